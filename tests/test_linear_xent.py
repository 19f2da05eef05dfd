"""Loss of a linear head without its logits, and its gradients (atom_k_linear_xent_*).

The reference is the definition in 64 bits.  Bounds are derived element by
element: u is the rounding of the element type (2^-8 bf16, 2^-24 fp32); a
product of k terms is off by at most (k / 32 + 64) 2^-24 of the sum of its
terms' magnitudes (chains of k / 32 matrix instructions, or fewer, joined by
splits and pieces)."""
import numpy as np
import pytest

from paper_2403_10504_amd import atom as A
from tests import gpu_util as U

U32 = 2.0 ** -24
LSE, DZ, SCALE, SCALE_F32, SCALE_ACC, SUM_SCALE = range(7, 13)  # internal epilogues, for the tile choice


def _u(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U32


def _gamma(k):
    return (k / 32 + 64) * U32


def _case(dtype, rows, V, d, ignored=0.0, seed=0, pad=0, spread=2.0):
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(1000 + seed)
    dt = t.bfloat16 if dtype == "bf16" else t.float32
    x = t.full((rows, d + pad), 7.0, device="cuda", dtype=dt)
    w = t.full((V, d + pad), 7.0, device="cuda", dtype=dt)
    x[:, :d] = t.randn((rows, d), device="cuda", generator=g).to(dt)
    w[:, :d] = (spread / d ** 0.5 * t.randn((V, d), device="cuda", generator=g)).to(dt)
    tgt = t.randint(0, V, (rows,), device="cuda", generator=g, dtype=t.int32)
    tgt[t.rand(rows, device="cuda", generator=g) < ignored] = A.ATOM_XENT_IGNORE
    return x, w, tgt


def _fwd(dtype, x, w, tgt, d, stream=None, ws=None):
    t = U.torch()
    rows, V, dt = x.shape[0], w.shape[0], U.dt_code(dtype)
    n = A.atom_k_linear_xent_fwd_ws_bytes(dt, rows, V, d)
    ws = t.full((n + 256,), 0xA5, device="cuda", dtype=t.uint8) if ws is None else ws
    lse = t.full((rows + 1,), 77.0, device="cuda")
    loss = t.full((rows + 1,), 77.0, device="cuda")
    A.atom_k_linear_xent_fwd(dt, x.data_ptr(), x.stride(0), w.data_ptr(), w.stride(0), tgt.data_ptr(), lse.data_ptr(),
                             loss.data_ptr(), rows, V, d, ws.data_ptr(), n, stream)
    return loss, lse, ws[n:]


def _ref(x, w, tgt, d):
    """64-bit loss, lse, logits and the largest sum of a logit's terms."""
    t = U.torch()
    xd, wd = x[:, :d].double(), w[:, :d].double()
    z = xd @ wd.T
    on = tgt >= 0
    lse = t.where(on, t.logsumexp(z, 1), 0.0)
    zt = z.gather(1, tgt.long().clamp(min=0).unsqueeze(1)).squeeze(1)
    return t.where(on, lse - zt, 0.0), lse, z, (xd.abs() @ wd.abs().T).max().item()


FWD = [("bf16", 1, 1, 8, 0), ("bf16", 1, 50257, 64, 0), ("bf16", 5, 7, 72, 8), ("bf16", 257, 1000, 136, 16),
       ("bf16", 999, 2049, 768, 0), ("bf16", 4100, 50257, 128, 0), ("bf16", 2048, 3333, 1024, 8),
       ("bf16", 3, 4096, 4104, 0), ("f32", 1, 1, 4, 0), ("f32", 33, 65, 68, 4), ("f32", 300, 5003, 260, 0),
       ("f32", 1025, 2049, 516, 4), ("f32", 2, 30011, 4096, 0),
       ("f32", 255, 1001, 100, 0), ("f32", 256, 1001, 100, 4), ("f32", 700, 9001, 1028, 0), ("f32", 2100, 4097, 36, 0),
       ("f32", 768, 43000, 132, 4), ("f32", 1030, 8201, 516, 0), ("f32", 2100, 4097, 516, 4), ("f32", 1100, 2001, 2052, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,V,d,pad", FWD)
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_forward(dtype, rows, V, d, pad, ignored):
    t = U.torch()
    x, w, tgt = _case(dtype, rows, V, d, ignored, rows + V, pad)
    loss, lse, behind = _fwd(dtype, x, w, tgt, d)
    rl, rs, z, terms = _ref(x, w, tgt, d)
    # logits off by gamma of their terms, the two base-2 logarithms' arguments
    # by 2^-24 of themselves, the sum of exponentials by a few roundings
    bound = _gamma(d) * terms + 2 ** -22 * (z.abs().max().item() + rs.abs().max().item()) + 2 ** -20
    assert (lse[:rows] - rs).abs().max().item() <= bound
    assert (loss[:rows] - rl).abs().max().item() <= 2 * bound
    off = tgt < 0
    assert (loss[:rows][off] == 0).all() and (lse[:rows][off] == 0).all()
    assert loss[rows] == 77.0 and lse[rows] == 77.0 and (behind == 0xA5).all()


# one size for every tile: (rows, V, d)
TILES = {(256, 256): (4096, 8192, 512), (256, 192): (512, 20000, 1024), (256, 128): (256, 30000, 2048),
         (128, 128): (700, 9000, 512), (64, 64): (128, 8192, 1024)}


@pytest.mark.gpu
@pytest.mark.parametrize("spread", [1e-3, 30.0])
def test_forward_spread(spread):
    """Logits that are all alike, and ones where a single term is the whole sum."""
    x, w, tgt = _case("bf16", 130, 777, 256, 0.1, 5, 0, spread)
    loss, lse, _ = _fwd("bf16", x, w, tgt, 256)
    rl, rs, z, terms = _ref(x, w, tgt, 256)
    bound = _gamma(256) * terms + 2 ** -22 * (z.abs().max().item() + rs.abs().max().item()) + 2 ** -20
    assert (lse[:-1] - rs).abs().max().item() <= bound
    assert (loss[:-1] - rl).abs().max().item() <= 2 * bound


def _bwd(dtype, x, w, tgt, lse, d, drow=None, scale=1.0, piece=0, epi=A.ATOM_EPI_STORE, want=("dx", "dw"), start=0.0,
         stream=None, opad=0):
    t = U.torch()
    rows, V, dt = x.shape[0], w.shape[0], U.dt_code(dtype)
    n = A.atom_k_linear_xent_bwd_ws_bytes(dt, rows, V, d, piece)
    ws = t.full((n + 256,), 0xA5, device="cuda", dtype=t.uint8)
    odt = x.dtype if epi == A.ATOM_EPI_STORE else t.float32
    dx = t.full((rows + 1, d + opad), 77.0, device="cuda", dtype=x.dtype)
    dw = t.full((V + 1, d + opad), 77.0, device="cuda", dtype=odt)
    dw[:V, :d] = start
    p = lambda v, k: v.data_ptr() if k in want else None  # noqa: E731
    A.atom_k_linear_xent_bwd(dt, x.data_ptr(), x.stride(0), w.data_ptr(), w.stride(0), tgt.data_ptr(), lse.data_ptr(),
                             None if drow is None else drow.data_ptr(), scale, p(dx, "dx"), dx.stride(0), p(dw, "dw"),
                             dw.stride(0), epi, rows, V, d, piece, ws.data_ptr(), n, stream)
    # rows behind the last, columns behind the last and the workspace's end stay
    assert (dx[rows] == 77.0).all() and (dw[V] == 77.0).all() and (ws[n:] == 0xA5).all()
    assert opad == 0 or ((dx[:, d:] == 77.0).all() and (dw[:, d:] == 77.0).all())
    return dx[:rows, :d], dw[:V, :d]


def _check_grads(dtype, x, w, tgt, d, dx, dw, drow=None, scale=1.0, out_u=None, start=0.0):
    t = U.torch()
    rows, V = x.shape[0], w.shape[0]
    on = tgt >= 0 if drow is None else (tgt >= 0) & (drow != 0)
    xd, wd = t.where(on.unsqueeze(1), x[:, :d].double(), 0.0), w[:, :d].double()
    terms = (xd.abs() @ wd.abs().T).max().item()
    z = xd @ wd.T
    lse = t.logsumexp(z, 1, keepdim=True)
    dz = t.exp(z - lse)
    p = dz.clone()
    dz.scatter_add_(1, tgt.long().clamp(min=0).unsqueeze(1), t.full_like(lse, -1.0))
    f = on.double() * (1.0 if drow is None else drow.double())
    f = f.unsqueeze(1)
    # p is off by its exponent's error: the logit, lse (as above) and their rounding
    ep = 2 * (_gamma(d) * terms + 2 ** -22 * (z.abs().max().item() + lse.abs().max().item()) + 2 ** -20)
    u = _u(dtype)
    edz = (u * dz.abs() + ep * p + U32) * f.abs()  # rounding of dz, then the error of p (and of 1 - p)
    dz = dz * f
    for got, ref, err, k, ou in ((dx, dz @ wd, edz @ wd.abs() + _gamma(V) * (dz.abs() @ wd.abs()), V, u),
                                 (dw, dz.T @ xd, edz.T @ xd.abs() + _gamma(rows) * (dz.abs().T @ xd.abs()), rows,
                                  u if out_u is None else out_u)):
        if got is None:
            continue
        if got is dw:
            ref = ref * scale + start
            bound = abs(scale) * err * 1.01 + 2 * ou * ref.abs() + abs(start) * U32 + 1e-37
        else:
            ref = ref * scale
            bound = abs(scale) * err * 1.01 + 2 * ou * ref.abs() + 1e-37
        worst = ((got.double() - ref).abs() / bound).max().item()
        assert worst <= 1.0, (worst, k)


# dtype, rows, V, d, piece, pad of the inputs' rows
BWD = [("bf16", 1, 1, 8, 0, 0), ("bf16", 1, 3000, 256, 0, 0), ("bf16", 5, 7, 72, 3, 8), ("bf16", 257, 1000, 136, 0, 16),
       ("bf16", 257, 1003, 136, 250, 8), ("bf16", 999, 2049, 768, 1024, 0), ("bf16", 4100, 9001, 128, 0, 0),
       ("bf16", 2048, 17000, 512, 0, 0), ("bf16", 130, 4097, 1032, 4096, 0), ("f32", 1, 1, 4, 0, 0),
       ("f32", 33, 65, 68, 8, 4), ("f32", 300, 3003, 260, 1000, 0), ("f32", 1025, 2049, 516, 0, 4),
       ("f32", 2, 9001, 1028, 4096, 0),
       ("f32", 256, 1003, 100, 250, 4), ("f32", 700, 9001, 1028, 0, 0), ("f32", 2100, 4097, 36, 0, 0),
       ("f32", 259, 20000, 772, 2048, 4), ("f32", 1030, 8201, 516, 0, 0), ("f32", 2100, 4097, 516, 1000, 4),
       ("f32", 512, 33000, 260, 0, 4), ("f32", 1100, 2001, 2052, 0, 0), ("bf16", 4100, 40001, 72, 0, 8),
       ("bf16", 2100, 33001, 2568, 0, 0), ("f32", 1300, 40001, 260, 0, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,V,d,piece,pad", BWD)
def test_backward(dtype, rows, V, d, piece, pad):
    x, w, tgt = _case(dtype, rows, V, d, 0.2, rows + V, pad)
    if rows == 1:
        tgt[:] = V - 1
    _, lse, _ = _fwd(dtype, x, w, tgt, d)
    scale = 1.0 / rows
    dx, dw = _bwd(dtype, x, w, tgt, lse, d, scale=scale, piece=piece, opad=pad)
    _check_grads(dtype, x, w, tgt, d, dx, dw, scale=scale)
    assert (dx[tgt < 0] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("epi", [A.ATOM_EPI_STORE, A.ATOM_EPI_STORE_F32, A.ATOM_EPI_ACC_F32])
@pytest.mark.parametrize("want", [("dx",), ("dw",), ("dx", "dw")])
def test_backward_forms(dtype, epi, want):
    """A weight per token (zero and negative ones too), each form of dW, and one gradient alone."""
    t = U.torch()
    rows, V, d = 190, 1111, 264
    x, w, tgt = _case(dtype, rows, V, d, 0.2, 3)
    _, lse, _ = _fwd(dtype, x, w, tgt, d)
    drow = t.randn(rows, device="cuda", generator=t.Generator(device="cuda").manual_seed(9))
    drow[::5] = 0
    start = 0.0 if epi == A.ATOM_EPI_STORE else 3.0
    dx, dw = _bwd(dtype, x, w, tgt, lse, d, drow, 0.37, 512, epi, want, start)
    if "dx" not in want:
        assert (dx == 77.0).all()
    if "dw" not in want:
        assert (dw == start).all()
    _check_grads(dtype, x, w, tgt, d, dx if "dx" in want else None, dw if "dw" in want else None, drow, 0.37,
                 None if epi == A.ATOM_EPI_STORE else U32, start if epi == A.ATOM_EPI_ACC_F32 else 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V,d", [(150, 700, 128), (400, 700, 128), (1100, 8000, 512)])
def test_tokens_without_part(dtype, rows, V, d):
    """Rows of masked tokens may hold anything; a batch of masked tokens only has no loss and no gradient."""
    t = U.torch()
    x, w, tgt = _case(dtype, rows, V, d, 0.5, 4)
    clean = x.clone()
    off = tgt < 0
    clean[off] = 0
    for k, v in enumerate((float("nan"), float("inf"), -float("inf"), 3e38)):
        x[off.nonzero()[k::4, 0]] = v
    loss, lse, _ = _fwd(dtype, x, w, tgt, d)
    l2, s2, _ = _fwd(dtype, clean, w, tgt, d)
    assert t.equal(loss, l2) and t.equal(lse, s2)
    got, want = _bwd(dtype, x, w, tgt, lse, d), _bwd(dtype, clean, w, tgt, lse, d)
    assert t.equal(got[0], want[0]) and t.equal(got[1], want[1])
    # the same by a weight of zero
    y = t.where(off, t.zeros_like(tgt), tgt)
    got = _bwd(dtype, x, w, y, lse, d, drow=(~off).float())
    assert t.equal(got[0], want[0]) and t.equal(got[1], want[1])
    tgt[:] = -5
    loss, lse, _ = _fwd(dtype, x, w, tgt, d)
    assert (loss[:-1] == 0).all() and (lse[:-1] == 0).all()
    dx, dw = _bwd(dtype, x, w, tgt, lse, d)
    assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.gpu
def test_bad_target_and_values():
    """A target past the vocabulary is never read: loss NaN, gradients NaN.  NaN and
    infinite logits make their own token's loss NaN and no other's."""
    t = U.torch()
    x, w, tgt = _case("bf16", 70, 300, 64, 0.0, 6)
    good, lse, _ = _fwd("bf16", x, w, tgt, 64)
    tgt2 = tgt.clone()
    tgt2[3], tgt2[69] = 300, 2 ** 31 - 1
    loss, l2, _ = _fwd("bf16", x, w, tgt2, 64)
    assert loss[[3, 69]].isnan().all() and t.equal(lse[:-1], l2[:-1])
    keep = [k for k in range(70) if k not in (3, 69)]
    assert t.equal(loss[keep], good[keep])
    dx, dw = _bwd("bf16", x, w, tgt2, l2, 64)
    assert dx[[3, 69]].isnan().all() and not dx[keep].isnan().any() and dw.isnan().all()
    x[5, 7], x[9, 1] = float("nan"), float("inf")
    loss, _, _ = _fwd("bf16", x, w, tgt, 64)
    assert loss[[5, 9]].isnan().all()
    keep = [k for k in range(70) if k not in (5, 9)]
    assert t.equal(loss[keep], good[keep])


@pytest.mark.gpu
def test_gradient_against_differences():
    """fp32: the loss's central difference along a direction is the gradient's product with it."""
    t = U.torch()
    rows, V, d = 40, 97, 32
    x, w, tgt = _case("f32", rows, V, d, 0.2, 8)
    loss, lse, _ = _fwd("f32", x, w, tgt, d)
    dx, dw = _bwd("f32", x, w, tgt, lse, d, scale=1.0 / rows)
    g = t.Generator(device="cuda").manual_seed(2)
    ex, ew = t.randn(x.shape, device="cuda", generator=g), t.randn(w.shape, device="cuda", generator=g)
    h = 2.0 ** -7
    hi = _fwd("f32", x + h * ex, w + h * ew, tgt, d)[0][:-1].double().sum().item() / rows
    lo = _fwd("f32", x - h * ex, w - h * ew, tgt, d)[0][:-1].double().sum().item() / rows
    want = ((dx.double() * ex).sum() + (dw.double() * ew).sum()).item()
    # third derivative times h^2 / 6 (directions of length sqrt(d) per row: a few
    # units), and the rounding of two losses of about 6 over 2 h
    assert abs((hi - lo) / (2 * h) - want) <= 0.02 * abs(want) + 6e-4


@pytest.mark.gpu
@pytest.mark.parametrize("tile", sorted(TILES))
def test_every_tile(tile):
    """The library's own rule takes each tile for some size; loss and gradients there, checked on sampled tokens."""
    t = U.torch()
    rows, V, d = TILES[tile]
    got = U.gemm_choice("bf16", 1, 1, LSE, rows, V, d)
    assert not got[0] and tuple(got[1:3]) == tile, got
    x, w, tgt = _case("bf16", rows, V, d, 0.1, 11)
    loss, lse, _ = _fwd("bf16", x, w, tgt, d)
    pick = slice(0, rows, max(1, rows // 97))
    rl, rs, z, terms = _ref(x[pick], w, tgt[pick], d)
    bound = _gamma(d) * terms + 2 ** -22 * (z.abs().max().item() + rs.abs().max().item()) + 2 ** -20
    assert (lse[:-1][pick] - rs).abs().max().item() <= bound
    assert (loss[:-1][pick] - rl).abs().max().item() <= 2 * bound
    dx, dw = _bwd("bf16", x, w, tgt, lse, d, scale=1.0 / rows)
    _check_grads("bf16", x, w, tgt, d, dx, dw, scale=1.0 / rows)


@pytest.mark.gpu
def test_streams_graphs_and_repeats():
    """The same bits on another stream, from a replayed graph beside eager work, and on every call."""
    t = U.torch()
    rows, V, d = 333, 5001, 192
    x, w, tgt = _case("bf16", rows, V, d, 0.1, 12)
    loss, lse, _ = _fwd("bf16", x, w, tgt, d)
    dx, dw = _bwd("bf16", x, w, tgt, lse, d, piece=2048)
    dt = A.ATOM_BF16
    bufs = [t.empty(n, device="cuda", dtype=t.uint8) for n in
            (A.atom_k_linear_xent_fwd_ws_bytes(dt, rows, V, d), A.atom_k_linear_xent_bwd_ws_bytes(dt, rows, V, d, 2048))]
    o = dict(loss=t.empty(rows, device="cuda"), lse=t.empty(rows, device="cuda"), dx=t.empty_like(x), dw=t.empty_like(w))

    def both(stream):
        A.atom_k_linear_xent_fwd(dt, x.data_ptr(), d, w.data_ptr(), d, tgt.data_ptr(), o["lse"].data_ptr(),
                                 o["loss"].data_ptr(), rows, V, d, bufs[0].data_ptr(), bufs[0].numel(), stream)
        A.atom_k_linear_xent_bwd(dt, x.data_ptr(), d, w.data_ptr(), d, tgt.data_ptr(), o["lse"].data_ptr(), None, 1.0,
                                 o["dx"].data_ptr(), d, o["dw"].data_ptr(), d, A.ATOM_EPI_STORE, rows, V, d, 2048,
                                 bufs[1].data_ptr(), bufs[1].numel(), stream)

    def same():
        t.cuda.synchronize()
        assert t.equal(o["loss"], loss[:-1]) and t.equal(o["lse"], lse[:-1])
        assert t.equal(o["dx"], dx) and t.equal(o["dw"], dw)

    s = t.cuda.Stream()
    s.wait_stream(t.cuda.current_stream())
    both(s.cuda_stream)
    same()
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g, stream=s):
        both(t.cuda.current_stream().cuda_stream)
    for _ in range(3):
        for v in o.values():
            v.fill_(5)
        g.replay()
        same()
        again = _bwd("bf16", x, w, tgt, lse, d, piece=2048)  # eager work between the replays
        assert t.equal(again[0], dx) and t.equal(again[1], dw)


def test_refusals():
    """Arguments that are refused before anything is enqueued (no GPU needed)."""
    P = 1 << 20  # never read
    ok = dict(dtype=A.ATOM_BF16, x=P, ldx=64, w=P, ldw=64, tgt=P, lse=P, loss=P, rows=10, V=100, d=64, ws=P, n=1 << 40)

    def fwd(**k):
        a = {**ok, **k}
        A.atom_k_linear_xent_fwd(a["dtype"], a["x"], a["ldx"], a["w"], a["ldw"], a["tgt"], a["lse"], a["loss"],
                                 a["rows"], a["V"], a["d"], a["ws"], a["n"])

    def bwd(**k):
        a = {**ok, **dict(drow=None, dx=P, lddx=64, dw=P, lddw=64, epi=A.ATOM_EPI_STORE, piece=0), **k}
        A.atom_k_linear_xent_bwd(a["dtype"], a["x"], a["ldx"], a["w"], a["ldw"], a["tgt"], a["lse"], a["drow"], 1.0,
                                 a["dx"], a["lddx"], a["dw"], a["lddw"], a["epi"], a["rows"], a["V"], a["d"], a["piece"],
                                 a["ws"], a["n"])

    common = [dict(dtype=2), dict(x=None), dict(w=None), dict(tgt=None), dict(lse=None), dict(ws=None), dict(x=P + 8),
              dict(w=P + 2), dict(ws=P + 4), dict(d=0), dict(d=60), dict(d=72), dict(ldx=63), dict(ldx=68), dict(ldw=56),
              dict(V=0), dict(V=-1), dict(rows=-1), dict(rows=1 << 31), dict(rows=1 << 27, V=1 << 24),
              dict(rows=(1 << 28) + 1), dict(V=(1 << 28) + 1), dict(d=(1 << 24) + 8, ldx=1 << 25, ldw=1 << 25), dict(n=0)]
    for call, more in ((fwd, [dict(loss=None), dict(n=A.atom_k_linear_xent_fwd_ws_bytes(1, 10, 100, 64) - 1)]),
                       (bwd, [dict(piece=-1), dict(epi=3), dict(epi=-1), dict(dx=P + 8), dict(dw=P + 8), dict(lddx=60),
                              dict(lddw=68), dict(n=A.atom_k_linear_xent_bwd_ws_bytes(1, 10, 100, 64, 0) - 1)])):
        for k in common + more:
            with pytest.raises(A.AtomError) as e:
                call(**k)
            assert e.value.status == A.ATOM_EINVAL, (call.__name__, k)
    # nothing to do: no launch, no workspace
    fwd(rows=0, x=None, w=None, tgt=None, lse=None, loss=None, ws=None, n=0)
    bwd(dx=None, dw=None)
    bwd(rows=0, x=None, w=None, tgt=None, lse=None, dx=None, ws=None, n=0, dw=None)
    for bad in ((2, 10, 100, 64), (1, -1, 100, 64), (1, 10, 0, 64), (1, 10, 100, 4)):
        assert A.atom_k_linear_xent_fwd_ws_bytes(*bad) == 0 and A.atom_k_linear_xent_bwd_ws_bytes(*bad, 0) == 0
    assert A.atom_k_linear_xent_bwd_ws_bytes(1, 10, 100, 64, -1) == 0
    # smaller pieces need less
    sizes = [A.atom_k_linear_xent_bwd_ws_bytes(1, 4096, 50257, 4096, p) for p in (1024, 4096, 8192)]
    assert np.all(np.diff(sizes) > 0)


@pytest.mark.gpu
def test_no_tokens():
    """No tokens: a stored gradient is zero, an accumulated one stays."""
    t = U.torch()
    x, w, tgt = _case("bf16", 1, 33, 64)
    x, tgt = x[:0], tgt[:0]
    lse = t.empty(1, device="cuda")
    for epi, want in ((A.ATOM_EPI_STORE, 0.0), (A.ATOM_EPI_STORE_F32, 0.0), (A.ATOM_EPI_ACC_F32, 3.0)):
        dw = t.full((34, 72), 3.0, device="cuda", dtype=t.bfloat16 if epi == A.ATOM_EPI_STORE else t.float32)
        A.atom_k_linear_xent_bwd(A.ATOM_BF16, x.data_ptr(), 64, w.data_ptr(), 64, tgt.data_ptr(), lse.data_ptr(), None,
                                 1.0, x.data_ptr(), 64, dw.data_ptr(), 72, epi, 0, 33, 64, 0, None, 0)
        assert (dw[:33, :64] == want).all() and (dw[33] == 3.0).all() and (dw[:, 64:] == 3.0).all()


@pytest.mark.gpu
def test_far_rows():
    """Rows of W, dW and x more than 2^31 elements from the first."""
    t = U.torch()
    rows, V, d, ld = 9, 1040, 64, 1 << 21
    x, w, tgt = _case("bf16", rows, V, d, 0.2, 50)
    tgt[0] = V - 1
    loss, lse, _ = _fwd("bf16", x, w, tgt, d)
    dx, dw = _bwd("bf16", x, w, tgt, lse, d)
    far = t.empty(V * ld, device="cuda", dtype=t.bfloat16)
    wf = far.as_strided((V, d), (ld, 1))
    wf.copy_(w)
    l2, s2, _ = _fwd("bf16", x, wf, tgt, d)
    assert t.equal(loss, l2) and t.equal(lse, s2)
    ws = t.empty(A.atom_k_linear_xent_bwd_ws_bytes(A.ATOM_BF16, rows, V, d), device="cuda", dtype=t.uint8)
    df = far.as_strided((V, d), (ld, 1), 4096)
    x2 = t.empty_like(x)
    A.atom_k_linear_xent_bwd(A.ATOM_BF16, x.data_ptr(), d, wf.data_ptr(), ld, tgt.data_ptr(), lse.data_ptr(), None, 1.0,
                             x2.data_ptr(), d, df.data_ptr(), ld, A.ATOM_EPI_STORE, rows, V, d, 0, ws.data_ptr(),
                             ws.numel())
    assert t.equal(x2, dx) and t.equal(df, dw)


@pytest.mark.parametrize("rows,V,d", [(2755581, 151936, 768), (2561241, 108983, 1024), (5923305, 50257, 4096)])
def test_parts_of_two_launches(rows, V, d):
    """Where the vocabulary is cut in two launches, the second one's parts lie behind the first one's and inside the
    workspace, also when that is more than 2^31 pairs (no GPU needed)."""
    cut, entries = U.lse_cut("bf16", rows, V, d)
    assert 0 < cut < V and entries % (2 * rows) == 0
    # a part is half a tile of 64 to 256 columns
    assert -(-cut // 128) <= entries // rows <= 2 * -(-cut // 64)
    assert entries > 2 ** 31
    rest = -(-(V - cut) // 128)
    assert 8 * (entries + rest * rows) <= A.atom_k_linear_xent_fwd_ws_bytes(A.ATOM_BF16, rows, V, d)


def test_refuses_more_workgroups_than_a_dispatch():
    """A dispatch counts its threads in 32 bits; sizes that need more in one launch are refused (no GPU needed)."""
    P = 1 << 20  # never read
    for dtype, rows, V, d in ((A.ATOM_F32, 700, 1 << 27, 4), (A.ATOM_BF16, 1 << 24, 1 << 15, 8)):
        assert A.atom_k_linear_xent_fwd_ws_bytes(dtype, rows, V, d) == 0
        with pytest.raises(A.AtomError) as e:
            A.atom_k_linear_xent_fwd(dtype, P, d, P, d, P, P, P, rows, V, d, P, 1 << 60)
        assert e.value.status == A.ATOM_EINVAL
    assert A.atom_k_linear_xent_fwd_ws_bytes(A.ATOM_F32, 700, 1 << 22, 4) > 0
    assert A.atom_k_linear_xent_fwd_ws_bytes(A.ATOM_BF16, 1 << 28, 8, 8) > 0


@pytest.mark.gpu
def test_most_tokens():
    """2^28 tokens, a block of them over and over: its loss over and over."""
    t = U.torch()
    n, rows, V, d = 1 << 16, 1 << 28, 8, 8
    x, w, tgt = _case("bf16", n, V, d, 0.2, 70)
    want, wlse, _ = _fwd("bf16", x, w, tgt, d)
    rl, rs, z, terms = _ref(x, w, tgt, d)
    bound = _gamma(d) * terms + 2 ** -22 * (z.abs().max().item() + rs.abs().max().item()) + 2 ** -20
    assert (want[:-1] - rl).abs().max().item() <= 2 * bound
    loss, lse, behind = _fwd("bf16", x.repeat(rows // n, 1), w, tgt.repeat(rows // n), d)
    assert loss[rows] == 77.0 and lse[rows] == 77.0 and (behind == 0xA5).all()
    # (another tile for so many tokens: other sums)
    assert (loss[:rows].view(-1, n) - want[:-1]).abs().max().item() <= 4 * bound
    assert (lse[:rows].view(-1, n) - wlse[:-1]).abs().max().item() <= 2 * bound


def _exact_case(dtype, rows, V, d, unit, gap, seed):
    """Logits that every product gives exactly: row n of x has `unit` at column n % d, w holds small integers there, and
    the target's is `gap` above all others."""
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(seed)
    dt = t.bfloat16 if dtype == "bf16" else t.float32
    x = t.zeros((rows, d), device="cuda", dtype=dt)
    n = t.arange(rows, device="cuda")
    x[n, n % d] = unit
    w = t.randint(-16, 9, (V, d), device="cuda", generator=g).to(dt)
    top = t.randint(0, V, (d,), device="cuda", generator=g)
    w[top, t.arange(d, device="cuda")] = 8.0 + gap
    return x, w, top[n % d].int()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,V,d", [("bf16", 300, 777, 64), ("bf16", 4100, 9001, 128), ("f32", 300, 777, 64),
                                            ("f32", 1100, 2001, 2052), ("bf16", 70, 50257, 64)])
def test_small_losses_of_large_logits(dtype, rows, V, d):
    """A target whose logit (1088) stands 64 above all others: the loss is nearly 0, and never below."""
    x, w, tgt = _exact_case(dtype, rows, V, d, 64.0, 9.0, 60)
    loss, lse, _ = _fwd(dtype, x, w, tgt, d)
    rl, rs, z, _ = _ref(x, w, tgt, d)
    assert z.max().item() == 64 * 17 and rl.max().item() < V * 1e-27
    assert (loss[:rows] >= 0).all() and loss[:rows].max().item() < V * 1e-27
    assert (lse[:rows] == 64 * 17).all()
    # 0 to 4 above the rest: the sum (1 to V) is off by at most 32 roundings (adds
    # of 8 columns, lanes, parts) and an exponential of up to 2^-20
    x, w, tgt = _exact_case(dtype, rows, V, d, 4.0, 1.0, 61)
    w += 200.0  # logits of 768 to 836
    loss, lse, _ = _fwd(dtype, x, w, tgt, d)
    rl, rs, z, _ = _ref(x, w, tgt, d)
    assert z.max().item() == 836
    assert (loss[:rows] - rl).abs().max().item() <= 32 * U32 + 2 ** -20 + U32 * rl.max().item()
    assert ((lse[:rows] - rs).abs().max().item() <= 32 * U32 + 2 ** -20 + U32 * 850)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_column(dtype):
    """A vocabulary of one: lse is the logit, the loss exactly 0."""
    t = U.torch()
    x, w, tgt = _case(dtype, 50, 1, 72, 0.2, 62, 0, 300.0)
    loss, lse, _ = _fwd(dtype, x, w, tgt, 72)
    z = (x[:, :72].double() @ w[:, :72].double().T)[:, 0]
    terms = (x.double().abs() @ w.double().abs().T).max().item()
    assert (loss[:50] == 0).all()
    assert (lse[:50] - t.where(tgt >= 0, z, 0.0)).abs().max().item() <= _gamma(72) * terms


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest_logits(dtype):
    """Logits next to the largest number of fp32, of both signs, alike and alone: loss and lse are those of the definition."""
    t = U.torch()
    V, d = 100, 64
    big = t.tensor(1.7e19).to(t.bfloat16).item()  # big^2 is 2.9e38
    dt = t.bfloat16 if dtype == "bf16" else t.float32
    x = t.zeros((4, d), device="cuda", dtype=dt)
    w = t.zeros((V, d), device="cuda", dtype=dt)
    for r, v in enumerate((big, -big, big, -big)):
        x[r, r] = v
    w[:, 0], w[:, 1], w[:, 2] = big, big, -big  # all alike: the largest, the lowest, the lowest
    w[:, 3], w[7, 3] = big, -big                # one largest among lowest
    tgt = t.tensor([5, 5, 5, 7], device="cuda", dtype=t.int32)
    loss, lse, _ = _fwd(dtype, x, w, tgt, d)
    want = t.tensor([1.0, 1.0, 1.0, 0.0], device="cuda") * np.log(V)
    # a sum of 100 ones is exact, its logarithm within 2^-22
    assert (loss[:4] - want).abs().max().item() <= 2 ** -21
    top = t.tensor([big * big, -big * big, -big * big, big * big], device="cuda", dtype=t.float32)
    assert ((lse[:4] - top).abs() <= 2.0 ** -22 * top.abs()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,V,d", [("bf16", 300, 777, 64), ("f32", 300, 777, 64), ("f32", 1100, 2001, 2052)])
def test_small_gradients_of_large_logits(dtype, rows, V, d):
    """The same targets' dz is p - 1 with p the nearest to 1: what is left are the other logits, e^-64 and less."""
    x, w, tgt = _exact_case(dtype, rows, V, d, 64.0, 9.0, 60)
    _, lse, _ = _fwd(dtype, x, w, tgt, d)
    dx, dw = _bwd(dtype, x, w, tgt, lse, d)
    assert dx.abs().max().item() <= V * 16 * 2e-28 and dw.abs().max().item() <= rows * 64 * 2e-28


@pytest.mark.parametrize("rows,V,d,tile", [(1030, 8201, 516, (256, 192)), (1300, 40001, 260, (256, 128)),
                                           (7688, 1000, 560, (256, 192))])
def test_planes_dx_takes_every_tile(rows, V, d, tile):
    """dx of fp32 operands in planes chooses among all five tiles for the first piece as for later ones (no GPU needed)."""
    _, _, planes, width, last, ws = U.xent_plan("f32", rows, V, d)
    assert planes
    for epi in (SCALE_F32, SCALE_ACC):
        assert U.loss_launches("planes", 1, 0, epi, rows, d, last if width == V else width, ws)[0][:2] == tile
