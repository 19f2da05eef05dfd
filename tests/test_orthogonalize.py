"""Newton-Schulz orthogonalisation (atom_k_orthogonalize).

The reference is the recursion in 64 bits.  How far the kernels may be off
comes from the same recursion in 64 bits with their roundings planted in it
(`_model`): X in two fp16 planes of 2^10 X, the factors of the products in one
(bf16) or two (fp32).  The kernels round the same numbers at the same places,
so their error is the model's up to other signs, plus the sums' own."""
import numpy as np
import pytest

from paper_2403_10504_amd import atom as A
from tests import gpu_util as U

QUINTIC = (3.4445, -4.7750, 2.0315)
SCALE = 1024.0


def _planes(x, n):
    hi = (x * SCALE).half().double()
    return (hi + (x * SCALE - hi).half().double() if n == 2 else hi) / SCALE


def _recursion(g, coef, dtype=None):
    """g: [rows][cols] in 64 bits; dtype: plant the roundings of that type's kernels."""
    t = U.torch()
    tall = g.shape[0] > g.shape[1]
    x = g.T if tall else g
    x = x / (t.linalg.vector_norm(x) + 1e-7)
    f = 2 if dtype == "f32" else 1
    for a, b, c in coef:
        a, b, c = (float(np.float32(v)) for v in (a, b, c))
        if dtype:
            x = _planes(x, 2)
            xf = _planes(x, f)
            s = _planes(xf @ xf.T, f)
            p = _planes(b * s + c * (s @ s), f)
            x = a * x + p @ xf
        else:
            s = x @ x.T
            x = a * x + (b * s + c * (s @ s)) @ x
    return x.T if tall else x


def _matrix(rows, cols, dtype, seed, kind="gradient"):
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: t.randn(s, device="cuda", generator=g, dtype=t.float64)  # noqa: E731
    k = max(1, min(rows, cols) // 16)
    x = 1e-4 * (r(rows, k) @ r(k, cols) + 2.0 * r(rows, cols)) if kind == "gradient" else r(rows, cols)
    if kind == "decay":  # singular values over four decades
        m = min(rows, cols)
        x = (r(rows, m) * t.logspace(0, -4, m, device="cuda", dtype=t.float64)) @ r(m, cols)
    return x.to(t.bfloat16 if dtype == "bf16" else t.float32)


def _run(dtype, g, coef, epi=A.ATOM_EPI_STORE, keep=0.0, scale=1.0, pad=0, start=None, stream=None, shift=0):
    """g: [batch][rows][cols] (any strides along the first two).  Returns out [batch][rows][cols]; rows, columns and
    workspace behind the ends are checked to stay."""
    t = U.torch()
    b, rows, cols = g.shape
    dt = U.dt_code(dtype)
    n = A.atom_k_orthogonalize_ws_bytes(dt, b, rows, cols)
    ws = t.full((n + 256,), 0xA5, device="cuda", dtype=t.uint8)
    odt = g.dtype if epi == A.ATOM_EPI_STORE else t.float32
    flat = t.full((shift + (b * (rows + 1)) * (cols + pad) + 8,), 77.0, device="cuda", dtype=odt)
    out = flat[shift:shift + b * (rows + 1) * (cols + pad)].view(b, rows + 1, cols + pad)
    if start is not None:
        out[:, :rows, :cols] = start
    A.atom_k_orthogonalize(dt, g.data_ptr(), g.stride(1), g.stride(0), out.data_ptr(), out.stride(1), out.stride(0), epi,
                           keep, scale, b, rows, cols, coef, ws.data_ptr(), n, stream)
    assert (ws[n:] == 0xA5).all() and (flat[:shift] == 77.0).all() and (flat[shift + out.numel():] == 77.0).all()
    assert (out[:, rows] == 77.0).all() and (pad == 0 or (out[:, :, cols:] == 77.0).all())
    return out[:, :rows, :cols]


def _check(dtype, got, g, coef, scale=1.0, out_bf16=None):
    t = U.torch()
    out_bf16 = dtype == "bf16" if out_bf16 is None else out_bf16
    for i in range(g.shape[0]):
        x = g[i].double()
        ref, mod = _recursion(x, coef), _recursion(x, coef, dtype)
        size = t.linalg.vector_norm(ref).item()
        err = t.linalg.vector_norm(got[i].double() / scale - ref).item()
        off = t.linalg.vector_norm(mod - ref).item()
        # the model's error with other signs; sums of k / 32 instructions per
        # pass, the square root of as many roundings, through the steps' growth
        # of weak directions (which the model's own error measures: at least one
        # rounding of 2^-23 of X per step); the rounding of the result
        if size == 0.0:
            assert err == 0.0
            continue
        k = max(g.shape[1:])
        grow = max(1.0, off / size / 2.0 ** -21) if dtype == "f32" else 1.0
        sums = 2.0 ** -24 * (4 + (3 * k / 32) ** 0.5) * len(coef) * (grow if dtype == "f32" else 100.0)
        bound = 2.0 * off + size * (sums + (2.0 ** -8 if out_bf16 else 2.0 ** -23))
        assert err <= bound, (i, err / size, bound / size, off / size)


SHAPES = [(1, 1), (1, 64), (64, 1), (5, 7), (33, 31), (64, 64), (100, 333), (333, 100), (129, 1000), (256, 256),
          (768, 256), (500, 501), (700, 1500), (1030, 1030)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_against_recursion(dtype, rows, cols):
    coef = [QUINTIC] * 5
    g = _matrix(rows, cols, dtype, rows * 7 + cols)[None]
    got = _run(dtype, g, coef)
    _check(dtype, got, g, coef)
    # the quintic by its number of steps
    assert U.torch().equal(got, _run(dtype, g, 5))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["gauss", "decay"])
def test_spectra(dtype, kind):
    g = _matrix(320, 512, dtype, 3, kind)[None]
    _check(dtype, _run(dtype, g, [QUINTIC] * 5), g, [QUINTIC] * 5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_result_is_orthogonal(dtype):
    """Cubic steps go on to singular values of one: O O^T is the identity."""
    t = U.torch()
    g = _matrix(96, 160, "f32", 4, "gauss").to(t.bfloat16 if dtype == "bf16" else t.float32)[None]
    o = _run(dtype, g, [QUINTIC] * 4 + [(1.875, -1.25, 0.375)] * 6)[0].double()
    off = (o @ o.T - t.eye(96, device="cuda", dtype=t.float64)).abs().max().item()
    # rows of length one, entries rounded to the type; and 11-bit factors of the last step
    assert off <= (2 ** -8 + 2 ** -10 if dtype == "bf16" else 2 ** -18)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("coef", [[], [(1.5, -0.5, 0.0)], [(1.5, -0.5, 0.0)] * 9, [(8.287, -23.596, 17.3), (4.107, -2.948, 0.545)],
                                  [(1.0, 0.0, 0.0)] * 2, [(0.0, 0.0, 0.0)]])
def test_coefficients(dtype, coef):
    g = _matrix(70, 130, dtype, 5)[None]
    _check(dtype, _run(dtype, g, coef), g, coef)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(48, 200, 0, 0), (200, 48, 3, 0), (65, 131, 1, 1), (128, 64, 4, 4),
                                                 (31, 4, 0, 2)])
@pytest.mark.parametrize("epi", [A.ATOM_EPI_STORE, A.ATOM_EPI_STORE_F32, A.ATOM_EPI_ACC_F32])
def test_output_forms(dtype, rows, cols, pad, shift, epi):
    """Strides and alignments of the result, its types, and the update of fp32 weights."""
    t = U.torch()
    g = t.stack([_matrix(rows, cols, dtype, 6 + i) for i in range(3)])
    coef = [QUINTIC] * 3
    got = _run(dtype, g, coef, epi, 0.75, -0.25, pad, 4.0 if epi == A.ATOM_EPI_ACC_F32 else None, None, shift)
    if epi == A.ATOM_EPI_ACC_F32:
        got = got.double() - 3.0
        # the sum's rounding: half a step of values below 4
        plain = _run(dtype, g, coef, A.ATOM_EPI_STORE_F32, 0.0, -0.25)
        assert (got - plain.double()).abs().max().item() <= 2.0 ** -23 * 2
    else:
        _check(dtype, got, g, coef, -0.25, dtype == "bf16" and epi == A.ATOM_EPI_STORE)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_batches(dtype):
    """Matrices side by side, on end, in place, and one read for all: each as if alone."""
    t = U.torch()
    dt, b, rows, cols = U.dt_code(dtype), 3, 60, 90
    big = _matrix(rows, b * cols, dtype, 8)
    alone = [_run(dtype, big[None, :, i * cols:(i + 1) * cols], 5)[0].clone() for i in range(b)]
    ws = t.empty(A.atom_k_orthogonalize_ws_bytes(dt, b, rows, cols), device="cuda", dtype=t.uint8)

    def call(src, ldg, sg, dst, ldo, so, n=b):
        A.atom_k_orthogonalize(dt, src.data_ptr(), ldg, sg, dst.data_ptr(), ldo, so, A.ATOM_EPI_STORE, 0.0, 1.0, n, rows,
                               cols, 5, ws.data_ptr(), ws.numel())

    side = t.zeros_like(big)
    call(big, b * cols, cols, side, b * cols, cols)
    ends = t.zeros((b, rows, cols), device="cuda", dtype=big.dtype)
    call(big, b * cols, cols, ends, cols, rows * cols)
    for i in range(b):
        assert t.equal(side[:, i * cols:(i + 1) * cols], alone[i]) and t.equal(ends[i], alone[i])
    same = t.zeros_like(ends)
    call(big, b * cols, 0, same, cols, rows * cols)
    assert all(t.equal(same[i], alone[0]) for i in range(b))
    call(big, b * cols, cols, big, b * cols, cols)
    assert t.equal(big, side)
    call(side, b * cols, cols, same, cols, rows * cols, 0)  # no matrices
    assert all(t.equal(same[i], alone[0]) for i in range(b))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_values(dtype):
    t = U.torch()
    coef = [QUINTIC] * 5
    g = _matrix(40, 72, dtype, 9, "gauss")
    # zeros: zeros; the norm neither overflows nor underflows
    assert (_run(dtype, t.zeros_like(g)[None], coef) == 0).all()
    base = _run(dtype, g[None], coef)
    for s in (2.0 ** 100, 2.0 ** -10):
        assert (_run(dtype, (g * s)[None], coef).double() - base.double()).abs().max().item() <= 2.0 ** -8
    tiny = (g * 2.0 ** -100)[None]
    _check(dtype, _run(dtype, tiny, coef), tiny, coef) if dtype == "f32" else None
    full = t.full_like(g, 3e38)[None]
    _check(dtype, _run(dtype, full, coef), full, coef)
    # an entry that is not finite: no number anywhere, in that matrix alone
    for v in (float("nan"), float("inf"), -float("inf")):
        two = t.stack([g, g])
        two[1, 39, 71] = v
        got = _run(dtype, two, coef)
        assert t.equal(got[0], base[0]) and got[1].isnan().all()


# type, batch, rows, cols, tiles of the three products and ranges of k of the first by the library's rule
TILES = [("bf16", 1, 1500, 1500, (64, 64, 128, 1)),
         ("bf16", 12, 700, 760, (128, 128, 128, 1)),
         ("bf16", 2, 2048, 2050, (128, 128, 192, 1)),
         ("bf16", 4, 2100, 2048, (256, 256, 192, 1)),
         ("f32", 2, 2100, 2048, (128, 192, 192, 1)),
         ("f32", 4, 2048, 2048, (256, 256, 256, 1)),
         ("bf16", 1, 4096, 4160, (192, 192, 192, 1)),
         ("bf16", 1, 4200, 4096, (192, 192, 192, 1)),
         ("f32", 1, 3300, 3200, (192, 192, 128, 1)),
         ("f32", 3, 700, 640, (64, 64, 64, 1)),
         ("f32", 12, 640, 700, (128, 128, 128, 1)),
         ("bf16", 1, 70, 20000, (64, 64, 64, 64)),
         ("bf16", 1, 20000, 70, (64, 64, 64, 64)),
         ("f32", 2, 100, 5000, (64, 64, 64, 32)),
         ("f32", 1, 768, 256, (64, 64, 64, 8)),
         ("bf16", 3, 700, 9001, (64, 64, 128, 2))]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,batch,rows,cols,tiles", TILES)
def test_every_tile(dtype, batch, rows, cols, tiles):
    assert U.ns_choice(dtype, batch, rows, cols) == tiles
    t = U.torch()
    g = t.stack([_matrix(rows, cols, dtype, 20 + i) for i in range(min(batch, 2))])
    g = g[t.arange(batch, device="cuda") % 2].contiguous() if batch > 2 else g
    got = _run(dtype, g, [QUINTIC] * 2)
    _check(dtype, got[:2], g[:2], [QUINTIC] * 2)
    for i in range(2, batch):
        assert t.equal(got[i], got[i % 2])


@pytest.mark.gpu
def test_streams_graphs_and_repeats():
    t = U.torch()
    b, rows, cols, dt = 2, 200, 330, A.ATOM_BF16
    g = t.stack([_matrix(rows, cols, "bf16", 30 + i) for i in range(b)])
    want = _run("bf16", g, 5).clone()
    ws = t.empty(A.atom_k_orthogonalize_ws_bytes(dt, b, rows, cols), device="cuda", dtype=t.uint8)
    out = t.empty_like(g)

    def call(stream):
        A.atom_k_orthogonalize(dt, g.data_ptr(), cols, rows * cols, out.data_ptr(), cols, rows * cols, A.ATOM_EPI_STORE,
                               0.0, 1.0, b, rows, cols, 5, ws.data_ptr(), ws.numel(), stream)

    s = t.cuda.Stream()
    s.wait_stream(t.cuda.current_stream())
    call(s.cuda_stream)
    t.cuda.synchronize()
    assert t.equal(out, want)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=s):
        call(t.cuda.current_stream().cuda_stream)
    for _ in range(3):
        out.fill_(5)
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(out, want)
        assert t.equal(_run("bf16", g, 5), want)  # eager work between the replays


def test_refusals():
    """Arguments that are refused before anything is enqueued (no GPU needed)."""
    P = 1 << 20  # never read
    ok = dict(dtype=A.ATOM_BF16, g=P, ldg=64, sg=6400, out=P, ldo=64, so=6400, epi=A.ATOM_EPI_STORE, batch=3, rows=100,
              cols=64, coef=5, ws=P, n=1 << 50)

    def call(**k):
        a = {**ok, **k}
        A.atom_k_orthogonalize(a["dtype"], a["g"], a["ldg"], a["sg"], a["out"], a["ldo"], a["so"], a["epi"], 0.0, 1.0,
                               a["batch"], a["rows"], a["cols"], a["coef"], a["ws"], a["n"])

    need = A.atom_k_orthogonalize_ws_bytes(A.ATOM_BF16, 3, 100, 64)
    for k in (dict(dtype=2), dict(g=None), dict(out=None), dict(ws=None), dict(g=P + 1), dict(out=P + 1),
              dict(out=P + 2, epi=A.ATOM_EPI_STORE_F32), dict(ws=P + 8), dict(ldg=63), dict(ldo=63), dict(sg=-1),
              dict(so=6399), dict(so=0), dict(so=64, ldo=191), dict(epi=3), dict(epi=-1), dict(batch=-1),
              dict(batch=65536), dict(rows=0), dict(cols=0), dict(rows=(1 << 24) + 1), dict(rows=1 << 22, cols=1 << 22),
              dict(coef=-1), dict(coef=65), dict(coef=[(float("nan"), 0, 0)]), dict(coef=[(1.0, float("inf"), 0)]),
              dict(coef=[(33.0, 0, 0)]), dict(coef=[(5.0, 0, 0)]), dict(coef=[(2.0, 0, 0)] * 3),
              dict(coef=[(1.0, -40.0, 40.0)] * 2),
              dict(coef=[(8.28, -23.6, 17.3), QUINTIC]), dict(n=need - 1)):
        with pytest.raises(A.AtomError) as e:
            call(**k)
        assert e.value.status == A.ATOM_EINVAL, k
    call(batch=0, g=None, out=None, ws=None, n=0)  # nothing to do
    with pytest.raises(ValueError):
        call(coef=[(1.0, 2.0)])
    for bad in ((2, 3, 100, 64), (1, 0, 100, 64), (1, 3, 0, 64), (1, 3, 100, -4)):
        assert A.atom_k_orthogonalize_ws_bytes(*bad) == 0


@pytest.mark.gpu
def test_far_rows():
    """Rows of the gradient and of the result more than 2^31 elements from the first."""
    t = U.torch()
    rows, cols, ld = 1040, 48, 1 << 21
    g = _matrix(rows, cols, "bf16", 60)
    want = _run("bf16", g[None], 5)[0]
    far = t.empty(rows * ld, device="cuda", dtype=t.bfloat16)
    src, dst = far.as_strided((rows, cols), (ld, 1)), far.as_strided((rows, cols), (ld, 1), 4097)
    src.copy_(g)
    ws = t.empty(A.atom_k_orthogonalize_ws_bytes(A.ATOM_BF16, 1, rows, cols), device="cuda", dtype=t.uint8)
    A.atom_k_orthogonalize(A.ATOM_BF16, src.data_ptr(), ld, 0, dst.data_ptr(), ld, 0, A.ATOM_EPI_STORE, 0.0, 1.0, 1, rows,
                           cols, 5, ws.data_ptr(), ws.numel())
    assert t.equal(dst, want)


def test_refuses_more_workgroups_than_a_dispatch():
    """A dispatch counts its threads in 32 bits; batches that need more in one launch are refused (no GPU needed)."""
    assert A.atom_k_orthogonalize_ws_bytes(A.ATOM_F32, 65535, 1, 64 * 1000) == 0
    assert A.atom_k_orthogonalize_ws_bytes(A.ATOM_BF16, 65535, 1, 64) > 0


def _small_norm_check(dtype, got, g, coef, scale=1.0):
    """The result against the recursion in 64 bits, bounded by the error of the recursion with the kernels' planes, which
    are taken of X times the power of two that brings the bound of its singular values into [1/2, 1)."""
    t = U.torch()
    x = g.double()
    ref = _recursion(x, coef) * scale
    tall = x.shape[0] > x.shape[1]
    y = x.T if tall else x
    y = y / (t.linalg.vector_norm(y) + 1e-7)
    f = 2 if dtype == "f32" else 1
    r = t.linalg.vector_norm(y).item()
    for a, b, c in coef:
        a, b, c = (float(np.float32(v)) for v in (a, b, c))
        e = 2.0 ** max(0.0, np.floor(-np.log2(r)))
        v = np.linspace(0.0, r, 4097)
        r = np.abs(a * v + b * v ** 3 + c * v ** 5).max()
        y = _planes(y * e, 2)
        yf = _planes(y, f)
        s = _planes(yf @ yf.T, f)
        p = _planes(b / e ** 2 * s + c / e ** 4 * (s @ s), f)
        y = (a * y + p @ yf) / e
    y = (y.T if tall else y) * scale
    size = t.linalg.vector_norm(ref).item()
    off = t.linalg.vector_norm(y - ref).item()
    k = max(g.shape)
    # as in _check; off counts four times: a bound next to a power of two may take
    # the other exponent
    sums = size * 2.0 ** -24 * (4 + (3 * k / 32) ** 0.5) * len(coef) * (8.0 if dtype == "f32" else 100.0)
    bound = 4.0 * off + sums + size * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) + 2.0 ** -149 * (g.numel() ** 0.5)
    err = t.linalg.vector_norm(got.double() - ref).item()
    assert size > 0 and err <= bound, (err / size, bound / size, off / size)
    assert bound <= size * (2.0 ** -5 if dtype == "bf16" else 2.0 ** -12)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("coef", [[], [QUINTIC] * 5, [(1.5, -0.5, 0.0)] * 20, [(0.25, 0.1, 0.0)] * 3 + [QUINTIC] * 8])
@pytest.mark.parametrize("rows,cols", [(40, 72), (200, 130)])
def test_small_norms(dtype, coef, rows, cols):
    """Norms far below the 1e-7 in the divisor, down to a few of the type's smallest numbers: X is small, and keeps its
    bits.  Beside matrices of ordinary norms in a batch, which stay as they are alone."""
    t = U.torch()
    base = _matrix(rows, cols, "f32", 71, "gauss").double()
    base = base / t.linalg.vector_norm(base)
    dt = t.bfloat16 if dtype == "bf16" else t.float32
    norms = [1.0, 1e-6, 3e-8, 1e-9, 1e-11, 1e-14, 1e-20, 1e-30, 1e-36]
    g = t.stack([(base * v).to(dt) for v in norms])
    # the result's scale keeps it out of the subnormal numbers
    got = _run(dtype, g, coef, scale=2.0 ** 40)
    for i, v in enumerate(norms):
        _small_norm_check(dtype, got[i], g[i], coef, 2.0 ** 40)
        assert t.equal(got[i], _run(dtype, g[i:i + 1], coef, scale=2.0 ** 40)[0]), v


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_entry(dtype):
    """A single entry is the norm itself, also the type's smallest: g / (g + 1e-7), and the recursion of a number."""
    t = U.torch()
    dt = t.bfloat16 if dtype == "bf16" else t.float32
    least = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    for v in (1.0, -3e-8, 1e-12, -1e-25, 1e-37, least, -7 * least):
        g = t.zeros((1, 33, 70), device="cuda", dtype=dt)
        g[0, 20, 50] = v
        v = g[0, 20, 50].double().item()
        x = v / (abs(v) + 1e-7)
        for coef in ([], [QUINTIC] * 5):
            want = x
            for a, b, c in coef:
                a, b, c = (float(np.float32(k)) for k in (a, b, c))
                want = a * want + b * want ** 3 + c * want ** 5
            got = _run(dtype, g, coef, A.ATOM_EPI_STORE_F32)[0]
            # per step X, A and B in 22 bits: B is off by (|b| x^2 + 2 |c| x^4 + |B|) 2^-23, up to 12 of them, and a step
            # next to |x| = 1 takes an error times 1.2.  bf16: A and B in 11, nothing beside a while X is small
            off = (2.0 ** -21 * (len(coef) + 1) * 8 if dtype == "f32" or abs(x) < 0.01 or not coef else 2.0 ** -5) * abs(want)
            assert abs(got[20, 50].item() - want) <= off + 2.0 ** -149
            assert (got != 0).sum().item() == 1


@pytest.mark.gpu
@pytest.mark.parametrize("batch,rows,cols", [(1, 33, 31), (2, 256, 256), (3, 100, 700), (1, 1030, 1000), (1, 3000, 128)])
def test_fp32_results_of_bf16_gradients(batch, rows, cols):
    """A result in fp32 is as accurate as of fp32 gradients: the bound is that of two planes of every factor."""
    t = U.torch()
    coef = [QUINTIC] * 5
    g = t.stack([_matrix(rows, cols, "bf16", 80 + i) for i in range(batch)])
    got = _run("bf16", g, coef, A.ATOM_EPI_STORE_F32)
    _check("f32", got, g, coef)
    # the same planes: the same bits
    assert t.equal(got, _run("f32", g.float(), coef))
    acc = _run("bf16", g, coef, A.ATOM_EPI_ACC_F32, 1.0, 1.0, start=0.0)
    assert t.equal(acc, got)


def test_workspace_of_many_small_matrices():
    """Partial sums of the norm take what is written: one per matrix of one row (no GPU needed)."""
    n = 65535
    # eight planes of 32 x 32, exponents of 64 steps, one partial sum, and the rounding of ten parts
    assert A.atom_k_orthogonalize_ws_bytes(A.ATOM_F32, n, 1, 1) <= n * (8 * 2048 + 256 + 8) + 10 * 256


@pytest.mark.parametrize("c", [0.0, 1e-20, -1e-20, 1e-38, 1e-3])
def test_refuses_an_extremum_inside(c):
    """12 s - 12 s^3 is 4.6 at 0.58 and 0 at 1: beyond 4, also with a last coefficient next to zero (no GPU needed)."""
    P = 1 << 20  # never read

    def call(a):
        A.atom_k_orthogonalize(A.ATOM_BF16, P, 64, 0, P, 64, 0, A.ATOM_EPI_STORE, 0.0, 1.0, 0, 64, 64, [(a, -a, c)], P,
                               1 << 40)

    with pytest.raises(A.AtomError) as e:
        call(12.0)
    assert e.value.status == A.ATOM_EINVAL
    call(10.0)  # 3.85; no matrices
