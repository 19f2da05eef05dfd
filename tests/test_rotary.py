"""Rotary positions (atom_k_rope) and the norms of queries and keys with the turn in the same pass
(atom_k_qknorm_rope_*), against the formulas in 64 bits.

Bounds.  A cosine or sine is off by its angle's rounding in fp32 (2^-25 half turns, below 2^-23 radians, and p freq 2^-52
in 64 bits), the function's own 2^-23 and the product with mscale: below 2^-21 with the products and the sum of a turn, so
a turned pair (u, w) is off by E = (|u| + |w|) mscale (2^-21 + p freq 2^-52).  r = 1 / sqrt(mean + eps) holds a sum of 256
squares at most in 16 terms of a lane and 6 shuffles, a root and a division: 2^-20 relative, 2^-19 with the products
behind it.  A result is rounded to its type: eps / 2 of the value.  fp32's denormal results may be off by 2^-126."""
import math
from fractions import Fraction

import numpy as np
import pytest

from paper_2403_10504_amd import atom as A
from tests import gpu_util as U

EPS = float(np.float32(1e-6))
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
LAYOUTS = {"half": A.ATOM_ROPE_HALF, "pairs": A.ATOM_ROPE_PAIRS}


def _type(dtype):
    t = U.torch()
    return t.bfloat16 if dtype == "bf16" else t.float32


def _freq(rot):
    t = U.torch()
    return t.from_numpy(A.atom_rope_freqs(rot)).cuda() if rot else None


def _ptr(x):
    return None if x is None else x.data_ptr()


def _padded(rows, width, pad, dtype, fill=77.0, shift=0):
    """A buffer of rows of width columns, pad behind each, and a row of guards at the end."""
    t = U.torch()
    flat = t.full((shift + (rows + 1) * (width + pad),), fill, device="cuda", dtype=_type(dtype))
    return flat[shift:].view(rows + 1, width + pad)


def _kept(buf, rows, width, fill=77.0):
    return bool((buf[rows:] == fill).all()) and bool((buf[:, width:] == fill).all())


def _angles(rows, T, pos, freq):
    t = U.torch()
    p = pos.double() if pos is not None else (t.arange(rows, device="cuda") % T).double()
    return t.outer(p, freq)


def _turn(x, angle, mscale, layout, back=False):
    """x [rows][heads][dh] in 64 bits; the turned x and the bound of its error."""
    t = U.torch()
    r = 2 * angle.shape[1]
    c, s = (f(angle).unsqueeze(1) * mscale for f in (t.cos, t.sin))
    s = -s if back else s
    y, e = x.clone(), t.zeros_like(x)
    i0 = slice(0, r // 2) if layout == "half" else slice(0, r, 2)
    i1 = slice(r // 2, r) if layout == "half" else slice(1, r, 2)
    u, w = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = u * c - w * s, u * s + w * c
    off = (u.abs() + w.abs()) * abs(mscale) * (2.0 ** -21 + angle.abs().unsqueeze(1) * 2.0 ** -52)
    e[..., i0], e[..., i1] = off, off
    return y, e


def _within(got, ref, bound, dtype):
    t = U.torch()
    slack = (got.double() - ref).abs() - (bound + (ref.abs() + bound) * HALF[dtype] + 2.0 ** -126)
    assert bool(t.isfinite(got.double()).all())
    assert slack.max().item() <= 0.0, slack.max().item()


SHAPES = [  # rows, Hq, Hk, Hv, dh, rot, pad
    (1, 1, 1, 1, 64, 64, 0), (2, 40, 40, 40, 128, 128, 0), (37, 4, 2, 2, 128, 96, 8), (130, 3, 1, 0, 64, 32, 16),
    (5, 7, 5, 3, 80, 40, 0), (9, 2, 2, 2, 256, 256, 0), (11, 1, 3, 2, 254, 252, 0), (300, 2, 1, 1, 130, 6, 3),
    (17, 5, 0, 0, 2, 2, 1), (33, 0, 4, 4, 36, 12, 0), (6, 2, 2, 2, 96, 0, 0), (1100, 12, 12, 12, 64, 64, 0)]


def _case(dtype, rows, heads, dh, rot, pad, seed, far=False, shift=0):
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(seed)
    x = _padded(rows, heads * dh, pad, dtype, shift=shift)
    x[:rows, :heads * dh] = t.randn(rows, heads * dh, device="cuda", generator=g) * 3
    pos = t.randint(0, 1 << 20, (rows,), device="cuda", generator=g, dtype=t.int32) if far else None
    return x, pos, _freq(rot), g


def _split(x, rows, heads, dh):
    return x[:rows, :heads * dh].double().reshape(rows, heads, dh)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rows,Hq,Hk,Hv,dh,rot,pad", SHAPES)
def test_rope(dtype, layout, rows, Hq, Hk, Hv, dh, rot, pad):
    t = U.torch()
    heads, mscale = Hq + Hk, 1.25
    for far in (False, True):
        x, pos, freq, _ = _case(dtype, rows, heads, dh, rot, pad, rows + dh, far)
        y = _padded(rows, heads * dh, pad + 1, dtype)
        T = 7
        for back in (0, 1):
            A.atom_k_rope(U.dt_code(dtype), x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), _ptr(pos), _ptr(freq),
                          mscale, LAYOUTS[layout], back, rows, T, heads, dh, rot)
            ref = _split(x, rows, heads, dh)
            bound = t.zeros_like(ref)
            if rot:
                ref, bound = _turn(ref, _angles(rows, T, pos, freq), mscale, layout, back)
            _within(_split(y, rows, heads, dh), ref, bound, dtype)
            assert _kept(y, rows, heads * dh)
            # what does not turn is copied
            assert t.equal(_split(y, rows, heads, dh)[..., rot:], _split(x, rows, heads, dh)[..., rot:])
        # in place: the same bits
        want = y[:rows, :heads * dh].clone()
        A.atom_k_rope(U.dt_code(dtype), x.data_ptr(), x.stride(0), x.data_ptr(), x.stride(0), _ptr(pos), _ptr(freq),
                      mscale, LAYOUTS[layout], 1, rows, T, heads, dh, rot)
        # (other alignments take other widths, with the same arithmetic on each pair)
        assert t.equal(x[:rows, :heads * dh], want) and _kept(x, rows, heads * dh)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rope_far_and_negative_positions(layout):
    t = U.torch()
    pos = t.tensor([0, 1, -1, 131071, -131072, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31], device="cuda", dtype=t.int32)
    rows, heads, dh = len(pos), 2, 64
    x, _, freq, _ = _case("f32", rows, heads, dh, dh, 0, 9)
    y = t.empty_like(x)
    A.atom_k_rope(A.ATOM_F32, x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), pos.data_ptr(), freq.data_ptr(), 1.0,
                  LAYOUTS[layout], 0, rows, 0, heads, dh, dh)
    ref, bound = _turn(_split(x, rows, heads, dh), _angles(rows, 1, pos, freq), 1.0, layout)
    _within(_split(y, rows, heads, dh), ref, bound, "f32")
    assert t.equal(y[0], x[0])  # position 0: nothing turns


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("back", [0, 1])
def test_angles_at_the_farthest_positions(layout, back):
    """Angles of 10^9 and more, the reference p freq reduced in rational numbers: heads of pairs (1, 0) give cosines and
    sines, off by the angle's cut to 2^-25 half turns and the function's own 2^-23, and nothing by the angle's size."""
    t = U.torch()
    r = np.random.default_rng(40)
    pos = np.concatenate([r.integers(2 ** 30, 2 ** 31, 40), [2 ** 31 - 1, -2 ** 31]]).astype(np.int32)
    freq = np.concatenate([r.uniform(0.4, 1.0, 124), [1.0, np.pi / 4, 1 / 3, 10000.0 ** (-1 / 64)]])
    rows, dh = len(pos), 256
    first = slice(0, 128) if layout == "half" else slice(0, dh, 2)
    second = slice(128, dh) if layout == "half" else slice(1, dh, 2)
    x = t.zeros(rows, dh, device="cuda")
    x[:, first] = 1.0
    y, p, f = t.empty_like(x), t.from_numpy(pos).cuda(), t.from_numpy(freq).cuda()
    A.atom_k_rope(A.ATOM_F32, x.data_ptr(), dh, y.data_ptr(), dh, p.data_ptr(), f.data_ptr(), 1.0, LAYOUTS[layout], back, rows,
                  0, 1, dh, dh)
    two_pi = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
    a = np.array([[float(int(i) * Fraction(w) % two_pi) for w in freq] for i in pos])
    bound = math.pi * 2.0 ** -25 + 2.0 ** -23
    got = y.double().cpu().numpy()
    off = max(np.abs(got[:, first] - np.cos(a)).max(), np.abs(got[:, second] - (-1) ** back * np.sin(a)).max())
    assert off <= bound, off


def _forward(x, gq, gk, rows, Hq, Hk, dh, angle, mscale, layout):
    """In 64 bits: y [rows][Hq + Hk][dh], its bound, x r and r."""
    t = U.torch()
    h = _split(x, rows, Hq + Hk, dh)
    r = 1.0 / t.sqrt((h * h).mean(-1, keepdim=True) + EPS)
    gain = t.cat([(gq if gq is not None else t.ones(dh, device="cuda")).double().expand(Hq, dh),
                  (gk if gk is not None else t.ones(dh, device="cuda")).double().expand(Hk, dh)])
    u = h * r * gain
    if angle is None:
        return u, u.abs() * 2.0 ** -19, h * r, r, gain
    y, e = _turn(u, angle, mscale, layout)
    # u's own error, turned: its pair's sum is in E already
    return y, e * (1 + 2.0 ** 2) + u.abs() * 2.0 ** -19, h * r, r, gain


def _norm_case(dtype, rows, Hq, Hk, Hv, dh, rot, pad, seed, far=False):
    t = U.torch()
    x, pos, freq, g = _case(dtype, rows, Hq + Hk + Hv, dh, rot, pad, seed, far)
    gq, gk = ((1 + 0.3 * t.randn(dh, device="cuda", generator=g)).to(_type(dtype)) for _ in range(2))
    return x, pos, freq, gq, gk, g


def _fwd(dtype, x, y, gq, gk, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot, stream=None):
    A.atom_k_qknorm_rope_fwd(U.dt_code(dtype), x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), _ptr(gq), _ptr(gk), EPS,
                             _ptr(pos), _ptr(freq), mscale, LAYOUTS[layout], rows, T, Hq, Hk, Hv, dh, rot, stream)


def _bwd(dtype, dy, x, dx, gq, gk, dgq, dgk, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot, ws, stream=None):
    A.atom_k_qknorm_rope_bwd(U.dt_code(dtype), dy.data_ptr(), dy.stride(0), x.data_ptr(), x.stride(0), dx.data_ptr(),
                             dx.stride(0), _ptr(gq), _ptr(gk), _ptr(dgq), _ptr(dgk), EPS, _ptr(pos), _ptr(freq), mscale,
                             LAYOUTS[layout], rows, T, Hq, Hk, Hv, dh, rot, _ptr(ws), 0 if ws is None else ws.numel(), stream)


def _ws(rows, Hq, Hk, dh):
    t = U.torch()
    return t.empty(A.atom_k_qknorm_rope_bwd_ws_bytes(rows, Hq, Hk, dh), device="cuda", dtype=t.uint8)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rows,Hq,Hk,Hv,dh,rot,pad", SHAPES)
def test_norm_forward(dtype, layout, rows, Hq, Hk, Hv, dh, rot, pad):
    t = U.torch()
    n, width, mscale, T = Hq + Hk, (Hq + Hk + Hv) * dh, 0.75, 5
    x, pos, freq, gq, gk, _ = _norm_case(dtype, rows, Hq, Hk, Hv, dh, rot, pad, 3 * rows + dh, far=rows % 2 == 1)
    for gains in ((gq, gk), (None, gk), (None, None)):
        y = _padded(rows, width, pad + 2, dtype)
        _fwd(dtype, x, y, *gains, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot)
        angle = _angles(rows, T, pos, freq) if rot else None
        ref, bound, *_ = _forward(x, *gains, rows, Hq, Hk, dh, angle, mscale, layout)
        _within(_split(y, rows, n, dh), ref, bound, dtype)
        assert t.equal(y[:rows, n * dh:width], x[:rows, n * dh:width]) and _kept(y, rows, width)
    before = x.clone()
    _fwd(dtype, x, x, None, None, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot)
    _within(_split(x, rows, n, dh), ref, bound, dtype)
    assert t.equal(x[:rows, n * dh:], before[:rows, n * dh:]) and _kept(x, rows, width)


def _gradients(dy, x, gq, gk, rows, Hq, Hk, dh, angle, mscale, layout):
    """dx, dgq, dgk in 64 bits and their bounds (see the file's head)."""
    t = U.torch()
    _, _, xh, r, gain = _forward(x, gq, gk, rows, Hq, Hk, dh, angle, mscale, layout)
    d = _split(dy, rows, Hq + Hk, dh)
    g, eg = (d, t.zeros_like(d)) if angle is None else _turn(d, angle, mscale, layout, True)
    gw = g * gain
    m = (gw * xh).mean(-1, keepdim=True)
    dx = r * (gw - xh * m)
    em = (eg * gain.abs() * xh.abs()).mean(-1, keepdim=True) + 2.0 ** -18 * (gw * xh).abs().mean(-1, keepdim=True)
    bound = r * (eg * gain.abs() + xh.abs() * em + 2.0 ** -18 * (gw.abs() + xh.abs() * m.abs()))
    terms = g * xh
    # sums: a lane's heads of each of its rows, 6 shuffles, 4 waves, 64 + 16 parts
    depth = math.ceil(rows / 4096) * (Hq + Hk) + 100
    eb = eg * xh.abs() + (2.0 ** -19 + depth * 2.0 ** -24) * terms.abs()
    return (dx, bound), (terms[:, :Hq].sum((0, 1)), eb[:, :Hq].sum((0, 1))), (terms[:, Hq:].sum((0, 1)), eb[:, Hq:].sum((0, 1)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rows,Hq,Hk,Hv,dh,rot,pad", SHAPES)
def test_norm_backward(dtype, layout, rows, Hq, Hk, Hv, dh, rot, pad):
    t = U.torch()
    n, width, mscale, T = Hq + Hk, (Hq + Hk + Hv) * dh, 1.5, 3
    x, pos, freq, gq, gk, g = _norm_case(dtype, rows, Hq, Hk, Hv, dh, rot, pad, 5 * rows + dh, far=rows % 2 == 0)
    dy = _padded(rows, width, pad + 1, dtype)
    dy[:rows, :width] = t.randn(rows, width, device="cuda", generator=g) * 0.01
    angle = _angles(rows, T, pos, freq) if rot else None
    for gains in ((gq, gk), (None, None)):
        dx = _padded(rows, width, pad, dtype)
        dg = t.full((2, dh + 4), 55.0, device="cuda")
        ws = _ws(rows, Hq, Hk, dh)
        _bwd(dtype, dy, x, dx, *gains, dg[0], dg[1], pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot, ws)
        refs = _gradients(dy, x, *gains, rows, Hq, Hk, dh, angle, mscale, layout)
        _within(_split(dx, rows, n, dh), *refs[0], dtype)
        assert t.equal(dx[:rows, n * dh:width], dy[:rows, n * dh:width]) and _kept(dx, rows, width)
        for k in (0, 1):
            _within(dg[k, :dh], *refs[1 + k], "f32")
        assert (dg[:, dh:] == 55.0).all()
    # one gain's gradient alone, and none; in place
    alone, other = t.empty(dh, device="cuda"), _padded(rows, width, pad, dtype)
    _bwd(dtype, dy, x, other, None, None, None, alone, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot, ws)
    assert t.equal(other, dx) and t.equal(alone, dg[1, :dh])
    _bwd(dtype, dy, x, other, None, None, alone, None, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot, ws)
    assert t.equal(alone, dg[0, :dh])
    _bwd(dtype, dy, x, dy, None, None, None, None, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot, None)
    _within(_split(dy, rows, n, dh), *refs[0], dtype)
    assert _kept(dy, rows, width)


# The widest accesses: every buffer aligned, in leading dimensions of its own.  One side and all of them in a group, two
# groups, several rows a wave (to 32) with some behind the last one, and as many heads as lanes for them.
ALIGNED = [  # rows, Hq, Hk, Hv, dh, rot, T
    (1, 1, 1, 1, 64, 64, 1), (37, 12, 2, 2, 128, 128, 5), (300, 8, 2, 2, 96, 0, 1), (4101, 4, 1, 1, 64, 64, 3),
    (4101, 1, 1, 1, 128, 96, 2048), (9001, 2, 1, 0, 64, 32, 1), (9001, 0, 1, 1, 64, 64, 100), (8200, 3, 0, 2, 32, 32, 7),
    (40003, 1, 0, 0, 64, 64, 3), (70001, 1, 0, 0, 16, 16, 1), (70001, 1, 1, 0, 16, 16, 40000), (2050, 5, 3, 2, 80, 80, 9),
    (600, 20, 4, 4, 256, 256, 77), (1030, 16, 16, 16, 128, 64, 1030)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rows,Hq,Hk,Hv,dh,rot,T", ALIGNED)
def test_aligned_rows(dtype, layout, rows, Hq, Hk, Hv, dh, rot, T):
    t = U.torch()
    n, heads, mscale = Hq + Hk, Hq + Hk + Hv, 1.25
    width = heads * dh
    for far in (False, True):
        x, pos, freq, gq, gk, g = _norm_case(dtype, rows, Hq, Hk, Hv, dh, rot, 0, rows + dh + far, far)
        angle = _angles(rows, T, pos, freq) if rot else None
        y = _padded(rows, width, 16, dtype)
        A.atom_k_rope(U.dt_code(dtype), x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), _ptr(pos), _ptr(freq), mscale,
                      LAYOUTS[layout], 0, rows, T, heads, dh, rot)
        ref = _split(x, rows, heads, dh)
        ref, bound = _turn(ref, angle, mscale, layout) if rot else (ref, t.zeros_like(ref))
        _within(_split(y, rows, heads, dh), ref, bound, dtype)
        assert _kept(y, rows, width)
        y = _padded(rows, width, 16, dtype)
        _fwd(dtype, x, y, gq, gk, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot)
        ref, bound, *_ = _forward(x, gq, gk, rows, Hq, Hk, dh, angle, mscale, layout)
        _within(_split(y, rows, n, dh), ref, bound, dtype)
        assert t.equal(y[:rows, n * dh:width], x[:rows, n * dh:width]) and _kept(y, rows, width)
        # gradients; infinities and NaN in the values' part are copied and touch nothing else
        dy, dx = _padded(rows, width, 8, dtype), _padded(rows, width, 24, dtype)
        dy[:rows, :width] = t.randn(rows, width, device="cuda", generator=g) * 0.01
        if Hv:
            dy[0, n * dh], dy[rows - 1, width - 1] = math.inf, float("nan")
        dg = t.full((2, dh), 55.0, device="cuda")
        _bwd(dtype, dy, x, dx, gq, gk, dg[0], dg[1], pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot,
             _ws(rows, Hq, Hk, dh))
        refs = _gradients(dy, x, gq, gk, rows, Hq, Hk, dh, angle, mscale, layout)
        _within(_split(dx, rows, n, dh), *refs[0], dtype)
        bits = t.int16 if dtype == "bf16" else t.int32
        assert t.equal(dx[:rows, n * dh:width].contiguous().view(bits), dy[:rows, n * dh:width].contiguous().view(bits))
        assert _kept(dx, rows, width)
        for k in (0, 1):
            _within(dg[k], *refs[1 + k], "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_gradient_against_differences(layout):
    """<dx, e> against the central difference of <dy, y> along e, the forward in 64 bits: h^2 of the third derivative
    (1e-8) and 2^-52 / h (1e-12) relative to the sums' terms, and the gradient's own fp32 (2^-18)."""
    t = U.torch()
    rows, Hq, Hk, dh, rot, h = 6, 3, 2, 64, 48, 1e-4
    x, pos, freq, gq, gk, g = _norm_case("f32", rows, Hq, Hk, 0, dh, rot, 0, 21, far=True)
    n = (Hq + Hk) * dh
    dy = t.randn(rows + 1, n, device="cuda", generator=g)
    dx, dg, ws = t.empty_like(x), t.empty(2, dh, device="cuda"), _ws(rows, Hq, Hk, dh)
    _bwd("f32", dy, x, dx, gq, gk, dg[0], dg[1], pos, freq, 1.25, layout, rows, 0, Hq, Hk, 0, dh, rot, ws)
    angle = _angles(rows, 1, pos, freq)

    def value(x, gq, gk):
        y, *_ = _forward(x, gq, gk, rows, Hq, Hk, dh, angle, 1.25, layout)
        return (y * _split(dy, rows, Hq + Hk, dh)).sum().item()

    X, Gq, Gk = x.double(), gq.double(), gk.double()
    for grad, move in ((dx[:rows], lambda e: (X + t.nn.functional.pad(e, (0, 0, 0, 1)), Gq, Gk)),
                       (dg[0], lambda e: (X, Gq + e, Gk)), (dg[1], lambda e: (X, Gq, Gk + e))):
        e = t.randn(grad.shape, device="cuda", generator=g, dtype=t.float64)
        diff = (value(*move(h * e)) - value(*move(-h * e))) / (2 * h)
        size = (grad.double() * e).abs().sum().item()
        assert abs(diff - (grad.double() * e).sum().item()) <= size * (2.0 ** -17 + 1e-6)


@pytest.mark.gpu
def test_rows_do_not_mix():
    """An infinity or a NaN stays in its head (and in its gradient's sum), and in its pair where nothing is normed."""
    t = U.torch()
    rows, H, dh = 3, 4, 64
    x, _, freq, gq, gk, _ = _norm_case("bf16", rows, H, H, H, dh, dh, 0, 31)
    clean, y, z = x.clone(), t.empty_like(x), t.empty_like(x)
    x[1, 2 * dh + 5] = float("nan")
    x[2, 11 * dh + 1] = float("inf")  # a value: copied
    _fwd("bf16", clean, z, gq, gk, None, freq, 1.0, "half", rows, rows, H, H, H, dh, dh)
    _fwd("bf16", x, y, gq, gk, None, freq, 1.0, "half", rows, rows, H, H, H, dh, dh)
    bad = t.zeros_like(x, dtype=t.bool)
    bad[1, 2 * dh:3 * dh] = True
    assert y[bad].isnan().all()
    bad[2, 11 * dh + 1] = True
    assert t.equal(y[:rows][~bad[:rows]], z[:rows][~bad[:rows]]) and y[2, 11 * dh + 1] == float("inf")
    A.atom_k_rope(A.ATOM_BF16, x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), None, freq.data_ptr(), 1.0,
                  A.ATOM_ROPE_HALF, 0, rows, rows, 2 * H, dh, 32)
    assert y[1, 2 * dh:3 * dh].isnan().sum() == 2  # its pair
    x[0, :2 * dh] = 0.0  # heads of zeros: zeros
    _fwd("bf16", x, y, gq, gk, None, freq, 1.0, "pairs", rows, rows, H, H, H, dh, dh)
    assert (y[0, :2 * dh] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,Hq,Hk,Hv,dh,rot,T", ALIGNED)
def test_aligned_rows_in_place(dtype, rows, Hq, Hk, Hv, dh, rot, T):
    """The widest accesses, several rows a wave, with results where the inputs were."""
    t = U.torch()
    n, width = Hq + Hk, (Hq + Hk + Hv) * dh
    x, pos, freq, gq, gk, g = _norm_case(dtype, rows, Hq, Hk, Hv, dh, rot, 16, rows + dh + 7)
    angle = _angles(rows, T, pos, freq) if rot else None
    dy = _padded(rows, width, 8, dtype)
    dy[:rows, :width] = t.randn(rows, width, device="cuda", generator=g) * 0.01
    dg, values = t.full((2, dh), 55.0, device="cuda"), dy[:rows, n * dh:width].clone()
    refs = _gradients(dy, x, gq, gk, rows, Hq, Hk, dh, angle, 0.75, "half")
    _bwd(dtype, dy, x, dy, gq, gk, dg[0], dg[1], pos, freq, 0.75, "half", rows, T, Hq, Hk, Hv, dh, rot, _ws(rows, Hq, Hk, dh))
    _within(_split(dy, rows, n, dh), *refs[0], dtype)
    assert t.equal(dy[:rows, n * dh:width], values) and _kept(dy, rows, width)
    for k in (0, 1):
        _within(dg[k], *refs[1 + k], "f32")
    y, values = x.clone(), x[:rows, n * dh:width].clone()
    ref, bound, *_ = _forward(x, gq, gk, rows, Hq, Hk, dh, angle, 0.75, "half")
    _fwd(dtype, y, y, gq, gk, pos, freq, 0.75, "half", rows, T, Hq, Hk, Hv, dh, rot)
    _within(_split(y, rows, n, dh), ref, bound, dtype)
    assert t.equal(y[:rows, n * dh:width], values) and _kept(y, rows, width)
    if rot:
        ref, bound = _turn(_split(x, rows, n, dh), angle, 0.75, "half")
        A.atom_k_rope(U.dt_code(dtype), x.data_ptr(), x.stride(0), x.data_ptr(), x.stride(0), None, _ptr(freq), 0.75,
                      A.ATOM_ROPE_HALF, 0, rows, T, n, dh, rot)
        _within(_split(x, rows, n, dh), ref, bound, dtype)
        assert t.equal(x[:rows, n * dh:width], values) and _kept(x, rows, width)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,Hv,dh,rot", [(65534, 1, 1, 2, 2), (1, 65535, 0, 16, 16), (0, 1, 65535, 4, 0)])
def test_most_heads(dtype, Hq, Hk, Hv, dh, rot):
    t = U.torch()
    rows, T, n, width = 3, 2, Hq + Hk, (Hq + Hk + Hv) * dh
    x, pos, freq, gq, gk, g = _norm_case(dtype, rows, Hq, Hk, Hv, dh, rot, 0, 61)
    angle = _angles(rows, T, pos, freq) if rot else None
    y, dx = _padded(rows, width, 0, dtype), _padded(rows, width, 0, dtype)
    _fwd(dtype, x, y, gq, gk, pos, freq, 1.0, "half", rows, T, Hq, Hk, Hv, dh, rot)
    ref, bound, *_ = _forward(x, gq, gk, rows, Hq, Hk, dh, angle, 1.0, "half")
    _within(_split(y, rows, n, dh), ref, bound, dtype)
    dy = t.randn(rows + 1, width, device="cuda", generator=g).to(_type(dtype))
    dg = t.full((2, dh), 55.0, device="cuda")
    _bwd(dtype, dy, x, dx, gq, gk, dg[0], dg[1], pos, freq, 1.0, "half", rows, T, Hq, Hk, Hv, dh, rot, _ws(rows, Hq, Hk, dh))
    refs = _gradients(dy, x, gq, gk, rows, Hq, Hk, dh, angle, 1.0, "half")
    _within(_split(dx, rows, n, dh), *refs[0], dtype)
    for k in (0, 1):
        _within(dg[k], *refs[1 + k], "f32")
    for a, b in ((x, y), (dy, dx)):
        assert t.equal(a[:rows, n * dh:], b[:rows, n * dh:]) and _kept(b, rows, width)


@pytest.mark.gpu
def test_most_rows():
    """2^31 - 1 rows, in place: they repeat with the positions, so every period has the first one's bits."""
    t = U.torch()
    rows, T = 2 ** 31 - 1, 1021
    base = t.randn(T, 2, device="cuda", generator=t.Generator(device="cuda").manual_seed(62)).to(t.bfloat16)
    x = base.repeat(rows // T + 1, 1)
    x[rows:] = 77.0
    freq, y = _freq(2), t.empty_like(base)
    for a, b, n in ((base, y, T), (x, x, rows)):
        A.atom_k_rope(A.ATOM_BF16, a.data_ptr(), 2, b.data_ptr(), 2, None, freq.data_ptr(), 1.0, A.ATOM_ROPE_HALF, 0, n, T, 1,
                      2, 2)
    whole, rest = rows // T, rows % T
    assert bool((x[:whole * T].view(whole, 2 * T) == y.view(1, 2 * T)).all())
    assert t.equal(x[whole * T:rows], y[:rest]) and bool((x[rows:] == 77.0).all())


@pytest.mark.gpu
def test_no_rows_and_no_heads():
    t = U.torch()
    A.atom_k_rope(A.ATOM_BF16, None, 0, None, 0, None, None, 1.0, 0, 0, 0, 0, 4, 64, 64)
    A.atom_k_rope(A.ATOM_BF16, None, 0, None, 0, None, None, 1.0, 0, 0, 5, 0, 0, 64, 64)
    A.atom_k_qknorm_rope_fwd(A.ATOM_F32, None, 0, None, 0, None, None, EPS, None, None, 1.0, 0, 0, 0, 1, 1, 1, 64, 64)
    dg = t.full((2, 64), 5.0, device="cuda")
    A.atom_k_qknorm_rope_bwd(A.ATOM_F32, None, 0, None, 0, None, 0, None, None, dg[0].data_ptr(), dg[1].data_ptr(), EPS,
                             None, None, 1.0, 0, 0, 0, 1, 1, 1, 64, 64, None, 0)
    assert (dg == 0).all()


@pytest.mark.gpu
def test_streams_graphs_and_repeats():
    """Two streams at once, and a captured call replayed on new inputs, give what each gives alone, to the bit."""
    t = U.torch()
    rows, H, dh = 700, 6, 128
    width = 3 * H * dh
    cases = [_norm_case("bf16", rows, H, H, H, dh, dh, 0, 50 + i) for i in range(2)]
    dys = [t.randn(rows + 1, width, device="cuda").to(t.bfloat16) for _ in cases]

    def buffers():
        return dict(y=t.zeros(rows + 1, width, device="cuda", dtype=t.bfloat16), dg=t.zeros(2, dh, device="cuda"),
                    dx=t.zeros(rows + 1, width, device="cuda", dtype=t.bfloat16), ws=_ws(rows, H, H, dh))

    def both(c, dy, b, stream):
        x, _, freq, gq, gk, _ = c
        _fwd("bf16", x, b["y"], gq, gk, None, freq, 1.0, "half", rows, 100, H, H, H, dh, dh, stream)
        _bwd("bf16", dy, x, b["dx"], gq, gk, b["dg"][0], b["dg"][1], None, freq, 1.0, "half", rows, 100, H, H, H, dh, dh,
             b["ws"], stream)

    alone, at_once = [buffers() for _ in cases], [buffers() for _ in cases]
    for c, dy, b in zip(cases, dys, alone):
        both(c, dy, b, None)
    t.cuda.synchronize()
    streams = [t.cuda.Stream(), t.cuda.Stream()]
    for _ in range(3):
        for c, dy, b, s in zip(cases, dys, at_once, streams):
            both(c, dy, b, s.cuda_stream)
    t.cuda.synchronize()
    for a, b in zip(alone, at_once):
        assert all(t.equal(a[k], b[k]) for k in ("y", "dx", "dg"))
    g, s, b, eager = t.cuda.CUDAGraph(), t.cuda.Stream(), buffers(), buffers()
    s.wait_stream(t.cuda.current_stream())
    with t.cuda.graph(g, stream=s):
        both(cases[0], dys[0], b, t.cuda.current_stream().cuda_stream)
    for i in range(3):
        cases[0][0].copy_(cases[1][0] * (i + 1))
        both(cases[0], dys[0], eager, None)
        g.replay()
        t.cuda.synchronize()
        assert all(t.equal(eager[k], b[k]) for k in ("y", "dx", "dg"))


@pytest.mark.gpu
def test_far_rows():
    """Offsets beyond 32 bits: rows 2^22 elements apart, the last of them behind 2^32."""
    t = U.torch()
    rows, ld, dh = 1030, 1 << 22, 64
    x = t.empty(rows * ld, device="cuda", dtype=t.bfloat16).view(rows, ld)
    x[:, :2 * dh] = t.randn(rows, 2 * dh, device="cuda")
    small = x[:, :2 * dh].contiguous()
    freq, y = _freq(dh), t.empty_like(small)
    for src, dst in ((small, y), (x, x)):
        A.atom_k_rope(A.ATOM_BF16, src.data_ptr(), src.stride(0), dst.data_ptr(), dst.stride(0), None, freq.data_ptr(), 1.0,
                      A.ATOM_ROPE_HALF, 0, rows, 4096, 2, dh, dh)
    assert t.equal(x[:, :2 * dh], y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_rows_several_a_wave(dtype):
    """Few heads of many rows, several rows a wave, 2^19 elements apart and the last of them behind 2^32: the bits of rows
    side by side, in every call."""
    t = U.torch()
    rows, T, dh, H = 8200, 77, 64, 3
    width, ld = H * dh, 2 ** 19 + 16
    near = _norm_case(dtype, rows, 1, 1, 1, dh, dh, 0, 41)
    x, _, freq, gq, gk, g = near
    dy = t.randn(rows, width, device="cuda", generator=g).to(_type(dtype))
    far = t.empty(rows * ld, device="cuda", dtype=_type(dtype)).view(rows, ld)
    fx, fdy, fy, fdx = (far[:, i * width:(i + 1) * width] for i in range(4))
    fx.copy_(x[:rows])
    fdy.copy_(dy)
    out = []
    for a, b, y, dx in ((x, dy, t.empty_like(x), t.empty_like(dy)), (fx, fdy, fy, fdx)):
        dg = t.empty(2, dh, device="cuda")
        A.atom_k_rope(U.dt_code(dtype), a.data_ptr(), a.stride(0), y.data_ptr(), y.stride(0), None, freq.data_ptr(), 1.0,
                      A.ATOM_ROPE_HALF, 0, rows, T, H, dh, dh)
        turned = y[:rows].clone()
        _fwd(dtype, a, y, gq, gk, None, freq, 1.0, "pairs", rows, T, 1, 1, 1, dh, dh)
        _bwd(dtype, b, a, dx, gq, gk, dg[0], dg[1], None, freq, 1.0, "pairs", rows, T, 1, 1, 1, dh, dh, _ws(rows, 1, 1, dh))
        out.append((turned, y[:rows].clone(), dx.clone(), dg))
    assert all(t.equal(p, q) for p, q in zip(*out))


def test_frequencies():
    i = np.arange(32)
    plain = 10000.0 ** (-i / 32)
    close = lambda a, b: np.allclose(a, b, rtol=1e-13, atol=0)  # noqa: E731
    assert close(A.atom_rope_freqs(64), plain)
    assert close(A.atom_rope_freqs(64, 500.0), 500.0 ** (-i / 32))
    assert close(A.atom_rope_freqs(64, scaling=A.ATOM_ROPE_LINEAR, factor=4.0), plain / 4)
    base = A.atom_rope_freqs(64, scaling=A.ATOM_ROPE_BASE, factor=8.0)
    assert base[0] == 1.0 and close(base[-1], plain[-1] / 8) and (base <= plain).all()
    parts = A.atom_rope_freqs(64, scaling=A.ATOM_ROPE_PARTS, factor=16.0, trained=4096.0, slow=1.0, fast=32.0)
    turns = 4096.0 * plain / (2 * np.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    assert close(parts, plain * (keep + (1 - keep) / 16))
    assert (parts[turns >= 32] == A.atom_rope_freqs(64)[turns >= 32]).all() and close(parts[turns <= 1], plain[turns <= 1] / 16)
    assert A.atom_rope_freqs(2, scaling=A.ATOM_ROPE_BASE, factor=8.0) == [1.0]


@pytest.mark.parametrize("rot,factor", [(4, 1e160), (4, 1e-200), (6, 1e250), (64, 1e300), (256, 1e-290)])
def test_frequencies_of_bases_beyond_the_numbers(rot, factor):
    """base factor^(rot/(rot-2)) need not be a double where the frequencies are: by logarithms, off by 2^-52 of 1000
    and a rounding of each power."""
    i = np.arange(rot // 2)
    got = A.atom_rope_freqs(rot, scaling=A.ATOM_ROPE_BASE, factor=factor)
    ref = -2.0 * i / rot * math.log(1e4) - 2.0 * i / (rot - 2) * math.log(factor)
    assert got[0] == 1.0 and np.abs(np.log(got) - ref).max() <= 1000 * 2.0 ** -50
    assert abs(got[-1] * factor * 1e4 ** ((rot - 2) / rot) - 1) <= 2.0 ** -50


@pytest.mark.parametrize("kw", [dict(rot=256, base=5e-324), dict(rot=64, scaling=1, factor=1e-320),
                                dict(rot=4, base=1e-300, scaling=2, factor=1e-300), dict(rot=64, scaling=3, factor=1e-320)])
def test_frequencies_that_are_not_finite(kw):
    with pytest.raises(A.AtomError) as e:
        A.atom_rope_freqs(**kw)
    assert e.value.status == A.ATOM_EINVAL


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=3), dict(rot=258), dict(rot=64, base=0.0), dict(rot=64, base=math.inf),
                                dict(rot=64, base=math.nan), dict(rot=64, scaling=4), dict(rot=64, scaling=1, factor=0.0),
                                dict(rot=64, scaling=3, slow=2.0, fast=2.0), dict(rot=64, scaling=3, trained=0.0),
                                dict(rot=64, scaling=2, factor=math.nan)])
def test_frequencies_refused(kw):
    with pytest.raises(A.AtomError) as e:
        A.atom_rope_freqs(**kw)
    assert e.value.status == A.ATOM_EINVAL


def _refused(fn, *args):
    with pytest.raises(A.AtomError) as e:
        fn(*args)
    assert e.value.status == A.ATOM_EINVAL


def test_refusals():
    """Each argument out of its range alone, on the host (no pointer is looked at)."""
    rope = dict(dtype=1, x=4096, ldx=512, y=8192, ldy=512, pos=None, freq=4096, mscale=1.0, layout=0, transposed=0, rows=4,
                T=4, heads=4, dh=128, rot=128)
    for k, v in [("dtype", 2), ("x", None), ("x", 4097), ("ldx", 511), ("y", None), ("y", 8193), ("ldy", 511), ("pos", 4098),
                 ("freq", None), ("freq", 4100), ("mscale", math.inf), ("mscale", math.nan), ("layout", 2), ("layout", -1),
                 ("rows", -1), ("rows", 1 << 31), ("T", 0), ("heads", -1), ("heads", (1 << 16) + 1), ("dh", 127), ("dh", 0),
                 ("dh", 258), ("rot", 130), ("rot", 63), ("rot", -2), ("ldx", 1 << 40)]:
        _refused(A.atom_k_rope, *{**rope, k: v}.values())
    _refused(A.atom_k_rope, *{**rope, "y": 4096, "ldy": 1024}.values())
    norm = dict(dtype=1, x=4096, ldx=1536, y=8192, ldy=1536, gq=4096, gk=4096, eps=1e-6, pos=None, freq=4096, mscale=1.0,
                layout=0, rows=4, T=4, Hq=4, Hk=4, Hv=4, dh=128, rot=128)
    for k, v in [("dtype", 7), ("x", None), ("y", None), ("ldx", 1535), ("ldy", 1535), ("gq", 4097), ("gk", 4097), ("eps", 0.0), ("eps", 1e-39),
                 ("eps", -1.0), ("eps", math.nan), ("eps", math.inf), ("freq", None), ("T", 0), ("Hq", -1), ("Hk", -1),
                 ("Hv", -1), ("Hv", 1 << 16), ("dh", 1), ("rot", 200)]:
        _refused(A.atom_k_qknorm_rope_fwd, *{**norm, k: v}.values())
    _refused(A.atom_k_qknorm_rope_fwd, *{**norm, "y": 4096, "ldy": 2048}.values())
    n = A.atom_k_qknorm_rope_bwd_ws_bytes(4, 4, 4, 128)
    assert n > 0
    bwd = dict(dtype=1, dy=12288, lddy=1536, x=4096, ldx=1536, dx=8192, lddx=1536, gq=4096, gk=4096, dgq=4096, dgk=4096,
               eps=1e-6, pos=None, freq=4096, mscale=1.0, layout=0, rows=4, T=4, Hq=4, Hk=4, Hv=4, dh=128, rot=128, ws=4096,
               ws_bytes=n)
    for k, v in [("dtype", -1), ("dy", None), ("x", None), ("dx", None), ("dx", 4096), ("lddy", 1535), ("ldx", 1), ("lddx", 0),
                 ("gq", 4097), ("dgq", 4098), ("dgk", 4098), ("eps", 0.0), ("mscale", math.nan), ("ws", None), ("ws", 4104),
                 ("ws_bytes", n - 1), ("layout", 3), ("rows", -1)]:
        _refused(A.atom_k_qknorm_rope_bwd, *{**bwd, k: v}.values())
    _refused(A.atom_k_qknorm_rope_bwd, *{**bwd, "dx": 12288, "lddx": 2048}.values())
    for args in [(-1, 4, 4, 128), (4, -1, 4, 128), (4, 4, -1, 128), (4, 4, 4, 127), (4, 4, 4, 0), (1 << 31, 4, 4, 128)]:
        assert A.atom_k_qknorm_rope_bwd_ws_bytes(*args) == 0
