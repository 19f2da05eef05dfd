"""The linear head's loss and gradients of fp32 operands in three bf16 planes (x = h + m + l), six products of planes.

A product of two numbers in planes keeps h h', h m', m h', m m', h l' and l h'; what is left out is at most 2^-24 of
it (m is up to 2^-8, l up to 2^-17).
Inputs in which every result is one such product show each of the six, at every tile that the library's rule takes:
without one of the last three, the smallest, a result of random mantissas is 2^-18.5 off on average."""
import pytest

from paper_2403_10504_amd import atom as A
from tests import gpu_util as U
from tests.test_linear_xent import DZ, LSE, SCALE_ACC, SCALE_F32, U32, _bwd, _case, _fwd

# What is left out, up to 2^-24, and roundings: of the last pass with what came
# before it, two of the accumulators' sets, one of the result (the passes before
# round numbers of 2^-8 of theirs)
SIX = 6 * U32

# rows, V, d, piece: together they take every tile of every product, with k whole and in ranges
SIZES = [(805, 41964, 428, 40731), (5456, 4742, 536, 1491), (2257, 7350, 404, 4435), (584, 32977, 360, 15424),
         (6672, 513, 1264, 251), (527, 1594, 5480, 0), (12524, 998, 344, 137), (4565, 340, 2772, 47),
         (881, 2323, 2100, 134), (803, 14816, 364, 756), (1565, 1332, 2660, 728)]
# W in two and three ranges of rows; the first one's end inside a tile, one cut in tiles of two kinds, whole tiles
RANGES = [(800, 20011, 2052, 0), (900, 50257, 1028, 0), (770, 43001, 1540, 0)]


def _ranges(rows, V, d):
    step = U.xent_plan("f32", rows, V, d)[1]
    return [(v, min(V, v + step)) for v in range(0, V, step)]


def _pieces(rows, V, d, piece):
    _, _, _, width, last, _ = U.xent_plan("f32", rows, V, d, piece)
    out, v = [], 0
    while v < V:
        n = V - v if V - v <= last else width
        out.append((v, v + n))
        v += n
    return out


def _products(rows, V, d, piece):
    """(product, tile, k in ranges) of each launch of the forward and both kinds of backward call."""
    ws = U.xent_plan("f32", rows, V, d, piece)[5]
    got = set()
    if U.xent_plan("f32", rows, V, d)[0]:
        for a, b in _ranges(rows, V, d):
            got |= {("loss", x[:2], False) for x in U.loss_launches("planes", 1, 1, LSE, rows, b - a, d)}
    for i, (a, b) in enumerate(_pieces(rows, V, d, piece)):
        got |= {("dz", x[:2], False) for x in U.loss_launches("planes", 1, 1, DZ, rows, b - a, d)}
        dx = SCALE_ACC if i else SCALE_F32
        got |= {(f"dx{dx}", x[:2], x[2] > 1) for x in U.loss_launches("planes", 1, 0, dx, rows, d, b - a, ws)}
        for dw in (SCALE_F32, SCALE_ACC):
            got |= {(f"dw{dw}", x[:2], x[2] > 1) for x in U.loss_launches("planes", 0, 0, dw, b - a, d, rows, ws)}
    return got


def test_sizes_take_every_product():
    """The sizes below reach every tile of every product, and several ranges of W (no GPU needed)."""
    tiles = [(256, 256), (256, 192), (256, 128), (128, 128), (64, 64)]
    want = {(p, t, False) for p in ("loss", "dz") for t in tiles}
    want |= {(f"{p}{e}", t, s) for p in ("dx", "dw") for e in (SCALE_F32, SCALE_ACC) for t in tiles for s in (False, True)}
    got = set()
    for s in SIZES:
        assert U.xent_plan("f32", *s)[2]
        got |= _products(*s)
    assert got >= want, sorted(want - got)
    assert [len(_ranges(*s[:3])) for s in RANGES] == [2, 2, 3]
    first = U.loss_launches("planes", 1, 1, LSE, RANGES[0][0], _ranges(*RANGES[0][:3])[0][1], RANGES[0][2])
    assert len(first) == 1 and _ranges(*RANGES[0][:3])[0][1] % first[0][1]
    assert len(U.loss_launches("planes", 1, 1, LSE, RANGES[1][0], _ranges(*RANGES[1][:3])[0][1], RANGES[1][2])) == 2


def test_single_products_show_each_pass():
    """The arithmetic of the bound: six products of planes are well inside it, any five are not (no GPU needed)."""
    t = U.torch()
    g = t.Generator().manual_seed(5)
    n = 513  # the fewest tokens of a size
    a, b = (2.0 + 2.0 * t.rand(n, generator=g) for _ in range(2))

    def planes(x):
        h = x.bfloat16().float()
        m = (x - h).bfloat16().float()
        return [h.double(), m.double(), (x - h - m).bfloat16().double()]

    pa, pb = planes(a), planes(b)
    assert t.equal(sum(pa), a.double())
    exact = a.double() * b.double()
    terms = [pa[i] * pb[j] for i, j in ((0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0))]
    off = lambda z: ((z - exact).abs() / exact).max().item()  # noqa: E731
    assert off(sum(terms)) <= U32
    for k in range(6):
        assert off(sum(terms) - terms[k]) > 4 * SIX


def _mantissas(g, shape, lo):
    """Random numbers in [lo, 2 lo) with all 24 bits."""
    t = U.torch()
    return lo * (1.0 + t.rand(shape, device="cuda", generator=g))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V,d,piece", SIZES + RANGES)
def test_loss_of_single_products(rows, V, d, piece):
    """A row of x has one entry; the target's logit is one product, at least 32 above all others: lse is that product."""
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(rows + V)
    n, c = t.arange(rows, device="cuda"), t.arange(d, device="cuda")
    sign = 1.0 - 2.0 * t.randint(0, 2, (d,), device="cuda", generator=g)
    x = t.zeros((rows, d), device="cuda")
    x[n, n % d] = _mantissas(g, (rows,), 2.0) * sign[n % d]
    w = -_mantissas(g, (V, d), 8.0) * sign
    # columns at the ends of the ranges are targets too
    edges = sorted({v for a, b in _ranges(rows, V, d) for v in (a, b - 1)})
    top = t.randint(0, V, (d,), device="cuda", generator=g)
    top[:len(edges)] = t.tensor(edges, device="cuda")
    w[top, c] *= -1.0
    tgt = top[n % d].int()
    loss, lse, behind = _fwd("f32", x, w, tgt, d)
    z = x[n, n % d].double() * w[top[n % d], n % d].double()
    assert z.min().item() >= 16.0
    assert ((lse[:rows].double() - z).abs() <= (SIX + U32) * z).all()
    # V others, e^-32 and less beside 1
    assert (loss[:rows] >= 0).all() and (loss[:rows] <= V * 2e-14 + U32).all()
    assert lse[rows] == 77.0 and (behind == 0xA5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("epi", [A.ATOM_EPI_STORE, A.ATOM_EPI_ACC_F32])
@pytest.mark.parametrize("rows,V,d,piece", SIZES)
def test_gradients_of_single_products(rows, V, d, piece, epi):
    """With lse infinite p is 0 and dz the weight of the token at its target; no two tokens share one.  Each entry of dx
    and dW is one product."""
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(rows + V + 1)
    sign = lambda s: 1.0 - 2.0 * t.randint(0, 2, s, device="cuda", generator=g)  # noqa: E731
    x = _mantissas(g, (rows, d), 1.0) * sign((rows, d))
    w = _mantissas(g, (V, d), 4.0) * sign((V, d))
    drow = _mantissas(g, (rows,), 1.0) * sign((rows,))
    m = min(rows, V)
    edges = t.tensor(sorted({v for a, b in _pieces(rows, V, d, piece) for v in (a, b - 1)}), device="cuda")[:m]
    rest = t.randperm(V, device="cuda", generator=g)
    pick = t.cat((edges, rest[~t.isin(rest, edges)]))[:m]
    who = t.randperm(rows, device="cuda", generator=g)[:m]
    tgt = t.full((rows,), A.ATOM_XENT_IGNORE, device="cuda", dtype=t.int32)
    tgt[who] = pick.int()
    lse = t.full((rows,), float("inf"), device="cuda")
    start = 0.0
    dx, dw = _bwd("f32", x, w, tgt, lse, d, drow, 1.0, piece, epi, start=start)
    want = t.zeros((rows, d), device="cuda", dtype=t.float64)
    want[who] = -drow[who].double().unsqueeze(1) * w[pick].double()
    assert ((dx.double() - want).abs() <= SIX * want.abs()).all()
    want = t.zeros((V, d), device="cuda", dtype=t.float64)
    want[pick] = -drow[who].double().unsqueeze(1) * x[who].double()
    assert ((dw.double() - want).abs() <= SIX * want.abs()).all()


def _rms(a):
    return a.double().square().mean().sqrt().item()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V,d", [(1030, 8201, 516), (2100, 4097, 516), (1100, 2001, 2052)])
def test_rms_error(rows, V, d):
    """Random inputs: how far loss and gradients are from 64 bits, all entries together.

    A sum of k terms of random signs is a chain of at most k / 4 roundings (matrix instructions add four products at
    least).  Each is off by at most 2^-24 of the partial sum, 2^-24 / sqrt 3 rms; partial sums grow with the root of
    their terms, so on average their squares are half the last one's: 2^-24 sqrt(k / 24) of the sum in all."""
    t = U.torch()
    assert U.xent_plan("f32", rows, V, d)[0] and U.xent_plan("f32", rows, V, d)[2]
    x, w, tgt = _case("f32", rows, V, d, 0.1, 90)
    loss, lse, _ = _fwd("f32", x, w, tgt, d)
    scale = 1.0 / rows
    z = x.double() @ w.double().T
    on = (tgt >= 0).double()
    rlse = t.logsumexp(z, 1)
    one = t.zeros_like(z).scatter_(1, tgt.long().clamp(min=0).unsqueeze(1), 1.0)
    rloss = (rlse - (z * one).sum(1)) * on
    dz = (t.exp(z - rlse.unsqueeze(1)) - one) * on.unsqueeze(1) * scale
    dx, dw = _bwd("f32", x, w, tgt, lse, d, scale=scale)
    chain = lambda k: U32 * (k / 24) ** 0.5  # noqa: E731
    # a logit; lse and loss: rounded (their size) and with a few roundings of the sum of exponentials
    ez = chain(d) * _rms(z)
    el = U32 * (rlse.abs().max().item() + 8.0)
    assert _rms(loss[:rows] - rloss) <= ez + el
    # p is off by ez and el of itself, which is no more than all of dz
    for got, ref, k in ((dx, dz @ w.double(), V), (dw, dz.T @ x.double(), rows)):
        assert _rms(got - ref) <= (chain(k) + ez + el + U32) * _rms(ref)
