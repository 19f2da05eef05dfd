"""The work of the operators around a GPT block's attention: rotary positions,
norms of queries and keys with the rotation in the same pass, and attention to
an encoder's states of another length.

Operations (field "op"):
  rope    y = mscale R(p) x for every head of a row: R turns pair i of the
          first `rot` elements by the angle p freq_i, p the row's position; the
          rest is copied.  Pairs are (i, i + rot/2) ("half") or (2i, 2i + 1)
          ("pairs")                                           (atom_k_rope)
  norm    y = R(p) (g * x rsqrt(mean x^2 + eps)) for each head of queries and of
          keys, the heads of values copied; "bwd": dx and the gradients of both
          gains from dy                          (atom_k_qknorm_rope_fwd, _bwd)
  cross   o = softmax(scale q k^T) v with lse, per sequence and head, Hq query
          heads on Hk heads of keys and values; "bwd": dq, dk, dv from dout, o
          and lse                                 (atom_k_cross_attn_fwd, _bwd)

Heads, widths and token counts are those of the GPT configurations: tiny (4
heads of 64, 2 x 128 tokens, fp32), Small (12 of 64, 8 x 2048), XL (16 of 128),
6.7B (32, 2 x 2048) and 13B (40, 1 x 2048); encoder lengths, shared heads and
short ragged batches are generic.
"""
from __future__ import annotations

import math
import random
import struct

import torch

own = False

EPS = 9.999999974752427e-07  # 1e-6 in fp32
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# frequencies for contexts beyond the trained one: by base, by length, or each
# by the turns that it makes in the trained length
SCALINGS = {"none": (1.0, 2048), "linear": (4.0, 2048), "base": (8.0, 2048), "parts": (16.0, 8192)}


def listed():
    return [
        # one token of four sequences far into a scaled context, 13B heads: the smallest call
        dict(name="rope_token", op="rope", dir="fwd", dtype="bf16", N=4, T=0, Hq=40, Hk=40, Hv=40, dh=128, rot=128,
             layout="half", scaling="parts"),
        # queries and keys of XL's batch, half of each head turned, neighbours paired
        dict(name="rope_xl", op="rope", dir="fwd", dtype="bf16", N=8192, T=2048, Hq=16, Hk=16, Hv=16, dh=128, rot=64,
             layout="pairs", scaling="none"),
        # the tiny fp32 decoder's batch
        dict(name="norm_tiny", op="norm", dir="fwd", dtype="f32", N=256, T=128, Hq=4, Hk=4, Hv=4, dh=64, rot=64,
             layout="half", scaling="none"),
        # the fused QKV rows of a 6.7B block
        dict(name="norm_6.7b", op="norm", dir="fwd", dtype="bf16", N=4096, T=2048, Hq=32, Hk=32, Hv=32, dh=128,
             rot=128, layout="half", scaling="none"),
        # fine-tuning on three ragged sequences of 333 tokens, sixteen query heads on four of keys
        dict(name="norm_grad_short", op="norm", dir="bwd", dtype="bf16", N=999, T=333, Hq=16, Hk=4, Hv=4, dh=128,
             rot=96, layout="pairs", scaling="linear"),
        # gradients at 13B
        dict(name="norm_grad_13b", op="norm", dir="bwd", dtype="bf16", N=2048, T=2048, Hq=40, Hk=40, Hv=40, dh=128,
             rot=128, layout="half", scaling="none"),
        # decoding: one token of eight sequences against 2048 encoder states at most
        dict(name="cross_token", op="cross", dir="fwd", dtype="bf16", B=8, Tq=1, Tk=2048, Hq=40, Hk=40, dh=128,
             rows="padded"),
        # Small's batch on short encoder states, padded
        dict(name="cross_small", op="cross", dir="fwd", dtype="bf16", B=8, Tq=2048, Tk=500, Hq=12, Hk=12, dh=64,
             rows="padded"),
        # 6.7B's batch on encoder states twice as long
        dict(name="cross_6.7b", op="cross", dir="fwd", dtype="bf16", B=2, Tq=2048, Tk=4096, Hq=32, Hk=32, dh=128,
             rows="full"),
        # gradients of the tiny fp32 decoder
        dict(name="cross_grad_tiny", op="cross", dir="bwd", dtype="f32", B=2, Tq=128, Tk=100, Hq=4, Hk=4, dh=64,
             rows="full"),
        # fine-tuning on three ragged sequences, packed, shared key heads
        dict(name="cross_grad_short", op="cross", dir="bwd", dtype="bf16", B=3, Tq=333, Tk=200, Hq=16, Hk=4, dh=128,
             rows="packed"),
        # gradients of 6.7B's batch
        dict(name="cross_grad_6.7b", op="cross", dir="bwd", dtype="bf16", B=2, Tq=2048, Tk=1500, Hq=32, Hk=32, dh=128,
             rows="full"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "norm", "norm", "cross", "cross", "cross"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    way = rng.choice(["fwd", "bwd"])
    group = rng.choice([1, 1, 2, 3, 4, 8])
    if op == "cross":
        dh = rng.choice([64, 128])
        Hk = rng.randint(1, 40 // group)
        # the work of the largest listed case, an eighth of it in fp32
        most = 2 * 2048 * 4096 * 32 * 128 // (group * Hk * dh) // (1 if dtype == "bf16" else 8) // (1 if way == "fwd" else 3)
        Tq = _log(rng, 1, min(4096, most))
        Tk = _log(rng, 1, min(8192, max(1, most // Tq)))
        rows = (group * Tq + Tk) * Hk * dh * (2 if dtype == "bf16" else 4) * (2 if way == "fwd" else 4)
        B = rng.randint(1, max(1, min(32, most // (Tq * Tk), 230_000_000 // rows)))
        return dict(op=op, dir=way, dtype=dtype, B=B, Tq=Tq, Tk=Tk, Hq=group * Hk, Hk=Hk, dh=dh,
                    rows=rng.choice(["full", "padded", "packed"]))
    dh = rng.choice([64, 128, 2 * rng.randint(8, 128)])
    rot = rng.choice([dh, 2 * rng.randint(1, dh // 2)])
    Hk = rng.randint(1, 40 // group)
    Hv = rng.choice([0, Hk])
    # the bytes of the largest listed case of each
    most = (8192 * 32 * 128 if op == "rope" else (4096 if way == "fwd" else 2730) * 96 * 128) // ((group + 2) * Hk * dh) // (1 if dtype == "bf16" else 2)
    N = _log(rng, 1, max(2, min(16384, most)))
    return dict(op=op, dir=way, dtype=dtype, N=N, T=rng.choice([0, rng.randint(1, N)]), Hq=group * Hk, Hk=Hk, Hv=Hv, dh=dh,
                rot=rot, layout=rng.choice(["half", "pairs"]), scaling=rng.choice(list(SCALINGS)))


# ------------------------------------------------------------------ inputs
def _frequencies(rot, scaling):
    """Radians per position of each pair, and the factor of the turned elements (in fp32)."""
    factor, trained = SCALINGS[scaling]
    base = 10000.0 * (factor ** (rot / (rot - 2)) if scaling == "base" and rot > 2 else 1.0)
    freq = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        freq = [f / factor for f in freq]
    if scaling == "parts":
        keep = [min(1.0, max(0.0, (trained * f / (2 * math.pi) - 1.0) / 31.0)) for f in freq]
        freq = [f * (k + (1.0 - k) / factor) for f, k in zip(freq, keep)]
    mscale = 1.0 + 0.1 * math.log(factor) if scaling == "parts" else 1.0
    return freq, struct.unpack("f", struct.pack("f", mscale))[0]


def _lengths(case, what):
    """Lengths of the sequences, from the case alone: one is whole, others may have no keys at all."""
    B, T = case["B"], case["T" + what]
    if case["rows"] == "full" or (case["rows"] == "padded" and what == "q"):
        return [T] * B
    r = random.Random(B * 8209 + T)
    return [T] + [r.randint(1 if what == "q" else 0, T) for _ in range(B - 1)]


def _starts(case, what, lens):
    """First row of each sequence, and the number of rows."""
    if case["rows"] != "packed":
        return [b * case["T" + what] for b in range(case["B"])], case["B"] * case["T" + what]
    starts = [sum(lens[:b]) for b in range(len(lens))]
    return starts, sum(lens)


def _i32(v):
    return torch.tensor(v, device="cuda", dtype=torch.int32)


def _inputs(case, seed):
    """The tensors an operator reads, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _TYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    if case["op"] == "cross":
        # normalised queries and keys, gradients of a mean over tokens
        ql, kl = _lengths(case, "q"), _lengths(case, "k")
        (qs, nq), (ks, nk) = _starts(case, "q", ql), _starts(case, "k", kl)
        Hq, Hk, dh = case["Hq"], case["Hk"], case["dh"]
        st = dict(q=(1.5 * randn(nq, Hq * dh)).to(dt), k=randn(nk, Hk * dh).to(dt), v=randn(nk, Hk * dh).to(dt),
                  q_start=_i32(qs), q_len=_i32(ql), k_start=_i32(ks), k_len=_i32(kl))
        if case["dir"] == "bwd":
            st.update(dout=(1e-3 * randn(nq, Hq * dh)).to(dt))
        return st
    # rows of a fused QKV product: channels of unlike sizes, and gains around one
    N, Hq, Hk, Hv, dh, rot = (case[k] for k in ("N", "Hq", "Hk", "Hv", "dh", "rot"))
    width = (Hq + Hk + Hv) * dh
    freq, _ = _frequencies(rot, case["scaling"])
    st = dict(x=(randn(N, width) * torch.exp(0.5 * randn(width))).to(dt),
              freq=torch.tensor(freq, device="cuda", dtype=torch.float64), pos=None)
    if case["T"] == 0:  # positions of single tokens, up to the scaled context's end
        most = int(SCALINGS[case["scaling"]][0] * SCALINGS[case["scaling"]][1])
        st.update(pos=torch.randint(0, most, (N,), device="cuda", generator=g, dtype=torch.int32))
    if case["op"] == "norm":
        st.update(gq=(1.0 + 0.2 * randn(dh)).to(dt), gk=(1.0 + 0.2 * randn(dh)).to(dt))
    if case["dir"] == "bwd":
        st.update(dy=(1e-3 * randn(N, width)).to(dt))
    return st


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    dt = _TYPES[case["dtype"]]
    if case["op"] == "cross":
        dh = case["dh"]
        st.update(scale=struct.unpack("f", struct.pack("f", dh ** -0.5))[0])
        if case["dir"] == "bwd":  # what the forward call left
            fwd = _plain_cross_fwd(st)
            st.update(fwd, dq=torch.empty_like(st["q"]), dk=torch.empty_like(st["k"]), dv=torch.empty_like(st["v"]))
        else:
            st.update(o=torch.empty_like(st["q"]), lse=torch.empty(st["q"].shape[0], case["Hq"], device="cuda"))
    else:
        heads = case["Hq"] + case["Hk"] + (case["Hv"] if case["op"] == "norm" else 0)
        st.update(mscale=_frequencies(case["rot"], case["scaling"])[1],
                  y=torch.empty(case["N"], heads * case["dh"], device="cuda", dtype=dt))
        if case["op"] == "norm" and case["dir"] == "bwd":
            st.update(dgq=torch.empty(case["dh"], device="cuda"), dgk=torch.empty(case["dh"], device="cuda"))
    if own:
        from paper_2403_10504_amd import atom as A

        st.update(A=A, dt=A.ATOM_BF16 if case["dtype"] == "bf16" else A.ATOM_F32)
        n = 0
        if case["op"] == "cross":
            ptr = {k: st[k].data_ptr() for k in ("q_start", "q_len", "k_start", "k_len")}
            if case["rows"] != "packed":
                ptr.update(q_start=None, k_start=None, q_len=None)
            if case["rows"] == "full":
                ptr.update(k_len=None)
            st.update(shape=A.atom_cross_shape(case["B"], case["Tq"], case["Tk"], case["Hq"], case["Hk"], case["dh"],
                                               st["q"].shape[0], st["k"].shape[0], **ptr))
            ws = A.atom_k_cross_attn_fwd_ws_bytes if case["dir"] == "fwd" else A.atom_k_cross_attn_bwd_ws_bytes
            n = ws(st["dt"], st["shape"])
        elif case["op"] == "norm" and case["dir"] == "bwd":
            n = A.atom_k_qknorm_rope_bwd_ws_bytes(case["N"], case["Hq"], case["Hk"], case["dh"])
        st.update(ws=torch.empty(max(16, n), device="cuda", dtype=torch.uint8))
    return st


# ------------------------------------------------------------- plain forms
def _positions(st):
    c = st["case"]
    return st["pos"].double() if st["pos"] is not None else (torch.arange(c["N"], device="cuda") % c["T"]).double()


def _turn(st, x, back):
    """mscale R x, or its transpose, of x [N][heads][dh] in fp32."""
    c = st["case"]
    rot = c["rot"]
    angle = (_positions(st).unsqueeze(1) * st["freq"]).unsqueeze(1)  # in 64 bits: far positions
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    sin = -sin if back else sin
    if c["layout"] == "half":
        a, b = x[..., : rot // 2], x[..., rot // 2 : rot]
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    y = (a * cos - b * sin) * st["mscale"], (a * sin + b * cos) * st["mscale"]
    y = torch.cat(y, -1) if c["layout"] == "half" else torch.stack(y, -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rope(st):
    c = st["case"]
    n = c["Hq"] + c["Hk"]
    x = st["x"] if c["dir"] == "fwd" else st["dy"]
    y = _turn(st, x.view(c["N"], -1, c["dh"])[:, :n].float(), c["dir"] == "bwd")
    return dict(y=y.reshape(c["N"], n * c["dh"]).to(x.dtype))


def _gains(st):
    """The gains of the query and key heads, [Hq + Hk][dh] in fp32."""
    c = st["case"]
    return torch.cat([st["gq"].float().expand(c["Hq"], -1), st["gk"].float().expand(c["Hk"], -1)])


def _plain_norm(st):
    c = st["case"]
    n, dt = c["Hq"] + c["Hk"], st["x"].dtype
    x = st["x"].view(c["N"], -1, c["dh"])
    h = x[:, :n].float()
    r = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    if c["dir"] == "fwd":
        y = _turn(st, h * r * _gains(st), False).to(dt)
        return dict(y=torch.cat([y, x[:, n:]], 1).reshape(c["N"], -1))
    dy = st["dy"].view(c["N"], -1, c["dh"])
    g = _turn(st, dy[:, :n].float(), True)
    xh = h * r
    gw = g * _gains(st)
    dx = (r * (gw - xh * (gw * xh).mean(-1, keepdim=True))).to(dt)
    dg = (g * xh).sum(0)
    return dict(dx=torch.cat([dx, dy[:, n:]], 1).reshape(c["N"], -1), dgq=dg[: c["Hq"]].sum(0), dgk=dg[c["Hq"]:].sum(0))


def _rows(start, length, T):
    """Row numbers [B][T] of padded sequences, and which of them hold one."""
    t = torch.arange(T, device="cuda")
    on = t < length.unsqueeze(1)
    return torch.where(on, start.long().unsqueeze(1) + t, 0), on


def _heads(x, rows, on, H, share):
    """[B][H * share][T][dh] in fp32 of the rows of x, zeros where there is none."""
    y = x.float()[rows] * on.unsqueeze(2)
    y = y.view(*rows.shape, H, -1).permute(0, 2, 1, 3)
    return y.repeat_interleave(share, 1).contiguous()


def _back(y, on):
    """The rows of [B][H][T][dh] that hold one, [rows][H * dh]."""
    return y.permute(0, 2, 1, 3).reshape(*on.shape, -1)[on]


def _plain_scores(st):
    c = st["case"]
    qr, qo = _rows(st["q_start"], st["q_len"], c["Tq"])
    kr, ko = _rows(st["k_start"], st["k_len"], c["Tk"])
    q = _heads(st["q"], qr, qo, c["Hq"], 1)
    k = _heads(st["k"], kr, ko, c["Hk"], c["Hq"] // c["Hk"])
    v = _heads(st["v"], kr, ko, c["Hk"], c["Hq"] // c["Hk"])
    z = torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"]
    return z.masked_fill_(~ko[:, None, None, :], -math.inf), q, k, v, (qr, qo), (kr, ko)


def _plain_cross_fwd(st):
    z, q, k, v, (qr, qo), _ = _plain_scores(st)
    m = z.max(-1, keepdim=True).values.clamp(min=-3e38)
    p = torch.exp(z - m)
    s = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(s > 0, s, 1.0)
    lse = (m + torch.log(s)).squeeze(-1).transpose(1, 2)
    return dict(o=_back(o, qo).to(st["q"].dtype), lse=lse[qo])


def _plain_cross_bwd(st):
    c, dt = st["case"], st["q"].dtype
    z, q, k, v, (qr, qo), (kr, ko) = _plain_scores(st)
    share = c["Hq"] // c["Hk"]
    do, o = (_heads(st[x], qr, qo, c["Hq"], 1) for x in ("dout", "o"))
    lse = torch.where(qo.unsqueeze(2), st["lse"][qr], math.inf).transpose(1, 2).unsqueeze(-1)
    p = torch.where(z > -math.inf, torch.exp(z - lse), 0.0)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = p * (torch.matmul(do, v.transpose(2, 3).contiguous()) - (do * o).sum(-1, keepdim=True)) * st["scale"]
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    dk, dv = (x.unflatten(1, (c["Hk"], share)).sum(2) for x in (dk, dv))
    if c["rows"] == "padded":  # rows behind a sequence's end: zero
        ko = torch.ones_like(ko)
    return dict(dq=_back(dq, qo).to(dt), dk=_back(dk, ko).to(dt), dv=_back(dv, ko).to(dt))


# --------------------------------------------------------- the framework's
def _own_rope(st, s):
    c, A = st["case"], st["A"]
    x = st["x"] if c["dir"] == "fwd" else st["dy"]
    A.atom_k_rope(st["dt"], x.data_ptr(), x.shape[1], st["y"].data_ptr(), st["y"].shape[1], _ptr(st["pos"]),
                  st["freq"].data_ptr(), st["mscale"], _layout(st), c["dir"] == "bwd", c["N"], c["T"], c["Hq"] + c["Hk"],
                  c["dh"], c["rot"], s)
    return dict(y=st["y"])


def _ptr(t):
    return None if t is None else t.data_ptr()


def _layout(st):
    return st["A"].ATOM_ROPE_HALF if st["case"]["layout"] == "half" else st["A"].ATOM_ROPE_PAIRS


def _own_norm(st, s):
    c, A, w = st["case"], st["A"], st["x"].shape[1]
    tail = (EPS, _ptr(st["pos"]), st["freq"].data_ptr(), st["mscale"], _layout(st), c["N"], c["T"], c["Hq"], c["Hk"],
            c["Hv"], c["dh"], c["rot"])
    if c["dir"] == "fwd":
        A.atom_k_qknorm_rope_fwd(st["dt"], st["x"].data_ptr(), w, st["y"].data_ptr(), w, st["gq"].data_ptr(),
                                 st["gk"].data_ptr(), *tail, s)
        return dict(y=st["y"])
    A.atom_k_qknorm_rope_bwd(st["dt"], st["dy"].data_ptr(), w, st["x"].data_ptr(), w, st["y"].data_ptr(), w,
                             st["gq"].data_ptr(), st["gk"].data_ptr(), st["dgq"].data_ptr(), st["dgk"].data_ptr(), *tail,
                             st["ws"].data_ptr(), st["ws"].numel(), s)
    return dict(dx=st["y"], dgq=st["dgq"], dgk=st["dgk"])


def _own_cross(st, s):
    A, lq, lk = st["A"], st["q"].shape[1], st["k"].shape[1]
    p = {k: st[k].data_ptr() for k in ("q", "k", "v", "o", "lse", "ws")}
    ins = (st["dt"], st["shape"], p["q"], lq, p["k"], lk, p["v"], lk, st["scale"], p["o"], lq)
    if st["case"]["dir"] == "fwd":
        A.atom_k_cross_attn_fwd(*ins, p["lse"], p["ws"], st["ws"].numel(), s)
        return dict(o=st["o"], lse=st["lse"])
    A.atom_k_cross_attn_bwd(*ins, st["dout"].data_ptr(), lq, p["lse"], st["dq"].data_ptr(), lq, st["dk"].data_ptr(), lk,
                            st["dv"].data_ptr(), lk, p["ws"], st["ws"].numel(), s)
    return dict(dq=st["dq"], dk=st["dk"], dv=st["dv"])


def run(state):
    op, way = state["case"]["op"], state["case"]["dir"]
    if own:
        s = torch.cuda.current_stream().cuda_stream
        return dict(rope=_own_rope, norm=_own_norm, cross=_own_cross)[op](state, s)
    if op == "cross":
        return (_plain_cross_fwd if way == "fwd" else _plain_cross_bwd)(state)
    return (_plain_rope if op == "rope" else _plain_norm)(state)


# --------------------------------------------------------------------- work
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    fwd = case["dir"] == "fwd"
    if case["op"] == "cross":
        ql, kl = _lengths(case, "q"), _lengths(case, "k")
        q, kv = sum(ql) * case["Hq"] * case["dh"], sum(kl) * case["Hk"] * case["dh"]
        pairs = sum(a * b for a, b in zip(ql, kl)) * case["Hq"] * case["dh"]
        # forward: q, k, v in, o and lse out, two products; backward: q, k, v, o, dout, lse in, three gradients out, five
        bytes_ = (2 * q + 2 * kv if fwd else 4 * q + 4 * kv) * e + 4 * sum(ql) * case["Hq"]
        return dict(bytes=bytes_, flops=(4 if fwd else 10) * pairs)
    turned = case["N"] * (case["Hq"] + case["Hk"]) * case["dh"]
    copied = case["N"] * case["Hv"] * case["dh"] if case["op"] == "norm" else 0
    at = 4 * case["N"] * (case["T"] == 0) + 4 * case["rot"]
    if case["op"] == "rope":
        return dict(bytes=2 * turned * e + at, flops=3 * turned)
    if fwd:
        return dict(bytes=2 * (turned + copied) * e + 2 * case["dh"] * e + at, flops=8 * turned)
    return dict(bytes=(3 * turned + 2 * copied) * e + 2 * case["dh"] * (e + 4) + at, flops=16 * turned)


# -------------------------------------------------------------------- exact
def _turns(case, inp):
    """cos + i sin of every row and pair, times mscale, in 64 bits."""
    p = inp["pos"] if inp["pos"] is not None else torch.arange(case["N"], device="cuda") % case["T"]
    angle = torch.outer(p.double(), inp["freq"])
    return torch.polar(torch.full_like(angle, _frequencies(case["rot"], case["scaling"])[1]), angle)


def _exact_turn(case, x, turns):
    """x [N][heads][dh] with its pairs as complex numbers, multiplied."""
    rot, half = case["rot"], case["layout"] == "half"
    y = x.clone()
    pairs = x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if half else x[..., :rot].unflatten(-1, (rot // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turns.unsqueeze(1))
    y[..., :rot] = (z.transpose(-1, -2) if half else z).flatten(-2)
    return y


def exact(case, seed):
    inp = _inputs(case, seed)
    if case["op"] == "cross":
        return _exact_cross(case, inp)
    N, dh, nq, n = case["N"], case["dh"], case["Hq"], case["Hq"] + case["Hk"]
    turns = _turns(case, inp)
    bwd = case["dir"] == "bwd"
    if case["op"] == "rope":
        x = inp["dy"] if bwd else inp["x"]
        y = _exact_turn(case, x[:, : n * dh].double().view(N, n, dh), turns.conj() if bwd else turns)
        return dict(y=y.reshape(N, -1))
    x = inp["x"].double().view(N, -1, dh).requires_grad_(bwd)
    gq, gk = (inp[k].double().requires_grad_(bwd) for k in ("gq", "gk"))
    size = torch.linalg.vector_norm(x[:, :n], dim=-1, keepdim=True) / math.sqrt(dh)
    u = x[:, :n] / torch.hypot(size, torch.full_like(size, math.sqrt(EPS)))
    u = torch.cat([u[:, :nq] * gq, u[:, nq:] * gk], 1)
    if not bwd:
        return dict(y=torch.cat([_exact_turn(case, u, turns), x[:, n:]], 1).reshape(N, -1))
    dy = inp["dy"].double().view(N, -1, dh)
    # the turn is linear: its gradient is the turn back, then u's by differentiation
    dx, dgq, dgk = torch.autograd.grad(u, (x, gq, gk), _exact_turn(case, dy[:, :n], turns.conj()))
    dx[:, n:] = dy[:, n:]
    return dict(dx=dx.reshape(N, -1), dgq=dgq, dgk=dgk)


def _exact_cross(case, inp):
    Hq, Hk, dh = case["Hq"], case["Hk"], case["dh"]
    bwd = case["dir"] == "bwd"
    scale = struct.unpack("f", struct.pack("f", dh ** -0.5))[0]
    q, k, v = (inp[x].double().unflatten(1, (-1, dh)) for x in ("q", "k", "v"))
    out = dict(dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v)) if bwd else dict(
        o=torch.zeros_like(q), lse=torch.full(q.shape[:2], -math.inf, device="cuda", dtype=torch.float64))
    seqs = zip(*(inp[x].tolist() for x in ("q_start", "q_len", "k_start", "k_len")))
    for q0, ql, k0, kl in seqs:
        for h in range(Hq if kl else 0):
            rows, keys, hk = slice(q0, q0 + ql), slice(k0, k0 + kl), h // (Hq // Hk)
            a, b, c = q[rows, h], k[keys, hk], v[keys, hk]
            z = scale * (a @ b.T)
            p = torch.softmax(z, 1)
            if not bwd:
                out["o"][rows, h] = p @ c
                out["lse"][rows, h] = torch.logsumexp(z, 1)
                continue
            g = inp["dout"].double().unflatten(1, (-1, dh))[rows, h]
            dp = g @ c.T
            ds = scale * p * (dp - (p * dp).sum(1, keepdim=True))
            out["dq"][rows, h] = ds @ b
            out["dk"][keys, hk] += ds.T @ a
            out["dv"][keys, hk] += p.T @ g
    return {name: (x.flatten(1) if name != "lse" else x) for name, x in out.items()}
