"""The work of two operators of a GPT training step's end: the loss of a linear
head without its logits (forward, and its gradients), and the orthogonalised
update of a weight matrix.

Operations (field "op"):
  loss   z = x W^T over a vocabulary of V, lse_n = log sum_v exp z_nv and
         loss_n = lse_n - z_n[t_n] per token; tokens whose target is -1 take
         no part (loss and lse 0)              (atom_k_linear_xent_fwd)
  grad   dz_nv = (exp(z_nv - lse_n) - [v = t_n]) s, 0 for tokens that take no
         part; dx = dz W, dW = dz^T x          (atom_k_linear_xent_bwd)
  ortho  X = G / (|G|_F + 1e-7); five times X <- a X + (b A + c A^2) X with
         A = X X^T; the result is X            (atom_k_orthogonalize)

Widths, vocabulary and token counts are those of the GPT configurations: tiny
(256, vocabulary 1024, 2 x 128 tokens, fp32), Small (768, 8 x 2048 tokens), XL
(2048), 6.7B (4096, 2 x 2048) and 13B (5120, 1 x 2048), vocabulary 50257; the
short ones stand for fine-tuning and scoring on a few ragged sequences.
"""
from __future__ import annotations

import math

import torch

own = False

NORM_EPS = 1e-7
COEF = (3.4445, -4.7750, 2.0315)  # the quintic's coefficients, every step
STEPS = 5
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # loss of the tiny fp32 decoder's batch: the smallest call, launches dominate
        dict(name="loss_tiny", op="loss", dtype="f32", N=256, d=256, V=1024, ignored=0.0),
        # scoring one token at XL width: the head's weights are read once
        dict(name="loss_token", op="loss", dtype="bf16", N=1, d=2048, V=50257, ignored=0.0),
        # evaluation loss of GPT-3 Small's batch: many tokens, narrow rows
        dict(name="loss_small", op="loss", dtype="bf16", N=16384, d=768, V=50257, ignored=0.0),
        # the same at 6.7B, some of the batch padding
        dict(name="loss_6.7b", op="loss", dtype="bf16", N=4096, d=4096, V=50257, ignored=0.1),
        # gradients of the tiny fp32 decoder's batch
        dict(name="grad_tiny", op="grad", dtype="f32", N=256, d=256, V=1024, ignored=0.1),
        # fine-tuning at XL width on three ragged sequences of 333 tokens, prompts masked
        dict(name="grad_short", op="grad", dtype="bf16", N=999, d=2048, V=50257, ignored=0.4),
        # gradients of 13B's batch
        dict(name="grad_13b", op="grad", dtype="bf16", N=2048, d=5120, V=50257, ignored=0.0),
        # update of one fp32 matrix of the tiny decoder (its QKV weights, taller than wide)
        dict(name="ortho_tiny", op="ortho", dtype="f32", batch=1, rows=768, cols=256),
        # update of the attention output weights of all twelve layers of GPT-3 Small
        dict(name="ortho_small", op="ortho", dtype="bf16", batch=12, rows=768, cols=768),
        # update of an XL block's first MLP weight, four times as tall as wide
        dict(name="ortho_xl", op="ortho", dtype="bf16", batch=1, rows=8192, cols=2048),
        # update of a 6.7B block's attention output weight from fp32 gradient sums
        dict(name="ortho_6.7b", op="ortho", dtype="f32", batch=1, rows=4096, cols=4096),
        # update of a 13B block's second MLP weight, the largest matrix
        dict(name="ortho_13b", op="ortho", dtype="bf16", batch=1, rows=5120, cols=20480),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["loss", "grad", "ortho"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "ortho":
        # any two lengths, odd ones among them; fp32 up to the 6.7B width
        hi = (5120, 20480) if dtype == "bf16" else (4096, 4096)
        short = _log(rng, 64, hi[0])
        long = max(short, min(hi[1], _log(rng, short, 5 * short)))
        batch = max(1, min(rng.choice([1, 1, 3, 12]), 5120 * 5120 // (short * long)))
        rows, cols = (short, long) if rng.random() < 0.5 else (long, short)
        return dict(op=op, dtype=dtype, batch=batch, rows=rows, cols=cols)
    # rows of x and W are whole 16-byte chunks, as the framework's products need
    d = 8 * _log(rng, 16, 640)
    V = _log(rng, 1000, 50257)
    most = 2048 * 5120 * 50257 // (d * V) // (1 if dtype == "bf16" else 8)
    N = _log(rng, 1, max(2, min(16384, most)))
    return dict(op=op, dtype=dtype, N=N, d=d, V=V, ignored=rng.choice([0.0, 0.1, 0.5]))


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    """The tensors an operator reads, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _TYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    if case["op"] == "ortho":
        # a gradient: a few strong directions over noise, and a small scale
        b, m, n = case["batch"], case["rows"], case["cols"]
        r = max(1, min(m, n) // 16)
        x = torch.empty(b, m, n, device="cuda", dtype=dt)
        for i in range(b):
            x[i] = (1e-4 * (randn(m, r) @ randn(r, n) + 2.0 * randn(m, n))).to(dt)
        return dict(g=x)
    # rows behind the final LayerNorm, and weights that spread the logits over
    # a few units, as a trained head's
    N, d, V = case["N"], case["d"], case["V"]
    x = randn(N, d).to(dt)
    w = (2.5 / math.sqrt(d) * randn(V, d)).to(dt)
    tgt = torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)
    tgt[torch.rand(N, device="cuda", generator=g) < case["ignored"]] = -1
    return dict(x=x, w=w, tgt=tgt)


def _row_chunks(case, budget=1 << 29):
    """Ranges of tokens whose logits hold about `budget` elements."""
    step = max(1, min(case["N"], budget // case["V"]))
    return [(r, min(case["N"], r + step)) for r in range(0, case["N"], step)]


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    dt = _TYPES[case["dtype"]]

    def empty(*shape, dtype=dt):
        return torch.empty(shape, device="cuda", dtype=dtype)

    if case["op"] == "ortho":
        st.update(out=torch.empty_like(st["g"]))
    else:
        N, d, V = case["N"], case["d"], case["V"]
        st.update(lse=empty(N, dtype=torch.float32))
        if case["op"] == "loss":
            st.update(loss=empty(N, dtype=torch.float32))
        else:
            # the forward's lse and the weight of a token in the mean
            for r0, r1 in _row_chunks(case):
                st["lse"][r0:r1] = _plain_lse(st["x"][r0:r1].float() @ st["w"].float().T)
            st["lse"][st["tgt"] < 0] = 0.0
            st.update(scale=1.0 / max(1, int((st["tgt"] >= 0).sum())), dx=empty(N, d), dw=empty(V, d))
    if own:
        from paper_2403_10504_amd import atom as A

        st.update(A=A, dt=A.ATOM_BF16 if case["dtype"] == "bf16" else A.ATOM_F32)
        if case["op"] == "ortho":
            n = A.atom_k_orthogonalize_ws_bytes(st["dt"], case["batch"], case["rows"], case["cols"])
        elif case["op"] == "loss":
            n = A.atom_k_linear_xent_fwd_ws_bytes(st["dt"], N, V, d)
        else:
            n = A.atom_k_linear_xent_bwd_ws_bytes(st["dt"], N, V, d)
        st.update(ws=torch.empty(n, device="cuda", dtype=torch.uint8))
    return st


# ------------------------------------------------------------- plain forms
def _plain_lse(z):
    m = z.max(1, keepdim=True).values
    return m.squeeze(1) + torch.log(torch.exp(z - m).sum(1))


def _plain_loss(st):
    t = st["tgt"].long()
    z = st["x"].float() @ st["w"].float().T
    lse = _plain_lse(z)
    loss = lse - z.gather(1, t.clamp(min=0).unsqueeze(1)).squeeze(1)
    return dict(loss=torch.where(t >= 0, loss, 0.0), lse=torch.where(t >= 0, lse, 0.0))


def _plain_grad(st):
    dt = st["x"].dtype
    x, w, t = st["x"].float(), st["w"].float(), st["tgt"].long()
    valid = t >= 0
    p = torch.exp(x @ w.T - st["lse"].unsqueeze(1))
    p.scatter_add_(1, t.clamp(min=0).unsqueeze(1), torch.full_like(st["lse"], -1.0).unsqueeze(1))
    p *= (valid * st["scale"]).unsqueeze(1)
    return dict(dx=(p @ w).to(dt), dw=(p.T @ x).to(dt))


def _newton_schulz(x):
    """x: [batch][rows][cols], rows <= cols."""
    a, b, c = COEF
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + NORM_EPS)
    for _ in range(STEPS):
        s = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * s + c * torch.matmul(s, s), x)
    return x


def _plain_ortho(st):
    g = st["g"].float()
    if g.shape[1] > g.shape[2]:
        return dict(out=_newton_schulz(g.transpose(1, 2).contiguous()).transpose(1, 2).contiguous().to(st["g"].dtype))
    return dict(out=_newton_schulz(g).to(st["g"].dtype))


# --------------------------------------------------------- the framework's
def _own_loss(st, s):
    c = st["case"]
    st["A"].atom_k_linear_xent_fwd(st["dt"], st["x"].data_ptr(), c["d"], st["w"].data_ptr(), c["d"],
                                   st["tgt"].data_ptr(), st["lse"].data_ptr(), st["loss"].data_ptr(), c["N"], c["V"],
                                   c["d"], st["ws"].data_ptr(), st["ws"].numel(), s)
    return dict(loss=st["loss"], lse=st["lse"])


def _own_grad(st, s):
    c, A = st["case"], st["A"]
    A.atom_k_linear_xent_bwd(st["dt"], st["x"].data_ptr(), c["d"], st["w"].data_ptr(), c["d"], st["tgt"].data_ptr(),
                             st["lse"].data_ptr(), None, st["scale"], st["dx"].data_ptr(), c["d"], st["dw"].data_ptr(),
                             c["d"], A.ATOM_EPI_STORE, c["N"], c["V"], c["d"], 0, st["ws"].data_ptr(),
                             st["ws"].numel(), s)
    return dict(dx=st["dx"], dw=st["dw"])


def _own_ortho(st, s):
    c, A = st["case"], st["A"]
    b, m, n = c["batch"], c["rows"], c["cols"]
    A.atom_k_orthogonalize(st["dt"], st["g"].data_ptr(), n, m * n, st["out"].data_ptr(), n, m * n, A.ATOM_EPI_STORE,
                           0.0, 1.0, b, m, n, [COEF] * STEPS, st["ws"].data_ptr(), st["ws"].numel(), s)
    return dict(out=st["out"])


def run(state):
    op = state["case"]["op"]
    if own:
        s = torch.cuda.current_stream().cuda_stream
        return dict(loss=_own_loss, grad=_own_grad, ortho=_own_ortho)[op](state, s)
    return dict(loss=_plain_loss, grad=_plain_grad, ortho=_plain_ortho)[op](state)


# --------------------------------------------------------------------- work
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "ortho":
        m, n = sorted((case["rows"], case["cols"]))
        # A = X X^T and A^2 are symmetric: half of each product; (b A + c A^2) X is a whole one
        return dict(bytes=case["batch"] * 2 * m * n * e, flops=case["batch"] * STEPS * (m * m * n + m ** 3 + 2 * m * m * n))
    N, d, V = case["N"], case["d"], case["V"]
    if case["op"] == "loss":
        return dict(bytes=(N * d + V * d) * e + 12 * N, flops=2 * N * d * V)
    # the logits are not kept, so the gradients take three products
    return dict(bytes=2 * (N * d + V * d) * e + 8 * N, flops=6 * N * d * V)


# -------------------------------------------------------------------- exact
def exact(case, seed):
    inp = _inputs(case, seed)
    if case["op"] == "ortho":
        out = torch.empty(inp["g"].shape, device="cuda", dtype=torch.float64)
        eye = None
        for i in range(case["batch"]):
            x = inp["g"][i].double()
            x = x / (torch.linalg.vector_norm(x) + NORM_EPS)
            # powers of the smaller Gram matrix, on the side it stands
            tall = x.shape[0] > x.shape[1]
            eye = torch.eye(min(x.shape), device="cuda", dtype=torch.float64) if eye is None else eye
            for _ in range(STEPS):
                s = x.T @ x if tall else x @ x.T
                p = COEF[0] * eye + s @ (COEF[1] * eye + COEF[2] * s)
                x = x @ p if tall else p @ x
            out[i] = x
        return dict(out=out)
    w, t = inp["w"].double(), inp["tgt"].long()
    N, d, V = case["N"], case["d"], case["V"]
    valid = t >= 0
    rows = torch.arange(N, device="cuda")
    if case["op"] == "loss":
        loss = torch.zeros(N, device="cuda", dtype=torch.float64)
        lse = torch.zeros_like(loss)
        for r0, r1 in _row_chunks(case, 1 << 28):
            z = inp["x"][r0:r1].double() @ w.T
            v = valid[r0:r1]
            lse[r0:r1] = torch.logsumexp(z, 1) * v
            loss[r0:r1] = (lse[r0:r1] - z[rows[: r1 - r0], t[r0:r1].clamp(min=0)]) * v
        return dict(loss=loss, lse=lse)
    scale = 1.0 / max(1, int(valid.sum()))
    dx = torch.zeros(N, d, device="cuda", dtype=torch.float64)
    dw = torch.zeros(V, d, device="cuda", dtype=torch.float64)
    for r0, r1 in _row_chunks(case, 1 << 28):
        x = inp["x"][r0:r1].double()
        dz = torch.softmax(x @ w.T, 1)
        dz[rows[: r1 - r0], t[r0:r1].clamp(min=0)] -= 1.0
        dz *= scale * valid[r0:r1].unsqueeze(1)
        dx[r0:r1] = dz @ w
        dw += dz.T @ x
    return dict(dx=dx, dw=dw)
