"""Measured operators of gated feed-forward blocks and of products in 8-bit integers.

A case is one of these kinds:
  "glu"      a gated block's first half, H = act(G) * U with [G | U] = P = X W^T + bias and W[2N x K]: forward ("fwd" as evaluated,
             "train" with P kept) or backward ("bwd": dX, dW, dbias from dH and the P that the forward call has kept);
  "gate"     the gate alone on a P that other layers (decomposed projections) have formed: H ("fwd"), or dP from dH ("bwd");
  "i8"       a served linear layer: the activations quantized to 8 bits a row, then their product with a quantized weight;
  "i8_glu"   the same of a gated block's first half.
X and dH ~ N(0, 1), weights scaled so that P stays at unit scale; the activations of the 8-bit layers have channels of unequal
size, as those of trained models have.
"""
from __future__ import annotations

import math

import torch

own = False          # False: the plain form in elementary torch operations; True: the calls of this package

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


def _glu(mode, M, K, N, dtype, act, bias=False):
    return {"kind": "glu", "mode": mode, "M": M, "K": K, "N": N, "dtype": dtype, "act": act, "bias": bias}


def _gate(mode, M, N, dtype, act):
    return {"kind": "gate", "mode": mode, "M": M, "N": N, "dtype": dtype, "act": act}


def _i8(kind, M, K, N, dtype, act="silu", bias=False):
    return {"kind": kind, "M": M, "K": K, "N": N, "dtype": dtype, "act": act, "bias": bias}


def listed():
    cases = [
        # one token through the gated block of a small model: all latency and weight traffic
        ("glu_token", _glu("fwd", 1, 1024, 2816, "bf16", "silu")),
        # a prompt of odd length through a block of odd width, with biases
        ("glu_prompt_odd", _glu("fwd", 333, 1024, 2731, "bf16", "gelu_tanh", True)),
        # training forward of a wide block on 8192 tokens, P kept for the backward pass
        ("glu_train_wide", _glu("train", 8192, 4096, 10752, "bf16", "silu")),
        # a small fp32 block
        ("glu_f32_small", _glu("train", 256, 512, 1376, "f32", "gelu", True)),
        # backward pass of a small model's block at 32 x 128 tokens
        ("glu_bwd", _glu("bwd", 4096, 1024, 2816, "bf16", "silu", True)),
        # backward pass of the wide block: the largest
        ("glu_bwd_wide", _glu("bwd", 8192, 4096, 10752, "bf16", "silu")),
        # the gate behind two decomposed projections, 8192 tokens
        ("gate", _gate("fwd", 8192, 4096, "bf16", "silu")),
        # its backward pass on a micro-batch of odd size and width
        ("gate_bwd_odd", _gate("bwd", 1021, 2731, "bf16", "gelu")),
        # one token through a served 4096 x 4096 layer
        ("i8_token", _i8("i8", 1, 4096, 4096, "bf16")),
        # the same layer on a long prompt
        ("i8_prompt", _i8("i8", 8192, 4096, 4096, "bf16")),
        # a decoding batch through the wide gated block
        ("i8_glu_batch", _i8("i8_glu", 16, 4096, 10752, "bf16")),
        # a small model's gated block on 4093 tokens, fp32 activations
        ("i8_glu_f32", _i8("i8_glu", 4093, 1024, 2816, "f32", "gelu_tanh", True)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width in the range: mostly a multiple of 8 to 256, at times as it falls."""
    n, m = _log(rng, lo, hi), rng.choice([1, 8, 64, 64, 128, 256])
    return max(m, n // m * m)


def draw(rng):
    top = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["glu", "glu", "glu", "gate", "i8", "i8", "i8_glu", "i8_glu"])
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        act, bias = rng.choice(list(ACTS)), rng.random() < 0.5
        M = _log(rng, 1, 8192)
        if kind == "gate":
            c = _gate(rng.choice(["fwd", "bwd"]), M, _width(rng, 256, 10752), dtype, act)
        elif kind == "glu":
            mode = rng.choice(["fwd", "train", "bwd"])
            if dtype == "f32":
                c = _glu(mode, _log(rng, 1, 1024), _width(rng, 64, 1024), _width(rng, 64, 2048), dtype, act, bias)
            else:
                c = _glu(mode, M, _width(rng, 256, 4096), _width(rng, 256, 10752), dtype, act, bias)
        else:
            c = _i8(kind, M, _width(rng, 256, 8192), _width(rng, 256, 10752), dtype, act, bias)
        if work(c)["flops"] <= top:
            return c


# ---- states -------------------------------------------------------------------------------------------------------
def _normal(g, tdt, *shape, std=1.0):
    return torch.randn(*shape, device="cuda", generator=g).mul_(std).to(tdt)


def _quantized(x):
    """Rows of x as 8-bit integers and their scales: s = max |x| / 127 (fp32), q = x / s rounded, ties to even.  The quotient is
    taken in 64 bits: it decides on which side of a border a value falls."""
    s = x.abs().amax(dim=1).float() / 127
    q = torch.where(s[:, None] > 0, torch.round(x.double() / s.double()[:, None]), torch.zeros((), dtype=torch.float64, device=x.device))
    return q.clamp_(-127, 127).to(torch.int8), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    tdt, M, N, kind = DTYPES[case["dtype"]], case["M"], case["N"], case["kind"]
    S = {"case": case}
    if kind == "gate":
        S["P"] = _normal(g, tdt, M, 2 * N)
        if case["mode"] == "bwd":
            S["dH"] = _normal(g, tdt, M, N)
    else:
        K = case["K"]
        rows = N if kind == "i8" else 2 * N
        S["X"] = _normal(g, tdt, M, K)
        W = _normal(g, tdt, rows, K, std=K ** -0.5)
        S["bias"] = _normal(g, tdt, rows, std=0.1) if case["bias"] else None
        if kind == "glu":
            S["W"] = W
            if case["mode"] == "bwd":
                S["dH"] = _normal(g, tdt, M, N)
                P = S["X"].float() @ W.float().T
                S["P"] = (P if S["bias"] is None else P + S["bias"].float()).to(tdt)
        else:
            S["X"] = (S["X"].float() * torch.randn(K, device="cuda", generator=g).mul_(0.5).exp_()).to(tdt)
            S["Wq"], S["ws"] = _quantized(W)
    if own:
        _own_buffers(S)
    return S


# ---- plain form ---------------------------------------------------------------------------------------------------
def _act(x, act):
    if act == "silu":
        return x / (1 + torch.exp(-x))
    if act == "gelu":
        return 0.5 * x * torch.erfc(x * -(0.5 ** 0.5))
    return x / (1 + torch.exp(-2 * (2 / math.pi) ** 0.5 * (x + 0.044715 * x * x * x)))


def _act_slope(x, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-x))
        return s * (1 + x * (1 - s))
    if act == "gelu":
        return 0.5 * torch.erfc(x * -(0.5 ** 0.5)) + x * torch.exp(-0.5 * x * x) * (2 * math.pi) ** -0.5
    c = (2 / math.pi) ** 0.5
    s = 1 / (1 + torch.exp(-2 * c * (x + 0.044715 * x * x * x)))
    return s + x * s * (1 - s) * (2 * c) * (1 + 3 * 0.044715 * x * x)


def _product(X, W, bias):
    P = X.float() @ W.float().T
    return P if bias is None else P + bias.float()


def _gate_plain(P, act):
    G, U = P.chunk(2, dim=1)
    return _act(G, act) * U


def _gate_bwd_plain(dH, P, act):
    G, U = P.chunk(2, dim=1)
    return torch.cat([dH * U * _act_slope(G, act), dH * _act(G, act)], dim=1)


def _run_plain(S):
    c = S["case"]
    tdt, act, kind = DTYPES[c["dtype"]], c["act"], c["kind"]
    if kind == "gate":
        P = S["P"].float()
        return [(_gate_plain(P, act) if c["mode"] == "fwd" else _gate_bwd_plain(S["dH"].float(), P, act)).to(tdt)]
    if kind == "glu" and c["mode"] != "bwd":
        P = _product(S["X"], S["W"], S["bias"])
        H = _gate_plain(P, act).to(tdt)
        return [H, P.to(tdt)] if c["mode"] == "train" else [H]
    if kind == "glu":
        dP = _gate_bwd_plain(S["dH"].float(), S["P"].float(), act)
        out = [dP @ S["W"].float(), dP.T @ S["X"].float()] + ([dP.sum(dim=0)] if c["bias"] else [])
        return [t.to(tdt) for t in out]
    q, s = _quantized(S["X"])
    P = (q.float() @ S["Wq"].float().T) * s[:, None] * S["ws"]
    P = P if S["bias"] is None else P + S["bias"].float()
    return [(P if kind == "i8" else _gate_plain(P, act)).to(tdt)]


# ---- the calls of the package -------------------------------------------------------------------------------------
def _empty(tdt, *shape):
    return torch.empty(*shape, dtype=tdt, device="cuda")


def _own_buffers(S):
    """Descriptor, outputs and workspace, as a user's program keeps them."""
    from paper_2309_03824_b200 import binding as b
    c = S["case"]
    tdt, code, act = DTYPES[c["dtype"]], {"bf16": b.LRD_BF16, "f32": b.LRD_F32}[c["dtype"]], ACTS[c["act"]]
    M, N, kind = c["M"], c["N"], c["kind"]
    S["b"] = b
    if kind == "gate":
        S["desc"] = b.glu_desc(M, 0, N, code, act)
        S["out"] = _empty(tdt, M, N if c["mode"] == "fwd" else 2 * N)
        return
    K = c["K"]
    if kind == "glu":
        S["desc"] = b.glu_desc(M, K, N, code, act)
        nbytes = b.lrd_glu_workspace_bytes(S["desc"], c["mode"] == "bwd")
        if c["mode"] == "bwd":
            S["dX"], S["dW"], S["db"] = _empty(tdt, M, K), _empty(tdt, 2 * N, K), _empty(tdt, 2 * N) if c["bias"] else None
        else:
            S["H"], S["P"] = _empty(tdt, M, N), _empty(tdt, M, 2 * N) if c["mode"] == "train" else None
    else:
        # rows of the 8-bit operands start at multiples of 16 bytes
        ld = (K + 15) // 16 * 16
        S["desc"] = b.i8_desc(M, K, N, code, act, ldx=ld, ldw=ld)
        nbytes = b.lrd_i8_workspace_bytes(S["desc"], kind == "i8_glu")
        Wq = torch.zeros(S["Wq"].shape[0], ld, dtype=torch.int8, device="cuda")
        Wq[:, :K] = S["Wq"]
        S["Wq"] = Wq
        S["Xq"], S["xs"], S["Y"] = _empty(torch.int8, M, ld), _empty(torch.float32, M), _empty(tdt, M, N)
    S["work"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda")


def _run_own(S):
    c, b = S["case"], S["b"]
    kind = c["kind"]
    if kind == "gate":
        if c["mode"] == "fwd":
            b.lrd_gate_fwd(S["desc"], S["P"], S["out"])
        else:
            b.lrd_gate_bwd(S["desc"], S["dH"], S["P"], S["out"])
        return [S["out"]]
    if kind == "glu" and c["mode"] != "bwd":
        b.lrd_dense_glu_fwd(S["desc"], S["X"], S["W"], S["bias"], S["H"], S["P"], S["work"])
        return [S["H"], S["P"]] if c["mode"] == "train" else [S["H"]]
    if kind == "glu":
        b.lrd_dense_glu_bwd(S["desc"], S["dH"], S["X"], S["W"], S["P"], S["dX"], S["dW"], S["db"], S["work"])
        return [S["dX"], S["dW"]] + ([S["db"]] if c["bias"] else [])
    b.lrd_i8_quantize(S["X"], 0, c["M"], c["K"], S["Xq"], S["Xq"].shape[1], S["xs"], S["desc"].dtype)
    call = b.lrd_i8_dense_fwd if kind == "i8" else b.lrd_i8_glu_fwd
    call(S["desc"], S["Xq"], S["xs"], S["Wq"], S["ws"], S["bias"], S["Y"], S["work"])
    return [S["Y"]]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- work and exact values ----------------------------------------------------------------------------------------
def work(case):
    M, N, e, kind = case["M"], case["N"], 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind == "gate":
        return {"bytes": e * M * N * (3 if case["mode"] == "fwd" else 5), "flops": 10 * M * N}
    K = case["K"]
    rows = N if kind == "i8" else 2 * N
    nb = rows if case["bias"] else 0
    if kind != "glu":
        return {"bytes": e * (M * K + M * N + nb) + rows * (K + 4), "flops": 2 * M * rows * K}
    if case["mode"] == "bwd":
        return {"bytes": e * (3 * M * N + 2 * (M * K + 2 * N * K) + nb), "flops": 8 * M * N * K}
    return {"bytes": e * (M * K + 2 * N * K + nb + M * N * (3 if case["mode"] == "train" else 1)), "flops": 4 * M * N * K}


def exact(case, seed):
    S = prepare(case, seed)
    d = {k: v.double() for k, v in S.items() if isinstance(v, torch.Tensor) and k not in ("Wq", "work")}
    kind, name, N = case["kind"], case["act"], case["N"]

    def phi(x):              # the activation and its derivative
        if name == "gelu":
            cdf = torch.special.ndtr(x)
            return x * cdf, cdf + x * torch.exp(-x ** 2 / 2) / math.sqrt(2 * math.pi)
        if name == "silu":
            t = torch.sigmoid(x)
            return x * t, t + x * t * torch.sigmoid(-x)
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (x + 0.044715 * x ** 3))
        return x / 2 * (1 + t), (1 + t) / 2 + x / 2 * (1 - t ** 2) * a * (1 + 0.134145 * x ** 2)

    if kind in ("gate", "glu") and case["mode"] == "bwd":
        G, U = d["P"][:, :N], d["P"][:, N:]
        f, slope = phi(G)
        dP = torch.hstack([d["dH"] * U * slope, d["dH"] * f])
        if kind == "gate":
            return [dP]
        return [torch.matmul(dP, d["W"]), torch.matmul(dP.t(), d["X"])] + ([dP.sum(0)] if case["bias"] else [])
    if kind == "gate":
        return [phi(d["P"][:, :N])[0] * d["P"][:, N:]]
    if kind == "glu":
        P = torch.matmul(d["X"], d["W"].t())
    else:
        scale = (d["X"].abs().max(dim=1, keepdim=True).values / 127).float().double()
        whole = torch.round(d["X"] / scale)
        P = torch.matmul(whole * scale, (S["Wq"][:, : case["K"]].double() * d["ws"][:, None]).t())
    if case["bias"]:
        P = P + d["bias"]
    if kind == "i8":
        return [P]
    H = phi(P[:, :N])[0] * P[:, N:]
    return [H, P] if kind == "glu" and case["mode"] == "train" else [H]
