"""Gated feed-forward block and gate against the fp64 oracle, through the C ABI.

Tolerances, element by element.  A rounding to the storage type is off by at most half a step (2^-8 of the value in bf16, 2^-24 in
fp32).  A sum of n products formed in fp32 is off by at most n 2^-23 times the sum of their magnitudes, whatever its order (the
tensor cores may cut where they round: a whole last place).  The activations: a few last places of fp32 (`ACT`), with the
bf16 results' fast exponential and divide some 2^-19; relative to |x| (the value) or 1 + |x| (the derivative), not to the result,
which passes through zero."""
import numpy as np
import pytest
import torch

from oracle import lrd_oracle as o
from paper_2309_03824_b200 import binding as b
from paper_2309_03824_b200 import workloads as wl

from helpers import DT, dev, host, workspace

pytestmark = pytest.mark.gpu
ACTS = [b.LRD_ACT_SILU, b.LRD_ACT_GELU, b.LRD_ACT_GELU_TANH]
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
ACT = {"bf16": 2.0 ** -18, "f32": 2.0 ** -20}
NAN = float("nan")


def make(M, K, N, dtype, seed, bias=True):
    c = {"M": M, "K": K, "N": N, "dtype": dtype, "X": wl.round_to(wl.normal(seed, (M, K)), dtype),
         "W": wl.round_to(wl.normal(seed + 1, (2 * N, K), K ** -0.5), dtype), "dH": wl.round_to(wl.normal(seed + 2, (M, N)), dtype)}
    c["b"] = wl.round_to(wl.normal(seed + 3, (2 * N,), 0.5), dtype) if bias else None
    return c


def padded(a, ld, dtype, fill=NAN, shift=0):
    """a on the device in rows of ld elements, the rest filled; `shift` elements past a 256-byte boundary."""
    rows, cols = a.shape
    t = torch.full((rows * ld + shift,), fill, dtype=DT[dtype][1], device="cuda")[shift:].view(rows, ld)
    t[:, :cols] = dev(a, dtype)
    return t


def fwd_tolerance(c, P, act):
    """(of H, of P): the projections' sums, then the gate on them, then the rounding."""
    X, W, N = np.abs(c["X"].astype(np.float64)), np.abs(c["W"].astype(np.float64)), c["N"]
    mag = X @ W.T + (0.0 if c["b"] is None else np.abs(c["b"].astype(np.float64)))
    off = (c["K"] + 2) * 2.0 ** -23 * mag
    G, U = P[:, :N], P[:, N:]
    value = np.abs(o.activation(G, act)[0])
    h = np.abs(G) * ACT[c["dtype"]] * np.abs(U) + 1.2 * off[:, :N] * (np.abs(U) + off[:, N:]) + value * off[:, N:]
    return h + HALF[c["dtype"]] * (np.abs(value * U) + h), off + HALF[c["dtype"]] * (np.abs(P) + off)


def gate_bwd_tolerance(dH, P, dtype):
    N = dH.shape[1]
    d, g, u = np.abs(dH), np.abs(P[:, :N]), np.abs(P[:, N:])
    return np.concatenate([d * u * (1 + g) * ACT[dtype], d * g * ACT[dtype]], axis=1)


def bwd_tolerance(c, ref, P):
    h, dt = HALF[c["dtype"]], c["dtype"]
    off = gate_bwd_tolerance(c["dH"].astype(np.float64), P, dt)
    off = off + h * (np.abs(ref["dP"]) + off)                # dP is rounded once
    mag = np.abs(ref["dP"]) + off
    W, X = np.abs(c["W"].astype(np.float64)), np.abs(c["X"].astype(np.float64))
    sums = {"dX": off @ W + (2 * c["N"] + 2) * 2.0 ** -23 * (mag @ W), "dW": off.T @ X + (c["M"] + 2) * 2.0 ** -23 * (mag.T @ X),
            "db": off.sum(axis=0) + (c["M"] + 2) * 2.0 ** -23 * mag.sum(axis=0)}
    return {k: v + h * (np.abs(ref[k]) + v) for k, v in sums.items()}


def close(got, want, tol, name):
    err = np.abs(host(got) - want)
    bad = ~(err <= tol)
    assert not bad.any(), (name, int(bad.sum()), err.max(), np.argwhere(bad)[:4].tolist())


def run_fwd(c, act, save=True, lds=None, shift=0, stream=None):
    """lds: leading dimensions (ldx, ldw, ldh, ldp); 0 = packed."""
    M, K, N, dt = c["M"], c["K"], c["N"], c["dtype"]
    ldx, ldw, ldh, ldp = lds or (0, 0, 0, 0)
    desc = b.glu_desc(M, K, N, DT[dt][0], act, ldx, ldw, ldh, ldp)
    X, W = padded(c["X"], ldx or K, dt, shift=shift), padded(c["W"], ldw or K, dt, shift=shift)
    H = padded(np.zeros((M, 0), np.float32), ldh or N, dt, 3.0, shift)
    P = padded(np.zeros((M, 0), np.float32), ldp or 2 * N, dt, 3.0, shift) if save else None
    need = b.lrd_glu_workspace_bytes(desc, 0)
    ws = workspace(need + 256)
    ws.fill_(0x5A)
    b.lrd_dense_glu_fwd(desc, X, W, dev(c["b"], dt), H, P, ws[:max(need, 256)], stream=stream)
    torch.cuda.synchronize()
    assert b.lrd_check_device_status() == b.LRD_OK
    assert (ws[need:] == 0x5A).all()
    for t, cols in ((H, N), (P, 2 * N)):                     # nothing written between the rows
        assert t is None or (t[:, cols:] == 3.0).all()
    return H[:, :N], None if P is None else P[:, :2 * N]


def check_fwd(c, act, **kw):
    Hr, Pr = o.glu_fwd(c["X"], c["W"], c["b"], act)
    H, P = run_fwd(c, act, **kw)
    th, tp = fwd_tolerance(c, Pr, act)
    close(H, Hr, th, "H")
    if P is not None:
        close(P, Pr, tp, "P")
    return H, P


def run_bwd(c, act, P, want_dx=True, want_db=True, lds=None, shift=0):
    M, K, N, dt = c["M"], c["K"], c["N"], c["dtype"]
    ldx, ldw, ldh, ldp = lds or (0, 0, 0, 0)
    desc = b.glu_desc(M, K, N, DT[dt][0], act, ldx, ldw, ldh, ldp)
    X, W, dH = padded(c["X"], ldx or K, dt, shift=shift), padded(c["W"], ldw or K, dt, shift=shift), padded(c["dH"], ldh or N, dt, shift=shift)
    Pd = padded(P, ldp or 2 * N, dt, shift=shift)
    none = lambda rows: np.zeros((rows, 0), np.float32)
    dX = padded(none(M), ldx or K, dt, 3.0, shift) if want_dx else None
    dW = padded(none(2 * N), ldw or K, dt, 3.0, shift)
    db = torch.full((2 * N,), NAN, dtype=DT[dt][1], device="cuda") if want_db else None
    need = b.lrd_glu_workspace_bytes(desc, 1)
    ws = workspace(need + 256)
    ws.fill_(0x5A)
    b.lrd_dense_glu_bwd(desc, dH, X, W, Pd, dX, dW, db, ws[:need])
    torch.cuda.synchronize()
    assert b.lrd_check_device_status() == b.LRD_OK
    assert (ws[need:] == 0x5A).all()
    for t in (dX, dW):
        assert t is None or (t[:, K:] == 3.0).all()
    return {"dX": None if dX is None else dX[:, :K], "dW": dW[:, :K], "db": db}


def check_bwd(c, act, **kw):
    P = wl.round_to(o.glu_fwd(c["X"], c["W"], c["b"], act)[1], c["dtype"])
    got = run_bwd(c, act, P, **kw)
    P = P.astype(np.float64)
    ref = o.glu_bwd(c["dH"], c["X"], c["W"], P, act)
    tol = bwd_tolerance(c, ref, P)
    for k, t in got.items():
        if t is not None:
            close(t, ref[k], tol[k], k)
    return got


SIZES = [(1, 64, 32), (1, 8, 8), (2, 1024, 264), (17, 200, 40), (32, 520, 1000), (33, 72, 40), (128, 64, 64), (129, 200, 136), (257, 64, 1000),
         (300, 520, 264), (1000, 1032, 520), (520, 136, 1288)]
ODD_SIZES = [(1, 1, 1), (3, 5, 2), (4, 17, 5), (31, 33, 7), (130, 65, 129), (77, 100, 51), (300, 1001, 333), (5, 64, 33), (200, 64, 173)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", SIZES + ODD_SIZES)
def test_forward(size, act):
    c = make(*size, "bf16", 500 + size[0], bias=size[0] % 2 == 1)
    H, _ = check_fwd(c, act)
    same, _ = check_fwd(c, act, save=False)
    assert torch.equal(H, same)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", SIZES + ODD_SIZES)
def test_backward(size, act):
    c = make(*size, "bf16", 600 + size[0])
    first = check_bwd(c, act)
    again = check_bwd(c, act)
    assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 300, 70), (3, 5, 2), (64, 64, 32), (65, 33, 33), (130, 129, 97), (256, 512, 172)])
def test_general_path(size, dtype):
    c = make(*size, dtype, 700 + size[0], bias=size[0] != 64)
    b.lrd_set_path(b.LRD_PATH_GENERAL)
    try:
        for act in ACTS:
            check_fwd(c, act)
            check_fwd(c, act, save=False)
            check_bwd(c, act)
    finally:
        b.lrd_set_path(b.LRD_PATH_AUTO)


@pytest.mark.parametrize("columns,blocks", [(32, 1), (64, 1), (128, 1), (256, 1), (128, 2), (256, 2)])
@pytest.mark.parametrize("size", [(1, 64, 16), (9, 264, 333), (32, 1096, 200), (33, 64, 200), (128, 72, 264), (129, 520, 129), (700, 136, 640), (513, 1032, 1000)])
def test_every_tile_shape(size, columns, blocks):
    M = size[0]
    c = make(*size, "bf16", 800 + M)
    b.lrd_glu_tuning(columns, blocks)
    try:
        if (columns == 32 and M > 128) or (blocks == 2 and M <= 128):
            d = b.glu_desc(*size, b.LRD_BF16)
            t = torch.zeros(1 << 20, dtype=torch.bfloat16, device="cuda")
            assert b.lrd_dense_glu_fwd(d, t, t, None, t, None, None, check=False) == b.LRD_ERR_UNSUPPORTED
            return
        for act in ACTS[:1] if M > 500 else ACTS:
            check_fwd(c, act)
    finally:
        b.lrd_glu_tuning()


# padded rows of even and odd length; every operand off a 16-byte boundary (then the general kernels take it)
@pytest.mark.parametrize("lds,shift", [((88, 96, 72, 160), 0), ((83, 96, 67, 131), 0), ((88, 81, 65, 133), 0), ((81, 83, 65, 129), 0), ((0, 0, 0, 0), 1), ((88, 96, 72, 160), 3),
                                       ((83, 0, 0, 0), 5)])
@pytest.mark.parametrize("M", [5, 150])
def test_strides_and_odd_bases(M, lds, shift):
    c = make(M, 80, 64, "bf16", 900 + M)
    check_fwd(c, b.LRD_ACT_SILU, lds=lds, shift=shift)
    check_bwd(c, b.LRD_ACT_SILU, lds=lds, shift=shift)
    f = make(M, 80, 64, "f32", 900 + M)
    check_fwd(f, b.LRD_ACT_GELU, lds=lds, shift=shift)
    check_bwd(f, b.LRD_ACT_GELU, lds=lds, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_that_are_not_wanted(dtype):
    c = make(140, 72, 48, dtype, 950)
    full = check_bwd(c, b.LRD_ACT_GELU_TANH)
    part = check_bwd(c, b.LRD_ACT_GELU_TANH, want_dx=False, want_db=False)
    assert torch.equal(full["dW"], part["dW"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens(dtype):
    d = b.glu_desc(0, 24, 8, DT[dtype][0])
    t = torch.full((16, 24), 3.0, dtype=DT[dtype][1], device="cuda")
    dW, db = t.clone(), t.reshape(-1)[:16].clone()
    ws = workspace(b.lrd_glu_workspace_bytes(d, 1))
    b.lrd_dense_glu_fwd(d, t, t, None, t, t, None)
    b.lrd_gate_fwd(d, t, t)
    b.lrd_gate_bwd(d, t, t, t)
    b.lrd_dense_glu_bwd(d, t, t, t, t, t, dW, db, ws)
    torch.cuda.synchronize()
    assert (t == 3.0).all() and not dW.any() and not db.any()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1), (1, 8), (3, 5), (70, 64), (257, 1000), (40, 333), (1000, 7)])
def test_gate(size, dtype, act):
    M, N = size
    for ldp, ldh, shift in ((2 * N, N, 0), (2 * N + 8, N + 8, 0), (2 * N + 3, N + 1, 0), (2 * N, N, 1)):
        P, dH = (wl.round_to(wl.normal(1000 + M + i, (M, (2 - i) * N), 2.0), dtype) for i in (0, 1))
        d = b.glu_desc(M, 0, N, DT[dtype][0], act, ldh=ldh, ldp=ldp)
        Pd, dHd = padded(P, ldp, dtype, shift=shift), padded(dH, ldh, dtype, shift=shift)
        H, dP = padded(P[:, :0], ldh, dtype, 3.0, shift), padded(P[:, :0], ldp, dtype, 3.0, shift)
        b.lrd_gate_fwd(d, Pd, H)
        b.lrd_gate_bwd(d, dHd, Pd, dP)
        P, dH = P.astype(np.float64), dH.astype(np.float64)
        Hr, dPr = o.gate_fwd(P, act), o.gate_bwd(dH, P, act)
        th = np.abs(P[:, :N] * P[:, N:]) * ACT[dtype]
        td = gate_bwd_tolerance(dH, P, dtype)
        close(H[:, :N], Hr, th + HALF[dtype] * (np.abs(Hr) + th), "H")
        close(dP[:, :2 * N], dPr, td + HALF[dtype] * (np.abs(dPr) + td), "dP")
        assert (H[:, N:] == 3.0).all() and (dP[:, 2 * N:] == 3.0).all()
        b.lrd_gate_bwd(d, dHd, Pd, Pd)                       # in place
        assert torch.equal(Pd[:, :2 * N], dP[:, :2 * N])


@pytest.mark.parametrize("N", [776, 777, 778, 779, 780, 781, 782, 783])
def test_gate_rows_off_16_bytes(N):
    """Longer rows whose halves and results start on boundaries of their own, NaN around them, and the backward pass in place."""
    M, act = 2736, ACTS[N % 3]
    P, dH = (wl.round_to(wl.normal(1050 + N + i, (M, (2 - i) * N), 2.0), "bf16") for i in (0, 1))
    P64, dH64 = P.astype(np.float64), dH.astype(np.float64)
    Hr, dPr = o.gate_fwd(P64, act), o.gate_bwd(dH64, P64, act)
    th, td = np.abs(P64[:, :N] * P64[:, N:]) * ACT["bf16"], gate_bwd_tolerance(dH64, P64, "bf16")
    for ldp, ldh, shift in ((2 * N, N, 0), (2 * N + 1, N + 6, 0), (2 * N + 3, N + 5, 1), (2 * N, N, 7)):
        d = b.glu_desc(M, 0, N, b.LRD_BF16, act, ldh=ldh, ldp=ldp)
        Pd, dHd = padded(P, ldp, "bf16", shift=shift), padded(dH, ldh, "bf16", shift=(shift + 3) % 8)
        H, dP = padded(P[:, :0], ldh, "bf16", 3.0, shift), padded(P[:, :0], ldp, "bf16", 3.0, 7 - shift)
        b.lrd_gate_fwd(d, Pd, H)
        b.lrd_gate_bwd(d, dHd, Pd, dP)
        close(H[:, :N], Hr, th + HALF["bf16"] * (np.abs(Hr) + th), "H")
        close(dP[:, :2 * N], dPr, td + HALF["bf16"] * (np.abs(dPr) + td), "dP")
        assert (H[:, N:] == 3.0).all() and (dP[:, 2 * N:] == 3.0).all()
        b.lrd_gate_bwd(d, dHd, Pd, Pd)
        assert torch.equal(Pd[:, :2 * N], dP[:, :2 * N]) and Pd[:, 2 * N:].isnan().all()


def test_bias_gradient_of_odd_halves():
    """The sums beside the gate over halves that start on no boundary."""
    c = make(2760, 2816, 777, "bf16", 1080)
    first, again = (check_bwd(c, b.LRD_ACT_GELU) for _ in range(2))
    assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_arguments(dtype, act):
    """Finite arguments of any size give finite values and slopes: the limits of the activation."""
    big = [1e3, 1e10, 1e19, 1e25, 1e30]
    G = np.array([[s * v for v in big] + [s * 80.0, s * 90.0, s * 13.0] for s in (1.0, -1.0)])
    U = np.full_like(G, 0.5)
    P = wl.round_to(np.concatenate([G, U], axis=1), dtype)
    d = b.glu_desc(2, 0, 8, DT[dtype][0], act)
    Pd, H, dP, one = dev(P, dtype), torch.zeros(2, 8, dtype=DT[dtype][1], device="cuda"), torch.zeros(2, 16, dtype=DT[dtype][1], device="cuda"), None
    one = torch.ones_like(H)
    b.lrd_gate_fwd(d, Pd, H)
    b.lrd_gate_bwd(d, one, Pd, dP)
    g = host(Pd)[:, :8]
    limit, step = np.where(g > 0, g, 0.0), np.where(g > 0, 1.0, 0.0)
    # (silu and both gelu are within 1e-4 of their limits from 13 on)
    assert np.abs(host(H) - 0.5 * limit).max() <= 1e-4 + 2.0 ** -7 * 0.5 * np.abs(limit).max()
    assert (np.abs(host(H) - 0.5 * limit) <= 1e-4 + 2.0 ** -8 * np.abs(limit)).all()
    assert (np.abs(host(dP)[:, :8] - 0.5 * step) <= 1e-4 + 2.0 ** -9).all()
    assert (np.abs(host(dP)[:, 8:] - limit) <= 2e-4 + 2.0 ** -8 * np.abs(limit)).all()


@pytest.mark.parametrize("M", [7, 200])
def test_a_row_with_nan_or_infinities_stays_by_itself(M):
    c = make(M, 136, 72, "bf16", 1100 + M)
    clean, _ = check_fwd(c, b.LRD_ACT_SILU)
    d = dict(c, X=c["X"].copy())
    d["X"][3, 5], d["X"][5, 0] = NAN, np.inf
    H, P = run_fwd(d, b.LRD_ACT_SILU)
    rest = [i for i in range(M) if i not in (3, 5)]
    assert torch.equal(H[rest], clean[rest]) and torch.isnan(H[3]).all() and torch.isnan(P[3]).all() and not torch.isfinite(P[5]).any()


def test_on_another_stream_and_in_a_graph():
    """Work goes to the stream it is given; a captured forward + backward replays on new contents of its buffers, beside a second
    graph with a workspace of its own."""
    size, act = (260, 136, 72), b.LRD_ACT_GELU
    cases = [make(*size, "bf16", 1200 + i) for i in range(3)]
    want = []
    for c in cases:
        P = wl.round_to(o.glu_fwd(c["X"], c["W"], c["b"], act)[1], "bf16")
        want.append((run_fwd(c, act), run_bwd(c, act, P)))
    M, K, N = size
    desc = b.glu_desc(M, K, N, b.LRD_BF16, act)
    new = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")

    class Step:
        def __init__(self):
            self.t = {k: new(*s) for k, s in (("X", (M, K)), ("W", (2 * N, K)), ("b", (2 * N,)), ("dH", (M, N)), ("H", (M, N)), ("P", (M, 2 * N)),
                                              ("dX", (M, K)), ("dW", (2 * N, K)), ("db", (2 * N,)))}
            self.ws = workspace(b.lrd_glu_workspace_bytes(desc, 1))

        def fill(self, c):
            for k in ("X", "W", "b", "dH"):
                self.t[k].copy_(dev(c[k], "bf16"))

        def run(self):
            t = self.t
            b.lrd_dense_glu_fwd(desc, t["X"], t["W"], t["b"], t["H"], t["P"], self.ws)
            b.lrd_dense_glu_bwd(desc, t["dH"], t["X"], t["W"], t["P"], t["dX"], t["dW"], t["db"], self.ws)

    def check(step, i):
        (H, P), g = want[i]
        assert torch.equal(step.t["H"], H) and torch.equal(step.t["P"], P)
        # (the forward's own P instead of the oracle's rounded one: off by a rounding here and there)
        for k in ("dX", "dW", "db"):
            a, r = host(step.t[k]), host(g[k])
            assert np.abs(a - r).max() <= 2e-2 * np.abs(r).max(), k

    side = torch.cuda.Stream()
    one, two = Step(), Step()
    one.fill(cases[0])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        one.run()
    side.synchronize()
    check(one, 0)
    graphs = []
    for step in (one, two):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step.run()
        graphs.append(g)
    for i in (1, 2):
        one.fill(cases[i])
        two.fill(cases[3 - i])
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        check(one, i)
        check(two, 3 - i)
    assert b.lrd_check_device_status() == b.LRD_OK


@pytest.mark.parametrize("M", [1, 333])
def test_a_whole_block_trained(M):
    """Gated half, plain second half, forward and backward, as a training step calls them: against the oracle fed with each stage's
    own (rounded) input."""
    K, N, act = 72, 136, b.LRD_ACT_SILU
    c = make(M, K, N, "bf16", 1300 + M)
    Wd, dY = wl.round_to(wl.normal(1, (K, N), N ** -0.5), "bf16"), wl.round_to(wl.normal(2, (M, K)), "bf16")
    bf = torch.bfloat16
    new = lambda *s: torch.empty(*s, dtype=bf, device="cuda")
    X, W, bias, Wdd, dYd = (dev(t, "bf16") for t in (c["X"], c["W"], c["b"], Wd, dY))
    desc, down = b.glu_desc(M, K, N, b.LRD_BF16, act), b.linear_desc(M, N, K, 0, b.LRD_BF16)
    ws = workspace(max(b.lrd_glu_workspace_bytes(desc, 1), b.lrd_dense_workspace_bytes(down, 1)))
    H, P, Y, dH, dWd, dX, dW, db = new(M, N), new(M, 2 * N), new(M, K), new(M, N), new(K, N), new(M, K), new(2 * N, K), new(2 * N)
    b.lrd_dense_glu_fwd(desc, X, W, bias, H, P, ws)
    b.lrd_dense_fwd(down, H, Wdd, None, Y, ws)
    b.lrd_dense_bwd(down, dYd, H, Wdd, dH, dWd, None, ws)
    b.lrd_dense_glu_bwd(desc, dH, X, W, P, dX, dW, db, ws)
    torch.cuda.synchronize()
    th, tp = fwd_tolerance(c, o.glu_fwd(c["X"], c["W"], c["b"], act)[1], act)
    close(H, o.glu_fwd(c["X"], c["W"], c["b"], act)[0], th, "H")
    Hn, Pn, dHn = host(H), host(P), host(dH)
    rounded = lambda a, b_, n: (n + 2) * 2.0 ** -23 * (np.abs(a) @ np.abs(b_)) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(a @ b_)
    close(Y, Hn @ Wd.T.astype(np.float64), rounded(Hn, Wd.T.astype(np.float64), N), "Y")
    close(dH, dY.astype(np.float64) @ Wd, rounded(dY.astype(np.float64), Wd.astype(np.float64), K), "dH")
    ref = o.glu_bwd(dHn, c["X"], c["W"], Pn, act)
    tol = bwd_tolerance(dict(c, dH=dHn), ref, Pn)
    for k, t in (("dX", dX), ("dW", dW), ("db", db)):
        close(t, ref[k], tol[k], k)


@pytest.mark.parametrize("freeze", [b.LRD_FREEZE_NONE, b.LRD_FREEZE_U, b.LRD_FREEZE_V])
def test_a_gate_behind_decomposed_projections(freeze):
    """Two decomposed layers write the halves of P, the gate follows, and its gradient goes back through both of them."""
    M, K, N, r, act = 300, 136, 200, 48, b.LRD_ACT_GELU_TANH
    layers = [wl.random_factor_case(M, K, N, r, "bf16", 1400 + 10 * i) for i in (0, 1)]
    X = layers[0]["X"]
    dH = wl.round_to(wl.normal(5, (M, N)), "bf16")
    new = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")
    Xd, dHd, P, dP, H = dev(X, "bf16"), dev(dH, "bf16"), new(M, 2 * N), new(M, 2 * N), new(M, N)
    lin, gate = b.linear_desc(M, K, N, r, b.LRD_BF16, ldy=2 * N), b.glu_desc(M, 0, N, b.LRD_BF16, act)
    V, U, bias = ([dev(L[k], "bf16") for L in layers] for k in ("V", "U", "b"))
    Z = None if freeze == b.LRD_FREEZE_U else [new(M, r) for _ in layers]
    ws = [workspace(max(b.lrd_linear_workspace_bytes(lin, freeze, i) for i in (0, 1))) for _ in layers]
    dX, dU, dV, db = [new(M, K) for _ in layers], [new(N, r) for _ in layers], [new(K, r) for _ in layers], [new(N) for _ in layers]
    halves = lambda t: [t[:, :N], t[:, N:]]
    b.lrd_linear_group_fwd([lin, lin], [Xd, Xd], V, U, bias, halves(P), Z, freeze, ws)
    b.lrd_gate_fwd(gate, P, H)
    b.lrd_gate_bwd(gate, dHd, P, dP)
    b.lrd_linear_group_bwd([lin, lin], halves(dP), [Xd, Xd], V, U, Z, dX, dU, dV, db, freeze, ws)
    torch.cuda.synchronize()
    Pn = host(P)
    th = np.abs(Pn[:, :N] * Pn[:, N:]) * ACT["bf16"]
    Hr = o.gate_fwd(Pn, act)
    close(H, Hr, th + 2.0 ** -8 * (np.abs(Hr) + th), "H")
    dPn, dPr, td = host(dP), o.gate_bwd(dH, Pn, act), gate_bwd_tolerance(dH.astype(np.float64), Pn, "bf16")
    close(dP, dPr, td + 2.0 ** -8 * (np.abs(dPr) + td), "dP")
    from helpers import TOL, rel_err
    for i, L in enumerate(layers):
        Zr, Yr = o.linear_fwd(X, L["V"], L["U"], L["b"])
        g = o.linear_bwd(dPn[:, i * N:(i + 1) * N], X, L["V"], L["U"], Zr, freeze)
        assert rel_err(P[:, i * N:(i + 1) * N], Yr) <= TOL["bf16"]
        for k, t in (("dX", dX[i]), ("dU", dU[i]), ("dV", dV[i]), ("db", db[i])):
            assert rel_err(t, g[k]) <= TOL["bf16"], (i, k)


def test_many_rows_of_the_result_past_32_bits():
    """Element offsets beyond 2^31: a gate over 2.2 G elements of P, its last rows looked at."""
    M, N = 1 << 20, 1056
    P = torch.empty(M, 2 * N, dtype=torch.bfloat16, device="cuda")
    H = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    P.fill_(1.0)
    P[-3:] = torch.randn(3, 2 * N, device="cuda").to(torch.bfloat16)
    d = b.glu_desc(M, 0, N, b.LRD_BF16)
    b.lrd_gate_fwd(d, P, H)
    b.lrd_gate_bwd(d, H, P, P)                               # (and back, in place)
    torch.cuda.synchronize()
    assert P.numel() > 2 ** 31
    one = o.activation(1.0, o.ACT_SILU)
    assert (H[:-3] == torch.tensor(float(one[0])).to(torch.bfloat16).item()).all()
    dP = P[: M - 3]
    assert (dP[:, N:] == dP[0, N]).all() and abs(float(dP[0, N]) - float(one[0]) ** 2) <= 3 * 2.0 ** -8
    assert torch.isfinite(P[-3:].float()).all() and torch.isfinite(H[-3:].float()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 2, 3, 4])
def test_few_tokens(M, dtype):
    """Decoding: short and long reductions, whole and ragged 16-byte pieces, padded rows and bases off 16 bytes."""
    for i, (K, N) in enumerate([(1, 1), (8, 7), (257, 33), (512, 40), (2056, 65), (4099, 18), (8192, 24)]):
        c = make(M, K, N, dtype, 1500 + 10 * M + i, bias=i % 2 == 0)
        for act in ACTS:
            check_fwd(c, act, save=act == b.LRD_ACT_SILU)
        check_fwd(c, b.LRD_ACT_SILU, lds=(K + 8, K + 16, N + 3, 2 * N + 5))
        check_fwd(c, b.LRD_ACT_SILU, lds=(K + 3, K + 1, N, 2 * N), shift=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_tokens_at_every_alignment(dtype):
    """Rows a few pieces long, off 16-byte boundaries: where the first and the last whole piece end, for each offset of X against W."""
    for K in (list(range(9, 50)) if dtype == "bf16" else list(range(5, 26))) + [333, 1031]:
        c = make(1 + K % 4, K, 9, dtype, 1600 + K, bias=K % 2 == 0)
        for dx in range(8 if dtype == "bf16" else 4):
            check_fwd(c, b.LRD_ACT_SILU, lds=(K + dx, K + 1, 9, 18), shift=dx % 2, save=False)


def split_fits(M, k_blocks, columns, split, gated=True):
    """Whether every block of the cluster gets a share of the k-blocks (two a stage up to 96 columns) and what they exchange (32 rows x
    32 columns of fp32 at a time) fits into shared memory's 150 KB and some."""
    g = 2 if columns <= 96 else 1
    share = -(-(-(-k_blocks // split)) // g) * g
    pieces = -(-(columns // 2 if gated else columns) // 32)
    rows = -(-min(M, 128) // 32) * 32
    return (split - 1) * share < k_blocks and split * -(-pieces // split) * (2 if gated else 1) * rows * 128 <= 131072


@pytest.mark.parametrize("columns", [32, 64, 128, 256])
@pytest.mark.parametrize("split", [2, 4, 8])
@pytest.mark.parametrize("size", [(1, 1024, 24), (9, 1100, 333), (32, 2048, 200), (61, 700, 136), (128, 1032, 264), (200, 1500, 129)])
def test_split_reductions(size, split, columns):
    """A tile's reduction shared by the blocks of a cluster: every share and width, ragged rows and columns, repeated bits."""
    M, K, N = size
    c = make(*size, "bf16", 1700 + M)
    b.lrd_glu_tuning(columns, 1, split)
    try:
        for lds in (None, ((K + 7) // 8 * 8, (K + 7) // 8 * 8 + 8, (N + 7) // 8 * 8, 2 * N + 1)):
            first = check_fwd(c, b.LRD_ACT_SILU, lds=lds)
            again = check_fwd(c, b.LRD_ACT_SILU, lds=lds)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    except b.LrdError as e:
        assert e.status == b.LRD_ERR_UNSUPPORTED and not split_fits(M, -(-K // 64), columns, split)
    finally:
        b.lrd_glu_tuning()


@pytest.mark.parametrize("size", [(4096, 1024, 704), (700, 1176, 640), (513, 1000, 1032), (1336, 256, 768), (300, 2056, 520), (2000, 264, 1544)])
def test_both_gradients_of_larger_layers(size):
    """Sizes at which dX and dW share a launch, or dW walks over its tiles unsplit, in tiles of every width: with and without the input and the
    bias gradient, repeated bits, the weights' gradient the same whether or not the input's is wanted."""
    c = make(*size, "bf16", 1800 + size[0])
    act = b.LRD_ACT_SILU
    full = check_bwd(c, act)
    again = check_bwd(c, act)
    assert all(torch.equal(full[k], again[k]) for k in full)
    part = check_bwd(c, act, want_dx=False)
    plain = check_bwd(c, act, want_db=False)
    for k, other in (("dW", part), ("db", part), ("dW", plain), ("dX", plain)):      # (another order of sums: off by a rounding of either)
        assert np.abs(host(full[k]) - host(other[k])).max() <= 2.0 ** -6 * np.abs(host(full[k])).max()
