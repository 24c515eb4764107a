"""Results whose rows end inside 16 bytes: what stands between a row's last column and the next row is left as it was.

Widths off multiples of 8 in rows that are padded to one, so that the tensor-core kernels take them; every result is a block of a wider
matrix filled with a number, next to a column of which the last row ends.  Values against the oracle within the suite's tolerance."""
import numpy as np
import pytest
import torch

from oracle import lrd_oracle as o
from paper_2309_03824_b200 import binding as b
from paper_2309_03824_b200 import workloads as wl

from helpers import TOL, dev, host, rel_err, workspace

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
FILL = 3.0
up8 = lambda n: (n + 7) // 8 * 8


def rows_of(a, ld):
    """a on the device in rows of ld elements, NaN behind each."""
    t = torch.full((a.shape[0], ld), float("nan"), dtype=BF, device="cuda")
    t[:, : a.shape[1]] = dev(a, "bf16")
    return t


def blank(rows, ld):
    return torch.full((rows, ld), FILL, dtype=BF, device="cuda")


def check(got, want, cols, name, tol=TOL["bf16"]):
    assert rel_err(got[:, :cols], want) <= tol, name
    assert (got[:, cols:] == FILL).all(), (name, np.argwhere(host(got[:, cols:]) != FILL)[:4].tolist())


def linear(M, K, N, r, seed, calls, accumulate=False):
    """Forward and backward of a layer, every leading dimension the next multiple of 8; calls(desc) around them."""
    c = wl.random_factor_case(M, K, N, r, "bf16", seed)
    ldx, ldr, ldy = up8(K), up8(r), up8(N)
    desc = b.linear_desc(M, K, N, r, b.LRD_BF16, ldx, ldr, ldr, ldy, ldr)
    X, V, U, dY = rows_of(c["X"], ldx), rows_of(c["V"], ldr), rows_of(c["U"], ldr), rows_of(c["dY"], ldy)
    Y, Z, dX, dU, dV, db = blank(M, ldy), blank(M, ldr), blank(M, ldx), blank(N, ldr), blank(K, ldr), blank(1, up8(N))
    ws = workspace(max(b.lrd_linear_workspace_bytes(desc, 0, i) for i in (0, 1, 2)))
    Zr, Yr = o.linear_fwd(c["X"], c["V"], c["U"], c["b"])
    g = o.linear_bwd(c["dY"], c["X"], c["V"], c["U"], Zr, 0)
    with calls:
        b.lrd_linear_fwd(desc, X, V, U, dev(c["b"], "bf16"), Y, Z, 0, ws)
        if accumulate:
            dU[:, :r], dV[:, :r] = 0.0, 0.0
            b.lrd_linear_bwd_accumulate(desc, dY, X, V, U, Z, dX, dU, dV, None, 0, ws)
        else:
            b.lrd_linear_bwd(desc, dY, X, V, U, Z, dX, dU, dV, db, 0, ws)
        torch.cuda.synchronize()
    assert b.lrd_check_device_status() == b.LRD_OK
    for name, t, want, cols in (("Y", Y, Yr, N), ("Z", Z, Zr, r), ("dX", dX, g["dX"], K), ("dU", dU, g["dU"], r), ("dV", dV, g["dV"], r)):
        check(t, want, cols, name)
    if not accumulate:
        check(db, g["db"][None], N, "db")


class Form:
    """Calls on one of the forms a layer takes."""
    def __init__(self, path, mma_blocks=0):
        self.path, self.mma_blocks = path, mma_blocks

    def __enter__(self):
        b.lrd_set_path(self.path)
        b.lrd_chain_pair_tuning(self.mma_blocks, 0, 0, 0)

    def __exit__(self, *e):
        b.lrd_set_path(b.LRD_PATH_AUTO)
        b.lrd_chain_pair_tuning(0, 0, 0, 0)


FORMS = {"auto": Form(b.LRD_PATH_AUTO), "products": Form(b.LRD_PATH_UNFUSED), "chain": Form(b.LRD_PATH_FUSED, 1), "pairs": Form(b.LRD_PATH_FUSED, 2)}


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("K,N,r", [(196, 204, 64), (260, 129, 32), (135, 327, 96), (513, 1030, 64), (90, 71, 64)])
@pytest.mark.parametrize("M", [5, 300])
def test_widths_off_multiples_of_8(M, K, N, r, form):
    linear(M, K, N, r, 2000 + K, FORMS[form])


@pytest.mark.parametrize("form", ["auto", "products"])
@pytest.mark.parametrize("r", [7, 44, 61, 75])
@pytest.mark.parametrize("M", [40, 300, 1500])
def test_ranks_off_multiples_of_8(M, r, form):
    """Z and the factors' gradients in rows padded by the caller."""
    linear(M, 264, 200, r, 2100 + r, FORMS[form])


@pytest.mark.parametrize("r", [44, 61])
@pytest.mark.parametrize("M", [40, 1500])
def test_accumulated_gradients(M, r):
    linear(M, 264, 200, r, 2200 + r, FORMS["auto"], accumulate=True)


@pytest.mark.parametrize("blocks,columns,split", [(1, 64, 1), (1, 64, 4), (1, 128, 1), (1, 192, 1), (1, 192, 2), (2, 128, 1), (2, 256, 2)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_every_form_of_the_gradients(blocks, columns, split, accumulate):
    b.lrd_wgrad_tuning(blocks, columns, split)
    try:
        linear(700, 520, 456, 205, 2300, FORMS["auto"], accumulate)
    finally:
        b.lrd_wgrad_tuning(0, 0, 0)


@pytest.mark.parametrize("M,K,N", [(300, 200, 204), (64, 1029, 77), (300, 196, 5), (700, 333, 1027), (4100, 264, 130)])
@pytest.mark.parametrize("blocks", [0, 1, 2])
def test_undecomposed_layers(M, K, N, blocks):
    X, W = wl.round_to(wl.normal(1, (M, K)), "bf16"), wl.round_to(wl.normal(2, (N, K), K ** -0.5), "bf16")
    bias, dY = wl.round_to(wl.normal(3, (N,), 0.1), "bf16"), wl.round_to(wl.normal(4, (M, N)), "bf16")
    ldk, ldy = up8(K), up8(N)
    desc = b.linear_desc(M, K, N, 0, b.LRD_BF16, ldx=ldk, ldv=ldk, ldy=ldy)
    Xd, Wd, dYd = rows_of(X, ldk), rows_of(W, ldk), rows_of(dY, ldy)
    Y, dX, dW, db = blank(M, ldy), blank(M, ldk), blank(N, ldk), blank(1, ldy)
    ws = workspace(b.lrd_dense_workspace_bytes(desc, 1))
    b.lrd_gemm_tuning(blocks)
    try:
        b.lrd_dense_fwd(desc, Xd, Wd, dev(bias, "bf16"), Y, ws)
        b.lrd_dense_bwd(desc, dYd, Xd, Wd, dX, dW, db, ws)
        torch.cuda.synchronize()
    finally:
        b.lrd_gemm_tuning(0)
    g = o.dense_bwd(dY, X, W)
    for name, t, want, cols in (("Y", Y, o.dense_fwd(X, W, bias), N), ("dX", dX, g["dX"], K), ("dW", dW, g["dW"], K), ("db", db, g["db"][None], N)):
        check(t, want, cols, name)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("N", [204, 333])
@pytest.mark.parametrize("order", ["up first", "gate first", "together"])
def test_halves_of_a_gated_block(order, N, form):
    """Two decomposed layers write the halves of P, in either order and side by side, and the gate reads them."""
    M, K, r = 300, 136, 64
    layers = [wl.random_factor_case(M, K, N, r, "bf16", 2400 + 10 * i) for i in (0, 1)]
    X, ldp = dev(layers[0]["X"], "bf16"), up8(2 * N)
    lin, gate = b.linear_desc(M, K, N, r, b.LRD_BF16, ldy=ldp), b.glu_desc(M, 0, N, b.LRD_BF16, b.LRD_ACT_SILU, ldp=ldp)
    V, U, bias = ([dev(L[k], "bf16") for L in layers] for k in ("V", "U", "b"))
    ws = [workspace(b.lrd_linear_workspace_bytes(lin, b.LRD_FREEZE_U, 0)) for _ in layers]
    P, H = blank(M, ldp), torch.empty(M, N, dtype=BF, device="cuda")
    halves = [P[:, :N], P[:, N:2 * N]]
    with FORMS[form]:
        if order == "together":
            b.lrd_linear_group_fwd([lin, lin], [X, X], V, U, bias, halves, None, b.LRD_FREEZE_U, ws)
        else:
            for i in (1, 0) if order == "up first" else (0, 1):
                b.lrd_linear_fwd(lin, X, V[i], U[i], bias[i], halves[i], None, b.LRD_FREEZE_U, ws[i])
        b.lrd_gate_fwd(gate, P, H)
        torch.cuda.synchronize()
    want = np.concatenate([o.linear_fwd(layers[0]["X"], L["V"], L["U"], L["b"])[1] for L in layers], axis=1)
    check(P, want, 2 * N, "P")
    assert rel_err(H, o.gate_fwd(host(P)[:, :2 * N], b.LRD_ACT_SILU)) <= TOL["bf16"]


@pytest.mark.parametrize("form", ["auto", "pairs"])
@pytest.mark.parametrize("K,N", [(196, 204), (333, 130), (264, 77)])
@pytest.mark.parametrize("n", [2, 4])
def test_groups_of_layers(n, K, N, form):
    """Layers that share a launch: each one's own results and leading dimensions."""
    M, r = 300, 64
    layers = [wl.random_factor_case(M, K, N, r, "bf16", 2500 + 10 * i) for i in range(n)]
    ldx, lds = up8(K), [up8(N) + 8 * i for i in range(n)]
    descs = [b.linear_desc(M, K, N, r, b.LRD_BF16, ldx=ldx, ldy=ld) for ld in lds]
    X, dY = [rows_of(L["X"], ldx) for L in layers], [rows_of(L["dY"], ld) for L, ld in zip(layers, lds)]
    V, U, bias = ([dev(L[k], "bf16") for L in layers] for k in ("V", "U", "b"))
    Y, Z, dX = [blank(M, ld) for ld in lds], [blank(M, r) for _ in layers], [blank(M, ldx) for _ in layers]
    dU, dV, db = [blank(N, r) for _ in layers], [blank(K, r) for _ in layers], [blank(1, N) for _ in layers]
    ws = [workspace(max(b.lrd_linear_workspace_bytes(d, 0, i) for i in (0, 1))) for d in descs]
    with FORMS[form]:
        b.lrd_linear_group_fwd(descs, X, V, U, bias, Y, Z, 0, ws)
        b.lrd_linear_group_bwd(descs, dY, X, V, U, Z, dX, dU, dV, db, 0, ws)
        torch.cuda.synchronize()
    for i, L in enumerate(layers):
        Zr, Yr = o.linear_fwd(L["X"], L["V"], L["U"], L["b"])
        g = o.linear_bwd(L["dY"], L["X"], L["V"], L["U"], Zr, 0)
        for name, t, want, cols in (("Y", Y, Yr, N), ("Z", Z, Zr, r), ("dX", dX, g["dX"], K), ("dU", dU, g["dU"], r), ("dV", dV, g["dV"], r), ("db", db, g["db"][None], N)):
            check(t[i], want, cols, (i, name))
