"""Gated and 8-bit products at the sizes where they take their larger forms, against products in 64 bits on the device.

Which form ran is read from the number of launches: the gate with the sums beside it is two launches, without them one, a shared launch
for dX and dW one, each of them alone one."""
import pytest
import torch

from paper_2309_03824_b200 import binding as b

from helpers import workspace

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def normal(seed, *shape, std=1.0):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).mul_(std).to(BF)


def silu(x):
    s = torch.sigmoid(x)
    return x * s, s * (1 + x * torch.sigmoid(-x))


def close(got, want, tol, name):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (name, float(err.max()), torch.nonzero(~(err <= tol))[:4].tolist())


def backward(M, K, N, want_dx, want_db):
    """(launches, dX, dW, db), checked: dP is rounded once (2^-8 of it, and 2^-18 (1 + |g|) of the factors for the approximated activation),
    sums of n products in fp32 are off by n 2^-23 of their magnitudes, results are rounded once."""
    X, W, dH, P = normal(1, M, K), normal(2, 2 * N, K, std=K ** -0.5), normal(3, M, N), normal(4, M, 2 * N)
    d = b.glu_desc(M, K, N, b.LRD_BF16)
    ldk = (K + 7) // 8 * 8
    dX, dW, db = torch.full((M, K), 3.0, dtype=BF, device="cuda"), torch.full((2 * N, K), 3.0, dtype=BF, device="cuda"), torch.full((2 * N,), 3.0, dtype=BF, device="cuda")
    ws = workspace(b.lrd_glu_workspace_bytes(d, 1))
    before = b.lrd_launch_count()
    b.lrd_dense_glu_bwd(d, dH, X, W, P, dX if want_dx else None, dW, db if want_db else None, ws)
    launches = b.lrd_launch_count() - before
    first = [t.clone() for t in (dX, dW, db)]
    b.lrd_dense_glu_bwd(d, dH, X, W, P, dX if want_dx else None, dW, db if want_db else None, ws)
    torch.cuda.synchronize()
    assert b.lrd_check_device_status() == b.LRD_OK and all(torch.equal(a, c) for a, c in zip(first, (dX, dW, db)))
    G, U, D = P[:, :N].double(), P[:, N:].double(), dH.double()
    value, slope = silu(G)
    dP = torch.hstack([D * U * slope, D * value])
    off = torch.hstack([(D * U).abs() * (1 + G.abs()), (D * G).abs()]) * 2.0 ** -18
    off = off + 2.0 ** -8 * (dP.abs() + off)
    mag = dP.abs() + off
    results = [("dW", dW, dP.T, off.T, X, M)] + ([("dX", dX, dP, off, W, 2 * N)] if want_dx else [])
    for name, got, left, loff, right, n in results:
        want, r = left @ right.double(), right.double().abs()
        tol = loff @ r + (n + 2) * 2.0 ** -23 * (mag.T if name == "dW" else mag) @ r
        close(got, want, tol + 2.0 ** -8 * (want.abs() + tol), name)
    if want_db:
        want, tol = dP.sum(0), off.sum(0) + (M + 2) * 2.0 ** -23 * mag.sum(0)
        close(db, want, tol + 2.0 ** -8 * (want.abs() + tol), "db")
    return launches


# tiles 256, 192 and 128 columns wide by the rounds they leave; ragged rows, columns and tokens; 42 and 57 MB of dP, walked over in groups of row
# tiles, the last of them smaller than the others; one token, and one more than a k-block
@pytest.mark.parametrize("M,K,N", [(330, 504, 4730), (300, 2000, 1160), (300, 104, 9476), (1500, 520, 7000), (1500, 88, 9500),
                                   (1, 104, 9476), (65, 520, 7000)])
def test_weight_gradients_by_an_unsplit_walk(M, K, N):
    assert backward(M, K, N, False, True) == 3               # (sums beside the gate: otherwise they would ride on dW)


# each width of dX's tiles with each of dW's, either's first; then weight gradients that would walk unsplit by themselves, and 42 MB of
# dP in groups of row tiles, the last of them smaller
@pytest.mark.parametrize("M,K,N", [(867, 168, 464), (893, 160, 440), (906, 192, 600), (861, 1256, 464), (521, 568, 392), (469, 2464, 296),
                                   (803, 1352, 344), (645, 264, 240), (968, 1416, 520), (649, 1888, 304), (632, 1944, 480), (715, 2136, 392),
                                   (840, 1552, 296), (994, 136, 264), (940, 1816, 424), (859, 1800, 264), (923, 1872, 600), (964, 2064, 440),
                                   (307, 1560, 1290), (3900, 1032, 2850)])
def test_both_products_in_one_launch(M, K, N):
    assert backward(M, K, N, True, False) == 2
    assert backward(M, K, N, True, True) == 3


def test_a_gated_product_in_groups_of_rows():
    """More rows of X than L2 keeps (42 MB): the tiles are walked over in groups of rows, the last one smaller."""
    M, K, N = 5000, 4200, 900
    X, W = normal(5, M, K), normal(6, 2 * N, K, std=K ** -0.5)
    H, P = torch.zeros(M, N, dtype=BF, device="cuda"), torch.zeros(M, 2 * N, dtype=BF, device="cuda")
    d = b.glu_desc(M, K, N, b.LRD_BF16)
    b.lrd_dense_glu_fwd(d, X, W, None, H, P, workspace(b.lrd_glu_workspace_bytes(d, 0)))
    want = X.double() @ W.double().T
    off = (K + 2) * 2.0 ** -23 * (X.double().abs() @ W.double().abs().T)
    close(P, want, off + 2.0 ** -8 * (want.abs() + off), "P")
    G, U = want[:, :N], want[:, N:]
    value = silu(G)[0]
    tol = (G * U).abs() * 2.0 ** -18 + 1.2 * off[:, :N] * (U.abs() + off[:, N:]) + value.abs() * off[:, N:]
    close(H, value * U, tol + 2.0 ** -8 * ((value * U).abs() + tol), "H")


@pytest.mark.parametrize("gated", [False, True])
def test_an_8_bit_product_in_groups_of_rows(gated):
    M, K, N = 10500, 4240, 700
    rows = 2 * N if gated else N
    g = torch.Generator(device="cuda").manual_seed(7)
    q, w = (torch.randint(-127, 128, (n, K), dtype=torch.int8, device="cuda", generator=g) for n in (M, rows))
    s, t = torch.rand(M, device="cuda", generator=g) / 127, torch.rand(rows, device="cuda", generator=g) / 127 / K ** 0.5
    Y = torch.zeros(M, N, dtype=BF, device="cuda")
    (b.lrd_i8_glu_fwd if gated else b.lrd_i8_dense_fwd)(b.i8_desc(M, K, N, b.LRD_BF16), q, s, w, t, None, Y, None)
    P = (q.double() @ w.double().T) * s.double()[:, None] * t.double()
    off = 4 * 2.0 ** -24 * P.abs()
    if not gated:
        close(Y, P, off + 2.0 ** -8 * (P.abs() + off), "Y")
        return
    G, U = P[:, :N], P[:, N:]
    value = silu(G)[0]
    tol = (G * U).abs() * 2.0 ** -18 + 1.2 * off[:, :N] * (U.abs() + off[:, N:]) + value.abs() * off[:, N:]
    close(Y, value * U, tol + 2.0 ** -8 * ((value * U).abs() + tol), "H")


@pytest.mark.parametrize("columns,blocks,split", [(0, 0, 0), (32, 1, 1), (256, 1, 4), (64, 1, 2), (256, 1, 1), (128, 2, 0), (256, 2, 0)])
@pytest.mark.parametrize("M", [9, 200])
@pytest.mark.parametrize("gated", [False, True])
def test_the_longest_sums_on_the_tensor_cores(M, gated, columns, blocks, split):
    """131071 products of -128 x -128 beside -128 x 127: 2^31 - 2^14, the largest a call can form, and next to the smallest."""
    if (columns == 32 and M > 128) or (blocks == 2 and M <= 128):
        pytest.skip("no such form")
    K, N = 131071, 40
    rows = 2 * N if gated else N
    q, w = torch.full((M, K + 1), -128, dtype=torch.int8, device="cuda"), torch.full((rows, K + 1), -128, dtype=torch.int8, device="cuda")
    w[1:rows:2] = 127
    one, t = torch.ones(M, device="cuda"), torch.full((rows,), 2.0 ** -31 if gated else 1.0, device="cuda")
    Y = torch.zeros(M, N, device="cuda")
    b.lrd_glu_tuning(columns, blocks, split)
    try:
        (b.lrd_i8_glu_fwd if gated else b.lrd_i8_dense_fwd)(b.i8_desc(M, K, N, b.LRD_F32, ldx=K + 1, ldw=K + 1), q, one, w, t, None, Y, None)
    finally:
        b.lrd_glu_tuning()
    sums = torch.where(torch.arange(rows, device="cuda") % 2 == 0, K * 2.0 ** 14, -K * 128.0 * 127.0).double()
    if not gated:
        assert (Y.double() == sums.float().double()).all()
        return
    P = sums.float().double() * 2.0 ** -31                  # (exact products with a power of two)
    want = silu(P[:N])[0] * P[N:]
    assert ((Y.double() - want).abs() <= 2.0 ** -20 * want.abs()).all()
