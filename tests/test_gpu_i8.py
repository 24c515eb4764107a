"""Rows quantized to 8 bits and products of 8-bit integers against the fp64 oracle, through the C ABI.

Quantized integers and scales are equal to the oracle's, bit for bit.  A product's sum is exact; times two scales plus bias in fp32 it
is off by at most four roundings of 2^-24 of the magnitudes, then rounded to the result's type (half a step)."""
import numpy as np
import pytest
import torch

from oracle import lrd_oracle as o
from paper_2309_03824_b200 import binding as b
from paper_2309_03824_b200 import workloads as wl

from helpers import DT, dev, host, workspace
from test_gpu_glu import ACT, ACTS, HALF, NAN, close, padded, split_fits

pytestmark = pytest.mark.gpu


def quantize(X, dtype, ldx=0, ldq=0, shift=0):
    M, K = X.shape
    Xd = padded(X, ldx or K, dtype, shift=shift)
    q = torch.full((M, ldq or K), 77, dtype=torch.int8, device="cuda")
    s = torch.full((M,), NAN, device="cuda")
    b.lrd_i8_quantize(Xd, ldx, M, K, q, ldq, s, DT[dtype][0])
    torch.cuda.synchronize()
    assert (q[:, K:] == 77).all()
    return q[:, :K], s


def check_quantize(X, dtype, **kw):
    q, s = quantize(X, dtype, **kw)
    qr, sr = o.i8_quantize(X)
    assert np.array_equal(s.cpu().numpy(), sr, equal_nan=True)
    assert np.array_equal(q.cpu().numpy().astype(np.int64), qr)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1), (1, 8), (3, 16), (5, 513), (9, 1024), (4, 1032), (2, 8192), (3, 8200), (2, 20000), (300, 72), (7, 4099), (1, 70001)])
def test_quantized_rows(size, dtype):
    X = wl.round_to(wl.normal(40 + size[0], size) * np.exp(wl.normal(41, (size[1],))), dtype)
    K = size[1]
    check_quantize(X, dtype)
    check_quantize(X, dtype, ldx=K + 8, ldq=(K + 15) // 16 * 16)
    check_quantize(X, dtype, ldx=K + 3, ldq=K + 1)
    check_quantize(X, dtype, shift=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_borders_between_integers(dtype):
    """Quotients on and beside every border: n + 1/2 exactly (ties to even), and one step of the type to either side."""
    rows = []
    for top in (127.0, 127.0 * 2.0 ** 40, 127.0 * 2.0 ** -60, 100.0, 3.0, 1.0, 0.7, 1e-20, 1e20):
        top = float(wl.round_to(np.array([top]), dtype)[0])
        mid = wl.round_to((np.arange(-126, 126) + 0.5) * (top / 127.0), dtype)
        step = np.spacing(mid.astype(np.float32)) * (65536 if dtype == "bf16" else 1)
        rows.append(np.concatenate([mid, wl.round_to(mid + step, dtype), wl.round_to(mid - step, dtype), [top, -top], np.zeros(2)]))
    check_quantize(np.array(rows, dtype=np.float32), dtype)


def test_every_bf16_pair_of_largest_and_value():
    """All 128 mantissas of a row's largest value against all values of the ten binades below it, both signs."""
    rows = []
    for m in range(128, 256):
        x = np.concatenate([np.arange(128, 256) * 2.0 ** -e for e in range(10)])
        x = np.where(x <= m, x, 0.0)
        rows.append(np.concatenate([x, -x, [m, 0.0, 0.0, 0.0]]))
    for scale in (1.0, 2.0 ** -40, 2.0 ** 100):
        check_quantize(np.array(rows, dtype=np.float32) * np.float32(scale), "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_zeros_tiny_and_huge_numbers_and_no_numbers(dtype):
    n = 64
    base = wl.round_to(wl.normal(50, (1, n)), "bf16")[0]
    rows = [np.zeros(n), base * 2.0 ** -120, base * 2.0 ** -130, base * 2.0 ** -135, base * 2.0 ** 120, np.full(n, 1e-45), np.full(n, -3e-44),
            np.where(np.arange(n) == 5, 3.38e38, 1.0), np.where(np.arange(n) == 9, NAN, base), np.where(np.arange(n) == 63, np.inf, base),
            np.where(np.arange(n) == 0, -np.inf, base), np.full(n, -0.0)]
    X = np.array(rows, dtype=np.float32)
    X = np.where(np.isnan(X), np.float32(NAN), wl.round_to(np.nan_to_num(X, nan=0.0, posinf=np.inf, neginf=-np.inf), dtype)).astype(np.float32)
    check_quantize(X, dtype)


def make(M, K, N, dtype, seed, gated=False, bias=True, full=False):
    g = np.random.default_rng(seed)
    rows = 2 * N if gated else N
    lo = -128 if full else -127
    c = {"M": M, "K": K, "N": N, "dtype": dtype, "q": g.integers(lo, 128, (M, K)), "w": g.integers(lo, 128, (rows, K)),
         "s": (np.exp(g.standard_normal(M)) / 127).astype(np.float32), "t": (np.exp(0.3 * g.standard_normal(rows)) / 127 / K ** 0.5).astype(np.float32)}
    c["b"] = wl.round_to(g.standard_normal(rows) * 0.5, dtype) if bias else None
    return c


def bytes_padded(a, ld):
    t = torch.full((a.shape[0], ld), 99, dtype=torch.int8, device="cuda")
    t[:, :a.shape[1]] = torch.from_numpy(a.astype(np.int8)).cuda()
    return t


def run(c, gated, act=0, ldx=0, ldw=0, ldy=0, shift=0):
    M, K, N, dt = c["M"], c["K"], c["N"], c["dtype"]
    d = b.i8_desc(M, K, N, DT[dt][0], act, ldx, ldw, ldy)
    Y = padded(np.zeros((M, 0), np.float32), ldy or N, dt, 3.0, shift)
    need = b.lrd_i8_workspace_bytes(d, gated)
    ws = workspace(need + 256)
    ws.fill_(0x5A)
    call = b.lrd_i8_glu_fwd if gated else b.lrd_i8_dense_fwd
    call(d, bytes_padded(c["q"], ldx or K), torch.from_numpy(c["s"]).cuda(), bytes_padded(c["w"], ldw or K), torch.from_numpy(c["t"]).cuda(), dev(c["b"], dt), Y, ws[:need])
    torch.cuda.synchronize()
    assert b.lrd_check_device_status() == b.LRD_OK
    assert (ws[need:] == 0x5A).all() and (Y[:, N:] == 3.0).all()
    return Y[:, :N]


def check(c, gated, act=0, **kw):
    got = run(c, gated, act, **kw)
    P = o.i8_product(c["q"], c["s"], c["w"], c["t"], c["b"])
    plain = o.i8_product(c["q"], c["s"], c["w"], c["t"], None)
    off = 4 * 2.0 ** -24 * (np.abs(plain) + (0.0 if c["b"] is None else np.abs(c["b"].astype(np.float64))))
    h, N = HALF[c["dtype"]], c["N"]
    if not gated:
        close(got, P, off + h * (np.abs(P) + off), "Y")
        return got
    G, U = P[:, :N], P[:, N:]
    value = np.abs(o.activation(G, act)[0])
    tol = np.abs(G) * ACT[c["dtype"]] * np.abs(U) + 1.2 * off[:, :N] * (np.abs(U) + off[:, N:]) + value * off[:, N:]
    close(got, o.gate_fwd(P, act), tol + h * (value * np.abs(U) + tol), "H")
    return got


SIZES = [(1, 1, 1), (1, 64, 16), (1, 4096, 72), (2, 17, 5), (16, 256, 1000), (31, 130, 33), (32, 1040, 200), (33, 128, 64), (128, 64, 40), (129, 200, 136),
         (300, 520, 264), (257, 2064, 129), (1000, 96, 1288)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_product(size, dtype):
    c = make(*size, dtype, size[0], bias=size[0] % 2 == 1, full=size[0] == 300)
    assert torch.equal(check(c, False), check(c, False))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_gated_product(size, dtype):
    c = make(*size, dtype, 60 + size[0], gated=True, bias=size[0] % 2 == 1)
    for act in ACTS:
        check(c, True, act)


@pytest.mark.parametrize("columns,blocks", [(32, 1), (64, 1), (128, 1), (256, 1), (128, 2), (256, 2)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("size", [(9, 264, 333), (32, 1096, 200), (129, 520, 129), (700, 144, 640), (513, 1032, 1000)])
def test_every_tile_shape(size, gated, columns, blocks):
    M = size[0]
    if (columns == 32 and M > 128) or (blocks == 2 and M <= 128):
        return
    b.lrd_glu_tuning(columns, blocks)
    try:
        for dtype in ("bf16", "f32"):
            check(make(*size, dtype, 70 + M, gated=gated), gated)
    finally:
        b.lrd_glu_tuning()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("ldx,ldw,ldy,shift", [(96, 112, 72, 0), (83, 96, 67, 0), (96, 81, 65, 0), (81, 83, 65, 1), (0, 0, 0, 1)])
def test_strides(ldx, ldw, ldy, shift, gated):
    for M in (5, 150):
        for dtype in ("bf16", "f32"):
            check(make(M, 80, 64, dtype, 80 + M, gated=gated), gated, ldx=ldx, ldw=ldw, ldy=ldy, shift=shift)


def test_the_longest_sum():
    """131071 products of -128 x -128: the sum is 2^31 - 2^14, the largest a call can form."""
    K = 131071
    for sign in (1, -1):
        q, w = torch.full((2, K + 1), -128, dtype=torch.int8, device="cuda"), torch.full((3, K + 1), -128, dtype=torch.int8, device="cuda")
        if sign < 0:
            w.fill_(127)
        one = torch.ones(3, device="cuda")
        Y = torch.zeros(2, 3, device="cuda")
        b.lrd_i8_dense_fwd(b.i8_desc(2, K, 3, b.LRD_F32, ldx=K + 1, ldw=K + 1), q, one, w, one, None, Y, None)
        assert (Y == float(np.float32(K * 128 * (128 if sign > 0 else -127)))).all()


def test_no_tokens_and_rows_without_a_scale():
    d = b.i8_desc(0, 32, 8, b.LRD_F32)
    q, f = torch.zeros(16, 32, dtype=torch.int8, device="cuda"), torch.full((16, 8), 3.0, device="cuda")
    b.lrd_i8_quantize(f, 0, 0, 8, q, 0, f, b.LRD_F32)
    for call in (b.lrd_i8_dense_fwd, b.lrd_i8_glu_fwd):
        call(d, q, f, q, f, None, f, None)
    torch.cuda.synchronize()
    assert (f == 3.0).all()
    # a row that could not be quantized stays one without numbers, and the others are as they were
    X = wl.round_to(wl.normal(90, (40, 64)), "bf16")
    X[7, 3], X[20] = NAN, 0.0
    w, t = o.i8_quantize(wl.normal(91, (24, 64)))
    q, s = quantize(X, "bf16")
    Y = torch.zeros(40, 24, device="cuda")
    b.lrd_i8_dense_fwd(b.i8_desc(40, 64, 24, b.LRD_F32), q, s, bytes_padded(w, 64), torch.from_numpy(t).cuda(), None, Y, None)
    assert torch.isnan(Y[7]).all() and not Y[20].any() and torch.isfinite(Y[[i for i in range(40) if i != 7]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 24, 300])
def test_a_block_served(M, dtype):
    """A gated block in 8 bits from end to end (quantize, gated product, quantize, product), captured once and replayed on two inputs,
    each stage against the oracle fed with the stage's own input."""
    K, N, act = 144, 200, b.LRD_ACT_SILU
    tdt, code = DT[dtype][1], DT[dtype][0]
    W, Wd = wl.normal(100, (2 * N, K), K ** -0.5), wl.normal(101, (K, N), N ** -0.5)
    ldn = (N + 15) // 16 * 16
    up, down = torch.zeros(2 * N, K, dtype=torch.int8, device="cuda"), torch.zeros(K, ldn, dtype=torch.int8, device="cuda")
    tu, td = torch.zeros(2 * N, device="cuda"), torch.zeros(K, device="cuda")
    b.lrd_i8_quantize(torch.from_numpy(W).float().cuda(), 0, 2 * N, K, up, 0, tu, b.LRD_F32)
    b.lrd_i8_quantize(torch.from_numpy(Wd).float().cuda(), 0, K, N, down, ldn, td, b.LRD_F32)
    X, H, Y = (torch.zeros(M, n, dtype=tdt, device="cuda") for n in (K, N, K))
    q, s, qh, sh = (torch.zeros(M, K, dtype=torch.int8, device="cuda"), torch.zeros(M, device="cuda"), torch.zeros(M, ldn, dtype=torch.int8, device="cuda"),
                    torch.zeros(M, device="cuda"))
    d1, d2 = b.i8_desc(M, K, N, code, act), b.i8_desc(M, N, K, code, ldx=ldn, ldw=ldn)

    def step():
        b.lrd_i8_quantize(X, 0, M, K, q, 0, s, code)
        b.lrd_i8_glu_fwd(d1, q, s, up, tu, None, H, None)
        b.lrd_i8_quantize(H, 0, M, N, qh, ldn, sh, code)
        b.lrd_i8_dense_fwd(d2, qh, sh, down, td, None, Y, None)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (102, 103):
        Xh = wl.round_to(wl.normal(seed, (M, K)), dtype)
        X.copy_(dev(Xh, dtype))
        graph.replay()
        torch.cuda.synchronize()
        qr, sr = o.i8_quantize(Xh)
        assert np.array_equal(q.cpu().numpy(), qr) and np.array_equal(s.cpu().numpy(), sr)
        P = o.i8_product(qr, sr, up.cpu().numpy(), tu.cpu().numpy(), None)
        G, U = P[:, :N], P[:, N:]
        off = 4 * 2.0 ** -24 * np.abs(P)
        tol = np.abs(G) * ACT[dtype] * np.abs(U) + 1.2 * off[:, :N] * np.abs(U) + np.abs(G) * off[:, N:] + 1e-12
        close(H, o.gate_fwd(P, act), tol + HALF[dtype] * (np.abs(o.gate_fwd(P, act)) + tol), "H")
        qhr, shr = o.i8_quantize(host(H))
        assert np.array_equal(qh.cpu().numpy()[:, :N], qhr) and np.array_equal(sh.cpu().numpy(), shr)
        Yr = o.i8_product(qhr, shr, down.cpu().numpy()[:, :N], td.cpu().numpy(), None)
        close(Y, Yr, (4 * 2.0 ** -24 + HALF[dtype]) * (1 + 2.0 ** -20) * np.abs(Yr), "Y")
    # and the quantized block is the block: a step of 1 / 127 of a row's largest (some three deviations) is off by 0.7 % of a deviation
    # in the middle, twice in each of two products; the largest of M x K such sums stays within 5 % of the largest result
    full = o.gate_fwd(host(X) @ W.T, act) @ Wd.T
    assert np.abs(host(Y) - full).max() <= 0.05 * np.abs(full).max()


def test_a_decomposed_layer_served():
    """Both factors in 8 bits: Z = X V, quantized again, Y = Z U^T."""
    M, K, N, r = 70, 256, 176, 64
    c = wl.random_factor_case(M, K, N, r, "bf16", 110)
    new8 = lambda *s: torch.zeros(*s, dtype=torch.int8, device="cuda")
    Vq, Uq, tv, tu = new8(r, K), new8(N, r), torch.zeros(r, device="cuda"), torch.zeros(N, device="cuda")
    b.lrd_i8_quantize(dev(np.ascontiguousarray(c["V"].T), "bf16"), 0, r, K, Vq, 0, tv, b.LRD_BF16)
    b.lrd_i8_quantize(dev(c["U"], "bf16"), 0, N, r, Uq, 0, tu, b.LRD_BF16)
    q, s, qz, sz = new8(M, K), torch.zeros(M, device="cuda"), new8(M, r), torch.zeros(M, device="cuda")
    Z, Y = torch.zeros(M, r, device="cuda"), torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    b.lrd_i8_quantize(dev(c["X"], "bf16"), 0, M, K, q, 0, s, b.LRD_BF16)
    b.lrd_i8_dense_fwd(b.i8_desc(M, K, r, b.LRD_F32), q, s, Vq, tv, None, Z, None)
    b.lrd_i8_quantize(Z, 0, M, r, qz, 0, sz, b.LRD_F32)
    b.lrd_i8_dense_fwd(b.i8_desc(M, r, N, b.LRD_BF16), qz, sz, Uq, tu, dev(c["b"], "bf16"), Y, None)
    want = o.i8_product(qz.cpu().numpy(), sz.cpu().numpy(), Uq.cpu().numpy(), tu.cpu().numpy(), c["b"])
    close(Y, want, (4 * 2.0 ** -24 + 2.0 ** -8) * (np.abs(want) + np.abs(c["b"])), "Y")
    full = o.linear_fwd(c["X"], c["V"], c["U"], c["b"])[1]
    assert np.abs(host(Y) - full).max() <= 0.05 * np.abs(full).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 7, 8, 9])
def test_few_tokens(M, dtype):
    """Decoding: whole and ragged 16-byte pieces, rows of any stride."""
    for i, (K, N) in enumerate([(1, 1), (16, 7), (513, 33), (1024, 40), (4112, 65), (8195, 18)]):
        for gated in (False, True):
            c = make(M, K, N, dtype, 200 + 10 * M + i, gated=gated, bias=i % 2 == 0, full=True)
            check(c, gated, ldx=K + 15, ldw=K + 1, ldy=N + 3)
            check(c, gated, act=b.LRD_ACT_GELU, ldx=(K + 15) // 16 * 16, ldw=(K + 31) // 16 * 16)


def test_few_tokens_at_every_alignment():
    """Rows a few pieces long, off 16-byte boundaries: where the first and the last whole piece end, for each offset of X against W."""
    for K in list(range(17, 84)) + [997, 2053]:
        c = make(1 + K % 4, K, 9, "f32", 500 + K, gated=K % 2 == 0)
        for dx in range(0, 16, 3):
            check(c, K % 2 == 0, ldx=K + dx, ldw=K + (1 if K % 16 else 3))


@pytest.mark.parametrize("columns", [32, 64, 128, 256])
@pytest.mark.parametrize("split", [2, 4, 8])
@pytest.mark.parametrize("size", [(9, 2200, 333), (32, 4096, 200), (61, 1400, 136), (128, 2064, 264), (200, 3000, 129)])
def test_split_reductions(size, split, columns):
    M, K, N = size
    for gated in (False, True):
        b.lrd_glu_tuning(columns, 1, split)
        try:
            for dtype in ("bf16", "f32"):
                c = make(*size, dtype, 300 + M, gated=gated)
                check(c, gated, ldx=(K + 15) // 16 * 16, ldw=(K + 15) // 16 * 16)
        except b.LrdError as e:
            assert e.status == b.LRD_ERR_UNSUPPORTED and not split_fits(M, -(-K // 128), columns, split, gated)
        finally:
            b.lrd_glu_tuning()


def test_two_streams_at_once():
    """Calls whose blocks wait for one another (reductions shared by clusters, pairs of SMs) and others beside them, on two streams: each gets
    its own bits."""
    shapes = [(16, 4096, 256, True), (300, 2048, 512, False), (24, 8192, 160, False), (2, 1024, 300, True), (640, 512, 1024, True)]
    cases = [make(M, K, N, "bf16", 400 + i, gated=g) for i, (M, K, N, g) in enumerate(shapes)]
    alone = [run(c, g, ldx=c["K"], ldw=c["K"]).clone() for c, (_, _, _, g) in zip(cases, shapes)]
    sides = []
    for c, (M, K, N, g) in zip(cases, shapes):
        args = [b.i8_desc(M, K, N, b.LRD_BF16), bytes_padded(c["q"], K), torch.from_numpy(c["s"]).cuda(), bytes_padded(c["w"], K), torch.from_numpy(c["t"]).cuda(), dev(c["b"], "bf16")]
        sides.append((args, g, [torch.zeros(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for turn in range(20):
        for k, s in enumerate(streams):
            for i in range(len(sides)):
                args, g, out = sides[(i + 2 * k + turn) % len(sides)]
                (b.lrd_i8_glu_fwd if g else b.lrd_i8_dense_fwd)(*args, out[k], None, stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert b.lrd_check_device_status() == b.LRD_OK
    for (_, _, out), want in zip(sides, alone):
        assert torch.equal(out[0], want) and torch.equal(out[1], want)
