"""Launches that start before the one in front of them has ended read what it wrote."""
import pytest
import torch

from paper_2309_03824_b200 import binding as b

pytestmark = pytest.mark.gpu


def normal(seed, *shape, std=1.0):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).mul_(std).to(torch.bfloat16)


def close(got, want, tol, name):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (name, float(err.max()), torch.nonzero(~(err <= tol))[:4].tolist())


@pytest.mark.parametrize("M", [1, 3, 17, 300])
def test_weights_written_by_the_launch_in_front(M):
    """Everything a product reads may come from the launch before it: rows quantized, weights quantized, then the product, many times over with
    other contents of the same buffers and nothing between the launches."""
    K, N = 512, 264
    X, W = [normal(20 + i, M, K) for i in range(4)], [normal(30 + i, N, K) for i in range(4)]
    new8 = lambda n: torch.zeros(n, K, dtype=torch.int8, device="cuda")
    q, w, s, t = new8(M), new8(N), torch.zeros(M, device="cuda"), torch.zeros(N, device="cuda")
    d = b.i8_desc(M, K, N, b.LRD_F32)
    Y = torch.zeros(80, M, N, device="cuda")
    for i in range(80):
        b.lrd_i8_quantize(X[i % 4], 0, M, K, q, 0, s, b.LRD_BF16)
        b.lrd_i8_quantize(W[i * 3 % 4], 0, N, K, w, 0, t, b.LRD_BF16)
        b.lrd_i8_dense_fwd(d, q, s, w, t, None, Y[i], None)
    torch.cuda.synchronize()
    want = {}
    for i in range(4):
        b.lrd_i8_quantize(X[i], 0, M, K, q, 0, s, b.LRD_BF16)
        b.lrd_i8_quantize(W[i * 3 % 4], 0, N, K, w, 0, t, b.LRD_BF16)
        torch.cuda.synchronize()
        sums = q.double() @ w.double().T
        off = sums.abs() * s.double()[:, None] * t.double()
        want[i] = (sums * s.double()[:, None] * t.double(), 4 * 2.0 ** -24 * off)
    for i in range(80):
        close(Y[i], *want[i % 4], i)
