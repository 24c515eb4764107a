"""8-bit gated products whose reduction is shared by the blocks of a cluster, at numbers of rows that fill no whole warp, against products in
64 bits on the device."""
import pytest
import torch

from paper_2309_03824_b200 import binding as b

pytestmark = pytest.mark.gpu


def silu(x):
    s = torch.sigmoid(x)
    return x * s, s * (1 + x * torch.sigmoid(-x))


def close(got, want, tol, name):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (name, float(err.max()), torch.nonzero(~(err <= tol))[:4].tolist())


@pytest.mark.parametrize("M", list(range(5, 33, 3)) + [33, 47, 63, 65, 97, 127])
def test_shared_reductions_of_every_number_of_rows(M):
    """Calls of few tokens over a long reduction, as they are dispatched and shared by two and four blocks: rows that fill no whole warp."""
    K, N = 4096, 264
    g = torch.Generator(device="cuda").manual_seed(M)
    q, w = (torch.randint(-127, 128, (n, K), dtype=torch.int8, device="cuda", generator=g) for n in (M, 2 * N))
    s, t = torch.rand(M, device="cuda", generator=g) / 127, torch.rand(2 * N, device="cuda", generator=g) / 127 / K ** 0.5
    P = (q.double() @ w.double().T) * s.double()[:, None] * t.double()
    off = 4 * 2.0 ** -24 * P.abs()
    for form in ((0, 0, 0), (64, 1, 2), (64, 1, 4), (128, 1, 4)):
        Y = torch.full((M + 2, N), 3.0, device="cuda")
        b.lrd_glu_tuning(*form)
        try:
            b.lrd_i8_glu_fwd(b.i8_desc(M, K, N, b.LRD_F32), q, s, w, t, None, Y, None)
        finally:
            b.lrd_glu_tuning()
        G, U = P[:, :N], P[:, N:]
        value = silu(G)[0]
        tol = (G * U).abs() * 2.0 ** -20 + 1.2 * off[:, :N] * (U.abs() + off[:, N:]) + value.abs() * off[:, N:]
        close(Y[:M], value * U, tol + 2.0 ** -24 * ((value * U).abs() + tol), form)
        assert (Y[M:] == 3.0).all()
