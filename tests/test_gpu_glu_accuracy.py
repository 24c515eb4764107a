"""Activations where their digits go: far tails, slopes next to 1, products that pass the type's range on the way.

Tolerances.  fp32: CUDA's expf is off by one last place (2^-23 of the value), the hardware's reciprocal by one, a sum or product by half.
With e = exp(-|z|), 1 / (1 + e) is then off by 4 and e / (1 + e) by 7 of 2^-24, beside what z's own roundings (7 of
2^-24 of z) make of e.  bf16: half a step of the result (2^-8) and 2^-11 for the approximations before it (exponential and reciprocal some 2^-20 in the
range used, the normal distribution's tail 2^-12)."""
import math

import numpy as np
import pytest
import torch

from oracle import lrd_oracle as o
from paper_2309_03824_b200 import binding as b
from paper_2309_03824_b200 import workloads as wl

from helpers import DT, dev, host, workspace

pytestmark = pytest.mark.gpu
SCALE, CUBIC = 2 * math.sqrt(2 / math.pi), 0.044715


def gate_bwd(P, dH, dtype, act):
    M, N = dH.shape
    d = b.glu_desc(M, 0, N, DT[dtype][0], act)
    dP = torch.zeros(M, 2 * N, dtype=DT[dtype][1], device="cuda")
    b.lrd_gate_bwd(d, dev(dH, dtype), dev(P, dtype), dP)
    torch.cuda.synchronize()
    return host(dP)


@pytest.mark.parametrize("act", [b.LRD_ACT_SILU, b.LRD_ACT_GELU_TANH])
@pytest.mark.parametrize("columns", [4096, 4099])
def test_slopes_keep_their_last_places(act, columns):
    """Slopes in fp32, relative to the terms they are the sum of: s and x s (1 - s) z', each positive or negative as a whole."""
    x = wl.round_to(np.concatenate([np.linspace(-25.0, 25.0, columns), wl.normal(1, (columns,))]).reshape(2, columns), "f32").astype(np.float64)
    P, one = np.concatenate([x, np.ones_like(x)], axis=1), np.ones_like(x)
    got = gate_bwd(P, one, "f32", act)[:, :columns]
    z, dz = (x, np.ones_like(x)) if act == b.LRD_ACT_SILU else (SCALE * (x + CUBIC * x ** 3), SCALE * (1 + 3 * CUBIC * x ** 2))
    e = np.exp(-np.abs(z))
    s, t = np.where(z >= 0, 1.0, e) / (1.0 + e), np.where(z >= 0, e, 1.0) / (1.0 + e)
    first, second = s, x * s * t * dz
    # units of 2^-24: s 7 and what it is multiplied and added with 3; the second term s 7, 1 - s 7, z' 5 and the products between them 4; z 7 in both
    tol = 2.0 ** -24 * (10 * np.abs(first) + 24 * np.abs(second))
    if act == b.LRD_ACT_GELU_TANH:
        tol = tol + 7 * 2.0 ** -24 * np.abs(z) * (s * t + np.abs(second))
    bad = ~(np.abs(got - (first + second)) <= tol + 1e-37)
    assert not bad.any(), (bad.sum(), x[bad][:4], got[bad][:4], (first + second)[bad][:4])


def through_the_block(G, U, act, dtype="bf16"):
    """act(G) * U by the product's own epilogue: X holds the numbers, W picks them out."""
    M, N = G.size, 16
    X, W = np.stack([G, U], axis=1), np.zeros((2 * N, 2), np.float32)
    W[:N, 0], W[N:, 1] = 1.0, 1.0
    pad = np.zeros((M, 6), np.float32)
    d = b.glu_desc(M, 8, N, DT[dtype][0], act)
    H = torch.zeros(M, N, dtype=DT[dtype][1], device="cuda")
    b.lrd_dense_glu_fwd(d, dev(np.concatenate([X, pad], axis=1), dtype), dev(np.concatenate([W, np.zeros((2 * N, 6))], axis=1), dtype), None, H, None,
                        workspace(b.lrd_glu_workspace_bytes(d, 0)))
    torch.cuda.synchronize()
    H = host(H)
    assert np.array_equal(H, np.repeat(H[:, :1], N, axis=1), equal_nan=True)
    return H[:, 0]


TAIL = wl.round_to(-np.concatenate([np.linspace(0.0, 12.0, 2001), np.linspace(4.0, 12.0, 999)]), "bf16").astype(np.float64)


@pytest.mark.parametrize("where", ["few tokens", "general", "tensor cores", "gate"])
def test_the_tail_of_gelu(where):
    """x Phi(x) down to -12 in bf16, relative to itself."""
    one = np.ones_like(TAIL)
    want, exact = o.activation(TAIL, o.ACT_GELU)
    if where == "gate":
        d = b.glu_desc(1, 0, TAIL.size, b.LRD_BF16, b.LRD_ACT_GELU)
        H = torch.zeros(1, TAIL.size, dtype=torch.bfloat16, device="cuda")
        b.lrd_gate_fwd(d, dev(np.concatenate([TAIL, one])[None], "bf16"), H)
        got = host(H)[0]
        slope = gate_bwd(np.concatenate([TAIL, one])[None], one[None], "bf16", b.LRD_ACT_GELU)[0]
        value, pdf = slope[TAIL.size:], np.exp(-TAIL ** 2 / 2) / math.sqrt(2 * math.pi)
        cdf = exact - TAIL * pdf
        assert (np.abs(value - want) <= (2.0 ** -8 + 2.0 ** -11) * np.abs(want)).all()
        assert (np.abs(slope[:TAIL.size] - exact) <= 2.0 ** -8 * np.abs(exact) + 2.0 ** -11 * (cdf + np.abs(TAIL) * pdf)).all()
    elif where == "few tokens":
        got = np.concatenate([through_the_block(TAIL[i:i + 4], one[i:i + 4], b.LRD_ACT_GELU) for i in range(0, TAIL.size, 300)])
        want = np.concatenate([want[i:i + 4] for i in range(0, TAIL.size, 300)])
    elif where == "general":
        b.lrd_set_path(b.LRD_PATH_GENERAL)
        try:
            got = through_the_block(TAIL, one, b.LRD_ACT_GELU)
        finally:
            b.lrd_set_path(b.LRD_PATH_AUTO)
    else:
        got = through_the_block(TAIL, one, b.LRD_ACT_GELU)
    bad = ~(np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -11) * np.abs(want))
    assert not bad.any(), (bad.sum(), np.stack([got, want], axis=1)[bad][:4])


@pytest.mark.parametrize("act", [b.LRD_ACT_SILU, b.LRD_ACT_GELU, b.LRD_ACT_GELU_TANH])
@pytest.mark.parametrize("M", [4, 400])
def test_a_vanishing_gate_before_a_huge_factor(M, act):
    """act(G) is taken before it meets U: far below zero it is nothing, whatever U is (G U alone would pass the type's range)."""
    G = np.resize(np.array([-200.0, -1000.0, -1e10, -150.0, -1e30]), M)
    U = wl.round_to(np.resize(np.array([1e38, -3e38, 2.5e38, 1e30, 3e38, 1e37, -1e38]), M), "bf16").astype(np.float64)
    got = through_the_block(G, U, act)
    assert not got.any(), got[:8]
    big = through_the_block(-G, U * 0 + 0.5, act)            # and the other end is G U
    assert (np.abs(big + 0.5 * wl.round_to(G, "bf16")) <= 2.0 ** -8 * np.abs(0.5 * G)).all()
