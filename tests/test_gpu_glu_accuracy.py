"""Activations where their digits go: far tails, products that pass the type's range on the way.

Tolerances.  bf16: half a step of the result (2^-8) and 2^-11 for the approximations before it (exponential and reciprocal some 2^-20 in the
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


def gate_bwd(P, dH, dtype, act):
    M, N = dH.shape
    d = b.glu_desc(M, 0, N, DT[dtype][0], act)
    dP = torch.zeros(M, 2 * N, dtype=DT[dtype][1], device="cuda")
    b.lrd_gate_bwd(d, dev(dH, dtype), dev(P, dtype), dP)
    torch.cuda.synchronize()
    return host(dP)


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
