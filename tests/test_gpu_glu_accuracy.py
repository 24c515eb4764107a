"""Activations where their digits go: products that pass the type's range on the way."""
import numpy as np
import pytest
import torch

from paper_2309_03824_b200 import binding as b
from paper_2309_03824_b200 import workloads as wl

from helpers import DT, dev, host, workspace

pytestmark = pytest.mark.gpu


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
