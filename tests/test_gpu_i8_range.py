"""Results of 8-bit products next to the ends of fp32's range: a result that fp32 holds is found, however large or small its row's scale."""
import numpy as np
import pytest
import torch

from oracle import lrd_oracle as o
from paper_2309_03824_b200 import binding as b
from paper_2309_03824_b200 import workloads as wl

from helpers import DT, dev, workspace
from test_gpu_glu import HALF, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,columns,blocks,split", [(1, 0, 0, 0), (4, 0, 0, 0), (16, 0, 0, 0), (16, 64, 1, 2), (300, 0, 0, 0), (300, 256, 2, 0)])
def test_rows_of_any_size(M, columns, blocks, split, dtype):
    """Rows of 2^116 times ordinary activations (sum times row scale alone would pass 2^128) beside rows of 2^-100 times them; weights of ordinary size."""
    K, N = 1024, 72
    size = np.where(np.arange(M) % 2 == 0, 2.0 ** 116, 2.0 ** -100)[:, None]
    X = wl.round_to(np.abs(wl.normal(120, (M, K))) * size, dtype)
    W = np.abs(wl.normal(121, (N, K), K ** -0.5))
    q, s, w, t = (torch.zeros(M, K, dtype=torch.int8, device="cuda"), torch.zeros(M, device="cuda"), torch.zeros(N, K, dtype=torch.int8, device="cuda"), torch.zeros(N, device="cuda"))
    b.lrd_i8_quantize(dev(X, dtype), 0, M, K, q, 0, s, DT[dtype][0])
    b.lrd_i8_quantize(torch.from_numpy(W).float().cuda(), 0, N, K, w, 0, t, b.LRD_F32)
    Y = torch.zeros(M, N, dtype=DT[dtype][1], device="cuda")
    d = b.i8_desc(M, K, N, DT[dtype][0])
    b.lrd_glu_tuning(columns, blocks, split)
    try:
        b.lrd_i8_dense_fwd(d, q, s, w, t, None, Y, workspace(b.lrd_i8_workspace_bytes(d, 0)))
        torch.cuda.synchronize()
    finally:
        b.lrd_glu_tuning()
    want = o.i8_product(q.cpu().numpy(), s.cpu().numpy(), w.cpu().numpy(), t.cpu().numpy(), None)
    sums = (q.double() @ w.double().T).max().item()
    assert want.max() < 3e38 and sums * s.double().max().item() > 2.0 ** 128          # the results fit, the sums with their rows' scales alone do not
    close(Y, want, (4 * 2.0 ** -24 + HALF[dtype]) * np.abs(want), "Y")
