"""What the gated block's and the 8-bit products' entry points refuse, before they look for a device (CPU)."""
import pytest
import torch

from paper_2309_03824_b200 import binding as b

T = torch.zeros(4096, dtype=torch.bfloat16)
F = torch.zeros(4096)
Q = torch.zeros(4096, dtype=torch.int8)
ODD = torch.zeros(4097, dtype=torch.uint8)[1:]           # off every element's boundary
WS = torch.zeros(1 << 20, dtype=torch.uint8)
WS = WS[(-WS.data_ptr()) % 256:]
BIG = (1 << 31) - 512


def fwd(d, X=T, W=T, bias=None, H=T, P=None, ws=WS):
    return b.lrd_dense_glu_fwd(d, X, W, bias, H, P, ws, stream=0, check=False)


def bwd(d, dH=T, X=T, W=T, P=T, dX=T, dW=T, db=None, ws=WS):
    return b.lrd_dense_glu_bwd(d, dH, X, W, P, dX, dW, db, ws, stream=0, check=False)


def i8(d, Xq=Q, xs=F, Wq=Q, w=F, bias=None, Y=F, ws=WS, call=b.lrd_i8_dense_fwd):
    return call(d, Xq, xs, Wq, w, bias, Y, ws, stream=0, check=False)


def good(**more):
    return b.glu_desc(**{**dict(M=4, K=16, N=8, dtype=b.LRD_BF16), **more})


def good8(**more):
    return b.i8_desc(**{**dict(M=4, K=16, N=8, dtype=b.LRD_F32), **more})


@pytest.mark.parametrize("more", [dict(M=-1), dict(K=0), dict(N=0), dict(dtype=2), dict(act=3), dict(act=-1), dict(ldx=15), dict(ldw=15), dict(ldh=7), dict(ldp=15)])
def test_bad_descriptors(more):
    d = good(**more)
    assert fwd(d) == bwd(d) == b.LRD_ERR_INVALID_ARG
    assert b.lrd_glu_workspace_bytes(d, 0) == b.lrd_glu_workspace_bytes(d, 1) == 0
    with pytest.raises(b.LrdError):
        b.lrd_dense_glu_fwd(d, T, T, None, T, None, WS, stream=0)
    if not set(more) & {"K", "ldx", "ldw"}:              # the gate does not look at those
        assert b.lrd_gate_fwd(d, T, T, stream=0, check=False) == b.lrd_gate_bwd(d, T, T, T, stream=0, check=False) == b.LRD_ERR_INVALID_ARG


@pytest.mark.parametrize("more", [dict(M=BIG), dict(K=BIG, ldx=BIG, ldw=BIG), dict(N=BIG // 2)])
def test_sizes_past_the_limit(more):
    assert fwd(good(**more)) == bwd(good(**more)) == b.LRD_ERR_TOO_LARGE


def test_missing_and_misplaced_pointers():
    d = good()
    for name in ("X", "W", "H"):
        assert fwd(d, **{name: None}) == b.LRD_ERR_INVALID_ARG
        assert fwd(d, **{name: ODD}) == b.LRD_ERR_ALIGNMENT
    assert fwd(d, bias=ODD) == fwd(d, P=ODD) == b.LRD_ERR_ALIGNMENT
    for name in ("dH", "X", "W", "P", "dW"):
        assert bwd(d, **{name: None}) == b.LRD_ERR_INVALID_ARG
        assert bwd(d, **{name: ODD}) == b.LRD_ERR_ALIGNMENT
    assert bwd(d, dX=ODD) == bwd(d, db=ODD) == b.LRD_ERR_ALIGNMENT
    assert b.lrd_gate_fwd(d, None, T, stream=0, check=False) == b.lrd_gate_fwd(d, T, None, stream=0, check=False) == b.LRD_ERR_INVALID_ARG
    assert b.lrd_gate_bwd(d, None, T, T, stream=0, check=False) == b.lrd_gate_bwd(d, T, T, None, stream=0, check=False) == b.LRD_ERR_INVALID_ARG
    assert b.lrd_gate_fwd(d, ODD, T, stream=0, check=False) == b.lrd_gate_bwd(d, ODD, T, T, stream=0, check=False) == b.LRD_ERR_ALIGNMENT


def test_workspaces():
    d = good()
    assert bwd(d, ws=None) == bwd(d, ws=WS[:128]) == b.LRD_ERR_WORKSPACE
    assert bwd(d, ws=WS[64:]) == b.LRD_ERR_ALIGNMENT
    odd = good(M=40, K=17)                               # rows that are repacked: the forward reads the workspace too
    assert b.lrd_glu_workspace_bytes(odd, 0) >= (40 + 16) * 24 * 2
    assert fwd(odd, ws=None) == fwd(odd, ws=WS[:256]) == b.LRD_ERR_WORKSPACE
    d8 = good8(M=40, K=17)
    assert b.lrd_i8_workspace_bytes(d8, 0) >= (40 + 8) * 32 and b.lrd_i8_workspace_bytes(d8, 1) >= (40 + 16) * 32
    assert i8(d8, ws=None) == i8(d8, ws=WS[:256], call=b.lrd_i8_glu_fwd) == b.LRD_ERR_WORKSPACE


@pytest.mark.parametrize("call", [b.lrd_i8_dense_fwd, b.lrd_i8_glu_fwd])
def test_8_bit_products(call):
    for more in (dict(M=-1), dict(K=0), dict(N=0), dict(dtype=5), dict(ldx=8), dict(ldw=8), dict(ldy=7)):
        assert i8(good8(**more), call=call) == b.LRD_ERR_INVALID_ARG
        assert b.lrd_i8_workspace_bytes(good8(**more), 0) == 0
    for name in ("Xq", "xs", "Wq", "w", "Y"):
        assert i8(good8(), call=call, **{name: None}) == b.LRD_ERR_INVALID_ARG
        assert i8(good8(), call=call, **{name: ODD}) == b.LRD_ERR_ALIGNMENT
    assert i8(good8(), bias=ODD, call=call) == b.LRD_ERR_ALIGNMENT
    for name in ("Xq", "Wq"):
        assert i8(good8(), call=call, **{name: Q[8:]}) == b.LRD_ERR_ALIGNMENT        # on no 16-byte boundary
    # a longer sum of products of -128 could pass 32 bits
    assert 131071 * 128 * 128 < 2 ** 31 <= 131072 * 128 * 128
    assert i8(good8(K=131072), call=call) == i8(good8(M=BIG), call=call) == i8(good8(N=BIG // 2), call=call) == b.LRD_ERR_TOO_LARGE


def test_activation_is_read_by_the_gated_product_alone():
    assert b.lrd_i8_workspace_bytes(good8(act=9), 0) > 0 and b.lrd_i8_workspace_bytes(good8(act=9), 1) == 0
    assert i8(good8(act=9), call=b.lrd_i8_glu_fwd) == b.LRD_ERR_INVALID_ARG


def test_quantizing():
    call = lambda X=F, ldx=0, M=4, K=8, Xq=Q, ldq=0, s=F, dt=b.LRD_F32: b.lrd_i8_quantize(X, ldx, M, K, Xq, ldq, s, dt, stream=0, check=False)
    for more in (dict(X=None), dict(Xq=None), dict(s=None), dict(M=-1), dict(K=0), dict(ldx=7), dict(ldq=7), dict(dt=2)):
        assert call(**more) == b.LRD_ERR_INVALID_ARG
    assert call(X=ODD) == call(s=ODD) == b.LRD_ERR_ALIGNMENT
    assert call(M=BIG) == b.LRD_ERR_TOO_LARGE


def test_launch_shapes_and_wrong_kinds():
    for bad in ((16, 0), (512, 1), (128, 3), (-1, 0), (128, 1, 3), (128, 1, 16), (128, 2, 2), (0, 1, 2), (128, 1, -1)):
        with pytest.raises(b.LrdError):
            b.lrd_glu_tuning(*bad)
    b.lrd_glu_tuning()
    with pytest.raises(TypeError):
        fwd(good8())
    with pytest.raises(TypeError):
        i8(good())
    with pytest.raises(AttributeError):
        fwd(good(), X=3)
