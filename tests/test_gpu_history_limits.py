"""Operators that read a history in order where their arguments end: strides, lengths, grids and values at the edge of what a call takes.
Values against the plain 64-bit forms of history_ref with its bounds; a tighter bound is derived where it stands."""
import math

import pytest
import torch

import paper_1906_00091_amd as hot

import history_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(autouse=True)
def hand_memory_back():
    yield
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def far_apart(n, H, d, stride, dtype, tensors=1):
    """Views [n, H, d] whose items lie `stride` elements apart, the views' rows side by side; what lies between is not touched."""
    assert tensors * H * d <= stride
    pool = torch.empty((n - 1) * stride + tensors * H * d, dtype=dtype, device=DEV)
    return [pool[i * H * d:].as_strided((n, H, d), (stride, d, 1), i * H * d) for i in range(tensors)]


# ------------------------------------------------------------------------------------------------ strides
@pytest.mark.parametrize("dtype,d,stride,slopes", [("f32", 16, 1 << 23, False), ("f32", 64, (1 << 22) + 8, True), ("f16", 64, 1 << 23, False), ("f32", 72, 1 << 22, False)])
def test_keys_a_large_stride_apart(dtype, d, stride, slopes):
    """Few queries over some hundred keys whose rows lie up to the largest stride apart: every row that a tile takes is its own."""
    g, dt, nq, nk, H = gen(d), DT[dtype], 3, 520, 2
    q, do = (rand(g, nq, H, d, dtype=dt) for _ in range(2))
    k, v = (rand(g, nk, H, d, dtype=dt) for _ in range(2))
    K, V, DK, DV = far_apart(nk, H, d, stride, dt, 4)
    K.copy_(k)
    V.copy_(v)
    Q, DO, DQ, O = far_apart(nq, H, d, stride, dt, 4)
    Q.copy_(q)
    DO.copy_(do)
    qo, ko = torch.tensor([0, nq], device=DEV), torch.tensor([0, nk], device=DEV)
    sl = torch.tensor([0.01, 0.0]) if slopes else None
    seq = hot.SeqBatch(qo, ko, nq, nk, nq, nk, slopes=None if sl is None else sl.to(DEV))
    lse = torch.empty(H, nq, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, Q, K, V, O, lse)
    hot.dlrm_seq_attn_bwd(seq, Q, K, V, O, lse, DO, DQ, DK, DV, hot.alloc_seq_attn_workspace(seq, H, H, d))
    want = ref.attention(q, k, v, qo.cpu(), ko.cpu(), True, None, sl, d ** -0.5, 0.0, do)
    for n, x in (("out", O), ("lse", lse), ("dq", DQ), ("dk", DK), ("dv", DV)):
        ref.close(x, want[n], want[n + "_tol"], n)
