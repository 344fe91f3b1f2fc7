"""Softmax attention where it can go wrong: heads without queries, wide strides,
long flat tails, large scores, and keys in parts.  Against the formulas in 64
bits with the tolerances of tests/test_gpu_attn.py, or those derived here."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_gpu_attn import DT, heads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("nq,nk", [(7, 300), (0, 5)])
def test_no_query_heads(dtype, causal, nq, nk):
    """Sums over no query head: dk and dv are written, as zeros."""
    t = DT[dtype]
    q, k, v = heads(2, 0, nq, 72, t, 1), heads(2, 3, nk, 72, t, 2), heads(2, 3, nk, 72, t, 3)
    o, lse = kb.kb_attn_forward(q, k, v, causal=causal)
    assert o.shape == q.shape and lse.shape == q.shape[:3]
    dk, dv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    dq, _, _ = kb.kb_attn_backward(q, q, k, v, o, lse, causal=causal, dk=dk, dv=dv)
    assert dq.numel() == 0 and torch.all(dk == 0) and torch.all(dv == 0)
