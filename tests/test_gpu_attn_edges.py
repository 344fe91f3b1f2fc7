"""Softmax attention where it can go wrong: heads without queries, wide strides,
long flat tails, large scores, and keys in parts.  Against the formulas in 64
bits with the tolerances of tests/test_gpu_attn.py, or those derived here."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_gpu_attn import DT, heads, normal

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


@pytest.mark.parametrize("dtype,d", [("f16", 128), ("f16", 40), ("bf16", 80), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("step", [(1 << 24) + (1 << 20), (1 << 25) - 16, 1 << 25])
def test_value_rows_far_apart(dtype, d, step):
    """Blocks of 128 value rows that are longer than the 2^31 bytes which one buffer descriptor reaches: strides of just
    over 2^31 / 128 bytes, of the largest that 64 rows allow, and of more.  As dense ones, to the bit."""
    t = DT[dtype]
    n, nq, elements = 130, 140, step // torch.finfo(t).bits * 8
    buf = torch.empty(n * elements, dtype=t, device="cuda")
    v = buf.as_strided((1, 1, n, d), (0, 0, elements, 1))
    k = buf.as_strided((1, 1, n, d), (0, 0, elements, 1), 1024)
    dense_k, dense_v = normal((1, 1, n, d), t, 1), normal((1, 1, n, d), t, 2)
    k.copy_(dense_k)
    v.copy_(dense_v)
    q, do = normal((1, 2, nq, d), t, 3), normal((1, 2, nq, d), t, 4)
    want = kb.kb_attn_forward(q, dense_k, dense_v, causal=True)
    got = kb.kb_attn_forward(q, k, v, causal=True)
    got += kb.kb_attn_backward(do, q, k, v, *want, causal=True)
    want += kb.kb_attn_backward(do, q, dense_k, dense_v, *want, causal=True)
    for a, c in zip(got, want):
        assert torch.equal(a, c)


@pytest.mark.parametrize("apart", [16.0, 17.4])
def test_long_flat_tails_in_f16(apart):
    """One score above 2^17 equal ones, whose terms (2^-23 and 2^-25.1 of it) count together.  A term is rounded to
    within 2^-11 of itself or, below f16's normal numbers, 2^-34 of the largest; a sum of 2^17 in 32 bits is off by at
    most 2^17 2^-24 of it; the result is rounded once.  66,000 rows: the keys are not in parts."""
    n, rows, d = 1 << 17, 66000, 64
    q, k = torch.zeros((1, 1, rows, d), device="cuda").half(), torch.zeros((1, 1, n, d), device="cuda").half()
    q[..., 0], k[:, :, 5, 0] = 1.0, apart
    v = torch.ones_like(k)
    v[:, :, 5] = 0.0
    o, _ = kb.kb_attn_forward(q, k, v, 1.0)
    assert kb.kb_attn_forward_workspace_bytes(q, k) == 0
    top = k[0, 0, 5, 0].double().exp().item()
    want = (n - 1) / (top + n - 1)
    err = float((o.double() - want).abs().max())
    assert err <= want * (2.0 ** -11 + 2.0 ** -11 + 2.0 ** -7) + n * 2.0 ** -34, (err, want)
