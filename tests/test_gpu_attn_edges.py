"""Softmax attention where it can go wrong: heads without queries, wide strides,
long flat tails, large scores, and keys or queries in parts.  Against the formulas
in 64 bits with the tolerances of tests/test_gpu_attn.py, or those derived here."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_gpu_attn import DT, U, check, heads, normal

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


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [0.125, 0.09, 0.3])
@pytest.mark.parametrize("nq,nk", [(40, 200), (2, 3000)])
def test_scores_of_the_types_lowest_value(dtype, scale, nq, nk):
    """Keys that a column of the type's lowest number takes out of the softmax, first, in the middle and last: what is
    left is as if they were not there.  Where they are all that a row has, their scores are equal: o is the mean of v
    (a rounding of each term, which is exact, of the sum and of o), and gradients stay finite."""
    t = DT[dtype]
    q, k, v, do = heads(1, 4, nq, 64, t, 1), heads(1, 2, nk, 64, t, 2), heads(1, 2, nk, 64, t, 3), heads(1, 4, nq, 64, t, 4)
    q[..., 0], k[..., 0] = 1.0, 0.0
    out = torch.zeros(nk, dtype=torch.bool, device="cuda")
    out[:70], out[100:131], out[-5:] = True, True, True
    k[:, :, out, 0] = torch.finfo(t).min
    kept, vkept = k[:, :, ~out].contiguous(), v[:, :, ~out].contiguous()
    o, lse = kb.kb_attn_forward(q, k, v, scale)
    want, want_lse = kb.kb_attn_forward(q, kept, vkept, scale)
    u = U[t]

    def same(a, c, f):  # the same terms in other tiles: a rounding each, one of the result, 3000 of them summed in 32 bits
        tol = (4 * u + 2 * 3000 * 2.0 ** -24) * f
        assert float((a.double() - c.double()).abs().max()) <= tol, (float((a.double() - c.double()).abs().max()), tol)
    same(o, want, float(v.abs().max()))
    assert torch.allclose(lse, want_lse, rtol=1e-5, atol=1e-5)
    dq, dk, dv = kb.kb_attn_backward(do, q, k, v, o, lse, scale)
    _, dk1, dv1 = kb.kb_attn_backward(do, q, kept, vkept, o, lse, scale)
    assert torch.all(dv[:, :, out] == 0) and torch.all(dk[:, :, out] == 0)
    assert torch.allclose(dv[:, :, ~out].float(), dv1.float(), rtol=16 * u, atol=16 * u)
    assert torch.allclose(dk[:, :, ~out].float(), dk1.float(), rtol=16 * u, atol=16 * u)
    q[:, :2] = 0.0  # two of the heads, on the first key head, see nothing else
    q[:, :2, :, 0] = 1.0
    k[:, 0, :, 0] = torch.finfo(t).min
    o, lse = kb.kb_attn_forward(q, k, v, scale)
    mean = v[:, :1].double().mean(2, keepdim=True)
    assert float((o[:, :2].double() - mean).abs().max()) <= (u + nk * 2.0 ** -24) * float(v.abs().max())
    assert torch.isfinite(lse).all()
    for grad in kb.kb_attn_backward(do, q, k, v, o, lse, scale):
        assert torch.isfinite(grad.float()).all()


@pytest.mark.parametrize("dtype,big", [("f32", 2.0 ** 50), ("f16", 2.0 ** 15), ("bf16", 2.0 ** 15), ("bf16", 2.0 ** 50)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("nq,nk", [(100, 150), (3, 2500)])
def test_scores_that_binary32_holds_coarsely(dtype, big, causal, nq, nk):
    """Scores of up to 2^28 and 2^98 that differ by more than exp's range: o is the v of the largest one to the last
    bit, and what follows from lse stays finite."""
    t = DT[dtype]
    q, k, v, do = heads(1, 2, nq, 64, t, 1), heads(1, 1, nk, 64, t, 2), heads(1, 1, nk, 64, t, 3), heads(1, 2, nq, 64, t, 4)
    q[..., 1:], k[..., 1:] = 0.0, 0.0
    q[..., 0] = torch.sign(q[..., 0]) * big
    size = torch.randperm(nk, device="cuda") % 200 - 100
    size[nk // 8], size[nk // 8 + 1] = 250, -250  # (whole numbers that bf16 holds)
    k[..., 0] = size[None, None] * (big / 4096)
    o, lse = kb.kb_attn_forward(q, k, v, 0.3, causal)
    s = (q[..., :1].double() * k[..., 0].double()[:, :, None]) * 0.3
    if causal:
        s = torch.where(torch.ones((nq, nk), dtype=torch.bool, device="cuda").tril(nk - nq), s, float("-inf"))
    top, at = s.max(-1)
    gap = top - s.scatter(-1, at[..., None], float("-inf")).max(-1).values
    clear = gap > 200
    assert clear.all()
    want = torch.gather(v.expand(1, 2, nk, 64), 2, at[..., None].expand(-1, -1, -1, 64))
    assert torch.equal(o[clear], want[clear])
    assert float(((lse.double() - top).abs() / top.abs())[clear].max()) <= 2.0 ** -22
    for grad in kb.kb_attn_backward(do, q * 0 + 1, k / big, v, o, lse, 0.3, causal):
        assert torch.isfinite(grad.float()).all()


def test_large_scores_in_f32():
    """Gradients where lse is far from 0 and the scores are exact (one element of q is not 0): for one query with
    dout = 1, dv is p = exp(s - lse).  The difference is rounded once (2^-24 of up to 20), brought to base 2 (twice
    2^-24 of it) and taken to a power (2^-22 or so): 3 x 20 x 2^-24 + 2^-22 = 3.9e-6."""
    n, d = 300, 64
    q, k = torch.zeros((1, 2, 1, d), device="cuda"), torch.zeros((1, 2, n, d), device="cuda")
    q[..., 0] = 1.0
    k[..., 0] = 5000.0 + normal((1, 2, n), torch.float32, 1, 2.0)
    v, do = normal((1, 2, n, d), torch.float32, 2), torch.ones_like(q)
    o, lse = kb.kb_attn_forward(q, k, v, 1.0)
    _, _, dv = kb.kb_attn_backward(do, q, k, v, o, lse, 1.0)
    want = (k[..., :1].double() - lse.double()[..., None]).exp()
    assert float(((dv.double() - want).abs() / want).max()) <= 3.9e-6


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [61, 97, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_parts_of_ragged_sequences(dtype, d, causal):
    """Keys in parts, with padded queries, sequences of no key and of one, and dimensions that are no multiple of 4."""
    nq, nk = 6, 2500
    q, k = (torch.empty(s, dtype=DT[dtype], device="cuda") for s in ((5, 4, nq, d), (5, 2, nk, d)))
    assert kb.kb_attn_forward_workspace_bytes(q, k) > 0
    check(dtype, 5, 4, 2, nq, nk, d, causal, "bshd", [6, 3, 1, 0, 5], [2500, 0, 1, 2000, 1300])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [61, 72])
def test_parts_of_queries_and_keys_backward(dtype, d):
    """dq, dk and dv in parts at odd dimensions."""
    check(dtype, 1, 2, 1, 700, 900, d, True, "bshd")
    check(dtype, 2, 2, 2, 600, 40, d, False, "bhsd", [600, 1], [3, 40])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq,nk,d", [(4, 2100, 64), (1, 3000, 128), (130, 400, 80)])
def test_rows_at_odd_addresses(dtype, nq, nk, d):
    """Views that start one element into a wider buffer give the bits of dense ones."""
    t = DT[dtype]

    def odd(x):
        wide = torch.full((*x.shape[:-1], x.shape[-1] + 3), 9.0, dtype=t, device="cuda")
        view = wide[..., 1:1 + x.shape[-1]]
        return view.copy_(x)
    q, k, v, do = heads(2, 4, nq, d, t, 1), heads(2, 2, nk, d, t, 2), heads(2, 2, nk, d, t, 3), heads(2, 4, nq, d, t, 4)
    want = kb.kb_attn_forward(q, k, v, causal=True)
    got = kb.kb_attn_forward(odd(q), odd(k), odd(v), causal=True, o=odd(torch.zeros_like(q)))
    wantg = kb.kb_attn_backward(do, q, k, v, *want, causal=True)
    gotg = kb.kb_attn_backward(odd(do), odd(q), odd(k), odd(v), odd(want[0]), want[1], causal=True)
    for a, c in zip(got + gotg, want + wantg):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [3, 1500, 2995, 2999])
def test_non_finite_values_in_one_part(dtype, bad, at):
    """A value row that is not finite, in keys that pass in parts, reaches one column of the queries that see it; a NaN
    key makes its queries NaN; the others keep their results (the same terms, maybe in another order: 16 u)."""
    t = DT[dtype]
    nq, nk, d = 8, 3000, 64
    q, k, v = heads(1, 4, nq, d, t, 1, 0.5), heads(1, 2, nk, d, t, 2), heads(1, 2, nk, d, t, 3)
    assert kb.kb_attn_forward_workspace_bytes(q, k) > 0
    clean, clean_lse = kb.kb_attn_forward(q, k, v, causal=True)
    tol = 16 * U[t]

    def same(a, c):
        assert torch.allclose(a.float(), c.float(), rtol=tol, atol=tol), float((a.float() - c.float()).abs().max())
    v[:, :, at, 7] = bad
    o, lse = kb.kb_attn_forward(q, k, v, causal=True)
    seen = torch.arange(nq, device="cuda") + nk - nq >= at
    other = [c for c in range(d) if c != 7]
    same(lse, clean_lse)
    same(o[..., other], clean[..., other])
    same(o[:, :, ~seen], clean[:, :, ~seen])
    assert not torch.isfinite(o[:, :, seen][..., 7].float()).any()
    if bad != bad:
        k[:, :, at, 2] = bad
        o, lse = kb.kb_attn_forward(q, k, v, causal=True)
        assert torch.isnan(o[:, :, seen]).all() and torch.isnan(lse[:, :, seen]).all()
        same(o[:, :, ~seen], clean[:, :, ~seen])
        same(lse[:, :, ~seen], clean_lse[:, :, ~seen])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_scores_of_minus_infinity_in_parts(dtype):
    """Scores of -infinity over whole parts of the keys, and over all of them."""
    t = DT[dtype]
    nq, nk, d = 3, 4000, 64
    q, k, v = heads(1, 2, nq, d, t, 1, 0.5), heads(1, 2, nk, d, t, 2), heads(1, 2, nk, d, t, 3)
    q[..., 0] = 1.0
    k[:, :, :1700, 0] = float("-inf")
    o, lse = kb.kb_attn_forward(q, k, v)
    want, want_lse = kb.kb_attn_forward(q, k[:, :, 1700:].contiguous(), v[:, :, 1700:].contiguous())
    # the same terms in other tiles: a rounding each and one of the result on either side, 2300 of them summed in 32 bits
    tol = 4 * U[t] + 2 * 2300 * 2.0 ** -24
    assert float((o.double() - want.double()).abs().max()) <= tol * float(v.abs().max())
    assert torch.allclose(lse, want_lse, rtol=1e-5, atol=1e-5)
    k[..., 0] = float("-inf")
    o, lse = kb.kb_attn_forward(q, k, v)
    assert torch.all(o == 0) and torch.all(lse == float("-inf"))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("at", [0, 300, 699])
@pytest.mark.parametrize("which", ["q", "k", "v", "do"])
def test_non_finite_values_backward_in_parts(dtype, at, which):
    """A NaN at one position of a causal sequence whose queries and keys pass in parts: gradients that it does not reach
    keep their values (the same terms, maybe in another order: 16 u)."""
    t = DT[dtype]
    n, d = 700, 64
    x = dict(q=heads(1, 2, n, d, t, 1), k=heads(1, 1, n, d, t, 2), v=heads(1, 1, n, d, t, 3), do=heads(1, 2, n, d, t, 4))
    o, lse = kb.kb_attn_forward(x["q"], x["k"], x["v"], causal=True)
    clean = kb.kb_attn_backward(x["do"], x["q"], x["k"], x["v"], o, lse, causal=True)
    x[which][:, :, at, 7] = float("nan")
    o, lse = kb.kb_attn_forward(x["q"], x["k"], x["v"], causal=True)
    dq, dk, dv = kb.kb_attn_backward(x["do"], x["q"], x["k"], x["v"], o, lse, causal=True)
    tol = 16 * U[t]

    def same(a, c):
        assert torch.allclose(a.float(), c.float(), rtol=tol, atol=8 * tol), float((a.float() - c.float()).abs().max())
    if which in ("k", "v"):
        same(dq[:, :, :at], clean[0][:, :, :at])
        assert torch.isnan(dq[:, :, at:]).all()
    else:
        others = [i for i in range(n) if i != at]
        same(dq[:, :, others], clean[0][:, :, others])
        assert torch.isnan(dq[:, :, at]).all() and torch.isnan(dk[:, :, :at + 1]).all()
        same(dk[:, :, at + 1:], clean[1][:, :, at + 1:])
        same(dv[:, :, at + 1:], clean[2][:, :, at + 1:])
