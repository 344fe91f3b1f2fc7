"""Softmax attention, forward and backward, against the formulas in 64 bits.

Tolerances, elementwise.  u is the unit roundoff of the storage type (2^-24,
2^-11, 2^-8), e = 2^-24, D the head dimension, n the terms of a sum.
  - A score is a binary32 sum of D products and is scaled, shifted and taken to
    a power in binary32: its term is off by a relative ES = (D + 16) e A, A the
    largest scaled sum of |q||k|, and 4 e for the power and the division.
  - A term is rounded to the storage type for its product: u.  A sum of n
    products in binary32 is off by at most n e of the sum of magnitudes.
  - dout . v is off by D e of the sum of magnitudes, and so is dout . o.
  - F16: t is held scaled so that its bound, 2 |dout| |v|, is at least 2^12: what
    it loses below the least normal number is under 2^-36 of that bound.
  - The result is rounded once: u of it, or the type's least subnormal."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def heads(b, h, n, d, dtype, seed, scale=1.0, layout="bhsd"):
    if layout == "bhsd":
        return normal((b, h, n, d), dtype, seed, scale)
    return normal((b, n, h, d), dtype, seed, scale).permute(0, 2, 1, 3)


def seen_of(nq, nk, causal):
    m = torch.ones((nq, nk), dtype=torch.bool, device="cuda")
    return m.tril(nk - nq) if causal else m


def close(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol) & ~(torch.isnan(want) & torch.isnan(got)) & ~(want == got)
    assert not bad.any(), "%s: %d of %d off, worst %.3g of the tolerance" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol)[bad].max()))


def check_forward(q, k, v, scale, causal, q_lens, k_lens, o, lse):
    u = U[q.dtype]
    grp = q.shape[1] // max(1, k.shape[1])
    D = q.shape[3]
    for b in range(q.shape[0]):
        nq = q.shape[2] if q_lens is None else min(max(int(q_lens[b]), 0), q.shape[2])
        nk = k.shape[2] if k_lens is None else min(max(int(k_lens[b]), 0), k.shape[2])
        assert torch.all(o[b, :, nq:] == 0) and torch.all(lse[b, :, nq:] == float("-inf"))
        if nq == 0:
            continue
        seen = seen_of(nq, nk, causal)
        for h in range(q.shape[1]):
            Q, K, V = q[b, h, :nq].double(), k[b, h // grp, :nk].double(), v[b, h // grp, :nk].double()
            s = torch.where(seen, (Q @ K.T) * scale, float("-inf"))
            want_lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), float("-inf"), device="cuda").double()
            p = torch.where(seen, torch.exp(s - want_lse[:, None]), 0.0)
            A = float((Q.abs() @ K.abs().T).max() * scale) if nk else 0.0
            es = (D + 16) * E * A + 4 * E
            mag = p @ V.abs()
            empty = want_lse == float("-inf")
            assert torch.all(o[b, h, :nq][empty] == 0) and torch.all(lse[b, h, :nq][empty] == float("-inf"))
            close(o[b, h, :nq], p @ V, (u + 2 * es + nk * E) * mag + 1.01 * u * (p @ V).abs() + TINY[q.dtype], "o")
            close(lse[b, h, :nq][~empty], want_lse[~empty], es + nk * E + 4 * E * want_lse[~empty].abs(), "lse")


def check_backward(do, q, k, v, o, lse, scale, causal, q_lens, k_lens, dq, dk, dv):
    u, tiny = U[q.dtype], TINY[q.dtype]
    grp = q.shape[1] // max(1, k.shape[1])
    D = q.shape[3]
    for b in range(q.shape[0]):
        nq = q.shape[2] if q_lens is None else min(max(int(q_lens[b]), 0), q.shape[2])
        nk = k.shape[2] if k_lens is None else min(max(int(k_lens[b]), 0), k.shape[2])
        assert torch.all(dq[b, :, nq:] == 0) and torch.all(dk[b, :, nk:] == 0) and torch.all(dv[b, :, nk:] == 0)
        seen = seen_of(nq, nk, causal)
        # F16: the bound of t over the key head's group
        for hk in range(k.shape[1]):
            K, V = k[b, hk, :nk].double(), v[b, hk, :nk].double()
            DO = do[b, hk * grp:(hk + 1) * grp, :nq].double()
            lost = 0.0
            if q.dtype == torch.float16 and nq and nk:
                lost = 2.0 ** -36 * 2 * float(DO.norm(dim=-1).max() * V.norm(dim=-1).max())
            wk, tk, wv, tv = (torch.zeros((nk, D), device="cuda").double() for _ in range(4))
            for r in range(grp):
                h = hk * grp + r
                Q, O, L = q[b, h, :nq].double(), o[b, h, :nq].double(), lse[b, h, :nq].double()
                s = (Q @ K.T) * scale
                p = torch.where(seen, torch.exp(s - torch.where(L == float("-inf"), 0.0, L)[:, None]), 0.0)
                p = torch.where((L == float("-inf"))[:, None], 0.0, p)
                A = float((Q.abs() @ K.abs().T).max() * scale) if nq and nk else 0.0
                top = float(L[torch.isfinite(L)].abs().max()) if torch.isfinite(L).any() else 0.0
                es = (D + 16) * E * A + 4 * E + 2 * E * top
                dp, dot = DO[r] @ V.T, (DO[r] * O).sum(1, keepdim=True)
                t = torch.where(seen, p * (dp - dot), 0.0)
                mag = torch.where(seen, p * (DO[r].abs() @ V.abs().T + (DO[r].abs() * O.abs()).sum(1, keepdim=True)), 0.0)
                et = (u + 2 * es) * t.abs() + D * E * mag + lost * seen
                n = E * nk
                close(dq[b, h, :nq], scale * (t @ K), scale * ((et + n * t.abs()) @ K.abs()) +
                      1.01 * u * scale * (t @ K).abs() + tiny, "dq")
                n = E * nq * grp
                wk += scale * (t.T @ Q)
                tk += scale * ((et + n * t.abs()).T @ Q.abs())
                wv += p.T @ DO[r]
                tv += (u + 2 * es + n) * (p.T @ DO[r].abs()) + (2.0 ** -34 if q.dtype == torch.float16 else 0.0) * \
                    DO[r].abs().sum(0)
            close(dk[b, hk, :nk], wk, tk + 1.01 * u * wk.abs() + tiny, "dk")
            close(dv[b, hk, :nk], wv, tv + 1.01 * u * wv.abs() + tiny, "dv")


def lens_tensor(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def check(dtype, b, h, hk, nq, nk, d, causal=False, layout="bhsd", q_lens=None, k_lens=None, seed=1, backward=True):
    t = DT[dtype]
    q, k = heads(b, h, nq, d, t, seed, 1.5, layout), heads(b, hk, nk, d, t, seed + 1, 1.0, layout)
    v, do = heads(b, hk, nk, d, t, seed + 2, 1.0, layout), heads(b, h, nq, d, t, seed + 3, 1.0, layout)
    scale = d ** -0.5
    ql, kl = lens_tensor(q_lens), lens_tensor(k_lens)
    o, lse = kb.kb_attn_forward(q, k, v, scale, causal, ql, kl)
    check_forward(q, k, v, scale, causal, q_lens, k_lens, o, lse)
    if backward:
        dq, dk, dv = kb.kb_attn_backward(do, q, k, v, o, lse, scale, causal, ql, kl)
        check_backward(do, q, k, v, o, lse, scale, causal, q_lens, k_lens, dq, dk, dv)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 2), (2, 1), (3, 31), (31, 32), (32, 33), (33, 64), (64, 65), (65, 63),
                                   (127, 128), (128, 129), (129, 127), (255, 257), (200, 17), (17, 200), (300, 300)])
def test_lengths(dtype, causal, nq, nk):
    check(dtype, 1, 2, 2, nq, nk, 64, causal)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [1, 3, 8, 15, 16, 32, 40, 63, 64, 65, 72, 80, 95, 96, 97, 100, 112, 127, 128])
def test_dimensions(dtype, d):
    check(dtype, 1, 2, 1, 70, 90, d, True, "bshd")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["bhsd", "bshd"])
@pytest.mark.parametrize("h,hk", [(1, 1), (3, 1), (8, 2), (12, 4), (6, 6), (32, 1)])
def test_shared_heads(dtype, layout, h, hk):
    check(dtype, 2, h, hk, 45, 77, 96, True, layout)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_ragged(dtype, causal, d):
    """Lengths of zero, of one, of all, and out of range (the nearer end); rows that see nothing."""
    check(dtype, 7, 4, 2, 130, 100, d, causal, "bshd", [130, 1, 0, 77, 128, 500, -3], [100, 100, 33, 0, 1, 64, 20])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("h,hk", [(4, 4), (8, 1), (16, 2), (40, 1)])
@pytest.mark.parametrize("nk", [1, 100, 1000, 5000])
def test_single_tokens(dtype, h, hk, nk):
    check(dtype, 3, h, hk, 1, nk, 128, True, "bshd", None, [nk, max(1, nk // 2), 1], backward=nk <= 1000)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(5, 3000), (64, 4100), (130, 9000)])
def test_pieces_of_a_prompt(dtype, nq, nk):
    check(dtype, 1, 8, 2, nq, nk, 128, True, "bshd", backward=False)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_long(dtype):
    check(dtype, 1, 2, 1, 1100, 1100, 128, True)
    check(dtype, 1, 1, 1, 1, 70000, 64, True, backward=False)
    check(dtype, 1, 2, 2, 2047, 513, 80, False)


def test_no_keys_and_no_queries():
    q, k = normal((2, 3, 5, 64), torch.float16, 1), normal((2, 3, 0, 64), torch.float16, 2)
    o, lse = kb.kb_attn_forward(q, k, k)
    assert torch.all(o == 0) and torch.all(lse == float("-inf"))
    dq, dk, dv = kb.kb_attn_backward(q, q, k, k, o, lse)
    assert torch.all(dq == 0) and dk.shape == (2, 3, 0, 64)
    k, q = normal((2, 3, 5, 64), torch.float16, 1), normal((2, 3, 0, 64), torch.float16, 2)
    o, lse = kb.kb_attn_forward(q, k, k)
    assert o.numel() == 0 and lse.shape == (2, 3, 0)
    dq, dk, dv = kb.kb_attn_backward(q, q, k, k, o, lse)
    assert dq.numel() == 0 and torch.all(dk == 0) and torch.all(dv == 0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_padding_holds_anything(dtype, bad):
    t = DT[dtype]
    ql, kl = lens_tensor([50, 1, 64]), lens_tensor([70, 33, 90])
    got = []
    for fill in (0.0, bad):
        q, k, v, do = (heads(3, 4 if s in (1, 4) else 2, 64 if s in (1, 4) else 90, 80, t, s) for s in (1, 2, 3, 4))
        for b in range(3):
            q[b, :, int(ql[b]):] = fill
            do[b, :, int(ql[b]):] = fill
            k[b, :, int(kl[b]):] = fill
            v[b, :, int(kl[b]):] = fill
        o, lse = kb.kb_attn_forward(q, k, v, None, True, ql, kl)
        o2 = o.clone()
        for b in range(3):
            o2[b, :, int(ql[b]):] = fill
        got.append((o, lse) + kb.kb_attn_backward(do, q, k, v, o2, lse, None, True, ql, kl))
    for a, c in zip(*got):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("at", [0, 5, 40, 63, 64, 100])
@pytest.mark.parametrize("which", ["q", "k", "v", "do"])
def test_non_finite_values_reach_who_sees_them(dtype, at, which):
    """A NaN at one position of a causal sequence: the queries before it, and the
    keys that only they see, keep their results."""
    t = DT[dtype]
    n, d = 130, 64
    x = dict(q=heads(1, 2, n, d, t, 1), k=heads(1, 1, n, d, t, 2), v=heads(1, 1, n, d, t, 3), do=heads(1, 2, n, d, t, 4))
    clean = {name: z.clone() for name, z in x.items()}
    x[which][:, :, at, 7] = float("nan")
    o, lse = kb.kb_attn_forward(x["q"], x["k"], x["v"], None, True)
    co, clse = kb.kb_attn_forward(clean["q"], clean["k"], clean["v"], None, True)
    tol = 16 * U[t]

    def same(a, c):
        assert torch.allclose(a.float(), c.float(), rtol=tol, atol=tol * 8), float((a.float() - c.float()).abs().max())
    if which == "q":
        rows = [i for i in range(n) if i != at]
        assert torch.isnan(o[:, :, at]).all() and torch.isnan(lse[:, :, at]).all()
    elif which == "do":
        rows = list(range(n))
    else:
        rows = list(range(at))
        hit = o[:, :, at:] if which == "k" else o[:, :, at:, 7]
        assert torch.isnan(hit).all()
    if rows:
        same(o[:, :, rows], co[:, :, rows])
        same(lse[:, :, rows], clse[:, :, rows])
    dq, dk, dv = kb.kb_attn_backward(x["do"], x["q"], x["k"], x["v"], o, lse, None, True)
    cq, ck, cv = kb.kb_attn_backward(clean["do"], clean["q"], clean["k"], clean["v"], co, clse, None, True)
    if which in ("k", "v"):
        if at:
            same(dq[:, :, :at], cq[:, :, :at])
        assert torch.isnan(dq[:, :, at:]).all()
    else:
        same(dq[:, :, [i for i in range(n) if i != at]], cq[:, :, [i for i in range(n) if i != at]])
        assert torch.isnan(dq[:, :, at]).all()
        # keys after the position are not seen by its query
        same(dk[:, :, at + 1:], ck[:, :, at + 1:])
        same(dv[:, :, at + 1:], cv[:, :, at + 1:])
        assert torch.isnan(dk[:, :, :at + 1]).all()


def test_scores_of_any_size():
    """Scores far beyond exp's range, equal scores, and scores of -infinity."""
    for t in DT.values():
        q, k, v = (heads(1, 2, 96, 64, t, s) for s in (1, 2, 3))
        o, lse = kb.kb_attn_forward(q * 60, k * 10, v, 1.0)
        assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
        s = (q * 60).double() @ (k * 10).double().transpose(2, 3)
        # a softmax this sharp picks the largest score (ties by the rounding of scores near 1e4 aside)
        gap = s.topk(2, -1).values
        clear = gap[..., 0] - gap[..., 1] > 40
        want = torch.gather(v.double(), 2, s.argmax(-1)[..., None].expand(-1, -1, -1, 64))
        assert torch.equal(o.double()[clear], want[clear])
        o, lse = kb.kb_attn_forward(torch.zeros_like(q), k, v, 1.0)
        mean = v.double().mean(2, keepdim=True)
        assert float((o.double() - mean).abs().max()) <= 2 * U[t] * float(v.abs().max())
        assert torch.allclose(lse, torch.full_like(lse, 96.0).log(), rtol=1e-6)
    q = torch.zeros((1, 1, 4, 64), device="cuda")
    k = torch.zeros((1, 1, 8, 64), device="cuda")
    q[..., 0] = 1.0
    k[0, 0, ::2, 0] = float("-inf")
    v = normal((1, 1, 8, 64), torch.float32, 5)
    o, lse = kb.kb_attn_forward(q, k, v, 1.0)
    assert torch.allclose(o[0, 0, 0], v[0, 0, 1::2].mean(0), atol=1e-6)
    k[..., 0] = float("-inf")
    o, lse = kb.kb_attn_forward(q, k, v, 1.0)
    assert torch.all(o == 0) and torch.all(lse == float("-inf"))


@pytest.mark.parametrize("size", [2.0 ** -12, 1.0, 2.0 ** 9])
def test_small_and_large_gradients_in_f16(size):
    """t under f16's normal range, and a bound of t past its largest number."""
    b, h, n, d = 1, 2, 600, 64
    q, k, v, do = (heads(b, h, n, d, torch.float16, s) for s in (1, 2, 3, 4))
    do, v = do * size, v * 8
    o, lse = kb.kb_attn_forward(q, k, v, 0.125, True)
    got = kb.kb_attn_backward(do, q, k, v, o, lse, 0.125, True)
    check_backward(do, q, k, v, o, lse, 0.125, True, None, None, *got)


def exact_loss(q, k, v, c, scale, causal):
    grp = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(grp, 1), v.repeat_interleave(grp, 1)
    s = torch.where(seen_of(q.shape[2], k.shape[2], causal), (q @ k.transpose(2, 3).contiguous()) * scale, float("-inf"))
    return ((torch.softmax(s, -1) @ v) * c).sum()


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("f16", 2e-2), ("bf16", 1e-1)])
def test_gradient_against_differences(dtype, tol):
    """Directional derivatives of S(o c) by central differences of the 64-bit formula.  tol: the gradient's terms are
    off by u each, at random over a few thousand of them; 16 u and a floor for the differences."""
    t = DT[dtype]
    q, k, v, c = heads(1, 4, 20, 40, t, 1), heads(1, 2, 33, 40, t, 2), heads(1, 2, 33, 40, t, 3), heads(1, 4, 20, 40, t, 4)
    o, lse = kb.kb_attn_forward(q, k, v, 0.2, True)
    grads = kb.kb_attn_backward(c, q, k, v, o, lse, 0.2, True)
    for i, grad in enumerate(grads):
        d = normal(grad.shape, torch.float32, 9 + i).double()
        ends = []
        for s in (1e-5, -1e-5):
            args = [x.double() for x in (q, k, v)]
            args[i] = args[i] + s * d
            ends.append(exact_loss(*args, c.double(), 0.2, True))
        diff = float((ends[0] - ends[1]) / 2e-5)
        assert abs(float((grad.double() * d).sum()) - diff) <= tol * (1 + abs(diff))


def test_strides_and_outputs_in_one_buffer():
    """q, k, v as columns of one projection, and their gradients as columns of another; nothing beside them is written."""
    b, n, h, hk, d = 2, 75, 4, 2, 72
    wide = h * d + 2 * hk * d + 5
    x = normal((b, n, wide), torch.bfloat16, 1)

    def views(t):
        cut = lambda a, heads: t[..., a:a + heads * d].unflatten(-1, (heads, d)).permute(0, 2, 1, 3)  # noqa: E731
        return cut(1, h), cut(1 + h * d, hk), cut(1 + (h + hk) * d, hk)
    q, k, v = views(x)
    out = torch.full((b, n, h * d + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    o = out[..., 2:2 + h * d].unflatten(-1, (h, d)).permute(0, 2, 1, 3)
    _, lse = kb.kb_attn_forward(q, k, v, None, True, o=o)
    want, want_lse = kb.kb_attn_forward(q.contiguous(), k.contiguous(), v.contiguous(), None, True)
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    assert torch.all(out[..., :2] == 7) and torch.all(out[..., -1] == 7)
    do = normal((b, h, n, d), torch.bfloat16, 2)
    grad = torch.full((b, n, wide), 7.0, dtype=torch.bfloat16, device="cuda")
    dq, dk, dv = views(grad)
    kb.kb_attn_backward(do, q, k, v, o, lse, None, True, dq=dq, dk=dk, dv=dv)
    dense = kb.kb_attn_backward(do, q.contiguous(), k.contiguous(), v.contiguous(), want, lse, None, True)
    for a, c in zip((dq, dk, dv), dense):
        assert torch.equal(a, c)
    assert torch.all(grad[..., 0] == 7) and torch.all(grad[..., -4:] == 7)


def test_broadcast_keys():
    """Keys and values of one sequence for the whole batch (stride 0)."""
    q = normal((3, 4, 20, 64), torch.float16, 1)
    k, v = normal((1, 2, 50, 64), torch.float16, 2), normal((1, 2, 50, 64), torch.float16, 3)
    a = kb.kb_attn_forward(q, k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1))
    c = kb.kb_attn_forward(q, k.repeat(3, 1, 1, 1), v.repeat(3, 1, 1, 1))
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


def test_wide_offsets():
    """Key rows whose offsets pass 2^31 elements and 2^32 bytes."""
    n, step = 300, 1 << 23
    buf = torch.empty(n * step + 64, dtype=torch.float16, device="cuda")
    k = buf.as_strided((1, 1, n, 64), (0, 0, step, 1))
    v = buf.as_strided((1, 1, n, 64), (0, 0, step, 1), 64)
    dense_k, dense_v = normal((1, 1, n, 64), torch.float16, 1), normal((1, 1, n, 64), torch.float16, 2)
    k.copy_(dense_k)
    v.copy_(dense_v)
    for nq in (1, 150):
        q, do = normal((1, 2, nq, 64), torch.float16, 3), normal((1, 2, nq, 64), torch.float16, 4)
        o, lse = kb.kb_attn_forward(q, k, v, None, True)
        co, clse = kb.kb_attn_forward(q, dense_k, dense_v, None, True)
        assert torch.equal(o, co) and torch.equal(lse, clse)
        for a, c in zip(kb.kb_attn_backward(do, q, k, v, o, lse, None, True),
                        kb.kb_attn_backward(do, q, dense_k, dense_v, o, lse, None, True)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("nq,nk", [(1, 6000), (200, 300)])
def test_repeats_streams_and_workspaces(nq, nk):
    """The same bits on every call, on another stream, and with a workspace that holds anything."""
    q, do = normal((2, 8, nq, 128), torch.float16, 1), normal((2, 8, nq, 128), torch.float16, 2)
    k, v = normal((2, 2, nk, 128), torch.float16, 3), normal((2, 2, nk, 128), torch.float16, 4)
    want = kb.kb_attn_forward(q, k, v, None, True)
    wantg = kb.kb_attn_backward(do, q, k, v, *want, None, True)
    fws = torch.full((max(16, kb.kb_attn_forward_workspace_bytes(q, k)),), 0xFF, dtype=torch.uint8, device="cuda")
    bws = torch.full((kb.kb_attn_backward_workspace_bytes(q, k),), 0xFF, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for stream in (None, None, side):
        if stream is not None:
            side.wait_stream(torch.cuda.current_stream())
        got = kb.kb_attn_forward(q, k, v, None, True, workspace=fws, stream=stream)
        gotg = kb.kb_attn_backward(do, q, k, v, *want, None, True, workspace=bws, stream=stream)
        torch.cuda.synchronize()
        for a, c in zip(got + gotg, want + wantg):
            assert torch.equal(a, c)
