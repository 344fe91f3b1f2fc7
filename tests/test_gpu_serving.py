"""Head norms, cache writes and attention run together: the serving workload, and a training step over the head norms."""
import pytest
import torch

import paper_2608_02611_amd as kb
from synth import serving
from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
HEADS, KV, DIM = 4, 2, 32
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def normed(x, w, positions, freqs):
    """A head norm with the rotation, in the type of x (64 bits, with gradients)."""
    g = x / (x.pow(2).mean(-1, keepdim=True) + serving.EPS).sqrt() * w
    t = positions.double()[:, None, None] * freqs.double()
    a, b = g.chunk(2, -1)
    return torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin()], -1)


def attended(q, k, v):
    """Causal attention of one sequence [tokens][heads][dim], in 64 bits; the queries are the last tokens."""
    out = []
    for h in range(HEADS):
        s = (q[:, h] @ k[:, h // (HEADS // KV)].T) * DIM ** -0.5
        hidden = torch.ones_like(s, dtype=torch.bool).triu(1 + s.shape[1] - s.shape[0])
        out.append(torch.softmax(s.masked_fill(hidden, float("-inf")), -1) @ v[:, h // (HEADS // KV)])
    return torch.stack(out, 1)


@pytest.mark.parametrize("prompts", [[40, 7, 1], [1, 1, 1], [0, 33, 90]])
@pytest.mark.parametrize("page", [16, 5])
def test_prompts_and_tokens_against_64_bits(prompts, page):
    """Prompts, a piece of three tokens each, then single tokens; outputs against whole sequences in 64 bits.

    Tolerance (32 bits): an element of a normalised key or query of 32 is off by (32 + 14) E of its pair's magnitude, a
    score, of magnitudes of up to 32, by three times that, and so is its term; sums of up to 100 terms are off by 100 E,
    twice: in all under (3 x 46 x 32 + 200) E, 2.8e-4 of the largest output."""
    to = serving.cache(3, 100, page, KV, DIM, torch.float32)
    w, freqs = serving.weights(DIM, torch.float32), serving.frequencies(DIM)
    kept = [[] for _ in prompts]
    for n, new in enumerate([prompts, [3, 3, 3], [1, 1, 1], [1, 1, 1]]):
        x = serving.projected(sum(new), HEADS, KV, DIM, torch.float32, sub=n)
        o = serving.step(x, new, to, w, freqs, HEADS, KV, DIM)
        first = 0
        for b, m in enumerate(new):
            kept[b].append(x[first:first + m])
            whole = torch.cat(kept[b]).double()
            if m:
                q, k, v = serving.columns(whole, HEADS, KV, DIM)
                at = torch.arange(len(whole), device="cuda")
                q, k = (normed(t, weight.double(), at, freqs) for t, weight in zip((q, k), w))
                want = attended(q[-m:], k, v)
                off = float((o[first:first + m].double() - want).abs().max())
                assert off <= 2.8e-4 * float(want.abs().max()), (n, b, off)
            first += m
    assert to.counts == [p + 5 for p in prompts] and to.lens.tolist() == to.counts


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_the_cache_gives_what_whole_sequences_give(dtype):
    """A prompt over its pages has the bits of the attention over dense keys, and single tokens its values to the terms'
    rounding."""
    n = 300
    to = serving.cache(2, 320, 16, KV, DIM, dtype)
    w, freqs = serving.weights(DIM, dtype), serving.frequencies(DIM)
    x = serving.projected(2 * n, HEADS, KV, DIM, dtype)
    o = serving.step(x, [n, n], to, w, freqs, HEADS, KV, DIM)
    q, k, v = serving.columns(x, HEADS, KV, DIM)
    positions = torch.arange(n, dtype=torch.int32, device="cuda").repeat(2)
    q, k = kb.kb_qk_norm_forward(q, k, *w, serving.EPS, positions, freqs)

    def dense(t):
        return t.unflatten(0, (2, n)).transpose(1, 2)
    want, _ = kb.kb_attn_forward(dense(q), dense(k), dense(v), causal=True)
    assert torch.equal(o.unflatten(0, (2, n)).transpose(1, 2), want)
    token = serving.cache(2, 320, 16, KV, DIM, dtype)
    most = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    u = torch.finfo(dtype).eps / 2
    assert u == most
    for i in range(20):
        got = serving.step(x.view(2, n, -1)[:, i], [1, 1], token, w, freqs, HEADS, KV, DIM)
        # a term's rounding in the prompt, of it and of its sum, both results', and sums of up to 20 terms in 32 bits
        top = float(v.abs().max())
        assert float((got.double() - o.view(2, n, HEADS, DIM)[:, i].double()).abs().max()) <= (4 * u + 40 * E) * top


def test_candidates_are_screened():
    """Noise below the tolerance passes, noise of four times the tolerance fails in every output."""
    to = serving.cache(2, 64, 16, KV, DIM, torch.bfloat16)
    w, freqs = serving.weights(DIM, torch.bfloat16), serving.frequencies(DIM)
    refs = [serving.step(serving.projected(sum(new), HEADS, KV, DIM, torch.bfloat16, sub=n), new, to, w, freqs, HEADS, KV, DIM)
            for n, new in enumerate([[50, 9], [1, 1]])]
    records, _, passed = kb.screen_multi(refs, serving.candidates(refs, [0.0, 2.0 ** -8, 2.0 ** -4]), 0.0, 2.0 ** -6)
    assert [bool(p) for p in passed] == [True, True, False]
    for out in records:
        assert out[0]["mismatches"] == 0 and out[1]["mismatches"] == 0 and out[2]["mismatches"] > 0


def test_a_training_step_against_64_bits():
    """x -> head norms -> attention and back: dx of the projection's columns and the weights' gradients.

    Tolerance (32 bits): sums over 16 products, 40 keys, 80 queries of a group and 160 rows, each off by n E of the
    magnitudes, which come to under ten times the largest result, through a norm and back: under 4 x 300 x 10 E, 7.2e-4."""
    n = 40
    x = serving.projected(2 * n, HEADS, KV, DIM, torch.float32)
    w, freqs = serving.weights(DIM, torch.float32), serving.frequencies(DIM)
    do = serving.projected(2 * n, HEADS, 0, DIM, torch.float32, sub=9).unflatten(1, (HEADS, DIM))
    positions = torch.arange(n, dtype=torch.int32, device="cuda").repeat(2)
    args = (serving.EPS, positions, freqs)

    def dense(t):
        return t.unflatten(0, (2, n)).transpose(1, 2)
    q, k, v = serving.columns(x, HEADS, KV, DIM)
    qn, kn = kb.kb_qk_norm_forward(q, k, *w, *args)
    o, lse = kb.kb_attn_forward(dense(qn), dense(kn), dense(v), causal=True)
    dx = torch.empty_like(x)
    dq, dk, dv = serving.columns(dx, HEADS, KV, DIM)
    dqn, dkn = torch.empty_like(qn), torch.empty_like(kn)
    kb.kb_attn_backward(dense(do), dense(qn), dense(kn), dense(v), o, lse, causal=True, dq=dense(dqn), dk=dense(dkn),
                        dv=dense(dv))
    _, _, dwq, dwk = kb.kb_qk_norm_backward(dqn, dkn, q, k, *w, *args, dq=dq, dk=dk)

    leaf, wq, wk = (t.double().requires_grad_() for t in (x, *w))
    q, k, v = serving.columns(leaf, HEADS, KV, DIM)
    q, k = normed(q, wq, positions, freqs), normed(k, wk, positions, freqs)
    loss = sum((attended(q[s], k[s], v[s]) * do[s].double()).sum() for s in (slice(0, n), slice(n, 2 * n)))
    for name, got, want in zip(("dx", "dwq", "dwk"), (dx, dwq, dwk), torch.autograd.grad(loss, (leaf, wq, wk))):
        off = float((got.double() - want).abs().max())
        assert off <= 7.2e-4 * float(want.abs().max()), (name, off)


def test_the_workload_runs(capsys):
    serving.main()
    lines = [line for line in capsys.readouterr().out.splitlines() if line.startswith("candidate")]
    assert len(lines) == 4 and "passed" in lines[0] and "failed" in lines[3]
