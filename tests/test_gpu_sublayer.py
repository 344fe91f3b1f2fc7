"""The attention sublayer workload: its operators run together, as one program uses them."""
import pytest
import torch

import paper_2608_02611_amd as kb
from synth import sublayer
from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
HEADS, KV, DIM = 4, 2, 16


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def given_of(dtype, length=33, wdtype=None):
    return sublayer.inputs(3, length, HEADS, KV, DIM, dtype, wdtype)


def exact(given, causal, lens):
    """The sublayer in 64 bits, with torch's own gradients."""
    x, w, b = (given[n].double().requires_grad_() for n in ("x", "w", "b"))
    c = x - x.mean(-1, keepdim=True)
    y = c / ((c * c).mean(-1, keepdim=True) + 1e-5).sqrt() * w + b
    q, k, v = sublayer.columns(y, HEADS, KV, DIM)
    loss, outs = 0.0, torch.zeros(given["do"].shape, dtype=torch.float64, device="cuda")
    for s in range(x.shape[0]):
        n = x.shape[1] if lens is None else int(lens[s])
        for h in range(HEADS):
            scores = (q[s, h, :n] @ k[s, h // (HEADS // KV), :n].T) * DIM ** -0.5
            if causal:
                scores = scores.masked_fill(torch.ones_like(scores, dtype=torch.bool).triu(1), float("-inf"))
            o = torch.softmax(scores, -1) @ v[s, h // (HEADS // KV), :n]
            outs[s, :n, h * DIM:(h + 1) * DIM] = o.detach()
            loss = loss + (o * given["do"][s, :n, h * DIM:(h + 1) * DIM].double()).sum()
    return (outs,) + torch.autograd.grad(loss, (x, w, b))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", [None, [33, 1, 20]])
def test_against_64_bits(causal, lens):
    """Tolerance: five sums in a row (rows of 128, scores of 16, keys of 33, queries of 66, rows of 99) are each off by
    at most n 2^-24 of the magnitudes that they add, which come to under ten times the largest result: in all under
    350 x 10 x 2^-24, 2.1e-4 of it."""
    given = given_of(torch.float32)
    lens_t = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = sublayer.reference(given, HEADS, KV, DIM, causal, lens_t)
    for name, a, want in zip(("o", "dx", "dw", "db"), got.outputs, exact(given, causal, lens)):
        off = float((a.double() - want).abs().max())
        assert off <= 2.1e-4 * float(want.abs().max()), (name, off)


@pytest.mark.parametrize("dtype,wdtype", [(torch.float16, None), (torch.bfloat16, torch.float32)])
def test_views_and_copies_agree(dtype, wdtype):
    """The columns of one buffer give the bits that dense tensors give, also on another stream."""
    given = given_of(dtype, 150, wdtype)
    got = sublayer.reference(given, HEADS, KV, DIM)
    y, mean, rstd = kb.kb_norm_forward(given["x"], given["w"], given["b"])
    q, k, v = (t.contiguous() for t in sublayer.columns(y, HEADS, KV, DIM))
    do = given["do"].unflatten(-1, (HEADS, DIM)).transpose(1, 2).contiguous()
    o, lse = kb.kb_attn_forward(q, k, v, causal=True)
    grads = kb.kb_attn_backward(do, q, k, v, o, lse, causal=True)
    dy = torch.cat([t.transpose(1, 2).flatten(2) for t in grads], -1)
    want = (o.transpose(1, 2).flatten(2),) + kb.kb_norm_backward(dy, given["x"], given["w"], mean, rstd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = sublayer.reference(given, HEADS, KV, DIM, stream=side)
    side.synchronize()
    assert torch.equal(got.lse, lse) and torch.equal(other.lse, lse)
    for a, c, d in zip(got.outputs, other.outputs, want):
        assert torch.equal(a, d) and torch.equal(c, d)


def test_candidates_are_screened():
    """Noise below the tolerance passes, noise of four times the tolerance fails in every output."""
    given = given_of(torch.bfloat16, 200, torch.float32)
    ref = sublayer.reference(given, HEADS, KV, DIM, lens=torch.tensor([200, 3, 77], dtype=torch.int32, device="cuda"))
    rows = sublayer.candidates(ref, [0.0, 2.0 ** -8, 2.0 ** -4])
    records, summary, passed = kb.screen_multi(ref.outputs, rows, 0.0, 2.0 ** -6)
    assert [bool(p) for p in passed] == [True, True, False]
    for out in records:
        assert out[0]["mismatches"] == 0 and out[1]["mismatches"] == 0 and out[2]["mismatches"] > 0
