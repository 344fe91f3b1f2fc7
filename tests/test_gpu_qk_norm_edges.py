"""Head norms: the views that the calls take."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_gpu_qk_norm import DT, EPS, check_backward, check_forward, freqs_of, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(0, 2), (3, 0), (3, 2)])
@pytest.mark.parametrize("lead", [(2, 5), (2, 1, 3), (2, 0), ()])
def test_leading_axes(dtype, heads, kv, lead):
    """Any number of axes before the heads, none of them, and no heads of one kind: the bits of [tokens][heads][dim]."""
    t, d, tokens = DT[dtype], 40, torch.Size(lead).numel()
    x = [normal((*lead, h, d), t, 1 + h) for h in (heads, kv, heads, kv)]
    w = normal((d,), t, 9)
    positions = torch.randint(0, 5000, lead, device="cuda", dtype=torch.int32)
    got = kb.kb_qk_norm_forward(*x[:2], w, w, EPS, positions, freqs_of(32))
    grads = kb.kb_qk_norm_backward(*x[2:], *x[:2], w, w, EPS, positions, freqs_of(32))
    flat = [v.reshape(tokens, v.shape[-2], d) for v in x]
    want = kb.kb_qk_norm_forward(*flat[:2], w, w, EPS, positions.reshape(tokens), freqs_of(32))
    want += kb.kb_qk_norm_backward(*flat[2:], *flat[:2], w, w, EPS, positions.reshape(tokens), freqs_of(32))
    for a, b in zip(got + grads, want):
        assert torch.equal(a.reshape(b.shape), b)
    assert [v.shape for v in got + grads[:2]] == [v.shape for v in x[:2]] * 2


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_heads_outside_a_sequence_at_a_time(dtype):
    """[batch][heads][len][dim], the layout of the dense attention: refused as a whole, one sequence at a time its values."""
    t, b, h, hk, n, d = DT[dtype], 3, 4, 2, 17, 64
    q, k = (normal((b, x, n, d), t, x).transpose(1, 2) for x in (h, hk))
    dq, dk = (torch.empty((b, x, n, d), dtype=t, device="cuda").transpose(1, 2) for x in (h, hk))
    args = (None, None, EPS)
    positions, freqs = torch.arange(n, device="cuda", dtype=torch.int32), freqs_of(64)
    with pytest.raises(ValueError, match="q: its axes"):
        kb.kb_qk_norm_forward(q, k, *args, positions.expand(b, n).contiguous(), freqs)
    with pytest.raises(ValueError, match="dq_out: its axes"):
        kb.kb_qk_norm_backward(q, k, q.contiguous(), k.contiguous(), *args, positions.expand(b, n).contiguous(), freqs)
    for i in range(b):
        yq, yk = kb.kb_qk_norm_forward(q[i], k[i], *args, positions, freqs)
        check_forward(q[i], *args[1:], positions, freqs, False, yq)
        check_forward(k[i], *args[1:], positions, freqs, False, yk)
        _, _, dwq, dwk = kb.kb_qk_norm_backward(yq, yk, q[i], k[i], *args, positions, freqs, dq=dq[i], dk=dk[i])
        check_backward(yq, q[i], *args[1:], positions, freqs, False, dq[i], dwq)
        check_backward(yk, k[i], *args[1:], positions, freqs, False, dk[i], dwk)
