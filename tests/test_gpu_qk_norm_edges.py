"""Head norms: cosines and sines of the exact angles, and the views that the calls take."""
import numpy as np
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_gpu_qk_norm import DT, EPS, check_backward, check_forward, freqs_of, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def exact_turns(positions, freqs):
    """cos and sin of positions x freqs, from two products that binary64 holds exactly: of the position's upper 16 bits and
    of its lower ones, 16 and 24 bits each, added by the angles' formula (off by a few 2^-53)."""
    high, low = (positions >> 16).astype(np.float64) * 65536.0, (positions & 0xFFFF).astype(np.float64)
    a, b = (part[:, None] * freqs.astype(np.float64) for part in (high, low))
    return np.cos(a) * np.cos(b) - np.sin(a) * np.sin(b), np.sin(a) * np.cos(b) + np.cos(a) * np.sin(b)


@pytest.mark.parametrize("interleaved", [False, True])
def test_turns_of_far_positions(interleaved):
    """cos and sin within 2^-23 for angles of up to 2^50, and nothing else: a row of 16 pairs (1, 0), 16 ones and 8 twos has
    the mean square 1, so that its norm without eps is the row itself, and its pairs become (cos, sin) unrounded."""
    n, dim = 16, 64
    rng = np.random.default_rng(1)
    positions = rng.integers(-2 ** 31, 2 ** 31, 3000)
    positions[:1500] >>= rng.integers(0, 28, 1500)
    positions[:8] = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 1 << 20, 3]
    x = torch.zeros((3000, 1, dim), device="cuda")
    first = torch.arange(n, device="cuda") * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    x[..., first] = 1.0
    x[..., 2 * n:3 * n], x[..., 3 * n:3 * n + 8] = 1.0, 2.0
    to = torch.from_numpy(positions.astype(np.int32)).cuda()
    beside = 0.0
    for low, high in ((-26, 0), (0, 12), (12, 18.9), (18, 18.99)):
        freqs = np.exp2(rng.uniform(low, high, n)).astype(np.float32)
        y, _ = kb.kb_qk_norm_forward(x, x, None, None, 0.0, to, torch.from_numpy(freqs).cuda(), interleaved)
        c, s = exact_turns(positions, freqs)
        for got, want in ((y[:, 0, first], c), (y[:, 0, second], s)):
            assert np.abs(got.double().cpu().numpy() - want).max() <= 2.0 ** -23
        assert torch.equal(y[..., 2 * n:], x[..., 2 * n:])
        beside = max(beside, np.abs(np.cos(positions[:, None] * freqs.astype(np.float64)) - c).max())
    assert beside > 2.0 ** -10  # the rounded product would be seen


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
