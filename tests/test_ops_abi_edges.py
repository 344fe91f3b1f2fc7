"""Argument ranges of the reference operators at their ends (no GPU: a call
whose arguments pass fails at its launch, KB_ERR_HIP)."""
import itertools
import random

import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_attn_abi import backward, forward, opts
from tests.test_norm_abi import view

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="descriptors of memory that does not exist")
ARG, OK, HIP = kb.KB_ERR_INVALID_ARG, kb.KB_OK, kb.KB_ERR_HIP


@pytest.fixture(scope="module")
def L():
    ensure_built()
    return kb.lib()


@pytest.mark.parametrize("dtype", [kb.KB_F32, kb.KB_F16, kb.KB_BF16])
@pytest.mark.parametrize("nq", [0, 16])
def test_no_query_heads_have_gradients_of_zero(L, dtype, nq):
    """Key heads that no query head reads: dk and dv are zeros that the call has to write; without keys, nothing."""
    none = view(0, (2, 0, nq, 64), dtype=dtype)
    for nk, code in ((32, HIP), (0, OK)):
        key = [view(p if nk else 0, (2, 4, nk, 64), dtype=dtype) for p in (0x100000, 0x200000, 0x300000, 0x400000)]
        size = L.kb_attn_backward_workspace_bytes(none, key[0])
        rc = backward(L, do=none, q=none, k=key[0], v=key[1], o=none, lse=None, dq=none, dk=key[2], dv=key[3], size=size)
        assert rc == code


def test_gradients_as_columns_of_a_padded_buffer(L):
    """dq, dk and dv of one buffer whose sequences lie a stride apart that is no multiple of a row: no element is shared.
    One element further they are refused, as they are where one's last row reaches the other's first."""
    n, h, hk, d = 32, 8, 4, 64
    wide = (h + 2 * hk) * d
    apart = n * wide + 40
    q, k = (3, h, n, d), (3, hk, n, d)

    def cut(first, heads, batch=apart):
        return view(0x7000000 + 4 * first, (3, heads, n, d), (batch, d, wide, 1))
    args = dict(do=view(0x1000000, q), q=view(0x2000000, q), k=view(0x3000000, k), v=view(0x4000000, k),
                o=view(0x5000000, q), lse=0x6000000, ws=0xa000000)
    assert backward(L, dq=cut(0, h), dk=cut(h * d, hk), dv=cut((h + hk) * d, hk), **args) == HIP
    assert backward(L, dq=cut(0, h), dk=cut(h * d - 1, hk), dv=cut((h + hk) * d, hk), **args) == ARG
    assert backward(L, dq=cut(0, h), dk=cut(h * d, hk), dv=cut((h + hk) * d + 41 + 1, hk, apart - 40), **args) == ARG


def test_overlap_of_views_of_three_strides(L):
    """Random q-like and k-like outputs of one buffer: one that shares an element is refused; columns that share none,
    with the buffer's strides and within its sequences, are not."""
    rng = random.Random(7)
    seen = [0, 0]
    for _ in range(2000):
        b, n, h, hk, d = (rng.randrange(1, 4) for _ in range(5))
        row = rng.randrange(h * d + hk * d, h * d + hk * d + 6)
        seq = rng.randrange((n - 1) * row + h * d + hk * d, n * row + 9)
        same = rng.random() < 0.7
        row2, seq2 = (row, seq) if same else (row + 1, seq + n)
        off = rng.randrange(0, seq + row) if rng.random() < 0.5 else h * d + rng.randrange(0, 4)
        q, k = (b, h, n, d), (b, hk, n, d)

        def places(base, shape, strides):
            return {base + sum(i * s for i, s in zip(at, strides)) for at in itertools.product(*map(range, shape))}
        sq, sk = (seq, d, row, 1), (seq2, d, row2, 1)
        shares = bool(places(0, q, sq) & places(off, k, sk))
        far = 1 << 20
        rc = backward(L, do=view(far, q), q=view(2 * far, q), k=view(3 * far, k), v=view(4 * far, k), o=view(5 * far, q),
                      lse=6 * far, dq=view(7 * far, q, sq), dk=view(7 * far + 4 * off, k, sk), dv=view(8 * far, k), ws=9 * far) \
            if h % hk == 0 else None
        if rc is None:
            continue
        assert rc in (ARG, HIP)
        if shares:
            assert rc == ARG, (q, k, sq, sk, off)
        elif same and off % row >= h * d and off % row + hk * d <= row and off + (n - 1) * row + hk * d <= seq:
            seen[1] += 1
            assert rc == HIP, (q, k, sq, sk, off)
        seen[0] += shares
    assert min(seen) > 200, seen


def test_outputs_on_the_lengths(L):
    """The lengths are inputs: an output or the workspace that holds them is refused."""
    lens = dict(op=opts(q_lens=0xb00000, k_lens=0xb00100))
    assert forward(L, **lens) == HIP and backward(L, **lens) == HIP
    q = (2, 8, 16, 64)
    assert forward(L, o=view(0xb00000 - 64, q), **lens) == ARG
    assert forward(L, lse=0xb00100 - 4, **lens) == ARG
    assert backward(L, dq=view(0xb00000 - 64, q), **lens) == ARG
    assert backward(L, dk=view(0xb00104, (2, 4, 32, 64)), **lens) == ARG
    assert backward(L, ws=0xb00100 - 256, **lens) == ARG
    assert "q_lens" in kb.kb_last_error()
