"""Argument checks of the attention calls: they run on the host before any HIP
call, so descriptors of memory that does not exist will do.  A call whose
arguments pass fails at its launch here (KB_ERR_HIP): no GPU."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_norm_abi import view

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="descriptors of memory that does not exist")
Q, K = (2, 8, 16, 64), (2, 4, 32, 64)
ARG, DTYPE, ALIGN, WS, HIP = (kb.KB_ERR_INVALID_ARG, kb.KB_ERR_DTYPE, kb.KB_ERR_ALIGNMENT, kb.KB_ERR_WORKSPACE,
                              kb.KB_ERR_HIP)


@pytest.fixture(scope="module")
def L():
    ensure_built()
    return kb.lib()


def opts(scale=0.125, flags=0, q_lens=0, k_lens=0):
    return kb._OPTS.pack(scale, flags, q_lens, k_lens)


def forward(L, q=view(0x100000, Q), k=view(0x200000, K), v=view(0x300000, K), op=opts(), o=view(0x400000, Q),
            lse=0x500000, ws=0x600000, size=1 << 20):
    return L.kb_attn_forward(q, k, v, op, o, lse, ws, size, None)


def backward(L, do=view(0x100000, Q), q=view(0x200000, Q), k=view(0x300000, K), v=view(0x400000, K),
             o=view(0x500000, Q), lse=0x600000, op=opts(), dq=view(0x700000, Q), dk=view(0x800000, K),
             dv=view(0x900000, K), ws=0xa00000, size=1 << 20):
    return L.kb_attn_backward(do, q, k, v, o, lse, op, dq, dk, dv, ws, size, None)


def test_good_arguments_reach_the_launch(L):
    assert forward(L) == HIP
    assert forward(L, op=opts(flags=kb.KB_ATTN_CAUSAL, q_lens=0x700000, k_lens=0x700100)) == HIP
    assert forward(L, k=view(0x200000, K, (0, 64, 64, 1))) == HIP  # shared keys, heads that overlap in memory
    assert backward(L) == HIP


@pytest.mark.parametrize("change,code", [
    (dict(q=None), ARG), (dict(op=None), ARG), (dict(o=None), ARG), (dict(lse=None), ARG),
    (dict(q=view(0, Q)), ARG),
    (dict(q=view(0x100000, Q[:3])), ARG),
    (dict(q=view(0x100000, (2, 6, 16, 64))), ARG),                    # 6 heads on 4
    (dict(k=view(0x200000, (2, 0, 32, 64)), v=view(0x300000, (2, 0, 32, 64))), ARG),
    (dict(k=view(0x200000, (3, 4, 32, 64))), ARG),
    (dict(k=view(0x200000, (2, 4, 32, 72))), ARG),
    (dict(v=view(0x300000, (2, 4, 31, 64))), ARG),
    (dict(q=view(0x100000, (2, 8, 16, 136)), k=view(0x200000, (2, 4, 32, 136))), ARG),
    (dict(q=view(0x100000, (2, 8, 16, 0)), k=view(0x200000, (2, 4, 32, 0))), ARG),
    (dict(q=view(0x100000, (2, 8, -16, 64))), ARG),
    (dict(q=view(0x100000, Q, (8192, 1024, 1, 16))), ARG),            # last dimension not contiguous
    (dict(k=view(0x200000, K, dtype=kb.KB_F16)), DTYPE),
    (dict(v=view(0x300000, K, dtype=kb.KB_F16)), DTYPE),
    (dict(o=view(0x400000, Q, dtype=kb.KB_BF16)), DTYPE),
    (dict(q=view(0x100000, Q, dtype=kb.KB_U32)), DTYPE),
    (dict(q=view(0x100002, Q)), ALIGN), (dict(lse=0x500002), ALIGN),
    (dict(op=opts(q_lens=0x700002)), ALIGN),
    (dict(op=opts(scale=0.0)), ARG), (dict(op=opts(scale=-1.0)), ARG), (dict(op=opts(scale=float("inf"))), ARG),
    (dict(op=opts(flags=2)), ARG),
    (dict(o=view(0x400000, (2, 8, 17, 64))), ARG),
    (dict(o=view(0x400000, Q, (8192, 0, 64, 1))), ARG),               # heads of o share memory
    (dict(o=view(0x100100, Q)), ARG), (dict(o=view(0x300100, Q)), ARG), (dict(lse=0x400100), ARG), (dict(lse=0x100100), ARG),
])
def test_forward_refusals(L, change, code):
    assert forward(L, **change) == code
    assert "kb_attn_forward" in kb.kb_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(do=None), ARG), (dict(dq=None), ARG), (dict(dk=None), ARG), (dict(dv=None), ARG), (dict(lse=None), ARG),
    (dict(do=view(0x100000, (2, 8, 15, 64))), ARG), (dict(o=view(0x500000, (2, 8, 15, 64))), ARG),
    (dict(dq=view(0x700000, K)), ARG), (dict(dk=view(0x800000, Q)), ARG),
    (dict(dv=view(0x900000, K, (8192, 2048, 0, 1))), ARG),
    (dict(dv=view(0x800000, K)), ARG), (dict(dq=view(0x200000, Q)), ARG), (dict(dk=view(0x100000, K)), ARG),
    (dict(dq=view(0x700000, Q, dtype=kb.KB_F16)), DTYPE),
    (dict(ws=None), WS), (dict(size=2047), WS), (dict(ws=0xa00004), ALIGN), (dict(ws=0x700000), ARG),
])
def test_backward_refusals(L, change, code):
    assert backward(L, **change) == code
    assert "kb_attn_backward" in kb.kb_last_error()


def test_workspace_bytes(L):
    # at least two values for each of 2 x 8 x 16 queries
    assert 4 * 512 <= L.kb_attn_backward_workspace_bytes(view(1, Q), view(1, K)) <= 4 * 600
    for q, k in (((2, 6, 16, 64), K), (Q, (1, 4, 32, 64)), ((2, 8, 16, 200), (2, 4, 32, 200))):
        assert L.kb_attn_backward_workspace_bytes(view(1, q), view(1, k)) == 0
        assert L.kb_attn_forward_workspace_bytes(view(1, q), view(1, k)) == 0
    # few rows on many keys: parts of their sums, binary32
    q, k = (1, 2, 1, 61), (1, 1, 5000, 61)
    assert L.kb_attn_forward_workspace_bytes(view(1, q), view(1, k)) == 4 * 2 * 39 * (64 + 4)
    assert L.kb_attn_backward_workspace_bytes(view(1, q), view(1, k)) >= 4 * 2 * 39 * 64
    assert L.kb_attn_forward_workspace_bytes(None, view(1, k)) == 0


def test_gradients_as_columns_of_one_buffer(L):
    """dq, dk and dv of one [batch][len][columns] buffer do not overlap; shifted by one element they do."""
    n, h, hk, d = 32, 8, 4, 64
    wide = (h + 2 * hk) * d
    q, k = (2, h, n, d), (2, hk, n, d)

    def cut(first, heads):
        return view(0x700000 + 4 * first, (2, heads, n, d), (n * wide, d, wide, 1))
    args = dict(do=view(0x100000, q), q=view(0x200000, q), k=view(0x300000, k), v=view(0x400000, k), o=view(0x500000, q))
    assert backward(L, dq=cut(0, h), dk=cut(h * d, hk), dv=cut((h + hk) * d, hk), **args) == HIP
    assert backward(L, dq=cut(0, h), dk=cut(h * d - 1, hk), dv=cut((h + hk) * d, hk), **args) == ARG
    assert backward(L, dq=cut(0, h), dk=cut(h * d, hk), dv=cut((h + hk) * d + 1, hk), **args) == ARG


def test_empty(L):
    for q, k in (((0, 8, 16, 64), (0, 4, 32, 64)), ((2, 0, 16, 64), (2, 0, 32, 64)), ((2, 8, 0, 64), K)):
        eq, ek = view(0, q), view(0 if 0 in k else 0x200000, k)
        assert forward(L, q=eq, k=ek, v=view(0 if 0 in k else 0x300000, k), o=eq, lse=None) == kb.KB_OK


def test_more_work_groups_than_a_launch_takes(L):
    """2^24 (batch, key head) pairs, and one fewer."""
    for n, code in ((1 << 24, ARG), ((1 << 24) - 1, HIP)):
        q = k = (n, 1, 1, 8)
        args = dict(q=view(1 << 32, q), k=view(2 << 32, k), v=view(3 << 32, k), o=view(4 << 32, q), lse=5 << 32)
        assert forward(L, **args) == code
        need = L.kb_attn_backward_workspace_bytes(view(1 << 32, q), view(2 << 32, k))
        assert (need == 0) == (code == ARG)
        args.update(do=view(6 << 32, q), dq=view(7 << 32, q), dk=view(8 << 32, k), dv=view(9 << 32, k), ws=10 << 32)
        assert backward(L, size=need or 1 << 20, **args) == code
    long = (1, 1, 1 << 30, 8)
    assert forward(L, q=view(1 << 40, (1, 1, 1, 8)), k=view(2 << 40, long), v=view(3 << 40, long),
                   o=view(4 << 40, (1, 1, 1, 8)), lse=5 << 40, ws=6 << 40) == ARG
