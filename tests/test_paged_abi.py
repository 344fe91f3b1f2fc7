"""Argument checks of the head norms, the cache writes and the attention over pages: they run on the host before any
HIP call, so descriptors of memory that does not exist will do.  A call whose arguments pass fails at its launch here
(KB_ERR_HIP): no GPU."""
import random

import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_norm_abi import view

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="descriptors of memory that does not exist")
ARG, DTYPE, ALIGN, WS, HIP = (kb.KB_ERR_INVALID_ARG, kb.KB_ERR_DTYPE, kb.KB_ERR_ALIGNMENT, kb.KB_ERR_WORKSPACE,
                              kb.KB_ERR_HIP)
F16, BF16 = kb.KB_F16, kb.KB_BF16
Q, K = (12, 4, 64), (12, 2, 64)
C = (40, 2, 16, 64)       # [pages][kv_heads][page][dim]
NAN = float("nan")


@pytest.fixture(scope="module")
def L():
    ensure_built()
    return kb.lib()


def qk_opts(eps=1e-6, flags=0, positions=0x700000, freqs=0x710000, rot=64):
    return kb._QK_OPTS.pack(eps, flags, positions, freqs, rot, 0)


def pages(table=0x700000, stride=10, lens=0x710000, starts=0x720000, batch=4, width=10):
    return kb._PAGES.pack(table, stride, lens, starts, batch, width)


def forward(L, q=view(0x100000, Q), k=view(0x200000, K), wq=view(0x300000, (64,)), wk=view(0x310000, (64,)), op=qk_opts(),
            yq=view(0x400000, Q), yk=view(0x500000, K)):
    return L.kb_qk_norm_forward(q, k, wq, wk, op, yq, yk, None)


def backward(L, dyq=view(0x100000, Q), dyk=view(0x180000, K), q=view(0x200000, Q), k=view(0x280000, K),
             wq=view(0x300000, (64,)), wk=view(0x310000, (64,)), op=qk_opts(), dq=view(0x400000, Q), dk=view(0x480000, K),
             dwq=view(0x500000, (64,)), dwk=view(0x510000, (64,)), ws=0x600000, size=1 << 20):
    return L.kb_qk_norm_backward(dyq, dyk, q, k, wq, wk, op, dq, dk, dwq, dwk, ws, size, None)


def write(L, k=view(0x100000, K), v=view(0x200000, K), pg=pages(), kc=view(0x300000, C), vc=view(0x500000, C)):
    return L.kb_cache_write(k, v, pg, kc, vc, None)


def attend(L, q=view(0x100000, Q), kc=view(0x300000, C), vc=view(0x500000, C), pg=pages(), scale=0.125, flags=1,
           o=view(0x200000, Q), lse=0x280000, ws=0x800000, size=1 << 26):
    return L.kb_attn_paged(q, kc, vc, pg, scale, flags, o, lse, ws, size, None)


def test_good_arguments_reach_the_launch(L):
    assert forward(L) == HIP
    assert forward(L, wq=None, wk=None, op=qk_opts(rot=0, positions=0, freqs=0)) == HIP
    assert forward(L, yq=view(0x100000, Q), yk=view(0x200000, K)) == HIP  # in place
    assert forward(L, q=view(0x100000, Q, (384, 64, 1)), k=view(0x100000 + 1024, K, (384, 64, 1))) == HIP  # columns
    assert forward(L, k=view(None, (12, 0, 64)), yk=view(None, (12, 0, 64))) == HIP
    assert backward(L) == HIP
    assert backward(L, dq=None, dk=None, dwq=None, dwk=None, ws=None, size=0) == HIP
    assert write(L) == HIP and attend(L) == HIP
    assert write(L, pg=pages(starts=0, batch=12)) == HIP and attend(L, pg=pages(starts=0, batch=12)) == HIP
    # pages of k and v beside each other, and shared by the heads of a page
    both = (2 * 2048, 16 * 64, 64, 1)
    assert write(L, kc=view(0x300000, C, both), vc=view(0x300000 + 4 * 2048, C, both)) == HIP
    assert attend(L, kc=view(0x300000, C), vc=view(0x300000, C)) == HIP
    assert attend(L, lse=None) == HIP


@pytest.mark.parametrize("change,code", [
    (dict(q=None), ARG), (dict(k=None), ARG), (dict(op=None), ARG), (dict(yq=None), ARG), (dict(yk=None), ARG),
    (dict(q=view(0, Q)), ARG),
    (dict(q=view(0x100000, (12, 256))), ARG),
    (dict(k=view(0x200000, (11, 2, 64))), ARG),
    (dict(k=view(0x200000, (12, 2, 32))), ARG),
    (dict(q=view(0x100000, (12, 4, 258)), k=view(0x200000, (12, 2, 258))), ARG),
    (dict(q=view(0x100000, (12, 4, 0)), k=view(0x200000, (12, 2, 0))), ARG),
    (dict(q=view(0x100000, (1, 65537, 64), (0, 0, 1))), ARG),
    (dict(q=view(0x100000, Q, (256, 1, 4))), ARG),
    (dict(q=view(0x100002, Q)), ALIGN),
    (dict(k=view(0x200000, K, dtype=F16)), DTYPE),
    (dict(yq=view(0x400000, Q, dtype=BF16)), DTYPE),
    (dict(yq=view(0x400000, Q, dtype=kb.KB_U32)), DTYPE),
    (dict(yk=view(0x500000, (12, 2, 63))), ARG),
    (dict(yq=view(0x400000, Q, (128, 64, 1))), ARG),                       # elements that share memory
    (dict(wq=view(0x300000, (63,))), ARG), (dict(wk=view(0x310000, (64,), (2,))), ARG),
    (dict(wq=view(0x300000, (64,), dtype=F16)), DTYPE),
    (dict(op=qk_opts(eps=-1.0)), ARG), (dict(op=qk_opts(eps=NAN)), ARG), (dict(op=qk_opts(flags=2)), ARG),
    (dict(op=qk_opts(rot=-2)), ARG), (dict(op=qk_opts(rot=33)), ARG), (dict(op=qk_opts(rot=66)), ARG),
    (dict(op=qk_opts(positions=0)), ARG), (dict(op=qk_opts(freqs=0)), ARG),
    (dict(op=qk_opts(positions=0x700002)), ALIGN), (dict(op=qk_opts(freqs=0x710001)), ALIGN),
    (dict(yq=view(0x100010, Q)), ARG),                                     # not in place, but on q
    (dict(yq=view(0x200000, Q)), ARG), (dict(yk=view(0x100000, K)), ARG),  # on k, on q
    (dict(yk=view(0x400100, K)), ARG),                                     # on q's output
    (dict(yq=view(0x300000, Q)), ARG), (dict(yq=view(0x6ffff0, Q)), ARG),  # on a weight, on the positions
])
def test_forward_refusals(L, change, code):
    assert forward(L, **change) == code
    assert "kb_qk_norm_forward" in kb.kb_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(dyq=None), ARG), (dict(dyk=view(0x180000, (12, 3, 64))), ARG),
    (dict(dyq=view(0x100000, Q, dtype=F16)), DTYPE),
    (dict(dq=view(0x100000, Q)), ARG), (dict(dq=view(0x200000, Q)), ARG),  # on dq_out, on q
    (dict(dk=view(0x400000, K)), ARG), (dict(dwq=view(0x510000, (64,))), ARG),
    (dict(dwq=view(0x500000, (64,), dtype=BF16)), DTYPE),
    (dict(dwk=view(0x510000, (64,), (0,))), ARG),
    (dict(op=None), ARG), (dict(op=qk_opts(eps=-1.0)), ARG),
    (dict(ws=None), WS), (dict(size=100), WS), (dict(ws=0x600004), ALIGN), (dict(ws=0x400000), ARG),
])
def test_backward_refusals(L, change, code):
    assert backward(L, **change) == code
    assert "kb_qk_norm_backward" in kb.kb_last_error()


def test_weights_types(L):
    half = dict(q=view(0x100000, Q, dtype=F16), k=view(0x200000, K, dtype=F16), yq=view(0x400000, Q, dtype=F16),
                yk=view(0x500000, K, dtype=F16))
    assert forward(L, **half) == HIP
    w16 = view(0x300000, (64,), dtype=F16)
    assert forward(L, wq=w16, wk=view(0x310000, (64,), dtype=F16), **half) == HIP
    assert forward(L, wq=w16, wk=None, **half) == HIP
    assert forward(L, wq=w16, **half) == DTYPE
    assert forward(L, wq=view(0x300000, (64,), dtype=BF16), wk=None, **half) == DTYPE


PAGE_CHANGES = [
    (dict(pg=None), ARG), (dict(kc=None), ARG), (dict(vc=None), ARG),
    (dict(kc=view(0x300000, C[:3])), ARG),
    (dict(vc=view(0x500000, (40, 2, 16, 32))), ARG), (dict(vc=view(0x500000, (39, 2, 16, 64))), ARG),
    (dict(kc=view(0x300000, (40, 2, 0, 64)), vc=view(0x500000, (40, 2, 0, 64))), ARG),
    (dict(kc=view(0x300000, (40, 2, 16, 32)), vc=view(0x500000, (40, 2, 16, 32))), ARG),
    (dict(kc=view(0x300000, C, dtype=F16), vc=view(0x500000, C, dtype=F16)), DTYPE),
    (dict(vc=view(0x500000, C, dtype=F16)), DTYPE),
    (dict(pg=pages(batch=-1)), ARG), (dict(pg=pages(width=-1)), ARG), (dict(pg=pages(batch=(1 << 20) + 1)), ARG),
    (dict(pg=pages(width=1 << 27, stride=1 << 27)), ARG),                  # 2^31 keys
    (dict(pg=pages(width=(1 << 28) + 1, stride=1 << 29), kc=view(0x300000, (40, 2, 1, 64)), vc=view(0x500000, (40, 2, 1, 64))), ARG),
    (dict(pg=pages(stride=9)), ARG), (dict(pg=pages(stride=-10)), ARG),
    (dict(pg=pages(table=0)), ARG), (dict(pg=pages(lens=0)), ARG),
    (dict(pg=pages(starts=0)), ARG),                                       # 12 tokens, 4 sequences
    (dict(pg=pages(table=0x700002)), ALIGN), (dict(pg=pages(lens=0x710001)), ALIGN), (dict(pg=pages(starts=0x720003)), ALIGN),
    (dict(kc=view(0x300002, C)), ALIGN),
]


@pytest.mark.parametrize("change,code", PAGE_CHANGES + [
    (dict(k=None), ARG), (dict(v=None), ARG), (dict(v=view(0x200000, (12, 2, 32))), ARG),
    (dict(v=view(0x200000, K, dtype=F16)), DTYPE),
    (dict(k=view(0x100000, (12, 4, 64)), v=view(0x200000, (12, 4, 64))), ARG),
    (dict(vc=view(0x300000, C)), ARG),                                     # v's pages on k's
    (dict(kc=view(0x300000, C, (0, 1024, 64, 1))), ARG),                   # pages that share memory
    (dict(k=view(0x300100, K)), ARG), (dict(pg=pages(table=0x300000)), ARG), (dict(pg=pages(lens=0x500000)), ARG),
    (dict(pg=pages(starts=0x300040)), ARG),
    (dict(k=view(0x100000, (12, 2, 136)), v=view(0x200000, (12, 2, 136)), kc=view(0x300000, (40, 2, 16, 136)),
          vc=view(0x600000, (40, 2, 16, 136))), ARG),
])
def test_write_refusals(L, change, code):
    assert write(L, **change) == code
    assert "kb_cache_write" in kb.kb_last_error()


@pytest.mark.parametrize("change,code", PAGE_CHANGES + [
    (dict(q=None), ARG), (dict(o=None), ARG), (dict(q=view(0x100000, (12, 3, 64)), o=view(0x200000, (12, 3, 64))), ARG),
    (dict(o=view(0x200000, (12, 4, 63))), ARG), (dict(o=view(0x200000, Q, dtype=F16)), DTYPE),
    (dict(o=view(0x200000, Q, (64, 64, 1))), ARG),
    (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG), (dict(scale=NAN), ARG), (dict(scale=float("inf")), ARG),
    (dict(flags=2), ARG), (dict(lse=0x280002), ALIGN),
    (dict(o=view(0x100000, Q)), ARG), (dict(o=view(0x300000, Q)), ARG), (dict(o=view(0x500100, Q)), ARG),
    (dict(lse=0x200010), ARG), (dict(lse=0x710000), ARG), (dict(o=view(0x6fff00, Q)), ARG),
    (dict(kc=view(0x300000, (40, 0, 16, 64)), vc=view(0x500000, (40, 0, 16, 64))), ARG),
    (dict(q=view(0x100000, (12, 4, 136)), o=view(0x200000, (12, 4, 136)), kc=view(0x300000, (40, 2, 16, 136)),
          vc=view(0x600000, (40, 2, 16, 136))), ARG),
    (dict(q=view(0x100000, (1 << 15, 1 << 16, 1), (0, 0, 1)), kc=view(0x300000, (4, 2, 16, 1)), vc=view(0x500000, (4, 2, 16, 1)),
          o=view(0x10000000, (1 << 15, 1 << 16, 1))), ARG),                # 2^31 (token, head) pairs
])
def test_attention_refusals(L, change, code):
    assert attend(L, **change) == code
    assert "kb_attn_paged" in kb.kb_last_error()


def test_workspaces(L):
    q, kc = view(0x100000, (4, 8, 64)), view(0x300000, (400, 2, 16, 64))
    need = L.kb_attn_paged_workspace_bytes(q, kc, pages(starts=0, width=100, stride=100))
    assert need > 0 and need % 16 == 0

    def call(**more):
        return attend(L, q=q, kc=kc, vc=view(0x700000 + (1 << 24), (400, 2, 16, 64)), o=view(0x180000, (4, 8, 64)),
                      pg=pages(0x710000, 100, 0x720000, 0, 4, 100), ws=0x10000000, **more)
    assert call(size=need) == HIP and call(size=need - 1) == WS
    assert L.kb_attn_paged_workspace_bytes(q, kc, pages(starts=0, width=32, stride=32)) == 0  # 512 keys: not split
    assert L.kb_attn_paged_workspace_bytes(q, kc, pages(starts=0, batch=3)) == 0              # (refused)
    assert L.kb_attn_paged_workspace_bytes(None, kc, pages()) == 0
    assert kb.kb_qk_norm_backward_workspace_bytes(0) == 0 and kb.kb_qk_norm_backward_workspace_bytes(257) == 0
    assert kb.kb_qk_norm_backward_workspace_bytes(64) > 0


def test_empty(L):
    none, kn = view(None, (0, 4, 64)), view(None, (0, 2, 64))
    assert forward(L, q=none, k=kn, yq=none, yk=kn) == kb.KB_OK
    assert backward(L, dyq=none, dyk=kn, q=none, k=kn, dq=none, dk=kn, dwq=None, dwk=None) == kb.KB_OK
    assert backward(L, dyq=none, dyk=kn, q=none, k=kn, dq=none, dk=kn) == HIP  # dw of no row is written
    assert write(L, k=kn, v=kn) == kb.KB_OK and attend(L, q=none, o=none) == kb.KB_OK
    assert write(L, pg=pages(batch=0)) == kb.KB_OK and attend(L, pg=pages(batch=0)) == kb.KB_OK
    assert write(L, pg=pages(table=0, width=0)) == kb.KB_OK
    assert attend(L, pg=pages(table=0, width=0)) == HIP                        # o of no key is written
    assert attend(L, kc=view(None, (0, 2, 16, 64)), vc=view(None, (0, 2, 16, 64))) == HIP


def test_pages_that_overlap_are_never_missed(L):
    """k's pages against v's over random views: two that share an element are refused."""
    rng = random.Random(3)
    seen = {True: 0, False: 0}
    shape = (3, 2, 4, 5)
    for _ in range(3000):
        order = rng.sample(range(3), 3)
        strides, n = [0, 0, 0, 1], 5
        for i in order:
            strides[i] = n + rng.choice([0, 0, 3, 40])
            n = strides[i] * shape[i]
        at = 0x300000 + 4 * rng.randrange(-200, 200)

        def elements(base):
            return {base + 4 * (a * strides[0] + b * strides[1] + c * strides[2] + d) for a in range(3) for b in range(2)
                    for c in range(4) for d in range(5)}
        shares = bool(elements(0x300000) & elements(at))
        rc = write(L, k=view(0x100000, (12, 2, 5)), v=view(0x200000, (12, 2, 5)), kc=view(0x300000, shape, strides),
                   vc=view(at, shape, strides))
        assert rc in (ARG, HIP)
        seen[shares] += 1
        if shares:
            assert rc == ARG, (strides, at - 0x300000)
    assert min(seen.values()) > 300
