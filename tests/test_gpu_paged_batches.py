"""The paged cache: starts that nobody should send, and batches of prompts beside single tokens."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.paged import DT, Batch, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch_size", [9, 90])
@pytest.mark.parametrize("tokens,keys", [(24, 300), (24, 3000), (700, 1500)])
def test_starts_out_of_order(dtype, batch_size, tokens, keys):
    """Starts that do not ascend, and lie outside the call's tokens: nothing but these tokens' rows is written."""
    b = Batch([(1, keys)] * batch_size, 16, 4, 2, 64, dtype, "hnd", one=True)
    g = torch.Generator().manual_seed(3)
    for n in range(4):
        starts = torch.randint(-tokens, 2 * tokens, (batch_size + 1,), generator=g).clamp(-5, tokens + 5).to(torch.int32).cuda()
        buf = torch.full((3 * tokens, 4, 64), 7.0, dtype=DT[dtype], device="cuda")
        norms = torch.full((3 * tokens, 4), 7.0, device="cuda")
        q = buf.new_ones((tokens, 4, 64))
        ws = torch.full((kb.kb_attn_paged_workspace_bytes(q, b.k_cache, b.table, b.lens, starts) + 16,), 255,
                        dtype=torch.uint8, device="cuda")
        kb.kb_attn_paged(q, b.k_cache, b.v_cache, b.table, b.lens, starts, o=buf[tokens:2 * tokens],
                         lse=norms[tokens:2 * tokens], workspace=ws)
        for t in (buf, norms):
            assert torch.all(t[:tokens] == 7.0) and torch.all(t[2 * tokens:] == 7.0)
        caches = [c.clone() for c in (b.k_cache, b.v_cache)]
        kb.kb_cache_write(q[:, :2], q[:, :2], *caches, b.table, b.lens, starts)
        spare = torch.ones(len(caches[0]), dtype=torch.bool, device="cuda")
        spare[b.table[:, :-(-keys // 16)].long()] = False
        assert int(spare.sum()) == 2 and all(torch.isnan(c[spare]).all() for c in caches)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("seqs", [
    [(1000, 1000), (1, 20000)],                              # by blocks of many rows
    [(300, 700), (1, 9000), (1, 1), (4, 2500), (1, 1200)],
    [(1, 500 + 90 * i) for i in range(40)] + [(70, 1000)],   # by blocks of few rows
])
def test_prompts_beside_single_tokens(dtype, seqs):
    b = Batch(seqs, 16, 8, 2, 64, dtype, "hnd")
    o, lse = kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, *b.pages)
    check(b, 0.125, True, o, lse)


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("first,last", [(-9, 0), (0, 7), (-9, 7)])
def test_starts_outside_the_tokens(many, first, last):
    """The first and the last start count as the nearer end of the tokens: the write and the attention have the same bits."""
    b = Batch([(3, 40), (2, 30)] + [(1, 20)] * (70 if many else 2) + [(4, 25)], 16, 4, 2, 64, "f16")
    outside = b.starts.clone()
    outside[0] += first
    outside[-1] += last
    k = b.q[:, :2].contiguous()
    got = []
    for starts in (b.starts, outside):
        caches = kb.kb_cache_write(k, k, b.k_cache.clone(), b.v_cache.clone(), b.table, b.lens, starts)
        got.append([torch.nan_to_num(c, 9.0) for c in caches] +
                   list(kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, b.table, b.lens, starts)))
    for a, c in zip(*got):
        assert torch.equal(a, c)
