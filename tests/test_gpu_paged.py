"""The paged cache: writes and attention, against the formulas in 64 bits (tests/paged.py has the tolerances)."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.paged import DT, E, U, Batch, check, ints, normal

pytestmark = pytest.mark.gpu
MANY, FEW = [(150, 150), (70, 300)], [(1, 130), (2, 70)]


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def attend(b, causal=True, scale=None, **given):
    """One call, into o and lse that hold 7 and a workspace that holds NaN."""
    o, lse = torch.full_like(b.q, 7.0), torch.full(b.q.shape[:2], 7.0, device="cuda")
    n = kb.kb_attn_paged_workspace_bytes(b.q, b.k_cache, *b.pages)
    ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
    kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, *b.pages, scale=scale, causal=causal, o=o, lse=lse, workspace=ws, **given)
    return o, lse


def run(b, causal=True, scale=None, missing=()):
    o, lse = attend(b, causal, scale)
    check(b, b.dim ** -0.5 if scale is None else scale, causal, o, lse, missing)
    for rows in (o[:b.before], o[b.ends[-1]:], lse[:b.before], lse[b.ends[-1]:]):
        assert torch.all(rows == 7.0)  # of no sequence
    return o, lse


def reordered(b):
    """How far apart o may be when the same sums are computed once more in other steps, and with another reference of
    the softmax: either has n terms, off by n E of the magnitudes, of which a mean of |v| is made, its terms rounded by u
    (16 bits), the result rounded by u."""
    n = max(nk for _, nk in b.seqs)
    return 2 * (2 * U[b.q.dtype] + 2 * n * E) * max(float(v.abs().max()) for v in b.values)


def reordered_lse(b, norm):
    """The same of lse: either is off by what check() allows, the terms' exponents being products of scores of up to A, a
    sum of |q| |k|, in 32 bits."""
    n, grp = max(nk for _, nk in b.seqs), b.heads // b.kv
    top = max(float((torch.nan_to_num(b.q[..., h, :]).double().abs() @ k[:, h // grp].double().abs().T).max())
              for k in b.keys for h in range(b.heads)) * b.dim ** -0.5
    return 2 * ((b.dim + 16) * E * top + 4 * E + n * E + 4 * E * float(norm.abs().max()) + E)


# ------------------------------------------------------------------- writes ---

@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["nhd", "hnd"])
@pytest.mark.parametrize("page,dim,kv", [(16, 128, 8), (1, 64, 1), (7, 40, 3), (24, 33, 2), (64, 2, 5), (5, 1, 1), (16, 126, 9)])
@pytest.mark.parametrize("one", [False, True])
def test_write(dtype, layout, page, dim, kv, one):
    """The new tokens' bits at their places, everything else as it was."""
    seqs = [(1, 1), (1, page), (1, 3 * page + 1), (1, 100)] if one else [(1, 1), (0, 5), (30, 30), (3, 2 * page + 2), (70, 100), (0, 0)]
    b = Batch(seqs, page, kv, kv, dim, dtype, layout, one=one, before=0 if one else 2, after=0 if one else 3)
    k, v = normal((b.q.shape[0], kv, dim), b.q.dtype, 50), normal((b.q.shape[0], kv, dim), b.q.dtype, 51)
    k[0, 0, 0] = float("nan")
    want = [c.clone() for c in (b.k_cache, b.v_cache)]
    for s, (nq, nk) in enumerate(seqs):
        for i in range(nq):
            j = nk - nq + i
            for c, x in zip(want, (k, v)):
                c[int(b.table[s, j // page]), :, j % page] = x[b.ends[s] + i]
    kb.kb_cache_write(k, v, b.k_cache, b.v_cache, *b.pages)
    for c, w in zip((b.k_cache, b.v_cache), want):
        raw = torch.int32 if dtype == "f32" else torch.int16
        assert torch.equal(c.view(raw) if c.is_contiguous() else c.contiguous().view(raw), w.contiguous().view(raw))


def test_write_skips_what_has_no_place():
    """Tokens before a sequence's first key, without a page, or past the table's end change nothing."""
    b = Batch([(5, 3), (4, 40), (2, 60)], 16, 2, 2, 32, "f16")
    b.table[1, 2] = -1   # keys 32 .. 39
    b.table[2, 3] = b.k_cache.shape[0]
    lens = ints([3, 40, 1000])  # counts as 64, the width of the table
    assert b.table.shape[1] == 4
    k = normal((11, 2, 32), torch.float16, 1)
    before = b.k_cache.clone(), b.v_cache.clone()
    kb.kb_cache_write(k, k, b.k_cache, b.v_cache, b.table, lens, b.starts)
    page = int(b.table[0, 0])
    for c, old in zip((b.k_cache, b.v_cache), before):
        assert torch.equal(c[page, :, :3].transpose(0, 1), k[2:5])  # its last three
        old[page, :, :3] = c[page, :, :3]
        assert torch.equal(torch.nan_to_num(c, 9.0), torch.nan_to_num(old, 9.0))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_write_from_columns_at_odd_addresses(dtype):
    t = DT[dtype]
    b = Batch([(9, 20), (3, 3)], 8, 3, 3, 40, dtype)
    buf = normal((12 * (6 * 40 + 3) + 1,), t, 1)[1:].view(12, -1)
    k, v = buf[:, :120].unflatten(1, (3, 40)), buf[:, 120:240].unflatten(1, (3, 40))
    caches = [c.clone() for c in (b.k_cache, b.v_cache)]
    kb.kb_cache_write(k, v, b.k_cache, b.v_cache, *b.pages)
    kb.kb_cache_write(k.contiguous(), v.contiguous(), *caches, *b.pages)
    for a, c in zip((b.k_cache, b.v_cache), caches):
        assert torch.equal(torch.nan_to_num(a, 9.0), torch.nan_to_num(c, 9.0))


def test_write_to_both_halves_of_one_buffer():
    """k's and v's pages beside each other in one buffer, and many sequences (the search over their starts)."""
    n = 5000
    both = torch.zeros((n, 2, 2, 4, 16), dtype=torch.bfloat16, device="cuda")  # [pages][k, v][heads][page][dim]
    table = torch.randperm(n, device="cuda", dtype=torch.int64).to(torch.int32).view(n, 1)
    counts = torch.arange(n, device="cuda") % 4
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]).to(torch.int32)
    k, v = (normal((int(starts[-1]), 2, 16), torch.bfloat16, s) for s in (1, 2))
    kb.kb_cache_write(k, v, both[:, 0], both[:, 1], table, torch.full((n,), 4, dtype=torch.int32, device="cuda"), starts)
    want = torch.zeros_like(both)
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), counts)
    place = 4 - starts[seq + 1].long() + torch.arange(len(k), device="cuda")
    want[table[seq, 0].long(), 0, :, place], want[table[seq, 0].long(), 1, :, place] = k, v
    assert torch.equal(both, want)


# ---------------------------------------------------------------- attention ---

@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("step", [0, 8, 32])
@pytest.mark.parametrize("seqs", [FEW, MANY])
def test_rows_that_share_memory(dtype, dim, step, seqs):
    """Keys and values that are windows of one another, or one row for all (strides less than a row, also 0), heads that
    are one: the bits of copies of them."""
    b = Batch(seqs, 16, 4, 2, dim, dtype, "hnd")
    n = b.k_cache.shape[0]
    buf = normal((n * 16 * max(step, 1) + dim,), b.q.dtype, 3)
    k = buf.as_strided((n, 2, 16, dim), (16 * step, 0, step, 1))
    v = buf.flip(0).as_strided((n, 2, 16, dim), (16 * step, 0, step, 1))
    b.k_cache, b.v_cache = k.contiguous(), v.contiguous()
    want = attend(b)
    b.k_cache, b.v_cache = k, v
    got = attend(b)
    u, terms = U[b.q.dtype], 2 * max(x for _, x in seqs) * E
    # the same sums in other steps, as reordered() and check() have them
    top = dim ** 0.5 * float(b.q.abs().max() * buf.abs().max())  # no score is larger, nor its magnitudes' sum
    assert float((got[0].double() - want[0].double()).abs().max()) <= 2 * (2 * u + terms) * float(buf.abs().max())
    off = 2 * ((dim + 16) * E * top + terms + 4 * E * (1 + float(want[1].abs().max())))
    assert float((got[1] - want[1]).abs().max()) <= off


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv", [(40, 1), (200, 2)])
def test_single_tokens_of_many_heads(dtype, heads, kv):
    """More query heads a key head than the blocks of few rows take, without starts."""
    run(Batch([(1, 90), (1, 1), (1, 700)], 16, heads, kv, 64, dtype, one=True))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["nhd", "hnd"])
@pytest.mark.parametrize("page", [1, 5, 8, 16, 24, 64, 100])
@pytest.mark.parametrize("seqs", [FEW, MANY])
def test_page_sizes(dtype, layout, page, seqs):
    run(Batch(seqs, page, 4, 2, 64, dtype, layout))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [1, 7, 32, 40, 64, 66, 72, 80, 96, 100, 128])
@pytest.mark.parametrize("seqs", [FEW, MANY])
def test_dimensions(dtype, dim, seqs):
    run(Batch(seqs, 16, 3, 1, dim, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 8), (8, 1), (16, 1), (32, 1), (33, 1), (128, 2), (12, 4), (20, 4)])
@pytest.mark.parametrize("new", [1, 2, 3, 40])
def test_head_groups(dtype, heads, kv, new):
    """Rows of a block end inside a query's heads; blocks of 16, 32 and 128 rows."""
    run(Batch([(new, 90), (min(new, 20), 20), (new, new)], 16, heads, kv, 64, dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("seqs", [
    [(0, 0), (1, 0), (3, 1), (1, 1), (0, 9), (2, 500), (9, 5)],     # lengths of zero and one, more queries than keys
    [(0, 40), (200, 130), (1, 1), (1, 0), (130, 130), (0, 0)],
    [(0, 0)], [(2, 0)], [(300, 0)], [(40, 40), (0, 0)],
])
def test_lengths(dtype, causal, seqs):
    run(Batch(seqs, 16, 4, 2, 64, dtype, before=3, after=2), causal)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("seqs,heads,kv", [
    ([(1, 5000)], 8, 2),                                   # a pair in more parts than waves read at once
    ([(1, 9000), (1, 3), (1, 700)], 4, 4),
    ([(5, 3001), (1, 513), (0, 50), (7, 2000)], 8, 2),      # several queries, in parts
    ([(1, 600 + 13 * i) for i in range(110)], 8, 8),        # more pairs than work-groups
    ([(9, 3000), (20, 1500)], 4, 2),                        # blocks of 128 rows, in parts
])
def test_parts(dtype, dim, seqs, heads, kv):
    run(Batch(seqs, 16, heads, kv, dim, dtype, "hnd", one=all(q == 1 for q, _ in seqs)))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("keys", [300, 800])
def test_many_sequences(dtype, keys):
    """More than a wave's lanes, some without new tokens; of keys that are split and that are not; also many rows each."""
    few = [(i % 3, 1 + (i * 37) % keys) for i in range(300)]
    run(Batch(few, 16, 8, 2, 64, dtype, before=1, after=1))
    many = [((i * 7) % 40, 40 + (i * 37) % keys) for i in range(70)]
    run(Batch(many, 16, 8, 2, 64, dtype, before=1, after=1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_wide_table_of_short_sequences(dtype):
    """Rooms for 100,000 keys, of which few are used: work-groups and parts without a key."""
    run(Batch([(1, 70), (1, 1), (1, 600)], 16, 4, 2, 64, dtype, width=6250, one=True))
    run(Batch([(40, 70), (1, 1), (3, 600)], 16, 4, 2, 64, dtype, width=6250))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [8, 16, 24])
@pytest.mark.parametrize("seqs", [[(1, 200), (1, 2000)], [(4, 200), (3, 2000)], [(100, 200), (70, 600)]])
def test_keys_without_a_page(dtype, page, seqs):
    """Pages taken out of the table, first, in the middle and last: their keys are not seen, whatever the numbers."""
    b = Batch(seqs, page, 4, 2, 64, dtype, one=all(q == 1 for q, _ in seqs))
    missing = []
    for s, (_, n) in enumerate(seqs):
        last = (n - 1) // page
        for i, number in ((0, -1), (3, 2 ** 31 - 1), (5, b.k_cache.shape[0]), (last, -2 ** 31)):
            b.table[s, i] = number
            missing += [(s, j) for j in range(i * page, min(n, (i + 1) * page))]
    run(b, missing=missing)
    b.table[0, :] = -1
    run(b, missing=missing + [(0, j) for j in range(seqs[0][1])])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("seqs", [[(4, 100), (6, 700)], [(100, 200), (64, 64)]])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_values_that_are_not_finite(dtype, seqs, value):
    """A NaN or an infinity of v at key j reaches the queries that see it, and no others."""
    b = Batch(seqs, 16, 4, 2, 64, dtype)
    want, norm = run(b)
    for s, (nq, nk) in enumerate(seqs):
        j = nk - 2  # the last query but one's own
        b.v_cache[int(b.table[s, j // 16]), 0, j % 16, 5] = value
    o, lse = attend(b)
    assert float((lse - norm).abs().max()) <= reordered_lse(b, norm)
    for s, (nq, nk) in enumerate(seqs):
        first = b.ends[s]
        got, old = o[first:first + nq], want[first:first + nq]
        assert not torch.isfinite(got[nq - 2:, :2, 5]).any()
        got, old = got.clone(), old.clone()
        got[nq - 2:, :2, 5] = old[nq - 2:, :2, 5] = 0
        assert float((got.double() - old.double()).abs().max()) <= reordered(b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs", [[(1, 300)], [(3, 90), (5, 700)], [(100, 200)]])
def test_a_row_of_the_query_that_is_not_finite(dtype, seqs):
    b = Batch(seqs, 16, 2, 2, 64, dtype)
    want, norm = run(b)
    b.q[0, 0, 3] = float("nan")
    o, lse = attend(b)
    assert torch.isnan(o[0, 0]).all() and torch.isnan(lse[0, 0])
    o[0, 0], lse[0, 0] = want[0, 0], norm[0, 0]
    assert float((o.double() - want.double()).abs().max()) <= reordered(b)
    assert float((lse - norm).abs().max()) <= reordered_lse(b, norm)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("seqs", [[(1, 300), (1, 3000)], [(3, 300), (3, 1300)], [(100, 300)]])
def test_scores_of_the_types_lowest_value(dtype, seqs):
    """Keys that a column of the type's lowest number takes out of the softmax; sequences where that leaves nothing have
    equal scores, so that o is the mean of v."""
    b = Batch(seqs, 16, 2, 2, 64, dtype)
    b.q[..., 0] = 1.0
    low = torch.finfo(b.q.dtype).min
    for s, (nq, nk) in enumerate(seqs):
        b.keys[s][:, :, 0] = 0.0
        b.keys[s][:70, :, 0] = low
        place = torch.arange(nk, device="cuda")
        b.k_cache[b.table[s, place // 16].long(), :, place % 16] = b.keys[s]
    o, lse = attend(b, causal=False, scale=0.125)
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
    keys, values, seqs0 = b.keys, b.values, b.seqs
    b.keys, b.values, b.seqs = [k[70:] for k in keys], [v[70:] for v in values], [(q, n - 70) for q, n in seqs]
    check(b, 0.125, False, o, lse)
    b.q[..., 1:] = 0.0
    b.k_cache[..., 0] = low
    o, _ = attend(b, causal=False, scale=0.125)
    for s, (nq, nk) in enumerate(seqs0):
        got, mean = o[b.ends[s]:b.ends[s + 1]].double(), values[s].double().mean(0)
        assert float((got - mean).abs().max()) <= (U[b.q.dtype] + 2 * nk * E) * float(values[s].abs().max())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_scores(dtype):
    """Scores that differ by more than exp's range: o is the v of the largest one to the last bit."""
    b = Batch([(1, 900), (2, 70)], 16, 2, 2, 64, dtype)
    big = 2.0 ** 15 if dtype == "f16" else 2.0 ** 40
    b.q[..., 1:] = 0.0
    b.q[..., 0] = big
    for s, (_, nk) in enumerate(b.seqs):
        place = torch.arange(nk, device="cuda")
        x = b.keys[s]
        x[..., 0] = -1.0
        x[nk // 3, :, 0] = 1.0
        b.k_cache[b.table[s, place // 16].long(), :, place % 16] = x
    o, lse = attend(b)
    for s, (nq, nk) in enumerate(b.seqs):
        for i in range(nq):
            assert torch.equal(o[b.ends[s] + i], b.values[s][nk // 3])
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("apart", [16.0, 17.4])
def test_long_flat_tails_in_f16(apart):
    """One score above 2^17 equal ones, whose terms (2^-23 and 2^-25.1 of it) count together.  In two parts a term is off
    by 2^-22 of itself or 2^-34 of the largest, a sum of 2^17 by 2^-7 of itself."""
    n = 1 << 17
    q = torch.zeros((1, 1, 64), device="cuda").half()
    k = torch.zeros((n // 64, 1, 64, 64), device="cuda").half()
    v = torch.ones_like(k)
    q[..., 0], k[0, 0, 5, 0], v[0, 0, 5] = 1.0, apart, 0.0
    o, _ = kb.kb_attn_paged(q, k, v, torch.arange(n // 64, device="cuda", dtype=torch.int32).view(1, -1), ints([n]), None, 1.0)
    top = k[0, 0, 5, 0].double().exp().item()
    want = (n - 1) / (top + n - 1)
    err = float((o.double() - want).abs().max())
    assert err <= want * (2.0 ** -11 + 2.0 ** -22 + 2.0 ** -7) + n * 2.0 ** -34, (err, want)


@pytest.mark.parametrize("dtype,dim", [("f16", 64), ("f32", 40)])
@pytest.mark.parametrize("seqs", [[(1, 50)], [(60, 60)]])
def test_pages_far_apart(dtype, dim, seqs):
    """Offsets that pass 2^31 elements, from page to page and from head to head; the bits of dense pages."""
    t = DT[dtype]
    step = (1 << 30) + 64
    b = Batch(seqs, 16, 4, 2, dim, dtype, "hnd", spare=0)
    n = b.k_cache.shape[0]
    buf = torch.empty((2 * n + 1) * step // 2 + 4096, dtype=t, device="cuda")
    k = buf.as_strided((n, 2, 16, dim), (step, step // 2, 2 * dim, 1))
    v = buf.as_strided((n, 2, 16, dim), (step, step // 2, 2 * dim, 1), dim)
    k.copy_(b.k_cache)
    v.copy_(b.v_cache)
    want = attend(b)
    b.k_cache, b.v_cache = k, v
    got = run(b)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    x = normal((b.q.shape[0], 2, dim), t, 3)
    kb.kb_cache_write(x, x, k, v, *b.pages)
    nq, nk = seqs[0]
    j = nk - 1
    assert torch.equal(k[int(b.table[0, j // 16]), :, j % 16], x[-1]) and torch.equal(v[int(b.table[0, j // 16]), :, j % 16], x[-1])


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("seqs", [FEW, MANY])
def test_odd_addresses(dtype, seqs):
    """q, o and the caches at addresses that are no multiple of 16, and q's heads apart."""
    t = DT[dtype]
    b = Batch(seqs, 16, 4, 2, 64, dtype, "hnd")
    want = attend(b)

    def moved(x, pad):
        buf = torch.full((x.numel() + pad * x.shape[0] * x.shape[1] + 8,), 7.0, dtype=t, device="cuda")
        inner = x[0, 0].numel() + pad
        y = buf[1:].as_strided(x.shape, (x.shape[1] * inner, inner) + ((x.shape[3], 1) if x.dim() == 4 else (1,)))
        return y.copy_(x)
    b.q, b.k_cache, b.v_cache = moved(b.q, 3), moved(b.k_cache, 5), moved(b.v_cache, 1)
    o, lse = moved(torch.zeros_like(want[0]), 2), torch.empty_like(want[1])
    kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, *b.pages, o=o, lse=lse)
    check(b, 0.125, True, o, lse)


def test_without_lse():
    """lse may be left out (the C interface)."""
    L = kb.lib()
    for seqs in (FEW, MANY, [(1, 3000)], [(20, 3000)]):
        b = Batch(seqs, 16, 4, 2, 64, "bf16")
        want, _ = attend(b)
        o = torch.empty_like(want)
        n = kb.kb_attn_paged_workspace_bytes(b.q, b.k_cache, *b.pages)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        rc = L.kb_attn_paged(kb.pack_view(b.q), kb.pack_view(b.k_cache), kb.pack_view(b.v_cache), kb._pages(*b.pages), 0.125,
                             1, kb.pack_view(o), None, ws.data_ptr(), n, kb._stream_handle(None))
        assert rc == 0 and torch.equal(o, want)


def test_shared_pages():
    """Two sequences with the same first pages read the same keys."""
    b = Batch([(1, 100), (1, 100), (3, 90)], 16, 4, 2, 64, "f16")
    b.table[1, :3] = b.table[0, :3]
    b.keys[1] = torch.cat([b.keys[0][:48], b.keys[1][48:]])
    b.values[1] = torch.cat([b.values[0][:48], b.values[1][48:]])
    run(b)


def test_lengths_out_of_range():
    """A length outside [0, max_pages page] counts as the nearer end."""
    b = Batch([(1, 64), (2, 10), (1, 0)], 16, 4, 2, 64, "f16")
    want = attend(b)
    b.lens = ints([2 ** 31 - 1, 10, -2 ** 31])
    got = attend(b)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_parts_of_a_batch():
    """Sequences of a batch in two calls, by slices of the table, the lengths and the starts: the tokens of the others are
    left as they are."""
    b = Batch([(1, 300), (1, 20), (200, 200), (40, 90)], 16, 4, 2, 64, "bf16")
    want = attend(b)
    o, lse = torch.full_like(b.q, 7.0), torch.full(b.q.shape[:2], 7.0, device="cuda")
    kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, b.table[:2], b.lens[:2], b.starts[:3], o=o, lse=lse)
    assert torch.all(o[2:] == 7.0) and torch.all(lse[2:] == 7.0)
    kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, b.table[2:], b.lens[2:], b.starts[2:], o=o, lse=lse)
    # the first two go by blocks of few rows here
    assert torch.equal(o[2:], want[0][2:])
    check(b, 0.125, True, o, lse)


@pytest.mark.parametrize("seqs", [[(1, 700 + 50 * i) for i in range(20)], [(300, 300), (50, 900)]])
def test_same_bits_on_every_call_and_stream(seqs):
    """Two streams at once, each with a workspace of its own."""
    b = Batch(seqs, 16, 8, 2, 128, "bf16", one=all(q == 1 for q, _ in seqs))
    first = attend(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(3):
        got.append(kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, *b.pages, stream=side))
        got.append(kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, *b.pages))
    torch.cuda.synchronize()
    for o, lse in got:
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("what", ["table dtype", "table rows", "lens length", "starts length", "cpu", "tokens", "dtype",
                                  "v shape", "heads", "lse", "o on q"])
def test_refusals_of_the_binding(what):
    b = Batch([(1, 20), (1, 30)], 16, 4, 2, 64, "f16", one=True)
    q, kc, vc, table, lens, starts, more = b.q, b.k_cache, b.v_cache, b.table, b.lens, None, {}
    if what == "table dtype":
        table = table.long()
    if what == "table rows":
        table = torch.stack([table, table], 2)[..., 0]
    if what == "lens length":
        lens = ints([20])
    if what == "starts length":
        starts = ints([0, 2])
    if what == "cpu":
        lens = lens.cpu()
    if what == "tokens":
        q = q[:1]
    if what == "dtype":
        q = q.float()
    if what == "v shape":
        vc = vc[:, :, :8]
    if what == "heads":
        q = q[:, :3].contiguous()
    if what == "lse":
        more = dict(lse=torch.empty((2, 3), device="cuda"))
    if what == "o on q":
        more = dict(o=q)
    with pytest.raises((ValueError, kb.KbError)):
        kb.kb_attn_paged(q, kc, vc, table, lens, starts, **more)
