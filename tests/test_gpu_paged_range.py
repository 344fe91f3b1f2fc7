"""Attention over pages with values of any size: finite ones give finite outputs, and an infinity gives itself.

o is a mean of the values that a row sees, so it is finite where they are, however large.  The tolerances are
tests/paged.py's, which are relative to S p |v|; the values are held at 15/16 of the type's largest at most, so that no
rounding of the mean reaches infinity."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.paged import DT, Batch, check, ints

pytestmark = pytest.mark.gpu

FEW = [
    dict(seqs=[(1, 1), (1, 2), (1, 90), (1, 700)], one=True),
    dict(seqs=[(4, 100), (6, 700), (1, 1)]),                     # queries whose keys differ share a block
    dict(seqs=[(1, 5000)], heads=8),                             # one pair in many parts
    dict(seqs=[(1, 9000), (1, 3), (5, 2000)], heads=4),
    dict(seqs=[(1, 600 + 13 * i) for i in range(40)], heads=8, kv=8, one=True),
]
MANY = [
    dict(seqs=[(150, 150), (70, 300)]),
    dict(seqs=[(200, 200), (1, 1), (33, 90), (1, 700)]),
    dict(seqs=[(20, 1500), (9, 3000)]),                          # in parts
    dict(seqs=[(130, 2100), (130, 130)], heads=1, kv=1),
]


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def batch(dtype, dim, page, seqs, heads=4, kv=2, one=False):
    return Batch(seqs, page, heads, kv, dim, dtype, "hnd", one=one)


def put(b):
    """The values of b.values to their places."""
    for s, (_, n) in enumerate(b.seqs):
        place = torch.arange(n, device="cuda")
        b.v_cache[b.table[s, place // b.page].long(), :, place % b.page] = b.values[s]


def enlarge(b, signs, heads=slice(None)):
    """Values of 1/4 to 15/16 of the type's largest in the key heads `heads`, of one sign or of both."""
    most = torch.finfo(b.q.dtype).max
    g = torch.Generator(device="cuda").manual_seed(5)
    for v in b.values:
        size = torch.rand(v.shape, generator=g, device="cuda", dtype=torch.float64) * (11 / 16) + 0.25
        if signs == 2:
            size *= torch.randint(0, 2, v.shape, generator=g, device="cuda") * 2 - 1
        v[:, heads] = (size * most).to(v.dtype)[:, heads]
    put(b)


def attend(b, causal):
    return kb.kb_attn_paged(b.q, b.k_cache, b.v_cache, *b.pages, causal=causal)


def large_values(dtype, dim, page, case, causal, signs):
    b = batch(dtype, dim, page, **case)
    enlarge(b, signs)
    o, lse = attend(b, causal)
    assert torch.isfinite(o).all()
    check(b, b.dim ** -0.5, causal, o, lse)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (128, 5)])
@pytest.mark.parametrize("case", FEW)
@pytest.mark.parametrize("causal,signs", [(True, 2), (False, 1)])
def test_large_values_few_rows(dtype, dim, page, case, causal, signs):
    large_values(dtype, dim, page, case, causal, signs)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (96, 5)])
@pytest.mark.parametrize("case", MANY)
@pytest.mark.parametrize("causal,signs", [(True, 2), (False, 1)])
def test_large_values_many_rows(dtype, dim, page, case, causal, signs):
    large_values(dtype, dim, page, case, causal, signs)


@pytest.mark.parametrize("dtype,value", [("f32", 3e37), ("bf16", 3e37), ("f16", 6e4)])
@pytest.mark.parametrize("page", [8, 16])
def test_a_large_value_after_a_smaller_score(dtype, value, page):
    """A score of 0, then one of 5 whose value is large, in the next tile of the same wave: o = value e^5 / S e^s."""
    t = DT[dtype]
    n = 65
    q = torch.zeros((1, 1, 64), dtype=t, device="cuda")
    k = torch.zeros((-(-n // page), 1, page, 64), dtype=t, device="cuda")
    v = torch.zeros_like(k)
    q[..., 0] = 1.0
    k[64 // page, 0, 64 % page, 0] = 5.0
    v[64 // page, 0, 64 % page] = value
    table = torch.arange(k.shape[0], dtype=torch.int32, device="cuda").view(1, -1)
    o, _ = kb.kb_attn_paged(q, k, v, table, ints([n]), None, 1.0)
    top = torch.tensor(5.0).double().exp().item()
    want = float(torch.tensor(value, dtype=t)) * top / (top + n - 1)
    # the terms by 4 E each and (16 bits) u^2, their sums by 65 E, the result by u
    err = abs(float(o[0, 0, 7]) - want)
    assert err <= want * (torch.finfo(t).eps * 0.5 * 1.01 + 2 * (2.0 ** -16 if t == torch.bfloat16 else 2.0 ** -22) + 150 * 2.0 ** -24)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", FEW[1:3] + MANY[:3])
def test_large_values_leave_other_heads_alone(dtype, case):
    """A key head of ordinary values beside one of large values keeps its bits."""
    b = batch(dtype, 64, 16, **case)
    want, _ = attend(b, True)
    enlarge(b, 1, slice(0, 1))
    got, _ = attend(b, True)
    half = b.heads // 2
    assert torch.equal(got[:, half:], want[:, half:]) and torch.isfinite(got).all()


def infinite(dtype, page, case, causal):
    """Of one sign at one key and column, of both at another column."""
    b = batch(dtype, 64, page, **case)
    grp, inf = b.heads // b.kv, float("inf")
    at = [max(0, n - 2) for _, n in b.seqs]
    for s, (_, n) in enumerate(b.seqs):
        page_of, j = (lambda k: int(b.table[s, k // page])), at[s]
        b.v_cache[page_of(j), 0, j % page, 3] = inf
        b.v_cache[page_of(j), 0, j % page, 5] = -inf
        if n > 1:
            b.v_cache[page_of(j), 0, j % page, 9] = inf
            b.v_cache[page_of(0), 0, 0, 9] = -inf
    o, lse = attend(b, causal)
    assert torch.isfinite(lse).all()
    for s, (nq, nk) in enumerate(b.seqs):
        rows = o[b.ends[s]:b.ends[s + 1], :grp].float()
        sees = torch.tensor([not causal or i + nk - nq >= at[s] for i in range(nq)], device="cuda")
        assert torch.all(rows[sees][..., 3] == inf) and torch.all(rows[sees][..., 5] == -inf)
        assert torch.isfinite(rows[~sees][..., 3]).all() and torch.isfinite(rows[~sees][..., 5]).all()
        if nk > 1 and at[s] > 0:
            assert torch.isnan(rows[sees][..., 9]).all() and torch.all(rows[~sees][..., 9] == -inf)
        rows[..., [3, 5, 9]] = 0.0
        assert torch.isfinite(rows).all()
    for v in b.values:
        v[:, 0, [3, 5, 9]] = 0.0
    o[:, :grp, [3, 5, 9]] = 0.0
    check(b, b.dim ** -0.5, causal, o, lse)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("case", FEW)
@pytest.mark.parametrize("causal", [True, False])
def test_infinite_values_few_rows(dtype, page, case, causal):
    infinite(dtype, page, case, causal)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("case", MANY)
@pytest.mark.parametrize("causal", [True, False])
def test_infinite_values_many_rows(dtype, page, case, causal):
    infinite(dtype, page, case, causal)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [16, 5, 64])
@pytest.mark.parametrize("seqs", [[(1, 200), (3, 2500)], [(100, 200), (70, 700)]])
@pytest.mark.parametrize("causal", [True, False])
def test_large_values_beside_keys_without_a_page(dtype, page, seqs, causal):
    b = batch(dtype, 64, page, seqs)
    enlarge(b, 2)
    missing = []
    for s, (_, n) in enumerate(seqs):
        for i, number in ((0, -1), (1, b.k_cache.shape[0])):
            b.table[s, i] = number
            missing += [(s, j) for j in range(i * page, (i + 1) * page)]
    o, lse = attend(b, causal)
    assert torch.isfinite(o).all()
    check(b, b.dim ** -0.5, causal, o, lse, missing)
