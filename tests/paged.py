"""Paged caches for the tests: sequences laid out over pages in any order, and the formulas in 64 bits."""
import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
E = 2.0 ** -24


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


class Batch:
    """Sequences of (new tokens, keys) over pages of `page` keys.  Places that are no sequence's hold NaN, table entries
    past a sequence's pages numbers that are no page's, and rows of the table lie apart.  before, after: tokens of no
    sequence.  one: no starts (every sequence has one new token)."""

    def __init__(self, seqs, page, heads, kv_heads, dim, dtype, layout="nhd", seed=0, before=0, after=0, one=False,
                 width=None, spare=2):
        t = DT[dtype]
        self.seqs, self.page, self.heads, self.kv, self.dim, self.before = seqs, page, heads, kv_heads, dim, before
        counts = [-(-n // page) for _, n in seqs]
        total = sum(counts) + spare
        g = torch.Generator().manual_seed(seed)
        order = torch.randperm(total, generator=g).tolist()
        width = max([width or 0] + counts + [1])
        # (the caches have fewer than 2^28 pages)
        table = torch.full((len(seqs), width + 3), 2 ** 31 - 1, dtype=torch.int32)
        table[:, ::2] = -5
        at = 0
        for b, n in enumerate(counts):
            table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.table = table.cuda()[:, :width]
        self.lens = ints([n for _, n in seqs])
        ends = [before]
        for q, _ in seqs:
            ends.append(ends[-1] + q)
        self.ends = ends
        self.starts = None if one else ints(ends)
        tokens = ends[-1] + after
        shape = (total, page, kv_heads, dim) if layout == "nhd" else (total, kv_heads, page, dim)
        turned = (lambda x: x.transpose(1, 2)) if layout == "nhd" else (lambda x: x)
        self.k_cache, self.v_cache = (turned(torch.full(shape, float("nan"), dtype=t, device="cuda")) for _ in range(2))
        self.keys, self.values = [], []
        for b, (_, n) in enumerate(seqs):
            for i, (cache, kept) in enumerate(((self.k_cache, self.keys), (self.v_cache, self.values))):
                x = normal((n, kv_heads, dim), t, seed + 100 * b + i + 1)
                kept.append(x)
                place = torch.arange(n, device="cuda")
                cache[self.table[b, place // page].long(), :, place % page] = x
        self.q = normal((tokens, heads, dim), t, seed + 7, 1.5)

    @property
    def pages(self):
        return self.table, self.lens, self.starts


def exact(batch, scale, causal, missing=()):
    """For each sequence (first token, o, lse, p, magnitudes of p |v|, of the scores): lists by head.  missing: keys
    (b, j) without a page."""
    grp = batch.heads // batch.kv
    for b, (nq, nk) in enumerate(batch.seqs):
        if nq == 0:
            continue
        first = batch.ends[b]
        seen = torch.ones((nq, nk), dtype=torch.bool, device="cuda")
        if causal:
            seen = seen.tril(nk - nq)
        for s, j in missing:
            if s == b:
                seen[:, j] = False
        for h in range(batch.heads):
            q = batch.q[first:first + nq, h].double()
            k, v = batch.keys[b][:, h // grp].double(), batch.values[b][:, h // grp].double()
            s = torch.where(seen, (q @ k.T) * scale, float("-inf"))
            lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), float("-inf"), dtype=torch.float64, device="cuda")
            p = torch.where(seen, torch.exp(s - lse[:, None]), 0.0)
            p = torch.where((lse == float("-inf"))[:, None], 0.0, p)
            top = float(((q.abs() @ k.abs().T) * scale).max()) if nk else 0.0
            yield first, nq, nk, h, p, p @ v, lse, p @ v.abs(), top, v


def close(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol) & ~(want == got)
    assert not bad.any(), "%s: %d of %d off, worst %.3g of the tolerance" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol)[bad].max()))


def check(batch, scale, causal, o, lse, missing=()):
    """o and lse against 64 bits.  A score is a sum of D products in 32 bits, scaled and shifted and taken to a power: its
    term is off by ES = (D + 16) E A + 4 E of itself, A the largest scaled sum of |q| |k|.  A term is rounded for its
    product: by u, or with few rows a sequence, where it goes in two parts, u^2 (F16: or 2^-34 of the row's largest).  A
    sum of n terms in 32 bits is off by n E of the magnitudes, twice (product and sum); the result is rounded once."""
    t = batch.q.dtype
    few = batch.q.shape[0] * (batch.heads // max(1, batch.kv)) <= 32 * len(batch.seqs)
    u = U[t]
    up = 2.0 ** -24 if t == torch.float32 else u * u if few else u
    for first, nq, nk, h, p, want, norm, mag, top, v in exact(batch, scale, causal, missing):
        es = (batch.dim + 16) * E * top + 4 * E
        empty = norm == float("-inf")
        go, gl = o[first:first + nq, h], lse[first:first + nq, h]
        assert torch.all(go[empty] == 0) and torch.all(gl[empty] == float("-inf"))
        tol = (2 * up + 2 * es + 2 * nk * E) * mag + 1.01 * u * want.abs() + TINY[t]
        if t == torch.float16 and nk:
            tol = tol + nk * 2.0 ** -34 * v.abs().max()
        close(go, want, tol, "o")
        close(gl[~empty], norm[~empty], es + nk * E + 4 * E * norm[~empty].abs() + E, "lse")
