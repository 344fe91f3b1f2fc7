"""A serving attention sublayer as a screening workload: its reference outputs are
computed on the device by the library's operators, prompts first and then single
tokens, and candidates' outputs are screened against them.

A projection leaves x [tokens][(heads + 2 kv_heads) dim] for the new tokens of a
batch, packed one sequence behind the other.  Its query and key columns are
normalised by head and rotated by their positions, keys and values go into the
pages of their sequences, and the queries attend over these.

    python -m synth.serving     (on the GPU: builds, screens, prints the verdicts)
"""
from dataclasses import dataclass, field

# purposes of the seeded streams, beside those of the other workloads
WORKLOAD = 7 << 8
X, WQ, WK, NOISE = range(4)
EPS = 1e-6


@dataclass
class Cache:
    """Pages of a batch: sequence b's key j lies in page table[b][j / page]."""
    k: "object"      # [pages][kv_heads][page][dim]
    v: "object"
    table: "object"  # int32 [batch][max_pages]
    lens: "object"   # int32 [batch]: keys so far
    counts: list = field(default_factory=list)  # the same on the host, which knows what it has sent


def cache(batch, max_keys, page, kv_heads, dim, dtype, device="cuda:0"):
    """An empty cache with room for max_keys keys a sequence, the sequences' pages interleaved."""
    import torch
    width = -(-max_keys // page)
    k, v = (torch.zeros((batch * width, page, kv_heads, dim), dtype=dtype, device=device).transpose(1, 2) for _ in range(2))
    table = torch.arange(batch * width, dtype=torch.int32, device=device).view(width, batch).T.contiguous()
    return Cache(k, v, table, torch.zeros(batch, dtype=torch.int32, device=device), [0] * batch)


def weights(dim, dtype, seed=0, device="cuda:0"):
    """The norms' weights of queries and keys, from the library's seeded generator."""
    import torch

    import paper_2608_02611_amd as kb
    return [kb.kb_gen_inputs(torch.empty(dim, dtype=dtype, device=device), kb.KB_DIST_NORMAL, 1.0, 0.1, seed=seed,
                             stream_id=WORKLOAD | purpose) for purpose in (WQ, WK)]


def projected(tokens, heads, kv_heads, dim, dtype, seed=0, sub=0, device="cuda:0"):
    """x of `tokens` new tokens; sub: another call's."""
    import torch

    import paper_2608_02611_amd as kb
    x = torch.empty((tokens, (heads + 2 * kv_heads) * dim), dtype=dtype, device=device)
    return kb.kb_gen_inputs(x, kb.KB_DIST_NORMAL, 0.0, 1.0, seed=seed, stream_id=WORKLOAD | X, sub=sub)


def frequencies(dim, base=10000.0, device="cuda:0"):
    import torch
    i = torch.arange(dim // 2, dtype=torch.float64, device=device)
    return (base ** (-2.0 * i / dim)).float()


def columns(x, heads, kv_heads, dim):
    """The queries, keys and values of x, as [tokens][heads][dim]."""
    return [part.unflatten(-1, (-1, dim)) for part in x.split([heads * dim, kv_heads * dim, kv_heads * dim], -1)]


def step(x, new, to, w, freqs, heads, kv_heads, dim):
    """The sublayer's output o [tokens][heads][dim] for the `new` tokens of each sequence (a list), whose keys and values
    are added to the cache `to`: whole prompts, pieces of them, or one token each.  A step that raises changes neither
    the cache's counts nor its lengths."""
    import torch

    import paper_2608_02611_amd as kb
    if len(new) != len(to.counts) or min(new, default=0) < 0:
        raise ValueError("new tokens %s for %d sequences" % (new, len(to.counts)))
    counts = [n + m for n, m in zip(to.counts, new)]
    ends, positions = [0], []
    for b, n in enumerate(counts):
        if n > to.table.shape[1] * to.k.shape[2]:
            raise ValueError("sequence %d has no room for %d keys" % (b, n))
        ends.append(ends[-1] + new[b])
        positions += range(to.counts[b], n)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=x.device)
    lens = ints(counts)
    starts = None if all(n == 1 for n in new) else ints(ends)
    q, k, v = columns(x, heads, kv_heads, dim)
    q, k = kb.kb_qk_norm_forward(q, k, w[0], w[1], EPS, ints(positions), freqs)
    kb.kb_cache_write(k, v, to.k, to.v, to.table, lens, starts)
    o, _ = kb.kb_attn_paged(q, to.k, to.v, to.table, lens, starts)
    to.counts[:] = counts
    to.lens.copy_(lens)
    return o


def candidates(refs, spreads, seed=0):
    """Candidate k: the reference outputs times 1 + U(-spreads[k], spreads[k]), an implementation's rounding noise."""
    import torch

    import paper_2608_02611_amd as kb
    return [[kb.kb_gen_perturb(torch.empty_like(t), t, kb.KB_PERTURB_REL_UNIFORM, -s, s, 0.0, seed=seed,
                               stream_id=WORKLOAD | NOISE, sub=len(refs) * k + n) for n, t in enumerate(refs)]
            for k, s in enumerate(spreads)]


def main():
    import torch

    import paper_2608_02611_amd as kb
    heads, kv_heads, dim, dtype = 32, 8, 128, torch.bfloat16
    prompts = [2000, 700, 33, 1]
    to = cache(len(prompts), 2100, 16, kv_heads, dim, dtype)
    w, freqs = weights(dim, dtype), frequencies(dim)
    refs = [step(projected(sum(prompts), heads, kv_heads, dim, dtype), prompts, to, w, freqs, heads, kv_heads, dim)]
    for n in range(3):
        x = projected(len(prompts), heads, kv_heads, dim, dtype, sub=1 + n)
        refs.append(step(x, [1] * len(prompts), to, w, freqs, heads, kv_heads, dim))
    spreads = [2.0 ** -9, 2.0 ** -7, 2.0 ** -5, 2.0 ** -3]
    records, _, passed = kb.screen_multi(refs, candidates(refs, spreads), 2.0 ** -10, 2.0 ** -6)
    for k, s in enumerate(spreads):
        wrong = [records[n][k]["mismatches"] for n in range(len(refs))]
        print("candidate %d, relative noise %.4f: %s, mismatches in the prompts %d, in single tokens %s"
              % (k, s, "passed" if passed[k] else "failed", wrong[0], wrong[1:]))


if __name__ == "__main__":
    main()
