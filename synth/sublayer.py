"""One attention sublayer as a screening workload: its reference outputs are
computed on the device by the library's operators, and candidates' outputs are
screened against them in one multi-output call.

The sublayer normalises x [batch][len][(heads + 2 kv_heads) dim] over its last
axis and attends with the columns of the result as queries, keys and values
(views of one buffer, as a fused projection leaves them).  Backward, dq, dk and
dv are written into the columns of one buffer, which is the gradient that the
layer norm's backward pass takes: no copy between the calls.

    python -m synth.sublayer     (on the GPU: builds, screens, prints the verdicts)
"""
from dataclasses import dataclass

# purposes of the seeded streams, beside those of the screening workloads
WORKLOAD = 6 << 8
X, W, B, DO, NOISE = range(5)


@dataclass
class Sublayer:
    o: "object"      # [batch][len][heads dim]
    lse: "object"    # [batch][heads][len]
    dx: "object"     # x's shape
    dw: "object"     # x's last axis
    db: "object"
    inputs: dict     # x, w, b, do: what a candidate is given

    @property
    def outputs(self):
        """The outputs that a candidate returns, in the order of a screening call."""
        return [self.o, self.dx, self.dw, self.db]


def inputs(batch, length, heads, kv_heads, dim, dtype, wdtype=None, seed=0, device="cuda:0"):
    """x, w, b and the gradient of o, from the library's seeded generator."""
    import torch

    import paper_2608_02611_amd as kb
    wide = (heads + 2 * kv_heads) * dim

    def make(shape, dt, purpose, mean=0.0, sigma=1.0):
        t = torch.empty(shape, dtype=dt, device=device)
        return kb.kb_gen_inputs(t, kb.KB_DIST_NORMAL, mean, sigma, seed=seed, stream_id=WORKLOAD | purpose)
    return dict(x=make((batch, length, wide), dtype, X, 0.25), w=make((wide,), wdtype or dtype, W, 1.0, 0.1),
                b=make((wide,), wdtype or dtype, B, 0.0, 0.1), do=make((batch, length, heads * dim), dtype, DO))


def columns(t, heads, kv_heads, dim):
    """The query, key and value columns of t [batch][len][(heads + 2 kv_heads) dim], as [batch][heads][len][dim]."""
    return [part.unflatten(-1, (-1, dim)).transpose(1, 2)
            for part in t.split([heads * dim, kv_heads * dim, kv_heads * dim], -1)]


def reference(given, heads, kv_heads, dim, causal=True, lens=None, eps=1e-5, stream=None):
    """The sublayer's outputs for inputs(); lens: int32 [batch] device tensor of sequence lengths, or None.
    With a stream, its caller has ordered it after the inputs."""
    import torch

    import paper_2608_02611_amd as kb
    x, w, b, do = (given[name] for name in ("x", "w", "b", "do"))
    y, mean, rstd = kb.kb_norm_forward(x, w, b, eps, stream=stream)
    q, k, v = columns(y, heads, kv_heads, dim)
    with torch.cuda.stream(stream):
        o, dy = torch.empty_like(do), torch.empty_like(x)
    o_heads, do_heads = (t.unflatten(-1, (heads, dim)).transpose(1, 2) for t in (o, do))
    _, lse = kb.kb_attn_forward(q, k, v, causal=causal, q_lens=lens, k_lens=lens, o=o_heads, stream=stream)
    dq, dk, dv = columns(dy, heads, kv_heads, dim)
    kb.kb_attn_backward(do_heads, q, k, v, o_heads, lse, causal=causal, q_lens=lens, k_lens=lens, dq=dq, dk=dk, dv=dv,
                        stream=stream)
    dx, dw, db = kb.kb_norm_backward(dy, x, w, mean, rstd, stream=stream)
    return Sublayer(o, lse, dx, dw, db, given)


def candidates(ref, spreads, seed=0):
    """Candidate k: the reference outputs times 1 + U(-spreads[k], spreads[k]), an implementation's rounding noise."""
    import torch

    import paper_2608_02611_amd as kb
    out = []
    for k, s in enumerate(spreads):
        row = []
        for n, t in enumerate(ref.outputs):
            c = torch.empty_like(t)
            row.append(kb.kb_gen_perturb(c, t, kb.KB_PERTURB_REL_UNIFORM, -s, s, 0.0, seed=seed,
                                         stream_id=WORKLOAD | NOISE, sub=4 * k + n))
        out.append(row)
    return out


def main():
    import torch

    import paper_2608_02611_amd as kb
    heads, kv_heads, dim = 32, 8, 128
    given = inputs(2, 2048, heads, kv_heads, dim, torch.bfloat16, torch.float32)
    lens = torch.tensor([2048, 1500], dtype=torch.int32, device="cuda:0")
    ref = reference(given, heads, kv_heads, dim, lens=lens)
    spreads = [2.0 ** -9, 2.0 ** -7, 2.0 ** -5, 2.0 ** -3]
    records, _, passed = kb.screen_multi(ref.outputs, candidates(ref, spreads), 2.0 ** -10, 2.0 ** -6)
    for k, s in enumerate(spreads):
        wrong = {name: records[n][k]["mismatches"] for n, name in enumerate(("o", "dx", "dw", "db"))}
        print("candidate %d, relative noise %.4f: %s, mismatches %s" % (k, s, "passed" if passed[k] else "failed", wrong))


if __name__ == "__main__":
    main()
