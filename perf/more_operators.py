"""Performance cases of the reference operators around a paged key-value cache, each through its public entry point.

Between the projection of an attention sublayer and its output lie four kernels
that a search works on and whose reference outputs these operators compute: the
norms of queries and keys with the position rotation, forward and backward, the
write of new keys and values into a paged cache, and the attention of new tokens
over that cache.  A case is a dict of plain values.  `op` names the call:

  qk_norm_forward   every head row of q [tokens][heads][dim] and k
                    [tokens][kv_heads][dim] times weight / its root mean square,
                    then its first `rot` elements rotated in pairs by position
                    times frequency;
  qk_norm_backward  dq, dk and the weights' gradients from those of the outputs;
  cache_write       the new tokens' rows of k and v to their places in the pages;
  attn_paged        o and lse of softmax(scale q k^T) v for the new tokens, the
                    last of their sequences, over the sequences' pages.

`pairs` says which elements rotate together: "halves" (i, i + rot / 2) or
"neighbours" (2i, 2i + 1).  `layout` says how a page lies in memory: "nhd"
[page size][kv_heads][dim] or "hnd" [kv_heads][page size][dim].  A batch has
`batch` sequences of up to `keys` keys, shorter ones down to a small part where
`ragged`; `new` tokens of each are new (0: all of them), packed one sequence
behind the other.  A sequence's pages lie anywhere in the cache.
"""
import math

import torch

own = False

DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
BASE = 500000.0


def listed():
    return [
        # one decoding step of a small batch: the call's latency
        dict(name="qk_fwd_tokens_bf16", op="qk_norm_forward", dtype="bf16", wdtype="bf16", tokens=16, heads=32, kv_heads=8,
             dim=128, rot=128, pairs="halves", far=131072),
        # the activations of a training batch, 8 sequences of 2048
        dict(name="qk_fwd_batch_f16", op="qk_norm_forward", dtype="f16", wdtype="f16", tokens=8 * 2048, heads=32, kv_heads=8,
             dim=128, rot=128, pairs="halves", far=2048),
        # 32-bit references at an odd length, half of a head's elements rotated, as neighbours
        dict(name="qk_fwd_partial_f32", op="qk_norm_forward", dtype="f32", wdtype="f32", tokens=4095, heads=12, kv_heads=12,
             dim=96, rot=48, pairs="neighbours", far=4095),
        # the gradient over a training batch, master weights in 32 bits
        dict(name="qk_bwd_batch_bf16", op="qk_norm_backward", dtype="bf16", wdtype="f32", tokens=8 * 2048, heads=32,
             kv_heads=8, dim=128, rot=128, pairs="halves", far=2048),
        # a small batch, as a search's first screens use, with shared heads
        dict(name="qk_bwd_small_f32", op="qk_norm_backward", dtype="f32", wdtype="f32", tokens=257, heads=16, kv_heads=4,
             dim=80, rot=40, pairs="halves", far=65536),
        # one decoding step's keys and values, each into the page of its own sequence
        dict(name="write_tokens_bf16", op="cache_write", dtype="bf16", layout="nhd", batch=64, kv_heads=8, dim=128, page=16,
             keys=4096, new=1, ragged=True),
        # the keys and values of prompts that have just arrived, of different lengths
        dict(name="write_prompts_f16", op="cache_write", dtype="f16", layout="hnd", batch=8, kv_heads=8, dim=128, page=64,
             keys=8191, new=0, ragged=True),
        # the smallest call: one token of one short sequence
        dict(name="attn_token_short_f32", op="attn_paged", dtype="f32", layout="nhd", batch=1, heads=8, kv_heads=8, dim=64,
             page=16, keys=200, new=1, ragged=False),
        # one decoding step of a serving batch, lengths from short to long
        dict(name="attn_tokens_bf16", op="attn_paged", dtype="bf16", layout="nhd", batch=64, heads=32, kv_heads=8, dim=128,
             page=16, keys=8191, new=1, ragged=True),
        # one decoding step of a single long sequence: few rows, one long axis
        dict(name="attn_token_long_f16", op="attn_paged", dtype="f16", layout="hnd", batch=1, heads=32, kv_heads=8, dim=128,
             page=128, keys=131071, new=1, ragged=False),
        # a few drafted tokens of each sequence checked at once
        dict(name="attn_drafts_bf16", op="attn_paged", dtype="bf16", layout="hnd", batch=32, heads=32, kv_heads=8, dim=128,
             page=32, keys=4000, new=5, ragged=True),
        # whole prompts of different lengths, packed, that the cache already holds
        dict(name="attn_prompts_bf16", op="attn_paged", dtype="bf16", layout="nhd", batch=6, heads=32, kv_heads=8, dim=128,
             page=64, keys=4095, new=0, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["qk_norm_forward", "qk_norm_backward", "cache_write", "attn_paged", "attn_paged", "attn_paged"])
    most = {k: max(work(c)[k] for c in listed() if c["op"] == op) for k in ("bytes", "flops")}
    while True:
        kv_heads = rng.choice([1, 2, 4, 8, 12, 16])
        heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 8) if kv_heads * g <= 32])
        c = dict(op=op, dtype=rng.choice(["f32", "f16", "bf16"]), kv_heads=kv_heads, dim=rng.choice([40, 64, 80, 96, 128, 128]))
        if op.startswith("qk"):
            c.update(wdtype=rng.choice([c["dtype"], "f32"]), heads=heads, tokens=_log_int(rng, 1, 16384),
                     rot=rng.choice([c["dim"], c["dim"], c["dim"] // 2]), pairs=rng.choice(["halves", "halves", "neighbours"]),
                     far=_log_int(rng, 2048, 1 << 20))
        else:
            kind = rng.choice(["token", "token", "drafts", "piece", "prompt"])
            keys = _log_int(rng, 16, 16384)
            new = {"token": 1, "drafts": min(keys, rng.randint(2, 8)), "piece": min(keys, _log_int(rng, 9, 512)), "prompt": 0}[kind]
            c.update(layout=rng.choice(["nhd", "hnd"]), batch=_log_int(rng, 1, 64), page=rng.choice([8, 16, 16, 32, 64, 128, 256]),
                     keys=keys, new=new, ragged=rng.random() < 0.75)
            if op == "attn_paged":
                c["heads"] = heads
                # scores and what is made of them in the plain form stay within a few GiB a sequence
                if max(q * k for q, k in _lens(c)) * heads > 1 << 29:
                    continue
        w = work(c)
        # 32-bit products take eight times as long as 16-bit ones
        if w["bytes"] <= most["bytes"] and w["flops"] * (8 if op == "attn_paged" and c["dtype"] == "f32" else 1) <= most["flops"]:
            return c


# ------------------------------------------------------------------ inputs ---

def _lens(case):
    """Each sequence's (new tokens, keys with them): the first has all, the others of a ragged batch less."""
    out = []
    for i in range(case["batch"]):
        part = (1.0 - ((7 * i) % case["batch"]) / case["batch"]) ** 2 if case["ragged"] else 1.0
        n = max(1, int(case["keys"] * part))
        out.append((min(n, case["new"]) if case["new"] else n, n))
    return out


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(0x9A6E + 104729 * int(seed))


def _normal(g, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(DT[dtype])


def _cache(g, case, pages, fill):
    """A view [pages][kv_heads][page size][dim] in the case's memory layout."""
    p, h, n, d = pages, case["kv_heads"], case["page"], case["dim"]
    shape = (p, n, h, d) if case["layout"] == "nhd" else (p, h, n, d)
    t = _normal(g, shape, case["dtype"]) if fill else torch.zeros(shape, dtype=DT[case["dtype"]], device=DEV)
    return t.transpose(1, 2) if case["layout"] == "nhd" else t


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pages(g, case, s):
    """The page table of the batch, its pages in any order, and the sequences' lengths."""
    lens = _lens(case)
    counts = [(n + case["page"] - 1) // case["page"] for _, n in lens]
    total, width = sum(counts) + 3, max(counts)
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    s["table"] = torch.zeros((case["batch"], width), dtype=torch.int32, device=DEV)
    first = 0
    for b, n in enumerate(counts):
        s["table"][b, :n] = order[first:first + n]
        first += n
    s["lens"] = _int([n for _, n in lens])
    ends = [0]
    for q, _ in lens:
        ends.append(ends[-1] + q)
    # one token of each sequence needs no starts
    s["starts"] = None if ends[-1] == case["batch"] else _int(ends)
    return total, ends[-1]


def prepare(case, seed):
    g = _gen(seed)
    op, dtype, d = case["op"], case["dtype"], case["dim"]
    s = dict(case=case)
    if op.startswith("qk"):
        n, h, kv = case["tokens"], case["heads"], case["kv_heads"]
        # the columns of one projection: queries, keys and values beside each other
        spread = torch.exp(0.5 * torch.randn((h + 2 * kv) * d, generator=g, device=DEV))
        x = torch.randn((n, (h + 2 * kv) * d), generator=g, device=DEV).mul_(spread).to(DT[dtype])
        s["q"] = x[:, :h * d].unflatten(1, (h, d))
        s["k"] = x[:, h * d:(h + kv) * d].unflatten(1, (kv, d))
        s["wq"], s["wk"] = ((1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(DT[case["wdtype"]]) for _ in range(2))
        s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device=DEV, dtype=torch.int32)
        i = torch.arange(case["rot"] // 2, device=DEV, dtype=torch.float64)
        s["freqs"] = (BASE ** (-2.0 * i / case["rot"])).float()
        new = lambda heads: torch.empty((n, heads, d), dtype=DT[dtype], device=DEV)  # noqa: E731
        if op == "qk_norm_forward":
            s["q_out"], s["k_out"] = new(h), new(kv)
        else:
            s["dq_out"], s["dk_out"] = _normal(g, (n, h, d), dtype), _normal(g, (n, kv, d), dtype)
            dx = torch.zeros_like(x)  # the gradient of the projection, its columns filled in by each operator
            s["dq"], s["dk"] = dx[:, :h * d].unflatten(1, (h, d)), dx[:, h * d:(h + kv) * d].unflatten(1, (kv, d))
            s["dwq"], s["dwk"] = torch.empty_like(s["wq"]), torch.empty_like(s["wk"])
        return s
    pages, tokens = _pages(g, case, s)
    s["k_cache"], s["v_cache"] = (_cache(g, case, pages, op == "attn_paged") for _ in range(2))
    if op == "cache_write":
        s["k"], s["v"] = (_normal(g, (tokens, case["kv_heads"], d), dtype) for _ in range(2))
        return s
    s["scale"] = d ** -0.5
    s["q"] = _normal(g, (tokens, case["heads"], d), dtype, 1.5)
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(s["q"].shape[:2], device=DEV)
    return s


# ------------------------------------------------------------- plain forms ---

def _angles(s):
    """cos and sin [tokens][1][rot / 2] of position times frequency: the product in 64 bits, positions reach far."""
    a = s["positions"].double()[:, None, None] * s["freqs"].double()
    return torch.cos(a).float(), torch.sin(a).float()


def _split(x, case):
    """The two elements of each rotating pair, and the elements that do not rotate."""
    r = case["rot"]
    if case["pairs"] == "halves":
        return x[..., :r // 2], x[..., r // 2:r], x[..., r:]
    return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]


def _joined(a, b, rest, case):
    pair = torch.cat((a, b), -1) if case["pairs"] == "halves" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((pair, rest), -1)


def _rms(x):
    return 1.0 / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)


def _plain_qk_norm_forward(s):
    case = s["case"]
    cos, sin = _angles(s)
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        x = x.float()
        a, b, rest = _split(x * _rms(x) * w.float(), case)
        out.append(_joined(a * cos - b * sin, b * cos + a * sin, rest, case).to(s["q"].dtype))
    return tuple(out)


def _plain_qk_norm_backward(s):
    case = s["case"]
    cos, sin = _angles(s)
    grads, weights = [], []
    for dy, x, w in ((s["dq_out"], s["q"], s["wq"]), (s["dk_out"], s["k"], s["wk"])):
        x = x.float()
        a, b, rest = _split(dy.float(), case)
        g = _joined(a * cos + b * sin, b * cos - a * sin, rest, case)
        r = _rms(x)
        z, u = x * r, g * w.float()
        grads.append((r * (u - z * ((u * z).sum(-1, keepdim=True) / x.shape[-1]))).to(s["q"].dtype))
        weights.append((g * z).sum((0, 1)).to(w.dtype))
    return tuple(grads + weights)


def _plain_cache_write(s):
    n, page = s["k"].shape[0], s["case"]["page"]
    token = torch.arange(n, device=DEV)
    if s["starts"] is None:
        seq, place = token, s["lens"].long() - 1
    else:
        ends = s["starts"][1:].long()
        seq = (token[:, None] >= ends[None, :]).sum(1)
        place = s["lens"].long()[seq] - ends[seq] + token
    at = s["table"][seq, place // page].long()
    s["k_cache"][at, :, place % page] = s["k"]
    s["v_cache"][at, :, place % page] = s["v"]
    return s["k_cache"], s["v_cache"]


def _matmul(a, b):
    """a b over the last two axes, in 32 bits, with a right operand that lies in rows."""
    return torch.matmul(a.contiguous(), b.contiguous())


def _attend(q, k, v, scale, hidden):
    """q [..][rows][dim] on k, v [..][keys][dim]; hidden: true where a row may not see a key."""
    scores = _matmul(q, k.transpose(-1, -2)).mul_(scale)
    if hidden is not None:
        scores.masked_fill_(hidden, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp_(scores.sub_(top))
    total = p.sum(-1, keepdim=True)
    return _matmul(p, v) / total, (top + torch.log(total))[..., 0]


def _plain_attn_paged(s):
    case = s["case"]
    kv, d, page = case["kv_heads"], case["dim"], case["page"]
    grp, dtype = case["heads"] // kv, s["q"].dtype
    if s["starts"] is None:  # one token of each sequence: all of them at once, padded to the longest
        k, v = (t[s["table"]].transpose(1, 2).reshape(case["batch"], kv, -1, d).float() for t in (s["k_cache"], s["v_cache"]))
        hidden = (torch.arange(k.shape[2], device=DEV)[None, :] >= s["lens"][:, None])[:, None, None, :]
        o, lse = _attend(s["q"].float().reshape(case["batch"], kv, grp, d), k, v, s["scale"], hidden)
        return o.reshape(s["q"].shape).to(dtype), lse.reshape(s["q"].shape[:2])
    outs, norms, first = [], [], 0
    for b, (nq, nk) in enumerate(_lens(case)):
        at = s["table"][b, :(nk + page - 1) // page]
        k, v = (t[at].transpose(0, 1).reshape(kv, -1, d)[:, :nk].float() for t in (s["k_cache"], s["v_cache"]))
        q = s["q"][first:first + nq].float().reshape(nq, kv, grp, d).permute(1, 2, 0, 3).reshape(kv, grp * nq, d)
        i = torch.arange(nq, device=DEV).repeat(grp)
        hidden = torch.arange(nk, device=DEV)[None, :] > i[:, None] + (nk - nq)
        o, lse = _attend(q, k, v, s["scale"], hidden)
        outs.append(o.reshape(kv * grp, nq, d).transpose(0, 1).to(dtype))
        norms.append(lse.reshape(kv * grp, nq).transpose(0, 1))
        first += nq
    return torch.cat(outs), torch.cat(norms)


PLAIN = {"qk_norm_forward": _plain_qk_norm_forward, "qk_norm_backward": _plain_qk_norm_backward,
         "cache_write": _plain_cache_write, "attn_paged": _plain_attn_paged}


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return PLAIN[op](s)
    import paper_2608_02611_amd as kb
    if op == "cache_write":
        return kb.kb_cache_write(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["starts"])
    if op == "attn_paged":
        return kb.kb_attn_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["starts"], s["scale"],
                                causal=True, o=s["o"], lse=s["lse"])
    interleaved = s["case"]["pairs"] == "neighbours"
    if op == "qk_norm_forward":
        return kb.kb_qk_norm_forward(s["q"], s["k"], s["wq"], s["wk"], EPS, s["positions"], s["freqs"], interleaved,
                                     q_out=s["q_out"], k_out=s["k_out"])
    return kb.kb_qk_norm_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["wq"], s["wk"], EPS, s["positions"],
                                  s["freqs"], interleaved, dq=s["dq"], dk=s["dk"], dwq=s["dwq"], dwk=s["dwk"])


# -------------------------------------------------------------------- work ---

def _seen(case):
    """(query, key) pairs that are seen, over the batch, for one head: query i sees i + 1 + keys - queries."""
    return sum(q * (k - q) + q * (q + 1) // 2 for q, k in _lens(case))


def work(case):
    op, size, d = case["op"], SIZE[case["dtype"]], case["dim"]
    if op.startswith("qk"):
        n, wsize = case["tokens"] * (case["heads"] + case["kv_heads"]) * d, SIZE[case["wdtype"]]
        table = 4 * case["tokens"] + 2 * case["rot"]
        if op == "qk_norm_forward":
            return {"bytes": 2 * n * size + 2 * d * wsize + table, "flops": 8 * n}
        return {"bytes": 3 * n * size + 4 * d * wsize + table, "flops": 14 * n}
    lens, kv = _lens(case), case["kv_heads"]
    tokens = sum(q for q, _ in lens)
    if op == "cache_write":
        return {"bytes": 4 * tokens * kv * d * size + 8 * case["batch"], "flops": 0}
    keys = sum(k for _, k in lens)
    rows = tokens * case["heads"]
    return {"bytes": 2 * rows * d * size + 4 * rows + 2 * keys * kv * d * size + 4 * sum(-(-k // case["page"]) for _, k in lens),
            "flops": 4 * _seen(case) * case["heads"] * d}


# ------------------------------------------------------------ exact values ---

def _exact_rotation(case, s):
    """The rotation of each token as complex numbers [tokens][1][rot / 2]."""
    a = torch.einsum("t,f->tf", s["positions"].double(), s["freqs"].double())[:, None]
    return torch.polar(torch.ones_like(a), a)


def _as_complex(x, case):
    r = case["rot"]
    order = torch.arange(r, device=DEV)
    order = order.view(2, -1).T if case["pairs"] == "halves" else order.view(-1, 2)
    return order, torch.view_as_complex(x[..., order].contiguous())


def _turned(x, turn, case):
    order, z = _as_complex(x, case)
    out = x.clone()
    out[..., order.reshape(-1)] = torch.view_as_real(z * turn).flatten(-2)
    return out


def _exact_qk(s, case):
    turn = _exact_rotation(case, s)
    d = case["dim"]
    res, extra = [], []
    for name, w in (("q", s["wq"].double()), ("k", s["wk"].double())):
        x = s[name].double()
        sd = (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        if case["op"] == "qk_norm_forward":
            res.append(_turned(x / sd * w, turn, case))
            continue
        # back through the rotation, whose transpose turns the other way, then the Jacobian (I - z z^T / dim) / sd
        g = _turned(s["d%s_out" % name].double(), turn.conj(), case)
        z, u = x / sd, g * w
        res.append((u - z * torch.einsum("thd,thd->th", u, z)[..., None] / d) / sd)
        extra.append(torch.einsum("thd,thd->d", g, z))
    return tuple(res + extra)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("qk"):
        return _exact_qk(s, case)
    page, table = case["page"], s["table"].tolist()
    if op == "cache_write":
        # a piece of a sequence at a time, as far as its page goes
        out = tuple(t.double() for t in (s["k_cache"], s["v_cache"]))
        first = 0
        for b, (nq, nk) in enumerate(_lens(case)):
            at = nk - nq
            while at < nk:
                n = min(page - at % page, nk - at)
                src = first + at - (nk - nq)
                for to, new in zip(out, (s["k"], s["v"])):
                    to[table[b][at // page], :, at % page:at % page + n] = new[src:src + n].transpose(0, 1).double()
                at += n
            first += nq
        return out
    grp = case["heads"] // case["kv_heads"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    first = 0
    for b, (nq, nk) in enumerate(_lens(case)):
        pages = table[b][:(nk + page - 1) // page]
        seen = torch.ones((nq, nk), dtype=torch.bool, device=DEV).tril(nk - nq)
        for h in range(case["kv_heads"]):
            k, v = (t[pages, h].reshape(-1, case["dim"])[:nk].double() for t in (s["k_cache"], s["v_cache"]))
            for j in range(h * grp, (h + 1) * grp):
                t = (s["q"][first:first + nq, j].double() @ k.T) * s["scale"]
                t = torch.where(seen, t, torch.full_like(t, -math.inf))
                norm = torch.logsumexp(t, 1)
                o[first:first + nq, j], lse[first:first + nq, j] = torch.exp(t - norm[:, None]) @ v, norm
        first += nq
    return o, lse
