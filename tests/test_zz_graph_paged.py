"""Head norms, cache writes and attention over pages captured in a HIP graph (GPU)."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.paged import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 3, 60])
def test_a_serving_step_in_a_captured_graph(new):
    """Recorded once and replayed as the sequences grow: with new inputs and lengths in place, eager work and
    synchronizations between the replays, each gives the bits of the eager calls.  One token each, in parts, a few, and
    many, in parts."""
    ensure_built()
    batch, h, hk, d, page, width = 3, 8, 2, 64, 16, 120
    gen = torch.Generator(device="cuda").manual_seed(5)
    tokens = batch * new
    # (defined values from the first call on: what it writes stays in the cache)
    x = torch.randn((tokens, (h + 2 * hk) * d), generator=gen, device="cuda").half()
    q, k, v = (t.unflatten(1, (-1, d)) for t in x.split([h * d, hk * d, hk * d], 1))
    dx, dy = torch.zeros_like(x), torch.randn((tokens, h, d), generator=gen, device="cuda").half()
    dq, dk, _ = (t.unflatten(1, (-1, d)) for t in dx.split([h * d, hk * d, hk * d], 1))
    w = torch.ones(d, dtype=torch.float32, device="cuda")
    freqs = torch.logspace(0, -4, d // 2, device="cuda")
    lens, positions = ints([5, 900, 1500]), torch.zeros(tokens, dtype=torch.int32, device="cuda")
    table = torch.randperm(batch * width, generator=gen, device="cuda").to(torch.int32).view(batch, width)
    starts = None if new == 1 else torch.arange(0, tokens + 1, new, dtype=torch.int32, device="cuda")
    kc, vc = (torch.randn((batch * width, hk, page, d), generator=gen, device="cuda").half() for _ in range(2))
    qo, ko = torch.empty((tokens, h, d), dtype=torch.float16, device="cuda"), torch.empty((tokens, hk, d), dtype=torch.float16, device="cuda")
    dk_out = torch.randn((tokens, hk, d), generator=gen, device="cuda").half()
    o, lse = torch.empty_like(qo), torch.empty((tokens, h), device="cuda")
    dwq, dwk = torch.empty_like(w), torch.empty_like(w)

    def space(n):
        return torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    ws, bws = space(kb.kb_attn_paged_workspace_bytes(qo, kc, table, lens, starts)), space(kb.kb_qk_norm_backward_workspace_bytes(d))
    outs = (qo, ko, kc, vc, o, lse, dx, dwq, dwk)

    def calls():
        kb.kb_qk_norm_forward(q, k, w, w, 1e-6, positions, freqs, q_out=qo, k_out=ko)
        kb.kb_cache_write(ko, v, kc, vc, table, lens, starts)
        kb.kb_attn_paged(qo, kc, vc, table, lens, starts, o=o, lse=lse, workspace=ws)
        kb.kb_qk_norm_backward(dy, dk_out, q, k, w, w, 1e-6, positions, freqs, dq=dq, dk=dk, dwq=dwq, dwk=dwk, workspace=bws)
    calls()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        for t in (x, dy, dk_out):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        lens += new
        positions.copy_((lens[:, None] - new + torch.arange(new, device="cuda", dtype=torch.int32)).view(-1))
        kept = kc.clone(), vc.clone()
        calls()
        want = [t.clone() for t in outs]
        kc.copy_(kept[0])
        vc.copy_(kept[1])
        for t in (qo, ko, o, lse, dx, dwq, dwk):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(outs, want):
            assert torch.equal(a, c), i
