"""The reference operators captured in a HIP graph (GPU)."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nk", [(70, 70), (1, 3000)])
def test_operators_in_a_captured_graph(nq, nk):
    """Layer norm and attention, forward and backward, recorded once and replayed: with new inputs in place, eager work
    and synchronizations between the replays, each gives the bits of the eager calls."""
    ensure_built()
    b, h, hk, d = 2, 4, 2, 64
    gen = torch.Generator(device="cuda").manual_seed(5)

    def make(*shape, dtype=torch.float16):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)
    x, w, bias, dy = make(33, 200), make(200), make(200), make(33, 200)
    q, do, k, v = make(b, h, nq, d), make(b, h, nq, d), make(b, hk, nk, d), make(b, hk, nk, d)
    f32 = dict(dtype=torch.float32, device="cuda")
    y, mean, rstd, dx = torch.empty_like(x), torch.empty(33, **f32), torch.empty(33, **f32), torch.empty_like(x)
    dw, db, o, lse = torch.empty_like(w), torch.empty_like(w), torch.empty_like(q), torch.empty((b, h, nq), **f32)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)

    def space(n):
        return torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    nws, fws = space(kb.kb_norm_backward_workspace_bytes(33, 200)), space(kb.kb_attn_forward_workspace_bytes(q, k))
    bws = space(kb.kb_attn_backward_workspace_bytes(q, k))
    outs = (y, mean, rstd, dx, dw, db, o, lse, dq, dk, dv)

    def calls():
        kb.kb_norm_forward(x, w, bias, y=y, mean=mean, rstd=rstd)
        kb.kb_norm_backward(dy, x, w, mean, rstd, dx=dx, dw=dw, db=db, workspace=nws)
        kb.kb_attn_forward(q, k, v, causal=True, o=o, lse=lse, workspace=fws)
        kb.kb_attn_backward(do, q, k, v, o, lse, causal=True, dq=dq, dk=dk, dv=dv, workspace=bws)
    calls()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        for t in (x, dy, q, k, v, do):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        calls()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(outs, want):
            assert torch.equal(a, c), i
