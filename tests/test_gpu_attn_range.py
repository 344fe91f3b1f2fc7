"""Attention over dense keys with values of any size: finite ones give finite outputs, and an infinity gives itself.

o is a mean of the values that a row sees.  The tolerances are tests/test_gpu_attn.py's, relative to S p |v|; the values are
held at 15/16 of the type's largest at most, so that no rounding of the mean reaches infinity."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_gpu_attn import DT, check_forward, heads, lens_tensor

pytestmark = pytest.mark.gpu

CASES = [
    dict(nq=130, nk=130),
    dict(nq=1, nk=2),
    dict(nq=200, nk=90, q_lens=[200, 17], k_lens=[33, 90]),
    dict(nq=3, nk=4000),                                    # in parts
    dict(nq=70, nk=3000, k_lens=[3000, 5]),
]


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def large(shape, dtype, signs):
    g = torch.Generator(device="cuda").manual_seed(5)
    size = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64) * (11 / 16) + 0.25
    if signs == 2:
        size *= torch.randint(0, 2, shape, generator=g, device="cuda") * 2 - 1
    return (size * torch.finfo(dtype).max).to(dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 96, 128, 33])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("causal,signs", [(True, 2), (False, 1)])
def test_large_values(dtype, d, case, causal, signs):
    t, nq, nk = DT[dtype], case["nq"], case["nk"]
    q, k = heads(2, 4, nq, d, t, 1, 1.5), heads(2, 2, nk, d, t, 2)
    v = large(k.shape, t, signs)
    ql, kl = case.get("q_lens"), case.get("k_lens")
    o, lse = kb.kb_attn_forward(q, k, v, d ** -0.5, causal, lens_tensor(ql), lens_tensor(kl))
    assert torch.isfinite(o).all()
    check_forward(q, k, v, d ** -0.5, causal, ql, kl, o, lse)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq,nk", [(130, 130), (1, 1), (3, 4000)])
@pytest.mark.parametrize("causal", [True, False])
def test_infinite_values(dtype, nq, nk, causal):
    """Of one sign at one key and column, of both at another column."""
    t, d, inf = DT[dtype], 64, float("inf")
    q, k, v = heads(1, 4, nq, d, t, 1, 1.5), heads(1, 2, nk, d, t, 2), heads(1, 2, nk, d, t, 3)
    at = max(0, nk - 2)
    v[0, 0, at, 3], v[0, 0, at, 5] = inf, -inf
    if nk > 1:
        v[0, 0, at, 9], v[0, 0, 0, 9] = inf, -inf
    o, lse = kb.kb_attn_forward(q, k, v, None, causal)
    sees = torch.tensor([not causal or i + nk - nq >= at for i in range(nq)], device="cuda")
    rows = o[0, :2].float()
    assert torch.isfinite(lse).all()
    assert torch.all(rows[:, sees, 3] == inf) and torch.all(rows[:, sees, 5] == -inf)
    assert torch.isfinite(rows[:, ~sees, 3]).all() and torch.isfinite(rows[:, ~sees, 5]).all()
    if nk > 1:
        assert torch.isnan(rows[:, sees, 9]).all() and torch.all(rows[:, ~sees, 9] == -inf)
    o[:, :2, :, [3, 5, 9]] = 0.0
    v[:, 0, :, [3, 5, 9]] = 0.0
    check_forward(q, k, v, d ** -0.5, causal, None, None, o, lse)
