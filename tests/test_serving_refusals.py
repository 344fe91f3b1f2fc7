"""A serving step that is refused changes nothing: host counts and device lengths stay equal, and the next step is the one
that an untouched cache takes."""
import pytest
import torch

import paper_2608_02611_amd as kb
from synth import serving
from tests.helpers import ensure_built

HEADS, KV, DIM = 4, 2, 32


def refuse(to, new, device, tokens=None):
    """A step that has to raise, with nothing changed."""
    counts, lens = list(to.counts), to.lens.clone()
    w = [torch.ones(DIM, device=device) for _ in range(2)]
    x = torch.zeros((sum(new) if tokens is None else tokens, (HEADS + 2 * KV) * DIM), device=device)
    with pytest.raises((ValueError, kb.KbError)):
        serving.step(x, new, to, w, torch.ones(DIM // 2, device=device), HEADS, KV, DIM)
    assert to.counts == counts and torch.equal(to.lens, lens)


@pytest.mark.parametrize("new", [[3, 5, 11], [0, 0, 99], [3, 11, 5], [1, 2], [1], [1, 2, 3, 4], [2, -1, 3]])
def test_no_room_or_not_its_sequences(new):
    """The third, or an earlier sequence has no room, there are fewer or more sequences, or less than no token."""
    to = serving.cache(3, 10, 5, KV, DIM, torch.float32, device="cpu")
    refuse(to, new, "cpu")


def test_no_room_later():
    to = serving.cache(3, 10, 5, KV, DIM, torch.float32, device="cpu")
    to.counts, to.lens = [9, 2, 8], torch.tensor([9, 2, 8], dtype=torch.int32)
    refuse(to, [1, 1, 3], "cpu")


@pytest.mark.gpu
def test_the_next_step_is_an_untouched_caches():
    ensure_built()
    w, freqs = serving.weights(DIM, torch.float32), serving.frequencies(DIM)
    one, other = (serving.cache(3, 40, 16, KV, DIM, torch.float32) for _ in range(2))
    for n, new in enumerate([[20, 7, 30], [4, 4, 4], [1, 1, 1]]):
        refuse(one, [1, 1, 49], "cuda")  # (there is room for 48)
        refuse(one, [2, 2, 2], "cuda", tokens=5)  # x has other tokens: a later call refuses
        refuse(one, [1, 1], "cuda")
        x = serving.projected(sum(new), HEADS, KV, DIM, torch.float32, sub=n)
        got, want = (serving.step(x, new, to, w, freqs, HEADS, KV, DIM) for to in (one, other))
        assert torch.equal(got, want) and one.counts == other.counts == one.lens.tolist()
    assert torch.equal(one.k, other.k) and torch.equal(one.v, other.v)
