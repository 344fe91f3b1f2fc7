"""Which views of [..., heads, dim] the head norm calls take: leading axes that one stride walks (no GPU needed)."""
import pytest
import torch

import paper_2608_02611_amd as kb


def base(*shape):
    return torch.arange(torch.Size(shape).numel(), dtype=torch.float32).view(shape)


TAKEN = {
    "dense": base(2, 3, 4, 8),
    "five axes": base(2, 3, 5, 4, 8),
    "one token": base(4, 8),
    "columns of a projection": base(2, 3, 96)[..., 32:64].unflatten(-1, (4, 8)),
    "some heads": base(2, 3, 6, 8)[:, :, 1:5],
    "a batch of one, its heads outside": base(1, 4, 3, 8).transpose(1, 2),
    "single tokens, their heads outside": base(3, 4, 1, 8).transpose(1, 2),
    "every other sequence of one token": base(6, 1, 4, 8)[::2],
    "part of one sequence": base(1, 9, 4, 8)[:, 2:7],
    "one token for all": base(1, 1, 4, 8).expand(2, 3, 4, 8),
    "no heads": base(2, 3, 0, 8),
    "no tokens": base(2, 0, 4, 8),
    "no sequences": base(0, 3, 4, 8),
    "no tokens, their heads outside": base(2, 4, 0, 8).transpose(1, 2),
}
REFUSED = {
    "heads outside": base(2, 4, 3, 8).transpose(1, 2),          # [batch][heads][len][dim]
    "a sliced batch": base(2, 9, 4, 8)[:, :5],
    "turned axes": base(3, 2, 4, 8).transpose(0, 1),
    "one sequence for all": base(1, 3, 4, 8).expand(2, 3, 4, 8),
    "a vector": base(8),
}


@pytest.mark.parametrize("name", TAKEN)
def test_taken(name):
    t = TAKEN[name]
    view = kb._tokens(t, "q")
    tokens = t.shape[:-2].numel()
    assert view.shape == (tokens, *t.shape[-2:]) and torch.equal(view, t.reshape(view.shape))
    assert view.data_ptr() == t.data_ptr()  # no copy
    if t.numel():
        assert view.storage_offset() == t.storage_offset()


@pytest.mark.parametrize("name", REFUSED)
def test_refused(name):
    with pytest.raises(ValueError, match="q_out"):
        kb._tokens(REFUSED[name], "q_out")


def test_three_axes_and_none_are_passed_on():
    t = base(3, 4, 8).transpose(0, 1)
    assert kb._tokens(t, "q") is t and kb._tokens(None, "dq") is None
