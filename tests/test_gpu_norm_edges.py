"""Layer norm at its ends: the longest rows, and binary32 sums to the bound of their own order."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def test_rows_of_nearly_2_to_31_columns():
    """The longest row that a descriptor can hold, where a thread's step passes 2^31.  Elements of 1 and -1 by turns
    sum to 1 exactly, so the mean is 2^-31 and rstd 1 within 2^-20 (eps 0): y is x, and of a dy that is 0 but for a few
    elements dx is dy and dw dy x, each after rounding to 16 bits (what is left of the row sums is under 2^-25)."""
    n = 2 ** 31 - 1
    row = torch.ones((1, n), dtype=torch.float16, device="cuda")
    row[:, 1::2] = -1.0
    y, mean, rstd = kb.kb_norm_forward(row, None, None, 0.0)
    assert float(mean) <= 2.0 ** -30 and abs(float(rstd) - 1) <= 2.0 ** -20
    assert torch.equal(y, row)
    del y
    at = torch.tensor([0, 1, 2047, 2 ** 30 + 3, n - 2049, n - 2048, n - 9, n - 8, n - 2, n - 1], device="cuda")
    dy = torch.zeros_like(row)
    dy[0, at] = torch.arange(1.0, 11.0, device="cuda").half()
    dx, dw, db = kb.kb_norm_backward(dy, row, None, mean, rstd)
    assert torch.equal(dx, dy) and torch.equal(db, dy[0])
    assert int((dw != 0).sum()) == len(at) and torch.equal(dw[at], (dy * row)[0, at])


def test_columns_of_more_threads_than_a_launch_takes():
    """Column sums of 2^27 columns and some, which would take 2^32 threads at once; whole numbers, so exact."""
    n = 2 ** 27 + 5
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randint(-8, 9, (2, n), generator=gen, device="cuda").float() for _ in range(2))
    mean, rstd = torch.zeros(2, device="cuda"), torch.ones(2, device="cuda")
    _, dw, db = kb.kb_norm_backward(dy, x, None, mean, rstd)
    assert torch.equal(db, dy.sum(0)) and torch.equal(dw, (dy * x).sum(0))
