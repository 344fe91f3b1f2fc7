"""Layer norm at its ends: the longest rows, and binary32 sums to the bound of their own order."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_gpu_norm import exact, normal

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


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


def within(got, want, tol, what):
    worst = float(((got.double() - want).abs() / tol).max())
    assert worst <= 1, "%s: %.3g of the tolerance" % (what, worst)


@pytest.mark.parametrize("rows,cols", [(37, 64), (1025, 65), (37, 500), (700, 1000), (37, 2048), (300, 4096), (5, 4097),
                                       (33, 6144), (33, 8192), (9, 9000), (9, 16384), (5, 20000), (1500, 16384)])
def test_sums_keep_32_bits(rows, cols):
    """A sum of n terms that is kept as chains of k joined in j steps is off by at most (k + j) e of the sum of
    magnitudes, e = 2^-24.  A row's chains have at most 24 terms up to 16,384 columns and 4 cols / 1024 beyond, joined in
    10 steps: R e in all.  A column's run over the rows of a part (at least 512 parts from 8192 rows on; each has a
    row at a time, four or sixteen rows beside each other), 32 parts and 16 sums: C e.  Mean: R e of mean |x|, and a
    rounding.  rstd: half of the variance's relative R e (the mean's error enters squared or against a sum of 0),
    and 4 roundings.  z = (x - mean) rstd: 4 roundings of it, rstd's error of it, the mean's of rstd.  Sums of
    products with z carry the error of z on top of their own.  Each result is rounded a few times more: 8 e."""
    x, w, b = normal((rows, cols), torch.float32, 1, 1.5, 0.25), normal((cols,), torch.float32, 2, 0.1, 1.0), normal((cols,), torch.float32, 3, 0.1)
    dy = normal((rows, cols), torch.float32, 4)
    y, mean, rstd = kb.kb_norm_forward(x, w, b)
    dx, dw, db = kb.kb_norm_backward(dy, x, w, mean, rstd)
    ey, em, er, edx, edw, edb = exact(x, w, b, dy, 1e-5)
    R = (24 if cols <= 16384 else 4 * cols // 1024 + 4) + 10
    C = -(-rows // 512) + 32 + 16 + 16
    size = x.double().abs().mean(1)
    t_mean = (R + 2) * E * size
    within(mean, em, t_mean, "mean")
    t_rstd = ((R + 8) / 2 + 4) * E * er
    within(rstd, er, t_rstd, "rstd")
    z = (x.double() - em[:, None]) * er[:, None]
    t_z = 4 * E * z.abs() + (t_rstd / er)[:, None] * z.abs() + (t_mean * er)[:, None] + E * (em.abs() * er)[:, None]
    aw, ag = w.double().abs(), (dy.double() * w.double()).abs()
    within(y, ey, t_z * aw + 8 * E * (z.abs() * aw + b.double().abs()), "y")
    g_mean, gz_mean = ag.mean(1, keepdim=True), (ag * z.abs()).mean(1, keepdim=True)
    t_gz = (R + 4) * E * gz_mean + (ag * t_z).mean(1, keepdim=True)
    t_dx = er[:, None] * ((R + 4) * E * g_mean + z.abs() * t_gz + t_z * gz_mean + 8 * E * (ag + g_mean + z.abs() * gz_mean))
    within(dx, edx, t_dx + (t_rstd / er)[:, None] * edx.abs(), "dx")
    ad = dy.double().abs()
    within(dw, edw, (ad * t_z).sum(0) + (C + 4) * E * (ad * z.abs()).sum(0), "dw")
    within(db, edb, (C + 4) * E * ad.sum(0), "db")
