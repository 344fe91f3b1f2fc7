"""Argument checks of the layer norm calls: they run on the host before any
HIP call, so descriptors of memory that does not exist will do.  A call whose
arguments pass fails at its launch here (KB_ERR_HIP): no GPU."""
import ctypes
import random

import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="descriptors of memory that does not exist")


@pytest.fixture(scope="module")
def L():
    ensure_built()
    return kb.lib()


def view(data, shape, strides=None, dtype=kb.KB_F32):
    if strides is None:
        strides, n = [], 1
        for s in reversed(shape):
            strides.insert(0, n)
            n *= s
    pad = (0,) * (kb.KB_MAX_DIMS - len(shape))
    return kb._VIEW.pack(data or 0, dtype, len(shape), *shape, *pad, *strides, *pad)


def forward(L, x=view(0x10000, (4, 8)), w=view(0x20000, (8,)), b=view(0x30000, (8,)), eps=1e-5,
            y=view(0x40000, (4, 8)), mean=0x50000, rstd=0x60000):
    return L.kb_norm_forward(x, w, b, eps, y, mean, rstd, None)


def backward(L, dy=view(0x10000, (4, 8)), x=view(0x20000, (4, 8)), w=view(0x30000, (8,)), mean=0x40000, rstd=0x50000,
             dx=view(0x60000, (4, 8)), dw=view(0x70000, (8,)), db=view(0x80000, (8,)), ws=0x90000, bytes=1 << 16):
    return L.kb_norm_backward(dy, x, w, mean, rstd, dx, dw, db, ws, bytes, None)


def test_good_arguments_reach_the_launch(L):
    assert forward(L) == kb.KB_ERR_HIP
    assert forward(L, w=None, b=None, mean=None, rstd=None) == kb.KB_ERR_HIP
    assert forward(L, y=view(0x10000, (4, 8))) == kb.KB_ERR_HIP  # in place
    assert backward(L) == kb.KB_ERR_HIP
    assert backward(L, dw=None, db=None, ws=None, bytes=0) == kb.KB_ERR_HIP


@pytest.mark.parametrize("change,code", [
    (dict(x=None), kb.KB_ERR_INVALID_ARG),
    (dict(x=view(None, (4, 8))), kb.KB_ERR_INVALID_ARG),
    (dict(x=view(0x10000, (4, 8, 1))), kb.KB_ERR_INVALID_ARG),
    (dict(x=view(0x10000, (4, -8))), kb.KB_ERR_INVALID_ARG),
    (dict(x=view(0x10000, (4, 8), (16, 2))), kb.KB_ERR_INVALID_ARG),
    (dict(x=view(0x10000, (4, 8), (-8, 1))), kb.KB_ERR_INVALID_ARG),
    (dict(x=view(0x10002, (4, 8))), kb.KB_ERR_ALIGNMENT),
    (dict(x=view(0x10000, (4, 8), dtype=kb.KB_U32)), kb.KB_ERR_DTYPE),
    (dict(x=view(0x10000, (4, 0)), y=view(0x40000, (4, 0)), w=None, b=None), kb.KB_ERR_INVALID_ARG),
    (dict(y=None), kb.KB_ERR_INVALID_ARG),
    (dict(y=view(0x40000, (4, 9))), kb.KB_ERR_INVALID_ARG),
    (dict(y=view(0x40000, (4, 8), (7, 1))), kb.KB_ERR_INVALID_ARG),
    (dict(y=view(0x40000, (4, 8), (0, 1))), kb.KB_ERR_INVALID_ARG),
    (dict(y=view(0x40000, (4, 8), dtype=kb.KB_F16)), kb.KB_ERR_DTYPE),
    (dict(y=view(0x10010, (4, 8))), kb.KB_ERR_INVALID_ARG),      # overlaps x
    (dict(y=view(0x20010, (4, 8))), kb.KB_ERR_INVALID_ARG),      # overlaps w
    (dict(mean=0x40010), kb.KB_ERR_INVALID_ARG),                 # overlaps y
    (dict(mean=0x60008), kb.KB_ERR_INVALID_ARG),                 # overlaps rstd
    (dict(mean=0x50002), kb.KB_ERR_ALIGNMENT),
    (dict(w=view(0x20000, (7,))), kb.KB_ERR_INVALID_ARG),
    (dict(w=view(0x20000, (8,), (2,))), kb.KB_ERR_INVALID_ARG),
    (dict(w=view(0x20000, (8,), dtype=kb.KB_F16)), kb.KB_ERR_DTYPE),
    (dict(eps=-1.0), kb.KB_ERR_INVALID_ARG),
    (dict(eps=float("nan")), kb.KB_ERR_INVALID_ARG),
])
def test_forward_refusals(L, change, code):
    assert forward(L, **change) == code
    assert "kb_norm_forward" in kb.kb_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(dy=None), kb.KB_ERR_INVALID_ARG),
    (dict(dy=view(0x10000, (5, 8))), kb.KB_ERR_INVALID_ARG),
    (dict(dy=view(0x10000, (4, 8), (0, 0))), kb.KB_ERR_INVALID_ARG),
    (dict(mean=None), kb.KB_ERR_INVALID_ARG),
    (dict(rstd=0x50001), kb.KB_ERR_ALIGNMENT),
    (dict(dx=view(0x10000, (4, 8))), kb.KB_ERR_INVALID_ARG),     # dx on dy
    (dict(dx=view(0x20000, (4, 8))), kb.KB_ERR_INVALID_ARG),     # dx on x
    (dict(dw=view(0x80000, (8,))), kb.KB_ERR_INVALID_ARG),       # dw on db
    (dict(dw=view(0x70000, (8,), dtype=kb.KB_BF16)), kb.KB_ERR_DTYPE),
    (dict(ws=None), kb.KB_ERR_WORKSPACE),
    (dict(bytes=255), kb.KB_ERR_WORKSPACE),                      # 4 rows x 2 x 8 floats = 256
    (dict(ws=0x90004), kb.KB_ERR_ALIGNMENT),
    (dict(ws=0x60000), kb.KB_ERR_INVALID_ARG),                   # the workspace on dx
])
def test_backward_refusals(L, change, code):
    assert backward(L, **change) == code
    assert "kb_norm_backward" in kb.kb_last_error()


def test_mixed_weight_types(L):
    half = dict(x=view(0x10000, (4, 8), dtype=kb.KB_F16), y=view(0x40000, (4, 8), dtype=kb.KB_F16))
    w16, b16 = view(0x20000, (8,), dtype=kb.KB_F16), view(0x30000, (8,), dtype=kb.KB_F16)
    assert forward(L, **half) == kb.KB_ERR_HIP
    assert forward(L, w=w16, b=b16, **half) == kb.KB_ERR_HIP
    assert forward(L, w=w16, **half) == kb.KB_ERR_DTYPE
    assert forward(L, w=view(0x20000, (8,), dtype=kb.KB_BF16), b=None, **half) == kb.KB_ERR_DTYPE


def test_empty(L):
    none = view(None, (0, 8))
    assert forward(L, x=none, y=none) == kb.KB_OK
    assert backward(L, dy=none, x=none, dx=none, dw=None, db=None) == kb.KB_OK


def test_workspace_bytes():
    assert kb.kb_norm_backward_workspace_bytes(0, 8) == 0
    assert kb.kb_norm_backward_workspace_bytes(4, 8) == 256
    assert kb.kb_norm_backward_workspace_bytes(-1, 8) == 0
    last = 0
    for rows in (1, 2, 100, 511, 512, 513, 100000):
        assert kb.kb_norm_backward_workspace_bytes(rows, 777) >= last
        last = kb.kb_norm_backward_workspace_bytes(rows, 777)


def elements(base, shape, strides):
    return {base + 4 * (i * strides[0] + j * strides[1]) for i in range(shape[0]) for j in range(shape[1])}


def test_overlap_is_never_missed(L):
    """dx against x over random views: one that shares an element is refused,
    and the columns of one wider buffer are not."""
    rng = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        shape = (rng.randrange(1, 6), rng.randrange(1, 9))
        sx = (rng.randrange(0, 24), 1)
        so = (rng.randrange(shape[1], 24), 1)
        if rng.random() < 0.5:
            sx = so
        bx, bo = 0x100000, 0x100000 + 4 * rng.randrange(-60, 60)
        shares = bool(elements(bx, shape, sx) & elements(bo, shape, so))
        rc = backward(L, x=view(bx, shape, sx), dy=view(0x200000, shape), dx=view(bo, shape, so), w=None,
                      dw=None, db=None)
        assert rc in (kb.KB_ERR_INVALID_ARG, kb.KB_ERR_HIP)
        seen[shares] += 1
        if shares:
            assert rc == kb.KB_ERR_INVALID_ARG, (shape, sx, so, bo - bx)
    assert min(seen.values()) > 500
    shape, s = (5, 8), (24, 1)
    assert backward(L, x=view(0x100000, shape, s), dy=view(0x100000 + 32, shape, s), w=None, dw=None, db=None,
                    dx=view(0x100000 + 64, shape, s)) == kb.KB_ERR_HIP
    assert ctypes.sizeof(kb.KbTensor) == kb._VIEW.size
