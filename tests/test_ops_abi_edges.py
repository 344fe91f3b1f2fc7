"""Argument ranges of the reference operators at their ends (no GPU: a call
whose arguments pass fails at its launch, KB_ERR_HIP)."""
import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built
from tests.test_attn_abi import backward
from tests.test_norm_abi import view

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="descriptors of memory that does not exist")
ARG, OK, HIP = kb.KB_ERR_INVALID_ARG, kb.KB_OK, kb.KB_ERR_HIP


@pytest.fixture(scope="module")
def L():
    ensure_built()
    return kb.lib()


@pytest.mark.parametrize("dtype", [kb.KB_F32, kb.KB_F16, kb.KB_BF16])
@pytest.mark.parametrize("nq", [0, 16])
def test_no_query_heads_have_gradients_of_zero(L, dtype, nq):
    """Key heads that no query head reads: dk and dv are zeros that the call has to write; without keys, nothing."""
    none = view(0, (2, 0, nq, 64), dtype=dtype)
    for nk, code in ((32, HIP), (0, OK)):
        key = [view(p if nk else 0, (2, 4, nk, 64), dtype=dtype) for p in (0x100000, 0x200000, 0x300000, 0x400000)]
        size = L.kb_attn_backward_workspace_bytes(none, key[0])
        rc = backward(L, do=none, q=none, k=key[0], v=key[1], o=none, lse=None, dq=none, dk=key[2], dv=key[3], size=size)
        assert rc == code
