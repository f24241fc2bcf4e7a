"""Sizes of the operators for several tokens at and past their limits: found on the host, in the C entries before
any launch and in the binding before a value is cut to 32 bits (no GPU)."""
import ctypes
import os

import pytest
import torch

from paper_2606_09682_amd import amk

BAD, UNSUPPORTED = amk.AMK_ERR_INVALID_ARGUMENT, amk.AMK_ERR_UNSUPPORTED
P = 4096  # a 256-byte aligned address that is never followed
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(amk.LIB_PATH):
        from paper_2606_09682_amd import build
        build.build()
    return amk.load()


@pytest.mark.parametrize("heads,kv,d,seqs,q,k", [
    (MOST, MOST, 64, 1, MOST, MOST), (MOST, 1, 128, 1, 2, 1), (1 << 20, 1 << 20, 64, 1, 4096, 1),
    (1, 1, 64, 1, 1, (1 << 30) + 1), (1, 1, 64, 1, (1 << 30) + 1, 1), (1 << 16, 1, 128, 1, 1 << 16, 1)])
def test_prompt_workspace_past_the_limits(lib, heads, kv, d, seqs, q, k):
    assert lib.amk_prompt_attention_workspace(heads, kv, d, seqs, q, k) == 0


@pytest.mark.parametrize("heads,kv,n,pos", [(MOST, MOST, 64, 0), (1 << 26, 1 << 26, 64, 0), (MOST, 1, 2, 9),
                                            (1, 1, 64, MOST - 64), (8, 8, 64, MOST), (1, 1, 1, 1 << 30)])
def test_tree_workspace_past_the_limits(lib, heads, kv, n, pos):
    assert lib.amk_tree_attention_workspace(heads, kv, 64, n, pos) == 0


def test_grids_past_the_limit(lib):
    """A grid holds fewer than 2^32 threads."""
    args = (P, 32, 1, 32, (1 << 26) + 1, P, None, amk.AMK_WEIGHTS_BF16, 0, P, (1 << 26) + 1, amk.AMK_F32, 0, None)
    assert lib.amk_linear(*args) == UNSUPPORTED
    args = (P, 32, 1 << 30, 32, 1 << 12, P, None, amk.AMK_WEIGHTS_BF16, 0, P, 1 << 12, amk.AMK_F32, 0, None)
    assert lib.amk_linear(*args) == UNSUPPORTED
    args = (P, amk.AMK_F32, 16, 1 << 24, 16, None, 0, None, P, None, None, P, 1 << 40, None)
    assert lib.amk_token_logprobs(*args) == UNSUPPORTED
    rows = (ctypes.c_int32 * 1)(1)
    assert lib.amk_kv_keep(P, 1 << 20, 1 << 6, 16, 64, 0, rows, 1, None) == UNSUPPORTED
    # a sequence adds a row tile per KV head: 2^20 of them with 2^12 KV heads
    a = amk.amk_attention_t(P, P, P, P, 64, 64, 64, 64, 64, 64, 64, 64, 1 << 10, 1 << 10, 64, 1.0)
    assert lib.amk_prompt_attention(a, P, P, 1 << 20, 1 << 20, 16, None, 0, None) == UNSUPPORTED


@pytest.mark.parametrize("value", [1 << 31, 1 << 32, -(1 << 31) - 1])
def test_binding_refuses_values_past_32_bits(value):
    with pytest.raises(ValueError, match="32 bits"):
        amk._int32(value, "a row")
    amk._int32((1 << 31) - 1, "a row"), amk._int32(-(1 << 31), "a row")
