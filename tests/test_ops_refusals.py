"""What the operators for several tokens refuse before anything is launched or allocated: sizes past 32 bits in the
binding, grids past the hardware's limit, texts that a later piece would refuse (no GPU)."""
import ctypes
import os

import pytest
import torch

from paper_2606_09682_amd import amk

P = 4096  # a 256-byte aligned address that is never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(amk.LIB_PATH):
        from paper_2606_09682_amd import build
        build.build()
    return amk.load()


class View:
    """What the binding asks of a device tensor, of a shape that would not fit this machine."""
    device = torch.device("cuda", 0)

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype = shape, dtype

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def stride(self, i=None):
        strides = [1]
        for s in self.shape[:0:-1]:
            strides.insert(0, strides[0] * s)
        return tuple(strides) if i is None else strides[i]

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return P


BIG = (1 << 32) + 64  # 64 if cut to 32 bits


@pytest.mark.parametrize("call", [
    lambda: amk.linear(View(BIG, 64), View(64, 64)),
    lambda: amk.linear(View(1, BIG), View(64, BIG)),
    lambda: amk.linear(View(1, 64), View(BIG, 64)),
    lambda: amk.prompt_attention(View(BIG, 4, 64), View(9, 4, 64), View(9, 4, 64), out=View(BIG, 4, 64)),
    lambda: amk.prompt_attention(View(9, BIG, 64), View(9, 4, 64), View(9, 4, 64), out=View(9, BIG, 64)),
    lambda: amk.prompt_attention(View(9, 4, BIG), View(9, 4, BIG), View(9, 4, BIG), out=View(9, 4, BIG)),
    lambda: amk.prompt_attention(View(9, 4, 64), View(BIG, 4, 64), View(BIG, 4, 64), out=View(9, 4, 64)),
    lambda: amk.prompt_attention(View(9, BIG, 64), View(9, BIG, 64), View(9, BIG, 64), out=View(9, BIG, 64)),
    lambda: amk.prompt_attention(View(9, 4, 64), View(9, 4, 64), View(9, 4, 64), View(BIG, dtype=torch.int32),
                                 View(BIG, dtype=torch.int32), out=View(9, 4, 64)),
    lambda: amk.tree_attention(View(1, 4, 64), View(BIG, 4, 64), View(BIG, 4, 64), 1 << 32, [1], out=View(1, 4, 64)),
    lambda: amk.token_logprobs(View(BIG, 100, dtype=torch.float32)),
    lambda: amk.token_logprobs(View(1, BIG, dtype=torch.float32)),
    lambda: amk.kv_keep(View(BIG, 2, 4, 100, 64), 0, [1]),
    lambda: amk.kv_keep(View(4, 2, BIG, 100, 64), 0, [1]),
    lambda: amk.kv_keep(View(4, 2, 4, BIG, 64), 0, [1]),
    lambda: amk.kv_keep(View(4, 2, 4, 100, BIG), 0, [1]),
])
def test_sizes_past_32_bits(lib, call):
    with pytest.raises(ValueError, match="does not fit 32 bits"):
        call()


@pytest.mark.parametrize("n,heads", [(1, 1 << 30), (8, 1 << 27)])
def test_tree_grid_past_the_limit(lib, n, heads):
    """A workgroup at least for every KV head, below 2^32 threads in all."""
    a = amk.amk_attention_t(P, P, P, P, 64, 64, 64, 64, 64, 64, 64, 64, heads, heads, 64, 1.0)
    masks = (ctypes.c_uint64 * n)(*[1] * n)
    assert lib.amk_tree_attention(a, n, 5, masks, None, 0, None) == amk.AMK_ERR_UNSUPPORTED


@pytest.mark.parametrize("tokens,top,error", [
    ([1] * 3000, 33, ValueError), ([1] * 3000, -1, ValueError), ([1] * 2999 + [100], 3, amk.AmkError),
    ([1] * 2999 + [-1], 3, amk.AmkError), ([1] * 2999 + [1 << 32], 3, ValueError), ([1], 3, ValueError),
    ([1] * 5000, 3, ValueError), ([1, 100], 0, amk.AmkError), ([1, 2], 33, ValueError)])
def test_score_refuses_before_it_runs(lib, tokens, top, error):
    """A text is taken in pieces: one that cannot be scored whole leaves the cache as it was."""
    dec = object.__new__(amk.Decoder)
    dec.handle = None
    dec.cfg = amk.make_config(64, 1, 1, 1, 64, 64, 100, 4096, 1e4)
    dec.extend = lambda *a, **k: pytest.fail("a piece was run")
    with pytest.raises(error):
        dec.score(tokens, 0, torch.zeros(1), top)
