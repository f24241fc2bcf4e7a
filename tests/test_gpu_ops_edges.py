"""Edges of the operators for several tokens: handles destroyed with work under way, attention rows whose bits
depend on nothing that they do not see."""
import numpy as np
import pytest

import synth
from synth.device import config_kwargs, kv_to_device, weights_to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import os
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2606_09682_amd import amk
    if not os.path.exists(amk.LIB_PATH):
        from paper_2606_09682_amd import build
        build.build()
    amk.load()
    return amk, torch


def randn(torch, seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


# ---- attention -----------------------------------------------------------------------------
HEADS = [(1, 1, 64), (8, 1, 64), (6, 2, 128), (32, 8, 128), (128, 1, 128)]


@pytest.mark.parametrize("heads,kv,d", HEADS)
@pytest.mark.parametrize("key", [45, 101, 198])
def test_prompt_rows_before_a_high_score(env, heads, kv, d, key):
    """A finite key that scores far above all others moves the running maximum of the rows that see it. The rows
    before it, some of them in the same wave, give the same bits with it and without."""
    amk, torch = env
    for seed in range(4):
        q = (randn(torch, seed, 230, heads, d) + 1).to(torch.bfloat16)
        k, v = (randn(torch, seed + s, 230, kv, d).to(torch.bfloat16) for s in (10, 20))
        clean = amk.prompt_attention(q, k, v)
        k[key] = 8.0
        got = amk.prompt_attention(q, k, v)
        assert torch.equal(got[:key], clean[:key])
        assert not torch.equal(got[key:], clean[key:])


@pytest.mark.parametrize("heads,kv,d", HEADS)
@pytest.mark.parametrize("n,pos", [(12, 10), (40, 300), (64, 3000)])
def test_tree_branches_beside_a_high_score(env, heads, kv, d, n, pos):
    """A token of one branch that scores far above all others: the other branch has the same bits."""
    amk, torch = env
    masks = [1 << i | sum(1 << j for j in range(i % 2, i, 2)) for i in range(n)]  # of odd and of even tokens
    for seed in range(4):
        q = (randn(torch, seed, n, heads, d) + 1).to(torch.bfloat16)
        k, v = (randn(torch, seed + s, pos + n, kv, d).to(torch.bfloat16) for s in (10, 20))
        clean = amk.tree_attention(q, k, v, pos, masks)
        k[pos + 7] = 8.0
        got = amk.tree_attention(q, k, v, pos, masks)
        assert torch.equal(got[0::2], clean[0::2])
        assert not torch.equal(got[7::2], clean[7::2])


# ---- handles -------------------------------------------------------------------------------
@pytest.mark.parametrize("static", [True, False])
def test_destroy_waits_for_extend(env, static):
    """A decoder that only extended (no step was taken) is closed while its work is under way on a side
    stream: the work is done when close returns, and a decoder made at once afterwards, of another shape and in
    the same static array, changes nothing of it."""
    amk, torch = env
    cap = 2304
    cfg = synth.get("tiny")
    other = cfg.with_(name="other", hidden=512, n_heads=8, n_kv_heads=2, intermediate=512, n_layers=2)
    w, w2 = synth.make_weights(cfg, seed=0), synth.make_weights(other, seed=1)
    tokens = [(5 * i * i + i) % cfg.vocab for i in range(2200)]

    def decoder(c, weights):
        return amk.Decoder(amk.make_config(**config_kwargs(c, "bf16", cap)), weights_to_device(weights, "bf16"),
                           static=static)

    kv = [kv_to_device(np.zeros((cfg.n_layers, 2, cfg.n_kv_heads, cap, cfg.head_dim), dtype=np.uint16))
          for _ in range(2)]
    dec = decoder(cfg, w)
    want = dec.extend(tokens, 0, kv[0], n_logits=9)
    torch.cuda.synchronize()
    dec.close()

    dec = decoder(cfg, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            got = dec.extend(tokens, 0, kv[1], n_logits=9)
    dec.close()
    assert side.query()
    decoder(other, w2).close()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(kv[1], kv[0])
