"""Edges of the operators for several tokens: handles destroyed with work under way."""
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
