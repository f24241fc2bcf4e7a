"""Several tokens through the decoder at once (Decoder.extend, score, keep): the operators together, as a
prompt, a drafted tree and a scored text use them, against the CPU oracle's step by step decode.

The oracle keeps activations in fp32; extend rounds the inputs of its products and attentions to bf16, about
six roundings of relative size up to 2^-8 a layer and one before the LM head, which add up like a random walk:
a logit may be off by 2^-8 sqrt(6 L + 1) of the largest, a cached row's elements (also rounded themselves) by
the same share of the row's largest."""
import math

import numpy as np
import pytest

import oracle
import synth
from synth.device import config_kwargs, kv_from_device, kv_to_device, weights_to_device

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


SHAPES = {
    "tiny": synth.get("tiny").with_(intermediate=768),
    "d128": synth.get("tiny").with_(name="d128", head_dim=128, n_heads=6, n_kv_heads=2, hidden=320, intermediate=640,
                                    n_layers=2, vocab=515),
    "tied": synth.get("tiny").with_(name="tied", n_heads=7, n_kv_heads=1, hidden=352, intermediate=416, n_layers=3,
                                    vocab=1001, tied_embeddings=True),
    "wide": synth.get("tiny").with_(name="wide", n_heads=4, n_kv_heads=2, hidden=256, intermediate=8192, n_layers=1,
                                    vocab=257),
}


def make(amk, name, fmt, max_seq, static=False, group=32):
    cfg = SHAPES[name]
    w = synth.make_weights(cfg, seed=0)
    if fmt == "w8a16":
        synth.add_w8a16(w)
    elif fmt == "w4a16":
        synth.add_w4a16(w, group=group)
    dec = amk.Decoder(amk.make_config(**config_kwargs(cfg, fmt, max_seq, group if fmt == "w4a16" else 0)),
                      weights_to_device(w, fmt), static=static)
    return cfg, dec, oracle.OracleModel(w, fmt, np.float32)


def empty_cache(cfg, max_seq):
    return np.zeros((cfg.n_layers, 2, cfg.n_kv_heads, max_seq, cfg.head_dim), dtype=np.uint16)


def rows_of(kv, a, b):
    """Cache rows [a, b) of every layer and head as fp32."""
    return (kv[:, :, :, a:b].astype(np.uint32) << 16).view(np.float32)


def share(cfg):
    return 2.0 ** -8 * math.sqrt(6 * cfg.n_layers + 1)


def check_logits(cfg, got, ref):
    err = np.max(np.abs(got - ref), axis=-1) / np.max(np.abs(ref), axis=-1)
    assert np.all(err <= share(cfg)), float(np.max(err))


def check_rows(cfg, got, ref):
    err = np.max(np.abs(got - ref), axis=-1) / np.max(np.abs(ref), axis=-1)
    assert np.all(err <= share(cfg) + 2.0 ** -8), float(np.max(err))


def oracle_prompt(model, tokens, pos, kv):
    return np.stack([oracle.decode_step(model, int(t), pos + i, kv) for i, t in enumerate(tokens)])


@pytest.mark.parametrize("name", ["d128", "tied", "tiny"])
@pytest.mark.parametrize("fmt", ["bf16", "w8a16", "w4a16"])
@pytest.mark.parametrize("pos,n", [(0, 1), (0, 37), (5, 64), (0, 65), (9, 131)])
def test_prompt(env, name, fmt, pos, n):
    """A prompt, at the start of a cache or behind positions that steps filled; a step goes on from it."""
    amk, torch = env
    cap = pos + n + 2
    cfg, dec, model = make(amk, name, fmt, cap)
    rng = np.random.RandomState(n)
    tokens = [int(t) for t in rng.randint(0, cfg.vocab, pos + n + 1)]
    ref_kv = empty_cache(cfg, cap)
    ref = oracle_prompt(model, tokens, 0, ref_kv)
    kv = kv_to_device(empty_cache(cfg, cap))
    logits = torch.empty(cfg.vocab, dtype=torch.float32, device="cuda")
    for i in range(pos):
        dec.step(tokens[i], i, kv, logits)
    got = dec.extend(tokens[pos:pos + n], pos, kv)
    check_logits(cfg, got.cpu().numpy(), ref[pos:pos + n])
    check_rows(cfg, rows_of(kv_from_device(kv), pos, pos + n), rows_of(ref_kv, pos, pos + n))
    assert not kv_from_device(kv)[:, :, :, pos + n:].any()
    dec.step(tokens[pos + n], pos + n, kv, logits)
    check_logits(cfg, logits.cpu().numpy()[None], ref[-1:])
    assert dec.status() == amk.AMK_OK
    dec.close()


@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("w8a16", 0), ("w4a16", 32), ("w4a16", 64), ("w4a16", 128)])
def test_prompts_of_many_tiles(env, fmt, group):
    """Q, K and V, and gate and up, are multiplied in one launch each, in tiles by the number of tokens: prompts of
    each kind of tile give what pieces of 20 tokens do, and those what the oracle gives."""
    amk, torch = env
    cfg, dec, model = make(amk, "wide", fmt, 2048, group=group)
    tokens = [int(t) for t in np.random.RandomState(6).randint(0, cfg.vocab, 2048)]
    kv, ref_kv = kv_to_device(empty_cache(cfg, 2048)), empty_cache(cfg, 2048)
    small = torch.cat([dec.extend(tokens[i:i + 20], i, kv) for i in range(0, 2048, 20)]).cpu().numpy()
    check_logits(cfg, small[:30], oracle_prompt(model, tokens[:30], 0, ref_kv))
    small_rows = rows_of(kv_from_device(kv), 0, 2048)
    check_rows(cfg, small_rows[:, :, :, :30], rows_of(ref_kv, 0, 30))
    for n in (100, 150, 300, 2048):  # each side may be off by the share
        kv.zero_()
        got = dec.extend(tokens[:n], 0, kv).cpu().numpy()
        rows = rows_of(kv_from_device(kv), 0, n)
        assert np.all(np.abs(got - small[:n]).max(-1) <= 2 * share(cfg) * np.abs(small[:n]).max(-1))
        top = np.abs(small_rows[:, :, :, :n]).max(-1)
        assert np.all(np.abs(rows - small_rows[:, :, :, :n]).max(-1) <= 2 * (share(cfg) + 2.0 ** -8) * top)
    dec.close()


def test_prompt_in_chunks(env):
    """A prompt longer than extend takes at once, all of its logits and the last few only, in one call and
    in two: later rows see all earlier ones."""
    amk, torch = env
    n, cap = 2100, 2304
    cfg, dec, model = make(amk, "tiny", "bf16", cap, static=True)
    tokens = [int(t) for t in np.random.RandomState(5).randint(0, cfg.vocab, n)]
    kv = kv_to_device(empty_cache(cfg, cap))
    full = dec.extend(tokens, 0, kv)
    assert full.shape == (n, cfg.vocab)
    again = kv_to_device(empty_cache(cfg, cap))
    last = dec.extend(tokens, 0, again, n_logits=70)
    # The cached rows are the same bits.  The LM head of 70 tokens may add its H products in another order
    # than that of all: each order is off by at most H 2^-24 sum |h w| <= H 2^-24 |h| |w|, with |h| at most
    # sqrt(H) times the largest norm gain (1.1 covers it and the rounding of h).
    assert torch.equal(kv, again)
    head = dec._keep["lm_head"].view(torch.bfloat16).double()
    bound = 2 * cfg.hidden * 2.0 ** -24 * math.sqrt(cfg.hidden) * 1.1 * float(head.norm(dim=1).max())
    assert float((last - full[-70:]).abs().max()) <= bound
    assert dec.extend(tokens[:5], 0, again, n_logits=0).shape == (0, cfg.vocab)
    two = kv_to_device(empty_cache(cfg, cap))
    dec.extend(tokens[:700], 0, two, n_logits=0)
    check_logits(cfg, dec.extend(tokens[700:], 700, two, n_logits=3).cpu().numpy(), full[-3:].cpu().numpy())
    ref_kv = empty_cache(cfg, cap)
    ref = oracle_prompt(model, tokens[:40], 0, ref_kv)
    check_logits(cfg, full[:40].cpu().numpy(), ref)
    # the oracle goes on from the cache that extend left
    ref_kv[:, :, :, :n - 1] = kv_from_device(kv)[:, :, :, :n - 1]
    check_logits(cfg, full[-1:].cpu().numpy(), oracle_prompt(model, tokens[-1:], n - 1, ref_kv))
    dec.close()


@pytest.mark.parametrize("name,fmt", [("tiny", "bf16"), ("d128", "w8a16"), ("tied", "w4a16")])
@pytest.mark.parametrize("pos", [0, 40])
def test_drafted_tree(env, name, fmt, pos):
    """A tree of drafted tokens: every branch has the logits of its own decode; the accepted branch's rows
    moved together carry on as if it alone had been decoded."""
    amk, torch = env
    n, cap = 13, pos + 20
    cfg, dec, model = make(amk, name, fmt, cap)
    rng = np.random.RandomState(pos + 1)
    text = [int(t) for t in rng.randint(0, cfg.vocab, pos)]
    drafted = [int(t) for t in rng.randint(0, cfg.vocab, n)]
    parents = [-1, 0, 0, 1, 1, 2, 3, -1, 7, 6, 5, 8, 9]
    ref_kv = empty_cache(cfg, cap)
    if pos:
        oracle_prompt(model, text, 0, ref_kv)
    kv = kv_to_device(empty_cache(cfg, cap))
    if pos:
        dec.extend(text, 0, kv, n_logits=0)
    got = dec.extend(drafted, pos, kv, parents=parents).cpu().numpy()
    for leaf in (4, 10, 11, 12):
        path = [leaf]
        while parents[path[0]] >= 0:
            path.insert(0, parents[path[0]])
        branch = ref_kv.copy()
        ref = oracle_prompt(model, [drafted[i] for i in path], pos, branch)
        check_logits(cfg, got[path], ref)
    # the longest branch is accepted: 0 1 3 6 9 12
    path = [0, 1, 3, 6, 9, 12]
    before = kv_from_device(kv)
    dec.keep(pos, path, kv)
    after = kv_from_device(kv)
    for i, r in enumerate(path):
        assert np.array_equal(after[:, :, :, pos + i], before[:, :, :, pos + r])
    check_rows(cfg, rows_of(after, pos, pos + len(path)), rows_of(branch, pos, pos + len(path)))
    logits = torch.empty(cfg.vocab, dtype=torch.float32, device="cuda")
    dec.step(7, pos + len(path), kv, logits)
    check_logits(cfg, logits.cpu().numpy()[None], oracle_prompt(model, [7], pos + len(path), branch))
    dec.close()


def test_score(env):
    """Log probabilities of a text's tokens from one call, against the oracle's decode."""
    amk, torch = env
    cfg, dec, model = make(amk, "tiny", "w8a16", 128)
    tokens = [int(t) for t in np.random.RandomState(9).randint(0, cfg.vocab, 90)]
    ref = oracle_prompt(model, tokens, 0, empty_cache(cfg, 128))[:-1].astype(np.float64)
    kv = kv_to_device(empty_cache(cfg, 128))
    logprob, entropy, ids, tops = dec.score(tokens, 0, kv, top=3)
    p = ref - np.log(np.sum(np.exp(ref - ref.max(1, keepdims=True)), 1, keepdims=True)) - ref.max(1, keepdims=True)
    bound = 2 * share(cfg) * np.abs(ref).max(1)  # the logit and the log of the sum each move by the logits' error
    assert np.all(np.abs(logprob.cpu().numpy() - p[np.arange(89), tokens[1:]]) <= bound)
    assert np.all(np.abs(tops.cpu().numpy() - -np.sort(-p, axis=1)[:, :3]) <= bound[:, None])
    assert np.all(entropy.cpu().numpy() <= math.log(cfg.vocab) + 1e-4) and ids.shape == (89, 3)
    with pytest.raises(ValueError):
        dec.score(tokens[:1], 0, kv)
    dec.close()


def test_extend_refusals(env):
    amk, torch = env
    cfg, dec, _ = make(amk, "tiny", "bf16", 32)
    kv = kv_to_device(empty_cache(cfg, 32))
    before = kv.clone()
    for tokens, pos, parents in (([0] * 33, 0, None), ([0] * 5, 28, None), ([cfg.vocab], 0, None), ([-1], 0, None),
                                 ([1], -1, None), ([1, 2], 0, [-1, 1]), ([1, 2], 0, [-2, 0])):
        with pytest.raises(amk.AmkError) as e:
            dec.extend(tokens, pos, kv, parents=parents)
        assert e.value.status == amk.AMK_ERR_INVALID_ARGUMENT
    for kw in ({"n_logits": 3}, {"n_logits": -1}, {"parents": [-1]}):
        with pytest.raises(ValueError):
            dec.extend([1, 2], 0, kv, **kw)
    with pytest.raises(ValueError):
        dec.extend([1], 0, kv.cpu())
    with pytest.raises(ValueError):
        dec.extend([1], 0, kv[:-1])
    with pytest.raises(ValueError):
        dec.keep(0, [0], kv[:-1])
    with pytest.raises(amk.AmkError):
        dec.keep(0, [32], kv)
    # the C entry point: buffers that are not device memory with room, and misaligned ones
    import ctypes
    lib, tok = amk.load(), (ctypes.c_int32 * 4)(1, 2, 3, 4)
    need = lib.amk_extend_workspace(dec.handle, 4)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.empty(4, cfg.vocab, device="cuda")
    host = torch.empty(need, dtype=torch.uint8)

    def call(k=kv.data_ptr(), lg=out.data_ptr(), w=ws.data_ptr(), size=need, n_logits=4):
        return lib.amk_extend(dec.handle, tok, 4, 0, None, k, lg, n_logits, w, size, None)
    for bad in (dict(k=kv.data_ptr() + 2), dict(lg=out.data_ptr() + 4), dict(w=ws.data_ptr() + 16), dict(size=need - 1),
                dict(k=None), dict(lg=None), dict(w=None), dict(k=host.data_ptr() // 256 * 256 + 256),
                dict(w=host.data_ptr() // 256 * 256 + 256), dict(n_logits=5)):
        assert call(**bad) == amk.AMK_ERR_INVALID_ARGUMENT, bad
    torch.cuda.synchronize()
    assert torch.equal(kv, before)
    assert call() == amk.AMK_OK and call(lg=None, n_logits=0) == amk.AMK_OK
    torch.cuda.synchronize()
    dec.close()


def test_extend_on_another_stream_and_in_a_graph(env):
    """The same bits on a side stream, and from a captured graph replayed with eager work between."""
    amk, torch = env
    cfg, dec, _ = make(amk, "d128", "w4a16", 256)
    tokens = [int(t) for t in np.random.RandomState(2).randint(0, cfg.vocab, 100)]
    kv = kv_to_device(empty_cache(cfg, 256))
    want = dec.extend(tokens, 0, kv).clone()
    tree = dec.extend(tokens[:20], 100, kv, parents=[i // 2 - 1 for i in range(20)]).clone()
    rows = kv.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kv2 = torch.zeros_like(kv)
        a = dec.extend(tokens, 0, kv2)
        b = dec.extend(tokens[:20], 100, kv2, parents=[i // 2 - 1 for i in range(20)])
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, tree) and torch.equal(kv2, rows)
    g = torch.cuda.CUDAGraph()
    kv3 = torch.zeros_like(kv)
    with torch.cuda.graph(g):
        a = dec.extend(tokens, 0, kv3)
        b = dec.extend(tokens[:20], 100, kv3, parents=[i // 2 - 1 for i in range(20)])
    logits = torch.empty(cfg.vocab, dtype=torch.float32, device="cuda")
    for _ in range(3):
        kv3.zero_()
        a.zero_()
        g.replay()
        dec.step(1, 130, kv, logits)
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, tree) and torch.equal(kv3, rows)
    dec.close()


@pytest.mark.parametrize("n", [2048, 2049, 2150])
def test_score_of_a_long_text_is_taken_in_pieces(env, n):
    """The pieces are those that extend makes itself, so one extend and one token_logprobs give the same bits."""
    amk, torch = env
    cfg, dec, _ = make(amk, "tiny", "bf16", 2304)
    tokens = [(7 * i * i + 3 * i) % cfg.vocab for i in range(n + 5)]
    kv, whole = (kv_to_device(empty_cache(cfg, 2304)) for _ in range(2))
    dec.extend(tokens[:5], 0, kv), dec.extend(tokens[:5], 0, whole)
    got = dec.score(tokens[5:], 5, kv, top=4)
    logits = dec.extend(tokens[5:], 5, whole)
    want = amk.token_logprobs(logits[:-1], torch.tensor(tokens[6:], dtype=torch.int32, device=logits.device), 4)
    for g, w in zip(got, want):
        assert g.shape == w.shape and torch.equal(g, w)
    assert torch.equal(kv, whole)
    before = kv.clone()
    with pytest.raises(ValueError):
        dec.score([1] * 2300, 5, kv)
    assert torch.equal(kv, before)
    dec.close()


def test_values_past_32_bits_are_refused(env):
    amk, torch = env
    cfg, dec, _ = make(amk, "tiny", "bf16", 16)
    kv = kv_to_device(empty_cache(cfg, 16))
    for args in (([1, 2], 1 << 32), ([1, (1 << 32) + 2], 0)):
        with pytest.raises(ValueError):
            dec.extend(*args, kv)
    with pytest.raises(ValueError):
        dec.extend([1, 2], 0, kv, parents=[(1 << 32) - 1, 0])
    for pos, rows in ((1 << 32, [1]), (0, [1 + (1 << 32)])):
        with pytest.raises(ValueError):
            dec.keep(pos, rows, kv)
    assert not kv.any()
    dec.close()
