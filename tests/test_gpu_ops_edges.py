"""Edges of the operators for several tokens: products of small codes, infinities and few tokens, handles destroyed with work under way, attention rows whose bits
depend on nothing that they do not see, infinities and NaN in V.

An fp32 sum of k exact products is off by at most k 2^-24 times the sum of their magnitudes, whatever the codes."""
import math

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


# ---- products ------------------------------------------------------------------------------
def packed(torch, codes):
    """Codes in [-8, 7] [out, in] in the packed layout: of 8 columns, the low nibbles are the first four."""
    u = (codes + 8).to(torch.uint8).view(codes.shape[0], -1, 2, 4)
    return (u[:, :, 0] | u[:, :, 1] << 4).reshape(codes.shape[0], -1).contiguous()


def codes_and_scale(torch, seed, low, high, out, width, group):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.randint(low, high + 1, (out, width), generator=g, device="cuda")
    return c, (torch.rand(out, width // group, generator=g, device="cuda") * 0.1 + 0.01).half()


# tokens, columns, rows, group: every kind of tile, columns that end inside a stage
TILES = [(1, 256, 40, 64), (9, 544, 8230, 32), (16, 1152, 300, 128), (30, 1056, 130, 32), (31, 1152, 8190, 128),
         (64, 1088, 4096, 64), (100, 1056, 4096, 32), (200, 1088, 4090, 64), (300, 416, 4090, 32), (511, 640, 4099, 128),
         (1030, 160, 4100, 32), (2050, 192, 8200, 64), (2050, 384, 2060, 128), (2050, 512, 8200, 256)]


@pytest.mark.parametrize("n,width,out,group", TILES)
def test_int4_codes_are_exact(env, n, width, out, group):
    """Zero codes give zero; a token of one 1 gives a column's codes times their scales, rounded nowhere; codes of
    -1, 0 and 1 are summed as closely as any."""
    amk, torch = env
    x = randn(torch, n, n, width).to(torch.bfloat16)
    c, s = codes_and_scale(torch, 1, 0, 0, out, width, group)
    assert not amk.linear(x, packed(torch, c), s, "w4a16", group).any()
    c, s = codes_and_scale(torch, 2, -1, 1, out, width, group)
    w64 = c.double() * s.double().repeat_interleave(group, 1)
    y = amk.linear(x, packed(torch, c), s, "w4a16", group)
    tol = (width + 4) * 2.0 ** -24 * (x.double().abs() @ w64.abs().t())
    assert float(((y.double() - x.double() @ w64.t()).abs() - tol).max()) <= 0
    c, s = codes_and_scale(torch, 3, -8, 7, out, width, group)
    w = c.float() * s.float().repeat_interleave(group, 1)
    at = torch.randint(0, width, (n,), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    one = torch.zeros(n, width, dtype=torch.bfloat16, device="cuda")
    one[torch.arange(n, device="cuda"), at] = 1
    assert torch.equal(amk.linear(one, packed(torch, c), s, "w4a16", group), w.t()[at])


@pytest.mark.parametrize("fmt", ["bf16", "w8a16", "w4a16"])
@pytest.mark.parametrize("n,width,out,group", TILES)
def test_infinite_tokens(env, fmt, n, width, out, group):
    """An infinity in x gives what the product's definition does: an infinity of its weight's sign, NaN where the
    weight is 0 or two infinities meet; other tokens do not change."""
    amk, torch = env
    x = randn(torch, n, n, width).to(torch.bfloat16)
    c, s = codes_and_scale(torch, 5, -8, 7, out, width, group)
    if fmt == "bf16":
        args, w64 = (c.to(torch.bfloat16),), c.double()
    elif fmt == "w8a16":
        args, w64 = (c.to(torch.int8), s[:, 0].float().contiguous(), fmt), c.double() * s[:, :1].double()
    else:
        args, w64 = (packed(torch, c), s, fmt, group), c.double() * s.double().repeat_interleave(group, 1)
    clean = amk.linear(x, *args)
    last, t = width - 1, n - 1
    for bad in ({3: math.inf}, {last: -math.inf}, {3: math.inf, last: math.inf}, {9: math.nan}):
        odd = x.clone()
        for k, value in bad.items():
            odd[t, k] = value
        y = amk.linear(odd, *args)
        want = sum(value * w64[:, k] for k, value in bad.items())  # what is finite does not count beside it
        assert torch.equal(torch.isnan(y[t]), torch.isnan(want))
        assert torch.equal(y[t][torch.isinf(want)].double(), want[torch.isinf(want)])
        assert torch.equal(y[:t], clean[:t])


def test_infinite_scales(env):
    """An infinite scale of the last group reaches its own row, also where the columns end inside a stage."""
    amk, torch = env
    for n, width, out, group in TILES:
        x = randn(torch, n, n, width).to(torch.bfloat16)
        c, s = codes_and_scale(torch, 6, 1, 7, out, width, group)
        x[:, -group:] = x[:, -group:].abs() + 1  # sums of the last group are positive
        clean = amk.linear(x, packed(torch, c), s, "w4a16", group)
        s[out // 2, -1] = math.inf
        y = amk.linear(x, packed(torch, c), s, "w4a16", group)
        rest = [r for r in range(out) if r != out // 2]
        assert (y[:, out // 2] == math.inf).all() and torch.equal(y[:, rest], clean[:, rest])


@pytest.mark.parametrize("fmt", ["bf16", "w8a16", "w4a16"])
@pytest.mark.parametrize("n", [17, 32, 33, 64, 100, 127])
@pytest.mark.parametrize("out", [32700, 128256])
def test_few_tokens_by_many_rows(env, fmt, n, out):
    """The logits of a drafted tree: tiles of more tokens than there are."""
    amk, torch = env
    width, group = 352, 32
    x = randn(torch, n, n, width).to(torch.bfloat16)
    c, s = codes_and_scale(torch, 7, -8, 7, out, width, group)
    if fmt == "bf16":
        y, w = amk.linear(x, c.to(torch.bfloat16)), c.float()
    elif fmt == "w8a16":
        one = s[:, 0].float().contiguous()
        y, w = amk.linear(x, c.to(torch.int8), one, fmt), c.float() * one[:, None]
    else:
        y, w = amk.linear(x, packed(torch, c), s, fmt, group), c.float() * s.float().repeat_interleave(group, 1)
    w = w.double()
    tol = (width + 4) * 2.0 ** -24 * (x.double().abs() @ w.abs().t())
    assert float(((y.double() - x.double() @ w.t()).abs() - tol).max()) <= 0


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


def odd_inputs(torch, seed, n, rows, heads, kv, d):
    """q [n], k, v [rows], every query's first element 1: k[j] = (x, 0, 0, ...) scores x for all."""
    q = randn(torch, seed, n, heads, d).to(torch.bfloat16)
    q[:, :, 0] = 1
    k, v = (randn(torch, seed + s, rows, kv, d).to(torch.bfloat16) for s in (10, 20))
    return q, k, v


def calls_of(amk, torch, q, k, v):
    """Attentions of the last queries to k's rows: as a prompt and (up to 64) as a chain: {name: result}"""
    n = q.shape[0]
    out = {"prompt": amk.prompt_attention(q, k, v)}
    if n <= 64:
        out["tree"] = amk.tree_attention(q, k, v, k.shape[0] - n, [(2 << i) - 1 for i in range(n)])
    return out


# queries, keys, and the key in question: in tiles that all rows see whole, in those of the diagonal, in ranges
# of keys that are split
ODD = [(200, 200, 20), (200, 200, 77), (90, 90, 0), (300, 300, 131), (40, 340, 100), (40, 340, 305), (12, 3012, 100),
       (60, 4060, 4010), (1, 3000, 1500), (1, 31, 30)]


@pytest.mark.parametrize("heads,kv,d", [(1, 1, 64), (6, 2, 64), (8, 1, 128), (128, 1, 128)])
@pytest.mark.parametrize("n,rows,key", ODD)
def test_odd_values_of_keys_without_weight(env, heads, kv, d, n, rows, key):
    """A key that scores minus infinity has no weight: what its V holds reaches no row, wherever tiles begin."""
    amk, torch = env
    q, k, v = odd_inputs(torch, 1, n, rows, heads, kv, d)
    k[key], k[key, :, 0] = 0, -math.inf
    clean = calls_of(amk, torch, q, k, v)
    for bad in (math.inf, -math.inf, math.nan):
        v[key, :, 5], v[key, :, d - 1] = bad, -bad
        for name, got in calls_of(amk, torch, q, k, v).items():
            assert torch.equal(got, clean[name]), (name, bad)


@pytest.mark.parametrize("heads,kv,d", [(1, 1, 64), (6, 2, 64), (8, 1, 128), (128, 1, 128)])
@pytest.mark.parametrize("n,rows,key", ODD)
@pytest.mark.parametrize("score", [0.0, -3e4])
def test_odd_values_reach_the_rows_that_see_them(env, heads, kv, d, n, rows, key, score):
    """However small a key's weight (2^-5000 here), an infinity or NaN of its V reaches every row that sees it, in
    its own column; all other rows and columns keep their bits."""
    amk, torch = env
    q, k, v = odd_inputs(torch, 2, n, rows, heads, kv, d)
    k[key], k[key, :, 0] = 0, score
    clean = calls_of(amk, torch, q, k, v)
    before = max(0, key - (rows - n))  # queries that do not see the key
    others = [c for c in range(d) if c != 5]
    for bad in (math.inf, -math.inf, math.nan):
        v[key, :, 5] = bad
        for name, got in calls_of(amk, torch, q, k, v).items():
            assert torch.equal(got[:before], clean[name][:before]), (name, bad)
            assert torch.equal(got[before:, :, others], clean[name][before:, :, others]), (name, bad)
            seen = got[before:, :, 5].float()
            assert bool(torch.isnan(seen).all() if math.isnan(bad) else (seen == bad).all()), (name, bad)
    if rows - n <= key < rows - 1:  # opposite infinities have no sum; query `before` is the last without the second
        v[key, :, 5], v[key + 1, :, 5] = math.inf, -math.inf
        for name, got in calls_of(amk, torch, q, k, v).items():
            assert (got[before, :, 5] == math.inf).all() and torch.isnan(got[before + 1:, :, 5]).all()


def test_rows_of_keys_without_weight_are_zeros(env):
    """Rows whose keys all score minus infinity get zeros, with infinities and NaN in V too; longer rows go on."""
    amk, torch = env
    for d, n in ((64, 150), (128, 150), (128, 64)):
        for none in (3, 64, 100):
            q, k, v = odd_inputs(torch, 3, n, n, 4, 2, d)
            k[:none], k[:none, :, 0] = 0, -math.inf
            clean = calls_of(amk, torch, q, k, v)
            v[:none:2], v[1:none:2] = math.inf, math.nan
            for name, got in calls_of(amk, torch, q, k, v).items():
                assert (got[:none] == 0).all() and torch.equal(got, clean[name])


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
