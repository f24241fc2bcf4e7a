"""The operators for several tokens against their definitions in 64 bits, at the sizes, strides and masks
where they can go wrong.

Tolerances count roundings (u = 2^-24 in fp32; bf16 2^-8 relative, half its step): an fp32 sum of k exact
products is off by at most k u times the sum of their magnitudes; an attention weight rounded to bf16 by
2^-8 of itself, so an output by 2^-8 of the weighted sum of |v|, and 2^-8 of itself for its own rounding."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8


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


# ---- products ----------------------------------------------------------------------------
def int4_words(torch, codes):
    """Codes in [-8, 7] [out, in] in the packed layout, column by column."""
    out, width = codes.shape
    w = torch.zeros(out, width // 2, dtype=torch.uint8, device="cuda")
    u = (codes + 8).to(torch.uint8)
    for t in range(8):
        w[:, t % 4::4] |= u[:, t::8] << (4 if t >= 4 else 0)
    return w


def matrix(torch, fmt, out, width, group, seed):
    """(w, scale, the matrix in 64 bits)"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if fmt == "bf16":
        w = randn(torch, seed, out, width).to(torch.bfloat16)
        return w, None, w.double()
    if fmt == "w8a16":
        w = torch.randint(-128, 128, (out, width), generator=g, device="cuda").to(torch.int8)
        s = torch.rand(out, generator=g, device="cuda") * 0.01
        return w, s, w.double() * s.double()[:, None]
    c = torch.randint(-8, 8, (out, width), generator=g, device="cuda")
    s = (torch.rand(out, width // group, generator=g, device="cuda") * 0.1).half()
    return int4_words(torch, c), s, c.double() * s.double().repeat_interleave(group, 1)


def check_linear(torch, y, x, w64, base=None):
    ref = x.double() @ w64.t()
    # width products and, in the last two steps, a scale and an addition
    tol = (x.shape[1] + 4) * U * (x.double().abs() @ w64.abs().t())
    if base is not None:
        ref = ref + base.double()
        tol = tol + 2 * U * base.double().abs()
    if y.dtype == torch.bfloat16:
        tol = tol + (ref.abs() + tol) * BF
    worst = float(((y.double() - ref).abs() - tol).max())
    assert worst <= 0, worst


LINEAR = [  # n, in, out, group
    (1, 64, 1, 64), (1, 256, 64, 32), (2, 96, 33, 32), (15, 320, 65, 64), (16, 576, 1536, 64), (17, 256, 4096, 256),
    (31, 1024, 129, 1024), (33, 2048, 63, 128), (48, 1024, 2500, 128), (64, 688 * 2, 130, 32), (65, 768, 127, 256),
    (129, 4096, 257, 128), (257, 512, 1040, 512), (300, 5632, 300, 64), (512, 320, 515, 64), (1000, 1152, 2051, 128),
    (2047, 320, 2051, 64), (4090, 576, 4091, 64),  # tiles of 128 and of 256
]


@pytest.mark.parametrize("fmt", ["bf16", "w8a16", "w4a16"])
@pytest.mark.parametrize("n,width,out,group", LINEAR)
def test_linear(env, fmt, n, width, out, group):
    amk, torch = env
    w, s, w64 = matrix(torch, fmt, out, width, group, n)
    x = randn(torch, 1, n, width).to(torch.bfloat16)
    for dtype in (torch.float32, torch.bfloat16):
        y = amk.linear(x, w, s, fmt, group, out_dtype=dtype)
        check_linear(torch, y, x, w64)


@pytest.mark.parametrize("fmt", ["bf16", "w8a16", "w4a16"])
@pytest.mark.parametrize("n,width,out,group", [(31, 1152, 8190, 128), (100, 1056, 4096, 32), (97, 5504, 14330, 64),
                                               (200, 1088, 4090, 64), (300, 416, 4090, 32), (511, 5504, 4099, 128)])
def test_linear_small_tiles(env, fmt, n, width, out, group):
    """More tiles of 32 than CUs, one round of tiles of 64 and two to a CU, columns that end inside a stage."""
    amk, torch = env
    w, s, w64 = matrix(torch, fmt, out, width, group, n)
    x = randn(torch, 1, n, width).to(torch.bfloat16)
    check_linear(torch, amk.linear(x, w, s, fmt, group), x, w64)


@pytest.mark.parametrize("n,width,out,group", [
    (2050, 384, 2060, 128), (2050, 512, 8200, 256), (2048, 1024, 8192, 1024), (2050, 128, 8200, 128),
    (2050, 96, 8200, 32), (2050, 192, 8200, 64), (1030, 160, 4100, 32)])
def test_linear_groups_in_large_tiles(env, n, width, out, group):
    amk, torch = env
    w, s, w64 = matrix(torch, "w4a16", out, width, group, n)
    x = randn(torch, 1, n, width).to(torch.bfloat16)
    check_linear(torch, amk.linear(x, w, s, "w4a16", group), x, w64)


@pytest.mark.parametrize("fmt", ["bf16", "w8a16"])
@pytest.mark.parametrize("width", [16, 48, 80, 2768])
def test_linear_widths_of_half_steps(env, fmt, width):
    amk, torch = env
    for n in (3, 70, 200):
        w, s, w64 = matrix(torch, fmt, 100, width, 0, width)
        x = randn(torch, 1, n, width).to(torch.bfloat16)
        check_linear(torch, amk.linear(x, w, s, fmt), x, w64)


@pytest.mark.parametrize("fmt", ["bf16", "w8a16", "w4a16"])
@pytest.mark.parametrize("n,out", [(1, 130), (20, 130), (90, 130), (300, 130), (64, 14001), (2050, 2050), (4090, 4090)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_linear_strides_and_accumulate(env, fmt, n, out, dtype):
    """Rows apart from each other, what lies between them untouched, and adding to what is there."""
    amk, torch = env
    width, group = 256, 64
    w, s, w64 = matrix(torch, fmt, out, width, group, n)
    store = torch.full((n, width + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    store[:, 8:8 + width] = randn(torch, 2, n, width).to(torch.bfloat16)
    x = store[:, 8:8 + width]
    held = randn(torch, 3, n, out + 7).to(getattr(torch, dtype))
    for accumulate in (False, True):
        full = held.clone()
        y = full[:, 3:3 + out]
        assert amk.linear(x, w, s, fmt, group, out=y, accumulate=accumulate) is y
        check_linear(torch, y, x, w64, held[:, 3:3 + out] if accumulate else None)
        assert torch.equal(full[:, :3], held[:, :3]) and torch.equal(full[:, 3 + out:], held[:, 3 + out:])


def test_linear_keeps_rows_apart(env):
    """A token of infinities and NaN, or such a row of W, reaches its own outputs only."""
    amk, torch = env
    for n in (5, 40, 140):
        x = randn(torch, 4, n, 320).to(torch.bfloat16)
        w = randn(torch, 5, 200, 320).to(torch.bfloat16)
        y = amk.linear(x, w)
        x[2, 7], x[2, 9], w[131, 300] = math.inf, math.nan, math.nan
        z = amk.linear(x, w)
        assert torch.isnan(z[2]).all() and torch.isnan(z[:, 131]).all()
        keep_t, keep_r = [i for i in range(n) if i != 2], [i for i in range(200) if i != 131]
        assert torch.equal(z[keep_t][:, keep_r], y[keep_t][:, keep_r])


def test_linear_of_nothing(env):
    amk, torch = env
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.empty(32, 64, dtype=torch.bfloat16, device="cuda")
    assert amk.linear(x, w).shape == (0, 32)


# ---- attention ---------------------------------------------------------------------------
def softmax_rows(torch, q, k, v, visible, scale):
    """(result, tolerance) in 64 bits: q [n, h, d], k, v [rows, kv, d], visible [n, rows]; what is not
    visible is left out, not multiplied by zero."""
    n, heads, d = q.shape
    group = heads // k.shape[1]
    ref = torch.zeros(n, heads, d, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(ref)
    for i in range(n):
        at = torch.nonzero(visible[i])[:, 0]
        if not len(at):
            continue
        for g in range(k.shape[1]):
            kk, vv = k[at, g].double(), v[at, g].double()
            qq = q[i, g * group:(g + 1) * group].double()
            s = (qq @ kk.t()) * scale
            p = torch.softmax(s, dim=1)
            o = p @ vv
            # scores are fp32 sums of d products, off by d u sum |q k|, and a weight by as much of itself
            ds = d * U * (qq.abs() @ kk.abs().t()) * scale + 4 * U * s.abs()
            mag = p @ vv.abs()
            ref[i, g * group:(g + 1) * group] = o
            tol[i, g * group:(g + 1) * group] = (BF + 2 * ds.max() + len(at) * U) * mag * (1 + BF) + BF * o.abs()
    return ref, tol


def close(torch, got, ref, tol):
    assert torch.isfinite(got.float()).all()
    worst = float(((got.double() - ref).abs() - tol).max()) if got.numel() else 0.0
    assert worst <= 1e-30, worst


def prompt_visible(torch, lens_q, lens_k):
    nq, nk = sum(lens_q), sum(lens_k)
    vis = torch.zeros(nq, nk, dtype=torch.bool, device="cuda")
    a = b = 0
    for m, n in zip(lens_q, lens_k):
        for i in range(m):
            vis[a + i, b:b + max(0, min(n, n - m + i + 1))] = True
        a, b = a + m, b + n
    return vis


def offsets(torch, lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


HEADS = [(4, 2, 64), (9, 3, 64), (7, 1, 128), (8, 8, 128), (32, 4, 64), (16, 2, 128)]
PROMPTS = [  # lengths of queries and keys
    ([1], [1]), ([5], [5]), ([33], [33]), ([64], [64]), ([65], [65]), ([150], [150]), ([1, 17, 100], [1, 17, 100]),
    ([3, 0, 40, 1], [70, 0, 40, 300]),       # earlier contexts, an empty sequence, a single token
    ([20, 9], [7, 0]),                        # fewer keys than queries, and none
    ([0, 0, 12], [5, 0, 12]), ([70, 1, 1, 1, 33], [130, 1, 257, 64, 33]),
]


@pytest.mark.parametrize("heads,kv,d", HEADS)
@pytest.mark.parametrize("lens_q,lens_k", PROMPTS)
def test_prompt_attention(env, heads, kv, d, lens_q, lens_k):
    amk, torch = env
    nq, nk = sum(lens_q), sum(lens_k)
    q = (randn(torch, 1, nq, heads, d) * 2).to(torch.bfloat16)
    k, v = randn(torch, 2, nk, kv, d).to(torch.bfloat16), randn(torch, 3, nk, kv, d).to(torch.bfloat16)
    got = amk.prompt_attention(q, k, v, offsets(torch, lens_q), offsets(torch, lens_k))
    close(torch, got, *softmax_rows(torch, q, k, v, prompt_visible(torch, lens_q, lens_k), d ** -0.5))
    if len(lens_q) == 1:
        assert torch.equal(amk.prompt_attention(q, k, v), got)


@pytest.mark.parametrize("heads,kv,d,nq,nk", [(8, 2, 128, 200, 700), (4, 4, 64, 90, 3000), (4, 1, 64, 513, 513),
                                              (8, 1, 128, 1030, 1100)])
def test_prompt_attention_longer(env, heads, kv, d, nq, nk):
    """Many key tiles, few row tiles: the keys of a tile may be split over workgroups."""
    amk, torch = env
    q = (randn(torch, 1, nq, heads, d) * 2).to(torch.bfloat16)
    k, v = randn(torch, 2, nk, kv, d).to(torch.bfloat16), randn(torch, 3, nk, kv, d).to(torch.bfloat16)
    got = amk.prompt_attention(q, k, v, scale=0.2)
    close(torch, got, *softmax_rows(torch, q, k, v, prompt_visible(torch, [nq], [nk]), 0.2))


def test_prompt_attention_long_contexts_of_several(env):
    """Sequences of few queries behind long contexts: keys split over workgroups, rows outside every
    sequence as they were."""
    amk, torch = env
    lens_q, lens_k, at = [30, 0, 41], [2999, 7, 2000], 5
    cu_q, cu_k = offsets(torch, lens_q) + at, offsets(torch, lens_k) + 3
    q = (randn(torch, 1, 90, 4, 64) * 2).to(torch.bfloat16)
    k, v = (randn(torch, s, 5100, 2, 64).to(torch.bfloat16) for s in (2, 3))
    held = randn(torch, 4, 90, 4, 64).to(torch.bfloat16)
    out = amk.prompt_attention(q, k, v, cu_q, cu_k, out=held.clone())
    ref, tol = softmax_rows(torch, q[at:76], k[3:5009], v[3:5009], prompt_visible(torch, lens_q, lens_k), 0.125)
    close(torch, out[at:76], ref, tol)
    assert torch.equal(out[:at], held[:at]) and torch.equal(out[76:], held[76:])


def test_prompt_attention_strides(env):
    """A cache layer as it lies, q in the middle of a wider projection, the output within a larger buffer
    whose other rows and columns stay."""
    amk, torch = env
    heads, kv, d, nq, nk = 6, 2, 128, 77, 109
    wide = randn(torch, 1, nq, heads + 4, d).to(torch.bfloat16)
    q = wide[:, 2:2 + heads]
    cache = randn(torch, 2, 2, kv, 200, d).to(torch.bfloat16)
    k, v = cache[0].transpose(0, 1)[:nk], cache[1].transpose(0, 1)[:nk]
    held = randn(torch, 3, nq + 5, heads + 1, d).to(torch.bfloat16)
    out = held.clone()
    amk.prompt_attention(q, k, v, offsets(torch, [70]), offsets(torch, [100]), out=out[:nq, 1:])
    ref, tol = softmax_rows(torch, q[:70], k[:100], v[:100], prompt_visible(torch, [70], [100]), d ** -0.5)
    close(torch, out[:70, 1:], ref, tol)
    assert torch.equal(out[70:], held[70:]) and torch.equal(out[:, 0], held[:, 0])


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("heads,kv,d", [(4, 2, 64), (8, 1, 128), (128, 1, 128)])
def test_prompt_attention_masked_values_stay_out(env, bad, heads, kv, d):
    """Infinities and NaN in K and V reach only the queries that see them: not those before, nor other
    sequences, nor through rows behind the last."""
    amk, torch = env
    lens, at = [100, 60], 43
    q = randn(torch, 1, 160, heads, d).to(torch.bfloat16)
    k, v = randn(torch, 2, 170, kv, d).to(torch.bfloat16), randn(torch, 3, 170, kv, d).to(torch.bfloat16)
    cu = offsets(torch, lens)
    clean = amk.prompt_attention(q, k, v, cu, cu)
    k[at, :, 5], v[at, :, 3], v[at + 1, :, 9] = bad, bad, bad
    k[160:], v[160:] = bad, bad
    got = amk.prompt_attention(q, k, v, cu, cu)
    assert torch.equal(got[:at], clean[:at]) and torch.equal(got[100:], clean[100:])
    if math.isnan(bad):
        assert torch.isnan(got[at:100]).all()


def test_prompt_attention_infinite_scores(env):
    """Visible keys scoring minus infinity have no weight; a row of only such keys gets zeros; a visible
    infinite value gives an infinite output."""
    amk, torch = env
    d = 64
    q = torch.ones(70, 1, d, dtype=torch.bfloat16, device="cuda")
    k, v = randn(torch, 2, 70, 1, d).to(torch.bfloat16), randn(torch, 3, 70, 1, d).to(torch.bfloat16)
    k[:3, :, 0] = -math.inf
    got = amk.prompt_attention(q, k, v)
    assert (got[:3] == 0).all()
    vis = prompt_visible(torch, [70], [70])
    vis[:, :3] = False
    ref, tol = softmax_rows(torch, q, k, v, vis, d ** -0.5)
    close(torch, got, ref, tol)
    v[20, 0, 7] = math.inf
    got = amk.prompt_attention(q, k, v)
    close(torch, got[:20], ref[:20], tol[:20])
    assert (got[20:, 0, 7] == math.inf).all()
    others = [i for i in range(d) if i != 7]
    close(torch, got[20:, :, others], ref[20:, :, others], tol[20:, :, others])


def test_prompt_attention_offsets_out_of_range(env):
    """Offsets past the tensors are cut to them."""
    amk, torch = env
    q = randn(torch, 1, 50, 4, 64).to(torch.bfloat16)
    k, v = randn(torch, 2, 50, 2, 64).to(torch.bfloat16), randn(torch, 3, 50, 2, 64).to(torch.bfloat16)
    cu = torch.tensor([-7, 50, 1 << 30], dtype=torch.int32, device="cuda")
    assert torch.equal(amk.prompt_attention(q, k, v, cu, cu), amk.prompt_attention(q, k, v))


def test_prompt_attention_many_sequences(env):
    """More sequences than a wave looks at at once, most of a few tokens."""
    amk, torch = env
    rng = np.random.RandomState(3)
    lens_q = [int(t) for t in rng.randint(0, 9, 150)]
    lens_k = [n + int(t) for n, t in zip(lens_q, rng.randint(0, 40, 150))]
    q = randn(torch, 1, sum(lens_q), 3, 64).to(torch.bfloat16)
    k, v = (randn(torch, s, sum(lens_k), 1, 64).to(torch.bfloat16) for s in (2, 3))
    got = amk.prompt_attention(q, k, v, offsets(torch, lens_q), offsets(torch, lens_k))
    close(torch, got, *softmax_rows(torch, q, k, v, prompt_visible(torch, lens_q, lens_k), 0.125))


def tree_visible(torch, n, pos, masks):
    vis = torch.zeros(n, pos + n, dtype=torch.bool, device="cuda")
    vis[:, :pos] = True
    for i, m in enumerate(masks):
        for j in range(n):
            vis[i, pos + j] = bool(m >> j & 1)
    return vis


TREES = [(1, 0), (1, 1), (1, 31), (1, 4000), (2, 63), (5, 0), (7, 127), (8, 300), (16, 128), (31, 1000), (33, 5),
         (64, 0), (64, 2017)]


@pytest.mark.parametrize("heads,kv,d", HEADS)
@pytest.mark.parametrize("n,pos", TREES)
def test_tree_attention(env, heads, kv, d, n, pos):
    amk, torch = env
    rng = np.random.RandomState(n + pos)
    parents = [int(rng.randint(max(-1, i - 5), i)) for i in range(n)]
    masks = amk.tree_masks(parents)
    q = (randn(torch, 1, n, heads, d) * 2).to(torch.bfloat16)
    cache = randn(torch, 2, 2, kv, pos + n + 3, d).to(torch.bfloat16)
    cache[:, :, pos + n:] = math.nan
    k, v = cache[0].transpose(0, 1), cache[1].transpose(0, 1)
    got = amk.tree_attention(q, k, v, pos, masks)
    close(torch, got, *softmax_rows(torch, q, k[:pos + n], v[:pos + n], tree_visible(torch, n, pos, masks), d ** -0.5))


def test_tree_attention_masks(env):
    """Any masks: none at all (a row behind no context gets zeros), bits past n ignored, a chain equals the
    causal prompt's rows."""
    amk, torch = env
    n, d = 40, 128
    q = randn(torch, 1, n, 4, d).to(torch.bfloat16)
    k, v = (randn(torch, s, 300, 2, d).to(torch.bfloat16) for s in (2, 3))
    rng = np.random.RandomState(1)
    masks = [int(rng.randint(0, 1 << 62)) & int(rng.randint(0, 1 << 62)) | 1 << 63 for _ in range(n)]
    masks[3] = masks[17] = 1 << 50
    for pos in (0, 100):
        got = amk.tree_attention(q, k, v, pos, masks)
        close(torch, got, *softmax_rows(torch, q, k[:pos + n], v[:pos + n], tree_visible(torch, n, pos, masks), d ** -0.5))
        if pos == 0:
            assert (got[3] == 0).all() and (got[17] == 0).all()
    chain = amk.tree_attention(q, k, v, 60, [(2 << i) - 1 for i in range(n)])
    ref, tol = softmax_rows(torch, q, k[:100], v[:100], prompt_visible(torch, [n], [100]), d ** -0.5)
    close(torch, chain, ref, tol)
    close(torch, amk.prompt_attention(q, k[:100], v[:100]), ref, tol)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_tree_attention_masked_values_stay_out(env, bad):
    """A sibling's infinities and NaN do not reach a branch, with keys in one range or in many, in small
    and large workgroups."""
    amk, torch = env
    for pos, n, d in ((10, 12, 64), (3000, 12, 64), (700, 50, 128)):
        q = randn(torch, 1, n, 8, d).to(torch.bfloat16)
        k, v = (randn(torch, s, pos + n, 2, d).to(torch.bfloat16) for s in (2, 3))
        masks = [1 << i | (1 << i % 2) for i in range(n)]  # two branches, of odd and even tokens
        clean = amk.tree_attention(q, k, v, pos, masks)
        k[pos + 1], v[pos + 1] = bad, bad
        got = amk.tree_attention(q, k, v, pos, masks)
        assert torch.equal(got[0::2], clean[0::2])
        assert not torch.isfinite(got[1::2].float()).any()


def test_attention_offsets_past_32_bits(env):
    """Heads of a long cache lie more than 2^32 bytes and 2^31 elements apart."""
    amk, torch = env
    cap, d = 6_000_000, 128
    store = torch.empty(2, 3, cap, d, dtype=torch.bfloat16, device="cuda")  # 9.2 GB
    rows = cap - 40
    store[:, :, rows - 50:rows + 8] = randn(torch, 1, 2, 3, 58, d).to(torch.bfloat16)
    q = randn(torch, 2, 8, 3, d).to(torch.bfloat16)
    tail = store[:, :, rows - 50:]
    k, v = tail[0].transpose(0, 1), tail[1].transpose(0, 1)
    masks = [(2 << i) - 1 for i in range(8)]
    ref, tol = softmax_rows(torch, q, k[:58], v[:58], tree_visible(torch, 8, 50, masks), d ** -0.5)
    close(torch, amk.tree_attention(q, k, v, 50, masks), ref, tol)
    close(torch, amk.prompt_attention(q, k[:58], v[:58]), ref, tol)


# ---- log probabilities -------------------------------------------------------------------
def check_logprobs(torch, amk, logits, tokens, top):
    lp, h, ids, tops = amk.token_logprobs(logits, tokens, top)
    x = logits.double()
    p = torch.log_softmax(x, dim=1)
    z = (x - x.amax(dim=1, keepdim=True)).clamp_min(-200.0)
    w = torch.softmax(x, dim=1)
    far = (w * z.abs()).sum(dim=1)
    # e^z is off by about (2 + 2 |z|) u, the sum by the depth of its tree (under 100 additions) u
    rel = U * (110 + 4 * far)
    for got, ref in ((lp, p.gather(1, tokens.long()[:, None])[:, 0]), ):
        assert torch.equal(torch.isinf(got), torch.isinf(ref))
        fine = torch.isfinite(ref)
        assert ((got.double() - ref).abs()[fine] <= (rel + 4 * U * (ref.abs() + x.abs().amax(dim=1)))[fine]).all()
    href = -(w * torch.where(w > 0, p, 0.0)).sum(dim=1)
    assert ((h.double() - href).abs() <= (1 + far) * rel * 2 + 4 * U * (href + far)).all()
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(ids.long(), order)
    ref = p.gather(1, order)
    assert torch.equal(torch.isinf(tops), torch.isinf(ref))
    fine = torch.isfinite(ref)
    assert ((tops.double() - ref).abs()[fine] <=
            (rel[:, None] + 4 * U * (ref.abs() + x.amax(dim=1)[:, None].abs()))[fine]).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("n,vocab,top", [(1, 1, 1), (1, 7, 3), (3, 33, 32), (2, 1000, 5), (5, 4096, 20), (4, 4097, 1),
                                         (1, 128256, 32), (130, 4099, 8), (100, 32003, 5), (3, 200001, 32),
                                         (1, 1 << 20, 32), (40, 16384, 0)])
def test_token_logprobs(env, dtype, n, vocab, top):
    amk, torch = env
    logits = (randn(torch, n, n, vocab) * 3).to(getattr(torch, dtype))
    tokens = torch.randint(0, vocab, (n,), device="cuda").to(torch.int32)
    check_logprobs(torch, amk, logits, tokens, top)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_token_logprobs_few_values(env, dtype):
    """Many equal logits: the lowest indices first, however many tie."""
    amk, torch = env
    for values in (1, 2, 5):
        logits = torch.randint(0, values, (6, 40003), device="cuda").to(getattr(torch, dtype))
        check_logprobs(torch, amk, logits, torch.arange(6, device="cuda").to(torch.int32), 32)
    # signed zeros are equal
    logits = torch.zeros(2, 100, device="cuda")
    logits[:, ::2] = -0.0
    assert amk.token_logprobs(logits, None, 5)[2].tolist() == [[0, 1, 2, 3, 4]] * 2


def test_token_logprobs_masked(env):
    """Impossible tokens, most or all but a few; an ascending and a descending row."""
    amk, torch = env
    n, vocab = 6, 50001
    logits = randn(torch, 1, n, vocab)
    logits[0, 100:] = -math.inf
    logits[1, :vocab - 3] = -math.inf
    logits[2] = -math.inf
    logits[2, 777] = 2.0
    logits[3, torch.rand(vocab, device="cuda") < 0.99] = -math.inf
    logits[4] = torch.arange(vocab, device="cuda") * 1e-3
    logits[5] = -torch.arange(vocab, device="cuda") * 1e-3
    check_logprobs(torch, amk, logits, torch.tensor([5, 5, 777, 9, 50000, 1], dtype=torch.int32, device="cuda"), 32)


def test_token_logprobs_without_softmax(env):
    """Rows with a NaN, plus infinity or nothing possible give NaN and -1; their neighbours do not change;
    tokens out of range give NaN."""
    amk, torch = env
    logits = randn(torch, 1, 6, 70000)
    tokens = torch.tensor([0, 1, 2, -1, 70000, 5], dtype=torch.int32, device="cuda")
    clean = amk.token_logprobs(logits, tokens, 4)
    logits[0, 69999], logits[2, 3], logits[5] = math.nan, math.inf, -math.inf
    lp, h, ids, tops = amk.token_logprobs(logits, tokens, 4)
    for i in (0, 2, 5):
        assert math.isnan(lp[i]) and math.isnan(h[i]) and torch.isnan(tops[i]).all() and (ids[i] == -1).all()
    assert torch.isnan(lp[3]) and torch.isnan(lp[4]) and lp[1] == clean[0][1]
    for i in (1, 3, 4):
        assert h[i] == clean[1][i] and torch.equal(ids[i], clean[2][i]) and torch.equal(tops[i], clean[3][i])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_token_logprobs_rows_apart(env, dtype):
    """Rows at every alignment, in the middle of a wider buffer of larger values."""
    amk, torch = env
    n, vocab = 9, 5003
    wide = torch.full((n, vocab + 10), 50.0, device="cuda").to(getattr(torch, dtype))
    for first in (0, 1, 3, 7):
        wide[:, first:first + vocab] = (randn(torch, first, n, vocab) * 3).to(wide.dtype)
        check_logprobs(torch, amk, wide[:, first:first + vocab], torch.arange(n, device="cuda").to(torch.int32), 8)
        wide[:, first:first + vocab] = 50.0


# ---- rows of a cache moved together --------------------------------------------------------
@pytest.mark.parametrize("layers,kv,cap,d,pos,rows", [
    (1, 1, 8, 64, 0, [0]), (2, 3, 20, 64, 3, [0, 2, 5, 16]), (3, 2, 100, 128, 36, [63]), (2, 4, 70, 128, 6, list(range(64))),
    (4, 1, 65, 64, 1, list(range(0, 64, 2))), (1, 2, 64, 128, 0, list(range(32, 64))), (2, 2, 9, 64, 4, [])])
def test_kv_keep(env, layers, kv, cap, d, pos, rows):
    amk, torch = env
    cache = randn(torch, 1, layers, 2, kv, cap, d).to(torch.bfloat16)
    cache[0, 0, 0, pos] = math.nan  # bits are moved, not values
    want = cache.clone()
    for i, r in enumerate(rows):
        want[:, :, :, pos + i] = cache[:, :, :, pos + r]
    amk.kv_keep(cache, pos, rows)
    assert torch.equal(cache.view(torch.int16), want.view(torch.int16))


# ---- streams, graphs, repetition -----------------------------------------------------------
def calls(amk, torch, seed):
    """One call of each operator on inputs of its own: (function, its outputs' list)."""
    x = randn(torch, seed, 100, 512).to(torch.bfloat16)
    w4, s4, _ = matrix(torch, "w4a16", 700, 512, 64, seed)
    q, k, v = (randn(torch, seed + i, 200, h, 64).to(torch.bfloat16) for i, h in enumerate((8, 2, 2)))
    cu = offsets(torch, [150, 50])
    kt, vt = (randn(torch, seed + i, 3000, 2, 64).to(torch.bfloat16) for i in (5, 6))
    logits = randn(torch, seed, 3, 70001)
    tokens = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    masks = [(2 << i) - 1 for i in range(20)]

    def run():
        return [amk.linear(x, w4, s4, "w4a16", 64), amk.linear(x[:9], w4, s4, "w4a16", 64),
                amk.prompt_attention(q, k, v, cu, cu), amk.prompt_attention(q[:70], kt, vt),
                amk.tree_attention(q[:20], kt, vt, 2900, masks), *amk.token_logprobs(logits, tokens, 7)]
    return run


def test_operators_on_two_streams(env):
    amk, torch = env
    runs = [calls(amk, torch, s) for s in (1, 2)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    got = [[], []]
    for _ in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(runs[i]())
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


def test_operators_in_graphs(env):
    """Two captured graphs replayed in turn with eager work between: every replay gives the eager bits."""
    amk, torch = env
    runs = [calls(amk, torch, s) for s in (3, 4)]
    want = [r() for r in runs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for r in runs:
            r()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for r in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(r())
        graphs.append(g)
    for _ in range(3):
        for i, g in enumerate(graphs):
            for o in outs[i]:
                o.zero_()
            g.replay()
            eager = runs[1 - i]()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))
            assert all(torch.equal(a, b) for a, b in zip(eager, want[1 - i]))
