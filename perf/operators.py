"""Measured cases of the operators for several tokens at once: what a program has them do around the decode step.

    linear    y = x W^T for n tokens, W in the decoder's weight formats (bf16, W8A16, W4A16)
    prompt    causal attention over whole prompts: packed sequences, grouped heads, an optional earlier context
    tree      attention of a tree of drafted tokens over a KV cache
    logprobs  log probabilities of given tokens, with the entropy and the most probable alternatives
    keep      the accepted rows of a drafted tree moved together in the KV cache of every layer

A case is a dict of plain values with the operator under "op".  ``run`` computes it in plain torch operations in
32 bits, or with the framework's operators where ``own`` is true; ``exact`` computes it in 64 bits from the
definition.  Shapes are those of ``synth/configs.py`` and generic odd ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False


# ------------------------------------------------------------------ cases
def _linear(fmt, n, inp, out, group=0, y="float32"):
    return {"op": "linear", "fmt": fmt, "n": n, "in": inp, "out": out, "group": group, "y": y}


def _prompt(heads, kv_heads, d, lens, context, cache):
    return {"op": "prompt", "heads": heads, "kv_heads": kv_heads, "d": d, "lens": lens, "context": context,
            "cache": cache}


def _tree(heads, kv_heads, d, n, pos):
    return {"op": "tree", "heads": heads, "kv_heads": kv_heads, "d": d, "n": n, "pos": pos}


def _logprobs(rows, vocab, dtype, top, masked=0.0):
    return {"op": "logprobs", "rows": rows, "vocab": vocab, "dtype": dtype, "top": top, "masked": masked}


def _keep(layers, kv_heads, d, cap, pos, drafted, kept):
    return {"op": "keep", "layers": layers, "kv_heads": kv_heads, "d": d, "cap": cap, "pos": pos,
            "drafted": drafted, "kept": kept}


def listed():
    cases = [
        # a small model checks five drafted tokens: int8 rows of odd width, all latency
        ("linear_w8a16_5", _linear("w8a16", 5, 576, 1536)),
        # a large model checks a tree of 32 drafted tokens: int4 weights stream past a few columns
        ("linear_w4a16_32", _linear("w4a16", 32, 4096, 14336, group=128)),
        # an odd number of prompt tokens through a ragged layer, the output in 16 bits
        ("linear_w8a16_301", _linear("w8a16", 301, 2768, 1043, y="bfloat16")),
        # the widest product of a long prompt
        ("linear_bf16_2048", _linear("bf16", 2048, 4096, 14336)),
        # several prompts of a 1B model together, one of a single token, some going on after an earlier context
        ("prompt_packed", _prompt(32, 4, 64, "1337,700,64,1,1500,490", "0,512,0,33,0,2000", False)),
        # one long prompt of an 8B model, read from its cache
        ("prompt_8192", _prompt(32, 8, 128, "8192", "0", True)),
        # a small model's tree of drafted tokens behind a short answer
        ("tree_8_at_300", _tree(9, 3, 64, 8, 300)),
        # a large tree of an 8B model at long context
        ("tree_64_at_32000", _tree(32, 8, 128, 64, 32001)),
        # one answer token and its alternatives, as a server returns them
        ("logprobs_1", _logprobs(1, 128256, "float32", 5)),
        # a text scored, most of its vocabulary allowed
        ("logprobs_1024", _logprobs(1024, 128256, "float32", 20, masked=0.1)),
        # seven of sixteen drafted tokens accepted in an 8B model's cache
        ("keep_7_of_16", _keep(32, 8, 128, 4096, 1000, 16, 7)),
        # a long branch of a large tree in a 1B model's cache, behind a single position
        ("keep_40_of_64", _keep(22, 4, 64, 2048, 1, 64, 40)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["linear", "prompt", "tree", "logprobs", "keep"])
    heads, kv_heads, d = rng.choice([(4, 2, 64), (9, 3, 64), (32, 4, 64), (32, 8, 64), (32, 8, 128), (15, 5, 64),
                                     (7, 1, 128), (8, 8, 128), (6, 2, 128)])
    if op == "linear":
        fmt = rng.choice(["bf16", "w8a16", "w4a16"])
        group = rng.choice([32, 64, 128, 256]) if fmt == "w4a16" else 0
        unit = group or 16
        inp = max(unit, _log(rng, 256, 14336) // unit * unit)
        out, n = _log(rng, 64, 14336), _log(rng, 1, 4096)
        while n * inp * out > 2048 * 4096 * 14336:
            n = max(1, n // 2)
        return _linear(fmt, n, inp, out, group, rng.choice(["float32", "bfloat16"]))
    if op == "prompt":
        count, room = _log(rng, 1, 24), 8000
        lens, context = [], []
        for _ in range(count):
            lens.append(_log(rng, 1, room if count == 1 else max(1, room // 2)))
            context.append(_log(rng, 1, max(1, (room - lens[-1]) // 4)) - 1 if rng.random() < 0.3 else 0)
            room = max(2, room - lens[-1] - context[-1])
        return _prompt(heads, kv_heads, d, ",".join(map(str, lens)), ",".join(map(str, context)),
                       rng.random() < 0.5)
    if op == "tree":
        return _tree(heads, kv_heads, d, _log(rng, 1, 64), _log(rng, 1, 30000) - 1)
    if op == "logprobs":
        vocab = _log(rng, 2000, 150000)
        rows = _log(rng, 1, min(2048, 131000000 // vocab))
        return _logprobs(rows, vocab, rng.choice(["float32", "bfloat16", "float16"]), rng.choice([0, 1, 5, 8, 20, 32]),
                         rng.choice([0.0, 0.1, 0.9]))
    drafted = _log(rng, 1, 64)
    pos = _log(rng, 1, 4000) - 1
    return _keep(rng.randint(1, 32), kv_heads, d, pos + drafted + rng.randint(0, 200), pos, drafted,
                 rng.randint(1, drafted))


# ------------------------------------------------------------------ inputs
class _State:
    pass


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(7000 + seed)


def _randn(gen, *shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def _ints(text):
    return [int(t) for t in text.split(",")]


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _pack_int4(codes):
    """Codes in [-8, 7], [out, in], in the decoder's nibble layout [out, in / 2]."""
    out, inp = codes.shape
    u = (codes + 8).to(torch.uint8).view(out, inp // 8, 2, 4)
    return (u[:, :, 0] | (u[:, :, 1] << 4)).reshape(out, inp // 2).contiguous()


def _prepare_linear(s, c, g, seed):
    n, inp, out = c["n"], c["in"], c["out"]
    s.x = _randn(g, n, inp)
    w = torch.randn(out, inp, generator=g, device="cuda") * 0.02
    s.scale = None
    if c["fmt"] == "bf16":
        s.w = w.to(torch.bfloat16)
    elif c["fmt"] == "w8a16":
        s.scale = w.abs().amax(dim=1) / 127.0
        s.w = torch.round(w / s.scale[:, None]).to(torch.int8)
    else:
        w = w.view(out, inp // c["group"], c["group"])
        s.scale = (w.abs().amax(dim=2) / 7.0).half()
        s.w = _pack_int4(torch.round(w / s.scale.float()[:, :, None]).clamp_(-8, 7).view(out, inp).to(torch.int16))


def _prepare_prompt(s, c, g, seed):
    lens, context = _ints(c["lens"]), _ints(c["context"])
    total_q, total_k = sum(lens), sum(lens) + sum(context)
    s.cu_q, s.cu_k = _offsets(lens), _offsets([a + b for a, b in zip(lens, context)])
    s.q = _randn(g, total_q, c["heads"], c["d"], std=2.0)
    if c["cache"]:  # one layer of a cache: [K, V][kv head][position][d]
        kv = _randn(g, 2, c["kv_heads"], total_k, c["d"])
        s.k, s.v = kv[0].transpose(0, 1), kv[1].transpose(0, 1)
    else:
        kv = _randn(g, total_k, 2, c["kv_heads"], c["d"])
        s.k, s.v = kv[:, 0], kv[:, 1]


def _prepare_tree(s, c, g, seed):
    n, pos = c["n"], c["pos"]
    r = random.Random(9000 + seed)
    s.masks = []
    for i in range(n):  # each drafted token under one of the few before it, or at the root
        parent = r.randint(max(-1, i - 6), i - 1)
        s.masks.append((1 << i) | (s.masks[parent] if parent >= 0 else 0))
    bits = [[(m >> j) & 1 for j in range(n)] for m in s.masks]
    s.visible = torch.tensor(bits, dtype=torch.bool, device="cuda")
    s.q = _randn(g, n, c["heads"], c["d"], std=2.0)
    kv = _randn(g, 2, c["kv_heads"], (pos + n + 255) // 256 * 256, c["d"])
    s.k, s.v = kv[0].transpose(0, 1), kv[1].transpose(0, 1)


def _prepare_logprobs(s, c, g, seed):
    rows, vocab = c["rows"], c["vocab"]
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 3.0
    if c["masked"]:
        x.masked_fill_(torch.rand(rows, vocab, generator=g, device="cuda") < c["masked"], -math.inf)
    s.tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    # a text's tokens are among those allowed
    x.scatter_(1, s.tokens.long()[:, None], torch.randn(rows, 1, generator=g, device="cuda") * 3.0)
    s.logits = x.to(getattr(torch, c["dtype"]))


def _prepare_keep(s, c, g, seed):
    s.kv = _randn(g, c["layers"], 2, c["kv_heads"], c["cap"], c["d"])
    s.rows = sorted(random.Random(9000 + seed).sample(range(c["drafted"]), c["kept"]))
    s.index = torch.tensor(s.rows, device="cuda") + c["pos"]


_PREPARE = {"linear": _prepare_linear, "prompt": _prepare_prompt, "tree": _prepare_tree, "logprobs": _prepare_logprobs,
            "keep": _prepare_keep}


def prepare(case, seed):
    s = _State()
    s.case = case
    _PREPARE[case["op"]](s, case, _gen(seed), seed)
    return s


# ------------------------------------------------------------------ one pass: the framework's operators
def _own(s):
    from paper_2606_09682_amd import amk
    c = s.case
    if c["op"] == "linear":
        return amk.linear(s.x, s.w, s.scale, weight_format=c["fmt"], group_size=c["group"],
                          out_dtype=getattr(torch, c["y"]))
    if c["op"] == "prompt":
        return amk.prompt_attention(s.q, s.k, s.v, s.cu_q, s.cu_k)
    if c["op"] == "tree":
        return amk.tree_attention(s.q, s.k, s.v, c["pos"], s.masks)
    if c["op"] == "logprobs":
        logprob, entropy, ids, top = amk.token_logprobs(s.logits, s.tokens, top=c["top"])
        return {"logprob": logprob, "entropy": entropy, "ids": ids, "top": top}
    amk.kv_keep(s.kv, c["pos"], s.rows)
    return s.kv


# ------------------------------------------------------------------ one pass: plain torch operations
def _weights(c, w, scale, dtype):
    """The dequantised matrix."""
    if c["fmt"] == "bf16":
        return w.to(dtype)
    if c["fmt"] == "w8a16":
        return w.to(dtype) * scale.to(dtype)[:, None]
    out, half = w.shape
    words = w.view(out, half // 4, 4)
    codes = torch.stack([words & 15, words >> 4], dim=2).reshape(out, -1, c["group"]).to(dtype) - 8
    return (codes * scale.to(dtype)[:, :, None]).view(out, 2 * half)


def _attention(q, k, v, visible):
    """softmax(q k^T / sqrt(d)) v over the visible keys in 32 bits; zeros where a row sees none."""
    heads, d = q.shape[1:]
    q = q.float().transpose(0, 1).contiguous()
    k = k.float().repeat_interleave(heads // k.shape[1], dim=1).permute(1, 2, 0).contiguous()
    v = v.float().repeat_interleave(heads // v.shape[1], dim=1).transpose(0, 1).contiguous()
    s = torch.bmm(q, k).mul_(1.0 / math.sqrt(d)).masked_fill_(~visible, -math.inf)
    m = s.amax(dim=2, keepdim=True)
    e = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    l = e.sum(dim=2, keepdim=True)
    return (torch.bmm(e, v) / torch.where(l == 0, 1.0, l)).transpose(0, 1).to(torch.bfloat16)


def _prompt_visible(s):
    """[queries, keys]: the key is of the query's sequence and not after the query."""
    i = torch.arange(s.q.shape[0], device="cuda", dtype=torch.int32)
    j = torch.arange(s.k.shape[0], device="cuda", dtype=torch.int32)
    seq_i = torch.bucketize(i, s.cu_q[1:], right=True)
    seq_j = torch.bucketize(j, s.cu_k[1:], right=True)
    last = i - s.cu_q[1:][seq_i] + s.cu_k[1:][seq_i]  # the sequences' last tokens are each other's
    return (seq_i[:, None] == seq_j[None, :]) & (j[None, :] <= last[:, None])


def _plain_logprobs(s):
    c = s.case
    x = s.logits.float() + 0.0
    m = x.amax(dim=1, keepdim=True)
    z = x - m
    e = z.exp()
    total = e.sum(dim=1, keepdim=True)
    lse = m + total.log()
    # an impossible token adds nothing to the entropy
    entropy = total.log()[:, 0] - torch.where(e > 0, z * e, 0.0).sum(dim=1) / total[:, 0]
    logprob = (x.gather(1, s.tokens.long()[:, None]) - lse)[:, 0]
    # the order of the values as whole numbers, the lowest index first among equal ones
    bits = x.view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
    at = torch.arange(c["vocab"], device="cuda")
    ids = torch.topk((order << 32) + (2 ** 31 - at), c["top"], dim=1).indices
    return {"logprob": logprob, "entropy": entropy, "ids": ids.to(torch.int32), "top": x.gather(1, ids) - lse}


def run(s):
    if own:
        return _own(s)
    c = s.case
    if c["op"] == "linear":
        y = torch.mm(s.x.float(), _weights(c, s.w, s.scale, torch.float32).t())
        return y.to(getattr(torch, c["y"]))
    if c["op"] == "prompt":
        return _attention(s.q, s.k, s.v, _prompt_visible(s))
    if c["op"] == "tree":
        pos, n = c["pos"], c["n"]
        context = torch.ones(n, pos, dtype=torch.bool, device="cuda")
        return _attention(s.q, s.k[:pos + n], s.v[:pos + n], torch.cat([context, s.visible], dim=1))
    if c["op"] == "logprobs":
        return _plain_logprobs(s)
    s.kv[:, :, :, c["pos"]:c["pos"] + c["kept"]] = s.kv.index_select(3, s.index)
    return s.kv


# ------------------------------------------------------------------ the same in 64 bits
def _exact_rows(q, k, v, scale):
    """One query head against the keys it sees all of: softmax in 64 bits."""
    w = (k @ q) * scale
    w = torch.exp(w - w.max())
    return (w @ v) / w.sum()


def _exact_prompt(s, c):
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    group, scale = c["heads"] // c["kv_heads"], 1.0 / math.sqrt(c["d"])
    q0 = k0 = 0
    for n, ctx in zip(_ints(c["lens"]), _ints(c["context"])):
        future = torch.arange(n + ctx, device="cuda")[None, :] > torch.arange(n, device="cuda")[:, None] + ctx
        for h in range(c["heads"]):
            q = s.q[q0:q0 + n, h].double()
            k, v = s.k[k0:k0 + n + ctx, h // group].double(), s.v[k0:k0 + n + ctx, h // group].double()
            w = torch.softmax((q @ k.t()).mul_(scale).masked_fill_(future, -math.inf), dim=1)
            out[q0:q0 + n, h] = w @ v
        q0, k0 = q0 + n, k0 + n + ctx
    return out


def _exact_tree(s, c):
    pos, n, group = c["pos"], c["n"], c["heads"] // c["kv_heads"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    for g in range(c["kv_heads"]):
        k, v = s.k[:pos + n, g].double(), s.v[:pos + n, g].double()
        for i, mask in enumerate(s.masks):
            see = torch.tensor(list(range(pos)) + [pos + j for j in range(n) if mask >> j & 1], device="cuda")
            ki, vi = k[see], v[see]
            for h in range(g * group, (g + 1) * group):
                out[i, h] = _exact_rows(s.q[i, h].double(), ki, vi, 1.0 / math.sqrt(c["d"]))
    return out


def _exact_logprobs(s, c):
    logprob, entropy, top = [], [], []
    for x, token in zip(s.logits.double(), s.tokens.tolist()):
        p = torch.log_softmax(x, dim=0)
        some = p[p > -math.inf]
        logprob.append(p[token])
        entropy.append(-(some.exp() * some).sum())
        top.append(p.sort(descending=True).values[:c["top"]])
    return {"logprob": torch.stack(logprob), "entropy": torch.stack(entropy), "ids": None, "top": torch.stack(top)}


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "linear":
        return torch.cat([s.x.double() @ _exact_weights(c, s, a, min(a + 2048, c["out"])).t()
                          for a in range(0, c["out"], 2048)], dim=1)
    if c["op"] == "prompt":
        return _exact_prompt(s, c)
    if c["op"] == "tree":
        return _exact_tree(s, c)
    if c["op"] == "logprobs":
        return _exact_logprobs(s, c)
    kv = s.kv.double()
    for i, row in enumerate(s.rows):
        kv[:, :, :, c["pos"] + i] = kv[:, :, :, c["pos"] + row]
    return kv


def _exact_weights(c, s, a, b):
    """Rows a to b of the matrix, column by column of its layout."""
    w = s.w[a:b]
    if c["fmt"] == "bf16":
        return w.double()
    if c["fmt"] == "w8a16":
        return w.double() * s.scale[a:b].double().view(-1, 1)
    full = torch.empty(b - a, c["in"], dtype=torch.float64, device="cuda")
    for t in range(8):  # column 8 d + t: byte 4 d + t % 4, the low nibble first
        byte = w[:, t % 4::4]
        full[:, t::8] = ((byte >> 4) if t >= 4 else (byte & 15)).double() - 8.0
    return full * s.scale[a:b].double().repeat_interleave(c["group"], dim=1)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "linear":
        n, inp, out = c["n"], c["in"], c["out"]
        weights = {"bf16": 2 * inp * out, "w8a16": inp * out + 4 * out,
                   "w4a16": inp * out // 2 + (2 * inp * out // c["group"] if c["group"] else 0)}[c["fmt"]]
        return {"bytes": weights + 2 * n * inp + n * out * (4 if c["y"] == "float32" else 2), "flops": 2 * n * inp * out}
    if c["op"] in ("prompt", "tree"):
        if c["op"] == "prompt":
            lens, context = _ints(c["lens"]), _ints(c["context"])
            pairs = sum(n * ctx + n * (n + 1) // 2 for n, ctx in zip(lens, context))
            q, k = sum(lens), sum(lens) + sum(context)
        else:
            q, k = c["n"], c["pos"] + c["n"]
            pairs = q * k
        return {"bytes": 4 * c["d"] * (q * c["heads"] + k * c["kv_heads"]), "flops": 4 * pairs * c["heads"] * c["d"]}
    if c["op"] == "logprobs":
        size = 4 if c["dtype"] == "float32" else 2
        return {"bytes": c["rows"] * (c["vocab"] * size + 12 + 8 * c["top"]), "flops": 6 * c["rows"] * c["vocab"]}
    return {"bytes": 8 * c["layers"] * c["kv_heads"] * c["d"] * c["kept"], "flops": 0}
