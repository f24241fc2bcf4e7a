"""Refusals of the operators for several tokens, all found on the host before any device call, and the
layout of their argument structure (no GPU)."""
import ctypes
import math
import os
import subprocess

import pytest

import synth
from paper_2606_09682_amd import amk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, UNSUPPORTED, OK = amk.AMK_ERR_INVALID_ARGUMENT, amk.AMK_ERR_UNSUPPORTED, amk.AMK_OK
P = 4096  # a 256-byte aligned address that is never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(amk.LIB_PATH):
        from paper_2606_09682_amd import build
        build.build()
    return amk.load()


def test_attention_struct_matches_header(tmp_path):
    fields = [n for n, _ in amk.amk_attention_t._fields_]
    src = "#include <stdio.h>\n#include <stddef.h>\n#include \"amk.h\"\nint main(void) {\n"
    src += 'printf("%zu\\n", sizeof(amk_attention_t));\n'
    src += "".join(f'printf("%zu\\n", offsetof(amk_attention_t, {f}));\n' for f in fields)
    src += 'printf("%d\\n%d\\n%d %d %d\\n", AMK_TREE_MAX, AMK_TOP_MAX, AMK_F32, AMK_BF16, AMK_F16);\nreturn 0; }\n'
    (tmp_path / "l.c").write_text(src)
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"),
                    "-o", str(tmp_path / "l")], check=True)
    got = subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()
    want = [ctypes.sizeof(amk.amk_attention_t)] + [getattr(amk.amk_attention_t, f).offset for f in fields]
    want += [amk.AMK_TREE_MAX, amk.AMK_TOP_MAX, amk.AMK_F32, amk.AMK_BF16, amk.AMK_F16]
    assert [int(t) for t in got] == want


LINEAR = dict(x=P, x_stride=64, n=3, width=64, out=5, w=P, scale=P, fmt=amk.AMK_WEIGHTS_BF16, group=0, y=P,
              y_stride=5, y_type=amk.AMK_F32, accumulate=0)
W8, W4 = {"fmt": amk.AMK_WEIGHTS_W8A16}, {"fmt": amk.AMK_WEIGHTS_W4A16, "width": 128, "x_stride": 128}


@pytest.mark.parametrize("over,status", [
    ({"x": None}, BAD), ({"w": None}, BAD), ({"y": None}, BAD), ({"x": P + 8}, BAD), ({"w": P + 4}, BAD),
    ({"y": P + 2}, BAD), ({"x_stride": 60}, BAD), ({"x_stride": 68}, BAD), ({"y_stride": 4}, BAD), ({"n": -1}, BAD),
    ({"out": -1}, BAD), ({"width": 0}, BAD), ({"width": 40}, UNSUPPORTED), ({"fmt": 3}, BAD), ({"fmt": -1}, BAD),
    ({"y_type": amk.AMK_F16}, BAD), ({"accumulate": 2}, BAD), ({**W8, "scale": None}, BAD), ({**W8, "scale": P + 2}, BAD),
    ({**W4, "scale": None}, BAD), ({**W4, "scale": P + 1}, BAD), ({**W4, "group": 48}, BAD), ({**W4, "group": 16}, BAD),
    ({**W4, "group": 2048}, BAD), ({**W4, "group": 256}, UNSUPPORTED), ({**W4, "width": 96}, UNSUPPORTED),
    ({"width": (1 << 22) + 16, "x_stride": (1 << 22) + 16}, UNSUPPORTED), ({"x_stride": (1 << 22) + 8}, UNSUPPORTED),
    ({"n": 0, "x": None, "y": None}, OK), ({"out": 0, "w": None}, OK)])
def test_linear_refusals(lib, over, status):
    a = {**LINEAR, **over}
    assert lib.amk_linear(a["x"], a["x_stride"], a["n"], a["width"], a["out"], a["w"], a["scale"], a["fmt"], a["group"],
                          a["y"], a["y_stride"], a["y_type"], a["accumulate"], None) == status


def attention(**over):
    a = amk.amk_attention_t(P, P, P, P, 256, 64, 128, 64, 128, 64, 256, 64, 4, 2, 64, 0.125)
    for name, value in over.items():
        setattr(a, name, value)
    return a


SHARED = [({"q": None}, BAD), ({"k": None}, BAD), ({"v": None}, BAD), ({"out": None}, BAD), ({"q": P + 2}, BAD),
          ({"k": P + 8}, BAD), ({"v": P + 4}, BAD), ({"out": P + 8}, BAD), ({"n_heads": 0}, BAD), ({"n_kv_heads": 0}, BAD),
          ({"n_heads": 5}, UNSUPPORTED), ({"head_dim": 96}, UNSUPPORTED), ({"scale": 0.0}, BAD), ({"scale": -1.0}, BAD),
          ({"k_token": (1 << 24) + 8}, UNSUPPORTED), ({"v_token": (1 << 24) + 8}, UNSUPPORTED), ({"scale": math.inf}, BAD), ({"scale": math.nan}, BAD)]
SHARED += [({f"{t}_{s}": v}, BAD) for t in ("q", "k", "v", "out") for s in ("token", "head") for v in (0, -64, 68)]


@pytest.mark.parametrize("over,status", SHARED)
def test_attention_refusals(lib, over, status):
    a = attention(**over)
    masks = (ctypes.c_uint64 * 3)(1, 3, 7)
    assert lib.amk_prompt_attention(a, P, P, 2, 10, 10, P, 1 << 40, None) == status
    assert lib.amk_tree_attention(a, 3, 5, masks, P, 1 << 40, None) == status


def test_prompt_attention_refusals(lib):
    a = attention()
    call = lambda *args: lib.amk_prompt_attention(a, *args)  # noqa: E731
    assert lib.amk_prompt_attention(None, P, P, 1, 1, 1, None, 0, None) == BAD
    for args in ((P, None, 1, 5, 5), (None, P, 1, 5, 5), (None, None, 2, 5, 5), (None, None, 0, 5, 5), (P, P, -1, 5, 5),
                 (P, P, 1, -1, 5), (P, P, 1, 5, -1), (P + 2, P, 1, 5, 5), (P, P + 1, 1, 5, 5)):
        assert call(*args, None, 0, None) == BAD, args
    assert call(P, P, 0, 5, 5, None, 0, None) == OK and call(P, P, 3, 0, 5, None, 0, None) == OK
    assert call(P, P, 1, (1 << 28) + 1, 5, P, 1 << 60, None) == UNSUPPORTED
    assert call(P, P, 1, 5, (1 << 30) + 1, P, 1 << 60, None) == UNSUPPORTED
    # a workspace that is missing, too small or not aligned, where one is needed
    need = lib.amk_prompt_attention_workspace(4, 2, 64, 1, 65, 20000)
    assert need > 0
    for ws, size in ((None, need), (P, need - 1), (P + 128, need)):
        assert call(None, None, 1, 65, 20000, ws, size, None) == BAD
    for bad in ((0, 2, 64, 1, 5, 5), (4, 0, 64, 1, 5, 5), (5, 2, 64, 1, 5, 5), (4, 2, 32, 1, 5, 5), (4, 2, 64, 0, 5, 5),
                (4, 2, 64, 1, 0, 5), (4, 2, 64, 1, 5, -1)):
        assert lib.amk_prompt_attention_workspace(*bad) == 0


def test_tree_attention_refusals(lib):
    a, masks = attention(), (ctypes.c_uint64 * 64)(*([1] * 64))
    assert lib.amk_tree_attention(None, 1, 0, masks, None, 0, None) == BAD
    for n, pos, m in ((-1, 0, masks), (65, 0, masks), (1, -1, masks), (1, (1 << 31) - 1, masks), (1, 0, None)):
        assert lib.amk_tree_attention(a, n, pos, m, P, 1 << 40, None) == BAD
    assert lib.amk_tree_attention(a, 0, 0, None, None, 0, None) == OK
    assert lib.amk_tree_attention(a, 1, 1 << 30, masks, P, 1 << 40, None) == UNSUPPORTED
    need = lib.amk_tree_attention_workspace(4, 2, 64, 8, 5000)
    assert need > 0
    for ws, size in ((None, need), (P, need - 1), (P + 64, need)):
        assert lib.amk_tree_attention(a, 8, 5000, masks, ws, size, None) == BAD
    for bad in ((0, 2, 64, 1, 5), (4, 2, 96, 1, 5), (4, 2, 64, 0, 5), (4, 2, 64, 65, 5), (4, 2, 64, 1, -1)):
        assert lib.amk_tree_attention_workspace(*bad) == 0


LOGPROBS = dict(logits=P, type=amk.AMK_F32, stride=100, n=2, vocab=100, tokens=P, top=3, logprob=P, entropy=P, ids=P,
                tops=P, ws=P, size=1 << 30)


@pytest.mark.parametrize("over,status", [
    ({"logits": None}, BAD), ({"logits": P + 2}, BAD), ({"type": 3}, BAD), ({"type": -1}, BAD), ({"stride": 99}, BAD),
    ({"n": -1}, BAD), ({"vocab": 0}, BAD), ({"vocab": (1 << 20) + 1, "stride": 1 << 21}, BAD), ({"top": -1}, BAD),
    ({"top": 33}, BAD), ({"vocab": 2}, BAD), ({"tokens": None}, BAD), ({"logprob": None}, BAD), ({"ids": None}, BAD),
    ({"tops": None}, BAD), ({"entropy": P + 1}, BAD), ({"ids": P + 2}, BAD), ({"tokens": P + 3}, BAD), ({"ws": None}, BAD),
    ({"ws": P + 4}, BAD), ({"size": 16}, BAD), ({"n": 0, "logits": None}, OK)])
def test_token_logprobs_refusals(lib, over, status):
    a = {**LOGPROBS, **over}
    assert lib.amk_token_logprobs(a["logits"], a["type"], a["stride"], a["n"], a["vocab"], a["tokens"], a["top"],
                                  a["logprob"], a["entropy"], a["ids"], a["tops"], a["ws"], a["size"], None) == status
    assert lib.amk_token_logprobs_workspace(0, 1, 0, 1) == lib.amk_token_logprobs_workspace(0, 1, 10, 33) == 0


KEEP = dict(kv=P, layers=2, heads=3, cap=50, d=64, pos=10, rows=(0, 2, 39), n=3)


@pytest.mark.parametrize("over,status", [
    ({"kv": None}, BAD), ({"kv": P + 8}, BAD), ({"layers": 0}, BAD), ({"heads": 0}, BAD), ({"cap": 0}, BAD),
    ({"d": 32}, UNSUPPORTED), ({"pos": -1}, BAD), ({"rows": None}, BAD), ({"rows": (0, 2, 40)}, BAD),
    ({"rows": (-1, 2, 3)}, BAD), ({"rows": (0, 2, 2)}, BAD), ({"rows": (3, 2, 4)}, BAD), ({"n": -1}, BAD),
    ({"n": 65, "rows": tuple(range(65)), "cap": 500}, BAD), ({"n": 0, "rows": None, "kv": None}, OK)])
def test_kv_keep_refusals(lib, over, status):
    a = {**KEEP, **over}
    rows = None if a["rows"] is None else (ctypes.c_int32 * len(a["rows"]))(*a["rows"])
    assert lib.amk_kv_keep(a["kv"], a["layers"], a["heads"], a["cap"], a["d"], a["pos"], rows, a["n"], None) == status


def test_extend_without_a_handle(lib):
    tok = (ctypes.c_int32 * 1)(0)
    assert lib.amk_extend(None, tok, 1, 0, None, P, P, 1, P, 1 << 40, None) == BAD
    assert lib.amk_extend_workspace(None, 1) == 0


def test_tree_masks():
    assert amk.tree_masks([-1, 0, 0, 1, -1]) == [1, 3, 5, 11, 16]
    for bad in ([0], [-2], [-1, 1]):
        with pytest.raises(ValueError):
            amk.tree_masks(bad)


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        amk.linear(x, x)
    with pytest.raises(ValueError, match="device tensor"):
        amk.prompt_attention(x.view(2, 1, 64), x.view(2, 1, 64), x.view(2, 1, 64))
    with pytest.raises(ValueError, match="device tensor"):
        amk.token_logprobs(x.float())
    with pytest.raises(ValueError, match="device tensor"):
        amk.kv_keep(torch.zeros(1, 2, 1, 8, 64, dtype=torch.bfloat16), 0, [0])
    with pytest.raises(ValueError, match="unknown weight format"):
        amk.linear(x, x, weight_format="fp8")


@pytest.mark.parametrize("name", sorted(synth.CONFIGS))
def test_every_shape_of_the_framework_is_taken(lib, name):
    """Workspaces of every model shape stay bounded: what amk_extend takes them from is one size for all
    prompts and positions."""
    c = synth.get(name)
    for tokens in (65, 70, 1000, 2048):
        for keys in (tokens, 5000, 100000, 1 << 20):
            need = lib.amk_prompt_attention_workspace(c.n_heads, c.n_kv_heads, c.head_dim, 1, tokens, keys)
            assert need <= 2048 * 32 * (4 * c.head_dim + 8) + 256
    for tokens in (1, 2, 17, 64):
        for keys in (0, 100, 5000, 1 << 20):
            need = lib.amk_tree_attention_workspace(c.n_heads, c.n_kv_heads, c.head_dim, tokens, keys)
            assert need <= 2048 * 32 * (4 * c.head_dim + 8) + 256
