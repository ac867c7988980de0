"""What sampling, log probabilities and the plan of a step refuse on the host: nothing is launched, so no GPU is needed."""
import ctypes
import re

import pytest

import paper_2508_11553_amd as sd
from tests.test_abi import HEADER, good_shape, lib  # noqa: F401


def good_logits(**over):
    f = dict(rows=3, vocab=1000, dtype=sd.SD_BF16, stride=0)
    f.update(over)
    return sd.Logits(**f)


def test_logits_struct_matches_header():
    body = re.search(r"typedef struct \{([^}]*)\} sd_logits;", open(HEADER).read(), flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = [(name, {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64}[kind]) for kind, name in re.findall(r"(int32_t|int64_t)\s+(\w+);", body)]
    assert fields == list(sd.Logits._fields_)


def sample(lib, shape, x=16, t=32, k=48, p=64, m=80, u=96, tokens=112, lp=128, dlp=144, ws=160, size=1 << 40):
    return lib.sample_tokens(ctypes.byref(shape) if shape else None, x, t, k, p, m, u, tokens, lp, dlp, ws, size, None)


def score(lib, shape, x=16, y=32, t=48, lp=64, H=80, stats=96, ws=112, size=1 << 40):
    return lib.token_logprobs(ctypes.byref(shape) if shape else None, x, y, t, lp, H, stats, ws, size, None)


def gradient(lib, shape, x=16, y=32, t=48, stats=64, H=80, g=96, h=112, d=128):
    return lib.token_logprobs_backward(ctypes.byref(shape) if shape else None, x, y, t, stats, H, g, h, d, None)


@pytest.mark.parametrize("over,code", [(dict(rows=-1), -1), (dict(vocab=0), -1), (dict(vocab=-5), -1), (dict(dtype=sd.SD_FP8_E4M3), -1), (dict(dtype=3), -1), (dict(stride=999), -1),
                                       (dict(stride=-1000), -1), (dict(vocab=2 ** 30), -2), (dict(stride=2 ** 41), -2)])
def test_bad_logits(lib, over, code):  # noqa: F811
    s = good_logits(**over)
    assert sample(lib, s) == code and score(lib, s) == code and gradient(lib, s) == code
    assert sd.sample_workspace_bytes(s) == 0 and sd.token_logprobs_workspace_bytes(s) == 0


def test_missing_logits(lib):  # noqa: F811
    assert sample(lib, None) == -1 and score(lib, None) == -1 and gradient(lib, None) == -1
    assert lib.sample_workspace_bytes(None) == 0 and lib.token_logprobs_workspace_bytes(None) == 0


@pytest.mark.parametrize("value", [None, 24])
def test_bad_pointers(lib, value):  # noqa: F811
    s = good_logits()
    for name in ("x", "u", "tokens", "ws"):
        assert sample(lib, s, **{name: value}) == -1
    for name in ("x", "y", "lp", "ws"):
        assert score(lib, s, **{name: value}) == -1
    for name in ("x", "y", "stats", "g", "d"):
        assert gradient(lib, s, **{name: value}) == -1
    for name in ("H", "h"):                                   # the two come together
        assert gradient(lib, s, **{name: value}) == -1
    if value:
        for name in ("t", "k", "p", "m", "lp", "dlp"):
            assert sample(lib, s, **{name: value}) == -1
        for name in ("t", "H", "stats"):
            assert score(lib, s, **{name: value}) == -1
        assert gradient(lib, s, t=value) == -1


def test_other_refusals_of_logits(lib):  # noqa: F811
    s = good_logits()
    need = sd.sample_workspace_bytes(s)
    assert need > 0 and sample(lib, s, size=need - 1) == -3
    need = sd.token_logprobs_workspace_bytes(s)
    assert need > 0 and score(lib, s, size=need - 1) == -3
    none = good_logits(rows=0)
    assert sample(lib, none, x=None, ws=None) == 0 and score(lib, none, x=None, ws=None) == 0 and gradient(lib, none, x=None) == 0
    assert sample(lib, good_logits(vocab=2 ** 20)) == -2 and sd.sample_workspace_bytes(good_logits(vocab=2 ** 20)) == 0
    many = good_logits(rows=2 ** 31 - 1, vocab=100000)
    assert sample(lib, many, size=2 ** 62) == -2 and score(lib, many) == -2 and gradient(lib, many) == -2


def test_workspaces_of_larger_calls_serve_smaller_ones(lib):  # noqa: F811
    for f in (sd.sample_workspace_bytes, sd.token_logprobs_workspace_bytes):
        for dtype in (sd.SD_BF16, sd.SD_F32):
            sizes = [[f(good_logits(rows=r, vocab=v, dtype=dtype)) for v in (1, 100, 4096, 50000, 131072, 200001, 1000000)] for r in (0, 1, 2, 15, 16, 17, 63, 64, 100, 255, 256, 257, 1000, 5000)]
            for x, y in zip(sizes, sizes[1:]):
                assert all(0 < i <= j for i, j in zip(x, y))
            for x in sizes:
                assert x == sorted(x)
    sizes = [sd.kv_plan_workspace_bytes(good_shape(batch=b)) for b in (0, 1, 2, 3, 4, 5, 100, 1023, 1024, 1025, 100000)]
    assert sizes == sorted(sizes) and sizes[0] > 0


PLAN = dict(new=16, shared=32, lens=48, lens_out=64, nxt=80, nxt_out=96, pages=112, free=128, free_out=144, table=160, granted=176, row_start=192, starts=208, seq=224, slots=240, positions=256, ws=272)


def plan(lib, shape, rows=8, size=1 << 40, **over):
    p = {**PLAN, **over}
    return lib.kv_plan_step(ctypes.byref(shape) if shape else None, p["new"], p["shared"], p["lens"], p["lens_out"], p["nxt"], p["nxt_out"], p["pages"], p["free"], p["free_out"], p["table"], rows,
                            p["granted"], p["row_start"], p["starts"], p["seq"], p["slots"], p["positions"], p["ws"], size, None)


@pytest.mark.parametrize("over,code", [(dict(batch=-1), -1), (dict(num_pages=-1), -1), (dict(page_size=32), -1), (dict(max_blocks_per_seq=0), -1), (dict(max_context_len=-1), -1),
                                       (dict(max_context_len=513), -1), (dict(batch=1 << 24), -2)])
def test_bad_shapes_of_a_plan(lib, over, code):  # noqa: F811
    s = good_shape(**over)
    assert plan(lib, s) == code and sd.kv_plan_workspace_bytes(s) == 0


def test_refusals_of_a_plan(lib):  # noqa: F811
    s = good_shape()
    assert plan(lib, None) == -1 and plan(lib, s, rows=-1) == -1
    for name in PLAN:
        assert plan(lib, s, **{name: 24}) == -1, name
        if name not in ("shared", "positions"):
            assert plan(lib, s, **{name: None}) == -1, name
    need = sd.kv_plan_workspace_bytes(s)
    assert plan(lib, s, size=need - 1) == -3
    assert plan(lib, good_shape(batch=0), new=None, ws=None) == 0
