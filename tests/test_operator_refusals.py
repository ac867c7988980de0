"""What the operators around the decode step refuse on the host: nothing is launched, so no GPU is needed."""
import ctypes
import re

import pytest

import paper_2508_11553_amd as sd
from tests.test_abi import HEADER, good_shape, lib  # noqa: F401


def good_norm(**over):
    f = dict(num_q_heads=8, num_kv_heads=2, head_dim=64, rotary_dim=64, interleaved=0, table_len=100, weight_dtype=sd.SD_BF16, eps=1e-6, q_stride=0, k_stride=0, v_stride=0)
    f.update(over)
    return sd.QkNorm(**f)


def test_norm_struct_matches_header():
    body = re.search(r"typedef struct \{([^}]*)\} sd_qk_norm;", open(HEADER).read(), flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = []
    for kind, names in re.findall(r"(int32_t|int64_t|float)\s+([\w, ]+);", body):
        fields += [(n.strip(), {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}[kind]) for n in names.split(",")]
    assert fields == list(sd.QkNorm._fields_)


NORM = dict(q=16, k=32, qw=48, kw=64, table=80, positions=96)


def rows(lib, norm, T=3, q_out=112, k_out=128, **over):
    p = {**NORM, **over}
    return lib.qk_norm_rope(ctypes.byref(norm), p["q"], p["k"], p["qw"], p["kw"], p["table"], p["positions"], T, q_out, k_out, None)


def append(lib, shape, norm, T=3, v=144, seq=160, slots=176, q_out=112, kp=192, vp=208, bt=224, **over):
    p = {**NORM, **over}
    return lib.qk_norm_rope_append(ctypes.byref(shape) if shape else None, ctypes.byref(norm), p["q"], p["k"], v, p["qw"], p["kw"], p["table"], p["positions"], seq, slots, T, q_out, kp, vp, bt, None)


def gradient(lib, norm, T=3, dqo=112, dko=128, dq=144, dk=160, dqw=176, dkw=192, ws=208, size=1 << 30, **over):
    p = {**NORM, **over}
    return lib.qk_norm_rope_backward(ctypes.byref(norm), dqo, dko, p["q"], p["k"], p["qw"], p["kw"], p["table"], p["positions"], T, dq, dk, dqw, dkw, ws, size, None)


BAD_NORMS = [
    (dict(num_q_heads=0), -1), (dict(num_kv_heads=-1), -1), (dict(head_dim=96), -2), (dict(head_dim=0), -1), (dict(rotary_dim=8), -1), (dict(rotary_dim=80), -1),
    (dict(rotary_dim=-16), -1), (dict(table_len=0), -1), (dict(interleaved=2), -1), (dict(weight_dtype=1), -1), (dict(weight_dtype=7), -1), (dict(eps=-1e-9), -1),
    (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(q_stride=511), -1), (dict(q_stride=504), -1), (dict(q_stride=516), -1), (dict(k_stride=120), -1),
    (dict(v_stride=-128), -1),
]


@pytest.mark.parametrize("over,code", BAD_NORMS)
def test_bad_norms(lib, over, code):
    n = good_norm(**over)
    assert rows(lib, n) == code and append(lib, good_shape(), n) in (code, -1) and gradient(lib, n) == code
    assert sd.qk_norm_rope_workspace_bytes(n, 5) == 0


@pytest.mark.parametrize("value", [None, 24])
def test_bad_pointers_of_the_norms(lib, value):
    n, s = good_norm(), good_shape()
    for name in NORM:
        assert rows(lib, n, **{name: value}) == -1 and append(lib, s, n, **{name: value}) == -1 and gradient(lib, n, **{name: value}) == -1
    for name in ("q_out", "k_out"):
        assert rows(lib, n, **{name: value}) == -1
    for name in ("v", "q_out", "kp", "vp", "bt"):
        assert append(lib, s, n, **{name: value}) == -1
    for name in ("dqo", "dko", "dq", "dk", "dqw", "dkw", "ws"):
        assert gradient(lib, n, **{name: value}) == -1
    if value:
        assert append(lib, s, n, seq=value) == -1 and append(lib, s, n, slots=value) == -1


def test_other_refusals_of_the_norms(lib):
    n, s = good_norm(), good_shape()
    assert lib.qk_norm_rope(None, 16, 32, 48, 64, 80, 96, 3, 112, 128, None) == -1
    assert rows(lib, n, T=-1) == -1 and append(lib, s, n, T=-1) == -1 and gradient(lib, n, T=-1) == -1
    assert rows(lib, n, T=0) == 0 and append(lib, s, n, T=0) == 0
    assert rows(lib, n, T=2 ** 28) == -2 and append(lib, s, n, T=2 ** 28) == -2 and gradient(lib, n, T=2 ** 28) == -2      # 2^28 x 12 rows of heads
    assert append(lib, None, n) == -1
    assert append(lib, good_shape(num_q_heads=4), n) == -1 and append(lib, good_shape(head_dim=128), n) == -1
    assert append(lib, good_shape(kv_dtype=sd.SD_FP8_E4M3), n) == -2
    assert append(lib, s, good_norm(rotary_dim=0), slots=None, positions=None) == -1       # nothing says where the rows go
    need = sd.qk_norm_rope_workspace_bytes(n, 3)
    assert need > 0 and gradient(lib, n, size=need - 1) == -3
    assert gradient(lib, n, T=0, size=0) == -3


def weights(lib, shape, q=16, qs=None, total=4, most=1, kp=48, ks=None, bt=64, lens=80, scale=0.125, decay=1.0, new=1, sin=96, sout=112, stride=512, ws=128, size=1 << 40):
    return lib.paged_weight_accumulate(ctypes.byref(shape), q, qs, total, most, kp, ks, bt, lens, scale, decay, new, sin, sout, stride, ws, size, None)


def test_weight_refusals(lib):
    s = good_shape()
    for value in (None, 24):
        for name in ("q", "kp", "bt", "lens", "sout", "ws"):
            assert weights(lib, s, **{name: value}) == -1
    assert weights(lib, s, sin=24) == -1 and weights(lib, s, qs=24, total=9, most=3) == -1
    assert weights(lib, s, total=3) == -1 and weights(lib, s, most=2) == -1       # without q_start one row each
    assert weights(lib, s, qs=32, total=-1) == -1 and weights(lib, s, qs=32, most=-1) == -1 and weights(lib, s, new=-1) == -1
    assert weights(lib, s, stride=508) == -1 and weights(lib, s, stride=514) == -1
    assert weights(lib, s, scale=float("nan")) == -1 and weights(lib, s, decay=float("nan")) == -1
    assert weights(lib, good_shape(kv_dtype=sd.SD_FP8_E4M3)) == -1                # fp8 pools come with scales
    assert weights(lib, good_shape(head_dim=96)) == -2 and weights(lib, good_shape(page_size=8)) == -1
    need = sd.paged_weight_workspace_bytes(s, 1)
    assert need > 0 and weights(lib, s, size=need - 1) == -3
    assert sd.paged_weight_workspace_bytes(s, -1) == 0 and sd.paged_weight_workspace_bytes(good_shape(head_dim=96), 1) == 0
    assert weights(lib, good_shape(batch=0), total=0, q=None, kp=None) == 0
    assert sd.paged_weight_workspace_bytes(s, 64) > 0


@pytest.mark.parametrize("heads,most", [(4, 1), (8, 1), (16, 1), (64, 1), (8, 3), (16, 40)])
def test_weight_workspace_of_a_large_call_serves_the_smaller(heads, most):
    sizes = [[sd.paged_weight_workspace_bytes(good_shape(batch=b, num_q_heads=heads, num_kv_heads=2, max_blocks_per_seq=8192, max_context_len=n), most)
              for n in (0, 1, 100, 1000, 1023, 4096, 5000, 9000, 70000, 131072)] for b in (1, 2, 13, 40, 79, 80, 81, 200, 499, 500, 1000)]
    for x, y in zip(sizes, sizes[1:]):
        assert all(0 < i <= j for i, j in zip(x, y))
    for x in sizes:
        assert x == sorted(x)


def evict(lib, shape, budget=100, sinks=4, recent=20, scores=16, stride=512, kp=32, vp=48, ks=None, vs=None, bt=64, lens=80, nbt=96, kept=112, nl=128, out=144, ostride=100):
    return lib.kv_evict(ctypes.byref(shape), budget, sinks, recent, scores, stride, kp, vp, ks, vs, bt, lens, nbt, kept, nl, out, ostride, None)


def test_evict_refusals(lib):
    s = good_shape()
    for value in (None, 24):
        for name in ("scores", "kp", "vp", "bt", "lens", "nbt", "kept", "nl"):
            assert evict(lib, s, **{name: value}) == -1
    assert evict(lib, s, out=24) == -1
    assert evict(lib, s, budget=0) == -1 and evict(lib, s, sinks=-1) == -1 and evict(lib, s, recent=-1) == -1 and evict(lib, s, sinks=50, recent=51) == -1
    assert evict(lib, s, sinks=2 ** 31 - 1, recent=2 ** 31 - 1) == -1
    assert evict(lib, s, stride=508) == -1 and evict(lib, s, stride=514) == -1 and evict(lib, s, ostride=99) == -1 and evict(lib, s, out=16, ostride=100) == -1
    assert evict(lib, good_shape(kv_dtype=sd.SD_FP8_E4M3)) == -1
    assert evict(lib, good_shape(head_dim=32)) == -2
    assert evict(lib, good_shape(batch=0), scores=None) == 0
