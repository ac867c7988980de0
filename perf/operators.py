"""Performance cases of the operators around the paged attention of a decode step: the rows that go into the cache,
and what the cache keeps of them.

A case is one pass of one of these (`path`):
  append    a step's or a resumed stretch's rows, straight from the fused projection: every head's query and key
            normalised and rotated to its position, keys and values put into the sequence's pages
  train     the same rows of a training step: normalised and rotated queries and keys, then the gradients of the
            projections and of the norms' weights
  weights   the attention weight that every cached token has received, brought up to date: one query row per
            sequence, or the last `window` rows of each
  evict     a cache cut down to `budget` tokens per sequence and head: the first `sinks`, the last `recent` and those
            of the largest accumulated weight stay, moved into new pages in their order

Lengths and positions follow from the case alone (`mix` seeds them); values, page placement and everything else come
from the seed.  With `own` the framework's entry points run; without it the same in elementary torch operations.
"""
import math
import random

import torch

own = False

PAGE = 16
FP8_MAX = 448.0
EPS = 1e-6
THETA = 10000.0


def listed():
    return [
        # one generated token for each of 64 sequences: as many rows as a decode step brings, nothing but latency
        dict(name="append_step", path="append", batch=64, new=1, lo=1024, hi=8192, heads=28, kv_heads=4, dim=128, rotary=128, interleaved=False, mix=1),
        # 16 paused sequences resume, 2048 stored tokens each go back into the cache
        dict(name="append_resume", path="append", batch=16, new=2048, lo=8192, hi=8192, heads=32, kv_heads=8, dim=128, rotary=128, interleaved=False, mix=2),
        # a tool's answer for a few sequences, small heads of which half is rotated, in neighbouring pairs
        dict(name="append_answers", path="append", batch=5, new=171, lo=300, hi=6000, heads=40, kv_heads=8, dim=64, rotary=32, interleaved=True, mix=3),
        # a small micro-batch of a training step
        dict(name="train_small", path="train", tokens=1531, lo=100, hi=700, heads=16, kv_heads=2, dim=128, rotary=128, interleaved=False, mix=4),
        # an ordinary one: 16 k tokens of packed trajectories
        dict(name="train_packed", path="train", tokens=16384, lo=1024, hi=8192, heads=64, kv_heads=8, dim=128, rotary=128, interleaved=False, mix=5),
        # a handful of short sequences: latency
        dict(name="weights_tiny", path="weights", kv="bf16", batch=4, window=1, dist="uniform", lo=1, hi=512, heads=8, kv_heads=2, dim=64, decay=1.0, mix=6),
        # an ordinary step of a rollout (64 sequences of 1 k to 8 k tokens)
        dict(name="weights_rollout", path="weights", kv="bf16", batch=64, window=1, dist="uniform", lo=1024, hi=8192, heads=28, kv_heads=4, dim=128, decay=1.0, mix=7),
        # a wide batch over an fp8 cache, old weight fading
        dict(name="weights_fp8_wide", path="weights", kv="fp8", batch=256, window=1, dist="uniform", lo=512, hi=4096, heads=64, kv_heads=8, dim=128, decay=0.97, mix=8),
        # prompts have gone into the cache: the weights of their last 64 tokens
        dict(name="weights_window", path="weights", kv="bf16", batch=8, window=64, dist="uniform", lo=5000, hi=8192, heads=32, kv_heads=8, dim=128, decay=1.0, mix=9),
        # three sequences have outgrown 1024 tokens by a little
        dict(name="evict_few", path="evict", kv="bf16", batch=3, dist="uniform", lo=1040, hi=1300, kv_heads=4, dim=128, budget=1024, sinks=4, recent=128, mix=10),
        # agent trajectories of 2 k to 64 k tokens cut to 4096
        dict(name="evict_agent", path="evict", kv="bf16", batch=32, dist="lognormal", lo=2048, hi=65536, kv_heads=8, dim=128, budget=4096, sinks=16, recent=1000, mix=11),
        # a wide batch over an fp8 cache
        dict(name="evict_fp8_wide", path="evict", kv="fp8", batch=200, dist="uniform", lo=1500, hi=4096, kv_heads=8, dim=128, budget=1500, sinks=4, recent=300, mix=12),
    ]


HEADS = [(28, 4), (32, 8), (64, 8), (40, 8), (32, 4), (16, 2), (8, 2)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Bytes and operations of a pass, and what the cache holds."""
    w = work(case)
    cached = 0 if case["path"] in ("append", "train") else sum(_lengths(case)) * case["kv_heads"] * case["dim"] * (1 if case["kv"] == "fp8" else 2)
    return w["bytes"], w["flops"], cached


def draw(rng):
    top = {}
    for c in listed():
        t = top.setdefault(c["path"], [0, 0, 0])
        t[:] = map(max, t, _cost(c))
    while True:
        path = rng.choice(["append", "train", "weights", "weights", "evict", "evict"])
        heads, kv_heads = rng.choice(HEADS)
        dim = 64 if rng.random() < 0.25 else 128
        c = dict(path=path, heads=heads, kv_heads=kv_heads, dim=dim, mix=rng.randrange(1 << 30))
        if path in ("append", "train"):
            c.update(rotary=rng.choice([dim, dim, dim, dim // 2, 16]), interleaved=rng.random() < 0.3)
            hi = _log(rng, 64, 32768)
            c.update(lo=max(1, int(hi * rng.uniform(0.1, 1))), hi=hi)
            if path == "append":
                c.update(batch=_log(rng, 1, 512), new=1 if rng.random() < 0.4 else _log(rng, 1, 2048))
                c["hi"] = max(hi, c["new"])
            else:
                c.update(tokens=_log(rng, 1, 20000))
        else:
            c["kv"] = rng.choice(["bf16", "bf16", "fp8"])
            hi = _log(rng, 32, 65536)
            c.update(batch=_log(rng, 1, 256), dist="uniform", lo=max(1, int(hi * rng.uniform(0.05, 1))), hi=hi)
            if hi > 8192 and rng.random() < 0.4:
                c.update(dist="lognormal", lo=2048)
            if path == "weights":
                c.update(window=1 if rng.random() < 0.6 else _log(rng, 2, 128), decay=rng.choice([1.0, 1.0, 0.97, 0.5]))
            else:
                del c["heads"]
                budget = _log(rng, 16, max(17, c["hi"]))
                c.update(budget=budget, sinks=rng.choice([0, 1, 4, 16]) if budget >= 16 else 0, recent=rng.randint(0, max(0, budget - 16)))
        if all(x <= y for x, y in zip(_cost(c), top[path])):
            return c


# ---------------------------------------------------------------------------
# what follows from the case alone
# ---------------------------------------------------------------------------
def _lengths(case):
    rng = random.Random(case["mix"])
    lo, hi = case["lo"], case["hi"]
    if case["path"] == "train":
        out = []
        while sum(out) < case["tokens"]:
            out.append(min(rng.randint(lo, hi), case["tokens"] - sum(out)))
        return out
    if case.get("dist") == "lognormal":
        return [min(hi, max(lo, int(round(rng.lognormvariate(math.log(16384), 1.0))))) for _ in range(case["batch"])]
    return [rng.randint(lo, hi) for _ in range(case["batch"])]


def _blocks(tokens):
    return (tokens + PAGE - 1) // PAGE


def work(case):
    """Every input once, every output once."""
    lens, hkv, d = _lengths(case), case["kv_heads"], case["dim"]
    if case["path"] in ("append", "train"):
        t = case["tokens"] if case["path"] == "train" else case["batch"] * case["new"]
        table = 4 * case["rotary"] * min(t, case["hi"])
        q, k = t * case["heads"] * d, t * hkv * d
        if case["path"] == "append":
            return dict(bytes=2 * 2 * (q + 2 * k) + table + 12 * t, flops=10 * (q + k))
        return dict(bytes=4 * 2 * (q + k) + table + 4 * t + 4 * 4 * d, flops=30 * (q + k))
    size = 1 if case["kv"] == "fp8" else 2
    total, B = sum(lens), len(lens)
    pages = sum(_blocks(n) for n in lens)
    if case["path"] == "weights":
        rows = [min(case["window"], n) for n in lens]
        scales = 4 * pages * hkv if size == 1 else 0
        return dict(bytes=total * hkv * (d * size + 8) + scales + 4 * pages + 2 * B * case["window"] * case["heads"] * d,
                    flops=sum(2 * n * r for n, r in zip(lens, rows)) * case["heads"] * d)
    kept = [min(n, case["budget"]) for n in lens]
    new_pages = sum(_blocks(n) for n in kept)
    scales = 8 * hkv * (pages + new_pages) if size == 1 else 0
    return dict(bytes=hkv * (4 * total + sum(kept) * (4 * d * size + 8)) + scales + 4 * (pages + new_pages), flops=hkv * (total + 2 * sum(kept) * d))


# ---------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------
def _normal(shape, gen, gain=1.0):
    """bf16 N(0, gain^2), drawn in pieces."""
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=gen, device="cuda") * gain
    return out


def _pool(case, pages, gen):
    """(pages, scales or None): every (page, head) tile of an fp8 pool has the scale of its largest value."""
    shape = (pages, case["kv_heads"], PAGE, case["dim"])
    if case["kv"] == "bf16":
        return _normal(shape, gen), None
    pool = torch.empty(shape, dtype=torch.uint8, device="cuda")
    scales = torch.empty(shape[:2], device="cuda")
    step = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3]))
    for i in range(0, pages, step):
        x = torch.randn((min(step, pages - i),) + shape[1:], generator=gen, device="cuda")
        s = x.abs().amax(dim=(2, 3)) / FP8_MAX
        pool[i:i + step] = (x / s[..., None, None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        scales[i:i + step] = s
    return pool, scales


def _spread(counts, first, pages, gen):
    """A block table: sequence b's counts[b] logical pages on physical pages first .. of a random order; -1 past them."""
    order = torch.randperm(sum(counts), generator=gen, device="cuda").int() + first
    table = torch.full((len(counts), max(1, max(counts))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rope_table(case, length):
    """[length][rotary]: the cosines, then the sines of every pair's angle."""
    m = case["rotary"]
    freq = THETA ** (-torch.arange(0, m, 2, dtype=torch.float64, device="cuda") / m)
    angle = torch.arange(length, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens, hkv, d = _lengths(case), case["kv_heads"], case["dim"]
    s = dict(case=case, lens=lens)
    if case["path"] in ("append", "train"):
        _prepare_rows(s, case, lens, gen)
    else:
        _prepare_cache(s, case, lens, gen)
    if own:
        import paper_2508_11553_amd as sd

        s["sd"] = sd
        if case["path"] in ("append", "train"):
            s["norm"] = sd.QkNorm(num_q_heads=case["heads"], num_kv_heads=hkv, head_dim=d, rotary_dim=case["rotary"], interleaved=int(case["interleaved"]),
                                  table_len=s["table"].shape[0], weight_dtype=sd.SD_BF16, eps=EPS,
                                  q_stride=s["q"].stride(0), k_stride=s["k"].stride(0), v_stride=s["k"].stride(0))
        if case["path"] == "train":
            s["ws_bytes"] = sd.qk_norm_rope_workspace_bytes(s["norm"], s["T"])
        else:
            s["shape"] = sd.Shape(batch=len(lens), num_q_heads=case.get("heads", hkv), num_kv_heads=hkv, head_dim=d, page_size=PAGE,
                                  num_pages=s["k_pages"].shape[0], max_blocks_per_seq=s["block_table"].shape[1],
                                  kv_dtype=sd.SD_FP8_E4M3 if case.get("kv") == "fp8" else sd.SD_BF16, max_context_len=max(lens), chunk_tokens=0)
        if case["path"] == "weights":
            s["ws_bytes"] = sd.paged_weight_workspace_bytes(s["shape"], case["window"])
        if "ws_bytes" in s:
            s["ws"] = torch.empty(max(s["ws_bytes"], 16), dtype=torch.uint8, device="cuda")
    return s


def _prepare_rows(s, case, lens, gen):
    hq, hkv, d = case["heads"], case["kv_heads"], case["dim"]
    if case["path"] == "append":
        n = case["new"]
        ends = [max(L, n) for L in lens]  # a sequence's true length; its cache holds less where it was cut before
        positions = [p for L in ends for p in range(L - n, L)]
        cached = [max(n, L - 37 * (b % 5)) for b, L in enumerate(ends)]
        s["seq_ids"] = _int([b for b in range(len(lens)) for _ in range(n)])
        s["slots"] = _int([p for L in cached for p in range(L - n, L)])
        # of the pool the pages that the new rows go to: nothing else is touched
        first = [(L - n) // PAGE for L in cached]
        counts = [_blocks(L) - f for L, f in zip(cached, first)]
        part = _spread(counts, 0, sum(counts), gen)
        s["block_table"] = torch.zeros((len(lens), max(_blocks(L) for L in cached)), dtype=torch.int32, device="cuda")
        for b, (f, k) in enumerate(zip(first, counts)):
            s["block_table"][b, f:f + k] = part[b, :k]
        s["k_pages"] = torch.zeros((sum(counts), hkv, PAGE, d), dtype=torch.bfloat16, device="cuda")
        s["v_pages"] = torch.zeros_like(s["k_pages"])
    else:
        positions = [p for n in lens for p in range(n)]
    T = s["T"] = len(positions)
    s["positions"] = _int(positions)
    s["table"] = _rope_table(case, max(case["hi"], max(positions) + 1))
    # the fused projection's rows: queries, keys, values of a token side by side
    qkv = _normal((T, (hq + 2 * hkv) * d), gen, 1.5)
    s["q"], s["k"], s["v"] = qkv[:, :hq * d], qkv[:, hq * d:(hq + hkv) * d], qkv[:, (hq + hkv) * d:]
    s["q_weight"], s["k_weight"] = 1 + _normal((d,), gen, 0.2), 1 + _normal((d,), gen, 0.2)
    s["q_out"] = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
    if case["path"] == "train":
        s["k_out"] = torch.empty((T, hkv, d), dtype=torch.bfloat16, device="cuda")
        s["dq_out"], s["dk_out"] = _normal((T, hq, d), gen, 0.01), _normal((T, hkv, d), gen, 0.01)
        dqkv = torch.empty_like(qkv)  # the gradient of the projection: dq and dk are laid out as q and k
        s["dq"], s["dk"] = dqkv[:, :hq * d], dqkv[:, hq * d:(hq + hkv) * d]
        s["dq_weight"], s["dk_weight"] = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")


def _prepare_cache(s, case, lens, gen):
    hkv, d = case["kv_heads"], case["dim"]
    counts = [_blocks(n) for n in lens]
    pages = sum(counts)
    kept = [_blocks(min(n, case["budget"])) for n in lens] if case["path"] == "evict" else []
    s["old"] = pages
    s["k_pages"], s["k_scales"] = _pool(case, pages + sum(kept), gen)
    s["block_table"] = _spread(counts, 0, pages, gen)
    s["context_lens"] = _int(lens)
    longest = (max(lens) + 3) // 4 * 4
    # weight that tokens have received is heavy-tailed; many have none
    x = torch.randn((len(lens), hkv, longest), generator=gen, device="cuda")
    s["scores"] = torch.where(x < -1, 0.0, torch.exp(2 * x - 3))
    if case["path"] == "weights":
        n = case["window"]
        s["rows"] = [min(n, L) for L in lens]
        s["q_start"] = [0]
        for r in s["rows"]:
            s["q_start"].append(s["q_start"][-1] + r)
        s["starts"] = _int(s["q_start"])
        s["q"] = _normal((s["q_start"][-1], case["heads"], d), gen, 1.5)
        # of a few steps before this one
        s["scores"] *= (case["heads"] // hkv / torch.tensor(lens, dtype=torch.float32, device="cuda"))[:, None, None]
        s["out"] = torch.zeros_like(s["scores"])
        s["scale"] = 1.0 / math.sqrt(d)
    else:
        s["v_pages"], s["v_scales"] = _pool(case, pages + sum(kept), gen)
        s["new_table"] = _spread(kept, pages, pages + sum(kept), gen)
        if s["new_table"].shape[1] < s["block_table"].shape[1]:
            more = s["block_table"].shape[1] - s["new_table"].shape[1]
            s["new_table"] = torch.cat([s["new_table"], torch.full((len(lens), more), -1, dtype=torch.int32, device="cuda")], dim=1)
        for x in (s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"]):
            if x is not None:
                x[pages:] = 0
        s["kept"] = torch.empty((len(lens), hkv, case["budget"]), dtype=torch.int32, device="cuda")
        s["new_lens"] = torch.empty_like(s["context_lens"])
        s["out"] = torch.zeros((len(lens), hkv, (min(case["budget"], max(lens)) + 3) // 4 * 4), device="cuda")


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)[s["case"]["path"]](s)


def _own_append(s):
    sd = s["sd"]
    sd.qk_norm_rope_append(s["shape"], s["norm"], s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["table"], s["positions"], s["seq_ids"], s["slots"],
                           s["T"], s["q_out"], s["k_pages"], s["v_pages"], s["block_table"])
    return dict(q=s["q_out"], k=s["k_pages"], v=s["v_pages"])


def _own_train(s):
    sd = s["sd"]
    sd.qk_norm_rope(s["norm"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["table"], s["positions"], s["T"], s["q_out"], s["k_out"])
    sd.qk_norm_rope_backward(s["norm"], s["dq_out"], s["dk_out"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["table"], s["positions"], s["T"],
                             s["dq"], s["dk"], s["dq_weight"], s["dk_weight"], s["ws"], s["ws_bytes"])
    return dict(q=s["q_out"], k=s["k_out"], dq=s["dq"], dk=s["dk"], dq_weight=s["dq_weight"], dk_weight=s["dk_weight"])


def _own_weights(s):
    sd, c = s["sd"], s["case"]
    sd.paged_weight_accumulate(s["shape"], s["q"], None if c["window"] == 1 else s["starts"], s["q_start"][-1], c["window"], s["k_pages"], s["k_scales"],
                               s["block_table"], s["context_lens"], s["scale"], c["decay"], c["window"], s["scores"], s["out"], s["scores"].shape[2], s["ws"], s["ws_bytes"])
    return s["out"]


def _own_evict(s):
    sd, c = s["sd"], s["case"]
    sd.kv_evict(s["shape"], c["budget"], c["sinks"], c["recent"], s["scores"], s["scores"].shape[2], s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"],
                s["block_table"], s["context_lens"], s["new_table"], s["kept"], s["new_lens"], s["out"], s["out"].shape[2])
    return _evicted(s)


def _evicted(s):
    got = dict(kept=s["kept"], lens=s["new_lens"], scores=s["out"])
    for name in ("k", "v"):
        pool = s[name + "_pages"][s["old"]:]
        got[name] = pool if s["k_scales"] is None else pool.view(torch.float8_e4m3fn)  # times its scale
        if s["k_scales"] is not None:
            got[name + "_scale"] = s[name + "_scales"][s["old"]:]
    return got


_own = dict(append=_own_append, train=_own_train, weights=_own_weights, evict=_own_evict)


# ---------------------------------------------------------------------------
# the same in elementary operations, 32 bits
# ---------------------------------------------------------------------------
def _angles(s, x):
    """Cosines and sines of the rows' positions, [T][1][rotary / 2]."""
    m = s["case"]["rotary"]
    row = s["table"][s["positions"].long()][:, None]
    return row[..., :m // 2], row[..., m // 2:]


def _rotate(x, cos, sin, interleaved):
    m = 2 * cos.shape[-1]
    a, b = (x[..., 0:m:2], x[..., 1:m:2]) if interleaved else (x[..., :m // 2], x[..., m // 2:m])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=-1).flatten(-2) if interleaved else torch.cat([a, b], dim=-1)
    return torch.cat([turned, x[..., m:]], dim=-1)


def _plain_norm(s, x, w, heads):
    x = x.reshape(s["T"], heads, -1).float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    cos, sin = _angles(s, x)
    return _rotate(x * r * w.float(), cos, sin, s["case"]["interleaved"]).bfloat16()


def _plain_append(s):
    c = s["case"]
    s["q_out"] = _plain_norm(s, s["q"], s["q_weight"], c["heads"])
    k = _plain_norm(s, s["k"], s["k_weight"], c["kv_heads"])
    slots = s["slots"].long()
    page = s["block_table"][s["seq_ids"].long(), slots // PAGE].long()
    s["k_pages"][page, :, slots % PAGE] = k
    s["v_pages"][page, :, slots % PAGE] = s["v"].reshape(s["T"], c["kv_heads"], -1)
    return dict(q=s["q_out"], k=s["k_pages"], v=s["v_pages"])


def _plain_gradient(s, dy, x, w, heads, dx_out):
    x = x.reshape(s["T"], heads, -1).float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    cos, sin = _angles(s, x)
    dz = _rotate(dy.float(), cos, -sin, s["case"]["interleaved"])
    g = dz * w.float()
    dx = r * (g - x * (r * r) * (g * x).mean(dim=-1, keepdim=True))
    dx_out.copy_(dx.reshape(s["T"], -1))
    return (dz * x * r).sum(dim=(0, 1))


def _plain_train(s):
    c = s["case"]
    q, k = _plain_norm(s, s["q"], s["q_weight"], c["heads"]), _plain_norm(s, s["k"], s["k_weight"], c["kv_heads"])
    dqw = _plain_gradient(s, s["dq_out"], s["q"], s["q_weight"], c["heads"], s["dq"])
    dkw = _plain_gradient(s, s["dk_out"], s["k"], s["k_weight"], c["kv_heads"], s["dk"])
    return dict(q=q, k=k, dq=s["dq"], dk=s["dk"], dq_weight=dqw, dk_weight=dkw)


def _plain_weights(s):
    c = s["case"]
    hkv, d = c["kv_heads"], c["dim"]
    for b, (L, n) in enumerate(zip(s["lens"], s["rows"])):
        pages = s["block_table"][b, :_blocks(L)].long()
        k = s["k_pages"][pages]
        k = k.float() if s["k_scales"] is None else k.view(torch.float8_e4m3fn).float() * s["k_scales"][pages][..., None, None]
        k = k.transpose(0, 1).reshape(hkv, -1, d)[:, :L]
        q = s["q"][s["q_start"][b]:s["q_start"][b + 1]].float().view(n, hkv, -1, d).transpose(0, 1).reshape(hkv, -1, d)  # [Hkv][n G][d]
        x = torch.matmul(q, k.transpose(1, 2).contiguous()).view(hkv, n, -1, L) * s["scale"]
        if n > 1:
            at = torch.arange(L, device="cuda")
            x = x.masked_fill((at > at[L - n:, None])[None, :, None], -math.inf)
        p = torch.exp(x - x.amax(dim=-1, keepdim=True))
        p = (p / p.sum(dim=-1, keepdim=True)).sum(dim=(1, 2))
        before = s["scores"][b, :, :L] * c["decay"]
        before[:, L - n:] = 0  # the rows' own tokens have received nothing yet
        s["out"][b, :, :L] = before + p
    return s["out"]


def _plain_select(s, scores):
    """Kept positions of one sequence and head set, ascending: [Hkv][n]."""
    c = s["case"]
    L = scores.shape[1]
    if L <= c["budget"]:
        return torch.arange(L, device="cuda").expand(scores.shape[0], L)
    middle = scores[:, c["sinks"]:L - c["recent"]]
    best = torch.sort(middle, dim=1, descending=True, stable=True).indices[:, :c["budget"] - c["sinks"] - c["recent"]] + c["sinks"]
    rest = torch.cat([torch.arange(c["sinks"], device="cuda"), torch.arange(L - c["recent"], L, device="cuda")]).expand(scores.shape[0], -1)
    return torch.sort(torch.cat([best, rest], dim=1), dim=1).values


def _plain_evict(s):
    c = s["case"]
    heads = torch.arange(c["kv_heads"], device="cuda")[:, None]
    s["kept"].fill_(-1)
    for b, L in enumerate(s["lens"]):
        scores = s["scores"][b, :, :L]
        kept = _plain_select(s, scores)
        n = kept.shape[1]
        s["kept"][b, :, :n] = kept
        s["new_lens"][b] = n
        s["out"][b, :, :n] = scores.gather(1, kept)
        page = s["block_table"][b].long()[kept // PAGE]
        at = torch.arange(n, device="cuda")
        new_page = s["new_table"][b].long()[at // PAGE]
        for pool, scales in ((s["k_pages"], s["k_scales"]), (s["v_pages"], s["v_scales"])):
            rows = pool[page, heads, kept % PAGE]  # [Hkv][n][d]
            if scales is not None:  # a new tile's scale is the largest of its rows' old ones
                old = scales[page, heads]
                blocks = _blocks(n)
                padded = torch.zeros((c["kv_heads"], blocks * PAGE), device="cuda")
                padded[:, :n] = old
                new = padded.view(c["kv_heads"], blocks, PAGE).amax(dim=2)
                scales[s["new_table"][b, :blocks].long()[None, :], heads] = new
                ratio = old / new[:, at // PAGE]
                rows = (rows.view(torch.float8_e4m3fn).float() * ratio[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            pool[new_page[None, :], heads, (at % PAGE)[None, :]] = rows
    return _evicted(s)


_plain = dict(append=_plain_append, train=_plain_train, weights=_plain_weights, evict=_plain_evict)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return dict(append=_exact_append, train=_exact_train, weights=_exact_weights, evict=_exact_evict)[case["path"]](s, case)


def _turn(case, s):
    """[T][d][d]-free rotation: complex numbers of the pairs times e^(i angle); -> a function of rows and a sign."""
    m = case["rotary"]
    table = s["table"].double()[s["positions"].long()]
    unit = torch.complex(table[:, :m // 2], table[:, m // 2:])[:, None]

    def turn(x, back):
        pair = x[..., :m].reshape(*x.shape[:-1], m // 2, 2) if case["interleaved"] else torch.stack([x[..., :m // 2], x[..., m // 2:m]], dim=-1)
        z = torch.view_as_complex(pair.contiguous()) * (unit.conj() if back else unit)
        z = torch.view_as_real(z)
        y = x.clone()
        y[..., :m] = z.reshape(*x.shape[:-1], m) if case["interleaved"] else torch.cat([z[..., 0], z[..., 1]], dim=-1)
        return y

    return turn


def _rows64(s, x, heads):
    return x.reshape(s["T"], heads, -1).double()


def _exact_append(s, case):
    turn = _turn(case, s)
    got = {}
    for name, heads in (("q", case["heads"]), ("k", case["kv_heads"])):
        x = _rows64(s, s[name], heads)
        got[name] = turn(x / (x.square().sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * s[name + "_weight"].double(), False)
    slots = s["slots"].tolist()
    sequence = s["seq_ids"].tolist()
    table = s["block_table"].tolist()
    at = torch.tensor([table[b][p // PAGE] * PAGE + p % PAGE for b, p in zip(sequence, slots)], device="cuda")
    pages = {}
    for name, rows in (("k", got["k"]), ("v", _rows64(s, s["v"], case["kv_heads"]))):
        flat = s["k_pages"].double().zero_().transpose(1, 2).reshape(-1, case["kv_heads"], case["dim"])
        flat[at] = rows
        pages[name] = flat.view(-1, PAGE, case["kv_heads"], case["dim"]).transpose(1, 2)
    return dict(q=got["q"], **pages)


def _exact_train(s, case):
    turn = _turn(case, s)
    got = {}
    for name, heads in (("q", case["heads"]), ("k", case["kv_heads"])):
        # in pieces of tokens: the gradient by autograd of the definition
        w = s[name + "_weight"].double().requires_grad_()
        x = _rows64(s, s[name], heads).requires_grad_()
        y = turn(x / (x.square().sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * w, False)
        dx, dw = torch.autograd.grad(y, (x, w), s["d%s_out" % name].double())
        got.update({name: y.detach(), "d" + name: dx.reshape(s["T"], -1), "d%s_weight" % name: dw})
    return got


def _exact_weights(s, case):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    group = case["heads"] // case["kv_heads"]
    for b, L in enumerate(s["lens"]):
        n = s["rows"][b]
        where = s["block_table"][b, :_blocks(L)].long()
        new = torch.ones(L, dtype=torch.float64, device="cuda")
        new[L - n:] = 0
        hidden = torch.ones((n, L), dtype=torch.bool, device="cuda").triu(L - n + 1).repeat_interleave(group, dim=0)
        for g in range(case["kv_heads"]):
            tile = s["k_pages"][where, g]
            k = tile.double() if case["kv"] == "bf16" else tile.view(torch.float8_e4m3fn).double() * s["k_scales"][where, g].double()[:, None, None]
            q = s["q"][s["q_start"][b]:s["q_start"][b + 1], g * group:(g + 1) * group].double().reshape(-1, case["dim"])
            x = (q @ k.reshape(-1, case["dim"])[:L].T.contiguous()) * s["scale"]
            x[hidden] = -math.inf
            out[b, g, :L] = torch.exp(x - torch.logsumexp(x, dim=1, keepdim=True)).sum(dim=0) + case["decay"] * s["scores"][b, g, :L].double() * new
    return out


def _exact_evict(s, case):
    got = dict(kept=None, lens=None, scores=torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"))
    fp8 = case["kv"] == "fp8"
    for name in ("k", "v"):
        got[name] = torch.zeros((s["k_pages"].shape[0] - s["old"],) + s["k_pages"].shape[1:], dtype=torch.float64, device="cuda")
        if fp8:
            got[name + "_scale"] = torch.zeros(got[name].shape[:2], dtype=torch.float64, device="cuda")
    for b, L in enumerate(s["lens"]):
        x = s["scores"][b, :, :L].double()
        n = min(L, case["budget"])
        rank = x.clone()
        rank[:, :case["sinks"]] = math.inf
        rank[:, L - case["recent"]:] = math.inf
        # by score, then by position: the position as a second key that no score reaches
        order = torch.argsort(-rank, dim=1, stable=True)[:, :n].sort(dim=1).values if n < L else torch.arange(L, device="cuda").expand(x.shape[0], L)
        to = s["new_table"][b, :_blocks(n)].long() - s["old"]
        for g in range(case["kv_heads"]):
            kept = order[g]
            got["scores"][b, g, :n] = x[g, kept]
            page = s["block_table"][b, kept // PAGE].long()
            for name in ("k", "v"):
                tile = torch.zeros((len(to) * PAGE, case["dim"]), dtype=torch.float64, device="cuda")
                if not fp8:
                    tile[:n] = s[name + "_pages"][page, g, kept % PAGE].double()
                else:
                    scale = torch.zeros(len(to) * PAGE, dtype=torch.float64, device="cuda")
                    scale[:n] = s[name + "_scales"][page, g].double()
                    top = scale.view(-1, PAGE).amax(dim=1)
                    got[name + "_scale"][to, g] = top
                    tile[:n] = s[name + "_pages"][page, g, kept % PAGE].view(torch.float8_e4m3fn).double() * (scale / top.repeat_interleave(PAGE))[:n, None]
                got[name][to, g] = tile.view(-1, PAGE, case["dim"])
    return got
