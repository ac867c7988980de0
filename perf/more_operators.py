"""Performance cases of what closes the loop of a rollout: from a step's logits to the next step's tables, and the log
probabilities of what was drawn with their gradient.

A case is one pass of one of these (`path`):
  sample    a token for every row of logits, drawn with the row's temperature, top-k, top-p and min-p from a given
            uniform number, and its log probabilities
  logprob   the log probabilities of given tokens, with the entropy of every row; with `train` the gradient of the logits too
  plan      places for the new tokens of every sequence, made on the device: pages off the free list (finished sequences
            give theirs back), block table, lengths, and the slot map of the rows

Lengths, counts and sizes follow from the case alone (`mix` seeds them); values and placement come from the seed.  With
`own` the framework's entry points run; without it the same in elementary torch operations.

A drawn token: with z = logit / temperature, largest first and of equal ones the lower index first, a row keeps its first top_k,
of those the shortest beginning that holds top_p of their probability, and of those the ones with at least min_p of the
largest's; in the order of their indices it takes the first whose probability, with all before it, exceeds uniform times
that of all that are kept.  Temperature 0 takes the largest logit.
"""
import math
import random

import torch

own = False

PAGE = 16


def listed():
    return [
        # a single sequence, plain sampling: nothing but latency
        dict(name="sample_one", path="sample", rows=1, vocab=32000, dtype="f32", logits="peaked", limits="none", masked=0.0, mix=1),
        # a decode step of 64 sequences with the usual limits
        dict(name="sample_step", path="sample", rows=64, vocab=131072, dtype="bf16", logits="peaked", limits="top", masked=0.0, mix=2),
        # a wide rollout for training: the whole distribution at one temperature, a vocabulary of odd size
        dict(name="sample_rollout", path="sample", rows=512, vocab=160001, dtype="bf16", logits="peaked", limits="none", masked=0.0, mix=3),
        # a model at the start of its training: top-p keeps tens of thousands of tokens
        dict(name="sample_flat", path="sample", rows=48, vocab=49999, dtype="f32", logits="flat", limits="top_p", masked=0.0, mix=4),
        # requests of many users in one batch, each with limits of its own, some greedy, a grammar hides most tokens
        dict(name="sample_mixed", path="sample", rows=200, vocab=100003, dtype="f32", logits="peaked", limits="mixed", masked=0.7, mix=5),
        # the few tokens of a short answer, trained on
        dict(name="logprob_few", path="logprob", rows=17, vocab=32000, dtype="f32", logits="peaked", train=True, pad=0.0, mix=6),
        # trajectories scored by the policy that is to be kept near: no gradient
        dict(name="logprob_score", path="logprob", rows=8192, vocab=65536, dtype="bf16", logits="peaked", train=False, pad=0.02, mix=7),
        # a micro-batch of a training step
        dict(name="logprob_train", path="logprob", rows=4096, vocab=131072, dtype="bf16", logits="peaked", train=True, pad=0.02, mix=8),
        # a small one in fp32, odd vocabulary, a batch padded to a fixed size
        dict(name="logprob_padded", path="logprob", rows=1531, vocab=49999, dtype="f32", logits="flat", train=True, pad=0.3, mix=9),
        # a decode step of 64 sequences: one new token each
        dict(name="plan_step", path="plan", batch=64, lo=1024, hi=8192, new_lo=1, new_hi=1, done=0.0, idle=0.0, shared=0.0, room=1.0, mix=10),
        # a wide step: some sequences finish and give their pages back, some wait, the pool runs short
        dict(name="plan_wide", path="plan", batch=2048, lo=1, hi=4096, new_lo=1, new_hi=1, done=0.05, idle=0.1, shared=0.5, room=0.3, mix=11),
        # paused sequences resume: up to 8 k stored tokens each go back into the cache
        dict(name="plan_resume", path="plan", batch=200, lo=0, hi=2048, new_lo=100, new_hi=8192, done=0.1, idle=0.2, shared=0.3, room=1.0, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = {}
    for c in listed():
        key = c["path"], c.get("train")
        w = work(c)
        top[key] = [max(a, b) for a, b in zip(top.get(key, [0, 0]), (w["bytes"], w["flops"]))]
    while True:
        path = rng.choice(["sample", "sample", "sample", "logprob", "logprob", "plan", "plan"])
        c = dict(path=path, mix=rng.randrange(1 << 30))
        if path == "plan":
            c.update(batch=_log(rng, 1, 4096), lo=0, hi=_log(rng, 16, 32768), new_lo=1, new_hi=1 if rng.random() < 0.5 else _log(rng, 2, 8192),
                     done=rng.choice([0.0, 0.05, 0.3]), idle=rng.choice([0.0, 0.1, 0.5]), shared=rng.choice([0.0, 0.5]), room=rng.choice([0.3, 1.0, 1.0]))
            c["lo"] = int(c["hi"] * rng.uniform(0, 1))
            if c["batch"] * c["hi"] > 64 * 131072:  # of the cache: 8 M tokens
                continue
        else:
            c.update(vocab=_log(rng, 200, 200000), dtype=rng.choice(["bf16", "bf16", "f32"]), logits="flat" if rng.random() < 0.25 else "peaked")
            if path == "sample":
                c.update(rows=_log(rng, 1, 1024), limits=rng.choice(["none", "top", "top_p", "mixed"]), masked=0.9 if rng.random() < 0.2 else 0.0)
            else:
                c.update(rows=_log(rng, 1, 8192), train=rng.random() < 0.6, pad=rng.choice([0.0, 0.02, 0.3]))
        w = work(c)
        if all(x <= y for x, y in zip((w["bytes"], w["flops"]), top[path, c.get("train")])):
            return c


# ---------------------------------------------------------------------------
# what follows from the case alone
# ---------------------------------------------------------------------------
def _real(case):
    """Rows of a logprob case that have a token."""
    return case["rows"] - int(case["rows"] * case["pad"])


def _blocks(tokens):
    return (tokens + PAGE - 1) // PAGE


def _step(case):
    """Per sequence (tokens in the cache, new ones: -1 where it is finished, tokens of a shared prefix, tokens cut from the cache before)."""
    rng = random.Random(case["mix"])
    out = []
    for _ in range(case["batch"]):
        n, x = rng.randint(case["lo"], case["hi"]), rng.random()
        new = -1 if x < case["done"] else 0 if x < case["done"] + case["idle"] else rng.randint(case["new_lo"], case["new_hi"])
        shared = rng.randint(0, n) // PAGE * PAGE if rng.random() < case["shared"] else 0
        out.append((n, new, shared, rng.choice([0, 0, 0, 977])))
    return out


def _free(case, step):
    """Pages that are free before the step."""
    need = sum(_blocks(n + new) - _blocks(n) for n, new, _, _ in step if new > 0)
    return max(1, int(need * case["room"])) + (5 if case["room"] >= 1 else 0)


def _max_rows(step):
    """A call of fixed size: the rows of all, rounded up."""
    return max(64, (sum(new for _, new, _, _ in step if new > 0) + 63) // 64 * 64)


def work(case):
    """Every input once, every output once."""
    if case["path"] == "plan":
        step = _step(case)
        pages = sum(_blocks(n + new) - _blocks(n) for n, new, _, _ in step if new > 0)
        back = sum(_blocks(n) - s // PAGE for n, new, s, _ in step if new < 0)
        return dict(bytes=4 * (9 * len(step) + 3 * _max_rows(step) + 2 * pages + 2 * back), flops=8 * len(step))
    size = 2 if case["dtype"] == "bf16" else 4
    if case["path"] == "sample":
        n = case["rows"] * case["vocab"]
        return dict(bytes=n * size + 16 * case["rows"], flops=4 * n)
    n = _real(case) * case["vocab"]
    whole = case["rows"] * case["vocab"]
    if not case["train"]:
        return dict(bytes=n * size + 24 * case["rows"], flops=6 * n)
    return dict(bytes=2 * n * size + whole * size + 40 * case["rows"], flops=13 * n)


# ---------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------
def _rand(gen, *shape):
    return torch.rand(shape, generator=gen, device="cuda")


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _logits(case, gen):
    """Peaked: a bulk of unlikely tokens, and some 60 per row of which the k-th lies about 1.3 log(k) below the first; flat: nearly alike."""
    rows, vocab = case["rows"], case["vocab"]
    out = torch.empty((rows, vocab), dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.float32, device="cuda")
    piece = max(1, (1 << 27) // vocab)
    for i in range(0, rows, piece):
        n = min(piece, rows - i)
        x = torch.randn((n, vocab), generator=gen, device="cuda") * (2.0 if case["logits"] == "peaked" else 0.7)
        if case["logits"] == "peaked":
            head = min(64, vocab // 2)
            where = torch.randint(0, vocab, (n, head), generator=gen, device="cuda")
            level = 11 + 4 * _rand(gen, n, 1) - 1.3 * torch.log(torch.arange(1, head + 1, device="cuda")) * (0.5 + 2 * _rand(gen, n, 1))
            x.scatter_reduce_(1, where, level + 0.3 * torch.randn((n, head), generator=gen, device="cuda"), "amax", include_self=False)
        if case.get("masked"):
            x.masked_fill_(_rand(gen, n, vocab) < case["masked"], -math.inf)
            x[:, vocab // 3] = 1.0  # something is always allowed
        out[i:i + n] = x
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=case)
    dict(sample=_prepare_sample, logprob=_prepare_logprob, plan=_prepare_plan)[case["path"]](s, case, gen)
    if own:
        import paper_2508_11553_amd as sd

        s["sd"] = sd
        if case["path"] == "plan":
            s["shape"] = sd.Shape(batch=case["batch"], num_q_heads=8, num_kv_heads=8, head_dim=128, page_size=PAGE, num_pages=s["free_pages"].shape[0],
                                  max_blocks_per_seq=s["block_table"].shape[1], kv_dtype=sd.SD_BF16, max_context_len=PAGE * s["block_table"].shape[1], chunk_tokens=0)
            s["ws_bytes"] = sd.kv_plan_workspace_bytes(s["shape"])
        else:
            s["desc"] = sd.Logits(rows=case["rows"], vocab=case["vocab"], dtype=sd.SD_BF16 if case["dtype"] == "bf16" else sd.SD_F32, stride=s["logits"].stride(0))
            s["ws_bytes"] = (sd.sample_workspace_bytes if case["path"] == "sample" else sd.token_logprobs_workspace_bytes)(s["desc"])
        s["ws"] = torch.empty(max(s["ws_bytes"], 16), dtype=torch.uint8, device="cuda")
    return s


def _prepare_sample(s, case, gen):
    rows = case["rows"]
    s["logits"] = _logits(case, gen)
    s["uniform"] = _rand(gen, rows)
    s["temperature"] = 0.6 + 0.6 * _rand(gen, rows)
    s["top_k"] = s["top_p"] = s["min_p"] = None
    pick = _rand(gen, rows)
    if case["limits"] in ("top", "mixed"):
        s["top_k"] = torch.randint(10, 101, (rows,), generator=gen, device="cuda").int()
    if case["limits"] in ("top", "top_p", "mixed"):
        s["top_p"] = 0.8 + 0.19 * _rand(gen, rows)
    if case["limits"] == "mixed":
        s["min_p"] = 0.1 * _rand(gen, rows)
        s["temperature"][pick < 0.15] = 0.0
        s["top_k"][pick > 0.3] = 0  # no limit
        s["top_p"][pick > 0.7] = 1.0
        s["min_p"][(pick > 0.5) & (pick < 0.9)] = 0.0
    s["tokens"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    s["logprobs"], s["draw_logprobs"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")


def _prepare_logprob(s, case, gen):
    rows, vocab = case["rows"], case["vocab"]
    s["logits"] = _logits(case, gen)
    best = s["logits"].argmax(dim=1)
    targets = torch.where(_rand(gen, rows) < 0.7, best, torch.randint(0, vocab, (rows,), generator=gen, device="cuda")).int()
    targets[_real(case):] = -1  # padding
    s["targets"] = targets
    s["temperature"] = torch.full((rows,), 0.8, device="cuda")
    s["logprobs"], s["entropy"], s["stats"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda")
    if case["train"]:
        s["d_logprobs"] = torch.randn(rows, generator=gen, device="cuda") / rows
        s["d_entropy"] = torch.full((rows,), -0.01 / rows, device="cuda")
        s["d_logits"] = torch.empty_like(s["logits"])


def _prepare_plan(s, case, gen):
    step = _step(case)
    B = len(step)
    counts = [_blocks(n) for n, _, _, _ in step]
    free = _free(case, step)
    pages = sum(counts) + free
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    blocks = max(1, max(_blocks(n + max(new, 0)) for n, new, _, _ in step))
    at = torch.arange(blocks, device="cuda")
    used = _int(counts)
    first = torch.cumsum(used, 0) - used
    s["block_table"] = torch.where(at < used[:, None], order[(first[:, None] + at).clamp(max=pages - 1)], -1).contiguous()
    s["free_pages"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    s["free_pages"][:free] = order[pages - free:]
    s["free_in"], s["free_out"] = _int([free]), _int([0])
    s["new_tokens"], s["shared"] = _int([new for _, new, _, _ in step]), _int([x for _, _, x, _ in step])
    s["lens_in"], s["next_in"] = _int([n for n, _, _, _ in step]), _int([n + cut for n, _, _, cut in step])
    s["max_rows"] = _max_rows(step)
    for name in ("lens_out", "next_out", "granted", "starts"):
        s[name] = torch.empty(B, dtype=torch.int32, device="cuda")
    s["row_start"] = torch.empty(B + 1, dtype=torch.int32, device="cuda")
    for name in ("seq_ids", "slots", "positions"):
        s[name] = torch.empty(s["max_rows"], dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
PLANNED = ("granted", "row_start", "starts", "lens_out", "next_out", "free_out", "seq_ids", "slots", "positions", "block_table", "free_pages")


def run(s):
    return (_own if own else _plain)[s["case"]["path"]](s)


def _own_sample(s):
    s["sd"].sample_tokens(s["desc"], s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["uniform"], s["tokens"], s["logprobs"], s["draw_logprobs"],
                          s["ws"], s["ws_bytes"])
    return dict(tokens=s["tokens"], logprobs=s["logprobs"], draw_logprobs=s["draw_logprobs"])


def _own_logprob(s):
    sd = s["sd"]
    sd.token_logprobs(s["desc"], s["logits"], s["targets"], s["temperature"], s["logprobs"], s["entropy"], s["stats"], s["ws"], s["ws_bytes"])
    got = dict(logprobs=s["logprobs"], entropy=s["entropy"])
    if s["case"]["train"]:
        sd.token_logprobs_backward(s["desc"], s["logits"], s["targets"], s["temperature"], s["stats"], s["entropy"], s["d_logprobs"], s["d_entropy"], s["d_logits"])
        got["d_logits"] = s["d_logits"]
    return got


def _own_plan(s):
    s["sd"].kv_plan_step(s["shape"], s["new_tokens"], s["shared"], s["lens_in"], s["lens_out"], s["next_in"], s["next_out"], s["free_pages"], s["free_in"], s["free_out"],
                         s["block_table"], s["max_rows"], s["granted"], s["row_start"], s["starts"], s["seq_ids"], s["slots"], s["positions"], s["ws"], s["ws_bytes"])
    return {name: s[name] for name in PLANNED}


_own = dict(sample=_own_sample, logprob=_own_logprob, plan=_own_plan)


# ---------------------------------------------------------------------------
# the same in elementary operations: 32 bits, the sums next to a border in 64
# ---------------------------------------------------------------------------
def _plain_sample(s):
    """In 64 bits: a draw ends next to borders between tokens."""
    vocab = s["case"]["vocab"]
    for i in range(0, s["case"]["rows"], 64):  # in pieces: they are large
        rows = slice(i, i + 64)
        order = torch.sort(s["logits"][rows].float(), dim=1, descending=True, stable=True)
        x = order.values.double()
        temperature = s["temperature"][rows].double()[:, None]
        greedy = temperature <= 0
        z = (x - x[:, :1]) / torch.where(greedy, 1.0, temperature)
        w = torch.exp(z)
        total = w.sum(dim=1, keepdim=True)
        rank = torch.arange(vocab, device="cuda")
        keep = torch.ones_like(w, dtype=torch.bool)
        if s["top_k"] is not None:
            k = s["top_k"][rows][:, None]
            keep &= (rank < k) | (k <= 0)
        if s["top_p"] is not None:
            p = s["top_p"][rows].double()[:, None]
            held = torch.where(keep, w, 0.0)
            keep &= (torch.cumsum(held, 1) - held < p * held.sum(dim=1, keepdim=True)) | (p >= 1)
        if s["min_p"] is not None:
            keep &= w >= s["min_p"][rows].double()[:, None]
        keep &= (rank == 0) | ~greedy
        held = torch.zeros_like(w).scatter_(1, order.indices, torch.where(keep, w, 0.0))  # in the order of the indices
        upto = torch.cumsum(held, 1)
        aim = s["uniform"][rows].double()[:, None] * upto[:, -1:]
        token = (upto <= aim).sum(dim=1, keepdim=True).clamp(max=vocab - 1)
        z = (s["logits"][rows].gather(1, token).double() - x[:, :1]) / torch.where(greedy, 1.0, temperature)
        s["tokens"][rows] = token[:, 0].int()
        s["logprobs"][rows] = (z - torch.log(total))[:, 0].float()
        s["draw_logprobs"][rows] = (z - torch.log(upto[:, -1:]))[:, 0].float()
    return dict(tokens=s["tokens"], logprobs=s["logprobs"], draw_logprobs=s["draw_logprobs"])


def _plain_logprob(s):
    c = s["case"]
    got = dict(logprobs=s["logprobs"], entropy=s["entropy"])
    piece = max(1, (1 << 28) // c["vocab"])
    for i in range(0, c["rows"], piece):
        rows = slice(i, i + piece)
        target = s["targets"][rows].long()[:, None]
        real = target >= 0
        target = target.clamp(min=0)
        temperature = s["temperature"][rows][:, None]
        z = s["logits"][rows].float() / temperature
        z = z - z.amax(dim=1, keepdim=True)
        logp = z - torch.log(torch.exp(z).sum(dim=1, keepdim=True))
        p = torch.exp(logp)
        entropy = -(p * logp).sum(dim=1, keepdim=True)
        s["logprobs"][rows] = torch.where(real, logp.gather(1, target), 0.0)[:, 0]
        s["entropy"][rows] = torch.where(real, entropy, 0.0)[:, 0]
        if c["train"]:
            g, h = s["d_logprobs"][rows][:, None], s["d_entropy"][rows][:, None]
            d = -p * (g + h * (logp + entropy))
            d.scatter_add_(1, target, g)
            s["d_logits"][rows] = torch.where(real, d / temperature, 0.0)
            got["d_logits"] = s["d_logits"]
    return got


def _plain_plan(s):
    lens, new, shared = s["lens_in"].long(), s["new_tokens"].long(), s["shared"].long()
    B, blocks = s["block_table"].shape
    pages = (lens + PAGE - 1) // PAGE
    # the free list with the finished sequences' pages on top
    at = torch.arange(blocks, device="cuda")
    back = (new < 0)[:, None] & (at >= (shared // PAGE)[:, None]) & (at < pages[:, None])
    held = s["free_in"].long()
    list_at = torch.where(back, held + torch.cumsum(back.flatten(), 0).view(B, blocks) - 1, s["free_pages"].shape[0])
    listed_pages = torch.cat([s["free_pages"], s["free_pages"].new_zeros(1)]).scatter(0, list_at.flatten(), s["block_table"].flatten())
    listed_pages = torch.where(torch.arange(listed_pages.shape[0], device="cuda") < held + back.sum(), listed_pages, -1)
    available = held + back.sum()
    # who gets what
    wants = torch.where((new > 0) & (lens + new <= PAGE * blocks), new, 0)
    need = torch.where(wants > 0, (lens + wants + PAGE - 1) // PAGE - pages, 0)
    ok = ((need == 0) | (torch.cumsum(need, 0) <= available)) & (torch.cumsum(wants, 0) <= s["max_rows"])
    granted, need = torch.where(ok, wants, 0), torch.where(ok, need, 0)
    ends, page_ends = torch.cumsum(granted, 0), torch.cumsum(need, 0)
    s["granted"].copy_(granted)
    s["row_start"][0] = 0
    s["row_start"][1:] = ends
    s["starts"].copy_(lens)
    s["lens_out"].copy_(torch.where(new < 0, 0, lens + granted))
    s["next_out"].copy_(torch.where(new < 0, 0, s["next_in"] + granted))
    left = available - page_ends[-1:]
    s["free_out"].copy_(left)
    # new pages from the top of the list down
    mine = (at >= pages[:, None]) & (at < (pages + need)[:, None])
    nth = (page_ends - need - pages)[:, None] + at
    s["block_table"].copy_(torch.where(mine, listed_pages[(available - 1 - nth).clamp(0, listed_pages.shape[0] - 1)], s["block_table"]))
    index = torch.arange(s["free_pages"].shape[0], device="cuda")
    s["free_pages"].copy_(torch.where((index >= held) & (index < left), listed_pages[:-1], s["free_pages"]))
    # the rows
    row = torch.arange(s["max_rows"], device="cuda")
    seq = torch.searchsorted(ends, row, right=True)
    some = seq < B
    seq = seq.clamp(max=B - 1)
    nth = row - (ends - granted)[seq]
    s["seq_ids"].copy_(torch.where(some, seq, -1))
    s["slots"].copy_(torch.where(some, lens[seq] + nth, 0))
    s["positions"].copy_(torch.where(some, s["next_in"][seq] + nth, 0))
    return {name: s[name] for name in PLANNED}


_plain = dict(sample=_plain_sample, logprob=_plain_logprob, plan=_plain_plan)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return dict(sample=_exact_sample, logprob=_exact_logprob, plan=_exact_plan)[case["path"]](s, case)


def _exact_sample(s, case):
    """Row by row, over the probabilities; the tokens that stay are counted, not marked."""
    tokens, logprobs, drawn = [], [], []
    value = lambda name, r, default: default if s[name] is None else s[name][r].item()  # noqa: E731
    for r in range(case["rows"]):
        x = s["logits"][r].double()
        temperature = value("temperature", r, 1.0)
        logp = torch.log_softmax(x / temperature if temperature > 0 else x, dim=0)
        if temperature <= 0:
            token = int((x == x.max()).nonzero()[0])
            tokens.append(token)
            logprobs.append(logp[token])
            drawn.append(torch.zeros_like(logp[token]))
            continue
        best = torch.argsort(-x, stable=True)
        p = logp[best].exp()
        k = value("top_k", r, 0)
        n = min(k, case["vocab"]) if k > 0 else case["vocab"]
        share = value("top_p", r, 1.0)
        if share < 1:
            n = min(n, 1 + int((p[:n].cumsum(0) < share * p[:n].sum()).sum()))
        n = min(n, int((p >= value("min_p", r, 0.0) * p[0]).sum()))
        kept = best[:n].sort().values
        upto = logp[kept].exp().cumsum(0)
        token = kept[min(int((upto <= s["uniform"][r].double() * upto[-1]).sum()), n - 1)]
        tokens.append(int(token))
        logprobs.append(logp[token])
        drawn.append(logp[token] - upto[-1].log())
    return dict(tokens=_int(tokens), logprobs=torch.stack(logprobs), draw_logprobs=torch.stack(drawn))


def _exact_logprob(s, case):
    """The gradient by autograd of the definition, some rows at a time."""
    rows, vocab, real = case["rows"], case["vocab"], _real(case)
    got = dict(logprobs=torch.zeros(rows, dtype=torch.float64, device="cuda"), entropy=torch.zeros(rows, dtype=torch.float64, device="cuda"))
    if case["train"]:
        got["d_logits"] = torch.zeros((rows, vocab), dtype=torch.float64, device="cuda")
    piece = max(1, (1 << 26) // vocab)
    for i in range(0, real, piece):
        at = slice(i, min(i + piece, real))
        x = s["logits"][at].double().requires_grad_(case["train"])
        logp = torch.log_softmax(x / s["temperature"][at].double()[:, None], dim=1)
        chosen = logp[torch.arange(logp.shape[0], device="cuda"), s["targets"][at].long()]
        entropy = -(logp.exp() * logp).sum(dim=1)
        got["logprobs"][at], got["entropy"][at] = chosen.detach(), entropy.detach()
        if case["train"]:
            loss = (chosen * s["d_logprobs"][at].double()).sum() + (entropy * s["d_entropy"][at].double()).sum()
            got["d_logits"][at] = torch.autograd.grad(loss, x)[0]
    return got


def _exact_plan(s, case):
    """One sequence after the other, with a list of pages."""
    table, step, limit = s["block_table"].tolist(), _step(case), PAGE * s["block_table"].shape[1]
    pages = s["free_pages"].tolist()
    stack = pages[:s["free_in"].item()]
    held = len(stack)
    for b, (n, new, shared, _) in enumerate(step):
        if new < 0:
            stack += table[b][shared // PAGE:_blocks(n)]
    available, asked, asked_rows = len(stack), 0, 0
    got = {name: [] for name in ("granted", "starts", "lens_out", "next_out", "seq_ids", "slots", "positions")}
    got["row_start"] = [0]
    for b, (n, new, _, cut) in enumerate(step):
        rows = new if new > 0 and n + new <= limit else 0
        need = _blocks(n + rows) - _blocks(n)
        asked, asked_rows = asked + need, asked_rows + rows
        if (need and asked > available) or asked_rows > s["max_rows"]:
            rows = need = 0
        for j in range(need):
            table[b][_blocks(n) + j] = stack.pop()
        got["granted"].append(rows)
        got["starts"].append(n)
        got["lens_out"].append(0 if new < 0 else n + rows)
        got["next_out"].append(0 if new < 0 else n + cut + rows)
        got["seq_ids"] += [b] * rows
        got["slots"] += range(n, n + rows)
        got["positions"] += range(n + cut, n + cut + rows)
        got["row_start"].append(got["row_start"][-1] + rows)
    rest = s["max_rows"] - len(got["slots"])
    got["seq_ids"] += [-1] * rest
    got["slots"] += [0] * rest
    got["positions"] += [0] * rest
    if len(stack) > held:
        pages[held:len(stack)] = stack[held:]
    got.update(free_out=[len(stack)], block_table=table, free_pages=pages)
    return {name: _int(got[name]) for name in PLANNED}
