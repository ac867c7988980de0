"""Sampling, log probabilities and the plan of a step in plain numpy, 64 bits: what the kernels are compared with."""
import numpy as np

ONE = 1 << 43   # of a weight


def bf16_bits(x):
    """float32 -> the nearest bf16's bits (ties to even; NaN stays NaN)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7fc0), r)


def bf16_values(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32)


def weights_of(x, temperature):
    """(whole weights, the logits relative to the largest over the temperature) of a row; None where there is nothing."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    top = x.max()
    if top == -np.inf:
        return None
    if top == np.inf:
        z = np.where(x == np.inf, 0.0, -np.inf)
    else:
        d = x - top
        with np.errstate(over="ignore"):
            z = np.where(d == -np.inf, -np.inf, d / temperature if np.isfinite(temperature) else 0 * np.where(np.isfinite(d), d, 0))
    return [int(w) for w in np.rint(np.exp(z) * ONE)], z


def sample(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, uniform=0.0):
    """(token, log probability, log probability of the draw) of a row of logits."""
    vocab = len(x)
    greedy = not temperature > 0
    got = weights_of(x, 1.0 if greedy else float(temperature))
    if got is None:
        return -1, -np.inf, -np.inf
    w, z = got
    total = sum(w)
    order = np.lexsort((np.arange(vocab), -np.where(np.isnan(x), -np.inf, x.astype(np.float64))))
    if greedy:
        token = int(order[0])
        return token, -np.log(total / ONE), 0.0
    n = vocab if top_k <= 0 else min(top_k, vocab)
    if top_p < 1:
        share = max(0.0, float(top_p)) * float(sum(w[i] for i in order[:n]))
        before, m = 0, 0
        while m < n and (m == 0 or before < share):
            before += w[order[m]]
            m += 1
        n = m
    kept = sorted(int(i) for i in order[:n])
    if min_p > 0:
        kept = [i for i in kept if np.exp(z[i]) >= min(float(min_p), 1.0)]
    mass = sum(w[i] for i in kept)
    u = float(uniform) if uniform > 0 else 0.0
    target = min(mass, int(u * float(mass)) + 1)
    upto = 0
    for token in kept:
        upto += w[token]
        if upto >= target:
            break
    return token, z[token] - np.log(total / ONE), z[token] - np.log(mass / ONE)


def logprobs(x, target, temperature=1.0):
    """(log probability, entropy, log2-domain moments E|z|, E z^2, log2 sum) of a row."""
    z = x.astype(np.float64) / temperature
    z = z - z.max()
    e = np.exp(z)
    s = e.sum()
    p = e / s
    logp = z - np.log(s)
    some = p > 0
    z2 = np.where(some, z, 0) / np.log(2)
    return logp[target], -(p[some] * logp[some]).sum(), (p * abs(z2)).sum(), (p * z2 * z2).sum(), np.log2(s)


def gradient(x, target, temperature, g, h):
    z = x.astype(np.float64) / temperature
    z = z - z.max()
    e = np.exp(z)
    p = e / e.sum()
    logp = np.where(p > 0, z - np.log(e.sum()), 0)
    entropy = -(p * logp).sum()
    d = -p * (g + h * (logp + entropy))
    d[target] += g
    return d / temperature


def plan(new, shared, lens, nxt, free, table, max_rows, limit):
    """A step's places, one sequence after the other; `free` is a list of pages, `table` rows of pages: both are changed."""
    blocks = lambda n: (n + 15) // 16  # noqa: E731
    lens = [max(0, min(n, limit)) for n in lens]
    for b, n in enumerate(new):
        if n < 0:
            free += table[b][max(0, min(shared[b], lens[b])) // 16:blocks(lens[b])]
    available, asked, asked_rows = len(free), 0, 0
    got = dict(granted=[], row_start=[0], starts=lens, lens_out=[], next_out=[], seq_ids=[], slots=[], positions=[])
    for b, n in enumerate(new):
        rows = n if n > 0 and lens[b] + n <= limit else 0
        need = blocks(lens[b] + rows) - blocks(lens[b])
        asked, asked_rows = asked + need, asked_rows + rows
        if (need and asked > available) or asked_rows > max_rows:
            rows = need = 0
        for j in range(need):
            table[b][blocks(lens[b]) + j] = free.pop()
        got["granted"].append(rows)
        got["row_start"].append(got["row_start"][-1] + rows)
        got["lens_out"].append(0 if n < 0 else lens[b] + rows)
        got["next_out"].append(0 if n < 0 else nxt[b] + rows)
        got["seq_ids"] += [b] * rows
        got["slots"] += range(lens[b], lens[b] + rows)
        got["positions"] += range(nxt[b], nxt[b] + rows)
    rest = max_rows - len(got["slots"])
    for name, fill in (("seq_ids", -1), ("slots", 0), ("positions", 0)):
        got[name] += [fill] * rest
    return got
