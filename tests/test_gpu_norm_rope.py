"""qk_norm_rope, qk_norm_rope_append and qk_norm_rope_backward against the formulas in 64 bits.

Tolerances.  An output is rounded to bf16 once, by at most half a unit in its last place: bf16 has 8 significant bits, so between
2^e and 2^(e+1) a unit is 2^(e-7) and half of it 2^(e-8).  What the fp32 steps before that add is far below: every factor is within a few 2^-24, and a rotated element is the sum of two products, so
the error is bounded by 2^-20 times the larger of the pair, for which the row's largest value stands.  The weights'
gradients are fp32 sums of products (u c + v s) x r, two a row: a product has at most ten roundings, and behind it stand the additions of a
lane (its share of the rows), of the wave, the workgroup and the final sum, at most 40; each is 2^-24 of the sum of the
products' absolute values (the two of a row may cancel, so |u c| + |v s| counts and not their sum).
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 1e-6
U = 2.0 ** -24


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


def f64(t):
    return t.detach().double().cpu().numpy()


def rope_table(length, m):
    angle = np.arange(length)[:, None] * 10000.0 ** (-np.arange(0, m, 2) / max(m, 1))
    return np.concatenate([np.cos(angle), np.sin(angle)], axis=1).astype(np.float32)


def pairs(x, m, interleaved):
    """Views of the first and the second of every pair."""
    return (x[..., 0:m:2], x[..., 1:m:2]) if interleaved else (x[..., :m // 2], x[..., m // 2:m])


def rotated(x, table, positions, m, interleaved, back=False):
    y = x.copy()
    if m:
        row = table[np.clip(positions, 0, len(table) - 1)].astype(np.float64)[:, None]
        c, s = row[..., :m // 2], row[..., m // 2:] * (-1 if back else 1)
        u, v = pairs(x, m, interleaved)
        y0, y1 = pairs(y, m, interleaved)
        y0[...], y1[...] = u * c - v * s, v * c + u * s
    return y


def forward(x, w, table, positions, m, interleaved, eps=EPS):
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rotated(x * r * w, table, positions, m, interleaved)


def backward(dy, x, w, table, positions, m, interleaved, eps=EPS):
    """-> dx, dw and the sum of the absolute products of dw"""
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dz = rotated(dy, table, positions, m, interleaved, back=True)
    g = dz * w
    dx = r * (g - x * r * r * (g * x).mean(-1, keepdims=True))
    size = np.abs(dy)
    if m:   # |u c| + |v s| for both of a pair
        u, v = pairs(np.abs(dy), m, interleaved)
        row = np.abs(table)[np.clip(positions, 0, len(table) - 1)].astype(np.float64)[:, None]
        s0, s1 = pairs(size, m, interleaved)
        s0[...], s1[...] = u * row[..., :m // 2] + v * row[..., m // 2:], v * row[..., :m // 2] + u * row[..., m // 2:]
    return dx, (dz * x * r).sum((0, 1)), (size * np.abs(x) * r).sum((0, 1))


class Rows:
    """Inputs of one call: queries, keys and values side by side in one tensor with a gap, as a fused projection leaves them."""

    def __init__(self, sd, T, hq, hkv, d, m, interleaved, seed, fp32=False, gap=0, table_len=512, side_by_side=False):
        import torch
        gen = torch.Generator().manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=gen)  # noqa: E731
        self.T, self.hq, self.hkv, self.d, self.m, self.interleaved = T, hq, hkv, d, m, interleaved
        width = (hq + 2 * hkv) * d + gap
        self.all = (normal(T, width) * torch.exp(normal(T, 1))).bfloat16().cuda()
        at = [0, hq * d, (hq + hkv) * d, (hq + 2 * hkv) * d]
        self.q, self.k, self.v = (self.all[:, i:j] for i, j in zip(at, at[1:]))
        if side_by_side:
            self.q, self.k, self.v = (x.contiguous() for x in (self.q, self.k, self.v))
        kind = torch.float32 if fp32 else torch.bfloat16
        self.qw, self.kw = ((1 + 0.3 * normal(d)).to(kind).cuda() for _ in range(2))
        self.table = torch.from_numpy(rope_table(table_len, m)).cuda() if m else None
        self.positions = torch.randint(0, table_len, (T,), generator=gen, dtype=torch.int32).cuda() if m else None
        strides = [0, 0, 0] if side_by_side else [width] * 3
        self.norm = sd.QkNorm(num_q_heads=hq, num_kv_heads=hkv, head_dim=d, rotary_dim=m, interleaved=int(interleaved), table_len=table_len if m else 0,
                              weight_dtype=sd.SD_F32 if fp32 else sd.SD_BF16, eps=EPS, q_stride=strides[0], k_stride=strides[1], v_stride=strides[2])

    def host(self, x, heads):
        return f64(x).reshape(self.T, heads, self.d)

    def rest(self):
        return (self.table.cpu().numpy() if self.m else None, self.positions.cpu().numpy() if self.m else None, self.m, self.interleaved)

    def expected(self):
        return (forward(self.host(self.q, self.hq), f64(self.qw), *self.rest()), forward(self.host(self.k, self.hkv), f64(self.kw), *self.rest()))


def check_rounded(got, want):
    top = np.abs(want).max(-1, keepdims=True)
    half_unit = 2.0 ** (np.frexp(want)[1] - 9)   # (frexp: |want| in [2^(e-1), 2^e))
    bad = ~(np.abs(got - want) <= half_unit + top * 2.0 ** -20)
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


SHAPES = [  # T, heads, kv heads, d, rotary, interleaved, fp32 weights, gap
    (1, 1, 1, 128, 128, False, False, 0),
    (1, 28, 4, 128, 128, False, False, 0),
    (7, 8, 2, 64, 64, False, True, 8),
    (33, 40, 8, 64, 32, True, False, 24),
    (64, 28, 4, 128, 64, False, False, 0),
    (5, 3, 1, 128, 16, False, True, 16),
    (19, 5, 5, 128, 128, True, False, 8),
    (9, 6, 2, 64, 16, True, True, 0),
    (130, 12, 3, 128, 112, False, False, 0),
    (11, 12, 3, 64, 48, False, False, 40),
    (23, 64, 8, 128, 0, False, False, 0),
    (1021, 16, 2, 128, 128, False, False, 0),
]


@pytest.mark.parametrize("T,hq,hkv,d,m,interleaved,fp32,gap", SHAPES)
def test_rows(sd, T, hq, hkv, d, m, interleaved, fp32, gap):
    import torch
    r = Rows(sd, T, hq, hkv, d, m, interleaved, T + hq, fp32, gap)
    q_out, k_out = torch.full((T, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((T, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    sd.qk_norm_rope(r.norm, r.q, r.k, r.qw, r.kw, r.table, r.positions, T, q_out, k_out)
    q, k = r.expected()
    check_rounded(f64(q_out), q)
    check_rounded(f64(k_out), k)


def test_rows_in_place(sd):
    r = Rows(sd, 37, 8, 2, 128, 128, False, 3, side_by_side=True)
    q, k = r.expected()
    sd.qk_norm_rope(r.norm, r.q, r.k, r.qw, r.kw, r.table, r.positions, r.T, r.q, r.k)
    check_rounded(r.host(r.q, 8), q)
    check_rounded(r.host(r.k, 2), k)


def test_zero_rows_tiny_rows_and_rows_that_are_not_finite(sd):
    import torch
    r = Rows(sd, 6, 4, 2, 128, 128, False, 4)
    r.q[0] = 0
    r.q[1] = 1e-30                      # eps outweighs it
    r.q[2, 5] = float("inf")            # head 0 only
    r.q[3, 128 + 7] = float("nan")      # head 1 only
    r.q[4] = 1e18                       # squares near the top of fp32
    q_out, k_out = torch.empty(6, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(6, 2, 128, dtype=torch.bfloat16, device="cuda")
    sd.qk_norm_rope(r.norm, r.q, r.k, r.qw, r.kw, r.table, r.positions, 6, q_out, k_out)
    got = f64(q_out)
    assert (got[0] == 0).all()
    want, _ = r.expected()
    finite = np.ones((6, 4), bool)
    finite[2, 0] = finite[3, 1] = False
    check_rounded(got[finite], want[finite])
    assert np.isnan(got[2, 0]).any() and np.isnan(got[3, 1]).all()   # x r is inf * 0; a NaN reaches its row through the mean
    assert np.isfinite(f64(k_out)).all()


def test_positions_outside_the_table_take_its_ends(sd):
    import torch
    r = Rows(sd, 5, 2, 1, 64, 64, False, 5)
    r.positions = torch.tensor([-1, -2 ** 31, 512, 2 ** 31 - 1, 511], dtype=torch.int32, device="cuda")
    q_out, k_out = torch.empty(5, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(5, 1, 64, dtype=torch.bfloat16, device="cuda")
    sd.qk_norm_rope(r.norm, r.q, r.k, r.qw, r.kw, r.table, r.positions, 5, q_out, k_out)
    q, k = r.expected()
    check_rounded(f64(q_out), q)
    check_rounded(f64(k_out), k)


@pytest.mark.parametrize("T,hq,hkv,d,m,interleaved,batch,with_slots", [(1, 28, 4, 128, 128, False, 3, True), (9, 8, 2, 64, 64, False, 9, False),
                                                                       (131, 40, 8, 64, 32, True, 4, True), (300, 32, 8, 128, 128, False, 5, True)])
def test_append(sd, T, hq, hkv, d, m, interleaved, batch, with_slots):
    import torch
    r = Rows(sd, T, hq, hkv, d, m, interleaved, T, gap=8)
    rng = np.random.default_rng(T)
    blocks, pages = 40, batch * 40 + 3
    table = rng.permutation(pages)[:batch * blocks].reshape(batch, blocks).astype(np.int32)
    if with_slots:
        cells = rng.choice(batch * blocks * 16, T, replace=False)
        seq, slot = cells // (blocks * 16), cells % (blocks * 16)
        seq[::5], slot[1::7] = -1, -3                       # rows that are not kept
        if T > 20:
            seq[3], slot[4] = batch, blocks * 16
            table[int(seq[6]), int(slot[6]) // 16] = pages     # no such page
    else:
        seq, slot = np.arange(T), f64(r.positions).astype(int)
    dev = lambda a: torch.tensor(a.astype(np.int32), device="cuda")  # noqa: E731
    k_pages = torch.full((pages, hkv, 16, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    v_pages = torch.full_like(k_pages, float("nan"))
    shape = sd.Shape(batch=batch, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, page_size=16, num_pages=pages, max_blocks_per_seq=blocks, kv_dtype=sd.SD_BF16,
                     max_context_len=blocks * 16, chunk_tokens=0)
    q_out = torch.full((T, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    sd.qk_norm_rope_append(shape, r.norm, r.q, r.k, r.v, r.qw, r.kw, r.table, r.positions, dev(seq) if with_slots else None, dev(slot) if with_slots else None, T,
                           q_out, k_pages, v_pages, dev(table))
    q, k = r.expected()
    check_rounded(f64(q_out), q)
    kp, vp, v = f64(k_pages), f64(v_pages), r.host(r.v, hkv)
    written = np.zeros((pages, 16), bool)
    for t in range(T):
        s, p = int(seq[t]), int(slot[t])
        if not (0 <= s < batch and 0 <= p < blocks * 16) or not 0 <= table[s, p // 16] < pages:
            continue
        page = table[s, p // 16]
        written[page, p % 16] = True
        check_rounded(kp[page, :, p % 16], k[t])
        assert np.array_equal(vp[page, :, p % 16], v[t])
    rest = np.broadcast_to(~written[:, None, :], (pages, hkv, 16))
    assert np.isnan(kp[rest]).all() and np.isnan(vp[rest]).all()


def run_backward(sd, r, dq_out, dk_out):
    import torch
    ws = sd.qk_norm_rope_workspace_bytes(r.norm, r.T)
    work = torch.empty(ws, dtype=torch.uint8, device="cuda").fill_(255)
    grads = torch.full_like(r.all, float("nan"))
    at = [0, r.hq * r.d, (r.hq + r.hkv) * r.d]
    dq, dk = grads[:, at[0]:at[1]], grads[:, at[1]:at[2]]
    dqw, dkw = torch.full((r.d,), float("nan"), device="cuda"), torch.full((r.d,), float("nan"), device="cuda")
    sd.qk_norm_rope_backward(r.norm, dq_out, dk_out, r.q, r.k, r.qw, r.kw, r.table, r.positions, r.T, dq, dk, dqw, dkw, work, ws)
    assert grads[:, at[2]:].isnan().all()   # nothing beside the two
    return dq, dk, dqw, dkw


@pytest.mark.parametrize("T,hq,hkv,d,m,interleaved,fp32,gap", SHAPES)
def test_gradient(sd, T, hq, hkv, d, m, interleaved, fp32, gap):
    import torch
    r = Rows(sd, T, hq, hkv, d, m, interleaved, 2 * T + hq, fp32, gap)
    gen = torch.Generator().manual_seed(T)
    dq_out, dk_out = (torch.randn(T, h, d, generator=gen).bfloat16().cuda() for h in (hq, hkv))
    dq, dk, dqw, dkw = run_backward(sd, r, dq_out, dk_out)
    for x, w, dy, dx, dw, heads in ((r.q, r.qw, dq_out, dq, dqw, hq), (r.k, r.kw, dk_out, dk, dkw, hkv)):
        want_x, want_w, size = backward(f64(dy), r.host(x, heads), f64(w), *r.rest())
        check_rounded(r.host(dx, heads), want_x)
        lane = T * heads / 32 + 1   # rows of a lane, were there one workgroup
        assert (np.abs(f64(dw) - want_w) <= (10 + min(lane, 64) + 40) * U * size).all()


def test_gradient_against_differences():
    """The formula that the gradient is held to is the derivative of the forward one (64 bits, central differences)."""
    rng = np.random.default_rng(0)
    for m, interleaved in ((8, False), (4, True)):
        T, H, d, h = 3, 2, 8, 1e-5
        x, w, dy = rng.normal(size=(T, H, d)), rng.normal(size=d), rng.normal(size=(T, H, d))
        table, pos = rope_table(9, m), rng.integers(0, 9, T)
        dx, dw, _ = backward(dy, x, w, table, pos, m, interleaved)
        loss = lambda x, w: (forward(x, w, table, pos, m, interleaved) * dy).sum()  # noqa: E731
        for i in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[i] = h
            assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[i]) < 1e-8
        for i in range(d):
            e = np.zeros_like(w)
            e[i] = h
            assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[i]) < 1e-8


def test_gradient_of_no_rows_and_twice_the_same(sd):
    import torch
    r = Rows(sd, 777, 16, 2, 128, 128, False, 6)
    dq_out, dk_out = (torch.randn(777, h, 128, device="cuda").bfloat16() for h in (16, 2))
    one, two = run_backward(sd, r, dq_out, dk_out), run_backward(sd, r, dq_out, dk_out)
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    r.T = 0
    _, _, dqw, dkw = run_backward(sd, r, dq_out, dk_out)
    assert (dqw == 0).all() and (dkw == 0).all()


def test_calls_of_many_rows_agree_with_their_halves(sd):
    """Rows of 64 MB and more stream past the caches: the same rows as from two smaller calls, bit for bit."""
    import torch
    T, hq, hkv, d = 4400, 56, 4, 128
    r = Rows(sd, T, hq, hkv, d, 128, False, 7)
    dq_out, dk_out = (torch.randn(T, h, d, device="cuda").bfloat16() for h in (hq, hkv))
    shape = sd.Shape(batch=T, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, page_size=16, num_pages=T, max_blocks_per_seq=1, kv_dtype=sd.SD_BF16, max_context_len=16, chunk_tokens=0)
    table, slots = torch.randperm(T).int().cuda(), (torch.arange(T) % 16).int().cuda()
    seq = torch.arange(T, dtype=torch.int32, device="cuda")

    def calls(t0, t1):
        n = t1 - t0
        outs = [torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hq)]
        pools = [torch.zeros(T, hkv, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        q, k, v, pos = r.q[t0:t1], r.k[t0:t1], r.v[t0:t1], r.positions[t0:t1].clone()
        sd.qk_norm_rope(r.norm, q, k, r.qw, r.kw, r.table, pos, n, outs[0], outs[1])
        sd.qk_norm_rope_append(shape, r.norm, q, k, v, r.qw, r.kw, r.table, pos, seq[t0:t1].clone(), slots[t0:t1].clone(), n, outs[2], *pools, table)
        ws = sd.qk_norm_rope_workspace_bytes(r.norm, n)
        work, grads, dw = torch.empty(ws, dtype=torch.uint8, device="cuda"), torch.zeros_like(r.all[t0:t1]), [torch.empty(d, device="cuda") for _ in range(2)]
        sd.qk_norm_rope_backward(r.norm, dq_out[t0:t1], dk_out[t0:t1], q, k, r.qw, r.kw, r.table, pos, n, grads, grads[:, hq * d:], *dw, work, ws)
        return outs + [grads], pools, dw

    assert T * (hq + hkv) * d * 2 >= 64 << 20
    rows, pools, dw = calls(0, T)
    parts = [calls(0, 2000), calls(2000, T)]
    for i, x in enumerate(rows):
        assert torch.equal(x, torch.cat([p[0][i] for p in parts]))
    for i in range(2):
        assert torch.equal(pools[i], parts[0][1][i] + parts[1][1][i])   # (each half leaves the other's slots 0)
        want = parts[0][2][i].double() + parts[1][2][i].double()
        _, _, size = backward(f64((dq_out, dk_out)[i]), r.host((r.q, r.k)[i], (hq, hkv)[i]), f64((r.qw, r.kw)[i]), *r.rest())
        assert (np.abs(f64(dw[i]) - want.cpu().numpy()) <= 2 * 114 * U * size).all()


def test_another_stream(sd):
    import torch
    r = Rows(sd, 50, 8, 2, 128, 128, False, 8)
    outs = [torch.zeros(50, h, 128, dtype=torch.bfloat16, device="cuda") for h in (8, 2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sd.qk_norm_rope(r.norm, r.q, r.k, r.qw, r.kw, r.table, r.positions, 50, *outs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for got, want in zip(outs, r.expected()):
        check_rounded(f64(got), want)
