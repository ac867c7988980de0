// The attention weight that every cached token receives, added to its running score:
//
//   s'[b][g][t] = decay s[b][g][t] + sum_rows softmax_t(scale <q_row, K_t>)      rows: the query rows of sequence b, heads of KV head g
//
// A weight needs its row's maximum and sum over all tokens, so K is walked, each row's statistics are joined, and the products become weights.
//
//   S[token][row] = K_page[token][d] . Q^T[d][row]     mfma 16x16x32 bf16, a page of 16 tokens at a time
//
// Up to 16 rows (a decode step: the heads of a KV head) fit one tile, and the products are kept, so K is read once.  Either one workgroup takes a whole
// (sequence, KV head) and keeps them in its registers (weight_whole_kernel), or they go through memory in fp32, rows * 4 bytes a token beside K's
// 64 to 256, between two launches (weight_products_kernel, weight_apply_kept_kernel).  Bound by reading K: 256 of 1 k - 8 k, bf16, 7 heads a group:
// 61 us, 4.4 TB/s of the 6.7 that a plain walk reads, for the longest of a compute unit's sequences ends last; 2048 of 0.5 k - 4 k, fp8: 117 us, 5.3 TB/s.
// With more rows (the last tokens of a prompt) the products would be more bytes than K: they are made twice, by weight_stats_kernel and
// weight_apply_kernel, rows stay in registers and K streams past.  Bound by matrix and vector units taking turns, for the waves of a workgroup do the same
// thing at the same time: 8 sequences of 5 k - 8 k, 8 KV heads, 256 rows 41 + 5 + 40 us, 660 and 670 TFLOP/s in the passes; vector units 62 - 69 % busy, matrix
// units 34 %, both at once 11 - 13 %.
//
// Where products are kept a lane holds four tokens (4 (lane / 16) ..) of row lane % 16.  Which d an operand's 16 bytes are differs between
// pools, and Q is read in the same order.  Weights, sums and scores are fp32 throughout.
#include <type_traits>

#include "attn_tile.h"

namespace sd {

namespace {

// One page of K: lane n + 16 c holds token n.  operand(s): the first operand of step s of the product.
template <int D>
struct Bf16Rows {
    static constexpr int kDim = D;
    static constexpr int kBytes = kPage * D * 2;
    static constexpr bool kScaled = false;
    u32x4 k[D / 32];
    SD_DEV static int q_offset(int s, int c) { return 32 * s + 8 * c; }
    SD_DEV u32x4 operand(int s) const { return k[s]; }
    static constexpr int kRowBytes = 2 * D;
};
template <int D>
struct Fp8Rows {
    static constexpr int kDim = D;
    static constexpr int kBytes = kPage * D;
    static constexpr bool kScaled = true;
    u32x4 k[D / 64];   // 16 codes each
    SD_DEV static int q_offset(int s, int c) { return 64 * (s / 2) + 16 * c + 8 * (s % 2); }
    SD_DEV u32x4 operand(int s) const
    {
        const unsigned lo = k[s / 2][2 * (s % 2)], hi = k[s / 2][2 * (s % 2) + 1];
        return u32x4{cvt_pk_bf16_fp8<false>(lo), cvt_pk_bf16_fp8<true>(lo), cvt_pk_bf16_fp8<false>(hi), cvt_pk_bf16_fp8<true>(hi)};
    }
    static constexpr int kRowBytes = D;
};

// A page on its way through LDS.  Lanes in operand layout ask for 64 bytes of each of 16 rows at a time, half a cache line; a workgroup that
// has a compute unit to itself gets 26 GB/s that way and 46 with loads of whole rows.  So 64 lanes bring 1 KB in one piece straight into
// LDS, 16 bytes each: piece p of row r goes to place p ^ (r mod the row's pieces), by which source a lane asks for, so that
// 16 rows' pieces of one column lie in different banks.
template <class K>
struct Staged {
    static constexpr int kNt = 2;   // cache policy bit nt
    static constexpr int kPieces = K::kRowBytes / 16, kLoads = K::kBytes / 1024;
    SD_DEV static void issue(const char *page, char *slot, int lane)
    {
#pragma unroll
        for (int s = 0; s < kLoads; ++s) {
            const int at = 64 * s + lane, r = at / kPieces, p = at % kPieces ^ r % kPieces;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(page + r * K::kRowBytes + p * 16),
                                             (__attribute__((address_space(3))) void *)(slot + s * 1024), 16, 0, kNt);
        }
    }
    SD_DEV static void fetch(K &k, const char *slot, int lane)
    {
        const int r = lane & 15, c = lane >> 4;
#pragma unroll
        for (int s = 0; s < kLoads; ++s) k.k[s] = *reinterpret_cast<const u32x4 *>(slot + r * K::kRowBytes + ((4 * s + c) ^ r % kPieces) * 16);
    }
};
// Waits for all but the newest N loads of this wave; for its LDS reads.  (s_waitcnt: vmcnt in bits 0-3 and 14-15, expcnt 4-6, lgkmcnt 8-11.)
template <int N>
SD_DEV void wait_loads()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
    asm volatile("" ::: "memory");
}
SD_DEV void wait_reads()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
}

// What a workgroup knows of its sequence.
struct Sequence {
    int L, first_q, n;   // tokens, first query row, query rows of it
    int base;            // position of the first one, which the whole range gives it; may be negative
};
SD_DEV Sequence sequence_of(const WeightArgs &a, int b)
{
    Sequence s;
    s.L = max(0, min(a.context_lens[b], a.max_context_len));
    s.first_q = b;
    s.n = 1;
    s.base = s.L - 1;
    if (a.q_start) {
        const int q0 = a.q_start[b], q1 = a.q_start[b + 1];
        const bool inside = q0 >= 0 && q1 <= a.total_q && q1 > q0;   // a range that leaves the rows has none
        s.first_q = inside ? q0 : 0;
        s.n = inside ? min(q1 - q0, a.max_q_len) : 0;
        s.base = inside ? s.L - (q1 - q0) : s.L;
    }
    return s;
}

// Row r of (sequence, KV head): query r / G, head r % G of the group.  The scale's sign is the queries' (q_flip): scaling keeps the order.
template <class K>
SD_DEV void load_q(u32x4 (&q)[K::kDim / 32], const WeightArgs &a, const Sequence &s, int g, int r, int rows, int lane)
{
    const int i = (int)a.per_group.of(r);
    const uint16_t *p = a.q + ((int64_t)(s.first_q + i) * a.Hq + g * a.G + (r - i * a.G)) * K::kDim;
#pragma unroll
    for (int j = 0; j < K::kDim / 32; ++j)
        q[j] = r < rows ? *reinterpret_cast<const u32x4 *>(p + K::q_offset(j, lane >> 4)) ^ a.q_flip : u32x4{0, 0, 0, 0};
}

// The tokens that row r attends: those before `end`.
SD_DEV int row_end(const WeightArgs &a, const Sequence &s, int r, int rows) { return r < rows ? min(s.L, s.base + 1 + (int)a.per_group.of(r)) : 0; }

struct Stat {
    float m, l;   // maximum (log2 domain) and sum of exp2(x - m)
};
SD_DEV float shrink_of(float from, float to) { return from == to ? 1.f : __builtin_amdgcn_exp2f(from - to); }   // (both may be -inf)
// What exponents are taken relative to: not a maximum of -inf, which is all that a stretch of tokens without any weight has.
SD_DEV float reference_of(float m) { return m == -INFINITY ? 0.f : m; }
SD_DEV Stat joined(Stat x, Stat y)
{
    const float m = fmaxf(x.m, y.m);
    return Stat{m, x.l * shrink_of(x.m, m) + y.l * shrink_of(y.m, m)};
}

}  // namespace

// A tile of few rows takes PACK pages: with W = 16 / PACK at least the rows, the rows stand W columns apart PACK times, every page's
// product gives all of them, and column n keeps that of page n / W.  So every lane holds four tokens of a row (row n % W), the
// exponentials are as many as there are products, and a tile of them is 1 KB in one piece.
template <int PACK>
struct Packed {
    static constexpr int kRows = kMaxGroup / PACK;
    int row, page, quarter;   // of the lane: row, page of the tile, four tokens of the page
    SD_DEV explicit Packed(int lane) : row(lane & (kRows - 1)), page((lane & 15) / kRows), quarter(lane >> 4) {}
    SD_DEV int token() const { return kPage * page + 4 * quarter; }   // the lane's first, counted from the tile's first
};

// A wave's walk over pages of one (sequence, KV head): those whose ids lanes 0 .. pages - 1 hold.  Two are on their way or in the wave's two
// slots of LDS: while it works on one, the next comes.
template <class K>
struct Walk {
    const char *pool;   // + id * stride: the page's tile of this head
    int64_t stride;
    char *slots;
    int ids, pages, lane;
    float scales;
    SD_DEV Walk(const WeightArgs &a, int b, int g, int page, int count, char *lds, int lane_) : slots(lds), pages(count), lane(lane_)
    {   // `page`: the lane's; `count`: of the wave
        ids = a.block_table[(int64_t)b * a.max_blocks + page];
        scales = K::kScaled ? a.k_scales[(int64_t)ids * a.Hkv + g] * a.scale_log2e : a.scale_log2e;
        stride = (int64_t)a.Hkv * K::kBytes;
        pool = static_cast<const char *>(a.k_pages) + (int64_t)g * K::kBytes;
    }
    SD_DEV void issue(int i) const
    {
        if (i < pages) Staged<K>::issue(pool + __builtin_amdgcn_readlane(ids, i) * stride, slots + i % 2 * K::kBytes, lane);
    }
    SD_DEV void start() const
    {
        wait_loads<0>();   // (what page() counts are its own loads)
        issue(0);
        issue(1);
    }
    // Scaled products of page i, which comes after i - 1.
    SD_DEV f32x4 page(int i, const u32x4 (&q)[K::kDim / 32]) const
    {
        if (i + 1 < pages) wait_loads<Staged<K>::kLoads>();
        else wait_loads<0>();
        K k;
        Staged<K>::fetch(k, slots + i % 2 * K::kBytes, lane);
        wait_reads();
        issue(i + 2);
        f32x4 y = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < K::kDim / 32; ++c) y = mfma_bf16_k32(k.operand(c), q[c], y);
        return y * (K::kScaled ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scales), i)) : scales);
    }
    // Of the PACK pages of tile i.
    template <int PACK>
    SD_DEV f32x4 tile(int i, const u32x4 (&q)[K::kDim / 32], const Packed<PACK> &at) const
    {
        f32x4 x = page(i * PACK, q);
#pragma unroll
        for (int j = 1; j < PACK; ++j) {
            const f32x4 y = page(i * PACK + j, q);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = at.page == j ? y[e] : x[e];
        }
        return x;
    }
};

// First step of a decode step: a.wave_tiles tiles to a wave, KV head fastest in the grid.
template <class K, int PACK>
__global__ __launch_bounds__(kWaves * 64) void weight_products_kernel(WeightArgs a)
{
    constexpr int W = kMaxGroup / PACK;
    __shared__ __attribute__((aligned(16))) char s_pages[kWaves][2 * K::kBytes];
    __shared__ Stat s_stat[kWaves][W];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.x % a.Hkv, c = blockIdx.x / a.Hkv % a.blocks, b = blockIdx.x / a.Hkv / a.blocks;
    const Sequence s = sequence_of(a, b);
    const int rows = s.n * a.G, last = (s.L + kPage - 1) / kPage - 1, all_tiles = last / PACK + 1, block0 = c * kWaves * a.wave_tiles;
    if (block0 >= all_tiles || s.L == 0 || rows == 0) return;   // workgroup-uniform
    const int64_t unit = (int64_t)b * a.Hkv + g;
    const int tile0 = block0 + wave * a.wave_tiles, tiles = max(0, min(a.wave_tiles, all_tiles - tile0));
    const Packed<PACK> at(lane);
    const Walk<K> walk(a, b, g, min(tile0 * PACK + lane, last), tiles * PACK, s_pages[wave], lane);
    u32x4 q[K::kDim / 32];
    load_q<K>(q, a, s, g, at.row, rows, lane);
    const int end = row_end(a, s, at.row, rows);
    float *to = a.products + ((unit * a.max_tiles + tile0) * 64 + lane) * 4;
    Stat stat = {-INFINITY, 0.f};
    walk.start();
    for (int i = 0; i < tiles; ++i) {
        const f32x4 x = walk.tile(i, q, at);
        *reinterpret_cast<f32x4 *>(to + i * 256) = x;
        const int t0 = (tile0 + i) * PACK * kPage + at.token();
        float m = stat.m;
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, t0 + e < end ? x[e] : -INFINITY);
        const float ref = reference_of(m);
        float l = stat.l * shrink_of(stat.m, m);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(x[e] - ref);
            l += t0 + e < end ? p : 0.f;
        }
        stat = Stat{m, l};
    }
    for (int off = W; off < 64; off *= 2) stat = joined(stat, Stat{__shfl_xor(stat.m, off, 64), __shfl_xor(stat.l, off, 64)});
    if (lane < W) s_stat[wave][lane] = stat;
    __syncthreads();
    if (threadIdx.x < W) {
        Stat all = s_stat[0][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) all = joined(all, s_stat[w][lane]);
        a.stats[(unit * a.blocks + c) * W + lane] = float2{all.m, all.l};
    }
}

// x plus that of the lane's partners in the 2^k columns of a row's packed stretch (DPP adds).
template <int W>
SD_DEV float over_rows(float x)
{
#define SD_DPP_ADD(ctrl) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xf, 0xf, false))
    SD_DPP_ADD(0xb1);                  // quad_perm 1 0 3 2
    SD_DPP_ADD(0x4e);                  // quad_perm 2 3 0 1
    if (W >= 8) SD_DPP_ADD(0x141);     // row_half_mirror
    if (W >= 16) SD_DPP_ADD(0x140);    // row_mirror
#undef SD_DPP_ADD
    return x;
}

// Its second step: kApplyTokens tokens to a workgroup, a tile at a time to a wave.
constexpr int kApplyTokens = 1024;
template <int PACK>
__global__ __launch_bounds__(256) void weight_apply_kept_kernel(WeightArgs a)
{
    constexpr int W = kMaxGroup / PACK, T = kApplyTokens / kPage / PACK / 4;   // tiles of a wave
    __shared__ float2 s_row[kMaxGroup];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.x % a.Hkv, j = blockIdx.x / a.Hkv % a.apply_blocks, b = blockIdx.x / a.Hkv / a.apply_blocks;
    const Sequence s = sequence_of(a, b);
    if (j * kApplyTokens >= s.L) return;
    const int64_t unit = (int64_t)b * a.Hkv + g;
    const int rows = s.n * a.G, tile0 = (j * 4 + wave) * T, tiles = (s.L + PACK * kPage - 1) / (PACK * kPage);
    const Packed<PACK> at(lane);
    // the products and the old scores are on their way while the statistics are joined
    f32x4 x[T];
    float before[T];
    const int64_t scores = unit * a.score_stride;
    const int t0 = tile0 * PACK * kPage + at.token(), mine = t0 + at.row;   // lane's first token; the one that it stores
#pragma unroll
    for (int i = 0; i < T; ++i) {
        if (tile0 + i < tiles && rows) x[i] = *reinterpret_cast<const f32x4 *>(a.products + ((unit * a.max_tiles + tile0 + i) * 64 + lane) * 4);
        const int t = mine + i * PACK * kPage;
        before[i] = a.scores_in && at.row < 4 && t < s.L - a.new_tokens ? a.scores_in[scores + t] : 0.f;
    }
    {   // row tid / 16, every 16th block to a lane
        const int r = threadIdx.x / 16, from = threadIdx.x % 16, blocks = (s.L + a.block_tokens - 1) / a.block_tokens;
        Stat sum = {-INFINITY, 0.f};
        if (r < rows)
            for (int c = from; c < blocks; c += 16) {
                const float2 v = a.stats[(unit * a.blocks + c) * W + r];
                sum = joined(sum, Stat{v.x, v.y});
            }
        for (int off = 1; off < 16; off *= 2) sum = joined(sum, Stat{__shfl_xor(sum.m, off, 64), __shfl_xor(sum.l, off, 64)});
        if (from == 0) s_row[r] = float2{sum.m, 1.f / sum.l};
    }
    __syncthreads();
    const float2 row = s_row[at.row];
    const int end = row_end(a, s, at.row, rows);
#pragma unroll
    for (int i = 0; i < T; ++i) {
        if (tile0 + i < tiles) {   // wave-uniform
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = __builtin_amdgcn_exp2f(x[i][e] - row.x) * row.y;
                const float all = over_rows<W>(t0 + i * PACK * kPage + e < end ? p : 0.f);
                sum = at.row == e ? all : sum;
            }
            const int t = mine + i * PACK * kPage;
            if (at.row < 4 && t < s.L) a.scores_out[scores + t] = sum + a.decay * before[i];
        }
    }
}

// The sequence of a workgroup where those longer than half the bound come first: as workgroups end, the next ones are short (us: 128 sequences of
// 1 k - 8 k, 4 KV heads 123 : 109; 256 of 0.5 k - 4 k, fp8, 8 KV heads 126 : 117; 200 of one length 164 : 164).
SD_DEV int long_first(const WeightArgs &a, int at, int lane)
{
    int len[kLaneLengths];
    unsigned long long longs[kLaneLengths];
    int all_long = 0;
#pragma unroll
    for (int j = 0; j < kLaneLengths; ++j) len[j] = 64 * j + lane < a.B ? a.context_lens[64 * j + lane] : 0;
#pragma unroll
    for (int j = 0; j < kLaneLengths; ++j) {
        longs[j] = __builtin_amdgcn_ballot_w64(len[j] > a.max_context_len / 2);
        all_long += __builtin_popcountll(longs[j]);
    }
    const bool is_long = at < all_long;   // wave-uniform: the at-th of the long ones, or of the others
    if (!is_long) at -= all_long;
    int b = 0;
#pragma unroll
    for (int j = 0; j < kLaneLengths; ++j) {
        const unsigned long long these = is_long ? longs[j] : ~longs[j];
        const int rank = __builtin_amdgcn_mbcnt_hi((unsigned)(these >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)these, 0));
        const unsigned long long it = __builtin_amdgcn_ballot_w64((these >> lane & 1) && rank == at);
        if (it) b = 64 * j + __builtin_ctzll(it);
        at -= __builtin_popcountll(these);
    }
    return b;
}

// Both steps in one: a workgroup takes a whole (sequence, KV head) and its products stay in its registers, whole_tiles to a wave.
template <class K, int PACK>
__global__ __launch_bounds__(1024) void weight_whole_kernel(WeightArgs a)
{
    constexpr int T = whole_tiles(PACK), W = kMaxGroup / PACK;
    extern __shared__ __attribute__((aligned(16))) char s_pages[];   // [waves][2][K::kBytes]
    __shared__ Stat s_stat[16][W];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x / 64;
    const int g = blockIdx.x % a.Hkv, b = a.long_first ? long_first(a, blockIdx.x / a.Hkv, lane) : blockIdx.x / a.Hkv;
    const Sequence s = sequence_of(a, b);
    if (s.L == 0) return;
    const int64_t unit = (int64_t)b * a.Hkv + g;
    const int rows = s.n * a.G, last = (s.L + kPage - 1) / kPage - 1, tiles = last / PACK + 1;
    const Packed<PACK> at(lane);
    // the wave's tile i is the sequence's tile i * waves + wave
    const Walk<K> walk(a, b, g, min((lane / PACK * waves + wave) * PACK + lane % PACK, last), (wave < tiles ? (tiles - 1 - wave) / waves + 1 : 0) * PACK,
                       s_pages + wave * (2 * K::kBytes), lane);
    u32x4 q[K::kDim / 32];
    load_q<K>(q, a, s, g, at.row, rows, lane);
    const int end = row_end(a, s, at.row, rows);
    const int64_t scores = unit * a.score_stride;
    f32x4 x[T];
    float m = -INFINITY;
    walk.start();
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const int tile = i * waves + wave;
        if (tile >= tiles) break;   // wave-uniform
        x[i] = walk.tile(i, q, at);
        const int t0 = tile * PACK * kPage + at.token();
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, t0 + e < end ? x[i][e] : -INFINITY);
    }
    for (int off = W; off < 64; off *= 2) m = fmaxf(m, __shfl_xor(m, off, 64));
    const float ref = reference_of(m);
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const int tile = i * waves + wave;
        if (tile >= tiles) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[i][e] = __builtin_amdgcn_exp2f(x[i][e] - ref);
            if (tile * PACK * kPage + at.token() + e >= end) x[i][e] = 0.f;
            l += x[i][e];
        }
    }
    for (int off = W; off < 64; off *= 2) l += __shfl_xor(l, off, 64);
    float before[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const int t = (i * waves + wave) * PACK * kPage + at.token() + at.row;
        before[i] = a.scores_in && at.row < 4 && t < s.L - a.new_tokens ? a.scores_in[scores + t] : 0.f;
    }
    if (lane < W) s_stat[wave][lane] = Stat{m, l};
    __syncthreads();
    Stat all = s_stat[0][at.row];
    for (int w = 1; w < waves; ++w) all = joined(all, s_stat[w][at.row]);
    const float weight = shrink_of(m, all.m) / all.l;
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const int tile = i * waves + wave;
        if (tile >= tiles) break;
        const int t0 = tile * PACK * kPage + at.token(), t = t0 + at.row;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = over_rows<W>(t0 + e < end ? x[i][e] * weight : 0.f);
            sum = at.row == e ? v : sum;
        }
        if (at.row < 4 && t < s.L) a.scores_out[scores + t] = sum + a.decay * before[i];
    }
}

// More rows than a tile: they stay, kRowTiles tiles of them in each wave's registers, and K streams past.  A workgroup walks up to a.wave_tiles groups of
// kGroupPages pages of one (sequence, KV head) for kRowTiles * 16 * waves rows; its waves bring a group into LDS, a page each, and all read it
// as operands, kAtOnce pages at a time, while the next one comes.  Where there are more rows, other workgroups take them: walking K again in
// the same one for each round of rows is a start-up each (us: 816 rows, one sequence of 37 k, 2 KV heads 88 : 65; 4096, one of 8 k, 8 KV heads 283 : 180).
constexpr int kGroupPages = 4, kGroupTokens = kGroupPages * kPage, kAtOnce = 2;
constexpr int kRowTiles = kRowsOfWave / kMaxGroup;
template <class K>
struct Stream {
    static constexpr int S = K::kDim / 32;
    const char *pool;   // + id * stride: the page's tile of this head
    int64_t stride;
    char *lds;          // [2][kGroupPages][K::kBytes]
    int ids, lane, wave, waves, groups;   // ids: of the workgroup's pages, a lane each
    float scales;
    unsigned long long below_zero;   // of the pages: those whose scale is
    SD_DEV Stream(const WeightArgs &a, int b, int g, int page0, int last, int groups_, char *lds_, int lane_, int wave_, int waves_)
        : lds(lds_), lane(lane_), wave(wave_), waves(waves_), groups(groups_)
    {
        ids = a.block_table[(int64_t)b * a.max_blocks + min(page0 + lane, last)];
        scales = K::kScaled ? a.k_scales[(int64_t)ids * a.Hkv + g] * a.scale_log2e : a.scale_log2e;
        below_zero = K::kScaled ? __builtin_amdgcn_ballot_w64(scales < 0.f) : 0;
        stride = (int64_t)a.Hkv * K::kBytes;
        pool = static_cast<const char *>(a.k_pages) + (int64_t)g * K::kBytes;
    }
    SD_DEV bool any_below_zero(int group) const { return below_zero >> group * kGroupPages & ((1u << kGroupPages) - 1); }
    SD_DEV char *slot(int group, int i) const { return lds + ((group & 1) * kGroupPages + i) * K::kBytes; }
    SD_DEV void issue(int group) const
    {
        for (int i = wave; i < kGroupPages; i += waves) Staged<K>::issue(pool + __builtin_amdgcn_readlane(ids, group * kGroupPages + i) * stride, slot(group, i), lane);
    }
    // Waits for a group, and sends the next one on its way: its slots were last read before the barrier.
    SD_DEV void next(int group) const
    {
        wait_loads<0>();
        __syncthreads();
        if (group + 1 < groups) issue(group + 1);
    }
    // Operands of kAtOnce of its pages.
    SD_DEV void fetch(int group, int first, u32x4 (&k)[kAtOnce][S], float (&scale)[kAtOnce]) const
    {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            K page;
            Staged<K>::fetch(page, slot(group, first + i), lane);
#pragma unroll
            for (int s = 0; s < S; ++s) k[i][s] = page.operand(s);
            scale[i] = K::kScaled ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scales), group * kGroupPages + first + i)) : scales;
        }
    }
};
// Which of a sequence's tokens a workgroup takes: a.wave_tiles groups of pages from group c of sequence b on; or, where a lane can hold every
// sequence's length (a.share), the fewest with which all workgroups run at once (or in as many turns as the bound on the lengths needs): they are
// as even as if all lengths were the bound's.  8 sequences of 5 k - 8 k, 256 rows, 8 KV heads: 13 groups each, not 16.
struct Share {
    int b, c, groups;   // b < 0: none
    int slot;           // of the statistics: sequence by sequence, a stretch of tokens each
};
SD_DEV int lane_groups(const WeightArgs &a, int lane) { return lane < a.B ? (max(0, min(a.context_lens[lane], a.max_context_len)) + kGroupTokens - 1) / kGroupTokens : 0; }
SD_DEV int wave_total(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }
SD_DEV int share_groups(const WeightArgs &a, int mine)
{
    if (a.share == 0) return a.wave_tiles;
    const int per_head = a.share / (a.Hkv * a.rounds);
    int w = max(1, (wave_total(mine) + per_head - 1) / per_head);
    while (w < a.wave_tiles && wave_total((mine + w - 1) / w) > per_head) ++w;   // (wave-uniform)
    return min(w, a.wave_tiles);
}
SD_DEV Share share_of(const WeightArgs &a, int lane)
{
    const int at = blockIdx.x / (a.Hkv * a.rounds);
    if (a.share == 0) return Share{at / a.blocks, at % a.blocks, a.wave_tiles, at};
    const int mine = lane_groups(a, lane), w = share_groups(a, mine), parts = (mine + w - 1) / w, upto = wave_scan(parts);
    const int b = __builtin_popcountll(__builtin_amdgcn_ballot_w64(upto <= at));
    if (b >= 64) return Share{-1, 0, 0, 0};
    return Share{b, at - __builtin_amdgcn_readlane(upto - parts, b), w, at};
}
// The first slot of sequence b, and its stretches' tokens.
SD_DEV Share first_share(const WeightArgs &a, int b, int lane)
{
    if (a.share == 0) return Share{b, 0, a.wave_tiles, b * a.blocks};
    const int mine = lane_groups(a, lane), w = share_groups(a, mine), parts = (mine + w - 1) / w;
    return Share{b, 0, w, __builtin_amdgcn_readlane(wave_scan(parts) - parts, b)};
}

template <int STEPS>
SD_DEV f32x4 products(const u32x4 (&k)[STEPS], const u32x4 (&q)[STEPS])
{
    f32x4 x = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) x = mfma_bf16_k32(k[s], q[s], x);
    return x;
}

// First step: every row's statistics over the workgroup's tokens.  What a row's exponents are taken relative to follows its maximum only
// once a product is kSlack (a factor of 2^16) above it: the sum of 2^31 such weights is far inside fp32, and a floating sum does not lose by its scale.
constexpr float kSlack = 16.f;
template <class K>
__global__ __launch_bounds__(kRowWaves * 64, 4) void weight_stats_kernel(WeightArgs a)
{
    constexpr int S = K::kDim / 32;
    __shared__ __attribute__((aligned(16))) char s_pages[2 * kGroupPages * K::kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x / 64;
    const Share share = share_of(a, lane);
    if (share.b < 0) return;   // workgroup-uniform, as all that follow
    const int b = share.b, c = share.c, g = blockIdx.x % a.Hkv;
    const Sequence s = sequence_of(a, b);
    const int rows = s.n * a.G, page0 = c * share.groups * kGroupPages, last = (s.L + kPage - 1) / kPage - 1, n = lane & 15;
    const int first = (blockIdx.x / a.Hkv % a.rounds * waves + wave) * kRowsOfWave;   // the wave's first row
    if (page0 > last || first - wave * kRowsOfWave >= rows) return;   // (L == 0: last is -1)
    const Stream<K> stream(a, b, g, page0, last, min(share.groups, (last - page0) / kGroupPages + 1), s_pages, lane, wave, waves);
    float2 *stats = a.stats + ((int64_t)share.slot * a.Hkv + g) * a.max_rows;
    u32x4 q[kRowTiles][S];
    Stat stat[kRowTiles];
#pragma unroll
    for (int i = 0; i < kRowTiles; ++i) {
        load_q<K>(q[i], a, s, g, first + i * kMaxGroup + n, rows, lane);
        stat[i] = Stat{-INFINITY, 0.f};
    }
    stream.issue(0);
    for (int group = 0; group < stream.groups; ++group) {
        stream.next(group);
        const int t0 = (page0 + group * kGroupPages) * kPage;
        auto tiles = [&](auto masked) {
#pragma unroll
            for (int half = 0; half < kGroupPages; half += kAtOnce) {
                u32x4 k[kAtOnce][S];
                float scale[kAtOnce];
                stream.fetch(group, half, k, scale);
#pragma unroll
                for (int i = 0; i < kRowTiles; ++i) {
                    const int end = masked ? row_end(a, s, first + i * kMaxGroup + n, rows) - t0 - half * kPage - 4 * (lane >> 4) : 0;
                    f32x4 x[kAtOnce];
                    float m = -INFINITY;
#pragma unroll
                    for (int p = 0; p < kAtOnce; ++p) {
                        x[p] = products(k[p], q[i]);
                        if (masked) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) m = fmaxf(m, 16 * p + e < end ? x[p][e] * scale[p] : -INFINITY);
                        } else {
                            m = max_of(m, scale[p] * max_of(max_of(x[p][0], x[p][1]), x[p][2], x[p][3]));
                        }
                    }
                    if (__builtin_amdgcn_ballot_w64(m > stat[i].m + kSlack)) {   // wave-uniform
                        const Stat old = stat[i];
                        stat[i].m = fmaxf(old.m, m);
                        stat[i].l = old.l * shrink_of(old.m, stat[i].m);
                    }
                    const float ref = reference_of(stat[i].m);
#pragma unroll
                    for (int p = 0; p < kAtOnce; ++p)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[p][e], scale[p], -ref));   // (as in the second pass)
                            stat[i].l += !masked || 16 * p + e < end ? w : 0.f;
                        }
                }
            }
        };
        if (first >= rows) continue;   // wave-uniform: rows that are not there
        // every row attends all of these tokens, and of the scores of a page the largest comes from the largest product
        if (t0 + kGroupTokens <= s.base + 1 && !stream.any_below_zero(group)) tiles(std::false_type{});
        else tiles(std::true_type{});
    }
#pragma unroll
    for (int i = 0; i < kRowTiles; ++i) {
        Stat all = stat[i];
        for (int off = 16; off < 64; off *= 2) all = joined(all, Stat{__shfl_xor(all.m, off, 64), __shfl_xor(all.l, off, 64)});
        const int r = first + i * kMaxGroup + n;
        if (lane < 16 && r < rows) stats[r] = float2{all.m, all.l};
    }
}

// Between the steps: every row's statistics over the sequence, four lanes to a row.
__global__ __launch_bounds__(256) void weight_rows_kernel(WeightArgs a)
{
    const int64_t unit = blockIdx.x / a.row_blocks;
    const int r = blockIdx.x % a.row_blocks * 64 + threadIdx.x % 64, slice = threadIdx.x / 64;
    __shared__ Stat s_stat[4][64];
    const Sequence s = sequence_of(a, (int)(unit / a.Hkv));
    const bool there = r < s.n * a.G;
    const Share share = first_share(a, (int)(unit / a.Hkv), threadIdx.x & 63);
    const int tokens = share.groups * kGroupTokens, blocks = (s.L + tokens - 1) / tokens;
    const int64_t step = (int64_t)a.Hkv * a.max_rows;   // from a stretch to the next
    Stat sum = {-INFINITY, 0.f};
    if (there) {
        const float2 *v = a.stats + share.slot * step + unit % a.Hkv * a.max_rows + r;
        for (int c = slice; c < blocks; c += 32) {
            float2 w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = v[min(c + 4 * i, blocks - 1) * step];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + 4 * i < blocks) sum = joined(sum, Stat{w[i].x, w[i].y});
        }
    }
    s_stat[slice][threadIdx.x % 64] = sum;
    __syncthreads();
    if (slice == 0 && there) {
#pragma unroll
        for (int i = 1; i < 4; ++i) sum = joined(sum, s_stat[i][threadIdx.x]);
        a.rows[unit * a.max_rows + r] = float2{sum.m, 1.f / sum.l};
    }
}

// x[p] summed over the four quarters of the wave, each for its own p: lane n + 16 p gets the sum of x[p] over lanes n, n + 16, n + 32, n + 48.
SD_DEV float over_quarters(const float (&x)[4])
{
    const auto bits = [](float f) { return __builtin_bit_cast(unsigned, f); };
    const auto sum = [](auto y) { return __builtin_bit_cast(float, (unsigned)y[0]) + __builtin_bit_cast(float, (unsigned)y[1]); };
    const float u = sum(__builtin_amdgcn_permlane32_swap(bits(x[0]), bits(x[2]), false, false));   // halves: x[0], x[2]
    const float v = sum(__builtin_amdgcn_permlane32_swap(bits(x[1]), bits(x[3]), false, false));   // x[1], x[3]
    return sum(__builtin_amdgcn_permlane16_swap(bits(u), bits(v), false, false));
}

// x of lane k of the wave's quarter that this lane is in (DPP row_newbcast; k a constant, below 8).
SD_DEV float quarter_lane(float x, int k)
{
#define SD_LANE(k) \
    case k: return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x150 + k, 0xf, 0xf, true))
    switch (k) {
        SD_LANE(0);
        SD_LANE(1);
        SD_LANE(2);
        SD_LANE(3);
        SD_LANE(4);
        SD_LANE(5);
        SD_LANE(6);
    default:
        SD_LANE(7);
    }
#undef SD_LANE
}

// Second step: the products once more, rows by tokens, so that a lane's sum runs over four rows of every tile and only the four quarters of the wave are
// left to add; and the weights' sums over the rows.  Grid as in the first.  A row's weights are taken relative to its maximum and multiplied with one over its
// sum, so their error does not grow with the scores; the factors of a lane's eight rows lie in one register of its quarter of the wave (in eight they spill).
template <class K>
__global__ __launch_bounds__(kRowWaves * 64, 4) void weight_apply_kernel(WeightArgs a)
{
    constexpr int S = K::kDim / 32;
    __shared__ __attribute__((aligned(16))) char s_pages[2 * kGroupPages * K::kBytes];
    extern __shared__ float s_sum[];   // [waves][a.block_tokens]: a wave's sums over its rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x / 64;
    const Share share = share_of(a, lane);
    if (share.b < 0) return;   // workgroup-uniform, as the next
    const int b = share.b, c = share.c, g = blockIdx.x % a.Hkv, round = blockIdx.x / a.Hkv % a.rounds;
    const Sequence s = sequence_of(a, b);
    const int rows = s.n * a.G, page0 = c * share.groups * kGroupPages, last = (s.L + kPage - 1) / kPage - 1, n = lane & 15;
    const int first = (round * waves + wave) * kRowsOfWave;
    if (page0 > last || (round && first - wave * kRowsOfWave >= rows)) return;
    const int64_t unit = (int64_t)b * a.Hkv + g;
    const Stream<K> stream(a, b, g, page0, last, min(share.groups, (last - page0) / kGroupPages + 1), s_pages, lane, wave, waves);
    if (rows) {
        u32x4 q[kRowTiles][S];
        float row[kRowTiles][4];   // maxima of rows 4 (lane / 16) .. of each tile
        const int ni = first + n / 4 % kRowTiles * kMaxGroup + 4 * (lane >> 4) + n % 4;
        const float inverse = ni < rows ? a.rows[unit * a.max_rows + ni].y : 0.f;   // of those rows: one each in lanes 0 .. 4 kRowTiles - 1 of the quarter
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) {
            load_q<K>(q[i], a, s, g, first + i * kMaxGroup + n, rows, lane);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = first + i * kMaxGroup + 4 * (lane >> 4) + e;
                row[i][e] = r < rows ? a.rows[unit * a.max_rows + r].x : 0.f;
            }
        }
        stream.issue(0);
        for (int group = 0; group < stream.groups; ++group) {
            stream.next(group);
            const int t0 = (page0 + group * kGroupPages) * kPage;
            float sum[kGroupPages] = {};   // of token n of each page over the lane's rows
            auto tiles = [&](auto masked) {
#pragma unroll
                for (int half = 0; half < kGroupPages; half += kAtOnce) {
                    u32x4 k[kAtOnce][S];
                    float scale[kAtOnce];
                    stream.fetch(group, half, k, scale);
#pragma unroll
                    for (int i = 0; i < kRowTiles; ++i) {
                        int end[4];
                        if (masked)
#pragma unroll
                            for (int e = 0; e < 4; ++e) end[e] = row_end(a, s, first + i * kMaxGroup + 4 * (lane >> 4) + e, rows) - t0 - half * kPage - n;
#pragma unroll
                        for (int p = 0; p < kAtOnce; ++p) {
                            const f32x4 x = products(q[i], k[p]);   // rows by tokens
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], scale[p], -row[i][e])), by = quarter_lane(inverse, 4 * i + e);
                                if (masked) sum[half + p] += 16 * p < end[e] ? w * by : 0.f;
                                else sum[half + p] = __builtin_fmaf(by, w, sum[half + p]);
                            }
                        }
                    }
                }
            };
            if (first < rows) {   // wave-uniform
                // every row is there and attends all of these tokens (one that is not there gives 0 * K, which an infinite K makes NaN)
                if (first + kRowsOfWave <= rows && t0 + kGroupTokens <= s.base + 1) tiles(std::false_type{});
                else tiles(std::true_type{});
            }
            s_sum[wave * a.block_tokens + group * kGroupTokens + lane] = over_quarters(sum);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < stream.groups * kGroupTokens; i += blockDim.x) {
        const int t = page0 * kPage + i;
        if (t >= s.L) break;
        float all = 0.f;
        if (rows)
            for (int w = 0; w < waves; ++w) all += s_sum[w * a.block_tokens + i];
        if (a.rounds > 1) {
            a.parts[((int64_t)round * a.B * a.Hkv + unit) * a.part_stride + t] = all;
            continue;
        }
        const int64_t at = unit * a.score_stride + t;
        a.scores_out[at] = all + (a.scores_in && t < s.L - a.new_tokens ? a.decay * a.scores_in[at] : 0.f);
    }
}

// Where the rows take several rounds: their sums, four tokens to a thread.
__global__ __launch_bounds__(256) void weight_join_kernel(WeightArgs a)
{
    const int64_t unit = blockIdx.x / a.apply_blocks;
    const int t0 = blockIdx.x % a.apply_blocks * kApplyTokens + 4 * threadIdx.x;
    const Sequence s = sequence_of(a, (int)(unit / a.Hkv));
    if (t0 >= s.L) return;
    f32x4 sum = {0, 0, 0, 0};
    for (int first = 0, round = 0; first < s.n * a.G; first += row_waves(a.max_rows) * kRowsOfWave, ++round)
        sum += *reinterpret_cast<const f32x4 *>(a.parts + ((int64_t)round * a.B * a.Hkv + unit) * a.part_stride + t0);
    const int64_t at = unit * a.score_stride + t0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (t0 + e < s.L) a.scores_out[at + e] = sum[e] + (a.scores_in && t0 + e < s.L - a.new_tokens ? a.decay * a.scores_in[at + e] : 0.f);
}

template <class K>
static void launch_streamed(const WeightArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.share ? a.share : (int64_t)a.B * a.blocks * a.Hkv * a.rounds)), block(row_waves(a.max_rows) * 64);
    hipLaunchKernelGGL(weight_stats_kernel<K>, grid, block, 0, stream, a);
    if (a.row_blocks) hipLaunchKernelGGL(weight_rows_kernel, dim3((unsigned)((int64_t)a.B * a.Hkv * a.row_blocks)), dim3(256), 0, stream, a);
    hipLaunchKernelGGL(weight_apply_kernel<K>, grid, block, block.x / 64 * a.block_tokens * 4, stream, a);
    if (a.rounds > 1) hipLaunchKernelGGL(weight_join_kernel, dim3((unsigned)((int64_t)a.B * a.Hkv * a.apply_blocks)), dim3(256), 0, stream, a);
}

template <class K, int PACK>
static void launch_kept(const WeightArgs &a, hipStream_t stream)
{
    if (a.whole_waves) {
        hipLaunchKernelGGL((weight_whole_kernel<K, PACK>), dim3((unsigned)((int64_t)a.B * a.Hkv)), dim3(a.whole_waves * 64), a.whole_waves * 2 * K::kBytes, stream, a);
        return;
    }
    hipLaunchKernelGGL((weight_products_kernel<K, PACK>), dim3((unsigned)((int64_t)a.B * a.blocks * a.Hkv)), dim3(kWaves * 64), 0, stream, a);
    hipLaunchKernelGGL(weight_apply_kept_kernel<PACK>, dim3((unsigned)((int64_t)a.B * a.apply_blocks * a.Hkv)), dim3(256), 0, stream, a);
}

template <class K>
static hipError_t launch_weights_of(const WeightArgs &a, int pack, hipStream_t stream)
{
    if (pack == 4) launch_kept<K, 4>(a, stream);
    else if (pack == 2) launch_kept<K, 2>(a, stream);
    else if (pack == 1) launch_kept<K, 1>(a, stream);
    else launch_streamed<K>(a, stream);
    return hipGetLastError();
}

hipError_t launch_weights(const WeightArgs &a, int pack, int head_dim, int kv_dtype, hipStream_t stream)
{
    if (kv_dtype == 0 && head_dim == 128) return launch_weights_of<Bf16Rows<128>>(a, pack, stream);
    if (kv_dtype == 0 && head_dim == 64) return launch_weights_of<Bf16Rows<64>>(a, pack, stream);
    if (kv_dtype == 1 && head_dim == 128) return launch_weights_of<Fp8Rows<128>>(a, pack, stream);
    if (kv_dtype == 1 && head_dim == 64) return launch_weights_of<Fp8Rows<64>>(a, pack, stream);
    return hipErrorNotSupported;
}

}  // namespace sd
