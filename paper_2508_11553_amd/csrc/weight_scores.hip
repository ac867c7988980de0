// The attention weight that every cached token receives, added to its running score:
//
//   s'[b][g][t] = decay s[b][g][t] + sum_rows softmax_t(scale <q_row, K_t>)      rows: the query rows of sequence b, heads of KV head g
//
// A weight needs its row's maximum and sum over all tokens, so there are two steps: one pass over K that makes the
// products and leaves every chunk's (max, sum) for each row, and one over the tokens that turns products into weights.
// The products of one tile of 16 query rows (a decode step: the heads of a KV head) are kept in fp32 between the two,
// rows * 4 bytes a token, a small part of K's 64 to 256; with more rows (the last tokens of a prompt) K is read again, from
// the caches or memory, and multiplied again.
//
//   S[token][row] = K_page[token][d] . Q^T[d][row]     mfma 16x16x32 bf16, a page of 16 tokens at a time
//
// A lane holds four tokens (4 (lane / 16) ..) of row lane % 16.  K goes from memory straight into operand layout: lane n + 16 c
// reads 16 bytes of token n; which d these are differs between pools, and Q is read in the same order.
// Weights, sums and scores are fp32 throughout.
#include "attn_tile.h"

namespace sd {

namespace {

constexpr int kScorePages = 4;   // pages in a wave's registers at a time

// One page of K as the first operand: lane n + 16 c holds token n.
template <int D>
struct Bf16Rows {
    static constexpr int kDim = D;
    static constexpr int kBytes = kPage * D * 2;
    static constexpr bool kScaled = false;
    u32x4 k[D / 32];
    SD_DEV static int q_offset(int s, int c) { return 32 * s + 8 * c; }
    template <bool STREAM>
    SD_DEV void load(const char *page, int lane)
    {
        const char *p = page + (lane & 15) * (D * 2) + (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) k[s] = kv_load<STREAM>(reinterpret_cast<const u32x4 *>(p + s * 64));
    }
    SD_DEV u32x4 operand(int s) const { return k[s]; }
};
template <int D>
struct Fp8Rows {
    static constexpr int kDim = D;
    static constexpr int kBytes = kPage * D;
    static constexpr bool kScaled = true;
    u32x4 k[D / 64];   // 16 codes each
    SD_DEV static int q_offset(int s, int c) { return 64 * (s / 2) + 16 * c + 8 * (s % 2); }
    template <bool STREAM>
    SD_DEV void load(const char *page, int lane)
    {
        const char *p = page + (lane & 15) * D + (lane >> 4) * 16;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) k[j] = kv_load<STREAM>(reinterpret_cast<const u32x4 *>(p + j * 64));
    }
    SD_DEV u32x4 operand(int s) const
    {
        const unsigned lo = k[s / 2][2 * (s % 2)], hi = k[s / 2][2 * (s % 2) + 1];
        return u32x4{cvt_pk_bf16_fp8<false>(lo), cvt_pk_bf16_fp8<true>(lo), cvt_pk_bf16_fp8<false>(hi), cvt_pk_bf16_fp8<true>(hi)};
    }
};

// What a workgroup knows of its sequence.
struct Sequence {
    int L, first_q, n;   // tokens, first query row, query rows of it
};
SD_DEV Sequence sequence_of(const WeightArgs &a, int b)
{
    Sequence s;
    s.L = max(0, min(a.context_lens[b], a.max_context_len));
    s.first_q = b;
    s.n = 1;
    if (a.q_start) {
        const int q0 = a.q_start[b], q1 = a.q_start[b + 1];
        const bool inside = q0 >= 0 && q1 <= a.total_q && q1 > q0;   // a range that leaves the rows has none
        s.first_q = inside ? q0 : 0;
        s.n = inside ? min(q1 - q0, a.max_q_len) : 0;
    }
    return s;
}

// Row r of (sequence, KV head): query r / G, head r % G of the group.
template <class K>
SD_DEV void load_q(u32x4 (&q)[K::kDim / 32], const WeightArgs &a, const Sequence &s, int g, int r, int rows, int lane)
{
    const int i = (int)a.per_group.of(r);
    const uint16_t *p = a.q + ((int64_t)(s.first_q + i) * a.Hq + g * a.G + (r - i * a.G)) * K::kDim;
#pragma unroll
    for (int j = 0; j < K::kDim / 32; ++j)
        q[j] = r < rows ? *reinterpret_cast<const u32x4 *>(p + K::q_offset(j, lane >> 4)) : u32x4{0, 0, 0, 0};
}

// The tokens that row r attends: those before `end`.
SD_DEV int row_end(const WeightArgs &a, const Sequence &s, int r, int rows) { return r < rows ? min(s.L, s.L - s.n + 1 + (int)a.per_group.of(r)) : 0; }

template <class K>
SD_DEV f32x4 products(const K &k, const u32x4 (&q)[K::kDim / 32], float scale)
{
    f32x4 x = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < K::kDim / 32; ++s) x = mfma_bf16_k32(k.operand(s), q[s], x);
    return x * scale;
}

// The pages of tiles [first, first + kScorePages) of a sequence; pages past the last one repeat it (their tokens are masked).
template <class K, bool STREAM>
SD_DEV void load_pages(K (&k)[kScorePages], float (&scale)[kScorePages], const WeightArgs &a, ConstTable bt, int g, int first, int last, int lane)
{
#pragma unroll
    for (int i = 0; i < kScorePages; ++i) {
        const int64_t at = (int64_t)bt[min(first + i, last)] * a.Hkv + g;
        k[i].template load<STREAM>(static_cast<const char *>(a.k_pages) + at * K::kBytes, lane);
        scale[i] = K::kScaled ? ((ConstScales)a.k_scales)[at] * a.scale_log2e : a.scale_log2e;
    }
}

struct Stat {
    float m, l;   // running maximum (log2 domain) and sum of exp2(x - m)
};
SD_DEV float shrink_of(float from, float to) { return from == to ? 1.f : __builtin_amdgcn_exp2f(from - to); }   // (both may be -inf)
SD_DEV Stat joined(Stat x, Stat y)
{
    const float m = fmaxf(x.m, y.m);
    return Stat{m, x.l * shrink_of(x.m, m) + y.l * shrink_of(y.m, m)};
}
SD_DEV Stat over_lanes(Stat s, int from, int to)
{
    for (int off = from; off < to; off *= 2) s = joined(s, Stat{__shfl_xor(s.m, off, 64), __shfl_xor(s.l, off, 64)});
    return s;
}

// x of four tokens (t0 ..), those before `end` attended: into the lane's statistics.
SD_DEV void take(Stat &s, const f32x4 (&x)[kScorePages], int t0, int end)
{
    float m = s.m;
#pragma unroll
    for (int i = 0; i < kScorePages; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = t0 + 16 * i + e < end ? fmaxf(m, x[i][e]) : m;
    s.l *= shrink_of(s.m, m);
    s.m = m;
#pragma unroll
    for (int i = 0; i < kScorePages; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s.l += t0 + 16 * i + e < end ? __builtin_amdgcn_exp2f(x[i][e] - m) : 0.f;
}

}  // namespace

// First step: workgroup (sequence, chunk, KV head), KV head fastest; its waves take the chunk's pages in turn, kScorePages at a time.
// KEEP: one tile of rows, whose products are kept.
template <class K, bool KEEP>
__global__ __launch_bounds__(kWaves * 64) void weight_stats_kernel(WeightArgs a)
{
    __shared__ Stat s_stat[kWaves][kMaxGroup];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.x % a.Hkv, c = blockIdx.x / a.Hkv % a.chunks, b = blockIdx.x / a.Hkv / a.chunks;
    const Sequence s = sequence_of(a, b);
    const int rows = s.n * a.G, page0 = c * a.chunk_pages, last = (s.L + kPage - 1) / kPage - 1;
    if (page0 > last || rows == 0) return;   // workgroup-uniform
    const int page1 = min(last + 1, page0 + a.chunk_pages), n = lane & 15;
    const ConstTable bt = (ConstTable)(a.block_table + (int64_t)b * a.max_blocks);
    const int64_t unit = (int64_t)b * a.Hkv + g;
    for (int r0 = 0; r0 < rows; r0 += kMaxGroup) {   // (one round with KEEP)
        u32x4 q[K::kDim / 32];
        load_q<K>(q, a, s, g, r0 + n, rows, lane);
        const int end = row_end(a, s, r0 + n, rows);
        Stat stat = {-INFINITY, 0.f};
        for (int p = page0 + wave * kScorePages; p < page1; p += kWaves * kScorePages) {
            K k[kScorePages];
            float scale[kScorePages];
            load_pages<K, KEEP>(k, scale, a, bt, g, p, last, lane);
            f32x4 x[kScorePages];
#pragma unroll
            for (int i = 0; i < kScorePages; ++i) x[i] = products(k[i], q, scale[i]);
            take(stat, x, p * kPage + 4 * (lane >> 4), end);
            if (KEEP && n < rows) {   // [page][row][token]
                float *to = a.products + ((unit * a.max_pages + p) * a.max_rows + n) * kPage + 4 * (lane >> 4);
#pragma unroll
                for (int i = 0; i < kScorePages; ++i)
                    if (p + i < page1) *reinterpret_cast<f32x4 *>(to + (int64_t)i * a.max_rows * kPage) = x[i];
            }
        }
        stat = over_lanes(stat, 16, 64);
        if (lane < 16) s_stat[wave][n] = stat;
        __syncthreads();
        if (threadIdx.x < 16 && r0 + n < rows) {
            Stat all = s_stat[0][n];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) all = joined(all, s_stat[w][n]);
            a.stats[(unit * a.chunks + c) * a.max_rows + r0 + n] = float2{all.m, all.l};
        }
        __syncthreads();
    }
}

// The statistics of a row over the sequence's chunks -> (max, 1 / sum), by one wave.
SD_DEV float2 whole_row(const WeightArgs &a, int64_t unit, int r, int chunks, int lane)
{
    Stat s = {-INFINITY, 0.f};
    for (int c = lane; c < chunks; c += 64) {
        const float2 v = a.stats[(unit * a.chunks + c) * a.max_rows + r];
        s = joined(s, Stat{v.x, v.y});
    }
    s = over_lanes(s, 1, 64);
    return float2{s.m, 1.f / s.l};
}

// Second step after KEEP: four tokens to a thread, 1024 to a workgroup.
__global__ __launch_bounds__(256) void weight_apply_kept_kernel(WeightArgs a)
{
    __shared__ float2 s_row[kMaxGroup];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int g = blockIdx.x % a.Hkv, j = blockIdx.x / a.Hkv % a.apply_blocks, b = blockIdx.x / a.Hkv / a.apply_blocks;
    const Sequence s = sequence_of(a, b);
    if (j * 1024 >= s.L) return;
    const int64_t unit = (int64_t)b * a.Hkv + g;
    const int rows = s.n * a.G, chunks = (s.L + a.chunk_pages * kPage - 1) / (a.chunk_pages * kPage);
    for (int r = wave; r < rows; r += 4) {
        const float2 v = whole_row(a, unit, r, chunks, lane);
        if (lane == 0) s_row[r] = v;
    }
    __syncthreads();
    const int t0 = j * 1024 + threadIdx.x * 4;
    if (t0 >= s.L) return;
    const float *x = a.products + ((unit * a.max_pages + t0 / kPage) * a.max_rows) * kPage + t0 % kPage;
    f32x4 sum = {0, 0, 0, 0};
    for (int r = 0; r < rows; ++r) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(x + r * kPage);
        const float2 row = s_row[r];
        const int end = row_end(a, s, r, rows);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += t0 + e < end ? __builtin_amdgcn_exp2f(v[e] - row.x) * row.y : 0.f;
    }
    const int64_t at = unit * a.score_stride + t0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (t0 + e < s.L) a.scores_out[at + e] = sum[e] + (a.scores_in && t0 + e < s.L - a.new_tokens ? a.decay * a.scores_in[at + e] : 0.f);
}

// Between the steps otherwise: every row's statistics once.
__global__ __launch_bounds__(256) void weight_rows_kernel(WeightArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = blockIdx.x;
    const Sequence s = sequence_of(a, (int)(unit / a.Hkv));
    const int chunks = (s.L + a.chunk_pages * kPage - 1) / (a.chunk_pages * kPage);
    for (int r = threadIdx.x >> 6; r < s.n * a.G; r += 4) {
        const float2 v = whole_row(a, unit, r, chunks, lane);
        if (lane == 0) a.rows[unit * a.max_rows + r] = v;
    }
}

// Second step with the products made again: grid as the first step's.
template <class K>
__global__ __launch_bounds__(kWaves * 64) void weight_apply_kernel(WeightArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.x % a.Hkv, c = blockIdx.x / a.Hkv % a.chunks, b = blockIdx.x / a.Hkv / a.chunks;
    const Sequence s = sequence_of(a, b);
    const int rows = s.n * a.G, page0 = c * a.chunk_pages, last = (s.L + kPage - 1) / kPage - 1;
    if (page0 > last) return;
    const int page1 = min(last + 1, page0 + a.chunk_pages), n = lane & 15;
    const ConstTable bt = (ConstTable)(a.block_table + (int64_t)b * a.max_blocks);
    const int64_t unit = (int64_t)b * a.Hkv + g;
    for (int p = page0 + wave * kScorePages; p < page1; p += kWaves * kScorePages) {
        K k[kScorePages];
        float scale[kScorePages];
        load_pages<K, false>(k, scale, a, bt, g, p, last, lane);
        f32x4 sum[kScorePages];
#pragma unroll
        for (int i = 0; i < kScorePages; ++i) sum[i] = f32x4{0, 0, 0, 0};
        const int t0 = p * kPage + 4 * (lane >> 4);
        for (int r0 = 0; r0 < rows; r0 += kMaxGroup) {
            u32x4 q[K::kDim / 32];
            load_q<K>(q, a, s, g, r0 + n, rows, lane);
            const int end = row_end(a, s, r0 + n, rows);
            const float2 row = a.rows[unit * a.max_rows + min(r0 + n, rows - 1)];
#pragma unroll
            for (int i = 0; i < kScorePages; ++i) {
                const f32x4 x = products(k[i], q, scale[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[i][e] += t0 + 16 * i + e < end ? __builtin_amdgcn_exp2f(x[e] - row.x) * row.y : 0.f;
            }
        }
        // over the rows of the tile: the 16 lanes of a group hold the same tokens
#pragma unroll
        for (int i = 0; i < kScorePages; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                for (int off = 1; off < 16; off *= 2) sum[i][e] += __shfl_xor(sum[i][e], off, 64);
        // lane n of a group stores token n % 4 of page n / 4
        const int t = t0 + 16 * (n / 4) + n % 4;
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < kScorePages; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine = n == 4 * i + e ? sum[i][e] : mine;
        if (t < min(s.L, page1 * kPage)) {
            const int64_t at = unit * a.score_stride + t;
            a.scores_out[at] = mine + (a.scores_in && t < s.L - a.new_tokens ? a.decay * a.scores_in[at] : 0.f);
        }
    }
}

template <class K>
static hipError_t launch_weights_of(const WeightArgs &a, bool keep, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.B * a.chunks * a.Hkv)), block(kWaves * 64);
    if (keep) {
        hipLaunchKernelGGL((weight_stats_kernel<K, true>), grid, block, 0, stream, a);
        hipLaunchKernelGGL(weight_apply_kept_kernel, dim3((unsigned)((int64_t)a.B * a.apply_blocks * a.Hkv)), dim3(256), 0, stream, a);
    } else {
        hipLaunchKernelGGL((weight_stats_kernel<K, false>), grid, block, 0, stream, a);
        hipLaunchKernelGGL(weight_rows_kernel, dim3((unsigned)(a.B * a.Hkv)), dim3(256), 0, stream, a);
        hipLaunchKernelGGL(weight_apply_kernel<K>, grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

hipError_t launch_weights(const WeightArgs &a, bool keep, int head_dim, int kv_dtype, hipStream_t stream)
{
    if (kv_dtype == 0 && head_dim == 128) return launch_weights_of<Bf16Rows<128>>(a, keep, stream);
    if (kv_dtype == 0 && head_dim == 64) return launch_weights_of<Bf16Rows<64>>(a, keep, stream);
    if (kv_dtype == 1 && head_dim == 128) return launch_weights_of<Fp8Rows<128>>(a, keep, stream);
    if (kv_dtype == 1 && head_dim == 64) return launch_weights_of<Fp8Rows<64>>(a, keep, stream);
    return hipErrorNotSupported;
}

}  // namespace sd
