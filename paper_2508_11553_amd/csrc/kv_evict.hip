// Cutting a cache down: which tokens of a (sequence, KV head) stay, and their move into new pages.
//
// Select: one workgroup per (sequence, KV head).  The first `sinks` and the last `recent` tokens stay; of those between, the `want`
// with the largest scores.  The want-th largest score is found digit by digit (11, 11 and 10 bits of a key that orders as the
// scores do): a histogram of the digit over the keys that agree so far, and the digit at which the count from above reaches
// `want`.  Then one walk over the tokens in order numbers those that stay: all above that score, and of those equal to it the first.
// Whole numbers throughout, so nothing depends on an order of additions.
//
// Move: a wave per (new page, KV head): 16 positions, their rows of K and V from wherever they lie, stored as one tile.  Bound by memory.
// fp8: a new tile's scale is the largest of its rows' old scales, so a row from the tile of that scale keeps its codes and
// no other row can overflow; e4m3 codes are floating point, so a smaller row loses nothing but what falls below the smallest exponent.
#include <climits>

#include "attn_tile.h"

namespace sd {

namespace {

constexpr int kSelectThreads = 1024;
constexpr int kBins = 2048;

// Keys order as scores do: NaN below everything, the two zeros equal.
SD_DEV unsigned key_of(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x == 0.f ? 0.f : x);
    return x != x ? 0u : u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
}

// Sum over a workgroup's threads before this one, and over all of them; two counts in the halves of a word pair.
struct Before {
    int before, all;
};
SD_DEV Before before_in_workgroup(int x, int *s_wave, int lane, int wave)
{
    const int upto = wave_scan(x);
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSelectThreads / 64; ++w) {
        const int n = s_wave[w];
        before += w < wave ? n : 0;
        all += n;
    }
    __syncthreads();
    return Before{before + upto - x, all};
}

}  // namespace

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a)
{
    __shared__ int s_bins[kBins];
    __shared__ int s_wave[kSelectThreads / 64];
    __shared__ int s_found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t unit = blockIdx.x;
    const int L = max(0, min(a.context_lens[unit / a.Hkv], a.max_context_len));
    const float *scores = a.scores + unit * a.score_stride;
    int32_t *kept = a.kept + unit * a.budget;
    const int stay = min(L, a.budget);
    const int lo = a.sinks, hi = L - a.recent;   // those between are chosen from
    unsigned bound = 0;                          // key of the last one that stays
    int ties = 0;                                // how many of that key stay
    const int want = a.budget - a.sinks - a.recent;
    const bool cut = L > a.budget;
    if (cut && want > 0) {
        int left = want;
        const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            for (int i = tid; i < kBins; i += kSelectThreads) s_bins[i] = 0;
            __syncthreads();
            for (int t = lo + tid; t < hi; t += kSelectThreads) {
                const unsigned key = key_of(scores[t]);
                if (pass == 0 || key >> (shifts[pass] + bits[pass]) == bound >> (shifts[pass] + bits[pass]))
                    atomicAdd(&s_bins[key >> shifts[pass] & ((1 << bits[pass]) - 1)], 1);
            }
            __syncthreads();
            // thread i holds bins 2 i and 2 i + 1 counted from the top
            const int top = (1 << bits[pass]) - 1, b0 = top - 2 * tid, b1 = b0 - 1;
            const int n0 = b0 >= 0 ? s_bins[b0] : 0, n1 = b1 >= 0 ? s_bins[b1] : 0;
            const int above = before_in_workgroup(n0 + n1, s_wave, lane, wave).before;
            if (above < left && left <= above + n0) s_found[0] = b0, s_found[1] = left - above;
            else if (above + n0 < left && left <= above + n0 + n1) s_found[0] = b1, s_found[1] = left - above - n0;
            __syncthreads();
            bound |= (unsigned)s_found[0] << shifts[pass];
            left = s_found[1];
            __syncthreads();
        }
        ties = left;
    }
    // in order; with nothing to cut all stay
    int more = 0, equal = 0;   // so far: above the bound (or kept anyway), equal to it
    for (int base = 0; base < L; base += kSelectThreads) {
        const int t = base + tid;
        const float x = t < L ? scores[t] : 0.f;
        const unsigned key = key_of(x);
        const bool always = t < L && (!cut || t < lo || t >= hi);
        const bool over = always || (t < L && want > 0 && key > bound), tie = !always && t < L && want > 0 && key == bound;
        const Before n = before_in_workgroup((int)over | (int)tie << 16, s_wave, lane, wave);
        const int m = more + (n.before & 0xffff), e = equal + (n.before >> 16);
        if (over || (tie && e < ties)) {
            const int to = m + min(e, ties);
            kept[to] = t;
            if (a.scores_out) a.scores_out[unit * a.scores_out_stride + to] = x;
        }
        more += n.all & 0xffff;
        equal += n.all >> 16;
    }
    for (int i = stay + tid; i < a.budget; i += kSelectThreads) kept[i] = -1;
}

// Rows of K and V of one new (page, head) tile by one wave.
template <int ROW_BYTES>
SD_DEV void move_rows(const char *pool, char *to, const int64_t from, int n, int lane)
{
    constexpr int kLanes = ROW_BYTES / 16, kAtOnce = 64 / kLanes;
    u32x4 x[kPage / kAtOnce];
#pragma unroll
    for (int i = 0; i < kPage / kAtOnce; ++i) {
        const int r = i * kAtOnce + lane / kLanes;
        const int64_t at = __shfl(from, r, 64);
        if (r < n) x[i] = kv_load<true>(reinterpret_cast<const u32x4 *>(pool + at * ROW_BYTES + lane % kLanes * 16));
    }
#pragma unroll
    for (int i = 0; i < kPage / kAtOnce; ++i) {
        const int r = i * kAtOnce + lane / kLanes;
        if (r < n) *reinterpret_cast<u32x4 *>(to + r * ROW_BYTES + lane % kLanes * 16) = x[i];
    }
}

// The same with codes and scales.
template <int D>
SD_DEV void move_codes(const char *pool, char *to, const float *scales, float *new_scale, const int64_t from, int n, int lane)
{
    constexpr int kLanes = D / 16, kAtOnce = 64 / kLanes;
    const float old = (lane & 15) < n ? scales[from / kPage] : 0.f;
    float top = old;
    for (int off = 1; off < 16; off *= 2) top = fmaxf(top, __shfl_xor(top, off, 64));
    const float ratio = top > 0.f ? old / top : 1.f;
    u32x4 x[kPage / kAtOnce];
#pragma unroll
    for (int i = 0; i < kPage / kAtOnce; ++i) {
        const int r = i * kAtOnce + lane / kLanes;
        const int64_t at = __shfl(from, r, 64);
        if (r < n) x[i] = kv_load<true>(reinterpret_cast<const u32x4 *>(pool + at * D + lane % kLanes * 16));
    }
#pragma unroll
    for (int i = 0; i < kPage / kAtOnce; ++i) {
        const int r = i * kAtOnce + lane / kLanes;
        const float by = __shfl(ratio, r, 64);
        if (r >= n) continue;
        if (by != 1.f)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const f32x2 u = __builtin_amdgcn_cvt_pk_f32_fp8(x[i][w], false), v = __builtin_amdgcn_cvt_pk_f32_fp8(x[i][w], true);
                const unsigned y = __builtin_amdgcn_cvt_pk_fp8_f32(u[0] * by, u[1] * by, 0, false);
                x[i][w] = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * by, v[1] * by, y, true);
            }
        *reinterpret_cast<u32x4 *>(to + r * D + lane % kLanes * 16) = x[i];
    }
    if (lane == 0) *new_scale = top;
}

template <int D, bool FP8>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a)
{
    constexpr int kRow = FP8 ? D : 2 * D;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);   // (sequence, new page, head), head fastest
    const int64_t page_item = item / a.Hkv;
    const int g = (int)(item - page_item * a.Hkv), b = (int)(page_item / a.new_pages), j = (int)(page_item - (int64_t)b * a.new_pages);
    if (b >= a.B) return;
    const int stay = max(0, min(min(a.context_lens[b], a.max_context_len), a.budget));
    if (g == 0 && j == 0 && lane == 0) a.new_lens[b] = stay;   // (new_lens may be context_lens: the smaller of it and the budget stays the same)
    const int n = min(kPage, stay - j * kPage);
    if (n <= 0) return;
    const int t = a.kept[((int64_t)b * a.Hkv + g) * a.budget + j * kPage + min(lane & 15, n - 1)];
    const int64_t from = ((int64_t)a.block_table[(int64_t)b * a.max_blocks + t / kPage] * a.Hkv + g) * kPage + t % kPage;   // row of the pool
    const int64_t tile = (int64_t)a.new_table[(int64_t)b * a.max_blocks + j] * a.Hkv + g;
    char *k = static_cast<char *>(a.k_pages), *v = static_cast<char *>(a.v_pages);
    if (FP8) {
        move_codes<D>(k, k + tile * kPage * kRow, a.k_scales, a.k_scales + tile, from, n, lane);
        move_codes<D>(v, v + tile * kPage * kRow, a.v_scales, a.v_scales + tile, from, n, lane);
    } else {
        move_rows<kRow>(k, k + tile * kPage * kRow, from, n, lane);
        move_rows<kRow>(v, v + tile * kPage * kRow, from, n, lane);
    }
}

hipError_t launch_evict(const EvictArgs &a, int head_dim, int kv_dtype, hipStream_t stream)
{
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)(a.B * a.Hkv)), dim3(kSelectThreads), 0, stream, a);
    const dim3 grid((unsigned)(((int64_t)a.B * a.new_pages * a.Hkv + 3) / 4)), block(256);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    if (kv_dtype == 0 && head_dim == 128) go(evict_move_kernel<128, false>);
    else if (kv_dtype == 0 && head_dim == 64) go(evict_move_kernel<64, false>);
    else if (kv_dtype == 1 && head_dim == 128) go(evict_move_kernel<128, true>);
    else if (kv_dtype == 1 && head_dim == 64) go(evict_move_kernel<64, true>);
    else return hipErrorNotSupported;
    return hipGetLastError();
}

}  // namespace sd
