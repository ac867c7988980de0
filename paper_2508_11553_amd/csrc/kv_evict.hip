// Cutting a cache down: which tokens of a (sequence, KV head) stay, and their move into new pages.
//
// Select: one workgroup per (sequence, KV head).  The first `sinks` and the last `recent` tokens stay; of those between, the `want`
// with the largest scores.  The want-th largest score is found digit by digit (11, 11 and 10 bits of a key that orders as the
// scores do): a histogram of the digit over the keys that agree so far, and the digit at which the count from above reaches
// `want`.  Then one walk over the tokens in order numbers those that stay: all above that score, and of those equal to it the first.
// Whole numbers throughout, so nothing depends on an order of additions.
//
// Move: a wave per (new page, KV head): 16 positions, their rows of K and V from wherever they lie, stored as one tile.  Bound by memory.
// fp8: a new tile's scale is the largest magnitude of its rows' old scales, so a row from the tile of that scale keeps its codes (or turns their signs) and
// no other row can overflow; e4m3 codes are floating point, so a smaller row loses nothing but what falls below the smallest exponent.
//
// Measured (d = 128): 256 sequences and heads of 2 k - 64 k, bf16, 4096 stay: choice 40 us (one workgroup's walk over 64 k: load 14, digits 13, places 13),
// move 207 us of 1.04 GB, 5.0 TB/s read and written, a copy's 4.9; 1600 of 1.5 k - 4 k, fp8, 1500 stay: 26 and 245 us (1.29 GB, 5.2 TB/s);
// 12 of about 1.2 k 7 and 4 us, two launches.
#include "attn_tile.h"

namespace sd {

namespace {

constexpr int kBins = 2048;
constexpr int kCopies = 4;   // of every bin, one to each lane of four: scores crowd into few bins, and additions to one address wait for each other

// Keys order as scores do: NaN below everything, the two zeros equal.
SD_DEV unsigned key_of(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x == 0.f ? 0.f : x);
    return x != x ? 0u : u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
}

}  // namespace

// THREADS: of a workgroup; HELD: keys in a thread's registers, in fours.  Scores are read once for the choice where the registers hold
// all of the sequence's keys, else once a pass.
template <int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a)
{
    constexpr int kWavesHere = THREADS / 64, kBlock = 4 * THREADS, kChunk = HELD * kBlock, kPer = kBins / THREADS;
    __shared__ int4 s_bins[kBins];   // kCopies each
    __shared__ int s_wave[kWavesHere];
    __shared__ int s_found[2];
    __shared__ int2 s_count[HELD * kWavesHere];   // of the tokens of a wave in a block: those above the bound, those equal to it
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t unit = blockIdx.x;
    const int L = max(0, min(a.context_lens[unit / a.Hkv], a.max_context_len));
    const float *scores = a.scores + unit * a.score_stride;
    float *scores_out = a.scores_out ? a.scores_out + unit * a.scores_out_stride : nullptr;
    int32_t *kept = a.kept + unit * a.budget;
    const int stay = min(L, a.budget);
    const bool cut = L > a.budget;
    const int lo = cut ? a.sinks : L, hi = cut ? L - a.recent : L;   // those between are chosen from (with nothing to cut all stay)
    auto four = [&](int t) { return t < L ? *reinterpret_cast<const f32x4 *>(scores + t) : f32x4{0, 0, 0, 0}; };   // (a row's stride is a multiple of four)
    // Keys: of tokens that stay anyway the largest, which no score has; of tokens past the end the smallest, which come last among equals.
    unsigned key[HELD][4];
    auto load = [&](int chunk0) {
        constexpr int kAhead = HELD < 8 ? HELD : 8;   // loads on their way at a time
#pragma unroll
        for (int i0 = 0; i0 < HELD; i0 += kAhead) {
            f32x4 x[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (chunk0 + (i0 + i) * kBlock < L) x[i] = four(chunk0 + (i0 + i) * kBlock + 4 * tid);   // workgroup-uniform
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (chunk0 + (i0 + i) * kBlock < L)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = chunk0 + (i0 + i) * kBlock + 4 * tid + e;
                        key[i0 + i][e] = t >= L ? 0u : t < lo || t >= hi ? ~0u : key_of(x[i][e]);
                    }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    load(0);
    unsigned bound = 0;   // key of the last one that stays
    int ties = 0;         // how many of that key stay
    if (cut) {
        int left = a.budget;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};
            const int shift = kShift[pass], bits = kBits[pass];
            for (int i = tid; i < kBins; i += THREADS) s_bins[i] = int4{0, 0, 0, 0};
            int *bins = &s_bins[0].x + lane % kCopies;
            __syncthreads();
            for (int chunk0 = 0; chunk0 < L; chunk0 += kChunk) {
                if (L > kChunk) load(chunk0);
#pragma unroll
                for (int i = 0; i < HELD; ++i) {
                    if (chunk0 + i * kBlock >= L) break;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int bin = __builtin_amdgcn_ubfe(key[i][e], shift, bits);
                        if (pass == 0) {
                            // (one addition where all lanes agree, as they do where no token has any weight)
                            const int first = __builtin_amdgcn_readfirstlane(bin);
                            if (__builtin_amdgcn_ballot_w64(bin != first) == 0) {
                                if (lane == 0) atomicAdd(&bins[first * kCopies], 64);
                            } else {
                                atomicAdd(&bins[bin * kCopies], 1);
                            }
                        } else if ((key[i][e] ^ bound) >> (shift + bits) == 0) {
                            atomicAdd(&bins[bin * kCopies], 1);
                        }
                    }
                }
            }
            __syncthreads();
            // thread i holds bins kPer i .. counted from the top
            int n[kPer], sum = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int4 c = s_bins[kBins - 1 - (kPer * tid + i)];
                n[i] = c.x + c.y + c.z + c.w;
                sum += n[i];
            }
            const int upto = wave_scan(sum);
            if (lane == 63) s_wave[wave] = upto;
            __syncthreads();
            int above = upto - sum;
#pragma unroll
            for (int w = 0; w < kWavesHere; ++w) above += w < wave ? s_wave[w] : 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (above < left && left <= above + n[i]) s_found[0] = kBins - 1 - (kPer * tid + i), s_found[1] = left - above;
                above += n[i];
            }
            __syncthreads();
            bound |= (unsigned)s_found[0] << shift;
            left = s_found[1];
        }
        ties = left;
    }
    // The places of those that stay: counted by waves and blocks of tokens, then added up in the tokens' order.
    const bool in_place = scores_out == scores;
    int more = 0, equal = 0;   // in the chunks so far
    for (int chunk0 = 0; chunk0 < L; chunk0 += kChunk) {
        if (L > kChunk) load(chunk0);
        unsigned before[HELD / 2] = {};   // in the wave before this thread's tokens of a block: above and equal, eight bits each (at most 252)
        __syncthreads();     // the last chunk's readers
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            if (chunk0 + i * kBlock >= L) break;
            int mine = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) mine += key[i][e] > bound ? 1 : key[i][e] == bound ? 0x10000 : 0;
            const int upto = wave_scan(mine);
            const unsigned b = upto - mine;
            before[i / 2] |= ((b & 0xff) | (b >> 8 & 0xff00)) << 16 * (i % 2);
            if (lane == 63) s_count[i * kWavesHere + wave] = int2{upto & 0xffff, upto >> 16};
        }
        __syncthreads();
        if (wave == 0) {   // exclusive sums over the chunk's counts, in the tokens' order
            constexpr int kCounts = HELD * kWavesHere, kPerLane = (kCounts + 63) / 64;
            const int blocks = min(HELD, (L - chunk0 + kBlock - 1) / kBlock);
            int2 c[kPerLane];
            int sx = 0, sy = 0;
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) {
                c[i] = kPerLane * lane + i < blocks * kWavesHere ? s_count[kPerLane * lane + i] : int2{0, 0};
                sx += c[i].x;
                sy += c[i].y;
            }
            const int ux = wave_scan(sx), uy = wave_scan(sy);
            int bx = more + ux - sx, by = equal + uy - sy;
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) {
                if (kPerLane * lane + i < kCounts) s_count[kPerLane * lane + i] = int2{bx, by};
                bx += c[i].x;
                by += c[i].y;
            }
            if (lane == 63) s_found[0] = bx, s_found[1] = by;
        }
        f32x4 x = {0, 0, 0, 0};
        if (scores_out) x = four(chunk0 + 4 * tid);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            if (chunk0 + i * kBlock >= L) break;
            // scores_out may be scores: tokens only move down, and a block's scores are all read before one of them is written
            const f32x4 now = x;
            if (scores_out) {
                if (i + 1 < HELD) x = four(chunk0 + (i + 1) * kBlock + 4 * tid);
                if (in_place) __syncthreads();
            }
            const int2 c = s_count[i * kWavesHere + wave];
            const unsigned b = before[i / 2] >> 16 * (i % 2);
            int m = c.x + (int)(b & 0xff), e0 = c.y + (int)(b >> 8 & 0xff);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool is_over = key[i][e] > bound, is_tie = key[i][e] == bound;
                if (is_over || (is_tie && e0 < ties)) {
                    const int to = m + min(e0, ties);
                    kept[to] = chunk0 + i * kBlock + 4 * tid + e;
                    if (scores_out) scores_out[to] = now[e];
                }
                m += is_over;
                e0 += is_tie;
            }
        }
        more = s_found[0];
        equal = s_found[1];
    }
    for (unsigned i = stay + tid; i < (unsigned)a.budget; i += THREADS) kept[i] = -1;   // (a budget may be the largest int)
}

// One new (page, head) tile of K or of V by one wave.  Row r comes from row `from` (of lane r) of the pool; rows past the n-th are left alone.
// Both ways stream past the caches: the rows that stay are next read by the attention, after many others.
template <int ROW_BYTES>
struct Rows {
    static constexpr int kLanes = ROW_BYTES / 16, kAtOnce = 64 / kLanes, kLoads = kPage / kAtOnce;
    u32x4 x[kLoads];
    SD_DEV void load(const char *pool, int64_t from, int n, int lane)
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = i * kAtOnce + lane / kLanes;
            const int64_t at = __shfl(from, r, 64);
            if (r < n) x[i] = kv_load<true>(reinterpret_cast<const u32x4 *>(pool + at * ROW_BYTES + lane % kLanes * 16));
        }
    }
    SD_DEV void store(char *to, int n, int lane) const
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = i * kAtOnce + lane / kLanes;
            if (r < n) __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4 *>(to + r * ROW_BYTES + lane % kLanes * 16));
        }
    }
    // Codes of rows whose scale was `old` (of lane r; past the last row its own), under the largest magnitude of those; -> that.
    SD_DEV float rescale(float old, int lane)
    {
        float top = fabsf(old);
        for (int off = 1; off < 16; off *= 2) top = fmaxf(top, __shfl_xor(top, off, 64));
        const float ratio = top > 0.f ? old / top : 1.f;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const float by = __shfl(ratio, i * kAtOnce + lane / kLanes, 64);
            if (by == 1.f) continue;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const f32x2 u = __builtin_amdgcn_cvt_pk_f32_fp8(x[i][w], false), v = __builtin_amdgcn_cvt_pk_f32_fp8(x[i][w], true);
                const unsigned y = __builtin_amdgcn_cvt_pk_fp8_f32(u[0] * by, u[1] * by, 0, false);
                x[i][w] = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * by, v[1] * by, y, true);
            }
        }
        return top;
    }
};

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
    const int64_t old_tile = (int64_t)a.block_table[(int64_t)b * a.max_blocks + t / kPage] * a.Hkv + g, from = old_tile * kPage + t % kPage;
    const int64_t tile = (int64_t)a.new_table[(int64_t)b * a.max_blocks + j] * a.Hkv + g;
    char *k = static_cast<char *>(a.k_pages), *v = static_cast<char *>(a.v_pages);
    Rows<kRow> kr, vr;
    kr.load(k, from, n, lane);
    vr.load(v, from, n, lane);
    if (FP8) {
        const float ks = kr.rescale(a.k_scales[old_tile], lane), vs = vr.rescale(a.v_scales[old_tile], lane);
        if (lane == 0) a.k_scales[tile] = ks, a.v_scales[tile] = vs;
    }
    kr.store(k + tile * kPage * kRow, n, lane);
    vr.store(v + tile * kPage * kRow, n, lane);
}

hipError_t launch_evict(const EvictArgs &a, int head_dim, int kv_dtype, hipStream_t stream)
{
    // The smallest workgroup whose registers hold the keys of the bound's tokens.  us per call, 512 threads of 8 keys : 1024 of 16 : 1024 of 64:
    //   1600 sequences and heads of 4096 (fp8, 256 stay) 70 : 88 : 92   128 of 16384 42 : 30 : 30   8 of 65536 101 : 69 : 52
    const dim3 units((unsigned)(a.B * a.Hkv));
    if (a.max_context_len <= 4 * 512 * 2) hipLaunchKernelGGL((evict_select_kernel<512, 2>), units, dim3(512), 0, stream, a);
    else if (a.max_context_len <= 4 * 1024 * 4) hipLaunchKernelGGL((evict_select_kernel<1024, 4>), units, dim3(1024), 0, stream, a);
    else hipLaunchKernelGGL((evict_select_kernel<1024, 16>), units, dim3(1024), 0, stream, a);
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
