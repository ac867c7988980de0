// A token for every row of logits, drawn with the row's temperature, top-k, top-p and min-p from a given uniform number.
//
//   z = x / temperature,  w = exp(z - max z),  order: x falling, equal x by rising index
//   kept: the first top_k;  of those the ones before which less than top_p of their weight lies;  of those w >= min_p
//   token: the first, by index, with (sum of the kept w up to it) > uniform * (sum of all kept w)
// All three limits keep a beginning of the order, so what is kept is known by its last logit (`bound`) and by how many of the equal
// ones stay (`ties`, the first by index).
//
// Weights are whole numbers: w 2^43, rounded, from an exponential in 64 bits (a polynomial of degree 11, the remainder of the series is
// below 2^-47).  Sums of up to 2^20 of them are exact in 64 bits, so that no order of additions, and no way to cut a row, changes a token.
#include "logits.h"

namespace sd {

namespace {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64, kBins = 2048;

// 2^t for t <= 0 (NaN counts as -inf) as a double in [0, 1].
SD_DEV double exp2_of(double t)
{
    t = __builtin_fmax(t, -1100.0);
    const double n = __builtin_rint(t), f = t - n;
    // ln(2)^k / k!
    double p = 4.4455382718708114976e-10;
    p = __builtin_fma(p, f, 7.0549116208011233299e-9);
    p = __builtin_fma(p, f, 1.0178086009239699728e-7);
    p = __builtin_fma(p, f, 1.3215486790144309489e-6);
    p = __builtin_fma(p, f, 1.5252733804059840280e-5);
    p = __builtin_fma(p, f, 1.5403530393381609954e-4);
    p = __builtin_fma(p, f, 1.3333558146428443423e-3);
    p = __builtin_fma(p, f, 9.6181291076284771620e-3);
    p = __builtin_fma(p, f, 5.5504108664821579953e-2);
    p = __builtin_fma(p, f, 2.4022650695910071233e-1);
    p = __builtin_fma(p, f, 6.9314718055994530942e-1);
    p = __builtin_fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}
SD_DEV uint64_t whole_weight(double w)   // w 2^43, rounded; w in [0, 1]
{
    constexpr double kMagic = 4503599627370496.0;   // 2^52
    return __builtin_bit_cast(uint64_t, __builtin_fma(w, 8796093022208.0, kMagic)) - __builtin_bit_cast(uint64_t, kMagic);
}

// How logits of a row weigh.  A row whose largest is +inf weighs those alone.
struct Weigher {
    double top, c;   // the largest logit, log2(e) / temperature
    bool infinite;
    SD_DEV double weight(float x) const
    {
        if (infinite) return x == __builtin_inff() ? 1.0 : 0.0;
        return exp2_of(((double)x - top) * c);
    }
    SD_DEV uint64_t whole(float x) const { return whole_weight(weight(x)); }
};

// Keys order as logits do: NaN below everything, the two zeros equal.  Those of bf16 have 16 bits.
template <bool F32>
SD_DEV unsigned key_of(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x == 0.f ? 0.f : x);
    const unsigned key = x != x ? 0u : u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
    return F32 ? key : key >> 16;
}
template <bool F32>
SD_DEV float value_of(unsigned key)
{
    if (!F32) key = key << 16 | (key & 0x8000u ? 0u : 0xffffu);
    return __builtin_bit_cast(float, key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu));
}

}  // namespace

template <bool F32>
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(SampleArgs a)
{
    using Row = LogitRow<F32>;
    __shared__ uint64_t s_mass[kBins];
    __shared__ uint64_t s_wave[kSampleWaves];
    __shared__ int s_equal[kSampleWaves];
    __shared__ float s_max[kSampleWaves];
    __shared__ uint64_t s_found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = blockIdx.x;
    const Row row(a.logits, r, a.stride, a.vocab);
    float temperature = a.temperature ? a.temperature[r] : 1.f;
    const bool greedy = !(temperature > 0.f);
    if (greedy) temperature = 1.f;
    int k = a.top_k ? a.top_k[r] : 0;
    float p = a.top_p ? a.top_p[r] : 1.f, least = a.min_p ? a.min_p[r] : 0.f;
    const bool by_count = k > 0 && k < a.vocab, by_mass = p < 1.f, by_least = least > 0.f;
    if (least > 1.f) least = 1.f;

    // a wave's part of the row: whole vectors, one after the other
    const int per_wave = (row.vectors + kSampleWaves - 1) / kSampleWaves;
    const int v0 = wave * per_wave, v1 = min(row.vectors, v0 + per_wave);
    auto walk = [&](auto &&use) {
        for (int v = v0 + lane; v < v1; v += 64) {
            const u32x4 w = row.load(v);
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) use(Row::value(w, e), v, e);
        }
    };
    auto sum_waves = [&](uint64_t x) {   // of all threads
        x = wave_reduce((unsigned long long)x, [](unsigned long long u, unsigned long long v) { return u + v; });
        __syncthreads();
        if (lane == 0) s_wave[wave] = x;
        __syncthreads();
        uint64_t all = 0;
        for (int w = 0; w < kSampleWaves; ++w) all += s_wave[w];
        return all;
    };

    float top = -__builtin_inff();
    walk([&](float x, int, int) { top = __builtin_fmaxf(top, x); });
    top = wave_reduce(top, [](float u, float v) { return __builtin_fmaxf(u, v); });
    if (lane == 0) s_max[wave] = top;
    __syncthreads();
    for (int w = 0; w < kSampleWaves; ++w) top = __builtin_fmaxf(top, s_max[w]);
    if (top == -__builtin_inff()) {   // nothing to draw from
        if (tid == 0) {
            a.tokens[r] = -1;
            if (a.logprobs) a.logprobs[r] = top;
            if (a.draw_logprobs) a.draw_logprobs[r] = top;
        }
        return;
    }
    Weigher weigh;
    weigh.infinite = top == __builtin_inff();
    weigh.top = top;
    weigh.c = kLog2e / (double)temperature;

    uint64_t mine = 0;
    walk([&](float x, int, int) { mine += weigh.whole(x); });
    const uint64_t total = sum_waves(mine);

    // The key at which what `of` gives, added up from the largest key down, reaches `aim`; what lies above that key goes to `above`.
    constexpr int kLevels = F32 ? 3 : 2;
    auto descend = [&](bool count, uint64_t aim, unsigned floor_key, uint64_t &above) {
        unsigned bound = 0;
        above = 0;
#pragma unroll
        for (int level = 0; level < kLevels; ++level) {
            constexpr int kShift32[3] = {21, 10, 0}, kBits32[3] = {11, 11, 10}, kShift16[3] = {5, 0, 0}, kBits16[3] = {11, 5, 0};
            const int shift = F32 ? kShift32[level] : kShift16[level], bits = F32 ? kBits32[level] : kBits16[level];
            __syncthreads();
            for (int i = tid; i < kBins; i += kSampleThreads) s_mass[i] = 0;
            __syncthreads();
            walk([&](float x, int v, int e) {
                const unsigned key = key_of<F32>(x);
                if ((level > 0 && (key ^ bound) >> (shift + bits) != 0) || key < floor_key || !row.inside(v, e)) return;
                const uint64_t add = count ? 1 : weigh.whole(x);
                if (add) atomicAdd(reinterpret_cast<unsigned long long *>(&s_mass[key >> shift & ((1u << bits) - 1)]), (unsigned long long)add);
            });
            __syncthreads();
            // thread i holds bins 2 i and 2 i + 1 counted from the top
            const uint64_t x0 = s_mass[kBins - 1 - 2 * tid], x1 = s_mass[kBins - 2 - 2 * tid];
            const uint64_t upto = wave_scan64(x0 + x1);
            if (lane == 63) s_wave[wave] = upto;
            __syncthreads();
            uint64_t before = above + upto - x0 - x1;
            for (int w = 0; w < wave; ++w) before += s_wave[w];
            if (before < aim && aim <= before + x0) s_found[0] = kBins - 1 - 2 * tid, s_found[1] = before;
            before += x0;
            if (before < aim && aim <= before + x1) s_found[0] = kBins - 2 - 2 * tid, s_found[1] = before;
            __syncthreads();
            bound |= (unsigned)s_found[0] << shift;
            above = s_found[1];
        }
        return bound;
    };

    // The last logit that is kept, and how many of those equal to it.
    unsigned bound = 0;
    int ties = a.vocab;
    if (greedy) {
        bound = key_of<F32>(top);
        ties = 1;
    } else {
        if (by_count) {
            uint64_t above;
            bound = descend(true, (uint64_t)k, 0, above);
            ties = k - (int)above;
        }
        if (by_mass) {
            uint64_t all = total;
            const uint64_t each = by_count ? weigh.whole(value_of<F32>(bound)) : 0;
            if (by_count) {
                uint64_t over = 0;
                walk([&](float x, int, int) { over += key_of<F32>(x) > bound ? weigh.whole(x) : 0; });
                all = sum_waves(over) + each * (uint64_t)ties;
            }
            const double share = p > 0.f ? (double)p * (double)all : 0.0;
            uint64_t aim = (uint64_t)__builtin_ceil(share);
            aim = aim < 1 ? 1 : aim > all ? all : aim;
            uint64_t above;
            const unsigned last = descend(false, aim, bound, above);
            const uint64_t one = weigh.whole(value_of<F32>(last));   // at least 1: the bin holds something
            const uint64_t needed = (aim - above + one - 1) / one;
            ties = !by_count || last != bound || needed < (uint64_t)ties ? (int)needed : ties;
            bound = last;
        }
    }

    // Weights of what is kept, wave by wave; those equal to the bound are counted first.
    auto heavy = [&](float x) { return !by_least || greedy || weigh.weight(x) >= (double)least; };
    uint64_t over = 0;
    int equal = 0;
    walk([&](float x, int v, int e) {
        const unsigned key = key_of<F32>(x);
        if (!row.inside(v, e)) return;
        if (key > bound && heavy(x)) over += weigh.whole(x);
        equal += key == bound;
    });
    over = wave_reduce((unsigned long long)over, [](unsigned long long u, unsigned long long v) { return u + v; });
    equal = wave_reduce(equal, [](int u, int v) { return u + v; });
    const float last = value_of<F32>(bound);
    const uint64_t one = heavy(last) ? weigh.whole(last) : 0;
    __syncthreads();
    if (lane == 0) s_wave[wave] = over, s_equal[wave] = equal;
    __syncthreads();
    uint64_t kept = 0, before = 0;
    int seen = 0, at_wave = 0;
    {
        int n = 0;
        for (int w = 0; w < kSampleWaves; ++w) {
            const int stay = max(0, min(s_equal[w], ties - n));
            kept += s_wave[w] + one * (uint64_t)stay;
            n += s_equal[w];
        }
        const double u = a.uniform[r];
        const double aim = u > 0.0 ? u * (double)kept : 0.0;
        uint64_t target = aim < (double)kept ? (uint64_t)aim + 1 : kept;
        target = target > kept ? kept : target;
        n = 0;
        for (int w = 0; w < kSampleWaves; ++w) {
            const int stay = max(0, min(s_equal[w], ties - n));
            const uint64_t part = s_wave[w] + one * (uint64_t)stay;
            if (before + part >= target) {
                at_wave = w;
                break;
            }
            before += part;
            n += s_equal[w];
        }
        seen = n;
        if (wave == at_wave) {
            for (int v = v0; v < v1; v += 64) {   // (wave-uniform)
                const bool some = v + lane < v1;
                const u32x4 w = some ? row.load(v + lane) : Row::nothing();
                int mine = 0;
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) mine += some && row.inside(v + lane, e) && key_of<F32>(Row::value(w, e)) == bound;
                const int upto = wave_scan(mine);
                int nth = seen + upto - mine;
                uint64_t weight[Row::kEach], sum = 0;
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) {
                    const float x = Row::value(w, e);
                    const unsigned key = key_of<F32>(x);
                    weight[e] = 0;
                    if (some && row.inside(v + lane, e)) {
                        if (key > bound && heavy(x)) weight[e] = weigh.whole(x);
                        if (key == bound && nth++ < ties) weight[e] = one;
                    }
                    sum += weight[e];
                }
                const uint64_t ends = before + wave_scan64(sum);
                const bool here = ends >= target && ends - sum < target;
                if (here) {
                    uint64_t x = ends - sum;
                    int e0 = 0;
#pragma unroll
                    for (int e = 0; e < Row::kEach; ++e) {
                        if (x < target && x + weight[e] >= target) e0 = e;
                        x += weight[e];
                    }
                    const int token = row.index(v + lane, e0);
                    a.tokens[r] = token;
                    const double x0 = row.at(token);
                    const double z = weigh.infinite ? 0.0 : (x0 - weigh.top) * (1.0 / (double)temperature);
                    constexpr double kOne = 8796093022208.0;
                    if (a.logprobs) a.logprobs[r] = (float)(z - log((double)total / kOne));
                    if (a.draw_logprobs) a.draw_logprobs[r] = greedy ? 0.f : (float)(z - log((double)kept / kOne));
                }
                if (__builtin_amdgcn_ballot_w64(here)) break;
                before = __shfl((unsigned long long)ends, 63, 64);
                seen += __builtin_amdgcn_readlane(upto, 63);
            }
        }
    }
}

hipError_t launch_sample(const SampleArgs &a, bool f32, hipStream_t stream)
{
    const dim3 grid((unsigned)a.rows), block(kSampleThreads);
    if (f32) hipLaunchKernelGGL(sample_row_kernel<true>, grid, block, 0, stream, a);
    else hipLaunchKernelGGL(sample_row_kernel<false>, grid, block, 0, stream, a);
    return hipGetLastError();
}

}  // namespace sd
