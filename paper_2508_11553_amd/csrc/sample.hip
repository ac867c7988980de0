// A token for every row of logits, drawn with the row's temperature, top-k, top-p and min-p from a given uniform number.
//
//   z = x / temperature,  w = exp(z - max z),  order: x falling, equal x by rising index
//   kept: the first top_k;  of those the ones before which less than top_p of their weight lies;  of those w >= min_p
//   token: the first, by index, with (sum of the kept w up to it) > uniform * (sum of all kept w)
// All three limits keep a beginning of the order, so what is kept is known by its last logit (`bound`) and by the index of the
// last one equal to it that stays.
//
// Weights are whole numbers: w 2^43, rounded, from an exponential in 64 bits (which costs this machine no more instructions' time than one in 32).  Their
// sums are exact, so neither atomics nor the number of waves on a row change a token: what is added in floating point, the sums of stretches of
// 2048 logits, is added in an order that the row alone fixes.
//
// First kernel, a wave per stretch: its largest logit, its weights' sum relative to that (one pass over the logits, in registers), and the largest logit
// of each lane's 32.  Second kernel: of a row without limits the stretch in which the draw ends, by one wave, and the token in it.  Of a row with
// limits a workgroup first looks at the lanes' maxima: the k-th largest of some of the logits, or one down to which some of them hold the
// share top_p, bounds what can be kept, and only lanes whose maximum lies above are read again, into a list in LDS.
// Where that list would be too long (nearly even logits) the workgroup goes over the row instead.
#include "logits.h"

namespace sd {

namespace {

constexpr int kChooseThreads = 512, kChooseWaves = kChooseThreads / 64;
constexpr int kBins = 2048, kList = 2048, kGroups = 1024, kRanked = 256;
constexpr int kFarBin = kBins - 1;   // logits whose weight is 0
constexpr int kMaxStretches = (kMaxVocab + kStretch - 1) / kStretch;
constexpr double kOne = 8796093022208.0;   // 2^43
constexpr float kInf = __builtin_inff();

// 2^t 2^BITS for t in [-60, 0], t below and NaN taken as -60.  A polynomial on [-1/2, 1/2] of the smallest relative error (2^-43.5) that is 1 at 0.
template <int BITS>
SD_DEV double exp2_of(double t)
{
    constexpr double kRound = 6755399441055744.0 + BITS;   // 1.5 2^52: the sum's low bits are t + BITS, rounded
    t = __builtin_fmax(t, -60.0);
    const double y = t + kRound, f = t - (y - kRound);
    double p = 9.168123000972248e-08;
    p = __builtin_fma(p, f, 1.3255182740764668e-06);
    p = __builtin_fma(p, f, 1.5258493043374333e-05);
    p = __builtin_fma(p, f, 0.00015403456036911954);
    p = __builtin_fma(p, f, 0.0013333547331502897);
    p = __builtin_fma(p, f, 0.00961812915917182);
    p = __builtin_fma(p, f, 0.05550410873971191);
    p = __builtin_fma(p, f, 0.2402265069581371);
    p = __builtin_fma(p, f, 0.6931471805585505);
    p = __builtin_fma(p, f, 1.0);
    const uint64_t bits = __builtin_bit_cast(uint64_t, p);
    const unsigned exponent = (unsigned)__builtin_bit_cast(uint64_t, y) << 20;
    return __builtin_bit_cast(double, (uint64_t)((unsigned)(bits >> 32) + exponent) << 32 | (unsigned)bits);
}
constexpr uint64_t kWholeBias = 0x4330000000000000ull;   // of 2^52
// How logits of a row weigh: relative to `top`, at log2(e) / temperature.
struct Weigher {
    double top, c;
    SD_DEV double exponent(float x) const { return ((double)x - top) * c; }
    SD_DEV double weight(float x) const { return exp2_of<0>(exponent(x)); }
    SD_DEV uint64_t biased(float x) const { return __builtin_bit_cast(uint64_t, exp2_of<43>(exponent(x)) + 4503599627370496.0); }
    SD_DEV uint64_t whole(float x) const { return biased(x) - kWholeBias; }
};
// Logits of a row whose largest is +inf: those alone count, alike.
SD_DEV float finite(float x, bool infinite) { return !infinite ? x : x == kInf ? 0.f : -kInf; }

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

struct RowLimits {
    double c;
    float temperature, top_p, min_p;
    int top_k;
    bool greedy, by_count, by_mass, by_least;
    SD_DEV RowLimits(const SampleArgs &a, int r)
    {
        temperature = a.temperature ? a.temperature[r] : 1.f;
        greedy = !(temperature > 0.f);
        if (greedy) temperature = 1.f;
        c = kLog2e / (double)temperature;
        top_k = a.top_k ? a.top_k[r] : 0;
        top_p = a.top_p ? a.top_p[r] : 1.f;
        min_p = a.min_p ? a.min_p[r] : 0.f;
        by_count = !greedy && top_k > 0 && top_k < a.vocab;
        by_mass = !greedy && top_p < 1.f;
        by_least = !greedy && min_p > 0.f;
        top_p = max(top_p, 0.f);
        min_p = min(min_p, 1.f);
    }
};

// What the stretches of a row come to, by one wave: the largest logit and the sum of all weights relative to it.
struct RowTotal {
    float top;
    double sum;
};
SD_DEV double stretch_scale(float m, float top, double c)
{
    const double t = ((double)m - top) * c;
    return m == top ? 1.0 : t > -60.0 ? exp2_of<0>(t) : 0.0;
}
SD_DEV double wave_scan_f64(double x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const double y = __shfl_up(x, off, 64);
        x += lane >= off ? y : 0.0;
    }
    return x;
}
SD_DEV RowTotal row_total(const SampleArgs &a, int64_t r, double c)
{
    const int lane = threadIdx.x & 63;
    const float *maxima = a.maxima + r * a.stretches;
    const uint64_t *sums = a.sums + r * a.stretches;
    RowTotal t{-kInf, 0.0};
    for (int s0 = 0; s0 < a.stretches; s0 += 64) t.top = max_of(t.top, wave_max_of(s0 + lane < a.stretches ? maxima[s0 + lane] : -kInf));
    for (int s0 = 0; s0 < a.stretches; s0 += 64) {
        double x = 0.0;
        if (s0 + lane < a.stretches) x = (double)sums[s0 + lane] * stretch_scale(maxima[s0 + lane], t.top, c);
        t.sum += __shfl(wave_scan_f64(x), 63, 64);
    }
    t.sum *= 1.0 / kOne;
    return t;
}

// The token of stretch s at which the kept weights' sum reaches `target` (no more than all of them), by one wave.
template <bool F32, typename W>
SD_DEV int walk(const LogitRow<F32> &row, int s, uint64_t target, W &&weight)
{
    using Row = LogitRow<F32>;
    constexpr int kLoads = kStretch / 64 / Row::kEach;
    const int lane = threadIdx.x & 63;
    u32x4 w[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) w[j] = row.load(s * (kStretch / Row::kEach) + j * 64 + lane);
    uint64_t before = 0;
    int token = -1;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int first = s * kStretch + (j * 64 + lane) * Row::kEach;
        uint64_t mine[Row::kEach], sum = 0;
#pragma unroll
        for (int e = 0; e < Row::kEach; ++e) {
            mine[e] = weight(Row::value(w[j], e), first + e);
            sum += mine[e];
        }
        const uint64_t ends = before + wave_scan64(sum);
        const uint64_t here = __builtin_amdgcn_ballot_w64(ends >= target);
        if (here) {   // (wave-uniform)
            uint64_t x = ends - sum;
            int e0 = 0;
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) {
                if (x < target && x + mine[e] >= target) e0 = e;
                x += mine[e];
            }
            token = __builtin_amdgcn_readlane(first + e0, (int)__builtin_ctzll(here));
            break;
        }
        before = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(ends >> 32), 63) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)ends, 63);
    }
    return token;
}

// kept: the weight that the token was drawn from, relative to the largest.
template <bool F32>
SD_DEV void write_token(const SampleArgs &a, int64_t r, const LogitRow<F32> &row, int token, const RowLimits &l, const RowTotal &t, double kept)
{
    if ((threadIdx.x & 63) != 0) return;
    a.tokens[r] = token;
    if (!a.logprobs && !a.draw_logprobs) return;
    const double z = t.top == kInf ? 0.0 : ((double)row.at(token) - t.top) * (1.0 / (double)l.temperature);
    if (a.logprobs) a.logprobs[r] = (float)(z - log(t.sum));
    if (a.draw_logprobs) a.draw_logprobs[r] = l.greedy ? 0.f : (float)(z - log(kept));
}
SD_DEV bool write_nothing(const SampleArgs &a, int64_t r, const RowTotal &t)
{
    if (t.top != -kInf) return false;
    if ((threadIdx.x & 63) == 0) {
        a.tokens[r] = -1;
        if (a.logprobs) a.logprobs[r] = -kInf;
        if (a.draw_logprobs) a.draw_logprobs[r] = -kInf;
    }
    return true;
}

// A row without limits, or the largest logit, by one wave.
template <bool F32>
SD_DEV void draw_from_all(const SampleArgs &a, int64_t r, const RowLimits &l)
{
    const int lane = threadIdx.x & 63;
    const LogitRow<F32> row(a.logits, r, a.stride, a.vocab);
    const RowTotal t = row_total(a, r, l.c);
    if (write_nothing(a, r, t)) return;
    const float *maxima = a.maxima + r * a.stretches;
    const uint64_t *sums = a.sums + r * a.stretches;
    if (l.greedy) {
        for (int s0 = 0; s0 < a.stretches; s0 += 64) {
            const uint64_t here = __builtin_amdgcn_ballot_w64(s0 + lane < a.stretches && maxima[s0 + lane] == t.top);
            if (!here) continue;
            const int token = walk<F32>(row, s0 + (int)__builtin_ctzll(here), 1, [&](float x, int) { return (uint64_t)(x == t.top); });
            write_token(a, r, row, token, l, t, 1.0);
            return;
        }
    }
    const double u = a.uniform[r], aim = (u > 0.0 ? u : 0.0) * (t.sum * kOne);
    double before = 0.0;
    int at = 0;          // the stretch, what it holds and how far into it
    uint64_t target = 1;
    for (int s0 = 0; s0 < a.stretches; s0 += 64) {
        const bool some = s0 + lane < a.stretches;
        const float m = some ? maxima[s0 + lane] : -kInf;
        const uint64_t sum = some ? sums[s0 + lane] : 0;
        const double scale = stretch_scale(m, t.top, l.c), x = (double)sum * scale, ends = before + wave_scan_f64(x);
        const uint64_t over = __builtin_amdgcn_ballot_w64(ends > aim && x > 0.0), some_weight = __builtin_amdgcn_ballot_w64(x > 0.0);
        const double below = __shfl_up(ends, 1, 64), start = lane ? below : before;
        if (some_weight) {   // the first that passes the aim, or else the last that has any weight, whole
            const int which = over ? (int)__builtin_ctzll(over) : 63 - (int)__builtin_clzll(some_weight);
            uint64_t want = sum;
            if (over) {
                const double into = (aim - start) / scale;
                want = into > 0.0 ? into < (double)sum ? (uint64_t)into + 1 : sum : 1;
                want = want > sum ? sum : want;
            }
            at = s0 + which;
            target = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(want >> 32), which) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)want, which);
        }
        if (over) break;
        before = __shfl(ends, 63, 64);
    }
    const float m = maxima[at];
    const bool infinite = m == kInf;
    const Weigher weigh{infinite ? 0.0 : (double)m, l.c};
    const int token = walk<F32>(row, at, target, [&](float x, int) { return weigh.whole(finite(x, infinite)); });
    write_token(a, r, row, token, l, t, t.sum);
}

}  // namespace

// GROUPS: the lanes' maxima are written too.
template <bool F32, bool GROUPS>
__global__ __launch_bounds__(256) void sample_stretch_kernel(SampleArgs a)
{
    using Row = LogitRow<F32>;
    constexpr int kLoads = kStretch / 64 / Row::kEach;
    const int lane = threadIdx.x & 63;
    const unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), r = a.per_row.of(item);
    if (r >= (unsigned)a.rows) return;
    const Row row(a.logits, r, a.stride, a.vocab);
    const RowLimits l(a, r);
    int s = (int)(item - r * a.runs) * a.run;
    const int end = min(a.stretches, s + a.run);
    u32x4 w[kLoads], next[kLoads];
    auto load = [&](u32x4 *to, int at) {
        if ((at + 1) * kStretch <= a.vocab) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) to[j] = *row.vector(at * (kStretch / Row::kEach) + j * 64 + lane);
        } else {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) to[j] = row.load(at * (kStretch / Row::kEach) + j * 64 + lane);
        }
    };
    if (s < end) load(w, s);
    for (; s < end; ++s) {
        if (s + 1 < end) load(next, s + 1);
        float m = -kInf;
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
#pragma unroll
            for (int e = 0; e < Row::kEach; e += 2) m = max_of(m, Row::value(w[j], e), Row::value(w[j], e + 1));
        if (__builtin_amdgcn_ballot_w64(m != m)) {   // NaN becomes -inf
            m = -kInf;
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) {
                    const float x = Row::value(w[j], e);
                    if (x != x) {
                        if (F32) w[j][F32 ? e : 0] = 0xff800000u;
                        else w[j][F32 ? 0 : e / 2] = e & 1 ? (w[j][F32 ? 0 : e / 2] & 0xffffu) | 0xff800000u : (w[j][F32 ? 0 : e / 2] & 0xffff0000u) | 0xff80u;
                    } else {
                        m = max_of(m, x);
                    }
                }
        }
        const float top = wave_max_of(m);
        uint64_t sum = 0;
        if (top == kInf) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) sum += Row::value(w[j], e) == kInf ? (uint64_t)kOne : 0;
        } else if (top != -kInf) {
            const Weigher weigh{(double)top, l.c};
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) sum += weigh.biased(Row::value(w[j], e));
            sum -= kLoads * Row::kEach * kWholeBias;
        }
        sum = wave_scan64(sum);
        const int64_t at = (int64_t)r * a.stretches + s;
        if (lane == 63) a.sums[at] = sum, a.maxima[at] = top;
        if (GROUPS) {
            if (F32) static_cast<float *>(a.group_maxima)[at * 64 + lane] = m;
            else static_cast<unsigned short *>(a.group_maxima)[at * 64 + lane] = (unsigned short)(__builtin_bit_cast(unsigned, m) >> 16);
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) w[j] = next[j];
    }
}

// Rows without limits: a wave each.
template <bool F32>
__global__ __launch_bounds__(64) void sample_pick_kernel(SampleArgs a)
{
    const int r = blockIdx.x;
    draw_from_all<F32>(a, r, RowLimits(a, r));
}

// Rows with limits: a workgroup each.
template <bool F32>
__global__ __launch_bounds__(kChooseThreads) void sample_choose_kernel(SampleArgs a)
{
    using Row = LogitRow<F32>;
    using ull = unsigned long long;
    constexpr int kLoads = kStretch / 64 / Row::kEach, kVectors = kStretch / Row::kEach;   // of a lane, of a stretch
    __shared__ uint64_t s_bins[kBins], s_list[kList], s_stretch[kMaxStretches + 1], s_wave[kChooseWaves];
    __shared__ int s_groups[kGroups], s_rank[kRanked];
    __shared__ uint64_t s_found[2];
    __shared__ int s_n[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t r = blockIdx.x;
    const RowLimits l(a, (int)r);
    if (!l.by_count && !l.by_mass && !l.by_least) {
        if (wave == 0) draw_from_all<F32>(a, r, l);
        return;
    }
    const Row row(a.logits, r, a.stride, a.vocab);
    const RowTotal total = row_total(a, r, l.c);
    if (total.top == -kInf) {
        if (wave == 0) write_nothing(a, r, total);
        return;
    }
    const bool infinite = total.top == kInf;
    const float top = infinite ? 0.f : total.top;
    const Weigher weigh{(double)top, l.c};

    // Bins of logits, from the largest down, 64 to the power of e; the last one's weights are 0.  (Halves: a difference of the largest floats is none.)
    const float steps = 2.f * min(64.f / l.temperature, 1e30f), half_top = 0.5f * top;
    auto bin_of = [&](float x) { return (int)__builtin_fminf((half_top - 0.5f * x) * steps, (float)kFarBin); };
    int limit = kFarBin - 1;   // the last bin that may hold something that is kept
    auto lower = [&](double least) { limit = min(limit, (int)__builtin_fmin(-64.0 * log(least) * 1.00001, 1e6) + 1); };   // nothing lighter than `least` is kept
    if (l.by_least && !(l.by_count && l.by_mass)) lower((double)l.min_p);   // (top_p asks for a share of all that top_k leaves, light ones too)
    // All that are as light as this or lighter hold less than 1 - top_p: they come after.
    if (l.by_mass && !l.by_count) lower((1.0 - (double)l.top_p) * total.sum / (double)a.vocab);

    auto clear_bins = [&] {
        __syncthreads();
        for (int i = tid; i < kBins; i += kChooseThreads) s_bins[i] = 0;
        if (tid == 0) s_found[0] = kBins;
        __syncthreads();
    };
    auto add_to_bin = [&](int bin, uint64_t x) { atomicAdd(reinterpret_cast<ull *>(&s_bins[bin]), (ull)x); };
    // The first bin at which the sum from bin 0 on reaches `aim`, and the sum before it; false: it does not.
    struct Found {
        bool some;
        int bin;
        uint64_t before;
    };
    auto find = [&](uint64_t aim) {
        __syncthreads();
        constexpr int kPer = kBins / kChooseThreads;
        uint64_t x[kPer], sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += x[i] = s_bins[kPer * tid + i];
        const uint64_t upto = wave_scan64(sum);
        if (lane == 63) s_wave[wave] = upto;
        __syncthreads();
        uint64_t before = upto - sum;
        for (int w = 0; w < wave; ++w) before += s_wave[w];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (before < aim && aim <= before + x[i]) s_found[0] = kPer * tid + i, s_found[1] = before;
            before += x[i];
        }
        __syncthreads();
        return Found{s_found[0] < kBins, (int)s_found[0], s_found[1]};
    };
    auto share_of = [&](double mass) {   // the whole weight that top_p of `mass` (whole weights) asks for
        const double share = (double)l.top_p * mass;
        return share > 1.0 ? (uint64_t)__builtin_ceil(share) : 1;
    };

    // What the lanes' maxima say.
    const int groups = a.stretches * 64;
    auto group_max = [&](int i) {
        const int64_t at = r * groups + i;
        const float x = F32 ? static_cast<const float *>(a.group_maxima)[at] : __builtin_bit_cast(float, (unsigned)static_cast<const unsigned short *>(a.group_maxima)[at] << 16);
        return finite(x, infinite);
    };
    if (l.by_count || l.by_mass) {
        clear_bins();
        for (int i = tid; i < groups; i += kChooseThreads) {
            const float x = group_max(i);
            const int bin = bin_of(x);
            if (bin <= limit) add_to_bin(bin, l.by_count ? 1 : weigh.whole(x));
        }
        const Found f = find(l.by_count ? (uint64_t)l.top_k : share_of(total.sum * kOne));
        if (f.some) limit = min(limit, f.bin);
    }
    // The lanes that hold something down to the limit, then what they hold: key and index, larger codes come earlier.
    if (tid < 2) s_n[tid] = 0;
    __syncthreads();
    for (int i = tid; i < groups; i += kChooseThreads)
        if (bin_of(group_max(i)) <= limit) {
            const int n = atomicAdd(&s_n[0], 1);
            if (n < kGroups) s_groups[n] = i;
        }
    __syncthreads();
    const int found_groups = s_n[0];
    auto code_of = [](unsigned key, int i) { return (uint64_t)key << 32 | ~(unsigned)i; };
    auto push = [&](float x, int i) {
        const int n = atomicAdd(&s_n[1], 1);
        if (n < kList) s_list[n] = code_of(key_of<F32>(x), i);
    };
    if (found_groups <= kGroups) {
        for (int i = tid; i < found_groups * kLoads; i += kChooseThreads) {
            const int g = s_groups[i / kLoads], v = (g / 64) * kVectors + i % kLoads * 64 + g % 64;
            const u32x4 w = row.load(v);
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) {
                const float x = finite(Row::value(w, e), infinite);
                if (bin_of(x) <= limit) push(x, v * Row::kEach + e);
            }
        }
    }
    __syncthreads();
    int listed = s_n[1];
    const bool complete = found_groups <= kGroups && listed <= kList;   // the list holds all down to the limit
    bool from_list = complete;

    // What is kept: all keys above `bound`, and of those equal to it the indices up to `last`.
    unsigned bound = 0;
    int last = INT_MAX;
    auto kept = [&](unsigned key, int i) { return key > bound || (key == bound && i <= last); };
    auto heavy = [&](float x) { return !l.by_least || weigh.weight(x) >= (double)l.min_p; };

    if (complete && listed <= kRanked && (l.by_count || l.by_mass)) {
        // Few: each one's rank is counted, the threads of a candidate sharing the others.
        const int width = listed <= 64 ? 64 : listed <= 128 ? 128 : 256, shares = kChooseThreads / width;
        const int i = tid & (width - 1), per = (listed + shares - 1) / shares, j0 = tid / width * per;
        const uint64_t code = i < listed ? s_list[i] : 0;
        if (tid < kRanked) s_rank[tid] = 0;
        __syncthreads();
        int rank = 0;
        for (int j = j0; j < min(listed, j0 + per); ++j) rank += s_list[j] > code;
        if (i < listed) atomicAdd(&s_rank[i], rank);
        __syncthreads();
        if (tid < listed) {
            s_bins[s_rank[tid]] = weigh.whole(value_of<F32>((unsigned)(code >> 32)));
            s_bins[kRanked + s_rank[tid]] = code;
        }
        __syncthreads();
        // by every wave alike
        uint64_t x[4], sum = 0;
        const int most = l.by_count ? min(l.top_k, listed) : listed;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += x[e] = 4 * lane + e < most ? s_bins[4 * lane + e] : 0;
        const uint64_t ends = wave_scan64(sum);
        int n = most;
        if (l.by_mass) {
            const uint64_t all = __shfl((ull)ends, 63, 64);
            const uint64_t aim = share_of(l.by_count ? (double)all : total.sum * kOne);
            uint64_t upto = ends - sum;
            int before = 0;   // those whose sum does not reach the aim
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                upto += x[e];
                before += 4 * lane + e < most && upto < aim;
            }
            n = min(most, 1 + wave_reduce(before, [](int u, int v) { return u + v; }));
        }
        const uint64_t end_code = s_bins[kRanked + max(0, n - 1)];
        bound = (unsigned)(end_code >> 32);
        last = (int)~(unsigned)end_code;
        __syncthreads();
    } else if (l.by_count || l.by_mass) {
        // By histograms, of the list or of the row.
        auto each = [&](auto &&use) {
            if (from_list) {
                for (int i = tid; i < listed; i += kChooseThreads) {
                    const unsigned key = (unsigned)(s_list[i] >> 32);
                    use(key, (int)~(unsigned)s_list[i], value_of<F32>(key));
                }
            } else {
                for (int v = tid; v < row.vectors; v += kChooseThreads) {
                    const u32x4 w = row.load(v);
#pragma unroll
                    for (int e = 0; e < Row::kEach; ++e) {
                        const float x = finite(Row::value(w, e), infinite);
                        use(key_of<F32>(x), v * Row::kEach + e, x);
                    }
                }
            }
        };
        for (int by = 0; by < 2; ++by) {   // first the count, then the weight of what it leaves
            const bool mass = by;
            if (mass ? !l.by_mass : !l.by_count) continue;
            from_list = complete;
            clear_bins();
            each([&](unsigned key, int i, float x) {
                const int bin = bin_of(x);
                if (bin <= limit && kept(key, i)) add_to_bin(bin, mass ? weigh.whole(x) : 1);
            });
            uint64_t aim = (uint64_t)l.top_k;
            if (mass) {
                aim = share_of(total.sum * kOne);
                if (l.by_count) {   // of what the count left
                    __syncthreads();
                    uint64_t all = 0;
                    for (int i = lane; i < kBins; i += 64) all += s_bins[i];
                    aim = share_of((double)wave_reduce((ull)all, [](ull u, ull v) { return u + v; }));
                }
            }
            const Found f = find(aim);
            if (!f.some) continue;   // all of them
            if (!from_list) {   // the bin's own, if the list holds them
                __syncthreads();
                if (tid == 0) s_n[1] = 0;
                __syncthreads();
                each([&](unsigned key, int i, float x) {
                    if (bin_of(x) == f.bin && kept(key, i)) push(x, i);
                });
                __syncthreads();
                from_list = s_n[1] <= kList;
                listed = s_n[1];
            }
            // digits of the key, then of the index of those equal to it
            constexpr int kLevels = F32 ? 3 : 2;
            uint64_t before = f.before;
            unsigned prefix = 0;
            int end = INT_MAX;
            for (int level = 0; level < kLevels + 2; ++level) {
                const bool of_key = level < kLevels;
                const int bits = of_key ? (F32 ? (level < 2 ? 11 : 10) : (level ? 5 : 11)) : 10;
                const int shift = of_key ? (F32 ? (level == 0 ? 21 : level == 1 ? 10 : 0) : (level ? 0 : 5)) : (level == kLevels ? 10 : 0);
                const unsigned mask = (1u << bits) - 1;
                clear_bins();
                each([&](unsigned key, int i, float x) {
                    if (bin_of(x) != f.bin || !kept(key, i)) return;
                    unsigned digit;
                    if (of_key) {
                        if (level > 0 && (key ^ prefix) >> (shift + bits) != 0) return;
                        digit = mask - (key >> shift & mask);
                    } else {
                        if (key != prefix || (level > kLevels && (i ^ end) >> 10 != 0)) return;
                        digit = i >> shift & mask;
                    }
                    add_to_bin((int)digit, of_key && mass ? weigh.whole(x) : 1);
                });
                const Found g = find(aim - before);
                before += g.before;
                if (of_key) prefix |= (mask - (unsigned)g.bin) << shift;
                else end = level == kLevels ? g.bin << 10 : end | g.bin;
                if (level == kLevels - 1) {
                    if (mass) {   // as many of that weight
                        const uint64_t one = weigh.whole(value_of<F32>(prefix));
                        aim = (aim - before + one - 1) / one;
                        before = 0;
                    } else {
                        aim -= before;
                        before = 0;
                    }
                }
            }
            bound = prefix;
            last = end;
        }
    }

    // The kept weights by stretches.
    __syncthreads();
    for (int i = tid; i < a.stretches; i += kChooseThreads) s_stretch[i] = 0;
    __syncthreads();
    if (complete) {
        for (int i = tid; i < listed; i += kChooseThreads) {
            const unsigned key = (unsigned)(s_list[i] >> 32);
            const int at = (int)~(unsigned)s_list[i];
            const float x = value_of<F32>(key);
            if (kept(key, at) && heavy(x)) atomicAdd(reinterpret_cast<ull *>(&s_stretch[at / kStretch]), (ull)weigh.whole(x));
        }
    } else {
        for (int s = wave; s < a.stretches; s += kChooseWaves) {
            uint64_t sum = 0;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int v = s * kVectors + j * 64 + lane;
                const u32x4 w = row.load(v);
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) {
                    const float x = finite(Row::value(w, e), infinite);
                    if (bin_of(x) <= limit && kept(key_of<F32>(x), v * Row::kEach + e) && heavy(x)) sum += weigh.whole(x);
                }
            }
            sum = wave_scan64(sum);
            if (lane == 63) s_stretch[s] = sum;
        }
    }
    __syncthreads();
    if (wave != 0) return;
    uint64_t all = 0;
    for (int s0 = 0; s0 < a.stretches; s0 += 64) all += s0 + lane < a.stretches ? s_stretch[s0 + lane] : 0;
    all = wave_reduce((ull)all, [](ull u, ull v) { return u + v; });
    const double u = a.uniform[r], aim = u > 0.0 ? u * (double)all : 0.0;
    uint64_t target = aim < (double)all ? (uint64_t)aim + 1 : all, before = 0;
    if (target > all) target = all;
    for (int s0 = 0; s0 < a.stretches; s0 += 64) {
        const uint64_t x = s0 + lane < a.stretches ? s_stretch[s0 + lane] : 0, ends = before + wave_scan64(x);
        const uint64_t here = __builtin_amdgcn_ballot_w64(ends >= target);
        if (here) {
            const int which = (int)__builtin_ctzll(here);
            const uint64_t want = target - __shfl((ull)(ends - x), which, 64);
            const int token = walk<F32>(row, s0 + which, want, [&](float y, int i) {
                y = finite(y, infinite);
                return bin_of(y) <= limit && kept(key_of<F32>(y), i) && heavy(y) ? weigh.whole(y) : 0;
            });
            write_token(a, r, row, token, l, total, (double)all * (1.0 / kOne));
            return;
        }
        before = __shfl((ull)ends, 63, 64);
    }
}

hipError_t launch_sample(const SampleArgs &a, bool f32, hipStream_t stream)
{
    const dim3 rows((unsigned)a.rows), runs((unsigned)(((int64_t)a.rows * a.runs + 3) / 4));
    const bool limits = a.top_k || a.top_p || a.min_p;
    auto go = [&](auto kernel, dim3 grid, unsigned threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, a); };
    if (f32) {
        if (limits) go(sample_stretch_kernel<true, true>, runs, 256), go(sample_choose_kernel<true>, rows, kChooseThreads);
        else go(sample_stretch_kernel<true, false>, runs, 256), go(sample_pick_kernel<true>, rows, 64);
    } else {
        if (limits) go(sample_stretch_kernel<false, true>, runs, 256), go(sample_choose_kernel<false>, rows, kChooseThreads);
        else go(sample_stretch_kernel<false, false>, runs, 256), go(sample_pick_kernel<false>, rows, 64);
    }
    return hipGetLastError();
}

}  // namespace sd
