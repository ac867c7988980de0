// A token for every row of logits, drawn with the row's temperature, top-k, top-p and min-p from a given uniform number.
//
//   z = x / temperature,  w = exp(z - max z),  order: x falling, equal x by rising index
//   kept: the first top_k;  of those the ones before which less than top_p of their weight lies;  of those w >= min_p
//   token: the first, by index, with (sum of the kept w up to it) > uniform * (sum of all kept w)
// All three limits keep a beginning of the order, so what is kept is known by its last logit (`bound`) and by the index of the
// last one equal to it that stays.
//
// Weights are whole numbers: w 2^43, rounded, from an exponential in 64 bits.  Their sums are exact, so neither atomics nor the number of waves on a row
// change a token: what is added in floating point, the sums of stretches of 2048 logits, is added in an order that the row alone fixes.  An instruction in
// 64 bits takes no longer here than one in 32, but a weight takes 11 where 32 bits would do with about half: some 15 of the first kernel's 43 us for many rows of
// bf16, none where memory bounds it.  Sums in 32 bits would be off by 1e-7 of a row and more, by how much depending on the waves' number: in nearly even rows, where a token of
// 10^5 holds 1e-5, a hundredth of the draws would end at a neighbour.
//
// First kernel, a wave per stretch: its largest logit, its weights' sum relative to that (one pass over the logits, in registers), and the largest logit
// of each lane's 32.  Bound by the vector units where there are many rows (512 of 160001 bf16: 43 us, 3.8 TB/s; 540 instructions a wave, 36 us at the 4 cycles that each
// takes at least: 358 for 32 weights a lane, 49 for its maxima, 42 for a power of the table, 55 for the wave's sum and maximum, 36 for the rest; memory alone 25; two or four
// stretches to a wave are no faster), by memory for fp32 (200 of 100003: 15 us, 5.3 TB/s).
//
// Second kernel: of a row without limits the stretch in which the draw ends, by one wave each for itself, and the token in it (7 us for 512 rows: five trips to memory).
// Of a row with limits a workgroup first looks at the lanes' maxima: the k-th largest of some of the logits, or one down to which some of them hold the
// share top_p, bounds what can be kept, and only lanes whose maximum lies above are read again, into a list in LDS.  Up to 256 of them are ranked by
// counting and the token drawn from them (64 rows of 131072: 12 us, half of it trips to memory, half barriers of short steps).
// Hundreds are cut at the bin in which the limit ends first, and what lies before that bin stays without a rank (1 row of 500: 37 -> 17 us).
// Where that list would be too long (nearly even logits) the workgroup goes over the row instead, twice: a histogram of weights in 32 bits brackets the
// share's end, then weights before it are summed exactly and those in the bracket listed (48 rows of 49999: 31 us, one compute unit each; more workgroups to a row need
// launches between the passes, 2 us each, which every call would have: the host does not know which rows are even).
#include "logits.h"

#include <type_traits>

// Products are fused where the code says so and nowhere else: what one kernel sums another one walks, and both have to round alike.
#pragma clang fp contract(off)

namespace sd {

namespace {

constexpr int kBins = 2048, kList = 2048, kGroups = 1024, kRanked = 256;
constexpr int kPowers = 256;
constexpr int kFarBin = kBins - 1;   // logits whose weight is 0
constexpr int kMaxStretches = (kMaxVocab + kStretch - 1) / kStretch;
constexpr double kOne = 8796093022208.0;   // 2^43
constexpr float kInf = __builtin_inff();

constexpr double kRound = 6755399441055744.0;   // 1.5 2^52: a sum's low bits are what is added to it, rounded

// 2^t for t in [-60, 1), t below and NaN taken as -60.  A polynomial on [-1/2, 1/2] of the smallest relative error (2^-51) that is 1 at 0.
SD_DEV double exp2_of(double t)
{
    t = __builtin_fmax(t, -60.0);
    const double y = t + kRound, f = t - (y - kRound);
    double p = 7.072585949269223e-09;
    p = __builtin_fma(p, f, 1.0208690299958306e-07);
    p = __builtin_fma(p, f, 1.321544258792169e-06);
    p = __builtin_fma(p, f, 1.5252657260200837e-05);
    p = __builtin_fma(p, f, 0.0001540353044173605);
    p = __builtin_fma(p, f, 0.0013333558230164974);
    p = __builtin_fma(p, f, 0.009618129107606888);
    p = __builtin_fma(p, f, 0.05550410866444772);
    p = __builtin_fma(p, f, 0.24022650695910097);
    p = __builtin_fma(p, f, 0.69314718055995);
    p = __builtin_fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)(unsigned)__builtin_bit_cast(uint64_t, y));
}
constexpr double kNone = 4503599627370496.0;   // 2^52
constexpr uint64_t kNoneBits = 0x4330000000000000ull;
constexpr int kOctaves = 64;   // below the largest logit; beyond there is no weight
// powers[j] = 2^(j / 256 - 21), its last bit set, less j << 44 (which the exponent's bits bring back, see Weigher), in LDS: by the first `threads` threads.
SD_DEV void make_powers(u32x2 *powers, int threads)
{
    for (int j = threadIdx.x; j < kPowers; j += threads)
        powers[j] = __builtin_bit_cast(u32x2, (__builtin_bit_cast(uint64_t, exp2_of(j * (1.0 / kPowers) + (43 - kOctaves))) | 1) - ((uint64_t)j << 44));
}
// How logits of a row weigh: relative to `top`, at log2(e) / temperature.  A logit's position is 2^14 less the 256ths of an octave that it lies below top.  Its whole
// part n (0 for all below 0, -inf and NaN) and the rest f make w 2^43 = 2^(n / 256 - 21) 2^(f / 256), the second by a polynomial (relative error 2^-45.7), the first
// from the table: n << 12 added to the high word makes the exponent of n >> 8 and takes back the j = n & 255 that the table holds too
// little.  Where top c is small its rounding is far below that of a weight, and one instruction makes the position.
// Sums are held above 2^52, where a fused product rounds to whole numbers: each weight by itself, as no weight lies halfway between two (its
// odd factor from the table has 53 bits, more than a whole number below 2^44 and a half).
struct Weigher {
    double top, c, shift;
    const u32x2 *powers;
    bool near;
    SD_DEV Weigher(float top_, double c_, const u32x2 *powers_)
        : top(top_), c(c_ * kPowers), shift(__builtin_fma(-top, c, (double)(kOctaves * kPowers))), powers(powers_), near(__builtin_fabs(top * c) < 65536.0)
    {
    }
    SD_DEV double weight(float x) const { return exp2_of(((double)x - top) * (c * (1.0 / kPowers))); }   // (of the largest exactly 1)
    // sum + w 2^43, rounded; sum is a whole number in [2^52, 2^53)
    template <bool NEAR>
    SD_DEV double add(double sum, float x) const
    {
        const double at = NEAR ? __builtin_fma((double)x, c, shift) : __builtin_fma((double)x - top, c, (double)(kOctaves * kPowers));
        unsigned n;
        asm("v_cvt_u32_f64 %0, %1" : "=v"(n) : "v"(at));   // (what is out of range becomes the nearest, NaN 0: the language leaves both open)
        const double f = __builtin_fmin(__builtin_fmax(__builtin_amdgcn_fract(at), 0.0), 1.0);   // (of -inf and NaN 0)
        double p = 3.3127842005945513e-09;
        p = __builtin_fma(p, f, 3.6655627958463705e-06);
        p = __builtin_fma(p, f, 0.002707606174622391);
        p = __builtin_fma(p, f, 0.9999999999999825);
        u32x2 power = powers[n & (kPowers - 1)];
        power[1] += n << 12;
        return __builtin_fma(p, __builtin_bit_cast(double, power), sum);
    }
    SD_DEV uint64_t whole(float x) const { return __builtin_bit_cast(uint64_t, near ? add<true>(kNone, x) : add<false>(kNone, x)) - kNoneBits; }
};
SD_DEV bool is_lone(float top) { return top == kInf; }   // then only those equal to it have weight
struct Lone {
    bool on;
    float top;
    SD_DEV float operator()(float x) const { return !on ? x : x == top ? 0.f : -kInf; }
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

struct RowLimits {
    double temperature, c;
    float top_p, min_p;
    int top_k;
    bool greedy, by_count, by_mass, by_least;
    SD_DEV RowLimits(const SampleArgs &a, int r)
    {
        temperature = a.temperature ? a.temperature[r] : 1.f;
        greedy = !(temperature > 0.0);
        if (greedy) temperature = 1.0;
        temperature = __builtin_fmin(temperature, 0x1p200);   // (infinity: far above all differences, which 0 times -inf would not be)
        c = kLog2e / temperature;
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
    return m == top ? 1.0 : t > -60.0 ? exp2_of(t) : 0.0;
}
SD_DEV double wave_scan_f64(double x)
{
#define SD_SCAN_STEP(ctrl, rows)                                                                                                    \
    {                                                                                                                               \
        const uint64_t u = __builtin_bit_cast(uint64_t, x);                                                                         \
        const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)u, ctrl, rows, 0xf, false);                               \
        const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), ctrl, rows, 0xf, false);                       \
        x += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);                                                                   \
    }
    SD_SCAN_STEP(0x111, 0xf) SD_SCAN_STEP(0x112, 0xf) SD_SCAN_STEP(0x114, 0xf) SD_SCAN_STEP(0x118, 0xf)
    SD_SCAN_STEP(0x142, 0xa) SD_SCAN_STEP(0x143, 0xc)
#undef SD_SCAN_STEP
    return x;
}
SD_DEV RowTotal row_total(const SampleArgs &a, int64_t r, double c)
{
    const int lane = threadIdx.x & 63;
    const float *maxima = a.maxima + r * a.stretches;
    const uint64_t *sums = a.sums + r * a.stretches;
    const float first = lane < a.stretches ? maxima[lane] : -kInf;
    const uint64_t first_sum = lane < a.stretches ? sums[lane] : 0;
    RowTotal t{wave_max_of(first), 0.0};
    for (int s0 = 64; s0 < a.stretches; s0 += 64) t.top = max_of(t.top, wave_max_of(s0 + lane < a.stretches ? maxima[s0 + lane] : -kInf));
    t.sum = read_lane(wave_scan_f64((double)first_sum * stretch_scale(first, t.top, c)), 63);
    for (int s0 = 64; s0 < a.stretches; s0 += 64) {
        double x = 0.0;
        if (s0 + lane < a.stretches) x = (double)sums[s0 + lane] * stretch_scale(maxima[s0 + lane], t.top, c);
        t.sum += read_lane(wave_scan_f64(x), 63);
    }
    t.sum *= 1.0 / kOne;
    return t;
}

struct Drawn {
    int token;   // < 0: not this wave's
    float x;
};
// The token of stretch s at which the kept weights' sum reaches `target` (no more than all of them), by WAVES waves that share the stretch's vectors:
// the wave whose vectors hold it has it.  s_part: a sum for each of a lane's vectors.
template <bool F32, int WAVES, typename W>
SD_DEV Drawn walk(const LogitRow<F32> &row, int s, uint64_t target, uint64_t *s_part, W &&weight)
{
    using Row = LogitRow<F32>;
    constexpr int kLoads = kStretch / 64 / Row::kEach, kMine = (kLoads + WAVES - 1) / WAVES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    u32x4 w[kMine];
    uint64_t upto[kMine];
#pragma unroll
    for (int j = 0; j < kMine; ++j)
        if (wave * kMine + j < kLoads) w[j] = row.load(s * (kStretch / Row::kEach) + (wave * kMine + j) * 64 + lane);
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        if (wave * kMine + j >= kLoads) break;
        uint64_t sum = 0;
#pragma unroll
        for (int e = 0; e < Row::kEach; ++e) sum += weight(Row::value(w[j], e), s * kStretch + ((wave * kMine + j) * 64 + lane) * Row::kEach + e);
        upto[j] = wave_scan64(sum);
        if (lane == 63) s_part[wave * kMine + j] = upto[j];
    }
    __syncthreads();
    Drawn d{-1, 0.f};
    uint64_t before = 0;
    for (int j = 0; j < wave * kMine && j < kLoads; ++j) before += s_part[j];
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        if (wave * kMine + j >= kLoads) break;
        const uint64_t all = read_lane(upto[j], 63);
        if (before < target && target <= before + all) {   // (wave-uniform)
            const int which = (int)__builtin_ctzll(__builtin_amdgcn_ballot_w64(before + upto[j] >= target));
            uint64_t x = before + (which ? read_lane(upto[j], which - 1) : 0);
            const int first = s * kStretch + ((wave * kMine + j) * 64 + which) * Row::kEach;
            const u32x4 at = {(unsigned)__builtin_amdgcn_readlane((int)w[j][0], which), (unsigned)__builtin_amdgcn_readlane((int)w[j][1], which),
                              (unsigned)__builtin_amdgcn_readlane((int)w[j][2], which), (unsigned)__builtin_amdgcn_readlane((int)w[j][3], which)};
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) {
                const uint64_t mine = weight(Row::value(at, e), first + e);
                if (x < target && x + mine >= target) d = Drawn{first + e, Row::value(at, e)};
                x += mine;
            }
        }
        before += all;
    }
    return d;
}

// kept: the weight that the token was drawn from, relative to the largest.
SD_DEV void write_token(const SampleArgs &a, int64_t r, const Drawn &d, const RowLimits &l, const RowTotal &t, double kept)
{
    const int lane = threadIdx.x & 63;
    if (d.token < 0) return;
    if (lane == 0) a.tokens[r] = d.token;
    float *to = lane == 0 ? a.logprobs : a.draw_logprobs;
    if (lane > 1 || !to) return;
    const double z = d.x == t.top ? 0.0 : ((double)d.x - t.top) * (1.0 / l.temperature);
    to[r] = lane == 1 && l.greedy ? 0.f : (float)(z - log(lane == 0 ? t.sum : kept));
}
SD_DEV bool write_nothing(const SampleArgs &a, int64_t r, const RowTotal &t)
{
    if (t.top != -kInf) return false;
    if (threadIdx.x == 0) {
        a.tokens[r] = -1;
        if (a.logprobs) a.logprobs[r] = -kInf;
        if (a.draw_logprobs) a.draw_logprobs[r] = -kInf;
    }
    return true;
}

// A row without limits, or the largest logit, by a workgroup of WAVES waves, each of which finds the stretch for itself.
template <bool F32, int WAVES>
SD_DEV void draw_from_all(const SampleArgs &a, int64_t r, const RowLimits &l, const u32x2 *powers, uint64_t *s_part)
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
            write_token(a, r, walk<F32, WAVES>(row, s0 + (int)__builtin_ctzll(here), 1, s_part, [&](float x, int) { return (uint64_t)(x == t.top); }), l, t, 1.0);
            return;
        }
    }
    const double u = a.uniform[r], aim = (u > 0.0 ? u : 0.0) * (t.sum * kOne);
    double before = 0.0;
    int at = 0;   // the stretch, its largest logit, how far into it
    float top = -kInf;
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
            top = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, m), which));
            target = read_lane(want, which);
        }
        if (over) break;
        before = read_lane(ends, 63);
    }
    const Lone lone{is_lone(top), top};
    const Weigher weigh(lone(top), l.c, powers);
    write_token(a, r, walk<F32, WAVES>(row, at, target, s_part, [&](float x, int) { return weigh.whole(lone(x)); }), l, t, t.sum);
}

}  // namespace

// A wave per stretch.  GROUPS: the lanes' maxima are written too.
template <bool F32, bool GROUPS>
__global__ __launch_bounds__(256) void sample_stretch_kernel(SampleArgs a)
{
    using Row = LogitRow<F32>;
    constexpr int kLoads = kStretch / 64 / Row::kEach;
    __shared__ u32x2 s_powers[kPowers];
    const int lane = threadIdx.x & 63;
    const unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), r = a.per_row.of(item);
    const int s = (int)(item - r * a.stretches);
    const bool some = r < (unsigned)a.rows;
    const Row row(a.logits, some ? r : 0, a.stride, a.vocab);
    u32x4 w[kLoads];
    if ((s + 1) * kStretch <= a.vocab) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) w[j] = *row.vector(s * (kStretch / Row::kEach) + j * 64 + lane);
    } else {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) w[j] = row.load(s * (kStretch / Row::kEach) + j * 64 + lane);
    }
    const RowLimits l(a, some ? (int)r : 0);
    make_powers(s_powers, 256);
    __syncthreads();
    if (!some) return;
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
    if (is_lone(top)) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) sum += Row::value(w[j], e) == top ? (uint64_t)kOne : 0;
    } else if (top != -kInf) {
        const Weigher weigh(top, l.c, s_powers);
        auto add = [&](auto near) {
            double all = kNone;
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) all = weigh.template add<decltype(near)::value>(all, Row::value(w[j], e));
            sum = __builtin_bit_cast(uint64_t, all) - kNoneBits;
        };
        if (weigh.near) add(std::true_type());
        else add(std::false_type());
    }
    sum = wave_scan64(sum);
    const int64_t at = (int64_t)r * a.stretches + s;
    if (lane == 63) a.sums[at] = sum, a.maxima[at] = top;
    if (GROUPS) {
        if (F32) static_cast<float *>(a.group_maxima)[at * 64 + lane] = m;
        else static_cast<unsigned short *>(a.group_maxima)[at * 64 + lane] = (unsigned short)(__builtin_bit_cast(unsigned, m) >> 16);
    }
}

// Rows without limits: a workgroup each.
template <bool F32>
__global__ __launch_bounds__(256) void sample_pick_kernel(SampleArgs a)
{
    __shared__ u32x2 s_powers[kPowers];
    __shared__ uint64_t s_part[8];
    const int r = blockIdx.x;
    const RowLimits l(a, r);
    make_powers(s_powers, 256);
    __syncthreads();
    draw_from_all<F32, 4>(a, r, l, s_powers, s_part);
}

// Rows with limits: a workgroup each.
template <bool F32, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_choose_kernel(SampleArgs a)
{
    constexpr int kChooseThreads = THREADS, kChooseWaves = THREADS / 64;
    using Row = LogitRow<F32>;
    using ull = unsigned long long;
    constexpr int kLoads = kStretch / 64 / Row::kEach, kVectors = kStretch / Row::kEach;   // of a lane, of a stretch
    constexpr int kHeld = 8;   // lanes' maxima that a thread holds
    __shared__ uint64_t s_bins[kBins], s_list[kList], s_stretch[kMaxStretches + 1], s_wave[kChooseWaves];
    __shared__ int s_groups[kGroups], s_rank[kRanked];
    __shared__ uint64_t s_found[2], s_base;
    __shared__ u32x2 s_powers[kPowers];
    __shared__ int s_n[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t r = blockIdx.x;
    const RowLimits l(a, (int)r);
    if (!l.by_count && !l.by_mass && !l.by_least) {
        make_powers(s_powers, kChooseThreads);
        __syncthreads();
        draw_from_all<F32, kChooseWaves>(a, r, l, s_powers, s_wave);
        return;
    }
    const Row row(a.logits, r, a.stride, a.vocab);
    // the lanes' maxima: a thread holds the first kHeld * kChooseThreads
    const int groups = a.stretches * 64;
    const char *maxima = static_cast<const char *>(a.group_maxima) + r * groups * Row::kSize;
    u32x4 held[kHeld / Row::kEach];
    auto load_maxima = [&](u32x4 *to, int first) {
#pragma unroll
        for (int j = 0; j < kHeld / Row::kEach; ++j) to[j] = first + kHeld * tid < groups ? reinterpret_cast<const u32x4 *>(maxima + (int64_t)(first + kHeld * tid) * Row::kSize)[j] : u32x4{};
    };
    load_maxima(held, 0);
    for (int i = tid; i < kBins; i += kChooseThreads) s_bins[i] = 0;
    for (int i = tid; i < a.stretches; i += kChooseThreads) s_stretch[i] = 0;
    if (tid < kRanked) s_rank[tid] = 0;
    if (tid < kPowers) make_powers(s_powers, kPowers);
    if (tid < 2) s_n[tid] = 0, s_found[tid] = kBins;
    const RowTotal total = row_total(a, r, l.c);
    if (write_nothing(a, r, total)) return;
    const Lone lone{is_lone(total.top), total.top};
    const float top = lone(total.top);
    const Weigher weigh(top, l.c, s_powers);
    __syncthreads();
    auto each_max = [&](auto &&use) {
        for (int first = 0; first < groups; first += kHeld * kChooseThreads) {
            u32x4 w[kHeld / Row::kEach];
#pragma unroll
            for (int j = 0; j < kHeld / Row::kEach; ++j) w[j] = held[j];
            if (first) load_maxima(w, first);
            if (first + kHeld * tid < groups)
#pragma unroll
                for (int i = 0; i < kHeld; ++i) use(first + kHeld * tid + i, lone(Row::value(w[i / Row::kEach], i % Row::kEach)));
        }
    };

    // Bins of logits, from the largest down, 64 to the power of e; the last one's weights are 0.
    float steps = (float)__builtin_fmin(64.0 / l.temperature, 1e30);
    auto bin_of = [&](float x) { return (int)__builtin_fminf((top - x) * steps, (float)kFarBin); };
    int limit = kFarBin - 1;   // the last bin that may hold something that is kept
    auto bins_to = [](double weight) { return __builtin_fmin(-64.0 * log(weight), 1e6); };
    auto lower = [&](double least) { limit = min(limit, (int)(bins_to(least) * 1.00001) + 1); };   // nothing lighter than `least` is kept
    float sure = kInf;   // (top - x) up to which a logit is as heavy as min_p without doubt
    if (l.by_least) sure = (float)(-log((double)l.min_p) * l.temperature * 0.99999);
    if (l.by_least && !(l.by_count && l.by_mass)) lower((double)l.min_p);   // (top_p asks for a share of all that top_k leaves, light ones too)
    // All that are as light as this or lighter hold less than 1 - top_p: they come after.
    if (l.by_mass && !l.by_count) lower((1.0 - (double)l.top_p) * total.sum / (double)a.vocab);
    auto heavy = [&](float x) { return top - x < sure || weigh.weight(x) >= (double)l.min_p; };

    auto clear_bins = [&] {
        __syncthreads();
        for (int i = tid; i < kBins; i += kChooseThreads) s_bins[i] = 0;
        if (tid < 2) s_found[tid] = kBins;
        __syncthreads();
    };
    auto add_to_bin = [&](int bin, uint64_t x) { atomicAdd(reinterpret_cast<ull *>(&s_bins[bin]), (ull)x); };
    // The first bin at which the sum from bin 0 on reaches `aim`, and the sum before it; false: it does not.
    struct Found {
        bool some;
        int bin;
        uint64_t before;
    };
    auto scan_bins = [&](uint64_t (&x)[kBins / kChooseThreads], auto &&value) {   // a thread's bins, and the sum before them
        __syncthreads();
        constexpr int kPer = kBins / kChooseThreads;
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += x[i] = value(s_bins[kPer * tid + i]);
        const uint64_t upto = wave_scan64(sum);
        if (lane == 63) s_wave[wave] = upto;
        __syncthreads();
        uint64_t before = upto - sum;
        for (int w = 0; w < wave; ++w) before += s_wave[w];
        return before;
    };
    auto find = [&](uint64_t aim) {
        constexpr int kPer = kBins / kChooseThreads;
        uint64_t x[kPer], before = scan_bins(x, [](uint64_t one) { return one; });
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
    if (l.by_count || l.by_mass) {
        each_max([&](int, float x) {
            const int bin = bin_of(x);
            if (bin <= limit) add_to_bin(bin, l.by_count ? 1 : weigh.whole(x));
        });
        const Found f = find(l.by_count ? (uint64_t)l.top_k : share_of(total.sum * kOne));
        if (f.some) limit = min(limit, f.bin);
    }
    // The lanes that hold something down to the limit, then what they hold: key and index, larger codes come earlier.
    each_max([&](int i, float x) {
        if (bin_of(x) > limit) return;
        const int n = atomicAdd(&s_n[0], 1);
        if (n < kGroups) s_groups[n] = i;
    });
    __syncthreads();
    const int found_groups = s_n[0];
    auto push = [&](float x, int i) {
        const int n = atomicAdd(&s_n[1], 1);
        if (n < kList) s_list[n] = (uint64_t)key_of<F32>(x) << 32 | ~(unsigned)i;
    };
    if (found_groups <= kGroups) {
        for (int i = tid; i < found_groups * kLoads; i += kChooseThreads) {
            const int g = s_groups[i / kLoads], v = (g / 64) * kVectors + i % kLoads * 64 + g % 64;
            const u32x4 w = row.load(v);
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) {
                const float x = lone(Row::value(w, e));
                if (bin_of(x) <= limit) push(x, v * Row::kEach + e);
            }
        }
        __syncthreads();
    }
    int listed = s_n[1];
    bool complete = found_groups <= kGroups && listed <= kList;   // the list holds all down to the limit

    // Rows that are gone over: a wave a part of the row, the next kBatch of its vectors on their way.  A stretch may lie in two waves' parts.
    auto each_vector = [&](auto &&use, auto &&ends) {   // use(vector, index of its first logit)
        constexpr int kBatch = F32 ? 2 : 1;
        const int items = (row.vectors + 63) / 64, per = ((items + kChooseWaves - 1) / kChooseWaves + kBatch - 1) / kBatch * kBatch, end = min(items, (wave + 1) * per);
        const int inside = a.vocab / (64 * Row::kEach) - (kBatch - 1);   // whole ones start below
        auto load = [&](u32x4 (&w)[kBatch], int i) {
            if (i < inside) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) w[j] = *row.vector((i + j) * 64 + lane);
            } else {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) w[j] = row.load((i + j) * 64 + lane);
            }
        };
        u32x4 next[kBatch];
        load(next, wave * per);
#pragma unroll 1
        for (int i = wave * per; i < end; i += kBatch) {
            u32x4 w[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) w[j] = next[j];
            if (i + kBatch < end) load(next, i + kBatch);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) use(w[j], ((i + j) * 64 + lane) * Row::kEach);
            if ((i + kBatch) % kLoads == 0 || i + kBatch >= end) ends(i / kLoads);
        }
    };
    auto each_plain = [&](auto &&use, auto &&ends) {
        each_vector([&](u32x4 w, int first) {
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) use(Row::value(w, e), first + e);
        }, ends);
    };
    auto each_logit = [&](auto &&use, auto &&ends) {
        each_vector([&](u32x4 w, int first) {
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) use(lone(Row::value(w, e)), first + e);
        }, ends);
    };

    // What is kept: all keys above `bound`, and of those equal to it the indices up to `last`.
    unsigned bound = 0;
    int last = INT_MAX;
    auto kept = [&](unsigned key, int i) { return key > bound || (key == bound && i <= last); };
    bool summed = false;    // s_stretch holds the weights of what lies in bins before `split`, the list all the others that may be kept
    int split = 0;
    uint64_t base = 0;      // the weight of what lies before `split`, light or not
    int ahead = 0;          // how many lie before it, where only those are counted
    auto stays = [&](float x, int i) {
        const int bin = bin_of(x);
        return (bin < split || (bin <= limit && kept(key_of<F32>(x), i))) && heavy(x);
    };

    if (!complete && l.by_mass && !l.by_count) {
        // The bin in which the share ends, from weights in 32 bits: whole ones of 2^-31 of the row's, each off by less than one and 2^-16 of itself.
        steps *= (float)(kBins - 2) / (float)(limit + 1);
        limit = kBins - 2;
        // (exponents from bins: log2(e) / temperature may pass the range of fp32, bins to octaves does not; no steps: all weigh alike)
        const float to_exponent = steps > 0.f ? (float)(-l.c / (double)steps) : 0.f, whole = (float)(31.0 - log2(total.sum));
        unsigned *bins = reinterpret_cast<unsigned *>(s_bins);
        clear_bins();
        const float past = (float)(limit + 1);
        auto add_up = [&](float x, int) {
            const float d = top - x, bin = d * steps;
            const unsigned w = (unsigned)__builtin_amdgcn_exp2f(__builtin_fmaf(bin, to_exponent, whole));
            if (bin < past) atomicAdd(&bins[2 * (int)bin + lane % 2], w);   // (two of each bin: logits crowd)
        };
        if (lone.on) each_logit(add_up, [](int) {});
        else each_plain(add_up, [](int) {});
        const double margin = 0x1p31 * (0x1p-15 + (double)a.vocab * 0x1p-31), aim = (double)l.top_p * 0x1p31;
        constexpr int kPer = kBins / kChooseThreads;
        uint64_t x[kPer], before = scan_bins(x, [](uint64_t two) { return (two & 0xffffffffu) + (two >> 32); });
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const double starts = (double)before, ends = (double)(before + x[i]);
            if (starts + margin < aim && ends + margin >= aim) s_found[0] = kPer * tid + i;   // the share ends in no bin before this one
            if (starts - margin < aim && ends - margin >= aim) s_found[1] = kPer * tid + i;   // nor in one after this one
            before += x[i];
        }
        if (tid == 0) s_n[1] = 0, s_base = 0;
        __syncthreads();
        const bool some = s_found[0] < kBins;
        split = some ? (int)s_found[0] : aim > margin ? kBins - 1 : 0;   // (down to the limit there is less than the share: all of that)
        limit = min(limit, (int)s_found[1]);
        // The weights of what lies before, by stretches, and the others into the list.
        double sum = kNone;
        uint64_t all = 0;
        const float upper = (float)split, lower_end = (float)(limit + 1);
        // (added as `whole` rounds them: the walk to the token has to come to the same sum)
        auto sum_up = [&](auto quick, auto near) {
            constexpr bool kQuick = decltype(quick)::value, kNear = decltype(near)::value;
            each_vector([&](u32x4 w, int first) {
                float x[Row::kEach];
                bool other = false;   // something is left over, or may be light
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) {
                    const float y = kQuick ? Row::value(w, e) : lone(Row::value(w, e)), d = top - y, bin = d * steps;
                    const bool in = bin < upper;
                    x[e] = in ? y : -kInf;
                    other |= kQuick ? bin < lower_end && !in : in ? !(d < sure) : bin < lower_end;
                }
                if (__builtin_amdgcn_ballot_w64(other)) {
#pragma unroll
                    for (int e = 0; e < Row::kEach; ++e) {
                        const float y = lone(Row::value(w, e));
                        if (x[e] == -kInf) {
                            if (bin_of(y) <= limit) push(y, first + e);
                        } else if (!kQuick && !heavy(y)) {
                            all += weigh.whole(y), x[e] = -kInf;
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < Row::kEach; ++e) sum = weigh.template add<kNear>(sum, x[e]);
            }, [&](int s) {
                const uint64_t whole = wave_scan64(__builtin_bit_cast(uint64_t, sum) - kNoneBits);
                if (lane == 63) atomicAdd(reinterpret_cast<ull *>(&s_stretch[s]), (ull)whole);
                all += lane == 63 ? whole : 0;
                sum = kNone;
            });
        };
        if (!weigh.near) sum_up(std::false_type(), std::false_type());
        else if (lone.on || l.by_least) sum_up(std::false_type(), std::true_type());
        else sum_up(std::true_type(), std::true_type());
        all = wave_scan64(all);
        if (lane == 63) atomicAdd(reinterpret_cast<ull *>(&s_base), (ull)all);
        __syncthreads();
        listed = s_n[1];
        summed = listed <= kList;
        if (summed) base = s_base;
        else split = 0;
    }
    auto mass_aim = [&] {   // of what the list holds, or the row
        const uint64_t aim = share_of(total.sum * kOne);
        return aim > base ? aim - base : 1;
    };

    if ((complete || summed) && listed > kRanked && (l.by_count || l.by_mass)) {
        // Fewer: what lies past the bin in which the count, or the share, ends leaves the list; and where that is not enough what lies before it too, as it stays.
        clear_bins();
        for (int i = tid; i < listed; i += kChooseThreads) {
            const float x = value_of<F32>((unsigned)(s_list[i] >> 32));
            if (bin_of(x) <= limit) add_to_bin(bin_of(x), l.by_count ? 1 : weigh.whole(x));
        }
        const Found f = find(l.by_count ? (uint64_t)l.top_k : mass_aim());
        if (f.some) {
            limit = f.bin;
            for (int round = 0; round < 2; ++round) {
                const int from = round ? limit : 0;
                if (listed <= kRanked || (round && (limit == 0 || (l.by_count && l.by_mass)))) break;   // (a share of what the count leaves is not known yet)
                uint64_t mine[kList / kChooseThreads];
#pragma unroll
                for (int j = 0; j < kList / kChooseThreads; ++j) mine[j] = tid + j * kChooseThreads < listed ? s_list[tid + j * kChooseThreads] : 0;
                if (tid == 0) s_n[1] = 0;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < kList / kChooseThreads; ++j) {
                    const float x = value_of<F32>((unsigned)(mine[j] >> 32));
                    const int bin = bin_of(x);
                    if (tid + j * kChooseThreads >= listed || bin > limit) continue;
                    if (bin >= from) s_list[atomicAdd(&s_n[1], 1)] = mine[j];
                    else if (heavy(x)) atomicAdd(reinterpret_cast<ull *>(&s_stretch[(int)~(unsigned)mine[j] / kStretch]), (ull)weigh.whole(x));
                }
                __syncthreads();
                listed = s_n[1];
                if (round) {
                    complete = false;
                    summed = true;
                    split = from;
                    if (l.by_count) ahead = (int)f.before;
                    else base += f.before;
                }
                __syncthreads();
            }
        }
    }
    if ((complete || summed) && listed <= kRanked && (l.by_count || l.by_mass)) {
        // Few: each one's rank is counted, the threads of a candidate sharing the others.
        const int width = listed <= 64 ? 64 : listed <= 128 ? 128 : 256, shares = kChooseThreads / width;
        const int i = tid & (width - 1), per = (listed + shares - 1) / shares, j0 = tid / width * per;
        const uint64_t code = i < listed ? s_list[i] : 0;
        int rank = 0;
        for (int j = j0; j < min(listed, j0 + per); ++j) rank += s_list[j] > code;
        if (i < listed) atomicAdd(&s_rank[i], rank);
        __syncthreads();
        if (tid < listed) {
            s_bins[s_rank[tid]] = weigh.whole(value_of<F32>((unsigned)(code >> 32)));
            s_bins[kRanked + s_rank[tid]] = code;
        }
        if (tid < kRanked) s_bins[2 * kRanked + tid] = 0;
        __syncthreads();
        // by every wave alike
        uint64_t x[4], sum = 0;
        const int most = l.by_count ? min(l.top_k - ahead, listed) : listed;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += x[e] = 4 * lane + e < most ? s_bins[4 * lane + e] : 0;
        const uint64_t ends = wave_scan64(sum);
        int n = most;
        if (l.by_mass) {
            const uint64_t aim = l.by_count ? share_of((double)read_lane(ends, 63)) : mass_aim();
            uint64_t upto = ends - sum;
            int before = 0;   // those whose sum does not reach the aim
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                upto += x[e];
                before += 4 * lane + e < most && upto < aim;
            }
            n = min(most, 1 + wave_reduce(before, [](int u, int v) { return u + v; }));
        }
        if (n > 0) {
            const uint64_t end_code = s_bins[kRanked + n - 1];
            bound = (unsigned)(end_code >> 32);
            last = (int)~(unsigned)end_code;
        }
        if (complete) {
            // All that is kept is at hand: the weight up to each one, by index, in the same way, and the draw.
            if (l.by_least) {
                __syncthreads();
                if (tid < n && !heavy(value_of<F32>((unsigned)(s_bins[kRanked + tid] >> 32)))) s_bins[tid] = 0;
                __syncthreads();
            }
            const unsigned mine = i < n ? (unsigned)s_bins[kRanked + i] : 0;   // (larger ones are lower indices)
            uint64_t upto = 0;
            for (int j = j0; j < min(n, j0 + per); ++j) upto += (unsigned)s_bins[kRanked + j] >= mine ? s_bins[j] : 0;
            if (i < n) atomicAdd(reinterpret_cast<ull *>(&s_bins[2 * kRanked + i]), (ull)upto);
            uint64_t all = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) all += 4 * lane + e < n ? s_bins[4 * lane + e] : 0;
            all = read_lane(wave_scan64(all), 63);
            const double u = a.uniform[r], aim = u > 0.0 ? u * (double)all : 0.0;
            const uint64_t target = aim < (double)all ? min((uint64_t)aim + 1, all) : all;
            __syncthreads();
            if (tid < n) {
                const uint64_t end = s_bins[2 * kRanked + tid], one = s_bins[tid];
                if (end - one < target && target <= end) s_found[0] = s_bins[kRanked + tid];
            }
            __syncthreads();
            if (wave == 0) write_token(a, r, Drawn{(int)~(unsigned)s_found[0], lone.on ? total.top : value_of<F32>((unsigned)(s_found[0] >> 32))}, l, total, (double)all * (1.0 / kOne));
            return;
        }
    } else if (l.by_count || l.by_mass) {
        // By histograms, of the list or of the row.
        bool from_list;
        auto each = [&](auto &&use) {
            if (from_list) {
                for (int i = tid; i < listed; i += kChooseThreads) {
                    const unsigned key = (unsigned)(s_list[i] >> 32);
                    use(key, (int)~(unsigned)s_list[i], value_of<F32>(key));
                }
            } else {
                each_logit([&](float x, int i) { use(key_of<F32>(x), i, x); }, [](int) {});
            }
        };
        for (int by = 0; by < 2; ++by) {   // first the count, then the weight of what it leaves
            const bool mass = by;
            if (mass ? !l.by_mass : !l.by_count) continue;
            from_list = complete || summed;
            clear_bins();
            each([&](unsigned key, int i, float x) {
                const int bin = bin_of(x);
                if (bin <= limit && kept(key, i)) add_to_bin(bin, mass ? weigh.whole(x) : 1);
            });
            uint64_t aim = (uint64_t)(l.top_k - ahead);
            if (mass) {
                aim = mass_aim();
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
            int end = 0;
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
                else end |= g.bin << shift;
                if (level == kLevels - 1) {   // as many of that weight, or of those that are left
                    const uint64_t one = mass ? weigh.whole(value_of<F32>(prefix)) : 1;
                    aim = (aim - before + one - 1) / one;
                    before = 0;
                }
            }
            bound = prefix;
            last = end;
        }
    }

    // The kept weights by stretches.
    if (complete || summed) {
        for (int i = tid; i < listed; i += kChooseThreads) {
            const unsigned key = (unsigned)(s_list[i] >> 32);
            const int at = (int)~(unsigned)s_list[i];
            const float x = value_of<F32>(key);
            if (kept(key, at) && heavy(x)) atomicAdd(reinterpret_cast<ull *>(&s_stretch[at / kStretch]), (ull)weigh.whole(x));
        }
    } else {
        __syncthreads();
        for (int i = tid; i < a.stretches; i += kChooseThreads) s_stretch[i] = 0;
        __syncthreads();
        uint64_t sum = 0;
        each_logit([&](float x, int i) {
            if (stays(x, i)) sum += weigh.whole(x);
        }, [&](int s) {
            sum = wave_scan64(sum);
            if (lane == 63) atomicAdd(reinterpret_cast<ull *>(&s_stretch[s]), (ull)sum);
            sum = 0;
        });
    }
    __syncthreads();
    // by every wave alike, up to the token's own
    uint64_t all = lane < a.stretches ? s_stretch[lane] : 0;
    const uint64_t first = all;
    for (int s0 = 64; s0 < a.stretches; s0 += 64) all += s0 + lane < a.stretches ? s_stretch[s0 + lane] : 0;
    all = read_lane(wave_scan64(all), 63);
    const double u = a.uniform[r], aim = u > 0.0 ? u * (double)all : 0.0;
    uint64_t target = aim < (double)all ? (uint64_t)aim + 1 : all, before = 0;
    if (target > all) target = all;
    for (int s0 = 0; s0 < a.stretches; s0 += 64) {
        const uint64_t x = s0 == 0 ? first : s0 + lane < a.stretches ? s_stretch[s0 + lane] : 0, ends = before + wave_scan64(x);
        const uint64_t here = __builtin_amdgcn_ballot_w64(ends >= target);
        if (here) {
            const int which = (int)__builtin_ctzll(here);
            const Drawn d = walk<F32, kChooseWaves>(row, s0 + which, target - read_lane(ends - x, which), s_wave, [&](float y, int i) {
                y = lone(y);
                return stays(y, i) ? weigh.whole(y) : 0;
            });
            write_token(a, r, d, l, total, (double)all * (1.0 / kOne));
            return;
        }
        before = read_lane(ends, 63);
    }
}

hipError_t launch_sample(const SampleArgs &a, bool f32, hipStream_t stream)
{
    const dim3 rows((unsigned)a.rows), runs((unsigned)(((int64_t)a.rows * a.stretches + 3) / 4));
    const bool limits = a.top_k || a.top_p || a.min_p;
    auto go = [&](auto kernel, dim3 grid, unsigned threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, a); };
    // (rows with limits: sixteen waves each while every row has a compute unit to itself, then two rows of eight.  us, 8 : 16 waves: 48 flat rows of 49999 40.4 : 37.6,
    // 200 mixed of 100003 66 : 59, 256 of 32000 22.4 : 23.0, 300 25.0 : 34.9, 260 flat rows of 50000 62 : 75)
    const bool few = a.rows <= 256;
    if (f32) {
        if (!limits) go(sample_stretch_kernel<true, false>, runs, 256), go(sample_pick_kernel<true>, rows, 256);
        else if (few) go(sample_stretch_kernel<true, true>, runs, 256), go(sample_choose_kernel<true, 1024>, rows, 1024);
        else go(sample_stretch_kernel<true, true>, runs, 256), go(sample_choose_kernel<true, 512>, rows, 512);
    } else {
        if (!limits) go(sample_stretch_kernel<false, false>, runs, 256), go(sample_pick_kernel<false>, rows, 256);
        else if (few) go(sample_stretch_kernel<false, true>, runs, 256), go(sample_choose_kernel<false, 1024>, rows, 1024);
        else go(sample_stretch_kernel<false, true>, runs, 256), go(sample_choose_kernel<false, 512>, rows, 512);
    }
    return hipGetLastError();
}

}  // namespace sd
