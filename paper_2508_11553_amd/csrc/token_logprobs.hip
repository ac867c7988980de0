// Log probabilities of given tokens with the entropy of every row, and their gradient.
//
//   z = x / temperature,  S = sum exp(z - max z),  log p = z - max z - log S
//   out: log p of the target,  H = -sum p log p = log S - sum exp(z - max z) (z - max z) / S
//   gradient, with g that of the log probability and h that of the entropy:
//   dx_j = (g ([j = target] - p_j) - h p_j (log p_j + H)) / temperature
//
// One pass over the logits for the first, one pass that reads and writes for the second: bound by memory (4096 rows of 131072 bf16: 160 us and 338, 6.5 and 6.3 TB/s;
// 1072 of 49999 fp32 39 and 91, 5.5 and 5.9).  A lane holds the largest logit so far and the two sums relative to it; where a larger one comes both sums
// are moved to it.  fp32, a row's logarithm and result in 64 bits.  Vectors go past the caches both ways: nothing of 1 GB is read again.
#include "logits.h"

namespace sd {

namespace {

constexpr float kLowest = -3.402823466e38f;
constexpr float kFar = -1e5f;   // 2^kFar is 0, and 0 times it too, which 0 times -inf is not

// sums relative to m: s = sum 2^((x - m) c), t = sum 2^((x - m) c) (x - m) c
struct RowSums {
    float m, s, t;
};
SD_DEV RowSums joined(RowSums a, RowSums b, float c)
{
    const float m = max_of(a.m, b.m);
    const float da = max_of((a.m - m) * c, kFar), db = max_of((b.m - m) * c, kFar);
    const float ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
    return RowSums{m, a.s * ea + b.s * eb, (a.t + a.s * da) * ea + (b.t + b.s * db) * eb};
}
// log2(e) / temperature; in fp32 finite and not 0, so that it times a difference of 0 is 0 and times one of -inf is -inf.
SD_DEV double log2_scale(const float *temperature, int64_t r)
{
    const float t = temperature ? temperature[r] : 1.f;
    return kLog2e / (t > 0.f ? __builtin_fmin(__builtin_fmax((double)t, 0x1p-126), 0x1p125) : 1.0);
}

SD_DEV void finish(const LogprobArgs &a, int64_t r, RowSums x, double c, float at_target)
{
    const float log2_sum = x.s > 0.f || x.s != x.s ? (float)log2((double)x.s) : -__builtin_inff();
    const bool nothing = log2_sum == -__builtin_inff();   // every logit is -inf
    // (in 64 bits: of a target masked by the type's lowest number 2-based logarithms pass the range of fp32, the result does not)
    const double z = ((double)at_target - x.m) * c;
    a.logprobs[r] = nothing ? log2_sum : (float)((z - log2_sum) * kLn2);
    if (a.entropy) a.entropy[r] = nothing ? 0.f : (float)((log2_sum - (double)x.t / x.s) * kLn2);
    // What the gradient needs: the largest logit and log2 of the sum; of a row with nothing a sum past all, which leaves no weight.
    if (a.stats) a.stats[2 * r] = nothing ? 0.f : x.m, a.stats[2 * r + 1] = nothing ? __builtin_inff() : log2_sum;
}
template <int LANES>
SD_DEV RowSums join_lanes(RowSums x, float c)
{
#pragma unroll
    for (int off = LANES / 2; off > 0; off /= 2) x = joined(x, RowSums{__shfl_xor(x.m, off, 64), __shfl_xor(x.s, off, 64), __shfl_xor(x.t, off, 64)}, c);
    return x;
}

}  // namespace

template <bool F32, int THREADS>
__global__ __launch_bounds__(THREADS) void logprob_kernel(LogprobArgs a)
{
    using Row = LogitRow<F32>;
    constexpr int kWaves = THREADS / 64, kAhead = 4;   // vectors of a lane on their way together
    __shared__ RowSums s_wave[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const unsigned r = a.per_row.of(blockIdx.x), part = blockIdx.x - r * a.slices;
    const int target = a.targets[r];
    if ((unsigned)target >= (unsigned)a.vocab) {
        if (tid == 0 && part == 0) {
            a.logprobs[r] = 0.f;
            if (a.entropy) a.entropy[r] = 0.f;
            if (a.stats) a.stats[2 * r] = a.stats[2 * r + 1] = 0.f;
        }
        return;
    }
    const Row row(a.logits, r, a.stride, a.vocab);
    const double to_log2 = log2_scale(a.temperature, r);
    const float c = (float)to_log2, at_target = row.at(target);
    const int per_part = (row.vectors + a.slices - 1) / a.slices;
    const int end = min(row.vectors, (int)(part + 1) * per_part);
    RowSums x{kLowest, 0.f, 0.f};
    for (int v0 = part * per_part + tid; v0 < end; v0 += kAhead * THREADS) {
        u32x4 w[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) w[j] = v0 + j * THREADS < end ? row.template load<true>(v0 + j * THREADS) : Row::nothing();
        float m = x.m;
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int e = 0; e < Row::kEach; e += 2) m = max_of(m, Row::value(w[j], e), Row::value(w[j], e + 1));
        const float d = max_of((x.m - m) * c, kFar), scale = __builtin_amdgcn_exp2f(d);
        float s = 0.f, t = 0.f;   // (summed by themselves: errors of 32 terms, not of all that a lane has had)
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int e = 0; e < Row::kEach; ++e) {
                const float z = max_of((Row::value(w[j], e) - m) * c, kFar), y = __builtin_amdgcn_exp2f(z);
                s += y;
                t += y * z;
            }
        x.t = (x.t + x.s * d) * scale + t;
        x.s = x.s * scale + s;
        x.m = m;
    }
    x = join_lanes<64>(x, c);
    if (lane == 0) s_wave[wave] = x;
    __syncthreads();
    if (wave != 0) return;
    x = join_lanes<kWaves>(lane < kWaves ? s_wave[lane] : RowSums{kLowest, 0.f, 0.f}, c);
    if (lane != 0) return;
    if (a.slices == 1) finish(a, r, x, to_log2, at_target);
    else a.parts[3 * (int64_t)blockIdx.x] = x.m, a.parts[3 * (int64_t)blockIdx.x + 1] = x.s, a.parts[3 * (int64_t)blockIdx.x + 2] = x.t;
}

// Joins the parts of a row: a wave per row.
template <bool F32>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a)
{
    const int64_t r = blockIdx.x;
    const int target = a.targets[r];
    if ((unsigned)target >= (unsigned)a.vocab) return;
    const double to_log2 = log2_scale(a.temperature, r);
    const float c = (float)to_log2, at_target = LogitRow<F32>(a.logits, r, a.stride, a.vocab).at(target);
    RowSums x{kLowest, 0.f, 0.f};
    for (int i = threadIdx.x; i < a.slices; i += 64) {
        const float *p = a.parts + 3 * (r * a.slices + i);
        x = joined(x, RowSums{p[0], p[1], p[2]}, c);
    }
    x = join_lanes<64>(x, c);
    if (threadIdx.x == 0) finish(a, r, x, to_log2, at_target);
}

template <bool F32>
__global__ __launch_bounds__(256) void logprob_backward_kernel(LogprobGradArgs a)
{
    using Row = LogitRow<F32>;
    const unsigned r = a.per_row.of(blockIdx.x), part = blockIdx.x - r * a.slices;
    const int target = a.targets[r];
    const bool padding = (unsigned)target >= (unsigned)a.vocab;
    const Row row(a.logits, r, a.stride, a.vocab);
    const LogitRow<F32> out(a.d_logits, r, a.stride, a.vocab);
    const float c = (float)log2_scale(a.temperature, r), inverse = c * (float)kLn2;
    const float m = a.stats[2 * (int64_t)r], log2_sum = a.stats[2 * (int64_t)r + 1];
    const float g = padding ? 0.f : a.d_logprobs[r], h = padding || !a.d_entropy ? 0.f : a.d_entropy[r];
    const float entropy = a.d_entropy && !padding ? a.entropy[r] : 0.f, at_target = log2_sum == __builtin_inff() ? 0.f : g;
    const int v0 = (int)part * kGradVectors * 256 + (int)threadIdx.x;
    u32x4 w[kGradVectors];
    if (!padding) {
#pragma unroll
        for (int j = 0; j < kGradVectors; ++j)
            if (v0 + j * 256 < row.vectors) w[j] = row.template load<true>(v0 + j * 256);
    }
#pragma unroll
    for (int j = 0; j < kGradVectors; ++j) {
        const int v = v0 + j * 256;
        if (v >= row.vectors) break;
        float y[Row::kEach];
#pragma unroll
        for (int e = 0; e < Row::kEach; ++e) {
            const float z = max_of((Row::value(w[j], e) - m) * c - log2_sum, kFar), q = __builtin_amdgcn_exp2f(z);   // log2 p, p
            // (p goes into each product first: what has no weight stays 0 whatever g, h and 1 / temperature come to; a p below 2^-126 has none)
            const float of_target = v * Row::kEach + e == target ? at_target : 0.f, of_g = __builtin_fmaf(-q, g, of_target);
            y[e] = padding ? 0.f : __builtin_fmaf(-h, q * __builtin_fmaf(z, (float)kLn2, entropy), of_g) * inverse;
        }
        u32x4 to;
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = F32 ? __builtin_bit_cast(unsigned, y[i]) : cvt_pk_bf16(y[F32 ? 0 : 2 * i], y[F32 ? 0 : 2 * i + 1]);
        out.template store<true>(v, to);
    }
}

hipError_t launch_logprobs(const LogprobArgs &a, bool f32, hipStream_t stream)
{
    const dim3 grid((unsigned)a.rows * (unsigned)a.slices), rows((unsigned)a.rows);
    auto go = [&](auto kernel, dim3 blocks, int threads) { hipLaunchKernelGGL(kernel, blocks, dim3(threads), 0, stream, a); };
    if (a.threads == 1024) f32 ? go(logprob_kernel<true, 1024>, grid, 1024) : go(logprob_kernel<false, 1024>, grid, 1024);
    else f32 ? go(logprob_kernel<true, 256>, grid, 256) : go(logprob_kernel<false, 256>, grid, 256);
    if (a.slices > 1) f32 ? go(logprob_join_kernel<true>, rows, 64) : go(logprob_join_kernel<false>, rows, 64);
    return hipGetLastError();
}

hipError_t launch_logprobs_backward(const LogprobGradArgs &a, bool f32, hipStream_t stream)
{
    const dim3 grid((unsigned)a.rows * (unsigned)a.slices);
    if (f32) hipLaunchKernelGGL(logprob_backward_kernel<true>, grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(logprob_backward_kernel<false>, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sd
