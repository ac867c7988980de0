// Rows on their way into the attention: every head's query and key divided by its root mean square, weighted,
// and rotated to its position; and the gradient of that.
//
//   r = 1 / sqrt(mean(x^2) + eps),  z = x r w,  y = R z       R turns the pairs of the first rotary_dim elements
//   dz = R^T dy,  dw += sum_rows dz x r,  g = dz w,  dx = r (g - x r^2 mean(g x))
//
// Bound by memory: a row is read once and written once (backward: two read, one written).  A row of d elements
// belongs to d / 16 lanes; lane l holds two 16-byte pieces of it, chosen so that both elements of every pair are
// its own: pieces l and l + rotary_dim / 16 where pairs are (i, i + rotary_dim / 2), pieces 2 l and 2 l + 1 where they are
// (2 i, 2 i + 1) and in the part that is not rotated.  So the rotation takes no exchange between lanes, and the mean
// three (d = 128) or two (64).  All of it in fp32, rounded to bf16 once at the end.
//
// Measured: 32768 tokens of 32/8 heads, d = 128, appended 135 us, 6.0 TB/s read and written, where a copy gets 4.9; 16384 of 64/8 heads 117 us (604 MB),
// their gradient 140 us (906 MB, 6.5 TB/s) and 4 for the weights' sums; 64 tokens of 28/4 heads 3.7 us, a launch.
#include "attn_tile.h"

namespace sd {

namespace {

constexpr int kRowThreads = 256;

struct Row16 {
    float x[16];   // [piece][element]
};

SD_DEV void widen(u32x4 w, float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
    }
}
SD_DEV u32x4 narrow(const float *x) { return u32x4{cvt_pk_bf16(x[0], x[1]), cvt_pk_bf16(x[2], x[3]), cvt_pk_bf16(x[4], x[5]), cvt_pk_bf16(x[6], x[7])}; }

// Calls whose rows no cache holds until they are read again stream them past the caches.
template <bool STREAM>
SD_DEV void store16(u32x4 *p, u32x4 x)
{
    if (STREAM) __builtin_nontemporal_store(x, p);
    else *p = x;
}

// Which two pieces of a row lane l holds.
struct Pieces {
    int a, b;
    bool turned;   // the lane's elements are rotated
};
SD_DEV Pieces pieces_of(const NormRopeArgs &n, int l)
{
    const int pairs = n.rotary_dim / 16;   // lanes whose pieces are rotated
    const bool halves = !n.interleaved && l < pairs;
    return Pieces{halves ? l : 2 * l, halves ? l + pairs : 2 * l + 1, l < pairs};
}

// The norm's weights of a lane's elements, bf16 or fp32.
SD_DEV Row16 weights_of(const void *w, bool fp32, const Pieces &p)
{
    Row16 r;
    if (fp32) {
        const f32x4 *f = static_cast<const f32x4 *>(w);
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4 *>(r.x + 4 * i) = f[2 * (i < 2 ? p.a : p.b) + (i & 1)];
    } else {
        widen(static_cast<const u32x4 *>(w)[p.a], r.x);
        widen(static_cast<const u32x4 *>(w)[p.b], r.x + 8);
    }
    return r;
}

// Cosines and sines of the lane's eight pairs at a position (positions outside the table take its nearest end).
struct Angles {
    float c[8], s[8];
};
SD_DEV Angles angles_of(const NormRopeArgs &n, int64_t token, int l, bool turned)
{
    Angles a;
    if (turned) {
        const int pos = min(max(n.positions[token], 0), n.table_len - 1);
        const f32x4 *row = reinterpret_cast<const f32x4 *>(n.table + (int64_t)pos * n.rotary_dim);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            *reinterpret_cast<f32x4 *>(a.c + 4 * i) = row[2 * l + i];
            *reinterpret_cast<f32x4 *>(a.s + 4 * i) = row[n.rotary_dim / 8 + 2 * l + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) a.c[i] = 1.f, a.s[i] = 0.f;
    }
    return a;
}

// Pair i of the lane: elements i and 8 + i (halves), or 2 i and 2 i + 1.
template <bool BACK>
SD_DEV void turn(float *x, const Angles &a, bool interleaved)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = BACK ? -a.s[i] : a.s[i];
        if (interleaved) {
            const float u = x[2 * i], v = x[2 * i + 1];
            x[2 * i] = u * a.c[i] - v * s;
            x[2 * i + 1] = v * a.c[i] + u * s;
        } else {
            const float u = x[i], v = x[8 + i];
            x[i] = u * a.c[i] - v * s;
            x[8 + i] = v * a.c[i] + u * s;
        }
    }
}

// Sum over the d / 16 lanes of a row (DPP: no LDS).
template <int D>
SD_DEV float row_sum(float x)
{
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xb1, 0xf, 0xf, false));   // quad_perm 1 0 3 2
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4e, 0xf, 0xf, false));   // quad_perm 2 3 0 1
    if (D == 128) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x141, 0xf, 0xf, false));   // row_half_mirror
    return x;
}

template <int D>
SD_DEV float inverse_rms(const float *x, float eps)
{
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += x[i] * x[i];
    return rsqrtf(row_sum<D>(sum) * (1.f / D) + eps);
}

}  // namespace

// One row per d / 16 lanes.  Rows of a token: its queries' heads, its keys' heads, and with pages (APPEND) its values' heads, which are copied.
template <int D, bool APPEND, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void norm_rope_kernel(NormRopeArgs n, RowPages p)
{
    constexpr int kLanes = D / 16;
    const int l = threadIdx.x % kLanes;
    const uint32_t row = blockIdx.x * (kRowThreads / kLanes) + threadIdx.x / kLanes, rows = n.Hq + (APPEND ? 2 : 1) * n.Hkv;
    if (row >= n.T * rows) return;   // all lanes of a row together
    const int64_t t = p.per_token.of(row);
    const int h = (int)(row - (uint32_t)t * rows);
    const bool is_q = h < n.Hq, is_v = APPEND && h >= n.Hq + n.Hkv;
    const int head = is_q ? h : is_v ? h - n.Hq - n.Hkv : h - n.Hq;
    const Pieces at = pieces_of(n, l);
    const uint16_t *src = is_q ? n.q + t * n.q_stride : is_v ? p.v + t * p.v_stride : n.k + t * n.k_stride;
    const u32x4 *in = reinterpret_cast<const u32x4 *>(src + (int64_t)head * D);
    u32x4 a = in[at.a], b = in[at.b];
    uint16_t *dst;
    if (is_q) {
        dst = n.q_out + (t * n.Hq + head) * D;
    } else if (APPEND) {
        // rows of no sequence, no slot or no page are not kept
        const int seq = p.seq_ids ? p.seq_ids[t] : (int)t, slot = p.slots ? p.slots[t] : n.positions[t];
        if (seq < 0 || seq >= p.batch || slot < 0 || slot / kPage >= p.max_blocks) return;
        const int page = p.block_table[(int64_t)seq * p.max_blocks + slot / kPage];
        if (page < 0 || page >= p.num_pages) return;
        dst = (is_v ? p.v_pages : p.k_pages) + (((int64_t)page * n.Hkv + head) * kPage + slot % kPage) * D;
    } else {
        dst = n.k_out + (t * n.Hkv + head) * D;
    }
    if (!is_v) {
        const Row16 w = weights_of(is_q ? n.q_weight : n.k_weight, n.fp32_weights, at);
        const Angles ang = angles_of(n, t, l, at.turned);
        float x[16];
        widen(a, x);
        widen(b, x + 8);
        const float r = inverse_rms<D>(x, n.eps);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w.x[i];
        turn<false>(x, ang, n.interleaved);
        a = narrow(x);
        b = narrow(x + 8);
    }
    u32x4 *out = reinterpret_cast<u32x4 *>(dst);
    store16<STREAM>(out + at.a, a);
    store16<STREAM>(out + at.b, b);
}

// Gradient.  The first n.q_blocks workgroups walk the queries' rows, the others the keys', so that a lane's weights and its share of
// dw stay in registers; a workgroup leaves one row of d sums, and norm_weight_kernel adds those up in a fixed order.
template <int D, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void norm_rope_backward_kernel(NormRopeArgs n, NormGradArgs d)
{
    constexpr int kLanes = D / 16, kRows = kRowThreads / kLanes;
    __shared__ float s_dw[kRowThreads / 64][D];
    const int l = threadIdx.x % kLanes;
    const bool is_q = (int)blockIdx.x < d.q_blocks;
    const uint32_t H = is_q ? n.Hq : n.Hkv, rows = n.T * H, step = (is_q ? d.q_blocks : gridDim.x - d.q_blocks) * kRows;
    const Division per_token = is_q ? d.per_q : d.per_k;
    const uint16_t *src = is_q ? n.q : n.k, *grad = is_q ? d.dq_out : d.dk_out;
    uint16_t *dst = is_q ? d.dq : d.dk;
    const int64_t stride = is_q ? n.q_stride : n.k_stride;
    const Pieces at = pieces_of(n, l);
    const Row16 w = weights_of(is_q ? n.q_weight : n.k_weight, n.fp32_weights, at);
    float dw[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) dw[i] = 0.f;
    for (uint32_t row = (is_q ? blockIdx.x : blockIdx.x - d.q_blocks) * kRows + threadIdx.x / kLanes; row < rows; row += step) {
        const int64_t t = per_token.of(row);
        const int64_t offset = t * stride + (int64_t)(row - (uint32_t)t * H) * D;
        const u32x4 *in = reinterpret_cast<const u32x4 *>(src + offset), *gin = reinterpret_cast<const u32x4 *>(grad + (int64_t)row * D);
        const u32x4 xa = kv_load<STREAM>(in + at.a), xb = kv_load<STREAM>(in + at.b), ga = kv_load<STREAM>(gin + at.a), gb = kv_load<STREAM>(gin + at.b);
        const Angles ang = angles_of(n, t, l, at.turned);
        float x[16], g[16];
        widen(xa, x);
        widen(xb, x + 8);
        widen(ga, g);
        widen(gb, g + 8);
        turn<true>(g, ang, n.interleaved);
        const float r = inverse_rms<D>(x, n.eps);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            dw[i] += g[i] * (x[i] * r);
            g[i] *= w.x[i];
            dot += g[i] * x[i];
        }
        const float c = row_sum<D>(dot) * (1.f / D) * (r * r);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = r * (g[i] - x[i] * c);
        u32x4 *out = reinterpret_cast<u32x4 *>(dst + offset);
        store16<STREAM>(out + at.a, narrow(x));
        store16<STREAM>(out + at.b, narrow(x + 8));
    }
    // the rows of a wave, then the waves
#pragma unroll
    for (int i = 0; i < 16; ++i)
        for (int off = kLanes; off < 64; off *= 2) dw[i] += __shfl_xor(dw[i], off, 64);
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 < kLanes) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_dw[wave][8 * at.a + i] = dw[i], s_dw[wave][8 * at.b + i] = dw[8 + i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < D; i += kRowThreads) {
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < kRowThreads / 64; ++v) sum += s_dw[v][i];
        d.parts[(int64_t)blockIdx.x * D + i] = sum;
    }
}

// dw = sum of the workgroups' rows: 16 elements to a workgroup, 64 rows at a time.
template <int D>
__global__ __launch_bounds__(1024) void norm_weight_kernel(NormGradArgs d, int k_blocks)
{
    __shared__ float s[64][17];
    const int groups = D / 16;
    const bool is_q = (int)blockIdx.x < groups;
    const int e = threadIdx.x % 16, slice = threadIdx.x / 16, element = (is_q ? blockIdx.x : blockIdx.x - groups) * 16 + e;
    const int first = is_q ? 0 : d.q_blocks, last = is_q ? d.q_blocks : d.q_blocks + k_blocks;
    float sum = 0.f;
    for (int i = first + slice; i < last; i += 8 * 64) {   // eight loads on their way at a time
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = i + 64 * j < last ? d.parts[(int64_t)(i + 64 * j) * D + element] : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[j];
    }
    s[slice][e] = sum;
    __syncthreads();
    for (int half = 32; half > 0; half /= 2) {
        if (slice < half) s[slice][e] += s[slice + half][e];
        __syncthreads();
    }
    if (slice == 0) (is_q ? d.dq_weight : d.dk_weight)[element] = s[0][e];
}

// From 64 MB of rows on, twice what the dies' L2 hold (32768 tokens, 32/8 heads, appended: 143 us, streamed 134; gradient of 16384, 64/8
// heads 182 and 160).
static bool streams(uint32_t rows, int head_dim, int32_t T) { return (int64_t)T * rows * head_dim * 2 >= 64 << 20; }

template <int D, bool APPEND>
static void launch_rows(const NormRopeArgs &n, const RowPages &p, uint32_t rows, hipStream_t stream)
{
    constexpr uint32_t kPer = kRowThreads / (D / 16);
    const dim3 grid((n.T * rows + kPer - 1) / kPer);
    if (streams(rows, D, n.T)) hipLaunchKernelGGL((norm_rope_kernel<D, APPEND, true>), grid, dim3(kRowThreads), 0, stream, n, p);
    else hipLaunchKernelGGL((norm_rope_kernel<D, APPEND, false>), grid, dim3(kRowThreads), 0, stream, n, p);
}

hipError_t launch_norm_rope(const NormRopeArgs &n, const RowPages *pages, int head_dim, hipStream_t stream)
{
    const uint32_t rows = n.Hq + (pages ? 2 : 1) * n.Hkv;
    if (n.T <= 0) return hipSuccess;
    RowPages p = {};
    if (pages) p = *pages;
    p.per_token = division_by(rows);
    if (head_dim == 128) pages ? launch_rows<128, true>(n, p, rows, stream) : launch_rows<128, false>(n, p, rows, stream);
    else if (head_dim == 64) pages ? launch_rows<64, true>(n, p, rows, stream) : launch_rows<64, false>(n, p, rows, stream);
    else return hipErrorNotSupported;
    return hipGetLastError();
}

template <int D>
static void launch_gradient(const NormRopeArgs &n, const NormGradArgs &d, int k_blocks, hipStream_t stream)
{
    const dim3 grid(d.q_blocks + k_blocks);
    if (streams(n.Hq + n.Hkv, D, n.T)) hipLaunchKernelGGL((norm_rope_backward_kernel<D, true>), grid, dim3(kRowThreads), 0, stream, n, d);
    else hipLaunchKernelGGL((norm_rope_backward_kernel<D, false>), grid, dim3(kRowThreads), 0, stream, n, d);
    hipLaunchKernelGGL(norm_weight_kernel<D>, dim3(2 * D / 16), dim3(1024), 0, stream, d, k_blocks);
}

hipError_t launch_norm_rope_backward(const NormRopeArgs &n, const NormGradArgs &d, int k_blocks, int head_dim, hipStream_t stream)
{
    if (head_dim == 128) launch_gradient<128>(n, d, k_blocks, stream);
    else if (head_dim == 64) launch_gradient<64>(n, d, k_blocks, stream);
    else return hipErrorNotSupported;
    return hipGetLastError();
}

}  // namespace sd
