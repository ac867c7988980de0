// Rows of logits: 16 bytes at a time, wherever a row begins.
//
// A row of `vocab` elements may begin at any element, so its vectors are loaded and stored at whatever address that gives (the memory
// takes any; a wave's 1024 bytes then touch one line more).  The last one may reach over the row's end: its elements are loaded one by one,
// and those outside are -inf, which no sum and no maximum sees.
#pragma once
#include "attn_tile.h"

namespace sd {

constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

typedef unsigned u32x4_anywhere __attribute__((ext_vector_type(4), aligned(2)));

template <bool F32>
struct LogitRow {
    static constexpr int kEach = F32 ? 4 : 8, kSize = F32 ? 4 : 2;
    const char *base;
    int vocab, vectors;

    SD_DEV LogitRow(const void *logits, int64_t row, int64_t stride, int vocab_)
        : base(static_cast<const char *>(logits) + row * stride * kSize), vocab(vocab_), vectors((vocab_ + kEach - 1) / kEach)
    {
    }
    SD_DEV const u32x4_anywhere *vector(int v) const { return reinterpret_cast<const u32x4_anywhere *>(base) + v; }
    SD_DEV bool whole(int v) const { return (v + 1) * kEach <= vocab; }

    // v may lie past the end
    template <bool STREAM = false>
    SD_DEV u32x4 load(int v) const
    {
        if (!whole(v)) return load_end(v);
        if (STREAM) return __builtin_nontemporal_load(vector(v));
        return *vector(v);
    }
    SD_DEV u32x4 load_end(int v) const
    {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (F32) {
                w[i] = v * kEach + i < vocab ? reinterpret_cast<const unsigned *>(vector(v))[i] : 0xff800000u;
            } else {
                const unsigned short *h = reinterpret_cast<const unsigned short *>(vector(v)) + 2 * i;
                const unsigned lo = v * kEach + 2 * i < vocab ? h[0] : 0xff80u, hi = v * kEach + 2 * i + 1 < vocab ? h[1] : 0xff80u;
                w[i] = lo | hi << 16;
            }
        }
        return u32x4{w[0], w[1], w[2], w[3]};
    }
    template <bool STREAM = false>
    SD_DEV void store(int v, u32x4 w) const   // of a row that is written
    {
        u32x4_anywhere *to = const_cast<u32x4_anywhere *>(vector(v));
        if (whole(v)) {
            if (STREAM) __builtin_nontemporal_store(w, to);
            else *to = w;
            return;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (v * kEach + e < vocab) {
                if (F32) reinterpret_cast<unsigned *>(to)[e] = w[F32 ? e : 0];
                else reinterpret_cast<unsigned short *>(to)[e] = (unsigned short)(w[F32 ? 0 : e / 2] >> 16 * (e & 1));
            }
    }
    SD_DEV static u32x4 nothing() { return F32 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
    SD_DEV static float value(u32x4 w, int e)
    {
        const unsigned u = w[F32 ? e : e / 2];   // (copied out: a bit cast of a vector's element reads element 0)
        return __builtin_bit_cast(float, F32 ? u : e & 1 ? u & 0xffff0000u : u << 16);
    }
    SD_DEV float at(int i) const
    {
        if (F32) return reinterpret_cast<const float *>(base)[i];
        return __builtin_bit_cast(float, (unsigned)reinterpret_cast<const unsigned short *>(base)[i] << 16);
    }
};

template <typename T, typename F>
SD_DEV T wave_reduce(T x, F f)
{
#pragma unroll
    for (int off = 32; off > 0; off /= 2) x = f(x, __shfl_xor(x, off, 64));
    return x;
}
// x of one lane (wave-uniform).
SD_DEV uint64_t read_lane(uint64_t x, int lane)
{
    return (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)x, lane);
}
SD_DEV double read_lane(double x, int lane) { return __builtin_bit_cast(double, read_lane(__builtin_bit_cast(uint64_t, x), lane)); }
// Sum of x over the lanes up to this one, 64 bits.
SD_DEV uint64_t wave_scan64(uint64_t x)
{
#define SD_SCAN_STEP(ctrl, rows)                                                                                                    \
    {                                                                                                                               \
        const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)x, ctrl, rows, 0xf, false);                               \
        const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(x >> 32), ctrl, rows, 0xf, false);                       \
        x += (uint64_t)hi << 32 | lo;                                                                                               \
    }
    SD_SCAN_STEP(0x111, 0xf) SD_SCAN_STEP(0x112, 0xf) SD_SCAN_STEP(0x114, 0xf) SD_SCAN_STEP(0x118, 0xf)
    SD_SCAN_STEP(0x142, 0xa) SD_SCAN_STEP(0x143, 0xc)
#undef SD_SCAN_STEP
    return x;
}
// The largest of a wave's values, none of them NaN.
SD_DEV float wave_max_of(float x)
{
#define SD_MAX_STEP(ctrl, rows) x = max_of(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), ctrl, rows, 0xf, false)));
    SD_MAX_STEP(0x111, 0xf) SD_MAX_STEP(0x112, 0xf) SD_MAX_STEP(0x114, 0xf) SD_MAX_STEP(0x118, 0xf)
    SD_MAX_STEP(0x142, 0xa) SD_MAX_STEP(0x143, 0xc)
#undef SD_MAX_STEP
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

}  // namespace sd
