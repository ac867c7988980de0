// Rows of logits: 16 bytes at a time, wherever a row begins.
//
// A row of `vocab` elements may begin at any element, so its 16-byte vectors are counted from the aligned address at or below its first
// element: element e of vector v is the row's element v * kEach - off + e.  The first and the last vector may reach over the row's
// ends; their elements are loaded one by one there, and those outside are -inf, which no sum and no maximum sees.
#pragma once
#include "attn_tile.h"

namespace sd {

constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

template <bool F32>
struct LogitRow {
    static constexpr int kEach = F32 ? 4 : 8, kSize = F32 ? 4 : 2;
    const char *base;
    int off, vocab, vectors;

    SD_DEV LogitRow(const void *logits, int64_t row, int64_t stride, int vocab_) : vocab(vocab_)
    {
        const uintptr_t p = reinterpret_cast<uintptr_t>(logits) + (uintptr_t)(row * stride * kSize);
        base = reinterpret_cast<const char *>(p & ~(uintptr_t)15);
        off = (int)(p & 15) / kSize;
        vectors = (off + vocab + kEach - 1) / kEach;
    }
    SD_DEV int index(int v, int e) const { return v * kEach - off + e; }
    SD_DEV bool whole(int v) const { return v * kEach >= off && (v + 1) * kEach <= off + vocab; }

    template <bool STREAM = false>
    SD_DEV u32x4 load(int v) const   // v in [0, vectors)
    {
        const u32x4 *at = reinterpret_cast<const u32x4 *>(base) + v;
        if (whole(v)) return kv_load<STREAM>(at);
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (F32) {
                w[i] = inside(v, i) ? reinterpret_cast<const unsigned *>(at)[i] : 0xff800000u;
            } else {
                const unsigned short *h = reinterpret_cast<const unsigned short *>(at) + 2 * i;
                const unsigned lo = inside(v, 2 * i) ? h[0] : 0xff80u, hi = inside(v, 2 * i + 1) ? h[1] : 0xff80u;
                w[i] = lo | hi << 16;
            }
        }
        return u32x4{w[0], w[1], w[2], w[3]};
    }
    SD_DEV void store(int v, u32x4 w) const   // of a row that is written; elements outside stay as they are
    {
        u32x4 *to = reinterpret_cast<u32x4 *>(const_cast<char *>(base)) + v;
        if (whole(v)) {
            *to = w;
            return;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (inside(v, e)) {
                if (F32) reinterpret_cast<unsigned *>(to)[e] = w[F32 ? e : 0];
                else reinterpret_cast<unsigned short *>(to)[e] = (unsigned short)(w[F32 ? 0 : e / 2] >> 16 * (e & 1));
            }
    }
    SD_DEV bool inside(int v, int e) const { return (unsigned)index(v, e) < (unsigned)vocab; }
    SD_DEV static u32x4 nothing() { return F32 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
    SD_DEV static float value(u32x4 w, int e)
    {
        const unsigned u = w[F32 ? e : e / 2];   // (copied out: a bit cast of a vector's element reads element 0)
        return __builtin_bit_cast(float, F32 ? u : e & 1 ? u & 0xffff0000u : u << 16);
    }
    SD_DEV float at(int i) const
    {
        const int j = i + off;
        if (F32) return reinterpret_cast<const float *>(base)[j];
        return __builtin_bit_cast(float, (unsigned)reinterpret_cast<const unsigned short *>(base)[j] << 16);
    }
};

template <typename T, typename F>
SD_DEV T wave_reduce(T x, F f)
{
#pragma unroll
    for (int off = 32; off > 0; off /= 2) x = f(x, __shfl_xor(x, off, 64));
    return x;
}
// Sum of x over the lanes up to this one, 64 bits.
SD_DEV uint64_t wave_scan64(uint64_t x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const uint64_t y = __shfl_up((unsigned long long)x, off, 64);
        x += lane >= off ? y : 0;
    }
    return x;
}

}  // namespace sd
