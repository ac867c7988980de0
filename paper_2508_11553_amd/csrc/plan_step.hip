// Places for the new tokens of every sequence: pages, block table, lengths and the rows' slot map.
//
// Sums over the batch by one workgroup, a thread four sequences: pages that come back; pages and rows that are asked for, in the batch's order, which says
// who is served; pages and rows of those that are.  Then the entries, each by one thread, which finds its sequence in those sums (kept in LDS, or
// a sample of them where the batch is too large).  The free list is a stack; the pages that come back lie on top of it, so they are the first to be taken, and
// only what is left of them is written to it.
//
// Bound by latency: a small call is one workgroup's, which keeps all sums in LDS (64 sequences 6 us: counts, sums, pages, three trips to memory and five barriers); a
// large one leaves them in the workspace for a second kernel (2048 sequences 5 us, then 6: counts -> sums into LDS -> search -> sequence -> page, each waits for
// the one before; 200 sequences with 0.6 M rows 5 and 5.5).
#include "logits.h"

namespace sd {

namespace {

constexpr int kPer = 4;   // sequences of a thread

SD_DEV int pages_of(int tokens) { return (int)(((int64_t)tokens + kPage - 1) / kPage); }
SD_DEV int length_of(const PlanArgs &a, int L) { return max(0, min(L, a.max_context_len)); }
SD_DEV int own_from(const PlanArgs &a, int b, int L) { return a.shared_len ? max(0, min(a.shared_len[b], L)) / kPage : 0; }

struct Four {
    int x[kPer];
};
SD_DEV Four load_four(const int32_t *p, int b, int B)
{
    Four f;
    if (b + kPer <= B) {
        const int4 v = *reinterpret_cast<const int4 *>(p + b);
        f = Four{v.x, v.y, v.z, v.w};
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) f.x[i] = b + i < B ? p[b + i] : 0;
    }
    return f;
}

SD_DEV void store_four(int32_t *p, int b, int B, const int (&x)[kPer])
{
    if (b + kPer <= B) {
        *reinterpret_cast<int4 *>(p + b) = int4{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (b + i < B) p[b + i] = x[i];
    }
}

// Sums over the workgroup's threads before this one; x becomes that, `all` the sums over all threads.
template <int N, int WAVES>
SD_DEV void scan(uint64_t (&x)[N], uint64_t (&all)[N], uint64_t (*s_wave)[N])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint64_t upto = wave_scan64(x[i]);
        if (lane == 63) s_wave[wave][i] = upto;
        x[i] = upto - x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint64_t upto = wave_scan64(lane < WAVES ? s_wave[lane][i] : 0);
        const uint64_t below = read_lane(upto, wave ? wave - 1 : 0);
        all[i] = read_lane(upto, 63);
        x[i] += wave ? below : 0;
    }
}

// The sums of every sequence, and what of the outputs has an entry per sequence.  put(b, ...) takes four sequences' first rows, first pages, pages that came
// back before, lengths and positions.
template <int THREADS, typename Put>
SD_DEV void sums(const PlanArgs &a, Put &&put, int &held, int64_t &back, int64_t &pages, int64_t &rows)
{
    constexpr int kWaves = THREADS / 64, kChunk = THREADS * kPer;
    __shared__ uint64_t s_three[kWaves][3], s_two[kWaves][2];
    held = max(0, min(a.free_in[0], a.num_pages));
    uint64_t all3[3], all2[2];
    const bool one_chunk = a.B <= kChunk;
    int64_t back_before = 0, asked_pages = 0, asked_rows = 0;
    back = pages = rows = 0;
    for (int pass = one_chunk; pass < 2; ++pass)   // of more sequences than the threads hold the pages that come back are counted first
        for (int b0 = 0; b0 < a.B; b0 += kChunk) {
            const int b = b0 + kPer * (int)threadIdx.x;
            const Four asks = load_four(a.new_tokens, b, a.B), lens = load_four(a.lens_in, b, a.B), shared = a.shared_len ? load_four(a.shared_len, b, a.B) : Four{},
                       nexts = a.next_in && pass ? load_four(a.next_in, b, a.B) : Four{};
            int L[kPer], n[kPer], need[kPer], returned[kPer];
            uint64_t x[3] = {0, 0, 0};
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                L[i] = length_of(a, lens.x[i]);
                returned[i] = asks.x[i] < 0 ? pages_of(L[i]) - max(0, min(shared.x[i], L[i])) / kPage : 0;
                n[i] = asks.x[i] > 0 && (int64_t)L[i] + asks.x[i] <= a.max_context_len ? asks.x[i] : 0;
                need[i] = pages_of(L[i] + n[i]) - pages_of(L[i]);
                x[0] += returned[i];
                x[1] += need[i];
                x[2] += n[i];
            }
            scan<3, kWaves>(x, all3, s_three);
            if (!pass || one_chunk) back += (int64_t)all3[0];
            if (!pass) continue;
            const int64_t available = held + back;
            int64_t back_at = back_before + (int64_t)x[0], page_sum = asked_pages + (int64_t)x[1], row_sum = asked_rows + (int64_t)x[2];
            back_before += (int64_t)all3[0];
            asked_pages += (int64_t)all3[1];
            asked_rows += (int64_t)all3[2];
            uint64_t y[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                page_sum += need[i];
                row_sum += n[i];
                if ((need[i] > 0 && page_sum > available) || row_sum > a.max_rows) n[i] = need[i] = 0;
                y[0] += need[i];
                y[1] += n[i];
            }
            scan<2, kWaves>(y, all2, s_two);
            int page[kPer], row[kPer], ends[kPer], next_ends[kPer];
            int64_t returned_before[kPer];
            int page_at = (int)(pages + (int64_t)y[0]), row_at = (int)(rows + (int64_t)y[1]);   // (of what is given; below 2^31)
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const bool done = asks.x[i] < 0;
                ends[i] = done ? 0 : L[i] + n[i];
                next_ends[i] = done ? 0 : nexts.x[i] + n[i];
                page[i] = page_at, row[i] = row_at, returned_before[i] = back_at;
                page_at += need[i];
                row_at += n[i];
                back_at += returned[i];
            }
            store_four(a.granted, b, a.B, n);
            store_four(a.starts, b, a.B, L);
            store_four(a.row_start, b, a.B, row);
            store_four(a.lens_out, b, a.B, ends);
            if (a.next_in) store_four(a.next_out, b, a.B, next_ends);
            put(b, row, page, returned_before, L, a.next_in ? nexts.x : L);
            pages += (int64_t)all2[0];
            rows += (int64_t)all2[1];
        }
    if (threadIdx.x == 0) {
        a.row_start[a.B] = (int)rows;
        a.free_out[0] = (int)min(held + back - pages, (int64_t)a.num_pages);
    }
}

// The last index of [0, n) whose entry is not above x, where entries ascend from 0.  Every `stride`-th is in LDS.
template <typename T>
SD_DEV int last_not_above(const T *s_from, const T *from, int stride, int n, T x)
{
    int lo = 0, hi = (n + stride - 1) / stride;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (s_from[mid] <= x) lo = mid;
        else hi = mid;
    }
    if (stride == 1) return lo;
    hi = min(n, (lo + 1) * stride);
    lo *= stride;
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (from[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Every `stride`-th of n entries into LDS, four loads of a thread on their way together.
template <typename T>
SD_DEV void hold(T *s_from, const T *from, int stride, int n)
{
    constexpr int kAtOnce = 4;
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += kAtOnce * 256) {
        T x[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) x[j] = from[min(i0 + j * 256 + (int)threadIdx.x, n - 1) * stride];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (i0 + j * 256 + (int)threadIdx.x < n) s_from[i0 + j * 256 + threadIdx.x] = x[j];
    }
}

// The i-th page of the list, where it came back: of sequence b, of length L.
SD_DEV int returned_page(const PlanArgs &a, int b, int L, int64_t nth) { return a.block_table[(int64_t)b * a.max_blocks + own_from(a, b, L) + nth]; }

}  // namespace

// A small call: all of it by one workgroup.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void plan_kernel(PlanArgs a)
{
    constexpr int kSums = THREADS * kPer;
    __shared__ int s_row[kSums], s_page[kSums], s_start[kSums], s_next[kSums];
    __shared__ int64_t s_back[kSums];
    const int tid = threadIdx.x;
    int held;
    int64_t back, pages, rows;
    sums<THREADS>(a, [&](int b, const int (&row)[kPer], const int (&page)[kPer], const int64_t (&returned)[kPer], const int (&L)[kPer], const int (&next)[kPer]) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) s_row[b + i] = row[i], s_page[b + i] = page[i], s_back[b + i] = returned[i], s_start[b + i] = L[i], s_next[b + i] = next[i];
    }, held, back, pages, rows);
    __syncthreads();
    for (int t = tid; t < a.max_rows; t += THREADS) {
        int b = -1, slot = 0, position = 0;
        if (t < rows) {
            b = last_not_above<int>(s_row, nullptr, 1, a.B, t);
            slot = s_start[b] + t - s_row[b];
            position = s_next[b] + t - s_row[b];
        }
        a.seq_ids[t] = b;
        a.slots[t] = slot;
        if (a.positions) a.positions[t] = position;
    }
    auto page_at = [&](int64_t i) {
        if (i < held) return a.free_pages[i];
        const int b = last_not_above<int64_t>(s_back, nullptr, 1, a.B, i - held);
        return returned_page(a, b, s_start[b], i - held - s_back[b]);
    };
    const int64_t available = held + back;
    for (int i = tid; i < pages; i += THREADS) {
        const int b = last_not_above<int>(s_page, nullptr, 1, a.B, i);
        a.block_table[(int64_t)b * a.max_blocks + pages_of(s_start[b]) + (i - s_page[b])] = page_at(available - 1 - i);
    }
    const int64_t left = min(available - pages, (int64_t)a.num_pages) - held;   // of the pages that came back
    constexpr int kAtOnce = 4;
    for (int64_t i0 = kAtOnce * tid; i0 < left; i0 += kAtOnce * THREADS) {   // (mostly of one sequence: found once)
        int b = last_not_above<int64_t>(s_back, nullptr, 1, a.B, i0), page[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i0 + j >= left) break;
            while (b + 1 < a.B && s_back[b + 1] <= i0 + j) ++b;
            page[j] = returned_page(a, b, s_start[b], i0 + j - s_back[b]);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (i0 + j < left) a.free_pages[held + i0 + j] = page[j];
    }
}

// A large one: the sums into the workspace,
template <int THREADS>
__global__ __launch_bounds__(THREADS) void plan_sums_kernel(PlanArgs a)
{
    int held;
    int64_t back, pages, rows;
    sums<THREADS>(a, [&](int b, const int (&)[kPer], const int (&page)[kPer], const int64_t (&returned)[kPer], const int (&)[kPer], const int (&next)[kPer]) {
        store_four(a.page_from, b, a.B, page);
        store_four(a.next_at, b, a.B, next);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (b + i < a.B) a.back_from[b + i] = returned[i];
    }, held, back, pages, rows);
    if (threadIdx.x == 0) {
        a.page_from[a.B] = (int)pages;
        a.back_from[a.B] = back;
        a.counts[0] = held;
    }
}

// then the entries: workgroups of 1024 rows, and behind those workgroups for pages, those that are taken and those that are left of the ones that came back.
__global__ __launch_bounds__(256) void plan_fill_kernel(PlanArgs a)
{
    __shared__ int s_from[kPlanHeld];
    __shared__ int64_t s_back[kPlanHeld];
    const int tid = threadIdx.x, row_blocks = (int)(((int64_t)a.max_rows + 1023) / 1024);
    const int stride = (a.B + kPlanHeld - 1) / kPlanHeld, sample = (a.B + stride - 1) / stride;
    if ((int)blockIdx.x < row_blocks) {
        const int rows = a.row_start[a.B];
        const int64_t row0 = (int64_t)blockIdx.x * 1024, t = row0 + kPer * tid;
        if (row0 < rows) {
            hold(s_from, a.row_start, stride, sample);
            __syncthreads();
        }
        if (t >= a.max_rows) return;
        int seq[kPer], slot[kPer], position[kPer];
        int b = -1, first = 0, end = 0, start = 0, next = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            seq[i] = -1;
            slot[i] = position[i] = 0;
            if (t + i >= rows) continue;
            if (b < 0 || t + i >= end) {
                b = last_not_above<int>(s_from, a.row_start, stride, a.B, (int)(t + i));
                first = a.row_start[b], end = a.row_start[b + 1], start = a.starts[b], next = a.next_at[b];
            }
            seq[i] = b;
            slot[i] = start + (int)(t + i - first);
            position[i] = next + (int)(t + i - first);
        }
        store_four(a.seq_ids, (int)t, a.max_rows, seq);
        store_four(a.slots, (int)t, a.max_rows, slot);
        if (a.positions) store_four(a.positions, (int)t, a.max_rows, position);
        return;
    }
    const int pages = a.page_from[a.B], held = a.counts[0];
    const int64_t back = a.back_from[a.B], available = held + back, left = min(available - pages, (int64_t)a.num_pages);
    const int64_t items = pages + max(left - held, (int64_t)0);
    const int64_t at = (int64_t)(blockIdx.x - row_blocks) * 256, step = (int64_t)(gridDim.x - row_blocks) * 256;
    if (at >= items) return;
    hold(s_from, a.page_from, stride, sample);
    if (back > 0) hold(s_back, a.back_from, stride, sample);
    __syncthreads();
    for (int64_t i = at + tid; i < items; i += step) {
        const int64_t place = i < pages ? available - 1 - i : held + i - pages;   // in the list
        const bool taken = i < pages, listed = place < held;
        // (both searches before the loads that they lead to)
        const int to = taken ? last_not_above<int>(s_from, a.page_from, stride, a.B, (int)i) : 0;
        const int from = listed ? 0 : last_not_above<int64_t>(s_back, a.back_from, stride, a.B, place - held);
        const int start = a.starts[to], first = a.page_from[to], length = a.starts[from];
        const int64_t returned = a.back_from[from];
        const int page = listed ? a.free_pages[place] : returned_page(a, from, length, place - held - returned);
        if (taken) a.block_table[(int64_t)to * a.max_blocks + pages_of(start) + (i - first)] = page;
        else a.free_pages[place] = page;
    }
}

hipError_t launch_plan(const PlanArgs &a, hipStream_t stream)
{
    // One workgroup is sooner while few pages come back, two kernels take the same whatever comes back.  us, one : two: 64 sequences 6.4 : 9.2, 3 of them finished with 900
    // pages 10.2 : 9.8, 6 with 7 k pages 22.6 : 9.9; 512 7.2 : 9.6; 1000 9.0 : 10.4, 100 of them finished with 6.5 k pages 35 : 10.5, 300 with 95 k 173 : 10.6.  In a rollout as
    // many pages come back as are taken, one in 16 tokens, though some steps see many, and the host does not know which: few sequences, one workgroup, which costs a step in
    // which long ones end up to 13 us; 257 to 1024 sequences, two kernels, which cost a step in which few end 1.4 to 2.4 us.
    if (a.B <= 256 && a.max_rows <= 1024) {
        hipLaunchKernelGGL((plan_kernel<256>), dim3(1), dim3(256), 0, stream, a);
    } else {
        if (a.B <= 256 * kPer) hipLaunchKernelGGL(plan_sums_kernel<256>, dim3(1), dim3(256), 0, stream, a);
        else if (a.B <= 512 * kPer) hipLaunchKernelGGL(plan_sums_kernel<512>, dim3(1), dim3(512), 0, stream, a);
        else hipLaunchKernelGGL(plan_sums_kernel<1024>, dim3(1), dim3(1024), 0, stream, a);
        // (pages: as many workgroups as might have one each, up to four to a compute unit)
        const int64_t row_blocks = ((int64_t)a.max_rows + 1023) / 1024, page_blocks = std::min<int64_t>(1024, (std::min<int64_t>(a.num_pages, (int64_t)a.B * a.max_blocks) + 255) / 256);
        hipLaunchKernelGGL(plan_fill_kernel, dim3((unsigned)(row_blocks + std::max<int64_t>(page_blocks, 1))), dim3(256), 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace sd
