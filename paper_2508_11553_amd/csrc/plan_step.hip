// Places for the new tokens of every sequence: pages, block table, lengths and the rows' slot map.
//
// First kernel, one workgroup: sums over the batch.  Pages that come back; pages and rows that are asked for, in the batch's order, which says
// who is served; pages and rows of those that are.  Second kernel: the entries, each by one thread, which finds its sequence in those sums.
// The free list is a stack; the pages that come back lie on top of it, so they are the first to be taken, and only what is left of them is written to it.
// Bound by latency: two launches and a workgroup's walk over the batch.
#include "logits.h"

namespace sd {

namespace {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

// Sum over the threads up to this one of two numbers; `all`: over all threads.
struct Pair {
    uint64_t x, y;
};
SD_DEV Pair scan_pair(Pair p, Pair *s_wave, Pair &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Pair upto{wave_scan64(p.x), wave_scan64(p.y)};
    __syncthreads();
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    all = Pair{0, 0};
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) upto.x += s_wave[w].x, upto.y += s_wave[w].y;
        all.x += s_wave[w].x;
        all.y += s_wave[w].y;
    }
    return upto;
}
SD_DEV int pages_of(int tokens) { return (int)(((int64_t)tokens + kPage - 1) / kPage); }

// The last index of [0, n) whose entry is not above x; entries ascend from 0.
template <typename T>
SD_DEV int last_not_above(const T *from, int n, T x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (from[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace

__global__ __launch_bounds__(kPlanThreads) void plan_sums_kernel(PlanArgs a)
{
    __shared__ Pair s_wave[kPlanWaves];
    const int tid = threadIdx.x;
    const int held = max(0, min(a.free_in[0], a.num_pages));
    auto length = [&](int b) { return max(0, min(a.lens_in[b], a.max_context_len)); };
    auto own_from = [&](int b, int L) { return a.shared_len ? max(0, min(a.shared_len[b], L)) / kPage : 0; };
    Pair all;
    // pages that come back
    int64_t back = 0;
    for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        const bool done = b < a.B && a.new_tokens[b] < 0;
        const int L = done ? length(b) : 0, n = done ? pages_of(L) - own_from(b, L) : 0;
        const Pair upto = scan_pair(Pair{(uint64_t)n, 0}, s_wave, all);
        if (b < a.B) a.back_from[b] = back + (int64_t)upto.x - n;
        back += (int64_t)all.x;
    }
    const int64_t available = held + back;
    int64_t asked_pages = 0, asked_rows = 0, pages = 0, rows = 0;
    for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        const bool some = b < a.B;
        const int L = some ? length(b) : 0, asks = some ? a.new_tokens[b] : 0;
        int n = asks > 0 && (int64_t)L + asks <= a.max_context_len ? asks : 0;
        int need = pages_of(L + n) - pages_of(L);
        const Pair asked = scan_pair(Pair{(uint64_t)need, (uint64_t)n}, s_wave, all);
        if ((need > 0 && asked_pages + (int64_t)asked.x > available) || asked_rows + (int64_t)asked.y > a.max_rows) n = need = 0;
        asked_pages += (int64_t)all.x;
        asked_rows += (int64_t)all.y;
        const Pair given = scan_pair(Pair{(uint64_t)need, (uint64_t)n}, s_wave, all);
        if (some) {
            const int next = a.next_in ? a.next_in[b] : 0;
            a.granted[b] = n;
            a.starts[b] = L;
            a.row_start[b] = (int)(rows + (int64_t)given.y - n);
            a.page_from[b] = (int)(pages + (int64_t)given.x - need);
            a.lens_out[b] = asks < 0 ? 0 : L + n;
            if (a.next_in) {
                a.next_at[b] = next;
                a.next_out[b] = asks < 0 ? 0 : next + n;
            }
        }
        pages += (int64_t)all.x;
        rows += (int64_t)all.y;
    }
    if (tid == 0) {
        a.row_start[a.B] = (int)rows;
        a.page_from[a.B] = (int)pages;
        a.back_from[a.B] = back;
        a.counts[0] = held;
        a.free_out[0] = (int)min(available - pages, (int64_t)a.num_pages);
    }
}

__global__ __launch_bounds__(256) void plan_fill_kernel(PlanArgs a)
{
    const int64_t step = (int64_t)gridDim.x * 256, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int rows = a.row_start[a.B], pages = a.page_from[a.B], held = a.counts[0];
    const int64_t back = a.back_from[a.B], available = held + back;
    for (int64_t t = at; t < a.max_rows; t += step) {
        int b = -1, slot = 0, position = 0;
        if (t < rows) {
            b = last_not_above(a.row_start, a.B, (int)t);
            const int nth = (int)t - a.row_start[b];
            slot = a.starts[b] + nth;
            position = a.next_in ? a.next_at[b] + nth : slot;
        }
        a.seq_ids[t] = b;
        a.slots[t] = slot;
        if (a.positions) a.positions[t] = position;
    }
    // the i-th page of the list, those that came back after those that were free
    auto page_at = [&](int64_t i) {
        if (i < held) return a.free_pages[i];
        const int b = last_not_above(a.back_from, a.B, i - held);
        const int L = a.starts[b], first = a.shared_len ? max(0, min(a.shared_len[b], L)) / kPage : 0;
        return a.block_table[(int64_t)b * a.max_blocks + first + (i - held - a.back_from[b])];
    };
    for (int64_t i = at; i < pages; i += step) {
        const int b = last_not_above(a.page_from, a.B, (int)i);
        a.block_table[(int64_t)b * a.max_blocks + pages_of(a.starts[b]) + (i - a.page_from[b])] = page_at(available - 1 - i);
    }
    const int64_t left = min(available - pages, (int64_t)a.num_pages);
    for (int64_t i = held + at; i < left; i += step) a.free_pages[i] = page_at(i);
}

hipError_t launch_plan(const PlanArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL(plan_sums_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
    const int64_t items = std::max<int64_t>(a.max_rows, a.B);
    hipLaunchKernelGGL(plan_fill_kernel, dim3((unsigned)std::min<int64_t>((items + 255) / 256, 2048)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sd
