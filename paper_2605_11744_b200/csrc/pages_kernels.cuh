// Pages handed out and taken back on the device: block tables, lengths, slot maps and positions from the lengths that requests
// ask for.  Integers only, and few of them: a decoding step's call is a launch and a chain of dependent reads (lengths, free
// list, table).  One block plans: who gives pages back, who gets some (first come, first served), by two prefix sums over the
// sequences.  Small calls are then filled in by the same block, from shared memory; larger ones by a second kernel with a grid
// over the sequences and their new rows.  64 sequences' steps and 48 prompts of up to 8192 rows (4.7 MB, mostly slots) take 8 us each.
#pragma once
#include <cstdint>

#include "decode_kernels.cuh"
#include "paged_cache.cuh"

namespace segattn {

constexpr int kPlanThreads = 1024;
constexpr int kPlanShared = 1024;  // sequences whose plans fit into shared memory
constexpr int kFillByPlanner = 4096;  // places in the slot map that the planning block fills in itself

struct PagePlan {
    int n_old, n_new;       // rows of the sequence before and after
    long long take, back;   // pages that sequences before it ask for, and give back
};

struct ResizeParams {
    const int32_t *want, *kv_len, *free_count, *pos_shift;
    int32_t *table, *free_pages;
    int32_t *kv_len_out, *free_count_out, *q_len;
    long long* slots;     // [B][Lq]
    int32_t* positions;   // [B][Lq]
    PagePlan* plan;       // [B]; unused where it fits into shared memory
    long long* counts;    // [3]: pages on the list before, with those given back, and after; unused like `plan`
    FastDiv f_page;
    int B, Lq, cap, n_pages, table_stride;
};

__device__ __forceinline__ int pages_for(const ResizeParams& p, int rows) { return (int)fdiv((uint32_t)rows + p.f_page.d - 1, p.f_page); }

// Sums of two numbers over the block's threads, and over those before this one.  In 64 bits: lengths that make no sense may add up
// past 32.
struct Pair {
    long long x, y;
};
__device__ __forceinline__ Pair block_scan(Pair v, Pair* total, Pair* red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    auto scan = [&](Pair s) {
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, s.x, k), y = __shfl_up_sync(0xffffffffu, s.y, k);
            if (lane >= k) {
                s.x += x;
                s.y += y;
            }
        }
        return s;
    };
    const Pair incl = scan(v);
    __syncthreads();
    if (lane == 31) red[warp] = incl;
    __syncthreads();
    const Pair all = scan(lane < warps ? red[lane] : Pair{0, 0});
    total->x = __shfl_sync(0xffffffffu, all.x, 31);
    total->y = __shfl_sync(0xffffffffu, all.y, 31);
    const long long x = __shfl_sync(0xffffffffu, all.x, warp ? warp - 1 : 0), y = __shfl_sync(0xffffffffu, all.y, warp ? warp - 1 : 0);
    return Pair{incl.x - v.x + (warp ? x : 0), incl.y - v.y + (warp ? y : 0)};
}

// What a sequence asks for, checked: its rows before and after (equal where a number is out of range).
__device__ __forceinline__ void asked(const ResizeParams& p, int b, int* n_old, int* n_new) {
    const int n = p.kv_len[b], w = p.want[b];
    *n_old = n;
    *n_new = w;
    const bool bad_n = n < 0 || n > p.cap;
    if (bad_n || w < 0 || w > p.cap || w - n > p.Lq) {
        refuse_input(bad_n ? 30 : 37);
        *n_new = n;
        if (bad_n) *n_old = *n_new = -1;
    }
}

// The whole plan, by one block.
__device__ __forceinline__ void plan_pages(const ResizeParams& p, PagePlan* plan, Pair* red, long long* counts) {
    const int tid = threadIdx.x, threads = blockDim.x;
    int count = *p.free_count;
    if (count < 0 || count > p.n_pages) {
        if (tid == 0) refuse_input(38);
        count = min(max(count, 0), p.n_pages);
    }
    auto pages = [&](int rows) { return rows < 0 ? 0 : pages_for(p, rows); };
    long long there = count;  // pages on the list, those given back among them
    if (p.B > threads) {  // else one scan gives their number as well
        Pair back{0, 0}, total;
        for (int b = tid; b < p.B; b += threads) {
            int o, n;
            asked(p, b, &o, &n);
            back.y += max(pages(o) - pages(n), 0);
        }
        block_scan(back, &total, red);
        there = count + total.y;
    }
    Pair before{0, 0};
    for (int b0 = 0; b0 < p.B; b0 += threads) {
        const int b = b0 + tid;
        int o = 0, n = 0;
        if (b < p.B) asked(p, b, &o, &n);
        const int more = pages(n) - pages(o), t = max(more, 0);
        Pair sum;
        Pair at = block_scan(Pair{t, max(-more, 0)}, &sum, red);
        at.x += before.x;
        at.y += before.y;
        before.x += sum.x;
        before.y += sum.y;
        if (p.B <= threads) there = count + sum.y;
        const bool served = t == 0 || at.x + t <= there;
        if (!served && at.x <= there) counts[2] = there - at.x;  // the first that has to wait: what those before it leave
        if (b < p.B) {
            if (!served) n = o;
            plan[b] = PagePlan{o, n, at.x, at.y};
            p.kv_len_out[b] = o < 0 ? p.kv_len[b] : n;
            p.q_len[b] = max(n - o, 0);
        }
    }
    if (tid == 0 && before.x <= there) counts[2] = there - before.x;
    __syncthreads();
    if (tid == 0) {
        const long long left = counts[2];
        counts[0] = count;
        counts[1] = there;
        if (left > p.n_pages) refuse_input(38);
        *p.free_count_out = (int)min(left, (long long)p.n_pages);
    }
}

// Sequence b, by the threads i0, i0 + step, ...
__device__ __forceinline__ void fill_sequence(const ResizeParams& p, const PagePlan* plan, const long long* counts, int b, int i0, int step) {
    const PagePlan q = plan[b];
    const int have = q.n_old < 0 ? 0 : pages_for(p, q.n_old), need = q.n_new < 0 ? 0 : pages_for(p, q.n_new);
    const long long count = counts[0], there = counts[1], left = counts[2];
    int32_t* row = p.table + (long long)b * p.table_stride;
    // The list is the pages that were on it and then those given back, sequence after sequence; pages are taken from its end.
    auto taken_page = [&](int i) {
        const long long v = there - 1 - q.take - i;
        if (v < count) return p.free_pages[v];
        int lo = 0, hi = p.B - 1;  // the last sequence with `back` at most v - count that gives something back
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (plan[mid].back <= v - count) lo = mid;
            else hi = mid - 1;
        }
        return p.table[(long long)lo * p.table_stride + pages_for(p, plan[lo].n_new) + (v - count - plan[lo].back)];
    };
    for (int i = i0; i < need - have; i += step) {
        const int page = taken_page(i);
        const bool fine = (unsigned)page < (unsigned)p.n_pages;
        if (!fine) refuse_input(33);
        row[have + i] = fine ? page : -1;
    }
    for (int i = i0; i < have - need; i += step) {
        const long long at = count + q.back + i;
        const int page = row[need + i];
        if ((unsigned)page >= (unsigned)p.n_pages) refuse_input(33);
        if (at < left && at < p.n_pages) p.free_pages[at] = page;
    }
    const int grown = q.n_new - q.n_old;
    int shift = p.pos_shift ? p.pos_shift[b] : 0;
    if (shift < 0 || (grown > 0 && shift > 0x7fffffff - (q.n_new - 1))) {  // or one that brings a position past its type
        if (i0 == 0) refuse_input(32);
        shift = 0;
    }
    for (int t = i0; t < p.Lq; t += step) {
        long long slot = -1;
        if (t < grown) {
            const int s = q.n_old + t, k = (int)fdiv((uint32_t)s, p.f_page);
            const int page = k < have ? row[k] : taken_page(k - have);
            if ((unsigned)page < (unsigned)p.n_pages) slot = (long long)page * p.f_page.d + (s - k * (int)p.f_page.d);
            else refuse_input(33);
        }
        p.slots[(long long)b * p.Lq + t] = slot;
        p.positions[(long long)b * p.Lq + t] = t < grown ? q.n_old + t + shift : 0;
    }
}

// FILL: the same block does the second part, a warp to a sequence, with the plan in shared memory.
template <bool FILL>
__global__ void __launch_bounds__(kPlanThreads) pages_plan_kernel(const ResizeParams p) {
    __shared__ Pair red[32];
    __shared__ long long counts[3];
    extern __shared__ uint8_t plan_smem[];
    PagePlan* shared_plan = reinterpret_cast<PagePlan*>(plan_smem);
    next_kernel_may_start();
    if (!FILL) {
        plan_pages(p, p.plan, red, p.counts);
        return;
    }
    plan_pages(p, shared_plan, red, counts);
    __syncthreads();
    for (int b = threadIdx.x >> 5; b < p.B; b += blockDim.x >> 5) fill_sequence(p, shared_plan, counts, b, threadIdx.x & 31, 32);
}

__global__ void __launch_bounds__(256) pages_fill_kernel(const ResizeParams p) {
    const int b = blockIdx.y;
    after_previous_kernel();
    fill_sequence(p, p.plan, p.counts, b, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

}  // namespace segattn
