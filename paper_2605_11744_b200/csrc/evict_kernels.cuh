// Eviction from the paged cache by accumulated attention weight: per (sequence, KV head) a selection of the slots to
// keep, then a copy of their rows to other pages.
#pragma once
#include <cstdint>

#include "paged_cache.cuh"

namespace segattn {

struct EvictParams {
    PagedView c;
    const float* weights;  // [B][Hkv][W]
    float* weights_out;    // [B][Hkv][W]
    int32_t* idx;          // [B][Hkv][budget]
    const int32_t* dst_table;
    int32_t *kv_len_out, *pos_shift_out;
    int W, sink, recent, heavy, budget;
    int dst_stride;
    int d16, d16_log;      // 16-byte pieces of a cache row
    int keys;              // keys a block of the selection has room for
    FastDiv f_heads;       // division by Hkv
};

// Order of the weights as unsigned numbers: NaN lowest, -0 equal to +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// ---- thread-block clusters -----------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// Every thread of every block of the cluster; writes to shared memory before it are seen after it.
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t load_from_block(const uint32_t* shared, uint32_t rank) {
    uint32_t addr, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(shared)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

constexpr int kEvictThreads = 1024;
constexpr int kEvictKeys = 40960;   // keys a block keeps in shared memory; more are read again from L2 in every pass
constexpr int kEvictAhead = 8;      // weights a thread has in flight
constexpr int kEvictBins = 2048;
constexpr int kEvictStatic = 3 * kEvictBins * 4;

// One cluster of up to eight blocks per (KV head, sequence), each with a contiguous slice of the slots between the sink and
// the recent rows.  The heavy-th largest key by a radix selection of 11, 11 and 10 bits, the blocks' histograms added up
// through distributed shared memory; then the kept slots written in ascending order, each warp with a segment of its block's
// slice, after one scan over the segments' counts.  Bound by the instructions of the passes over the keys and the barriers
// between them, not by the one read of the weights: 33 us for 128 heads of 26K slots.  Keys are taken four at a time once they
// are in shared memory, and a histogram's warp looks for one common bin over all of its keys at once (19.1M -> 13.8M
// instructions, 38 -> 33 us); re-reading the weights in every pass and scanning 1024 slots at a time it was 95.
__global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(const EvictParams prm) {
    extern __shared__ uint32_t evict_smem[];
    uint32_t* hist = evict_smem;                    // [3][kEvictBins]
    uint32_t* keys = evict_smem + 3 * kEvictBins;   // [prm.keys]
    __shared__ uint32_t scan[32], seg_gt[32], seg_eq[32], found[2], totals[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int CS = (int)cluster_size(), rank = (int)cluster_rank(), unit = blockIdx.x / CS;
    const int b = unit / prm.c.Hkv;
    const int n = seq_len(prm.c, b);
    const float* w = prm.weights + (long long)unit * prm.W;
    float* w_out = prm.weights_out + (long long)unit * prm.W;
    int32_t* out = prm.idx + (long long)unit * prm.budget;
    const int t0 = rank * kEvictThreads + tid, step = CS * kEvictThreads;
    const bool all = n <= prm.budget;
    // rows kept whatever they weigh, and the zeros behind the kept ones
    auto keep_the_rest = [&]() {
        const int kept = all ? n : prm.budget, front = all ? n : prm.sink, gap = all ? 0 : prm.heavy;
        for (int i = t0; i < kept - gap; i += step) {
            const int r = i < front ? i : i + gap, src = i < front ? i : n - kept + r;
            out[r] = src;
            w_out[r] = w[src];
        }
        for (int r = kept + t0; r < prm.budget; r += step) out[r] = -1;
#pragma unroll 4
        for (int r = kept + t0; r < prm.W; r += step) w_out[r] = 0.f;
    };
    if (all || prm.heavy == 0) {
        keep_the_rest();
        return;
    }

    const int m0 = prm.sink, len = n - prm.recent - m0;  // the slots between: more than `heavy` of them, since n > budget
    const int slice = ((len + CS - 1) / CS + 31) & ~31, a = min(rank * slice, len), cnt = min(slice, len - a);
    const float* mine = w + m0 + a;
    const bool cached = cnt <= prm.keys;
    // four keys from index i on (a multiple of four); what lies behind the slice's end counts as no key
    const int n4 = (cnt + 3) / 4;
    auto keys_at = [&](int i4, uint32_t (&k)[4]) {
        if (cached) {
            const uint4 v = reinterpret_cast<const uint4*>(keys)[i4];
            k[0] = v.x;
            k[1] = v.y;
            k[2] = v.z;
            k[3] = v.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) k[e] = 4 * i4 + e < cnt ? weight_key(mine[4 * i4 + e]) : 0u;
        }
    };
    auto there = [&](int i4, int e) { return 4 * i4 + e < cnt; };
    for (int i = tid; i < 3 * kEvictBins; i += kEvictThreads) hist[i] = 0;
    __syncthreads();
    uint32_t prefix = 0, need = prm.heavy;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        uint32_t* mh = hist + pass * kEvictBins;
        // N keys of each lane into the histogram.  A warp whose keys all fall into one bin (zeros that nothing ever looked at)
        // adds them at once.
        auto count = [&](auto& k, const uint32_t in) {
            constexpr int N = sizeof(k) / sizeof(k[0]);
            const uint32_t mask = (1u << bits) - 1, b0 = (k[0] >> shift) & mask;
            bool same = in == (1u << N) - 1;
#pragma unroll
            for (int e = 1; e < N; ++e) same = same && ((k[e] >> shift) & mask) == b0;
            const uint32_t lead = __shfl_sync(0xffffffffu, b0, 0);  // by every lane, before anything that only some evaluate
            if (__all_sync(0xffffffffu, same && b0 == lead)) {
                if (lane == 0) atomicAdd(mh + b0, 32u * N);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if ((in >> e) & 1) atomicAdd(mh + ((k[e] >> shift) & mask), 1u);
            }
        };
        if (pass == 0) {
            for (int i0 = 0; i0 < cnt; i0 += kEvictAhead * kEvictThreads) {
                float x[kEvictAhead];
#pragma unroll
                for (int y = 0; y < kEvictAhead; ++y) x[y] = i0 + y * kEvictThreads + tid < cnt ? mine[i0 + y * kEvictThreads + tid] : 0.f;
                uint32_t k[kEvictAhead], in = 0;
#pragma unroll
                for (int y = 0; y < kEvictAhead; ++y) {
                    const int i = i0 + y * kEvictThreads + tid;
                    k[y] = weight_key(x[y]);
                    if (i < cnt) {
                        in |= 1u << y;
                        if (cached) keys[i] = k[y];
                    }
                }
                count(k, in);
            }
        } else {
            // few keys share the leading bits found so far: most warps only look
            for (int i = tid; i - tid < n4; i += kEvictThreads) {
                uint32_t k[4];
                uint32_t in = 0;
                if (i < n4) {
                    keys_at(i, k);
#pragma unroll
                    for (int e = 0; e < 4; ++e) in |= ((k[e] >> (shift + bits)) == prefix && there(i, e) ? 1u : 0u) << e;
                }
                if (__any_sync(0xffffffffu, in)) count(k, in);
            }
        }
        __syncthreads();
        if (CS > 1) cluster_sync();
        // bins from the top down: thread t has bins 2047 - 2 t and 2046 - 2 t
        uint32_t c[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t* at = mh + kEvictBins - 1 - 2 * tid - k;
            c[k] = CS == 1 ? *at : 0u;
            if (CS > 1) {
                uint32_t v[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = r < CS ? load_from_block(at, r) : 0u;
#pragma unroll
                for (int r = 0; r < 8; ++r) c[k] += v[r];
            }
        }
        uint32_t before = c[0] + c[1];
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, before, x);
            if (lane >= x) before += y;
        }
        if (lane == 31) scan[warp] = before;
        before -= c[0] + c[1];
        __syncthreads();
        before += __reduce_add_sync(0xffffffffu, lane < warp ? scan[lane] : 0u);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (need > before && need <= before + c[k]) {
                found[0] = kEvictBins - 1 - 2 * tid - k;
                found[1] = need - before;
            }
            before += c[k];
        }
        __syncthreads();
        prefix = (prefix << bits) | found[0];
        need = found[1];
    }
    // keys above `prefix` are all kept, of those equal to it the first `need`
    const int seg = ((n4 + 31) / 32 + 31) & ~31, s0 = min(warp * seg, n4), s1 = min(s0 + seg, n4);  // in fours
    uint32_t gt = 0, eq = 0;
    for (int i = s0 + lane; i < s1; i += 32) {
        uint32_t k[4];
        keys_at(i, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            gt += there(i, e) && k[e] > prefix;
            eq += there(i, e) && k[e] == prefix;
        }
    }
    gt = __reduce_add_sync(0xffffffffu, gt);
    eq = __reduce_add_sync(0xffffffffu, eq);
    if (lane == 0) {
        seg_gt[warp] = gt;
        seg_eq[warp] = eq;
    }
    __syncthreads();
    uint32_t gt_before = __reduce_add_sync(0xffffffffu, lane < warp ? seg_gt[lane] : 0u);
    uint32_t eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? seg_eq[lane] : 0u);
    const uint32_t gt_all = __reduce_add_sync(0xffffffffu, seg_gt[lane]), eq_all = __reduce_add_sync(0xffffffffu, seg_eq[lane]);
    if (CS > 1) {
        if (tid == 0) {
            totals[0] = gt_all;
            totals[1] = eq_all;
        }
        cluster_sync();
        for (int r = 0; r < rank; ++r) {
            gt_before += load_from_block(totals, r);
            eq_before += load_from_block(totals + 1, r);
        }
    }
    uint32_t at = prm.sink + gt_before + min(eq_before, need);
    for (int i = s0 + lane; i - lane < s1; i += 32) {
        uint32_t k[4], keep = 0, equal = 0;
        const uint32_t below = (1u << lane) - 1;
        if (i < s1) {
            keys_at(i, k);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                keep |= (there(i, e) && k[e] > prefix ? 1u : 0u) << e;
                equal |= (there(i, e) && k[e] == prefix ? 1u : 0u) << e;
            }
        }
        if (__any_sync(0xffffffffu, equal)) {
            // ranks among the equal ones: lane after lane, four slots each
            uint32_t before = eq_before, total = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t b = __ballot_sync(0xffffffffu, (equal >> e) & 1);
                before += __popc(b & below);
                total += __popc(b);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if ((equal >> e) & 1) keep |= (before++ < need ? 1u : 0u) << e;
            eq_before += total;
        }
        uint32_t r = at, total = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t b = __ballot_sync(0xffffffffu, (keep >> e) & 1);
            r += __popc(b & below);
            total += __popc(b);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if ((keep >> e) & 1) {
                out[r] = m0 + a + 4 * i + e;
                w_out[r++] = mine[4 * i + e];
            }
        at += total;
    }
    keep_the_rest();
    if (CS > 1) cluster_sync();  // no block leaves while another may still read its shared memory
}

// Row r of the compacted cache from slot idx[b][h][r]: a thread moves 16 bytes of K and of V for four rows, whose reads are
// all in flight together (205 -> 160 us for 16 x 8 heads of 8036 rows against one row a thread; 1.05 GB).  Runs after the selection's end; the new
// lengths and shifts are written here and not there because kv_len_out may be kv_len, which the selection's blocks read.
constexpr int kMoveRows = 4;
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictParams prm) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.y;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        const int n = seq_len(prm.c, b), m = min(n, prm.budget), s = shift_of(prm.c, b);
        prm.kv_len_out[b] = m;
        prm.pos_shift_out[b] = s + n - m;
    }
    const uint32_t i = blockIdx.x * 256 + threadIdx.x, e = i & (prm.d16 - 1), u = i >> prm.d16_log;
    const uint32_t r4 = fdiv(u, prm.f_heads);
    const int h = (int)(u - r4 * prm.c.Hkv), r0 = (int)r4 * kMoveRows;
    if (r0 >= prm.budget) return;
    int src[kMoveRows];
    const int32_t* idx = prm.idx + ((long long)b * prm.c.Hkv + h) * prm.budget;
#pragma unroll
    for (int k = 0; k < kMoveRows; ++k) src[k] = r0 + k < prm.budget ? idx[r0 + k] : -1;
    uint4 kx[kMoveRows], vx[kMoveRows];
#pragma unroll
    for (int k = 0; k < kMoveRows; ++k) {
        int row, page = -1;
        if (src[k] >= 0) page = page_of(prm.c, b, src[k], &row);
        kx[k] = vx[k] = make_uint4(0, 0, 0, 0);
        if (page >= 0) {
            kx[k] = *reinterpret_cast<const uint4*>(prm.c.K + page * prm.c.k_stride[0] + row * prm.c.k_stride[1] + h * prm.c.k_stride[2] + 16 * e);
            vx[k] = *reinterpret_cast<const uint4*>(prm.c.V + page * prm.c.v_stride[0] + row * prm.c.v_stride[1] + h * prm.c.v_stride[2] + 16 * e);
        }
    }
#pragma unroll
    for (int k = 0; k < kMoveRows; ++k) {
        if (src[k] < 0) continue;
        const int entry = (int)fdiv((uint32_t)(r0 + k), prm.c.f_page), row = r0 + k - entry * (int)prm.c.f_page.d;
        const int to = prm.dst_table[(long long)b * prm.dst_stride + entry];
        if ((unsigned)to >= (unsigned)prm.c.n_pages) {
            if (e == 0) refuse_input(36);
            continue;
        }
        *reinterpret_cast<uint4*>(prm.c.K + to * prm.c.k_stride[0] + row * prm.c.k_stride[1] + h * prm.c.k_stride[2] + 16 * e) = kx[k];
        *reinterpret_cast<uint4*>(prm.c.V + to * prm.c.v_stride[0] + row * prm.c.v_stride[1] + h * prm.c.v_stride[2] + 16 * e) = vx[k];
    }
}

}  // namespace segattn
