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
    int d16;               // 16-byte pieces of a cache row
};

// Order of the weights as unsigned numbers: NaN lowest, -0 equal to +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int kEvictThreads = 1024;

// One block per (KV head, sequence).  The threshold (the heavy-th largest key between the sink and the recent rows) by
// a radix selection of eight bits a pass, then the kept slots written out in ascending order.
__global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(const EvictParams prm) {
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int n = seq_len(prm.c, b);
    const long long unit = (long long)b * prm.c.Hkv + h;
    const float* w = prm.weights + unit * prm.W;
    int32_t* out = prm.idx + unit * prm.budget;
    if (n <= prm.budget) {
        for (int r = tid; r < prm.budget; r += kEvictThreads) out[r] = r < n ? r : -1;
        return;
    }
    __shared__ uint32_t hist[256];
    __shared__ uint32_t s_prefix, s_need;
    const int m0 = prm.sink, m1 = n - prm.recent;  // the slots between: more than `heavy` of them, since n > budget
    uint32_t prefix = 0, need = prm.heavy;
    for (int shift = 24; need > 0 && shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kEvictThreads) hist[i] = 0;
        __syncthreads();
        for (int j = m0 + tid; j < m1; j += kEvictThreads) {
            const uint32_t k = weight_key(w[j]);
            if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            uint32_t left = need;
            int bin = 255;
            while (bin > 0 && hist[bin] < left) left -= hist[bin--];
            s_prefix = (prefix << 8) | (uint32_t)bin;
            s_need = left;
        }
        __syncthreads();
        prefix = s_prefix;
        need = s_need;
    }
    // keys above `prefix` are all kept, of those equal to it the first `need` (heavy == 0: none)
    __shared__ uint32_t warp_sum[32];
    uint32_t kept = 0, equal = 0;
    for (int base = 0; base < n; base += kEvictThreads) {
        const int j = base + tid;
        bool keep = false, eq = false;
        if (j < n) {
            if (j < m0 || j >= m1) keep = true;
            else if (prm.heavy > 0) {
                const uint32_t k = weight_key(w[j]);
                keep = k > prefix;
                eq = k == prefix;
            }
        }
        // rank of the equal ones first, then of all kept ones
        const int lane = tid & 31, wid = tid >> 5;
        const uint32_t beq = __ballot_sync(0xffffffffu, eq);
        if (lane == 0) warp_sum[wid] = __popc(beq);
        __syncthreads();
        uint32_t before = equal, total = 0;
        for (int k = 0; k < 32; ++k) {
            if (k < wid) before += warp_sum[k];
            total += warp_sum[k];
        }
        equal += total;
        if (eq) keep = before + __popc(beq & ((1u << lane) - 1)) < need;
        __syncthreads();
        const uint32_t bk = __ballot_sync(0xffffffffu, keep);
        if (lane == 0) warp_sum[wid] = __popc(bk);
        __syncthreads();
        before = kept;
        total = 0;
        for (int k = 0; k < 32; ++k) {
            if (k < wid) before += warp_sum[k];
            total += warp_sum[k];
        }
        kept += total;
        if (keep) out[before + __popc(bk & ((1u << lane) - 1))] = j;
        __syncthreads();
    }
}

// Row r of the compacted cache from slot idx[b][h][r]: one thread per 16 bytes (K and V both).
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictParams prm) {
    const long long n = (long long)prm.c.B * prm.budget * prm.c.Hkv * prm.d16;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int e = (int)(i % prm.d16);
    const int h = (int)((i / prm.d16) % prm.c.Hkv);
    const int r = (int)((i / ((long long)prm.d16 * prm.c.Hkv)) % prm.budget);
    const int b = (int)(i / ((long long)prm.d16 * prm.c.Hkv * prm.budget));
    const int src = prm.idx[((long long)b * prm.c.Hkv + h) * prm.budget + r];
    if (src < 0) return;
    int row, to_row;
    const int page = page_of(prm.c, b, src, &row);
    const int entry = (int)fdiv((uint32_t)r, prm.c.f_page);
    to_row = r - entry * (int)prm.c.f_page.d;
    const int to = prm.dst_table[(long long)b * prm.dst_stride + entry];
    if ((unsigned)to >= (unsigned)prm.c.n_pages) {
        if (e == 0) refuse_input(36);
        return;
    }
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (page >= 0) {
        k = *reinterpret_cast<const uint4*>(prm.c.K + page * prm.c.k_stride[0] + row * prm.c.k_stride[1] + h * prm.c.k_stride[2] + 16 * e);
        v = *reinterpret_cast<const uint4*>(prm.c.V + page * prm.c.v_stride[0] + row * prm.c.v_stride[1] + h * prm.c.v_stride[2] + 16 * e);
    }
    *reinterpret_cast<uint4*>(prm.c.K + to * prm.c.k_stride[0] + to_row * prm.c.k_stride[1] + h * prm.c.k_stride[2] + 16 * e) = k;
    *reinterpret_cast<uint4*>(prm.c.V + to * prm.c.v_stride[0] + to_row * prm.c.v_stride[1] + h * prm.c.v_stride[2] + 16 * e) = v;
}

// weights_out = the kept slots' weights, then zeros; and, by the first threads, the new lengths and shifts (here and
// not in the selection: kv_len_out may be kv_len, which the selection's blocks read).
__global__ void __launch_bounds__(256) evict_finish_kernel(const EvictParams prm) {
    const long long units = (long long)prm.c.B * prm.c.Hkv;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i < prm.c.B) {
        const int b = (int)i, n = seq_len(prm.c, b), m = min(n, prm.budget), s = shift_of(prm.c, b);
        prm.kv_len_out[b] = m;
        prm.pos_shift_out[b] = s + n - m;
    }
    if (i >= units * prm.W) return;
    const int j = (int)(i % prm.W);
    const long long unit = i / prm.W;
    float x = 0.f;
    if (j < prm.budget) {
        const int src = prm.idx[unit * prm.budget + j];
        if (src >= 0) x = prm.weights[unit * prm.W + src];
    }
    prm.weights_out[i] = x;
}

}  // namespace segattn
