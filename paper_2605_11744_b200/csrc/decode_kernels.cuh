// Attention of a sequence's newest rows over its paged cache.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "paged_cache.cuh"

namespace segattn {

struct DecodeParams {
    PagedView c;
    const __nv_bfloat16* Q;
    __nv_bfloat16* O;
    float* LSE;                      // [B][Hq][Lq]
    const float* w_in;               // [B][Hkv][W] or null
    float* w_out;                    // or null
    const float *k_scale, *v_scale;  // e4m3 only
    long long q_stride[3], o_stride[3];
    FastDiv f_S;
    int S, T, W, Hq, g;
    float scale_log2;                // sm_scale * log2(e)
    uint8_t head_class[64];
};

// Slots [lo, hi) that new row t of sequence b sees through a KV head of class cls.
__device__ __forceinline__ void visible_slots(const DecodeParams& p, int n, int rows, int shift, int t, int cls, int* lo, int* hi) {
    const int slot = n - rows + t;
    *hi = slot + 1;
    *lo = 0;
    if (cls != kHeadPast && slot >= 0) {
        const uint32_t pos = (uint32_t)slot + (uint32_t)shift;
        long long start = (long long)fdiv(pos, p.f_S) * p.S;
        if (cls == kHeadLocal) start = max(0ll, start - p.T);
        *lo = (int)max(0ll, start - shift);
    }
}

template <bool FP8>
__device__ __forceinline__ float cache_value(const char* row, int e) {
    if (FP8) return float(reinterpret_cast<const __nv_fp8_e4m3*>(row)[e]);
    return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[e]);
}

// One block per (new row, query head, sequence): each warp walks every eighth key with its own running maximum and sum.
template <int D, bool FP8>
__global__ void __launch_bounds__(256) decode_kernel(const DecodeParams p) {
    const int t = blockIdx.x, hq = blockIdx.y, b = blockIdx.z;
    const int rows = new_rows(p.c, b);
    if (t >= rows) return;
    const int h = hq / p.g, n = seq_len(p.c, b), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int lo, hi;
    visible_slots(p, n, rows, shift_of(p.c, b), t, p.head_class[h], &lo, &hi);
    constexpr int E = D / 32;
    float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
    const float ks = FP8 ? p.k_scale[h] : 1.f, vs = FP8 ? p.v_scale[h] : 1.f;
    for (int k = 0; k < E; ++k)
        q[k] = __bfloat162float(p.Q[b * p.q_stride[0] + t * p.q_stride[1] + hq * p.q_stride[2] + lane * E + k]);
    for (int j = lo + warp; j < hi; j += 8) {
        int row;
        const int page = page_of(p.c, b, j, &row);
        if (page < 0) continue;
        const char* kr = p.c.K + page * p.c.k_stride[0] + row * p.c.k_stride[1] + h * p.c.k_stride[2];
        const char* vr = p.c.V + page * p.c.v_stride[0] + row * p.c.v_stride[1] + h * p.c.v_stride[2];
        float s = 0.f;
        for (int k = 0; k < E; ++k) s += q[k] * cache_value<FP8>(kr, lane * E + k);
        for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= p.scale_log2 * ks;
        const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn, w = exp2f(s - base), f = exp2f(m - base);
        l = l * f + w;
        for (int k = 0; k < E; ++k) o[k] = o[k] * f + w * cache_value<FP8>(vr, lane * E + k);
        m = mn;
    }
    __shared__ float sm[8], sl[8], so[8][D];
    if (lane == 0) {
        sm[warp] = m;
        sl[warp] = l;
    }
    for (int k = 0; k < E; ++k) so[warp][lane * E + k] = o[k];
    __syncthreads();
    float M = -INFINITY, L = 0.f;
    for (int k = 0; k < 8; ++k) M = fmaxf(M, sm[k]);
    const float base = M == -INFINITY ? 0.f : M;
    for (int k = 0; k < 8; ++k) L += sl[k] * exp2f(sm[k] - base);
    if (threadIdx.x == 0) p.LSE[((long long)b * p.Hq + hq) * p.c.Lq + t] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
    for (int e = threadIdx.x; e < D; e += 256) {
        float x = 0.f;
        for (int k = 0; k < 8; ++k) x += so[k][e] * exp2f(sm[k] - base);
        p.O[b * p.o_stride[0] + t * p.o_stride[1] + hq * p.o_stride[2] + e] = __float2bfloat16(L == 0.f ? 0.f : x / L * vs);
    }
}

// Attention weight of every slot, from the LSE: one warp per slot.
template <int D, bool FP8>
__global__ void __launch_bounds__(256) decode_weights_kernel(const DecodeParams p) {
    const int j = blockIdx.x * 8 + (threadIdx.x >> 5), h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 31;
    const int rows = new_rows(p.c, b), n = seq_len(p.c, b), shift = shift_of(p.c, b);
    if (j >= n || rows == 0) return;
    constexpr int E = D / 32;
    float k[E], sum = 0.f;
    int row;
    const int page = page_of(p.c, b, j, &row);
    if (page >= 0) {
        const char* kr = p.c.K + page * p.c.k_stride[0] + row * p.c.k_stride[1] + h * p.c.k_stride[2];
        for (int e = 0; e < E; ++e) k[e] = cache_value<FP8>(kr, lane * E + e);
        for (int t = 0; t < rows; ++t) {
            int lo, hi;
            visible_slots(p, n, rows, shift, t, p.head_class[h], &lo, &hi);
            if (j < lo || j >= hi) continue;
            for (int hq = h * p.g; hq < (h + 1) * p.g; ++hq) {
                float s = 0.f;
                const __nv_bfloat16* q = p.Q + b * p.q_stride[0] + t * p.q_stride[1] + hq * p.q_stride[2] + lane * E;
                for (int e = 0; e < E; ++e) s += __bfloat162float(q[e]) * k[e];
                for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
                const float lse = p.LSE[((long long)b * p.Hq + hq) * p.c.Lq + t];
                if (lse != -INFINITY) sum += exp2f(s * (p.scale_log2 * (FP8 ? p.k_scale[h] : 1.f)) - lse * 1.4426950408889634f);
            }
        }
    }
    if (lane == 0) {
        const long long at = ((long long)b * p.c.Hkv + h) * p.W + j;
        p.w_out[at] = (p.w_in ? p.w_in[at] : 0.f) + sum;
    }
}

}  // namespace segattn
