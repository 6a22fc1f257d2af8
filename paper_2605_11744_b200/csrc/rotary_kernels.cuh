// Rotary positions in general form: both pairings, part of the head, scaled frequencies, rows at positions of their own.
// y = a Rot(p) x on the pairs of the first rot_dim elements, the rest copied.  All of it is a stream over HBM; a thread
// takes 16 elements of a head row (eight pairs) for a few heads of the same row, so that the table entry it reads (64
// bytes of cosines and sines for 32 bytes of data) is read once for those heads.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "paged_cache.cuh"

namespace segattn {

struct RopeFreq {
    double base, factor, trained_len, turns_lo, turns_hi, amplitude;
    int kind;  // SEGATTN_ROPE_*
};

// table[pos][i] = a (cos, sin)(pos * w_i): angles and their cosines and sines in double, rounded once to fp32 (an
// angle of 10^5 in fp32 would already be off by 4e-3)
__global__ void __launch_bounds__(256) rope_table_scaled_kernel(float2* table, int n_pos, int half, const RopeFreq f) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long long)n_pos * half) return;
    const int k = (int)(i % half);
    const int pos = (int)(i / half);
    double w = pow(f.base, -(double)k / (double)half);
    if (f.kind == 1) {
        w /= f.factor;
    } else if (f.kind == 2) {
        const double turns = f.trained_len * w * 0.15915494309189535;  // 1 / (2 pi)
        const double g = fmin(fmax((turns - f.turns_lo) / (f.turns_hi - f.turns_lo), 0.0), 1.0);
        w = (1.0 - g) * w / f.factor + g * w;
    }
    double s, c;
    sincos((double)pos * w, &s, &c);
    table[i] = make_float2((float)(f.amplitude * c), (float)(f.amplitude * s));
}

// Where the two 16-byte halves of unit u (16 elements) of a head row lie, in elements.
template <bool INTERLEAVED>
__device__ __forceinline__ void unit_offsets(int u, int rot, int* e0, int* e1) {
    if (INTERLEAVED || u * 16 >= rot) {
        *e0 = u * 16;
        *e1 = u * 16 + 8;
    } else {
        *e0 = u * 8;
        *e1 = rot / 2 + u * 8;
    }
}

__device__ __forceinline__ void unpack8(const uint4& v, float* x) {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = __bfloat1622float2(p[k]);
        x[2 * k] = f.x;
        x[2 * k + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 pack8(const float* x) {
    uint4 v;
    __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
    return v;
}

// Cosines and sines of a unit's eight pairs, in registers.
struct UnitAngles {
    float c[8], s[8];
    __device__ __forceinline__ void load(const float2* __restrict__ t, float sign) {
        const float4* t4 = reinterpret_cast<const float4*>(t);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 v = __ldg(t4 + k);
            c[2 * k] = v.x;
            s[2 * k] = sign * v.y;
            c[2 * k + 1] = v.z;
            s[2 * k + 1] = sign * v.w;
        }
    }
};

// Rotates the 16 elements x (first and second 16 bytes of the unit).  Products are rounded separately: the result is
// that of the formula evaluated operation by operation, whatever the compiler would contract.
template <bool INTERLEAVED>
__device__ __forceinline__ void rotate16(float* x, const UnitAngles& t) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int i = INTERLEAVED ? 2 * k : k, j = INTERLEAVED ? 2 * k + 1 : 8 + k;
        const float a = x[i], b = x[j];
        x[i] = __fsub_rn(__fmul_rn(a, t.c[k]), __fmul_rn(b, t.s[k]));
        x[j] = __fadd_rn(__fmul_rn(a, t.s[k]), __fmul_rn(b, t.c[k]));
    }
}

struct RotateParams {
    const __nv_bfloat16* X;
    __nv_bfloat16* Y;
    const float2* table;       // [n_pos][rot/2]
    const int32_t* positions;  // [B][L] or null
    long long x_stride[3], y_stride[3];
    uint32_t n;                // B * L * head groups * units
    FastDiv f_units, f_groups, f_L;  // units = d / 16
    int H, rot, pos0, n_pos;
    float sign;
};
template <bool INTERLEAVED, int HPT>
__global__ void __launch_bounds__(256) rope_rotate_kernel(const RotateParams prm) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= prm.n) return;
    // 32-bit reciprocals: four 64-bit divisions would be most of the kernel's instructions
    const uint32_t hu = fdiv(i, prm.f_units), row = fdiv(hu, prm.f_groups);
    const int u = (int)(i - hu * prm.f_units.d), g = (int)(hu - row * prm.f_groups.d);
    const int b = (int)fdiv(row, prm.f_L), r = (int)(row - (uint32_t)b * prm.f_L.d);
    int e0, e1;
    unit_offsets<INTERLEAVED>(u, prm.rot, &e0, &e1);
    const int h0 = g * HPT;
    const __nv_bfloat16* x = prm.X + b * prm.x_stride[0] + r * prm.x_stride[1] + h0 * prm.x_stride[2];
    __nv_bfloat16* y = prm.Y + b * prm.y_stride[0] + r * prm.y_stride[1] + h0 * prm.y_stride[2];
    uint4 lo[HPT], hi[HPT];
#pragma unroll
    for (int k = 0; k < HPT; ++k)
        if (h0 + k < prm.H) {
            lo[k] = *reinterpret_cast<const uint4*>(x + k * prm.x_stride[2] + e0);
            hi[k] = *reinterpret_cast<const uint4*>(x + k * prm.x_stride[2] + e1);
        }
    const int pos = prm.positions ? prm.positions[row] : prm.pos0 + r;
    const bool known = (unsigned)pos < (unsigned)prm.n_pos;
    if (!known && u == 0 && g == 0) refuse_input(34);
    UnitAngles t;
    const bool turns = u * 16 < prm.rot && known;
    if (turns) t.load(prm.table + (long long)pos * (prm.rot / 2) + u * 8, prm.sign);
#pragma unroll
    for (int k = 0; k < HPT; ++k)
        if (h0 + k < prm.H) {
            if (turns) {
                float v[16];
                unpack8(lo[k], v);
                unpack8(hi[k], v + 8);
                rotate16<INTERLEAVED>(v, t);
                lo[k] = pack8(v);
                hi[k] = pack8(v + 8);
            } else if (!known) {
                lo[k] = hi[k] = make_uint4(0, 0, 0, 0);
            }
            *reinterpret_cast<uint4*>(y + k * prm.y_stride[2] + e0) = lo[k];
            *reinterpret_cast<uint4*>(y + k * prm.y_stride[2] + e1) = hi[k];
        }
}

// ---- new rows into the paged cache ------------------------------------------------------------------------------
struct AppendParams {
    PagedView c;
    const __nv_bfloat16 *Kn, *Vn, *Q;  // Q may be null
    __nv_bfloat16* Qo;
    const float2* table;               // may be null: no rotation
    const float *k_scale, *v_scale;    // e4m3 only
    long long kn_stride[3], vn_stride[3], q_stride[3], qo_stride[3];
    uint32_t n;                        // B * Lq * head groups * units
    FastDiv f_units, f_groups, f_Lq;   // units = d / 16
    int Hq, rot, n_pos;
};

// Eight values as e4m3, nearest even and saturated (a NaN stays one).
__device__ __forceinline__ uint2 e4m3x8(const float* x) {
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const __nv_fp8x2_storage_t a = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * k], x[4 * k + 1]), __NV_SATFINITE, __NV_E4M3);
        const __nv_fp8x2_storage_t b = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * k + 2], x[4 * k + 3]), __NV_SATFINITE, __NV_E4M3);
        w[k] = (uint32_t)a | ((uint32_t)b << 16);
    }
    return make_uint2(w[0], w[1]);
}
// The heads of a token are listed as [query heads ; key heads ; value heads]; a thread takes unit u of HPT of them.
template <bool INTERLEAVED, bool FP8, int HPT>
__global__ void __launch_bounds__(256) kv_append_kernel(const AppendParams prm) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= prm.n) return;
    const uint32_t hu = fdiv(i, prm.f_units), row = fdiv(hu, prm.f_groups);
    const int u = (int)(i - hu * prm.f_units.d), g = (int)(hu - row * prm.f_groups.d);
    const int b = (int)fdiv(row, prm.f_Lq), t = (int)(row - (uint32_t)b * prm.f_Lq.d);
    const int rows = new_rows(prm.c, b);
    if (t >= rows) return;
    const int Hkv = prm.c.Hkv, all = prm.Hq + 2 * Hkv, h0 = g * HPT;
    int r0, r1;  // this unit's two 16-byte halves where the head is rotated, and where it is copied
    unit_offsets<INTERLEAVED>(u, prm.rot, &r0, &r1);
    const int v0 = u * 16, v1 = u * 16 + 8;
    uint4 lo[HPT], hi[HPT];
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
        const int h = h0 + k;
        if (h < all) {
            const bool val = h >= prm.Hq + Hkv;
            const __nv_bfloat16* x =
                h < prm.Hq ? prm.Q + b * prm.q_stride[0] + t * prm.q_stride[1] + h * prm.q_stride[2]
                : val      ? prm.Vn + b * prm.vn_stride[0] + t * prm.vn_stride[1] + (h - prm.Hq - Hkv) * prm.vn_stride[2]
                           : prm.Kn + b * prm.kn_stride[0] + t * prm.kn_stride[1] + (h - prm.Hq) * prm.kn_stride[2];
            lo[k] = *reinterpret_cast<const uint4*>(x + (val ? v0 : r0));
            hi[k] = *reinterpret_cast<const uint4*>(x + (val ? v1 : r1));
        }
    }
    float inv[HPT];
    if (FP8) {
#pragma unroll
        for (int k = 0; k < HPT; ++k) {
            const int h = h0 + k - prm.Hq;
            inv[k] = h >= 0 && h < 2 * Hkv ? __frcp_rn(h < Hkv ? prm.k_scale[h] : prm.v_scale[h - Hkv]) : 1.f;
        }
    }
    // From the numbers as they are given: a length or a count of rows cut to its range would move the rows to slots, and
    // turn them by positions, that are not theirs.
    const int n = prm.c.kv_len[b], shift = prm.c.pos_shift ? prm.c.pos_shift[b] : 0;
    const uint32_t slot = (uint32_t)n - (uint32_t)(rows - t), pos = slot + (uint32_t)shift;
    if (n < 0 || slot >= (uint32_t)prm.c.cap || (prm.c.q_len && prm.c.q_len[b] != rows) ||
        (prm.table && (shift < 0 || pos >= (uint32_t)prm.n_pos))) {
        if (u == 0 && g == 0) refuse_input(35);
        return;
    }
    UnitAngles ang;
    const bool turns = prm.table && u * 16 < prm.rot;
    if (turns && h0 < prm.Hq + Hkv) ang.load(prm.table + (long long)pos * (prm.rot / 2) + u * 8, 1.f);
    int prow = 0, page = -1;
    if (h0 + HPT > prm.Hq) page = page_of(prm.c, b, (int)slot, &prow);
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
        const int h = h0 + k;
        if (h >= all) continue;
        const bool val = h >= prm.Hq + Hkv;
        float x[16];
        unpack8(lo[k], x);
        unpack8(hi[k], x + 8);
        if (turns && !val) rotate16<INTERLEAVED>(x, ang);
        if (h < prm.Hq) {
            __nv_bfloat16* y = prm.Qo + b * prm.qo_stride[0] + t * prm.qo_stride[1] + h * prm.qo_stride[2];
            *reinterpret_cast<uint4*>(y + r0) = pack8(x);
            *reinterpret_cast<uint4*>(y + r1) = pack8(x + 8);
        } else if (page >= 0) {
            const int hk = val ? h - prm.Hq - Hkv : h - prm.Hq;
            char* dst = val ? prm.c.V + page * prm.c.v_stride[0] + prow * prm.c.v_stride[1] + hk * prm.c.v_stride[2]
                            : prm.c.K + page * prm.c.k_stride[0] + prow * prm.c.k_stride[1] + hk * prm.c.k_stride[2];
            const int o0 = val ? v0 : r0, o1 = val ? v1 : r1;
            if (FP8) {
                // times the inverse: with a division for each value the kernel took 84 us instead of 49 (12K rows)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = __fmul_rn(x[e], inv[k]);
                const uint2 y0 = e4m3x8(x), y1 = e4m3x8(x + 8);
                if (INTERLEAVED) {
                    *reinterpret_cast<uint4*>(dst + o0) = make_uint4(y0.x, y0.y, y1.x, y1.y);
                } else {
                    *reinterpret_cast<uint2*>(dst + o0) = y0;
                    *reinterpret_cast<uint2*>(dst + o1) = y1;
                }
            } else {
                *reinterpret_cast<uint4*>(dst + 2 * o0) = pack8(x);
                *reinterpret_cast<uint4*>(dst + 2 * o1) = pack8(x + 8);
            }
        }
    }
}

}  // namespace segattn
