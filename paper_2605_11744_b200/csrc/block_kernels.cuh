// Blocks of rows of the paged cache: 8-bit values with a scale for each block and head, means of blocks, and the choice of blocks
// by their means.  A block is 2^k rows of a page, 16 to 128, and starts at a multiple of its size in its page and its sequence.
#pragma once
#include <cfloat>
#include <cstdint>

#include "decode_kernels.cuh"
#include "evict_kernels.cuh"
#include "paged_cache.cuh"
#include "rotary_kernels.cuh"

namespace segattn {

// ---- new rows into a cache with a scale for each block ---------------------------------------------------------------
struct AppendBlocksParams {
    AppendParams a;                        // a.n: threads that rotate queries
    float *ks, *vs;
    long long ks_stride[3], vs_stride[3];  // elements, for (page, block of the page, head)
    uint32_t units, unit_blocks;           // (sequence, block, K and V heads); thread blocks that work on them
    FastDiv f_heads2, f_blocks;            // 2 Hkv; blocks that the new rows of a sequence can touch
    int log;                               // log2 of a block's rows
};

// The exponent of the scale of a block whose largest value is `top`: 2^e >= top / 448, the smallest such, cut to [-40, 119].  (2^119 times
// 448 is 1.75 * 2^127: what lies between that and bf16's end at 1.99 * 2^127 saturates, as infinities do.  2^-40 lies below every
// value that matters and keeps the scales of a cache within reach of each other.)
__device__ __forceinline__ int scale_exponent(float top) {
    const uint32_t bits = __float_as_uint(top);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 * 2^8
    return min(max(e, -40), 119);
}
// 16 values in 8 bits times r, in 8 bits again
__device__ __forceinline__ uint4 rescale16(const uint4& v, float r) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float x[16];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t lo, hi;
        e4m3x4_to_half(w[k], lo, hi);
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
        x[4 * k] = __fmul_rn(a.x, r);
        x[4 * k + 1] = __fmul_rn(a.y, r);
        x[4 * k + 2] = __fmul_rn(b.x, r);
        x[4 * k + 3] = __fmul_rn(b.y, r);
    }
    const uint2 y0 = e4m3x8(x), y1 = e4m3x8(x + 8);
    return make_uint4(y0.x, y0.y, y1.x, y1.y);
}

// The queries' part of the call: as kv_append_kernel does it.
template <bool INTERLEAVED, int HPT>
__device__ __forceinline__ void rotate_queries(const AppendParams& prm, uint32_t i) {
    const uint32_t hu = fdiv(i, prm.f_units), row = fdiv(hu, prm.f_groups);
    const int u = (int)(i - hu * prm.f_units.d), h0 = (int)(hu - row * prm.f_groups.d) * HPT;
    const int b = (int)fdiv(row, prm.f_Lq), t = (int)(row - (uint32_t)b * prm.f_Lq.d);
    const int rows = new_rows(prm.c, b);
    if (t >= rows) return;
    int r0, r1;
    unit_offsets<INTERLEAVED>(u, prm.rot, &r0, &r1);
    const __nv_bfloat16* x = prm.Q + b * prm.q_stride[0] + t * prm.q_stride[1] + h0 * prm.q_stride[2];
    __nv_bfloat16* y = prm.Qo + b * prm.qo_stride[0] + t * prm.qo_stride[1] + h0 * prm.qo_stride[2];
    uint4 lo[HPT], hi[HPT];
#pragma unroll
    for (int k = 0; k < HPT; ++k)
        if (h0 + k < prm.Hq) {
            lo[k] = *reinterpret_cast<const uint4*>(x + k * prm.q_stride[2] + r0);
            hi[k] = *reinterpret_cast<const uint4*>(x + k * prm.q_stride[2] + r1);
        }
    const int n = prm.c.kv_len[b], shift = prm.c.pos_shift ? prm.c.pos_shift[b] : 0;
    const uint32_t slot = (uint32_t)n - (uint32_t)(rows - t), pos = slot + (uint32_t)shift;
    if (n < 0 || slot >= (uint32_t)prm.c.cap || (prm.c.q_len && prm.c.q_len[b] != rows) || shift < 0 || pos >= (uint32_t)prm.n_pos) {
        if (u == 0 && h0 == 0) refuse_input(35);
        return;
    }
    UnitAngles ang;
    const bool turns = u * 16 < prm.rot;
    if (turns) ang.load(prm.table + (long long)pos * (prm.rot / 2) + u * 8, 1.f);
#pragma unroll
    for (int k = 0; k < HPT; ++k)
        if (h0 + k < prm.Hq) {
            float v[16];
            unpack8(lo[k], v);
            unpack8(hi[k], v + 8);
            if (turns) rotate16<INTERLEAVED>(v, ang);
            *reinterpret_cast<uint4*>(y + k * prm.qo_stride[2] + r0) = pack8(v);
            *reinterpret_cast<uint4*>(y + k * prm.qo_stride[2] + r1) = pack8(v + 8);
        }
}

// G threads (a warp, or the thread block) take one block of one K or V head: its new rows into registers, rotated, their largest value,
// the block's scale, and the rows in 8 bits.  Where the block has rows already its scale can only grow, and with it those rows are
// brought to the new one: by a power of two, which costs a value nothing but at the lowest octave of its range.  A stream over HBM:
// 12K rows of 8 heads with 32 query heads take 55 us for 281 MB (5.1 TB/s; 43 us at the rate of a copy), with issue slots half used and
// loads waited for; five and six thread blocks to an SM (51 and 42 registers) took 56 and 71 us, the queries' blocks first or in turn
// with the others 56 and 61.  64 sequences' tokens: 2.8 us.
template <int D, bool INTERLEAVED, int G, int STEPS>
__global__ void __launch_bounds__(256) append_blocks_kernel(const __grid_constant__ AppendBlocksParams p) {
    const AppendParams& a = p.a;
    if (blockIdx.x >= p.unit_blocks) {
        const uint32_t i = (blockIdx.x - p.unit_blocks) * 256u + threadIdx.x;
        if (i < a.n) rotate_queries<INTERLEAVED, 2>(a, i);
        return;
    }
    constexpr int U = D / 16, RP = G / U;  // threads to a row, rows at a time
    __shared__ uint32_t red[8];
    const uint32_t unit = blockIdx.x * (256 / G) + threadIdx.x / G;
    if (unit >= p.units) return;
    const int tid = threadIdx.x % G, u = tid % U, rr = tid / U;
    const uint32_t bk = fdiv(unit, p.f_heads2), b = fdiv(bk, p.f_blocks);
    const int hh = (int)(unit - bk * p.f_heads2.d), k = (int)(bk - b * p.f_blocks.d), Hkv = a.c.Hkv;
    const bool val = hh >= Hkv;
    const int h = val ? hh - Hkv : hh;
    const int rows = new_rows(a.c, b), n = a.c.kv_len[b], shift = a.c.pos_shift ? a.c.pos_shift[b] : 0;
    if (rows == 0) return;
    // From the numbers as they are given; rows that they give no place are left out.
    const int first = n - rows;
    int lo = max(first, 0), hi = min(n, a.c.cap);
    if (a.table) hi = (int)min((long long)hi, (long long)a.n_pos - shift);
    if (n < 0 || (a.c.q_len && a.c.q_len[b] != rows) || (a.table && shift < 0)) hi = lo;
    if (hi - lo < rows && k == 0 && hh == 0 && tid == 0) refuse_input(35);
    const int start = ((lo >> p.log) + k) << p.log, from = max(lo, start), to = (int)min((long long)hi, (long long)start + (1 << p.log));
    if (from >= to) return;

    // the new rows, whose places do not depend on the page: on their way while it is looked up
    int e0, e1;  // this thread's two halves of a row
    unit_offsets<INTERLEAVED>(u, val ? 0 : a.rot, &e0, &e1);
    const __nv_bfloat16* src = val ? a.Vn + b * a.vn_stride[0] + h * a.vn_stride[2] : a.Kn + b * a.kn_stride[0] + h * a.kn_stride[2];
    const long long src_row = val ? a.vn_stride[1] : a.kn_stride[1], dst_row = val ? a.c.v_stride[1] : a.c.k_stride[1];
    const bool turns = !val && a.table && u * 16 < a.rot;
    uint4 raw[STEPS][2];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int slot = from + s * RP + rr;
        if (slot < to) {
            const __nv_bfloat16* x = src + (slot - first) * src_row;
            raw[s][0] = *reinterpret_cast<const uint4*>(x + e0);
            raw[s][1] = *reinterpret_cast<const uint4*>(x + e1);
        }
    }
    int prow;
    const int page = page_of(a.c, b, start, &prow);
    if (page < 0) return;
    float* scale_at = val ? p.vs + page * p.vs_stride[0] + (prow >> p.log) * p.vs_stride[1] + h * p.vs_stride[2]
                          : p.ks + page * p.ks_stride[0] + (prow >> p.log) * p.ks_stride[1] + h * p.ks_stride[2];
    const float old = start < lo ? *scale_at : 0.f;
    float x[STEPS][16], top = 0.f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int slot = from + s * RP + rr;
        if (slot < to) {
            unpack8(raw[s][0], x[s]);
            unpack8(raw[s][1], x[s] + 8);
            if (turns) {
                UnitAngles ang;
                ang.load(a.table + (long long)(slot + shift) * (a.rot / 2) + u * 8, 1.f);
                rotate16<INTERLEAVED>(x[s], ang);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float m = fabsf(x[s][e]);
                if (m <= FLT_MAX) top = fmaxf(top, m);  // neither an infinity, which saturates, nor a NaN has a say
            }
        }
    }
    uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
    if (G > 32) {
        if ((tid & 31) == 0) red[tid >> 5] = most;
        __syncthreads();
        most = __reduce_max_sync(0xffffffffu, red[tid & 7]);
    }
    // An append's own scales are positive; of others the magnitude counts, and one that is not finite has no say (its rows become NaN, or
    // saturate).
    const float size = fabsf(old), need = __uint_as_float((uint32_t)(127 + scale_exponent(__uint_as_float(most))) << 23);
    const float scale = size <= FLT_MAX ? fmaxf(size, need) : need;
    char* dst = val ? a.c.V + page * a.c.v_stride[0] + prow * dst_row + h * a.c.v_stride[2]
                    : a.c.K + page * a.c.k_stride[0] + prow * dst_row + h * a.c.k_stride[2];
    if (start < lo && scale != old) {
        const float r = __fdiv_rn(old, scale);
        for (int row = rr; row < lo - start; row += RP) {
            uint4* at = reinterpret_cast<uint4*>(dst + row * dst_row + u * 16);
            *at = rescale16(*at, r);
        }
    }
    if (tid == 0 && scale != old) *scale_at = scale;
    const float inv = __frcp_rn(scale);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int slot = from + s * RP + rr;
        if (slot < to) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[s][e] = __fmul_rn(x[s][e], inv);
            const uint2 y0 = e4m3x8(x[s]), y1 = e4m3x8(x[s] + 8);
            char* row = dst + (slot - start) * dst_row;
            if (INTERLEAVED || val || !turns) {
                *reinterpret_cast<uint4*>(row + e0) = make_uint4(y0.x, y0.y, y1.x, y1.y);
            } else {
                *reinterpret_cast<uint2*>(row + e0) = y0;
                *reinterpret_cast<uint2*>(row + e1) = y1;
            }
        }
    }
}

// ---- eviction from a cache with a scale for each block -------------------------------------------------------------------
struct EvictBlocksParams {
    EvictParams e;
    float *ks, *vs;
    long long ks_stride[3], vs_stride[3];
    int log;
};

// A warp writes one block of the compacted cache for one head: its rows come from blocks of all kinds, so it takes the largest of their
// scales in magnitude, and a row of another scale is brought to it (exactly but at the lowest octave where both are powers of two, as in an
// append; no row's largest value has to be looked for).  A scale that is not finite has no say: its row becomes NaN, or saturates.  Runs after evict_select_kernel; the lengths and shifts are written here as in evict_move_kernel.
template <int D>
__global__ void __launch_bounds__(256) evict_move_blocks_kernel(const __grid_constant__ EvictBlocksParams p) {
    const EvictParams& prm = p.e;
    after_previous_kernel();
    const int b = blockIdx.y, lane = threadIdx.x & 31;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        const int n = seq_len(prm.c, b), m = min(n, prm.budget), s = shift_of(prm.c, b);
        prm.kv_len_out[b] = m;
        prm.pos_shift_out[b] = s + n - m;
    }
    const uint32_t unit = blockIdx.x * 8 + (threadIdx.x >> 5), k = fdiv(unit, prm.f_heads);
    const int h = (int)(unit - k * prm.f_heads.d), r0 = (int)(k << p.log);
    if (r0 >= prm.budget) return;
    const int rows = min(1 << p.log, prm.budget - r0);
    const int32_t* idx = prm.idx + ((long long)b * prm.c.Hkv + h) * prm.budget + r0;
    // rows 32 j + lane: where they are (-1: nowhere, -2: on a page that is not there), and their scales
    int page[4], row[4];
    float ks[4], vs[4], k_top = 0.f, v_top = 0.f;
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = 32 * j + lane, slot = r < rows ? idx[r] : -1;
        page[j] = -1;
        row[j] = 0;
        ks[j] = vs[j] = 0.f;
        if (slot >= 0) {
            any = true;
            page[j] = page_of(prm.c, b, slot, &row[j]);
            if (page[j] < 0) {
                page[j] = -2;
            } else {
                ks[j] = p.ks[page[j] * p.ks_stride[0] + (row[j] >> p.log) * p.ks_stride[1] + h * p.ks_stride[2]];
                vs[j] = p.vs[page[j] * p.vs_stride[0] + (row[j] >> p.log) * p.vs_stride[1] + h * p.vs_stride[2]];
            }
        }
        const float k_size = fabsf(ks[j]), v_size = fabsf(vs[j]);
        if (k_size <= FLT_MAX) k_top = fmaxf(k_top, k_size);
        if (v_size <= FLT_MAX) v_top = fmaxf(v_top, v_size);
    }
    if (!__any_sync(0xffffffffu, any)) return;
    const int entry = (int)fdiv((uint32_t)r0, prm.c.f_page), first = r0 - entry * (int)prm.c.f_page.d;
    const int to = prm.dst_table[(long long)b * prm.dst_stride + entry];
    if ((unsigned)to >= (unsigned)prm.c.n_pages) {
        if (lane == 0) refuse_input(36);
        return;
    }
    k_top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(k_top)));
    v_top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v_top)));
    if (k_top == 0.f) k_top = 0x1p-40f;  // no row had a page, or a scale to go by
    if (v_top == 0.f) v_top = 0x1p-40f;
    if (lane == 0) {
        p.ks[to * p.ks_stride[0] + (first >> p.log) * p.ks_stride[1] + h * p.ks_stride[2]] = k_top;
        p.vs[to * p.vs_stride[0] + (first >> p.log) * p.vs_stride[1] + h * p.vs_stride[2]] = v_top;
    }
    constexpr int U = D / 16, RP = 32 / U;  // lanes to a row, rows at a time
    const int e = lane % U * 16;
#pragma unroll 4
    for (int r = lane / U; r - lane / U < rows; r += RP) {
        const int from = r & 31, j = r >> 5;
        auto of = [&](auto (&v)[4]) { return __shfl_sync(0xffffffffu, j == 0 ? v[0] : j == 1 ? v[1] : j == 2 ? v[2] : v[3], from); };
        const int pg = of(page), rw = of(row);
        const float kr = of(ks), vr = of(vs);
        if (pg == -1) continue;
        uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
        if (pg >= 0) {
            kx = *reinterpret_cast<const uint4*>(prm.c.K + pg * prm.c.k_stride[0] + rw * prm.c.k_stride[1] + h * prm.c.k_stride[2] + e);
            vx = *reinterpret_cast<const uint4*>(prm.c.V + pg * prm.c.v_stride[0] + rw * prm.c.v_stride[1] + h * prm.c.v_stride[2] + e);
            if (kr != k_top) kx = rescale16(kx, __fdiv_rn(kr, k_top));
            if (vr != v_top) vx = rescale16(vx, __fdiv_rn(vr, v_top));
        }
        *reinterpret_cast<uint4*>(prm.c.K + to * prm.c.k_stride[0] + (first + r) * prm.c.k_stride[1] + h * prm.c.k_stride[2] + e) = kx;
        *reinterpret_cast<uint4*>(prm.c.V + to * prm.c.v_stride[0] + (first + r) * prm.c.v_stride[1] + h * prm.c.v_stride[2] + e) = vx;
    }
}

constexpr float kOver127 = 1.f / 127.f;  // steps are max / 127 as the product with this number, rounded

// ---- means of blocks --------------------------------------------------------------------------------------------------
struct SummariseParams {
    PagedView c;
    const float* ks;            // e4m3: scales by strides (0, 0, 1) for one to a head
    long long ks_stride[3];
    int ks_log;
    int8_t* sums;               // [n_pages][blocks of a page][Hkv][D]
    float* sum_scale;           // [n_pages][blocks of a page][Hkv]
    FastDiv f_heads, f_blocks;  // Hkv; blocks whose means the new rows of a sequence can change
    uint32_t units;             // B * blocks * Hkv
    int log, per_page;          // log2 of a block's rows; blocks of a page
};

// A bf16 number times 2^-896, as the upper half of a double: its exponent and mantissa bits where a double has them.  (An infinity or
// a NaN comes out as a number: they are looked for apart.)
__device__ __forceinline__ double bf16_in_double(uint32_t b) { return __hiloint2double((int)((b & 0x8000u) << 16 | (b & 0x7fffu) << 13), 0); }

// sum + the two fp16 numbers of a register, exactly as long as the sum has room
__device__ __forceinline__ void add_halves(float& lo, float& hi, uint32_t x) {
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tadd.f32.f16 %0, a, %0;\n\tadd.f32.f16 %1, b, %1;\n\t}" : "+f"(lo), "+f"(hi) : "r"(x));
}

// A warp takes one head's block of rows, if it is full and the new rows may have changed it, 16 rows (which have one scale) at a time: the mean of its
// keys in double, then c = max |mean| / 127 and the mean in steps of c.  HBM is to bound it, so a value costs few instructions and
// hardly any of them in double precision, where a conversion alone takes the time of a dozen others: values of an 8-bit cache are
// multiples of 2^-9, of which a lane adds up 32 at most in fp32, and the lanes their sums as integers, exactly; bf16 numbers are put
// into doubles bit by bit.  8 sequences of 16-65K rows, 8 heads in 8 bits: 79 us for 384 MB (4.9 TB/s; 317 us with every value made a
// double), 1080 instructions to a block of 64 rows, half of them the additions; issue slots and DRAM are both at 57%, as a warp looks up and
// loads one block alone and waits for it.  Small thread blocks: a step's few blocks spread out.
constexpr int kSumWarps = 4;
template <int D, bool FP8>
__global__ void __launch_bounds__(32 * kSumWarps, 6) summarise_kernel(const __grid_constant__ SummariseParams p) {
    constexpr int PER = FP8 ? 16 : 8, T = D / PER, RW = 32 / T, ROWS = 16 / RW;  // values of a lane's piece, lanes to a row, rows at a time, of a lane
    constexpr int KEEP = PER / RW;  // dims a lane has in the end
    constexpr int AHEAD = 8 / ROWS;  // groups of 16 rows whose loads are in flight together
    const int lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * kSumWarps + (threadIdx.x >> 5);
    if (unit >= p.units) return;
    const uint32_t bk = fdiv(unit, p.f_heads), b = fdiv(bk, p.f_blocks);
    const int h = (int)(unit - bk * p.f_heads.d), k = (int)(bk - b * p.f_blocks.d);
    const int rows = new_rows(p.c, b), n = seq_len(p.c, b);
    if (rows == 0) return;
    // from the block that the first new row lies in, or all of its scale's block: an append may have raised that, with all its rows
    const int whole = max(p.log, p.ks_log), start = (max(n - rows, 0) >> whole << whole) + (k << p.log);
    if ((long long)start + (1 << p.log) > n) return;
    int prow;
    const int page = page_of(p.c, b, start, &prow);
    if (page < 0) return;
    const int c = lane % T;
    const char* src = p.c.K + page * p.c.k_stride[0] + (prow + lane / T * ROWS) * p.c.k_stride[1] + h * p.c.k_stride[2] + c * 16;
    const float* scale_at = FP8 ? p.ks + page * p.ks_stride[0] + h * p.ks_stride[2] : nullptr;
    bool odd = false;  // an infinity or a NaN among the values
    double mine[KEEP];
#pragma unroll
    for (int e = 0; e < KEEP; ++e) mine[e] = 0.0;
    // The lanes with the same piece of different rows halve their values at every step: what they keep, they add up.
    int dim = c * PER;
#pragma unroll
    for (int half = PER / 2, x = T; half >= KEEP; half >>= 1, x <<= 1)
        if (lane & x) dim += half;
    auto gather = [&](auto& t) {
#pragma unroll
        for (int half = PER / 2, x = T; half >= KEEP; half >>= 1, x <<= 1) {
            const bool upper = lane & x;
#pragma unroll
            for (int e = 0; e < half; ++e) {
                const auto give = upper ? t[e] : t[e + half], keep = upper ? t[e + half] : t[e];
                t[e] = keep + __shfl_xor_sync(0xffffffffu, give, x);
            }
        }
    };
    auto load = [&](auto& v, int r0) {
#pragma unroll
        for (int g = 0; g < AHEAD; ++g)
            if (r0 + 16 * g < 1 << p.log) {
#pragma unroll
                for (int i = 0; i < ROWS; ++i) v[g][i] = *reinterpret_cast<const uint4*>(src + (r0 + 16 * g + i) * p.c.k_stride[1]);
            }
    };
    if (FP8) {
        float sum[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = 0.f;
        float scale = scale_at[(prow >> p.ks_log) * p.ks_stride[1]];
        auto flush = [&]() {
            int t[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                odd |= sum[e] != sum[e];
                t[e] = __float2int_rn(sum[e] * 512.f);
                sum[e] = 0.f;
            }
            gather(t);
#pragma unroll
            for (int e = 0; e < KEEP; ++e) mine[e] += (double)scale * 0.001953125 * (double)t[e];
        };
        for (int r0 = 0; r0 < 1 << p.log; r0 += 16 * AHEAD) {
            uint4 v[AHEAD][ROWS];
            float next[AHEAD];
            load(v, r0);
#pragma unroll
            for (int g = 0; g < AHEAD; ++g)
                if (r0 + 16 * g < 1 << p.log) next[g] = scale_at[((prow + r0 + 16 * g) >> p.ks_log) * p.ks_stride[1]];
#pragma unroll
            for (int g = 0; g < AHEAD; ++g) {
                if (r0 + 16 * g >= 1 << p.log) break;
                if (__float_as_uint(next[g]) != __float_as_uint(scale)) {
                    flush();
                    scale = next[g];
                }
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    const uint32_t w[4] = {v[g][i].x, v[g][i].y, v[g][i].z, v[g][i].w};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t lo, hi;
                        e4m3x4_to_half(w[q], lo, hi);
                        add_halves(sum[4 * q], sum[4 * q + 1], lo);
                        add_halves(sum[4 * q + 2], sum[4 * q + 3], hi);
                    }
                }
            }
        }
        flush();
    } else {
        double sum[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.0;
        for (int r0 = 0; r0 < 1 << p.log; r0 += 16 * AHEAD) {
            uint4 v[AHEAD][ROWS];
            load(v, r0);
#pragma unroll
            for (int g = 0; g < AHEAD; ++g) {
                if (r0 + 16 * g >= 1 << p.log) break;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    const uint32_t w[4] = {v[g][i].x, v[g][i].y, v[g][i].z, v[g][i].w};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        odd |= (w[q] & 0x7f80u) == 0x7f80u || (w[q] & 0x7f800000u) == 0x7f800000u;
                        sum[2 * q] += bf16_in_double(w[q] & 0xffffu);
                        sum[2 * q + 1] += bf16_in_double(w[q] >> 16);
                    }
                }
            }
        }
        gather(sum);
#pragma unroll
        for (int e = 0; e < KEEP; ++e) mine[e] = sum[e] * __hiloint2double((1023 + 896) << 20, 0);
    }
    float mean[KEEP];
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < KEEP; ++e) {
        mean[e] = (float)(mine[e] * __hiloint2double((1023 - p.log) << 20, 0));  // over a power of two
        most = max(most, __float_as_uint(fabsf(mean[e])));                       // as bits: an infinity or a NaN is the largest
    }
    most = __reduce_max_sync(0xffffffffu, most);
    const bool fine = most < 0x7f800000u && !__any_sync(0xffffffffu, odd);
    const float step = fine ? __fmul_rn(__uint_as_float(most), kOver127) : __uint_as_float(0x7fffffffu);
    const long long at = ((long long)page * p.per_page + (prow >> p.log)) * p.c.Hkv + h;
    uint32_t q = 0;  // cut to +-127: a subnormal step is rounded so coarsely that the largest mean comes to more of them
#pragma unroll
    for (int e = 0; e < KEEP; ++e)
        q |= (fine && step > 0.f ? (uint32_t)min(max(__float2int_rn(__fdiv_rn(mean[e], step)), -127), 127) & 0xffu : 0u) << (8 * e);
    int8_t* out = p.sums + at * D + dim;
    if (KEEP == 4) *reinterpret_cast<uint32_t*>(out) = q;
    else *reinterpret_cast<uint16_t*>(out) = (uint16_t)q;
    if (lane == 0) p.sum_scale[at] = step;
}

// ---- the choice of blocks ---------------------------------------------------------------------------------------------
struct SelectParams {
    PagedView c;                // K, V and their strides unused
    const __nv_bfloat16* Q;
    long long q_stride[3];
    const int8_t* sums;
    const float* sum_scale;
    int32_t* idx;               // [B][Lq][Hkv][n]
    FastDiv f_S;
    int S, T, g, n, sink, log, per_page, keys;
    int n_past;                 // heads with a past
    uint8_t heads[64];          // those, then the others
};

constexpr int kSelThreads = 512;
constexpr int kSelBins = 2048;
constexpr int kSelFew = 256;                // as many are compared with each other one by one
constexpr int kSelMost = 128;               // blocks that can be chosen
constexpr int kSelKeys = 49152;             // blocks to choose from
constexpr int kSelSlice = 512;              // blocks that a thread block of a cluster has at least
constexpr uint32_t kSinkKey = 0xffffffffu;  // above every score's
static_assert(kSelKeys / 32 <= kSelBins, "a bin for 32 neighbouring blocks");

// The lowest slot that a row at `slot` sees whole through a head with a past: its tail's start, rounded down to a block.
__device__ __forceinline__ int whole_from(const SelectParams& p, int slot, int shift) {
    const uint32_t pos = (uint32_t)slot + (uint32_t)shift;
    const long long start = (long long)fdiv(pos, p.f_S) * p.S;
    return (int)max(0ll, max(0ll, start - p.T) - shift) >> p.log << p.log;
}

// Lists of row t of sequence b for the heads from p.heads[from] on: no blocks.
__device__ __forceinline__ void no_choice(const SelectParams& p, int bt, int from, int tid, int step) {
    for (int i = tid; i < (p.c.Hkv - from) * p.n; i += step) p.idx[((long long)bt * p.c.Hkv + p.heads[from + i / p.n]) * p.n + i % p.n] = -1;
}
__global__ void __launch_bounds__(128) no_choice_kernel(const __grid_constant__ SelectParams p) {
    const int b = blockIdx.x / p.c.Lq, t = blockIdx.x - b * p.c.Lq;
    if (t < new_rows(p.c, b)) no_choice(p, blockIdx.x, 0, threadIdx.x, 128);
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// into the same place of another block's shared memory
__device__ __forceinline__ void store_to_block(uint32_t* shared, uint32_t rank, uint32_t v) {
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(shared)), "r"(rank));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// A cluster takes one (new row, KV head with a past).  The query, summed over the head's query heads and brought to 8 bits, against
// the means of the blocks before the row's tail: integer products, so that a score is the same in whatever order it is added up.
// Then the first block of the cluster chooses: digits of the keys (11, 11 and 10 bits, then the block's number over 32, lower numbers
// first) narrow down where the n-th lies until few keys are left there, most times after one of them; those are compared one by
// one, and the chosen numbers put in order in the same way.  Barriers and dependent reads are what it costs (16 x 4 heads of 2800-4000
// blocks: 13.8 us for 28 MB of means, of which reading them takes 5), so there are few of them; a selection over histograms of the
// whole cluster, with ordered scans for the numbers, took 17.5.
template <int D>
__global__ void __launch_bounds__(kSelThreads, 2) select_kernel(const __grid_constant__ SelectParams p) {
    extern __shared__ uint32_t sel_smem[];
    uint32_t* hist = sel_smem;             // [kSelBins]
    uint32_t* keys = sel_smem + kSelBins;  // [p.keys]
    __shared__ __align__(16) int8_t query[D];
    __shared__ __align__(16) uint32_t near[kSelFew];    // keys about the n-th, then zeros
    __shared__ int32_t near_at[kSelFew];                // their blocks
    __shared__ __align__(16) int32_t chosen[kSelMost];  // the chosen blocks, then larger numbers
    __shared__ uint32_t red[kSelThreads / 32], found[3];
    __shared__ int n_chosen, n_near;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int CS = (int)cluster_size(), rank = (int)cluster_rank(), unit = blockIdx.x / CS;
    const int which = unit % p.n_past, h = p.heads[which], bt = unit / p.n_past, b = bt / p.c.Lq, t = bt - b * p.c.Lq;
    float q = 0.f;  // the query; asked for before anything that depends on the lengths
    if (tid < D) {
        double sum = 0.0;
        const __nv_bfloat16* at = p.Q + b * p.q_stride[0] + t * p.q_stride[1] + (long long)h * p.g * p.q_stride[2] + tid;
#pragma unroll 8
        for (int x = 0; x < p.g; ++x) sum += (double)__bfloat162float(at[x * p.q_stride[2]]);
        q = (float)sum;
    }
    const int rows = new_rows(p.c, b), n = seq_len(p.c, b), shift = shift_of(p.c, b);
    if (t >= rows) return;
    int32_t* out = p.idx + ((long long)bt * p.c.Hkv + h) * p.n;
    if (which == 0) no_choice(p, bt, p.n_past, rank * kSelThreads + tid, CS * kSelThreads);
    const int slot = n - rows + t;
    const int m = slot >= 0 ? whole_from(p, slot, shift) >> p.log : 0;  // blocks to choose from
    if (m <= p.n) {
        for (int i = rank * kSelThreads + tid; i < p.n; i += CS * kSelThreads) out[i] = i < m ? i : -1;
        return;
    }
    if (CS > 1) cluster_arrive();

    // this block's slice, and the pages of its blocks (in the keys' place, in the first block of the cluster until the scores take it)
    const int slice = (((m + CS - 1) / CS + 31) & ~31), j0 = min(rank * slice, m), cnt = min(slice, m - j0);
    for (int i = tid; i < cnt; i += kSelThreads) keys[i] = (uint32_t)table_entry(p.c, b, (j0 + i) << p.log);

    const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(fabsf(q)));
    if (lane == 0) red[warp] = most;
    if (tid == 0) n_chosen = n_near = 0;
    if (tid < kSelFew) near[tid] = 0;
    if (tid < kSelMost) chosen[tid] = 0x7fffffff;
    for (int i = tid; i < kSelBins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t top = __reduce_max_sync(0xffffffffu, lane < D / 32 ? red[lane] : 0u);
    const float step = __fmul_rn(__uint_as_float(top), kOver127);
    if (tid < D) query[tid] = top > 0 && top < 0x7f800000u && step > 0.f ? (int8_t)__float2int_rn(__fdiv_rn(q, step)) : (int8_t)0;
    __syncthreads();
    if (CS > 1) cluster_wait();  // the first block is there

    // The scores, as unsigned numbers of the same order.  T lanes read a mean, so that a load of the warp touches few lines (a lane
    // to a mean touches 32, and their look-ups took three times as long as the bytes); a lane's partial sums of its T means are then
    // handed on by halves, after which it has the sum of one.
    constexpr int T = D / 16, PW = 32 / T;  // lanes to a mean, means of a load
    const uint4 q16 = reinterpret_cast<const uint4*>(query)[lane % T];
    for (int i0 = warp * 32; i0 < cnt; i0 += kSelThreads) {
        uint4 k16[T];
#pragma unroll
        for (int y = 0; y < T; ++y) {
            const int i = i0 + y * PW + lane / T;
            const uint32_t page = i < cnt ? keys[i] : 0xffffffffu;
            k16[y] = make_uint4(0, 0, 0, 0);
            if (page < (uint32_t)p.c.n_pages) {
                const long long at = ((long long)page * p.per_page + (row_in_page(p.c, (j0 + i) << p.log) >> p.log)) * p.c.Hkv + h;
                k16[y] = reinterpret_cast<const uint4*>(p.sums + at * D)[lane % T];
            }
        }
        const int i = i0 + lane % T * PW + lane / T;  // this lane's mean
        float scale = __uint_as_float(0x7fffffffu);   // of a page that is not there: lowest
        if (i < cnt) {
            const uint32_t page = keys[i];
            if (page < (uint32_t)p.c.n_pages)
                scale = p.sum_scale[((long long)page * p.per_page + (row_in_page(p.c, (j0 + i) << p.log) >> p.log)) * p.c.Hkv + h];
            else refuse_input(33);
        }
        int s[T];
#pragma unroll
        for (int y = 0; y < T; ++y)
            s[y] = __dp4a((int)k16[y].x, (int)q16.x, __dp4a((int)k16[y].y, (int)q16.y, __dp4a((int)k16[y].z, (int)q16.z, __dp4a((int)k16[y].w, (int)q16.w, 0))));
#pragma unroll
        for (int half = T / 2; half >= 1; half >>= 1) {
            const bool upper = lane & half;
#pragma unroll
            for (int y = 0; y < half; ++y) {
                const int give = upper ? s[y] : s[y + half], keep = upper ? s[y + half] : s[y];
                s[y] = keep + __shfl_xor_sync(0xffffffffu, give, half);
            }
        }
        __syncwarp();
        if (i < cnt) {
            const uint32_t key = j0 + i < p.sink ? kSinkKey : weight_key(__fmul_rn((float)s[0], scale));
            if (rank == 0) keys[i] = key;
            else store_to_block(keys + j0 + i, 0, key);
        }
        __syncwarp();
    }
    if (CS > 1) {
        cluster_sync();
        if (rank > 0) return;
    } else {
        __syncthreads();
    }

    // Where the n-th is: among `about` keys that share the digits found so far, the need-th of them.
    constexpr int BT = kSelBins / kSelThreads;
    uint32_t prefix = 0, need = p.n;
    int done = 32, numbers = -1, about = m;  // bits of a key that are left, the bin of the numbers once there are none
    auto place = [&](int i, uint32_t key) {  // 2: in front of them, 1: one of them, 0: behind
        if (done == 32) return 1;
        const uint32_t d = key >> done;
        if (d != prefix) return d > prefix ? 2 : 0;
        return numbers < 0 || i >> 5 == numbers ? 1 : i >> 5 < numbers ? 2 : 0;
    };
#pragma unroll 1
    for (int pass = 0; about > kSelFew; ++pass) {  // four at most: 32 numbers to a bin
        const int bits = pass < 2 ? 11 : 10, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        if (pass > 0) {
            for (int i = tid; i < kSelBins; i += kSelThreads) hist[i] = 0;
            __syncthreads();
        }
        for (int i = tid; i < m; i += kSelThreads) {
            const uint32_t key = keys[i];
            if (place(i, key) == 1) atomicAdd(hist + (pass < 3 ? (key >> shift) & ((1u << bits) - 1) : (uint32_t)(kSelBins - 1 - (i >> 5))), 1u);
        }
        __syncthreads();
        // bins from the top down, BT to a thread
        const uint4 v = *reinterpret_cast<const uint4*>(hist + kSelBins - BT - BT * tid);
        const uint32_t c[BT] = {v.w, v.z, v.y, v.x};
        uint32_t before = c[0] + c[1] + c[2] + c[3];
        const uint32_t mine = before;
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, before, x);
            if (lane >= x) before += y;
        }
        if (lane == 31) red[warp] = before;
        before -= mine;
        __syncthreads();
        before += __reduce_add_sync(0xffffffffu, lane < warp ? red[lane] : 0u);
#pragma unroll
        for (int k = 0; k < BT; ++k) {
            if (need > before && need <= before + c[k]) {
                found[0] = kSelBins - 1 - BT * tid - k;
                found[1] = need - before;
                found[2] = c[k];
            }
            before += c[k];
        }
        __syncthreads();
        if (pass < 3) {
            prefix = (prefix << bits) | found[0];
            done = shift;
        } else {
            numbers = kSelBins - 1 - (int)found[0];
        }
        need = found[1];
        about = (int)found[2];
    }
    for (int i = tid; i < m; i += kSelThreads) {
        const uint32_t key = keys[i];
        const int at = place(i, key);
        if (at == 2) chosen[atomicAdd(&n_chosen, 1)] = i;
        if (at == 1) {
            const int k = atomicAdd(&n_near, 1);
            near[k] = key;
            near_at[k] = i;
        }
    }
    __syncthreads();
    const uint32_t mine = tid < about ? near[tid] : 0u;
    uint32_t front = 0;
    if (warp * 32 < about)
#pragma unroll 4
        for (int i = 0; i < about; i += 4) {
            const uint4 k = *reinterpret_cast<const uint4*>(near + i);
            front += (k.x > mine) + (k.y > mine) + (k.z > mine) + (k.w > mine);
        }
    const bool may = tid < about && front < need;
    if (__syncthreads_count(may) > (int)need && may)  // equal ones on the border: the lower blocks
        for (int i = 0; i < about; ++i) front += near[i] == mine && near_at[i] < near_at[tid];
    if (may && front < need) chosen[atomicAdd(&n_chosen, 1)] = near_at[tid];
    __syncthreads();
    if (tid < p.n) {
        const int32_t number = chosen[tid];
        int at = 0;
#pragma unroll 4
        for (int i = 0; i < p.n; i += 4) {
            const int4 k = *reinterpret_cast<const int4*>(chosen + i);
            at += (k.x < number) + (k.y < number) + (k.z < number) + (k.w < number);
        }
        out[at] = number;
    }
}

}  // namespace segattn
