// Attention of a sequence's newest rows over its paged cache.
//
// The work is a stream over the visible K and V rows (HBM bound: 4 g flops per byte for g query heads to a KV head), so the
// kernel is built around the loads.  Its unit is a tile of 64 slots of one item, an item being up to 16 WM rows (new row,
// query head) of one (sequence, KV head).  All tiles of all items form one list, which the grid - two blocks to an SM -
// cuts into equal ranges by the lengths found in device memory: whatever the batch's mix of lengths and head classes, every
// SM reads the same number of bytes.  Where a range ends inside an item the block leaves an unnormalised part (O, running
// maximum, sum) in the workspace, and decode_join_kernel adds the parts up in the order of the ranges.
//
// Inside a block four warps load 16 slots of a tile each with cp.async into a ring of their own, several tiles ahead and
// across item borders.  For up to 16 rows (WM = 1) each warp attends over its own 16 slots with its own running maximum
// and sum and needs no block barrier until an item ends; for more rows WM = 2 or 4 warps share 32 or 64 slots, so that a
// row of K is read once for 32 or 64 rows.  Products run on mma.sync: 16 rows fill one of its tiles, while tcgen05.mma
// starts at 64 and would leave nine tenths of its rows empty for the same bytes.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "paged_cache.cuh"

namespace segattn {

constexpr int kDecThreads = 128;
constexpr int kDecTile = 64;     // slots in a tile
constexpr int kDecBlocksPerSm = 2;

struct DecodeParams {
    PagedView c;
    const __nv_bfloat16* Q;
    __nv_bfloat16* O;
    float* LSE;                      // [B][Hq][Lq]
    const float* w_in;               // [B][Hkv][W] or null
    float* w_out;                    // or null
    const float *k_scale, *v_scale;  // e4m3 only
    // workspace
    float* part_o;                   // [grid][2][16 WM][D]
    float2* part_ml;                 // [grid][2][16 WM] (maximum in log2 units, sum)
    int2* item_blocks;               // [B][Hkv][row blocks]: first and last block of the item's tiles
    float* scores;                   // [B][Hkv][g Lq][pitch], log2 units; null unless weights are asked for
    long long q_stride[3], o_stride[3];
    FastDiv f_S, f_g;
    int S, T, W, Hq, g;
    int row_blocks;                  // ceil(g Lq / (16 WM))
    int pitch;                       // slots in a row of scores
    int min_tiles;                   // a block's range has at least this many tiles
    float scale_log2;                // sm_scale * log2(e)
    int n_class[3];                  // KV heads of each class
    uint8_t head_class[64];
};

// Slots [lo, hi) that new row t of a sequence sees through a KV head of class cls.
__device__ __forceinline__ void visible_slots(const DecodeParams& p, int n, int rows, int shift, int t, int cls, int* lo, int* hi) {
    const int slot = n - rows + t;
    *hi = max(slot + 1, 0);
    *lo = 0;
    if (cls != kHeadPast && slot >= 0) {
        const uint32_t pos = (uint32_t)slot + (uint32_t)shift;
        long long start = (long long)fdiv(pos, p.f_S) * p.S;
        if (cls == kHeadLocal) start = max(0ll, start - p.T);
        *lo = (int)max(0ll, start - shift);
    }
}

// ---- the list of tiles -------------------------------------------------------------------------------------------
// Slots the rows of one row block see between them (their lower and upper ends both grow with the row), and its tiles:
// whole tiles of 64 slots, at least one, so that rows that see nothing are written too.
template <int MB>
__device__ __forceinline__ int item_tiles(const DecodeParams& p, int n, int rows, int shift, int cls, int rb, int* lo, int* hi) {
    const int last = min((rb + 1) * MB, rows * p.g) - 1;
    int l0, h0, l1, h1;
    visible_slots(p, n, rows, shift, (int)fdiv((uint32_t)(rb * MB), p.f_g), cls, &l0, &h0);
    visible_slots(p, n, rows, shift, (int)fdiv((uint32_t)last, p.f_g), cls, &l1, &h1);
    *lo = l0;
    *hi = max(h1, l0);
    return max(1, (*hi + kDecTile - 1) / kDecTile - l0 / kDecTile);
}

// Tiles of one sequence's heads of class cls (one head).
template <int MB>
__device__ __forceinline__ int class_tiles(const DecodeParams& p, int n, int rows, int shift, int cls) {
    int sum = 0, lo, hi;
    for (int rb = 0; rb * MB < rows * p.g; ++rb) sum += item_tiles<MB>(p, n, rows, shift, cls, rb, &lo, &hi);
    return sum;
}

// A place in the list: an item and a tile of it.
template <int MB>
struct TileCursor {
    int b, h, rb, n, rows, shift;
    int lo, hi;     // visible slots of the item
    int tile, end;  // next tile of the item and the number of its tiles
    __device__ __forceinline__ void read_sequence(const DecodeParams& p) {
        n = seq_len(p.c, b);
        rows = new_rows(p.c, b);
        shift = shift_of(p.c, b);
    }
    __device__ __forceinline__ void enter(const DecodeParams& p, int at) {
        end = item_tiles<MB>(p, n, rows, shift, p.head_class[h], rb, &lo, &hi);
        tile = at;
    }
    // the item after this one; the caller knows that there is one
    __device__ __forceinline__ void next_item(const DecodeParams& p) {
        if (++rb * MB >= rows * p.g) {
            rb = 0;
            if (++h == p.c.Hkv) {
                h = 0;
                do {
                    ++b;
                    read_sequence(p);
                } while (rows == 0 && b + 1 < p.c.B);
            }
        }
        enter(p, 0);
    }
    __device__ __forceinline__ int first_slot() const { return (lo / kDecTile + tile) * kDecTile; }
};

// This block's range of tiles, and the item it begins in.  Every block counts the tiles of all sequences: they are read
// from device memory, so that a captured call follows the lengths.
struct BlockRange {
    int begin, end, per, b, h, rb, tile;
};
template <int MB>
__device__ __forceinline__ void find_range(const DecodeParams& p, BlockRange* out, int* warp_sum) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int seg = (p.c.B + kDecThreads - 1) / kDecThreads;
    const int b0 = min(tid * seg, p.c.B), b1 = min(b0 + seg, p.c.B);
    auto tiles_of = [&](int b) {
        const int rows = new_rows(p.c, b);
        if (rows == 0) return 0;
        const int n = seq_len(p.c, b), shift = shift_of(p.c, b);
        int sum = 0;
#pragma unroll
        for (int cls = 0; cls < 3; ++cls)
            if (p.n_class[cls]) sum += p.n_class[cls] * class_tiles<MB>(p, n, rows, shift, cls);
        return sum;
    };
    int mine = 0;
    for (int b = b0; b < b1; ++b) mine += tiles_of(b);
    int before = mine;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, before, x);
        if (lane >= x) before += y;
    }
    if (lane == 31) warp_sum[warp] = before;
    if (tid == 0) out->begin = out->end = 0;
    __syncthreads();
    int total = 0;
    before -= mine;
    for (int k = 0; k < kDecThreads / 32; ++k) {
        if (k < warp) before += warp_sum[k];
        total += warp_sum[k];
    }
    const int per = max(p.min_tiles, (total + (int)gridDim.x - 1) / (int)gridDim.x);
    const int begin = min((int)blockIdx.x * per, total), end = min(begin + per, total);
    if (begin < end && begin >= before && begin < before + mine) {
        int off = begin - before, b = b0;
        for (;; ++b) {
            const int t = tiles_of(b);
            if (off < t) break;
            off -= t;
        }
        const int n = seq_len(p.c, b), rows = new_rows(p.c, b), shift = shift_of(p.c, b);
        int of_class[3], h = 0, rb = 0;
#pragma unroll
        for (int cls = 0; cls < 3; ++cls) of_class[cls] = p.n_class[cls] ? class_tiles<MB>(p, n, rows, shift, cls) : 0;
        for (;; ++h) {
            const int c = p.head_class[h], t = c == 0 ? of_class[0] : c == 1 ? of_class[1] : of_class[2];
            if (off < t) break;
            off -= t;
        }
        for (;; ++rb) {
            int lo, hi;
            const int t = item_tiles<MB>(p, n, rows, shift, p.head_class[h], rb, &lo, &hi);
            if (off < t) break;
            off -= t;
        }
        out->begin = begin;
        out->end = end;
        out->per = per;
        out->b = b;
        out->h = h;
        out->rb = rb;
        out->tile = off;
    }
    __syncthreads();
}

// ---- shared memory and operand fragments -----------------------------------------------------------------------------
// 16-byte piece c of row r in a tile of RB-byte rows: XORed with the row, so that eight rows at one piece (ldmatrix) and a
// row's pieces (16-byte loads and stores) fall into different banks.
template <int RB>
__device__ __forceinline__ uint32_t swizzled(int r, int c) {
    return (uint32_t)(r * RB + ((c ^ (RB == 64 ? (r >> 1) & 3 : r & 7)) << 4));
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
    // without `there` nothing is read and the 16 bytes become zero
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// d (16 x 8, fp32) += a (16 x 16) b (16 x 8); fp16 operands where HALF, else bf16
template <bool HALF>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two e4m3 values to two fp16 ones (exact)
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3);
    return (uint32_t)h.x | ((uint32_t)h.y << 16);
}
template <bool HALF>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if (HALF) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    return pack_bf16(lo, hi);
}

template <int D, bool FP8, int WM>
struct DecodeShape {
    static constexpr int RB = D * (FP8 ? 1 : 2);           // bytes of a cache row
    static constexpr int kStages = RB == 256 ? 3 : RB == 128 ? 6 : 8;
    static constexpr int kWarpStage = 2 * 16 * RB;         // a warp's 16 K rows and 16 V rows
    static constexpr int kRing = kStages * 4 * kWarpStage;
    static constexpr int MB = 16 * WM;                     // rows of an item
    static constexpr int kMergeRows = WM == 4 ? 0 : 32;    // rows handed over between warps at an item's end
    static constexpr int kMergePitch = D + 4;              // floats
    static constexpr int kMerge = kMergeRows * kMergePitch * 4;
    static constexpr int kDynamic = kRing + kMerge + 128;
};

// One warp's running state for 16 rows.  Lane l holds rows l/4 and l/4 + 8 in the layout of an mma accumulator.
template <int D>
struct RowState {
    float o[D / 8][4];
    float m[2], l[2];  // maximum in log2 units; sum over this lane's columns
};

template <int D, bool FP8, int WM>
__global__ void __launch_bounds__(kDecThreads, kDecBlocksPerSm) decode_kernel(const __grid_constant__ DecodeParams p) {
    using Sh = DecodeShape<D, FP8, WM>;
    constexpr int RB = Sh::RB, C = RB / 16, MB = Sh::MB, ST = Sh::kStages, KS = D / 16;
    extern __shared__ uint8_t smem_raw[];
    __shared__ BlockRange range;
    __shared__ int warp_sum[4];
    __shared__ uint32_t there[ST][4];  // which of a warp's 16 slots were loaded, per stage
    const uint32_t ring = (smem_u32(smem_raw) + 127u) & ~127u;
    float* merge = reinterpret_cast<float*>(smem_raw + (ring - smem_u32(smem_raw)) + Sh::kRing);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q4 = lane & 3;
    const int group = warp / WM, wrow = warp % WM;  // key group of this warp, and its 16 rows of the item

    find_range<MB>(p, &range, warp_sum);
    if (range.begin >= range.end) return;
    const int per = range.per;
    TileCursor<MB> put, get;  // what is loaded next, and what is computed next
    get.b = range.b;
    get.h = range.h;
    get.rb = range.rb;
    get.read_sequence(p);
    get.enter(p, range.tile);
    put = get;
    int put_left = range.end - range.begin, get_left = put_left;

    // One tile's 16 slots of this warp into stage s.
    auto load_tile = [&](int s) {
        if (put_left > 0) {
            if (put.tile == put.end) put.next_item(p);
            const int r = lane & 15, slot = put.first_slot() + warp * 16 + r;
            long long off = -1;  // of row r: lanes 0-15 in K, 16-31 in V
            if (slot >= put.lo && slot < put.hi) {
                int prow;
                const int page = page_of(p.c, put.b, slot, &prow);
                const long long* st = lane < 16 ? p.c.k_stride : p.c.v_stride;
                if (page >= 0) off = page * st[0] + prow * st[1] + put.h * st[2];
            }
            const uint32_t loaded = __ballot_sync(0xffffffffu, off >= 0) & 0xffffu;
            if (lane == 0) there[s][warp] = loaded;
            const uint32_t dst = ring + (uint32_t)(s * 4 + warp) * Sh::kWarpStage;
            constexpr int RPI = 32 / C;  // rows one instruction covers
            const int r0 = lane / C, ch = lane % C;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv)
#pragma unroll
                for (int i = 0; i < 16 / RPI; ++i) {
                    const int row = i * RPI + r0;
                    const long long o = __shfl_sync(0xffffffffu, off, kv * 16 + row);
                    const char* src = (kv ? p.c.V : p.c.K) + (o >= 0 ? o + ch * 16 : 0);
                    cp_async16(dst + kv * 16 * RB + swizzled<RB>(row, ch), src, o >= 0);
                }
            ++put.tile;
            --put_left;
        }
        cp_async_commit();
    };

#pragma unroll
    for (int s = 0; s < ST - 1; ++s) load_tile(s);
    int stage = 0, slot_stage = ST - 1;

    RowState<D> st;
    uint32_t qf[KS][4];
    float qscale[2];     // score scale of the lane's two rows, log2 units
    int rlo[2], rhi[2];  // their visible slots
    while (get_left > 0) {
        // ---- a piece: this block's tiles of one item ----
        const int first = get.tile, count = min(get.end - first, get_left);
        const int cls = p.head_class[get.h], rows = get.rows * p.g;
        const float vs = FP8 ? p.v_scale[get.h] : 1.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = get.rb * MB + wrow * 16 + (lane >> 2) + 8 * i;
            const bool real = r < rows;
            const int t = (int)fdiv((uint32_t)(real ? r : 0), p.f_g), qh = get.h * p.g + (real ? r - t * p.g : 0);
            visible_slots(p, get.n, get.rows, get.shift, t, cls, &rlo[i], &rhi[i]);
            const __nv_bfloat16* q = p.Q + get.b * p.q_stride[0] + t * p.q_stride[1] + qh * p.q_stride[2];
            if (FP8) {
                // Lane q4 of a row takes D/4 consecutive elements, in the order in which it meets the bytes of K.  They go
                // to fp16 after a division by a power of two that brings the row's largest below 2: what a bf16 value
                // then loses lies under 2^-25 of that largest one.
                uint4 raw[D / 32];
                float x[D / 4], big = 0.f;
#pragma unroll
                for (int k = 0; k < D / 32; ++k) raw[k] = *reinterpret_cast<const uint4*>(q + q4 * (D / 4) + 8 * k);
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    const __nv_bfloat162* b2 = reinterpret_cast<const __nv_bfloat162*>(&raw[k]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 f = __bfloat1622float2(b2[e]);
                        x[8 * k + 2 * e] = f.x;
                        x[8 * k + 2 * e + 1] = f.y;
                        big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
                    }
                }
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                const int e = big > 0.f ? min(max((int)(__float_as_uint(big) >> 23) - 127, -126), 126) : 0;
                const float down = __uint_as_float((uint32_t)(127 - e) << 23);
                qscale[i] = p.scale_log2 * p.k_scale[get.h] * __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    qf[k][i] = real ? pack16<true>(x[4 * k] * down, x[4 * k + 1] * down) : 0u;
                    qf[k][2 + i] = real ? pack16<true>(x[4 * k + 2] * down, x[4 * k + 3] * down) : 0u;
                }
            } else {
                qscale[i] = p.scale_log2;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    qf[k][i] = real ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 2 * q4) : 0u;
                    qf[k][2 + i] = real ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 8 + 2 * q4) : 0u;
                }
            }
            st.m[i] = -INFINITY;
            st.l[i] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < D / 8; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) st.o[k][e] = 0.f;
        // slots that every row of the item sees: no mask there
        int all_lo, all_hi;
        {
            const int r_last = min((get.rb + 1) * MB, rows) - 1;
            int x;
            visible_slots(p, get.n, get.rows, get.shift, (int)fdiv((uint32_t)r_last, p.f_g), cls, &all_lo, &x);
            visible_slots(p, get.n, get.rows, get.shift, (int)fdiv((uint32_t)(get.rb * MB), p.f_g), cls, &x, &all_hi);
        }
        float* score_row[2];
        if (p.scores) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = get.rb * MB + wrow * 16 + (lane >> 2) + 8 * i;
                score_row[i] = r < rows ? p.scores + (((long long)get.b * p.c.Hkv + get.h) * p.g * p.c.Lq + r) * p.pitch : nullptr;
            }
        }

        for (int left = count; left > 0; --left) {
            cp_async_wait<ST - 2>();
            if (WM == 1) __syncwarp();
            else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(32 * WM) : "memory");
            load_tile(slot_stage);
            slot_stage = stage;
            // this warp's key group: 16 WM slots, loaded by the group's WM warps
            const int slot0 = get.first_slot() + group * 16 * WM;
            float s[WM][2][4];
#pragma unroll
            for (int k = 0; k < WM; ++k) {
                const uint32_t kb = ring + (uint32_t)(stage * 4 + group * WM + k) * Sh::kWarpStage;
#pragma unroll
                for (int n8 = 0; n8 < 2; ++n8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[k][n8][e] = 0.f;
                if (FP8) {
#pragma unroll
                    for (int n8 = 0; n8 < 2; ++n8) {
                        const int row = n8 * 8 + (lane >> 2);
#pragma unroll
                        for (int v = 0; v < D / 64; ++v) {
                            const uint4 w = lds128(kb + swizzled<RB>(row, q4 * (D / 64) + v));
                            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                mma16816<true>(s[k][n8], qf[v * 4 + j], e4m3x2_to_half2(ww[j]), e4m3x2_to_half2(ww[j] >> 16));
                        }
                    }
                } else {
#pragma unroll
                    for (int c2 = 0; c2 < KS; ++c2) {
                        // matrices: (slots 0-7, piece 2 c2), (slots 0-7, next piece), (slots 8-15, ...) x 2
                        uint32_t b[4];
                        ldsm_x4(kb + swizzled<RB>((lane & 7) + ((lane >> 4) << 3), 2 * c2 + ((lane >> 3) & 1)), b);
                        mma16816<false>(s[k][0], qf[c2], b[0], b[1]);
                        mma16816<false>(s[k][1], qf[c2], b[2], b[3]);
                    }
                }
            }
            // scores in log2 units, masked where this tile is not seen whole by every row
            const bool edge_range = slot0 < all_lo || slot0 + 16 * WM > all_hi;
            bool edge = edge_range;
#pragma unroll
            for (int k = 0; k < WM; ++k) edge |= there[stage][group * WM + k] != 0xffffu;
            float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int k = 0; k < WM; ++k)
#pragma unroll
                for (int n8 = 0; n8 < 2; ++n8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = s[k][n8][e] * qscale[e >> 1];
                        if (edge) {
                            const int j = n8 * 8 + q4 * 2 + (e & 1), slot = slot0 + k * 16 + j;
                            if (slot < rlo[e >> 1] || slot >= rhi[e >> 1] || !((there[stage][group * WM + k] >> j) & 1)) x = -INFINITY;
                        }
                        s[k][n8][e] = x;
                        mx[e >> 1] = fmaxf(mx[e >> 1], x);
                    }
            if (p.scores) {
#pragma unroll
                for (int k = 0; k < WM; ++k)
#pragma unroll
                    for (int n8 = 0; n8 < 2; ++n8)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (score_row[i])
                                *reinterpret_cast<float2*>(score_row[i] + slot0 + k * 16 + n8 * 8 + q4 * 2) =
                                    make_float2(s[k][n8][2 * i], s[k][n8][2 * i + 1]);
            }
            float base[2];
            bool grows = false;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
                grows |= mx[i] > st.m[i];
            }
            if (__any_sync(0xffffffffu, grows)) {
                float f[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float mn = fmaxf(st.m[i], mx[i]);
                    f[i] = mn == -INFINITY ? 1.f : ex2(st.m[i] - mn);
                    st.m[i] = mn;
                    st.l[i] *= f[i];
                }
#pragma unroll
                for (int k = 0; k < D / 8; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.o[k][e] *= f[e >> 1];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) base[i] = st.m[i] == -INFINITY ? 0.f : st.m[i];
#pragma unroll
            for (int k = 0; k < WM; ++k) {
                const uint32_t vb = ring + (uint32_t)(stage * 4 + group * WM + k) * Sh::kWarpStage + 16 * RB;
#pragma unroll
                for (int n8 = 0; n8 < 2; ++n8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[k][n8][e] = ex2(s[k][n8][e] - base[e >> 1]);
                        st.l[e >> 1] += s[k][n8][e];
                    }
                const uint32_t a[4] = {pack16<FP8>(s[k][0][0], s[k][0][1]), pack16<FP8>(s[k][0][2], s[k][0][3]),
                                       pack16<FP8>(s[k][1][0], s[k][1][1]), pack16<FP8>(s[k][1][2], s[k][1][3])};
                // A weight of zero does not undo an infinite or NaN V: slots that some rows of the item see and others do not
                // (rows behind a row, slots across a segment's border) are looked at, and where V is not finite its product is
                // taken out of the mma and added to the rows that see it one by one.
                uint32_t bad = 0;
                if (edge_range) {
                    const int b0 = slot0 + k * 16;
                    uint32_t part = 0;
                    for (int j = 0; j < 16; ++j)
                        if (b0 + j < all_lo || b0 + j >= all_hi) part |= 1u << j;
                    part &= there[stage][group * WM + k];
                    while (part) {
                        const int j = __ffs(part) - 1;
                        part &= part - 1;
                        bool odd = false;
                        if (lane < C) {
                            const uint4 w = lds128(vb + swizzled<RB>(j, lane));
                            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if (FP8) {
#pragma unroll
                                    for (int y = 0; y < 4; ++y) odd |= ((ww[e] >> (8 * y)) & 0x7fu) == 0x7fu;
                                } else {
                                    odd |= (ww[e] & 0x7f80u) == 0x7f80u || (ww[e] & 0x7f800000u) == 0x7f800000u;
                                }
                            }
                        }
                        if (__any_sync(0xffffffffu, odd)) bad |= 1u << j;
                    }
                }
                uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;  // of the lane's V fragments: slots 2 q4, 2 q4 + 1 and 8 on
                if (bad) {
                    const uint32_t t0 = bad >> (2 * q4), t1 = bad >> (2 * q4 + 8);
                    keep0 = (t0 & 1 ? 0u : 0xffffu) | (t0 & 2 ? 0u : 0xffff0000u);
                    keep1 = (t1 & 1 ? 0u : 0xffffu) | (t1 & 2 ? 0u : 0xffff0000u);
                }
#pragma unroll
                for (int c2 = 0; c2 < C / 2; ++c2) {
                    if (FP8) {
                        // (slots 0-7, piece 2 c2), (slots 8-15, same), and the next piece: 16 dims of V to a piece; even and odd
                        // dims of it go to two mma tiles
                        uint32_t b[4];
                        ldsm_x4_t(vb + swizzled<RB>(lane & 15, 2 * c2 + (lane >> 4)), b);
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint32_t l0 = e4m3x2_to_half2(b[2 * x]), h0 = e4m3x2_to_half2(b[2 * x] >> 16);
                            const uint32_t l1 = e4m3x2_to_half2(b[2 * x + 1]), h1 = e4m3x2_to_half2(b[2 * x + 1] >> 16);
                            mma16816<true>(st.o[4 * c2 + 2 * x], a, __byte_perm(l0, h0, 0x5410) & keep0, __byte_perm(l1, h1, 0x5410) & keep1);
                            mma16816<true>(st.o[4 * c2 + 2 * x + 1], a, __byte_perm(l0, h0, 0x7632) & keep0, __byte_perm(l1, h1, 0x7632) & keep1);
                        }
                    } else {
                        uint32_t b[4];
                        ldsm_x4_t(vb + swizzled<RB>(lane & 15, 2 * c2 + (lane >> 4)), b);
                        mma16816<false>(st.o[2 * c2], a, b[0] & keep0, b[1] & keep1);
                        mma16816<false>(st.o[2 * c2 + 1], a, b[2] & keep0, b[3] & keep1);
                    }
                }
                while (bad) {
                    const int j = __ffs(bad) - 1;
                    bad &= bad - 1;
                    const int slot = slot0 + k * 16 + j;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        // the weight of (row, j): column j & 7 of n8 = j / 8, held by lane (row, (j & 7) / 2)
                        const float x0 = j & 8 ? s[k][1][2 * i] : s[k][0][2 * i], x1 = j & 8 ? s[k][1][2 * i + 1] : s[k][0][2 * i + 1];
                        const float w = __shfl_sync(0xffffffffu, j & 1 ? x1 : x0, (lane & ~3) | ((j & 7) >> 1));
                        if (slot < rlo[i] || slot >= rhi[i]) continue;
#pragma unroll
                        for (int nt = 0; nt < D / 8; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int dim = FP8 ? (nt >> 1) * 16 + 4 * q4 + 2 * e + (nt & 1) : nt * 8 + 2 * q4 + e;
                                const uint32_t at = vb + swizzled<RB>(j, dim * (FP8 ? 1 : 2) / 16) + dim * (FP8 ? 1 : 2) % 16;
                                float v;
                                if (FP8) {
                                    uint32_t byte;
                                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(byte) : "r"(at));
                                    v = __half2float(__ushort_as_half((unsigned short)(e4m3x2_to_half2(byte) & 0xffffu)));
                                } else {
                                    uint16_t h16;
                                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h16) : "r"(at));
                                    v = __uint_as_float((uint32_t)h16 << 16);
                                }
                                st.o[nt][2 * i + e] += w * v;
                            }
                    }
                }
            }
            stage = stage + 1 == ST ? 0 : stage + 1;
            ++get.tile;
        }
        get_left -= count;

        // ---- the piece's rows: over the lanes of a row, then over the key groups ----
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            st.l[i] += __shfl_xor_sync(0xffffffffu, st.l[i], 1);
            st.l[i] += __shfl_xor_sync(0xffffffffu, st.l[i], 2);
        }
        // warps [half, 2 half) hand their state to warps [0, half); only rows that are there
#pragma unroll
        for (int half = 2; half >= WM; half >>= 1) {
            if (WM == 4) break;
            float* mine = merge + ((warp % half) * 16 + (lane >> 2)) * Sh::kMergePitch;
            if (warp >= half && warp < 2 * half) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float* to = mine + 8 * i * Sh::kMergePitch;
#pragma unroll
                    for (int nt = 0; nt < D / 8; ++nt)
                        *reinterpret_cast<float2*>(to + nt * 8 + 2 * q4) = make_float2(st.o[nt][2 * i], st.o[nt][2 * i + 1]);
                    if (q4 == 0) *reinterpret_cast<float2*>(to + D) = make_float2(st.m[i], st.l[i]);
                }
            }
            __syncthreads();
            if (warp < half) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float* from = mine + 8 * i * Sh::kMergePitch;
                    const float2 ml = *reinterpret_cast<const float2*>(from + D);
                    const float mn = fmaxf(st.m[i], ml.x), zero = mn == -INFINITY ? 0.f : mn;
                    const float fa = ex2(st.m[i] - zero), fb = ex2(ml.x - zero);
                    st.m[i] = mn;
                    st.l[i] = st.l[i] * fa + ml.y * fb;
#pragma unroll
                    for (int nt = 0; nt < D / 8; ++nt) {
                        const float2 v = *reinterpret_cast<const float2*>(from + nt * 8 + 2 * q4);
                        st.o[nt][2 * i] = st.o[nt][2 * i] * fa + v.x * fb;
                        st.o[nt][2 * i + 1] = st.o[nt][2 * i + 1] * fa + v.y * fb;
                    }
                }
            }
            __syncthreads();
        }
        if (group == 0) {
            // the item's tiles are numbered from here on in the list of all tiles
            const int list0 = range.end - get_left - count - first;
            const int b_first = list0 / per, b_last = (list0 + get.end - 1) / per;
            if (first == 0 && wrow == 0 && lane == 0)
                p.item_blocks[((long long)get.b * p.c.Hkv + get.h) * p.row_blocks + get.rb] = make_int2(b_first, b_last);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int rl = wrow * 16 + (lane >> 2) + 8 * i, r = get.rb * MB + rl;
                if (r >= rows) continue;
                if (b_first == b_last) {
                    const int t = (int)fdiv((uint32_t)r, p.f_g), qh = get.h * p.g + r - t * p.g;
                    const float inv = st.l[i] == 0.f ? 0.f : vs / st.l[i];
                    __nv_bfloat16* o = p.O + get.b * p.o_stride[0] + t * p.o_stride[1] + qh * p.o_stride[2];
                    if (FP8) {
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) {
                            const uint32_t lo2 = pack_bf16(st.o[2 * x][2 * i] * inv, st.o[2 * x + 1][2 * i] * inv);
                            const uint32_t hi2 = pack_bf16(st.o[2 * x][2 * i + 1] * inv, st.o[2 * x + 1][2 * i + 1] * inv);
                            *reinterpret_cast<uint2*>(o + 16 * x + 4 * q4) = make_uint2(lo2, hi2);
                        }
                    } else {
#pragma unroll
                        for (int nt = 0; nt < D / 8; ++nt)
                            *reinterpret_cast<uint32_t*>(o + nt * 8 + 2 * q4) = pack_bf16(st.o[nt][2 * i] * inv, st.o[nt][2 * i + 1] * inv);
                    }
                    if (q4 == 0)
                        p.LSE[((long long)get.b * p.Hq + qh) * p.c.Lq + t] =
                            st.l[i] == 0.f ? -INFINITY : (st.m[i] + log2f(st.l[i])) * 0.6931471805599453f;
                } else {
                    // a part: slot 0 where the block's range begins inside the item, else slot 1
                    const long long at = ((long long)blockIdx.x * 2 + (first == 0 ? 1 : 0)) * MB + rl;
                    float* o = p.part_o + at * D;
#pragma unroll
                    for (int nt = 0; nt < D / 8; ++nt) {
                        if (FP8) {
                            if (nt & 1) continue;
                            *reinterpret_cast<float4*>(o + nt * 8 + 4 * q4) = make_float4(
                                st.o[nt][2 * i] * vs, st.o[nt + 1][2 * i] * vs, st.o[nt][2 * i + 1] * vs, st.o[nt + 1][2 * i + 1] * vs);
                        } else {
                            *reinterpret_cast<float2*>(o + nt * 8 + 2 * q4) = make_float2(st.o[nt][2 * i], st.o[nt][2 * i + 1]);
                        }
                    }
                    if (q4 == 0) p.part_ml[at] = make_float2(st.m[i], st.l[i]);
                }
            }
        }
        if (get_left > 0) get.next_item(p);
    }
    cp_async_wait<0>();
}

// Adds the parts of one row of an item that several blocks share; block.x = the row, block.y = the item.
template <int D>
__global__ void __launch_bounds__(D) decode_join_kernel(const __grid_constant__ DecodeParams p, int MB) {
    const int rb = blockIdx.y % p.row_blocks, u = blockIdx.y / p.row_blocks, h = u % p.c.Hkv, b = u / p.c.Hkv;
    const int rl = blockIdx.x, r = rb * MB + rl;
    if (r >= new_rows(p.c, b) * p.g) return;
    const int2 blocks = p.item_blocks[blockIdx.y];
    if (blocks.x == blocks.y) return;
    // the item's first block holds its part in slot 1 (its range began at or before the item), the others in slot 0
    auto at = [&](int k) { return ((long long)k * 2 + (k == blocks.x ? 1 : 0)) * MB + rl; };
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int k = blocks.x; k <= blocks.y; ++k) m = fmaxf(m, p.part_ml[at(k)].x);
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 4
    for (int k = blocks.x; k <= blocks.y; ++k) {
        const float2 ml = p.part_ml[at(k)];
        const float f = ex2(ml.x - base);
        l += ml.y * f;
        o += p.part_o[at(k) * D + threadIdx.x] * f;
    }
    const int t = (int)fdiv((uint32_t)r, p.f_g), qh = h * p.g + r - t * p.g;
    p.O[b * p.o_stride[0] + t * p.o_stride[1] + qh * p.o_stride[2] + threadIdx.x] = __float2bfloat16(l == 0.f ? 0.f : o / l);
    if (threadIdx.x == 0) p.LSE[((long long)b * p.Hq + qh) * p.c.Lq + t] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// Attention weight of every slot, from the scores and the finished LSE: one thread per slot.
__global__ void __launch_bounds__(256) decode_weights_kernel(const __grid_constant__ DecodeParams p) {
    const int j = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int rows = new_rows(p.c, b), n = seq_len(p.c, b);
    if (j >= n || rows == 0) return;
    const int shift = shift_of(p.c, b), cls = p.head_class[h];
    const long long unit = (long long)b * p.c.Hkv + h;
    const float* s = p.scores + unit * p.g * p.c.Lq * p.pitch + j;
    float sum = 0.f;
    for (int t = 0; t < rows; ++t) {
        int lo, hi;
        visible_slots(p, n, rows, shift, t, cls, &lo, &hi);
        if (j < lo || j >= hi) continue;
        for (int k = 0; k < p.g; ++k) {
            const float lse = p.LSE[((long long)b * p.Hq + h * p.g + k) * p.c.Lq + t];
            if (lse != -INFINITY) sum += ex2(s[(long long)(t * p.g + k) * p.pitch] - lse * 1.4426950408889634f);
        }
    }
    const long long at = unit * p.W + j;
    p.w_out[at] = (p.w_in ? p.w_in[at] : 0.f) + sum;
}

}  // namespace segattn
