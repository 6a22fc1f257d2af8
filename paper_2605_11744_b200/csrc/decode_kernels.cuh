// Attention of a sequence's newest rows over its paged cache.
//
// The work is a stream over the visible K and V rows (HBM bound: 4 g flops per byte for g query heads to a KV head), so the
// kernel is built around the loads.  Its unit is a tile of 64 slots of one item, an item being up to 8 NT WM rows (new row,
// query head) of one (sequence, KV head).  All tiles of all items form one list, which the grid - two or three blocks to an SM -
// cuts into equal ranges by the lengths found in device memory: whatever the batch's mix of lengths and head classes, every
// SM reads the same number of bytes.  Where a range ends inside an item the block leaves an unnormalised part (O, running
// base, sum) in the workspace, and decode_join_kernel adds the parts up in the order of the ranges.
//
// Inside a block four warps load 16 slots of a tile each with cp.async into a ring of their own, several tiles ahead and
// across item borders.  For up to 16 rows (WM = 1) each warp attends over its own 16 slots with its own base and sum and
// needs no block barrier until an item ends; for more rows WM = 2 or 4 warps share 32 or 64 slots, so that a row of K is
// read once for 32 or 64 rows.
//
// Products run on mma.sync with the slots in M and the query rows in N: S^T = K Q^T (16 slots x 8 rows) and O^T = V^T P^T
// (16 dims x 8 rows).  Eight query heads fill a tile of that shape; with the rows in M half of it would be padding, and
// tcgen05.mma, which starts at 64 (the slots could fill that, but P^T would have to pass through shared memory for every
// tile), buys nothing where three quarters of the issue slots are free.
//
// 16 sequences of 16-32K slots, 8 KV heads with their whole past, 8 query heads each, d = 128: 248 us for 1.69 GB (6.8 TB/s);
// with the rows in M, a maximum per tile and a look-up per row it was 389 us.  8-bit caches are held up by what a value costs to
// convert (453 instructions per 16 slots at first, 240 now) and by DRAM pieces of 64 or 128 bytes.
//
// Two more forms of the same kernel: with a scale for each block of rows (BS: 8 sequences of 100-131K slots, every second of 8 heads,
// 168-181 us on different cards for 1.04 GB, 5.8-6.2 TB/s), and with chosen blocks in the place of the far past (SEL; with scales, 16 sequences of 90-131K slots,
// four rows each of 64 blocks and 2-3K slots of their own: 123-129 us for the 595 MB that they cannot do without).  The latter
// waits: three warps to a scheduler leave half of the issue slots empty (5.7 cycles to an instruction of a warp) and DRAM at 58%.  Four query
// heads leave half of each product empty, and a start of 7 us (length, list, page, rows) weighs more.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "paged_cache.cuh"

namespace segattn {

constexpr int kDecThreads = 128;
constexpr int kDecMaxBlocks = 480;  // blocks a launch has at most: what the parts in the workspace are laid out for

struct DecodeParams {
    PagedView c;
    const __nv_bfloat16* Q;
    __nv_bfloat16* O;
    float* LSE;                      // [B][Hq][Lq]
    const float* w_in;               // [B][Hkv][W] or null
    float* w_out;                    // or null
    const float *k_scale, *v_scale;  // e4m3 only
    // workspace
    float* part_o;                   // [grid][2][rows of a unit][D]
    float2* part_ml;                 // [grid][2][rows of a unit] (base in log2 units, sum)
    int2* item_blocks;               // [B][Hkv][row blocks]: first and last block of the item's tiles
    float* scores;                   // [B][Hkv][g Lq][pitch], log2 units; null unless weights are asked for
    long long q_stride[3], o_stride[3];
    FastDiv f_S, f_g;
    int S, T, W, Hq, g;
    int row_blocks;                  // ceil(g Lq / (rows of an item))
    int blocks;                      // blocks the workspace has parts for
    int page_whole;                  // page_size is a multiple of 16: a warp's slots lie in one page
    int pitch;                       // slots in a row of scores
    float scale_log2;                // sm_scale * log2(e)
    // KV heads are taken in units of one class: 1, 2 or 4 of them, side by side in the block's warps
    int unit_log[3], units[3];       // by class: heads to a unit (log2), and units
    uint8_t head_class[64];
    uint8_t head_order[64];          // the heads by class, unit after unit
    uint8_t head_in_unit[64];        // by head
    // an 8-bit cache with a scale for each block of 2^scale_log rows of a page and head
    const float *ks, *vs;
    long long ks_stride[3], vs_stride[3];  // elements, for (page, block of the page, head)
    int scale_log;
    // blocks of 2^choice_log slots that heads with a past read of what lies behind their tail
    int choice_log, n_chosen;
    const int32_t* chosen;           // [B][Lq][Hkv][n_chosen]; null: no choice, the whole past
    int page_pair;                   // 32 slots or numbers from a multiple of 32 on lie in one page, one after the other
    int head_blocks;                 // ceil(g / (rows of an item)), an item being of one new row
};

// Programmatic launch: the next kernel of the stream may be set up from here on, and this kernel waits for the end (and the
// writes) of the one before it.
__device__ __forceinline__ void next_kernel_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void after_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

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

// With chosen blocks an item is up to MB query heads of one new row, and its slots are numbered through: a head with a past has
// the chosen blocks one after the other in [0, far), then what it sees whole, from its tail's start (rounded down to a block) on:
// number v stands for slot v + off there.  Every number in [*lo, *hi) is visible to every row of the item.
__device__ __forceinline__ void numbered_slots(const DecodeParams& p, int n, int rows, int shift, int t, int cls, int* lo, int* hi, int* far, int* off) {
    visible_slots(p, n, rows, shift, t, cls == kHeadPast ? kHeadLocal : cls, lo, hi);
    *far = *off = 0;
    if (cls == kHeadPast) {
        const int blocks = *lo >> p.choice_log, whole = blocks << p.choice_log;
        *far = min(blocks, p.n_chosen) << p.choice_log;
        *off = whole - *far;
        *hi = max(*hi - *off, *far);
        *lo = 0;
    }
    *hi = max(*hi, *lo);
}

// ---- the list of tiles -------------------------------------------------------------------------------------------
// Slots the rows of one row block see between them (their lower and upper ends both grow with the row), and its tiles:
// whole tiles of 2^tile_log slots, at least one, so that rows that see nothing are written too.
template <int MB, bool SEL = false>
__device__ __forceinline__ int item_tiles(const DecodeParams& p, int n, int rows, int shift, int cls, int tile_log, int rb, int* lo, int* hi) {
    if (SEL) {
        int far, off;
        numbered_slots(p, n, rows, shift, rb / p.head_blocks, cls, lo, hi, &far, &off);
        return max(1, ((*hi + (1 << tile_log) - 1) >> tile_log) - (*lo >> tile_log));
    }
    const int last = min((rb + 1) * MB, rows * p.g) - 1;
    int l0, h0, l1, h1;
    visible_slots(p, n, rows, shift, (int)fdiv((uint32_t)(rb * MB), p.f_g), cls, &l0, &h0);
    visible_slots(p, n, rows, shift, (int)fdiv((uint32_t)last, p.f_g), cls, &l1, &h1);
    *lo = l0;
    *hi = max(h1, l0);
    return max(1, ((*hi + (1 << tile_log) - 1) >> tile_log) - (l0 >> tile_log));
}

// whether row block rb of a sequence has a row
template <int MB, bool SEL>
__device__ __forceinline__ bool has_rows(const DecodeParams& p, int rows, int rb) {
    return SEL ? rb < rows * p.head_blocks : rb * MB < rows * p.g;
}
// New row t and query head hq (of its KV head) that row i of a row block stands for; whether it is there (else t of a row that is).
template <int MB, bool SEL>
__device__ __forceinline__ bool row_of(const DecodeParams& p, int rows, int rb, int i, int* t, int* hq) {
    if (SEL) {
        *t = rb / p.head_blocks;
        *hq = (rb - *t * p.head_blocks) * MB + i;
        return *hq < p.g;
    }
    const int r = rb * MB + i;
    const bool real = r < rows * p.g;
    *t = (int)fdiv((uint32_t)(real ? r : 0), p.f_g);
    *hq = r - *t * p.g;
    return real;
}

// Tiles of one unit of class cls of a sequence.  A unit's tile has 2^(TILE_LOG - unit_log) slots: the same bytes for all.
template <int MB, int TILE_LOG, bool SEL = false>
__device__ __forceinline__ int unit_tiles(const DecodeParams& p, int n, int rows, int shift, int cls) {
    int sum = 0, lo, hi;
    for (int rb = 0; has_rows<MB, SEL>(p, rows, rb); ++rb) sum += item_tiles<MB, SEL>(p, n, rows, shift, cls, TILE_LOG - p.unit_log[cls], rb, &lo, &hi);
    return sum;
}

__device__ __forceinline__ int class_of_unit(const DecodeParams& p, int u, int* first_head) {
    int cls = 0, first = 0;
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (cls == c && u >= p.units[c]) {
            u -= p.units[c];
            first += p.units[c] << p.unit_log[c];
            cls = c + 1;
        }
    *first_head = first + (u << p.unit_log[cls]);
    return cls;
}

// A place in the list: an item (a row block of a unit of a sequence) and a tile of it.
template <int MB, int TILE_LOG, bool SEL = false>
struct TileCursor {
    int b, u, rb, n, rows, shift;
    int cls, log, first_head;    // of the unit; it has 2^log heads
    int lo, hi;                  // visible slots of the item
    int tile, end;               // next tile of the item and the number of its tiles
    __device__ __forceinline__ void read_sequence(const DecodeParams& p) {
        n = seq_len(p.c, b);
        rows = new_rows(p.c, b);
        shift = shift_of(p.c, b);
    }
    __device__ __forceinline__ void enter(const DecodeParams& p, int at) {
        cls = class_of_unit(p, u, &first_head);
        log = p.unit_log[cls];
        end = item_tiles<MB, SEL>(p, n, rows, shift, cls, TILE_LOG - log, rb, &lo, &hi);
        tile = at;
    }
    // the item after this one; the caller knows that there is one
    __device__ __forceinline__ void next_item(const DecodeParams& p) {
        if (!has_rows<MB, SEL>(p, rows, ++rb)) {
            rb = 0;
            if (++u == p.units[0] + p.units[1] + p.units[2]) {
                u = 0;
                do {
                    ++b;
                    read_sequence(p);
                } while (rows == 0 && b + 1 < p.c.B);
            }
        }
        enter(p, 0);
    }
    __device__ __forceinline__ int first_slot() const {
        return ((lo >> (TILE_LOG - log)) + tile) << (TILE_LOG - log);
    }
};

// This block's range of tiles, and the item it begins in.  Every block counts the tiles of all sequences: they are read
// from device memory, so that a captured call follows the lengths.
struct BlockRange {
    int begin, end, per, b, u, rb, tile;
};
template <int MB, int TILE_LOG, bool SEL = false>
__device__ __forceinline__ void find_range(const DecodeParams& p, BlockRange* out, int* warp_sum) {
    // A thread takes a run of (sequence, class) pairs, four to a sequence (the last is empty), so that for up to 32 sequences none
    // has more than one of them: this part of the kernel is a chain of few instructions on data that nothing waits beside.
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int pairs = 4 * p.c.B, seg = (pairs + kDecThreads - 1) / kDecThreads;
    const int e0 = min(tid * seg, pairs), e1 = min(e0 + seg, pairs);
    auto tiles_of = [&](int e) {
        const int b = e >> 2, cls = e & 3;
        if (cls == 3 || p.units[cls] == 0) return 0;
        const int rows = new_rows(p.c, b);
        return rows == 0 ? 0 : p.units[cls] * unit_tiles<MB, TILE_LOG, SEL>(p, seq_len(p.c, b), rows, shift_of(p.c, b), cls);
    };
    int mine = 0;
    for (int e = e0; e < e1; ++e) mine += tiles_of(e);
    int before = mine;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, before, x);
        if (lane >= x) before += y;
    }
    if (lane == 31 && warp < kDecThreads / 32) warp_sum[warp] = before;  // the block's further warps have no sequence
    if (tid == 0) out->begin = out->end = 0;
    __syncthreads();
    int total = 0;
    before -= mine;
    for (int k = 0; k < kDecThreads / 32; ++k) {
        if (k < warp) before += warp_sum[k];
        total += warp_sum[k];
    }
    const int per = max(1, (total + (int)gridDim.x - 1) / (int)gridDim.x);
    const int begin = min((int)blockIdx.x * per, total), end = min(begin + per, total);
    if (begin < end && begin >= before && begin < before + mine) {
        int off = begin - before, e = e0, t = mine;
        if (seg > 1)
            for (;; ++e) {
                t = tiles_of(e);
                if (off < t) break;
                off -= t;
            }
        const int b = e >> 2, cls = e & 3;
        const int n = seq_len(p.c, b), rows = new_rows(p.c, b), shift = shift_of(p.c, b);
        int u = cls > 0 ? p.units[0] : 0, rb = 0;
        if (cls > 1) u += p.units[1];
        t /= p.units[cls];  // of one unit
        u += off / t;
        off %= t;
        for (;; ++rb) {
            int lo, hi;
            const int t = item_tiles<MB, SEL>(p, n, rows, shift, cls, TILE_LOG - p.unit_log[cls], rb, &lo, &hi);
            if (off < t) break;
            off -= t;
        }
        out->begin = begin;
        out->end = end;
        out->per = per;
        out->b = b;
        out->u = u;
        out->rb = rb;
        out->tile = off;
    }
    __syncthreads();
}

// The block table and the lists of chosen blocks, on their way to L2 while a block finds its range: each is the next link of a chain
// of dependent reads (length, list, page, rows) that the first tile waits for, and all but the length's would come from DRAM.  A
// few KB to a block at most: a table with much more room than the sequences fill is left alone.
__device__ __forceinline__ void prefetch_numbers(const DecodeParams& p) {
    auto fetch = [](const void* at) { asm volatile("prefetch.global.L2 [%0];" ::"l"(at)); };
    const int i0 = blockIdx.x * kDecThreads + threadIdx.x, step = gridDim.x * kDecThreads;
    const int row = (p.c.max_pages + 31) / 32;  // lines of 128 bytes
    if ((long long)p.c.B * row <= step)
        for (int i = i0; i < p.c.B * row; i += step) fetch(p.c.block_table + (long long)(i / row) * p.c.table_stride + i % row * 32);
    const long long lines = p.chosen ? ((long long)p.c.B * p.c.Lq * p.c.Hkv * p.n_chosen + 31) / 32 : 0;
    if (lines <= step)
        for (int i = i0; i < (int)lines; i += step) fetch(p.chosen + i * 32);
}

// ---- shared memory and operand fragments -----------------------------------------------------------------------------
// 16-byte piece c of row r in a tile of RB-byte rows: XORed with the row, so that eight rows at one piece (ldmatrix) and a
// row's pieces (16-byte loads and stores) fall into different banks.
template <int RB>
__device__ __forceinline__ uint32_t swizzled(int r, int c) {
    return (uint32_t)(r * RB + ((c ^ (RB == 64 ? (r >> 1) & 3 : r & 7)) << 4));
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16_if(uint32_t dst, const void* src, bool there) {
    // without `there` nothing is read and the 16 bytes become zero
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16_hint(uint32_t dst, const void* src, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
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
// two 16 x 16 blocks of bytes, transposed: lane l gets column l/4 (then l/4 + 8), rows 4 (l%4) .. + 3, of each
__device__ __forceinline__ void ldsm8_x2_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];"
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
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// four e4m3 values to four fp16 ones (exact): the lower two bytes to lo, the upper two to hi
__device__ __forceinline__ void e4m3x4_to_half(uint32_t x, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(x));
}
template <bool HALF>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if (HALF) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    return pack_bf16(lo, hi);
}

__device__ __forceinline__ uint32_t movm_t(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

template <bool V>
struct Flag {
    static constexpr bool value = V;
};

template <int D, bool FP8, int NT, int WM, bool BS = false, bool SEL = false>
struct DecodeShape {
    static constexpr int RB = D * (FP8 ? 1 : 2);           // bytes of a cache row
    static constexpr int KG = RB == 256 ? 1 : 2;           // blocks of 16 slots of a warp in a tile
    static constexpr int kTileLog = KG == 1 ? 6 : 7;       // log2 of 64 KG, slots of a tile of one head
    static constexpr int kBlock = 2 * 16 * RB;             // 16 K rows and 16 V rows
    static constexpr int kWarpStage = KG * kBlock;
    // with scales or a choice there are more instructions to a row and less of a warp's time is waiting for loads: a third warp to
    // a scheduler, for a stage less (16 x 4 rows of chosen blocks 150 -> 139 us, 8 x 100-131K slots with scales 174 -> 172)
    static constexpr bool kThree = (BS || SEL) && RB == 128 && NT == 1 && FP8;
    static constexpr int kBlocksPerSm = kThree || (RB == 64 && NT == 1) ? 3 : 2;
    static constexpr int KP = KG == 2 || WM > 1 ? 2 : 1;   // blocks of 16 slots taken through the products at once
    static constexpr int kStages = kThree ? 2 : RB == 64 ? (NT == 1 ? 4 : 6) : 3;
    static constexpr int kWR = 8 * NT;                     // rows of a warp
    static constexpr int MB = kWR * WM;                    // rows of an item, of each of its heads
    static constexpr int kPartRows = WM == 1 ? 4 * kWR : MB;  // rows of a unit's item
    static constexpr int kDynamic = kStages * 4 * kWarpStage + 128;
    static_assert(8 * D * 4 <= kWarpStage, "eight rows of an item's end go through a warp's free stage");
};

// A weight of exp2(score - base) may exceed 1 by this power of two before the base is moved up to the row's maximum: most
// tiles then need no maximum across lanes and no rescaling.  A weight in bf16 keeps its relative precision wherever it lies.
constexpr float kDecSlack = 8.f;
// One in fp16, beside an 8-bit cache, keeps it down to 2^-14 only, and from 2^-25 on it is zero: a base at the maximum would
// lose the small weights of a long cache that one key dominates (32K slots that share a hundredth of the weight came out wrong
// by an eighth).  So the base is put 2^13 under the maximum, and moved when a weight would pass 2^15, fp16's largest power:
// weights are exact to fp16's half step down to 2^-27 of the largest.
constexpr float kHalfRoom = 13.f, kHalfTop = 15.f;
// With a scale for each block of rows a weight goes into the product with V times its block's scale m 2^e (1 <= |m| < 2): as
// m exp2(score + e - base), so that fp16's range is spent on what a weight adds to O and not on the scale, whatever its size.  The
// sum takes exp2(score + e - base) 2^(ref - e), exactly, ref being the smallest e that the warp has met in the item: no weight adds more
// than 2^14, so the sum cannot overflow wherever the scales lie.  Bases are whole numbers there (e - base is exact), and one lower for m.
// A scale that has no such form - zero, an infinity, NaN - goes into the product as it is, at e = ref; a subnormal one has e = -126.
constexpr float kScaledRoom = 12.f, kScaledTop = 14.f;
// Beside such scales O is in units of this where a block's four warps add it up and in the parts: their sums may come to 8, and the
// numbers of V to the end of fp32's range.  The join divides its parts' weights first, and not its O in the end, for the same reason.
constexpr int kScaledUnitLog = 4;
constexpr float kScaledUnit = 16.f;
constexpr uint32_t kOneBits = 0x3f800000u, kInfBits = 0x7f800000u;
// LSE of a row from its base (log2 units) and sum.
__device__ __forceinline__ float lse_of(float base, float sum) { return sum == 0.f ? -INFINITY : (base + log2f(sum)) * 0.6931471805599453f; }

// BS: a scale for each block of rows (the members of DecodeParams from ks on), for FP8.  SEL: heads with a past read chosen blocks of
// it and what their own segment and tail show them (from choice_log on); WM = 1.
template <int D, bool FP8, int NT, int WM, bool BS = false, bool SEL = false>
__global__ void __launch_bounds__(kDecThreads, DecodeShape<D, FP8, NT, WM, BS, SEL>::kBlocksPerSm) decode_kernel(const __grid_constant__ DecodeParams p) {
    using Sh = DecodeShape<D, FP8, NT, WM, BS, SEL>;
    static_assert(!BS || (FP8 && Sh::KG == 2 && Sh::KP == 2), "the warp's two blocks of 16 slots have a scale each");
    static_assert(!SEL || WM == 1, "an item's rows all see the same slots");
    constexpr float kTop = BS ? kScaledTop : kHalfTop;
    constexpr int RB = Sh::RB, C = RB / 16, MB = Sh::MB, WR = Sh::kWR, ST = Sh::kStages, KS = D / 16, MT = D / 16, KG = Sh::KG, KP = Sh::KP;
    extern __shared__ uint8_t smem_raw[];
    __shared__ BlockRange range;
    __shared__ int warp_sum[4];
    __shared__ uint32_t there[ST][4];  // which of a warp's 16 KG slots were loaded, per stage
    __shared__ float2 end_ml[4][8];    // an item's end: base and sum of eight rows of each warp
    __shared__ float2 end_power[BS ? 4 : 1][8];  // and the power of two that their O is in units of, as a product
    __shared__ __align__(16) float block_scale[(BS ? ST : 1) * 16];  // of K and V, for each of a warp's blocks of 16 slots: [ST][4][2][2]
    const uint32_t ring = (smem_u32(smem_raw) + 127u) & ~127u;
    uint8_t* ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q4 = lane & 3, l4 = lane >> 2;
    const int wrow = WM == 1 ? 0 : warp % WM;  // this warp's eight NT rows of the item
    // with one head to a unit warps WM g .. WM g + WM - 1 share the slots of key group g; with several heads each warp has a
    // head and a key group of its own
    auto key_group = [&](int log) { return WM == 1 ? warp >> log : warp / WM; };
    auto head_of = [&](int first_head, int log) { return (int)p.head_order[first_head + (WM == 1 ? warp & ((1 << log) - 1) : 0)]; };

    next_kernel_may_start();
    if (BS || SEL) prefetch_numbers(p);
    find_range<MB, Sh::kTileLog, SEL>(p, &range, warp_sum);
    if (range.begin >= range.end) return;
    const int per = range.per;
    TileCursor<MB, Sh::kTileLog, SEL> put, get;  // what is loaded next, and what is computed next
    get.b = range.b;
    get.u = range.u;
    get.rb = range.rb;
    get.read_sequence(p);
    get.enter(p, range.tile);
    put = get;
    int put_left = range.end - range.begin, get_left = put_left;

    // ---- one tile's 16 KG slots of this warp into stage s ----
    constexpr int RPI = 32 / C;  // rows that one instruction of the warp covers
    const int r0 = lane / C, ch = lane % C;
    const uint32_t put_lane = swizzled<RB>(r0, ch);
    const char *k_item, *v_item;  // of the item being loaded: this lane's piece of row r0 of page 0
    const float* s_item = nullptr;  // its scales: of K for even lanes, of V for odd ones
    int far = 0, off = 0;         // its numbered slots
    uint64_t read_once = 0, read_again = 0;
    if (SEL) {
        asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(read_once));
        asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(read_again));
    }
    int chosen[SEL ? 4 : 1], n_chosen = 0;  // its blocks, 32 k + lane in chosen[k], and how many of them are in order
    auto enter_item = [&]() {
        const int h = head_of(put.first_head, put.log);
        if (BS) s_item = (lane & 1) == 0 ? p.ks + h * p.ks_stride[2] : p.vs + h * p.vs_stride[2];
        if (SEL) {
            int lo, hi;
            const int t = put.rb / p.head_blocks;
            numbered_slots(p, put.n, put.rows, put.shift, t, put.cls, &lo, &hi, &far, &off);
            n_chosen = 0;
            if (far > 0) {
                // Blocks count while they ascend within the past: none is read twice, nor one that the row sees whole.
                const int32_t* list = p.chosen + (((long long)put.b * p.c.Lq + t) * p.c.Hkv + h) * p.n_chosen;
                const int past = (off + far) >> p.choice_log;
#pragma unroll
                for (int k = 0; k < 4; ++k) chosen[k] = 32 * k + lane < p.n_chosen ? list[32 * k + lane] : -1;
                bool more = true;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (32 * k >= p.n_chosen) break;
                    const int last = k ? __shfl_sync(0xffffffffu, chosen[k ? k - 1 : 0], 31) : -1, up = __shfl_up_sync(0xffffffffu, chosen[k], 1);
                    const bool fine = (unsigned)chosen[k] < (unsigned)past && chosen[k] > (lane ? up : last);
                    const uint32_t wrong = __ballot_sync(0xffffffffu, !fine);
                    if (more) {
                        n_chosen += wrong ? __ffs(wrong) - 1 : 32;
                        more = wrong == 0;
                        if (wrong && lane == __ffs(wrong) - 1 && chosen[k] != -1) refuse_input(39);
                    }
                }
            }
        }
        k_item = p.c.K + r0 * p.c.k_stride[1] + h * p.c.k_stride[2] + ch * 16;
        v_item = p.c.V + r0 * p.c.v_stride[1] + h * p.c.v_stride[2] + ch * 16;
    };
    // the first slot of 16 that are numbered from v0 on; -1 for those of a block that is not there
    auto slot_from = [&](int v0) {
        if (!SEL || v0 >= far) return v0 + (SEL ? off : 0);
        const int i = v0 >> p.choice_log;
        const int from = i < 32 ? chosen[0] : i < 64 ? chosen[SEL ? 1 : 0] : i < 96 ? chosen[SEL ? 2 : 0] : chosen[SEL ? 3 : 0];
        const int block = __shfl_sync(0xffffffffu, from, i & 31);
        return i < n_chosen ? (block << p.choice_log) + (v0 & ((1 << p.choice_log) - 1)) : -1;
    };
    // The pages of the tile to be loaded next, looked up one tile ahead: the look-up is a load of its own, and the loads of the
    // rows wait for it.  An entry of the table outside the visible slots is not read.
    int page_next[KG], slot_next[KG];
    auto look_up = [&]() {
        const int slot0 = put.first_slot() + (WM == 1 ? key_group(put.log) : warp) * 16 * KG;
        if ((BS || SEL) && KG == 2 && p.page_pair) {
            // one look-up for both blocks of 16, if either is needed
            const int from = slot_from(slot0);
            const bool full0 = slot0 >= put.lo && slot0 + 16 <= put.hi, full1 = slot0 + 16 >= put.lo && slot0 + 32 <= put.hi;
            const int page = from >= 0 && (full0 || full1) ? table_entry(p.c, put.b, from) : -1;
            slot_next[0] = from;
            slot_next[KG - 1] = from >= 0 ? from + 16 : -1;
            page_next[0] = full0 ? page : -1;
            page_next[KG - 1] = full1 ? page : -1;
            return;
        }
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const int s0 = slot0 + 16 * k;
            page_next[k] = -1;
            slot_next[k] = slot_from(s0);
            if (p.page_whole && s0 >= put.lo && s0 + 16 <= put.hi && (!SEL || slot_next[k] >= 0)) page_next[k] = table_entry(p.c, put.b, slot_next[k]);
        }
    };
    enter_item();
    look_up();
    auto load_tile = [&](int s) {
        if (put_left > 0) {
            const int slot0 = put.first_slot() + (WM == 1 ? key_group(put.log) : warp) * 16 * KG;
            uint32_t loaded = 0;
            constexpr bool PAIR = (BS || SEL) && KG == 2;
            // chosen blocks are read once; what a sequence's rows see whole is read again by the next of them, and stays in L2
            const uint64_t policy = SEL ? (slot0 < far ? read_once : read_again) : 0;
            auto rows_from = [&](uint32_t dst, const char* src, long long stride) {
#pragma unroll
                for (int i = 0; i < 16 / RPI; ++i) {
                    const uint32_t to = (dst ^ swizzled<RB>(i * RPI, 0) % RB) + i * RPI * RB;
                    if (SEL) cp_async16_hint(to, src, policy);
                    else cp_async16(to, src);
                    src += RPI * stride;
                }
                return src;
            };
            const bool both = PAIR && p.page_pair && (unsigned)page_next[0] < (unsigned)p.c.n_pages && page_next[0] == page_next[KG - 1];
            if (both) {
                const int page = page_next[0], prow = row_in_page(p.c, slot_next[0]);
                const uint32_t dst = ring + (uint32_t)(s * 4 + warp) * Sh::kWarpStage + put_lane;
                const char* src = rows_from(dst, k_item + page * p.c.k_stride[0] + prow * p.c.k_stride[1], p.c.k_stride[1]);
                rows_from(dst + Sh::kBlock, src, p.c.k_stride[1]);
                src = rows_from(dst + 16 * RB, v_item + page * p.c.v_stride[0] + prow * p.c.v_stride[1], p.c.v_stride[1]);
                rows_from(dst + Sh::kBlock + 16 * RB, src, p.c.v_stride[1]);
                loaded = 0xffffffffu;
                if (BS && lane < 4) {
                    const long long* st = lane & 1 ? p.vs_stride : p.ks_stride;
                    cp_async4(smem_u32(block_scale) + (s * 16 + warp * 4 + lane) * 4,
                              s_item + page * st[0] + ((prow + 16 * (lane >> 1)) >> p.scale_log) * st[1]);
                }
            }
            constexpr int APART = PAIR ? 1 : KG;  // blocks of 16 side by side in the code: seldom ones take turns
#pragma unroll APART
            for (int k = both ? KG : 0; k < KG; ++k) {
                const int s0 = slot0 + 16 * k;
                const uint32_t dst = ring + (uint32_t)((s * 4 + warp) * KG + k) * Sh::kBlock + put_lane;
                const int slot_k = k == 0 ? slot_next[0] : slot_next[KG - 1];
                int prow, page = k == 0 ? page_next[0] : page_next[KG - 1];
                if ((unsigned)page < (unsigned)p.c.n_pages) {
                    // 16 visible slots in one page: one look-up, and rows a stride apart
                    prow = row_in_page(p.c, SEL ? slot_k : s0);
                    rows_from(dst, k_item + page * p.c.k_stride[0] + prow * p.c.k_stride[1], p.c.k_stride[1]);
                    rows_from(dst + 16 * RB, v_item + page * p.c.v_stride[0] + prow * p.c.v_stride[1], p.c.v_stride[1]);
                    loaded |= 0xffffu << (16 * k);
                } else {
                    const int slot = s0 + (lane & 15);
                    long long row_off = -1;  // of one row: lanes 0-15 in K, 16-31 in V
                    page = -1;
                    if (slot >= put.lo && slot < put.hi && (!SEL || slot_k >= 0) &&
                        (page = page_of(p.c, put.b, SEL ? slot_k + (lane & 15) : slot, &prow)) >= 0) {
                        const long long* st = lane < 16 ? p.c.k_stride : p.c.v_stride;
                        row_off = page * st[0] + prow * st[1] + head_of(put.first_head, put.log) * st[2];
                    }
                    const uint32_t found = __ballot_sync(0xffffffffu, row_off >= 0);
                    loaded |= (found & 0xffffu) << (16 * k);
                    if (BS) {  // 16 slots of one page
                        const int from = found ? __ffs(found) - 1 : 0;
                        page = __shfl_sync(0xffffffffu, page, from);
                        prow = __shfl_sync(0xffffffffu, prow, from);
                    }
#pragma unroll 1
                    for (int i = 0; i < 32 / RPI; ++i) {
                        const int row = i * RPI + r0;  // 0-15 of K, then of V
                        const long long o = __shfl_sync(0xffffffffu, row_off, row);
                        cp_async16_if(dst - put_lane + (row >> 4) * 16 * RB + swizzled<RB>(row & 15, ch),
                                      (row & 16 ? p.c.V : p.c.K) + (o >= 0 ? o + ch * 16 : 0), o >= 0);
                    }
                }
                if (BS && lane < 2) {
                    const int to = s * 16 + warp * 4 + 2 * k + lane;
                    const long long* st = lane == 0 ? p.ks_stride : p.vs_stride;
                    if ((unsigned)page < (unsigned)p.c.n_pages) cp_async4(smem_u32(block_scale) + to * 4, s_item + page * st[0] + (prow >> p.scale_log) * st[1]);
                    else block_scale[to] = 0.f;  // none of the 16 is there
                }
            }
            if (lane == 0) there[s][warp] = loaded;
            ++put.tile;
            if (--put_left > 0) {
                if (put.tile == put.end) {
                    put.next_item(p);
                    enter_item();
                }
                look_up();
            }
        }
        cp_async_commit();
    };

#pragma unroll
    for (int s = 0; s < ST - 1; ++s) load_tile(s);
    int stage = 0, free_stage = ST - 1;

    // Which slot of its 16 the row m of an S^T tile stands for.  The transposing 8-bit load of V hands a lane four
    // neighbouring slots, so with an e4m3 cache rows 2q, 2q + 1, 8 + 2q, 9 + 2q stand for slots 4q .. 4q + 3.
    auto slot_of = [](int m) { return FP8 ? 4 * ((m & 7) >> 1) + (m & 1) + 2 * (m >> 3) : m; };
    const int js[2] = {slot_of(l4), slot_of(l4 + 8)};  // slots of this lane's scores
    // byte offsets of this lane's operand pieces within a 16-slot block; piece 2c is reached by XOR with 32 c
    const uint32_t k_lane = FP8 ? 0u : swizzled<RB>(lane & 15, lane >> 4);
    const uint32_t k8_lane[2] = {swizzled<RB>(js[0], q4 * (D / 64)), swizzled<RB>(js[1], q4 * (D / 64))};
    const uint32_t v_lane = 16 * RB + (FP8 ? swizzled<RB>(lane & 15, lane >> 4) : swizzled<RB>((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1));

    float o[MT][NT][4];        // O^T: (dim l4, row 2 q4), (dim l4, row 2 q4 + 1), (dim l4 + 8, ...) of 16-dim tiles
    // A row's weights are exp2(score - base) so far: the base (0, or the scales' exponent, until the row has seen a key), the sum over this lane's slots,
    // and how far over the base a score has to be for the base to move (-inf until the row has seen a key).
    float base[NT][2], l[NT][2], slack[NT][2];
    uint32_t qf[KS][NT][2];
    float qscale[NT][2];       // score scale of the lane's rows, log2 units
    int rlo[NT][2], rhi[NT][2];  // their visible slots
    while (get_left > 0) {
        // ---- a piece: this block's tiles of one item ----
        const int first = get.tile, count = min(get.end - first, get_left);
        const int cls = get.cls, rows = get.rows * p.g, group = key_group(get.log), head = head_of(get.first_head, get.log);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            int t, hq;  // of the row whose elements this lane holds
            const bool real = row_of<MB, SEL>(p, get.rows, get.rb, wrow * WR + nt * 8 + l4, &t, &hq);
            const int qh = head * p.g + (real ? hq : 0);
            const __nv_bfloat16* q = p.Q + get.b * p.q_stride[0] + t * p.q_stride[1] + qh * p.q_stride[2];
            float scale = p.scale_log2;
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
                scale *= (BS ? 1.f : p.k_scale[head]) * __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    qf[k][nt][0] = real ? pack16<true>(x[4 * k] * down, x[4 * k + 1] * down) : 0u;
                    qf[k][nt][1] = real ? pack16<true>(x[4 * k + 2] * down, x[4 * k + 3] * down) : 0u;
                }
            } else {
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    qf[k][nt][0] = real ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 2 * q4) : 0u;
                    qf[k][nt][1] = real ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 8 + 2 * q4) : 0u;
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int rc = get.rb * MB + wrow * WR + nt * 8 + 2 * q4 + e;  // a row whose scores this lane holds
                qscale[nt][e] = FP8 ? __shfl_sync(0xffffffffu, scale, (2 * q4 + e) * 4) : scale;
                if (SEL) {
                    rlo[nt][e] = get.lo;
                    rhi[nt][e] = get.hi;
                } else {
                    visible_slots(p, get.n, get.rows, get.shift, (int)fdiv((uint32_t)min(rc, rows - 1), p.f_g), cls, &rlo[nt][e], &rhi[nt][e]);
                }
                base[nt][e] = l[nt][e] = 0.f;
                slack[nt][e] = -INFINITY;
            }
        }
#pragma unroll
        for (int k = 0; k < MT; ++k)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[k][nt][e] = 0.f;
        // slots that every row of the item sees: no mask there
        int all_lo = get.lo, all_hi = get.hi;
        if (!SEL) {
            const int r_last = min((get.rb + 1) * MB, rows) - 1;
            int x;
            visible_slots(p, get.n, get.rows, get.shift, (int)fdiv((uint32_t)r_last, p.f_g), cls, &all_lo, &x);
            visible_slots(p, get.n, get.rows, get.shift, (int)fdiv((uint32_t)(get.rb * MB), p.f_g), cls, &x, &all_hi);
        }
        float* scores = p.scores;
        if (scores) scores += (((long long)get.b * p.c.Hkv + head) * p.g * p.c.Lq + get.rb * MB + wrow * WR) * p.pitch;

        uint32_t ref_bits = kInfBits;  // the bits of 2^ref; infinity: no scale of the piece has been seen that has an exponent

        for (int left = count; left > 0; --left) {
            cp_async_wait<ST - 2>();
            if (WM == 1) __syncwarp();
            else asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / WM), "n"(32 * WM) : "memory");
            load_tile(free_stage);
            // this warp's key group: 16 KG WM slots, loaded by the group's WM warps
#pragma unroll 1
            for (int w = 0; w < WM * KG; w += KP) {
                const int slot0 = get.first_slot() + group * WM * KG * 16 + w * 16;
                const int from = WM == 1 ? warp : group * WM + w / KG;  // the warp that loaded them, or the first of two
                const uint32_t blk = ring + (uint32_t)(stage * 4 + from) * Sh::kWarpStage;
                uint32_t have = there[stage][from];
                if (KP > KG) have |= there[stage][from + 1] << 16;
                // Products with an accumulator wait for one another, some 30 cycles each: four chains are kept going, over blocks of
                // slots, rows, and where those are too few over even and odd pieces of the head.
                constexpr int CH = KP * NT >= 4 ? 1 : 2;
                float s[KP][NT][4], s2[CH][KP][NT][4];
#pragma unroll
                for (int x = 0; x < CH; ++x)
#pragma unroll
                    for (int k = 0; k < KP; ++k)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s2[x][k][nt][e] = 0.f;
                // the scales of K and V in each of the two blocks of slots; asked for in front of the products, which they are needed behind
                float4 sc = make_float4(1.f, 1.f, 1.f, 1.f);
                if (BS) sc = *reinterpret_cast<const float4*>(block_scale + stage * 16 + from * 4);
                if (FP8) {
#pragma unroll
                    for (int v = 0; v < D / 64; ++v) {
                        uint4 w0[KP], w1[KP];
#pragma unroll
                        for (int k = 0; k < KP; ++k) {
                            w0[k] = lds128(blk + k * Sh::kBlock + (k8_lane[0] ^ (v << 4)));
                            w1[k] = lds128(blk + k * Sh::kBlock + (k8_lane[1] ^ (v << 4)));
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int k = 0; k < KP; ++k) {
                                uint32_t a[4];
                                e4m3x4_to_half(j == 0 ? w0[k].x : j == 1 ? w0[k].y : j == 2 ? w0[k].z : w0[k].w, a[0], a[2]);
                                e4m3x4_to_half(j == 0 ? w1[k].x : j == 1 ? w1[k].y : j == 2 ? w1[k].z : w1[k].w, a[1], a[3]);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
                                    mma16816<true>(s2[j % CH][k][nt], a, qf[v * 4 + j][nt][0], qf[v * 4 + j][nt][1]);
                            }
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < KS; ++c)
#pragma unroll
                        for (int k = 0; k < KP; ++k) {
                            uint32_t a[4];
                            ldsm_x4(blk + k * Sh::kBlock + (k_lane ^ (c << 5)), a);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma16816<false>(s2[c % CH][k][nt], a, qf[c][nt][0], qf[c][nt][1]);
                        }
                }
#pragma unroll
                for (int k = 0; k < KP; ++k)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[k][nt][e] = CH == 1 ? s2[0][k][nt][e] : s2[0][k][nt][e] + s2[CH - 1][k][nt][e];
                // score scales of the rows in each block of slots; m, e and 2^(ref - e) of V's scales
                float qs[KP][NT][2], vsc[KP], vexp[KP], vinv[KP];
                // Scales that are read in the plain way: positive, with exponents from ref to ref + 126.
                const uint32_t span = min(126u << 23, kInfBits - ref_bits);
                bool plain = true;
#pragma unroll
                for (int k = 0; k < KP; ++k) {
                    const float ks = k == 0 ? sc.x : sc.z, vs = k == 0 ? sc.y : sc.w;
                    if (BS) {
                        const uint32_t bits = __float_as_uint(vs);
                        plain = plain && bits - ref_bits < span;
                        vsc[k] = __uint_as_float((bits & 0x7fffffu) | kOneBits);
                        vexp[k] = __uint_as_float(0x4b000000u | (bits >> 23)) - 8388735.f;  // 2^23 + 127
                        vinv[k] = __uint_as_float(ref_bits + kOneBits - (bits & kInfBits));
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) qs[k][nt][e] = BS ? qscale[nt][e] * ks : qscale[nt][e];
                }
                if (BS && !plain) {
                    const bool first = ref_bits == kInfBits;
                    int ref = first ? 127 : (int)(ref_bits >> 23), low = 255, ve[KP];  // exponents as they stand in a number's bits
#pragma unroll
                    for (int k = 0; k < KP; ++k) {
                        const float vs = k == 0 ? sc.y : sc.w;
                        const uint32_t size = __float_as_uint(vs) & 0x7fffffffu;
                        ve[k] = size == 0 ? 255 : max((int)(size >> 23), 1);
                        vsc[k] = size == 0 || size >= kInfBits ? vs
                                 : size < 1u << 23 ? vs * 0x1p126f : __uint_as_float((__float_as_uint(vs) & 0x807fffffu) | kOneBits);
                        low = min(low, ve[k]);
                    }
                    if (low < (first ? 255 : ref)) {
                        // Bases begin where the scales are: a score is not rounded by how far that is from zero.  Scales without an exponent in
                        // front of the first may have moved them: from there, with nothing in O that depends on it.  Later ref only falls.
                        const float f = __uint_as_float((uint32_t)max(127 + low - ref, 0) << 23);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                if (first) base[nt][e] += (float)(low - ref);
                                else l[nt][e] *= f;
                            }
                        ref = low;
                        ref_bits = (uint32_t)ref << 23;
                    }
#pragma unroll
                    for (int k = 0; k < KP; ++k) {
                        if (ve[k] == 255) ve[k] = ref;
                        vexp[k] = (float)(ve[k] - 127);
                        vinv[k] = __uint_as_float((uint32_t)max(127 + ref - ve[k], 0) << 23);
                    }
                }
                // element e of s[k][nt]: slot 16 k + js[e >> 1], row 2 q4 + (e & 1) of the warp's eight; log2 units over the base
                const bool edge_range = slot0 < all_lo || slot0 + 16 * KP > all_hi;
                if (scores) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int r = nt * 8 + 2 * q4 + (e & 1);
                            if (get.rb * MB + wrow * WR + r < rows)
#pragma unroll
                                for (int k = 0; k < KP; ++k)
                                    scores[(long long)r * p.pitch + slot0 + 16 * k + js[e >> 1]] =
                                        (have >> (16 * k + js[e >> 1])) & 1 ? s[k][nt][e] * qs[k][nt][e & 1] : -INFINITY;
                        }
                }
                bool grows = false;
#pragma unroll
                for (int k = 0; k < KP; ++k)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[k][nt][e] = fmaf(s[k][nt][e], qs[k][nt][e & 1], BS ? vexp[k] - base[nt][e & 1] : -base[nt][e & 1]);
                if (edge_range || have != (KP == 1 ? 0xffffu : 0xffffffffu)) {
#pragma unroll
                    for (int k = 0; k < KP; ++k)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int j = 16 * k + js[e >> 1];
                                if (slot0 + j < rlo[nt][e & 1] || slot0 + j >= rhi[nt][e & 1] || !((have >> j) & 1)) s[k][nt][e] = -INFINITY;
                            }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(s[0][nt][e], s[0][nt][e + 2]);
                        if (KP > 1) mx = fmaxf(mx, fmaxf(s[KP - 1][nt][e], s[KP - 1][nt][e + 2]));
                        grows |= mx > slack[nt][e];
                    }
                if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float f[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float mx = fmaxf(s[0][nt][e], s[0][nt][e + 2]);
                            if (KP > 1) mx = fmaxf(mx, fmaxf(s[KP - 1][nt][e], s[KP - 1][nt][e + 2]));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                            // row by row: what one row sees must not move another row's base (and with it its rounding)
                            f[e] = 1.f;
                            if (mx > slack[nt][e]) {
                                const float moved = BS ? floorf(base[nt][e] + (mx - kScaledRoom)) : base[nt][e] + (FP8 ? mx - kHalfRoom : mx);
                                mx = moved - base[nt][e];  // by what the rounded base has moved: scores and sums follow it
                                f[e] = slack[nt][e] == -INFINITY ? 0.f : ex2(-mx);
                                base[nt][e] = moved;
                                slack[nt][e] = FP8 ? kTop : kDecSlack;
                                // a base past 2^26 is rounded by whole powers of two: what that leaves over fp16's top is cut
                                auto over_new_base = [&](float x) { return FP8 && x - mx > kTop ? kTop : x - mx; };
#pragma unroll
                                for (int k = 0; k < KP; ++k) {
                                    s[k][nt][e] = over_new_base(s[k][nt][e]);
                                    s[k][nt][e + 2] = over_new_base(s[k][nt][e + 2]);
                                }
                            }
                            l[nt][e] *= f[e];
                        }
#pragma unroll
                        for (int k2 = 0; k2 < MT; ++k2)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[k2][nt][e] *= f[e & 1];
                    }
                }
                uint32_t pf[KP][NT][2];
#pragma unroll
                for (int k = 0; k < KP; ++k)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[k][nt][e] = ex2(s[k][nt][e]);
                            l[nt][e & 1] = BS ? fmaf(s[k][nt][e], vinv[k], l[nt][e & 1]) : l[nt][e & 1] + s[k][nt][e];
                        }
                if (BS && (vsc[0] != 1.f || vsc[KP - 1] != 1.f)) {  // scales that are no (positive) powers of two
#pragma unroll
                    for (int k = 0; k < KP; ++k)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[k][nt][e] = s[k][nt][e] == 0.f ? 0.f : s[k][nt][e] * vsc[k];  // hidden: not 0 times NaN
                }
#pragma unroll
                for (int k = 0; k < KP; ++k)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        pf[k][nt][0] = movm_t(pack16<FP8>(s[k][nt][0], s[k][nt][1]));
                        pf[k][nt][1] = movm_t(pack16<FP8>(s[k][nt][2], s[k][nt][3]));
                    }
                // A weight of zero does not undo an infinite or NaN V: slots that some rows of the item see and others do not
                // (rows behind a row, slots across a segment's border) are looked at, and where V is not finite its product is
                // taken out of the mma and added to the rows that see it one by one.
                uint32_t bad = 0;
                if (edge_range) {
                    uint32_t part = 0;
#pragma unroll 1
                    for (int j = 0; j < 16 * KP; ++j)
                        if (slot0 + j < all_lo || slot0 + j >= all_hi) part |= 1u << j;
                    part &= have;
#pragma unroll 1
                    for (; part; part &= part - 1) {
                        const int j = __ffs(part) - 1;
                        bool odd = false;
                        if (lane < C) {
                            const uint4 w4 = lds128(blk + (j >> 4) * Sh::kBlock + 16 * RB + swizzled<RB>(j & 15, lane));
                            const uint32_t ww[4] = {w4.x, w4.y, w4.z, w4.w};
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
                auto add_values = [&](auto masked) {
#pragma unroll
                    for (int k = 0; k < KP; ++k) {
                        // the lane's V fragments hold slots slot_of(2 q4), slot_of(2 q4 + 1) and slot_of(8 + 2 q4), slot_of(9 + 2 q4)
                        uint32_t keep0 = 0, keep1 = 0;
                        if (masked.value) {
                            const uint32_t b16 = bad >> (16 * k);
                            keep0 = ((b16 >> slot_of(2 * q4)) & 1 ? 0u : 0xffffu) | ((b16 >> slot_of(2 * q4 + 1)) & 1 ? 0u : 0xffff0000u);
                            keep1 = ((b16 >> slot_of(8 + 2 * q4)) & 1 ? 0u : 0xffffu) | ((b16 >> slot_of(9 + 2 * q4)) & 1 ? 0u : 0xffff0000u);
                        }
                        auto product = [&](float (&acc)[NT][4], uint32_t (&a)[4]) {
                            if (masked.value) {
                                a[0] &= keep0;
                                a[1] &= keep0;
                                a[2] &= keep1;
                                a[3] &= keep1;
                            }
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma16816<FP8>(acc[nt], a, pf[k][nt][0], pf[k][nt][1]);
                        };
#pragma unroll
                        for (int c = 0; c < (FP8 ? MT / 2 : MT); ++c) {
                            uint32_t b[4];
                            if (FP8) {
                                ldsm8_x2_t(blk + k * Sh::kBlock + (v_lane ^ (c << 5)), b);
#pragma unroll
                                for (int x = 0; x < 2; ++x) {
                                    uint32_t a[4];
                                    e4m3x4_to_half(b[2 * x], a[0], a[2]);
                                    e4m3x4_to_half(b[2 * x + 1], a[1], a[3]);
                                    product(o[2 * c + x], a);
                                }
                            } else {
                                ldsm_x4_t(blk + k * Sh::kBlock + (v_lane ^ (c << 5)), b);
                                product(o[c], b);
                            }
                        }
                    }
                };
                if (bad == 0) {
                    add_values(Flag<false>());
                } else {
                    add_values(Flag<true>());
#pragma unroll 1
                    for (; bad; bad &= bad - 1) {
                        const int j = __ffs(bad) - 1, slot = slot0 + j, j16 = j & 15;
                        const int mrow = FP8 ? (j16 >> 2) * 2 + (j16 & 1) + ((j16 >> 1) & 1) * 8 : j16;  // slot_of(mrow) = j16
                        const uint32_t vrow = blk + (j >> 4) * Sh::kBlock + 16 * RB;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float lo_w = j & 16 ? s[KP - 1][nt][e] : s[0][nt][e], hi_w = j & 16 ? s[KP - 1][nt][2 + e] : s[0][nt][2 + e];
                                const float wt = __shfl_sync(0xffffffffu, mrow & 8 ? hi_w : lo_w, (mrow & 7) * 4 + q4);
                                if (slot < rlo[nt][e] || slot >= rhi[nt][e]) continue;
#pragma unroll
                                for (int k2 = 0; k2 < MT; ++k2)
#pragma unroll
                                    for (int hh = 0; hh < 2; ++hh) {
                                        const int byte = (k2 * 16 + l4 + 8 * hh) * (FP8 ? 1 : 2);
                                        const uint32_t at = vrow + swizzled<RB>(j16, byte >> 4) + (byte & 15);
                                        float x;
                                        if (FP8) {
                                            uint32_t raw, h0, h1;
                                            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(raw) : "r"(at));
                                            e4m3x4_to_half(raw, h0, h1);
                                            x = __half2float(__ushort_as_half((unsigned short)(h0 & 0xffffu)));
                                        } else {
                                            uint16_t raw;
                                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(raw) : "r"(at));
                                            x = __uint_as_float((uint32_t)raw << 16);
                                        }
                                        o[k2][nt][2 * hh + e] += wt * x;
                                    }
                            }
                    }
                }
            }
            free_stage = stage;
            stage = stage + 1 == ST ? 0 : stage + 1;
            ++get.tile;
        }
        get_left -= count;

        // ---- the item's end: sums over the lanes of a row, then over the key groups, eight rows of each warp at a time
        // through the stage that was computed last (the next load into it comes after the barriers here) ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 4);
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 8);
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 16);
            }
        // the item's tiles are numbered from list0 on in the list of all tiles
        const int list0 = range.end - get_left - count - first;
        const int b_first = list0 / per, b_last = (list0 + get.end - 1) / per;
        if (first == 0 && threadIdx.x < 1 << get.log)
            p.item_blocks[((long long)get.b * p.c.Hkv + p.head_order[get.first_head + threadIdx.x]) * p.row_blocks + get.rb] =
                make_int2(b_first, b_last);
        const int side = WM == 1 ? 1 << get.log : WM;  // warps w, w + side, ... hold parts of the same rows
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0 && (SEL ? get.rb % p.head_blocks * MB + nt * 8 >= p.g : get.rb * MB + nt * 8 >= rows)) break;  // none of the warps' rows from here on is there (WM = 1)
            float* mine = reinterpret_cast<float*>(ring_ptr + (size_t)(free_stage * 4 + warp) * Sh::kWarpStage);
            __syncthreads();
            // row r8 at r8 D, its dims XORed with the row so that the lanes' writes fall into different banks
#pragma unroll
            for (int k2 = 0; k2 < MT; ++k2)
#pragma unroll
                for (int e = 0; e < 4; ++e) mine[(2 * q4 + (e & 1)) * D + ((k2 * 16 + l4 + 8 * (e >> 1)) ^ (q4 << 3))] = o[k2][nt][e];
            if (l4 == 0) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float m = slack[nt][e] == -INFINITY ? -INFINITY : base[nt][e], sum = l[nt][e];
                    if (BS) {
                        // The true sum is sum 2^(base - ref) and O in units of 2^(base - ref) 2^ref.  The sum is brought to [1, 2): whole
                        // numbers are added up first, and the LSE is not rounded by how far the scales are from one.
                        const uint32_t bits = __float_as_uint(sum);
                        int power = ref_bits == kInfBits ? 0 : (int)(ref_bits >> 23) - 127;
                        m -= (float)power;
                        if (bits - 0x00800000u < 0x7f000000u) {  // a normal number
                            const int up = (int)(bits >> 23) - 127;
                            m += (float)up;
                            sum = __uint_as_float((bits & 0x7fffffu) | 0x3f800000u);
                            power -= up;
                        }
                        // in two factors, as their product may be out of range
                        power -= kScaledUnitLog;
                        const int half = power >> 1;
                        end_power[warp][2 * q4 + e] =
                            make_float2(__uint_as_float((uint32_t)max(127 + half, 0) << 23), __uint_as_float((uint32_t)max(127 + power - half, 0) << 23));
                    }
                    end_ml[warp][2 * q4 + e] = make_float2(m, sum);
                }
            }
            __syncthreads();
            constexpr int TPR = D / 4;  // threads to a row
            const int d0 = (threadIdx.x % TPR) * 4;
            // rows of the eight that are there, the same for all heads of the unit (with several warps to a tile they differ)
            const int there8 = WM > 1 ? 8 : min(8, SEL ? p.g - get.rb % p.head_blocks * MB - nt * 8 : rows - get.rb * MB - nt * 8);
            for (int i = threadIdx.x / TPR; i < side * there8; i += kDecThreads / TPR) {
                const int w0 = i / there8, r8 = i - w0 * there8;
                int t, hq;
                if (!row_of<MB, SEL>(p, get.rows, get.rb, (WM == 1 ? 0 : w0 * WR) + nt * 8 + r8, &t, &hq)) continue;
                const int h = p.head_order[get.first_head + (WM == 1 ? w0 : 0)];
                const float vs = BS ? kScaledUnit : FP8 ? p.v_scale[h] : 1.f;
                float mm = -INFINITY, ll = 0.f;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int w = w0; w < 4; w += side) mm = fmaxf(mm, end_ml[w][r8].x);
                const float top = mm == -INFINITY ? 0.f : mm;
                for (int w = w0; w < 4; w += side) {
                    const float2 ml = end_ml[w][r8];
                    float f = ex2(ml.x - top);
                    float4 y = *reinterpret_cast<const float4*>(
                        ring_ptr + (size_t)(free_stage * 4 + w) * Sh::kWarpStage + (r8 * D + (d0 ^ ((r8 >> 1) << 3))) * 4);
                    ll += ml.y * f;
                    if (BS) {
                        const float2 power = end_power[w][r8];
                        f *= power.x;
                        y.x *= power.y;
                        y.y *= power.y;
                        y.z *= power.y;
                        y.w *= power.y;
                    }
                    x.x += y.x * f;
                    x.y += y.y * f;
                    x.z += y.z * f;
                    x.w += y.w * f;
                }
                if (b_first == b_last) {
                    const int qh = h * p.g + hq;
                    const float inv = ll == 0.f ? 0.f : vs / ll;
                    *reinterpret_cast<uint2*>(p.O + get.b * p.o_stride[0] + t * p.o_stride[1] + qh * p.o_stride[2] + d0) =
                        make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
                    if (d0 == 0)
                        p.LSE[((long long)get.b * p.Hq + qh) * p.c.Lq + t] = lse_of(mm, ll);
                } else {
                    // a part: slot 0 where the block's range begins inside the item, else slot 1
                    const long long at = ((long long)blockIdx.x * 2 + (first == 0 ? 1 : 0)) * Sh::kPartRows + w0 * WR + nt * 8 + r8;
                    *reinterpret_cast<float4*>(p.part_o + at * D + d0) = BS ? x : make_float4(x.x * vs, x.y * vs, x.z * vs, x.w * vs);
                    if (d0 == 0) p.part_ml[at] = make_float2(mm, ll);
                }
            }
        }
        __syncthreads();
        if (get_left > 0) get.next_item(p);
    }
    cp_async_wait<0>();
}

// Whether an item's first and last block, as found in the workspace, name parts to be added up: not where one block holds all
// of the item, and not where nobody wrote them (the block that should have may have left after an expired wait; the workspace
// is scratch memory and can hold anything there).
__host__ __device__ inline bool parts_to_join(int first, int last, int blocks) { return first >= 0 && first < last && last < blocks; }

// Adds the parts of one row of an item that several blocks share; block.x = the item, block.y = the row, a thread one dim.
// A row has at most as many parts as the grid has blocks: their bases and sums are read by all threads at once, and the first
// values of O beside them, so that two dependent reads are all the latency there is.
template <int D, bool SEL = false>
__global__ void __launch_bounds__(D) decode_join_kernel(const __grid_constant__ DecodeParams p, int MB, int part_rows) {
    constexpr int AHEAD = 8;
    const int rb = blockIdx.x % p.row_blocks, u = blockIdx.x / p.row_blocks, h = u % p.c.Hkv, b = u / p.c.Hkv;
    const int rl = blockIdx.y, r = rb * MB + rl, tid = threadIdx.x;
    after_previous_kernel();
    if (SEL ? rb / p.head_blocks >= new_rows(p.c, b) || rb % p.head_blocks * MB + rl >= p.g : r >= new_rows(p.c, b) * p.g) return;
    const int2 blocks = p.item_blocks[blockIdx.x];
    if (!parts_to_join(blocks.x, blocks.y, p.blocks)) return;
    __shared__ float weight[kDecMaxBlocks];
    __shared__ float red[2][D / 32];
    const int n = blocks.y - blocks.x + 1;
    // the item's first block holds its part in slot 1 (its range began at or before the item), the others in slot 0
    auto at = [&](int k) { return ((long long)(blocks.x + k) * 2 + (k == 0 ? 1 : 0)) * part_rows + p.head_in_unit[h] * MB + rl; };
    float ahead[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) ahead[k] = k < n ? p.part_o[at(k) * D + tid] : 0.f;
    float m = -INFINITY;
    for (int k = tid; k < n; k += D) m = fmaxf(m, p.part_ml[at(k)].x);
#pragma unroll
    for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    if ((tid & 31) == 0) red[0][tid >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < D / 32; ++k) m = fmaxf(m, red[0][k]);
    const float base = m == -INFINITY ? 0.f : m;
    const bool scaled = p.ks != nullptr;
    float l = 0.f;
    for (int k = tid; k < n; k += D) {
        const float2 ml = p.part_ml[at(k)];
        weight[k] = ex2(ml.x - base);
        l += ml.y * weight[k];
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
    if ((tid & 31) == 0) red[1][tid >> 5] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) l += red[1][k];
    float o = 0.f;
    const float share = scaled ? kScaledUnit / l : 1.f;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (k < n) o += ahead[k] * (weight[k] * share);
#pragma unroll 8
    for (int k = AHEAD; k < n; ++k) o += p.part_o[at(k) * D + tid] * (weight[k] * share);
    const int t = SEL ? rb / p.head_blocks : (int)fdiv((uint32_t)r, p.f_g), qh = h * p.g + (SEL ? rb % p.head_blocks * MB + rl : r - t * p.g);
    p.O[b * p.o_stride[0] + t * p.o_stride[1] + qh * p.o_stride[2] + tid] = __float2bfloat16(l == 0.f ? 0.f : scaled ? o : o / l);
    if (tid == 0) p.LSE[((long long)b * p.Hq + qh) * p.c.Lq + t] = lse_of(m, l);
}

// Attention weight of every slot, from the scores and the finished LSE: a block takes 256 slots of one (sequence, KV head), a
// thread one slot, over the rows in chunks whose LSE and visible slots lie in shared memory.  A stream over the scores: eight
// loads are in flight per thread (a slot a row does not see is loaded and dropped: the workspace has room for every slot).
constexpr int kWeightRows = 128;
__global__ void __launch_bounds__(256) decode_weights_kernel(const __grid_constant__ DecodeParams p) {
    const int j = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
    after_previous_kernel();
    const int rows = new_rows(p.c, b), n = seq_len(p.c, b);
    if (blockIdx.x * 256 >= n || rows == 0) return;
    __shared__ float lse2[kWeightRows];
    __shared__ int lo[kWeightRows], hi[kWeightRows];
    const int shift = shift_of(p.c, b), cls = p.head_class[h];
    const long long unit = (long long)b * p.c.Hkv + h;
    float sum = 0.f;
    for (int r0 = 0; r0 < rows * p.g; r0 += kWeightRows) {
        const int m = min(kWeightRows, rows * p.g - r0);
        if (threadIdx.x < m) {
            const int r = r0 + threadIdx.x, t = (int)fdiv((uint32_t)r, p.f_g);
            const float x = p.LSE[((long long)b * p.Hq + h * p.g + r - t * p.g) * p.c.Lq + t];
            visible_slots(p, n, rows, shift, t, cls, &lo[threadIdx.x], &hi[threadIdx.x]);
            lse2[threadIdx.x] = x * 1.4426950408889634f;
            if (x == -INFINITY) hi[threadIdx.x] = lo[threadIdx.x];
        }
        __syncthreads();
        if (j < n && j >= lo[0]) {  // the rows' lower ends only grow
            const float* s = p.scores + (unit * p.g * p.c.Lq + r0) * p.pitch + j;
            for (int r = 0; r < m; r += 8) {
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = r + k < m ? s[(long long)(r + k) * p.pitch] : 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (r + k < m && j >= lo[r + k] && j < hi[r + k]) sum += ex2(x[k] - lse2[r + k]);
            }
        }
        __syncthreads();
    }
    if (j >= n) return;
    const long long at = unit * p.W + j;
    p.w_out[at] = (p.w_in ? p.w_in[at] : 0.f) + sum;
}

}  // namespace segattn
