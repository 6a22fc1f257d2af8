// The paged cache's attention for many new rows to a KV head (a prompt's last tokens, a long speculation): 128 rows fill
// tcgen05.mma's M, so the products go to the tensor memory's accumulators.  bf16 caches; more than kDecRowsMin rows.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>

#include "decode_kernels.cuh"

namespace segattn {

// Rows to a KV head from which these kernels take over: at 32 rows both take 46 us (4 x 14000 slots, half of the heads with
// their whole past), at 24 and fewer decode_kernel is ahead, by far where weights are asked for; at 64 it takes 66 us to 49.
constexpr int kDecRowsMin = 33;

// 16-byte piece c of row r in an operand tile of 64-element panels with 128-byte swizzled rows.
__device__ __forceinline__ uint32_t panel_at(int r, int c, int panel_bytes) {
    return (uint32_t)((c >> 3) * panel_bytes + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

// 16 slots from slot0 on of one (sequence, KV head) into rows row0 .. row0 + 15 of an operand tile (K, or V), by one warp;
// slots outside [lo, hi) and of pages that are none become zeros.  Returns which were loaded, one bit each.
template <int D>
__device__ __forceinline__ uint32_t load_16_slots(const PagedView& c, int b, int h, int slot0, int lo, int hi, uint32_t k_tile, uint32_t v_tile,
                                                  bool with_v, int row0, int panel_bytes, bool page_whole) {
    constexpr int C = D / 8, RPI = 32 / C;  // 16-byte pieces of a row; rows one instruction of the warp covers
    const int lane = threadIdx.x & 31, slot = slot0 + (lane & 15), r0 = lane / C, ch = lane % C;
    int prow, page;
    if (page_whole && slot0 >= lo && slot0 + 16 <= hi && (page = page_of(c, b, slot0, &prow)) >= 0) {
        // 16 visible slots in one page: one look-up, and rows a stride apart
        const char* k = c.K + page * c.k_stride[0] + (prow + r0) * c.k_stride[1] + h * c.k_stride[2] + ch * 16;
        const char* v = c.V + page * c.v_stride[0] + (prow + r0) * c.v_stride[1] + h * c.v_stride[2] + ch * 16;
#pragma unroll
        for (int i = 0; i < 16 / RPI; ++i) {
            const uint32_t at = panel_at(row0 + i * RPI + r0, ch, panel_bytes);
            cp_async16(k_tile + at, k);
            if (with_v) cp_async16(v_tile + at, v);
            k += RPI * c.k_stride[1];
            v += RPI * c.v_stride[1];
        }
        return 0xffffu;
    }
    long long off = -1;  // of one row: lanes 0-15 in K, 16-31 in V
    if (slot >= lo && slot < hi && (page = page_of(c, b, slot, &prow)) >= 0) {
        const long long* st = lane < 16 ? c.k_stride : c.v_stride;
        off = page * st[0] + prow * st[1] + h * st[2];
    }
    const uint32_t loaded = __ballot_sync(0xffffffffu, off >= 0) & 0xffffu;
#pragma unroll
    for (int i = 0; i < 16 / RPI; ++i) {
        const int r = i * RPI + r0;
        const uint32_t at = panel_at(row0 + r, ch, panel_bytes);
        const long long ok = __shfl_sync(0xffffffffu, off, r);
        cp_async16_if(k_tile + at, c.K + (ok >= 0 ? ok + ch * 16 : 0), ok >= 0);
        if (with_v) {
            const long long ov = __shfl_sync(0xffffffffu, off, 16 + r);
            cp_async16_if(v_tile + at, c.V + (ov >= 0 ? ov + ch * 16 : 0), ov >= 0);
        }
    }
    return loaded;
}

// Row r of a sequence's KV head (r = new row * g + query head of the group) into row r - r_base of an operand tile, `count` rows
// from `first` on by one warp; rows that are not there become zeros.
template <int D>
__device__ __forceinline__ void load_query_rows(const DecodeParams& p, int b, int h, int rows, int r_base, int first, int count, uint32_t tile, int panel_bytes) {
    constexpr int C = D / 8, RPI = 32 / C;
    const int lane = threadIdx.x & 31, r0 = lane / C, ch = lane % C;
    for (int i = first; i < first + count; i += RPI) {
        const int r = r_base + i + r0;
        const bool real = r < rows;
        const int t = (int)fdiv((uint32_t)(real ? r : 0), p.f_g), qh = h * p.g + (real ? r - t * p.g : 0);
        const __nv_bfloat16* q = p.Q + b * p.q_stride[0] + t * p.q_stride[1] + qh * p.q_stride[2] + ch * 8;
        cp_async16_if(tile + panel_at(i + r0, ch, panel_bytes), q, real);
    }
}

// One arrival on `bar` when all copies that this thread has issued so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- attention -----------------------------------------------------------------------------------------------------
// One block to an SM walks its range of 64-slot tiles of the same list that decode_kernel uses (items of up to QR rows).
//   loaders      16 or 32 slots of K and V a warp with cp.async into a ring of stages, queries into one of two buffers
//   issuer       S(i) = Q K^T (128 x 64), then O += P(i-1) V (128 x D)
//   softmax      one group of warps for the even tiles, one for the odd ones: thread = row = TMEM lane; scores out of the
//                group's S buffer, weights (bf16) into its P buffer, an O and a base of its own; joined at an item's end
// TMEM (512 columns): S at 0 and 64, P at 128 and 160, O at 192 and 320.  A row's base moves as in decode_kernel, past a
// slack only: most tiles leave O alone.  The rows of an MMA do not mix, so that with items of QR = 64 rows the upper half of
// the lanes computes on whatever is there and nobody reads it; its two warps of each softmax group are not needed (two of
// them load), and the queries' smaller buffers leave room for six stages instead of four.  4 x 14000 slots, half of the heads with
// their whole past, 64 rows: 49 us, 2900 cycles for each of a block's 31 tiles, of which the twelve products take some 770.  No
// part of the SM is full (DRAM 33%, tensor pipe 22%, issue slots 23%): a tile goes from scores through softmax and weights to its
// product in one dependent chain, and two tiles, one to a group, are on their way at a time.  With the scores issued after the
// products it took 52 us, with four stages 57, with one softmax group 97, with tiles of 128 slots, whose P has to share S's columns,
// 60.  Every wait is bounded.
template <int D, int QR>
struct RowsShape {
    static constexpr int kStages = D == 64 ? 8 : QR == 64 ? 6 : 4;
    static constexpr int kKv = (D / 64) * 8192;       // a K or V tile: 64 rows, panels of 64 elements
    static constexpr int kQPanel = QR * 128;
    static constexpr int kQ = (D / 64) * kQPanel;
    static constexpr int kDynamic = kStages * 2 * kKv + 2 * kQ + 1024;
    static constexpr int MB = QR, kTileLog = 6;
    static_assert(QR == 128 || 128 * 128 + (D / 64 - 1) * kQPanel <= kQ + kStages * 2 * kKv, "an MMA's 128 rows of the second query buffer end in the ring");
    static constexpr int kThreads = QR == 64 ? 320 : 384;
    static constexpr int kLoaders = QR == 64 ? 4 : 2; // warps 0, 1 (, 6, 7); the issuer is warp 2, the groups start at warps 4 and 8
};
constexpr int kRowsBlocks = 160;  // blocks a launch has at most

template <int D, int QR>
__global__ void __launch_bounds__(RowsShape<D, QR>::kThreads, 1) decode_rows_kernel(const __grid_constant__ DecodeParams p) {
    using Sh = RowsShape<D, QR>;
    constexpr int ST = Sh::kStages, MB = Sh::MB, C = D / 8, NL = Sh::kLoaders, SW = 4 / NL * 16;  // slots of a loader warp
    enum { kFull = 0, kEmpty = ST, kSFull = 2 * ST, kPFull = 2 * ST + 2, kPvDone = 2 * ST + 4, kQFull = 2 * ST + 6, kQEmpty = 2 * ST + 8, kScan = 2 * ST + 10, kSRead = 2 * ST + 12, kBars = 2 * ST + 14 };
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ BlockRange range;
    __shared__ int warp_sum[4];
    __shared__ uint32_t there[ST][4], tmem_slot;
    __shared__ float2 end_ml[2][QR];  // an item's end: base and sum of each row in the two groups
    const uint32_t base_s = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // The queries come first: an MMA reads 128 rows of them, with QR = 64 up to 16 KB past the second buffer's end, which has
    // to stay within the block's shared memory (the ring's 96 KB and more).
    auto sQ = [&](int s) { return base_s + s * Sh::kQ; };
    auto sK = [&](int s) { return base_s + 2 * Sh::kQ + s * 2 * Sh::kKv; };
    auto sV = [&](int s) { return sK(s) + Sh::kKv; };
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    next_kernel_may_start();
    find_range<MB, Sh::kTileLog>(p, &range, warp_sum);
    if (range.begin >= range.end) return;
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i)
            mbar_init(bar(i), i < kEmpty ? NL * 33 : i >= kQFull && i < kQEmpty ? NL * 32 : (i >= kPFull && i < kPvDone) || i >= kScan ? QR / 32 : 1);
        fence_mbar_init();
    }
    if (warp == 2) {
        tmem_alloc(smem_u32(&tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tS = tmem, tP = tmem + 128, tO = tmem + 192;  // of group g: + 64 g, + 32 g, + 128 g
    const int n_tiles = range.end - range.begin;
    TileCursor<MB, Sh::kTileLog> cur;
    cur.b = range.b;
    cur.u = range.u;
    cur.rb = range.rb;
    cur.read_sequence(p);
    cur.enter(p, range.tile);

    const int loader = warp < 2 ? warp : NL == 4 && (warp == 6 || warp == 7) ? warp - 4 : -1;
    if (loader >= 0) {
        // ---------------- loaders ----------------
        // A stage's barrier counts every loader thread, when its copies have landed, and the warps' notes of what they loaded.
        bool ok = true;
        int piece = 0;
        for (int i = 0; i < n_tiles; ++i) {
            const bool first = i == 0 || cur.tile == cur.end;
            if (i > 0 && first) {
                cur.next_item(p);
                ++piece;
            }
            const int head = p.head_order[cur.first_head];
            if (first) {
                if (!(ok = warp_wait<true>(bar(kQEmpty + (piece & 1)), ((uint32_t)(piece >> 1) & 1) ^ 1, 42))) break;
                load_query_rows<D>(p, cur.b, head, cur.rows * p.g, cur.rb * MB, loader * (QR / NL), QR / NL, sQ(piece & 1), Sh::kQPanel);
                cp_async_arrive(bar(kQFull + (piece & 1)));
            }
            const int s = i % ST;
            if (!(ok = warp_wait<true>(bar(kEmpty + s), ((uint32_t)(i / ST) & 1) ^ 1, 43))) break;
#pragma unroll
            for (int k = 0; k < SW; k += 16) {
                const uint32_t got = load_16_slots<D>(p.c, cur.b, head, cur.first_slot() + loader * SW + k, cur.lo, cur.hi, sK(s), sV(s), true,
                                                      loader * SW + k, 8192, p.page_whole);
                if (lane == 0) there[s][(loader * SW + k) / 16] = got;
            }
            cp_async_arrive(bar(kFull + s));
            if (lane == 0) mbar_arrive(bar(kFull + s));
            ++cur.tile;
        }
    } else if (warp == 2) {
        // ---------------- issuer ----------------
        // S(i) as soon as its tile has landed and its buffer's scores have been read, O += P(j) V as soon as P(j) is there,
        // whichever comes first.  What the loaders' copies wrote is in the generic proxy's order and the products read through
        // the async one: the fence between the two stands here, after the barrier that the copies complete.
        constexpr uint32_t idesc_s = make_idesc_bf16(128, 64, 0, 0), idesc_o = make_idesc_bf16(128, D, 0, 1);
        int i = 0, j = 0, piece = 0, piece_start = 0;
        uint32_t fresh = 0;  // bit k & 31: tile k is the first of its group in its piece
        bool first = true, tile_there = false;
        for (int idle = 0; j < n_tiles; ++idle) {
            if (idle > (1 << 18)) {  // a long time without either: a bounded wait for what has to come next
                if (!(j < i ? warp_wait<true>(bar(kPFull + (j & 1)), (uint32_t)(j >> 1) & 1, 46)
                            : warp_wait<true>(bar(kFull + i % ST), (uint32_t)(i / ST) & 1, 45) &&
                                  (!first || warp_wait<true>(bar(kQFull + (piece & 1)), (uint32_t)(piece >> 1) & 1, 44))))
                    break;
                idle = 0;
            }
            if (j < i && __all_sync(0xffffffffu, mbar_test_wait(bar(kPFull + (j & 1)), (uint32_t)(j >> 1) & 1))) {
                tc_fence_after();
                const uint64_t vd = make_sdesc(sV(j % ST), 8192, 1024);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mma_ts(tO + (j & 1) * 128, tP + (j & 1) * 32 + k * 8, vd + ((k * 2048) >> 4), idesc_o, k > 0 || !((fresh >> (j & 31)) & 1));
                mma_commit(bar(kPvDone + (j & 1)));
                mma_commit(bar(kEmpty + j % ST));
                ++j;
                idle = 0;
            }
            if (i == n_tiles) continue;
            if (!tile_there) {
                if (!__all_sync(0xffffffffu, mbar_test_wait(bar(kFull + i % ST), (uint32_t)(i / ST) & 1) &&
                                                 (!first || mbar_test_wait(bar(kQFull + (piece & 1)), (uint32_t)(piece >> 1) & 1))))
                    continue;
                fence_proxy_async_smem();
                tile_there = true;
            }
            if (i >= 2 && !__all_sync(0xffffffffu, mbar_test_wait(bar(kSRead + (i & 1)), (uint32_t)((i >> 1) - 1) & 1))) continue;
            tc_fence_after();
            const uint64_t qd = make_sdesc(sQ(piece & 1), 16, 1024), kd = make_sdesc(sK(i % ST), 16, 1024);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                mma_ss(tS + (i & 1) * 64, qd + (((k / 4) * Sh::kQPanel + (k % 4) * 32) >> 4), kd + (((k / 4) * 8192 + (k % 4) * 32) >> 4), idesc_s, k > 0);
            mma_commit(bar(kSFull + (i & 1)));
            fresh = (fresh & ~(1u << (i & 31))) | ((i - piece_start < 2 ? 1u : 0u) << (i & 31));
            ++i;
            ++cur.tile;
            tile_there = first = false;
            idle = 0;
            if (cur.tile == cur.end || i == n_tiles) {
                mma_commit(bar(kQEmpty + (piece & 1)));
                if (i < n_tiles) {
                    cur.next_item(p);
                    ++piece;
                    piece_start = i;
                    first = true;
                }
            }
        }
    } else if (warp >= 4 && (warp & 3) < QR / 32) {
        // ---------------- softmax ----------------
        bool ok = true;
        const int grp = (warp - 4) >> 2, row = tid & 127, quarter = warp & 3;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, tSg = tS + lanes + grp * 64, tPg = tP + lanes + grp * 32;
        // All softmax warps meet at an item's end, whatever has become of them: a warp whose wait has failed gets there at once,
        // the others when theirs fail too, and none goes on when one has failed.
        auto both_agree = [](bool mine) {
            uint32_t all;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 3, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                         : "=r"(all) : "r"((uint32_t)mine), "n"(2 * QR) : "memory");
            return all != 0;
        };
        auto scores_read = [&] {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kSRead + grp));
        };
        // O += P V of the group's tile q (of the one before its tile, or its last): waited for tile by tile, so that a wait by
        // parity cannot take one phase for another
        auto products_done = [&](int q) {
            const bool y = q < 0 || warp_wait<true>(bar(kPvDone + grp), (uint32_t)(q >> 1) & 1, 49);
            tc_fence_after();
            return y;
        };
        int scans = 0;
        int i0 = 0;  // the piece's first tile
        while (i0 < n_tiles && ok) {
            const int first = cur.tile, count = min(cur.end - first, n_tiles - i0), head = p.head_order[cur.first_head];
            const int rows = cur.rows * p.g, r = cur.rb * MB + row;
            const bool real = r < rows;
            int lo, hi, all_lo, all_hi, x;
            const int t = (int)fdiv((uint32_t)min(r, rows - 1), p.f_g);
            visible_slots(p, cur.n, cur.rows, cur.shift, t, cur.cls, &lo, &hi);
            visible_slots(p, cur.n, cur.rows, cur.shift, (int)fdiv((uint32_t)(min((cur.rb + 1) * MB, rows) - 1), p.f_g), cur.cls, &all_lo, &x);
            visible_slots(p, cur.n, cur.rows, cur.shift, (int)fdiv((uint32_t)(cur.rb * MB), p.f_g), cur.cls, &x, &all_hi);
            const bool idle = cur.rb * MB + quarter * 32 >= rows;  // none of this warp's rows is there: it only keeps step
            float base = 0.f, l = 0.f, slack = -INFINITY;
            int done = -1;  // the group's last tile of the piece
            const int slot_first = cur.first_slot();
            for (int i = i0 + ((i0 ^ grp) & 1); i < i0 + count; i += 2) {
                if (!(ok = warp_wait<true>(bar(kSFull + grp), (uint32_t)(i >> 1) & 1, 47))) break;
                const int st = i % ST, slot0 = slot_first + (i - i0) * 64;
                if (!(ok = warp_wait<true>(bar(kFull + st), (uint32_t)(i / ST) & 1, 51))) break;  // done: for what the loaders wrote
                tc_fence_after();
                uint32_t pk[32];
                unsigned long long bad = 0;
                const unsigned long long have = (unsigned long long)(there[st][0] | there[st][1] << 16) |
                                                (unsigned long long)(there[st][2] | there[st][3] << 16) << 32;
                const bool edge_range = slot0 < all_lo || slot0 + 64 > all_hi;
                if (!idle) {
                    uint32_t s0[32], s1[32];
                    tmem_ld_x32(tSg, s0);
                    tmem_ld_x32(tSg + 32, s1);
                    tmem_wait_ld_dep(s0);
                    reg_fence32(s1);
                    scores_read();
                    const uint64_t scale2 = f32x2(p.scale_log2, p.scale_log2), base2 = f32x2(-base, -base);
                    auto over_base = [&](uint32_t (&s)[32]) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float a, b;
                            f32x2_unpack(fma_f32x2(f32x2_bits(s[e], s[e + 1]), scale2, base2), a, b);
                            s[e] = __float_as_uint(a);
                            s[e + 1] = __float_as_uint(b);
                        }
                    };
                    over_base(s0);
                    over_base(s1);
                    if (edge_range || have != ~0ull) {
                        auto masked = [&](uint32_t (&s)[32], int c) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (slot0 + c + e < lo || slot0 + c + e >= hi || !((have >> (c + e)) & 1)) s[e] = 0xff800000u;
                        };
                        masked(s0, 0);
                        masked(s1, 32);
                    }
                    float m0 = __uint_as_float(s0[0]), m1 = __uint_as_float(s1[0]);
#pragma unroll
                    for (int e = 1; e < 31; e += 2) {
                        m0 = fmax3(m0, __uint_as_float(s0[e]), __uint_as_float(s0[e + 1]));
                        m1 = fmax3(m1, __uint_as_float(s1[e]), __uint_as_float(s1[e + 1]));
                    }
                    const float mx = fmaxf(fmax3(m0, m1, __uint_as_float(s0[31])), __uint_as_float(s1[31]));
                    const bool up = mx > slack;
                    if (__any_sync(0xffffffffu, up)) {
                        float moved = 0.f, f = 1.f;
                        if (up) {
                            const float to = base + mx;
                            moved = to - base;  // by what the rounded base moves: scores and sums follow it
                            f = slack == -INFINITY ? 0.f : ex2(-moved);
                            base = to;
                            slack = kDecSlack;
                            l *= f;
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                s0[e] = __float_as_uint(__uint_as_float(s0[e]) - moved);
                                s1[e] = __float_as_uint(__uint_as_float(s1[e]) - moved);
                            }
                        }
                        if (done >= 0) {  // O holds the group's earlier tiles of the piece
                            if (!(ok = products_done(i - 2))) break;
#pragma unroll 1
                            for (int c = 0; c < D; c += 32) {
                                uint32_t o[32];
                                tmem_ld_x32(tO + lanes + grp * 128 + c, o);
                                tmem_wait_ld_dep(o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st_x32(tO + lanes + grp * 128 + c, o);
                            }
                            tmem_wait_st();
                        }
                    }
                    float la = 0.f, lb = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float a0 = ex2(__uint_as_float(s0[2 * e])), a1 = ex2(__uint_as_float(s0[2 * e + 1]));
                        const float b0 = ex2(__uint_as_float(s1[2 * e])), b1 = ex2(__uint_as_float(s1[2 * e + 1]));
                        la += a0 + a1;
                        lb += b0 + b1;
                        pk[e] = pack_bf16(a0, a1);
                        pk[16 + e] = pack_bf16(b0, b1);
                    }
                    l += la + lb;
                } else {
                    scores_read();
#pragma unroll
                    for (int e = 0; e < 32; ++e) pk[e] = 0u;
                }
                if (edge_range) {
                    // Slots that some rows see and others do not: a weight of zero does not undo an infinite or NaN V.  Such
                    // rows of V are taken out of the product and added one by one to the rows that see them, from the cache.
#pragma unroll 1
                    for (int j = 0; j < 64; ++j) {
                        const bool part = (slot0 + j < all_lo || slot0 + j >= all_hi) && ((have >> j) & 1);
                        if (!part) continue;
                        bool odd = false;
                        if (lane < C) {
                            const uint4 w4 = lds128(sV(st) + panel_at(j, lane, 8192));
                            const uint32_t ww[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) odd |= (ww[e] & 0x7f80u) == 0x7f80u || (ww[e] & 0x7f800000u) == 0x7f800000u;
                        }
                        if (__any_sync(0xffffffffu, odd)) bad |= 1ull << j;
                    }
                    if (bad) {  // the four warps have found the same; the first clears them once all have looked
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(kScan + grp));
                        if (quarter == 0) {
                            if (!(ok = warp_wait<true>(bar(kScan + grp), (uint32_t)scans & 1, 52))) break;
#pragma unroll 1
                            for (int j = 0; j < 64; ++j)
                                if (((bad >> j) & 1) && lane < C) st_shared_v4(sV(st) + panel_at(j, lane, 8192), 0u, 0u, 0u, 0u);
                            fence_proxy_async_smem();
                        }
                        ++scans;
                    }
                }
                if (!(ok = products_done(i - 2))) break;  // they have read the P buffer
                tmem_st_x32(tPg, pk);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kPFull + grp));
                done = i;
                if (bad) {
                    if (!(ok = products_done(i))) break;
                    float w[64];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        w[2 * e] = __uint_as_float(pk[e] << 16);
                        w[2 * e + 1] = __uint_as_float(pk[e] & 0xffff0000u);
                    }
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        tmem_ld_x32(tO + lanes + grp * 128 + c, o);
                        tmem_wait_ld_dep(o);
#pragma unroll 1
                        for (int j = 0; j < 64; ++j) {
                            const int slot = slot0 + j;
                            int prow, page;
                            if (!((bad >> j) & 1) || !real || slot < lo || slot >= hi || (page = page_of(p.c, cur.b, slot, &prow)) < 0) continue;
                            const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(
                                p.c.V + page * p.c.v_stride[0] + prow * p.c.v_stride[1] + head * p.c.v_stride[2]) + c;
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(fmaf(w[j], __bfloat162float(v[e]), __uint_as_float(o[e])));
                        }
                        tmem_st_x32(tO + lanes + grp * 128 + c, o);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                }
            }
            // ---- the piece's rows: both groups' parts joined, each group writing one half of the dims ----
            if (ok && done >= 0) ok = products_done(done);
            end_ml[grp][row] = make_float2(done < 0 || slack == -INFINITY ? -INFINITY : base, l);
            tc_fence_before();
            ok = both_agree(ok);
            tc_fence_after();
            if (!ok) break;
            const int list0 = range.begin + i0 - first, b_first = list0 / range.per, b_last = (list0 + cur.end - 1) / range.per;
            if (first == 0 && row == 0 && grp == 0)
                p.item_blocks[((long long)cur.b * p.c.Hkv + head) * p.row_blocks + cur.rb] = make_int2(b_first, b_last);
            if (!idle) {
                const float2 ma = end_ml[0][row], mb = end_ml[1][row];
                const float top = fmaxf(ma.x, mb.x), zero = top == -INFINITY ? 0.f : top, fa = ex2(ma.x - zero), fb = ex2(mb.x - zero);
                const float sum = ma.y * fa + mb.y * fb, inv = b_first != b_last ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
                // a group without a tile in the piece, or whose rows saw nothing, has nothing (or something old) in its O
                const bool ua = ma.x != -INFINITY, ub = mb.x != -INFINITY;
                const int qh = head * p.g + (real ? r - t * p.g : 0);
                const long long part = ((long long)blockIdx.x * 2 + (first == 0 ? 1 : 0)) * MB + row;
#pragma unroll 1
                for (int c = grp * (D / 2); c < (grp + 1) * (D / 2); c += 32) {
                    uint32_t o[32], o2[32];
                    tmem_ld_x32(tO + lanes + c, o);
                    tmem_ld_x32(tO + lanes + 128 + c, o2);
                    tmem_wait_ld_dep(o);
                    reg_fence32(o2);
                    if (!real) continue;
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        o[e] = __float_as_uint(((ua ? __uint_as_float(o[e]) * fa : 0.f) + (ub ? __uint_as_float(o2[e]) * fb : 0.f)) * inv);
                    if (b_first == b_last) {
                        uint4* to = reinterpret_cast<uint4*>(p.O + cur.b * p.o_stride[0] + t * p.o_stride[1] + qh * p.o_stride[2] + c);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t q[4];
#pragma unroll
                            for (int y = 0; y < 4; ++y) q[y] = pack_bf16(__uint_as_float(o[8 * e + 2 * y]), __uint_as_float(o[8 * e + 2 * y + 1]));
                            to[e] = make_uint4(q[0], q[1], q[2], q[3]);
                        }
                    } else {
                        uint4* to = reinterpret_cast<uint4*>(p.part_o + part * D + c);
#pragma unroll
                        for (int e = 0; e < 8; ++e) to[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                    }
                }
                if (real && grp == 0) {
                    if (b_first == b_last)
                        p.LSE[((long long)cur.b * p.Hq + qh) * p.c.Lq + t] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
                    else
                        p.part_ml[part] = make_float2(top, sum);
                }
            }
            tc_fence_before();
            both_agree(true);
            tc_fence_after();
            i0 += count;
            if (i0 < n_tiles) cur.next_item(p);
        }
    }
    // ---------------- teardown ----------------
    cp_async_commit();  // the loaders' copies report to barriers: after a failed wait nobody else may have waited for them
    cp_async_wait<0>();
    drain_if_failed();
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        __syncwarp();
        tmem_dealloc(tmem, 512);
    }
}

// ---- attention weights ---------------------------------------------------------------------------------------------
// Sum over the rows of each slot's weight, from the finished LSE: S^T = K Q^T again, 128 slots in M and up to 128 rows in N, a
// thread with its slot's row of the accumulator.  Keeping the scores of the first pass instead would write and read 8 bytes a
// (row, slot), more than the 256 bytes of K from 32 rows on.  A block takes four tiles of 128 slots of one (sequence, KV head)
// one after the other; three or four blocks to an SM cover each other's loads (two blocks with the next tile on its way while
// one is computed took longer).  Where QR rows hold all of them the queries are loaded once.
constexpr int kWeightTiles = 4;
template <int D, int QR>
struct RowWeightsShape {
    static constexpr int kTile = (D / 64) * 16384, kQPanel = QR * 128;
    static constexpr int kDynamic = kTile + (D / 64) * kQPanel + 1024;
};
template <int D, int QR>
__global__ void __launch_bounds__(128) decode_row_weights_kernel(const __grid_constant__ DecodeParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) float lse2[QR];
    __shared__ int lo[QR], hi[QR];
    __shared__ uint32_t tmem_slot, loaded[8];
    __shared__ __align__(8) uint64_t bar_mem;
    after_previous_kernel();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, h = blockIdx.y, b = blockIdx.z;
    const int new_r = new_rows(p.c, b), n = seq_len(p.c, b), first = blockIdx.x * (128 * kWeightTiles);
    if (first >= n || new_r == 0) return;
    const int shift = shift_of(p.c, b), cls = p.head_class[h], rows = new_r * p.g;
    const float* w_in = p.w_in ? p.w_in + ((long long)b * p.c.Hkv + h) * p.W : nullptr;
    float* w_out = p.w_out + ((long long)b * p.c.Hkv + h) * p.W;
    int all_lo, all_hi, inner_lo, inner_hi;  // slots that some row sees, and that every row sees
    visible_slots(p, n, new_r, shift, 0, cls, &all_lo, &inner_hi);
    visible_slots(p, n, new_r, shift, new_r - 1, cls, &inner_lo, &all_hi);
    // this block's tiles with a visible slot: [t0, t1) of its kWeightTiles; the others take over what they had
    const int end = min(n, first + 128 * kWeightTiles);
    const int t0 = min(max((all_lo - first) / 128, 0), kWeightTiles), t1 = min(max((min(all_hi, end) - first + 127) / 128, t0), kWeightTiles);
    for (int j = first + tid; j < end; j += 128)
        if (j < first + t0 * 128 || j >= first + t1 * 128) w_out[j] = w_in ? w_in[j] : 0.f;
    if (t0 == t1) return;
    using Sh = RowWeightsShape<D, QR>;
    const uint32_t k_tile = (smem_u32(smem_raw) + 1023u) & ~1023u, q_tile = k_tile + Sh::kTile, bar = smem_u32(&bar_mem);
    if (tid == 0) {
        mbar_init(bar, 1);
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_slot), 128);
        tmem_relinquish();
    }
    auto load_rows = [&](int r0) {
        load_query_rows<D>(p, b, h, rows, r0, warp * (QR / 4), QR / 4, q_tile, Sh::kQPanel);
        if (tid < QR && r0 + tid < rows) {
            const int r = r0 + tid, t = (int)fdiv((uint32_t)r, p.f_g);
            const float l = p.LSE[((long long)b * p.Hq + h * p.g + r - t * p.g) * p.c.Lq + t];
            visible_slots(p, n, new_r, shift, t, cls, &lo[tid], &hi[tid]);
            // a row without a finite score weighs nothing anywhere: exp2(score - inf) is 0 on the path that looks at no mask too
            lse2[tid] = l == -INFINITY ? INFINITY : l * 1.4426950408889634f;
        }
    };
    bool ok = true;
    uint32_t turn = 0;
    for (int t = t0; t < t1 && ok; ++t) {
        const int slot0 = first + t * 128, j = slot0 + tid;
        const bool inner = slot0 >= inner_lo && slot0 + 128 <= inner_hi;
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t got = load_16_slots<D>(p.c, b, h, slot0 + warp * 32 + k * 16, all_lo, all_hi, k_tile, 0, false, warp * 32 + k * 16, 16384,
                                                  p.page_whole);
            if (lane == 0) loaded[warp * 2 + k] = got;
        }
        for (int r0 = 0; r0 < rows && ok; r0 += QR, ++turn) {
            const int m = min(QR, rows - r0);
            if (rows > QR || t == t0) load_rows(r0);
            cp_async_commit();
            cp_async_wait<0>();
            fence_proxy_async_smem();
            tc_fence_before();
            __syncthreads();
            tc_fence_after();
            if (warp == 0) {
                const uint64_t kd = make_sdesc(k_tile, 16, 1024), qd = make_sdesc(q_tile, 16, 1024);
                const uint32_t idesc = make_idesc_bf16(128, (m + 15) & ~15, 0, 0);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    mma_ss(tmem_slot, kd + (((k / 4) * 16384 + (k % 4) * 32) >> 4), qd + (((k / 4) * Sh::kQPanel + (k % 4) * 32) >> 4), idesc, k > 0);
                }
                mma_commit(bar);
            }
            ok = warp_wait<true>(bar, turn & 1, 41);
            tc_fence_after();
            const bool have = ok && (loaded[tid >> 4] >> (tid & 15)) & 1;
            for (int c = 0; c < m && ok; c += 32) {
                uint32_t s[32];
                tmem_ld_x32(tmem_slot + ((uint32_t)(warp * 32) << 16) + c, s);
                tmem_wait_ld_dep(s);
                if (have && inner && c + 32 <= m) {
                    float x[4] = {};
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 l = *reinterpret_cast<const float4*>(lse2 + c + i);
                        x[0] += ex2(fmaf(__uint_as_float(s[i]), p.scale_log2, -l.x));
                        x[1] += ex2(fmaf(__uint_as_float(s[i + 1]), p.scale_log2, -l.y));
                        x[2] += ex2(fmaf(__uint_as_float(s[i + 2]), p.scale_log2, -l.z));
                        x[3] += ex2(fmaf(__uint_as_float(s[i + 3]), p.scale_log2, -l.w));
                    }
                    sum += (x[0] + x[1]) + (x[2] + x[3]);
                } else if (have) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c + i < m && j >= lo[c + i] && j < hi[c + i]) sum += ex2(__uint_as_float(s[i]) * p.scale_log2 - lse2[c + i]);
                }
            }
            tc_fence_before();
            ok = __syncthreads_and(ok);
        }
        if (j < n) w_out[j] = (w_in ? w_in[j] : 0.f) + sum;
    }
    cp_async_wait<0>();
    drain_if_failed();
    __syncthreads();
    if (warp == 0) {
        __syncwarp();
        tmem_dealloc(tmem_slot, 128);
    }
}

}  // namespace segattn
