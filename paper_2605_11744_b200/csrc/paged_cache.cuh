// The paged key/value cache as the kernels see it: slot j of sequence b is row j % page_size of page
// block_table[b][j / page_size].  Every number that comes from device memory is checked here before it becomes an
// address; what is out of range is recorded (g_refused_input) and not followed.
#pragma once
#include <cstdint>

#include "mask.cuh"
#include "ptx.cuh"

namespace segattn {

struct PagedView {
    char* K;
    char* V;
    long long k_stride[3], v_stride[3];  // BYTES, for (page, row, head)
    const int32_t* block_table;
    const int32_t* kv_len;
    const int32_t* q_len;      // may be null: Lq for every sequence
    const int32_t* pos_shift;  // may be null: 0
    FastDiv f_page;            // division by page_size
    int table_stride, n_pages, max_pages;
    int cap;                   // max_pages * page_size
    int B, Hkv, Lq;
};

__device__ __forceinline__ void refuse_input(int site) { atomicCAS(&g_refused_input, 0, (1 << 8) | site); }

// Length of sequence b, cut to what its row of the block table can hold.
__device__ __forceinline__ int seq_len(const PagedView& c, int b) {
    const int n = c.kv_len[b];
    if (n < 0 || n > c.cap) refuse_input(30);
    return min(max(n, 0), c.cap);
}
// New rows of sequence b, cut to [0, Lq].
__device__ __forceinline__ int new_rows(const PagedView& c, int b) {
    if (!c.q_len) return c.Lq;
    const int q = c.q_len[b];
    if (q < 0 || q > c.Lq) refuse_input(31);
    return min(max(q, 0), c.Lq);
}
__device__ __forceinline__ int shift_of(const PagedView& c, int b) {
    if (!c.pos_shift) return 0;
    const int s = c.pos_shift[b];
    if (s < 0) refuse_input(32);
    return max(s, 0);
}
// The block table's entry for a slot in [0, cap), unchecked, and the slot's row in its page.
__device__ __forceinline__ int table_entry(const PagedView& c, int b, int slot) {
    return __ldg(c.block_table + (long long)b * c.table_stride + fdiv((uint32_t)slot, c.f_page));
}
__device__ __forceinline__ int row_in_page(const PagedView& c, int slot) {
    return slot - (int)(fdiv((uint32_t)slot, c.f_page) * c.f_page.d);
}
// Page of a slot in [0, cap) and the row in it; -1 for a page number out of range.
__device__ __forceinline__ int page_of(const PagedView& c, int b, int slot, int* row) {
    *row = row_in_page(c, slot);
    const int page = table_entry(c, b, slot);
    if ((unsigned)page >= (unsigned)c.n_pages) {
        refuse_input(33);
        return -1;
    }
    return page;
}

}  // namespace segattn
