// What the kernels of the paged key-value cache share: its description, lookups with their checks, how the work of an
// attention is dealt.
#pragma once
#include "common.cuh"

namespace lsp {

// bits of the status word (lsp_paged_kv.status)
constexpr int PG_BAD_LEN = 1, PG_BAD_PAGE = 2, PG_BAD_ROWS = 4;

struct PagedView {
  char *k, *v;                                  // pools (element type T of the kernel)
  const int* table;                             // [batch][max_pages], or null: page p of sequence b is b * max_pages + p
  int* status;
  long long page_stride, row_stride, head_stride;      // elements
  int n_pages, page, max_pages, batch, hkv;
};

// floor(a / b), a >= 0, b > 0, for quotients below 2^20: in floating point it is off by less than 3 2^-23 of itself, that is by one at most.
// (A third of the instructions of the integer division, and what a launch begins with is a chain of them.)
__device__ __forceinline__ int pg_div(int a, int b) {
  int q = (int)__fdividef((float)a, (float)b);
  const int r = a - q * b;
  if (r < 0) --q;
  if (r >= b) ++q;
  return q;
}

__device__ __forceinline__ void pg_flag(const PagedView& pv, int bit) {
  if (pv.status) atomicOr(pv.status, bit);
}
__device__ __forceinline__ int pg_capacity(const PagedView& pv) { return pv.max_pages * pv.page; }

// Slots in use, n as the caller's array has it, inside [0, capacity].
__device__ __forceinline__ int pg_len(const PagedView& pv, int n) {
  const int cap = pg_capacity(pv);
  if (n < 0 || n > cap) {
    pg_flag(pv, PG_BAD_LEN);
    return n < 0 ? 0 : cap;
  }
  return n;
}
// Id of page p of sequence b (0 <= p < max_pages); -1 with the flag set where the table names no page of the pool.
__device__ __forceinline__ int pg_page(const PagedView& pv, int b, int p) {
  const int id = pv.table ? pv.table[(long long)b * pv.max_pages + p] : b * pv.max_pages + p;
  if (id < 0 || id >= pv.n_pages) {
    pg_flag(pv, PG_BAD_PAGE);
    return -1;
  }
  return id;
}
// Asks for bytes at p to come to L2 (thread `i` of n, a line each).  Ahead of the wait for a preceding kernel: nothing is read.
// (64 bits: a launch may have 2^23 blocks and more, 2^31 threads.)
__device__ __forceinline__ void pg_prefetch(const void* p, long long bytes, long long i, long long n) {
  for (long long at = i * 128; p && at < bytes; at += n * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"((const char*)p + at));
}
// By the whole grid, neighbouring lines by neighbouring blocks.
__device__ __forceinline__ void pg_prefetch_grid(const void* p, long long bytes) {
  pg_prefetch(p, bytes, (long long)threadIdx.x * gridDim.x + blockIdx.x, (long long)gridDim.x * blockDim.x);
}
// The page table, a megabyte of it at most, by the whole grid.
__device__ __forceinline__ void pg_prefetch_table(const PagedView& pv) {
  pg_prefetch_grid(pv.table, min((long long)pv.batch * pv.max_pages * 4, 1ll << 20));
}
// Where slot j of sequence b begins (0 <= j < capacity), in elements from the pool's start; -1 where its page is none.
__device__ __forceinline__ long long pg_slot(const PagedView& pv, int b, int j) {
  const int p = pg_div(j, pv.page), id = pg_page(pv, b, p);
  return id < 0 ? -1 : (long long)id * pv.page_stride + (long long)(j - p * pv.page) * pv.row_stride;
}
// Packed rows of sequence b: first one and count (0 with the flag set where the offsets leave the caller's rows).
struct RowSpan { int first, n; };
__device__ __forceinline__ RowSpan pg_rows(const PagedView& pv, const int* row_off, int b, int max_rows, int n_rows) {
  if (!row_off) return RowSpan{b * max_rows, max_rows};
  const int r0 = row_off[b], r1 = row_off[b + 1];
  if (r0 < 0 || r1 < r0 || r1 > n_rows || r1 - r0 > max_rows) {
    pg_flag(pv, PG_BAD_ROWS);
    return RowSpan{0, 0};
  }
  return RowSpan{r0, r1 - r0};
}

}  // namespace lsp
