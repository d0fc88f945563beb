// What the kernels over a paged key/value cache share: the arguments of a batch, and where a sequence's new rows, slots
// and pages lie.  Everything read from the device's tables is checked against the host's sizes before it becomes an
// address: a length is cut to [0, max_len], a chunk to max_new rows inside [0, n_rows), and a page outside the pool is no
// page (its tokens are neither stored nor seen).
#pragma once
#include "common.h"

namespace llmc {

struct PagedArgs {
  const int32_t* table;       // [n_seqs, max_pages]
  const int32_t* length;      // [n_seqs]
  const int32_t* new_start;   // [n_seqs + 1], or NULL: row b is the one new token of sequence b
  int32_t n_seqs, max_pages, n_rows, max_new, max_len;
  int32_t n_pages, page_shift, n_kv;
};

struct SeqRange {
  int len;      // tokens in the cache, with the new ones
  int first;    // first row of the new tokens
  int q;        // new tokens
};

__device__ __forceinline__ SeqRange seq_range(const PagedArgs& a, int b) {
  SeqRange s;
  s.len = min(max(a.length[b], 0), a.max_len);
  if (a.new_start) {
    const int lo = a.new_start[b], hi = a.new_start[b + 1];
    s.first = lo;
    const bool ok = lo >= 0 && hi <= a.n_rows && lo < hi;
    s.q = ok ? min(hi - lo, a.max_new) : 0;
  } else {
    s.first = b;
    s.q = 1;
  }
  return s;
}

// The sequence whose rows [new_start[b], new_start[b + 1]) hold `row`, or -1: every wavefront counts the starts that are not
// beyond the row, 64 at a time (no chain of dependent loads, as a binary search would be).  All lanes ask for one row.
__device__ __forceinline__ int seq_of_row(const PagedArgs& a, int row) {
  if (!a.new_start) return row < a.n_seqs ? row : -1;
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int i = 0; i <= a.n_seqs; i += 64)
    n += __popcll(__ballot(i + lane <= a.n_seqs && a.new_start[min(i + lane, a.n_seqs)] <= row));
  return n >= 1 && n <= a.n_seqs ? n - 1 : -1;
}

// page of a slot, or -1
__device__ __forceinline__ int page_of(const PagedArgs& a, int b, int slot) {
  const int col = slot >> a.page_shift;
  const int p = a.table[(size_t)b * a.max_pages + min(col, a.max_pages - 1)];
  return (uint32_t)p < (uint32_t)a.n_pages ? p : -1;
}

// Workgroups numbered over two dimensions, since no dimension of a launch may have 2^32 threads: their number may be exceeded.
inline dim3 flat_grid(int64_t workgroups) {
  const int64_t most = 1 << 22;
  return dim3((unsigned)(workgroups < most ? workgroups : most), (unsigned)((workgroups + most - 1) / most));
}
__device__ __forceinline__ uint32_t flat_block() { return blockIdx.x + blockIdx.y * gridDim.x; }

}  // namespace llmc
