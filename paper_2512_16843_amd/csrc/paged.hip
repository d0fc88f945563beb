// The paged key/value cache: storing new tokens, and evicting those of least accumulated attention weight.
//
// Pages of keys and of values are [n_pages, n_kv_heads, page_size, head_dim], so the tokens of one head in one page are
// contiguous (page_size * head_dim elements): what an attention kernel reads for a head comes in whole cache lines.
#include <algorithm>
#include "paged.h"

namespace llmc {
namespace {

// ---- storing ---------------------------------------------------------------------------------------
// A wavefront stores one new token, keys and values of all heads, 16 bytes a lane: the row is read contiguously and lands in
// pieces of head_dim elements (128 bytes or more: whole lines).  Bound: memory (each element once read, once written).
struct AppendArgs {
  PagedArgs p;
  const uint4 *k_new, *v_new;
  uint4 *k, *v;
  int64_t ld_k, ld_v;          // row strides of the new tokens, in 16-byte vectors
  const int32_t* pos_new;
  int32_t* pos;
  float* weight;
  int32_t vec_shift;           // log2 of the vectors of one head
};

__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  const int row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= a.p.n_rows) return;
  const int b = seq_of_row(a.p, row);
  if (b < 0) return;
  const SeqRange s = seq_range(a.p, b);
  const int i = row - s.first, slot = s.len - s.q + i;
  if (i >= s.q || slot < 0) return;
  const int page = page_of(a.p, b, slot);
  const int nv = a.p.n_kv << a.vec_shift, off = slot & ((1 << a.p.page_shift) - 1);
  if (page >= 0) {
    const uint4 *ks = a.k_new + row * a.ld_k, *vs = a.v_new + row * a.ld_v;
    const size_t base = (size_t)page * a.p.n_kv << a.p.page_shift;
    for (int v = lane; v < nv; v += 64) {
      const int h = v >> a.vec_shift, c = v & ((1 << a.vec_shift) - 1);
      const size_t dst = ((base + ((size_t)h << a.p.page_shift) + off) << a.vec_shift) + c;
      const uint4 x = ks[v], y = vs[v];
      a.k[dst] = x;
      a.v[dst] = y;
    }
  }
  if (lane == 0) {
    const size_t at = ((size_t)b * a.p.max_pages << a.p.page_shift) + slot;
    if (a.pos) a.pos[at] = a.pos_new ? a.pos_new[row] : slot;
    if (a.weight) a.weight[at] = 0.f;
  }
}

// ---- eviction --------------------------------------------------------------------------------------
// Of a sequence with n tokens and a budget of k < n, the n - k tokens that come first by (protected, weight, position, slot)
// go.  Tokens are then moved only where they must be: the kept tokens in slots k .. n - 1 fill the holes in slots 0 .. k - 1,
// the i-th one the i-th hole, both ascending.  Source and destination slots are disjoint, so the moves need no order, and
// their number is at most the number of evicted tokens (closing the gaps in order would move nearly every token for each
// one that goes).
//
// The choice: one workgroup per sequence narrows a 64-bit key (protected flag, weight, position) to the (n - k)-th smallest
// by its digits of 8 bits, most significant first (a histogram in LDS a digit), then numbers holes and movers by a prefix
// sum over the slots.
constexpr int kSelThreads = 1024;

struct EvictArgs {
  const int32_t* table;
  const int32_t* length;
  int32_t n_seqs, max_pages, max_len, n_pages, page_shift, n_kv;
  int32_t* pos;
  float* weight;
  const int32_t* keep;
  int32_t sink, recent;
  int32_t* length_out;
  int32_t* counts;             // [n_seqs] number of moves
  int2* moves;                 // [n_seqs, max_moves] (source slot, destination slot)
  int32_t max_moves;
};

// order of a weight: ascending, -0 as +0, NaN above every number (a token whose weight cannot be told is kept)
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (w != w) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint64_t evict_key(float w, int pos, int last, int sink, int recent) {
  const uint32_t p = (uint32_t)max(pos, 0);
  const bool safe = pos < sink || (int64_t)pos > (int64_t)last - recent;
  return ((uint64_t)safe << 63) | ((uint64_t)weight_order(w) << 31) | p;
}

__global__ __launch_bounds__(kSelThreads) void kv_evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t wave_sum_s[2][kSelThreads / 64];
  __shared__ int sh_last;
  __shared__ uint32_t sh_digit, sh_before;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(a.length[b], 0), a.max_len);
  const int keep = min(max(a.keep[b], 0), n);
  const size_t slots = (size_t)a.max_pages << a.page_shift;
  int32_t* pos = a.pos + b * slots;
  float* weight = a.weight + b * slots;
  if (tid == 0) a.length_out[b] = keep;
  if (keep >= n) {
    if (tid == 0) a.counts[b] = 0;
    return;
  }
  if (tid == 0) sh_last = INT32_MIN;
  __syncthreads();
  int last = INT32_MIN;
  for (int j = tid; j < n; j += kSelThreads) last = max(last, pos[j]);
  atomicMax(&sh_last, last);
  __syncthreads();
  last = sh_last;
  // the digits of the (n - keep)-th smallest key
  uint64_t prefix = 0;
  uint32_t need = n - keep;            // still to be found among the keys that share the prefix
  for (int shift = 56; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += kSelThreads) {
      const uint64_t key = evict_key(weight[j], pos[j], last, a.sink, a.recent);
      if (shift == 56 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) { c[i] = hist[lane * 4 + i]; sum += c[i]; }
      uint32_t incl = sum;
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(incl, o, 64);
        if (lane >= o) incl += v;
      }
      uint32_t before = incl - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < need && need <= before + c[i]) { sh_digit = lane * 4 + i; sh_before = before; }
        before += c[i];
      }
    }
    __syncthreads();
    prefix |= (uint64_t)sh_digit << shift;
    need -= sh_before;
    __syncthreads();
  }
  // `need` tokens whose key equals the prefix go too, those in the lowest slots (positions of one sequence differ, so it is one)
  uint32_t eq_before = 0, hole_base = 0, mover_base = 0;
  int2* moves = a.moves + (size_t)b * a.max_moves;
  for (int j0 = 0; j0 < n; j0 += kSelThreads) {
    const int j = j0 + tid;
    const uint64_t key = j < n ? evict_key(weight[j], pos[j], last, a.sink, a.recent) : ~0ull;
    const bool eq = j < n && key == prefix;
    const uint64_t m_eq = __ballot(eq);
    if (lane == 0) wave_sum_s[0][wave] = __popcll(m_eq);
    __syncthreads();
    uint32_t my_eq = eq_before, all_eq = 0;
    for (int w = 0; w < kSelThreads / 64; ++w) {
      if (w < wave) my_eq += wave_sum_s[0][w];
      all_eq += wave_sum_s[0][w];
    }
    eq_before += all_eq;
    my_eq += __popcll(m_eq & ((1ull << lane) - 1));
    __syncthreads();
    const bool gone = j < n && (key < prefix || (eq && my_eq < need));
    const bool hole = gone && j < keep, mover = j < n && !gone && j >= keep;
    const uint64_t m_hole = __ballot(hole), m_move = __ballot(mover);
    if (lane == 0) { wave_sum_s[0][wave] = __popcll(m_hole); wave_sum_s[1][wave] = __popcll(m_move); }
    __syncthreads();
    uint32_t my_hole = hole_base, my_move = mover_base;
    for (int w = 0; w < kSelThreads / 64; ++w) {
      const uint32_t ch = wave_sum_s[0][w], cm = wave_sum_s[1][w];
      if (w < wave) { my_hole += ch; my_move += cm; }
      hole_base += ch;
      mover_base += cm;
    }
    my_hole += __popcll(m_hole & ((1ull << lane) - 1));
    my_move += __popcll(m_move & ((1ull << lane) - 1));
    if (hole && my_hole < (uint32_t)a.max_moves) moves[my_hole].y = j;
    if (mover && my_move < (uint32_t)a.max_moves) moves[my_move].x = j;
    __syncthreads();
  }
  // as many holes as movers
  const uint32_t n_moves = min(hole_base, (uint32_t)a.max_moves);
  if (tid == 0) a.counts[b] = (int)n_moves;
  __threadfence_block();
  __syncthreads();
  for (uint32_t i = tid; i < n_moves; i += kSelThreads) {
    const int2 m = moves[i];
    pos[m.y] = pos[m.x];
    weight[m.y] = weight[m.x];
  }
}

// moves keys and values: 16 bytes a lane, the vectors of one head's token on neighbouring lanes; grid (pieces, n_seqs)
__global__ __launch_bounds__(256) void kv_evict_move_kernel(EvictArgs a, uint4* __restrict__ k, uint4* __restrict__ v,
                                                            int vec_shift) {
  const int b = blockIdx.y;
  const int n_moves = a.counts[b];
  const int2* moves = a.moves + (size_t)b * a.max_moves;
  const int32_t* table = a.table + (size_t)b * a.max_pages;
  const int mask = (1 << a.page_shift) - 1, per = a.n_kv << vec_shift;
  const int64_t total = (int64_t)n_moves * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int mv = (int)(i / per), r = (int)(i - (int64_t)mv * per);
    const int h = r >> vec_shift, c = r & ((1 << vec_shift) - 1);
    const int2 m = moves[mv];
    const int ps = table[m.x >> a.page_shift], pd = table[m.y >> a.page_shift];
    if ((uint32_t)ps >= (uint32_t)a.n_pages || (uint32_t)pd >= (uint32_t)a.n_pages) continue;
    const size_t src = (((((size_t)ps * a.n_kv + h) << a.page_shift) + (m.x & mask)) << vec_shift) + c;
    const size_t dst = (((((size_t)pd * a.n_kv + h) << a.page_shift) + (m.y & mask)) << vec_shift) + c;
    const uint4 x = k[src], y = v[src];
    k[dst] = x;
    v[dst] = y;
  }
}

int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

}  // namespace

PagedArgs paged_args(const llmc_kv_desc_t* kv, const llmc_kv_batch_t* bt) {
  PagedArgs p{};
  p.table = bt->d_table; p.length = bt->d_length; p.new_start = bt->d_new_start;
  p.n_seqs = bt->n_seqs; p.max_pages = bt->max_pages; p.n_rows = bt->n_rows; p.max_new = bt->max_new; p.max_len = bt->max_len;
  p.n_pages = kv->n_pages; p.page_shift = log2_of(kv->page_size); p.n_kv = kv->n_kv_heads;
  return p;
}

llmc_status_t launch_kv_append(const llmc_kv_desc_t* kv, const llmc_kv_batch_t* bt, const void* k_new, int64_t ld_k,
                               const void* v_new, int64_t ld_v, const int32_t* pos_new, hipStream_t st) {
  if (bt->n_rows == 0) return LLMC_OK;
  const int e = (int)elem_size(kv->dtype);
  AppendArgs a{};
  a.p = paged_args(kv, bt);
  a.k_new = (const uint4*)k_new; a.v_new = (const uint4*)v_new;
  a.k = (uint4*)kv->d_k; a.v = (uint4*)kv->d_v;
  a.ld_k = ld_k * e / 16; a.ld_v = ld_v * e / 16;
  a.pos_new = pos_new; a.pos = bt->d_pos; a.weight = bt->d_weight;
  a.vec_shift = log2_of(kv->head_dim * e / 16);
  ProfScope ps_("kv_append_kernel", st);
  LLMC_KERNEL_GGL(kv_append_kernel, dim3((unsigned)((bt->n_rows + 3) / 4)), dim3(256), 0, st, a);
  LLMC_LAUNCH_CHECK("kv_append");
  return LLMC_OK;
}

// a sequence moves at most half of its tokens: as many as stay and as many as go
size_t kv_evict_ws_bytes(int n_seqs, int max_len) {
  return align_up((size_t)n_seqs * 4, 256) + (size_t)n_seqs * (max_len / 2 + 1) * sizeof(int2);
}

llmc_status_t launch_kv_evict(const llmc_kv_desc_t* kv, const llmc_kv_batch_t* bt, const int32_t* keep, int sink, int recent,
                              int32_t* length_out, void* ws, hipStream_t st) {
  EvictArgs a{};
  a.table = bt->d_table; a.length = bt->d_length;
  a.n_seqs = bt->n_seqs; a.max_pages = bt->max_pages; a.max_len = bt->max_len; a.n_pages = kv->n_pages;
  a.page_shift = log2_of(kv->page_size); a.n_kv = kv->n_kv_heads;
  a.pos = bt->d_pos; a.weight = bt->d_weight; a.keep = keep; a.sink = sink; a.recent = recent; a.length_out = length_out;
  a.counts = (int32_t*)ws;
  a.moves = (int2*)((char*)ws + align_up((size_t)bt->n_seqs * 4, 256));
  a.max_moves = bt->max_len / 2 + 1;
  { ProfScope ps_("kv_evict_select_kernel", st);
    LLMC_KERNEL_GGL(kv_evict_select_kernel, dim3((unsigned)bt->n_seqs), dim3(kSelThreads), 0, st, a); }
  LLMC_LAUNCH_CHECK("kv_evict_select");
  const int vec_shift = log2_of(kv->head_dim * (int)elem_size(kv->dtype) / 16);
  const int64_t most = (int64_t)a.max_moves * (kv->n_kv_heads << vec_shift);
  const unsigned pieces = (unsigned)std::max<int64_t>(1, std::min<int64_t>((most + 255) / 256, std::max(8, 4096 / bt->n_seqs)));
  { ProfScope ps_("kv_evict_move_kernel", st);
    LLMC_KERNEL_GGL(kv_evict_move_kernel, dim3(pieces, (unsigned)bt->n_seqs), dim3(256), 0, st, a, (uint4*)kv->d_k,
                    (uint4*)kv->d_v, vec_shift); }
  LLMC_LAUNCH_CHECK("kv_evict_move");
  return LLMC_OK;
}

}  // namespace llmc
