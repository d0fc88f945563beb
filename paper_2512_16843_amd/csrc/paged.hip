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
  const uint32_t idx = flat_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (idx >= (uint32_t)a.p.n_rows) return;
  const int row = idx;
  const int b = seq_of_row(a.p, row);
  if (b < 0) return;
  const SeqRange s = seq_range(a.p, b);
  const int i = row - s.first, slot = s.len - s.q + i;
  if ((uint32_t)i >= (uint32_t)s.q || slot < 0) return;
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
// A slot whose page is none can neither give its token away nor take one: below k it stays as it is, from k on its token goes,
// and the others are chosen among the slots that have pages.  Holes and movers are then as many as each other, all in pages.
//
// The choice: one workgroup per sequence.  A token's key is 64 bits (protected flag, weight, position); the (n - k)-th smallest is
// narrowed by digits of 11 bits, most significant first, a histogram in LDS a digit, until at most 64 keys share the digits
// so far (two digits, as weights go); a wavefront then ranks those by key and slot.  Holes and movers are numbered by counts
// of ballots.  Up to 24576 tokens the keys are read once and stay in registers.  Bound: latency, one workgroup's chain of loads and
// barriers (64 sequences of 1040 tokens 8.6 us, 8 of up to 8192 14.5; eight digits of 8 bits and keys read in each pass 17.4 and 42).
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64, kDigit = 11, kBins = 1 << kDigit;

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
  int4* moves;                 // [n_seqs, max_moves] source slot and page, destination slot and page
  int32_t max_moves;
};

// order of a weight: ascending, -0 as +0, NaN above every number (a token whose weight cannot be told is kept).  The lowest and
// the highest value are no weight's: evict_key's ends of the order are left to slots without a page.
constexpr uint64_t kGoesFirst = 0, kGoesLast = ~0ull;
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (w != w) return 0xFFFFFFFEu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint64_t evict_key(float w, int pos, int last, int sink, int recent) {
  const uint32_t p = (uint32_t)max(pos, 0);
  const bool safe = pos < sink || (int64_t)pos > (int64_t)last - recent;
  return ((uint64_t)safe << 63) | ((uint64_t)weight_order(w) << 31) | p;
}

// E: tokens of a thread, kept in registers; 0: read again in every pass
template <int E>
__global__ __launch_bounds__(kSelThreads) void kv_evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t totals[kSelWaves];
  __shared__ uint32_t sh_digit, sh_before, sh_count, sh_n;
  __shared__ int2 sh_last[kSelWaves];                            // a wavefront's highest position, and whether it found a bad page
  __shared__ int sh_slot;
  __shared__ uint64_t sh_key;
  __shared__ uint64_t cand_key[64];
  __shared__ int cand_slot[64];
  __shared__ uint32_t ballots[2][kSelWaves * (E ? E : 1)];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(a.length[b], 0), a.max_len);
  const int keep = min(max(a.keep[b], 0), n);
  const size_t slots = (size_t)a.max_pages << a.page_shift;
  const int32_t* pos = a.pos + b * slots;
  const float* weight = a.weight + b * slots;
  if (keep >= n) {
    if (tid == 0) {
      a.length_out[b] = keep;
      a.counts[b] = 0;
    }
    return;
  }
  const int32_t* table = a.table + (size_t)b * a.max_pages;
  const auto page = [&](int slot) {
    const int p = table[slot >> a.page_shift];
    return (uint32_t)p < (uint32_t)a.n_pages ? p : -1;
  };
  const int rounds = E ? E : (n + kSelThreads - 1) / kSelThreads;
  uint64_t key[E ? E : 1];
  int last = INT32_MIN;
  if (E) {
    float w[E ? E : 1];
    int p[E ? E : 1];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = min(e * kSelThreads + tid, n - 1);
      w[e] = weight[j];
      p[e] = pos[j];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) last = max(last, p[e]);
#pragma unroll
    for (int e = 0; e < E; ++e) key[e] = ((uint64_t)__float_as_uint(w[e]) << 32) | (uint32_t)p[e];
  } else {
    for (int j = tid; j < n; j += kSelThreads) last = max(last, pos[j]);
  }
  bool some_bad = false;                                         // is there a slot without a page?
  for (int i = tid; i <= (n - 1) >> a.page_shift; i += kSelThreads) some_bad |= (uint32_t)table[i] >= (uint32_t)a.n_pages;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) last = max(last, __shfl_xor(last, o, 64));
  const bool wave_bad = __ballot(some_bad) != 0;
  if (lane == 0) sh_last[wave] = make_int2(last, wave_bad);
  for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
  if (tid == 0) sh_n = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    last = max(last, sh_last[w].x);
    some_bad |= sh_last[w].y != 0;
  }
  const auto order = [&](float w, int p, int j) {
    if (some_bad && page(j) < 0) return j < keep ? kGoesLast : kGoesFirst;
    return evict_key(w, p, last, a.sink, a.recent);
  };
  if (E) {
#pragma unroll
    for (int e = 0; e < E; ++e)
      key[e] = order(__uint_as_float((uint32_t)(key[e] >> 32)), (int)(uint32_t)key[e], min(e * kSelThreads + tid, n - 1));
  }
  const auto key_at = [&](int e, int j) { return E ? key[E ? e : 0] : order(weight[j], pos[j], j); };
  // digits of the key, then (equal keys only) of the slot, until at most 64 tokens are left to choose among
  uint64_t prefix = 0;
  uint32_t slot_prefix = 0, need = n - keep, count = n;
  int shift = 64, slot_shift = 31;
  while (count > 64) {
    const bool by_slot = shift == 0;
    const int to = by_slot ? max(slot_shift - kDigit, 0) : max(shift - kDigit, 0);
    const uint32_t mask = (1u << ((by_slot ? slot_shift : shift) - to)) - 1;
#pragma unroll
    for (int e = 0; e < rounds; ++e) {
      const int j = e * kSelThreads + tid;
      if (j < n) {
        const uint64_t k = key_at(e, j);
        if (by_slot) {
          if (k == prefix && (slot_shift == 31 || ((uint32_t)j >> slot_shift) == (slot_prefix >> slot_shift)))
            atomicAdd(&hist[((uint32_t)j >> to) & mask], 1u);
        } else if (shift == 64 || (k >> shift) == (prefix >> shift)) {
          atomicAdd(&hist[(uint32_t)(k >> to) & mask], 1u);
        }
      }
    }
    __syncthreads();
    const uint32_t c0 = hist[2 * tid], c1 = hist[2 * tid + 1];
    uint32_t incl = c0 + c1;
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t v = __shfl_up(incl, o, 64);
      if (lane >= o) incl += v;
    }
    if (lane == 63) totals[wave] = incl;
    hist[2 * tid] = 0;
    hist[2 * tid + 1] = 0;
    __syncthreads();
    uint32_t before = incl - c0 - c1;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) before += w < wave ? totals[w] : 0;
    if (before < need && need <= before + c0) { sh_digit = 2 * tid; sh_before = before; sh_count = c0; }
    before += c0;
    if (before < need && need <= before + c1) { sh_digit = 2 * tid + 1; sh_before = before; sh_count = c1; }
    __syncthreads();
    if (by_slot) {
      slot_prefix |= sh_digit << to;
      slot_shift = to;
    } else {
      prefix |= (uint64_t)sh_digit << to;
      shift = to;
    }
    need -= sh_before;
    count = sh_count;
    if (by_slot && to == 0) break;                               // one token is left
  }
#pragma unroll
  for (int e = 0; e < rounds; ++e) {
    const int j = e * kSelThreads + tid;
    if (j >= n) continue;
    const uint64_t k = key_at(e, j);
    const bool in = shift == 64 || ((k >> shift) == (prefix >> shift) &&
                                    (slot_shift == 31 || ((uint32_t)j >> slot_shift) == (slot_prefix >> slot_shift)));
    if (in) {
      const uint32_t at = atomicAdd(&sh_n, 1u);                   // at most 64; their order does not matter
      if (at < 64) { cand_key[at] = k; cand_slot[at] = j; }
    }
  }
  __syncthreads();
  if (wave == 0) {
    const uint64_t mine = lane < (int)count ? cand_key[lane] : ~0ull;
    const int my_slot = lane < (int)count ? cand_slot[lane] : INT32_MAX;
    uint32_t rank = 0;
    for (int i = 0; i < (int)count; ++i) rank += cand_key[i] < mine || (cand_key[i] == mine && cand_slot[i] < my_slot);
    if (lane < (int)count && rank == need - 1) { sh_key = mine; sh_slot = my_slot; }
  }
  __syncthreads();
  // gone: up to this key and, among equal keys, up to this slot
  const uint64_t top = sh_key;
  const int top_slot = sh_slot;
  int4* moves = a.moves + (size_t)b * a.max_moves;
  // 0: stays where it is, 1: a hole, 2: moves
  const auto part_of = [&](uint64_t k, int j) {
    const bool gone = k < top || (k == top && j <= top_slot);
    return j >= n ? 0 : gone ? (j < keep ? 1 : 0) : (j >= keep ? 2 : 0);
  };
  const auto put = [&](int part, int j, uint32_t hole_at, uint32_t move_at) {
    if (part == 1 && hole_at < (uint32_t)a.max_moves) {
      moves[hole_at].z = j;
      moves[hole_at].w = page(j);
    }
    if (part == 2 && move_at < (uint32_t)a.max_moves) {
      moves[move_at].x = j;
      moves[move_at].y = page(j);
    }
  };
  const uint64_t below = (1ull << lane) - 1;
  uint32_t holes = 0;
  if (E) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = e * kSelThreads + tid, part = part_of(key[E ? e : 0], j);
      const uint64_t h = __ballot(part == 1), m = __ballot(part == 2);
      if (lane == 0) {
        ballots[0][e * kSelWaves + wave] = __popcll(h);
        ballots[1][e * kSelWaves + wave] = __popcll(m);
      }
    }
    __syncthreads();
    if (wave < 2) {                                              // running sums in the tokens' order, in place
      uint32_t base = 0;
      for (int i0 = 0; i0 < E * kSelWaves; i0 += 64) {
        const int i = i0 + lane;
        const uint32_t c = i < E * kSelWaves ? ballots[wave][i] : 0;
        uint32_t incl = c;
        for (int o = 1; o < 64; o <<= 1) {
          const uint32_t v = __shfl_up(incl, o, 64);
          if (lane >= o) incl += v;
        }
        if (i < E * kSelWaves) ballots[wave][i] = base + incl - c;
        base += __shfl(incl, 63, 64);
      }
      if (wave == 0 && lane == 0) sh_count = base;
    }
    __syncthreads();
    holes = sh_count;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = e * kSelThreads + tid, part = part_of(key[E ? e : 0], j);
      const uint64_t h = __ballot(part == 1), m = __ballot(part == 2);
      put(part, j, ballots[0][e * kSelWaves + wave] + __popcll(h & below), ballots[1][e * kSelWaves + wave] + __popcll(m & below));
    }
  } else {
    uint32_t movers = 0;
    for (int e = 0; e < rounds; ++e) {
      const int j = e * kSelThreads + tid, part = part_of(key_at(0, min(j, n - 1)), j);
      const uint64_t h = __ballot(part == 1), m = __ballot(part == 2);
      __syncthreads();
      if (lane == 0) { totals[wave] = __popcll(h); ballots[1][wave] = __popcll(m); }
      __syncthreads();
      uint32_t my_hole = holes + __popcll(h & below), my_move = movers + __popcll(m & below);
      for (int w = 0; w < kSelWaves; ++w) {
        const uint32_t ch = totals[w], cm = ballots[1][w];
        if (w < wave) { my_hole += ch; my_move += cm; }
        holes += ch;
        movers += cm;
      }
      put(part, j, my_hole, my_move);
    }
  }
  if (tid == 0) {
    a.length_out[b] = keep;
    a.counts[b] = (int)min(holes, (uint32_t)a.max_moves);        // as many holes as movers
  }
}

// moves keys and values, 16 bytes a lane, the vectors of one head's token on neighbouring lanes, and positions and weights; grid
// (pieces, n_seqs)
__global__ __launch_bounds__(256) void kv_evict_move_kernel(EvictArgs a, uint4* __restrict__ k, uint4* __restrict__ v,
                                                            int vec_shift) {
  const int b = blockIdx.y;
  const int n_moves = a.counts[b];
  const int4* moves = a.moves + (size_t)b * a.max_moves;
  const int mask = (1 << a.page_shift) - 1, per = a.n_kv << vec_shift;
  const int64_t total = (int64_t)n_moves * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int mv = (int)(i / per), r = (int)(i - (int64_t)mv * per);
    const int h = r >> vec_shift, c = r & ((1 << vec_shift) - 1);
    const int4 m = moves[mv];
    if (r == 0) {
      const size_t row = ((size_t)b * a.max_pages) << a.page_shift;
      a.pos[row + m.z] = a.pos[row + m.x];
      a.weight[row + m.z] = a.weight[row + m.x];
    }
    const size_t src = (((((size_t)m.y * a.n_kv + h) << a.page_shift) + (m.x & mask)) << vec_shift) + c;
    const size_t dst = (((((size_t)m.w * a.n_kv + h) << a.page_shift) + (m.z & mask)) << vec_shift) + c;
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
  LLMC_KERNEL_GGL(kv_append_kernel, flat_grid(((int64_t)bt->n_rows + 3) / 4), dim3(256), 0, st, a);
  LLMC_LAUNCH_CHECK("kv_append");
  return LLMC_OK;
}

// a sequence moves at most half of its tokens: as many as stay and as many as go
size_t kv_evict_ws_bytes(int n_seqs, int max_len) {
  return align_up((size_t)n_seqs * 4, 256) + (size_t)n_seqs * (max_len / 2 + 1) * sizeof(int4);
}

llmc_status_t launch_kv_evict(const llmc_kv_desc_t* kv, const llmc_kv_batch_t* bt, const int32_t* keep, int sink, int recent,
                              int32_t* length_out, void* ws, hipStream_t st) {
  EvictArgs a{};
  a.table = bt->d_table; a.length = bt->d_length;
  a.n_seqs = bt->n_seqs; a.max_pages = bt->max_pages; a.max_len = bt->max_len; a.n_pages = kv->n_pages;
  a.page_shift = log2_of(kv->page_size); a.n_kv = kv->n_kv_heads;
  a.pos = bt->d_pos; a.weight = bt->d_weight; a.keep = keep; a.sink = sink; a.recent = recent; a.length_out = length_out;
  a.counts = (int32_t*)ws;
  a.moves = (int4*)((char*)ws + align_up((size_t)bt->n_seqs * 4, 256));
  a.max_moves = bt->max_len / 2 + 1;
  { ProfScope ps_("kv_evict_select_kernel", st);
    const dim3 grid((unsigned)bt->n_seqs), block(kSelThreads);
    if (bt->max_len <= 2 * kSelThreads) LLMC_KERNEL_GGL(kv_evict_select_kernel<2>, grid, block, 0, st, a);
    else if (bt->max_len <= 8 * kSelThreads) LLMC_KERNEL_GGL(kv_evict_select_kernel<8>, grid, block, 0, st, a);
    else if (bt->max_len <= 24 * kSelThreads) LLMC_KERNEL_GGL(kv_evict_select_kernel<24>, grid, block, 0, st, a);
    else LLMC_KERNEL_GGL(kv_evict_select_kernel<0>, grid, block, 0, st, a); }
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
