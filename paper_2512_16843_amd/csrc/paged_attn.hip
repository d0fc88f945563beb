// Attention of new tokens over a paged key/value cache (one token of each sequence when decoding, a chunk of each when a
// prompt is read), and the attention weight that every cached token receives from them.
//
// Row m of a (sequence, key/value head) is new token m / G under query head m % G of the head's group of G, so the heads that
// share keys are rows of one product.  With x = <q, k> * scale, optionally capped (cap * tanh(x / cap)) and lowered with
// distance (slope_h * (pos_q - pos_k)), a row's output is sum_j p_j v_j, p = softmax of x over the keys that it sees: those
// not behind its own slot and, with a window, less than `window` positions away.  Softmax runs once over the keys with a
// running maximum and sum in fp32, in base 2.
//
// Both products are computed transposed, so that a lane holds ONE query column: S^T = K Q^T (A = keys, B = queries) and
// O^T += V^T P^T (A = values by head dimension, B = probabilities straight from the accumulators of S^T).  The key index of
// the second product is a free permutation, so the values are fetched in the order in which S^T delivers the keys.
#include <algorithm>
#include "paged.h"
#include "mma.h"
#include "gemm.h"

namespace llmc {
namespace {

typedef const __attribute__((address_space(4))) int32_t scalar_i32;    // read through the scalar cache
constexpr float kLog2e = 1.4426950408889634f;
// The maximum that a row's sums count from follows its scores only where they outgrow it by this much in base 2: weights up to
// 2^8 are as good as weights up to one in floating point, and most steps then rescale nothing.  (Where weights are rounded to bf16 the largest
// is then not exactly one: chunks in tiles 2.4e-4 from the exact result on average, 2.2e-4 without the slack, and 2 to 6 % slower: 16
// prompts of 1024 tokens 49.9 and 50.9 us, a chunk of 512 over 16384 tokens, 32 heads of 128, 200 and 208.)
constexpr float kSlack = 8.f;
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

struct AttnArgs {
  PagedArgs p;
  const void* q;               // [n_rows, H, DH], rows ld_q elements apart
  void* out;                   // [n_rows, H, DH], rows ld_out elements apart
  const void *k, *v;
  int64_t ld_q, ld_out;
  int32_t H, G;
  uint64_t g_magic, split_magic;   // row_magic of G and of split
  float softcap;
  float mul, add;              // a score in base 2 from a product (scale * log2(e), 0) or from what cap_scores makes of it
  float cap_in;                // scale / softcap; fast: times 2 log2(e)
  int32_t window;              // 0: none
  const float* slopes;
  const int32_t* pos;          // NULL: slots are positions
  int32_t split;               // keys of one piece of a long axis, a multiple of 128
  int32_t n_split;             // pieces that the grid provides for
  int32_t blocks;              // row blocks of all sequences, at most
  float* part_o;               // [n_rows * H, n_split, DH], not normalised
  float2* part_ml;             // [n_rows * H, n_split] (maximum in base 2, sum)
  float* lse;                  // [n_rows * H] log2 of the normaliser with the maximum in it, or NULL
  float* scores;               // [n_seqs, n_kv, join_rows, ld_scores] scores in base 2 of up to 16 rows a head, or NULL
  int32_t join_rows, ld_scores;
  int32_t by_length;           // the rows kernel takes the sequences by length
  int32_t by_level;            // row blocks of a sequence, at most, where the kernels take them level by level; else 0
};

__device__ __forceinline__ float max_over_groups(float v) {      // over the four groups of 16 lanes
  uint32_t a, b;
  butterfly_pair_u32<32>(__float_as_uint(v), a, b);
  v = fmaxf(__uint_as_float(a), __uint_as_float(b));
  butterfly_pair_u32<16>(__float_as_uint(v), a, b);
  return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ float sum_over_groups(float v) {
  uint32_t a, b;
  butterfly_pair_u32<32>(__float_as_uint(v), a, b);
  v = __uint_as_float(a) + __uint_as_float(b);
  butterfly_pair_u32<16>(__float_as_uint(v), a, b);
  return __uint_as_float(a) + __uint_as_float(b);
}

// r / d by row_magic(d), r >= 0: a short launch runs through its code once, from a cold cache, and a division is thirty instructions
__device__ __forceinline__ int div_by(int r, uint64_t magic) {
  return (int)(((uint64_t)(uint32_t)r * (uint32_t)(magic >> 32) + __umulhi((uint32_t)r, (uint32_t)magic)) >> 29);
}
__device__ __forceinline__ int token_of(const AttnArgs& a, int m) { return a.G == 1 ? m : div_by(m, a.g_magic); }

// the keys that rows [m0, m0 + rows) of a sequence's head can see: [lo, hi), lo a multiple of 64
struct KeyRange { int lo, hi; };
__device__ __forceinline__ KeyRange key_range(const AttnArgs& a, const SeqRange& s, int m0, int rows) {
  const int t0 = s.len - s.q + token_of(a, m0);                            // slot of the first row's token
  const int t1 = s.len - s.q + min(token_of(a, m0 + rows - 1), s.q - 1);
  KeyRange r;
  r.hi = max(t1 + 1, 0);
  // positions rise by one at least from slot to slot unless tokens were moved, so a slot `window` away is out of the window
  r.lo = (a.window > 0 && !a.pos) ? (int)max((int64_t)t0 - a.window + 1, (int64_t)0) & ~63 : 0;
  return r;
}

// Capped scores take the place of the products in the one fma of the exponent.
//   FAST, for the 128-row blocks whose weights are rounded to bf16: c + 2 c y with y = -1 / (1 + 2^(2 log2(e) x / c)), one exponential and
//   one reciprocal, exact at both ends; near zero it is off by 2^-23 c, far below that rounding for c up to 1024.  The normalisers
//   of weights that are accumulated in fp32 take it up to 64: 2^-17 at most, 2^-23 as the keys' errors average (a chunk capped at 30,
//   12 heads of 64: 45 us, 64 with the exact form).
//   Else, where memory is the bound or the result has 24 bits: c t with t = tanh(x / c) to the last bits, (1 - E) / (1 + E) with
//   E = 2^(-2 log2(e) |x| / c), and below 0.45 the power series, whose first term left out is 2 * 10^-8 of the sum there.
template <bool FAST, int N>
__device__ __forceinline__ void cap_scores(const AttnArgs& a, float (&y)[N]) {
  if constexpr (FAST) {
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(y[i] * a.cap_in));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float z = y[i] * a.cap_in, u = fabsf(z), q = u * u;
      const float e = __builtin_amdgcn_exp2f(u * (-2.f * kLog2e));
      const float big = (1.f - e) * __builtin_amdgcn_rcpf(1.f + e);
      float p = 21844.f / 6081075.f;
      p = fmaf(p, q, -1382.f / 155925.f);
      p = fmaf(p, q, 62.f / 2835.f);
      p = fmaf(p, q, -17.f / 315.f);
      p = fmaf(p, q, 2.f / 15.f);
      p = fmaf(p, q, -1.f / 3.f);
      y[i] = copysignf(u < 0.45f ? fmaf(u * q, p, u) : big, z);
    }
  }
}

// Scores in base 2 from N products, lowered by slope2 * away(i) and hidden at and beyond the window.  The branches are uniform
// and outside the loops.
template <int N, typename Away>
__device__ __forceinline__ void bias_scores(const AttnArgs& a, float (&x)[N], Away away, float slope2) {
  if (a.softcap > 0.f) cap_scores<false>(a, x);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = fmaf(-slope2, (float)away(i), fmaf(x[i], a.mul, a.add));
  if (a.window > 0) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (away(i) >= a.window) x[i] = -INFINITY;
  }
}

// a block of rows of a sequence and a piece of its keys
struct Item { int b, mb, piece; SeqRange s; };      // b < 0: nothing

// ---- rows that may have met a value which they do not see ------------------------------------------------------------------
// A row's sum is over the keys that it sees, but the value product multiplies every key of a step by a weight, zero where the key is
// hidden, and zero times an infinity or a NaN is no zero.  Where a row's output is not finite although its normaliser is, the values of
// the keys that are hidden from some row of the wavefront are looked at; if one of those is not finite, the row is summed again,
// over what it sees and nothing else.  That is far slower; where all is finite it costs the test of the outputs, which no time
// shows.  (An infinity in the first token of each of 16 prompts of 1024 tokens, 12 heads of 64, 48 us without it: 61 us this way, 5 ms if
// every row that sees it were summed again.)

// whether a value of a key hidden from some of the rows with slots t_first to t_last is not finite, of keys [lo, hi) and those behind
// that share their last step
template <typename T, int DH>
__device__ __forceinline__ bool hides_odd_values(const AttnArgs& a, const Item& it, int h, int t_first, int t_last, int lo, int hi) {
  constexpr int PER = DH / Vec16<T>::N;                          // 16-byte vectors of a key
  hi = min(it.s.len, lo + ((hi - lo + 63) & ~63));
  const int from = max(lo, t_first + 1);                         // hidden from here on, and up to here
  const int upto = a.window <= 0 ? lo : a.pos ? hi : (int)min((int64_t)hi, (int64_t)t_last - a.window + 1);
  const int lane = threadIdx.x & 63;
  bool any = false;
#pragma unroll 1
  for (int key = (upto > lo ? lo : from) + lane / PER; key < hi; key += 64 / PER) {
    const int page = key < from && key >= upto ? -1 : page_of(a.p, it.b, key);
    if (page < 0) continue;
    float v[Vec16<T>::N];
    Vec16<T>::load((const T*)a.v + ((((size_t)page * a.p.n_kv + h) << a.p.page_shift) + (key & ((1 << a.p.page_shift) - 1))) * DH +
                       lane % PER * Vec16<T>::N, v);
#pragma unroll
    for (int e = 0; e < Vec16<T>::N; ++e) any |= !(fabsf(v[e]) < INFINITY);
  }
  return __any(any) != 0;
}

// A row's sum over what it sees: a lane a key for the scores and a lane a dim for the values.  m: the row of the head; ref: what its
// weights count from; keys: `width` from first, every `step`, up to hi; the DH sums go to part, or times scale to out.  FAST: see cap_scores.
template <typename T, int DH, bool FAST>
__device__ __forceinline__ void sum_seen(const AttnArgs& a, const Item& it, int h, int m, float ref, int first, int hi, int step,
                                         int width, float* part, T* out, float scale) {
  constexpr int N = DH / 64;
  const int lane = threadIdx.x & 63, i = token_of(a, m), head = h * a.G + m - i * a.G, t = it.s.len - it.s.q + i;
  const T* q = (const T*)a.q + (size_t)(it.s.first + i) * a.ld_q + head * DH;
  const size_t seq = ((size_t)it.b * a.p.max_pages) << a.p.page_shift;
  const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.f;
  const int t_pos = a.pos && t >= 0 ? a.pos[seq + t] : t;
  const auto place = [&](int page, int key) {
    return ((((size_t)page * a.p.n_kv + h) << a.p.page_shift) + (key & ((1 << a.p.page_shift) - 1))) * DH;
  };
  float o[N] = {};
  for (int kb = first; kb < hi; kb += step) {
    const int key = kb + lane;
    const int page = lane < width && key < hi && key <= t ? page_of(a.p, it.b, key) : -1;
    int away = 0;
    float x[1] = {0.f};
    if (page >= 0) {
      const T* k = (const T*)a.k + place(page, key);
#pragma unroll 2
      for (int d = 0; d < DH; d += Vec16<T>::N) {
        float qd[Vec16<T>::N], kd[Vec16<T>::N];
        Vec16<T>::load(q + d, qd);
        Vec16<T>::load(k + d, kd);
#pragma unroll
        for (int e = 0; e < Vec16<T>::N; ++e) x[0] = fmaf(qd[e], kd[e], x[0]);
      }
      away = t_pos - (a.pos ? a.pos[seq + key] : key);
    }
    if constexpr (FAST) {
      if (a.softcap > 0.f) cap_scores<true>(a, x);
      x[0] = fmaf(x[0], a.mul, a.add);
    } else {
      bias_scores(a, x, [&](int) { return away; }, slope2);
    }
    const float w = __builtin_amdgcn_exp2f(x[0] - ref);
    const uint64_t seen = __ballot(page >= 0 && !(a.window > 0 && away >= a.window));
#pragma unroll 2
    for (int l = 0; l < width; ++l) {                            // the loads of hidden keys are of some page, and not used
      const float wl = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), l));
      const T* v = (const T*)a.v + place(max(__builtin_amdgcn_readlane(page, l), 0), kb + l);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float ve = Elem<T>::load(v + e * 64 + lane);
        o[e] = seen >> l & 1 ? fmaf(wl, ve, o[e]) : o[e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (part) part[e * 64 + lane] = o[e];
    else Elem<T>::store(out + e * 64 + lane, o[e] * scale);
  }
}

// ---- pieces of the products for the two element types, 16 query columns a wavefront -----------------------------------
template <typename T, int DH> struct Frag;

template <int DH> struct Frag<bf16_t, DH> {
  static constexpr int KEYS = 32, SUB = 2, NV = DH / 16;       // keys a step, 16-key products, output tiles of 16 dims
  typedef uint16_t E;
  struct Q { bf16x8_t v[DH / 32]; };
  struct K { bf16x8_t v[SUB][DH / 32]; };
  struct V { uint32_t w[8][NV / 2]; };                          // keys 4 g + r and 16 + 4 g + r, NV consecutive dims
  static __device__ __forceinline__ void load_q(Q& q, const E* row, int g) {
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) q.v[i] = *reinterpret_cast<const bf16x8_t*>(row + i * 32 + g * 8);
  }
  static __device__ __forceinline__ void load_k(K& k, int u, const E* tile, int c, int g) {   // tile: 16 keys of one page
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) k.v[u][i] = *reinterpret_cast<const bf16x8_t*>(tile + c * DH + i * 32 + g * 8);
  }
  static __device__ __forceinline__ void load_v(V& v, int u, const E* tile, int c, int g) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const E* p = tile + (4 * g + r) * DH + c * NV;
      if constexpr (NV == 4) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        v.w[u * 4 + r][0] = x.x; v.w[u * 4 + r][1] = x.y;
      } else {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        v.w[u * 4 + r][0] = x.x; v.w[u * 4 + r][1] = x.y; v.w[u * 4 + r][2] = x.z; v.w[u * 4 + r][3] = x.w;
      }
    }
  }
  static __device__ __forceinline__ void clear_v(V& v, int u, int r) {
#pragma unroll
    for (int i = 0; i < NV / 2; ++i) v.w[u * 4 + r][i] = 0;
  }
  static __device__ __forceinline__ f32x4_t qk(const K& k, int u, const Q& q, float from = 0.f) {
    f32x4_t s = {from, from, from, from};
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.v[u][i], q.v[i], s, 0, 0, 0);
    return s;
  }
  // A weight goes in as two bf16 numbers, itself rounded and what that left: off by 2^-16 of itself, where one number would be off
  // by 2^-8 and would be most of an output's error (one sequence of 777 tokens, 12 heads of 64: 2.1e-4 from the exact result on average
  // with one number, 1.5e-4 with one and kSlack = 0, 1.23e-4 with two, which is what the output's own rounding leaves).  The second product costs
  // nothing where memory is the bound: 43.8 us for 43.7 with one (64 sequences of up to 2048), 7.3 for 7.2 (the one of 777).
  static __device__ __forceinline__ void pv(const V& v, const float (&p)[SUB][4], f32x4_t (&o)[NV]) {
    union Weights { uint32_t u[4]; bf16x8_t v; } b, rest;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float p0 = p[u][2 * i], p1 = p[u][2 * i + 1];
        const uint32_t w = f32x2_to_bf16x2(p0, p1);
        b.u[2 * u + i] = w;
        rest.u[2 * u + i] = f32x2_to_bf16x2(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xFFFF0000u));
      }
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      union { uint32_t u[4]; bf16x8_t v; } x;
      const uint32_t sel = (t & 1) ? 0x07060302u : 0x05040100u;      // the high or the low halves of two keys' words
#pragma unroll
      for (int i = 0; i < 4; ++i) x.u[i] = __builtin_amdgcn_perm(v.w[2 * i + 1][t >> 1], v.w[2 * i][t >> 1], sel);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, rest.v, o[t], 0, 0, 0);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, b.v, o[t], 0, 0, 0);
    }
  }
};

template <int DH> struct Frag<float, DH> {
  static constexpr int KEYS = 16, SUB = 1, NV = DH / 16;
  typedef float E;
  struct Q { f32x4_t v[DH / 16]; };
  struct K { f32x4_t v[SUB][DH / 16]; };
  struct V { f32x4_t w[4][NV / 4]; };
  static __device__ __forceinline__ void load_q(Q& q, const E* row, int g) {
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) q.v[i] = *reinterpret_cast<const f32x4_t*>(row + i * 16 + g * 4);
  }
  static __device__ __forceinline__ void load_k(K& k, int u, const E* tile, int c, int g) {
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) k.v[u][i] = *reinterpret_cast<const f32x4_t*>(tile + c * DH + i * 16 + g * 4);
  }
  static __device__ __forceinline__ void load_v(V& v, int, const E* tile, int c, int g) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NV / 4; ++i)
        v.w[r][i] = *reinterpret_cast<const f32x4_t*>(tile + (4 * g + r) * DH + c * NV + i * 4);
  }
  static __device__ __forceinline__ void clear_v(V& v, int, int r) {
#pragma unroll
    for (int i = 0; i < NV / 4; ++i) v.w[r][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  static __device__ __forceinline__ f32x4_t qk(const K& k, int u, const Q& q, float from = 0.f) {
    f32x4_t s = {from, from, from, from};
#pragma unroll
    for (int i = 0; i < DH / 16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k.v[u][i][j], q.v[i][j], s, 0, 0, 0);
    return s;
  }
  static __device__ __forceinline__ void pv(const V& v, const float (&p)[SUB][4], f32x4_t (&o)[NV]) {
#pragma unroll
    for (int t = 0; t < NV; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.w[r][t >> 2][t & 3], p[0][r], o[t], 0, 0, 0);
  }
};

template <typename T, int N> __device__ __forceinline__ void store_vec(T* p, const float* x);
template <> __device__ __forceinline__ void store_vec<float, 4>(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
template <> __device__ __forceinline__ void store_vec<float, 8>(float* p, const float* x) {
  store_vec<float, 4>(p, x);
  store_vec<float, 4>(p + 4, x + 4);
}
template <> __device__ __forceinline__ void store_vec<bf16_t, 4>(bf16_t* p, const float* x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]));
}
template <> __device__ __forceinline__ void store_vec<bf16_t, 8>(bf16_t* p, const float* x) { Vec16<bf16_t>::store(p, x); }

// v of all lanes up to this one added up
__device__ __forceinline__ int sum_up_to_lane(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);            // from 1, 2, 4, 8 lanes below within 16, then the last of
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);            // the 16, of the 32 before
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

// the pieces that the keys of rows [m0, m0 + rows) are cut into, as every kernel counts them
__device__ __forceinline__ int pieces_of(const AttnArgs& a, const KeyRange& kr) {
  return max(1, div_by(max(kr.hi - kr.lo, 0) + a.split - 1, a.split_magic));
}

// What the idx-th workgroups of a launch (one a head) work on: a block of ROWS rows of a sequence, and a piece of its keys.  A later
// block of a chunk sees more keys, so the last blocks of all sequences come first, then those before them (16 prompts of 1024
// tokens, 12 heads: 61.7 us sequence by sequence, 51 in this order); the pieces of a level are numbered without gaps.
// Workgroups are dealt to compute units in turn, whatever they have to do, and idle ones in between leave the work uneven
// (4 ragged fp32 chunks of 256 tokens over 1024, 12 heads: 33 us with gaps, 28 without; 16 of up to 300 over 4000 in bf16: 60 and
// 46).  That takes a step a level and lanes for all sequences; larger calls go sequence by sequence from the end, 64 a step.
template <int ROWS>
__device__ __forceinline__ Item item_of(const AttnArgs& a, int idx) {
  const int lane = threadIdx.x & 63;
  const Item none = {-1, 0, 0, {0, 0, 0}};
  if (a.by_level) {
    SeqRange s = {0, 0, 0};
    if (lane < a.p.n_seqs) s = seq_range(a.p, lane);
    const int n = (s.q * a.G + ROWS - 1) / ROWS;
    for (int level = a.by_level - 1; level >= 0; --level) {
      int count = n > level;
      if (a.n_split > 1 && n > level) count = pieces_of(a, key_range(a, s, level * ROWS, ROWS));
      const int upto = sum_up_to_lane(count), total = __builtin_amdgcn_readlane(upto, 63);
      if (idx < total) {
        const int l = (int)__builtin_ctzll(__ballot(upto > idx));
        return Item{l, level, idx - __builtin_amdgcn_readlane(upto, l) + __builtin_amdgcn_readlane(count, l),
                    {__builtin_amdgcn_readlane(s.len, l), __builtin_amdgcn_readlane(s.first, l), __builtin_amdgcn_readlane(s.q, l)}};
      }
      idx -= total;
    }
    return none;
  }
  const int at = idx / a.n_split, piece = idx - at * a.n_split, blk = a.blocks - 1 - at;
  if (blk < 0) return none;
  if (!a.p.new_start) {
    const int per = (a.G + ROWS - 1) / ROWS, b = blk / per;
    return b < a.p.n_seqs ? Item{b, blk - b * per, piece, seq_range(a.p, b)} : none;
  }
  int before = 0;
  for (int i = 0; i < a.p.n_seqs; i += 64) {
    const int b = i + lane;
    const int n = b < a.p.n_seqs ? (seq_range(a.p, b).q * a.G + ROWS - 1) / ROWS : 0;
    const int upto = before + sum_up_to_lane(n);
    const uint64_t hit = __ballot(upto > blk);
    if (hit) {
      const int l = (int)__builtin_ctzll(hit);
      return Item{i + l, blk - __builtin_amdgcn_readlane(upto, l) + __builtin_amdgcn_readlane(n, l), piece, seq_range(a.p, i + l)};
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return none;
}

// The n-th sequence when each group of 64 is ordered by length, longest first.  In the order of the batch, lengths may repeat with the period
// in which workgroups come back to a compute unit (64 sequences of up to 2048 tokens, 12 heads: 50 us, 42 in order).  Pieces of a
// long axis are better mixed (6 sequences of up to 32768, 8 heads of 128: 91 us, 100 in order).
__device__ __forceinline__ int nth_longest(const PagedArgs& p, int n) {
  const int lane = threadIdx.x & 63, first = n & ~63;
  const int len = first + lane < p.n_seqs ? max(p.length[first + lane], 0) : -1;
  int rank = 0;
#pragma unroll 8
  for (int k = 0; k < 64; ++k) {
    const int other = __builtin_amdgcn_readlane(len, k);
    rank += other > len || (other == len && k < lane);
  }
  return first + __builtin_ctzll(__ballot(rank == n - first));
}

// ---- few rows, or fp32: keys straight from memory to registers ----------------------------------------------------------
// A wavefront owns 16 rows and walks the keys in steps of 32 (bf16) or 16 (fp32), the next step's keys and values in flight
// while it works on this one's.  ROWSPLIT 0: the four wavefronts of a workgroup take the same 16 rows and every fourth step, and
// join their maxima, sums and outputs in LDS: a single token's keys are read once.  (8 wavefronts a workgroup gain where all
// sequences are long and lose elsewhere, and the host does not know the lengths: 12 heads of 64, 64 sequences of up to 2048 tokens 40.8 us
// for 43.5, 256 of up to 300 45 for 31.)
// ROWSPLIT 1: they take 64 rows and the same steps.
// FEAT 0: plain scores, 1: capped, biased or in a window, 2: the same with positions that are not the slots' numbers.
template <typename T, int DH, int FEAT, bool ROWSPLIT>
__global__ __launch_bounds__(256) void attention_paged_rows_kernel(AttnArgs a) {
  typedef Frag<T, DH> F;
  typedef typename F::E E;
  constexpr int NW = 4, NV = F::NV, SUB = F::SUB, KEYS = F::KEYS, ROWS = ROWSPLIT ? 16 * NW : 16, LDO = DH + 4;
  constexpr int STEP = ROWSPLIT ? KEYS : NW * KEYS;
  extern __shared__ __attribute__((aligned(16))) float rows_lds[];          // ROWSPLIT 0: [NW][join_rows][LDO], then maxima, sums
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int h = blockIdx.x, idx = blockIdx.y + blockIdx.z * gridDim.y;
  Item rb;
  if (ROWSPLIT || a.n_split > 1) {
    rb = item_of<ROWS>(a, idx);
    if (rb.b < 0) return;
  } else {
    if (idx >= a.p.n_seqs) return;
    rb.b = a.by_length ? nth_longest(a.p, idx) : idx;
    rb.mb = rb.piece = 0;
    rb.s = seq_range(a.p, rb.b);
  }
  const int piece = rb.piece;
  const SeqRange s = rb.s;
  const int rows = s.q * a.G;
  if (rb.mb * ROWS >= rows) return;
  const KeyRange kr = key_range(a, s, rb.mb * ROWS, ROWS);
  const int n_pieces = pieces_of(a, kr);
  if (piece >= n_pieces) return;
  const int k_lo = kr.lo + piece * a.split;
  int k_hi = min(kr.hi, k_lo + a.split);
  const int m0 = rb.mb * ROWS + (ROWSPLIT ? wave * 16 : 0);
  const int m = m0 + c;                                         // this lane's column
  const bool row_there = m < rows;
  const int mc = min(m, rows - 1), i_new = token_of(a, mc), head = h * a.G + mc - i_new * a.G;
  const int row = s.first + i_new, t_slot = s.len - s.q + i_new;
  const int t_first = s.len - s.q + token_of(a, m0);                   // the first row's slot: all rows see the keys up to it
  if (ROWSPLIT) k_hi = min(k_hi, max(0, s.len - s.q + min(token_of(a, m0 + 15), s.q - 1) + 1));
  const int slots = a.p.max_pages << a.p.page_shift;
  const int32_t* pos = FEAT == 2 ? a.pos + (size_t)rb.b * slots : nullptr;
  float slope = 0.f;
  int t_pos = t_slot;
  if (FEAT) {
    if (a.slopes) slope = a.slopes[head] * kLog2e;
    if (FEAT == 2 && t_slot >= 0) t_pos = pos[t_slot];
  }
  typename F::Q fq;
  F::load_q(fq, (const E*)a.q + (size_t)row * a.ld_q + head * DH, g);
  f32x4_t o[NV];
#pragma unroll
  for (int t = 0; t < NV; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;
  const int page_mask = (1 << a.p.page_shift) - 1;
  // scores of these rows, for the weights that the keys receive
  float* score = a.scores && row_there ? a.scores + (((size_t)rb.b * a.p.n_kv + h) * a.join_rows + mc) * a.ld_scores + 4 * g : nullptr;

  // A step's keys and values.  The next step's keys are asked for as soon as the scores have consumed this one's, the values after
  // the value product, into the same registers: one copy of the code (a second buffer, or a third, gains nothing where memory is
  // the bound, and a longer code costs short calls).  Pages are scalar loads, so waiting for them waits for no other load in flight; they
  // are asked for a step earlier than the keys.  Beyond the last step the last one is read again (a conditional load would have
  // to be waited for together with what is in flight).
  struct Step {
    typename F::K k;
    typename F::V v;
    int4 pos[SUB];
    int k_page[SUB], v_page[SUB];
  };
  scalar_i32* table = (scalar_i32*)(uintptr_t)(a.p.table + (size_t)rb.b * a.p.max_pages);
  const int k_first = k_lo + (ROWSPLIT ? 0 : wave * KEYS);
  const int k_last = k_first + max(0, k_hi - 1 - k_first) / STEP * STEP;     // this wavefront's last step
  int page_next[SUB];
  auto ask_pages = [&](int kb) {
#pragma unroll
    for (int u = 0; u < SUB; ++u)
      page_next[u] = table[min((min(kb, k_last) + 16 * u) >> a.p.page_shift, a.p.max_pages - 1)];
  };
  auto place = [&](int page, int key) {
    return ((((size_t)max(page, 0) * a.p.n_kv + h) << a.p.page_shift) + (key & page_mask)) * DH;
  };
  auto fetch_k = [&](Step& st, int kb) {
    kb = min(kb, k_last);
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      st.k_page[u] = (uint32_t)page_next[u] < (uint32_t)a.p.n_pages ? page_next[u] : -1;
      F::load_k(st.k, u, (const E*)a.k + place(st.k_page[u], kb + 16 * u), c, g);
      if (FEAT == 2) st.pos[u] = reinterpret_cast<const int4*>(pos)[min(kb + 16 * u + 4 * g, slots - 4) >> 2];
    }
  };
  auto fetch_v = [&](Step& st, int kb) {
    kb = min(kb, k_last);
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      st.v_page[u] = st.k_page[u];
      F::load_v(st.v, u, (const E*)a.v + place(st.v_page[u], kb + 16 * u), c, g);
    }
  };
  if (k_first < k_hi) {
    Step st;
    ask_pages(k_first);
    fetch_k(st, k_first);
    fetch_v(st, k_first);
    ask_pages(k_first + STEP);
    for (int kb = k_first; kb < k_hi; kb += STEP) {
    float x[SUB * 4];
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      const f32x4_t sc = F::qk(st.k, u, fq);
#pragma unroll
      for (int r = 0; r < 4; ++r) x[u * 4 + r] = sc[r];
    }
    bool edge = kb + KEYS - 1 > t_first || kb + KEYS > s.len;
#pragma unroll
    for (int u = 0; u < SUB; ++u) edge |= st.v_page[u] < 0;
    int key_pos[8];
    if (FEAT == 2) {
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        key_pos[u * 4] = st.pos[u].x; key_pos[u * 4 + 1] = st.pos[u].y; key_pos[u * 4 + 2] = st.pos[u].z; key_pos[u * 4 + 3] = st.pos[u].w;
      }
    }
    fetch_k(st, kb + STEP);
    ask_pages(kb + 2 * STEP);
    if (FEAT == 2) {
      bias_scores(a, x, [&](int i) { return t_pos - key_pos[i]; }, slope);
    } else if (FEAT == 1) {
      const int away0 = t_slot - kb - 4 * g;
      bias_scores(a, x, [&](int i) { return away0 - 16 * (i >> 2) - (i & 3); }, slope);
    } else {
#pragma unroll
      for (int i = 0; i < SUB * 4; ++i) x[i] *= a.mul;
    }
    if (edge) {
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = kb + 16 * u + 4 * g + r;
          if (key > t_slot || st.v_page[u] < 0) x[u * 4 + r] = -INFINITY;
          // what lies behind the sequence in its last page may be anything, and 0 * anything is not always 0
          if (key >= s.len || st.v_page[u] < 0) F::clear_v(st.v, u, r);
        }
    }
    if (!ROWSPLIT && score) {
#pragma unroll
      for (int u = 0; u < SUB; ++u)
        if (kb + 16 * u < k_hi)
          *reinterpret_cast<float4*>(score + kb + 16 * u) = make_float4(x[u * 4], x[u * 4 + 1], x[u * 4 + 2], x[u * 4 + 3]);
    }
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < SUB * 4; ++i) mx = fmaxf(mx, x[i]);
    const float m_new = max_over_groups(mx);
    if (__any(m_new > m_run + kSlack)) {
      const float m_top = fmaxf(m_run, m_new), corr = m_top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_top);
      m_run = m_top;
      l_run *= corr;
#pragma unroll
      for (int t = 0; t < NV; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[t][r] *= corr;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;        // a row that has seen no key so far
    float pr[SUB][4];
#pragma unroll
    for (int i = 0; i < SUB * 4; ++i) {
      pr[i >> 2][i & 3] = __builtin_amdgcn_exp2f(x[i] - m_use);
      l_run += pr[i >> 2][i & 3];
    }
    F::pv(st.v, pr, o);
    fetch_v(st, kb + STEP);
    }
  }
  l_run = sum_over_groups(l_run);

  // lane: column c, dims (4 g + r) * NV + t
  const int R = a.join_rows;                                     // at least as many as this block has
  float* sM = rows_lds + NW * R * LDO;
  float* sL = sM + NW * R;
  const bool whole = ROWSPLIT && n_pieces == 1;
  const size_t rh = (size_t)row * a.H + head;
  const float scale = !whole ? 1.f : l_run > 0.f ? 1.f / l_run : (l_run == 0.f ? 0.f : l_run);
  float zero = 0.f;                                              // or NaN
#pragma unroll
  for (int t = 0; t < NV; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) zero = fmaf(o[t][r], 0.f, zero);
  const uint64_t odd = __ballot(zero != 0.f && l_run < INFINITY && row_there);
  uint32_t again = (uint32_t)(odd | odd >> 16 | odd >> 32 | odd >> 48) & 0xFFFFu;    // a bit a column
  // (bf16 has two parts of a weight, of any sign or none, and is not right about an infinity that a row does see)
  if (__builtin_expect(again != 0, 0) && sizeof(T) == 4 &&
      !hides_odd_values<T, DH>(a, rb, h, t_first, s.len - s.q + min(token_of(a, m0 + 15), s.q - 1), k_lo, k_hi))
    again = 0;
  if (ROWSPLIT ? row_there : c < R) {
    if (!(again >> c & 1)) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float y[NV];
#pragma unroll
        for (int t = 0; t < NV; ++t) y[t] = o[t][r] * scale;
        if (whole) store_vec<T, NV>((T*)a.out + (size_t)row * a.ld_out + head * DH + (4 * g + r) * NV, y);
        else if (ROWSPLIT) store_vec<float, NV>(a.part_o + (rh * a.n_split + piece) * DH + (4 * g + r) * NV, y);
        else store_vec<float, NV>(&rows_lds[(wave * R + c) * LDO + (4 * g + r) * NV], y);
      }
    }
    if (g == 0) {
      if (!ROWSPLIT) { sM[wave * R + c] = m_run; sL[wave * R + c] = l_run; }
      else if (!whole) a.part_ml[rh * a.n_split + piece] = make_float2(m_run, l_run);
      else if (a.lse) a.lse[rh] = l_run == 0.f ? INFINITY : m_run + __builtin_amdgcn_logf(l_run);
    }
  }
  for (; __builtin_expect(again != 0, 0); again &= again - 1) {
    const int col = __builtin_ctz(again), mr = m0 + col;
    const auto of_row = [&](float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), col)); };
    const float ref = of_row(m_run) == -INFINITY ? 0.f : of_row(m_run), sc = of_row(scale);
    const int i = token_of(a, mr), r = s.first + i, hd = h * a.G + mr - i * a.G;
    float* part = whole ? nullptr : ROWSPLIT ? a.part_o + (((size_t)r * a.H + hd) * a.n_split + piece) * DH : rows_lds + (wave * R + col) * LDO;
    sum_seen<T, DH, false>(a, rb, h, mr, ref, k_first, k_hi, STEP, KEYS, part, (T*)a.out + (size_t)r * a.ld_out + hd * DH, sc);
  }
  if (ROWSPLIT) return;
  __syncthreads();
  // joined by a thread a row and dim
  for (int e = threadIdx.x; e < rows * DH; e += NW * 64) {
    const int jr = e / DH, jd = e % DH;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, sM[w * R + jr]);
    const float top_use = top == -INFINITY ? 0.f : top;
    float l = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(sM[w * R + jr] - top_use);
      l += f * sL[w * R + jr];
      y += f * rows_lds[(w * R + jr) * LDO + jd];
    }
    const int ji = token_of(a, jr), jrow = s.first + ji, jhead = h * a.G + jr - ji * a.G;
    const size_t rh = (size_t)jrow * a.H + jhead;
    if (n_pieces == 1) {
      Elem<T>::store((T*)a.out + (size_t)jrow * a.ld_out + jhead * DH + jd, y * (l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l)));
      if (a.lse && jd == 0) a.lse[rh] = l == 0.f ? INFINITY : top + __builtin_amdgcn_logf(l);
    } else {
      a.part_o[(rh * a.n_split + piece) * DH + jd] = y;
      if (jd == 0) a.part_ml[rh * a.n_split + piece] = make_float2(top, l);
    }
  }
}

// ---- the pieces of a long axis joined: a workgroup a (row, head), its wavefronts a quarter of the pieces each -------------
template <typename T, int DH>
__device__ __forceinline__ void join_pieces(const AttnArgs& a, int row, int head, int n) {
  // 16 bytes a lane: a wavefront takes 256 / DH pieces a step
  constexpr int L = DH / 4, STEP = 64 / L;
  __shared__ float4 part_y[3][L];
  __shared__ float part_l[3];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = lane / L, dim = lane % L * 4;
  const size_t rh = (size_t)row * a.H + head;
  const float2* ml = a.part_ml + rh * a.n_split;
  const float* po = a.part_o + rh * a.n_split * DH;
  float top = -INFINITY;
  for (int j = lane; j < n; j += 64) top = fmaxf(top, ml[j].x);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float top_use = top == -INFINITY ? 0.f : top;
  float l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int j = wave * STEP + sub; j < n; j += 4 * STEP) {
    const float2 v = ml[j];
    const float4 p = *reinterpret_cast<const float4*>(po + (size_t)j * DH + dim);
    const float f = __builtin_amdgcn_exp2f(v.x - top_use);
    l += f * v.y;
    y[0] += f * p.x; y[1] += f * p.y; y[2] += f * p.z; y[3] += f * p.w;
  }
#pragma unroll
  for (int o = 32; o >= L; o >>= 1) {
    l += __shfl_xor(l, o, 64);
#pragma unroll
    for (int t = 0; t < 4; ++t) y[t] += __shfl_xor(y[t], o, 64);
  }
  if (wave > 0 && sub == 0) {
    part_y[wave - 1][lane] = make_float4(y[0], y[1], y[2], y[3]);
    if (lane == 0) part_l[wave - 1] = l;
  }
  __syncthreads();
  if (wave > 0 || sub > 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const float4 v = part_y[w][lane];
    l += part_l[w];
    y[0] += v.x; y[1] += v.y; y[2] += v.z; y[3] += v.w;
  }
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
#pragma unroll
  for (int t = 0; t < 4; ++t) y[t] *= inv;
  store_vec<T, 4>((T*)a.out + (size_t)row * a.ld_out + head * DH + dim, y);
  if (a.lse && lane == 0) a.lse[rh] = l == 0.f ? INFINITY : top + __builtin_amdgcn_logf(l);
}

// one token of each sequence, or few: grid (heads, rows)
template <typename T, int DH>
__global__ __launch_bounds__(256) void attention_paged_join_kernel(AttnArgs a) {
  const int head = blockIdx.x, row = blockIdx.y + blockIdx.z * gridDim.y;
  if (row >= a.p.n_rows) return;
  const int b = seq_of_row(a.p, row);
  if (b < 0) return;
  const SeqRange s = seq_range(a.p, b);
  if ((uint32_t)(row - s.first) >= (uint32_t)s.q) return;
  const KeyRange kr = key_range(a, s, 0, 16);
  const int n = pieces_of(a, kr);
  if (n > 1) join_pieces<T, DH>(a, row, head, n);               // else written where it was computed
}

// many rows of few pieces: a wavefront takes 256 / DH heads of a row, DH / 4 lanes each (24576 rows and heads of two pieces: 10.4 us
// with a wavefront each, 5.7 so)
template <typename T, int DH, int ROWS>
__global__ __launch_bounds__(256) void attention_paged_join_rows_kernel(AttnArgs a) {
  constexpr int L = DH / 4, HEADS = 64 / L;
  const int lane = threadIdx.x & 63, dim = lane % L * 4;
  const uint32_t idx = flat_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), per_row = (a.H + HEADS - 1) / HEADS;
  if (idx / per_row >= (uint32_t)a.p.n_rows) return;
  const int row = idx / per_row, head = (idx - row * per_row) * HEADS + lane / L;
  const int b = seq_of_row(a.p, row);
  if (b < 0) return;
  const SeqRange s = seq_range(a.p, b);
  const int i = row - s.first;
  if ((uint32_t)i >= (uint32_t)s.q || head >= a.H) return;
  const int h = token_of(a, head), m = i * a.G + head - h * a.G;
  const KeyRange kr = key_range(a, s, m / ROWS * ROWS, ROWS);
  const int n = pieces_of(a, kr);
  if (n <= 1) return;
  const size_t rh = (size_t)row * a.H + head;
  const float2* ml = a.part_ml + rh * a.n_split;
  const float* po = a.part_o + rh * a.n_split * DH + dim;
  float top = -INFINITY, l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < n; ++j) top = fmaxf(top, ml[j].x);
  const float top_use = top == -INFINITY ? 0.f : top;
#pragma unroll 4
  for (int j = 0; j < n; ++j) {
    const float2 v = ml[j];
    const float4 p = *reinterpret_cast<const float4*>(po + (size_t)j * DH);
    const float f = __builtin_amdgcn_exp2f(v.x - top_use);
    l += f * v.y;
    y[0] += f * p.x; y[1] += f * p.y; y[2] += f * p.z; y[3] += f * p.w;
  }
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
#pragma unroll
  for (int t = 0; t < 4; ++t) y[t] *= inv;
  store_vec<T, 4>((T*)a.out + (size_t)row * a.ld_out + head * DH + dim, y);
  if (a.lse && dim == 0) a.lse[rh] = l == 0.f ? INFINITY : top + __builtin_amdgcn_logf(l);
}

// ---- many rows in bf16: 128 rows a workgroup share key tiles in LDS -----------------------------------------------------
// Four wavefronts of 32 rows; tiles of 64 keys and values, double buffered, filled by direct global -> LDS loads.  Each
// wavefront fetches 16 rows of a tile: rows of one page, so its page is a scalar, loaded a tile ahead through the scalar cache (whose
// loads are waited for apart from the tiles in flight).  Values stay as they lie in memory and are transposed by the LDS's
// transposing reads (a group of 16 lanes gets 4 keys of 16 dims, 4 keys a lane).  The 16-byte chunks of a row are XOR-swizzled by
// the row, on the global side: 16 consecutive rows then offer one chunk in 16 places (the keys' 16-byte reads), and four
// consecutive rows four neighbouring chunks in 4 different quarters of the banks (the values' transposing reads).
// The score products run at a raised priority (one chunk of 512 over 16384 tokens, 32 heads of 128: 166 -> 154 us; the value
// products too: 165).
// FEAT 0: plain or (FAST) capped scores, with or without a window; 1: bias by distance, or exact capping; 2: positions that are not
// the slots' numbers.
template <int DH>
struct TileCfg {
  static constexpr int KT = 64, ROWS = 128;
  static constexpr int CH = DH / 8;                               // 16-byte chunks of a row
  static constexpr int RPI = 64 / CH;                             // rows that one load instruction of a wavefront fills
  static constexpr int NI = 16 / RPI;                             // load instructions of a wavefront, for K and for V
  static constexpr int TILE = KT * DH;                            // elements
  static constexpr int POS = 2 * 2 * TILE;                      // the tiles' positions follow, then a word a wavefront
  static constexpr size_t LDS_BYTES = POS * 2 + 2 * KT * 4 + 16;           // 33 and 65 KiB: four and two workgroups a compute unit
  // place of chunk c of row r: c ^ swz(r)
  static __device__ __forceinline__ int swz(int r) {
    if (DH == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    return (((r >> 1) & 1) << 2) | (((r >> 2) & 1) << 1) | ((r >> 3) & 1);
  }
};

typedef short v4s16_t __attribute__((ext_vector_type(4)));
// (`restrict` gives the read alias information once inlined.  Without any, the compiler takes it to depend on every direct
// global -> LDS load in flight and waits for the next tile here.)
typedef __attribute__((address_space(3))) v4s16_t lds_v4s16_t;
__device__ __forceinline__ v4s16_t lds_read_tr(lds_v4s16_t* __restrict__ p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }
__device__ __forceinline__ uint2 lds_read_transposed(const uint16_t* p) {
  return __builtin_bit_cast(uint2, lds_read_tr((lds_v4s16_t*)p));
}

template <int DH, int FEAT>
__global__ __launch_bounds__(256, DH == 128 ? 2 : FEAT ? 3 : 4) void attention_paged_tile_kernel(AttnArgs a) {
  typedef TileCfg<DH> C;
  constexpr int NF = DH / 32, KS = DH / 16;
  // Heads of 128: LDS reads two products ahead (one chunk of 512 over 16384 tokens, 32 heads: 158 -> 153 us).  Of 64, four workgroups a
  // compute unit leave no registers for it (16 prompts of 1024: 51 -> 54).
  constexpr int AHEAD = DH == 128 ? 2 : 0;
  extern __shared__ __attribute__((aligned(16))) uint16_t tile_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  // (Heads dealt so that all blocks of a sequence's head share one XCD's L2 are slower: 16 prompts of 1024 tokens, 12 heads, 68 us for 62.)
  const int h = blockIdx.x;
  const Item rb = item_of<C::ROWS>(a, blockIdx.y + blockIdx.z * gridDim.y);
  if (rb.b < 0) return;
  const int piece = rb.piece;
  const SeqRange s = rb.s;
  const int rows = s.q * a.G;
  if (rb.mb * C::ROWS >= rows) return;
  const KeyRange kr = key_range(a, s, rb.mb * C::ROWS, C::ROWS);
  const int n_pieces = pieces_of(a, kr);
  if (piece >= n_pieces) return;
  const int k_lo = kr.lo + piece * a.split, k_hi = min(kr.hi, k_lo + a.split);
  const int n_tiles = (k_hi - k_lo + C::KT - 1) / C::KT;
  const int m0 = rb.mb * C::ROWS + wave * 32, m = m0 + (lane & 31);
  const bool row_there = m < rows;
  const int mc = min(m, rows - 1), i_new = token_of(a, mc), head = h * a.G + mc - i_new * a.G;
  const int row = s.first + i_new, t_slot = s.len - s.q + i_new;
  const int t_first = s.len - s.q + token_of(a, m0);
  const int t_last = s.len - s.q + min(token_of(a, m0 + 31), s.q - 1);
  const int slots = a.p.max_pages << a.p.page_shift;
  const int32_t* pos = FEAT == 2 ? a.pos + (size_t)rb.b * slots : nullptr;
  // keys below this slot are out of the window of some row of the wavefront
  const int w_first = FEAT == 2 || a.window <= 0 ? INT32_MIN : (int)max((int64_t)t_last - a.window + 1, (int64_t)INT32_MIN);

  const uint16_t* qp = (const uint16_t*)a.q + (size_t)row * a.ld_q + head * DH;
  bf16x8_t fq[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) fq[ks] = *reinterpret_cast<const bf16x8_t*>(qp + ks * 16 + half * 8);
  float slope = 0.f;
  int t_pos = t_slot;
  if (FEAT) {
    if (a.slopes) slope = a.slopes[head] * kLog2e;
    if (FEAT == 2 && t_slot >= 0) t_pos = pos[t_slot];
  }
  // Whether the piece has a page that is none: such tiles are masked key by key.  Each wavefront leaves its answer in LDS.
  int* bad_words = reinterpret_cast<int*>(tile_lds + C::POS + 2 * C::KT * 2);
  {
    bool bad = false;
    for (int col = (k_lo >> a.p.page_shift) + tid; col <= (k_hi - 1) >> a.p.page_shift; col += 256)
      bad |= (uint32_t)a.p.table[(size_t)rb.b * a.p.max_pages + col] >= (uint32_t)a.p.n_pages;
    const int any = __ballot(bad) != 0;
    if (lane == 0) bad_words[wave] = any;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // written before the first tile's barrier
  }

  scalar_i32* table = (scalar_i32*)(uintptr_t)(a.p.table + (size_t)rb.b * a.p.max_pages);
  const int page_mask = (1 << a.p.page_shift) - 1;
  const int r0 = wave * 16;                                       // this wavefront's rows of a tile
  int src_off[C::NI];                                             // this lane's chunk in each of its load instructions
#pragma unroll
  for (int j = 0; j < C::NI; ++j) {
    const int r = j * C::RPI + lane / C::CH;
    src_off[j] = r * DH + ((lane % C::CH) ^ C::swz(r)) * 8;
  }
  int page_next = 0;
  auto ask_page = [&](int t) { page_next = table[min((k_lo + t * C::KT + r0) >> a.p.page_shift, a.p.max_pages - 1)]; };
  auto load = [&](int t, int stage) {
    const int key = k_lo + t * C::KT + r0;
    const int page = (uint32_t)page_next < (uint32_t)a.p.n_pages ? page_next : 0;
    const size_t at = ((((size_t)page * a.p.n_kv + h) << a.p.page_shift) + (key & page_mask)) * DH;
    uint16_t* dst = tile_lds + stage * 2 * C::TILE + r0 * DH;
#pragma unroll
    for (int j = 0; j < C::NI; ++j)
      __builtin_amdgcn_global_load_lds(LLMC_GPTR((const uint16_t*)a.k + at + src_off[j]), LLMC_LPTR(dst + j * C::RPI * DH), 16, 0, 0);
#pragma unroll
    for (int j = 0; j < C::NI; ++j)
      __builtin_amdgcn_global_load_lds(LLMC_GPTR((const uint16_t*)a.v + at + src_off[j]),
                                       LLMC_LPTR(dst + C::TILE + j * C::RPI * DH), 16, 0, 0);
    if (FEAT == 2)                                                // every wavefront the same 64 words
      __builtin_amdgcn_global_load_lds(LLMC_GPTR(pos + min(k_lo + t * C::KT + lane, slots - 1)),
                                       LLMC_LPTR(tile_lds + C::POS + stage * 2 * C::KT), 4, 0, 0);
  };
  ask_page(0);
  if (n_tiles > 0) load(0, 0);
  ask_page(1);

  f32x16_t o[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[f][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};
  const bool exact_sum = a.lse != nullptr;
  bool bad = false;
  // fragment places: keys' row lane % 32 (the swizzle looks at 16 rows), values' row (lane % 16) / 4 of a group of four keys
  const int k_row = lane & 31, k_swz = C::swz(k_row);
  const int v_row = half * 4 + ((lane & 15) >> 2), v_col = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;

  for (int t = 0; t < n_tiles; ++t) {
    const int kb = k_lo + t * C::KT, stage = t & 1;
    LLMC_WAIT_VM(0);
    dma::barrier();                                               // this tile is there, and the other buffer has no readers
    if (t + 1 < n_tiles) {
      load(t + 1, stage ^ 1);
      ask_page(t + 2);
    }
    uint16_t* sk = tile_lds + stage * 2 * C::TILE;
    uint16_t* sv = sk + C::TILE;
    const int* tile_pos = reinterpret_cast<const int*>(tile_lds + C::POS + stage * 2 * C::KT);
    if (t == 0) bad = __builtin_amdgcn_readfirstlane(bad_words[0] | bad_words[1] | bad_words[2] | bad_words[3]) != 0;
    if (kb + C::KT > s.len || bad) {
      // what lies behind the sequence in its last page may be anything, and 0 * anything is not always 0
      const int r = tid >> 2, key = kb + r;
      if (key >= s.len || page_of(a.p, rb.b, key) < 0) {
#pragma unroll
        for (int i = 0; i < C::CH / 4; ++i)
          *reinterpret_cast<uint4*>(sv + r * DH + ((tid & 3) * (C::CH / 4) + i) * 8) = make_uint4(0, 0, 0, 0);
      }
      __syncthreads();
    }
    if (kb > t_last || m0 >= rows) continue;                      // nothing that this wavefront's rows see
    f32x16_t sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[u][r] = 0.f;
    __builtin_amdgcn_s_setprio(1);                                // the other wavefronts of the SIMD have their exponentials to do
    {
      bf16x8_t fk[AHEAD + 1][2];
      const auto read_k = [&](int ks) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          fk[ks % (AHEAD + 1)][u] = *reinterpret_cast<const bf16x8_t*>(sk + (u * 32 + k_row) * DH + (((ks * 2 + half) ^ k_swz) << 3));
      };
#pragma unroll
      for (int ks = 0; ks < AHEAD; ++ks) read_k(ks);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + AHEAD < KS) read_k(ks + AHEAD);
#pragma unroll
        for (int u = 0; u < 2; ++u) sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[ks % (AHEAD + 1)][u], fq[ks], sc[u], 0, 0, 0);
      }
      if (AHEAD) {                                                // reads (0x100) and products (0x8) in this order
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * AHEAD, 0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          if (ks + AHEAD < KS) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    float x[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = sc[i >> 4][i & 15];
    const auto off = [](int i) { return 32 * (i >> 4) + 8 * ((i & 15) >> 2) + (i & 3); };
    const int key0 = kb + half * 4, away0 = t_slot - key0;
    if (FEAT == 2) {
      bias_scores(a, x, [&](int i) { return t_pos - tile_pos[half * 4 + off(i)]; }, slope);
    } else if (FEAT == 1) {
      if (a.softcap > 0.f) cap_scores<false>(a, x);
      const float base = (float)away0;                            // distances below 2^24 are exact
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] = fmaf(-slope, base - (float)off(i), fmaf(x[i], a.mul, a.add));
    } else if (a.softcap > 0.f) {
      cap_scores<true>(a, x);
    }
    if (FEAT != 2 && kb < w_first) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (away0 - off(i) >= a.window) x[i] = -INFINITY;
    }
    if (kb + C::KT - 1 > t_first) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (off(i) > away0) x[i] = -INFINITY;
    }
    if (bad) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (page_of(a.p, rb.b, min(key0 + off(i), a.p.max_len - 1)) < 0) x[i] = -INFINITY;
    }
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) mx = fmaxf(mx, x[i]);
    uint32_t ma, mb_;
    butterfly_pair_u32<32>(__float_as_uint(mx), ma, mb_);
    mx = fmaxf(__uint_as_float(ma), __uint_as_float(mb_));
    const float m_new = FEAT ? mx : fmaf(mx, a.mul, a.add);
    if (__any(m_new > m_run + kSlack)) {
      const float m_top = fmaxf(m_run, m_new), corr = m_top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_top);
      m_run = m_top;
      l_run *= corr;
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[f][r] *= corr;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;         // a row that has seen no key so far
    const float minus = a.add - m_use;
    uint32_t pk[2][8];
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      x[i] = __builtin_amdgcn_exp2f(FEAT ? x[i] - m_use : fmaf(x[i], a.mul, minus));
      x[i + 1] = __builtin_amdgcn_exp2f(FEAT ? x[i + 1] - m_use : fmaf(x[i + 1], a.mul, minus));
      pk[i >> 4][(i & 15) >> 1] = f32x2_to_bf16x2(x[i], x[i + 1]);
    }
    // The value product takes the weights rounded to bf16, in one number each (16 prompts of 1024 tokens, 12 heads of 64: 50 us and 2.4e-4
    // from the exact result on average; with two numbers, as few rows have it, 78 us and 1.7e-4, which is the output's own rounding).
    // The sum is that of the rounded weights, two an instruction: the weights of the value product then add up to one.  Where
    // the cached tokens' weights are wanted too, which are not rounded, it is that of the weights as they are.
    if (exact_sum) {
      float l_tile = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) l_tile += x[i];
      l_run += l_tile;
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pk[e >> 3][e & 7]), ones, l_run, false);
    }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      union { uint32_t u[4]; bf16x8_t v; } pb;
#pragma unroll
      for (int e = 0; e < 4; ++e) pb.u[e] = pk[ks >> 1][(ks & 1) * 4 + e];
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        union { uint2 u[2]; bf16x8_t v; } va;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = ks * 16 + i * 8 + v_row, col = f * 32 + v_col;
          va.u[i] = lds_read_transposed(sv + r * DH + (((col >> 3) ^ C::swz(r)) << 3) + (col & 7));
        }
        o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va.v, pb.v, o[f], 0, 0, 0);
      }
    }
    if (AHEAD) {
      __builtin_amdgcn_sched_group_barrier(0x100, 6, 1);
#pragma unroll
      for (int i = 0; i < 4 * NF; ++i) {
        if (i + 3 < 4 * NF) __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 1);
      }
    }
  }
  const float l = l_run + __shfl_xor(l_run, 32, 64);
  const size_t rh = (size_t)row * a.H + head;
  const bool whole = n_pieces == 1;
  const float scale = !whole ? 1.f : l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
  float zero = 0.f;                                               // or NaN
#pragma unroll
  for (int f = 0; f < NF; ++f)
#pragma unroll
    for (int r = 0; r < 16; ++r) zero = fmaf(o[f][r], 0.f, zero);
  const uint64_t odd = __ballot(zero != 0.f && l < INFINITY && row_there);
  uint32_t again = (uint32_t)(odd | odd >> 32);                   // a bit a row
  if (__builtin_expect(again != 0, 0) && !hides_odd_values<bf16_t, DH>(a, rb, h, t_first, t_last, k_lo, k_hi)) again = 0;
  if (row_there) {
    if (!(again >> (lane & 31) & 1)) {
      if (whole) {
        uint16_t* dst = (uint16_t*)a.out + (size_t)row * a.ld_out + head * DH + half * 4;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint2 w;
            w.x = f32x2_to_bf16x2(o[f][4 * j] * scale, o[f][4 * j + 1] * scale);
            w.y = f32x2_to_bf16x2(o[f][4 * j + 2] * scale, o[f][4 * j + 3] * scale);
            *reinterpret_cast<uint2*>(dst + f * 32 + 8 * j) = w;
          }
      } else {
        float* dst = a.part_o + (rh * a.n_split + piece) * DH + half * 4;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<float4*>(dst + f * 32 + 8 * j) =
                make_float4(o[f][4 * j], o[f][4 * j + 1], o[f][4 * j + 2], o[f][4 * j + 3]);
      }
    }
    if (half == 0) {
      if (!whole) a.part_ml[rh * a.n_split + piece] = make_float2(m_run, l);
      else if (a.lse) a.lse[rh] = l == 0.f ? INFINITY : m_run + __builtin_amdgcn_logf(l);
    }
  }
  for (; __builtin_expect(again != 0, 0); again &= again - 1) {
    const int col = __builtin_ctz(again), mr = m0 + col;
    const auto of_row = [&](float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), col)); };
    const float ref = of_row(m_run) == -INFINITY ? 0.f : of_row(m_run), sc = of_row(scale);
    const int i = token_of(a, mr), r = s.first + i, hd = h * a.G + mr - i * a.G;
    float* part = whole ? nullptr : a.part_o + (((size_t)r * a.H + hd) * a.n_split + piece) * DH;
    sum_seen<bf16_t, DH, FEAT == 0>(a, rb, h, mr, ref, k_lo, k_hi, 64, 64, part, (bf16_t*)a.out + (size_t)r * a.ld_out + hd * DH, sc);
  }
}

// ---- the weight that every key received ---------------------------------------------------------------------------------
// sum over the rows of p = 2^(x - lse), the scores computed a second time with the finished normalisers.  A wavefront, a workgroup
// of its own, holds 16 to 64 keys of one head in registers and walks the rows, the next ones in flight; where there are few, several share a
// head's rows.  Its sums go to sums[b][share][h][key]; a second kernel adds them up in one order: no atomics.  The first keys, which
// every row sees, come first.  (Workgroups that take all heads of some keys and add in LDS spare that launch, 4.6 us, but
// are few and uneven: 16 prompts of 1024 tokens, 12 heads: 71 us, 54 this way.)
// FEAT as in the tile kernel.
template <typename T, int DH> struct WeightCfg {
  static constexpr int TILES = sizeof(T) == 2 ? 4 : DH == 64 ? 2 : 1;        // of 16 keys: 32 or 64 registers
  static constexpr int RT = sizeof(T) == 2 && DH == 64 ? 2 : 1;              // 16-row tiles of a step
  static constexpr int KEYS = 16 * TILES;
};

template <typename T, int DH, int FEAT>
__global__ __launch_bounds__(64) void attention_paged_weight_kernel(AttnArgs a, float* __restrict__ sums, int shares) {
  typedef Frag<T, DH> F;
  typedef typename F::E E;
  typedef WeightCfg<T, DH> W;
  constexpr int SUB = F::SUB, TILES = W::TILES, NK = TILES / SUB, RT = W::RT;
  const int lane = threadIdx.x, c = lane & 15, g = lane >> 4;
  const int h = blockIdx.y;
  uint32_t share = blockIdx.z, idx = blockIdx.x;
  for (; share >= (uint32_t)shares; share -= shares) idx += gridDim.x;             // more workgroups than fit one dimension
  const int b = idx % (uint32_t)a.p.n_seqs;
  const SeqRange s = seq_range(a.p, b);
  const int kb = key_range(a, s, 0, 1).lo + (int)(idx / (uint32_t)a.p.n_seqs) * W::KEYS;      // from the first key that a window leaves
  if (kb >= s.len || s.q == 0) return;
  const int slots = a.p.max_pages << a.p.page_shift;
  const int32_t* pos = FEAT == 2 ? a.pos + (size_t)b * slots : nullptr;
  const int rows = s.q * a.G, t_base = s.len - s.q;
  scalar_i32* table = (scalar_i32*)(uintptr_t)(a.p.table + (size_t)b * a.p.max_pages);
  const int page_mask = (1 << a.p.page_shift) - 1;
  int page[TILES];
  bool bad = false;
  typename F::K fk[NK];
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    const int p = table[min((kb + 16 * u) >> a.p.page_shift, a.p.max_pages - 1)];
    page[u] = (uint32_t)p < (uint32_t)a.p.n_pages ? p : -1;
    bad |= page[u] < 0;
    const size_t at = ((((size_t)max(page[u], 0) * a.p.n_kv + h) << a.p.page_shift) + ((kb + 16 * u) & page_mask)) * DH;
    F::load_k(fk[u / SUB], u % SUB, (const E*)a.k + at, c, g);
  }
  int key_pos[TILES][4];
  if (FEAT == 2) {
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
      const int4 v = reinterpret_cast<const int4*>(pos)[min(kb + 16 * u + 4 * g, slots - 4) >> 2];
      key_pos[u][0] = v.x; key_pos[u][1] = v.y; key_pos[u][2] = v.z; key_pos[u][3] = v.w;
    }
  }
  // rows whose tokens do not lie before the first key, and, with a window and slots as positions, not too far behind the last
  const int m_lo = max(0, kb - t_base) * a.G;
  int m_hi = rows;
  if (FEAT != 2 && a.window > 0)
    m_hi = (int)min((int64_t)rows, max((int64_t)0, (int64_t)kb + W::KEYS - 1 - t_base + a.window) * a.G);
  struct Rows {
    typename F::Q q[RT];
    float lse[RT], slope[RT];
    int t_slot[RT], t_pos[RT];
  };
  float w[TILES][4];
#pragma unroll
  for (int u = 0; u < TILES; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r) w[u][r] = 0.f;
  auto fetch = [&](Rows& R, int m0) {
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int m = m0 + 16 * i + c, mc = min(m, rows - 1), i_new = token_of(a, mc), head = h * a.G + mc - i_new * a.G;
      const int row = s.first + i_new;
      F::load_q(R.q[i], (const E*)a.q + (size_t)row * a.ld_q + head * DH, g);
      R.lse[i] = a.lse[(size_t)row * a.H + head];
      R.t_slot[i] = t_base + i_new;
      if (FEAT) R.slope[i] = a.slopes ? a.slopes[head] * kLog2e : 0.f;
      if (FEAT == 2) R.t_pos[i] = pos[max(R.t_slot[i], 0)];
    }
  };
  auto work = [&](Rows& R, int m0) {
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int first = t_base + token_of(a, min(m0 + 16 * i, rows - 1)), last = t_base + token_of(a, min(m0 + 16 * i + 15, rows - 1));
      const bool edge = first < kb + W::KEYS - 1 || bad || (FEAT != 2 && a.window > 0 && (int64_t)last - kb >= a.window);
      float lse = m0 + 16 * i + c < m_hi ? R.lse[i] : INFINITY;             // no such row, or out of the window: weights of zero
      // a row of NaN gives NaN to the keys that it sees, through its products, and nothing to hidden ones (-inf - NaN is NaN too)
      const float from = lse == lse ? 0.f : lse;
      lse = lse == lse ? lse : 0.f;
#pragma unroll
      for (int u = 0; u < TILES; ++u) {
        const f32x4_t sc = F::qk(fk[u / SUB], u % SUB, R.q[i], from);
        const int key0 = kb + 16 * u + 4 * g;
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = sc[r];
        if (FEAT == 2) {
          bias_scores(a, x, [&](int r) { return R.t_pos[i] - key_pos[u][r]; }, R.slope[i]);
        } else {
          if (a.softcap > 0.f) cap_scores<false>(a, x);
          if (FEAT == 1) {
            const float base = (float)(R.t_slot[i] - key0);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = fmaf(-R.slope[i], base - (float)r, fmaf(x[r], a.mul, a.add));
          }
        }
        if (edge) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int away = R.t_slot[i] - key0 - r;
            if (away < 0 || page[u] < 0 || (FEAT != 2 && a.window > 0 && away >= a.window)) x[r] = -INFINITY;
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
          w[u][r] += __builtin_amdgcn_exp2f(FEAT ? x[r] - lse : fmaf(x[r], a.mul, a.add - lse));
      }
    }
  };
  const int step = shares * RT * 16;
  int m0 = (m_lo & ~15) + share * RT * 16;
  if (m0 < m_hi) {
    Rows r0, r1;
    fetch(r0, m0);
    for (;;) {
      fetch(r1, m0 + step);                                      // beyond the last row the last one is read again
      work(r0, m0);
      if ((m0 += step) >= m_hi) break;
      fetch(r0, m0 + step);
      work(r1, m0);
      if ((m0 += step) >= m_hi) break;
    }
  }
#pragma unroll
  for (int u = 0; u < TILES; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v = w[u][r];
      v += __uint_as_float(butterfly_u32<8>(__float_as_uint(v)));
      v += __uint_as_float(butterfly_u32<4>(__float_as_uint(v)));
      v += __uint_as_float(butterfly_u32<2>(__float_as_uint(v)));
      v += __uint_as_float(butterfly_u32<1>(__float_as_uint(v)));
      w[u][r] = v;
    }
  if (c == 0) {                                                  // a row of sums has room for whole tiles
    float* dst = sums + (((size_t)b * shares + share) * a.p.n_kv + h) * a.ld_scores + kb + 4 * g;
#pragma unroll
    for (int u = 0; u < TILES; ++u) *reinterpret_cast<float4*>(dst + 16 * u) = make_float4(w[u][0], w[u][1], w[u][2], w[u][3]);
  }
}

__global__ __launch_bounds__(256) void attention_paged_add_weights_kernel(AttnArgs a, const float* __restrict__ sums, int n,
                                                                          float* __restrict__ weight) {
  const int b = blockIdx.y;
  const SeqRange s = seq_range(a.p, b);
  const int key = key_range(a, s, 0, 1).lo + blockIdx.x * 256 + threadIdx.x;
  if (key >= s.len || s.q == 0) return;
  const float* src = sums + (size_t)b * n * a.ld_scores + key;
  float v = 0.f;
#pragma unroll 8
  for (int h = 0; h < n; ++h) v += src[(size_t)h * a.ld_scores];
  weight[((size_t)b * a.p.max_pages << a.p.page_shift) + key] += v;
}

// The same from the scores that the attention itself left, for calls of up to 16 rows a head.  A workgroup takes 256 keys, four a
// lane; its wavefronts take a quarter of the rows of all heads each, and the four sums are added in order: the loads of a
// thread are few and independent, which is what this is bound by.  Keys outside the rows' range have no scores.  Where the key
// axis was cut, the normalisers are made from the pieces' here, and workgroups beyond the keys' join the outputs (a launch
// of their own takes 7 us for 6 sequences of up to 32768 tokens).
template <typename T, int DH>
__global__ __launch_bounds__(256) void attention_paged_score_weights_kernel(AttnArgs a, float* __restrict__ weight, int n_kb) {
  __shared__ float4 part[3][64];
  const int b = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SeqRange s = seq_range(a.p, b);
  const int rows = s.q * a.G, n = a.p.n_kv * rows;
  if (rows == 0) return;
  const KeyRange kr = key_range(a, s, 0, 16);                    // lo is a multiple of 64
  const int n_pieces = pieces_of(a, kr);
  if ((int)blockIdx.x >= n_kb) {
    const int r = (int)blockIdx.x - n_kb, h = r / rows, m = r - h * rows;
    const int i = token_of(a, m);
    if (r < n && n_pieces > 1) join_pieces<T, DH>(a, s.first + i, h * a.G + m - i * a.G, n_pieces);
    return;
  }
  const int key = blockIdx.x * 256 + lane * 4;
  if ((int)blockIdx.x * 256 >= kr.hi || (int)blockIdx.x * 256 + 256 <= kr.lo) return;
  const bool there = key >= kr.lo && key < kr.hi;
  const int per = (n + 3) / 4, r0 = wave * per, r1 = min(n, r0 + per);
  const float* src = a.scores + (size_t)b * a.p.n_kv * a.join_rows * a.ld_scores + (there ? key : kr.lo);
  float w[4] = {0.f, 0.f, 0.f, 0.f};
  for (int q0 = r0; q0 < r1; q0 += 8) {
    // eight rows' normalisers side by side, by eight lanes each
    const int r = min(q0 + (lane >> 3), r1 - 1), h = r / rows, m = r - h * rows, i_new = token_of(a, m);
    const int at = h * a.join_rows + m;
    const size_t rh = (size_t)(s.first + i_new) * a.H + h * a.G + m - i_new * a.G;
    float lse;
    if (n_pieces > 1) {
      const float2* ml = a.part_ml + rh * a.n_split;
      float top = -INFINITY, l = 0.f;
      for (int j = lane & 7; j < n_pieces; j += 8) top = fmaxf(top, ml[j].x);
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      const float top_use = top == -INFINITY ? 0.f : top;
      for (int j = lane & 7; j < n_pieces; j += 8) {
        const float2 v = ml[j];
        l += v.y * __builtin_amdgcn_exp2f(v.x - top_use);
      }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) l += __shfl_xor(l, o, 64);
      lse = l == 0.f ? INFINITY : top + __builtin_amdgcn_logf(l);
    } else {
      lse = a.lse[rh];
    }
    float4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = *reinterpret_cast<const float4*>(src + (size_t)__builtin_amdgcn_readlane(at, i * 8) * a.ld_scores);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (q0 + i >= r1) break;
      const float z = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lse), i * 8));
      w[0] += x[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[i].x - z);
      w[1] += x[i].y == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[i].y - z);
      w[2] += x[i].z == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[i].z - z);
      w[3] += x[i].w == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[i].w - z);
    }
  }
  if (wave > 0) part[wave - 1][lane] = make_float4(w[0], w[1], w[2], w[3]);
  __syncthreads();
  if (wave > 0 || !there) return;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const float4 v = part[i][lane];
    w[0] += v.x; w[1] += v.y; w[2] += v.z; w[3] += v.w;
  }
  float* dst = weight + ((size_t)b * a.p.max_pages << a.p.page_shift) + key;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (key + i < kr.hi) dst[i] += w[i];
}

// ---- host ---------------------------------------------------------------------------------------------------------------
struct Plan {
  bool tile, rowsplit;
  int rows;                    // of a row block
  int join_rows;               // rows a head at most, where a workgroup's wavefronts are joined
  int64_t blocks;              // row blocks of all sequences, at most
  int split, n_split;
  int shares;                  // of a head's rows, for the weights of its keys
};

// How a call is cut.  Up to 16 rows a head (single tokens above all): 16-row products with the keys dealt to wavefronts.  More
// rows in bf16 share key tiles in LDS, in fp32 (bound by the matrix instructions of that type) 64 rows walk the keys together.
// The key axis is cut where there are too few row blocks to fill the chip.
// The line at 16 rows is what one product of a wavefront holds.  In bf16 the tiles would be slower below it where the call is short (one sequence
// of 1000 tokens, 12 heads of 64, 8 and 16 new ones: 8.9 and 9.5 us, in tiles 14.4 and 14.0; 64 sequences of up to 300, 8 and 16 new:
// 14.1 and 15.7, in tiles 13.9 and 14.6) and faster where it is long (16 of up to 2048, 8 and 16 new: 27.6 and 29.0, in tiles 24.5 and
// 23.7; 4 of up to 8192, 8 heads of 128 shared by four each, 2 and 4 new: 37 and 42, in tiles 32 and 33), but they round weights to 8 bits for
// 16, and the weights of cached tokens would take a second pass over the keys.
// span: the longest range of keys that a row block can see (a window may make it shorter than max_len); workspaces are sized
// for span = max_len, and a shorter one never gets more pieces.
Plan make_plan(int dtype, int head_dim, int n_rows, int n_seqs, int n_kv, int G, int max_new, int max_len, int span) {
  Plan p{};
  const int64_t rows = (int64_t)max_new * G;
  p.tile = rows > 16 && dtype == LLMC_BF16;
  p.rowsplit = rows > 16 && !p.tile;
  p.rows = p.tile ? 128 : p.rowsplit ? 64 : 16;
  p.join_rows = (int)std::min<int64_t>(rows, 16);
  p.blocks = rows <= p.rows ? n_seqs : std::min<int64_t>((rows + p.rows - 1) / p.rows * n_seqs, (int64_t)n_rows * G / p.rows + n_seqs);
  const int64_t units = std::max<int64_t>(1, p.blocks * n_kv);
  const auto cut = [&](int len, int most) {
    int64_t want;                // pieces of the key axis
    int least = p.tile || (p.rowsplit && head_dim == 64) ? 256 : 128;        // keys of a piece
    if (p.tile || p.rowsplit) {
      // bf16: as many as are resident, four a compute unit, of 128-wide heads two.  Where there is a workgroup a compute unit anyway,
      // only in pieces that are long on average (the rows of a whole prompt see half of it) and pay for being joined: 12 chunks of up
      // to 333 tokens over 3000, 12 heads, 55 us whole, 34 + 5 in two; in a window of 1024, 30 and 22 + 5; 5 prompts of
      // 1024: 24 whole, 24 + 7 in two.
      // fp32: twice as many, a step is long there (8 chunks of up to 256 tokens over 1024, 12 heads of 64: 66 us whole, 38 + 5 in
      // pieces; 4 of them with heads of 128: 68 + 5.5 us in pieces of 256 keys, 58 + 7 of 128).
      want = (p.rowsplit ? 2048 : head_dim == 128 ? 512 : 1024) / units;
      if (p.tile && units >= 256) want = std::min<int64_t>(want, (len < max_len ? len : len - max_new / 2) / 512);
    } else {
      // Eight steps of a workgroup take as long as the second launch that joins pieces (one sequence of 777 tokens, 12 heads of 64:
      // 8.0 us in one piece, 4.4 + 4.0 in seven).  From two workgroups a compute unit on, cutting gains less than that launch
      // (64 sequences of up to 2048: 42 and 47 + 4); below, pieces even out ragged lengths (6 of up to 32768, 8 heads of 128: 1024
      // workgroups 106 + 4.5 us, 2048 92 + 7, 4096 93 + 10).  Down to a step of a workgroup, two in fp32 (8 of up to 1000 in fp32, 12
      // heads of 64, biased: 13.4 us in pieces of 256 keys, 10.5 of 128; 8 of up to 1200 in bf16: 7.7 and 6.8).
      // More than 128 pieces of one axis only where there would be less than two workgroups a compute unit (one of 100000 tokens, 8 heads of
      // 128: 78 + 6.6 us in 256, 76 + 5 in 128).
      const int steps8 = 8 * 4 * (dtype == LLMC_BF16 ? 32 : 16);
      want = len <= steps8 || units >= 512 ? 1 : std::min<int64_t>(2048 / units, std::max<int64_t>(128, 512 / units));
    }
    want = std::max<int64_t>(1, std::min<int64_t>({want, most, len / least}));
    p.split = (int)std::max<int64_t>(least, align_up((size_t)((len + want - 1) / want), 128));
    p.n_split = std::max(1, (int)((len + p.split - 1) / p.split));
  };
  cut(max_len, max_len);
  if (span < max_len) cut(span, p.n_split);
  // Wavefronts that sum weights: two a SIMD at least as long as each has 128 rows, and none with many more than 256 rows: the first keys
  // of a long chunk would keep the call waiting (16 prompts of 1024 tokens, 12 heads: 64 us in one share, 54 in four).
  const int64_t waves = (int64_t)n_seqs * n_kv * ((max_len + 63) / 64);
  p.shares = (int)std::max<int64_t>(1, std::min<int64_t>({std::max<int64_t>(2048 / waves, rows / 256), rows / 128, 16}));
  return p;
}

struct Layout { size_t part_o, part_ml, lse, scores, sums, total; int ld_scores; };
Layout ws_layout(const Plan& p, int n_rows, int H, int DH, int n_seqs, int n_kv, int max_len, bool weights) {
  Layout l{};
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t r = at; at += align_up(bytes, 256); return r; };
  const size_t rh = (size_t)n_rows * H;
  const bool scores = weights && !p.tile && !p.rowsplit;
  l.ld_scores = (int)align_up((size_t)max_len, 64);
  l.part_o = take(p.n_split > 1 ? rh * p.n_split * DH * 4 : 0);
  l.part_ml = take(p.n_split > 1 ? rh * p.n_split * 8 : 0);
  l.lse = take(weights ? rh * 4 : 0);
  l.scores = take(scores ? (size_t)n_seqs * n_kv * p.join_rows * l.ld_scores * 4 : 0);
  l.sums = take(weights && !scores ? (size_t)n_seqs * n_kv * p.shares * l.ld_scores * 4 : 0);
  l.total = std::max<size_t>(at, 256);
  return l;
}

void set_scores(AttnArgs& a, const llmc_attn_desc_t* at, bool fast_cap) {
  if (at->softcap > 0.f) {
    const float c2 = at->softcap * kLog2e;
    a.cap_in = (float)((fast_cap ? 2.0 * 1.4426950408889634 : 1.0) * at->scale / at->softcap);
    a.mul = fast_cap ? 2.f * c2 : c2;
    a.add = fast_cap ? c2 : 0.f;
  } else {
    a.mul = at->scale * kLog2e;
  }
}

template <int DH, int FEAT>
llmc_status_t launch_tile(const AttnArgs& a, dim3 grid, hipStream_t st) {
  static std::atomic<bool> lds_set[64];
  const auto kernel = attention_paged_tile_kernel<DH, FEAT>;
  LLMC_TRY(ensure_dynamic_lds((const void*)kernel, TileCfg<DH>::LDS_BYTES, lds_set));
  LLMC_KERNEL_GGL(kernel, grid, dim3(256), TileCfg<DH>::LDS_BYTES, st, a);
  return LLMC_OK;
}

template <typename T, int DH, int FEAT>
llmc_status_t launch_t(AttnArgs a, const llmc_attn_desc_t* at, const Plan& p, float* sums, float* weight, hipStream_t st) {
  const bool fast_cap = p.tile && FEAT == 1 && !a.slopes && at->softcap <= (weight ? 64.f : 1024.f);
  set_scores(a, at, fast_cap);
  const int64_t items = p.blocks * p.n_split;
  const dim3 grid((unsigned)a.p.n_kv, (unsigned)std::min<int64_t>(items, 32768), (unsigned)((items + 32767) / 32768));
  {
    ProfScope ps_("attention_paged_kernel", st);
    if (!p.tile && !p.rowsplit) {
      // 16 rows of 128 dims take 33.8 KiB: no more than a kernel may have without asking
      const size_t lds = (size_t)4 * p.join_rows * (DH + 4 + 2) * 4;
      LLMC_KERNEL_GGL((attention_paged_rows_kernel<T, DH, FEAT, false>), grid, dim3(256), lds, st, a);
    } else if constexpr (sizeof(T) == 2) {
      if (FEAT == 1 && !a.slopes && (fast_cap || at->softcap == 0.f)) LLMC_TRY((launch_tile<DH, 0>(a, grid, st)));
      else LLMC_TRY((launch_tile<DH, FEAT>(a, grid, st)));
    } else {
      LLMC_KERNEL_GGL((attention_paged_rows_kernel<T, DH, FEAT, true>), grid, dim3(256), 0, st, a);
    }
  }
  LLMC_LAUNCH_CHECK("attention_paged");
  if (p.n_split > 1 && !a.scores) {
    ProfScope ps_("attention_paged_join_kernel", st);
    constexpr int heads = 256 / DH;
    const dim3 one((unsigned)a.H, (unsigned)std::min(a.p.n_rows, 32768), (unsigned)((a.p.n_rows + 32767) / 32768));
    const dim3 many = flat_grid(((int64_t)a.p.n_rows * ((a.H + heads - 1) / heads) + 3) / 4);
    if (p.rows == 128) LLMC_KERNEL_GGL((attention_paged_join_rows_kernel<T, DH, 128>), many, dim3(256), 0, st, a);
    else if (p.rows == 64) LLMC_KERNEL_GGL((attention_paged_join_rows_kernel<T, DH, 64>), many, dim3(256), 0, st, a);
    else LLMC_KERNEL_GGL((attention_paged_join_kernel<T, DH>), one, dim3(256), 0, st, a);
    LLMC_LAUNCH_CHECK("attention_paged_join");
  }
  if (weight && a.scores) {
    { ProfScope ps_("attention_paged_weight_kernel", st);
      const int n_kb = (a.p.max_len + 255) / 256, n_join = p.n_split > 1 ? p.join_rows * a.p.n_kv : 0;
      LLMC_KERNEL_GGL((attention_paged_score_weights_kernel<T, DH>), dim3(n_kb + n_join, a.p.n_seqs), dim3(256), 0, st, a, weight,
                      n_kb); }
    LLMC_LAUNCH_CHECK("attention_paged_score_weights");
  } else if (weight) {
    constexpr int keys = WeightCfg<T, DH>::KEYS;
    // keys that the new tokens of a sequence see, at most; the first one rounded down to a multiple of 64
    const int seen = a.window > 0 && !a.pos ? (int)std::min<int64_t>(a.p.max_len, (int64_t)a.window + a.p.max_new + 62) : a.p.max_len;
    set_scores(a, at, false);
    { ProfScope ps_("attention_paged_weight_kernel", st);
      dim3 wg = flat_grid((int64_t)((seen + keys - 1) / keys) * a.p.n_seqs);
      wg = dim3(wg.x, (unsigned)a.p.n_kv, wg.y * (unsigned)p.shares);
      if (FEAT == 1 && !a.slopes) LLMC_KERNEL_GGL((attention_paged_weight_kernel<T, DH, 0>), wg, dim3(64), 0, st, a, sums, p.shares);
      else LLMC_KERNEL_GGL((attention_paged_weight_kernel<T, DH, FEAT>), wg, dim3(64), 0, st, a, sums, p.shares); }
    LLMC_LAUNCH_CHECK("attention_paged_weight");
    { ProfScope ps_("attention_paged_add_weights_kernel", st);
      LLMC_KERNEL_GGL(attention_paged_add_weights_kernel, dim3((seen + 255) / 256, a.p.n_seqs), dim3(256), 0, st, a, sums,
                      a.p.n_kv * p.shares, weight); }
    LLMC_LAUNCH_CHECK("attention_paged_add_weights");
  }
  return LLMC_OK;
}

}  // namespace

size_t attention_paged_ws_bytes(int dtype, int head_dim, int n_kv, int H, int n_rows, int n_seqs, int max_new, int max_len,
                                bool weights) {
  const Plan p = make_plan(dtype, head_dim, n_rows, n_seqs, n_kv, H / n_kv, max_new, max_len, max_len);
  return ws_layout(p, n_rows, H, head_dim, n_seqs, n_kv, max_len, weights).total;
}

bool attention_paged_grid_ok(int dtype, int head_dim, int n_kv, int H, int n_rows, int n_seqs, int max_new, int max_len, bool weights) {
  const Plan p = make_plan(dtype, head_dim, n_rows, n_seqs, n_kv, H / n_kv, max_new, max_len, max_len);
  const int64_t most = 0x7FFFFFFF;
  return p.blocks <= most / n_kv / p.n_split && (int64_t)n_rows * H <= most &&
         (!weights || (int64_t)((max_len + 15) / 16) <= most / n_seqs);
}

llmc_status_t launch_attention_paged(const llmc_kv_desc_t* kv, const llmc_kv_batch_t* bt, const llmc_attn_desc_t* at,
                                     const void* q, int64_t ld_q, void* out, int64_t ld_out, void* ws, hipStream_t st) {
  if (bt->n_rows == 0) return LLMC_OK;
  const int G = at->n_heads / kv->n_kv_heads;
  const bool by_slot = at->window > 0 && !bt->d_pos;             // a block of 128 rows sees a window behind each, rounded to 64 keys
  const int span = by_slot ? (int)std::min<int64_t>(bt->max_len, (int64_t)at->window + std::min(bt->max_new, 127 / G + 1) + 63) : bt->max_len;
  const Plan p = make_plan(kv->dtype, kv->head_dim, bt->n_rows, bt->n_seqs, kv->n_kv_heads, G, bt->max_new, bt->max_len, span);
  const bool weights = bt->d_weight && at->accumulate;
  const Layout l = ws_layout(p, bt->n_rows, at->n_heads, kv->head_dim, bt->n_seqs, kv->n_kv_heads, bt->max_len, weights);
  AttnArgs a{};
  a.p = paged_args(kv, bt);
  a.q = q; a.out = out; a.k = kv->d_k; a.v = kv->d_v; a.ld_q = ld_q; a.ld_out = ld_out;
  a.H = at->n_heads; a.G = G;
  a.g_magic = row_magic(a.G); a.split_magic = row_magic(p.split);
  a.softcap = at->softcap;
  a.window = at->window; a.slopes = at->d_slopes;
  a.pos = (at->window > 0 || at->d_slopes) ? bt->d_pos : nullptr;
  a.split = p.split; a.n_split = p.n_split; a.blocks = (int)p.blocks;
  char* w = (char*)ws;
  a.part_o = (float*)(w + l.part_o); a.part_ml = (float2*)(w + l.part_ml);
  a.lse = weights ? (float*)(w + l.lse) : nullptr;
  const int64_t levels = ((int64_t)bt->max_new * a.G + p.rows - 1) / p.rows;
  a.by_level = bt->n_seqs <= 64 && levels <= 64 ? (int)levels : 0;
  a.by_length = bt->n_seqs > 1 && p.n_split == 1 && p.blocks * kv->n_kv_heads > 256;
  a.join_rows = p.join_rows; a.ld_scores = l.ld_scores;
  a.scores = weights && !p.tile && !p.rowsplit ? (float*)(w + l.scores) : nullptr;
  float* sums = weights ? (float*)(w + l.sums) : nullptr;
  float* weight = weights ? bt->d_weight : nullptr;
  const int feat = a.pos ? 2 : at->softcap > 0.f || at->window > 0 || at->d_slopes ? 1 : 0;
#define LLMC_PAGED(T_, DH_)                                                  \
  return feat == 2   ? launch_t<T_, DH_, 2>(a, at, p, sums, weight, st)          \
         : feat == 1 ? launch_t<T_, DH_, 1>(a, at, p, sums, weight, st)          \
                     : launch_t<T_, DH_, 0>(a, at, p, sums, weight, st)
  if (kv->dtype == LLMC_BF16) {
    if (kv->head_dim == 64) LLMC_PAGED(bf16_t, 64);
    LLMC_PAGED(bf16_t, 128);
  }
  if (kv->head_dim == 64) LLMC_PAGED(float, 64);
  LLMC_PAGED(float, 128);
#undef LLMC_PAGED
}

}  // namespace llmc
