// The kernels of attention to a cache of keys and values in four bits (kernels_cache.hip).
//
// A row is a token of one of the query heads that share a key head.  With a = scale * log2(e) and m the largest of a row's a q.k so far, o = sum_j 2^(a q.k_j - m) v_j
// and l = sum_j 2^(a q.k_j - m) are formed in one pass over the keys; o / l is what comes out.  Keys and values are widened to 16 bits on their way into the matrix
// cores, which rounds nothing (cache_pages.hpp); fp32 queries and probabilities go in as the three bf16 numbers that they are the sum of (24 bits: exact, and
// three products of 16 bits where products of 32 would take eight times as long).
//
// What bounds it.  Few rows: the one read of the cache, and behind short ones the trips (length, page number, codes), what a wavefront alone on its SIMD waits for from
// step to step, and the second launch.  Many rows: the power that the matrix cores may draw, beside it the exponentials and what widening costs; of those 207
// vector instructions a wavefront and tile of 64 keys at 64 channels, 32 are exponentials of four times the cycles.
// us on inputs that are not the call's before, host included, over several boxes: one token of 32 / 8 heads of 128 against 4 x 65536 tokens (ragged) in bf16 39 to 41 (under the tracer the
// first kernel 35 = 4.0 TB/s and the second 4.8), in fp32 51 to 54, against 65536 21 to 22, 16 x 4096 in f16 20.3 to 23 (18.1 and 4.6), in fp32 28 to 32, 2000 10 to 11, 300 7.3 to 7.9; 30 heads of 64
// against 4 x 32768 62 to 66 = 4.1 to 4.3 TB/s; 5400x10800 of 30 of 64 in f16 618 to 700 = 725 to 640 TFLOP/s, 8192x8192 of 32 / 8 of 128 in bf16 1100 to 1120 = 1000 to 982, in f16 1130 to 1215
// (the longer the call is repeated, the slower), 2 x 4096x4096 of 16 of 256 680 = 806, 3000x3000 of 8 of 128 in fp32 108 to 113 = 341 to 326 (products of 32 bits reach 155 at most).
// Steps, us for 4 x 65536, 16 x 4096, 5400x10800: sixteen rows a wavefront for all sizes, two sets of codes under way 46.7, 24.8, 1157; 128 rows a workgroup 669 of the last; one
// set, asked for again as soon as it has been used, four wavefronts a SIMD 39.5, 20.8; pages by the wavefront where they are multiples of 16; places from tile to tile 653 to 624 of the last;
// infinities of f16 taken out, no more than 1 %.
// Measured and not kept: two sets of codes under way with few rows (300 to 500 keys 3 % faster, 16 x 4096 26.0 against 22.7), 32 rows a wavefront for few rows (half the wavefronts: 16 x 64 tokens against 4096 294 against 181), 16 wavefronts a workgroup in place of ranges of
// keys (2000 tokens 14.1 against 10.7, eight samples of 1000 11.8 against 15.7: no better but there), the sum of the probabilities as a product with ones (5400x10800 672), four wavefronts a
// SIMD at 64 channels and many rows, with what a thread widens worked out anew (645).
#pragma once
#include <algorithm>

#include "cache_pages.hpp"

namespace wmdec {

constexpr int kFewRows = 16, kManyRows = 128, kCacheMaxSplits = 64;

// How the work is divided (kernels_cache.hip decides).  A block is a number of rows of a key head; its keys are a workgroup's each `range` of them.  Blocks that need
// one range only write the output, the others partial outputs, and a second launch joins these.
struct CachePlan {
  int nb = 1;                                        // blocks of 32 channels
  bool few = true;                                   // blocks of kFewRows rows, else of kManyRows
  bool halves = false;                               // many: the wavefronts of a workgroup are eight and take halves of a tile's keys
  int rows = 0, row_blocks = 0, range = 0, splits = 1;
  __host__ __device__ int bq() const { return few ? kFewRows : kManyRows; }
  __host__ __device__ int block_rows() const { return rows < bq() ? rows : bq(); }   // of partial outputs
};
struct CacheLaunch {
  CacheAttentionArgs a;
  CachePlan plan;
  float* part;                                       // [sample][key head][row block][split][block_rows][32 nb] sums of probabilities times values
  float2* ml;                                        // [sample][key head][row block][split][block_rows] reference and sum of the probabilities
};

template <typename T> struct CacheOperand { typedef T type; static constexpr int pieces = 1; };   // what the matrix cores get
template <> struct CacheOperand<float> { typedef bf16_t type; static constexpr int pieces = 3; };

// the sum of the pieces is x (to 24 bits)
__device__ __forceinline__ void split_rest(float a, float b, unsigned (&w)[3]) {
  w[1] = pack2<bf16_t>(a, b);
  a -= unpack_lo<bf16_t>(w[1]); b -= unpack_hi<bf16_t>(w[1]);
  w[2] = pack2<bf16_t>(a, b);
}
__device__ __forceinline__ void split3(float a, float b, unsigned (&w)[3]) {
  w[0] = pack2<bf16_t>(a, b);
  split_rest(a - unpack_lo<bf16_t>(w[0]), b - unpack_hi<bf16_t>(w[0]), w);
}
// eight of any numbers: those that bf16 would round to infinity have its largest as their first piece, and infinities have no rest
__device__ __forceinline__ void split3_any(f32x4 x, f32x4 y, unsigned (&w)[4][3]) {
  float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]}, top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i]));
  if (!__ballot(top > 0x1.fep127f)) {                // bf16's largest
#pragma unroll
    for (int i = 0; i < 4; ++i) split3(v[2 * i], v[2 * i + 1], w[i]);
    return;
  }
  float first[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool past = fabsf(v[i]) > 0x1.fep127f, infinite = fabsf(v[i]) == INFINITY;
    first[i] = past && !infinite ? copysignf(0x1.fep127f, v[i]) : v[i];
    if (infinite) v[i] = 0.f;
    else v[i] -= past ? first[i] : unpack_lo<bf16_t>(pack2<bf16_t>(first[i], 0.f));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i][0] = pack2<bf16_t>(first[2 * i], first[2 * i + 1]);
    split_rest(v[2 * i], v[2 * i + 1], w[i]);
  }
}

// what is in the cache for a sample, and how far a block of rows sees of it
struct CacheView {
  int len, count;                                    // tokens of the sample, rows of tokens among the queries
  int rows;                                          // rows of a key head
  int end;                                           // keys that the block's rows see at most
};
__device__ __forceinline__ CacheView view_of(const CacheAttentionArgs& a, int n, int first_row, int block_rows) {
  CacheView v;
  v.len = min(max(a.lens[n], 0), a.reach);
  v.count = a.counts ? min(max(a.counts[n], 0), a.tq) : a.tq;
  v.rows = v.count * a.group;
  const int last = min(first_row + block_rows, v.rows) - 1;
  v.end = a.causal ? min(v.len, max(0, v.len - v.count + last / a.group + 1)) : v.len;
  return v;
}

__device__ __forceinline__ float cache_weight(float m, float top) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top); }

template <typename T> __device__ __forceinline__ void store_four(T* row, int at, int d, f32x4 v) {   // (d is a multiple of 8)
  if (at >= d) return;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(row + at) = v;
  else *reinterpret_cast<u32x2*>(row + at) = u32x2{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
}
template <typename T> __device__ __forceinline__ T* output_row(const CacheAttentionArgs& a, int n, int h, int row) {
  const int tok = row / a.group;
  return (T*)a.o + n * a.os.sample + tok * a.os.token + (long)(h * a.group + (row - tok * a.group)) * a.os.head;
}

// 16-byte chunk c of row r of a tile of `chunks` to a row lies at c ^ turn: eight rows of a chunk, and four rows of two, have banks of their own
template <int CHUNKS> __device__ __forceinline__ int tile_turn(int row) {
  if constexpr (CHUNKS % 8 == 0) return ((row & 3) << 1) | ((row >> 2) & 1);
  else return (row & 2) | ((row >> 2) & 1);
}

// F16 does not hold every value: of what another type wrote with exponents past 13, what exceeds 65504 is infinite.  Infinities must not get into the products, where
// nothing times them is not a number for the rows that do not see them (and for those whose probability is nothing in f16).  They are zeros there; where there were
// any, they are looked for once more behind the last key, and added to the outputs of the rows that see theirs.  (Among the products there are no registers for that.)
template <typename T> constexpr bool kHasInfinities = std::is_same<T, f16_t>::value;
constexpr unsigned kLastFiniteExponent = 13 + 127;
__device__ __forceinline__ bool may_be_infinite(unsigned exponent) { return exponent > kLastFiniteExponent && exponent < 255u; }
// how many codes of a sign are finite where some may not be: up to 3 * 2^14, 1.5 * 2^15, 0.5 * 2^16, 0
__device__ __forceinline__ unsigned finite_codes(unsigned exponent) { return exponent == 141 ? 6 : exponent == 142 ? 4 : exponent == 143 ? 2 : 1; }
__device__ __forceinline__ unsigned infinite_codes(unsigned codes, unsigned finite) { return ((codes & 0x77777777u) + (8 - finite) * 0x11111111u) & 0x88888888u; }   // bit 3 of those
__device__ __forceinline__ unsigned without_infinities(unsigned codes, unsigned finite) { return codes & ~((infinite_codes(codes, finite) >> 3) * 15u); }
__device__ __forceinline__ unsigned without_infinities(unsigned word) {   // (of two f16 values)
  return word & ((word & 0x7fffu) == 0x7c00u ? 0xffff0000u : ~0u) & ((word & 0x7fff0000u) == 0x7c000000u ? 0xffffu : ~0u);
}
// bit 7 of the bytes that are above kLastFiniteExponent, where `ones` has a 1 in them
template <typename E> __device__ __forceinline__ E past_f16(E e, E ones) { return ((e & 127 * ones) + (128 - (kLastFiniteExponent - 127)) * ones) & e & 128 * ones; }
// A lane's row sees keys up to `see`; element j of its fours of channels STEP i + first .. + 3 is o(i, j).  All lanes of the wavefront, with the same keys.
template <int NB, int STEP, typename F>
__device__ __forceinline__ void add_infinities(const CachePages& cp, const int* table, int h, int begin, int end, int see, int first, F o) {
  const unsigned values_at = 16 * NB * cp.page_tokens, exps_at = 2 * values_at + exponent_bytes(NB) * cp.page_tokens;
  auto page_of = [&](int key, int& slot) { return head_of_page(cp, table[div_rem((unsigned)key, cp.page_tokens, cp.inv_page_tokens, slot)], h); };
#pragma unroll 1
  for (int k0 = begin; k0 < end; k0 += 64) {
    const int own = k0 + (threadIdx.x & 63);
    bool any = false;
    int slot;
    if (own < end) {
      if (const unsigned char* page = page_of(own, slot))
        for (int b = 0; b < NB; ++b) any = any || may_be_infinite(page[exps_at + (unsigned)slot * exponent_bytes(NB) + b]);
    }
#pragma unroll 1
    for (unsigned long keys = __ballot(any); keys; keys &= keys - 1) {
      const int key = k0 + __builtin_ctzl(keys);
      const unsigned char* page = page_of(key, slot);
#pragma unroll
      for (int i = 0; i < 32 / STEP * NB; ++i) {
        const unsigned e = page[exps_at + (unsigned)slot * exponent_bytes(NB) + STEP * i / 32];
        const unsigned codes = *reinterpret_cast<const unsigned short*>(page + (values_at + (unsigned)slot * 16 * NB + (STEP * i + first) / 2));
        if (!may_be_infinite(e) || key > see) continue;
        const unsigned infinite = infinite_codes(codes, finite_codes(e));
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if ((infinite >> (4 * j + 3)) & 1u) o(i, j) += (codes >> (4 * j + 3)) & 1u ? -INFINITY : INFINITY;
      }
    }
  }
}

constexpr float kCacheSlack = 8.0f;   // log2 of how far a maximum may exceed the reference before that moves
// (The difference, not the sum: from 2^27 on the reference and eight more may round to the next score, whose probability of 2^16 is infinite in f16.)
__device__ __forceinline__ bool is_past(float mx, float m) {
#pragma clang fp contract(off)
  return mx - m > kCacheSlack;
}

template <int N> struct Words { unsigned w[N]; };

// ---------------------------------------------------------------- few rows
// A wavefront takes 16 rows and every fourth 32 keys of its workgroup's range by itself: S^T = K Q^T of 16x16x32 products, whose keys come straight from memory (a lane
// has 1 / 4 of a key's channels; the queries are in the same order), the softmax, and O^T += V^T P^T with the values turned in LDS.  The next 32 keys are on
// their way meanwhile.
template <typename T, int NB> constexpr int kFewWaves = sizeof(T) == 4 ? (NB <= 2 ? 3 : 2) : NB <= 4 ? 4 : 2;   // a SIMD

// EVEN: pages hold a multiple of 16 tokens, so that 16 keys lie together in one of them: its number and address are the wavefront's, not a lane's.
template <typename T, int NB, bool EVEN>
__global__ __launch_bounds__(256, (kFewWaves<T, NB>)) void cache_few_kernel(CacheLaunch launch) {
  typedef typename CacheOperand<T>::type O;
  constexpr int PIECES = CacheOperand<T>::pieces, CH = 4 * NB, ROW = 16 * NB, EXP = exponent_bytes(NB), D = 32 * NB, TILES = 2 * NB, RED = D + 4;
  constexpr int TILE_BYTES = 32 * CH * 16, JOIN_BYTES = 2 * 16 * (RED + 2) * 4, SMEM = 4 * TILE_BYTES > JOIN_BYTES ? 4 * TILE_BYTES : JOIN_BYTES;
  __shared__ __align__(16) unsigned char smem[SMEM];
  __shared__ bool s_infinite[4];
  const CacheAttentionArgs& a = launch.a;
  const CachePages& cp = a.pages;
  const CachePlan& p = launch.plan;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // workgroup id -> (sample, key head, range, row block); the ids of one XCD (id % 8) are neighbours within a sample, and row blocks share their keys
  const int per_sample = cp.heads * p.splits * p.row_blocks, n = blockIdx.x / per_sample;
  int L;
  {
    const int i = blockIdx.x - n * per_sample, per = per_sample / 8, rem = per_sample % 8, x = i % 8, j = i / 8;
    L = x * per + (x < rem ? x : rem) + j;
  }
  const int rb = L % p.row_blocks, split = L / p.row_blocks % p.splits, h = L / (p.row_blocks * p.splits);
  // pages of 32 keys; where they are the wavefront's, the first are asked for before the sample's length is known
  struct Place { int number[2], slot[2]; };          // of keys k0 and k0 + 16, or k0 + l16 and k0 + 16 + l16; no page past the range
  const int* table = cp.table + n * cp.table_stride;
  auto find_even = [&](int k0) {
    typedef const __attribute__((address_space(4))) int* uniform_t;
    Place w;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int page = div_rem((unsigned)(k0 + 16 * t), cp.page_tokens, cp.inv_page_tokens, w.slot[t]);
      w.number[t] = ((uniform_t)(uintptr_t)table)[min(page, cp.table_pages - 1)];   // (past the range: not used)
    }
    return w;
  };
  Place next;
  if constexpr (EVEN) next = find_even(split * p.range + 32 * wave);

  const CacheView view = view_of(a, n, rb * kFewRows, kFewRows);
  if (rb * kFewRows >= view.rows) return;
  const int begin = (int)min((long)split * p.range, (long)view.end), end = (int)min((long)begin + p.range, (long)view.end);
  if (split > 0 && begin >= end) return;
  const bool whole = view.end <= p.range;            // the block has one range

  // ---- queries: lane (row l16, g) has channels 8 (NB g + s) .. + 7
  const int row = rb * kFewRows + l16, row_tok = row / a.group;
  u32x4 q[NB][PIECES];
  {
    const int r = min(row, view.rows - 1), tok = r / a.group, hq = h * a.group + (r - tok * a.group);
    const T* src = (const T*)a.q + n * a.qs.sample + tok * a.qs.token + hq * a.qs.head;
#pragma unroll
    for (int s = 0; s < NB; ++s) {
      const int at = 8 * (NB * g + s);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) q[s][i] = u32x4{0, 0, 0, 0};
      if (at < cp.d) {
        if constexpr (sizeof(T) == 4) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(src + at), y = *reinterpret_cast<const f32x4*>(src + at + 4);
          unsigned w[4][3];
          split3_any(x, y, w);
#pragma unroll
          for (int i = 0; i < 3; ++i) q[s][i] = u32x4{w[0][i], w[1][i], w[2][i], w[3][i]};
        } else {
          q[s][0] = *reinterpret_cast<const u32x4*>(src + at);
        }
      }
    }
  }

  // ---- 32 keys: lane (key l16 of either half, g) has words NB g .. NB g + NB - 1 of a key's and a value's codes
  typedef typename std::conditional<EXP == 1, unsigned char, typename std::conditional<EXP == 2, unsigned short, typename std::conditional<EXP == 4, unsigned, unsigned long>::type>::type>::type E;
  typedef typename std::conditional<EXP == 8, unsigned long, unsigned>::type EW;
  struct Half { Words<NB> w[2]; EW e[2]; };          // keys, or values
  Half xk, xv;
  unsigned there = 0;                                // which of the 32 are keys
  const unsigned values_at = ROW * cp.page_tokens, exps_at = 2 * values_at;
  auto find = [&](int k0) {
    Place w;
    if constexpr (EVEN) {
      w = find_even(k0);
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = k0 + 16 * t + l16, page = div_rem((unsigned)key, cp.page_tokens, cp.inv_page_tokens, w.slot[t]);
        w.number[t] = -1;
        if (key < end) w.number[t] = table[page];
      }
    }
    return w;
  };
  auto ask = [&](Half& x, bool values, const Place& w) {
    const unsigned codes_at = values ? values_at : 0, to_exps = exps_at + (values ? EXP * cp.page_tokens : 0);
    if constexpr (EVEN) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        // (no page: none of them is a key, and what page 0 has instead is taken for zeros)
        const unsigned char* page = head_of_page(cp, (unsigned)w.number[t] < (unsigned)cp.pages ? w.number[t] : 0, h);
        x.w[t] = *reinterpret_cast<const Words<NB>*>(page + (codes_at + (unsigned)w.slot[t] * ROW + (l16 * ROW + 4 * NB * g)));
        x.e[t] = *reinterpret_cast<const E*>(page + (to_exps + (unsigned)w.slot[t] * EXP + l16 * EXP));
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const unsigned char* page = head_of_page(cp, w.number[t], h);
        x.w[t] = Words<NB>{};
        x.e[t] = 0;
        if (page) {
          x.w[t] = *reinterpret_cast<const Words<NB>*>(page + (codes_at + (unsigned)w.slot[t] * ROW + 4 * NB * g));
          x.e[t] = *reinterpret_cast<const E*>(page + (to_exps + (unsigned)w.slot[t] * EXP));
        }
      }
    }
  };
  auto keys_of = [&](const Place& w, int k0) {
    if constexpr (EVEN) {
      const unsigned here = end - k0 >= 32 ? ~0u : (1u << (end - k0)) - 1;
      return here & (((unsigned)w.number[0] < (unsigned)cp.pages ? 0xffffu : 0u) | ((unsigned)w.number[1] < (unsigned)cp.pages ? 0xffff0000u : 0u));
    }
    else return ((unsigned)__ballot((unsigned)w.number[0] < (unsigned)cp.pages) & 0xffffu) | (unsigned)__ballot((unsigned)w.number[1] < (unsigned)cp.pages) << 16;
  };
  // what is no key: zeros (its exponents may be anything)
  auto cut = [&](Half& x) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (!((there >> (16 * t + l16)) & 1u)) {
        x.w[t] = Words<NB>{};
        x.e[t] = 0;
      }
  };
  auto unit = [&](EW e, int s) {                     // the power of two of word NB g + s
    const int block = NB % 4 == 0 ? NB / 4 * g + s / 4 : NB == 2 ? g / 2 : (NB * g + s) / 4;
    if constexpr (NB == 1) return unit_of((unsigned)e);
    unsigned half = (unsigned)e;
    if constexpr (NB > 4) half = block >= 4 ? (unsigned)(e >> 32) : half;
    return unit_of((half >> (8 * (block & 3))) & 255u);
  };

  u32x4* tile = reinterpret_cast<u32x4*>(smem + wave * TILE_BYTES);   // [32 keys][CH] chunks of eight channels
  // lane i of 16 reads four channels of key 4 g + i / 4, and gets channel i of the four keys
  constexpr int VB = CH % 8 == 0 ? 4 : 2;
  int vb[VB];
#pragma unroll
  for (int i = 0; i < VB; ++i) {
    const int r = 4 * g + (l16 >> 2), c = 2 * i + ((l16 & 3) >> 1);
    vb[i] = (r * CH + (c ^ tile_turn<CH>(r))) * 16 + (l16 & 1) * 8;
  }

  const float c = a.scale * 1.4426950408889634f;
  // keys that the lane's row sees, and that all rows of the block see
  const int see = a.causal ? view.len - view.count + row_tok : view.len - 1;
  const int all_see = a.causal ? view.len - view.count + rb * kFewRows / a.group : view.len - 1;
  f32x4 o[TILES];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < TILES; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Where some rows do not see some of the keys: a block of values that is not a number is zero to the products (its codes are), as nothing times it is not
  // nothing, and reaches the rows that see it here.
  auto take_out = [&](int k0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      bool any = false;
#pragma unroll
      for (int b = 0; b < NB; ++b) any = any || ((xv.e[t] >> (8 * b)) & 255u) == 255u;
      if (!__ballot(any)) continue;
#pragma unroll 1
      for (int i = 0; i < 16; ++i) {
        const unsigned lo = __builtin_amdgcn_readlane((int)xv.e[t], i), hi = __builtin_amdgcn_readlane((int)((unsigned long)xv.e[t] >> 32), i);
#pragma unroll
        for (int b = 0; b < NB; ++b)
          if ((((b < 4 ? lo : hi) >> (8 * (b & 3))) & 255u) == 255u && k0 + 16 * t + i <= see) o[2 * b] = o[2 * b + 1] = f32x4{NAN, NAN, NAN, NAN};
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
        if (((xv.e[t] >> (8 * b)) & 255u) == 255u) xv.e[t] &= ~((EW)255 << (8 * b));
    }
  };

  bool infinite = false;                             // whether there were infinities
  auto take_out_infinities = [&]() {                 // of the tile
    infinite = true;
    int at = lane;
    asm volatile("" : "+v"(at));                     // (not worked out ahead: there are no registers for that)
#pragma unroll 1
    for (; at < 32 * CH * 4; at += 64) reinterpret_cast<unsigned*>(tile)[at] = without_infinities(reinterpret_cast<const unsigned*>(tile)[at]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };

  auto work = [&](int k0) {                          // and asks for the wavefront's next keys as soon as there is room for them
    const bool more = k0 + 128 < end;
    f32x4 s[2];
    if constexpr (EVEN) {
      if (there != ~0u) { cut(xk); cut(xv); }
    }
    if (k0 + 31 > all_see) take_out(k0);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NB; ++w) {
        const u32x4 k = widen<O>(xk.w[t].w[w], unit(xk.e[t], w));
#pragma unroll
        for (int i = 0; i < PIECES; ++i) s[t] = Mma<O>::m16(k, q[w][i], s[t]);
      }
    }
    if (more) ask(xk, false, next);
    bool past = false;
    if constexpr (kHasInfinities<T>) {
      constexpr EW ones = (EW)0x0101010101010101ul >> (8 * (sizeof(EW) - NB));
      past = __ballot((past_f16<EW>(xv.e[0], ones) | past_f16<EW>(xv.e[1], ones)) != 0) != 0;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (the tile has been read)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 16 * t + l16;
#pragma unroll
      for (int w = 0; w < NB; ++w) tile[r * CH + ((NB * g + w) ^ tile_turn<CH>(r))] = widen<O>(xv.w[t].w[w], unit(xv.e[t], w));
    }
    if (more) ask(xv, true, next);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (past) take_out_infinities();
    if (there != ~0u || k0 + 31 > all_see) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = 16 * t + 4 * g + r;
          if (!((there >> at) & 1u) || k0 + at > see) s[t][r] = -INFINITY;
        }
    }
    {
      // the products are rounded as the reference is, so that the largest is at most the reference, however large both are
#pragma clang fp contract(off)
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[t][r] = s[t][r] * c;
          mx = __builtin_elementwise_maximum(mx, s[t][r]);
        }
      if (__ballot(is_past(mx, m))) {               // all lanes of a row move together
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const bool moves = is_past(mx, m);
        const float factor = moves ? __builtin_amdgcn_exp2f(m - mx) : 1.f;
        m = moves ? mx : m;
        l = l * factor;
#pragma unroll
        for (int i = 0; i < TILES; ++i) o[i] = o[i] * factor;
      }
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[t][r] = __builtin_amdgcn_exp2f(s[t][r] - ref);
          l = l + s[t][r];
        }
    }
    u32x4 pr[PIECES];                                // probabilities of keys 4 g .. + 3 of either half
    if constexpr (PIECES == 3) {
      unsigned w[4][3];
      split3(s[0][0], s[0][1], w[0]); split3(s[0][2], s[0][3], w[1]); split3(s[1][0], s[1][1], w[2]); split3(s[1][2], s[1][3], w[3]);
#pragma unroll
      for (int i = 0; i < 3; ++i) pr[i] = u32x4{w[0][i], w[1][i], w[2][i], w[3][i]};
    } else {
      pr[0] = u32x4{pack2<O>(s[0][0], s[0][1]), pack2<O>(s[0][2], s[0][3]), pack2<O>(s[1][0], s[1][1]), pack2<O>(s[1][2], s[1][3])};
    }
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* tptr_t;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const unsigned char* at = reinterpret_cast<const unsigned char*>(tile) + vb[i % VB] + i / VB * VB * 32;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)at));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)(at + 16 * CH * 16)));
#pragma unroll
      for (int j = 0; j < PIECES; ++j) o[i] = Mma<O>::m16(u32x4{lo.x, lo.y, hi.x, hi.y}, pr[j], o[i]);
    }
  };

  int k0 = begin + 32 * wave;
  if (k0 < end) {
    if (!EVEN) next = find(k0);
    ask(xk, false, next);
    ask(xv, true, next);
  }
  while (k0 < end) {
    there = keys_of(next, k0);
    next = find(k0 + 128);
    work(k0);
    k0 += 128;
  }

  // ---- the wavefronts' sums are joined: 2 and 3 to 0 and 1, then 1 to 0.  A lane has channels 16 i + 4 g .. + 3 of its row
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (kHasInfinities<T> && lane == 0) s_infinite[wave] = infinite;
  float* s_o = reinterpret_cast<float*>(smem);                       // [2][16][RED]
  float2* s_ml = reinterpret_cast<float2*>(s_o + 2 * 16 * RED);      // [2][16]
#pragma unroll
  for (int step = 2; step >= 1; step /= 2) {
    __syncthreads();
    if (wave >= step && wave < 2 * step) {
      const int w = wave - step;
      if (g == 0) s_ml[w * 16 + l16] = make_float2(m, l);
#pragma unroll
      for (int i = 0; i < TILES; ++i) *reinterpret_cast<f32x4*>(s_o + (w * 16 + l16) * RED + 16 * i + 4 * g) = o[i];
    }
    __syncthreads();
    if (wave < step) {
      const float2 e = s_ml[wave * 16 + l16];
      const float top = fmaxf(m, e.x), own = cache_weight(m, top), other = cache_weight(e.x, top);
      m = top;
      l = l * own + e.y * other;
#pragma unroll
      for (int i = 0; i < TILES; ++i) o[i] = o[i] * own + *reinterpret_cast<const f32x4*>(s_o + (wave * 16 + l16) * RED + 16 * i + 4 * g) * other;
    }
  }
  if (wave > 0) return;
  if constexpr (kHasInfinities<T>) {
    if (s_infinite[0] | s_infinite[1] | s_infinite[2] | s_infinite[3]) add_infinities<NB, 16>(cp, table, h, begin, end, see, 4 * g, [&](int i, int j) -> float& { return ((float*)&o[i])[j]; });
  }
  if (row >= view.rows) return;
  if (whole) {
    T* dst = output_row<T>(a, n, h, row);
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int i = 0; i < TILES; ++i) store_four<T>(dst, 16 * i + 4 * g, cp.d, o[i] * inv);
  } else {
    const int br = p.block_rows();
    const long at = ((((long)n * cp.heads + h) * p.row_blocks + rb) * p.splits + split) * br + l16;
    if (g == 0) launch.ml[at] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < TILES; ++i) *reinterpret_cast<f32x4*>(launch.part + at * D + 16 * i + 4 * g) = o[i];
  }
}

// ---------------------------------------------------------------- many rows
// The four wavefronts of a workgroup take 32 rows each of the same tiles of KT keys and values, which the workgroup widens into LDS while it works on the tile
// before; the codes of the tile after that are on their way meanwhile.  Per 32 keys a wavefront forms S^T = K Q^T of 32x32x16 products (keys along the accumulator's
// registers, one row a lane), the softmax, and O^T += V^T P^T with the probabilities as they are in their registers: an accumulator's keys of lane half lk
// are 8 (r / 4) + 4 lk + r % 4, so V^T is read from LDS in that order of keys, transposed on the way.
__host__ __device__ constexpr bool has_halves(int nb) { return nb != 4; }   // (measured beside the rule in kernels_cache.hip)

// KW: 1, or 2 where there are few blocks: eight wavefronts, of which the first and the last four take half of a tile's keys each, joined at the end.
template <int NB, int KW>
struct ManyForm {
  static constexpr int D = 32 * NB, KT = NB <= 4 || KW == 2 ? 64 : 32, CH = 4 * NB, TILE = KT * CH, WAVES = KW == 2 ? 2 : NB <= 1 ? 4 : NB == 2 ? 3 : 2;   // (TILE: chunks of a tile)
  static constexpr bool TIGHT = NB >= 7;             // queries and outputs leave few registers
  static constexpr bool PAIR = NB >= (KW == 2 ? 5 : 3);   // a thread widens a block of 32 channels of a key and of its value, else of one of them
};

// every LDS access of this wavefront is done, and so for the others: codes on their way are not waited for
__device__ __forceinline__ void sync_tiles_of_cache() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// SMALL: for pages of any size; else they hold a tile or more.
template <typename T, int NB, int KW, bool SMALL>
__global__ __launch_bounds__(256 * KW, (ManyForm<NB, KW>::WAVES)) void cache_many_kernel(CacheLaunch launch) {
  typedef ManyForm<NB, KW> F;
  constexpr int CH = F::CH, D = F::D, KT = F::KT, NS = KT / 32 / KW, QS = CH / 2, TILE = F::TILE, ROW = 16 * NB, EXP = exponent_bytes(NB);
  constexpr int GP = CH % 8 == 0 ? 8 : 4;            // chunks that are exchanged among each other
  constexpr bool TIGHT = F::TIGHT;
  __shared__ __align__(16) u32x4 s_k[4 * TILE];      // two tiles of keys, and two of values
  u32x4* const s_v = s_k + 2 * TILE;
  // what is out of the ordinary in a tile: bits of the keys whose values are not a number, by block; whether there are any (1), or keys without a page (2); those
  constexpr int FLAGS = 2 * NB, GONE = FLAGS + 1, BAD = FLAGS + 3;
  __shared__ unsigned s_bad[3][BAD];
  __shared__ bool s_infinite;                        // whether there were infinities
  const CacheAttentionArgs& a = launch.a;
  const CachePages& cp = a.pages;
  const CachePlan& p = launch.plan;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, lk = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6) % 4, kw = __builtin_amdgcn_readfirstlane(tid >> 6) / 4;

  // workgroup id -> (sample, key head, range, row block), as for few rows
  const int per_sample = cp.heads * p.splits * p.row_blocks, n = blockIdx.x / per_sample;
  int L;
  {
    const int i = blockIdx.x - n * per_sample, per = per_sample / 8, rem = per_sample % 8, x = i % 8, j = i / 8;
    L = x * per + (x < rem ? x : rem) + j;
  }
  const int rb = L % p.row_blocks, split = L / p.row_blocks % p.splits, h = L / (p.row_blocks * p.splits), row0 = rb * kManyRows;
  const CacheView view = view_of(a, n, row0, kManyRows);
  if (row0 >= view.rows) return;
  const int begin = (int)min((long)split * p.range, (long)view.end), end = (int)min((long)begin + p.range, (long)view.end);
  if (split > 0 && begin >= end) return;
  const bool whole = view.end <= p.range;
  const int tiles = (end - begin + KT - 1) / KT;

  // ---- queries: chunk 2 s + lk of the lane's row
  const int row = row0 + wave * 32 + l32, first_row = row0 + wave * 32;
  const bool idle = first_row >= view.rows;          // a wavefront past the last row only widens
  u32x4 q[QS];
  {
    const int r = min(row, view.rows - 1), tok = r / a.group, hq = h * a.group + (r - tok * a.group);
    const T* src = (const T*)a.q + n * a.qs.sample + tok * a.qs.token + hq * a.qs.head;
#pragma unroll
    for (int s = 0; s < QS; ++s) {
      const int at = 8 * (2 * s + lk);
      q[s] = u32x4{0, 0, 0, 0};
      if (at < cp.d) q[s] = *reinterpret_cast<const u32x4*>(src + at);
    }
  }
  // keys up to which the lane's row, all rows of the wavefront, and its last row see
  const int behind = view.len - view.count;
  const int see = a.causal ? behind + row / a.group : view.len - 1, all_see = a.causal ? behind + first_row / a.group : view.len - 1;
  const int last_see = a.causal ? behind + min(first_row + 31, view.rows - 1) / a.group : view.len - 1;

  // ---- tiles.  A thread widens a block of 32 channels of a key, of a value, or of both.  Its place goes from tile to tile: page numbers are asked for a tile before
  // they are needed, and with large pages only where the last one ends.
  constexpr int ITEMS = F::PAIR ? 2 : 1;
  constexpr unsigned kGone = 256;                    // instead of an exponent: there is no page
  struct Mine { int key, block; bool live, values; };
  auto mine_of = [&]() {
    int t = tid;
    if constexpr (TIGHT) asm volatile("" : "+v"(t));   // (worked out again wherever it is needed: there are no registers to keep it)
    const bool second = !F::PAIR && t >= KT * NB;
    if (second) t -= KT * NB;
    return Mine{t / NB, t % NB, t < KT * NB, second};
  };
  const int* table = cp.table + n * cp.table_stride;
  const unsigned char* page = nullptr;
  int slot = 0, page_index = 0, next_number = -1, next_slot = 0;
  u32x4 codes[ITEMS];
  unsigned held[ITEMS];
  auto number_at = [&](int index) { return index < cp.table_pages ? table[index] : -1; };
  auto first_place = [&]() {
    const int key = mine_of().key;
    page_index = div_rem((unsigned)(begin + key), cp.page_tokens, cp.inv_page_tokens, slot);
    page = head_of_page(cp, number_at(page_index), h);
    if constexpr (SMALL) next_number = number_at(div_rem((unsigned)(begin + KT + key), cp.page_tokens, cp.inv_page_tokens, next_slot));
    else next_number = number_at(page_index + 1);
  };
  auto next_place = [&](int j) {                     // from tile j - 1 to tile j
    if constexpr (SMALL) {
      const int key = mine_of().key;
      page = head_of_page(cp, next_number, h);
      slot = next_slot;
      next_number = number_at(div_rem((unsigned)(begin + (j + 1) * KT + key), cp.page_tokens, cp.inv_page_tokens, next_slot));
    } else {
      slot += KT;
      if (slot >= (int)cp.page_tokens) {
        slot -= (int)cp.page_tokens;
        ++page_index;
        page = head_of_page(cp, next_number, h);
        next_number = number_at(page_index + 1);
      }
    }
  };
  const unsigned values_at = ROW * cp.page_tokens, exps_at = 2 * values_at, value_exps_at = EXP * cp.page_tokens;
  auto ask = [&]() {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      codes[i] = u32x4{0, 0, 0, 0};
      held[i] = kGone;
    }
    const Mine x = mine_of();
    if (x.live && page) {
      const unsigned char *c = page + (16 * x.block + (unsigned)slot * ROW), *e = page + (exps_at + x.block + (unsigned)slot * EXP);
      if constexpr (F::PAIR) {
        codes[0] = *reinterpret_cast<const u32x4*>(c);
        codes[ITEMS - 1] = *reinterpret_cast<const u32x4*>(c + values_at);
        held[0] = *e;
        held[ITEMS - 1] = e[value_exps_at];
      } else {
        codes[0] = *reinterpret_cast<const u32x4*>(c + (x.values ? values_at : 0u));
        held[0] = e[x.values ? value_exps_at : 0u];
      }
    }
  };
  auto fill = [&](int j) {
    const int left = end - begin - j * KT;           // keys of the tile
    const Mine x = mine_of();
    const int key = x.key, block = x.block;
    if (!x.live) return;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const bool values = F::PAIR ? i == 1 : x.values;
      if (left < KT && key >= left) {                // (a page has room for keys that are not there; their exponents may be anything)
        codes[i] = u32x4{0, 0, 0, 0};
        held[i] = 0;
      }
      if (held[i] > (kHasInfinities<T> ? kLastFiniteExponent : 254u)) {
        const bool gone = held[i] == kGone, bad = held[i] == 255u && a.causal && values;   // (as take_out does for few rows)
        if (gone ? !values && block == 0 : bad) {
          atomicOr(&s_bad[j % 3][(gone ? GONE : 2 * block) + (key >> 5)], 1u << (key & 31));
          atomicOr(&s_bad[j % 3][FLAGS], gone ? 2u : 1u);
        }
        if (gone || bad) held[i] = 0;
        if (kHasInfinities<T> && values && may_be_infinite(held[i])) {
          s_infinite = true;
          unsigned most = finite_codes(held[i]);
          if constexpr (TIGHT) asm volatile("" : "+v"(most));   // (2 x 4096x4096 of 16 heads of 256 680 us, else 710)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            __builtin_amdgcn_sched_barrier(0);
            codes[i][c] = without_infinities(codes[i][c], most);
          }
        }
      }
      u32x4* to = (values ? s_v : s_k) + (j & 1) * TILE + key * CH;
      const float unit = unit_of(held[i]);
#pragma unroll
      for (int c = 0; c < 4; ++c) to[(4 * block + c) ^ tile_turn<CH>(key)] = widen<T>(codes[i][c], unit);
    }
  };
  unsigned long there = 0;                           // which of a tile's keys are there

  // ---- where a lane reads its operands (chunks, and bytes, of a tile)
  int kb[GP / 2];
#pragma unroll
  for (int s = 0; s < GP / 2; ++s) kb[s] = l32 * CH + ((2 * s + lk) ^ tile_turn<CH>(l32));
  int vb[GP / 4];
#pragma unroll
  for (int i = 0; i < GP / 4; ++i) {   // channels 16 (l32 / 16) + 4 (lane % 4) .. + 3 of key 4 lk + lane / 4 % 4, of which the lane gets channel l32 of four keys
    const int r = 4 * lk + ((lane >> 2) & 3), c = 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    vb[i] = (r * CH + (c ^ tile_turn<CH>(r))) * 16 + (lane & 1) * 8;
  }

  f32x16 o[NB], s[NS];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int dt = 0; dt < NB; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  const float c = a.scale * 1.4426950408889634f;

  auto scores = [&](const u32x4* tk, int k0) {
    int k_at[GP / 2];
    k_at[0] = kb[0];
    if constexpr (TIGHT) asm volatile("" : "+v"(k_at[0]));
#pragma unroll
    for (int i = 1; i < GP / 2; ++i) k_at[i] = GP == 8 ? k_at[0] ^ 2 * i : kb[i];   // (eight chunks are exchanged by their three bits)
#pragma unroll
    for (int ns = 0; ns < NS; ++ns) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[ns][r] = 0.f;
#pragma unroll
      for (int st = 0; st < QS; ++st) {
        s[ns] = Mma<T>::m32(tk[k_at[st % (GP / 2)] + st / (GP / 2) * GP + (kw * NS + ns) * 32 * CH], q[st], s[ns]);
      }
    }
#pragma unroll
    for (int ns = 0; ns < NS; ++ns) {
      const int at = k0 + 32 * (kw * NS + ns);
      const unsigned is_there = (unsigned)(there >> (32 * (kw * NS + ns)));
      if (is_there != ~0u || at + 31 > all_see) {
        const int seen = see - at + 1;
        const unsigned b = (is_there & (seen >= 32 ? ~0u : seen <= 0 ? 0u : (1u << seen) - 1)) >> (4 * lk);
#pragma unroll
        for (int r = 0; r < 16; ++r) {   // -inf where the bit is not set, in two instructions: the bit spread over the word, and a choice by it
          const unsigned is = (unsigned)((int)(b << (31 - 8 * (r / 4) - r % 4)) >> 31);
          s[ns][r] = __uint_as_float((is & __float_as_uint(s[ns][r])) | (~is & 0xff800000u));
        }
      }
    }
  };
  // The reference is a rounded product.  From 2^24 on a fused multiply-add would find the largest score half a step of the reference away from it, 1 and more: there
  // the products are rounded like the reference, and then subtracted.
  bool far = false;   // (of any of the wavefront's rows)
  auto round_and_subtract = [&](float ref) {
#pragma clang fp contract(off)
#pragma unroll
    for (int ns = 0; ns < NS; ++ns)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = s[ns][r] * c;
        s[ns][r] = x - ref;
      }
  };
  auto maximum = [](float x, float y) { return __builtin_elementwise_maximum(x, y); };
  auto softmax = [&]() {
    float mx = maximum(maximum(s[0][0], s[0][1]), s[0][2]);
#pragma unroll
    for (int i = 3; i + 1 < 16 * NS; i += 2) mx = maximum(maximum(mx, s[i / 16][i % 16]), s[(i + 1) / 16][(i + 1) % 16]);
    mx = maximum(mx, s[NS - 1][15]);
    mx = half_max(mx) * c;
    const bool moves = is_past(mx, m);
    if (__ballot(moves)) {
      const float to = moves ? mx : m, factor = moves ? __builtin_amdgcn_exp2f(m - mx) : 1.f;
      m = to;
      far = __ballot(fabsf(m) >= 0x1p24f && m != -INFINITY) != 0;
      l *= factor;
#pragma unroll
      for (int dt = 0; dt < NB; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= factor;
    }
    float ref = m == -INFINITY ? 0.f : m, by = c;
    if (far) {
      round_and_subtract(ref);
      by = 1.f;
      ref = 0.f;
    }
#pragma unroll
    for (int ns = 0; ns < NS; ++ns)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[ns][r] = __builtin_amdgcn_exp2f(fmaf(s[ns][r], by, -ref));
        l += s[ns][r];
      }
  };
  auto values = [&](const unsigned char* tv) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* tptr_t;
    int v_at[GP / 4];
    v_at[0] = vb[0];
    if constexpr (TIGHT) asm volatile("" : "+v"(v_at[0]));
#pragma unroll
    for (int i = 1; i < GP / 4; ++i) v_at[i] = GP == 8 ? v_at[0] ^ 64 * i : vb[i];
#pragma unroll
    for (int i = 0; i < 2 * NS; ++i) {               // 16 keys
      u32x4 pr;                                      // the one rounding inside the operator: probabilities as operands of T
#pragma unroll
      for (int e = 0; e < 4; ++e) pr[e] = pack2<T>(s[i / 2][8 * (i % 2) + 2 * e], s[i / 2][8 * (i % 2) + 2 * e + 1]);
#pragma unroll
      for (int dt = 0; dt < NB; ++dt) {
        const unsigned char* at = tv + v_at[dt % (GP / 4)] + dt / (GP / 4) * GP * 16 + (kw * 2 * NS + i) * 16 * CH * 16;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)at));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)(at + 8 * CH * 16)));
        o[dt] = Mma<T>::m32(u32x4{lo.x, lo.y, hi.x, hi.y}, pr, o[dt]);
      }
    }
  };

  if (tid < 3 * BAD) s_bad[0][tid] = 0;
  if (kHasInfinities<T> && tid == 0) s_infinite = false;
  if (tiles > 0) {
    first_place();
    ask();
    sync_tiles_of_cache();                           // (s_bad is clear)
    fill(0);
    next_place(1);
    ask();
  }
  for (int j = 0; j < tiles; ++j) {
    sync_tiles_of_cache();                           // the tile is there, and every wavefront is done with the other buffer
    if (j + 1 < tiles) {
      fill(j + 1);
      next_place(j + 2);
      ask();
    }
    if (tid < BAD) s_bad[(j + 2) % 3][tid] = 0;
    const int k0 = begin + j * KT, left = end - k0;
    if (idle || k0 + 32 * kw * NS > last_see) continue;
    there = left >= 64 ? ~0ul : (1ul << left) - 1;
    const unsigned* bad = s_bad[j % 3];
    const unsigned flags = __builtin_amdgcn_readfirstlane((int)bad[FLAGS]);
    if (flags & 2u) there &= ~((unsigned)__builtin_amdgcn_readfirstlane((int)bad[GONE]) | (unsigned long)(unsigned)__builtin_amdgcn_readfirstlane((int)bad[GONE + 1]) << 32);
    if (flags & 1u) {
#pragma unroll
      for (int dt = 0; dt < NB; ++dt)
#pragma unroll 1
        for (int i = 0; i < KT; ++i)
          if (((bad[2 * dt + (i >> 5)] >> (i & 31)) & 1u) && k0 + i <= see)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] = NAN;
    }
    __builtin_amdgcn_sched_barrier(0);
    scores(s_k + (j & 1) * TILE, k0);
    softmax();
    values(reinterpret_cast<const unsigned char*>(s_v + (j & 1) * TILE));
  }

  // ---- output.  A lane holds channels 32 dt + 8 g + 4 lk .. + 3 of its row
  l += __shfl_xor(l, 32);
  if constexpr (KW == 2) {                           // the last four wavefronts' sums to the first four, through the tiles' memory
    __shared__ float2 s_ml[kManyRows];
    f32x4* s_o = reinterpret_cast<f32x4*>(s_k) + (wave * 32 + l32) * (D / 4);
    sync_tiles_of_cache();
    if (kw == 1) {
      if (lk == 0) s_ml[wave * 32 + l32] = make_float2(m, l);
#pragma unroll
      for (int dt = 0; dt < NB; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) s_o[(8 * dt + 2 * g + lk) ^ (l32 & 7)] = f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
    }
    sync_tiles_of_cache();
    if (kw == 1) return;
    const float2 e = s_ml[wave * 32 + l32];
    const float top = fmaxf(m, e.x), own = cache_weight(m, top), other = cache_weight(e.x, top);
    m = top;
    l = l * own + e.y * other;
#pragma unroll
    for (int dt = 0; dt < NB; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 x = s_o[(8 * dt + 2 * g + lk) ^ (l32 & 7)];
#pragma unroll
        for (int r = 0; r < 4; ++r) o[dt][4 * g + r] = o[dt][4 * g + r] * own + x[r] * other;
      }
  }
  if constexpr (kHasInfinities<T>) {
    if (tiles > 0 && !idle && s_infinite) add_infinities<NB, 8>(cp, table, h, begin, end, see, 4 * lk, [&](int i, int j) -> float& { return ((float*)&o[i / 4])[i % 4 * 4 + j]; });
  }
  if (row >= view.rows) return;
  if (whole) {
    T* dst = output_row<T>(a, n, h, row);
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int dt = 0; dt < NB; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) store_four<T>(dst, 32 * dt + 8 * g + 4 * lk, cp.d, f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]} * inv);
  } else {
    const long at = ((((long)n * cp.heads + h) * p.row_blocks + rb) * p.splits + split) * p.block_rows() + wave * 32 + l32;
    if (lk == 0) launch.ml[at] = make_float2(m, l);
    float* dst = launch.part + at * D + 4 * lk;
#pragma unroll
    for (int dt = 0; dt < NB; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4*>(dst + 32 * dt + 8 * g) = f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
  }
}

// o = sum_s part_s 2^(m_s - M) / sum_s l_s 2^(m_s - M) for the rows whose keys were several ranges (`total` of all key heads, `bq` a block).  A thread takes four
// channels of a row and every groups-th range, eight at a time; the groups of a row are joined in order.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheLaunch launch, int bq, int groups, unsigned total) {
  constexpr int QUADS = D / 4, UNITS = 256 / QUADS, B = 8;
  __shared__ f32x4 s_num[UNITS][QUADS];
  __shared__ float2 s_ml[UNITS];
  const CacheAttentionArgs& a = launch.a;
  const CachePlan& p = launch.plan;
  const int unit = threadIdx.x / QUADS, quad = threadIdx.x % QUADS, g = unit % groups, in_block = UNITS / groups, br = p.block_rows();
  for (unsigned r0 = blockIdx.x * in_block; r0 < total; r0 += gridDim.x * in_block) {
    const unsigned r = min(r0 + unit / groups, total - 1), nh = r / p.rows;           // row among those of all key heads, its sample and key head
    const int row = (int)(r - nh * p.rows), n = nh / a.pages.heads, h = nh - n * a.pages.heads, rb = row / bq, in = row - rb * bq;
    const CacheView view = view_of(a, n, rb * bq, bq);
    const int ranges = row < view.rows && view.end > p.range ? (view.end + p.range - 1) / p.range : 0;
    const long pb = ((long)nh * p.row_blocks + rb) * p.splits;
    const bool there = unit < in_block * groups && r0 + unit / groups < total && ranges > 0;
    float top = -INFINITY, den = 0.f;
    f32x4 num{0.f, 0.f, 0.f, 0.f};
    auto join = [&](float m, float l, f32x4 v) {
      const float now = fmaxf(top, m), keep = cache_weight(top, now), f = cache_weight(m, now);
      den = den * keep + l * f;
      num = num * keep + v * f;
      top = now;
    };
    if (there && quad * 4 < a.pages.d) {
      for (int s0 = g; s0 < ranges; s0 += B * groups) {
        float2 e[B];
        f32x4 v[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
          const long at = (pb + min(s0 + b * groups, ranges - 1)) * br + in;
          e[b] = launch.ml[at];
          v[b] = *reinterpret_cast<const f32x4*>(launch.part + at * D + quad * 4);
        }
#pragma unroll
        for (int b = 0; b < B; ++b)
          if (s0 + b * groups < ranges) join(e[b].x, e[b].y, v[b]);
      }
    }
    if (groups > 1) {
      if (unit < UNITS) {
        s_num[unit][quad] = num;
        if (quad == 0) s_ml[unit] = make_float2(top, den);
      }
      __syncthreads();
      if (g == 0 && there)
        for (int i = 1; i < groups; ++i) join(s_ml[unit + i].x, s_ml[unit + i].y, s_num[unit + i][quad]);
      __syncthreads();   // (read before the next rows' are written)
    }
    if (g == 0 && there) store_four<T>(output_row<T>(a, n, h, row), quad * 4, a.pages.d, num * (den == 0.f ? 0.f : 1.f / den));
  }
}

template <typename T, int NB, int KW>
void cache_launch_many(const CacheLaunch& l, dim3 grid, hipStream_t s) {
  if (l.a.pages.page_tokens < ManyForm<NB, KW>::KT) hipLaunchKernelGGL((cache_many_kernel<T, NB, KW, true>), grid, dim3(256 * KW), 0, s, l);
  else hipLaunchKernelGGL((cache_many_kernel<T, NB, KW, false>), grid, dim3(256 * KW), 0, s, l);
}

template <typename T, int NB>
int cache_attention_width(const CacheLaunch& l, hipStream_t s) {
  const CachePlan& p = l.plan;
  const int heads = l.a.pages.heads;
  const dim3 grid((unsigned)((long)l.a.n * heads * p.row_blocks * p.splits));
  const bool even = l.a.pages.page_tokens % 16 == 0;   // (us, the wavefront's places / a lane's: 4 x 32768 tokens of 30 heads of 64 in pages of 16 64 / 78, of 48 64 / 76, 8 of 128 38 / 40)
  if (!p.few) {
    if constexpr (sizeof(T) == 2) {
      if (!p.halves) cache_launch_many<T, NB, 1>(l, grid, s);
      else if constexpr (has_halves(NB)) cache_launch_many<T, NB, 2>(l, grid, s);
    }
  } else if (even) {
    hipLaunchKernelGGL((cache_few_kernel<T, NB, true>), grid, dim3(256), 0, s, l);
  } else {
    hipLaunchKernelGGL((cache_few_kernel<T, NB, false>), grid, dim3(256), 0, s, l);
  }
  WMDEC_HIP(hipGetLastError());
  if (p.splits > 1) {
    constexpr int units = 256 / (8 * NB);
    int groups = 1;
    while (groups * 2 <= units && groups * 8 < p.splits) groups *= 2;
    const long total = (long)l.a.n * heads * p.rows, in_block = units / groups, most = 8192;   // rows (below 2^26: cache_attention_fits); rows and most workgroups of a launch
    hipLaunchKernelGGL((cache_join_kernel<T, 32 * NB>), dim3((unsigned)std::min(most, (total + in_block - 1) / in_block)), dim3(256), 0, s, l, p.bq(), groups, (unsigned)total);
    WMDEC_HIP(hipGetLastError());
  }
  return WMDEC_OK;
}

template <typename T>
int cache_attention_launch(const CacheLaunch& l, hipStream_t s) {
  switch (l.plan.nb) {
    case 1: return cache_attention_width<T, 1>(l, s);
    case 2: return cache_attention_width<T, 2>(l, s);
    case 3: return cache_attention_width<T, 3>(l, s);
    case 4: return cache_attention_width<T, 4>(l, s);
    case 5: return cache_attention_width<T, 5>(l, s);
    case 6: return cache_attention_width<T, 6>(l, s);
    case 7: return cache_attention_width<T, 7>(l, s);
    default: return cache_attention_width<T, 8>(l, s);
  }
}
extern template int cache_attention_launch<f16_t>(const CacheLaunch&, hipStream_t);
extern template int cache_attention_launch<bf16_t>(const CacheLaunch&, hipStream_t);
extern template int cache_attention_launch<float>(const CacheLaunch&, hipStream_t);

}  // namespace wmdec
