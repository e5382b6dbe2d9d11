// A cache of keys and values in four bits: states are rounded to it as they are written, and read back.  (Attention to it: cache_device.hpp.)
//
// Bound by HBM: 16-bit states are 3.8 times what is held of them, so the dense side counts.  A wavefront takes tokens of one head: its reads of the
// states are whole rows of a head, what it writes of a page lies together, and neighbouring wavefronts have the next heads of the same tokens.  A lane has 16 bytes of a
// state; the four lanes of a block (eight in fp32) find its largest magnitude among themselves.
// us on inputs that are not the call's before: 32768 tokens of 8 heads of 128 read back in bf16 26.8 = 6.3 TB/s (a copy reaches 5.1 to 5.4), written and read back 63; a frame of
// 5400 tokens of 30 heads of 64 and its twin written and read back 43 = 4.8 TB/s; rows that are no whole pieces of 64 bytes run at half of that (27962 of 30 of 40 read back 64).
// Steps, reading 32768 / writing and reading two frames: 40.9, 54.6; states that are whole pieces pass by the caches 27.4, 45 (else a kernel ends with waiting for what lies in
// the L2s; codes that pass by them too make the pair 55); two tokens of a lane under way, not four or eight 26.8, 43.  Neighbouring heads on one XCD: no difference.
#include <algorithm>
#include <cmath>

#include "cache_device.hpp"

namespace wmdec {

template int cache_attention_launch<f16_t>(const CacheLaunch&, hipStream_t);

namespace {

constexpr int kSteps = 2;   // tokens of a lane, on their way together

struct TokenParams { CacheTokens a; int chunks; unsigned units; };   // units: (sample, chunk of tokens, head), a wavefront each

// A lane has 16 bytes of a state; lanes of a token, tokens of a wavefront at a time.
template <typename T> constexpr int kLaneChannels = 16 / (int)sizeof(T);
__host__ __device__ constexpr int lanes_of(int nb, int channels) { return 32 / channels * nb; }
__host__ __device__ constexpr int tokens_abreast(int nb, int channels) { return 64 / lanes_of(nb, channels); }

// Calls f(sample, head, lane's place in the row, tokens, page numbers, places in the pages) for the lane's tokens.
template <typename T, int NB, typename F>
__device__ __forceinline__ void for_tokens(const TokenParams& p, F f) {
  constexpr int LANES = lanes_of(NB, kLaneChannels<T>), ABREAST = tokens_abreast(NB, kLaneChannels<T>);
  const CachePages& c = p.a.pages;
  const unsigned unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // (below 2^26: cache_tokens_fit)
  if (unit >= p.units) return;
  const unsigned above = unit / (unsigned)c.heads;
  const int lane = threadIdx.x & 63, h = (int)(unit - above * (unsigned)c.heads), n = (int)(above / (unsigned)p.chunks), chunk = (int)(above - (unsigned)n * (unsigned)p.chunks);
  const int count = p.a.counts ? min(p.a.counts[n], p.a.t) : p.a.t;
  const long first = p.a.first ? p.a.first[n] : 0, most = (long)c.table_pages * c.page_tokens;
  const int own = lane / LANES;
  int token[kSteps], number[kSteps], slot[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    token[i] = (chunk * kSteps + i) * ABREAST + own;
    if (own >= ABREAST || token[i] >= count) token[i] = -1;
    const long at = first + token[i];
    number[i] = -1;
    slot[i] = 0;
    if (token[i] >= 0 && at >= 0 && at < most) number[i] = c.table[n * c.table_stride + div_rem((unsigned)at, c.page_tokens, c.inv_page_tokens, slot[i])];
  }
  f(n, h, lane % LANES, token, number, slot);
}

// f16 reads back what it wrote
template <typename T> constexpr int kTopExponent = 125 + 127;
template <> constexpr int kTopExponent<f16_t> = 13 + 127;

// (by the caches or not at compile time: the compiler makes an ordinary access of two branches)
template <bool STREAM> __device__ __forceinline__ u32x4 load_state(const void* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load((const u32x4*)p);
  else return *(const u32x4*)p;
}
template <bool STREAM> __device__ __forceinline__ void store_state(void* p, u32x4 v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, (u32x4*)p);
  else *(u32x4*)p = v;
}

template <typename T, int NB, bool STREAM>
__global__ __launch_bounds__(256) void cache_write_kernel(TokenParams p) {
  for_tokens<T, NB>(p, [&](int n, int h, int c, const int (&token)[kSteps], const int (&number)[kSteps], const int (&slot)[kSteps]) {
    constexpr int E = kLaneChannels<T>, PER = 32 / E, ROW = 16 * NB, EXP = exponent_bytes(NB);   // PER: lanes of a block
    const CachePages& cp = p.a.pages;
    u32x4 x[2][kSteps];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const T* src = (const T*)(which ? p.a.v : p.a.k);
      const wmdec_strides& st = which ? p.a.vs : p.a.ks;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        x[which][i] = u32x4{0, 0, 0, 0};
        if (src && number[i] >= 0 && E * c < cp.d) x[which][i] = load_state<STREAM>(src + n * st.sample + token[i] * st.token + h * st.head + E * c);
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      unsigned char* page = head_of_page(cp, number[i], h);
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        if (!(which ? p.a.v : p.a.k)) continue;
        float v[E];
        unsigned top = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if constexpr (E == 4) v[e] = __uint_as_float(x[which][i][e]);
          else v[e] = e % 2 ? unpack_hi<T>(x[which][i][e / 2]) : unpack_lo<T>(x[which][i][e / 2]);
          top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
        }
#pragma unroll
        for (int step = 1; step < PER; step *= 2) top = max(top, (unsigned)__shfl_xor((int)top, step));
        // the exponent of the largest value as three bits of it round, which is one more from 1.75 on
        const int held = min(max((int)((top + 0x200000u) >> 23) - 2, 2), kTopExponent<T>);
        const bool finite = top < 0x7f800000u;
        const unsigned codes = finite ? narrow(v, unit_of(held)) : 0;
        if (page) {
          unsigned char* at = page + which * ROW * cp.page_tokens + (unsigned)slot[i] * ROW + E / 2 * c;
          if constexpr (E == 4) *reinterpret_cast<unsigned short*>(at) = (unsigned short)codes;
          else *reinterpret_cast<unsigned*>(at) = codes;
          if (c % PER == 0) page[(2 * ROW + which * EXP) * cp.page_tokens + slot[i] * EXP + c / PER] = (unsigned char)(finite ? held : 255);
        }
      }
    }
  });
}

template <typename T, int NB, bool STREAM>
__global__ __launch_bounds__(256) void cache_read_kernel(TokenParams p) {
  for_tokens<T, NB>(p, [&](int n, int h, int c, const int (&token)[kSteps], const int (&number)[kSteps], const int (&slot)[kSteps]) {
    constexpr int E = kLaneChannels<T>, PER = 32 / E, ROW = 16 * NB, EXP = exponent_bytes(NB);
    typedef typename std::conditional<E == 4, unsigned short, unsigned>::type Codes;
    const CachePages& cp = p.a.pages;
    if (E * c >= cp.d) return;
    unsigned codes[2][kSteps], held[2][kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const unsigned char* page = head_of_page(cp, number[i], h);
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        codes[which][i] = held[which][i] = 0;   // no page: zeros
        if (page && (which ? p.a.v : p.a.k)) {
          codes[which][i] = *reinterpret_cast<const Codes*>(page + which * ROW * cp.page_tokens + (unsigned)slot[i] * ROW + E / 2 * c);
          held[which][i] = page[(2 * ROW + which * EXP) * cp.page_tokens + slot[i] * EXP + c / PER];
        }
      }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      T* dst = (T*)(which ? p.a.v : p.a.k);
      if (!dst) continue;
      const wmdec_strides& st = which ? p.a.vs : p.a.ks;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        if (token[i] < 0) continue;
        const float unit = unit_of(held[which][i]);
        u32x4 v;
        if constexpr (E == 4) {
          const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[which][i], unit, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[which][i], unit, 1);
          v = __builtin_bit_cast(u32x4, f32x4{lo.x, lo.y, hi.x, hi.y});
        } else {
          v = widen<T>(codes[which][i], unit);
        }
        store_state<STREAM>(dst + n * st.sample + token[i] * st.token + h * st.head + E * c, v);
      }
    }
  });
}

int blocks_of(int d) { return (d + 31) / 32; }
int chunks_of(int t, int d, int channels) { const int per = kSteps * tokens_abreast(blocks_of(d), channels); return (int)(((long)t + per - 1) / per); }

// States that are whole 64-byte pieces of memory pass by the caches (us, by them or not: read back in bf16, 30 heads of 32 35 / 44, of 64 27 / 41, 8 of 128 27 / 41, but 30 of 40 79 / 65, of
// 72 59 / 57, of 8 50 / 20); those to be written only from 128 bytes on (30 of 32 77 / 70, of 64 64 / 76).
bool pieces(const void* p, const wmdec_strides& s, int d, size_t es) {
  return !p || ((uintptr_t)p % 64 == 0 && d * es % 64 == 0 && s.sample * es % 64 == 0 && s.token * es % 64 == 0 && s.head * es % 64 == 0);
}

template <typename T, bool WRITE, int NB>
int launch_tokens(const TokenParams& p, bool stream, hipStream_t s) {
  const dim3 grid((unsigned)((p.units + 3) / 4));
  auto kern = WRITE ? (stream ? cache_write_kernel<T, NB, true> : cache_write_kernel<T, NB, false>) : (stream ? cache_read_kernel<T, NB, true> : cache_read_kernel<T, NB, false>);
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, p);
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

template <typename T, bool WRITE>
int launch_width(const TokenParams& p, bool stream, hipStream_t s) {
  switch (blocks_of(p.a.pages.d)) {
    case 1: return launch_tokens<T, WRITE, 1>(p, stream, s);
    case 2: return launch_tokens<T, WRITE, 2>(p, stream, s);
    case 3: return launch_tokens<T, WRITE, 3>(p, stream, s);
    case 4: return launch_tokens<T, WRITE, 4>(p, stream, s);
    case 5: return launch_tokens<T, WRITE, 5>(p, stream, s);
    case 6: return launch_tokens<T, WRITE, 6>(p, stream, s);
    case 7: return launch_tokens<T, WRITE, 7>(p, stream, s);
    default: return launch_tokens<T, WRITE, 8>(p, stream, s);
  }
}

template <bool WRITE>
int launch_type(const CacheTokens& a, int dtype, hipStream_t s) {
  TokenParams p;
  p.a = a;
  const size_t es = dtype_size(dtype);
  p.chunks = chunks_of(a.t, a.pages.d, 16 / (int)es);
  const bool stream = pieces(a.k, a.ks, a.pages.d, es) && pieces(a.v, a.vs, a.pages.d, es) && (!WRITE || a.pages.d * es >= 128);
  p.units = (unsigned)((long)a.n * p.chunks * a.pages.heads);
  if (dtype == WMDEC_F32) return launch_width<float, WRITE>(p, stream, s);
  return dtype == WMDEC_BF16 ? launch_width<bf16_t, WRITE>(p, stream, s) : launch_width<f16_t, WRITE>(p, stream, s);
}

}  // namespace

size_t cache_head_bytes(int page_tokens, int d) {
  const int nb = blocks_of(d);
  return ((size_t)page_tokens * 2 * (16 * nb + exponent_bytes(nb)) + 15) / 16 * 16;
}

bool cache_tokens_fit(int n, int t, int heads, int d) { return (double)n * chunks_of(t, d, 4) * heads <= 0x1p26 - 4; }   // (64 threads each, in whole workgroups of 256)

int launch_cache_write(const CacheTokens& a, int dtype, hipStream_t s) { return launch_type<true>(a, dtype, s); }
int launch_cache_read(const CacheTokens& a, int dtype, hipStream_t s) { return launch_type<false>(a, dtype, s); }

// ---------------------------------------------------------------- attention: what is decided on sizes alone
namespace {

// Nothing here looks at the number of samples, so that the bits of a sample do not depend on what it is batched with.
CachePlan plan_of(int dtype, int tq, int tk, int heads, int group, int d) {
  CachePlan p;
  p.nb = blocks_of(d);
  p.rows = tq * group;
  // us, blocks of 16 rows / of 128: bf16, causal, 32 / 8 heads of 128, 64 rows a key head against 2048 keys 11.2 / 16.0, 16384 21.4 / 31.1, 16 x 4096 80 / 72; 128 rows against
  // 2048 13.3 / 18.1, 16 x 4096 137 / 90; 100 of 30 heads of 64 against 2000 15.0 / 18.7, 16 x 1000 62 / 31.  In fp32, where products weigh more than what is widened for
  // them, all: 1000x1000 of 12 of 64 19 / 30, four of 1000x3000 of 8 of 128 161 / 221, 2000x2000 of 16 of 160 138 / 205, of 192 161 / 226.
  p.few = p.rows <= 64 || dtype == WMDEC_F32;
  p.row_blocks = (p.rows + p.bq() - 1) / p.bq();
  const long blocks = (long)heads * p.row_blocks;
  long ranges;
  if (p.few) {
    // One range below 640 keys, then of 256 up to eight of them, then of 512 or more and at most 64, as long as there are no more than four workgroups a compute unit (us, one
    // token of 32 / 8 heads of 128 against 500 keys in one range / two 8.3 / 9.7, 1000 in three / four 10.5 / 9.9, 4000 in eight / sixteen 11.7 / 9.9 but 16 x 4096 20.3 / 22.7, 16384 in 32
    // / 64 15.8 / 17.0, 65536 in 64 / 128 20.5 / 22.8).
    ranges = tk < 640 ? 1 : std::min({1024 / blocks, std::max(std::min(8L, (tk + 255L) / 256L), tk / 512L), (long)kCacheMaxSplits});
  } else {
    // Partial outputs of 128 rows weigh: s ranges take a / s for their keys, b * s for writing and reading what they leave, and the second launch.
    const double a = 1.8e-4 * tk * 32 * p.nb, b = 1.2e-6 * 512 * 32 * p.nb * blocks;   // us
    ranges = std::min({512 / blocks, tk / 256L, (long)kCacheMaxSplits, (long)std::sqrt(a / b)});
    if (ranges < 2 || a - a / ranges < 5 + b * ranges) ranges = 1;
  }
  ranges = std::max(ranges, 1L);
  p.range = std::max(128, (int)(((long)tk + ranges - 1) / ranges + 127) / 128 * 128);
  p.splits = std::max(1, (int)(((long)tk + p.range - 1) / p.range));
  // us, four wavefronts / eight that halve the keys: one workgroup a compute unit or less, bf16, 2048x2048 of 16 of 256 137 / 98, 2000x2000 of 16 of 160 91 / 68, 1000x2000 of 30 of
  // 64 45 / 38, 1000x1000 of 12 of 96 29 / 27, but 5 to 64 x 2048 of 32 / 8 of 128 14.1 .. 22.1 / 15.0 .. 23.3; more workgroups, 2 x 4096x4096 of 16 of 256 677 / 733, 2 x 5400x5400
  // of 30 of 64 599 / 634.
  p.halves = !p.few && has_halves(p.nb) && blocks * p.splits <= 256;
  return p;
}

size_t part_rows(const CachePlan& p, int n, int heads) { return p.splits == 1 ? 0 : (size_t)n * heads * p.row_blocks * p.splits * p.block_rows(); }

}  // namespace

bool cache_attention_fits(int dtype, int n, int tq, int tk, int heads, int group, int d) {
  const CachePlan p = plan_of(dtype, tq, tk, heads, group, d);
  const double blocks = (double)n * heads * p.row_blocks;
  return blocks * p.splits * (p.halves ? 512 : 256) < 0x1p32 && (p.splits == 1 || (double)n * heads * p.rows < 0x1p26);   // threads of a launch; rows that are joined
}

size_t cache_attention_scratch_bytes(int dtype, int n, int tq, int tk, int heads, int group, int d) {
  const CachePlan p = plan_of(dtype, tq, tk, heads, group, d);
  return part_rows(p, n, heads) * (32 * p.nb + 2) * sizeof(float);
}

int launch_cache_attention(const CacheAttentionArgs& a, int dtype, hipStream_t s) {
  CacheLaunch l;
  l.a = a;
  l.plan = plan_of(dtype, a.tq, a.tk, a.pages.heads, a.group, a.pages.d);
  l.part = (float*)a.scratch;
  l.ml = (float2*)(l.part + part_rows(l.plan, a.n, a.pages.heads) * 32 * l.plan.nb);
  if (dtype == WMDEC_F32) return cache_attention_launch<float>(l, s);
  return dtype == WMDEC_BF16 ? cache_attention_launch<bf16_t>(l, s) : cache_attention_launch<f16_t>(l, s);
}

}  // namespace wmdec
