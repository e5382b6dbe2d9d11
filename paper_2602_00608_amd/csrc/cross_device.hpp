// The kernel of kernels_cross.hip: attention of rows (a token of one of the query heads that share a key head) to the keys of a sample.
//
// Tiles of KT keys and values stream through two LDS buffers, straight from memory (16 bytes a lane), while the tile before is worked on.  Per 32 keys a
// wavefront forms S^T = K Q^T (keys along the accumulator's registers, one row a lane), the softmax against a running maximum, and O^T += V^T P^T with the
// probabilities as they are in their registers: an accumulator's keys of lane half lk are 8 (r / 4) + 4 lk + r % 4, so V^T is read from LDS in that order of
// keys (16-bit types: transposed on the way, four keys of one channel a lane).  fp32 takes the same steps with 32x32x2 products.
// The wavefronts of a workgroup take QT * 32 rows each (QW of them), or, where there are few rows, the same rows and a part of a tile's keys (KW), joined at the end.
//
// 16-byte chunk c of key r lies at chunk c ^ turn(r) of its row in LDS: the eight lanes of a pass over K (eight keys, one chunk) and the sixteen over V (four
// keys, two chunks) then have banks of their own.  The loads bring the chunks in that order, as a lane chooses what it reads and not where it lands.
#pragma once
#include <mutex>

#include "mfma.hpp"

namespace wmdec {

struct CrossLaunch {
  CrossArgs a;
  int rows, row_blocks, splits;   // rows of a key head, blocks of them, ranges of keys
  float* part;                    // [split][sample][key head][row][D] sums of probabilities times values
  float2* ml;                     // [split][sample][key head][row] reference and sum of the probabilities
};

template <typename T> constexpr int kChunkElems = 16 / (int)sizeof(T);

template <int CH> __device__ __forceinline__ int chunk_turn(int row) {   // CH: chunks of a key, a multiple of 4
  if constexpr (CH % 8 == 0) return ((row & 3) << 1) | ((row >> 2) & 1);
  else return (row & 2) | ((row >> 2) & 1);   // (rows alternate between the halves of 128 bytes by themselves)
}

__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }   // (NaN if one is: one instruction for three)

constexpr int kMaskKeys = 32768;      // keys whose mask is staged as bits at a time

// D: channels, rounded up to a multiple of 32; a wavefront has QT * 32 rows; QW x KW wavefronts
template <typename T, int D, int QT, int QW, int KW, int KT>
struct CrossForm {
  static constexpr int EC = kChunkElems<T>, CH = D / EC, NW = QW * KW, NT = 64 * NW, SUB = KT / KW, NS = SUB / 32, LOADS = KT * CH / NT, BQ = 32 * QT * QW;
  static constexpr int TILE = KT * D;
  static constexpr int kTiles = 4 * TILE * (int)sizeof(T), kSmem = kTiles + kMaskKeys / 8;
  static constexpr int RED = D + 4;   // floats from row to row of the outputs that are joined
  static_assert(D % 32 == 0 && KT % (32 * KW) == 0 && KT * CH % NT == 0 && (KW == 1 || (QW == 1 && QT == 1)));
  static_assert(kTiles <= 128 * 1024 && 3 * LOADS < 64 && (KW == 1 || KW * 32 * (RED + 2) * 4 <= kTiles));
};

// Tiles are asked for and waited for in assembly: the compiler would wait for all of them in front of every transposed read.  No registers are written.
// 16 bytes a lane from `offset` of the buffer to lds + 16 * lane; past the buffer's end the LDS gets zeros.
__device__ __forceinline__ void load_to_lds(u32x4 buffer, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(offset), "s"(buffer) : "memory", "m0");
}
// all but the last N loads of this wavefront have landed
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }
// every load and LDS access of this wavefront is done, and so for the others
__device__ __forceinline__ void sync_tiles() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory"); }
// the same for LDS accesses alone: tiles on their way are not waited for
__device__ __forceinline__ void sync_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }
constexpr unsigned kPastEnd = 0x80000000u;   // an offset that no buffer reaches

constexpr float kCrossSlack = 8.0f;   // log2 of how far a tile's maximum may exceed the reference before that moves

template <typename T, int D, int QT, int QW, int KW, int KT, int WAVES>
__global__ __launch_bounds__(64 * QW * KW, WAVES) void cross_attention_kernel(CrossLaunch p) {
  using F = CrossForm<T, D, QT, QW, KW, KT>;
  constexpr int EC = F::EC, CH = F::CH, NW = F::NW, NS = F::NS, LOADS = F::LOADS, TILE = F::TILE, QS = CH / 2, ND = D / 32;
  constexpr int GP = CH % 8 == 0 ? 8 : 4;   // chunks that are exchanged among each other
  constexpr bool WIDE = sizeof(T) == 4, OWN = KW > 1;   // OWN: a wavefront loads the keys it works on, and waits for nobody
  extern __shared__ __align__(16) unsigned char smem[];
  T* s_k = reinterpret_cast<T*>(smem);      // [2] tiles
  T* s_v = s_k + 2 * TILE;
  unsigned* s_bits = reinterpret_cast<unsigned*>(smem + F::kTiles);   // the mask, 32 keys a word
  const CrossArgs& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, lk = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), qw = wave / KW, kw = wave % KW;
  // workgroup id -> (sample, key head, key range, row block); the ids of one XCD (id % 8) are neighbours and share their keys
  int L;
  {
    const int i = blockIdx.x, total = gridDim.x, per = total / 8, rem = total % 8, x = i % 8, j = i / 8;
    L = x * per + (x < rem ? x : rem) + j;
  }
  const int rb = L % p.row_blocks, split = L / p.row_blocks % p.splits, nh = L / (p.row_blocks * p.splits), h = nh % a.heads, n = nh / a.heads;
  const int len = a.lens ? min(max(a.lens[n], 0), a.tk) : a.tk;
  const int tiles = (len + KT - 1) / KT, first = (int)((long)split * tiles / p.splits), nt = (int)((long)(split + 1) * tiles / p.splits) - first;

  // ---- tiles.  A load is 64 consecutive chunks of a tile; chunks past the last channel and keys past the last one are read past the buffer's end
  const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const char* kp = (const char*)a.k + (n * a.ks.sample + h * a.ks.head) * (long)sizeof(T);
  const char* vp = (const char*)a.v + (n * a.vs.sample + h * a.vs.head) * (long)sizeof(T);
  const int kstep = (int)(a.ks.token * (long)sizeof(T)), vstep = (int)(a.vs.token * (long)sizeof(T));   // (128 of them are below 2^31: checked on the host)
  const unsigned char* mask = a.mask ? a.mask + (long)n * a.tk : nullptr;
  auto slot0 = [&](int i) { return OWN ? wave * F::SUB * CH + i * 64 : (i * NW + wave) * 64; };
  unsigned koff[LOADS], voff[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = (slot0(i) + lane) / CH, c = ((slot0(i) + lane) % CH) ^ chunk_turn<CH>(r);
    koff[i] = c * EC < a.d ? (unsigned)(r * kstep + c * 16) : kPastEnd;
    voff[i] = c * EC < a.d ? (unsigned)(r * vstep + c * 16) : kPastEnd;
  }
  auto ask = [&](const char* base, int step, const unsigned (&off)[LOADS], int at, int j) {
    const int k0 = (first + j) * KT, left = len - k0;
    const uint64_t from = (uint64_t)(base + (long)k0 * step);
    const u32x4 buffer{(unsigned)from, (unsigned)(from >> 32) & 0xffffu, kPastEnd - 1, 0x00020000u};
    const unsigned to = lds + (at + (j & 1) * TILE) * (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      unsigned o = off[i];
      if (left < KT) o = (slot0(i) + lane) / CH < left ? o : kPastEnd;
      load_to_lds(buffer, o, to + slot0(i) * 16);
    }
  };
  auto ask_k = [&](int j) { ask(kp, kstep, koff, 0, j); };
  auto ask_v = [&](int j) { ask(vp, vstep, voff, 2 * TILE, j); };

  // ---- queries: chunk 2 s + lk of the lane's row
  const int row0 = rb * F::BQ + qw * QT * 32 + l32;
  u32x4 q[QT][QS];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int row = min(row0 + t * 32, p.rows - 1), tok = row / a.group, hq = h * a.group + (row - tok * a.group);
    const T* src = (const T*)a.q + n * a.qs.sample + tok * a.qs.token + hq * a.qs.head;
#pragma unroll
    for (int s = 0; s < QS; ++s) {
      const int c = (2 * s + lk) * EC;
      q[t][s] = u32x4{0, 0, 0, 0};
      if (c < a.d) q[t][s] = *reinterpret_cast<const u32x4*>(src + c);
    }
  }

  // ---- where a lane reads its operands (elements of a tile)
  int kb[GP / 2];   // chunks 2 s + lk of key l32, by s modulo the chunks that are exchanged
#pragma unroll
  for (int s = 0; s < GP / 2; ++s) kb[s] = (l32 * CH + ((2 * s + lk) ^ chunk_turn<CH>(l32))) * EC;
  constexpr int VB = WIDE ? 4 : GP / 4;
  int vb[VB];
#pragma unroll
  for (int i = 0; i < VB; ++i) {
    if constexpr (WIDE) {   // channel l32 of key 4 lk + i
      const int r = 4 * lk + i;
      vb[i] = (r * CH + ((l32 >> 2) ^ chunk_turn<CH>(r))) * EC + (l32 & 3);
    } else {                // channels 16 (l32 / 16) + 4 (lane % 4) .. + 3 of key 4 lk + lane / 4 % 4, of which the lane gets channel l32 of four keys
      const int r = 4 * lk + ((lane >> 2) & 3), c = 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      vb[i] = (r * CH + (c ^ chunk_turn<CH>(r))) * EC + (lane & 1) * 4;
    }
  }

  f32x16 o[QT][ND];
  float m[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY; l[t] = 0.f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][dt][r] = 0.f;
  }
  const float c = a.scale * 1.4426950408889634f;

  f32x16 s[QT][NS];
  // scores of a tile (its valid keys in `bits`)
  auto scores = [&](const T* tk, const unsigned (&bits)[NS]) {
#pragma unroll
    for (int ns = 0; ns < NS; ++ns) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][ns][r] = 0.f;
#pragma unroll
      for (int st = 0; st < QS; ++st) {
        const u32x4 kf = *reinterpret_cast<const u32x4*>(tk + kb[st % (GP / 2)] + st / (GP / 2) * GP * EC + ns * 32 * D);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          if constexpr (WIDE) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][ns] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(q[t][st][e]), s[t][ns], 0, 0, 0);
          } else {
            s[t][ns] = Mma<T>::m32(kf, q[t][st], s[t][ns]);
          }
        }
      }
      if (bits[ns] != ~0u) {
        const unsigned b = bits[ns] >> (4 * lk);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!((b >> (8 * (r / 4) + r % 4)) & 1)) {
#pragma unroll
            for (int t = 0; t < QT; ++t) s[t][ns][r] = -INFINITY;
          }
      }
    }
  };
  auto softmax = [&]() {
    // softmax: the reference moves when a maximum exceeds it by 2^kCrossSlack; until then probabilities may reach that, well inside the 16-bit types
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float mx = maximum(maximum(s[t][0][0], s[t][0][1]), s[t][0][2]);
#pragma unroll
      for (int i = 3; i + 1 < 16 * NS; i += 2) mx = maximum(maximum(mx, s[t][i / 16][i % 16]), s[t][(i + 1) / 16][(i + 1) % 16]);
      mx = maximum(mx, s[t][NS - 1][15]);
      mx = half_max(mx) * c;
      const bool moves = mx > m[t] + kCrossSlack;
      if (__ballot(moves)) {
        const float to = moves ? mx : m[t], factor = moves ? __builtin_amdgcn_exp2f(m[t] - mx) : 1.f;
        m[t] = to;
        l[t] *= factor;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[t][dt][r] *= factor;
      }
      const float ref = m[t] == -INFINITY ? 0.f : m[t];
#pragma unroll
      for (int ns = 0; ns < NS; ++ns)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[t][ns][r] = __builtin_amdgcn_exp2f(fmaf(s[t][ns][r], c, -ref));
          l[t] += s[t][ns][r];
        }
    }
  };
  auto values = [&](const T* tv) {
#pragma unroll
    for (int ns = 0; ns < NS; ++ns) {
      if constexpr (WIDE) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) {
            const float vf = to_float(tv[vb[r % 4] + (ns * 32 + 8 * (r / 4)) * D + dt * 32]);
#pragma unroll
            for (int t = 0; t < QT; ++t) o[t][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[t][ns][r], o[t][dt], 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          u32x4 pf[QT];   // the one rounding inside the operator: probabilities as operands of T
#pragma unroll
          for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int w = 0; w < 4; ++w) pf[t][w] = pack2<T>(s[t][ns][8 * ks + 2 * w], s[t][ns][8 * ks + 2 * w + 1]);
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4* tptr_t;
            const T* at = tv + vb[dt % (GP / 4)] + dt / (GP / 4) * GP * EC + (ns * 32 + ks * 16) * D;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)at));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)(at + 8 * D)));
            const u32x4 vf{lo.x, lo.y, hi.x, hi.y};
#pragma unroll
            for (int t = 0; t < QT; ++t) o[t][dt] = Mma<T>::m32(vf, pf[t], o[t][dt]);
          }
        }
      }
    }
  };

  // The mask of up to kMaskKeys keys is staged at a time; without one all keys are one block.
  constexpr int MB = kMaskKeys / KT;
  for (int b0 = 0; b0 < nt;) {
    const int b1 = mask ? min(nt, b0 + MB) : nt;
    if (mask) {
      if (b0) sync_tiles();   // (the bits before have been read)
      const int k0 = (first + b0) * KT, words = ((b1 - b0) * KT + 63) / 64;
#pragma unroll 4
      for (int w = wave; w < words; w += NW) {
        const int key = k0 + w * 64 + lane;
        const unsigned long long bit = __ballot(key < len && mask[min(key, len - 1)] != 0);
        if (lane == 0) *reinterpret_cast<u32x2*>(s_bits + 2 * w) = u32x2{(unsigned)bit, (unsigned)(bit >> 32)};
      }
      sync_lds();
    }
    // valid keys of the wavefront's part of tile j
    bool none, all;
    auto valid = [&](int j, unsigned (&bits)[NS]) {
      none = true; all = true;
#pragma unroll
      for (int ns = 0; ns < NS; ++ns) {
        const int at = kw * F::SUB + ns * 32, left = len - (first + j) * KT - at;
        unsigned u = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1;
        if (mask) u &= __builtin_amdgcn_readfirstlane(s_bits[((j - b0) * KT + at) / 32]);
        bits[ns] = u;
        none = none && u == 0;
        all = all && u == ~0u;
      }
    };
    // what a masked value holds times a probability of zero need not be zero (keys past the last one are zeros already)
    auto clear = [&](T* tile, const unsigned (&bits)[NS]) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int r = (slot0(i) + lane) / CH - kw * F::SUB;
        unsigned u = bits[0];
#pragma unroll
        for (int ns = 1; ns < NS; ++ns) u = r / 32 == ns ? bits[ns] : u;
        if (!((u >> (r & 31)) & 1)) *reinterpret_cast<u32x4*>(tile + (slot0(i) + lane) * EC) = u32x4{0, 0, 0, 0};
      }
    };
    unsigned bits[NS];
    // (the queries are waited for here: the compiler, which does not see the tiles' loads, would wait for all of them wherever it first uses a query)
    auto queries_landed = [&]() {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int s = 0; s < QS; ++s) asm volatile("" : "+v"(q[t][s]));
    };
    if constexpr (OWN) {
      // keys and values each have two tiles on their way while a third is worked on
      ask_k(b0);
      ask_v(b0);
      if (b0 + 1 < b1) { ask_k(b0 + 1); ask_v(b0 + 1); }
      queries_landed();
      for (int j = b0; j < b1; ++j) {
        T *tk = s_k + (j & 1) * TILE + kw * F::SUB * D, *tv = s_v + (j & 1) * TILE;
        const int more = b1 - 1 - j;
        valid(j, bits);
        if (more > 0) wait_loads<3 * LOADS>();
        else wait_loads<LOADS>();
        if (!none) scores(tk, bits);
        __builtin_amdgcn_sched_barrier(0);
        if (more > 1) ask_k(j + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (!none) softmax();
        if (more > 1) wait_loads<3 * LOADS>();
        else if (more > 0) wait_loads<2 * LOADS>();
        else wait_loads<0>();
        if (!none) {
          if (mask && !all) { clear(tv, bits); asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }
          values(tv + kw * F::SUB * D);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more > 1) ask_v(j + 2);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      ask_k(b0);
      ask_v(b0);
      queries_landed();
      for (int j = b0; j < b1; ++j) {
        sync_tiles();       // the tile has landed, and every wavefront is done with the other buffer
        T *tk = s_k + (j & 1) * TILE, *tv = s_v + (j & 1) * TILE;
        if (j + 1 < b1) { ask_k(j + 1); ask_v(j + 1); }
        valid(j, bits);
        if (none) continue;
        if (mask && !all) { clear(tv, bits); sync_lds(); }
        scores(tk, bits);
        softmax();
        values(tv);
      }
    }
    b0 = b1;
  }

  // ---- output.  A lane holds channels 32 dt + 8 g + 4 lk .. + 3 of its row
#pragma unroll
  for (int t = 0; t < QT; ++t) l[t] += __shfl_xor(l[t], 32);
  const long unit = ((long)split * a.n + n) * a.heads + h;
  if constexpr (KW == 1) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int row = row0 + t * 32;
      if (row >= p.rows) continue;
      if (p.splits > 1) {
        if (lk == 0) p.ml[unit * p.rows + row] = make_float2(m[t], l[t]);
        float* dst = p.part + (unit * p.rows + row) * D + 4 * lk;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4*>(dst + 32 * dt + 8 * g) = f32x4{o[t][dt][4 * g], o[t][dt][4 * g + 1], o[t][dt][4 * g + 2], o[t][dt][4 * g + 3]};
        continue;
      }
      const int tok = row / a.group, hq = h * a.group + (row - tok * a.group);
      T* dst = (T*)a.o + n * a.os.sample + tok * a.os.token + hq * a.os.head;
      const float inv = l[t] == 0.f ? 0.f : 1.f / l[t];
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int at = 32 * dt + 8 * g + 4 * lk;
          const float v0 = o[t][dt][4 * g] * inv, v1 = o[t][dt][4 * g + 1] * inv, v2 = o[t][dt][4 * g + 2] * inv, v3 = o[t][dt][4 * g + 3] * inv;
          if (at >= a.d) continue;
          if constexpr (WIDE) *reinterpret_cast<f32x4*>(dst + at) = f32x4{v0, v1, v2, v3};
          else *reinterpret_cast<u32x2*>(dst + at) = u32x2{pack2<T>(v0, v1), pack2<T>(v2, v3)};
        }
    }
  } else {
    float* s_o = reinterpret_cast<float*>(smem);                          // [KW][32][RED]
    float2* s_ml = reinterpret_cast<float2*>(s_o + KW * 32 * F::RED);     // [KW][32]
    sync_tiles();
    if (lk == 0) s_ml[kw * 32 + l32] = make_float2(m[0], l[0]);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(s_o + (kw * 32 + l32) * F::RED + 32 * dt + 8 * g + 4 * lk) = f32x4{o[0][dt][4 * g], o[0][dt][4 * g + 1], o[0][dt][4 * g + 2], o[0][dt][4 * g + 3]};
    sync_lds();
    for (int i = tid; i < 32 * D / 4; i += F::NT) {
      const int r = i / (D / 4), at = i % (D / 4) * 4, row = rb * 32 + r;
      if (row >= p.rows || at >= a.d) continue;
      float top = s_ml[r].x, den = 0.f;
#pragma unroll
      for (int w = 1; w < KW; ++w) top = fmaxf(top, s_ml[w * 32 + r].x);
      f32x4 num{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float2 e = s_ml[w * 32 + r];
        const float f = e.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(e.x - top);
        den = fmaf(e.y, f, den);
        num += f * *reinterpret_cast<const f32x4*>(s_o + (w * 32 + r) * F::RED + at);
      }
      if (p.splits > 1) {
        if (at == 0) p.ml[unit * p.rows + row] = make_float2(top, den);
        *reinterpret_cast<f32x4*>(p.part + (unit * p.rows + row) * D + at) = num;
        continue;
      }
      const int tok = row / a.group, hq = h * a.group + (row - tok * a.group);
      T* dst = (T*)a.o + n * a.os.sample + tok * a.os.token + hq * a.os.head + at;
      const float inv = den == 0.f ? 0.f : 1.f / den;
      if constexpr (WIDE) *reinterpret_cast<f32x4*>(dst) = num * inv;
      else *reinterpret_cast<u32x2*>(dst) = u32x2{pack2<T>(num[0] * inv, num[1] * inv), pack2<T>(num[2] * inv, num[3] * inv)};
    }
  }
}

// o = sum_s part_s 2^(m_s - M) / sum_s l_s 2^(m_s - M), ranges in index order, eight at a time.  A thread takes four channels of a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_combine_kernel(CrossLaunch p) {
  const CrossArgs& a = p.a;
  const long i = (long)blockIdx.x * 256 + threadIdx.x, count = (long)a.n * a.heads * p.rows, r = i / (D / 4);
  const int at = (int)(i % (D / 4)) * 4;
  if (r >= count || at >= a.d) return;
  float top = -INFINITY, den = 0.f;
  f32x4 num{0.f, 0.f, 0.f, 0.f};
  constexpr int B = 8;
  for (int s0 = 0; s0 < p.splits; s0 += B) {
    float2 e[B];
    f32x4 v[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {   // (past the last: the last again, with weight zero)
      const long s = min(s0 + b, p.splits - 1);
      e[b] = p.ml[s * count + r];
      v[b] = *reinterpret_cast<const f32x4*>(p.part + (s * count + r) * D + at);
    }
    float now = top;
#pragma unroll
    for (int b = 0; b < B; ++b) now = fmaxf(now, e[b].x);
    const float keep = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - now);
    den *= keep;
    num *= keep;
    top = now;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (s0 + b >= p.splits) continue;
      const float f = e[b].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(e[b].x - top);
      den = fmaf(e[b].y, f, den);
      num += f * v[b];
    }
  }
  const int row = (int)(r % p.rows), h = (int)(r / p.rows % a.heads), n = (int)(r / ((long)p.rows * a.heads));
  const int tok = row / a.group, hq = h * a.group + (row - tok * a.group);
  T* dst = (T*)a.o + n * a.os.sample + tok * a.os.token + hq * a.os.head + at;
  const float inv = den == 0.f ? 0.f : 1.f / den;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(dst) = num * inv;
  else *reinterpret_cast<u32x2*>(dst) = u32x2{pack2<T>(num[0] * inv, num[1] * inv), pack2<T>(num[2] * inv, num[3] * inv)};
}

// What the kernels of a type are launched with: rows per wavefront, whether wavefronts share rows.
template <typename T, int D, int QT, int QW, int KW, int KT, int WAVES>
int cross_launch_form(const CrossLaunch& p, hipStream_t s) {
  using F = CrossForm<T, D, QT, QW, KW, KT>;
  auto kern = cross_attention_kernel<T, D, QT, QW, KW, KT, WAVES>;
  static std::once_flag attr_once;
  hipError_t attr_err = hipSuccess;
  std::call_once(attr_once, [&] { attr_err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, F::kSmem); });
  WMDEC_HIP(attr_err);
  CrossLaunch q = p;
  q.row_blocks = (p.rows + F::BQ - 1) / F::BQ;
  hipLaunchKernelGGL(kern, dim3((unsigned)((long)q.row_blocks * q.splits * q.a.n * q.a.heads)), dim3(F::NT), F::kSmem, s, q);
  WMDEC_HIP(hipGetLastError());
  if (p.splits > 1) {
    const long threads = (long)q.a.n * q.a.heads * q.rows * (D / 4);
    hipLaunchKernelGGL((cross_combine_kernel<T, D>), dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, q);
    WMDEC_HIP(hipGetLastError());
  }
  return WMDEC_OK;
}

template <typename T, int D>
int cross_launch_width(const CrossLaunch& p, bool few, hipStream_t s) {
  constexpr int bytes = D * (int)sizeof(T);   // of a key
  constexpr int KT = bytes <= 512 ? 64 : 32;
  if constexpr (bytes <= 256) {
    if (few) return cross_launch_form<T, D, 1, 1, 4, 128, 1>(p, s);
  } else if constexpr (bytes <= 512) {
    if (few) return cross_launch_form<T, D, 1, 1, 2, 64, 1>(p, s);
  }
  if constexpr (sizeof(T) == 2 && D <= 128) {
    if (p.rows > 128) return cross_launch_form<T, D, 2, 4, 1, KT, (D <= 64 ? 2 : 1)>(p, s);
  }
  return cross_launch_form<T, D, 1, 4, 1, KT, (D <= 128 ? 2 : 1)>(p, s);
}

// few: at most 32 rows
template <typename T>
int cross_launch(const CrossLaunch& p, int width, bool few, hipStream_t s) {
  switch (width) {
    case 32: return cross_launch_width<T, 32>(p, few, s);
    case 64: return cross_launch_width<T, 64>(p, few, s);
    case 96: return cross_launch_width<T, 96>(p, few, s);
    case 128: return cross_launch_width<T, 128>(p, few, s);
    case 192: return cross_launch_width<T, 192>(p, few, s);
    default: return cross_launch_width<T, 256>(p, few, s);
  }
}
extern template int cross_launch<f16_t>(const CrossLaunch&, int, bool, hipStream_t);
extern template int cross_launch<bf16_t>(const CrossLaunch&, int, bool, hipStream_t);
extern template int cross_launch<float>(const CrossLaunch&, int, bool, hipStream_t);

}  // namespace wmdec
