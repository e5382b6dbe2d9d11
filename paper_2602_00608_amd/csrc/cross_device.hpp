// The kernel of kernels_cross.hip: attention of rows (a token of one of the query heads that share a key head) to the keys of a sample.
//
// Tiles of KT keys and values stream through LDS, straight from memory (16 bytes a lane), while the tile before is worked on.  With a mask a tile is made of
// valid keys alone: a lane chooses what it reads, so their places are worked out first and the others are neither read nor reckoned with.  Per 32 keys a
// wavefront forms S^T = K Q^T (keys along the accumulator's registers, one row a lane), the softmax against a running maximum, and O^T += V^T P^T with the
// probabilities as they are in their registers: an accumulator's keys of lane half lk are 8 (r / 4) + 4 lk + r % 4, so V^T is read from LDS in that order of
// keys (16-bit types: transposed on the way, four keys of one channel a lane).  fp32 takes the same steps with 32x32x2 products.
// The wavefronts of a workgroup take 32 rows each (QW of them), or, where there are few rows, the same rows and a part of a tile's keys (KW), joined at the end.
//
// 16-byte chunk c of key r lies at chunk c ^ turn(r) of its row in LDS: eight neighbouring lanes over K (eight keys, one chunk) and sixteen over V (four keys, two
// chunks) then have banks of their own.  (Twice as many lanes do not: a third of the LDS cycles at 64 channels and half at 128 are conflicts.  A turn of 32 keys that
// frees V of them, half of those at 128, is no faster: 3 x 4096x4096 of 16 heads 474 / 474 us.)  The loads bring the chunks in that order, as a lane chooses what it reads and not where it lands.
//
// What bounds it.  Few rows: the one read of the keys and values; two workgroups of 32 rows a compute unit, with 128 KB of tiles under way.  Many rows in
// 16 bits: the power that the matrix cores may draw, and at 64 channels the exponentials, which take as many cycles as the products (32 rows and 64 keys of a
// wavefront: 16 products of 32 cycles, 32 exponentials of 8 beside 32 each of multiply-add, add and half a maximum and a conversion).  fp32: its products.
// Rates: one token of 32 heads against 16 x 4096 keys of 8 heads of 128 48.1 us = 5.58 TB/s on the inputs of the call before, 58.9 on others; 8192x8192 of 32 / 8 heads
// of 128 1040 to 1150 us = 1060 to 950 TFLOP/s (a large library product on this card 1090 to 1150); 5400x5400 of 30 heads of 64 280 to 310 us = 720 to 800, of 96
// heads 870 to 890 (1290 workgroups are 1.26 rounds of the 1024 that run at once); fp32 4000x2000 of 8 heads of 128 266 us = 123 of 155.
// Steps, us for 5400x5400 of 30 of 64 f16, 2 x 5400x512 of 30 of 64 bf16 (two lengths), 1 token against 4 x 32768 (ragged) of 8 of 128: a wavefront a row 92950, 9854,
// 50355; matrix cores, tiles through LDS, transposed reads 298, 66, 128; tiles by instructions that the compiler does not wait for 298, 66, 110; 128 rows a workgroup
// and the XCDs divided within a sample 297, 50, 65; wavefronts past the last row idle 290, 50, 65; ranges joined by as many threads as there are rows 62 of the last.  With a fifth of the keys masked, by a mask on the scores and zeros in place of masked values / by tiles of valid
// keys: 5400x5400 of 30 of 64 in bf16 361 / 240 (280 without a mask), 4096x4096 of 16 of 128 168 / 117, 333x301 of 8 of 72 in fp32 20.0 / 15.3.  160 channels as 192 / as
// themselves, with two workgroups a compute unit: 4000x4000 of 30 heads in f16 528 / 338.
// Measured and not kept: 64 rows a wavefront (128 channels 818 TFLOP/s against 1005: half the wavefronts), wave priorities around the products, the compiler's own
// interleaving of them, sums by dot products (4 cycles against 2), a loop over pairs of tiles, tiles of 32 keys and three workgroups a compute unit at 128 channels (8192x8192 1026
// against 1045, but 4096x4096 of 16 heads 168 against 158), ranges for the last round's blocks alone (partial outputs cost what
// they gain).
#pragma once
#include <algorithm>
#include <atomic>

#include "conv_device.hpp"

namespace wmdec {

// How the work is divided (kernels_cross.hip decides).  A block is BQ rows of a key head; it is a workgroup that writes the output, or `splits` workgroups that
// take a range of the keys each and leave partial outputs, and a launch that joins these.
struct CrossPlan {
  int width = 0;                  // channels that the kernel is made for
  bool few = false;               // 32 rows a workgroup, whose wavefronts share them; else 128
  int rows = 0, row_blocks = 0, splits = 1;   // rows of a key head, blocks of them
};
struct CrossLaunch {
  CrossArgs a;
  CrossPlan plan;
  float* part;                    // [sample][key head][row block][split][BQ][width] sums of probabilities times values
  float2* ml;                     // [sample][key head][row block][split][BQ] reference and sum of the probabilities
};

template <typename T> constexpr int kChunkElems = 16 / (int)sizeof(T);

template <int CH> __device__ __forceinline__ int chunk_turn(int row) {   // CH: chunks of a key, a multiple of 4
  if constexpr (CH % 8 == 0) return ((row & 3) << 1) | ((row >> 2) & 1);
  else return (row & 2) | ((row >> 2) & 1);   // (rows alternate between the halves of 128 bytes by themselves)
}

__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }   // (NaN if one is: one instruction for three)

constexpr int kMaskKeys = 2048;       // keys whose mask is read at a time; the places of the valid ones among them, as 16 bits

// D: channels, rounded up to a multiple of 32; QW x KW wavefronts of 32 rows and 1 / KW of a tile's keys
template <typename T, int D, int QW, int KW, int KT>
struct CrossForm {
  static constexpr int EC = kChunkElems<T>, CH = D / EC, NW = QW * KW, NT = 64 * NW, SUB = KT / KW, NS = SUB / 32, LOADS = KT * CH / NT, BQ = 32 * QW;
  static constexpr int TILE = KT * D, NB = KW == 1 ? 2 : 1;   // buffers of keys, and of values
  static constexpr int RED = D + 4;   // floats from row to row of the outputs that are joined
  static constexpr int kTiles = 2 * NB * TILE * (int)sizeof(T), kRed = KW == 1 ? 0 : KW * 32 * (RED + 2) * 4, kLow = kTiles > kRed ? kTiles : kRed, kMask = kMaskKeys * 2 + kMaskKeys / 64 * 4;   // (the last only with a mask)
  static_assert(D % 32 == 0 && KT % (32 * KW) == 0 && KT * CH % NT == 0 && (KW == 1 || QW == 1));
  static_assert(kLow + kMask <= 160 * 1024 && LOADS < 64);
};

// Tiles are asked for and waited for in assembly: the compiler would wait for all of them in front of every transposed read.  No registers are written.
// 16 bytes a lane from `offset` + `more` of the buffer to lds + AT + 16 * lane; past the buffer's end the LDS gets zeros.  (Nothing else here uses M0.)
template <int AT> __device__ __forceinline__ void load_to_lds(u32x4 buffer, unsigned offset, unsigned more, unsigned lds) {
  asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(lds), "v"(offset), "s"(buffer), "s"(more), "n"(AT) : "memory", "scc");
}
// all but the last N loads of this wavefront have landed
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }
// every load and LDS access of this wavefront is done, and so for the others
__device__ __forceinline__ void sync_tiles() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory"); }
// the same for LDS accesses alone: tiles on their way are not waited for
__device__ __forceinline__ void sync_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }
constexpr unsigned kPastEnd = 0x80000000u;   // an offset that no buffer reaches

// what a sum taken against the reference m counts for against the reference `top`, which is at least m (nothing seen yet: nothing)
__device__ __forceinline__ float weight_of(float m, float top) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top); }
// four channels of a row from channel `at` on, if it has them
template <typename T> __device__ __forceinline__ void store_quad(T* row, int at, int d, f32x4 v) {
  if (at >= d) return;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(row + at) = v;
  else *reinterpret_cast<u32x2*>(row + at) = u32x2{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
}

constexpr float kCrossSlack = 8.0f;   // log2 of how far a tile's maximum may exceed the reference before that moves

// MASKED: tiles are made of the valid keys alone, whose places are worked out for up to kMaskKeys keys at a time
template <typename T, int D, int QW, int KW, int KT, int WAVES, bool MASKED>
__global__ __launch_bounds__(64 * QW * KW, WAVES) void cross_attention_kernel(CrossLaunch launch) {
  using F = CrossForm<T, D, QW, KW, KT>;
  constexpr int EC = F::EC, CH = F::CH, NW = F::NW, NS = F::NS, LOADS = F::LOADS, TILE = F::TILE, NB = F::NB, QS = CH / 2, ND = D / 32;
  constexpr int GP = CH % 8 == 0 ? 8 : 4;   // chunks that are exchanged among each other
  constexpr bool WIDE = sizeof(T) == 4, OWN = KW > 1;   // OWN: a wavefront loads the keys it works on, and waits for nobody
  extern __shared__ __align__(16) unsigned char smem[];
  T* s_k = reinterpret_cast<T*>(smem);      // [NB] tiles
  T* s_v = s_k + NB * TILE;
  unsigned short* s_place = reinterpret_cast<unsigned short*>(smem + F::kLow);   // [kMaskKeys] valid keys
  int* s_count = reinterpret_cast<int*>(smem + F::kLow + kMaskKeys * 2);          // [kMaskKeys / 64] how many of 64 keys are valid
  const CrossArgs& a = launch.a;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, lk = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), qw = wave / KW, kw = wave % KW;
  // workgroup id -> (sample, key head, range of keys, row block); within a sample the ids of one XCD (id % 8) are neighbours and share their keys.  (Neighbours over
  // all samples: an XCD had one sample's work, and where samples have different lengths those with long ones ran alone.)
  const CrossPlan& p = launch.plan;
  const int per_sample = a.heads * p.splits * p.row_blocks, turn = blockIdx.x / per_sample;
  // Samples of many blocks come longest first (a short one's workgroups end the launch sooner together).
  int n = turn;
  if (KW == 1 && a.lens && a.n > 1 && a.n <= 64) {
    const int mine = lane < a.n ? min(max(a.lens[lane], 0), a.tk) : -1;
    int before = 0;
    for (int j = 0; j < a.n; ++j) {
      const int other = __builtin_amdgcn_readlane(mine, j);
      before += other > mine || (other == mine && j < lane);
    }
    n = __builtin_ctzll(__ballot(before == turn));
  }
  int L;
  {
    const int i = blockIdx.x - turn * per_sample, per = per_sample / 8, rem = per_sample % 8, x = i % 8, j = i / 8;
    L = x * per + (x < rem ? x : rem) + j;
  }
  const int rb = L % p.row_blocks, split = L / p.row_blocks % p.splits, h = L / (p.row_blocks * p.splits);
  const int len = a.lens ? min(max(a.lens[n], 0), a.tk) : a.tk;
  const int tiles = (len + KT - 1) / KT, first = (int)((long)split * tiles / p.splits), nt = (int)((long)(split + 1) * tiles / p.splits) - first;
  const int begin = first * KT, end = min((long)len, (long)(first + nt) * KT);   // keys of the range

  // ---- tiles.  A load is 64 consecutive chunks of a tile; chunks past the last channel and keys past the last one are read past the buffer's end
  const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const char* kp = (const char*)a.k + (n * a.ks.sample + h * a.ks.head) * (long)sizeof(T);
  const char* vp = (const char*)a.v + (n * a.vs.sample + h * a.vs.head) * (long)sizeof(T);
  const int kstep = (int)(a.ks.token * (long)sizeof(T)), vstep = (int)(a.vs.token * (long)sizeof(T));   // (128 of them are below 2^31: checked on the host)
  auto slot0 = [&](int i) { return OWN ? wave * F::SUB * CH + i * 64 : (i * NW + wave) * 64; };
  // Offsets of the loads: every PER-th one has the same chunks of keys that are a multiple of eight further, a scalar part of the address.
  constexpr int ROWS = 64 % CH == 0 ? 64 / CH * (OWN ? 1 : NW) : 0;   // keys from a load to the next; 0: loads end inside a key
  constexpr int PER = ROWS == 0 ? LOADS : ROWS % 8 == 0 ? 1 : 8 / ROWS < LOADS ? 8 / ROWS : LOADS;
  unsigned koff[PER], voff[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = (slot0(i) + lane) / CH, c = ((slot0(i) + lane) % CH) ^ chunk_turn<CH>(r);
    koff[i] = c * EC < a.d ? (unsigned)((MASKED ? 0 : r * kstep) + c * 16) : kPastEnd;
    voff[i] = c * EC < a.d ? (unsigned)((MASKED ? 0 : r * vstep) + c * 16) : kPastEnd;
  }
  int k0 = begin, count = 0;   // the keys at work: `count` from k0 on, or the valid ones among those from k0 on
  constexpr int PLACES = MASKED ? LOADS : 1;
  // Outputs and queries of 256 channels leave no registers for a lane's chunks and keys: worked out for every tile, from a lane number that the compiler does not know.
  constexpr bool AGAIN = MASKED && !WIDE && D == 256 && !OWN;
  auto keys_of = [&](int j, int& ln, unsigned (&place)[PLACES]) {
    ln = lane;
    if constexpr (AGAIN) asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(ln));
    if constexpr (MASKED) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) place[i] = s_place[j * KT + (slot0(i) + ln) / CH];   // (past the last one: below kMaskKeys still, and not used)
    }
  };
  auto ask = [&](const char* base, int step, const unsigned (&off)[PER], int at, int j, int ln, const unsigned (&place)[PLACES]) {
    const int left = count - j * KT;
    const uint64_t from = (uint64_t)(base + (k0 + (MASKED ? 0L : (long)j * KT)) * step);
    const u32x4 buffer{(unsigned)from, (unsigned)(from >> 32) & 0xffffu, kPastEnd - 1, 0x00020000u};
    const unsigned to = lds + (at + (NB == 2 ? j & 1 : 0) * TILE) * (int)sizeof(T) + slot0(0) * 16;
    unsigned more = 0;
    static_for<LOADS>([&](auto i_c) {
      constexpr int i = decltype(i_c)::value;
      if constexpr (!MASKED && i > 0 && i % PER == 0) {
        more += PER * ROWS * step;
        asm volatile("" : "+s"(more));   // (one after the other: worked out beforehand for all loads they do not fit the scalar registers)
      }
      const int r = (slot0(i) + ln) / CH;
      unsigned o;
      if constexpr (AGAIN) {
        const int c = ((slot0(i) + ln) % CH) ^ chunk_turn<CH>(r);
        o = c * EC < a.d ? (unsigned)(c * 16) : kPastEnd;
      } else {
        o = off[i % PER];
      }
      if constexpr (MASKED) o = r < left ? o + place[i] * (unsigned)step : kPastEnd;   // (below 2^32: a place times the step is below 2^31)
      else if (left < KT) o = r < left ? o : kPastEnd;
      load_to_lds<i * (OWN ? 1 : NW) * 1024>(buffer, o, more, to);
    });
  };
  auto ask_one = [&](bool values, int j) {
    int ln;
    unsigned place[PLACES];
    keys_of(j, ln, place);
    if (values) ask(vp, vstep, voff, NB * TILE, j, ln, place);
    else ask(kp, kstep, koff, 0, j, ln, place);
  };
  auto ask_k = [&](int j) { ask_one(false, j); };
  auto ask_v = [&](int j) { ask_one(true, j); };
  auto ask_both = [&](int j) {
    int ln;
    unsigned place[PLACES];
    keys_of(j, ln, place);
    ask(kp, kstep, koff, 0, j, ln, place);
    ask(vp, vstep, voff, NB * TILE, j, ln, place);
  };

  // ---- queries: chunk 2 s + lk of the lane's row
  const int row = rb * F::BQ + qw * 32 + l32;
  const bool idle = rb * F::BQ + qw * 32 >= p.rows;   // a wavefront past the last row only loads
  u32x4 q[QS];
  {
    const int r = min(row, p.rows - 1), tok = r / a.group, hq = h * a.group + (r - tok * a.group);
    const T* src = (const T*)a.q + n * a.qs.sample + tok * a.qs.token + hq * a.qs.head;
#pragma unroll
    for (int s = 0; s < QS; ++s) {
      const int c = (2 * s + lk) * EC;
      q[s] = u32x4{0, 0, 0, 0};
      if (c < a.d) q[s] = *reinterpret_cast<const u32x4*>(src + c);
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

  f32x16 o[ND];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  const float c = a.scale * 1.4426950408889634f;

  f32x16 s[NS];
  // Fragments.  Where a SIMD has few wavefronts (EAGER) they are read RK and RV ahead of their products, in that order; else the compiler places them.
  constexpr bool EAGER = OWN || WIDE;
  constexpr int KF = NS * QS, RK = WIDE || D > 192 ? 4 : 8, VF = NS * (WIDE ? 16 : 2) * ND, RV = D > 192 ? 4 : 8;
  u32x4 kr[RK];
  typename std::conditional<WIDE, float, u32x4>::type vr[RV];
  auto key_fragment = [&](const T* tk, auto i_c) -> u32x4 {        // i = ns * QS + step
    constexpr int i = decltype(i_c)::value, ns = i / QS, st = i % QS;
    return *reinterpret_cast<const u32x4*>(tk + kb[st % (GP / 2)] + st / (GP / 2) * GP * EC + ns * 32 * D);
  };
  auto value_fragment = [&](const T* tv, auto i_c) {               // i = (ns, register or half of 32 keys, channel tile)
    constexpr int i = decltype(i_c)::value, dt = i % ND;
    if constexpr (WIDE) {
      constexpr int r = i / ND % 16, ns = i / ND / 16;
      return to_float(tv[vb[r % 4] + (ns * 32 + 8 * (r / 4)) * D + dt * 32]);
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4* tptr_t;
      const T* at = tv + vb[dt % (GP / 4)] + dt / (GP / 4) * GP * EC + i / ND * 16 * D;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)at));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)(at + 8 * D)));
      return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  };
  auto score_step = [&](const u32x4& kf, auto i_c) {
    constexpr int i = decltype(i_c)::value, ns = i / QS, st = i % QS;
    if constexpr (st == 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[ns][r] = 0.f;
    }
    if constexpr (WIDE) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[ns] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(q[st][e]), s[ns], 0, 0, 0);
    } else {
      s[ns] = Mma<T>::m32(kf, q[st], s[ns]);
    }
  };
  // scores of a tile (its valid keys in `bits`)
  auto scores = [&](const T* tk, const unsigned (&bits)[NS]) {
    if constexpr (EAGER) {
      static_for<(RK < KF ? RK : KF)>([&](auto i) { kr[decltype(i)::value] = key_fragment(tk, i); });
      static_for<KF>([&](auto i_c) {
        constexpr int i = decltype(i_c)::value;
        __builtin_amdgcn_sched_barrier(0);
        score_step(kr[i % RK], i_c);
        if constexpr (i + RK < KF) kr[i % RK] = key_fragment(tk, std::integral_constant<int, i + RK>{});
      });
      __builtin_amdgcn_sched_barrier(0);
    } else {
      static_for<KF>([&](auto i) { score_step(key_fragment(tk, i), i); });
    }
#pragma unroll
    for (int ns = 0; ns < NS; ++ns)
      if (bits[ns] != ~0u) {
        const unsigned b = bits[ns] >> (4 * lk);
#pragma unroll
        for (int r = 0; r < 16; ++r) {   // -inf where the bit is not set, in two instructions: the bit spread over the word, and a choice by it
          const unsigned is = (unsigned)((int)(b << (31 - 8 * (r / 4) - r % 4)) >> 31);
          s[ns][r] = __uint_as_float((is & __float_as_uint(s[ns][r])) | (~is & 0xff800000u));
        }
      }
  };
  // The reference is a rounded product.  From 2^24 on a fused multiply-add would find the largest score half a step of the reference away from it, 1 and more: its
  // probability is not 1 but anything between none and infinity.  There the products are rounded like the reference, and then subtracted.
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
  // The reference moves when a maximum exceeds it by 2^kCrossSlack; until then probabilities may reach that, well inside the 16-bit types.
  auto softmax = [&]() {
    float mx = maximum(maximum(s[0][0], s[0][1]), s[0][2]);
#pragma unroll
    for (int i = 3; i + 1 < 16 * NS; i += 2) mx = maximum(maximum(mx, s[i / 16][i % 16]), s[(i + 1) / 16][(i + 1) % 16]);
    mx = maximum(mx, s[NS - 1][15]);
    mx = half_max(mx) * c;
    const bool moves = mx > m + kCrossSlack;
    if (__ballot(moves)) {
      const float to = moves ? mx : m, factor = moves ? __builtin_amdgcn_exp2f(m - mx) : 1.f;
      m = to;
      far = __ballot(fabsf(m) >= 0x1p24f && m != -INFINITY) != 0;
      l *= factor;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
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
  auto values_head = [&](const T* tv) {
    if constexpr (EAGER) {
      static_for<(RV < VF ? RV : VF)>([&](auto i) { vr[decltype(i)::value] = value_fragment(tv, i); });
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto values = [&](const T* tv) {
    u32x4 pf;   // the one rounding inside the operator: probabilities as operands of T
    auto value_step = [&](const auto& vf, auto i_c) {
      constexpr int i = decltype(i_c)::value, dt = i % ND;
      if constexpr (WIDE) {
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[i / ND / 16][i / ND % 16], o[dt], 0, 0, 0);
      } else {
        constexpr int ns = i / ND / 2, ks = i / ND % 2;
        if constexpr (dt == 0) {
#pragma unroll
          for (int w = 0; w < 4; ++w) pf[w] = pack2<T>(s[ns][8 * ks + 2 * w], s[ns][8 * ks + 2 * w + 1]);
        }
        o[dt] = Mma<T>::m32(vf, pf, o[dt]);
      }
    };
    if constexpr (EAGER) {
      static_for<VF>([&](auto i_c) {
        constexpr int i = decltype(i_c)::value;
        __builtin_amdgcn_sched_barrier(0);
        value_step(vr[i % RV], i_c);
        if constexpr (i + RV < VF) vr[i % RV] = value_fragment(tv, std::integral_constant<int, i + RV>{});
      });
    } else {
      static_for<VF>([&](auto i) { value_step(value_fragment(tv, i), i); });
    }
  };

  const int stage = min(kMaskKeys, (int)((kPastEnd - 1) / (unsigned)max(max(kstep, vstep), 1)) & -64);   // (at least 64; all of them within a buffer)
  while (k0 < end) {   // without a mask once
    const int here = MASKED ? min(end - k0, stage) : end - k0;
    if constexpr (MASKED) {
      constexpr int WORDS = kMaskKeys / 64 / NW;
      const unsigned char* mask = a.mask + (long)n * a.tk + k0;
      if (k0 != begin) sync_tiles();   // (the places before have been read)
      bool set[WORDS];
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        const int key = (i * NW + wave) * 64 + lane;
        set[i] = mask[min(key, here - 1)] != 0 && key < here;
      }
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        const int valid = __popcll(__ballot(set[i]));
        if (lane == 0) s_count[i * NW + wave] = valid;
      }
      sync_lds();
      const int own = s_count[l32];
      int upto = own;                  // valid keys up to the 64 of number l32
#pragma unroll
      for (int step = 1; step < kMaskKeys / 64; step *= 2) {
        const int before = __shfl_up(upto, step, kMaskKeys / 64);
        if (l32 >= step) upto += before;
      }
      count = __builtin_amdgcn_readlane(upto, kMaskKeys / 64 - 1);
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        const int at = __builtin_amdgcn_readlane(upto - own, i * NW + wave);
        const unsigned long long word = __ballot(set[i]);
        if (set[i]) s_place[at + __builtin_amdgcn_mbcnt_hi((unsigned)(word >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)word, 0))] = (unsigned short)((i * NW + wave) * 64 + lane);
      }
      sync_lds();
    } else {
      count = here;
    }
    const int nb = (count + KT - 1) / KT;
    // valid keys of the wavefront's part of tile j
    bool none;
    auto valid = [&](int j, unsigned (&bits)[NS]) {
      none = true;
#pragma unroll
      for (int ns = 0; ns < NS; ++ns) {
        const int left = count - j * KT - kw * F::SUB - ns * 32;
        bits[ns] = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1;
        none = none && bits[ns] == 0;
      }
    };
    unsigned bits[NS];
    // (the queries are waited for here: the compiler, which does not see the tiles' loads, would wait for all of them wherever it first uses a query)
    auto queries_landed = [&]() {
#pragma unroll
      for (int s = 0; s < QS; ++s) asm volatile("" : "+v"(q[s]));
    };
    if constexpr (OWN) {
      // One buffer of either, asked for again as soon as it has been read: the next keys travel behind the softmax and the values, the next values behind the
      // scores.  (Two buffers each: half the workgroups a compute unit, and slower throughout, the main launch of 16 x 4096 keys of 8 heads of 128 channels by 19 us.)
      if (nb) { ask_k(0); ask_v(0); }
      queries_landed();
      static_assert(!OWN || NS == 1, "a wavefront has 32 keys of a tile");
      T *tk = s_k + kw * F::SUB * D, *tv = s_v + kw * F::SUB * D;
      for (int j = 0; j < nb; ++j) {
        const bool more = j + 1 < nb;
        valid(j, bits);
        wait_loads<LOADS>();
        if (!none) scores(tk, bits);
        __builtin_amdgcn_sched_barrier(0);
        if (more) { ask_k(j + 1); wait_loads<LOADS>(); }
        else wait_loads<0>();
        if (!none) {
          values_head(tv);
          softmax();
          values(tv);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) ask_v(j + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      if (nb) ask_both(0);
      queries_landed();
      for (int j = 0; j < nb; ++j) {
        sync_tiles();       // the tile has landed, and every wavefront is done with the other buffer
        T *tk = s_k + (j & 1) * TILE, *tv = s_v + (j & 1) * TILE;
        if (j + 1 < nb) ask_both(j + 1);
        valid(j, bits);
        if (idle) continue;
        scores(tk, bits);
        values_head(tv);
        softmax();
        values(tv);
      }
    }
    k0 += here;
  }

  // ---- output.  A lane holds channels 32 dt + 8 g + 4 lk .. + 3 of its row
  l += __shfl_xor(l, 32);
  const long part0 = ((((long)n * a.heads + h) * p.row_blocks + rb) * p.splits + split) * F::BQ;   // first row of the partial outputs
  auto output = [&](int r) -> T* {
    const int tok = r / a.group, hq = h * a.group + (r - tok * a.group);
    return (T*)a.o + n * a.os.sample + tok * a.os.token + hq * a.os.head;
  };
  if constexpr (KW == 1) {
    if (row >= p.rows) return;
    if (p.splits > 1) {
      const long at = part0 + qw * 32 + l32;
      if (lk == 0) launch.ml[at] = make_float2(m, l);
      float* dst = launch.part + at * D + 4 * lk;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4*>(dst + 32 * dt + 8 * g) = f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
      return;
    }
    T* dst = output(row);
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) store_quad<T>(dst, 32 * dt + 8 * g + 4 * lk, a.d, f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]} * inv);
  } else {
    float* s_o = reinterpret_cast<float*>(smem);                          // [KW][32][RED]
    float2* s_ml = reinterpret_cast<float2*>(s_o + KW * 32 * F::RED);     // [KW][32]
    sync_tiles();
    if (lk == 0) s_ml[kw * 32 + l32] = make_float2(m, l);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(s_o + (kw * 32 + l32) * F::RED + 32 * dt + 8 * g + 4 * lk) = f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
    sync_lds();
    for (int i = tid; i < 32 * D / 4; i += F::NT) {
      const int r = i / (D / 4), at = i % (D / 4) * 4;
      if (rb * 32 + r >= p.rows || at >= a.d) continue;
      float top = s_ml[r].x, den = 0.f;
#pragma unroll
      for (int w = 1; w < KW; ++w) top = fmaxf(top, s_ml[w * 32 + r].x);
      f32x4 num{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float2 e = s_ml[w * 32 + r];
        const float f = weight_of(e.x, top);
        den = fmaf(e.y, f, den);
        num += f * *reinterpret_cast<const f32x4*>(s_o + (w * 32 + r) * F::RED + at);
      }
      if (p.splits > 1) {
        if (at == 0) launch.ml[part0 + r] = make_float2(top, den);
        *reinterpret_cast<f32x4*>(launch.part + (part0 + r) * D + at) = num;
      } else {
        store_quad<T>(output(rb * 32 + r), at, a.d, num * (den == 0.f ? 0.f : 1.f / den));
      }
    }
  }
}

// o = sum_s part_s 2^(m_s - M) / sum_s l_s 2^(m_s - M) for the rows of the blocks that are split (`total` of all key heads, `bq` a block).  A thread takes four
// channels of a row and every groups-th range, eight at a time; the groups of a row are joined in order.  Bound by latency: one trip.
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_combine_kernel(CrossLaunch launch, int bq, int groups, unsigned total) {
  constexpr int QUADS = D / 4, UNITS = 256 / QUADS, B = 8;
  __shared__ f32x4 s_num[UNITS][QUADS];
  __shared__ float2 s_ml[UNITS];
  const CrossArgs& a = launch.a;
  const CrossPlan& p = launch.plan;
  const int unit = threadIdx.x / QUADS, quad = threadIdx.x % QUADS, g = unit % groups, in_block = UNITS / groups;
  for (unsigned r0 = blockIdx.x * in_block; r0 < total; r0 += gridDim.x * in_block) {
    const unsigned r = r0 + unit / groups, nh = r / p.rows;                          // row among those of all key heads, its sample and key head
    const int row = (int)(r - nh * p.rows), n = nh / a.heads, h = nh - n * a.heads, in = row % bq;
    const long pb = (long)nh * p.row_blocks + row / bq;
    const bool there = unit < in_block * groups && r < total;
    float top = -INFINITY, den = 0.f;
    f32x4 num{0.f, 0.f, 0.f, 0.f};
    auto join = [&](float m, float l, f32x4 v) {
      const float now = fmaxf(top, m), keep = weight_of(top, now), f = weight_of(m, now);
      den = den * keep + l * f;
      num = num * keep + v * f;
      top = now;
    };
    if (there && quad * 4 < a.d) {
      for (int s0 = g; s0 < p.splits; s0 += B * groups) {
        float2 e[B];
        f32x4 v[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
          const long at = (pb * p.splits + min(s0 + b * groups, p.splits - 1)) * bq + in;
          e[b] = launch.ml[at];
          v[b] = *reinterpret_cast<const f32x4*>(launch.part + at * D + quad * 4);
        }
#pragma unroll
        for (int b = 0; b < B; ++b)
          if (s0 + b * groups < p.splits) join(e[b].x, e[b].y, v[b]);
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
    if (g == 0 && there) {
      const int tok = row / a.group, hq = h * a.group + (row - tok * a.group);
      store_quad<T>((T*)a.o + n * a.os.sample + tok * a.os.token + hq * a.os.head, quad * 4, a.d, num * (den == 0.f ? 0.f : 1.f / den));
    }
  }
}

template <typename T, int D, int QW, int KW, int KT, int WAVES, bool MASKED>
int cross_launch_kernel(const CrossLaunch& l, hipStream_t s) {
  using F = CrossForm<T, D, QW, KW, KT>;
  constexpr int smem = F::kLow + (MASKED ? F::kMask : 0);
  auto kern = cross_attention_kernel<T, D, QW, KW, KT, WAVES, MASKED>;
  static std::atomic<unsigned long long> known{0};   // devices that the kernel's LDS has been asked for on
  int device = 0;
  WMDEC_HIP(hipGetDevice(&device));
  const unsigned long long bit = 1ull << (device & 63);
  if (!(known.load() & bit)) {
    WMDEC_HIP(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, smem));
    known.fetch_or(bit);
  }
  const CrossPlan& p = l.plan;
  hipLaunchKernelGGL(kern, dim3((unsigned)((long)l.a.n * l.a.heads * p.row_blocks * p.splits)), dim3(F::NT), smem, s, l);
  WMDEC_HIP(hipGetLastError());
  if (p.splits > 1) {
    constexpr int units = 256 / (D / 4);
    // As many groups as there are eights of ranges; nothing that depends on the number of samples, as the groups decide which ranges are added before which.  us, with
    // as many as there are ranges / so: 700x3000 of 4 heads of 96 in f16 (6 ranges) 22.4 / 18.7, four samples 52.8 / 36.0, 16 x 4096 keys of 8 of 128 (16) 60.3 / 59.6,
    // 32768 keys (64) 34.1 / 34.1.
    int groups = 1;
    while (groups * 2 <= units && groups * 8 < p.splits) groups *= 2;
    const long total = (long)l.a.n * l.a.heads * p.rows, in_block = units / groups, most = 8192;   // rows (below 2^26: cross_attention_fits); rows and most workgroups of a launch
    hipLaunchKernelGGL((cross_combine_kernel<T, D>), dim3((unsigned)std::min(most, (total + in_block - 1) / in_block)), dim3(256), 0, s, l, F::BQ, groups, (unsigned)total);
    WMDEC_HIP(hipGetLastError());
  }
  return WMDEC_OK;
}

template <typename T, int D, int QW, int KW, int KT, int WAVES>
int cross_launch_form(const CrossLaunch& l, hipStream_t s) {
  return l.a.mask ? cross_launch_kernel<T, D, QW, KW, KT, WAVES, true>(l, s) : cross_launch_kernel<T, D, QW, KW, KT, WAVES, false>(l, s);
}

// Keys of a tile, wavefronts a SIMD.  Where 128 rows have a workgroup: 64 keys in 16 bits while the tiles of two workgroups fit a compute unit (up to 160 channels), else 32
// (us, 64 keys and one workgroup / 32 and two: 3 x 4096x4096 of 16 heads of 256 in bf16 1088 / 792, 3 x 3000x3000 of 16 of 192 in f16 459 / 362).  fp32: 64 up to 128 channels,
// where 32 and two workgroups gain nothing (2000x2000 of 8 of 128 154 / 150, 3 x 2402x1124 of 8 / 2 of 72 111 / 129), else 32.
template <typename T, int D>
int cross_launch_width(const CrossLaunch& l, hipStream_t s) {
  constexpr int bytes = D * (int)sizeof(T);   // of a key
  if constexpr (bytes <= 768) {
    if (l.plan.few) return cross_launch_form<T, D, 1, (bytes <= 512 ? 4 : 2), (bytes <= 512 ? 128 : 64), (bytes <= (sizeof(T) == 2 ? 320 : 256) ? 2 : 1)>(l, s);
  }
  return cross_launch_form<T, D, 4, 1, (bytes <= (sizeof(T) == 2 ? 320 : 512) ? 64 : 32), (sizeof(T) == 2 && D <= 64 ? 4 : bytes <= 640 ? 2 : 1)>(l, s);
}

template <typename T>
int cross_launch(const CrossLaunch& l, hipStream_t s) {
  switch (l.plan.width) {
    case 32: return cross_launch_width<T, 32>(l, s);
    case 64: return cross_launch_width<T, 64>(l, s);
    case 96: return cross_launch_width<T, 96>(l, s);
    case 128: return cross_launch_width<T, 128>(l, s);
    case 160: return cross_launch_width<T, 160>(l, s);
    case 192: return cross_launch_width<T, 192>(l, s);
    default: return cross_launch_width<T, 256>(l, s);
  }
}
extern template int cross_launch<f16_t>(const CrossLaunch&, hipStream_t);
extern template int cross_launch<bf16_t>(const CrossLaunch&, hipStream_t);
extern template int cross_launch<float>(const CrossLaunch&, hipStream_t);

}  // namespace wmdec
