// Gated residual with the norms on both of its sides: x' = x + s * g * P(h), y = N(x') * (1 + c) + b, rows of d channels.
//
// Bound by HBM: x and h are read once, x' and y written once, some twenty operations an element.  The vectors of a sample (gate, shift, scale, the
// norms' weights and biases: up to seven times four bytes a channel, more than a row of 16-bit tensors has) would be read again for every row, so a
// thread owns eight channels of many rows and keeps what they come to in registers, two multiply-adds an element:
//   x' = x + ((h - mean) * rstd) * ga + gb,   ga = s * g * w, gb = s * g * u;     y = ((x' - mean) * rstd) * ya + yb,   ya = w (1 + c), yb = u (1 + c) + b.
// A row is 8 to 64 lanes of a wavefront (up to 512 channels, four rows of them and more a workgroup), or whole wavefronts of one; the next row is requested before the present one
// is reduced.  Moments: mean and squares about it over the values of a wavefront, joined over the wavefronts (Chan, Golub, LeVeque) behind one barrier a norm.
// us on inputs from memory, with the rate: 2x5400 rows of 1920 in bf16 38.1 (4.36 TB/s), 4x5400 rows of 1152, fp32 beside f16, 62.7 (4.76; a copy of 4 GiB 4.89).
// Steps: a row a workgroup 318 and 405; this form with ranges of rows, two rows at a time, in 1.3 rounds of workgroups 50.5 and 84.2; one round 42.7 and 71.0; a row at
// a time 40.8 and 68.6; the workgroups' rows side by side, so that what is under way lies together in memory, 38.1 and 62.7.  Measured and not kept: two and
// eight rounds of workgroups (39.8 and 69.4, 50.4 and 72.3), stores or loads that pass the caches by (42.1 and 72.4, 44.9 and 74.6).
#include "conv_device.hpp"

namespace wmdec {
namespace {

constexpr int kMaxThreads = 512;   // of a workgroup: 4096 channels at a vector a thread
constexpr int E = 8;               // channels of a vector

struct Params {
  ResidualNormArgs a;
  int tpr, segs;   // threads of a row, workgroups of a sample
};

// A thread's eight channels of a vector are consecutive where rows are aligned; where they are not, they are `gap` apart, so that the lanes of every load and
// store are next to each other.  `count` of them are there.
template <typename T, bool VEC> __device__ __forceinline__ void load8(const T* p, int count, int gap, T (&v)[E]) {
  if constexpr (VEC) {
    u32x4 q[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = u32x4{0, 0, 0, 0};
    if (count > 0) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = reinterpret_cast<const u32x4*>(p)[i];
    }
    __builtin_memcpy(&v, &q, sizeof(v));
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < count ? p[e * gap] : T{};
  }
}
template <typename T, bool VEC> __device__ __forceinline__ void store8(T* p, int count, int gap, const float (&v)[E]) {
  T t[E];
#pragma unroll
  for (int e = 0; e < E; ++e) t[e] = from_float<T>(v[e]);
  if constexpr (VEC) {
    u32x4 q[sizeof(T) / 2];
    __builtin_memcpy(&q, &t, sizeof(t));
    if (count > 0) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<u32x4*>(p)[i] = q[i];
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < count) p[e * gap] = t[e];
  }
}
// Eight of a vector that may be missing.  Places past the row's end get zeros either way: what a norm makes of them (minus its mean) is multiplied by these, and
// has to be nothing in the next norm's sums.
template <bool VEC> __device__ __forceinline__ void vector8(const float* p, long at, int count, int gap, float missing, float (&v)[E]) {
  if (p) load8<float, VEC>(p + at, count, gap, v);
  else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (VEC ? count > 0 : e < count) ? missing : 0.f;
  }
}

// VPT vectors a thread
template <typename TX, typename TA, int VPT, bool VEC>
__global__ __launch_bounds__(kMaxThreads, VPT == 1 ? 4 : 2) void residual_norm_kernel(Params p) {
  __shared__ float4 s_red[2][2][kMaxThreads / 64];
  const ResidualNormArgs& a = p.a;
  const int d = a.d, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool shared = p.tpr <= 64;        // rows of a wavefront's lanes
  const int groups = shared ? (int)blockDim.x / p.tpr : 1, group = shared ? tid / p.tpr : 0, lane = shared ? tid % p.tpr : tid;
  const int n = blockIdx.x / p.segs, seg = blockIdx.x % p.segs;
  const int row0 = seg * groups, step = p.segs * groups;   // (workgroups side by side: the rows under way at a time are next to each other in memory)
  const bool has_h = a.h != nullptr, has_y = a.y != nullptr;
  const int gap = min(p.tpr, 64);
  int col[VPT], count[VPT];
  float held = 0.f;                       // values of this wavefront in a row
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    col[i] = VEC ? (i * p.tpr + lane) * E : i * p.tpr * E + (shared ? lane : wave * 64 * E + (tid & 63));
    count[i] = min(VEC ? max(d - col[i], 0) : max(d - col[i] + gap - 1, 0) / gap, E);
    held += (float)min(max(d - (i * p.tpr + wave * 64) * E, 0), 64 * E);
  }
  const TX* x = (const TX*)a.x + (long)n * a.t * d;
  const TA* h = (const TA*)a.h + (has_h ? (long)n * a.t * d : 0);
  TX* x_out = (TX*)a.x_out + (has_h ? (long)n * a.t * d : 0);
  TA* y = (TA*)a.y + (has_y ? (long)n * a.t * d : 0);

  TX rx[VPT][E];
  TA rh[VPT][E];
  auto ask = [&](int first) {             // past the last row: that one again, not stored
    const long at = (long)min(first + group, a.t - 1) * d;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      load8<TX, VEC>(x + at + col[i], count[i], gap, rx[i]);
      if (has_h) load8<TA, VEC>(h + at + col[i], count[i], gap, rh[i]);
    }
  };
  constexpr bool AHEAD = VPT < 4;         // (four vectors a thread leave no registers for the next rows)
  if (AHEAD) ask(row0);
  __builtin_amdgcn_sched_barrier(0);

  float ga[VPT][E], gb[VPT][E], ya[VPT][E], yb[VPT][E];
  const long mod = (long)n * a.mod_stride;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    float w[E], u[E], m[E];
    if (has_h) {
      vector8<VEC>(a.gate, mod + col[i], count[i], gap, 1.f, m);
      vector8<VEC>(a.post.weight, col[i], count[i], gap, 1.f, w);
      vector8<VEC>(a.post.bias, col[i], count[i], gap, 0.f, u);
#pragma unroll
      for (int e = 0; e < E; ++e) { ga[i][e] = a.res_scale * m[e] * w[e]; gb[i][e] = a.res_scale * m[e] * u[e]; }
    }
    if (has_y) {
      vector8<VEC>(a.scale, mod + col[i], count[i], gap, 0.f, m);
      vector8<VEC>(a.pre.weight, col[i], count[i], gap, 1.f, w);
      vector8<VEC>(a.pre.bias, col[i], count[i], gap, 0.f, u);
#pragma unroll
      for (int e = 0; e < E; ++e) { ya[i][e] = w[e] * (1.f + m[e]); yb[i][e] = u[e] * (1.f + m[e]); }
      vector8<VEC>(a.shift, mod + col[i], count[i], gap, 0.f, m);
#pragma unroll
      for (int e = 0; e < E; ++e) yb[i][e] += m[e];
    }
  }

  const float inv_d = 1.f / (float)d, inv_held = shared ? inv_d : 1.f / fmaxf(held, 1.f);
  auto row_sum = [&](float v) {           // over the lanes of a row, or of a wavefront of it
    v = lane_group_sum<8>(v);
    if (p.tpr > 8) v += mirror16(v);
    if (p.tpr > 16) v = swap_sum<16>(v);
    if (p.tpr > 32) v = swap_sum<32>(v);
    return v;
  };
  // mean and 1 / sqrt(variance + eps) of the row; RMS: the mean is zero
  auto statistics = [&](const wmdec_norm& norm, const float (&v)[VPT][E], int which, int parity, float& mean, float& rstd) {
    mean = 0.f;
    if (norm.kind == WMDEC_NORM_LAYER) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) sum += v[i][e];
      mean = row_sum(sum) * inv_held;
    }
    float m2 = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float part = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float dev = v[i][e] - mean;
        part = VEC || e < count[i] ? fmaf(dev, dev, part) : part;
      }
      m2 += VEC && count[i] == 0 ? 0.f : part;
    }
    m2 = row_sum(m2);
    if (!shared) {
      if ((tid & 63) == 0) s_red[parity][which][wave] = make_float4(mean, m2, held, 0.f);
      __syncthreads();
      const int waves = blockDim.x >> 6;
      float sum = 0.f;
      for (int w = 0; w < waves; ++w) { const float4 q = s_red[parity][which][w]; sum = fmaf(q.x, q.z, sum); }
      mean = sum * inv_d;
      m2 = 0.f;
      for (int w = 0; w < waves; ++w) { const float4 q = s_red[parity][which][w]; m2 += fmaf(q.z * (q.x - mean), q.x - mean, q.y); }
    }
    rstd = __builtin_amdgcn_rsqf(fmaf(m2, inv_d, norm.eps));
  };

  int parity = 0;
  for (int first = row0; first < a.t; first += step, parity ^= 1) {
    if (!AHEAD) ask(first);
    float v[VPT][E], b[VPT][E];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[i][e] = to_float(rx[i][e]);
        if (has_h) b[i][e] = to_float(rh[i][e]);
      }
    if (AHEAD && first + step < a.t) ask(first + step);
    __builtin_amdgcn_sched_barrier(0);
    const int row = first + group;
    const long at = (long)row * d;
    float mean, rstd;
    if (has_h) {
      if (a.post.kind != WMDEC_NORM_NONE) {
        statistics(a.post, b, 0, parity, mean, rstd);
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
          for (int e = 0; e < E; ++e) b[i][e] = (b[i][e] - mean) * rstd;
      }
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = round_through<TX>(v[i][e] + fmaf(b[i][e], ga[i][e], gb[i][e]));   // (what is stored is what is normalised)
        if (row < a.t) store8<TX, VEC>(x_out + at + col[i], count[i], gap, v[i]);
      }
    }
    if (!has_y) continue;
    if (a.pre.kind != WMDEC_NORM_NONE) {
      statistics(a.pre, v, 1, parity, mean, rstd);
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = (v[i][e] - mean) * rstd;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[i][e] = fmaf(v[i][e], ya[i][e], yb[i][e]);
      if (row < a.t) store8<TA, VEC>(y + at + col[i], count[i], gap, v[i]);
    }
  }
}

template <typename TX, typename TA, int VPT, bool VEC>
int launch_form(const ResidualNormArgs& a, int tpr, int threads, hipStream_t s) {
  Params p{a, tpr, 1};
  const int groups = tpr <= 64 ? threads / tpr : 1;
  const int most = (a.t + groups - 1) / groups;
  // Wavefronts of a compute unit; four where each has a row of more than 3200 bytes to itself (from 401 channels on in fp32).  us, 16 / 4: fp32 20000 rows of 512 36.1 / 33.7,
  // 100000 rows 161.7 / 143.9, 2 x 5400 of 448 22.2 / 20.3; but 100000 of 320 105.8 / 113.6, fp32 beside bf16 20000 of 448 25.4 / 26.4, bf16 20000 of 512 19.6 / 24.7.
  const long row_bytes = (long)a.d * (sizeof(TX) + (a.h ? sizeof(TA) : 0));
  const int waves = tpr == 64 && row_bytes > 3200 ? 4 : VPT == 1 ? 16 : 8;
  const int target = 256 * (waves / (threads / 64)) / a.n;   // all workgroups at once: those of a second round would run alone
  p.segs = max(1, min(most, target));
  hipLaunchKernelGGL((residual_norm_kernel<TX, TA, VPT, VEC>), dim3((unsigned)a.n * p.segs), dim3(threads), 0, s, p);
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

template <typename TX, typename TA, bool VEC>
int launch_width(const ResidualNormArgs& a, hipStream_t s) {
  const int vectors = (a.d + E - 1) / E;
  int tpr = 8;
  while (tpr < 64 && tpr < vectors) tpr *= 2;
  if (vectors <= 64) return launch_form<TX, TA, 1, VEC>(a, tpr, 256, s);
  if (vectors <= kMaxThreads) return launch_form<TX, TA, 1, VEC>(a, (vectors + 63) / 64 * 64, (vectors + 63) / 64 * 64, s);
  tpr = ((vectors + 1) / 2 + 63) / 64 * 64;
  if (tpr <= kMaxThreads) return launch_form<TX, TA, 2, VEC>(a, tpr, tpr, s);
  tpr = ((vectors + 3) / 4 + 63) / 64 * 64;
  static_assert(4 * kMaxThreads * E == kResidualNormMaxD, "four vectors a thread hold the widest row");
  return launch_form<TX, TA, 4, VEC>(a, tpr, tpr, s);
}

template <typename TX, typename TA>
int launch(const ResidualNormArgs& a, hipStream_t s) {
  auto aligned = [](const void* p) { return ((uintptr_t)p & 15) == 0; };
  const bool vec = a.d % E == 0 && a.mod_stride % 4 == 0 && aligned(a.x) && aligned(a.h) && aligned(a.x_out) && aligned(a.y) && aligned(a.gate) && aligned(a.scale) &&
                   aligned(a.shift) && aligned(a.post.weight) && aligned(a.post.bias) && aligned(a.pre.weight) && aligned(a.pre.bias);
  return vec ? launch_width<TX, TA, true>(a, s) : launch_width<TX, TA, false>(a, s);
}

}  // namespace

int launch_residual_norm(const ResidualNormArgs& a, int x_dtype, int act_dtype, hipStream_t s) {
  if (x_dtype == WMDEC_BF16) return launch<bf16_t, bf16_t>(a, s);
  if (x_dtype == WMDEC_F16) return launch<f16_t, f16_t>(a, s);
  if (act_dtype == WMDEC_BF16) return launch<float, bf16_t>(a, s);
  if (act_dtype == WMDEC_F16) return launch<float, f16_t>(a, s);
  return launch<float, float>(a, s);
}

}  // namespace wmdec
