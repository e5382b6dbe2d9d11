// Rotary positions: pairs of channels of a head turn by position * frequency.
//
// Bound by HBM: q and k are read and written once.  An angle belongs to a token and a pair, not to a head: it is worked out once for all heads (in 64 bits,
// as positions times frequencies pass what fp32 resolves), and what is left an element is a multiplication and a multiply-add.
#include <algorithm>

#include "mfma.hpp"

namespace wmdec {
namespace {

constexpr int NT = 256;
constexpr double kTwoPi = 6.283185307179586476925286766559;

struct FreqParams { double* freq; int axes; int dim[3]; wmdec_rope_scaling sc; };

__global__ void rope_frequencies_kernel(FreqParams p) {
  int j = blockIdx.x * blockDim.x + threadIdx.x, axis = 0;
  const int at = j;
  while (axis < p.axes && j >= p.dim[axis] / 2) j -= p.dim[axis++] / 2;
  if (axis == p.axes) return;
  const double d = p.dim[axis];
  const double base = p.sc.kind == WMDEC_ROPE_BASE ? p.sc.base * pow(p.sc.factor, d / (d - 2)) : p.sc.base;
  double f = pow(base, -2.0 * j / d);
  if (p.sc.kind == WMDEC_ROPE_LINEAR) f /= p.sc.factor;
  if (p.sc.kind == WMDEC_ROPE_RAMP) {
    const double w = fmin(fmax((p.sc.trained_length * f / kTwoPi - p.sc.low_turns) / (p.sc.high_turns - p.sc.low_turns), 0.0), 1.0);
    f *= w + (1.0 - w) / p.sc.factor;
  }
  p.freq[at] = f;
}

// sin and cos of the angle theta: quarter turns and the rest within an eighth of a turn, in 64 bits, then Taylor's polynomials in fp32 (the terms left out
// are below 2^-29 of the sine and 2^-33).
__device__ __forceinline__ float2 sin_cos(double theta) {
  const double quarters = theta * (4.0 / kTwoPi), whole = rint(quarters);
  const float r = (float)((quarters - whole) * (kTwoPi / 4.0)), z = r * r;
  const float sn = fmaf(r * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), r);
  const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  const int q = (int)(long)whole & 3;
  const float s = q & 1 ? cs : sn, c = q & 1 ? sn : cs;
  return make_float2(q & 2 ? -s : s, (q + 1) & 2 ? -c : c);
}

template <typename T, int W> struct Vec { T v[W]; };
template <typename T, int W> __device__ __forceinline__ Vec<T, W> load(const T* p) {
  Vec<T, W> r;
  if constexpr (W == 1) r.v[0] = *p;
  else {
    u32x4 q[sizeof(T) * W / 16];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * W / 16); ++i) q[i] = reinterpret_cast<const u32x4*>(p)[i];
    __builtin_memcpy(&r, &q, sizeof(r));
  }
  return r;
}
template <typename T, int W> __device__ __forceinline__ void store(T* p, const Vec<T, W>& r) {
  if constexpr (W == 1) *p = r.v[0];
  else {
    u32x4 q[sizeof(T) * W / 16];
    __builtin_memcpy(&q, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * W / 16); ++i) reinterpret_cast<u32x4*>(p)[i] = q[i];
  }
}

// Work of a workgroup: `tokens` consecutive tokens, all heads.  Its angles are worked out once, a thread each, into LDS; then the threads walk over
// (token, head, unit).  A unit is two vectors of W channels (or one channel and its partner): of the rotated part W / 2 or W pairs, else copied.
struct Params {
  RopeArgs a;
  int tokens;                       // of a workgroup
  int pairs, rotated, units;        // pairs of a head, units of them, units of a head
  int du, dh, dt;                   // NT = (dt * heads + dh) * units + du: a thread's step
  int split;                        // workgroups that share a range of tokens, each with every split-th step
  long total;                       // tokens of all samples
};

template <typename T, int W, bool INTERLEAVED>
__global__ __launch_bounds__(NT) void rope_kernel(Params p) {
  extern __shared__ __align__(16) float2 s_turn[];   // [tokens][pairs] cosine, sine
  const RopeArgs& a = p.a;
  const int heads = a.q.heads + a.k.heads, tid = threadIdx.x;
  const long first = (long)(blockIdx.x / p.split) * p.tokens;
  const int count = (int)min((long)p.tokens, p.total - first), part = blockIdx.x % p.split;
  const int n0 = (int)(first / a.t), t0 = (int)(first - (long)n0 * a.t);
  auto sample_of = [&](int i, int& n, int& t) {      // of the i-th token of the workgroup
    n = n0; t = t0 + i;
    if (t >= a.t) { n += t / a.t; t %= a.t; }
  };

  struct Place { int u, h, t; };
  auto advance = [&](Place& w, int du, int dh, int dt) {
    w.u += du; w.h += dh; w.t += dt;
    if (w.u >= p.units) { w.u -= p.units; ++w.h; }
    if (w.h >= heads) { w.h -= heads; ++w.t; }
  };
  // where the two vectors of a unit are; both the same channel where there is no second one
  auto channels = [&](int u, int& c0, int& c1) {
    if (u >= p.rotated) { c0 = a.rot + (u - p.rotated) * 2 * W; c1 = c0 + W < a.d ? c0 + W : c0; return; }
    if (INTERLEAVED) { c0 = u * 2 * W; c1 = c0 + W; if (c1 >= a.rot) c1 = c0; return; }
    int j = u * W, at = 0, axis = 0;
    while (j >= a.layout.axis_dim[axis] / 2) { at += a.layout.axis_dim[axis]; j -= a.layout.axis_dim[axis++] / 2; }
    c0 = at + j; c1 = c0 + a.layout.axis_dim[axis] / 2;
  };
  auto address = [&](const Place& w, const T*& in, T*& out) {
    int n, t;
    sample_of(w.t, n, t);
    const bool second = w.h >= a.q.heads;
    const int h = second ? w.h - a.q.heads : w.h;
    const wmdec_strides &si = second ? a.k.si : a.q.si, &so = second ? a.k.so : a.q.so;
    in = (const T*)(second ? a.k.in : a.q.in) + n * si.sample + t * si.token + h * si.head;
    out = (T*)(second ? a.k.out : a.q.out) + n * so.sample + t * so.token + h * so.head;
  };
  constexpr int U = 4;              // steps in flight
  Place w{0, 0, 0};
  {
    const int i = part * NT + tid, hu = heads * p.units;
    w.t = i / hu; w.h = (i - w.t * hu) / p.units; w.u = i - w.t * hu - w.h * p.units;
  }
  Vec<T, W> v[U][2];
  Place at[U];
  auto ask = [&]() {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      at[i] = w;
      if (w.t < count) {
        const T* in; T* out; int c0, c1;
        address(w, in, out); channels(w.u, c0, c1);
        v[i][0] = load<T, W>(in + c0);
        v[i][1] = load<T, W>(in + c1);
      }
      advance(w, p.du, p.dh, p.dt);
    }
  };
  ask();
  for (int i = tid; i < count * p.pairs; i += NT) {
    const int t = i / p.pairs, u = i - t * p.pairs;
    int axis = 0, j = u;
    while (j >= a.layout.axis_dim[axis] / 2) j -= a.layout.axis_dim[axis++] / 2;
    int n, row;
    sample_of(t, n, row);
    const long pos = n * a.positions_stride + (long)row * a.layout.axes + axis;
    float2 sc = sin_cos((double)a.positions[pos] * a.freq[u]);
    if (a.layout.inverse) sc.x = -sc.x;
    s_turn[i] = make_float2(sc.y * a.layout.magnitude, sc.x * a.layout.magnitude);
  }
  __syncthreads();
  while (true) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (at[i].t >= count) continue;
      const T* in; T* out; int c0, c1;
      address(at[i], in, out); channels(at[i].u, c0, c1);
      Vec<T, W> o0 = v[i][0], o1 = v[i][1];
      if (at[i].u < p.rotated) {
        const float2* turn = s_turn + at[i].t * p.pairs;
        if constexpr (INTERLEAVED && W > 1) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            Vec<T, W>& o = half ? o1 : o0;
#pragma unroll
            for (int e = 0; e < W; e += 2) {
              const float2 c = turn[(half ? c1 : c0) / 2 + e / 2];
              const float x = to_float(o.v[e]), y = to_float(o.v[e + 1]);
              o.v[e] = from_float<T>(x * c.x - y * c.y);
              o.v[e + 1] = from_float<T>(x * c.y + y * c.x);
            }
          }
        } else {
#pragma unroll
          for (int e = 0; e < W; ++e) {
            const float2 c = turn[at[i].u * W + e];
            const float x = to_float(o0.v[e]), y = to_float(o1.v[e]);
            o0.v[e] = from_float<T>(x * c.x - y * c.y);
            o1.v[e] = from_float<T>(x * c.y + y * c.x);
          }
        }
      }
      store<T, W>(out + c0, o0);
      if (c1 != c0) store<T, W>(out + c1, o1);
    }
    if (w.t >= count) break;        // (steps go upwards)
    ask();
  }
}

template <typename T, int W, bool INTERLEAVED>
int launch_form(const RopeArgs& a, hipStream_t s) {
  Params p;
  p.a = a;
  p.pairs = a.rot / 2;
  p.rotated = W == 1 ? p.pairs : (a.rot + 2 * W - 1) / (2 * W);
  p.units = p.rotated + (a.d - a.rot + 2 * W - 1) / (2 * W);
  p.total = (long)a.n * a.t;
  const long per_token = (long)(a.q.heads + a.k.heads) * p.units;
  // Tokens of a workgroup: an angle for every thread, or 16 steps of work where that is less, and workgroups for all compute units; few tokens with much work
  // are shared.
  const long fill = std::max(1L, (p.total + 1023) / 1024), angles = std::max(1, NT / p.pairs), steps = std::max(1L, 16L * NT / per_token);
  p.tokens = (int)std::min(fill, std::max(1L, std::min(angles, steps)));
  const long groups = (p.total + p.tokens - 1) / p.tokens, work = (p.tokens * per_token + NT - 1) / NT;
  p.split = (int)std::max(1L, std::min(work, 1024 / groups));
  const long step = (long)NT * p.split;
  p.du = (int)(step % p.units); p.dh = (int)(step / p.units % (a.q.heads + a.k.heads)); p.dt = (int)(step / per_token);
  WMDEC_REQUIRE(groups * p.split < (1L << 31), WMDEC_ERR_UNSUPPORTED, "rope: too many tokens");
  hipLaunchKernelGGL((rope_kernel<T, W, INTERLEAVED>), dim3((unsigned)(groups * p.split)), dim3(NT), p.tokens * p.pairs * sizeof(float2), s, p);
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

template <typename T>
int launch(const RopeArgs& a, hipStream_t s) {
  // Vectors of eight channels: every head starts on 16 bytes, the rotated part and its halves are whole vectors.
  constexpr int W = 8;
  auto fits = [&](const RopeTensor& t) {
    auto part = [](const void* p, const wmdec_strides& st) {
      return ((uintptr_t)p & 15) == 0 && st.sample * sizeof(T) % 16 == 0 && st.token * sizeof(T) % 16 == 0 && st.head * sizeof(T) % 16 == 0;
    };
    return t.heads == 0 || (part(t.in, t.si) && part(t.out, t.so));
  };
  bool vec = a.d % W == 0 && a.rot % W == 0 && fits(a.q) && fits(a.k);
  for (int i = 0; i < a.layout.axes; ++i) vec = vec && (a.layout.interleaved || a.layout.axis_dim[i] % (2 * W) == 0);
  if (a.layout.interleaved) return vec ? launch_form<T, W, true>(a, s) : launch_form<T, 1, true>(a, s);
  return vec ? launch_form<T, W, false>(a, s) : launch_form<T, 1, false>(a, s);
}

}  // namespace

int launch_rope_frequencies(double* freq, int axes, const int* axis_dim, const wmdec_rope_scaling& sc, hipStream_t s) {
  FreqParams p{freq, axes, {0, 0, 0}, sc};
  int pairs = 0;
  for (int i = 0; i < axes; ++i) { p.dim[i] = axis_dim[i]; pairs += axis_dim[i] / 2; }
  hipLaunchKernelGGL(rope_frequencies_kernel, dim3((unsigned)((pairs + 63) / 64)), dim3(64), 0, s, p);
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

int launch_rope(const RopeArgs& a, int dtype, hipStream_t s) {
  switch (dtype) {
    case WMDEC_F32: return launch<float>(a, s);
    case WMDEC_BF16: return launch<bf16_t>(a, s);
    default: return launch<f16_t>(a, s);
  }
}

}  // namespace wmdec
