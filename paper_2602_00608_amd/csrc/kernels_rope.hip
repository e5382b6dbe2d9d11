// Rotary positions: pairs of channels of a head turn by position * frequency.
//
// Bound by HBM: q and k are read and written once.  An angle belongs to a token and a pair, not to a head: it is worked out once for all heads (in 64 bits,
// as positions times frequencies pass what fp32 resolves), and what is left an element is a multiplication and a multiply-add.
// us on inputs from memory, with the rate: 2x5400 tokens of 30 + 30 heads of 64 in bf16 38.1 (4.36 TB/s; a copy of as many bytes 32.6), 16385 tokens of
// 32 + 8 heads of 128 in f16 70.1 (4.79).  Steps: a thread a pair 139 and 350; angles through LDS and vectors of eight channels, four of them at a time 48.9 and
// 77.4; workgroups side by side in memory, where a token's q and k are from LDS, one unit on its way behind the other 38.1 and 72.6.
#include <algorithm>

#include "mfma.hpp"

namespace wmdec {
namespace {

constexpr int NT = 256;
constexpr int kMaxTokens = 256, kMaxAngles = 2048;   // of a workgroup
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
// are below 2^-28 of the sine and 2^-32 of the cosine).  The quarter turns are taken off by fused steps with pi / 2 in two parts
// (the reduction of Cody and Waite), in which their product is not rounded.  (The fraction of theta / (pi / 2): up to 5 steps of 2^-24 off at 2^31.)
constexpr double kQuarterTurn = kTwoPi / 4, kQuarterTurnRest = 6.123233995736766e-17;   // pi / 2 and what is left of it
__device__ __forceinline__ float2 sin_cos(double theta) {
  const double whole = rint(theta * (4.0 / kTwoPi));
  const float r = (float)fma(-whole, kQuarterTurnRest, fma(-whole, kQuarterTurn, theta)), z = r * r;
  const float sn = fmaf(r * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), r);
  const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  const int q = (int)(long)whole & 3;
  const float s = q & 1 ? cs : sn, c = q & 1 ? sn : cs;
  return make_float2(q & 2 ? -s : s, (q + 1) & 2 ? -c : c);
}

// W channels next to each other, in loads and stores of up to 16 bytes
template <typename T, int W> struct alignas(sizeof(T) * W < 16 ? sizeof(T) * W : 16) Vec { T v[W]; };
template <typename T, int W> __device__ __forceinline__ Vec<T, W> load(const T* p) { return *reinterpret_cast<const Vec<T, W>*>(p); }
template <typename T, int W> __device__ __forceinline__ void store(T* p, const Vec<T, W>& r) { *reinterpret_cast<Vec<T, W>*>(p) = r; }

// Work of a workgroup: `tokens` tokens, all heads.  Its angles are worked out once, a thread each, into LDS; then the threads walk over
// (token, head, unit).  The tokens of a workgroup are as far apart as there are workgroups, so that what is under way at a time lies together in memory.  A unit is two vectors of W channels (or one channel and its partner): of the rotated part W / 2 or W pairs, else copied.
struct Params {
  RopeArgs a;
  int tokens;                       // of a workgroup
  int pairs, rotated, units;        // pairs of a head, units of them, units of a head
  int du, dh, dt;                   // NT = (dt * heads + dh) * units + du: a thread's step
  int groups, split;                // ranges of tokens, workgroups that share one, each with every split-th step
  long total;                       // tokens of all samples
};

template <typename T, int W, bool INTERLEAVED>
__global__ __launch_bounds__(NT) void rope_kernel(Params p) {
  extern __shared__ __align__(16) float2 s_turn[];   // [tokens][pairs] cosine, sine
  struct Places { const T* in; T* out; };
  __shared__ Places s_place[kMaxTokens][2];          // where a token's q and k are
  const RopeArgs& a = p.a;
  const int heads = a.q.heads + a.k.heads, tid = threadIdx.x;
  const int first = blockIdx.x / p.split, part = blockIdx.x % p.split;
  const int count = (int)((p.total - first + p.groups - 1) / p.groups);   // tokens first, first + groups, ...
  auto token_of = [&](int i, int& n, int& t) {
    const int token = first + i * p.groups;          // (below 2^31: checked on the host)
    n = token / a.t; t = token - n * a.t;
  };
  for (int i = tid; i < 2 * count; i += NT) {
    const RopeTensor& x = i & 1 ? a.k : a.q;
    int n, t;
    token_of(i / 2, n, t);
    s_place[i / 2][i & 1] = Places{(const T*)x.in + n * x.si.sample + t * x.si.token, (T*)x.out + n * x.so.sample + t * x.so.token};
  }
  __syncthreads();

  struct Unit { Vec<T, W> v[2]; T* out; const float2* turn; int c0, c1; bool live; };   // turn: null for channels that are copied
  int wu, wh, wt;                                    // the next unit, its head, its token
  {
    const int i = part * NT + tid, hu = heads * p.units;
    wt = i / hu; wh = (i - wt * hu) / p.units; wu = i - wt * hu - wh * p.units;
  }
  // where the two vectors of a unit are; both the same channel where there is no second one
  auto channels = [&](int u, int& c0, int& c1) {
    if (u >= p.rotated) { c0 = a.rot + (u - p.rotated) * 2 * W; c1 = c0 + W < a.d ? c0 + W : c0; return; }
    if (INTERLEAVED) { c0 = u * 2 * W; c1 = c0 + W; if (c1 >= a.rot) c1 = c0; return; }
    int j = u * W, at = 0, axis = 0;
    while (j >= a.layout.axis_dim[axis] / 2) { at += a.layout.axis_dim[axis]; j -= a.layout.axis_dim[axis++] / 2; }
    c0 = at + j; c1 = c0 + a.layout.axis_dim[axis] / 2;
  };
  auto ask = [&](Unit& x) {
    x.live = wt < count;
    if (x.live) {
      const bool second = wh >= a.q.heads;
      const Places at = s_place[wt][second];
      const int h = second ? wh - a.q.heads : wh;
      channels(wu, x.c0, x.c1);
      const T* in = at.in + h * (second ? a.k.si.head : a.q.si.head);
      x.out = at.out + h * (second ? a.k.so.head : a.q.so.head);
      x.turn = wu < p.rotated ? s_turn + wt * p.pairs + wu * W : nullptr;
      x.v[0] = load<T, W>(in + x.c0);
      x.v[1] = load<T, W>(in + x.c1);
    }
    wu += p.du; wh += p.dh; wt += p.dt;
    if (wu >= p.units) { wu -= p.units; ++wh; }
    if (wh >= heads) { wh -= heads; ++wt; }
  };
  auto finish = [&](Unit& x) {
    Vec<T, W> &o0 = x.v[0], &o1 = x.v[1];
    if (x.turn) {
      if constexpr (INTERLEAVED && W > 1) {        // (the second vector has its pairs behind the first one's; where there is none they are not used)
#pragma unroll
        for (int e = 0; e < 2 * W; e += 2) {
          Vec<T, W>& o = e < W ? o0 : o1;
          const float2 c = x.turn[e / 2 < W / 2 || x.c1 != x.c0 ? e / 2 : 0];
          const float v = to_float(o.v[e % W]), w = to_float(o.v[e % W + 1]);
          o.v[e % W] = from_float<T>(v * c.x - w * c.y);
          o.v[e % W + 1] = from_float<T>(v * c.y + w * c.x);
        }
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float2 c = x.turn[e];
          const float v = to_float(o0.v[e]), w = to_float(o1.v[e]);
          o0.v[e] = from_float<T>(v * c.x - w * c.y);
          o1.v[e] = from_float<T>(v * c.y + w * c.x);
        }
      }
    }
    store<T, W>(x.out + x.c0, o0);
    if (x.c1 != x.c0) store<T, W>(x.out + x.c1, o1);
  };
  Unit s0, s1;                      // one travels while the other is worked on
  ask(s0);
  for (int i = tid; i < count * p.pairs; i += NT) {
    const int t = i / p.pairs, u = i - t * p.pairs;
    int axis = 0, j = u, n, row;
    while (j >= a.layout.axis_dim[axis] / 2) j -= a.layout.axis_dim[axis++] / 2;
    token_of(t, n, row);
    float2 sc = sin_cos((double)a.positions[n * a.positions_stride + (long)row * a.layout.axes + axis] * a.freq[u]);
    if (a.layout.inverse) sc.x = -sc.x;
    s_turn[i] = make_float2(sc.y * a.layout.magnitude, sc.x * a.layout.magnitude);
  }
  __syncthreads();
  while (s0.live) {                 // (units go upwards: where one is past the end, all that follow are)
    ask(s1);
    finish(s0);
    if (!s1.live) break;
    ask(s0);
    finish(s1);
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
  // 4096 workgroups where there are as many tokens (1024, one round of them: 16385 tokens of 40 heads of 128 72.6 us against 70.1, 2x5400 of 60 of 64 the same), but
  // 1024 while four steps a thread are not reached; few tokens with much work are shared.
  const long tokens = std::max((p.total + 4095) / 4096, std::min((p.total + 1023) / 1024, 4L * NT / per_token));
  p.tokens = (int)std::min(tokens, std::max(1L, std::min((long)kMaxAngles / p.pairs, (long)kMaxTokens)));
  const long groups = (p.total + p.tokens - 1) / p.tokens, work = (p.tokens * per_token + NT - 1) / NT;
  p.groups = (int)groups;
  p.split = (int)std::max(1L, std::min(work, 1024 / groups));
  const long step = (long)NT * p.split;
  p.du = (int)(step % p.units); p.dh = (int)(step / p.units % (a.q.heads + a.k.heads)); p.dt = (int)(step / per_token);
  WMDEC_REQUIRE(groups * p.split < (1L << 24), WMDEC_ERR_UNSUPPORTED, "rope: too many tokens");
  hipLaunchKernelGGL((rope_kernel<T, W, INTERLEAVED>), dim3((unsigned)(groups * p.split)), dim3(NT), p.tokens * p.pairs * sizeof(float2), s, p);
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

template <typename T>
int launch(const RopeArgs& a, hipStream_t s) {
  // Vectors of eight channels, or of four: every head starts on one, the rotated part and its halves are whole vectors.
  auto fits = [&](int w) {
    const size_t to = std::min<size_t>(16, w * sizeof(T));
    auto part = [&](const void* p, const wmdec_strides& st) {
      return (uintptr_t)p % to == 0 && st.sample * sizeof(T) % to == 0 && st.token * sizeof(T) % to == 0 && st.head * sizeof(T) % to == 0;
    };
    auto tensor = [&](const RopeTensor& t) { return t.heads == 0 || (part(t.in, t.si) && part(t.out, t.so)); };
    bool ok = a.d % w == 0 && a.rot % w == 0 && tensor(a.q) && tensor(a.k);
    for (int i = 0; i < a.layout.axes; ++i) ok = ok && (a.layout.interleaved || a.layout.axis_dim[i] % (2 * w) == 0);
    return ok;
  };
  if (a.layout.interleaved) return fits(8) ? launch_form<T, 8, true>(a, s) : fits(4) ? launch_form<T, 4, true>(a, s) : launch_form<T, 1, true>(a, s);
  return fits(8) ? launch_form<T, 8, false>(a, s) : fits(4) ? launch_form<T, 4, false>(a, s) : launch_form<T, 1, false>(a, s);
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
