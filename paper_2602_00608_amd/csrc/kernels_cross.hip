// Attention to states of another length: o = softmax(scale * q k^T over the valid keys) v.  The kernels are in cross_device.hpp; here is what is decided on
// sizes alone, and the f16 kernels.
#include <algorithm>

#include "cross_device.hpp"

namespace wmdec {

template int cross_launch<f16_t>(const CrossLaunch&, hipStream_t);

namespace {

// Nothing here looks at the number of samples, so that the bits of a sample do not depend on what it is batched with.
CrossPlan plan_of(int dtype, int tq, int tk, int heads, int group, int d) {
  CrossPlan p;
  p.width = d <= 128 ? (d + 31) / 32 * 32 : d <= 192 ? 192 : 256;
  p.rows = tq * group;
  const int bytes = p.width * (int)dtype_size(dtype);   // of a key
  auto blocks = [&](int bq) { return (long)heads * ((p.rows + bq - 1) / bq); };
  // Few rows: the wavefronts of a workgroup share 32 rows and take a part of the keys each; so do those of more rows that would not give work to all.
  p.few = bytes <= 768 && (p.rows <= 32 || (dtype == WMDEC_F32 && bytes <= 512 && blocks(128) <= 64));
  const int bq = p.few ? 32 : 128;
  p.row_blocks = (p.rows + bq - 1) / bq;
  // Ranges of keys, where blocks are fewer than workgroups run at once: as many as tiles fit into the LDS of a compute unit (and four, or what the registers allow).
  const int tiles = p.few ? (bytes <= 512 ? 128 : 64) * 2 * bytes : (bytes <= 512 ? 64 : 32) * 4 * bytes;
  const int slots = 256 * std::min(160 * 1024 / (tiles + 4096), !p.few && p.width <= 64 ? 4 : 2);
  const long range = dtype != WMDEC_F32 || (p.few && bytes <= 512) ? 256 : p.few ? 128 : 64;   // fewest keys of a range: two tiles, or what is worth a launch
  p.splits = (int)std::max(1L, std::min({slots / blocks(bq), tk / range, (long)kCrossMaxSplits}));
  return p;
}

size_t part_rows(const CrossPlan& p, int n, int heads) { return p.splits == 1 ? 0 : (size_t)n * heads * p.row_blocks * p.splits * (p.few ? 32 : 128); }

}  // namespace

bool cross_attention_fits(int dtype, int n, int tq, int tk, int heads, int group, int d) {
  const CrossPlan p = plan_of(dtype, tq, tk, heads, group, d);
  const double blocks = (double)n * heads * p.row_blocks;
  return blocks * p.splits < 0x1p24 && (p.splits == 1 || blocks * (p.few ? 32 : 128) < 0x1p26);   // workgroups of 256 threads; rows that are joined, four of them
}

size_t cross_attention_scratch_bytes(int dtype, int n, int tq, int tk, int heads, int group, int d) {
  const CrossPlan p = plan_of(dtype, tq, tk, heads, group, d);
  return part_rows(p, n, heads) * (p.width + 2) * sizeof(float);
}

int launch_cross_attention(const CrossArgs& a, int dtype, hipStream_t s) {
  CrossLaunch l;
  l.a = a;
  l.plan = plan_of(dtype, a.tq, a.tk, a.heads, a.group, a.d);
  l.part = (float*)a.scratch;
  l.ml = (float2*)(l.part + part_rows(l.plan, a.n, a.heads) * l.plan.width);
  if (dtype == WMDEC_F32) return cross_launch<float>(l, s);
  return dtype == WMDEC_BF16 ? cross_launch<bf16_t>(l, s) : cross_launch<f16_t>(l, s);
}

}  // namespace wmdec
