// Attention to states of another length: o = softmax(scale * q k^T over the valid keys) v.  The kernels are in cross_device.hpp; here is what is decided on
// sizes alone, and the f16 kernels.
#include <algorithm>
#include <cmath>

#include "cross_device.hpp"

namespace wmdec {

template int cross_launch<f16_t>(const CrossLaunch&, hipStream_t);

namespace {

// Nothing here looks at the number of samples, so that the bits of a sample do not depend on what it is batched with.
CrossPlan plan_of(int dtype, int tq, int tk, int heads, int group, int d) {
  CrossPlan p;
  p.width = d <= 192 ? (d + 31) / 32 * 32 : 256;
  p.rows = tq * group;
  const int bytes = p.width * (int)dtype_size(dtype);   // of a key
  auto blocks = [&](int bq) { return (long)heads * ((p.rows + bq - 1) / bq); };
  // Few rows: the wavefronts of a workgroup share 32 rows and take a part of the keys each.  us, shared / 128 rows: 4 rows a key head against 32768 keys of 8 heads
  // of 128 channels in bf16 34.2 / 36.9, 16 x 4096 of them 58.9 / 58.8; in f16 30 against 500 of 8 of 64 7.1 / 9.6, 32 against 8192 of 4 of 128 12.5 / 15.6, but against
  // 8 x 4096 of 8 of 64 26.0 / 23.8; 48 rows of that 30.9 / 26.3.
  // In fp32 also more rows whose blocks of 128 would not give work to all: 333x301 of 8 heads of 72 (24 blocks) 16.8 / 21.5, 1000x1000 of 12 of 64 (96) 42 / 45, 2000x500
  // of 8 of 64 (128) 24 / 28; but 2500x2500 of 10 of 64 (200) 178 / 172, 700x700 of 12 of 96 (72) 54 / 36, 2 x 700x700 of 32 of 128 (192) 210 / 191 (and 3000x3000 of 8 of
  // 64 (192), where the blocks of 128 leave a quarter of the compute units idle, 172 / 199).
  p.few = bytes <= 768 && (p.rows <= 32 || (dtype == WMDEC_F32 && bytes <= 512 && blocks(128) <= (bytes <= 256 ? 128 : 64)));
  const int bq = p.few ? 32 : 128;
  p.row_blocks = (p.rows + bq - 1) / bq;
  // Ranges of keys, where blocks are fewer than workgroups run at once: as many as tiles fit into the LDS of a compute unit (and four, or what the registers
  // allow; a mask takes 4 KB more, which 160 channels in 16 bits do not have twice).
  // us without / with ranges: 4 rows a key head against 32768 keys of 8 heads of 128 in bf16 336 / 34, 200 rows against 4096 of 8 of 64 in f16 55.9 / 14.7.
  const int tiles = p.few ? (bytes <= 512 ? 128 : 64) * 2 * bytes : (bytes <= (dtype == WMDEC_F32 ? 512 : 320) ? 64 : 32) * 4 * bytes;
  const int slots = 256 * std::min(160 * 1024 / tiles, !p.few && p.width <= 64 ? 4 : 2);
  // (us with 128, 256 or 512 keys: bf16 1 token of 32 / 8 heads of 128 against 4 x 1024 10.6, 10.5, 11.8, against 16 x 1024 21.5, 20.4, 21.0.  fp32 with 64, 128 or 256: 5 rows
  // against 699 keys of 10 heads of 256 34, 50, 98, four samples 59, 54, 102; of 10 of 160, four samples, 25, 28, 44.  Shared rows of up to 512 bytes: 500x500 of 12 of 64 19.3,
  // 19.5, 15.1, 3 x 333x301 of 8 of 72 33.7, 33.7, 32.8; but up to 32 rows 30x2000 of 4 of 128 15.4, 19.6, 24.3, 1x1024 of 8 of 128 13.3, 13.1, 18.0.)
  const long range = dtype != WMDEC_F32 || (p.few && bytes <= 512) ? 256 : p.few ? 128 : 64;   // fewest keys of a range: two tiles, or what is worth a launch
  p.splits = (int)std::max(1L, std::min({slots / blocks(bq), tk / range, (long)kCrossMaxSplits}));
  if (!p.few && p.splits > 1) {
    // Partial outputs of 128 rows weigh: s ranges take a / s for their keys, b * s for writing and reading what they leave, and the second launch.  (b counts half as
    // much again as one sample alone has, for batches: what batches gain, single samples lose.)  us, ranges as slots allow / so: f16 1000x1000 of 16 / 4 heads of 128 30.5 / 27.4,
    // four samples 87 / 47, 2000x2000 of 8 of 128 37 / 48, three samples 95 / 71, 700x3000 of 4 of 96 18.5 / 18.4, three 35 / 28, 150x8000 of 4 of 64 12.7 / 14.5, four 25 / 24; fp32
    // 257x893 of 8 / 2 of 160 30 / 33, three 69 / 62.
    const double a = (dtype == WMDEC_F32 ? 1e-3 : 1.8e-4) * tk * p.width, b = 1.2e-6 * 512 * p.width * blocks(bq);   // us
    p.splits = std::min(p.splits, (int)std::sqrt(a / b));
    if (p.splits < 2 || a - a / p.splits < 5 + b * p.splits) p.splits = 1;
  }
  return p;
}

size_t part_rows(const CrossPlan& p, int n, int heads) { return p.splits == 1 ? 0 : (size_t)n * heads * p.row_blocks * p.splits * (p.few ? 32 : 128); }

}  // namespace

bool cross_attention_fits(int dtype, int n, int tq, int tk, int heads, int group, int d) {
  const CrossPlan p = plan_of(dtype, tq, tk, heads, group, d);
  const double blocks = (double)n * heads * p.row_blocks;
  return blocks * p.splits < 0x1p24 && (p.splits == 1 || blocks * (p.few ? 32 : 128) < 0x1p26);   // workgroups of 256 threads; rows that are joined, numbered in 32 bits
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
