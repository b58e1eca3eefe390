// The dispatch rule of the tile and pair GEMMs (linear.cu, linear_act.cu), by sizes.
#pragma once

#include "common.cuh"

namespace grace {

constexpr int kGemmBM = 128;
constexpr int kGemmBK = 64;                                 // bf16 elements of a k-block; a k-block is 128 bytes of a row

// Which kernel runs a problem: the estimate below, in microseconds, of every form that can, and the least of them.
// linear_kernel: a wave of CTAs takes a fixed part (launch, first loads, epilogue: it grows with the columns a CTA
// finishes) and a part per k-block of its range of K; CTAs beyond a wave wait for it.  The constants are fits to
// chains of dependent launches on a B200 (x [M][K] times [N][K], M 1 .. 4096, N 128 .. 8192, K 128 .. 8192; most
// estimates are within 10 %).  What it gives against the rule before (pair kernel from M = 1024 on, else 32- or 128-wide
// tiles without a split), LayerNorm included: 512 x 1536 x 512: 10.3 -> 5.8 us, 512 x 2048 x 512: 10.5 -> 6.1,
// 512 x 512 x 2048: 10.3 -> 5.8, 16 x 512 x 2048: 9.9 -> 4.3, 1024 x 512 x 2048: 13.1 -> 7.1, 1024 x 512 x 512:
// 7.6 -> 5.0, 2048 x 512 x 2048: 13.1 -> 9.1.
// Row statistics formed from the operand tiles are free for eight k-blocks, which are in flight at once; beyond, the ring
// waits for the warps that form them (as if free: 10000 x 512 x 2048 45 us where the pair kernel behind the statistics
// kernel takes 28, 16384 x 512 x 2048 45 / 33, 4096 x 1024 x 2048 23 / 19).  Two CTAs per SM take an SM's time from each other: a last
// wave of one per SM is shorter (1000 x 6144 x 2048: 36.3 us in the form estimated before, 28.7 so); seen with long K only.
// Rows beyond the problem's last cost no exchange and no stores: both parts grow from few rows to a full tile of 128.
struct LinearForm {
  int bn, split, per_sm;                   // bn = 0: the CTA-pair kernel
  float fixed, per_kb;                     // with few rows
  float fixed_rows, per_kb_rows;           // added with 128 rows or more
};
constexpr LinearForm kLinearForms[] = {
    {32, 1, 1, 1.9f, 0.243f, 0.1f, 0.f}, {32, 2, 1, 2.35f, 0.235f, 0.4f, 0.02f},     // whole K range in flight
    {64, 1, 1, 2.35f, 0.243f, 0.4f, 0.f}, {64, 2, 1, 2.55f, 0.236f, 0.7f, 0.014f}, {64, 4, 1, 2.4f, 0.233f, 0.9f, 0.08f},
    {128, 1, 1, 3.25f, 0.245f, 0.85f, 0.f}, {128, 2, 1, 3.15f, 0.246f, 1.2f, 0.f}, {128, 4, 1, 2.95f, 0.237f, 1.4f, 0.01f},
    {64, 1, 2, 3.85f, 0.318f, 0.f, 0.f}, {128, 1, 2, 5.0f, 0.46f, 0.f, 0.f}};        // two CTAs per SM, three or four stages
enum LinearStats { kStatsNone, kStatsFormed, kStatsFormedNarrow };
// stats: whether the call's row statistics are still to be formed, and if so whether the pair kernel would form them itself
// (narrow) or need the statistics kernel in front.  whole_k: no split of K, so that the sums are those of the pair kernel bit
// for bit (fp32 products: grace_linear_f32_lse promises those of grace_linear).
inline LinearForm linear_form(int M, int N, int K, bool pair_possible, LinearStats stats, bool whole_k, int products = 1) {
  const int64_t tiles_m = (M + kGemmBM - 1) / kGemmBM;
  const int kb = K / kGemmBK;
  LinearForm best = {};
  const float rows = M < kGemmBM ? (float)M / (float)kGemmBM : 1.f;
  float least = 3.4e38f;
  if (pair_possible) {
    const int64_t waves = ((int64_t)((M + 255) / 256) * ((N + 255) / 256) * products + kSmsInTwos / 2 - 1) / (kSmsInTwos / 2);
    least = 2.7f + (float)waves * (1.0f + 0.33f * (float)kb) + (stats == kStatsFormed ? 3.2f + 3.6e-7f * (float)M * (float)K : 0.f);
    if (tiles_m > 65535) return best;                        // more row tiles than gridDim.y takes: the persistent kernel
  }
  for (const LinearForm& f : kLinearForms) {
    if (f.split > kb || (whole_k && f.split > 1)) continue;
    const int64_t ctas = tiles_m * ((N + f.bn - 1) / f.bn) * f.split * products;
    const int wave = f.split == 1 ? kSms * f.per_sm : (f.split == 2 ? kSmsInTwos : kSmsInFours);
    const int64_t waves = (ctas + wave - 1) / wave;
    const int long_kb = (kb + f.split - 1) / f.split;
    float one = f.fixed + rows * f.fixed_rows + (f.per_kb + rows * f.per_kb_rows) * (float)long_kb;
    if (stats != kStatsNone && long_kb > 8) one += (f.per_sm == 1 ? 0.07f : 0.15f) * (float)(long_kb - 8);
    float t = (float)waves * one;
    if (f.per_sm == 2 && waves > 1 && long_kb > 8 && ctas - (waves - 1) * wave <= kSms) t -= 0.35f * one;
    if (t < least) { least = t; best = f; }
  }
  return best;
}
// The pair kernel takes whole 256 x 256 tiles and adds into the residual stream by TMA only in place.
inline bool linear_pair_possible(int M, int N, bool residual_elsewhere) { return M >= 1024 && N >= 256 && !residual_elsewhere; }

}  // namespace grace
