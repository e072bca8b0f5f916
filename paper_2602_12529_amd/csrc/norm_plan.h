// How the affine norm and the norms' gradients take a row: plain C++, so that the rule can be checked without a GPU.
#pragma once

#include <cstdint>
#include <initializer_list>

namespace ff {

// Threads a row and chunks of 8 columns a thread for a width.  ni = 0: the row is too wide for this.
//   - Up to 1536 columns a wave takes a row: no barriers (32760 x 1536 backward: 52 us, 192 threads 64).
//   - Wider rows have several waves.  A chunk takes 60 registers in the backward pass, so three of them halve the waves
//     in flight: one chunk up to 2048 columns (32768 x 2048: 256 threads 103 us, 192 threads of two 111) and of 3073 to
//     4096 in the backward pass (16384 x 4096: 512 threads 102, 256 threads of two 109), else two (8192 x 5000: 384
//     threads 61, 512 threads 65), past 8192 columns three.  The forward pass takes three of 2049 to 3072 columns
//     (32768 x 3072: 128 threads 61 us, 192 threads 63).
//   - Few rows leave compute units idle, so as many threads as can work on each (1665 x 2560, five samples: 384 threads
//     17.8 us, 192 threads 18.6; 3000 x 1536: 192 threads 21.7, a wave 13.7).
// (Both sides of each with plain loads of x.)
struct RowPlanH { int tpr, ni; };
inline RowPlanH row_plan_h(int64_t rows, int64_t H, bool forward = false) {
  for (int tpr : {8, 16, 32, 64})
    if (H <= 8 * tpr) return {tpr, 1};
  const bool few = rows <= 2048;
  if (H <= 1536 && !few) return {64, static_cast<int>((H + 511) / 512)};
  if (forward && !few && H > 2048 && H <= 3072) return {128, 3};
  if (!few && H <= 2048) return {256, 1};
  if (!forward && !few && H > 3072 && H <= 4096) return {512, 1};
  for (int tpr : {128, 192, 256, 384, 512}) {
    const int ni = static_cast<int>((H + 8 * tpr - 1) / (8 * tpr));
    if (ni == 1 || (ni == 2 && (!few || H > 4096))) return {tpr, ni};
  }
  return {512, H <= 12288 ? 3 : 0};
}

// The plans that row_plan_h gives for each pass, which are the kernels that are built (ni = 0 has kernels of its own).
#define FF_NORM_BOTH(CALL) \
  CALL(8, 1) CALL(16, 1) CALL(32, 1) CALL(64, 1) CALL(64, 2) CALL(64, 3) CALL(128, 1) CALL(192, 1) CALL(256, 1) \
  CALL(384, 1) CALL(384, 2) CALL(512, 1) CALL(512, 2) CALL(512, 3)
#define FF_NORM_FORWARD(CALL) FF_NORM_BOTH(CALL) CALL(128, 3) CALL(256, 2)
#define FF_NORM_BACKWARD(CALL) FF_NORM_BOTH(CALL) CALL(192, 2)

}  // namespace ff
