// The shape of a product's tiles, and the tensor maps of its operands.  Host code without CUDA calls.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "as_fp8.h"
#include "fp8_context.h"

constexpr int LIN_BM = 128;                  // rows of results of a CTA
constexpr int LIN_BK = 64;                   // steps of the summed index of a stage

namespace as_lin {

// cg: CTAs that share a tile's rows; bn: its columns; parts: of the summed index, shared by a cluster of CTAs or left in the workspace.
struct Plan { int cg, bn, parts; bool shared; double ns; };

// By the time that the turns of all SMs take: turns x steps x ns a step, and what the reading out of the last turn and the meeting of a pair add.  What a step takes is its bytes into an SM, 64 a
// clock, and beside them, from 256 x 256 on, its MMAs.  A tile's results take the warps 1.9 us (two strips of 32 columns each: 3.3), which a short sum does not hide: 6144 x 1280 from 3 rows takes 18 us in
// tiles of 128 x 64 and 11 of 128 x 256.  A part more costs its sums' way to the workspace and back, and a launch; a cluster costs the meeting and the sums, and more with every CTA beyond
// two, and holds as many tiles at once as the device has such clusters.  most_steps: that a cluster's CTA may add up by itself.  clusters == nullptr: single CTAs alone.
inline Plan plan_of(long long entries, long long T, long long M, long long N, long long ksteps, bool b_mn, int most_steps, int sms, const int* clusters) {
  static const int ns[2][8] = {{230, 250, 265, 300, 345, 385, 440, 500}, {228, 230, 240, 262, 297, 320, 365, 410}};
  Plan best{1, 64, 1, false, 1e300};
  for (int cg = 1; cg <= (clusters != nullptr ? 2 : 1); ++cg)
    for (int i = 0; i < 8; ++i) {
      const int bn = 32 * (i + 1);
      if (b_mn && bn % (64 * cg) != 0) continue;
      const long long tiles = entries * ((T + LIN_BM * cg - 1) / (LIN_BM * cg)) * ((N + bn - 1) / bn), units = sms / cg;
      for (int parts = 1; parts <= 16 && parts <= ksteps; ++parts) {
        const long long steps = (ksteps + parts - 1) / parts;
        if (parts == 1 || tiles * parts <= 2 * units) {
          const long long all = tiles * parts, whole = (all + units - 1) / units;
          const double turns = whole == 1 ? 1. : 0.5 * ((double)all / units + whole);
          const double step = (double)steps * ns[cg - 1][i];
          double t = (turns - 1.) * std::max(step, bn <= 128 ? 1900. : 3300.) + step + 10. * bn + (cg == 2 ? 400. : 0.);
          if (parts > 1) t += 3000. + 200. * parts + (double)M * (double)N * 4. * (parts + 1) / 6000.;
          if (t < best.ns) best = {cg, bn, parts, false, t};
        }
        if (clusters != nullptr && cg == 1 && parts > 1 && parts <= MAX_PARTS && tiles <= clusters[parts] && steps <= most_steps) {
          const double t = (double)steps * ns[0][i] + 10. * bn + 1700. + 8. * std::max(bn - 64, 0) + (parts - 2) * (100. + 4. * bn);
          if (t < best.ns) best = {1, bn, parts, true, t};
        }
      }
    }
  return best;
}

}  // namespace as_lin

namespace as_tc {

// A bf16 matrix [rows, cols] in rows or heads as a 4-D tensor: column of a head, token, head, batch entry; boxes of 64 columns x box_rows tokens with the 128-byte swizzle; what
// lies outside reads as 0.  (Defined in tensor_init.cu.)
bool make_map_boxes(CUtensorMap* m, const as_rows_t& x, long long rows, long long cols, int box_rows);
// A matrix in bf16 or fp32 the same way, in boxes of 64 bytes x 32 tokens with the 64-byte swizzle.
bool make_map_strips(CUtensorMap* m, const as_rows_t& x, long long rows, long long cols);

}  // namespace as_tc

// Per-device set-up of the linear layers' kernels (shared-memory opt-in).
cudaError_t as_linear_init();
