// What linfusion_keep8.hip offers the library's other translation units.
#pragma once
#include "lf_rows_api.hpp"

namespace lf { struct KeepArgs; }

namespace lfh {
// How workgroups of 256 threads share C channels, eight a lane: lanes of a token (a multiple of four) and workgroups across, so that most of
// them have work (C = 320: 40 lanes and six tokens, where 32 lanes would take two workgroups, the second a quarter full).
struct Across { int lanes, blocks; };
inline Across across(int C) {
  const int wide = C / 8;
  Across best{32, (wide + 31) / 32};
  double most = 0.0;
  for (int blocks = (wide + 255) / 256; blocks <= (wide + 15) / 16; ++blocks) {
    const int lanes = ((wide + blocks - 1) / blocks + 3) / 4 * 4;
    if (lanes > 256) continue;
    const double used = (double)wide / blocks * (256 / lanes) / 256.0;
    if (used > most + 0.02) {
      most = used;
      best = Across{lanes, (wide + lanes - 1) / lanes};
    }
  }
  return best;
}

// Values of `dtype` from codes and exponents; the tokens per workgroup are chosen here.
void launch_unkeep8(const lf::KeepArgs& a, int B, int dtype, hipStream_t st);
}  // namespace lfh
