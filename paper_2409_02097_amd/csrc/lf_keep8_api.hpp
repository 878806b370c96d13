// What linfusion_keep8.hip offers the library's other translation units.
#pragma once
#include "lf_rows_api.hpp"

namespace lf { struct KeepArgs; }

namespace lfh {
// Values of `dtype` from codes and exponents; the tokens per workgroup are chosen here.
void launch_unkeep8(const lf::KeepArgs& a, int B, int dtype, hipStream_t st);
}  // namespace lfh
