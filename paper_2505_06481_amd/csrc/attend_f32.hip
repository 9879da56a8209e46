// Attention over fp32 pages.
#include "attend_kernel.h"

namespace mmoe {

void attend_f32(int D, const Shares& r, const AttendArgs& g, hipStream_t st) { attend_kind<kF32>(D, r, g, st); }

}  // namespace mmoe
