// Attention over e4m3 pages.
#include "attend_kernel.h"

namespace mmoe {

void attend_fp8(int D, const Shares& r, const AttendArgs& g, hipStream_t st) { attend_kind<kFp8>(D, r, g, st); }

}  // namespace mmoe
