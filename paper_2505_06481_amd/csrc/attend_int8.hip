// Attention over int8 pages.
#include "attend_kernel.h"

namespace mmoe {

void attend_int8(int D, const Shares& r, const AttendArgs& g, hipStream_t st) { attend_kind<kInt8>(D, r, g, st); }

}  // namespace mmoe
