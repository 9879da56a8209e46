// Attention over bf16 pages.
#include "attend_kernel.h"

namespace mmoe {

void attend_bf16(int D, const Shares& r, const AttendArgs& g, hipStream_t st) { attend_kind<kBf16>(D, r, g, st); }

}  // namespace mmoe
