// wm_attend_128.hip -- attention over the paged cache, heads of 128.
#include "wm_attend.h"

namespace wm {
int launch_attend_128(const AttendArgs &a, void *stream) { return attend_dim<128>(a, stream); }
}  // namespace wm
