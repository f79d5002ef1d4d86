// wm_attend_64.hip -- attention over the paged cache, heads of 64.
#include "wm_attend.h"

namespace wm {
int launch_attend_64(const AttendArgs &a, void *stream) { return attend_dim<64>(a, stream); }
}  // namespace wm
