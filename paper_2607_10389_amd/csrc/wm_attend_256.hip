// wm_attend_256.hip -- attention over the paged cache, heads of 256.
#include "wm_attend.h"

namespace wm {
int launch_attend_256(const AttendArgs &a, void *stream) { return attend_dim<256>(a, stream); }
}  // namespace wm
