// wm_attend_192.hip -- attention over the paged cache, heads of 192.
#include "wm_attend.h"

namespace wm {
int launch_attend_192(const AttendArgs &a, void *stream) { return attend_dim<192>(a, stream); }
}  // namespace wm
