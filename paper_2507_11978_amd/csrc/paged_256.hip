// Paged attention, head sizes up to 256
#include "paged_launch.h"

namespace nt {

nt_status launch_paged_256(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream) { return launch_paged_size<256>(a, rows, programs, bf16, kind, stream); }

}  // namespace nt
