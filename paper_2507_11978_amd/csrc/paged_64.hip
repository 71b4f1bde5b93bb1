// Paged attention, head sizes up to 64
#include "paged_launch.h"

namespace nt {

nt_status launch_paged_64(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream) { return launch_paged_size<64>(a, rows, programs, bf16, kind, stream); }

}  // namespace nt
