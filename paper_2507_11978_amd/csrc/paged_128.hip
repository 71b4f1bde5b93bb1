// Paged attention, head sizes up to 128
#include "paged_launch.h"

namespace nt {

nt_status launch_paged_128(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream) { return launch_paged_size<128>(a, rows, programs, bf16, kind, stream); }

}  // namespace nt
