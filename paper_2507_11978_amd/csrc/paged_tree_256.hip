// Attention for trees of drafted tokens over a paged cache, head sizes up to 256
#include "paged_tree.h"

namespace nt {

nt_status launch_paged_tree_256(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream) { return launch_paged_tree_size<256>(a, rows, programs, bf16, kind, stream); }

}  // namespace nt
