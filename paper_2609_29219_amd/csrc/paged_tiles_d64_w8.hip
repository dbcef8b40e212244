// The paged tile kernels for d = 64, blocks of 256 rows.
#include "paged_tiles.h"

namespace attn {

hipError_t launch_paged_tiles_d64_w8(const PagedArgs& a, int form, hipStream_t stream) {
    return launch_paged_tiles_d<64, 8>(a, form, stream);
}

}  // namespace attn
