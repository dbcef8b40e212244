// The paged tile kernels for d = 128, blocks of 256 rows.
#include "paged_tiles.h"

namespace attn {

hipError_t launch_paged_tiles_d128_w8(const PagedArgs& a, int form, hipStream_t stream) {
    return launch_paged_tiles_d<128, 8>(a, form, stream);
}

}  // namespace attn
