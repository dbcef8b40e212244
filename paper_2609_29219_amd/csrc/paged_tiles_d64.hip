// The paged tile kernels for d = 64.
#include "paged_tiles.h"

namespace attn {

hipError_t launch_paged_tiles_d64(const PagedArgs& a, int form, hipStream_t stream) {
    return launch_paged_tiles_d<64>(a, form, stream);
}

}  // namespace attn
