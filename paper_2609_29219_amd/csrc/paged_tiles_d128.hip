// The paged tile kernels for d = 128.
#include "paged_tiles.h"

namespace attn {

hipError_t launch_paged_tiles_d128(const PagedArgs& a, int form, hipStream_t stream) {
    return launch_paged_tiles_d<128>(a, form, stream);
}

}  // namespace attn
