// The paged tile kernels for d = 128, blocks of 128 rows.
#include "paged_tiles.h"

namespace attn {

hipError_t launch_paged_tiles_d128_w4(const PagedArgs& a, int form, hipStream_t stream) {
    if (form == 0) return launch_paged_tiles_form<128, 4, 0>(a, stream);
    if (form == 1) return launch_paged_tiles_form<128, 4, 1>(a, stream);
    if (form == 2) return launch_paged_tiles_form<128, 4, 2>(a, stream);
    if (form == 3) return launch_paged_tiles_form<128, 4, 3>(a, stream);
    return hipErrorInvalidValue;
}

}  // namespace attn
