// Paged attention of chunks over keys and values of 8 bits.
#include "paged_many.h"

namespace jx {

hipError_t launch_paged_many8(const PagedArgs& g, int rows, hipStream_t st) {
    return g.a.dtype == JX_BF16 ? launch_many_dim<__bf16, uint8_t>(g, rows, st) : launch_many_dim<_Float16, uint8_t>(g, rows, st);
}

}  // namespace jx
