// Paged attention of few rows for each request over keys and values of 16 bits.
#include "paged_few.h"

namespace jx {

hipError_t launch_paged_few(const PagedArgs& g, int rows, hipStream_t st) {
    if (g.a.dtype == JX_BF16) return rows == 16 ? launch_few_dim<__bf16, __bf16, 1>(g, st) : launch_few_dim<__bf16, __bf16, 2>(g, st);
    return rows == 16 ? launch_few_dim<_Float16, _Float16, 1>(g, st) : launch_few_dim<_Float16, _Float16, 2>(g, st);
}

}  // namespace jx
