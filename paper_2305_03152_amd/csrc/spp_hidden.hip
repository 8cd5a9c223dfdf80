// The product of hidden rows in 8 bits with weights in the same format.
#include "spp_hidden_kernels.h"

extern "C" int spp_fp8_product(spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, const void* d_weights, int32_t n_groups,
                               int32_t D, int32_t H, int32_t type, uint32_t flags) {
    return spp::hidden<spp::kProduct>("spp_fp8_product", ctx, lists, nullptr, n_lists, d_weights, n_groups, D, H, type, 0, flags);
}
