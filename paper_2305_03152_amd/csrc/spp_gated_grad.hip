// The backward pass of the gated layer on hidden rows in 8 bits.
#include "spp_hidden_kernels.h"

extern "C" int spp_fp8_gated_grad(spp_ctx* ctx, const spp_row_list* lists, const spp_row_list* grads, int32_t n_lists, const void* d_weights,
                                  int32_t n_groups, int32_t D, int32_t H, int32_t type, int32_t activation, uint32_t flags) {
    return spp::hidden<spp::kGatedGrad>("spp_fp8_gated_grad", ctx, lists, grads, n_lists, d_weights, n_groups, D, H, type, activation, flags);
}
