// The gated layer on hidden rows in 8 bits.
#include "spp_hidden_kernels.h"

extern "C" int spp_fp8_gated(spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, const void* d_weights, int32_t n_groups,
                             int32_t D, int32_t H, int32_t type, int32_t activation, uint32_t flags) {
    return spp::hidden<spp::kGated>("spp_fp8_gated", ctx, lists, nullptr, n_lists, d_weights, n_groups, D, H, type, activation, flags);
}
