// The weight gradient over hidden rows in 8 bits.
#include "spp_fp8.h"
#include "spp_grad.h"

extern "C" int spp_fp8_weight_grad(spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, int32_t n_groups, int32_t D, int32_t H,
                                   int32_t type, float* d_grad, uint32_t flags) {
    return spp::weight_grad<spp::GradFp8>("spp_fp8_weight_grad", ctx, lists, n_lists, n_groups, D, H, type, d_grad, spp::fp8_bytes(D), flags);
}
