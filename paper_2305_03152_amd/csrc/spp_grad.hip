// The weight gradient over feature rows in MXFP4.
#include "spp_grad.h"

extern "C" int spp_mx4_weight_grad(spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, int32_t n_groups, int32_t D, int32_t H,
                                   int32_t type, float* d_grad, uint32_t flags) {
    return spp::weight_grad<spp::GradMx4>("spp_mx4_weight_grad", ctx, lists, n_lists, n_groups, D, H, type, d_grad, spp::mx4_bytes(D), flags);
}
