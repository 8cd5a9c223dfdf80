#include "spp_hidden.h"

namespace spp {

// A workgroup takes 128 rows of X by 128 columns: of the product, or 64 of the gate's and the same 64 of the other factor.  Steps of 128
// columns of X and W go through LDS, the next asked for while one is multiplied.
constexpr int kTileRows = 128, kTileBlock = 256, kTileLd = kFp8Block + 16;
constexpr int kTileBuffer = 2 * kTileRows * kTileLd + 2 * kTileRows;       // rows of X, rows of W, their scales

template <class T, int Mode>
__global__ void __launch_bounds__(kTileBlock) hidden_tile_kernel(HiddenArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Lists lists(a.t, kTileRows);
    const int total = lists.total();
    if (total == 0) return;
    const int wave = threadIdx.x >> 6, l = lane_id(), m = l & 15, q = l >> 4;
    constexpr int cols = Mode == kProduct ? 128 : 64;
    const int parts = (a.H + cols - 1) / cols;
    const Share share((int64_t)total * parts);
    for (int64_t item = share.at; item < share.end; item += share.step) {
        const int tile = (int)(item / parts), h0 = (int)(item - (int64_t)tile * parts) * cols;
        const int list = lists.list_of(tile);
        const int64_t r0 = (int64_t)(tile - lists.first_tile(list)) * kTileRows;
        const int64_t left = lists.rows_in(list) - r0;
        const int here = left < kTileRows ? (int)left : kTileRows;
        const uint8_t* x = a.t.rows[list] + r0 * a.rb;
        const uint8_t* w = a.w + (int64_t)a.t.group[list] * a.H * (Mode == kProduct ? 1 : 2) * a.rb;
        // Row r of the 128 of W: a column of the result.
        auto w_row = [&](int r) {
            int h = h0 + (Mode == kProduct ? r : r & 63);
            h = h < a.H ? h : a.H - 1;
            return w + (int64_t)(Mode == kProduct || r < 64 ? h : a.H + h) * a.rb;
        };
        u32x4 next[8];
        uint8_t next_scale;
        auto ask = [&](int s) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = k * kTileBlock + (int)threadIdx.x, r = i >> 3, at = 128 * s + 16 * (i & 7);
                const bool in = at < a.cb;
                next[k] = *reinterpret_cast<const u32x4*>(x + (int64_t)(r < here ? r : here - 1) * a.rb + (in ? at : 0));
                next[4 + k] = *reinterpret_cast<const u32x4*>(w_row(r) + (in ? at : 0));
                if (!in) next[k] = next[4 + k] = u32x4{0, 0, 0, 0};
            }
            const int r = (int)threadIdx.x & 127;
            next_scale = (threadIdx.x < 128 ? x + (int64_t)(r < here ? r : here - 1) * a.rb : w_row(r))[a.cb + s];
        };
        // by operand: columns 4m + f of each 64 as row 16 f + m
        auto operand = [](int r) { return (r & 64) + (r & 3) * 16 + ((r & 63) >> 2); };
        auto keep = [&](uint8_t* to) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = k * kTileBlock + (int)threadIdx.x, r = i >> 3, at = 16 * (i & 7);
                *reinterpret_cast<u32x4*>(to + r * kTileLd + at) = next[k];
                *reinterpret_cast<u32x4*>(to + (kTileRows + operand(r)) * kTileLd + at) = next[4 + k];
            }
            const int r = (int)threadIdx.x & 127;
            to[2 * kTileRows * kTileLd + (threadIdx.x < 128 ? r : 128 + operand(r))] = next_scale;
        };
        f32x4 acc[2][8];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int f = 0; f < 8; ++f) acc[c][f] = f32x4{0.f, 0.f, 0.f, 0.f};
        ask(0);
        __syncthreads();                                 // the item before has been worked off
        for (int s = 0; s < a.steps; ++s) {
            uint8_t* buffer = lds + (s & 1) * kTileBuffer;
            keep(buffer);
            if (s + 1 < a.steps) ask(s + 1);
            __syncthreads();                             // (and the buffer of the step after next has been read by all)
            const uint8_t* scales = buffer + 2 * kTileRows * kTileLd;
            auto operand_at = [&](int row) {
                const uint8_t* p = buffer + row * kTileLd + 16 * q;
                return Operand{*reinterpret_cast<const u32x4*>(p), *reinterpret_cast<const u32x4*>(p + 64), scales[row]};
            };
            Operand xv[2], wv[8];
#pragma unroll
            for (int c = 0; c < 2; ++c) xv[c] = operand_at(32 * wave + 16 * c + m);
#pragma unroll
            for (int f = 0; f < 8; ++f) wv[f] = operand_at(kTileRows + 16 * f + m);
            multiply<sizeof(T) == 4>(acc, xv, wv);
        }
        const int64_t ld = a.t.ld[list];
        T* y = static_cast<T*>(a.t.y[list]) + r0 * ld;
        const bool wide = ((uintptr_t)a.t.y[list] | (uint64_t)(ld * (int64_t)sizeof(T))) % (4 * sizeof(T)) == 0;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int row = 32 * wave + 16 * c + 4 * q, have = here - row;
            f32x4(&one)[4] = reinterpret_cast<f32x4(&)[4]>(acc[c][0]);
            f32x4(&two)[4] = reinterpret_cast<f32x4(&)[4]>(acc[c][4]);
            if constexpr (Mode == kProduct) {
                put_tile<T>(y + row * ld, ld, have, h0 + 4 * m, a.H, wide, one);
                put_tile<T>(y + row * ld, ld, have, h0 + 64 + 4 * m, a.H, wide, two);
            } else if constexpr (Mode == kGated) {
                with_activation(a.act, [&](auto act) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) one[k][i] = activate<decltype(act)::value>(one[k][i]) * two[k][i];
                });
                put_tile<T>(y + row * ld, ld, have, h0 + 4 * m, a.H, wide, one);
            } else {
                f32x4 dy[4];
                get_tile<T>(y + row * ld, ld, have, h0 + 4 * m, a.H, wide, dy);
                with_activation(a.act, [&](auto act) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float f, d;
                            activate_both<decltype(act)::value>(one[k][i], f, d);
                            one[k][i] = dy[k][i] * two[k][i] * d;
                            two[k][i] = dy[k][i] * f;
                        }
                });
                const int64_t pld = a.dp_ld[list];
                T* p = static_cast<T*>(a.dp[list]) + (r0 + row) * pld;
                const bool pwide = ((uintptr_t)a.dp[list] | (uint64_t)(pld * (int64_t)sizeof(T)) | (uint64_t)(a.H * (int)sizeof(T))) % (4 * sizeof(T)) == 0;
                put_tile<T>(p, pld, have, h0 + 4 * m, a.H, pwide, one);
                put_tile<T>(p + a.H, pld, have, h0 + 4 * m, a.H, pwide, two);
            }
        }
    }
}

template <class T, int Mode>
static int launch_hidden(spp_ctx* ctx, const HiddenArgs& a) {
    auto kernel = hidden_tile_kernel<T, Mode>;
    static LdsLimit limit;
    SPP_TRY(limit.allow(ctx, reinterpret_cast<const void*>(kernel), 2 * kTileBuffer));
    int64_t tiles = 0;
    for (int j = 0; j < a.t.n_lists; ++j) tiles += (a.t.n[j] + (int64_t)kTileRows - 1) / kTileRows;
    constexpr int cols = Mode == kProduct ? 128 : 64;
    const int64_t want = tiles * ((a.H + cols - 1) / cols), most = (int64_t)ctx->num_cu * 64;
    kernel<<<(unsigned)(want < most ? want : most), kTileBlock, 2 * kTileBuffer, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}

// The checks of the three entries, and the launch.
template <int Mode>
static int hidden(const char* who, spp_ctx* ctx, const spp_row_list* lists, const spp_row_list* grads, int32_t n_lists, const void* d_weights,
                  int32_t n_groups, int32_t D, int32_t H, int32_t type, int32_t activation, uint32_t flags) {
    SPP_CHECK(ctx && d_weights, SPP_E_ARG, "%s: null argument", who);
    SPP_CHECK((uintptr_t)d_weights % 16 == 0, SPP_E_ARG, "%s: weights must be 16-byte aligned", who);
    HiddenArgs a;
    memset(&a, 0, sizeof(a));
    int64_t most = 0;
    SPP_TRY(row_table(who, lists, n_lists, n_groups, D, H, type, a.t, &most));
    if (Mode != kProduct) {
        SPP_CHECK(H <= SPP_MAX_HIDDEN / 2, SPP_E_ARG, "%s: H = %d (1 .. %d)", who, H, SPP_MAX_HIDDEN / 2);
        SPP_CHECK(activation == SPP_SILU || activation == SPP_GELU || activation == SPP_SIGMOID, SPP_E_ARG, "%s: activation %d", who, activation);
    }
    if (Mode == kGatedGrad) {
        RowTable p;
        int64_t also = 0;
        SPP_CHECK(grads || n_lists == 0, SPP_E_ARG, "%s: null argument", who);
        SPP_TRY(row_table(who, grads, n_lists, n_groups, D, 2 * H, type, p, &also));
        for (int j = 0; j < n_lists; ++j)
            SPP_CHECK(lists[j].d_rows == grads[j].d_rows && lists[j].n == grads[j].n && lists[j].d_n == grads[j].d_n && lists[j].group == grads[j].group,
                      SPP_E_ARG, "%s: list %d: the gradient's rows, count or group are not the list's", who, j);
        for (int j = 0; j < n_lists; ++j) { a.dp[j] = p.y[j]; a.dp_ld[j] = p.ld[j]; }
    }
    if (most > 0) {
        a.w = static_cast<const uint8_t*>(d_weights);
        a.D = D; a.H = H; a.rb = fp8_bytes(D); a.cb = fp8_code_bytes(D); a.steps = fp8_blocks(D); a.act = activation;
        SPP_HIP(hipSetDevice(ctx->device));
        ScopedTimer timer(ctx, SPP_T_LAYER, ctx->stream);
        SPP_TRY(type == SPP_F32 ? (launch_hidden<float, Mode>(ctx, a)) : type == SPP_F16 ? (launch_hidden<_Float16, Mode>(ctx, a))
                                                                                          : (launch_hidden<__bf16, Mode>(ctx, a)));
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}

}  // namespace spp

extern "C" int spp_fp8_product(spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, const void* d_weights, int32_t n_groups,
                               int32_t D, int32_t H, int32_t type, uint32_t flags) {
    return spp::hidden<spp::kProduct>("spp_fp8_product", ctx, lists, nullptr, n_lists, d_weights, n_groups, D, H, type, 0, flags);
}

extern "C" int spp_fp8_gated(spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, const void* d_weights, int32_t n_groups,
                             int32_t D, int32_t H, int32_t type, int32_t activation, uint32_t flags) {
    return spp::hidden<spp::kGated>("spp_fp8_gated", ctx, lists, nullptr, n_lists, d_weights, n_groups, D, H, type, activation, flags);
}

extern "C" int spp_fp8_gated_grad(spp_ctx* ctx, const spp_row_list* lists, const spp_row_list* grads, int32_t n_lists, const void* d_weights,
                                  int32_t n_groups, int32_t D, int32_t H, int32_t type, int32_t activation, uint32_t flags) {
    return spp::hidden<spp::kGatedGrad>("spp_fp8_gated_grad", ctx, lists, grads, n_lists, d_weights, n_groups, D, H, type, activation, flags);
}
