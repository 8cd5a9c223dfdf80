// Feature rows in MXFP4: quantisation of rows of 16- or 32-bit floats, and back.
//
//   block of 32 columns, a = max |x|:  e = max(floor(log2 a) - 2, -127),  code = nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} to |x| / 2^e,
//   ties to the even code, 6 for what lies above; the scale byte is e + 127.  A block with a NaN or an infinity is NaN as a whole.
//
// Both directions move each byte once and are bound by HBM.  A lane has 8 columns, so four lanes share a block and find its
// largest value with two exchanges between neighbours; the lanes of a wavefront read and write side by side.
#include "spp_mx4.h"

namespace spp {

constexpr int kMxBlock = 256;

struct MxArgs {
    const void*    x;
    void*          rows;
    const int64_t* d_n;
    int64_t        n, ld;        // ld: elements from a row of x to the next
    int32_t        D, nb, rb;
    int32_t        units;        // lanes per row: 4 nb
    uint32_t       magic;        // ceil(2^32 / units)
    int32_t        tile;         // rows of a workgroup's round
    int32_t        wide;         // x may be taken 16 bytes at a time
};

template <class T>
__device__ __forceinline__ void load8(const T* p, int have, bool wide, float (&x)[8]) {
    if (have >= 8 && wide) {
        if constexpr (sizeof(T) == 4) {
            const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
        } else {
            const typename Elem<T>::v8 a = *reinterpret_cast<const typename Elem<T>::v8*>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < have ? (float)p[i] : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void store8(T* p, int have, bool wide, const float (&x)[8]) {
    if (have >= 8 && wide) {
        if constexpr (sizeof(T) == 4) {
            const f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
            *reinterpret_cast<f32x4*>(p) = a;
            *reinterpret_cast<f32x4*>(p + 4) = b;
        } else {
            typename Elem<T>::v8 a;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = (T)x[i];
            *reinterpret_cast<typename Elem<T>::v8*>(p) = a;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = (T)x[i];
    }
}

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {           // over the four lanes of a block
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);      // lanes 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);               // lanes 2 3 0 1
    return v > o ? v : o;
}

template <class T>
__global__ void __launch_bounds__(kMxBlock) mx4_quantize_kernel(MxArgs a) {
    const int64_t n = rows_of(a.n, a.d_n);
    const int all = a.tile * a.units;
    for (int64_t r0 = (int64_t)blockIdx.x * a.tile; r0 < n; r0 += (int64_t)gridDim.x * a.tile) {
        // the four lanes of a block stay together: units and the workgroup's size are multiples of four
        for (int u = threadIdx.x; u < all; u += kMxBlock) {
            const int row = (int)__umulhi((uint32_t)u, a.magic), j = u - row * a.units;
            if (r0 + row >= n) break;
            float x[8];
            load8(static_cast<const T*>(a.x) + (r0 + row) * a.ld + 8 * j, a.D - 8 * j, a.wide, x);
            uint32_t top = 0;                    // bits of |x| order as the values do, NaN above infinity above the rest
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
                top = top > b ? top : b;
            }
            top = quad_max(top);
            const bool bad = top >= 0x7F800000u;
            int e = (int)(top >> 23) - 127 - 2;              // a subnormal block has the least scale, as has a block of zeros
            e = e < -127 ? -127 : e;
            uint32_t code = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = ldexpf(x[2 * i], -e), hi = ldexpf(x[2 * i + 1], -e);
                uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, lo, hi, 1.0f, 0);
                code |= (c & 255u) << (8 * i);
            }
            uint8_t* out = static_cast<uint8_t*>(a.rows) + (r0 + row) * a.rb;
            *reinterpret_cast<uint32_t*>(out + 4 * j) = bad ? 0u : code;
            if ((j & 3) == 0) out[16 * a.nb + (j >> 2)] = bad ? (uint8_t)255 : (uint8_t)(e + 127);
            for (int k = 17 * a.nb + j; k < a.rb; k += a.units) out[k] = 0;
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kMxBlock) mx4_dequantize_kernel(MxArgs a) {
    const int64_t n = rows_of(a.n, a.d_n);
    const int all = a.tile * a.units;
    for (int64_t r0 = (int64_t)blockIdx.x * a.tile; r0 < n; r0 += (int64_t)gridDim.x * a.tile)
        for (int u = threadIdx.x; u < all; u += kMxBlock) {
            const int row = (int)__umulhi((uint32_t)u, a.magic), j = u - row * a.units;
            if (r0 + row >= n) break;
            const uint8_t* in = static_cast<const uint8_t*>(a.rows) + (r0 + row) * a.rb;
            const uint32_t code = *reinterpret_cast<const uint32_t*>(in + 4 * j);
            const float s = mx4_scale(in[16 * a.nb + (j >> 2)]);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t c = (code >> (4 * i)) & 15u;
                // E2M1 to fp32: exponent codes 1..3 are 2^0..2^2 with one bit of mantissa, 0 and 1 alone are 0 and a half
                const uint32_t m = c & 7u;
                const uint32_t bits = m >= 2u ? (m << 22) + (126u << 23) : m ? 0x3F000000u : 0u;
                x[i] = __uint_as_float(bits | (c & 8u) << 28) * s;
            }
            store8(static_cast<T*>(const_cast<void*>(a.x)) + (r0 + row) * a.ld + 8 * j, a.D - 8 * j, a.wide, x);
        }
}

static int mx4_args(const char* who, spp_ctx* ctx, const void* x, int32_t type, int64_t n, const int64_t* d_n, int32_t D, int64_t ld,
                    const void* rows, MxArgs& a) {
    SPP_CHECK(ctx, SPP_E_ARG, "%s: ctx is null", who);
    SPP_CHECK(is_type(type), SPP_E_ARG, "%s: element type %d", who, type);
    SPP_CHECK(D >= 1 && D <= SPP_MX4_MAX_COLS, SPP_E_ARG, "%s: D = %d (1 .. %d)", who, D, SPP_MX4_MAX_COLS);
    SPP_CHECK(n >= 0 && n <= 0x7FFFFFFFll && ld >= D, SPP_E_ARG, "%s: n = %lld, ld = %lld", who, (long long)n, (long long)ld);
    SPP_CHECK(n == 0 || (x && rows), SPP_E_ARG, "%s: null argument", who);
    SPP_CHECK((uintptr_t)x % type_bytes(type) == 0 && (uintptr_t)rows % 16 == 0, SPP_E_ARG,
              "%s: rows must be 16-byte aligned, values aligned to their type", who);
    a.x = x; a.rows = const_cast<void*>(rows); a.d_n = d_n; a.n = n; a.ld = ld; a.D = D;
    a.nb = mx4_blocks(D); a.rb = mx4_bytes(D); a.units = 4 * a.nb;
    a.magic = (uint32_t)((0x100000000ull + a.units - 1) / a.units);
    a.tile = a.units < 1024 ? 1024 / a.units : 1;
    a.wide = (uintptr_t)x % 16 == 0 && ld * (int64_t)type_bytes(type) % 16 == 0;
    return SPP_OK;
}
static unsigned mx4_grid(const spp_ctx* ctx, const MxArgs& a) {
    const int64_t tiles = (a.n + a.tile - 1) / a.tile, most = (int64_t)ctx->num_cu * 32;
    return (unsigned)(tiles < most ? tiles : most);
}

}  // namespace spp

extern "C" int64_t spp_mx4_row_bytes(int32_t D) {
    SPP_CHECK(D >= 1 && D <= SPP_MX4_MAX_COLS, SPP_E_ARG, "spp_mx4_row_bytes: D = %d (1 .. %d)", D, SPP_MX4_MAX_COLS);
    return spp::mx4_bytes(D);
}

extern "C" int spp_mx4_quantize(spp_ctx* ctx, const void* d_x, int32_t type, int64_t n, const int64_t* d_n, int32_t D, int64_t ld,
                                void* d_rows, uint32_t flags) {
    using namespace spp;
    MxArgs a;
    SPP_TRY(mx4_args("spp_mx4_quantize", ctx, d_x, type, n, d_n, D, ld, d_rows, a));
    if (n > 0) {
        SPP_HIP(hipSetDevice(ctx->device));
        ScopedTimer timer(ctx, SPP_T_MX4, ctx->stream);
        const unsigned grid = mx4_grid(ctx, a);
        if (type == SPP_F32) mx4_quantize_kernel<float><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        else if (type == SPP_F16) mx4_quantize_kernel<_Float16><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        else mx4_quantize_kernel<__bf16><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        SPP_HIP(hipGetLastError());
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}

extern "C" int spp_mx4_dequantize(spp_ctx* ctx, const void* d_rows, int64_t n, const int64_t* d_n, int32_t D, void* d_x, int32_t type,
                                  int64_t ld, uint32_t flags) {
    using namespace spp;
    MxArgs a;
    SPP_TRY(mx4_args("spp_mx4_dequantize", ctx, d_x, type, n, d_n, D, ld, d_rows, a));
    if (n > 0) {
        SPP_HIP(hipSetDevice(ctx->device));
        ScopedTimer timer(ctx, SPP_T_MX4, ctx->stream);
        const unsigned grid = mx4_grid(ctx, a);
        if (type == SPP_F32) mx4_dequantize_kernel<float><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        else if (type == SPP_F16) mx4_dequantize_kernel<_Float16><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        else mx4_dequantize_kernel<__bf16><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        SPP_HIP(hipGetLastError());
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}
