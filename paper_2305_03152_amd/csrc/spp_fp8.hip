// Hidden rows in 8 bits: quantisation of rows of 16- or 32-bit floats, and back.
//
//   block of 128 columns, a = max |x| of what is finite:  e = the smallest integer with a <= 448 2^e, at least -117 and at most 119,
//   code = nearest E4M3 to x / 2^e, ties to even, 448 for what lies above (of more than 448 2^119 only);  NaN for what is not finite.
//
// The scale is a power of two, so that a code under it is exact in bf16, and rounded up, so that nothing saturates: an E4M3's
// relative step is the same under any scale, and a block has 15 powers of two below its largest value before its steps widen.
// A block's lanes find its largest value together: sixteen of 8 columns each, of rows of up to 64 and 32 columns eight and four, so
// that fewer are idle.
//
// Bound by HBM: 2.56M rows of 256 in bf16 quantised in 336 us, read back in 344, 5.9 TB/s both.
#include "spp_fp8.h"
#include "spp_rows.h"

namespace spp {

struct Fp8Rows {
    static constexpr int lds = 4128, columns = kFp8Block;
    static constexpr bool skips = true;
    static void layout(MxArgs& a) {
        a.nb = fp8_blocks(a.D); a.rb = fp8_bytes(a.D); a.cb = fp8_code_bytes(a.D);
        a.share = a.D > 64 ? 16 : a.D > 32 ? 8 : 4;
    }
    static __device__ __forceinline__ int scale_at(const MxArgs& a, int column) { return a.cb + column / kFp8Block; }
    static __device__ __forceinline__ uint32_t block_max(uint32_t v, int share) {
        v = quad_max(v);
        if (share > 4) {
            const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true);      // eight lanes mirrored
            v = v > o ? v : o;
        }
        if (share > 8) {
            const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true);      // sixteen
            v = v > o ? v : o;
        }
        return v;
    }
    // The scale's byte: 448 = 1.75 2^8, so what is above 1.75 times its own power of two takes one more.
    static __device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
        const int e = (int)((top + 0x1FFFFFu) >> 23) - 8;
        return (uint32_t)(e < kFp8LeastScale ? kFp8LeastScale : e > kFp8MostScale ? kFp8MostScale : e);
    }
    template <class T>
    static __device__ __forceinline__ void put(const Eight<T>& v, const MxArgs& a, uint8_t* out, int piece) {
        uint32_t top = v.top();
        u32x2 code;
        uint32_t byte;
        if (__any(top > kFp8Most)) {                         // seldom: a value that is not finite, or too large for the largest scale
            Eight<float> w;
            uint32_t nan[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x = v.at(i);
                const bool odd = (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u;
                if (odd) nan[i >> 2] |= 0xFFu << (8 * (i & 3));
                const float most = __uint_as_float(kFp8Most);
                x = odd ? 0.0f : x > most ? most : x < -most ? -most : x;
                if (i < 4) w.a[i] = x; else w.b[i - 4] = x;
            }
            top = block_max(w.top(), a.share);
            byte = scale_byte(top);
            code = w.codes8(mx4_scale(byte));
            code = u32x2{(code.x & ~nan[0]) | (0x7F7F7F7Fu & nan[0]), (code.y & ~nan[1]) | (0x7F7F7F7Fu & nan[1])};
        } else {
            top = block_max(top, a.share);
            byte = scale_byte(top);
            code = v.codes8(mx4_scale(byte));
        }
        if (8 * piece < a.cb) *reinterpret_cast<u32x2*>(out + 8 * piece) = code;
        if ((piece & (a.share - 1)) == 0) out[a.cb + piece / 16] = (uint8_t)byte;
    }
    template <int VE>
    struct Codes {
        uint32_t code[VE / 4];
        __device__ __forceinline__ void fetch(const uint8_t* row, int piece) {
            if constexpr (VE == 8) {
                const u32x2 c = reinterpret_cast<const u32x2*>(row)[piece];
                code[0] = c.x; code[1] = c.y;
            } else {
                code[0] = reinterpret_cast<const uint32_t*>(row)[piece];
            }
        }
        template <class T>
        __device__ __forceinline__ auto value(float s) const {
            typedef T V __attribute__((ext_vector_type(VE)));
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            V v;
#pragma unroll
            for (int i = 0; i < VE / 4; ++i) {
                if constexpr (__is_same(T, __bf16)) {
                    const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[i], s, false), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[i], s, true);
                    v[4 * i] = v0[0]; v[4 * i + 1] = v0[1]; v[4 * i + 2] = v1[0]; v[4 * i + 3] = v1[1];
                } else {                                     // by way of fp32, which holds every value, and rounded to 16 bits from there
                    const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[i], s, false), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[i], s, true);
                    v[4 * i] = (T)v0[0]; v[4 * i + 1] = (T)v0[1]; v[4 * i + 2] = (T)v1[0]; v[4 * i + 3] = (T)v1[1];
                }
            }
            return v;
        }
    };
};

}  // namespace spp

extern "C" int64_t spp_fp8_row_bytes(int32_t D) {
    SPP_CHECK(D >= 1 && D <= SPP_MX4_MAX_COLS, SPP_E_ARG, "spp_fp8_row_bytes: D = %d (1 .. %d)", D, SPP_MX4_MAX_COLS);
    return spp::fp8_bytes(D);
}

extern "C" int spp_fp8_quantize(spp_ctx* ctx, const void* d_x, int32_t type, int64_t n, const int64_t* d_n, int32_t D, int64_t ld,
                                void* d_rows, uint32_t flags) {
    return spp::quantize_rows<spp::Fp8Rows>("spp_fp8_quantize", SPP_T_MX4, ctx, d_x, type, n, d_n, D, ld, d_rows, flags);
}

extern "C" int spp_fp8_dequantize(spp_ctx* ctx, const void* d_rows, int64_t n, const int64_t* d_n, int32_t D, void* d_x, int32_t type,
                                  int64_t ld, uint32_t flags) {
    return spp::dequantize_rows<spp::Fp8Rows>("spp_fp8_dequantize", SPP_T_MX4, ctx, d_rows, n, d_n, D, d_x, type, ld, flags);
}
