// Feature rows in MXFP4: quantisation of rows of 16- or 32-bit floats, and back.
//
//   block of 32 columns, a = max |x|:  e = max(floor(log2 a) - 2, -127),  code = nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} to |x| / 2^e,
//   ties to the even code, 6 for what lies above; the scale byte is e + 127.  A block with a NaN or an infinity is NaN as a whole.
//
// Four lanes share a block.  800k rows of 768 fp16: 273 us, and 274 back to bf16, 5.7 TB/s each; 2M rows of 100 in fp32 166 and 169, in
// fp16, 200-byte rows, 107 and 79.
#include "spp_rows.h"

namespace spp {

struct Mx4Rows {
    static constexpr int lds = 2304, columns = 32;
    static constexpr bool skips = false;
    static void layout(MxArgs& a) { a.nb = mx4_blocks(a.D); a.rb = mx4_bytes(a.D); a.cb = 16 * a.nb; a.share = 4; }
    static __device__ __forceinline__ int scale_at(const MxArgs& a, int column) { return 16 * a.nb + column / 32; }
    template <class T>
    static __device__ __forceinline__ void put(const Eight<T>& v, const MxArgs& a, uint8_t* out, int piece) {
        const uint32_t top = quad_max(v.top());
        const bool bad = top >= 0x7F800000u;
        int e = (int)(top >> 23) - 2;                                // the scale's byte; subnormal and zero blocks have the least
        e = e < 0 ? 0 : e;
        const uint32_t code = v.codes(mx4_scale((uint32_t)e));
        *reinterpret_cast<uint32_t*>(out + 4 * piece) = bad ? 0u : code;
        if ((piece & 3) == 0) out[16 * a.nb + (piece >> 2)] = bad ? (uint8_t)255 : (uint8_t)e;
    }
    template <int VE>
    struct Codes {
        uint32_t code;
        __device__ __forceinline__ void fetch(const uint8_t* row, int piece) {
            code = VE == 8 ? reinterpret_cast<const uint32_t*>(row)[piece] : reinterpret_cast<const uint16_t*>(row)[piece];
        }
        template <class T>
        __device__ __forceinline__ auto value(float s) const {
            typedef T V __attribute__((ext_vector_type(VE)));
            V v;
            if constexpr (__is_same(T, __bf16)) {
                const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 1),
                             v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 3);
                v = V{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
            } else {
                // by way of fp32, which holds every value, and rounded to 16 bits from there
                typedef float f32x2 __attribute__((ext_vector_type(2)));
                const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1);
                v[0] = (T)v0[0]; v[1] = (T)v0[1]; v[2] = (T)v1[0]; v[3] = (T)v1[1];
                if constexpr (VE == 8) {
                    const f32x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3);
                    v[4] = (T)v2[0]; v[5] = (T)v2[1]; v[6] = (T)v3[0]; v[7] = (T)v3[1];
                }
            }
            return v;
        }
    };
};

}  // namespace spp

extern "C" int64_t spp_mx4_row_bytes(int32_t D) {
    SPP_CHECK(D >= 1 && D <= SPP_MX4_MAX_COLS, SPP_E_ARG, "spp_mx4_row_bytes: D = %d (1 .. %d)", D, SPP_MX4_MAX_COLS);
    return spp::mx4_bytes(D);
}

extern "C" int spp_mx4_quantize(spp_ctx* ctx, const void* d_x, int32_t type, int64_t n, const int64_t* d_n, int32_t D, int64_t ld,
                                void* d_rows, uint32_t flags) {
    return spp::quantize_rows<spp::Mx4Rows>("spp_mx4_quantize", SPP_T_MX4, ctx, d_x, type, n, d_n, D, ld, d_rows, flags);
}

extern "C" int spp_mx4_dequantize(spp_ctx* ctx, const void* d_rows, int64_t n, const int64_t* d_n, int32_t D, void* d_x, int32_t type,
                                  int64_t ld, uint32_t flags) {
    return spp::dequantize_rows<spp::Mx4Rows>("spp_mx4_dequantize", SPP_T_MX4, ctx, d_rows, n, d_n, D, d_x, type, ld, flags);
}
