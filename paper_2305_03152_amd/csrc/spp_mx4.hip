// Feature rows in MXFP4: quantisation of rows of 16- or 32-bit floats, and back.
//
//   block of 32 columns, a = max |x|:  e = max(floor(log2 a) - 2, -127),  code = nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} to |x| / 2^e,
//   ties to the even code, 6 for what lies above; the scale byte is e + 127.  A block with a NaN or an infinity is NaN as a whole.
//
// Both directions move each byte once and are bound by HBM.  A lane has 8 columns, so four lanes share a block and find its
// largest value with two exchanges between neighbours; the lanes of a wavefront read and write side by side.  The conversion
// instruction takes the scale and rounds as the format asks.  800k rows of 768 fp16: 273 us, and 274 back to bf16, 5.7 TB/s each; 2M rows of
// 100 in fp32 166 and 169, in fp16, 200-byte rows, 107 and 79.
#include "spp_mx4.h"

namespace spp {

constexpr int kMxBlock = 256, kMxWaves = kMxBlock / kWave, kMxSlots = 4, kMxLds = 2304;
constexpr int kMxGroups = 256;          // workgroups per CU: one or a few rounds each.  800k rows of 768 fp16: quantised in 305, 273 us with 8, 256; back in 332, 274

struct MxArgs {
    const void*    x;
    void*          rows;
    const int64_t* d_n;
    int64_t        n, ld;        // ld: elements from a row of x to the next
    int32_t        D, nb, rb;
    int32_t        units;        // lanes per row
    uint32_t       magic;        // ceil(2^32 / units)
    int32_t        tile;         // rows of a wavefront's round: as many as 256 lanes have whole, or one
    int32_t        wide, even;   // rows of x begin at multiples of 16 bytes, of 4
};

// Which row and which piece of it each of the lane's slots of a round is; the same in every round.
struct Slots {
    int row[kMxSlots], piece[kMxSlots];
    __device__ __forceinline__ explicit Slots(const MxArgs& a) {
#pragma unroll
        for (int k = 0; k < kMxSlots; ++k) {
            const uint32_t u = lane_id() + k * kWave;
            row[k] = a.units > 1 ? (int)__umulhi(u, a.magic) : (int)u;
            piece[k] = (int)u - row[k] * a.units;
        }
    }
};

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {           // over the four lanes of a block
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);      // lanes 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);               // lanes 2 3 0 1
    return v > o ? v : o;
}

// Eight columns of a block: their largest magnitude as bits of an fp32 (these order as the magnitudes do, NaN above infinity above
// the rest), and their codes under a scale.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <class T> struct Eight {
    u32x4 v;
    static constexpr uint32_t kOne = sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu;
    __device__ __forceinline__ void load(const T* p) { v = reinterpret_cast<const Loose<u32x4>*>(p)->v; }
    __device__ __forceinline__ void load_wide(const T* p) { v = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ void load_some(const T* p, int have) {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < have ? p[i] : (T)0.0f;
        v = __builtin_bit_cast(u32x4, t);
    }
    __device__ __forceinline__ void keep(int have) {                 // the columns behind the row's last are zeros
        const int bits = have * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int left = bits - 32 * i;
            v[i] = left >= 32 ? v[i] : left <= 0 ? 0u : v[i] & 0xFFFFu;
        }
    }
    __device__ __forceinline__ uint32_t top() const {
        u16x2 m = __builtin_bit_cast(u16x2, v[0] & kOne);
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & kOne));
        const uint16_t t = m[0] > m[1] ? m[0] : m[1];
        return __float_as_uint((float)__builtin_bit_cast(T, t)) & 0x7FFFFFFFu;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const {
        // (a bit_cast of a vector's element itself takes the vector's first)
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t c = 0;
        if constexpr (__is_same(T, __bf16)) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
        } else {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w[0]), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w[1]), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w[2]), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w[3]), scale, 3);
        }
        return c;
    }
};
template <> struct Eight<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const Loose<f32x4>*>(p)->v; b = reinterpret_cast<const Loose<f32x4>*>(p + 4)->v; }
    __device__ __forceinline__ void load_wide(const float* p) { a = *reinterpret_cast<const f32x4*>(p); b = *reinterpret_cast<const f32x4*>(p + 4); }
    __device__ __forceinline__ void load_some(const float* p, int have) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i] = i < have ? p[i] : 0.0f; b[i] = 4 + i < have ? p[4 + i] : 0.0f; }
    }
    __device__ __forceinline__ void keep(int have) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i] = i < have ? a[i] : 0.0f; b[i] = 4 + i < have ? b[i] : 0.0f; }
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = __float_as_uint(a[i]) & 0x7FFFFFFFu, y = __float_as_uint(b[i]) & 0x7FFFFFFFu;
            t = t > x ? t : x;
            t = t > y ? t : y;
        }
        return t;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[0], a[1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[2], a[3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, b[0], b[1], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, b[2], b[3], scale, 3);
        return c;
    }
};

// A wavefront's rows are put together in LDS, codes, scales and the zeros behind them, and go out as one run of 16-byte pieces.
template <class T>
__global__ void __launch_bounds__(kMxBlock) mx4_quantize_kernel(MxArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[kMxWaves][kMxLds];
    const int64_t n = rows_of(a.n, a.d_n);
    uint8_t* mine = lds[threadIdx.x >> 6];
    const int l = lane_id(), all = a.tile * a.units;
    for (int i = l; i < kMxLds / 16; i += kWave) reinterpret_cast<u32x4*>(mine)[i] = u32x4{0, 0, 0, 0};
    wave_lds_order();
    const Slots slots(a);
    const int64_t behind = (n - 1) * a.ld + a.D - 8;                 // the last element that eight can be read from
    const Share share((n + a.tile - 1) / a.tile, kMxWaves);
    for (int64_t t = share.at; t < share.end; t += share.step) {
        const int64_t r0 = t * a.tile;
        const int here = n - r0 < a.tile ? (int)(n - r0) : a.tile;
        const T* x = static_cast<const T*>(a.x) + r0 * a.ld;
        for (int u0 = 0; u0 < all; u0 += kMxSlots * kWave) {         // one round but for rows of more than 2048 columns
            Eight<T> v[kMxSlots];
            int row[kMxSlots], piece[kMxSlots];
            int64_t off[kMxSlots];
            // the four lanes of a block stay together: units are multiples of four
#pragma unroll
            for (int k = 0; k < kMxSlots; ++k) {
                row[k] = slots.row[k]; piece[k] = slots.piece[k] + u0;
                if (u0 + k * kWave + l >= all || row[k] >= here) row[k] = -1;
                off[k] = row[k] < 0 ? 0 : row[k] * a.ld + 8 * piece[k];
            }
            if ((r0 + here - 1) * a.ld + 8 * (a.units - 1) <= behind) {          // all of the round can be read whole
                if (a.wide)
#pragma unroll
                    for (int k = 0; k < kMxSlots; ++k) v[k].load_wide(x + off[k]);
                else
#pragma unroll
                    for (int k = 0; k < kMxSlots; ++k) v[k].load(x + off[k]);
            } else {
#pragma unroll
                for (int k = 0; k < kMxSlots; ++k) v[k].load_some(x + off[k], a.D - 8 * piece[k]);
            }
            if (a.D & 31) {
#pragma unroll
                for (int k = 0; k < kMxSlots; ++k) v[k].keep(a.D - 8 * piece[k]);
            }
#pragma unroll
            for (int k = 0; k < kMxSlots; ++k) {
                if (row[k] < 0) continue;
                const uint32_t top = quad_max(v[k].top());
                const bool bad = top >= 0x7F800000u;
                int e = (int)(top >> 23) - 2;                        // the scale's byte; subnormal and zero blocks have the least
                e = e < 0 ? 0 : e;
                const uint32_t code = v[k].codes(mx4_scale((uint32_t)e));
                uint8_t* out = mine + row[k] * a.rb;
                *reinterpret_cast<uint32_t*>(out + 4 * piece[k]) = bad ? 0u : code;
                if ((piece[k] & 3) == 0) out[16 * a.nb + (piece[k] >> 2)] = bad ? (uint8_t)255 : (uint8_t)e;
            }
        }
        wave_lds_order();
        u32x4* out = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.rows) + r0 * a.rb);
        for (int i = l; i < here * (a.rb / 16); i += kWave) __builtin_nontemporal_store(reinterpret_cast<const u32x4*>(mine)[i], &out[i]);
        wave_lds_order();
    }
}

// A lane has 16 bytes of the result: eight columns of 16 bits, four of 32.  Rows that follow each other without a gap but not at
// multiples of 16 bytes (Run) are put together in LDS and go out as one run of 16-byte pieces, its ends by element.
template <class T, bool Run>
__global__ void __launch_bounds__(kMxBlock) mx4_dequantize_kernel(MxArgs a) {
    constexpr int VE = 16 / (int)sizeof(T), kRun = kMxSlots * kWave * 16 + 16;
    typedef T V __attribute__((ext_vector_type(VE)));
    __shared__ __attribute__((aligned(16))) uint8_t lds[Run ? kMxWaves : 1][Run ? kRun : 16];
    uint8_t* mine = lds[Run ? threadIdx.x >> 6 : 0];
    const int64_t n = rows_of(a.n, a.d_n);
    const int all = a.tile * a.units, l = lane_id();
    const Slots slots(a);
    const Share share((n + a.tile - 1) / a.tile, kMxWaves);
    for (int64_t t = share.at; t < share.end; t += share.step) {
        const int64_t r0 = t * a.tile;
        const int here = n - r0 < a.tile ? (int)(n - r0) : a.tile;
        const uint8_t* in = static_cast<const uint8_t*>(a.rows) + r0 * a.rb;
        T* x = static_cast<T*>(const_cast<void*>(a.x)) + r0 * a.ld;
        for (int u0 = 0; u0 < all; u0 += kMxSlots * kWave) {
            // one run a round: rows of more than 256 pieces in parts
            char* start = reinterpret_cast<char*>(x + VE * u0);
            const int head = (int)((uintptr_t)start & 15);
            uint32_t code[kMxSlots], scale[kMxSlots];
#pragma unroll
            for (int k = 0; k < kMxSlots; ++k) {
                const bool there = u0 + k * kWave + l < all && slots.row[k] < here;
                const uint8_t* row = in + (there ? slots.row[k] : 0) * a.rb;
                const int piece = there ? slots.piece[k] + u0 : 0;
                code[k] = VE == 8 ? reinterpret_cast<const uint32_t*>(row)[piece] : reinterpret_cast<const uint16_t*>(row)[piece];
                scale[k] = row[16 * a.nb + piece * VE / 32];
            }
#pragma unroll
            for (int k = 0; k < kMxSlots; ++k) {
                if (u0 + k * kWave + l >= all || slots.row[k] >= here) continue;
                const float s = mx4_scale(scale[k]);
                V v;
                if constexpr (__is_same(T, __bf16)) {
                    const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[k], s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[k], s, 1),
                                 v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[k], s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[k], s, 3);
                    v = V{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
                } else {
                    // by way of fp32, which holds every value, and rounded to 16 bits from there
                    typedef float f32x2 __attribute__((ext_vector_type(2)));
                    const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], s, 1);
                    v[0] = (T)v0[0]; v[1] = (T)v0[1]; v[2] = (T)v1[0]; v[3] = (T)v1[1];
                    if constexpr (VE == 8) {
                        const f32x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], s, 3);
                        v[4] = (T)v2[0]; v[5] = (T)v2[1]; v[6] = (T)v3[0]; v[7] = (T)v3[1];
                    }
                }
                const int piece = slots.piece[k] + u0, have = a.D - VE * piece;
                if constexpr (Run) {
                    uint8_t* out = mine + head + (slots.row[k] * a.D + VE * slots.piece[k]) * (int)sizeof(T);
                    if (have < VE) {                                 // the next row lies behind
#pragma unroll
                        for (int i = 0; i < VE; ++i)
                            if (i < have) reinterpret_cast<T*>(out)[i] = v[i];
                    } else if (a.even) {                             // an LDS write that is not aligned to its size takes many times one that is
                        struct Words { uint32_t w[4]; } w = __builtin_bit_cast(Words, v);
#pragma unroll
                        for (int i = 0; i < 4; ++i) reinterpret_cast<volatile uint32_t*>(out)[i] = w.w[i];
                    } else {
                        struct Halves { uint16_t w[8]; } w = __builtin_bit_cast(Halves, v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) reinterpret_cast<volatile uint16_t*>(out)[i] = w.w[i];
                    }
                } else {
                    T* out = x + slots.row[k] * a.ld + VE * piece;
                    if (have >= VE) {
                        if (a.wide) __builtin_nontemporal_store(v, reinterpret_cast<V*>(out));
                        else reinterpret_cast<Loose<V>*>(out)->v = v;
                    } else
#pragma unroll
                        for (int i = 0; i < VE; ++i)
                            if (i < have) out[i] = v[i];
                }
            }
            if constexpr (Run) {
                wave_lds_order();
                const int columns = a.tile > 1 || a.D - VE * u0 < VE * kMxSlots * kWave ? a.D - VE * u0 : VE * kMxSlots * kWave;
                const int len = ((here - 1) * a.D + columns) * (int)sizeof(T), end = (head + len) / 16;
                u32x4* to = reinterpret_cast<u32x4*>(start - head);
                for (int k = (head ? 1 : 0) + l; k < end; k += kWave) __builtin_nontemporal_store(reinterpret_cast<const u32x4*>(mine)[k], &to[k]);
                // lanes 0..7: what lies before the first whole piece; 8..15: behind the last; a run inside one piece that it begins, too
                const int kk = l & 7, off = (l < 8 ? head : 16 * end) + kk * (int)sizeof(T);
                if (l < 8 ? head && off < 16 && off < head + len : l < 16 && off < head + len && (end > 0 || !head))
                    *reinterpret_cast<T*>(start - head + off) = *reinterpret_cast<const T*>(mine + off);
                wave_lds_order();
            }
        }
    }
}

static int mx4_args(const char* who, spp_ctx* ctx, const void* x, int32_t type, int64_t n, const int64_t* d_n, int32_t D, int64_t ld,
                    const void* rows, int per_lane, MxArgs& a) {
    SPP_CHECK(ctx, SPP_E_ARG, "%s: ctx is null", who);
    SPP_CHECK(is_type(type), SPP_E_ARG, "%s: element type %d", who, type);
    SPP_CHECK(D >= 1 && D <= SPP_MX4_MAX_COLS, SPP_E_ARG, "%s: D = %d (1 .. %d)", who, D, SPP_MX4_MAX_COLS);
    SPP_CHECK(n >= 0 && n <= 0x7FFFFFFFll && ld >= D, SPP_E_ARG, "%s: n = %lld, ld = %lld", who, (long long)n, (long long)ld);
    SPP_CHECK(n == 0 || (x && rows), SPP_E_ARG, "%s: null argument", who);
    SPP_CHECK((uintptr_t)x % type_bytes(type) == 0 && (uintptr_t)rows % 16 == 0, SPP_E_ARG,
              "%s: rows must be 16-byte aligned, values aligned to their type", who);
    a.x = x; a.rows = const_cast<void*>(rows); a.d_n = d_n; a.n = n; a.ld = ld; a.D = D;
    a.nb = mx4_blocks(D); a.rb = mx4_bytes(D);
    a.units = per_lane ? (D + per_lane - 1) / per_lane : 4 * a.nb;
    a.magic = a.units > 1 ? (uint32_t)((0x100000000ull + a.units - 1) / a.units) : 0;
    a.tile = a.units < kMxSlots * kWave ? kMxSlots * kWave / a.units : 1;
    const uint64_t bits = (uintptr_t)x | (uint64_t)(ld * (int64_t)type_bytes(type));
    a.wide = bits % 16 == 0; a.even = bits % 4 == 0;
    return SPP_OK;
}
static unsigned mx4_grid(const spp_ctx* ctx, const MxArgs& a) {
    const int64_t rounds = (a.n + a.tile - 1) / a.tile, groups = (rounds + kMxWaves - 1) / kMxWaves, most = (int64_t)ctx->num_cu * kMxGroups;
    return (unsigned)(groups < most ? groups : most);
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
    SPP_TRY(mx4_args("spp_mx4_quantize", ctx, d_x, type, n, d_n, D, ld, d_rows, 0, a));
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
    SPP_TRY(mx4_args("spp_mx4_dequantize", ctx, d_x, type, n, d_n, D, ld, d_rows, type == SPP_F32 ? 4 : 8, a));
    if (n > 0) {
        SPP_HIP(hipSetDevice(ctx->device));
        ScopedTimer timer(ctx, SPP_T_MX4, ctx->stream);
        const unsigned grid = mx4_grid(ctx, a);
        const bool run = !a.wide && (ld == D || n == 1);
        auto launch = [&](auto kernel) { kernel<<<grid, kMxBlock, 0, ctx->stream>>>(a); };
        if (type == SPP_F32) run ? launch(mx4_dequantize_kernel<float, true>) : launch(mx4_dequantize_kernel<float, false>);
        else if (type == SPP_F16) run ? launch(mx4_dequantize_kernel<_Float16, true>) : launch(mx4_dequantize_kernel<_Float16, false>);
        else run ? launch(mx4_dequantize_kernel<__bf16, true>) : launch(mx4_dequantize_kernel<__bf16, false>);
        SPP_HIP(hipGetLastError());
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}
