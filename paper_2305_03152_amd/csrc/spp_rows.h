// Feature and hidden rows in few bits: what quantising rows of 16- or 32-bit floats and reading them back share, whatever the format.
//
// Both directions move each byte once and are bound by HBM.  A lane has 8 columns, so some lanes share a block and find its
// largest value with exchanges between neighbours; the lanes of a wavefront read and write side by side.  The conversion
// instructions take the scale and round as the formats ask.
//
// A format F says how many bytes of LDS a wavefront's rows need (lds), how many columns a block has, whether lanes behind a row's
// last column load nothing (skips), and
//   layout     where in a row its codes and scales are, and how many lanes share a block
//   put        eight columns' codes, and their block's scale, to their places in a row in LDS
//   scale_at   where in a row the scale of a column is
//   Codes      the codes of four or eight columns: fetch, and the values that they stand for under a scale
#pragma once

#include "spp_mx4.h"

namespace spp {

constexpr int kMxBlock = 256, kMxWaves = kMxBlock / kWave, kMxSlots = 4;
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
    int32_t        cb;           // bytes of a row's codes
    int32_t        share;        // lanes that share a block
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

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {           // over four lanes
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);      // lanes 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);               // lanes 2 3 0 1
    return v > o ? v : o;
}

// Eight columns of a block: their largest magnitude as bits of an fp32 (these order as the magnitudes do, NaN above infinity above
// the rest), and their codes under a scale.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
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
    __device__ __forceinline__ u32x2 codes8(float scale) const {     // E4M3
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        i16x2 c[2] = {{0, 0}, {0, 0}};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (__is_same(T, __bf16)) {
                c[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c[i], __builtin_bit_cast(bf16x2, w[2 * i]), scale, false);
                c[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c[i], __builtin_bit_cast(bf16x2, w[2 * i + 1]), scale, true);
            } else {
                c[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c[i], __builtin_bit_cast(f16x2, w[2 * i]), scale, false);
                c[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c[i], __builtin_bit_cast(f16x2, w[2 * i + 1]), scale, true);
            }
        }
        return u32x2{__builtin_bit_cast(uint32_t, c[0]), __builtin_bit_cast(uint32_t, c[1])};
    }
    __device__ __forceinline__ float at(int i) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        return (float)__builtin_bit_cast(T, (uint16_t)(w[i / 2] >> (16 * (i & 1))));
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
    __device__ __forceinline__ u32x2 codes8(float scale) const {
        i16x2 c = {0, 0}, d = {0, 0};
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, a[0], a[1], scale, false);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, a[2], a[3], scale, true);
        d = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(d, b[0], b[1], scale, false);
        d = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(d, b[2], b[3], scale, true);
        return u32x2{__builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
    }
    __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i] : b[i - 4]; }
};

// A wavefront's rows are put together in LDS, codes, scales and the zeros behind them, and go out as one run of 16-byte pieces.
template <class F, class T>
__global__ void __launch_bounds__(kMxBlock) quantize_rows_kernel(MxArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[kMxWaves][F::lds];
    const int64_t n = rows_of(a.n, a.d_n);
    uint8_t* mine = lds[threadIdx.x >> 6];
    const int l = lane_id(), all = a.tile * a.units;
    for (int i = l; i < F::lds / 16; i += kWave) reinterpret_cast<u32x4*>(mine)[i] = u32x4{0, 0, 0, 0};
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
            // the lanes of a block stay together: units are multiples of their number
#pragma unroll
            for (int k = 0; k < kMxSlots; ++k) {
                row[k] = slots.row[k]; piece[k] = slots.piece[k] + u0;
                if (u0 + k * kWave + l >= all || row[k] >= here) row[k] = -1;
                off[k] = row[k] < 0 ? 0 : row[k] * a.ld + (F::skips && 8 * piece[k] >= a.D ? 0 : 8 * piece[k]);
            }
            const int last = F::skips ? (a.D - 1) / 8 : a.units - 1;             // the last piece of a row that is loaded
            if ((r0 + here - 1) * a.ld + 8 * last <= behind) {          // all of the round can be read whole
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
            if (a.D & (F::columns - 1)) {
#pragma unroll
                for (int k = 0; k < kMxSlots; ++k) v[k].keep(a.D - 8 * piece[k]);
            }
#pragma unroll
            for (int k = 0; k < kMxSlots; ++k) {
                if (row[k] < 0) continue;
                F::put(v[k], a, mine + row[k] * a.rb, piece[k]);
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
template <class F, class T, bool Run>
__global__ void __launch_bounds__(kMxBlock) dequantize_rows_kernel(MxArgs a) {
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
            typename F::template Codes<VE> code[kMxSlots];
            uint32_t scale[kMxSlots];
#pragma unroll
            for (int k = 0; k < kMxSlots; ++k) {
                const bool there = u0 + k * kWave + l < all && slots.row[k] < here;
                const uint8_t* row = in + (there ? slots.row[k] : 0) * a.rb;
                const int piece = there ? slots.piece[k] + u0 : 0;
                code[k].fetch(row, piece);
                scale[k] = row[F::scale_at(a, piece * VE)];
            }
#pragma unroll
            for (int k = 0; k < kMxSlots; ++k) {
                if (u0 + k * kWave + l >= all || slots.row[k] >= here) continue;
                const float s = mx4_scale(scale[k]);
                const V v = code[k].template value<T>(s);
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

template <class F>
static int rows_args(const char* who, spp_ctx* ctx, const void* x, int32_t type, int64_t n, const int64_t* d_n, int32_t D, int64_t ld,
                    const void* rows, int per_lane, MxArgs& a) {
    SPP_CHECK(ctx, SPP_E_ARG, "%s: ctx is null", who);
    SPP_CHECK(is_type(type), SPP_E_ARG, "%s: element type %d", who, type);
    SPP_CHECK(D >= 1 && D <= SPP_MX4_MAX_COLS, SPP_E_ARG, "%s: D = %d (1 .. %d)", who, D, SPP_MX4_MAX_COLS);
    SPP_CHECK(n >= 0 && n <= 0x7FFFFFFFll && ld >= D, SPP_E_ARG, "%s: n = %lld, ld = %lld", who, (long long)n, (long long)ld);
    SPP_CHECK(n == 0 || (x && rows), SPP_E_ARG, "%s: null argument", who);
    SPP_CHECK((uintptr_t)x % type_bytes(type) == 0 && (uintptr_t)rows % 16 == 0, SPP_E_ARG,
              "%s: rows must be 16-byte aligned, values aligned to their type", who);
    a.x = x; a.rows = const_cast<void*>(rows); a.d_n = d_n; a.n = n; a.ld = ld; a.D = D;
    F::layout(a);
    a.units = per_lane ? (D + per_lane - 1) / per_lane : a.share * a.nb;
    a.magic = a.units > 1 ? (uint32_t)((0x100000000ull + a.units - 1) / a.units) : 0;
    a.tile = a.units < kMxSlots * kWave ? kMxSlots * kWave / a.units : 1;
    const uint64_t bits = (uintptr_t)x | (uint64_t)(ld * (int64_t)type_bytes(type));
    a.wide = bits % 16 == 0; a.even = bits % 4 == 0;
    return SPP_OK;
}
static unsigned rows_grid(const spp_ctx* ctx, const MxArgs& a) {
    const int64_t rounds = (a.n + a.tile - 1) / a.tile, groups = (rounds + kMxWaves - 1) / kMxWaves, most = (int64_t)ctx->num_cu * kMxGroups;
    return (unsigned)(groups < most ? groups : most);
}

template <class F>
static int quantize_rows(const char* who, int timer_index, spp_ctx* ctx, const void* d_x, int32_t type, int64_t n, const int64_t* d_n, int32_t D,
                         int64_t ld, void* d_rows, uint32_t flags) {
    MxArgs a;
    SPP_TRY(rows_args<F>(who, ctx, d_x, type, n, d_n, D, ld, d_rows, 0, a));
    if (n > 0) {
        SPP_HIP(hipSetDevice(ctx->device));
        ScopedTimer timer(ctx, timer_index, ctx->stream);
        const unsigned grid = rows_grid(ctx, a);
        if (type == SPP_F32) quantize_rows_kernel<F, float><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        else if (type == SPP_F16) quantize_rows_kernel<F, _Float16><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        else quantize_rows_kernel<F, __bf16><<<grid, kMxBlock, 0, ctx->stream>>>(a);
        SPP_HIP(hipGetLastError());
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}

template <class F>
static int dequantize_rows(const char* who, int timer_index, spp_ctx* ctx, const void* d_rows, int64_t n, const int64_t* d_n, int32_t D, void* d_x,
                           int32_t type, int64_t ld, uint32_t flags) {
    MxArgs a;
    SPP_TRY(rows_args<F>(who, ctx, d_x, type, n, d_n, D, ld, d_rows, type == SPP_F32 ? 4 : 8, a));
    if (n > 0) {
        SPP_HIP(hipSetDevice(ctx->device));
        ScopedTimer timer(ctx, timer_index, ctx->stream);
        const unsigned grid = rows_grid(ctx, a);
        const bool run = !a.wide && (ld == D || n == 1);
        auto launch = [&](auto kernel) { kernel<<<grid, kMxBlock, 0, ctx->stream>>>(a); };
        if (type == SPP_F32) run ? launch(dequantize_rows_kernel<F, float, true>) : launch(dequantize_rows_kernel<F, float, false>);
        else if (type == SPP_F16) run ? launch(dequantize_rows_kernel<F, _Float16, true>) : launch(dequantize_rows_kernel<F, _Float16, false>);
        else run ? launch(dequantize_rows_kernel<F, __bf16, true>) : launch(dequantize_rows_kernel<F, __bf16, false>);
        SPP_HIP(hipGetLastError());
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}

}  // namespace spp
