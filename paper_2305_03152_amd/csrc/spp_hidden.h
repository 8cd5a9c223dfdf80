// The layers that read hidden rows in 8 bits, and the backward pass of the gated one, over the lists of the product:
//
//   product      Y_j = X_j W[g_j]^T                                 X_j [n_j, D], W[g] [H, D] in 8 bits
//   gated        Y_j = act(X_j Wg[g_j]^T) * (X_j Wu[g_j]^T)         W[g] = Wg, then Wu, H rows each
//   its gradient [dY_j * u * act'(g) | dY_j * act(g)]               g and u formed again from X_j and W[g_j], as in the forward pass
//
// Codes are E4M3 and scales powers of two: a code under a scale is exact in bf16, so the values are decoded in registers and multiplied by
// the bf16 instruction: products are exact, sums fp32, whatever the type of the result.  The instruction for 8-bit floats would take the
// codes and the scales themselves, at twice the rate, but it adds the products of eight neighbouring columns after cutting each off at
// 2^-13 of the power of two of the largest (measured: beside 2^16 an addend of 2^3 counts and one of 2^2 does not): where large terms cancel
// each other, the small ones, which are then the result, are lost.  The activation is computed in fp32, and what is written is rounded once.
#pragma once

#include "spp_fp8.h"
#include "spp_rows_out.h"

namespace spp {

enum HiddenMode { kProduct, kGated, kGatedGrad };

struct HiddenArgs {
    RowTable       t;
    void*          dp[kRowLists];        // gradient of the gated layer: where each list's goes, [n_j, 2H]
    int64_t        dp_ld[kRowLists];
    const uint8_t* w;
    int32_t        D, H, rb, cb, steps;  // steps of 128 columns
    int32_t        act;
    // the form that holds W in LDS
    int32_t        fill;         // workgroups that few rows are dealt out to
    int32_t        w_lds;        // bytes of W; behind them, per wavefront, room for rows on their way:
    int32_t        out_lds;      // bytes
    // the form that holds W in registers
    int32_t        blocks;       // workgroups that share a row's columns
    int32_t        shares;       // and the rows of an XCD; 0: few rows, dealt out to all
};

// Lane j has list j's group: fetched byte by byte where it is needed, it would make the wavefront wait for all that it has under way.
__device__ __forceinline__ int group_of_lane(const RowTable& t) { return lane_id() < t.n_lists ? t.group[lane_id()] : 0; }

// ---- operands -------------------------------------------------------------------------------------

// A lane's 32 codes of a step of 128 columns, 16 from 16 q and 16 from 64 + 16 q on, q being its quarter of the wavefront, and the
// scales of four steps, a byte each.
struct Operand {
    u32x4 lo, hi;
    uint32_t scale;
};
// The values of eight of its codes.
__device__ __forceinline__ bf16x8 eight_of(uint32_t a, uint32_t b, float s) {
    const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true),
                 v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false), v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true);
    return bf16x8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
}
struct Decoded { bf16x8 v[4]; };
template <int Byte>
__device__ __forceinline__ Decoded decode(const Operand& o) {
    const float s = mx4_scale((o.scale >> (8 * Byte)) & 255u);
    return Decoded{{eight_of(o.lo.x, o.lo.y, s), eight_of(o.lo.z, o.lo.w, s), eight_of(o.hi.x, o.hi.y, s), eight_of(o.hi.z, o.hi.w, s)}};
}
// acc[c][f] += X[c] W[f]^T over a step, rows of X as rows of the result.
template <int Byte, int RN, int FN>
__device__ __forceinline__ void multiply(f32x4 (&acc)[RN][FN], const Operand (&x)[RN], const Operand (&w)[FN]) {
    Decoded xd[RN];
#pragma unroll
    for (int c = 0; c < RN; ++c) xd[c] = decode<Byte>(x[c]);
#pragma unroll
    for (int f = 0; f < FN; ++f) {
        const Decoded wd = decode<Byte>(w[f]);
#pragma unroll
        for (int c = 0; c < RN; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[c][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xd[c].v[j], wd.v[j], acc[c][f], 0, 0, 0);
    }
}

// ---- activations ----------------------------------------------------------------------------------

// 1 / (1 + exp(-g)) and 1 / (1 + exp(g)), from exp(-|g|), which is at most 1: neither loses its small values.
__device__ __forceinline__ void sigmoids(float g, float& s, float& r) {
    const float t = __builtin_amdgcn_exp2f(__builtin_fabsf(g) * -1.44269504f);
    const float p = __builtin_amdgcn_rcpf(1.0f + t), q = t * p;
    s = g >= 0.0f ? p : q;
    r = g >= 0.0f ? q : p;
}
// The normal distribution function of g, and exp(-g^2 / 2).  Below -x, x = |g|, it is exp(-x^2 / 2) R(x) with R falling from 1/2 to
// about 0.4 / x: t P(t) with t = 1 / (1 + 0.345 x) and P of degree 8, fitted here for the least relative error over x from 0 to 14; with the
// constants as they stand here, in fp32, 6.6e-8 (half a step of fp32 is 6.0e-8); behind that the exponential is 0.  In fp32 2^-23 (3 + 0.5 x^2) off,
// relative (the exponential's argument), at both ends.  The library's erfc takes some four times as long.
__device__ __forceinline__ float normal(float g, float& e) {
    const float x = __builtin_fabsf(g);
    e = __builtin_amdgcn_exp2f(x * x * -0.72134752f);
    const float t = __builtin_amdgcn_rcpf(__fmaf_rn(0.345f, x, 1.0f));
    float p = -0.028387917205691338f;
    p = __fmaf_rn(p, t, 0.14530695974826813f);
    p = __fmaf_rn(p, t, -0.2712171971797943f);
    p = __fmaf_rn(p, t, 0.18723931908607483f);
    p = __fmaf_rn(p, t, -0.03762628510594368f);
    p = __fmaf_rn(p, t, 0.11180825531482697f);
    p = __fmaf_rn(p, t, 0.11723647266626358f);
    p = __fmaf_rn(p, t, 0.1380210965871811f);
    p = __fmaf_rn(p, t, 0.137619286775589f);
    const float below = e * (t * p);
    return g >= 0.0f ? 1.0f - below : below;
}
template <int Act> __device__ __forceinline__ float activate(float g) {
    if constexpr (Act == SPP_GELU) {
        float e;
        return g * normal(g, e);
    } else if constexpr (Act == SPP_SILU) {
        return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));       // an infinite exponential leaves 0
    } else {
        float s, r;
        sigmoids(g, s, r);
        return s;
    }
}
// act(g) and act'(g)
template <int Act> __device__ __forceinline__ void activate_both(float g, float& f, float& d) {
    if constexpr (Act == SPP_GELU) {
        float e;
        const float p = normal(g, e);
        f = g * p;
        d = __fmaf_rn(g, e * 0.39894228f, p);
    } else {
        float s, r;
        sigmoids(g, s, r);
        f = Act == SPP_SILU ? g * s : s;
        d = Act == SPP_SILU ? s * __fmaf_rn(g, r, 1.0f) : s * r;
    }
}
// The activation is the same for the whole call: a branch around a tile's worth of work.
template <class Use> __device__ __forceinline__ void with_activation(int act, Use use) {
    if (act == SPP_SILU) use(std::integral_constant<int, SPP_SILU>());
    else if (act == SPP_GELU) use(std::integral_constant<int, SPP_GELU>());
    else use(std::integral_constant<int, SPP_SIGMOID>());
}

// Columns h .. h+N-1 of rows y[0..3], of which `have` are there: read, others as zeros, and written.  `wide`: N are aligned.
template <class T, int N>
__device__ __forceinline__ void get_columns(const T* y, int64_t ld, int have, int h, int H, bool wide, f32x4 (&v)[N]) {
    typedef T V __attribute__((ext_vector_type(N)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        V x;
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = (T)0.0f;
        const T* from = y + i * ld + h;
        if (i < have) {
            if (wide && h + N <= H) x = *reinterpret_cast<const V*>(from);
            else if (h + N <= H) x = reinterpret_cast<const Loose<V>*>(from)->v;
            else
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (h + k < H) x[k] = from[k];
        }
#pragma unroll
        for (int k = 0; k < N; ++k) v[k][i] = (float)x[k];
    }
}
template <class T, int N>
__device__ __forceinline__ void put_columns(T* y, int64_t ld, int have, int h, int H, bool wide, const f32x4 (&v)[N]) {
    typedef T V __attribute__((ext_vector_type(N)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        V x;
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = (T)v[k][i];
        T* out = y + i * ld + h;
        if (i >= have) continue;
        if (wide && h + N <= H) *reinterpret_cast<V*>(out) = x;
        else if (h + N <= H) reinterpret_cast<Loose<V>*>(out)->v = x;
        else
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (h + k < H) out[k] = x[k];
    }
}

// What columns of the two factors become: of the gated layer Y, in `one`; of its gradient dG and dU, in `one` and `two`.
template <int Mode, int N>
__device__ __forceinline__ void combine(int act, f32x4 (&one)[N], f32x4 (&two)[N], const f32x4 (&dy)[N]) {
    if constexpr (Mode == kGated) {
        with_activation(act, [&](auto kind) {
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) one[k][i] = activate<decltype(kind)::value>(one[k][i]) * two[k][i];
        });
    } else if constexpr (Mode == kGatedGrad) {
        with_activation(act, [&](auto kind) {
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float f, d;
                    activate_both<decltype(kind)::value>(one[k][i], f, d);
                    one[k][i] = dy[k][i] * two[k][i] * d;
                    two[k][i] = dy[k][i] * f;
                }
        });
    }
}

// A tile of a matrix of results by way of a buffer (rows_buffer) that begins with its first row: 16 RN rows, of which `here` are there, and of
// each N columns from h0 + N m on.
// Whole vectors where all begin at multiples of four bytes, which is all that the instructions ask for; the last columns of a row where they
// are no whole vector, and 16-bit matrices at odd places, go element by element (1M rows 172 -> 86, every column by element: gated layer in
// fp32 212 us, its gradient 477; so 174 and 360).  All of it is branches that a whole wavefront takes: where a kernel's values fill the
// registers the compiler (of ROCm 7.2) has copied some of them at the end of a masked piece of code before it restored the mask, and the
// lanes that were masked out lost theirs.
template <class T, int RN, int N, bool Whole = false>        // Whole: the caller knows that all are whole vectors
struct Tile {
    typedef T V __attribute__((ext_vector_type(N)));
    __amdgpu_buffer_rsrc_t at;
    uint32_t step;               // bytes from a row to the next
    int      h0, h, H;
    int      single;             // columns from this one on go element by element
    int      last;               // of the tile's
    uint32_t first;              // the lane's first element
    // `front`: columns of the matrix before these `columns`; a row has `all`
    __device__ __forceinline__ Tile(const T* y, int64_t ld, int64_t r0, int here, int h0, int front, int columns, int all) {
        step = (uint32_t)ld * (uint32_t)sizeof(T);
        at = rows_buffer(y + r0 * ld, (uint32_t)(here - 1) * step + (uint32_t)all * (uint32_t)sizeof(T));
        h = h0 + N * (lane_id() & 15);
        this->h0 = h0;
        H = columns;
        const bool vectors = sizeof(T) == 4 || N == 1 || ((uint32_t)(uintptr_t)y | step | (uint32_t)(front * (int)sizeof(T))) % 4 == 0;
        single = Whole ? columns : vectors ? columns / N * N : 0;
        last = h0 + 16 * N < columns ? h0 + 16 * N : columns;
        first = 4 * (uint32_t)(lane_id() >> 4) * step + (uint32_t)(front + h) * (uint32_t)sizeof(T);
    }
    template <class Use> __device__ __forceinline__ void each(Use use) const {
#pragma unroll
        for (int c = 0; c < RN; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) use(c, i, (uint32_t)(16 * c + i) * step);
    }
    // v(c, n): column n of the lane's rows of the c-th sixteen
    template <int Kind = 0, class Get> __device__ __forceinline__ void put(Get v) const {
        if (Whole || single > h0) {
            const uint32_t from = h < single ? first : kNowhere;
            each([&](int c, int i, uint32_t row) {
                V x;
#pragma unroll
                for (int n = 0; n < N; ++n) x[n] = (T)v(c, n)[i];
                buffer_store<Kind>(x, at, from + row);
            });
        }
        if (!Whole && single < last) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const uint32_t from = h >= single && h + n < H ? first + n * (uint32_t)sizeof(T) : kNowhere;
                each([&](int c, int i, uint32_t row) { buffer_store<Kind>((T)v(c, n)[i], at, from + row); });
            }
        }
    }
    // Asked for, and the values of what came: where the compiler may not move code, the first use is what waits.
    __device__ __forceinline__ void ask(V (&x)[RN][4]) const {
        if (Whole || single >= last) {
            const uint32_t from = h < single ? first : kNowhere;
            each([&](int c, int i, uint32_t row) { x[c][i] = buffer_load<V>(at, from + row); });
        } else {
            each([&](int c, int i, uint32_t row) {
                struct { T v[N]; } e;
#pragma unroll
                for (int n = 0; n < N; ++n) e.v[n] = buffer_load<T>(at, (h + n < H ? first + n * (uint32_t)sizeof(T) : kNowhere) + row);
                x[c][i] = __builtin_bit_cast(V, e);
            });
        }
    }
    static __device__ __forceinline__ void values(const V (&x)[4], f32x4 (&v)[N]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n][i] = (float)x[i][n];
    }
};
// Whether a tile's rows span what a buffer can.
static inline bool spans(int64_t ld, int bytes, int rows) { return (rows + 1) * ld * bytes < (1ll << 31); }

// A list's matrices of results: Y, read or written, and dP.  `row`: of the list; `have`: rows that are there from it on.
template <class T, int Mode>
struct Results {
    T*      y;
    T*      p;
    int64_t ld, pld;
    bool    wide, pwide;
    __device__ __forceinline__ Results(const HiddenArgs& a, int list) {
        y = static_cast<T*>(a.t.y[list]);
        ld = a.t.ld[list];
        wide = ((uintptr_t)y | (uint64_t)(ld * (int64_t)sizeof(T))) % (4 * sizeof(T)) == 0;
        if constexpr (Mode == kGatedGrad) {
            p = static_cast<T*>(a.dp[list]);
            pld = a.dp_ld[list];
            pwide = ((uintptr_t)p | (uint64_t)(pld * (int64_t)sizeof(T)) | (uint64_t)(a.H * (int)sizeof(T))) % (4 * sizeof(T)) == 0;
        }
    }
    template <int N>
    __device__ __forceinline__ void get(const HiddenArgs& a, int64_t row, int have, int h, f32x4 (&v)[N]) const {
        get_columns<T, N>(y + row * ld, ld, have, h, a.H, wide, v);
    }
    template <int N>
    __device__ __forceinline__ void put(const HiddenArgs& a, int64_t row, int have, int h, const f32x4 (&v)[N]) const {
        if constexpr (Mode == kGatedGrad) put_columns<T, N>(p + row * pld, pld, have, h, a.H, pwide, v);
        else put_columns<T, N>(y + row * ld, ld, have, h, a.H, wide, v);
    }
    template <int N>
    __device__ __forceinline__ void put_second(const HiddenArgs& a, int64_t row, int have, int h, const f32x4 (&v)[N]) const {
        put_columns<T, N>(p + row * pld + a.H, pld, have, h, a.H, pwide, v);
    }
};

}  // namespace spp
