// The gradient of the layers that read rows in 4 or 8 bits by their weights, over the product's lists:
//
//   dW[g] = sum over the lists j of group g of dY_j^T X_j        dY_j [n_j, H] fp32, fp16 or bf16, X_j [n_j, D] in few bits, dW fp32
//
// What a code and a scale stand for is exact in bf16, as is an fp16 as the sum of two bf16 and an fp32 of at least 2^-110 as that of three:
// the products of the matrix instruction are exact and are added in fp32, up to kGradChain times, those sums in 64 bits.  Of a smaller fp32 the bits
// below 2^-133, the smallest bf16, are lost: off by less than 2^-133 each, whatever X.

#pragma once

#include "spp_mx4.h"

#include <type_traits>

namespace spp {

// How a format F's rows are read here, 16 bytes of codes a piece: columns of a piece, pieces of a row (count), bytes of its codes, where
// in the row its scale is, and what its codes stand for, eight bf16 at a time.
struct GradMx4 {
    static constexpr int columns = 32;
    static __host__ __device__ __forceinline__ int count(int D) { return (D + 31) / 32; }
    static __device__ __forceinline__ int scale_at(int pieces, int piece) { return 16 * pieces + piece; }
    // the j-th eight of a piece
    static __device__ __forceinline__ bf16x8 eight(const u32x4& c, int j, float s) {
        const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], s, 1),
                     v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], s, 3);
        return bf16x8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
    }
};
struct GradFp8 {
    static constexpr int columns = 16;
    static __host__ __device__ __forceinline__ int count(int D) { return (D + 15) / 16; }
    static __device__ __forceinline__ int scale_at(int pieces, int piece) { return 16 * pieces + piece / 8; }
    static __device__ __forceinline__ bf16x8 eight(const u32x4& c, int j, float s) {
        const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * j], s, false), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * j], s, true),
                     v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * j + 1], s, false), v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * j + 1], s, true);
        return bf16x8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
    }
};

// The rows of all lists, in the order of their groups, are cut into chunks, and the chunks into `splits` runs of equal length.  A
// workgroup has one run and one tile of dW; where its run passes from a group to the next it writes down what it has as piece
// (run + group) and starts again, and the second kernel adds up each group's pieces in the order of the rows.  No atomics, and how
// many runs there are follows from the chunks that the lists have, not from those that their buffers could hold: on GPUs of as
// many CUs the same counts give the same bits.
//
// Both operands have the rows as the axis that is summed over, so their tiles lie in LDS as they lie in memory and are read
// transposed (ds_read_b64_tr_b16).  A chunk's operands are asked for two chunks ahead, into registers; X is unpacked to bf16 on
// its way to LDS, dY cut into its pieces.
//
// Bound by HBM where dW is one tile: 2.56M rows of 128 with 256 gradients in bf16 280 to 300 us, 5.0 to 5.3 TB/s; fp16 480, fp32 (half the rows) 345
// to 355, by the cutting and its two and three products.  For larger dW by the turns that writing a chunk to LDS and multiplying it take:
// 390k rows of 768 with 1024 in bf16 590 to 600 us, 1.0 PFLOP/s.  Few chunks a run leave little to overlap: 45k rows of 128 with
// 256 in bf16 26 us, 60k of 100 with 172 in eight groups in fp32 38 (their pieces, written and read again: 18 MB beside 72 of operands).
// Those are rows in 4 bits.  In 8: 2.5M rows of 256 with 512 gradients in bf16 740 us, 890 TFLOP/s, in fp16 1280, half of them in fp32 950; 380k of
// 1024 with 1024 775, 1.03 PFLOP/s; 93k of 172 with 200 in eight groups in fp32 55 to 59.
constexpr int kGradPad = 16;         // elements behind an LDS row: the four rows that 16 lanes read at once are then 4 x 32 bytes of other banks

struct GradArgs {
    RowTable t;
    void*    pieces;       // [splits + groups][H * D], fp32 or fp64
    float*   dw;           // [groups][H * D]
    int32_t  D, H, nb, rb; // nb: pieces of a row (GradMx4, GradFp8)
    int32_t  splits, tiles_d;        // runs that the grid and the pieces have room for
    int32_t  most;         // runs at most, by the matrix's shape
    int32_t  chunk;        // rows of a chunk
    int32_t  direct;       // one run and one group, within a chain: its sums are dW
    int32_t  wide;         // runs that may be longer than a chain: pieces in 64 bits
};

constexpr int kFewGradRows = 128;
// The runs of so many chunks: two chunks for each, but one run for a few rows.  Never more for fewer chunks: the host counts with
// what the lists can hold and the kernels with what they have.
__host__ __device__ __forceinline__ int grad_runs(int64_t chunks, int rows, int most) {
    if (chunks * rows <= kFewGradRows) return 1;
    const int64_t half = (chunks + 1) / 2;
    return half < most ? (int)half : most;
}

// The additions that an accumulator takes at most.  Rows that are alike are rounded alike: where dW filled the CUs, so that a group's rows were one
// run, 800k of them were off by 1.5e-3 in bf16 and 4e-3 in fp32, and by more the more they were.  Behind a chain of so many a run adds what it has to its
// piece in 64 bits and begins anew: reading and writing a piece is 1 MB a workgroup (256 x 256) beside some 25 MB of operands (1M rows of
// 2048 with 2048 gradients in bf16 7642 and 7764 us), and runs are as long only where there are many rows for the CUs (2.5M rows of 256 with 512
// gradients in bf16 have 610 additions a run).
constexpr int kGradChain = 1024;

// dY as bf16 numbers that add up to it exactly (above): one, two of an fp16, three of an fp32.  Cut off rather than rounded, so that no
// finite value becomes infinite; what is not finite is its first piece alone.
template <class T> struct Pieces { static constexpr int n = 1; };
template <> struct Pieces<_Float16> { static constexpr int n = 2; };
template <> struct Pieces<float> { static constexpr int n = 3; };
template <int P, bool Finite>
__device__ __forceinline__ void cut(float x, __bf16 (&out)[P]) {
    const bool finite = Finite || (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const uint32_t head = __float_as_uint(x) & 0xFFFF0000u;
        out[p] = p == 0 && !finite ? (__bf16)x : __builtin_bit_cast(__bf16, (uint16_t)(head >> 16));
        x = finite ? x - __uint_as_float(head) : 0.0f;
    }
}

// Eight rows of the lane's column, four and the four sixteen rows on: of 16 lanes, lane i names row i/4 and columns 4 (i mod 4) ..,
// and gets column i of four rows.  The wavefront's 64 lanes so read 16 rows that follow each other, 32 lanes eight: with
// the pad behind each row these are 256 bytes of different banks.  In what order the 32 rows are summed is the same to both operands.
template <int LD>
__device__ __forceinline__ bf16x8 column8(const __bf16* p) {
    typedef __attribute__((address_space(3))) i16x4* lds4;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 16 * LD));
    const bf16x4 x = __builtin_bit_cast(bf16x4, a), y = __builtin_bit_cast(bf16x4, b);
    return bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

template <class F, class T, int WH, int WD, int FH>
struct GradShape {
    typedef F format;
    static constexpr int columns = F::columns, row_pieces = 64 * WD / columns;     // of a row of the tile
    static constexpr int P = Pieces<T>::n, wh = WH, wd = WD, fh = FH;
    static constexpr int rows = P == 1 ? 64 : 32;                    // of a chunk: two buffers of it fit the LDS
    static constexpr int threads = 64 * WH * WD;
    static constexpr int chain = kGradChain / (rows / 32 * P);       // in chunks
    static constexpr int th = 16 * FH * WH, td = 64 * WD;            // the tile of dW: a wavefront has 16 FH x 64 of it
    static constexpr int ly = th + kGradPad, lx = td + kGradPad;     // elements of an LDS row
    static constexpr int buffer = rows * (P * ly + lx);              // elements of a buffer
    static constexpr int lds = 2 * buffer * 2;
    static constexpr int ve = 16 / (int)sizeof(T);                   // elements of a 16-byte vector of dY
    static constexpr int ahead = FH > 4 ? 1 : 2;                     // chunks in registers: the largest tile leaves room for one
    static constexpr int ny = rows * th / ve / threads;              // vectors of dY, pieces of X per thread and chunk
    static constexpr int nx = (rows * row_pieces + threads - 1) / threads;
};

// Some shapes take up to 466 of 512 registers: no code here is masked behind the first product but what a whole wavefront does or does not.
template <class F, class T, int WH, int WD, int FH>
__global__ void __launch_bounds__(64 * WH * WD) weight_grad_kernel(GradArgs a) {
    typedef GradShape<F, T, WH, WD, FH> S;
    constexpr int RP = S::row_pieces;
    constexpr int P = S::P;
    extern __shared__ __attribute__((aligned(16))) __bf16 lds[];
    const Lists lists(a.t, S::rows);
    const int total = lists.total();
    const int splits = grad_runs(total, S::rows, a.most);
    const int tiles = (int)gridDim.x / a.splits;
    // the tiles of a run, which read the same rows, share an XCD's L2
    const int id = (int)own_piece();
    const int tile = id % tiles, split = id / tiles;
    if (split >= splits || (total == 0 && !a.direct)) return;          // (no chunk: dW is zeros)
    const int from = (int)((int64_t)split * total / splits), to = (int)((int64_t)(split + 1) * total / splits);
    const int h0 = tile / a.tiles_d * S::th, d0 = tile % a.tiles_d * S::td;
    const int wave = threadIdx.x >> 6, l = lane_id();
    const int wh = wave / WD * (16 * FH), wd = wave % WD * 64;

    u32x4 ry[S::ahead][S::ny], rx[S::ahead][S::nx];
    uint32_t rs[S::ahead][S::nx];
    int here[S::ahead], group[S::ahead];

    // Where the next chunk is; chunks are asked for in their order, so that most follow the one before in its list.
    const T* y = nullptr;
    const uint8_t* x = nullptr;
    int64_t ld = 0;
    int until = from, list_group = 0, left = 0;                      // the list's last chunk + 1, its group, its rows from the chunk on
    bool wide = false;
    uint32_t oy[S::ny], ox[S::nx], os[S::nx];                        // a whole chunk's vectors, pieces and scales
#pragma unroll
    for (int k = 0; k < S::nx; ++k) {
        const int i = k * S::threads + (int)threadIdx.x, b = d0 / S::columns + i % RP;
        const int r = i / RP < S::rows ? i / RP : S::rows - 1, in = b < a.nb ? b : a.nb - 1;
        ox[k] = (uint32_t)(r * a.rb + 16 * in);
        os[k] = (uint32_t)(r * a.rb + F::scale_at(a.nb, in));
    }
    // Behind the last chunk (more false) the last one again: a path without loads would make the compiler wait for all that are under way.
    auto load = [&](int u, int chunk, bool more) {
        if (more && chunk >= until) {
            const int list = lists.list_of(chunk);
            const int before = chunk - lists.first_tile(list);
            until = __builtin_amdgcn_readlane(lists.upto, list);
            left = lists.rows_in(list) - before * S::rows;
            list_group = a.t.group[list];
            ld = a.t.ld[list];
            y = static_cast<const T*>(a.t.y[list]) + (int64_t)before * S::rows * ld;
            x = a.t.rows[list] + (int64_t)before * S::rows * a.rb;
            wide = ((uintptr_t)a.t.y[list] | (uint64_t)(ld * (int64_t)sizeof(T))) % 16 == 0 && a.H % S::ve == 0;
#pragma unroll
            for (int k = 0; k < S::ny; ++k) {
                const int i = k * S::threads + (int)threadIdx.x, h = h0 + i % (S::th / S::ve) * S::ve;
                oy[k] = (uint32_t)(i / (S::th / S::ve) * (int)ld + (h < a.H ? h : 0));
            }
        } else if (more) {
            y += S::rows * ld;
            x += S::rows * a.rb;
            left -= S::rows;
        }
        here[u] = left < S::rows ? left : S::rows;
        group[u] = list_group;
        // Columns behind H or D: others in their place, as those columns of dW are not written; rows behind the list's last: the last,
        // put() clears them.  A vector may reach over a row's end into the next row, but not over the list's.
        uint32_t py[S::ny], px[S::nx], ps[S::nx];
#pragma unroll
        for (int k = 0; k < S::ny; ++k) py[k] = oy[k];
#pragma unroll
        for (int k = 0; k < S::nx; ++k) { px[k] = ox[k]; ps[k] = os[k]; }
        if (left < S::rows) {
#pragma unroll
            for (int k = 0; k < S::ny; ++k) {
                const int i = k * S::threads + (int)threadIdx.x, r = i / (S::th / S::ve);
                py[k] -= (uint32_t)(max(r - left + 1, 0) * (int)ld);
            }
#pragma unroll
            for (int k = 0; k < S::nx; ++k) {
                const int i = k * S::threads + (int)threadIdx.x, r = i / RP < S::rows ? i / RP : S::rows - 1;
                const uint32_t back = (uint32_t)(max(r - left + 1, 0) * a.rb);
                px[k] -= back; ps[k] -= back;
            }
        }
        if (ld < (1 << 24) && (wide || (left > S::rows && a.H >= S::ve))) {
            if (wide)
#pragma unroll
                for (int k = 0; k < S::ny; ++k) ry[u][k] = *reinterpret_cast<const u32x4*>(y + py[k]);
            else
#pragma unroll
                for (int k = 0; k < S::ny; ++k) ry[u][k] = reinterpret_cast<const Loose<u32x4>*>(y + py[k])->v;
        } else {
#pragma unroll
            for (int k = 0; k < S::ny; ++k) {
                const int i = k * S::threads + (int)threadIdx.x, h = h0 + i % (S::th / S::ve) * S::ve;
                int r = i / (S::th / S::ve);
                r = r < here[u] ? r : here[u] - 1;
                T v[S::ve];
#pragma unroll
                for (int j = 0; j < S::ve; ++j) v[j] = y[r * ld + (h + j < a.H ? h + j : a.H - 1)];
                ry[u][k] = __builtin_bit_cast(u32x4, v);
            }
        }
#pragma unroll
        for (int k = 0; k < S::nx; ++k) {
            rx[u][k] = *reinterpret_cast<const u32x4*>(x + px[k]);
            rs[u][k] = x[ps[k]];
        }
    };
    auto put = [&](int u, int buffer) {
        __bf16* gy = lds + buffer * S::buffer;
        __bf16* gx = gy + P * S::rows * S::ly;
        if (here[u] < S::rows) {                           // the list's last chunk: rows behind its last are zeros
#pragma unroll
            for (int k = 0; k < S::ny; ++k) ry[u][k] &= (k * S::threads + (int)threadIdx.x) / (S::th / S::ve) < here[u] ? ~0u : 0u;
#pragma unroll
            for (int k = 0; k < S::nx; ++k) {
                const uint32_t there = (k * S::threads + (int)threadIdx.x) / RP < here[u] ? ~0u : 0u;
                rx[u][k] &= there;
                rs[u][k] &= there;                         // (2^-127: not NaN)
            }
        }
#pragma unroll
        for (int k = 0; k < S::ny; ++k) {
            const int i = k * S::threads + (int)threadIdx.x;
            const int r = i / (S::th / S::ve), h = i % (S::th / S::ve) * S::ve;
            const u32x4 raw = ry[u][k];
            if constexpr (P == 1) {
                *reinterpret_cast<u32x4*>(gy + r * S::ly + h) = raw;
            } else {
                struct Vec { T v[S::ve]; } in = __builtin_bit_cast(Vec, raw);
                struct Cut { __bf16 v[S::ve]; } out[P];
                auto each = [&](auto finite) {
#pragma unroll
                    for (int j = 0; j < S::ve; ++j) {
                        __bf16 c[P];
                        cut<P, decltype(finite)::value>((float)in.v[j], c);
#pragma unroll
                        for (int p = 0; p < P; ++p) out[p].v[j] = c[p];
                    }
                };
                bool odd;                                  // infinite or NaN
                if constexpr (S::ve == 8) {
                    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
                    u16x2 top = __builtin_bit_cast(u16x2, raw.x & 0x7FFF7FFFu);
#pragma unroll
                    for (int j = 1; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, raw[j] & 0x7FFF7FFFu));
                    odd = top[0] >= 0x7C00u || top[1] >= 0x7C00u;
                } else {
                    uint32_t top = raw.x & 0x7FFFFFFFu;
#pragma unroll
                    for (int j = 1; j < 4; ++j) top = top > (raw[j] & 0x7FFFFFFFu) ? top : raw[j] & 0x7FFFFFFFu;
                    odd = top >= 0x7F800000u;
                }
                if (__any(odd)) each(std::false_type());
                else each(std::true_type());
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if constexpr (S::ve == 8) *reinterpret_cast<u32x4*>(gy + (p * S::rows + r) * S::ly + h) = __builtin_bit_cast(u32x4, out[p]);
                    else *reinterpret_cast<u32x2*>(gy + (p * S::rows + r) * S::ly + h) = __builtin_bit_cast(u32x2, out[p]);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < S::nx; ++k) {
            const int i = k * S::threads + (int)threadIdx.x;
            const int r = i / RP;
            if (S::rows * RP % S::threads && __builtin_amdgcn_readfirstlane(r) >= S::rows) continue;       // a wavefront's are, or are not: 64 divide them
            const float s = mx4_scale(rs[u][k]);
            u32x4 c = rx[u][k];
            __bf16* to_x = gx + r * S::lx + i % RP * S::columns;
            if constexpr (S::columns == 32) {
                // 16 lanes' pieces of 16 bytes, 64 bytes apart, in banks of their own: half of the lanes begin with the second
                const int turn = WD == 2 ? (l >> 3) & 1 : (l >> 2) & 1;
                c = turn ? u32x4{c.y, c.z, c.w, c.x} : c;
#pragma unroll
                for (int j = 0; j < 4; ++j) *reinterpret_cast<bf16x8*>(to_x + 8 * ((j + turn) & 3)) = F::eight(c, j, s);
            } else {
                // and 32 bytes apart
                const int turn = (l >> 3) & 1;
                c = turn ? u32x4{c.z, c.w, c.x, c.y} : c;
#pragma unroll
                for (int j = 0; j < 2; ++j) *reinterpret_cast<bf16x8*>(to_x + 8 * ((j + turn) & 1)) = F::eight(c, j, s);
            }
        }
    };

    f32x4 acc[FH][4];
    auto clear = [&]() {
#pragma unroll
        for (int f = 0; f < FH; ++f)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[f][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    // By way of a buffer, whose range check takes the place of masks: what lies behind H or D goes nowhere.  `more`: to what the piece has already.
    auto flush = [&](int g, bool more) {
        // from values made anew: addresses worked out ahead of the loop would take the registers that it needs
        const int lane = spp::here(l);
        const int64_t size = (int64_t)a.H * a.D, piece = (int64_t)(split + __builtin_amdgcn_readfirstlane(g)) * size;
        const uint32_t h = h0 + wh + 4 * (lane >> 4), d = d0 + wd + (lane & 15);
        auto place = [&](int f, int c, int i, int es) {
            const uint32_t at = ((h + 16 * f + i) * (uint32_t)a.D + d + 16 * c) * es;
            return (h + 16 * f + i < (uint32_t)a.H) & (d + 16 * c < (uint32_t)a.D) ? at : kNowhere;
        };
        if (!a.wide) {
            const auto out = rows_buffer(a.direct ? a.dw : static_cast<float*>(a.pieces) + piece, (uint32_t)size * 4);
#pragma unroll
            for (int f = 0; f < FH; ++f)
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) buffer_store<0>(acc[f][c][i], out, place(f, c, i, 4));
        } else {
            const auto out = rows_buffer(static_cast<double*>(a.pieces) + piece, (uint32_t)size * 8);       // at most 2^31 bytes
#pragma unroll
            for (int f = 0; f < FH; ++f)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t at[4];
                    double v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        at[i] = place(f, c, i, 8);
                        v[i] = 0.0;
                    }
                    if (more)
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(double, buffer_load<u32x2>(out, at[i]));
#pragma unroll
                    for (int i = 0; i < 4; ++i) buffer_store<0>(__builtin_bit_cast(u32x2, v[i] + (double)acc[f][c][i]), out, at[i]);
                }
        }
    };
    const int n = to - from;
    clear();
    int now = 0, held = 0;                                           // the group, chunks in the accumulators
    bool more = false;                                               // the group's piece has been begun
    if (n > 0) {
        load(0, from, true);
        if (S::ahead > 1) load(S::ahead - 1, from + 1, n > 1);
        now = group[0];
    }
    for (int j = 0; j < n; j += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (j + u >= n) break;
            constexpr int mask = S::ahead - 1;
            if (group[u & mask] != now || (a.wide && held == S::chain)) {
                flush(now, more);
                clear();
                more = group[u & mask] == now;
                now = group[u & mask];
                held = 0;
            }
            ++held;
            put(u & mask, u);
            load(u & mask, from + j + u + S::ahead, j + u + S::ahead < n);
            __syncthreads();         // the other buffer has been read by all before this one is read by any
            const __bf16* gy = lds + u * S::buffer;
            const __bf16* gx = gy + P * S::rows * S::ly;
#pragma unroll
            for (int k = 0; k < S::rows; k += 32) {
                const int row = k + 4 * (l >> 4) + ((l & 15) >> 2), col = 4 * (l & 3);
                bf16x8 bx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) bx[c] = column8<S::lx>(gx + row * S::lx + col + wd + 16 * c);
                // the next rows of dY are read during the products of these
                auto read = [&](int e) { return column8<S::ly>(gy + (e / FH * S::rows + row) * S::ly + col + wh + 16 * (e % FH)); };
                bf16x8 ay[2];
                ay[0] = read(0);
#pragma unroll
                for (int e = 0; e < P * FH; ++e) {
                    if (e + 1 < P * FH) ay[(e + 1) & 1] = read(e + 1);
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[e % FH][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ay[e & 1], bx[c], acc[e % FH][c], 0, 0, 0);
                }
            }
        }
    }
    flush(now, more);
}

// The pieces of 256 elements side by side, four a lane, are added by a workgroup's wavefronts in turn, then the wavefronts' sums:
// always in the same order.
constexpr int kSumWaves = 16;
// The wavefronts that share a group's pieces, by the runs there are; those that a grid with room for more runs has beyond them add nothing.
__host__ __device__ __forceinline__ int grad_sum_waves(int runs, int groups) {
    const int each = runs / groups + 1;
    return each > 64 ? kSumWaves : each > 16 ? 8 : 4;
}
typedef double f64x4 __attribute__((ext_vector_type(4)));
template <class V>       // of a piece
static __global__ void __launch_bounds__(64 * kSumWaves) weight_grad_sum_kernel(GradArgs a) {
    typedef V V4 __attribute__((ext_vector_type(4)));
    __shared__ f64x4 part[kSumWaves][kWave];
    const Lists lists(a.t, a.chunk);
    const int total = lists.total(), group = blockIdx.y, wave = threadIdx.x >> 6, l = lane_id();
    const int splits = grad_runs(total, a.chunk, a.most), waves = grad_sum_waves(splits, (int)gridDim.y);
    const int64_t size = (int64_t)a.H * a.D;
    // the chunks of the group: from its first list's first to its last list's last
    const uint64_t mine = __ballot(l < a.t.n_lists && (int)a.t.group[l] == group && lists.tiles > 0);
    int lo = 0, hi = -1;
    if (mine) {
        const int first = lists.first_tile(__builtin_ctzll(mine)), last = __builtin_amdgcn_readlane(lists.upto, 63 - __builtin_clzll(mine)) - 1;
        lo = (int)((((int64_t)first + 1) * splits - 1) / total);
        hi = wave < waves ? (int)((((int64_t)last + 1) * splits - 1) / total) : -1;
    }
    const int64_t i = ((int64_t)blockIdx.x * kWave + l) * 4;
    // a vector at the matrix' end begins earlier: its last elements are the matrix' last
    const int64_t at = size < 4 ? 0 : i + 4 <= size ? i : size - 4;
    const V* p = static_cast<const V*>(a.pieces) + group * size + at;
    f64x4 sum = {0.0, 0.0, 0.0, 0.0};
    auto add = [&](V4 v) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += (double)v[k];
    };
    auto take = [&](int s) {
        const V* from = p + (int64_t)s * size;
        if (size >= 4) return reinterpret_cast<const Loose<V4>*>(from)->v;
        V4 v = {0, 0, 0, 0};
        for (int k = 0; k < (int)size; ++k) v[k] = from[k];
        return v;
    };
    int s = lo + wave;
    for (; s + 7 * waves <= hi; s += 8 * waves) {
        V4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = take(s + k * waves);
#pragma unroll
        for (int k = 0; k < 8; ++k) add(v[k]);
    }
    for (; s + 3 * waves <= hi; s += 4 * waves) {
        V4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = take(s + k * waves);
#pragma unroll
        for (int k = 0; k < 4; ++k) add(v[k]);
    }
    for (; s <= hi; s += waves) add(take(s));
    part[wave][l] = sum;
    __syncthreads();
    if (wave == 0) {
        for (int k = 1; k < waves; ++k) sum += part[k][l];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at + k >= i && at + k < size) a.dw[group * size + at + k] = (float)sum[k];
    }
}

template <class S>
static int64_t grad_tiles(const GradArgs& a) { return (int64_t)((a.D + S::td - 1) / S::td) * ((a.H + S::th - 1) / S::th); }
template <class T, class S>
static int launch_grad(spp_ctx* ctx, GradArgs& a, int n_groups, bool sum_only) {
    auto kernel = weight_grad_kernel<typename S::format, T, S::wh, S::wd, S::fh>;
    static LdsLimit limit;
    a.chunk = S::rows;
    a.tiles_d = (a.D + S::td - 1) / S::td;
    const int64_t tiles = grad_tiles<S>(a), size = (int64_t)a.H * a.D;
    int64_t chunks = 0;
    for (int j = 0; j < a.t.n_lists; ++j) chunks += (a.t.n[j] + (int64_t)S::rows - 1) / S::rows;
    a.splits = grad_runs(chunks, S::rows, a.most);
    // What the lists can hold decides the pieces' type, which does not show in the result: a run within a chain gives the same sum in either.
    a.wide = (chunks + a.splits - 1) / a.splits > S::chain;
    a.direct = !sum_only && !a.wide && a.splits == 1 && n_groups == 1;
    if (!a.direct) SPP_TRY(ctx->gradws.reserve((size_t)(a.splits + n_groups) * size * (a.wide ? sizeof(double) : sizeof(float)), ctx->stream));
    a.pieces = ctx->gradws.ptr;
    if (!sum_only) {
        SPP_TRY(limit.allow(ctx, reinterpret_cast<const void*>(kernel), S::lds));
        kernel<<<(unsigned)(a.splits * tiles), S::threads, S::lds, ctx->stream>>>(a);
        SPP_HIP(hipGetLastError());
    }
    if (a.direct) return SPP_OK;
    const int64_t sums = (size + 4 * kWave - 1) / (4 * kWave);       // at most 2^20: SPP_MAX_HIDDEN rows of SPP_MX4_MAX_COLS
    auto sum = a.wide ? weight_grad_sum_kernel<double> : weight_grad_sum_kernel<float>;
    sum<<<dim3((unsigned)sums, n_groups), 64 * grad_sum_waves(a.splits, n_groups), 0, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}
// Tiles of dW: as few as 256 x 256 (of 128 columns: 256 x 128) allow, of as few wavefronts as these need.  The larger the tile, the
// less is read from LDS per product and the less often dY and X are read.
template <class F, class T, class Use>
static int grad_shape(const GradArgs& a, Use use) {
    const int tiles = (a.H + 255) / 256, h = (a.H + tiles - 1) / tiles;
    if (a.D > 128) {
        if (h > 128) return use(GradShape<F, T, 2, 4, 8>());
        return h > 64 ? use(GradShape<F, T, 2, 4, 4>()) : use(GradShape<F, T, 1, 4, 4>());
    }
    if (a.D > 64) {
        // (six wavefronts: of 16-column pieces and one product the registers would not hold the chunks ahead)
        if constexpr (F::columns == 16 && Pieces<T>::n == 1) { if (h > 128) return use(GradShape<F, T, 4, 2, 4>()); }
        else if (h > 128) return h > 192 ? use(GradShape<F, T, 4, 2, 4>()) : use(GradShape<F, T, 3, 2, 4>());
        return h > 64 ? use(GradShape<F, T, 2, 2, 4>()) : use(GradShape<F, T, 1, 2, 4>());
    }
    if (h > 128) return h > 192 ? use(GradShape<F, T, 4, 1, 4>()) : use(GradShape<F, T, 3, 1, 4>());
    return h > 64 ? use(GradShape<F, T, 2, 1, 4>()) : use(GradShape<F, T, 1, 1, 4>());
}
// kFewGradRows rows and less take tiles of 128 x 128 and, in one list, one run, so that more CUs have something to write and no pieces
// need adding.  Large tiles and two launches against this, us: 128 x 256 in bf16 100 rows 15 and 10.5, 256 15 and 12, 512 15 and
// 16; in fp32 100 rows 16 and 13.5, 160 15 both, 256 15.5 and 20; 768 x 1024 in bf16 128 rows 15 and 10, 512 27 and 17, 1000 30 and 26; in
// fp32 128 rows 28 and 14, 384 30 and 27, 512 31 and 33.  (So large matrices and 16 bits would gain up to 384 rows and more; the limit
// is where no shape or type loses.)
// The runs are those of the ordinary tiles: a tile's size does not change the order in which an element's rows are added.
template <class F, class T>
static int grad_of(spp_ctx* ctx, GradArgs& a, int n_groups, int64_t most) {
    const bool sum_only = most == 0;
    a.most = grad_shape<F, T>(a, [&](auto shape) {
        typedef decltype(shape) S;
        // as many workgroups as run at once
        const int fit = 163840 / S::lds, wish = 8 / (S::wh * S::wd);
        const int64_t at_once = (int64_t)ctx->num_cu * (fit < 1 || wish < 1 ? 1 : fit < wish ? fit : wish), runs = at_once / grad_tiles<S>(a);
        return (int)(runs < 1 ? 1 : runs);
    });
    auto launch = [&](auto shape) { return launch_grad<T, decltype(shape)>(ctx, a, n_groups, sum_only); };
    const int tiles = (a.H + 255) / 256, h = (a.H + tiles - 1) / tiles;
    return most <= kFewGradRows && a.D > 64 && h > 64 ? launch(GradShape<F, T, 2, 2, 4>()) : grad_shape<F, T>(a, launch);
}

template <class F>
static int weight_grad(const char* who, spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, int32_t n_groups, int32_t D, int32_t H,
                       int32_t type, float* d_grad, int row_bytes, uint32_t flags) {
    SPP_CHECK(ctx && d_grad, SPP_E_ARG, "%s: null argument", who);
    SPP_CHECK((uintptr_t)d_grad % 4 == 0, SPP_E_ARG, "%s: the gradient must be 4-byte aligned", who);
    GradArgs a;
    int64_t most = 0;
    SPP_TRY(row_table(who, lists, n_lists, n_groups, D, H, type, a.t, &most));
    SPP_HIP(hipSetDevice(ctx->device));
    a.dw = d_grad; a.D = D; a.H = H; a.nb = F::count(D); a.rb = row_bytes;
    hipStream_t st = ctx->stream;
    ScopedTimer timer(ctx, SPP_T_LAYER, st);
    SPP_TRY(type == SPP_F32 ? (grad_of<F, float>(ctx, a, n_groups, most)) : type == SPP_F16 ? (grad_of<F, _Float16>(ctx, a, n_groups, most))
                                                                                              : (grad_of<F, __bf16>(ctx, a, n_groups, most)));
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(st));
    return SPP_OK;
}

}  // namespace spp
