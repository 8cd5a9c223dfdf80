// The layer that reads feature rows in MXFP4, and its gradient, over up to 64 lists of rows whose lengths may be known on the
// device only (the minibatches that a pipeline keeps in flight; rows of several kinds, each kind with a matrix of its own):
//
//   product       Y_j = X_j W[g_j]^T           X_j [n_j, D] and W[g] [H, D] in MXFP4, Y_j fp32, fp16 or bf16
//   weight grad   dW[g] = sum_j dY_j^T X_j     over the lists of group g; dY_j fp32, fp16 or bf16, dW fp32
//
// What a code and a scale stand for is exact in bf16, as is an fp32 as the sum of three bf16: the products of both kernels are
// exact and are added in fp32, so the only other roundings are those of the sums and of Y.
#include "spp_mx4.h"

namespace spp {

// Lane j has list j: its rows, and the tiles of all lists up to it.  The count of a list may have to be fetched: one round trip.
struct Lists {
    int rows, upto, tiles;
    __device__ __forceinline__ Lists(const RowTable& t, int tile_rows) {
        const int j = lane_id();
        rows = j < t.n_lists ? (int)rows_of(t.n[j], t.d_n[j]) : 0;
        tiles = (int)(((int64_t)rows + tile_rows - 1) / tile_rows);
        upto = wave_inclusive_scan(tiles);
    }
    __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(upto, kWave - 1); }
    __device__ __forceinline__ int list_of(int tile) const { return __builtin_amdgcn_readfirstlane(__popcll(__ballot(upto <= tile))); }
    __device__ __forceinline__ int rows_in(int list) const { return __builtin_amdgcn_readlane(rows, list); }
    __device__ __forceinline__ int first_tile(int list) const { return __builtin_amdgcn_readlane(upto - tiles, list); }
};

// ---- product --------------------------------------------------------------------------------------

struct ProductArgs {
    RowTable       t;
    const uint8_t* w;
    int32_t        D, H, nb, rb;
    int32_t        ls;           // bytes of a row of W in LDS: an odd number of 16, so that 16 rows lie in banks of their own
    uint32_t       magic;        // ceil(2^32 / (rb / 16))
    int32_t        fill;         // workgroups that few rows are dealt out to
    int32_t        w_lds;        // bytes of W in LDS; behind them, per wavefront, room for rows of Y on their way:
    int32_t        out_lds;      // bytes
};

constexpr int kProdBlock = 256, kProdWaves = 4;

// Four consecutive 32-bit words of operand for a scaled 16x16x128 product in E2M1: the lane's block of 32 columns.
__device__ __forceinline__ i32x8 mx4_operand(u32x4 v) {
    return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
}

// A product's operands: rows of X as the 16 rows of the result, columns 4m + f of a 64-column tile of Y as column m of result f.
// A lane then has four columns side by side, and the 16 lanes of a row 64: stores of whole 128-byte lines.
__device__ __forceinline__ int tile_column(int f, int m) { return 4 * m + f; }

// Columns h .. h+3 of rows y[0..3], of which `have` are there.
template <class T>
__device__ __forceinline__ void put_tile(T* y, int64_t ld, int have, int h, int H, bool wide, const f32x4 (&acc)[4]) {
    typedef typename Elem<T>::v4 V;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const V v = {(T)acc[0][i], (T)acc[1][i], (T)acc[2][i], (T)acc[3][i]};
        T* out = y + i * ld + h;
        if (i >= have) continue;
        if (wide && h + 4 <= H) *reinterpret_cast<V*>(out) = v;
        else if (h + 4 <= H) reinterpret_cast<Loose<V>*>(out)->v = v;
        else
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (h + k < H) out[k] = v[k];
    }
}
// All of them, aligned.
template <class T>
__device__ __forceinline__ void put_whole(T* y, int64_t ld, const f32x4 (&acc)[4]) {
    typedef typename Elem<T>::v4 V;
#pragma unroll
    for (int i = 0; i < 4; ++i) __builtin_nontemporal_store(V{(T)acc[0][i], (T)acc[1][i], (T)acc[2][i], (T)acc[3][i]}, reinterpret_cast<V*>(y + i * ld));
}

// A wavefront's 16 RN rows of Y on their way to memory where they do not begin with a line each.  They are put together in LDS and
// written by whole 16-byte pieces, side by side; the ends of a row or a run, less than a piece, by element.
//   run    the rows follow each other without a gap and fit: all of them are put together as one run of bytes
//   lines  64 columns of every row at a time, each byte where it lies in its 128-byte line: what they fill of lines goes out, the
//          begun line stays for the next 64
// Offsets that every 64 columns share are computed once a tile of rows: a tile of 16 x 64 results costs a SIMD some 150 clocks of
// matrix work, which is not many instructions.
template <class T, int RN>
struct RowsOut {
    static constexpr int kBytes = 64 * (int)sizeof(T), kPitch = kBytes + 128, kPieces = 2 * RN;     // per lane: rows lane/8 + 8j, a piece of each line
    typedef typename Elem<T>::v4 V;
    uint8_t* lds;
    char*    y;              // first row, first of the wavefront's columns
    int64_t  step;           // bytes from a row to the next
    int      rows, bytes;    // bytes of the wavefront's columns of a row
    bool     run;
    int      to[RN][4];      // where in LDS the lane's four columns of its rows go
    __device__ __forceinline__ int phase(int row) const { return (int)(((uintptr_t)y + row * step) & 127); }
    __device__ __forceinline__ void begin() {
        const int q = lane_id() >> 4, m = lane_id() & 15;
#pragma unroll
        for (int c = 0; c < RN; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * c + 4 * q + i;
                to[c][i] = 4 * m * (int)sizeof(T) + (run ? (int)((uintptr_t)y & 15) + row * (int)step : row * kPitch + phase(row));
            }
    }
    // The t-th 64 columns from the wavefront's first.  An LDS write that is not aligned to its size takes many times one that is
    // (rows of 2002 bytes 424 us, of 2008 246), so each alignment has writes of its own.
    template <class W>
    __device__ __forceinline__ void put_as(uint8_t* at, const f32x4 (&acc)[RN][4]) const {
        constexpr int n = (int)(sizeof(V) / sizeof(W));
#pragma unroll
        for (int c = 0; c < RN; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const V v = {(T)acc[c][0][i], (T)acc[c][1][i], (T)acc[c][2][i], (T)acc[c][3][i]};
                struct Words { W w[n]; } words = __builtin_bit_cast(Words, v);
#pragma unroll
                for (int k = 0; k < n; ++k) {
                    if constexpr (sizeof(W) == 2) reinterpret_cast<volatile W*>(at + to[c][i])[k] = words.w[k];      // the compiler would join them again
                    else reinterpret_cast<W*>(at + to[c][i])[k] = words.w[k];
                }
            }
    }
    __device__ __forceinline__ void put(int t, const f32x4 (&acc)[RN][4]) const {
        uint8_t* at = lds + (run ? t * kBytes : 0);
        if (run && (t + 1) * kBytes > bytes) {                   // behind a row's last column the next one lies
            const int left = (bytes - t * kBytes) / (int)sizeof(T) - 4 * (lane_id() & 15);
#pragma unroll
            for (int c = 0; c < RN; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < left) reinterpret_cast<T*>(at + to[c][i])[k] = (T)acc[c][k][i];
            return;
        }
        const uintptr_t bits = (uintptr_t)y | (uintptr_t)step;
        if (bits % sizeof(V) == 0) put_as<V>(at, acc);
        else if (sizeof(T) == 4 && bits % 8 == 0) put_as<uint64_t>(at, acc);
        else if (bits % 4 == 0) put_as<uint32_t>(at, acc);
        else if constexpr (sizeof(T) == 2) put_as<uint16_t>(at, acc);
    }
    __device__ __forceinline__ void flush_run() const {
        wave_lds_order();
        const int head = (int)((uintptr_t)y & 15), len = (rows - 1) * (int)step + bytes, end = (head + len) / 16;
        u32x4* out = reinterpret_cast<u32x4*>(y - head);
        const u32x4* from = reinterpret_cast<const u32x4*>(lds);
        int k = (head ? 1 : 0) + lane_id();
        for (; k + 3 * kWave < end; k += 4 * kWave) {
            u32x4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = from[k + u * kWave];
#pragma unroll
            for (int u = 0; u < 4; ++u) __builtin_nontemporal_store(v[u], &out[k + u * kWave]);
        }
        for (; k < end; k += kWave) __builtin_nontemporal_store(from[k], &out[k]);
        if (((uintptr_t)y | (uintptr_t)len) & 15) {
            // lanes 0..7: what lies before the first whole piece; 8..15: behind the last; a run inside one piece that it begins, too
            const int l = lane_id(), kk = l & 7, off = l < 8 ? head + kk * (int)sizeof(T) : 16 * end + kk * (int)sizeof(T);
            if (l < 8 ? head && off < 16 && off < head + len : l < 16 && off < head + len && (end > 0 || !head))
                *reinterpret_cast<T*>(y - head + off) = *reinterpret_cast<const T*>(lds + off);
        }
        wave_lds_order();
    }
    // After the t-th 64 columns.
    __device__ __forceinline__ void flush_lines(int t, bool first, bool last) const {
        wave_lds_order();
        const int l = lane_id(), k = l & 7;
        const uint8_t* mine = lds + (l >> 3) * kPitch + 16 * k;
        char* out = y + t * kBytes;
        if (!first && !last) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const int r = (l >> 3) + 8 * j;
                char* line = out + r * step;
                line -= (uintptr_t)line & 127;
#pragma unroll
                for (int u = 0; u < kBytes / 128; ++u) {
                    const u32x4 v = *reinterpret_cast<const u32x4*>(mine + 8 * j * kPitch + 128 * u);
                    if (r < rows) *reinterpret_cast<u32x4*>(line + 128 * u + 16 * k) = v;
                }
            }
        } else {
            const int fresh = last ? bytes - t * kBytes : kBytes;
            for (int j = 0; j < kPieces; ++j) {
                const int r = (l >> 3) + 8 * j, head = phase(r);
                char* line = out + r * step - head;
                const int from = first ? head : 0, end = last ? head + fresh : kBytes;
                if (r < rows)
                    for (int u = 0; u <= kBytes; u += 128) {
                        const int at = u + 16 * k;
                        if (at >= from && at + 16 <= end) {
                            *reinterpret_cast<u32x4*>(line + at) = *reinterpret_cast<const u32x4*>(mine + 8 * j * kPitch + u);
                        } else if (at + 16 > from && at < end) {             // the row's first or last piece, a part of it
                            for (int e = 0; e < 16; e += (int)sizeof(T))
                                if (at + e >= from && at + e < end)
                                    *reinterpret_cast<T*>(line + at + e) = *reinterpret_cast<const T*>(mine + 8 * j * kPitch + u + e);
                        }
                    }
            }
        }
        if (!last) {                                             // the begun line to where the next columns will find it
            u32x4 v[kPieces];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) v[j] = *reinterpret_cast<const u32x4*>(mine + 8 * j * kPitch + kBytes);
#pragma unroll
            for (int j = 0; j < kPieces; ++j) *reinterpret_cast<u32x4*>(const_cast<uint8_t*>(mine) + 8 * j * kPitch) = v[j];
        }
        wave_lds_order();
    }
};

// The ordinary form, for D up to 768.  A wavefront holds its 16 RN rows of X in registers, all columns of them, and goes over the
// columns of Y 64 at a time; W comes from LDS, where a workgroup's wavefronts share it.  If all of W fits it stays there
// (Stream false), else 64 of its rows at a time, the next ones asked for while these are used.  X is read once and Y, which is most
// of what moves, written once.
template <class T, int KS, int RN, int WAVES, bool Stream, bool Lines>
__global__ void __launch_bounds__(64 * WAVES) mx4_rows_kernel(ProductArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t ws[];
    constexpr int TB = WAVES * 16 * RN, threads = 64 * WAVES;
    constexpr int kVec = (64 * ((KS * 4 * 17 + 15) / 16) + threads - 1) / threads;       // vectors of 64 rows of W per thread
    const Lists lists(a.t, TB);
    const int total = lists.total();
    if (total == 0) return;
    const int wave = threadIdx.x >> 6, l = lane_id(), m = l & 15, q = l >> 4;
    const int ht = (a.H + 63) / 64;
    int parts = a.fill / total;                        // few rows: the columns of Y are dealt out too
    parts = parts < 1 ? 1 : parts > ht ? ht : parts;
    const int64_t items = (int64_t)total * parts;
    const int rv = a.rb / 16, lv = a.ls / 16;          // vectors of a row of W in memory and in LDS
    int held_group = -1, held_from = -1;
    RowsOut<T, RN> out;
    out.lds = ws + a.w_lds + wave * a.out_lds;
    struct Item { int part, list, here, group; int64_t r0; };
    auto find = [&](int64_t item) {
        Item it;
        it.part = (int)(item / total);
        const int tile = (int)(item - (int64_t)it.part * total);
        it.list = lists.list_of(tile);
        it.r0 = (int64_t)(tile - lists.first_tile(it.list)) * TB;
        const int64_t left = lists.rows_in(it.list) - it.r0;
        it.here = left < TB ? (int)left : TB;
        it.group = a.t.group[it.list];
        return it;
    };
    // X: a lane has row m of each 16 and every fourth block.  Asked for an item ahead.
    u32x4 ahead[KS][RN];
    uint32_t ahead_scale[KS][RN];
    auto ask_rows = [&](const Item& it) {
        const uint8_t* x = a.t.rows[it.list] + it.r0 * a.rb;
#pragma unroll
        for (int c = 0; c < RN; ++c) {
            const int row = (wave * RN + c) * 16 + m;
            const uint8_t* p = x + (row < it.here ? row : it.here - 1) * a.rb;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bool in = 4 * s + q < a.nb;
                ahead[s][c] = *reinterpret_cast<const u32x4*>(p + 16 * (in ? 4 * s + q : 0));
                ahead_scale[s][c] = *reinterpret_cast<const uint32_t*>(p + 16 * a.nb + 4 * s);
            }
        }
    };
    const Share share(items);
    if (share.at >= share.end) return;
    constexpr bool kAhead = !Stream;                   // streams have fewer registers than KS = 6 would need for it
    Item it = find(share.at);
    if (kAhead) ask_rows(it);
    for (int64_t item = share.at; item < share.end; item += share.step) {
        if (!kAhead) { it = find(item); ask_rows(it); }
        const int t0 = (int)((int64_t)it.part * ht / parts), t1 = (int)((int64_t)(it.part + 1) * ht / parts);
        const int list = it.list, here = it.here, group = it.group, mine = here - wave * 16 * RN;       // rows of the workgroup, of the wavefront
        const int64_t r0 = it.r0;
        const uint8_t* w = a.w + (int64_t)group * a.H * a.rb;
        const int64_t ld = a.t.ld[list];
        T* y = static_cast<T*>(a.t.y[list]) + (r0 + wave * 16 * RN) * ld;
        if (!Lines) {
            out.rows = mine < 16 * RN ? mine : 16 * RN;
            out.step = ld * (int64_t)sizeof(T);
            out.y = reinterpret_cast<char*>(y + 64 * t0);
            out.bytes = ((64 * t1 < a.H ? 64 * t1 : a.H) - 64 * t0) * (int)sizeof(T);
            out.run = !Stream && out.bytes == out.step && 16 * RN * out.bytes + 16 <= a.out_lds;
            out.begin();
        }

        u32x4 next[kVec];
        auto ask = [&](int t) {                        // rows 64 t .. of W
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                const uint32_t i = k * threads + threadIdx.x, r = __umulhi(i, a.magic);
                const int h = 64 * t + (int)r < a.H ? 64 * t + (int)r : a.H - 1;
                next[k] = *reinterpret_cast<const u32x4*>(w + (int64_t)h * a.rb + 16 * (i - r * rv));
            }
        };
        auto keep = [&](uint8_t* to) {
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                const uint32_t i = k * threads + threadIdx.x, r = __umulhi(i, a.magic);
                if (r < 64) reinterpret_cast<u32x4*>(to)[((r & 3) * 16 + (r >> 2)) * lv + (i - r * rv)] = next[k];        // by operand
            }
        };
        if (Stream) {
            ask(t0);
            __syncthreads();                           // the item before has been worked off
            keep(ws + (t0 & 1) * (64 * a.ls + 64));
            __syncthreads();
        } else if (group != held_group || t0 != held_from) {
            __syncthreads();
            for (int t = t0; t < t1; ++t) {
                ask(t);
                keep(ws + (t - t0) * 64 * a.ls);
            }
            held_group = group; held_from = t0;
            __syncthreads();
        }
        u32x4 xv[KS][RN];
        uint32_t xc[KS][RN];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int c = 0; c < RN; ++c) {
                const bool in = 4 * s + q < a.nb;
                xc[s][c] = in ? ahead_scale[s][c] >> (8 * q) : 127u;
                xv[s][c] = in ? ahead[s][c] : u32x4{0, 0, 0, 0};
            }
        if (kAhead && item + share.step < share.end) { it = find(item + share.step); ask_rows(it); }
        for (int t = t0; t < t1; ++t) {
            const uint8_t* tile_w = Stream ? ws + (t & 1) * (64 * a.ls + 64) : ws + (t - t0) * 64 * a.ls;
            if (Stream && t + 1 < t1) ask(t + 1);
            f32x4 acc[RN][4];
#pragma unroll
            for (int c = 0; c < RN; ++c)
#pragma unroll
                for (int f = 0; f < 4; ++f) acc[c][f] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (mine > 0)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    u32x4 wv[4];
                    uint32_t wc[4];
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        // a lane without a block at this step reads what lies behind: X has zeros there, the scale is made finite
                        const uint8_t* p = tile_w + (16 * f + m) * a.ls;
                        wv[f] = *reinterpret_cast<const u32x4*>(p + 16 * (4 * s + q));
                        wc[f] = *reinterpret_cast<const uint32_t*>(p + 16 * a.nb + 4 * s) >> (8 * q);
                        if (s == KS - 1) wc[f] = 4 * s + q < a.nb ? wc[f] : 127u;
                    }
#pragma unroll
                    for (int f = 0; f < 4; ++f)
#pragma unroll
                        for (int c = 0; c < RN; ++c)
                            acc[c][f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(xv[s][c]), mx4_operand(wv[f]), acc[c][f], 4, 4,
                                                                                         0, (int)xc[s][c], 0, (int)wc[f]);
                }
            if (Stream && t + 1 < t1) keep(ws + ((t + 1) & 1) * (64 * a.ls + 64));
            if constexpr (Lines) {
                if (mine >= 16 * RN && 64 * t + 64 <= a.H) {
#pragma unroll
                    for (int c = 0; c < RN; ++c) put_whole<T>(y + (16 * c + 4 * q) * ld + 64 * t + 4 * m, ld, acc[c]);
                } else {
#pragma unroll
                    for (int c = 0; c < RN; ++c) put_tile<T>(y + (16 * c + 4 * q) * ld, ld, mine - 16 * c - 4 * q, 64 * t + 4 * m, a.H, true, acc[c]);
                }
            } else if (mine > 0) {
                out.put(t - t0, acc);
                if (!out.run) out.flush_lines(t - t0, t == t0, t + 1 == t1);
                else if (t + 1 == t1) out.flush_run();
            }
            if (Stream) __syncthreads();
        }
    }
}

// The form for wider rows, and for calls of few rows, whose W is better read once by those who need it: a workgroup takes a tile of
// TR rows into LDS and its wavefronts take 16 RN of them by 64 columns of Y at a time, W straight from memory.
template <class T, int TR, int RN>
__global__ void __launch_bounds__(kProdBlock) mx4_product_kernel(ProductArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t xs[];
    constexpr int RS = TR / (16 * RN);
    const Lists lists(a.t, TR);
    const int total = lists.total();
    if (total == 0) return;
    const int wave = threadIdx.x >> 6, l = lane_id(), m = l & 15, q = l >> 4;
    const int tasks = (a.H + 63) / 64 * RS;
    const int most = (tasks + kProdWaves - 1) / kProdWaves;
    int parts = (int)gridDim.x / total;
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    const int64_t items = (int64_t)total * parts;
    const int steps = (a.nb + 3) / 4;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int tile = (int)(item / parts), part = (int)(item - (int64_t)tile * parts);
        const int list = lists.list_of(tile);
        const int64_t r0 = (int64_t)(tile - lists.first_tile(list)) * TR;
        const int64_t left = lists.rows_in(list) - r0;
        const int here = left < TR ? (int)left : TR;
        const u32x4* src = reinterpret_cast<const u32x4*>(a.t.rows[list] + r0 * a.rb);
        __syncthreads();                                   // the tile before has been read
        for (int i = threadIdx.x; i < here * (a.rb / 16); i += kProdBlock) reinterpret_cast<u32x4*>(xs)[i] = src[i];
        __syncthreads();
        const uint8_t* w = a.w + (int64_t)a.t.group[list] * a.H * a.rb;
        const int64_t ld = a.t.ld[list];
        T* y = static_cast<T*>(a.t.y[list]) + r0 * ld;
        const bool wide = ((uintptr_t)a.t.y[list] | (uint64_t)(ld * (int64_t)sizeof(T))) % 16 == 0;
        for (int task = part * kProdWaves + wave; task < tasks; task += parts * kProdWaves) {
            const int h0 = task / RS * 64, c0 = task % RS * (16 * RN);
            if (c0 >= here) continue;
            f32x4 acc[RN][4];
#pragma unroll
            for (int c = 0; c < RN; ++c)
#pragma unroll
                for (int f = 0; f < 4; ++f) acc[c][f] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int s = 0; s < steps; ++s) {
                const bool in = 4 * s + q < a.nb;                  // else the lane has no block at this step: zeros
                const int b = in ? 4 * s + q : a.nb - 1;
                u32x4 wv[4], xv[RN];
                uint32_t wc[4], xc[RN];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    int h = h0 + tile_column(f, m);
                    h = h < a.H ? h : a.H - 1;
                    const uint8_t* p = w + (int64_t)h * a.rb;
                    wv[f] = *reinterpret_cast<const u32x4*>(p + 16 * b);
                    wc[f] = *reinterpret_cast<const uint32_t*>(p + 16 * a.nb + 4 * s) >> (8 * q);
                    if (!in) { wv[f] = u32x4{0, 0, 0, 0}; wc[f] = 127; }
                }
#pragma unroll
                for (int c = 0; c < RN; ++c) {
                    const uint8_t* p = xs + (c0 + 16 * c + m) * a.rb;
                    xv[c] = *reinterpret_cast<const u32x4*>(p + 16 * b);
                    xc[c] = *reinterpret_cast<const uint32_t*>(p + 16 * a.nb + 4 * s) >> (8 * q);
                    if (!in) { xv[c] = u32x4{0, 0, 0, 0}; xc[c] = 127; }
                }
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int c = 0; c < RN; ++c)
                        acc[c][f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(xv[c]), mx4_operand(wv[f]), acc[c][f],
                                                                                     4, 4, 0, (int)xc[c], 0, (int)wc[f]);
            }
#pragma unroll
            for (int c = 0; c < RN; ++c)
                put_tile<T>(y + (c0 + 16 * c + 4 * q) * ld, ld, here - c0 - 16 * c - 4 * q, h0 + 4 * m, a.H, wide, acc[c]);
        }
    }
}

// ---- weight gradient ------------------------------------------------------------------------------

// The rows of all lists, in the order of their groups, are cut into chunks, and the chunks into `splits` runs of equal length.  A
// workgroup has one run and one tile of dW; where its run passes from a group to the next it writes down what it has as piece
// (run + group) and starts again, and the second kernel adds up each group's pieces in the order of the rows.  No atomics: the
// same counts give the same bits.
//
// Both operands have the rows as the axis that is summed over, so their tiles lie in LDS as they lie in memory and are read
// transposed (ds_read_b64_tr_b16).  A chunk's operands are asked for two chunks ahead, into registers; X is unpacked to bf16 on
// its way to LDS, dY cut into its pieces.
constexpr int kGradPad = 16;         // elements behind an LDS row: the four rows that 16 lanes read at once are then 4 x 32 bytes of other banks

struct GradArgs {
    RowTable t;
    float*   pieces;       // [splits + groups][H * D]
    float*   dw;           // [groups][H * D]
    int32_t  D, H, nb, rb;
    int32_t  splits, tiles_d;
    int32_t  chunk;        // rows of a chunk
};

// dY as bf16 numbers that add up to it exactly: one, two of an fp16, three of an fp32.  Cut off rather than rounded, so that no
// finite value becomes infinite; what is not finite is its first piece alone.
template <class T> struct Pieces { static constexpr int n = 1; };
template <> struct Pieces<_Float16> { static constexpr int n = 2; };
template <> struct Pieces<float> { static constexpr int n = 3; };
template <int P>
__device__ __forceinline__ void cut(float x, __bf16 (&out)[P]) {
    const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const float head = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
        out[p] = (__bf16)(p == 0 && !finite ? x : head);
        x = finite ? x - head : 0.0f;
    }
}

// Eight rows of the lane's column: of 16 lanes, lane i names row i/4 and columns 4 (i mod 4) .., and gets column i of four rows.
template <int LD>
__device__ __forceinline__ bf16x8 column8(const __bf16* p) {
    typedef __attribute__((address_space(3))) i16x4* lds4;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 4 * LD));
    const bf16x4 x = __builtin_bit_cast(bf16x4, a), y = __builtin_bit_cast(bf16x4, b);
    return bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

template <class T, int WH, int WD>
struct GradShape {
    static constexpr int P = Pieces<T>::n;
    static constexpr int rows = P == 1 ? 64 : 32;                    // of a chunk: two buffers of it fit the LDS
    static constexpr int threads = 64 * WH * WD;
    static constexpr int th = 64 * WH, td = 64 * WD;                 // the tile of dW: a wavefront has 64 x 64 of it
    static constexpr int ly = th + kGradPad, lx = td + kGradPad;     // elements of an LDS row
    static constexpr int buffer = rows * (P * ly + lx);              // elements of a buffer
    static constexpr int lds = 2 * buffer * 2;
    static constexpr int ve = 16 / (int)sizeof(T);                   // elements of a 16-byte vector of dY
    static constexpr int ny = rows * th / ve / threads;              // vectors of dY, blocks of X per thread and chunk
    static constexpr int nx = (rows * 2 * WD + threads - 1) / threads;
};

template <class T, int WH, int WD>
__global__ void __launch_bounds__(64 * WH * WD) mx4_grad_kernel(GradArgs a) {
    typedef GradShape<T, WH, WD> S;
    constexpr int P = S::P;
    extern __shared__ __attribute__((aligned(16))) __bf16 lds[];
    const Lists lists(a.t, S::rows);
    const int total = lists.total();
    const int splits = a.splits < total ? a.splits : total;
    const int tiles = (int)gridDim.x / a.splits;
    // the tiles of a run, which read the same rows, share an XCD's L2
    const int id = (int)own_piece();
    const int tile = id % tiles, split = id / tiles;
    if (split >= splits) return;
    const int from = (int)((int64_t)split * total / splits), to = (int)((int64_t)(split + 1) * total / splits);
    const int h0 = tile / a.tiles_d * S::th, d0 = tile % a.tiles_d * S::td;
    const int wave = threadIdx.x >> 6, l = lane_id();
    const int wh = wave / WD * 64, wd = wave % WD * 64;

    u32x4 ry[2][S::ny], rx[2][S::nx];
    uint32_t rs[2][S::nx];
    int here[2], group[2];

    auto load = [&](int u, int chunk) {
        const int list = lists.list_of(chunk);
        const int64_t r0 = (int64_t)(chunk - lists.first_tile(list)) * S::rows;
        const int64_t left = lists.rows_in(list) - r0;
        here[u] = left < S::rows ? (int)left : S::rows;
        group[u] = a.t.group[list];
        const int64_t ld = a.t.ld[list];
        const T* y = static_cast<const T*>(a.t.y[list]) + r0 * ld;
        const uint8_t* x = a.t.rows[list] + r0 * a.rb;
        // rows behind the last and columns behind H or D: others in their place; put() clears the rows, and those columns of dW
        // are not written
        if (((uintptr_t)a.t.y[list] | (uint64_t)(ld * (int64_t)sizeof(T))) % 16 == 0 && a.H % S::ve == 0) {
#pragma unroll
            for (int k = 0; k < S::ny; ++k) {
                const int i = k * S::threads + (int)threadIdx.x;
                int r = i / (S::th / S::ve), h = h0 + i % (S::th / S::ve) * S::ve;
                r = r < here[u] ? r : here[u] - 1;
                h = h < a.H ? h : 0;
                ry[u][k] = *reinterpret_cast<const u32x4*>(y + r * ld + h);
            }
        } else {
#pragma unroll
            for (int k = 0; k < S::ny; ++k) {
                const int i = k * S::threads + (int)threadIdx.x;
                int r = i / (S::th / S::ve);
                const int h = h0 + i % (S::th / S::ve) * S::ve;
                r = r < here[u] ? r : here[u] - 1;
                T v[S::ve];
#pragma unroll
                for (int j = 0; j < S::ve; ++j) v[j] = y[r * ld + (h + j < a.H ? h + j : a.H - 1)];
                ry[u][k] = __builtin_bit_cast(u32x4, v);
            }
        }
#pragma unroll
        for (int k = 0; k < S::nx; ++k) {
            const int i = k * S::threads + (int)threadIdx.x;
            int r = i / (2 * WD), b = d0 / 32 + i % (2 * WD);
            r = r < here[u] ? r : here[u] - 1;
            b = b < a.nb ? b : a.nb - 1;
            const uint8_t* p = x + r * a.rb;
            rx[u][k] = *reinterpret_cast<const u32x4*>(p + 16 * b);
            rs[u][k] = p[16 * a.nb + b];
        }
    };
    auto put = [&](int u) {
        __bf16* gy = lds + u * S::buffer;
        __bf16* gx = gy + P * S::rows * S::ly;
#pragma unroll
        for (int k = 0; k < S::ny; ++k) {
            const int i = k * S::threads + (int)threadIdx.x;
            const int r = i / (S::th / S::ve), h = i % (S::th / S::ve) * S::ve;
            const u32x4 raw = r < here[u] ? ry[u][k] : u32x4{0, 0, 0, 0};
            if constexpr (P == 1) {
                *reinterpret_cast<u32x4*>(gy + r * S::ly + h) = raw;
            } else {
                struct Vec { T v[S::ve]; } in = __builtin_bit_cast(Vec, raw);
                struct Cut { __bf16 v[S::ve]; } out[P];
#pragma unroll
                for (int j = 0; j < S::ve; ++j) {
                    __bf16 c[P];
                    cut<P>((float)in.v[j], c);
#pragma unroll
                    for (int p = 0; p < P; ++p) out[p].v[j] = c[p];
                }
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
            const int r = i / (2 * WD);
            if (S::rows * 2 * WD % S::threads && r >= S::rows) continue;
            const float s = r < here[u] ? mx4_scale(rs[u][k]) : 0.0f;
            const u32x4 c = r < here[u] ? rx[u][k] : u32x4{0, 0, 0, 0};
            __bf16* to_x = gx + r * S::lx + i % (2 * WD) * 32;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], s, 1),
                             v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], s, 3);
                *reinterpret_cast<bf16x8*>(to_x + 8 * j) = bf16x8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
            }
        }
    };

    f32x4 acc[4][4];
    auto clear = [&]() {
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[f][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    auto flush = [&](int g) {
        float* out = a.pieces + (int64_t)(split + g) * a.H * a.D;
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int h = h0 + wh + 16 * f + 4 * (l >> 4) + i, d = d0 + wd + 16 * c + (l & 15);
                    if (h < a.H && d < a.D) out[(int64_t)h * a.D + d] = acc[f][c][i];
                }
    };
    const int n = to - from;
    load(0, from);
    if (n > 1) load(1, from + 1);
    clear();
    int now = group[0];
    for (int j = 0; j < n; j += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (j + u >= n) break;
            if (group[u] != now) { flush(now); clear(); now = group[u]; }
            put(u);
            __syncthreads();         // the other buffer has been read by all before this one is read by any
            if (j + u + 2 < n) load(u, from + j + u + 2);
            const __bf16* gy = lds + u * S::buffer;
            const __bf16* gx = gy + P * S::rows * S::ly;
#pragma unroll
            for (int k = 0; k < S::rows; k += 32) {
                const int row = k + 8 * (l >> 4) + ((l & 15) >> 2), col = 4 * (l & 3);
                bf16x8 bx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) bx[c] = column8<S::lx>(gx + row * S::lx + col + wd + 16 * c);
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const bf16x8 ay = column8<S::ly>(gy + (p * S::rows + row) * S::ly + col + wh + 16 * f);
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ay, bx[c], acc[f][c], 0, 0, 0);
                    }
            }
        }
    }
    flush(now);
}

// Each element's pieces are added by four lanes, then the four sums: always in the same order.
constexpr int kSumLanes = 4;
__global__ void __launch_bounds__(256) mx4_grad_sum_kernel(GradArgs a) {
    const Lists lists(a.t, a.chunk);
    const int total = lists.total(), group = blockIdx.y;
    const int splits = a.splits < total ? a.splits : total;
    const int64_t size = (int64_t)a.H * a.D;
    // the chunks of the group: from its first list's first to its last list's last
    const uint64_t mine = __ballot(lane_id() < a.t.n_lists && (int)a.t.group[lane_id()] == group && lists.tiles > 0);
    int lo = 0, hi = -1;
    if (mine) {
        const int first = lists.first_tile(__builtin_ctzll(mine)), last = __builtin_amdgcn_readlane(lists.upto, 63 - __builtin_clzll(mine)) - 1;
        lo = (int)((((int64_t)first + 1) * splits - 1) / total);
        hi = (int)((((int64_t)last + 1) * splits - 1) / total);
    }
    // 16 elements side by side, the four lanes of each 16 apart
    const int part = (lane_id() >> 4) & (kSumLanes - 1);
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), waves = (int64_t)gridDim.x * 4;
    for (int64_t i0 = wave * 16; i0 < size; i0 += waves * 16) {
        const int64_t i = i0 + (lane_id() & 15);
        const float* p = a.pieces + (i < size ? i : size - 1);
        double sum = 0.0;
#pragma unroll 8
        for (int s = lo + part; s <= hi; s += kSumLanes) sum += p[(int64_t)(s + group) * size];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (part == 0 && i < size) a.dw[group * size + i] = (float)sum;
    }
}

template <class T, int WH, int WD>
static int launch_grad(spp_ctx* ctx, GradArgs& a, int n_groups, bool sum_only) {
    typedef GradShape<T, WH, WD> S;
    auto kernel = mx4_grad_kernel<T, WH, WD>;
    a.chunk = S::rows;
    a.tiles_d = (a.D + S::td - 1) / S::td;
    const int64_t tiles = (int64_t)a.tiles_d * ((a.H + S::th - 1) / S::th), size = (int64_t)a.H * a.D;
    int64_t chunks = 0;
    for (int j = 0; j < a.t.n_lists; ++j) chunks += (a.t.n[j] + (int64_t)S::rows - 1) / S::rows;
    const int fit = 163840 / S::lds, wish = 8 / (WH * WD);
    const int64_t at_once = (int64_t)ctx->num_cu * (fit < 1 || wish < 1 ? 1 : fit < wish ? fit : wish);
    int64_t splits = at_once / tiles;
    if (splits > (chunks + 1) / 2) splits = (chunks + 1) / 2;
    a.splits = (int32_t)(splits < 1 ? 1 : splits);
    SPP_TRY(ctx->gradws.reserve((size_t)(a.splits + n_groups) * size * sizeof(float)));
    a.pieces = ctx->gradws.as<float>();
    if (!sum_only) {
        if (S::lds > 65536) SPP_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::lds));
        kernel<<<(unsigned)(a.splits * tiles), S::threads, S::lds, ctx->stream>>>(a);
        SPP_HIP(hipGetLastError());
    }
    const int64_t sums = (size + 63) / 64;
    mx4_grad_sum_kernel<<<dim3((unsigned)(sums < 8192 ? sums : 8192), n_groups), 256, 0, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}
template <class T, int WH>
static int grad_by_width(spp_ctx* ctx, GradArgs& a, int n_groups, bool sum_only) {
    // as few tiles as 128 columns allow, of as few wavefronts as these need
    const int tiles = (a.D + 127) / 128;
    return (a.D + tiles - 1) / tiles > 64 ? launch_grad<T, WH, 2>(ctx, a, n_groups, sum_only) : launch_grad<T, WH, 1>(ctx, a, n_groups, sum_only);
}
template <class T>
static int grad_of(spp_ctx* ctx, GradArgs& a, int n_groups, bool sum_only) {
    const int tiles = (a.H + 255) / 256, wh = (a.H + 64 * tiles - 1) / (64 * tiles);
    return wh == 1 ? grad_by_width<T, 1>(ctx, a, n_groups, sum_only) : wh == 2 ? grad_by_width<T, 2>(ctx, a, n_groups, sum_only)
         : wh == 3 ? grad_by_width<T, 3>(ctx, a, n_groups, sum_only) : grad_by_width<T, 4>(ctx, a, n_groups, sum_only);
}

int row_table(const char* who, const spp_row_list* lists, int32_t n_lists, int32_t n_groups, int32_t D, int32_t H, int32_t type,
              RowTable& t, int64_t* most) {
    SPP_CHECK(n_lists >= 0 && n_lists <= kRowLists && (lists || n_lists == 0), SPP_E_ARG, "%s: %d lists (at most %d)", who, n_lists, kRowLists);
    SPP_CHECK(n_groups >= 1 && n_groups <= kRowLists, SPP_E_ARG, "%s: %d groups (1 .. %d)", who, n_groups, kRowLists);
    SPP_CHECK(D >= 1 && D <= SPP_MX4_MAX_COLS && H >= 1 && H <= SPP_MAX_HIDDEN, SPP_E_ARG, "%s: D = %d (1 .. %d), H = %d (1 .. %d)", who, D,
              SPP_MX4_MAX_COLS, H, SPP_MAX_HIDDEN);
    SPP_CHECK(is_type(type), SPP_E_ARG, "%s: element type %d", who, type);
    memset(&t, 0, sizeof(t));
    *most = 0;
    for (int j = 0; j < n_lists; ++j) {
        const spp_row_list& a = lists[j];
        SPP_CHECK(a.n >= 0 && a.n <= 0x7FFFFFFFll && a.ld >= H && a.group >= 0 && a.group < n_groups, SPP_E_ARG,
                  "%s: list %d: n = %lld, ld = %lld, group = %d", who, j, (long long)a.n, (long long)a.ld, a.group);
        SPP_CHECK(a.n == 0 || (a.d_rows && a.d_y), SPP_E_ARG, "%s: list %d: null argument", who, j);
        SPP_CHECK((uintptr_t)a.d_rows % 16 == 0 && (uintptr_t)a.d_y % type_bytes(type) == 0 && (uintptr_t)a.d_n % 8 == 0, SPP_E_ARG,
                  "%s: list %d: rows must be 16-byte aligned, Y to its type and the count to 8 bytes", who, j);
        *most += a.n;
    }
    for (int g = 0, k = 0; g < n_groups; ++g)               // the lists in the order of their groups
        for (int j = 0; j < n_lists; ++j) {
            if (lists[j].group != g) continue;
            t.rows[k] = static_cast<const uint8_t*>(lists[j].d_rows);
            t.y[k] = lists[j].d_y; t.d_n[k] = lists[j].n ? lists[j].d_n : nullptr; t.ld[k] = lists[j].ld;
            t.n[k] = (int32_t)lists[j].n; t.group[k] = (uint8_t)g;
            ++k;
        }
    t.n_lists = n_lists;
    return SPP_OK;
}

template <class T, int TR, int RN>
static int launch_product(spp_ctx* ctx, const ProductArgs& a) {
    const int lds = TR * a.rb;
    auto kernel = mx4_product_kernel<T, TR, RN>;
    if (lds > 65536) SPP_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    int64_t tiles = 0;
    for (int j = 0; j < a.t.n_lists; ++j) tiles += (a.t.n[j] + (int64_t)TR - 1) / TR;
    const int64_t parts = ((a.H + 63) / 64 * (TR / (16 * RN)) + kProdWaves - 1) / kProdWaves;
    const int64_t want = tiles * parts, most = (int64_t)ctx->num_cu * 4;
    kernel<<<(unsigned)(want < most ? want : most), kProdBlock, lds, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}
constexpr int kHeldW = 65536;            // LDS for a W that stays
constexpr int kRowOut = 768;             // bytes of Y's rows that go out in one run
template <class T, int KS, int RN, int WAVES, bool Stream, bool Lines>
static int launch_rows_as(spp_ctx* ctx, ProductArgs& a) {
    auto kernel = mx4_rows_kernel<T, KS, RN, WAVES, Stream, Lines>;
    const int ht = (a.H + 63) / 64, row = a.H * (int)sizeof(T);
    a.w_lds = Stream ? 2 * (64 * a.ls + 64) : ht * 64 * a.ls + 64;
    a.out_lds = 16 * RN * RowsOut<T, RN>::kPitch;
    if (!Stream && row <= kRowOut && a.out_lds < 16 * RN * row + 16) a.out_lds = 16 * RN * row + 16;
    const int lds = a.w_lds + (Lines ? 0 : WAVES * a.out_lds);
    if (lds > 65536) SPP_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    int64_t tiles = 0;
    for (int j = 0; j < a.t.n_lists; ++j) tiles += (a.t.n[j] + (int64_t)(WAVES * 16 * RN) - 1) / (WAVES * 16 * RN);
    // Workgroups per CU.  A stream of whole lines is fastest from few wavefronts (2.56M rows 128 -> 256: 221 us with one workgroup per CU,
    // 245 to 250 with two to eight) once each has enough to do; with less, or two steps of columns and more to wait for (800k
    // rows 256 -> 256: 102, 86, 92 us with one, two, three), more are better.  Rows of other lengths take unequal times: many
    // workgroups even them out where there are many more tiles (2.56M rows 100 -> 172: 236 us with four per CU, 197 with
    // sixteen; 300k rows in fp32 42 and 49).
    a.fill = 2 * ctx->num_cu;
    const int64_t want = tiles >= a.fill ? tiles : tiles * ht < a.fill ? tiles * ht : a.fill;
    const int per_cu = Stream ? 2 : Lines ? (KS > 1 ? 2 : tiles >= 8 * ctx->num_cu ? 1 : 3) : tiles >= 64 * ctx->num_cu ? 16 : 4;
    const int64_t most = (int64_t)ctx->num_cu * per_cu;
    kernel<<<(unsigned)(want < most ? want : most), 64 * WAVES, lds, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}
template <class T, int KS>
static int launch_rows(spp_ctx* ctx, ProductArgs& a) {
    const int ht = (a.H + 63) / 64;
    // Y's rows begin with a line each: stored as they come, 128 or 256 bytes of a row at a time
    bool lines = true;
    for (int j = 0; j < a.t.n_lists; ++j) lines = lines && ((uintptr_t)a.t.y[j] | (uint64_t)(a.t.ld[j] * (int64_t)sizeof(T))) % 128 == 0;
    if (ht * 64 * a.ls <= kHeldW)
        return lines ? launch_rows_as<T, KS, 2, 4, false, true>(ctx, a) : launch_rows_as<T, KS, 1, 4, false, false>(ctx, a);
    return lines ? launch_rows_as<T, KS, 2, 8, true, true>(ctx, a) : launch_rows_as<T, KS, KS >= 4 ? 1 : 2, 8, true, false>(ctx, a);
}
constexpr int kFewRows = 64;
template <class T>
static int product_of(spp_ctx* ctx, ProductArgs& a, int64_t most) {
    if (most <= kFewRows) return launch_product<T, 64, 1>(ctx, a);
    const int rv = a.rb / 16;
    a.ls = 16 * (rv | 1);
    a.magic = (uint32_t)((0x100000000ull + rv - 1) / rv);
    switch ((a.nb + 3) / 4) {
        case 1: return launch_rows<T, 1>(ctx, a);
        case 2: return launch_rows<T, 2>(ctx, a);
        case 3: return launch_rows<T, 3>(ctx, a);
        case 4: return launch_rows<T, 4>(ctx, a);
        case 5: return launch_rows<T, 5>(ctx, a);
        case 6: return launch_rows<T, 6>(ctx, a);
        default: return a.rb <= 544 ? launch_product<T, 128, 4>(ctx, a) : launch_product<T, 64, 4>(ctx, a);
    }
}

}  // namespace spp

extern "C" int spp_mx4_product(spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, const void* d_weights, int32_t n_groups,
                               int32_t D, int32_t H, int32_t type, uint32_t flags) {
    using namespace spp;
    SPP_CHECK(ctx && d_weights, SPP_E_ARG, "spp_mx4_product: null argument");
    SPP_CHECK((uintptr_t)d_weights % 16 == 0, SPP_E_ARG, "spp_mx4_product: weights must be 16-byte aligned");
    ProductArgs a;
    int64_t most = 0;
    SPP_TRY(row_table("spp_mx4_product", lists, n_lists, n_groups, D, H, type, a.t, &most));
    if (most > 0) {
        a.w = static_cast<const uint8_t*>(d_weights);
        a.D = D; a.H = H; a.nb = mx4_blocks(D); a.rb = mx4_bytes(D);
        SPP_HIP(hipSetDevice(ctx->device));
        ScopedTimer timer(ctx, SPP_T_LAYER, ctx->stream);
        SPP_TRY(type == SPP_F32 ? product_of<float>(ctx, a, most) : type == SPP_F16 ? product_of<_Float16>(ctx, a, most) : product_of<__bf16>(ctx, a, most));
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}

extern "C" int spp_mx4_weight_grad(spp_ctx* ctx, const spp_row_list* lists, int32_t n_lists, int32_t n_groups, int32_t D, int32_t H,
                                   int32_t type, float* d_grad, uint32_t flags) {
    using namespace spp;
    SPP_CHECK(ctx && d_grad, SPP_E_ARG, "spp_mx4_weight_grad: null argument");
    SPP_CHECK((uintptr_t)d_grad % 4 == 0, SPP_E_ARG, "spp_mx4_weight_grad: the gradient must be 4-byte aligned");
    GradArgs a;
    int64_t most = 0;
    SPP_TRY(row_table("spp_mx4_weight_grad", lists, n_lists, n_groups, D, H, type, a.t, &most));
    SPP_HIP(hipSetDevice(ctx->device));
    a.dw = d_grad; a.D = D; a.H = H; a.nb = mx4_blocks(D); a.rb = mx4_bytes(D);
    hipStream_t st = ctx->stream;
    ScopedTimer timer(ctx, SPP_T_LAYER, st);
    SPP_TRY(type == SPP_F32 ? grad_of<float>(ctx, a, n_groups, most == 0) : type == SPP_F16 ? grad_of<_Float16>(ctx, a, n_groups, most == 0)
                                                                                          : grad_of<__bf16>(ctx, a, n_groups, most == 0));
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(st));
    return SPP_OK;
}
