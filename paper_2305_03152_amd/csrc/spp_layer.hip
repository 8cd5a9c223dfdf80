// The layer that reads feature rows in MXFP4, over up to 64 lists of rows whose lengths may be known on the device only (the
// minibatches that a pipeline keeps in flight; rows of several kinds, each kind with a matrix of its own):
//
//   Y_j = X_j W[g_j]^T           X_j [n_j, D] and W[g] [H, D] in MXFP4, Y_j fp32, fp16 or bf16
//
// Two values of the format have 6 bits as a product: the products of the matrix instruction are exact, sums are formed in fp32,
// and Y is rounded once.
#include "spp_mx4.h"

namespace spp {

// ---- product --------------------------------------------------------------------------------------

struct ProductArgs {
    RowTable       t;
    const uint8_t* w;
    int32_t        D, H, nb, rb;
    int32_t        ls;           // bytes of a row of W in LDS: an odd number of 16, so that a lane group's 16 rows lie in banks of their own
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
// written by whole 16-byte pieces, side by side; the ends of a row or a run, less than a piece, by element.  Stored as they come, 2.56M
// rows 100 -> 172 in bf16 took 432 us, so 230 to 237 (4.5 TB/s).  Where W is a stream rows go out by lines, and the narrower their LDS writes
// have to be the longer it takes: 400k rows 256 -> 1001 313 us, -> 1002 263, -> 1004 242, -> 1008 225, -> 1024, stored as they come, 154.
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
// of what moves, written once, past the L2, which reads of the next rows would otherwise share with it (2.56M rows 128 -> 256 301 us
// with plain stores, 250 so, both from a cached X).  Bound by HBM for narrow rows: 2.56M rows 128 -> 256 in bf16 264 us, 5.6 TB/s;
// 400k rows 256 -> 1024 157 us, 5.7 TB/s; for wide ones by the wavefronts' waits for each other at every 64 columns: 390k
// rows 768 -> 1024 225 to 230 us, 2.7 PFLOP/s.  Two rows of 16 per wavefront, three where kManyRows says so: one reads W from LDS twice as
// often, four (768 -> 1024) leave a wavefront per SIMD.  Eight wavefronts share a stream of W, four where rows are short (256 -> 1024
// 167 and 157 us, 768 -> 1024 with two rows of 16 250 and 279).
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

// The form for wider rows, of which a wavefront's registers would not hold enough: a workgroup takes a tile of TR rows into LDS and its
// wavefronts take 16 RN of them by 64 columns of Y at a time, W straight from memory.  300k rows 800 -> 256 in bf16: 158 us, 1.7 TB/s,
// 1024 -> 256 205, 800 -> 1024 463; 50k rows 4096 -> 256 188.  Bound by the way of W's blocks from the L2, a step of 128 columns at a
// time: every wavefront fetches them itself, and nothing is asked for ahead.
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
    SPP_CHECK(*most <= (int64_t)1 << 35, SPP_E_ARG, "%s: the lists' n add up to %lld (at most 2^35)", who, (long long)*most);
    int at[kRowLists + 1] = {};                             // the lists in the order of their groups
    for (int j = 0; j < n_lists; ++j) ++at[lists[j].group + 1];
    for (int g = 0; g < n_groups; ++g) at[g + 1] += at[g];
    for (int j = 0; j < n_lists; ++j) {
        const int k = at[lists[j].group]++;
        t.rows[k] = static_cast<const uint8_t*>(lists[j].d_rows);
        t.y[k] = lists[j].d_y; t.d_n[k] = lists[j].n ? lists[j].d_n : nullptr; t.ld[k] = lists[j].ld;
        t.n[k] = (int32_t)lists[j].n; t.group[k] = (uint8_t)lists[j].group;
    }
    t.n_lists = n_lists;
    return SPP_OK;
}

template <class T, int TR, int RN>
static int launch_product(spp_ctx* ctx, const ProductArgs& a) {
    const int lds = TR * a.rb;
    auto kernel = mx4_product_kernel<T, TR, RN>;
    static LdsLimit limit;
    SPP_TRY(limit.allow(ctx, reinterpret_cast<const void*>(kernel), lds));
    int64_t tiles = 0;
    for (int j = 0; j < a.t.n_lists; ++j) tiles += (a.t.n[j] + (int64_t)TR - 1) / TR;
    const int64_t parts = ((a.H + 63) / 64 * (TR / (16 * RN)) + kProdWaves - 1) / kProdWaves;
    const int64_t want = tiles * parts, most = (int64_t)ctx->num_cu * 4;
    kernel<<<(unsigned)(want < most ? want : most), kProdBlock, lds, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}
constexpr int kHeldW = 65536;            // LDS for a W that stays: two workgroups fit a CU
// Rows per CU from which wide rows with a result of 16 bits go 48 to a wavefront instead of 32: W is read from LDS two thirds as
// often, but tiles are larger and the last round of them emptier.  768 -> 1024, 32 and 48: 100k rows 75 and 92 us, 200k 149 both, 300k
// 209 and 200, 390k 247 and 230, 800k 533 and 489; 500 -> 1024: 100k 58 and 71, 200k 111 both, 390k 191 and 176, 800k 410 and 387.
// (150k rows, a round less: 110 and 100, not taken.)  In fp32 the stores bound both: 390k rows 355 and 362.
constexpr int kManyRows = 2 * 8 * 48;
constexpr int kRowOut = 768;             // bytes of Y's rows that go out in one run
template <class T, int KS, int RN, int WAVES, bool Stream, bool Lines>
static int launch_rows_as(spp_ctx* ctx, ProductArgs& a) {
    auto kernel = mx4_rows_kernel<T, KS, RN, WAVES, Stream, Lines>;
    const int ht = (a.H + 63) / 64, row = a.H * (int)sizeof(T);
    a.w_lds = Stream ? 2 * (64 * a.ls + 64) : ht * 64 * a.ls + 64;
    a.out_lds = 16 * RN * RowsOut<T, RN>::kPitch;
    if (!Stream && row <= kRowOut && a.out_lds < 16 * RN * row + 16) a.out_lds = 16 * RN * row + 16;
    const int lds = a.w_lds + (Lines ? 0 : WAVES * a.out_lds);
    static LdsLimit limit;
    SPP_TRY(limit.allow(ctx, reinterpret_cast<const void*>(kernel), lds));
    int64_t tiles = 0;
    for (int j = 0; j < a.t.n_lists; ++j) tiles += (a.t.n[j] + (int64_t)(WAVES * 16 * RN) - 1) / (WAVES * 16 * RN);
    // Workgroups per CU.  Many tiles are fastest with a workgroup each (2.56M rows 128 -> 256: 264 us, 285 with one workgroup per CU
    // that goes over its tiles, 298 to 302 with two to sixteen); some with one per CU; few with what runs at once.  With 1, 2, 3, 8 and 128
    // per CU, 128 -> 256: 200k rows 23.4, 22.5, 24.1, 26.1, 26.2 us; 270k 30.3, 31.4, 33.6, 31.6, 32.6; 500k 47.9, 47.4, 47.7, 48.3, 48.7;
    // 540k 53.3, 55.2, 57.3, 55.6, 53.7; 800k 73.7, 74.5, 76.0, 77.3, 74.1.  Of other shapes: 256 -> 256 200k 29.4, 26.2, 27.5, 30.6, 30.5;
    // 400k 49.6, 44.1, 47.8, 47.1, 49.7; 800k 110, 108, 111, 104, 104; 32 -> 64 200k 12.3, 8.7, 8.3, 10.8, 10.7; 400k 19.6, 14.1, 12.6, 15.3,
    // 17.2; 800k 33.4, 23.2, 21.8, 24.3, 30.3.  (The limits, 262k and 524k rows, are those of 128 -> 256, and within a few per cent there;
    // narrow rows would be up to a third faster with three throughout.)
    // Rows of other lengths take unequal times: many workgroups even them out where there are many more tiles (2.56M rows
    // 100 -> 172: 289 us with four per CU, 238 with 32; 300k rows in fp32 42 and 49).
    a.fill = 2 * ctx->num_cu;
    const int64_t want = tiles >= a.fill ? tiles : tiles * ht < a.fill ? tiles * ht : a.fill;
    const int64_t load = tiles / ctx->num_cu;
    const int per_cu = Stream ? 2 : Lines ? (load >= 16 ? 128 : load >= 8 ? 1 : 3) : load >= 64 ? 32 : 4;
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
    if constexpr (KS >= 4 && sizeof(T) == 2) {
        int64_t rows = 0;
        for (int j = 0; j < a.t.n_lists; ++j) rows += a.t.n[j];
        if (lines && rows >= kManyRows * ctx->num_cu) return launch_rows_as<T, KS, 3, 8, true, true>(ctx, a);
    }
    return lines ? launch_rows_as<T, KS, 2, KS <= 3 ? 4 : 8, true, true>(ctx, a) : launch_rows_as<T, KS, KS >= 4 ? 1 : 2, 8, true, false>(ctx, a);
}
template <class T>
static int product_of(spp_ctx* ctx, ProductArgs& a) {
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
        SPP_TRY(type == SPP_F32 ? product_of<float>(ctx, a) : type == SPP_F16 ? product_of<_Float16>(ctx, a) : product_of<__bf16>(ctx, a));
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}
