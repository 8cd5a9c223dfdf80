// How a wavefront's results of 16x16 products go to memory: straight from registers where rows begin with a line each, else by way of LDS.
#pragma once

#include "spp_mx4.h"

namespace spp {

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

}  // namespace spp
