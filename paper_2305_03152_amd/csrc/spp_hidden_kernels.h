// The kernels of the layers on hidden rows and what chooses between them; one source per layer instantiates them.
#pragma once

#include "spp_hidden.h"

namespace spp {

// Bytes behind a row in LDS, its scales among them.  The wavefront reads 16 bytes of 16 rows and four places each, eight lanes at a time and of these
// half from one place and half from the next: rows an even number of 16 bytes apart, but not of 32, put them in banks of their own (16
// bytes behind a row each read took twice its time).
constexpr int kLdsPad = 32;

// ---- W and X in LDS --------------------------------------------------------------------------------

// The form for rows of any length.  A workgroup takes 128 rows of X by 128 columns: of the product, or 64 of the gate's and the same 64 of the other
// factor.  Steps of 128 columns of X and W go through LDS, the next asked for while one is multiplied: bound by that turn, a wait and a barrier a
// step, by one workgroup a CU, whose LDS holds no second one.  In bf16 300k rows 1100 -> 256 499 us, 340 TFLOP/s; 50k 4096 -> 256 369, gated 606, its
// gradient 620.
constexpr int kTileRows = 128, kTileBlock = 256, kTileLd = kFp8Block + kLdsPad;
constexpr int kTileBuffer = 2 * kTileRows * kTileLd + 2 * kTileRows;       // rows of X, rows of W, their scales

template <class T, int Mode>
__global__ void __launch_bounds__(kTileBlock) hidden_tile_kernel(HiddenArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Lists lists(a.t, kTileRows);
    const int total = lists.total();
    if (total == 0) return;
    const int wave = threadIdx.x >> 6, l = lane_id(), m = l & 15, q = l >> 4;
    constexpr int cols = Mode == kProduct ? 128 : 64;
    const int parts = (a.H + cols - 1) / cols;
    const Share share((int64_t)total * parts);
    for (int64_t item = share.at; item < share.end; item += share.step) {
        const int tile = (int)(item / parts), h0 = (int)(item - (int64_t)tile * parts) * cols;
        const int list = lists.list_of(tile);
        const int64_t r0 = (int64_t)(tile - lists.first_tile(list)) * kTileRows;
        const int64_t left = lists.rows_in(list) - r0;
        const int here = left < kTileRows ? (int)left : kTileRows;
        const uint8_t* x = a.t.rows[list] + r0 * a.rb;
        const uint8_t* w = a.w + (int64_t)a.t.group[list] * a.H * (Mode == kProduct ? 1 : 2) * a.rb;
        // Row r of the 128 of W: a column of the result.
        auto w_row = [&](int r) {
            int h = h0 + (Mode == kProduct ? r : r & 63);
            h = h < a.H ? h : a.H - 1;
            return w + (int64_t)(Mode == kProduct || r < 64 ? h : a.H + h) * a.rb;
        };
        u32x4 next[8];
        uint8_t next_scale;
        auto ask = [&](int s) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = k * kTileBlock + (int)threadIdx.x, r = i >> 3, at = 128 * s + 16 * (i & 7);
                const bool in = at < a.cb;
                next[k] = *reinterpret_cast<const u32x4*>(x + (int64_t)(r < here ? r : here - 1) * a.rb + (in ? at : 0));
                next[4 + k] = *reinterpret_cast<const u32x4*>(w_row(r) + (in ? at : 0));
                if (!in) next[k] = next[4 + k] = u32x4{0, 0, 0, 0};
            }
            const int r = (int)threadIdx.x & 127;
            next_scale = (threadIdx.x < 128 ? x + (int64_t)(r < here ? r : here - 1) * a.rb : w_row(r))[a.cb + s];
        };
        // by operand: columns 4m + f of each 64 as row 16 f + m
        auto operand = [](int r) { return (r & 64) + (r & 3) * 16 + ((r & 63) >> 2); };
        auto keep = [&](uint8_t* to) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = k * kTileBlock + (int)threadIdx.x, r = i >> 3, at = 16 * (i & 7);
                *reinterpret_cast<u32x4*>(to + r * kTileLd + at) = next[k];
                *reinterpret_cast<u32x4*>(to + (kTileRows + operand(r)) * kTileLd + at) = next[4 + k];
            }
            const int r = (int)threadIdx.x & 127;
            to[2 * kTileRows * kTileLd + (threadIdx.x < 128 ? r : 128 + operand(r))] = next_scale;
        };
        f32x4 acc[2][8];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int f = 0; f < 8; ++f) acc[c][f] = f32x4{0.f, 0.f, 0.f, 0.f};
        ask(0);
        __syncthreads();                                 // the item before has been worked off
        for (int s = 0; s < a.steps; ++s) {
            uint8_t* buffer = lds + (s & 1) * kTileBuffer;
            keep(buffer);
            if (s + 1 < a.steps) ask(s + 1);
            __syncthreads();                             // (and the buffer of the step after next has been read by all)
            const uint8_t* scales = buffer + 2 * kTileRows * kTileLd;
            auto operand_at = [&](int row) {
                const uint8_t* p = buffer + row * kTileLd + 16 * q;
                return Operand{*reinterpret_cast<const u32x4*>(p), *reinterpret_cast<const u32x4*>(p + 64), scales[row]};
            };
            Operand xv[2], wv[8];
#pragma unroll
            for (int c = 0; c < 2; ++c) xv[c] = operand_at(32 * wave + 16 * c + m);
#pragma unroll
            for (int f = 0; f < 8; ++f) wv[f] = operand_at(kTileRows + 16 * f + m);
            multiply<0>(acc, xv, wv);
        }
        const Results<T, Mode> out(a, list);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int row = 32 * wave + 16 * c + 4 * q;
            f32x4(&one)[4] = reinterpret_cast<f32x4(&)[4]>(acc[c][0]);
            f32x4(&two)[4] = reinterpret_cast<f32x4(&)[4]>(acc[c][4]);
            f32x4 dy[4];
            if constexpr (Mode == kGatedGrad) out.get(a, r0 + row, here - row, h0 + 4 * m, dy);
            combine<Mode>(a.act, one, two, dy);
            if constexpr (Mode == kProduct) {
                out.put(a, r0 + row, here - row, h0 + 4 * m, one);
                out.put(a, r0 + row, here - row, h0 + 64 + 4 * m, two);
            } else {
                out.put(a, r0 + row, here - row, h0 + 4 * m, one);
                if constexpr (Mode == kGatedGrad) out.put_second(a, r0 + row, here - row, h0 + 4 * m, two);
            }
        }
    }
}

// ---- W in LDS --------------------------------------------------------------------------------------

// The form for weights that LDS holds.  A wavefront keeps its 16 RN rows of X in registers, all columns of them, and goes over the columns of
// the result 64 at a time (64 of the gate's and the same 64 of the other factor); a workgroup's wavefronts share W and wait for each other only
// where the matrix changes.  X is asked for an item ahead and read once, results are written once, past the L2.  The product of many rows is bound by
// HBM: 2.5M rows 256 -> 256 in bf16 406 us, 4.8 TB/s (the same reads and writes without the products 390).  The gated layer, 717, is by the
// vector pipe, which decodes W for every 32 rows of X and forms the activation (67 % busy, the matrix pipe 42 %); its gradient, 1109, by both (the same reads
// and writes alone 885).  In fp32 the product 658, the gated layer 816.
constexpr int kHeldWaves = 8, kHeldBlock = 64 * kHeldWaves;
// Bytes of a row of W in LDS: codes, zeros up to whole steps, scales; or values (bf16, exact), decoded on their way there.
template <int KS, bool Values> constexpr int held_row() { return (Values ? 256 : 128) * KS + kLdsPad; }
// How results leave: rows that begin with a line each straight from registers past the L2, others by way of LDS, or straight too.
enum HeldOut { kLines, kRagged, kStraight };
template <class T, int Mode, int KS, int RN, int Out, bool Values>
__global__ void __launch_bounds__(kHeldBlock) hidden_held_kernel(HiddenArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    constexpr int TB = kHeldWaves * 16 * RN, MR = Mode == kProduct ? 64 : 128;       // rows of X per workgroup, rows of W per 64 columns
    constexpr int kLs = held_row<KS, Values>();
    constexpr bool kAhead = KS * RN <= (Mode == kGatedGrad || KS > 2 ? 2 : 4);
    const Lists lists(a.t, TB);
    const int total = lists.total(), groups = group_of_lane(a.t);
    if (total == 0) return;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = lane_id(), m = l & 15, q = l >> 4;
    const int ht = (a.H + 63) / 64;
    int parts = a.fill / total;                        // few rows: the columns of the result are dealt out too
    parts = parts < 1 ? 1 : parts > ht ? ht : parts;
    const int64_t items = (int64_t)total * parts;
    int held_group = -1, held_from = -1;
    struct Item { int part, list, here, group; int64_t r0; };
    auto find = [&](int64_t item) {
        Item it;
        it.part = (int)(item / total);
        const int tile = (int)(item - (int64_t)it.part * total);
        it.list = lists.list_of(tile);
        it.r0 = (int64_t)(tile - lists.first_tile(it.list)) * TB;
        const int64_t left = lists.rows_in(it.list) - it.r0;
        it.here = left < TB ? (int)left : TB;
        it.group = __builtin_amdgcn_readlane(groups, it.list);
        return it;
    };
    u32x4 ahead[KS][RN][2];
    uint32_t ahead_scale[(KS + 3) / 4][RN];
    auto ask_rows = [&](const Item& it) {
        const uint8_t* x = a.t.rows[it.list] + it.r0 * a.rb;
#pragma unroll
        for (int c = 0; c < RN; ++c) {
            const int row = (wave * RN + c) * 16 + m;
            const uint8_t* p = x + (int64_t)(row < it.here ? row : it.here - 1) * a.rb;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int at = 128 * s + 64 * k + 16 * q;
                    ahead[s][c][k] = *reinterpret_cast<const u32x4*>(p + (at < a.cb ? at : 0));
                }
#pragma unroll
            for (int s = 0; s < (KS + 3) / 4; ++s) ahead_scale[s][c] = *reinterpret_cast<const uint32_t*>(p + a.cb + 4 * s);
        }
    };
    const Share share(items);
    if (share.at >= share.end) return;
    Item it = find(share.at);
    if (kAhead) ask_rows(it);
    for (int64_t item = share.at; item < share.end; item += share.step) {
        if (!kAhead) { it = find(item); ask_rows(it); }
        const int t0 = (int)((int64_t)it.part * ht / parts), t1 = (int)((int64_t)(it.part + 1) * ht / parts);
        const int list = it.list, here = it.here, group = it.group, mine = here - wave * 16 * RN;       // rows of the workgroup, of the wavefront
        const int64_t r0 = it.r0 + wave * 16 * RN;
        if (group != held_group || t0 != held_from) {
            const uint8_t* w = a.w + (int64_t)group * a.H * (MR / 64) * a.rb;
            constexpr uint32_t lv = Values ? 8 * KS : kLs / 16;
            const uint32_t all = (uint32_t)(t1 - t0) * MR * lv;
            __syncthreads();
            // eight vectors of a thread under way together
            for (uint32_t i0 = threadIdx.x; i0 < all; i0 += 8 * kHeldBlock) {
                u32x4 v[8];
                uint8_t scale[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t i = i0 + k * kHeldBlock < all ? i0 + k * kHeldBlock : all - 1;
                    const uint32_t r = i / lv, c = i - r * lv;                       // LDS row: by operand, columns 4m + f of 64 as row 16 f + m
                    int h = 64 * (t0 + (int)(r / MR)) + 4 * (int)(r & 15) + (int)(r >> 4 & 3);
                    h = h < a.H ? h : a.H - 1;
                    const uint8_t* from = w + (int64_t)(MR == 128 && (r & 64) ? a.H + h : h) * a.rb;
                    const int at = c >= 8 * KS ? a.cb : 16 * (int)c;
                    v[k] = *reinterpret_cast<const u32x4*>(from + (c >= 8 * KS || at < a.cb ? at : 0));
                    if (c < 8 * KS && at >= a.cb) v[k] = u32x4{0, 0, 0, 0};
                    if constexpr (Values) scale[k] = from[a.cb + (int)(c / 8)];
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t i = i0 + k * kHeldBlock;
                    if (i >= all) continue;
                    if constexpr (Values) {          // a step's 16-byte pieces in the order in which lanes take them: of four quarters the first, ..
                        const uint32_t r = i / lv, c = i - r * lv;
                        uint8_t* to = lds + r * kLs + 256 * (c / 8) + 128 * (c / 4 & 1) + 16 * (c & 3);
                        const float s = mx4_scale(scale[k]);
                        *reinterpret_cast<bf16x8*>(to) = eight_of(v[k].x, v[k].y, s);
                        *reinterpret_cast<bf16x8*>(to + 64) = eight_of(v[k].z, v[k].w, s);
                    } else {
                        reinterpret_cast<u32x4*>(lds)[i] = v[k];
                    }
                }
            }
            held_group = group; held_from = t0;
            __syncthreads();
        }
        Operand x[KS][RN];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int c = 0; c < RN; ++c) {
                const int at = 128 * s + 16 * q;
                x[s][c].lo = at < a.cb ? ahead[s][c][0] : u32x4{0, 0, 0, 0};
                x[s][c].hi = at + 64 < a.cb ? ahead[s][c][1] : u32x4{0, 0, 0, 0};
                x[s][c].scale = ahead_scale[s / 4][c];
            }
        Decoded xd[Values ? KS : 1][RN];
        if constexpr (Values)
            steps_of<KS>([&](auto step) {
                constexpr int s = decltype(step)::value;
#pragma unroll
                for (int c = 0; c < RN; ++c) xd[s][c] = decode<(s & 3)>(x[s][c]);
            });
        if (kAhead && item + share.step < share.end) { it = find(item + share.step); ask_rows(it); }
        if (mine <= 0) continue;
        const int rows = mine < 16 * RN ? mine : 16 * RN;
        const Results<T, Mode> res(a, list);
        T* const y = res.y;
        const int64_t ld = res.ld;
        RowsOut<T, RN> out;
        if constexpr (Out == kRagged) {
            out.lds = lds + a.w_lds + wave * a.out_lds;
            out.rows = rows;
            out.step = ld * (int64_t)sizeof(T);
            out.y = reinterpret_cast<char*>(y + r0 * ld + 64 * t0);
            out.bytes = ((64 * t1 < a.H ? 64 * t1 : a.H) - 64 * t0) * (int)sizeof(T);
            out.run = out.bytes == out.step && 16 * RN * out.bytes + 16 <= a.out_lds;
            out.begin();
        }
        for (int t = t0; t < t1; ++t) {
            const uint8_t* tile_w = lds + (t - t0) * MR * kLs;
            typedef Tile<T, RN, 4, Out == kLines> Rows;
            typename Rows::V raw[RN][4];
            if constexpr (Mode == kGatedGrad) Rows(res.y, res.ld, r0, rows, 64 * t, 0, a.H, a.H).ask(raw);
            f32x4 acc[MR / 64][RN][4];
#pragma unroll
            for (int k = 0; k < MR / 64; ++k) {
#pragma unroll
                for (int c = 0; c < RN; ++c)
#pragma unroll
                    for (int f = 0; f < 4; ++f) acc[k][c][f] = f32x4{0.f, 0.f, 0.f, 0.f};
                steps_of<KS>([&](auto step) {
                    constexpr int s = decltype(step)::value;
                    if constexpr (Values) {
#pragma unroll
                        for (int f = 0; f < 4; ++f) {
                            const uint8_t* p = tile_w + (64 * k + 16 * f + m) * kLs + 256 * s + 16 * q;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const bf16x8 w = *reinterpret_cast<const bf16x8*>(p + 64 * j);
#pragma unroll
                                for (int c = 0; c < RN; ++c) acc[k][c][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xd[s][c].v[j], w, acc[k][c][f], 0, 0, 0);
                            }
                        }
                    } else {
                        Operand w[4];
#pragma unroll
                        for (int f = 0; f < 4; ++f) {
                            const uint8_t* p = tile_w + (64 * k + 16 * f + m) * kLs;
                            w[f].lo = *reinterpret_cast<const u32x4*>(p + 128 * s + 16 * q);
                            w[f].hi = *reinterpret_cast<const u32x4*>(p + 128 * s + 64 + 16 * q);
                            w[f].scale = *reinterpret_cast<const uint32_t*>(p + 128 * KS + 4 * (s / 4));
                        }
                        multiply<(s & 3)>(acc[k], x[s], w);
                        if constexpr (KS > 6) __builtin_amdgcn_sched_barrier(0);      // W of steps to come would take the registers that there are
                    }
                });
            }
#pragma unroll
            for (int c = 0; c < RN; ++c) {
                f32x4 dy[4];
                if constexpr (Mode == kGatedGrad) Rows::values(raw[c], dy);
                combine<Mode>(a.act, acc[0][c], acc[MR / 64 - 1][c], dy);
            }
            if constexpr (Mode == kGatedGrad) {
                                constexpr int kind = Out == kLines ? kPastL2 : 0;
                Rows(res.p, res.pld, r0, rows, 64 * t, 0, a.H, 2 * a.H).template put<kind>([&](int c, int n) { return acc[0][c][n]; });
                Rows(res.p, res.pld, r0, rows, 64 * t, a.H, a.H, 2 * a.H).template put<kind>([&](int c, int n) { return acc[1][c][n]; });
            } else if constexpr (Out != kRagged) {
                constexpr int kind = Out == kLines ? kPastL2 : 0;
                Rows(y, ld, r0, rows, 64 * t, 0, a.H, a.H).template put<kind>([&](int c, int n) { return acc[0][c][n]; });
            } else {
                out.put(t - t0, acc[0]);
                if (!out.run) out.flush_lines(t - t0, t == t0, t + 1 == t1);
                else if (t + 1 == t1) out.flush_run();
            }
        }
    }
}

constexpr int kHeldLds = 163840;         // all of a CU's
constexpr int kHeldRowOut = 768;         // bytes of rows that go out in one run
template <class T, int Mode, int KS, int RN, int Out, bool Values>
static int launch_held_as(spp_ctx* ctx, HiddenArgs& a, bool* done) {
    constexpr int MR = Mode == kProduct ? 64 : 128, TB = kHeldWaves * 16 * RN;
    auto kernel = hidden_held_kernel<T, Mode, KS, RN, Out, Values>;
    const int ht = (a.H + 63) / 64, row = a.H * (int)sizeof(T);
    a.out_lds = Out != kRagged ? 0 : 16 * RN * RowsOut<T, RN>::kPitch;
    if (Out == kRagged && row <= kHeldRowOut && a.out_lds < 16 * RN * row + 16) a.out_lds = 16 * RN * row + 16;
    const int64_t need = (int64_t)ht * MR * held_row<KS, Values>(), most_lds = kHeldLds - (int64_t)kHeldWaves * a.out_lds;
    *done = need <= most_lds;
    if (!*done) return SPP_OK;
    a.w_lds = (int)need;
    const int lds = a.w_lds + kHeldWaves * a.out_lds;
    static LdsLimit limit;
    SPP_TRY(limit.allow(ctx, reinterpret_cast<const void*>(kernel), lds));
    int64_t tiles = 0;
    for (int j = 0; j < a.t.n_lists; ++j) tiles += (a.t.n[j] + (int64_t)TB - 1) / TB;
    a.fill = ctx->num_cu;
    const int fit = kHeldLds / lds, per_cu = fit < 1 ? 1 : fit > 2 ? 2 : fit;
    const int64_t want = tiles >= a.fill ? tiles : tiles * ht < a.fill ? tiles * ht : a.fill, most = (int64_t)ctx->num_cu * per_cu;
    kernel<<<(unsigned)(want < most ? want : most), kHeldBlock, lds, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}
// Whether W is held as values: where the code that decodes a row of W for 16 RN rows of X takes longer than its products, of the
// gated layer, and of the product where RN is 1; not for few rows, which have W but once.  W as codes and as values, in bf16: 200k rows gated 172 -> 100
// 51 and 42 us, 128 -> 256 56 and 47, 512 -> 64 51 and 43; the product 1M rows 172 -> 100 166 and 140, 300k 256 -> 86 55 and 43; in fp32 200k rows gated
// 172 -> 100 65 and 54, the product 172 -> 100 38 and 33, with two sixteens 100 -> 64 18 and 20; the gated gradient 172 -> 100 110 both.
template <class T, int Mode, int KS, int RN, int Out>
static int launch_held(spp_ctx* ctx, HiddenArgs& a, bool few, bool* done) {
    if constexpr (KS <= 4 && ((Mode == kGated && (RN == 2 || KS > 2)) || (Mode == kProduct && RN == 1 && (Out == kRagged || KS > 2)))) {
        if (!few) SPP_TRY((launch_held_as<T, Mode, KS, RN, Out, true>(ctx, a, done)));
        if (*done) return SPP_OK;
    }
    return launch_held_as<T, Mode, KS, RN, Out, false>(ctx, a, done);
}
template <class T, int Mode>
static int try_held(spp_ctx* ctx, HiddenArgs& a, bool* done) {
    // rows of whole vectors that begin with a line each are stored as they come, 128 or 256 bytes of a row at a time
    bool lines = Mode == kGatedGrad ? a.H * sizeof(T) % 128 == 0 : a.H % 4 == 0;
    int64_t pairs = 0;                                   // tiles of two sixteens
    for (int j = 0; j < a.t.n_lists; ++j) {
        void* const y = Mode == kGatedGrad ? a.dp[j] : a.t.y[j];
        const int64_t ld = Mode == kGatedGrad ? a.dp_ld[j] : a.t.ld[j];
        lines = lines && ((uintptr_t)y | (uint64_t)(ld * (int64_t)sizeof(T))) % 128 == 0;
        if (Mode == kGatedGrad) lines = lines && ((uintptr_t)a.t.y[j] | (uint64_t)(a.t.ld[j] * (int64_t)sizeof(T))) % 4 == 0;       // dY
        pairs += (a.t.n[j] + 32 * kHeldWaves - 1) / (32 * kHeldWaves);
    }
    // Few rows: tiles of two sixteens and 64 columns are no more than there are CUs.  One sixteen then: 16k rows 256 -> 256 in bf16 10.7 and 8.1 us,
    // gated 14.2 and 12.5, its gradient 17.6 and 15.5; 24k, which are more tiles, 12.4 and 10.7, 19.2
    // and 16.0, 24.2 and 21.5, with one sixteen and with two.
    const bool few = pairs * ((a.H + 63) / 64) <= ctx->num_cu;
    auto with = [&](auto steps) {
        constexpr int KS = decltype(steps)::value;
        auto put = [&](auto out) {
            constexpr int Out = decltype(out)::value;
            if constexpr (KS <= 2) {
                if (!few) return launch_held<T, Mode, KS, 2, Out>(ctx, a, few, done);
            }
            return launch_held<T, Mode, KS, 1, Out>(ctx, a, few, done);
        };
        if constexpr (KS > 6 && Mode == kGatedGrad) {
            return (int)SPP_OK;                              // (registers)
        } else if constexpr (KS > 4) {
            // with few columns most wavefronts of the other form would have none: 200k rows 1024 -> 24 in bf16 120 and 67 us, 640 -> 128 80 and 64, of 16
            // bits 640 -> 192 81 and 86
            if (sizeof(T) == 2 && a.H > 128) return (int)SPP_OK;
            return launch_held<T, Mode, KS, 1, kStraight>(ctx, a, few, done);
        } else if (lines) {
            return put(std::integral_constant<int, kLines>());
        } else if constexpr (Mode == kGatedGrad) {
            // One sixteen: with two, what the CUs have under way is more than the L2 holds, and lines that two stores share leave it in between.
            // 1M rows with two and one in bf16 172 -> 100 304 and 299 us, 100 -> 172 456 and 410, in fp32 449 and 419, 709 and 679; 16k 172 -> 100 19 and
            // 14, 18 and 14.  But two where these are one tile a CU and one sixteen would be a few more: 40k 21 and 26, 23 and 26, 64k 24 and 34, 26 and 34
            if constexpr (KS <= 2) {
                if (2 * pairs > ctx->num_cu && pairs <= ctx->num_cu) return launch_held<T, Mode, KS, 2, kStraight>(ctx, a, few, done);
            }
            return launch_held<T, Mode, KS, 1, kStraight>(ctx, a, few, done);
        } else if constexpr (Mode == kGated) {
            // beside two products the LDS that rows need is worth more to W and to a second sixteen rows of X (1M rows 172 -> 100 in bf16 by way of
            // LDS 243 us, so 167; in fp32 240 and 193)
            return put(std::integral_constant<int, kStraight>());
        } else {
            // Results of 16 bits and few columns straight, with two sixteens: by way of LDS and so 1M rows 172 -> 100 in bf16 130 and 104 us, 300k 128 -> 86
            // 31 and 28, 256 -> 86 43 and 41; but 256 -> 172 53 and 59, 1M 128 -> 250 172 and 236; in fp32 172 -> 100 137 and 161, 300k 128 -> 86 34 and 46.
            // By way of LDS with one sixteen and two 300k 128 -> 86 in bf16 38 and 31, in fp32 38 and 34 (two sixteens of two steps fill the registers)
            if constexpr (sizeof(T) == 2 && KS <= 2) {
                if (a.H <= 128) return put(std::integral_constant<int, kStraight>());
            }
            if constexpr (KS == 1) {
                if (!few) SPP_TRY((launch_held<T, Mode, KS, 2, kRagged>(ctx, a, few, done)));
                if (*done) return (int)SPP_OK;
            }
            return launch_held<T, Mode, KS, 1, kRagged>(ctx, a, few, done);
        }
    };
    switch (a.steps) {
        case 1: return with(std::integral_constant<int, 1>());
        case 2: return with(std::integral_constant<int, 2>());
        case 3: return with(std::integral_constant<int, 3>());
        case 4: return with(std::integral_constant<int, 4>());
        case 5: return with(std::integral_constant<int, 5>());
        case 6: return with(std::integral_constant<int, 6>());
        case 7: return with(std::integral_constant<int, 7>());
        case 8: return with(std::integral_constant<int, 8>());
    }
    return SPP_OK;
}

// ---- W in registers --------------------------------------------------------------------------------

// The form for weights that LDS does not hold.  A wavefront keeps 64 rows of W in registers (32 of the gate's and the same 32 of the other
// factor), all columns of them, and a workgroup goes over its share of the rows of X, 32 at a time, which its wavefronts read from LDS:
// W is read once per workgroup, and per product half as much from LDS as with X in registers and W in LDS.  The workgroups that have the same
// rows and other columns share an XCD's L2 and take the rows in the same order at the same time.  With one wavefront per SIMD nothing else
// works while it waits, so that a tile's work is one piece of code without branches, the next tile's way to LDS in the middle of its products.
// Bound by the decoding of W for every tile of rows, beside which the matrix pipe is busy 41 % of the time: 380k rows 1024 -> 1024 in bf16 770 to 820 us,
// 1.0 PFLOP/s, gated to 512 825, its gradient 924; in fp32 832, 831 and 1240.
// Rows of X at a time, in sixteens: one where the registers would not hold what two need.  No kernel here may spill registers: the compiler (of
// ROCm 7.2) has lost some of those that it had to put away where a kernel fills all 512.
template <class T, int Mode, int KS> constexpr int kWideRows = Mode == kGatedGrad && KS == 8 && sizeof(T) == 4 ? 1 : 2;
template <class T, int Mode, int KS, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, WAVES > 4 ? 2 : 1) hidden_wide_kernel(HiddenArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    constexpr int RN = kWideRows<T, Mode, KS>, TB = 16 * RN, threads = 64 * WAVES, cols = Mode == kProduct ? 64 : 32;
    constexpr int kLs = 128 * KS + kLdsPad;                   // bytes of a row of X in LDS: codes, zeros up to whole steps, scales
    constexpr int kVec = (TB * (8 * KS + 1) + threads - 1) / threads;
    const Lists lists(a.t, TB);
    const int total = lists.total(), groups = group_of_lane(a.t);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = lane_id(), m = l & 15, q = l >> 4;
    // which columns, which rows
    int block, at, end, step;
    if (a.shares > 0) {
        const int xcd = blockIdx.x & 7, k = (int)blockIdx.x >> 3;
        block = k % a.blocks;
        at = (int)((int64_t)total * xcd >> 3) + k / a.blocks;
        end = (int)((int64_t)total * (xcd + 1) >> 3);
        step = a.shares;
    } else {
        block = (int)blockIdx.x % a.blocks;
        at = (int)blockIdx.x / a.blocks;
        end = total;
        step = (int)gridDim.x / a.blocks;
    }
    if (at >= end) return;
    const int h0 = (block * WAVES + wave) * cols;
    constexpr int buffer = TB * kLs;
    for (int i = threadIdx.x; i < 2 * buffer / 16; i += threads) reinterpret_cast<u32x4*>(lds)[i] = u32x4{0, 0, 0, 0};

    Operand w[KS][4];
    int held_group = -1;
    auto hold = [&](int group) {
        const uint8_t* base = a.w + (int64_t)group * a.H * (Mode == kProduct ? 1 : 2) * a.rb;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            int h = h0 + (Mode == kProduct ? 4 * m + f : 2 * m + (f & 1));
            h = h < a.H ? h : a.H - 1;
            const uint8_t* p = base + (int64_t)(Mode != kProduct && f >= 2 ? a.H + h : h) * a.rb;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int lo = 128 * s + 16 * q, hi = lo + 64;
                const u32x4 x = *reinterpret_cast<const u32x4*>(p + (lo < a.cb ? lo : 0)), y = *reinterpret_cast<const u32x4*>(p + (hi < a.cb ? hi : 0));
                w[s][f].lo = lo < a.cb ? x : u32x4{0, 0, 0, 0};
                w[s][f].hi = hi < a.cb ? y : u32x4{0, 0, 0, 0};
                w[s][f].scale = *reinterpret_cast<const uint32_t*>(p + a.cb + 4 * (s / 4));
            }
        }
        held_group = group;
    };

    // X: where the thread's vectors of a tile come from and go to; the zeros between codes and scales are never written
    uint32_t places[kVec];                                    // 16 bits each
    static_assert(TB * kLs <= 65536, "");
    {
        const uint32_t per = (uint32_t)a.cb / 16 + 1, all = TB * per;
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            uint32_t i = k * threads + threadIdx.x;
            i = i < all ? i : all - 1;
            const uint32_t r = i / per, v = i - r * per;
            places[k] = (r * (uint32_t)a.rb + 16 * v) | (r * kLs + (v + 1 < per ? 16 * v : 128 * KS)) << 16;
        }
    }
    struct Piece { int list, here, r0; };
    const uint8_t* x_list = nullptr;                          // of the list of the tile that was asked for last
    int x_until = at, x_first = 0, x_rows = 0, x_of = 0;
    u32x4 ahead[kVec];
    auto find = [&](int tile) {                               // behind the last tile the last one again
        tile = tile < end ? tile : end - 1;
        if (tile >= x_until) {
            x_of = lists.list_of(tile);
            x_first = lists.first_tile(x_of);
            x_until = __builtin_amdgcn_readlane(lists.upto, x_of);
            x_rows = lists.rows_in(x_of);
            x_list = a.t.rows[x_of];
        }
        Piece t;
        t.list = x_of;
        t.r0 = (tile - x_first) * TB;                         // (below the list's rows, which are at most 2^31 - 1)
        t.here = x_rows - t.r0 < TB ? x_rows - t.r0 : TB;
        return t;
    };
    auto ask = [&](const Piece& t) {
        const auto x = rows_buffer(x_list + (int64_t)t.r0 * a.rb, (uint32_t)(t.here * a.rb));
#pragma unroll
        for (int k = 0; k < kVec; ++k) ahead[k] = __builtin_amdgcn_raw_buffer_load_b128(x, (int)(places[k] & 0xFFFF), 0, 0);
    };
    auto keep = [&](uint8_t* buf) {
#pragma unroll
        for (int k = 0; k < kVec; ++k) *reinterpret_cast<u32x4*>(buf + (places[k] >> 16)) = ahead[k];
    };
    Piece now = find(at);
    ask(now);
    __syncthreads();
    keep(lds);
    hold(__builtin_amdgcn_readlane(groups, now.list));
    Piece next = find(at + step);
    ask(next);
    int out_list = -1;
    T *y = nullptr, *p = nullptr;                             // the list's Y and dP
    int ld = 0, pld = 0;                                      // (32 rows are below 2^31 bytes)
    for (int tile = at, j = 0; tile < end; tile += step, ++j) {
        __syncthreads();                                      // this tile is in LDS, and the one before has been read by all
        if (now.list != out_list) {
            const int group = __builtin_amdgcn_readlane(groups, now.list);
            if (group != held_group) hold(group);
            out_list = now.list;
            y = static_cast<T*>(a.t.y[now.list]);
            ld = (int)a.t.ld[now.list];
            if constexpr (Mode == kGatedGrad) { p = static_cast<T*>(a.dp[now.list]); pld = (int)a.dp_ld[now.list]; }
        }
        const Piece after = find(tile + 2 * step);
        const uint8_t* x = lds + (j & 1) * buffer;
        uint8_t* const other = lds + (~j & 1) * buffer;
        constexpr int N = cols / 16;                          // columns of a lane
        typedef Tile<T, RN, N> Rows;
        typename Rows::V raw[RN][4];
        if constexpr (Mode == kGatedGrad) Rows(y, ld, now.r0, now.here, h0, 0, a.H, a.H).ask(raw);
        f32x4 acc[RN][4];
#pragma unroll
        for (int c = 0; c < RN; ++c)
#pragma unroll
            for (int f = 0; f < 4; ++f) acc[c][f] = f32x4{0.f, 0.f, 0.f, 0.f};
        // The next tile goes to LDS and the one behind it is asked for during the products.  One wavefront per SIMD also reads each step's rows
        // before the products of the step before; the compiler, short of registers, would put every load right before its use (380k rows
        // 1024 -> 1024 854 us, 777 so).
        constexpr bool kOrdered = WAVES == 4;
        Operand xv[kOrdered ? 2 : 1][RN];
        uint32_t scales[kOrdered ? 2 : 1][RN];                // of four steps
        auto read = [&](auto index) {
            constexpr int s = decltype(index)::value;
#pragma unroll
            for (int c = 0; c < RN; ++c) {
                const uint8_t* p = x + (16 * c + m) * kLs;
                xv[kOrdered ? s & 1 : 0][c].lo = *reinterpret_cast<const u32x4*>(p + 128 * s + 16 * q);
                xv[kOrdered ? s & 1 : 0][c].hi = *reinterpret_cast<const u32x4*>(p + 128 * s + 64 + 16 * q);
                if constexpr (s % 4 == 0) scales[kOrdered ? s / 4 & 1 : 0][c] = *reinterpret_cast<const uint32_t*>(p + 128 * KS + s);
            }
        };
        if constexpr (kOrdered) read(std::integral_constant<int, 0>());
        steps_of<KS>([&](auto index) {
            constexpr int s = decltype(index)::value;
            if constexpr (!kOrdered) read(index);
            else if constexpr (s + 1 < KS) read(std::integral_constant<int, s + 1>());
            if (kOrdered) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = 0; c < RN; ++c) xv[kOrdered ? s & 1 : 0][c].scale = scales[kOrdered ? s / 4 & 1 : 0][c];
            multiply<(s & 3)>(acc, xv[kOrdered ? s & 1 : 0], w[s]);
            if (s == (KS > 2 ? 1 : 0)) keep(other);
            if (s == (KS > 2 ? 2 : KS - 1)) ask(after);
            if (kOrdered) __builtin_amdgcn_sched_barrier(0);
        });
#pragma unroll
        for (int c = 0; c < RN; ++c)
            if constexpr (Mode != kProduct) {
                f32x4 dy[N];
                if constexpr (Mode == kGatedGrad) Rows::values(raw[c], dy);
                combine<Mode>(a.act, reinterpret_cast<f32x4(&)[2]>(acc[c][0]), reinterpret_cast<f32x4(&)[2]>(acc[c][2]), dy);
            }
        if constexpr (Mode == kGatedGrad) {
            Rows(p, pld, now.r0, now.here, h0, 0, a.H, 2 * a.H).put([&](int c, int n) { return acc[c][n]; });
            Rows(p, pld, now.r0, now.here, h0, a.H, a.H, 2 * a.H).put([&](int c, int n) { return acc[c][N + n]; });
        } else {
            // whole lines past the L2 (200k rows 256 -> 1024 in bf16: 152 us with plain stores, 133 so)
            const Rows to(y, ld, now.r0, now.here, h0, 0, a.H, a.H);
            if (Mode == kProduct && (((uint32_t)(uintptr_t)y | to.step) & 127) == 0) to.template put<kPastL2>([&](int c, int n) { return acc[c][n]; });
            else to.put([&](int c, int n) { return acc[c][n]; });
        }
        now = next;
        next = after;
    }
}

template <class T, int Mode, int KS, int WAVES>
static int launch_wide(spp_ctx* ctx, HiddenArgs& a) {
    constexpr int TB = 16 * kWideRows<T, Mode, KS>, cols = WAVES * (Mode == kProduct ? 64 : 32);
    auto kernel = hidden_wide_kernel<T, Mode, KS, WAVES>;
    constexpr int lds = 2 * TB * (128 * KS + kLdsPad);
    static LdsLimit limit;
    SPP_TRY(limit.allow(ctx, reinterpret_cast<const void*>(kernel), lds));
    int64_t tiles = 0;
    for (int j = 0; j < a.t.n_lists; ++j) tiles += (a.t.n[j] + (int64_t)TB - 1) / TB;
    a.blocks = (a.H + cols - 1) / cols;
    const int64_t at_once = ctx->num_cu;
    a.shares = (int)(at_once / 8 / a.blocks);
    int64_t grid = (int64_t)a.shares * 8 * a.blocks;
    if (a.shares == 0 || tiles < 8 * a.shares) {
        const int64_t fill = at_once / a.blocks < 1 ? 1 : at_once / a.blocks;
        a.shares = 0;
        grid = (tiles < fill ? tiles : fill) * a.blocks;
    }
    kernel<<<(unsigned)grid, 64 * WAVES, lds, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}

template <class T, int Mode>
static int launch_hidden(spp_ctx* ctx, HiddenArgs& a) {
    bool done = false, near = true;                      // whether 32 rows of results are within what a buffer spans
    for (int j = 0; j < a.t.n_lists; ++j)
        near = near && spans(a.t.ld[j], sizeof(T), 32) && (Mode != kGatedGrad || spans(a.dp_ld[j], sizeof(T), 32));
    if (near) SPP_TRY((try_held<T, Mode>(ctx, a, &done)));
    if (done) return SPP_OK;
    if (near) switch (a.steps) {
        case 1: return launch_wide<T, Mode, 1, 8>(ctx, a);
        case 2: return launch_wide<T, Mode, 2, 8>(ctx, a);
        case 3: return launch_wide<T, Mode, 3, 8>(ctx, a);
        case 4: return launch_wide<T, Mode, 4, Mode == kGatedGrad ? 4 : 8>(ctx, a);
        case 5: return launch_wide<T, Mode, 5, 4>(ctx, a);
        case 6: return launch_wide<T, Mode, 6, 4>(ctx, a);
        case 7: return launch_wide<T, Mode, 7, 4>(ctx, a);
        case 8: return launch_wide<T, Mode, 8, 4>(ctx, a);
    }
    auto kernel = hidden_tile_kernel<T, Mode>;
    static LdsLimit limit;
    SPP_TRY(limit.allow(ctx, reinterpret_cast<const void*>(kernel), 2 * kTileBuffer));
    int64_t tiles = 0;
    for (int j = 0; j < a.t.n_lists; ++j) tiles += (a.t.n[j] + (int64_t)kTileRows - 1) / kTileRows;
    constexpr int cols = Mode == kProduct ? 128 : 64;
    const int64_t want = tiles * ((a.H + cols - 1) / cols), most = (int64_t)ctx->num_cu * 64;
    kernel<<<(unsigned)(want < most ? want : most), kTileBlock, 2 * kTileBuffer, ctx->stream>>>(a);
    SPP_HIP(hipGetLastError());
    return SPP_OK;
}

// Whether two matrices of rows share a byte: n rows of `bytes` bytes each, `step` bytes from a row to the next.  Rows of the same step, and of steps that differ where
// one matrix has no gaps, exactly: columns of one buffer may lie side by side.  Of two with gaps and other steps the first 4096 rows are looked at.
struct Span {
    uint64_t at;
    int64_t  n, bytes, step;
    uint64_t end() const { return at + (uint64_t)(n - 1) * step + bytes; }
};
static inline bool overlap(Span a, Span b) {
    if (a.n == 0 || b.n == 0) return false;
    if (a.n == 1) a.step = a.bytes;
    if (b.n == 1) b.step = b.bytes;
    if (a.at >= b.end() || b.at >= a.end()) return false;
    // a row from `from` of `bytes` bytes against rows: the first that ends behind its beginning begins before its end
    auto meets = [](uint64_t from, int64_t bytes, const Span& s) {
        const uint64_t i = from < s.at + s.bytes ? 0 : (from - s.at - s.bytes) / s.step + 1;
        return (int64_t)i < s.n && s.at + i * s.step < from + bytes;
    };
    if (a.step == a.bytes) return meets(a.at, a.n * a.bytes, b);
    if (b.step == b.bytes) return meets(b.at, b.n * b.bytes, a);
    if (a.at > b.at) { const Span c = a; a = b; b = c; }
    if (a.step == b.step) {                              // b's first row lies among a's, and all others as it does
        const uint64_t d = (b.at - a.at) % a.step;
        return (int64_t)d < a.bytes || ((int64_t)d + b.bytes > a.step && (int64_t)((b.at - a.at) / a.step) + 1 < a.n);
    }
    for (int64_t i = 0; i < b.n && i < 4096; ++i)
        if (meets(b.at + i * b.step, b.bytes, a)) return true;
    return false;
}

// The checks of the three entries, and the launch.
template <int Mode>
static int hidden(const char* who, spp_ctx* ctx, const spp_row_list* lists, const spp_row_list* grads, int32_t n_lists, const void* d_weights,
                  int32_t n_groups, int32_t D, int32_t H, int32_t type, int32_t activation, uint32_t flags) {
    SPP_CHECK(ctx && d_weights, SPP_E_ARG, "%s: null argument", who);
    SPP_CHECK((uintptr_t)d_weights % 16 == 0, SPP_E_ARG, "%s: weights must be 16-byte aligned", who);
    HiddenArgs a;
    memset(&a, 0, sizeof(a));
    int64_t most = 0;
    SPP_TRY(row_table(who, lists, n_lists, n_groups, D, H, type, a.t, &most));
    if (Mode != kProduct) SPP_CHECK(H <= SPP_MAX_HIDDEN / 2, SPP_E_ARG, "%s: H = %d (1 .. %d)", who, H, SPP_MAX_HIDDEN / 2);
    if (Mode == kGatedGrad) {
        RowTable p;
        int64_t also = 0;
        SPP_CHECK(grads || n_lists == 0, SPP_E_ARG, "%s: null argument", who);
        SPP_TRY(row_table(who, grads, n_lists, n_groups, D, 2 * H, type, p, &also));
        for (int j = 0; j < n_lists; ++j)
            SPP_CHECK(lists[j].d_rows == grads[j].d_rows && lists[j].n == grads[j].n && lists[j].d_n == grads[j].d_n && lists[j].group == grads[j].group,
                      SPP_E_ARG, "%s: list %d: the gradient's rows, count or group are not the list's", who, j);
        auto span = [&](const spp_row_list& l, int cols) {
            const int64_t es = (int64_t)type_bytes(type);
            return Span{(uint64_t)(uintptr_t)l.d_y, l.n, cols * es, l.ld * es};
        };
        uint64_t lo = ~0ull, hi = 0;                     // all dY lie there: most gradients, in buffers of their own, need no closer look
        for (int j = 0; j < n_lists; ++j)
            if (lists[j].n > 0) {
                const Span s = span(lists[j], H);
                lo = s.at < lo ? s.at : lo;
                hi = s.end() > hi ? s.end() : hi;
            }
        for (int k = 0; k < n_lists; ++k) {
            const Span dp = span(grads[k], 2 * H);
            if (dp.n == 0 || dp.at >= hi || dp.end() <= lo) continue;
            for (int j = 0; j < n_lists; ++j)
                SPP_CHECK(!overlap(span(lists[j], H), dp), SPP_E_ARG, "%s: the gradient of list %d overlaps the dY of list %d", who, k, j);
        }
        for (int j = 0; j < n_lists; ++j) { a.dp[j] = p.y[j]; a.dp_ld[j] = p.ld[j]; }
    }
    if (Mode != kProduct)
        SPP_CHECK(activation == SPP_SILU || activation == SPP_GELU || activation == SPP_SIGMOID, SPP_E_ARG, "%s: activation %d", who, activation);
    if (most > 0) {
        a.w = static_cast<const uint8_t*>(d_weights);
        a.D = D; a.H = H; a.rb = fp8_bytes(D); a.cb = fp8_code_bytes(D); a.steps = fp8_blocks(D); a.act = activation;
        SPP_HIP(hipSetDevice(ctx->device));
        ScopedTimer timer(ctx, SPP_T_LAYER, ctx->stream);
        SPP_TRY(type == SPP_F32 ? (launch_hidden<float, Mode>(ctx, a)) : type == SPP_F16 ? (launch_hidden<_Float16, Mode>(ctx, a))
                                                                                          : (launch_hidden<__bf16, Mode>(ctx, a)));
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}

}  // namespace spp
