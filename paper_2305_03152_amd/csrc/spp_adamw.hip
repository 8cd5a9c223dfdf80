// One AdamW step over many tensors at once, with the two moments in 32 bits or in 8.
//
//   m' = b1 m + (1-b1) g      v' = b2 v + (1-b2) g^2
//   p' = (1 - lr wd) p - lr/(1-b1^t) * m' / (sqrt(v') / sqrt(1-b2^t) + eps)
//
// each operation rounded once, in the order written.  An element whose v' is not finite (its gradient is not, or its square is
// not) is left as it was, its moments too.
//
// In 8 bits the moments of 256 consecutive elements share a scale each: the largest |m| and the largest sqrt(v) of the block
// are the largest code, and a code is a small float: m a sign, 4 bits of exponent and 3 of mantissa, sqrt(v) 4 and 4.  Steps
// of a constant ratio, because both moments are divided by each other: an evenly spaced code would hold small second moments as
// zero, and their updates would be m / eps.  For the same reason a v that is not zero keeps at least the smallest code.  The
// update itself uses the moments before they are rounded to 8 bits.
//
// All of it is element by element.  With moments in 32 bits it is bound by HBM: 128M fp32 parameters and bf16 gradients, 26 bytes each,
// 549 to 623 us by the box, 5.3 to 6.1 TB/s.  In 8 bits, 14 bytes each, 330 us, 5.4 TB/s: as much by its arithmetic (some 80 instructions
// an element, a root and a quotient rounded correctly among them).  Chunks in the order of the workgroups: with a contiguous part per
// XCD, as streams that are only written like it, 650 and 390 us.  A step that leaves all elements alone takes 3.0 ms either way: the
// threads that have such elements count them on one word, each by an add of its own.
#include "spp_mx4.h"

#include <math.h>

namespace spp {

constexpr int kAdamTensors = kWave;          // of one launch: a lane has a tensor's first chunk
constexpr int kAdamBlock = 256, kAdamPer = 8, kAdamChunk = kAdamBlock * kAdamPer;
constexpr int kAdamShared = SPP_ADAMW_BLOCK;
static_assert(kAdamShared == 4 * kWave, "a wavefront has a block, four elements per lane");

struct AdamTable {
    void*       p[kAdamTensors];
    const void* g[kAdamTensors];
    void*       m[kAdamTensors];
    void*       v[kAdamTensors];
    float*      scale[kAdamTensors];
    int64_t     n[kAdamTensors];
    uint32_t    first[kAdamTensors];         // first chunk; behind the last tensor: all ones
    uint8_t     kind[kAdamTensors];          // type of p, type of g << 2, and 16 if four elements may be taken at a time
};
struct AdamHyper { float b1, c1, b2, c2, rs, eps, decay, step; };

// The tensor that a chunk is of.
__device__ __forceinline__ uint32_t chunk_owner(const AdamTable& t, uint32_t chunk) {
    return (uint32_t)__builtin_amdgcn_readfirstlane(__popcll(__ballot(t.first[lane_id()] <= chunk)) - 1);
}

template <class T>
__device__ __forceinline__ void load4(const void* base, int64_t i, int have, bool wide, float (&x)[4]) {
    const T* p = static_cast<const T*>(base) + i;
    if (have >= 4 && wide) {
        const typename Elem<T>::v4 a = *reinterpret_cast<const typename Elem<T>::v4*>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = (float)a[k];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = k < have ? (float)p[k] : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void store4(void* base, int64_t i, int have, bool wide, const float (&x)[4]) {
    T* p = static_cast<T*>(base) + i;
    if (have >= 4 && wide) {
        typename Elem<T>::v4 a;
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = (T)x[k];
        __builtin_nontemporal_store(a, reinterpret_cast<typename Elem<T>::v4*>(p));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < have) p[k] = (T)x[k];
    }
}
__device__ __forceinline__ void load_codes(const void* base, int64_t i, int have, bool wide, uint32_t (&c)[4]) {
    const uint8_t* p = static_cast<const uint8_t*>(base) + i;
    if (have >= 4 && wide) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = (w >> (8 * k)) & 255u;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = k < have ? p[k] : 0u;
    }
}
__device__ __forceinline__ void store_codes(void* base, int64_t i, int have, bool wide, const uint32_t (&c)[4]) {
    uint8_t* p = static_cast<uint8_t*>(base) + i;
    if (have >= 4 && wide) __builtin_nontemporal_store(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, reinterpret_cast<uint32_t*>(p));
    else
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < have) p[k] = (uint8_t)c[k];
}

// False: the element stays as it was.  root: of the v that it then has.
__device__ __forceinline__ bool adam_element(const AdamHyper& h, float g, float& p, float& m, float& v, float& root) {
    const float m1 = m * h.b1 + g * h.c1;
    const float v1 = v * h.b2 + (g * g) * h.c2;
    const bool finite = (__float_as_uint(v1) & 0x7F800000u) != 0x7F800000u;
    v = finite ? v1 : v;
    root = sqrtf(v);
    const float den = root * h.rs + h.eps;
    const float p1 = p * h.decay - (m1 / den) * h.step;
    p = finite ? p1 : p;
    m = finite ? m1 : m;
    return finite;
}

// The moments of a block as codes and back.  `most` is the largest code's value before the scale.
constexpr float kMostM = 1.875f, kMostV = 1.9375f, kLeastScale = 0x1p-100f;
struct Moment { float inv, scale; };
__device__ __forceinline__ Moment moment_scale(float largest, float most) {
    // below this 1 / scale would not be finite: the block counts as zeros
    return largest >= kLeastScale ? Moment{most / largest, largest * (1.0f / most)} : Moment{0.0f, 0.0f};
}
// The nearest code, ties to the even one: the float's bits without the last DROP, whose first code, 0, would be 2^-15.  Rounding goes by
// that value also where the code then reads as 0.
template <int DROP, int BASE, int TOP>
__device__ __forceinline__ uint32_t small_float(float q) {
    const uint32_t u = __float_as_uint(q);
    const int c = (int)((u + ((1u << (DROP - 1)) - 1) + ((u >> DROP) & 1u)) >> DROP) - BASE;
    return (uint32_t)(c < 0 ? 0 : c > TOP ? TOP : c);
}
__device__ __forceinline__ uint32_t code_m(float m, const Moment& s) {
    const uint32_t c = small_float<20, 896, 127>(fabsf(m) * s.inv);
    return c ? c | (__float_as_uint(m) >> 31) << 7 : 0u;
}
__device__ __forceinline__ uint32_t code_v(float r, const Moment& s) {
    const uint32_t c = small_float<19, 1792, 255>(r * s.inv);
    return r > 0.0f && s.scale > 0.0f ? (c ? c : 1u) : 0u;
}
__device__ __forceinline__ float value_m(uint32_t c, float scale) {
    const float a = __uint_as_float(((c & 127u) + 896u) << 20) * scale;
    return (c & 127u) ? (c & 128u ? -a : a) : 0.0f;
}
__device__ __forceinline__ float value_v(uint32_t c, float scale) {
    const float r = __uint_as_float((c + 1792u) << 19) * scale;
    return c ? r * r : 0.0f;
}
__device__ __forceinline__ float wave_max(float x) {            // of values that are not negative
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)wave_inclusive_max(__float_as_uint(x)), kWave - 1));
}
__device__ __forceinline__ void put_moments(const AdamTable& t, uint32_t j, int64_t i, int have, bool wide, const float (&m)[4], const float (&r)[4]) {
    float am = 0.f, ar = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        am = fmaxf(am, fabsf(m[k]));
        ar = fmaxf(ar, r[k]);
    }
    const Moment sm = moment_scale(wave_max(am), kMostM), sv = moment_scale(wave_max(ar), kMostV);
    uint32_t cm[4], cv[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) { cm[k] = code_m(m[k], sm); cv[k] = code_v(r[k], sv); }
    store_codes(t.m[j], i, have, wide, cm);
    store_codes(t.v[j], i, have, wide, cv);
    if (lane_id() == 0) {
        float* s = t.scale[j] + 2 * (i / kAdamShared);
        s[0] = sm.scale; s[1] = sv.scale;
    }
}
__device__ __forceinline__ void get_moments(const AdamTable& t, uint32_t j, int64_t i, int have, bool wide, float (&m)[4], float (&v)[4]) {
    uint32_t cm[4], cv[4];
    load_codes(t.m[j], i, have, wide, cm);
    load_codes(t.v[j], i, have, wide, cv);
    const float* s = t.scale[j] + 2 * (i / kAdamShared);
    const float sm = s[0], sv = s[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) { m[k] = value_m(cm[k], sm); v[k] = value_v(cv[k], sv); }
}

// A workgroup's chunk: kAdamPer elements per thread, four at a time; all of them are asked for before any is worked on, so that
// a wavefront's loads are under way together.  Whole: a chunk without an end in it, all arrays aligned.
template <bool Small, class P, class G, bool Whole>
__device__ __forceinline__ int adam_chunk(const AdamTable& t, const AdamHyper& h, uint32_t j, int64_t at, int64_t n, bool wide) {
    constexpr int R = kAdamPer / 4;
    float p[R][4], g[R][4], m[R][4], v[R][4];
    int have[R];
    int left_alone = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t i = at + (r * kAdamBlock + (int)threadIdx.x) * 4, rest = n - i;
        have[r] = Whole || rest >= 4 ? 4 : rest > 0 ? (int)rest : 0;
        // in 8 bits a wavefront has a block: all of it goes or none, and lanes behind the last element bring zeros
        if (!Whole && (Small ? n - (i - 4 * lane_id()) <= 0 : rest <= 0)) { have[r] = -1; continue; }
        load4<P>(t.p[j], i, have[r], Whole || wide, p[r]);
        load4<G>(t.g[j], i, have[r], Whole || wide, g[r]);
        if constexpr (Small) get_moments(t, j, have[r] ? i : n - 1, have[r], Whole || wide, m[r], v[r]);
        else { load4<float>(t.m[j], i, have[r], Whole || wide, m[r]); load4<float>(t.v[j], i, have[r], Whole || wide, v[r]); }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!Whole && have[r] < 0) continue;
        const int64_t i = at + (r * kAdamBlock + (int)threadIdx.x) * 4;
        float root[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) left_alone += adam_element(h, g[r][k], p[r][k], m[r][k], v[r][k], root[k]) ? 0 : 1;
        store4<P>(t.p[j], i, have[r], Whole || wide, p[r]);
        if constexpr (Small) put_moments(t, j, i, have[r], Whole || wide, m[r], root);
        else { store4<float>(t.m[j], i, have[r], Whole || wide, m[r]); store4<float>(t.v[j], i, have[r], Whole || wide, v[r]); }
    }
    return left_alone;
}
template <bool Small, class P, class G>
__device__ __forceinline__ int adam_chunk(const AdamTable& t, const AdamHyper& h, uint32_t j, int64_t at, int64_t n, bool wide) {
    return wide && n - at >= kAdamChunk ? adam_chunk<Small, P, G, true>(t, h, j, at, n, true) : adam_chunk<Small, P, G, false>(t, h, j, at, n, wide);
}

template <bool Small>
__global__ void __launch_bounds__(kAdamBlock) adamw_kernel(AdamTable t, AdamHyper h, int64_t* skipped) {
    const uint32_t chunk = blockIdx.x, j = chunk_owner(t, chunk);
    const int64_t n = t.n[j], at = (int64_t)(chunk - t.first[j]) * kAdamChunk;
    const int kind = t.kind[j];
    const bool wide = kind & 16;
    int left_alone = 0;
    switch (kind & 15) {
        case SPP_F32 | SPP_F32 << 2: left_alone = adam_chunk<Small, float, float>(t, h, j, at, n, wide); break;
        case SPP_F32 | SPP_F16 << 2: left_alone = adam_chunk<Small, float, _Float16>(t, h, j, at, n, wide); break;
        case SPP_F32 | SPP_BF16 << 2: left_alone = adam_chunk<Small, float, __bf16>(t, h, j, at, n, wide); break;
        case SPP_BF16 | SPP_F32 << 2: left_alone = adam_chunk<Small, __bf16, float>(t, h, j, at, n, wide); break;
        case SPP_BF16 | SPP_F16 << 2: left_alone = adam_chunk<Small, __bf16, _Float16>(t, h, j, at, n, wide); break;
        case SPP_BF16 | SPP_BF16 << 2: left_alone = adam_chunk<Small, __bf16, __bf16>(t, h, j, at, n, wide); break;
    }
    if (left_alone) atomicAdd(reinterpret_cast<unsigned long long*>(skipped), (unsigned long long)left_alone);
}

// m and the root of v, as codes, from fp32 arrays, and back.  t.p: fp32 m, t.g: fp32 v.
__global__ void __launch_bounds__(kAdamBlock) adamw_load_kernel(AdamTable t) {
    const uint32_t chunk = blockIdx.x, j = chunk_owner(t, chunk);
    const int64_t n = t.n[j], at = (int64_t)(chunk - t.first[j]) * kAdamChunk;
    const bool wide = t.kind[j] & 16;
    for (int round = 0; round < kAdamPer / 4; ++round) {
        const int64_t i = at + (round * kAdamBlock + (int)threadIdx.x) * 4;
        if (n - (i - 4 * lane_id()) <= 0) break;
        const int have = n - i >= 4 ? 4 : n - i > 0 ? (int)(n - i) : 0;
        float m[4], v[4];
        load4<float>(t.p[j], i, have, wide, m);
        load4<float>(t.g[j], i, have, wide, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {                       // what no step can have left there counts as zero
            if ((__float_as_uint(m[k]) & 0x7F800000u) == 0x7F800000u) m[k] = 0.0f;
            if (!(v[k] >= 0.0f) || (__float_as_uint(v[k]) & 0x7F800000u) == 0x7F800000u) v[k] = 0.0f;
            v[k] = sqrtf(v[k]);
        }
        put_moments(t, j, i, have, wide, m, v);
    }
}
__global__ void __launch_bounds__(kAdamBlock) adamw_values_kernel(AdamTable t) {
    constexpr int R = kAdamPer / 4;
    const uint32_t chunk = blockIdx.x, j = chunk_owner(t, chunk);
    const int64_t n = t.n[j], at = (int64_t)(chunk - t.first[j]) * kAdamChunk;
    const bool wide = t.kind[j] & 16;
    if (wide && n - at >= kAdamChunk) {                     // all codes asked for before any is worked on
        const uint32_t* pm = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.m[j]) + at) + threadIdx.x;
        const uint32_t* pv = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.v[j]) + at) + threadIdx.x;
        const float* ps = t.scale[j] + 2 * (at / kAdamShared + (threadIdx.x >> 6));
        uint32_t cm[R], cv[R];
        float sm[R], sv[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            cm[r] = pm[r * kAdamBlock];
            cv[r] = pv[r * kAdamBlock];
            sm[r] = ps[2 * r * (kAdamBlock / kWave)];
            sv[r] = ps[2 * r * (kAdamBlock / kWave) + 1];
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t i = at + (r * kAdamBlock + (int)threadIdx.x) * 4;
            float m[4], v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) { m[k] = value_m((cm[r] >> (8 * k)) & 255u, sm[r]); v[k] = value_v((cv[r] >> (8 * k)) & 255u, sv[r]); }
            store4<float>(t.p[j], i, 4, true, m);
            store4<float>(const_cast<void*>(t.g[j]), i, 4, true, v);
        }
        return;
    }
    for (int r = 0; r < R; ++r) {
        const int64_t i = at + (r * kAdamBlock + (int)threadIdx.x) * 4;
        if (i >= n) break;
        const int have = n - i >= 4 ? 4 : (int)(n - i);
        float m[4], v[4];
        get_moments(t, j, i, have, wide, m, v);
        store4<float>(t.p[j], i, have, wide, m);
        store4<float>(const_cast<void*>(t.g[j]), i, have, wide, v);
    }
}

static int adam_check(const char* who, const spp_ctx* ctx, const spp_adamw_tensor* tensors, int32_t n_tensors, int32_t bits) {
    SPP_CHECK(ctx && (tensors || n_tensors == 0), SPP_E_ARG, "%s: null argument", who);
    SPP_CHECK(n_tensors >= 0, SPP_E_ARG, "%s: %d tensors", who, n_tensors);
    SPP_CHECK(bits == 32 || bits == 8, SPP_E_ARG, "%s: states of %d bits (32 or 8)", who, bits);
    for (int k = 0; k < n_tensors; ++k) {
        const spp_adamw_tensor& a = tensors[k];
        SPP_CHECK(a.n >= 0 && a.n <= SPP_ADAMW_MAX_ELEMENTS, SPP_E_ARG, "%s: tensor %d: n = %lld", who, k, (long long)a.n);
        SPP_CHECK((a.p_type == SPP_F32 || a.p_type == SPP_BF16) && is_type(a.g_type), SPP_E_ARG, "%s: tensor %d: types %d, %d", who, k, a.p_type,
                  a.g_type);
        SPP_CHECK(a.n == 0 || (a.d_p && a.d_g && a.d_m && a.d_v && (bits == 32 || a.d_scale)), SPP_E_ARG, "%s: tensor %d: null argument", who, k);
        const size_t state = bits == 32 ? 4 : 1;
        SPP_CHECK((uintptr_t)a.d_p % type_bytes(a.p_type) == 0 && (uintptr_t)a.d_g % type_bytes(a.g_type) == 0 && (uintptr_t)a.d_m % state == 0 &&
                      (uintptr_t)a.d_v % state == 0 && (bits == 32 || (uintptr_t)a.d_scale % 4 == 0),
                  SPP_E_ARG, "%s: tensor %d: an array is not aligned to its type", who, k);
    }
    return SPP_OK;
}
// Launches over as many tensors at a time as a table holds.  run(table, chunks)
template <class Run>
static int adam_launches(const spp_adamw_tensor* tensors, int32_t n_tensors, int32_t bits, Run run) {
    for (int k = 0; k < n_tensors;) {
        AdamTable t;
        memset(&t, 0, sizeof(t));
        memset(t.first, 0xFF, sizeof(t.first));
        int64_t chunks = 0;
        for (int j = 0; j < kAdamTensors && k < n_tensors; ++k) {
            const spp_adamw_tensor& a = tensors[k];
            if (a.n == 0) continue;
            const int64_t more = (a.n + kAdamChunk - 1) / kAdamChunk;
            if (chunks + more > 0xFFFFFFll) break;             // a grid has fewer than 2^32 threads
            const size_t state = bits == 32 ? 4 : 1;
            const bool wide = (uintptr_t)a.d_p % (4 * type_bytes(a.p_type)) == 0 && (uintptr_t)a.d_g % (4 * type_bytes(a.g_type)) == 0 &&
                              (uintptr_t)a.d_m % (4 * state) == 0 && (uintptr_t)a.d_v % (4 * state) == 0;
            t.p[j] = a.d_p; t.g[j] = a.d_g; t.m[j] = a.d_m; t.v[j] = a.d_v; t.scale[j] = a.d_scale; t.n[j] = a.n;
            t.first[j] = (uint32_t)chunks;
            t.kind[j] = (uint8_t)(a.p_type | a.g_type << 2 | (wide ? 16 : 0));
            chunks += more;
            ++j;
        }
        if (chunks == 0) break;
        run(t, (unsigned)chunks);
        SPP_HIP(hipGetLastError());
    }
    return SPP_OK;
}

}  // namespace spp

extern "C" int spp_adamw_step(spp_ctx* ctx, const spp_adamw_tensor* tensors, int32_t n_tensors, int32_t state_bits, const spp_adamw_hyper* hyper,
                              int64_t t, uint32_t flags) {
    using namespace spp;
    SPP_TRY(adam_check("spp_adamw_step", ctx, tensors, n_tensors, state_bits));
    SPP_CHECK(hyper, SPP_E_ARG, "spp_adamw_step: hyper is null");
    const double b1 = hyper->beta1, b2 = hyper->beta2;
    SPP_CHECK(b1 >= 0.0 && b1 < 1.0 && b2 >= 0.0 && b2 < 1.0 && (float)b1 < 1.0f && (float)b2 < 1.0f, SPP_E_ARG, "spp_adamw_step: betas %g, %g", b1, b2);
    SPP_CHECK((float)hyper->eps >= 0x1p-126f && isfinite((float)hyper->eps) && isfinite(hyper->lr) && hyper->lr >= 0.0 && isfinite(hyper->weight_decay) &&
                  hyper->weight_decay >= 0.0,
              SPP_E_ARG, "spp_adamw_step: lr %g, eps %g, weight decay %g", hyper->lr, hyper->eps, hyper->weight_decay);
    SPP_CHECK(t >= 1, SPP_E_ARG, "spp_adamw_step: step %lld (the first is 1)", (long long)t);
    SPP_HIP(hipSetDevice(ctx->device));
    // the bias corrections of step t and the learning rate are arguments of the kernel: replays would repeat step t
    hipStreamCaptureStatus recording = hipStreamCaptureStatusNone;
    SPP_HIP(hipStreamIsCapturing(ctx->stream, &recording));
    SPP_CHECK(recording == hipStreamCaptureStatusNone, SPP_E_ARG, "spp_adamw_step: the stream records a graph, whose replays would repeat step %lld",
              (long long)t);
    AdamHyper h;
    h.b1 = (float)b1; h.c1 = (float)(1.0 - b1); h.b2 = (float)b2; h.c2 = (float)(1.0 - b2);
    h.rs = (float)(1.0 / sqrt(1.0 - pow(b2, (double)t)));
    h.eps = (float)hyper->eps;
    h.decay = (float)(1.0 - hyper->lr * hyper->weight_decay);
    h.step = (float)(hyper->lr / (1.0 - pow(b1, (double)t)));
    ScopedTimer timer(ctx, SPP_T_ADAMW, ctx->stream);
    int64_t* skipped = ctx->totals + 9;
    SPP_TRY(adam_launches(tensors, n_tensors, state_bits, [&](const AdamTable& table, unsigned chunks) {
        if (state_bits == 32) adamw_kernel<false><<<chunks, kAdamBlock, 0, ctx->stream>>>(table, h, skipped);
        else adamw_kernel<true><<<chunks, kAdamBlock, 0, ctx->stream>>>(table, h, skipped);
    }));
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}

// Load and values: the 8-bit state of `tensors`, their fp32 moments in place of parameter and gradient.
static int adam_moments(const char* who, spp_ctx* ctx, const spp_adamw_tensor* tensors, int32_t n_tensors, float* const* d_m, float* const* d_v,
                        uint32_t flags, bool load) {
    using namespace spp;
    SPP_CHECK(ctx && ((tensors && d_m && d_v) || n_tensors == 0), SPP_E_ARG, "%s: null argument", who);
    SPP_CHECK(n_tensors >= 0, SPP_E_ARG, "%s: %d tensors", who, n_tensors);
    for (int k = 0; k < n_tensors; ++k) {                   // all of them before any work
        spp_adamw_tensor a = tensors[k];
        a.d_p = d_m[k]; a.d_g = d_v[k]; a.p_type = SPP_F32; a.g_type = SPP_F32;
        SPP_TRY(adam_check(who, ctx, &a, 1, 8));
    }
    SPP_HIP(hipSetDevice(ctx->device));
    for (int k = 0; k < n_tensors; k += kAdamTensors) {
        spp_adamw_tensor part[kAdamTensors];
        const int here = n_tensors - k < kAdamTensors ? n_tensors - k : kAdamTensors;
        for (int j = 0; j < here; ++j) {
            part[j] = tensors[k + j];
            part[j].d_p = d_m[k + j]; part[j].d_g = d_v[k + j]; part[j].p_type = SPP_F32; part[j].g_type = SPP_F32;
        }
        SPP_TRY(adam_launches(part, here, 8, [&](const AdamTable& table, unsigned chunks) {
            if (load) adamw_load_kernel<<<chunks, kAdamBlock, 0, ctx->stream>>>(table);
            else adamw_values_kernel<<<chunks, kAdamBlock, 0, ctx->stream>>>(table);
        }));
    }
    if (flags & SPP_SYNC) SPP_HIP(hipStreamSynchronize(ctx->stream));
    return SPP_OK;
}
extern "C" int spp_adamw_load(spp_ctx* ctx, const spp_adamw_tensor* tensors, int32_t n_tensors, const float* const* d_m, const float* const* d_v,
                              uint32_t flags) {
    return adam_moments("spp_adamw_load", ctx, tensors, n_tensors, const_cast<float* const*>(d_m), const_cast<float* const*>(d_v), flags, true);
}
extern "C" int spp_adamw_values(spp_ctx* ctx, const spp_adamw_tensor* tensors, int32_t n_tensors, float* const* d_m, float* const* d_v,
                                uint32_t flags) {
    return adam_moments("spp_adamw_values", ctx, tensors, n_tensors, d_m, d_v, flags, false);
}
