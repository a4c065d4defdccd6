// AdamW over many tensors in one launch, optimiser state in fp32 or in 8 bits.
#pragma once
#include "adamw_element.cuh"
#include "local_common.cuh"
#include <cuda_fp16.h>
#include <type_traits>

namespace {

// The recurrence is that of adamw1.  A work unit is 256 consecutive elements of one tensor, held by a
// warp, eight a lane; the table of tensors travels in the launch's parameters (nothing on the device can
// be stale).  A warp finds its first unit's tensor by bisection and walks the table from there.
//
// States in 8 bits: blocks of 256 elements counted from the tensor's start, which is what a warp holds.
//   m = code_m * scale_m,  sqrt(v) = code_r * scale_r,  codes e4m3, scale = (block's largest) / 448.
// The root is stored because e4m3 spans 2^18: of v itself that would be nine binary orders of the
// gradient's size.  m is rounded to nearest.  sqrt(v) is rounded up or down at random (in proportion,
// from a hash of element number and seed): with beta2 = 0.999 a step changes sqrt(v) by less than half
// of e4m3's spacing, and rounded to nearest it would never move.  A root that is not zero is never
// stored as zero, so no update is divided by eps alone.  The parameters' update uses the new
// moments before they are rounded.  The state arithmetic is a fixed sequence of separately rounded fp32
// operations (no fused multiply-adds), so that a few lines of plain code give the same codes.

constexpr int kTensorThreads = 256;
constexpr int kTensorWarps = kTensorThreads / 32;
constexpr int kStateBlock = 256;                       // elements of a work unit, and of a block of 8-bit states
constexpr int kSmallTable = 60, kLargeTable = 500;     // table sizes: 4 KB and 32 KB of launch parameters

struct TensorEntry {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    long long n;
    float decay;                 // 1 - lr * weight decay of this tensor
    int first_unit;
};

template <int kEntries>
struct TensorTable {
    TensorEntry e[kEntries];
    const float *grad_scale;
    AdamArgs args;               // scalars only
    float b1;
    unsigned seed_term;
    int n, units;
};

// ---------------------------------------------------------------- eight elements of a lane, as stored
// kVec: elements 8 lane .. 8 lane + 7 of the unit, in 16-byte accesses (8-byte for codes); otherwise elements
// lane, lane + 32, ..., which any alignment allows.  Elements past the tensor's end read as zero.

template <typename T> struct Raw { unsigned w[2 * sizeof(T)]; };

template <bool kVec> __device__ __forceinline__ long long element_at(long long e0, int k) { return kVec ? e0 + k : e0 + 32 * k; }

template <typename T, bool kVec>
__device__ __forceinline__ Raw<T> load_raw(const void *base, long long e0, long long n) {
    const T *p = static_cast<const T *>(base);
    constexpr int kWords = 2 * (int)sizeof(T);
    Raw<T> r;
    if (kVec && e0 + 8 <= n) {
        if constexpr (kWords == 2) {
            const uint2 u = __ldcs(reinterpret_cast<const uint2 *>(p + e0));
            r.w[0] = u.x; r.w[1] = u.y;
        } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(p + e0) + i);
                r.w[4 * i] = u.x; r.w[4 * i + 1] = u.y; r.w[4 * i + 2] = u.z; r.w[4 * i + 3] = u.w;
            }
        }
        return r;
    }
    using U = typename std::conditional<sizeof(T) == 4, unsigned, typename std::conditional<sizeof(T) == 2, unsigned short, unsigned char>::type>::type;
    constexpr int kPer = 4 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        r.w[i] = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const long long e = element_at<kVec>(e0, i * kPer + j);
            if (e < n) r.w[i] |= (unsigned)__ldcs(reinterpret_cast<const U *>(p) + e) << (8 * (int)sizeof(T) * j);
        }
    }
    return r;
}

template <typename T, bool kVec>
__device__ __forceinline__ void store_raw(void *base, long long e0, long long n, const Raw<T> &r) {
    T *p = static_cast<T *>(base);
    constexpr int kWords = 2 * (int)sizeof(T);
    if (kVec && e0 + 8 <= n) {
        if constexpr (kWords == 2) {
            __stcs(reinterpret_cast<uint2 *>(p + e0), make_uint2(r.w[0], r.w[1]));
        } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i)
                __stcs(reinterpret_cast<uint4 *>(p + e0) + i, make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]));
        }
        return;
    }
    using U = typename std::conditional<sizeof(T) == 4, unsigned, typename std::conditional<sizeof(T) == 2, unsigned short, unsigned char>::type>::type;
    constexpr int kPer = 4 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < kWords; ++i)
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const long long e = element_at<kVec>(e0, i * kPer + j);
            if (e < n) __stcs(reinterpret_cast<U *>(p) + e, (U)(r.w[i] >> (8 * (int)sizeof(T) * j)));
        }
}

__device__ __forceinline__ float2 pair_of(const Raw<float> &r, int i) { return make_float2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1])); }
__device__ __forceinline__ float2 pair_of(const Raw<bf16> &r, int i) { return make_float2(bf16_low(r.w[i]), bf16_high(r.w[i])); }
__device__ __forceinline__ void set_pair(Raw<float> &r, int i, float2 f) { r.w[2 * i] = __float_as_uint(f.x); r.w[2 * i + 1] = __float_as_uint(f.y); }
__device__ __forceinline__ void set_pair(Raw<bf16> &r, int i, float2 f) { r.w[i] = bf16_pair(f.x, f.y); }

// ---------------------------------------------------------------- 8-bit states

using code8 = unsigned char;

__device__ __forceinline__ float2 e4m3_values(const Raw<code8> &r, int i) {       // codes 2 i, 2 i + 1
    unsigned h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)(r.w[i >> 1] >> (16 * (i & 1)))));   // exact
    return __half22float2(*reinterpret_cast<__half2 *>(&h));
}
__device__ __forceinline__ unsigned e4m3_nearest(float2 y) {
    unsigned short c;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(y.y), "f"(y.x));
    return c;
}
// Two elements of a pair share one 32-bit hash (the finalizer of MurmurHash3, by Austin Appleby).
__device__ __forceinline__ unsigned pair_hash(unsigned pair, unsigned seed_term) {
    unsigned h = pair + seed_term;
    h ^= h >> 16; h *= 0x85ebca6bu;
    h ^= h >> 13; h *= 0xc2b2ae35u;
    return h ^ (h >> 16);
}
// e4m3 magnitudes are an fp32 number's bits from bit 20 on, once 2^-120 has matched the exponents'
// offsets (z = y 2^-120; y is at most 448 and a few ulp).  16 random bits are added below bit 20; the code comes
// back in the top byte.  What is not zero does not become zero.
__device__ __forceinline__ unsigned e4m3_random_top(float y, float z, unsigned random_at_8) {
    const unsigned t = (__float_as_uint(z) << 4) + random_at_8;
    return y > 0.f ? max(t, 1u << 24) : t;
}
__device__ __forceinline__ float max_abs(float a, float b) {                      // NaN if either is
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(fabsf(b)));
    return d;
}
// Scale of a block from its largest magnitude (fp32 bits order as magnitudes do; NaN is above infinity).
__device__ __forceinline__ void block_scale(float top, float &scale, float &over) {
    scale = __fmul_rn(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu)), 1.0f / 448.0f);
    if (scale < 0x1p-126f) scale = 0.f;
    over = scale == 0.f ? 0.f : __fdiv_rn(1.f, scale);
}

template <typename TP, typename TG>
struct Unit8 {
    Raw<TP> p;
    Raw<TG> g;
    Raw<code8> m, r;
    float ms, rs;
};

template <typename TP, typename TG, bool kVec>
__device__ __forceinline__ void load_unit8(const TensorEntry &t, int blk, int lane, Unit8<TP, TG> &u) {
    const long long e0 = (long long)blk * kStateBlock + (kVec ? lane * 8 : lane);
    u.p = load_raw<TP, kVec>(t.param, e0, t.n);
    u.g = load_raw<TG, kVec>(t.grad, e0, t.n);
    u.m = load_raw<code8, kVec>(t.m, e0, t.n);
    u.r = load_raw<code8, kVec>(t.v, e0, t.n);
    u.ms = __ldcg(t.m_scale + blk);
    u.rs = __ldcg(t.v_scale + blk);
}

template <typename TP, typename TG, bool kVec>
__device__ __forceinline__ void step_unit8(const TensorEntry &t, int blk, int lane, Unit8<TP, TG> &u, const AdamArgs &a, float b1,
                                           float gs, unsigned seed_term) {
    const long long e0 = (long long)blk * kStateBlock + (kVec ? lane * 8 : lane);
    float2 m[4], r[4];
    float mtop = 0.f, rtop = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 g = mul2(pair_of(u.g, i), both(gs));
        const float2 old = mul2(e4m3_values(u.m, i), both(u.ms)), root = mul2(e4m3_values(u.r, i), both(u.rs));
        const float2 m0 = mul2(old, both(b1)), m1 = mul2(g, both(a.one_minus_b1));
        const float2 v0 = mul2(mul2(root, root), both(a.b2)), v1 = mul2(mul2(g, g), both(a.one_minus_b2));
        m[i] = make_float2(__fadd_rn(m0.x, m1.x), __fadd_rn(m0.y, m1.y));
        r[i] = make_float2(__fsqrt_rn(__fadd_rn(v0.x, v1.x)), __fsqrt_rn(__fadd_rn(v0.y, v1.y)));
        mtop = max_abs(max_abs(mtop, m[i].x), m[i].y);
        rtop = max_abs(max_abs(rtop, r[i].x), r[i].y);
        // the update itself, in 2 ulp: it is small against the parameter that it is added to
        const float2 den = fma2(r[i], both(a.inv_sqrt_bc2), both(a.eps));
        const float2 step = make_float2(__fdividef(m[i].x, den.x), __fdividef(m[i].y, den.y));
        set_pair(u.p, i, fma2(both(-a.step_size), step, mul2(pair_of(u.p, i), both(t.decay))));
    }
    store_raw<TP, kVec>(t.param, e0, t.n, u.p);
    float msc, mover, rsc, rover;
    block_scale(mtop, msc, mover);
    block_scale(rtop, rsc, rover);
    unsigned top[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned c = e4m3_nearest(mul2(m[i], both(mover)));
        if (i & 1) u.m.w[i >> 1] |= c << 16;
        else u.m.w[i >> 1] = c;
        const float2 y = mul2(r[i], both(rover)), z = mul2(y, both(0x1p-120f));
        if (kVec) {
            const unsigned h = pair_hash(((unsigned)e0 >> 1) + i, seed_term);
            top[2 * i] = e4m3_random_top(y.x, z.x, __byte_perm(h, 0, 0x4104));          // low half at bit 8
            top[2 * i + 1] = e4m3_random_top(y.y, z.y, __byte_perm(h, 0, 0x4324));      // high half at bit 8
        } else {
            const unsigned first = (unsigned)element_at<kVec>(e0, 2 * i);          // both of the lane's parity
            const unsigned h0 = pair_hash(first >> 1, seed_term), h1 = pair_hash((first >> 1) + 16, seed_term);
            const unsigned pick = (first & 1) ? 0x4324 : 0x4104;
            top[2 * i] = e4m3_random_top(y.x, z.x, __byte_perm(h0, 0, pick));
            top[2 * i + 1] = e4m3_random_top(y.y, z.y, __byte_perm(h1, 0, pick));
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        u.r.w[i] = __byte_perm(__byte_perm(top[4 * i], top[4 * i + 1], 0x0073), __byte_perm(top[4 * i + 2], top[4 * i + 3], 0x0073), 0x5410);
    store_raw<code8, kVec>(t.m, e0, t.n, u.m);
    store_raw<code8, kVec>(t.v, e0, t.n, u.r);
    if (lane == 0) {
        t.m_scale[blk] = msc;
        t.v_scale[blk] = rsc;
    }
}

// ---------------------------------------------------------------- fp32 states

template <typename TP, typename TG, bool kVec>
__device__ __forceinline__ void step_unit32(const TensorEntry &t, int blk, int lane, const AdamArgs &a, float gs) {
    const long long e0 = (long long)blk * kStateBlock + (kVec ? lane * 8 : lane);
    AdamArgs mine = a;
    mine.decay = t.decay;
    Raw<TP> p = load_raw<TP, kVec>(t.param, e0, t.n);
    const Raw<TG> g = load_raw<TG, kVec>(t.grad, e0, t.n);
    Raw<float> m = load_raw<float, kVec>(t.m, e0, t.n), v = load_raw<float, kVec>(t.v, e0, t.n);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 pp = pair_of(p, i), mm = pair_of(m, i), vv = pair_of(v, i);
        const float2 gg = pair_of(g, i);
        adamw1(pp.x, mm.x, vv.x, __fmul_rn(gg.x, gs), mine);
        adamw1(pp.y, mm.y, vv.y, __fmul_rn(gg.y, gs), mine);
        set_pair(p, i, pp);
        set_pair(m, i, mm);
        set_pair(v, i, vv);
    }
    store_raw<TP, kVec>(t.param, e0, t.n, p);
    store_raw<float, kVec>(t.m, e0, t.n, m);
    store_raw<float, kVec>(t.v, e0, t.n, v);
}

// ---------------------------------------------------------------- the kernel

template <int kBits>
__device__ __forceinline__ bool takes_vectors(const TensorEntry &t) {
    const uintptr_t wide = reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.grad);
    const uintptr_t states = reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v);
    return kBits == 32 ? ((wide | states) & 15u) == 0 : (wide & 15u) == 0 && (states & 7u) == 0;
}

template <typename TP, typename TG, int kBits, int kEntries>
__global__ void __launch_bounds__(kTensorThreads, kBits == 8 ? 4 : 3)
adamw_tensors_kernel(const __grid_constant__ TensorTable<kEntries> tab) {
    const float gs = tab.grad_scale ? __ldg(tab.grad_scale) : 1.f;
    if (!isfinite(gs)) return;                              // a step whose gradients overflowed is skipped whole
    const int lane = threadIdx.x & 31;
    const int stride = gridDim.x * kTensorWarps;
    int u = blockIdx.x * kTensorWarps + (threadIdx.x >> 5);
    if (u >= tab.units) return;
    int k = 0, hi = tab.n;                                  // the last tensor with first_unit <= u
    while (hi - k > 1) {
        const int mid = (k + hi) >> 1;
        if (tab.e[mid].first_unit <= u) k = mid; else hi = mid;
    }
    for (; u < tab.units; u += stride) {
        while (k + 1 < tab.n && tab.e[k + 1].first_unit <= u) ++k;
        const TensorEntry &t = tab.e[k];
        const int blk = u - t.first_unit;
        if constexpr (kBits == 32) {
            if (takes_vectors<kBits>(t)) step_unit32<TP, TG, true>(t, blk, lane, tab.args, gs);
            else step_unit32<TP, TG, false>(t, blk, lane, tab.args, gs);
        } else {
            Unit8<TP, TG> x;
            if (takes_vectors<kBits>(t)) {
                load_unit8<TP, TG, true>(t, blk, lane, x);
                step_unit8<TP, TG, true>(t, blk, lane, x, tab.args, tab.b1, gs, tab.seed_term);
            } else {
                load_unit8<TP, TG, false>(t, blk, lane, x);
                step_unit8<TP, TG, false>(t, blk, lane, x, tab.args, tab.b1, gs, tab.seed_term);
            }
        }
    }
}

}  // namespace
