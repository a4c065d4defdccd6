// AdamW over many tensors in one launch, optimiser state in fp32 or in 8 bits.
#pragma once
#include "adamw_element.cuh"
#include "local_common.cuh"

namespace {

// The recurrence is that of adamw1.  A work unit is 2048 consecutive elements of one tensor, eight
// warps of 256; the table of tensors travels in the launch's parameters (nothing on the device can be
// stale), and a block finds a unit's tensor by bisection.
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
constexpr int kUnit = 2048;
constexpr int kStateBlock = 256;
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

// Two elements of a pair share one 32-bit hash (the finalizer of MurmurHash3, by Austin Appleby).
__device__ __forceinline__ unsigned pair_hash(unsigned pair, unsigned seed_term) {
    unsigned h = pair + seed_term;
    h ^= h >> 16; h *= 0x85ebca6bu;
    h ^= h >> 13; h *= 0xc2b2ae35u;
    return h ^ (h >> 16);
}

// e4m3 magnitudes: an fp32 number's bits from bit 20 on, once 2^-120 has matched the exponents' offsets.
__device__ __forceinline__ float e4m3_value(unsigned code) { return __uint_as_float((code & 0x7fu) << 20) * 0x1p120f; }
__device__ __forceinline__ unsigned e4m3_random(float y, unsigned bits20) {
    const unsigned c = (__float_as_uint(__fmul_rn(y, 0x1p-120f)) + bits20) >> 20;
    return min(c, 0x7eu);
}
__device__ __forceinline__ unsigned e4m3_nearest2(float lo, float hi) {       // two codes
    unsigned short c;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(hi), "f"(lo));
    return c;
}
// Scale of a block from its largest magnitude (fp32 bits order as magnitudes do; NaN is above infinity).
__device__ __forceinline__ void block_scale(unsigned top_bits, float &scale, float &over) {
    scale = __fmul_rn(__uint_as_float(__reduce_max_sync(0xffffffffu, top_bits)), 1.0f / 448.0f);
    if (scale < 0x1p-126f) scale = 0.f;
    over = scale == 0.f ? 0.f : __fdiv_rn(1.f, scale);
}

// Eight elements of a lane: consecutive (kVec) or 32 apart (any alignment).
template <typename TP, typename TG, bool kVec>
__device__ __forceinline__ void adamw8_elements(const TensorEntry &t, long long base, int lane, const AdamArgs &a, float b1,
                                                float gs, unsigned seed_term) {
    const long long blk = base / kStateBlock;
    const float ms = __ldcg(t.m_scale + blk), rs = __ldcg(t.v_scale + blk);
    TP *param = static_cast<TP *>(t.param);
    const TG *grad = static_cast<const TG *>(t.grad);
    unsigned char *mc = static_cast<unsigned char *>(t.m), *rc = static_cast<unsigned char *>(t.v);
    float p[8], g[8], m[8], r[8];
    unsigned cm[8], cr[8];
    const long long e0 = base + (kVec ? lane * 8 : lane);
    auto at = [&](int k) { return kVec ? e0 + k : e0 + 32 * k; };
    const bool whole = kVec && e0 + 8 <= t.n;
    if (whole) {
        load_vec<TP, 8>(param + e0, p);
        load_vec<TG, 8>(grad + e0, g);
        const uint2 um = __ldcs(reinterpret_cast<const uint2 *>(mc + e0)), ur = __ldcs(reinterpret_cast<const uint2 *>(rc + e0));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            cm[k] = ((k < 4 ? um.x : um.y) >> (8 * (k & 3))) & 0xffu;
            cr[k] = ((k < 4 ? ur.x : ur.y) >> (8 * (k & 3))) & 0xffu;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool in = at(k) < t.n;
            p[k] = in ? to_float(param[at(k)]) : 0.f;
            g[k] = in ? to_float(grad[at(k)]) : 0.f;
            cm[k] = in ? mc[at(k)] : 0u;
            cr[k] = in ? rc[at(k)] : 0u;
        }
    }
    unsigned mtop = 0, rtop = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float mag = e4m3_value(cm[k]);
        const float old = __fmul_rn((cm[k] & 0x80u) ? -mag : mag, ms);
        const float root = __fmul_rn(e4m3_value(cr[k]), rs);
        const float gk = __fmul_rn(g[k], gs);
        m[k] = __fadd_rn(__fmul_rn(old, b1), __fmul_rn(gk, a.one_minus_b1));
        const float v = __fadd_rn(__fmul_rn(__fmul_rn(root, root), a.b2), __fmul_rn(__fmul_rn(gk, gk), a.one_minus_b2));
        r[k] = __fsqrt_rn(v);
        mtop = max(mtop, __float_as_uint(m[k]) & 0x7fffffffu);
        rtop = max(rtop, __float_as_uint(r[k]) & 0x7fffffffu);
        p[k] = __fmul_rn(p[k], t.decay);
        p[k] = __fmaf_rn(-a.step_size, __fdiv_rn(m[k], __fmaf_rn(r[k], a.inv_sqrt_bc2, a.eps)), p[k]);
    }
    float msc, mover, rsc, rover;
    block_scale(mtop, msc, mover);
    block_scale(rtop, rsc, rover);
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const unsigned c = e4m3_nearest2(__fmul_rn(m[k], mover), __fmul_rn(m[k + 1], mover));
        cm[k] = c & 0xffu;
        cm[k + 1] = (c >> 8) & 0xffu;
    }
    unsigned h = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const unsigned idx = (unsigned)at(k);
        if (!kVec || (k & 1) == 0) h = pair_hash(idx >> 1, seed_term);
        const unsigned half = (idx & 1u) ? h >> 16 : h & 0xffffu;
        cr[k] = e4m3_random(__fmul_rn(r[k], rover), half << 4);
        if (r[k] > 0.f && rover > 0.f) cr[k] = max(cr[k], 1u);
    }
    if (whole) {
        uint2 um, ur;
        um.x = cm[0] | cm[1] << 8 | cm[2] << 16 | cm[3] << 24;
        um.y = cm[4] | cm[5] << 8 | cm[6] << 16 | cm[7] << 24;
        ur.x = cr[0] | cr[1] << 8 | cr[2] << 16 | cr[3] << 24;
        ur.y = cr[4] | cr[5] << 8 | cr[6] << 16 | cr[7] << 24;
        store_vec<TP, 8>(param + e0, p);
        __stcs(reinterpret_cast<uint2 *>(mc + e0), um);
        __stcs(reinterpret_cast<uint2 *>(rc + e0), ur);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (at(k) < t.n) {
                param[at(k)] = from_float<TP>(p[k]);
                mc[at(k)] = (unsigned char)cm[k];
                rc[at(k)] = (unsigned char)cr[k];
            }
    }
    if (lane == 0) {
        t.m_scale[blk] = msc;
        t.v_scale[blk] = rsc;
    }
}

template <typename TP, typename TG, bool kVec>
__device__ __forceinline__ void adamw32_elements(const TensorEntry &t, long long base, int lane, const AdamArgs &a, float gs) {
    TP *param = static_cast<TP *>(t.param);
    const TG *grad = static_cast<const TG *>(t.grad);
    float *pm = static_cast<float *>(t.m), *pv = static_cast<float *>(t.v);
    AdamArgs mine = a;
    mine.decay = t.decay;
    float p[8], g[8], m[8], v[8];
    const long long e0 = base + (kVec ? lane * 8 : lane);
    auto at = [&](int k) { return kVec ? e0 + k : e0 + 32 * k; };
    const bool whole = kVec && e0 + 8 <= t.n;
    if (whole) {
        load_vec<TP, 8>(param + e0, p);
        load_vec<TG, 8>(grad + e0, g);
        load_vec<float, 8>(pm + e0, m);
        load_vec<float, 8>(pv + e0, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (at(k) < t.n) {
                p[k] = to_float(param[at(k)]);
                g[k] = to_float(grad[at(k)]);
                m[k] = pm[at(k)];
                v[k] = pv[at(k)];
            } else {
                p[k] = g[k] = m[k] = v[k] = 0.f;
            }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) adamw1(p[k], m[k], v[k], __fmul_rn(g[k], gs), mine);
    if (whole) {
        store_vec<TP, 8>(param + e0, p);
        store_vec<float, 8>(pm + e0, m);
        store_vec<float, 8>(pv + e0, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (at(k) < t.n) {
                param[at(k)] = from_float<TP>(p[k]);
                pm[at(k)] = m[k];
                pv[at(k)] = v[k];
            }
    }
}

template <typename TP, typename TG, int kBits, int kEntries>
__global__ void __launch_bounds__(kTensorThreads) adamw_tensors_kernel(const __grid_constant__ TensorTable<kEntries> tab) {
    const float gs = tab.grad_scale ? __ldg(tab.grad_scale) : 1.f;
    if (!isfinite(gs)) return;                              // a step whose gradients overflowed is skipped whole
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int u = blockIdx.x; u < tab.units; u += gridDim.x) {
        int lo = 0, hi = tab.n;                             // the last tensor with first_unit <= u
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (tab.e[mid].first_unit <= u) lo = mid; else hi = mid;
        }
        const TensorEntry &t = tab.e[lo];
        const long long base = (long long)(u - t.first_unit) * kUnit + warp * kStateBlock;
        if (base >= t.n) continue;
        const uintptr_t wide = reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.grad);
        const uintptr_t states = reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v);
        if constexpr (kBits == 32) {
            if (((wide | states) & 15u) == 0) adamw32_elements<TP, TG, true>(t, base, lane, tab.args, gs);
            else adamw32_elements<TP, TG, false>(t, base, lane, tab.args, gs);
        } else {
            if ((wide & 15u) == 0 && (states & 7u) == 0) adamw8_elements<TP, TG, true>(t, base, lane, tab.args, tab.b1, gs, tab.seed_term);
            else adamw8_elements<TP, TG, false>(t, base, lane, tab.args, tab.b1, gs, tab.seed_term);
        }
    }
}

}  // namespace
