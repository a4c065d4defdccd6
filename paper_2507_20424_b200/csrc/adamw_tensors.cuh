// AdamW over many tensors in one launch, optimiser state in fp32 or in 8 bits.
#pragma once
#include "adamw_element.cuh"
#include "local_common.cuh"
#include <cuda_fp16.h>
#include <type_traits>

namespace {

// The recurrence is that of adamw1.  A work unit is 256 consecutive elements of one tensor, held by a
// warp, eight a lane; the table of tensors travels in the launch's parameters (nothing on the device can
// be stale).  A warp finds a unit's tensor in it.
//
// States in 8 bits: blocks of 256 elements counted from the tensor's start, which is what a warp holds.
//   m = code_m * scale_m,  sqrt(v) = code_r * scale_r,  codes e4m3, scale = (block's largest) / 448.
// The root is stored because e4m3 spans 2^18: of v itself that would be nine binary orders of the
// gradient's size.  m is rounded to nearest.  sqrt(v) is rounded up or down at random (in proportion,
// from a hash of element number and seed): with beta2 = 0.999 a step changes sqrt(v) by less than half
// of e4m3's spacing, and rounded to nearest it would never move.  (m stops short in the same way where
// (1 - beta1) |g - m| stays below half of its spacing, 3 to 6 % of m, and the gradients bring no noise of their own: 1.8
// times its average after a drop to 0.3 with beta1 = 0.9, not at all with noise of 30 %.)  A root that is not zero is never
// stored as zero, so no update is divided by eps alone.  The parameters' update uses the new
// moments before they are rounded.  The state arithmetic is a fixed sequence of separately rounded fp32
// operations (no fused multiply-adds), so that a few lines of plain code give the same codes.

constexpr int kTensorThreads = 256;
constexpr int kTensorWarps = kTensorThreads / 32;
constexpr int kStateBlock = 256;                       // elements of a work unit, and of a block of 8-bit states
constexpr int kGroup = 4;                              // units that a warp takes at a time with 8-bit states, where there are enough
constexpr int kSmallTable = 50, kLargeTable = 440;     // table sizes: under 4 KB and 32 KB of launch parameters

// Resident blocks an SM.  Fewer loads in flight run faster once there are enough of them, since reads and writes
// share the memory: fp32 states with fp32 parameters and gradients 2 blocks (86.6M elements: 365 us; 3: 433 us, 4: 445), with
// bf16 ones 3 (297 us; 2 and 4: 333 us), with one of each 3 as well, although fp32 parameters with bf16 gradients take 393 us so and
// 355 with 2 (4: 422).  8-bit states are bound by instructions and registers: 2 blocks of 128 registers and groups of four units
// (300M bf16: 534 us; 3 blocks and groups of 2: 587 us; 4 blocks and single units: 726 us).  fp32 parameters with fp32 gradients
// are 28 bytes a thread short of registers there (86.6M in packed rows: 266 us; groups of 2: 299).
template <typename TP, typename TG, int kBits>
struct TensorShape { static constexpr int kBlocks = kBits == 8 || sizeof(TP) + sizeof(TG) == 8 ? 2 : 3; };

struct TensorEntry {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    long long n;
    float decay;                 // 1 - lr * weight decay of this tensor
    int first_unit;              // 8 bits: of those that are taken one at a time
    union {
        int lead;                // 32 bits: elements that the first unit begins before the tensor (0 .. 255); -1: only accesses of
                                 // any alignment
        int first_group;         // 8 bits
    };
};

template <int kEntries>
struct TensorTable {
    TensorEntry e[kEntries];
    const float *grad_scale;
    AdamArgs args;               // scalars only
    float b1;
    unsigned seed_term;
    int n, units, groups;        // 8 bits: a tensor begins with its groups of kGroup units, the units are the rest
};

// ---------------------------------------------------------------- eight elements of a lane, as stored
enum Access {
    kAnyAlignment,   // elements lane, lane + 32, ... of the unit; those outside the tensor read as zero and are not written
    kAligned,        // elements 8 lane .. 8 lane + 7 of a unit that lies inside its tensor, in 16-byte accesses (8-byte ones for codes)
    kSkewed          // the same for a unit that does not start on a 16-byte boundary: read and written in the aligned 16-byte
                     // pieces that cover it, and moved into place between neighbouring lanes.  Pieces reach over the unit's ends
                     // into the same 16 bytes as one of its elements: what is read there is not used, and those two pieces are
                     // written element by element.  Codes have to be 8-byte aligned all the same.
};

template <typename T> struct Raw { unsigned w[2 * sizeof(T)]; };
template <typename T> struct Bits { using type = unsigned; };
template <> struct Bits<bf16> { using type = unsigned short; };
template <> struct Bits<unsigned char> { using type = unsigned char; };

// Bytes by which a tensor's units start after a 16-byte boundary: the same for all of them.
__device__ __forceinline__ unsigned skew(const void *p) { return (unsigned)(reinterpret_cast<uintptr_t>(p) & 15u); }

// A lane's element k of eight, counted from the unit's first.
template <int kAccess> __device__ __forceinline__ int lane_element(int lane, int k) { return kAccess == kAnyAlignment ? lane + 32 * k : 8 * lane + k; }

// `first`: the unit's first element (may be negative with kAnyAlignment).
template <typename T, int kAccess>
__device__ __forceinline__ Raw<T> load_raw(const void *base, long long first, long long n, int lane) {
    const T *p = static_cast<const T *>(base);
    constexpr int kWords = 2 * (int)sizeof(T), kPer = 4 / (int)sizeof(T);
    Raw<T> r;
    if constexpr (kAccess == kAnyAlignment) {
        using U = typename Bits<T>::type;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            r.w[i] = 0;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const long long e = first + lane_element<kAccess>(lane, i * kPer + j);
                if (e >= 0 && e < n) r.w[i] |= (unsigned)__ldcs(reinterpret_cast<const U *>(p) + e) << (8 * (int)sizeof(T) * j);
            }
        }
    } else if constexpr (kWords == 2) {
        const uint2 u = __ldcs(reinterpret_cast<const uint2 *>(p + first + 8 * lane));
        r.w[0] = u.x; r.w[1] = u.y;
    } else {                                                  // kSkewed: the covering pieces, for settle()
        const char *q = reinterpret_cast<const char *>(p + first + 8 * lane) - (kAccess == kSkewed ? skew(p) : 0u);
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
            const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(q) + i);
            r.w[4 * i] = u.x; r.w[4 * i + 1] = u.y; r.w[4 * i + 2] = u.z; r.w[4 * i + 3] = u.w;
        }
    }
    return r;
}

// x[j] <- the 32 bits that start `off` bytes after word j (off even, below 16)
template <int kWords>
__device__ __forceinline__ void move_down(unsigned (&x)[kWords + 4], unsigned off) {
    if (off & 8u) {
#pragma unroll
        for (int j = 0; j < kWords + 2; ++j) x[j] = x[j + 2];
    }
    if (off & 4u) {
#pragma unroll
        for (int j = 0; j < kWords + 1; ++j) x[j] = x[j + 1];
    }
    if (off & 2u) {
#pragma unroll
        for (int j = 0; j < kWords; ++j) x[j] = __byte_perm(x[j], x[j + 1], 0x5432);
    }
}

// The pieces that cover a stretch of whole units end 16 bytes later if they are skewed: that last piece, in lane 0.
template <typename T>
__device__ __forceinline__ uint4 load_end(const void *base, long long end, int lane) {
    const T *p = static_cast<const T *>(base);
    uint4 u = make_uint4(0, 0, 0, 0);
    if (lane == 0 && skew(p)) u = __ldcs(reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p + end) - skew(p)));
    return u;
}
template <typename T>
__device__ __forceinline__ uint4 first_piece(const Raw<T> &r) { return make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]); }
// Moves a skewed unit's elements to their lanes; `next`: the 16 bytes that follow the unit's pieces (lane 0's counts).
template <typename T>
__device__ __forceinline__ void settle(const void *base, Raw<T> &r, uint4 next, int lane) {
    constexpr int kWords = 2 * (int)sizeof(T);
    if (skew(base)) {
        unsigned x[kWords + 4];
#pragma unroll
        for (int i = 0; i < kWords; ++i) x[i] = r.w[i];
        x[kWords] = __shfl_sync(0xffffffffu, lane ? x[0] : next.x, lane + 1);
        x[kWords + 1] = __shfl_sync(0xffffffffu, lane ? x[1] : next.y, lane + 1);
        x[kWords + 2] = __shfl_sync(0xffffffffu, lane ? x[2] : next.z, lane + 1);
        x[kWords + 3] = __shfl_sync(0xffffffffu, lane ? x[3] : next.w, lane + 1);
        move_down<kWords>(x, skew(base));
#pragma unroll
        for (int i = 0; i < kWords; ++i) r.w[i] = x[i];
    }
}

template <typename T, int kAccess>
__device__ __forceinline__ void store_raw(void *base, long long first, long long n, int lane, const Raw<T> &r) {
    T *p = static_cast<T *>(base);
    using U = typename Bits<T>::type;
    constexpr int kWords = 2 * (int)sizeof(T), kPer = 4 / (int)sizeof(T), kShift = 8 * (int)sizeof(T);
    if constexpr (kAccess == kAnyAlignment) {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const long long e = first + lane_element<kAccess>(lane, i * kPer + j);
                if (e >= 0 && e < n) __stcs(reinterpret_cast<U *>(p) + e, (U)(r.w[i] >> (kShift * j)));
            }
    } else if constexpr (kWords == 2) {
        __stcs(reinterpret_cast<uint2 *>(p + first + 8 * lane), make_uint2(r.w[0], r.w[1]));
    } else {
        const unsigned off = kAccess == kSkewed ? skew(p) : 0u;
        uint4 *q = reinterpret_cast<uint4 *>(reinterpret_cast<char *>(p + first + 8 * lane) - off);
        if (off == 0) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) __stcs(q + i, make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]));
        } else {
            unsigned x[kWords + 4];                           // the lane before's last 16 bytes (lane 0: lane 31's), then this one's
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = __shfl_sync(0xffffffffu, r.w[kWords - 4 + j], lane + 31);
#pragma unroll
            for (int j = 0; j < kWords; ++j) x[4 + j] = r.w[j];
            move_down<kWords>(x, 16u - off);
            if (lane) __stcs(q, make_uint4(x[0], x[1], x[2], x[3]));
            if constexpr (kWords == 8) __stcs(q + 1, make_uint4(x[4], x[5], x[6], x[7]));
            if (lane == 0) {                                  // first bytes: the unit's last piece; the others: its first
                U *head = reinterpret_cast<U *>(q), *tail = reinterpret_cast<U *>(q + kStateBlock * sizeof(T) / 16);
                const int split = (int)(off / sizeof(T));
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < kPer; ++j) (i * kPer + j < split ? tail : head)[i * kPer + j] = (U)(x[i] >> (kShift * j));
            }
        }
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
// Square roots: an approximate root s = v y, y ~ 1/sqrt(v), corrected by its residual, s + (v - s s) y / 2 (Markstein, IBM J. Res.
// Dev. 34, 1990).  The residual's last bits are 2^-46 of v: down to 2^-102 it is exact and the roots are correctly rounded.  Smaller
// numbers come out near enough as long as they are normal, and below 2^-126, where y stays at 2^63, as something above 0 (0 as 0)
// that is below 2^-62, as their roots are.  Infinity gives NaN.
__device__ __forceinline__ float2 sqrt2(float2 v) {
    float2 y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(v.x, 0x1p-126f)));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(v.y, 0x1p-126f)));
    const float2 s = mul2(v, y), half = mul2(y, both(0.5f));
    const float2 rest = fma2(make_float2(-s.x, -s.y), s, v);
    return fma2(rest, half, s);
}
// Correctly rounded for every v: small ones are multiplied by 2^64 (exactly) and their roots by 2^-32.
__device__ __forceinline__ float2 sqrt2_any(float2 v) {
    const bool a = v.x < 0x1p-100f, b = v.y < 0x1p-100f;
    const float2 s = sqrt2(mul2(v, make_float2(a ? 0x1p64f : 1.f, b ? 0x1p64f : 1.f)));
    return mul2(s, make_float2(a ? 0x1p-32f : 1.f, b ? 0x1p-32f : 1.f));
}
// sqrt2 stands for it in two cases, which is nearly always (300M bf16: 565 us with sqrt2_any everywhere, 534 so, 531 with sqrt2
// alone; a branch on the smallest of a lane's second moments 573 to 595).  For the parameters' update, where eps is large enough
// (kExactRoots is false): it divides by root * inv_sqrt_bc2 + eps, in which roots below 2^-62 do not show.
__host__ __forceinline__ bool sqrt2_is_enough(float eps, float inv_sqrt_bc2) { return eps >= 0x1p-36f * inv_sqrt_bc2; }
// For the states, where a block's largest root is at least this: what is below 2^-51 is below half of the smallest code's value then, and
// gets code 1 whatever it is.  The other blocks' states are done once more.
constexpr float kTopRoot = 0x1p-32f;
__device__ __forceinline__ float reciprocal(float x) {                            // 1 ulp; infinity below 2^-126
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_abs(float a, float b) {                      // NaN if either is
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(fabsf(b)));
    return d;
}
__device__ __forceinline__ float2 first_moment(float2 g, float2 old, const AdamArgs &a, float b1) {
    const float2 m0 = mul2(old, both(b1)), m1 = mul2(g, both(a.one_minus_b1));
    return make_float2(__fadd_rn(m0.x, m1.x), __fadd_rn(m0.y, m1.y));
}
__device__ __forceinline__ float2 second_moment(float2 g, float2 root, const AdamArgs &a) {
    const float2 v0 = mul2(mul2(root, root), both(a.b2)), v1 = mul2(mul2(g, g), both(a.one_minus_b2));
    return make_float2(__fadd_rn(v0.x, v1.x), __fadd_rn(v0.y, v1.y));
}
// A block's largest magnitude from its lanes' (fp32 bits order as magnitudes do; NaN is above infinity)
__device__ __forceinline__ unsigned block_top(float top) { return __reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu); }
__device__ __forceinline__ float scale_of(unsigned top) {
    const float scale = __fmul_rn(__uint_as_float(top), 1.0f / 448.0f);
    return scale < 0x1p-126f ? 0.f : scale;
}
__device__ __forceinline__ float one_over(float scale) { return scale == 0.f ? 0.f : __fdiv_rn(1.f, scale); }
__device__ __forceinline__ Raw<code8> moment_codes(const float2 (&m)[4], float over) {
    Raw<code8> c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned two = e4m3_nearest(mul2(m[i], both(over)));
        if (i & 1) c.w[i >> 1] |= two << 16;
        else c.w[i >> 1] = two;
    }
    return c;
}
// Codes of a lane's roots; e: the unit's first element.
template <int kAccess>
__device__ __forceinline__ Raw<code8> root_codes(const float2 (&r)[4], float over, long long e, int lane, unsigned seed_term) {
    unsigned top[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = mul2(r[i], both(over)), z = mul2(y, both(0x1p-120f));
        const unsigned pair = (unsigned)(e + lane_element<kAccess>(lane, 2 * i)) >> 1;
        if (kAccess != kAnyAlignment) {
            const unsigned h = pair_hash(pair, seed_term);
            top[2 * i] = e4m3_random_top(y.x, z.x, __byte_perm(h, 0, 0x4104));              // low half at bit 8
            top[2 * i + 1] = e4m3_random_top(y.y, z.y, __byte_perm(h, 0, 0x4324));          // high half at bit 8
        } else {                                                                            // 32 elements apart, both of the lane's parity
            const unsigned h0 = pair_hash(pair, seed_term), h1 = pair_hash(pair + 16, seed_term), pick = (lane & 1) ? 0x4324 : 0x4104;
            top[2 * i] = e4m3_random_top(y.x, z.x, __byte_perm(h0, 0, pick));
            top[2 * i + 1] = e4m3_random_top(y.y, z.y, __byte_perm(h1, 0, pick));
        }
    }
    Raw<code8> c;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        c.w[i] = __byte_perm(__byte_perm(top[4 * i], top[4 * i + 1], 0x0073), __byte_perm(top[4 * i + 2], top[4 * i + 3], 0x0073), 0x5410);
    return c;
}
// New states of block blk, of which the parameters have had their step, with roots by sqrt2_any.  Seldom called: not in line, so that
// the registers of the caller are its own.
template <typename TG>
__device__ __noinline__ void step_states8(const TensorEntry &t, int blk, int lane, const AdamArgs &a, float b1, float gs, unsigned seed_term) {
    const long long first = (long long)blk * kStateBlock;
    const Raw<TG> grad = load_raw<TG, kAnyAlignment>(t.grad, first, t.n, lane);
    Raw<code8> mc = load_raw<code8, kAnyAlignment>(t.m, first, t.n, lane);
    const Raw<code8> rc = load_raw<code8, kAnyAlignment>(t.v, first, t.n, lane);
    const float ms = __ldcg(t.m_scale + blk), rs = __ldcg(t.v_scale + blk);
    float2 m[4], r[4];
    float mtop = 0.f, rtop = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 g = mul2(pair_of(grad, i), both(gs));
        m[i] = first_moment(g, mul2(e4m3_values(mc, i), both(ms)), a, b1);
        r[i] = sqrt2_any(second_moment(g, mul2(e4m3_values(rc, i), both(rs)), a));
        mtop = max_abs(max_abs(mtop, m[i].x), m[i].y);
        rtop = max_abs(max_abs(rtop, r[i].x), r[i].y);
    }
    const float mscale = scale_of(block_top(mtop)), rscale = scale_of(block_top(rtop));
    if (lane == 0) { t.m_scale[blk] = mscale; t.v_scale[blk] = rscale; }
    store_raw<code8, kAnyAlignment>(t.m, first, t.n, lane, moment_codes(m, one_over(mscale)));
    store_raw<code8, kAnyAlignment>(t.v, first, t.n, lane, root_codes<kAnyAlignment>(r, one_over(rscale), first, lane, seed_term));
}
template <typename TP, typename TG>
struct Unit8 {
    Raw<TP> p;
    Raw<TG> g;
    Raw<code8> m, r;
    float ms, rs;
};

// kUnits consecutive units of one tensor, so that constants, addresses and the division behind a unit's two scales
// are shared: lane i works out the i-th scale of the 2 kUnits.
template <typename TP, typename TG, int kAccess, int kUnits, bool kExactRoots>
__device__ __forceinline__ void step_units8(const TensorEntry &t, int blk, int lane, const AdamArgs &a, float b1, float gs, unsigned seed_term) {
    const long long first = (long long)blk * kStateBlock;
    Unit8<TP, TG> us[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const long long e = first + k * kStateBlock;
        us[k].p = load_raw<TP, kAccess>(t.param, e, t.n, lane);
        us[k].g = load_raw<TG, kAccess>(t.grad, e, t.n, lane);
        us[k].m = load_raw<code8, kAccess>(t.m, e, t.n, lane);
        us[k].r = load_raw<code8, kAccess>(t.v, e, t.n, lane);
        us[k].ms = __ldcg(t.m_scale + blk + k);
        us[k].rs = __ldcg(t.v_scale + blk + k);
    }
    uint4 pend, gend;
    if constexpr (kAccess == kSkewed) {
        pend = load_end<TP>(t.param, first + kUnits * kStateBlock, lane);
        gend = load_end<TG>(t.grad, first + kUnits * kStateBlock, lane);
    }
    float2 m[kUnits][4], r[kUnits][4];
    unsigned top_of = 0;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        Unit8<TP, TG> &u = us[k];
        if constexpr (kAccess == kSkewed) {
            constexpr int kLast = kUnits - 1;
            settle<TP>(t.param, u.p, k < kLast ? first_piece(us[k < kLast ? k + 1 : k].p) : pend, lane);
            settle<TG>(t.grad, u.g, k < kLast ? first_piece(us[k < kLast ? k + 1 : k].g) : gend, lane);
        }
        float mtop = 0.f, rtop = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 g = mul2(pair_of(u.g, i), both(gs));
            const float2 old = mul2(e4m3_values(u.m, i), both(u.ms)), root = mul2(e4m3_values(u.r, i), both(u.rs));
            const float2 v = second_moment(g, root, a);
            m[k][i] = first_moment(g, old, a, b1);
            r[k][i] = kExactRoots ? sqrt2_any(v) : sqrt2(v);
            mtop = max_abs(max_abs(mtop, m[k][i].x), m[k][i].y);
            rtop = max_abs(max_abs(rtop, r[k][i].x), r[k][i].y);
            // the update itself, in 2 ulp: it is small against the parameter that it is added to
            const float2 den = fma2(r[k][i], both(a.inv_sqrt_bc2), both(a.eps));
            const float2 step = mul2(m[k][i], make_float2(reciprocal(den.x), reciprocal(den.y)));
            set_pair(u.p, i, fma2(both(-a.step_size), step, mul2(pair_of(u.p, i), both(t.decay))));
        }
        store_raw<TP, kAccess>(t.param, first + k * kStateBlock, t.n, lane, u.p);
        const unsigned mt = block_top(mtop), rt = block_top(rtop);
        if (lane == 2 * k) top_of = mt;
        if (lane == 2 * k + 1) top_of = rt;
    }
    if constexpr (!kExactRoots) {
        if (__any_sync(0xffffffffu, (lane & 1) && lane < 2 * kUnits && top_of != 0 && top_of < __float_as_uint(kTopRoot))) {
            for (int k = 0; k < kUnits; ++k) step_states8<TG>(t, blk + k, lane, a, b1, gs, seed_term);
            return;
        }
    }
    const float scale = scale_of(top_of), over = one_over(scale);
    if (lane < 2 * kUnits) ((lane & 1) ? t.v_scale : t.m_scale)[blk + (lane >> 1)] = scale;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const long long e = first + k * kStateBlock;
        const float mover = __shfl_sync(0xffffffffu, over, 2 * k), rover = __shfl_sync(0xffffffffu, over, 2 * k + 1);
        store_raw<code8, kAccess>(t.m, e, t.n, lane, moment_codes(m[k], mover));
        store_raw<code8, kAccess>(t.v, e, t.n, lane, root_codes<kAccess>(r[k], rover, e, lane, seed_term));
    }
}

// ---------------------------------------------------------------- fp32 states
// Units need not begin where the tensor does: with `lead` elements before its start they lie on multiples of their own size
// (else of 16 bytes) in all four arrays wherever the arrays' offsets allow it (tensors at the same places of packed rows: 86.6M
// elements in 152 tensors 365 us; on multiples of 16 bytes 390, in accesses of any alignment 420).

template <typename TP, typename TG, int kAccess>
__device__ __forceinline__ void step_unit32(const TensorEntry &t, long long first, int lane, const AdamArgs &a, float gs) {
    AdamArgs mine = a;
    mine.decay = t.decay;
    Raw<TP> p = load_raw<TP, kAccess>(t.param, first, t.n, lane);
    Raw<TG> g = load_raw<TG, kAccess>(t.grad, first, t.n, lane);
    Raw<float> m = load_raw<float, kAccess>(t.m, first, t.n, lane), v = load_raw<float, kAccess>(t.v, first, t.n, lane);
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
    store_raw<TP, kAccess>(t.param, first, t.n, lane, p);
    store_raw<float, kAccess>(t.m, first, t.n, lane, m);
    store_raw<float, kAccess>(t.v, first, t.n, lane, v);
}

// ---------------------------------------------------------------- the kernel

// The last tensor whose first unit (or group) is not past u, at or after tensor k: a few steps, or else bisection (few large
// tensors lie between a warp's units, or many small ones).
template <bool kGroups>
__device__ __forceinline__ int first_of(const TensorEntry &t) { return kGroups ? t.first_group : t.first_unit; }
template <bool kGroups, int kEntries>
__device__ __forceinline__ int find_tensor(const TensorTable<kEntries> &tab, int u, int k) {
    for (int i = 0; i < 4; ++i, ++k)
        if (k + 1 >= tab.n || first_of<kGroups>(tab.e[k + 1]) > u) return k;
    int hi = tab.n;
    while (hi - k > 1) {
        const int mid = (k + hi) >> 1;
        if (first_of<kGroups>(tab.e[mid]) <= u) k = mid; else hi = mid;
    }
    return k;
}
__host__ __device__ __forceinline__ bool codes_on_8(const TensorEntry &t) {
    return ((reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v)) & 7u) == 0;
}

template <typename TP, typename TG, int kBits, bool kExactRoots, int kEntries>
__global__ void __launch_bounds__(kTensorThreads, TensorShape<TP, TG, kBits>::kBlocks)
adamw_tensors_kernel(const __grid_constant__ TensorTable<kEntries> tab) {
    const float gs = tab.grad_scale ? __ldg(tab.grad_scale) : 1.f;
    if (!isfinite(gs)) return;                              // a step whose gradients overflowed is skipped whole
    const int lane = threadIdx.x & 31;
    const int step = gridDim.x * kTensorWarps, warp = blockIdx.x * kTensorWarps + (threadIdx.x >> 5);
    int u = warp;
    for (int k = 0; u < tab.units; u += step) {
        k = find_tensor<false>(tab, u, k);
        const TensorEntry &t = tab.e[k];
        if constexpr (kBits == 32) {
            const long long e = (long long)(u - t.first_unit) * kStateBlock - max(t.lead, 0);
            if (t.lead >= 0 && e >= 0 && e + kStateBlock <= t.n) step_unit32<TP, TG, kAligned>(t, e, lane, tab.args, gs);
            else step_unit32<TP, TG, kAnyAlignment>(t, e, lane, tab.args, gs);
        } else {
            const int grouped = ((k + 1 < tab.n ? tab.e[k + 1].first_group : tab.groups) - t.first_group) * kGroup;
            const int blk = grouped + u - t.first_unit;
            if (codes_on_8(t) && (long long)(blk + 1) * kStateBlock <= t.n)
                step_units8<TP, TG, kSkewed, 1, kExactRoots>(t, blk, lane, tab.args, tab.b1, gs, tab.seed_term);
            else
                step_units8<TP, TG, kAnyAlignment, 1, kExactRoots>(t, blk, lane, tab.args, tab.b1, gs, tab.seed_term);
        }
    }
    if constexpr (kBits == 8) {
        // Groups go on from the warp after the last unit's.  Groups hold whole units of one tensor only: taken across the tensors' ends,
        // a unit at a time there, the warps that met an end finished late (25.7M bf16 in 150 tensors 65 us, now 54; 4.4M in 116 27, 16).
        u -= tab.units;
        for (int k = 0; u < tab.groups; u += step) {
            k = find_tensor<true>(tab, u, k);
            const TensorEntry &t = tab.e[k];
            const int blk = (u - t.first_group) * kGroup;
            if (skew(t.param) | skew(t.grad)) step_units8<TP, TG, kSkewed, kGroup, kExactRoots>(t, blk, lane, tab.args, tab.b1, gs, tab.seed_term);
            else step_units8<TP, TG, kAligned, kGroup, kExactRoots>(t, blk, lane, tab.args, tab.b1, gs, tab.seed_term);
        }
    }
}

}  // namespace
