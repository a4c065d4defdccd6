// Clipped policy loss with a KL term from logits: loss, log-probabilities and the logits' gradient.
#pragma once
#include "local_common.cuh"

namespace {

// One row of logits x[V] (bf16 or fp32), target y, z = x / temperature:
//   lse = log sum_v exp z_v;  lp = z_y - lse;  q = exp(lp - old)
//   L   = -min(q A, clip(q, lo, hi) A) + kl_coef (exp(ref - lp) - (ref - lp) - 1)
//   s   = dL/dlp = -[not clipped] q A + kl_coef (1 - exp(ref - lp))
//   dx_v = w s / temperature ([v = y] - exp(z_v - lse))
// The gradient needs the row's statistics and the row again.  A cluster of 1 to 8 blocks keeps the row in its shared
// memory between the two, so that the row is read once and its gradient written once: the pass is bound by those bytes.
// Each block copies its slice in with bulk asynchronous copies (each with its own mbarrier, so that the first is
// used while the last is under way), forms a running maximum and sum per thread, and the warps of the cluster tell one
// another a pair of numbers, by asynchronous stores that the receiver counts (a cluster barrier instead, whose arrival
// is a fence behind all of a block's traffic, cost 33 us of 350 for 4,096 x 131,072 bf16, a quarter masked; now 319).  Without a
// gradient nothing is kept: the chunks go through a ring of buffers.
// Exponentials are base 2: e_v = 2^((x_v - max) log2e / temperature), with the difference formed first, so that rows of the
// type's lowest value, and -inf entries, need no special case.  The rows' terms are summed by a second launch, in a
// fixed order (a counter of finished rows cost each block another fence: 22 us for the same rows).

constexpr int kPolicyThreads = 128, kPolicyShortThreads = 64;   // ... for rows whose blocks would not fill an SM by their memory
constexpr int kPolicyChunks = 4;                 // buffers, and copies of a slice that is kept
constexpr int kPolicyRing = 512;                 // vectors of a buffer of the ring
constexpr int kPolicyMaxCluster = 8;

struct PolicyHeader {           // first bytes of the workspace; all zero before the first call
    int status;                 // dppf_status of the last call
    int failed;                 // a bounded wait gave up in this call; back at 0 when the call ends
};

struct PolicyArgs {
    const void *logits;
    void *grad;                 // null: no gradient
    long long ld, ld_grad;      // elements
    const void *targets;
    const float *old_logp, *ref_logp, *advantage, *weight;   // ref_logp may be null
    float *logp, *sums;         // [T], [3] (loss, KL, clipped)
    float *terms;               // workspace [3][T]
    PolicyHeader *hdr;
    int T, V;
    int targets64;
    int slice;                  // 16-byte vectors of a row that each block of the cluster holds
    int chunk;                  // ... and that a bulk copy brings, into one of kPolicyChunks buffers (in turn, without a gradient)
    int spin;
    float clip_lo, clip_hi, kl_coef, inv_t;
    float log2e_t, log2e_t_rest;                             // log2(e) / temperature = their sum, both above zero: for the sums
    float log2e_t_near;                                      // ... to the nearest: for single exponentials
};

template <typename T> struct Vec16;      // the elements of a 16-byte vector, in pairs
template <> struct Vec16<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(uint4 u, float2 *x) {
        x[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
        x[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
    }
    static __device__ __forceinline__ uint4 nothing() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }   // -inf
    static __device__ __forceinline__ uint4 put(const float2 *x) {
        return make_uint4(__float_as_uint(x[0].x), __float_as_uint(x[0].y), __float_as_uint(x[1].x), __float_as_uint(x[1].y));
    }
};
template <> struct Vec16<bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(uint4 u, float2 *x) {
        x[0] = make_float2(bf16_low(u.x), bf16_high(u.x));
        x[1] = make_float2(bf16_low(u.y), bf16_high(u.y));
        x[2] = make_float2(bf16_low(u.z), bf16_high(u.z));
        x[3] = make_float2(bf16_low(u.w), bf16_high(u.w));
    }
    static __device__ __forceinline__ uint4 nothing() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    static __device__ __forceinline__ uint4 put(const float2 *x) {
        return make_uint4(bf16_pair(x[0].x, x[0].y), bf16_pair(x[1].x, x[1].y), bf16_pair(x[2].x, x[2].y), bf16_pair(x[3].x, x[3].y));
    }
};

// (m, s) stands for s 2^(m k); the maxima start at -FLT_MAX, so differences never are inf - inf
// unless the row holds +inf or NaN.
__device__ __forceinline__ void merge(float &m, float &s, float m2, float s2, float k) {
    const float top = fmaxf(m, m2);
    s = s * exp2_fast((m - top) * k) + s2 * exp2_fast((m2 - top) * k);
    m = top;
}

// (x - m) k for the sums: with the part of k below its fp32 value, since that error would be the same in all of a row's
// terms (as much as 1e-6 of a log-probability).  The rest is above zero, so that -inf stays -inf.
__device__ __forceinline__ float2 scaled2(float2 x, float m, float k, float rest) {
    const float2 d = add2(x, both(-m));
    return fma2(d, both(rest), mul2(d, both(k)));
}

// Running maximum m and sum s = sum 2^((x - m) k) of a thread, over G vectors at once.
template <typename T, int G, int kThreads>
__device__ __forceinline__ void take(const uint4 *v, float k, float rest, float &m, float &s) {
    constexpr int kPairs = Vec16<T>::N / 2 * G;
    float2 x[kPairs];
#pragma unroll
    for (int i = 0; i < G; ++i) Vec16<T>::get(v[i * kThreads], x + i * (Vec16<T>::N / 2));
    float top = m;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) top = fmaxf(fmaxf(top, x[i].x), x[i].y);
    s *= exp2_fast((m - top) * k);
    m = top;
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const float2 t = scaled2(x[i], top, k, rest);
        sum = add2(sum, make_float2(exp2_fast(t.x), exp2_fast(t.y)));
    }
    s += sum.x + sum.y;
}

// Gradient of one vector, without the target's own term: -c exp(z - lse), cn = -c / s.
template <typename T>
__device__ __forceinline__ uint4 slope_vector(uint4 v, float k, float m, float cn) {
    constexpr int kPairs = Vec16<T>::N / 2;
    float2 x[kPairs];
    Vec16<T>::get(v, x);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const float2 t = mul2(add2(x[i], both(-m)), both(k));
        x[i] = mul2(make_float2(exp2_fast(t.x), exp2_fast(t.y)), both(cn));
    }
    return Vec16<T>::put(x);
}

// Over the warp's pairs: one maximum, one exponential a lane, one sum.
__device__ __forceinline__ void warp_merge(float &m, float &s, float k) {
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    s *= exp2_fast((m - top) * k);
    m = top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
}

struct RowTerms { float lp, loss, kl, slope; bool clipped; };     // slope: dL/dlp

__device__ __forceinline__ RowTerms row_terms(const PolicyArgs &a, float lp, float old, float ref, float A) {
    RowTerms r;
    r.lp = lp;
    const float q = expf(lp - old);
    r.clipped = (A > 0.f && q > a.clip_hi) || (A < 0.f && q < a.clip_lo);
    r.loss = A == 0.f ? 0.f : r.clipped ? -fminf(fmaxf(q, a.clip_lo), a.clip_hi) * A : -q * A;
    r.slope = A == 0.f || r.clipped ? 0.f : -q * A;
    r.kl = 0.f;
    if (a.ref_logp) {
        const float gap = ref - lp, eg = expm1f(gap);
        r.kl = isinf(eg) ? eg : eg - gap;                         // (a gap of infinity is infinitely far, not NaN)
        if (a.kl_coef != 0.f) {                                   // watched only: no part in either, however large it is
            r.loss += a.kl_coef * r.kl;
            r.slope -= a.kl_coef * eg;
        }
    }
    return r;
}
__device__ __forceinline__ void put_terms(const PolicyArgs &a, int row, float lp, float loss, float kl, float part) {
    a.logp[row] = lp;
    a.terms[row] = loss;
    a.terms[(size_t)a.T + row] = kl;
    a.terms[2 * (size_t)a.T + row] = part;
}
__device__ __forceinline__ long long target_of(const PolicyArgs &a, int row) {
    return a.targets64 ? __ldg(static_cast<const long long *>(a.targets) + row) : (long long)__ldg(static_cast<const int *>(a.targets) + row);
}

// Fixed-order sums of the rows' terms: one block each for the loss, the KL term and the clipped weights.
constexpr int kFinishThreads = 1024;

__global__ void __launch_bounds__(kFinishThreads) policy_finish_kernel(const PolicyArgs a) {
    __shared__ double s_sum[kFinishThreads / 32];
    wait_for_previous();
    const float *t = a.terms + (size_t)blockIdx.x * a.T;
    double sum = 0.0;
#pragma unroll 16
    for (int i = threadIdx.x; i < a.T; i += kFinishThreads) sum += (double)__ldcg(t + i);
    sum = warp_sum(sum);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int w = 0; w < kFinishThreads / 32; ++w) all += s_sum[w];
        a.sums[blockIdx.x] = (float)all;
        if (blockIdx.x == 0) {
            a.hdr->status = __ldcg(&a.hdr->failed) ? DPPF_ERR_TIMEOUT : DPPF_OK;
            a.hdr->failed = 0;
        }
    }
}

template <typename T, int kThreads>
__global__ void __launch_bounds__(kThreads) policy_kernel(const PolicyArgs a) {
    constexpr int N = Vec16<T>::N, kTake = 4, kWarps = kThreads / 32;
    static_assert(kPolicyMaxCluster * kWarps <= 32, "a warp merges the pairs of all warps of a cluster");
    extern __shared__ __align__(128) uint4 s_row[];              // this block's slice, as aligned in the row, or the ring
    __shared__ unsigned long long s_bar[kPolicyChunks], s_told;  // s_told: the pairs of the cluster's warps
    __shared__ float2 s_stats[kPolicyMaxCluster * kWarps]; // one entry from each warp of the cluster
    __shared__ int s_failed;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = (int)cluster_size(), rank = (int)cluster_rank();
    const int row = blockIdx.x / C;
    const T *x = static_cast<const T *>(a.logits) + (long long)row * a.ld;
    T *g = static_cast<T *>(a.grad) + (long long)row * a.ld_grad;

    if (tid == 0) {
        for (int c = 0; c < kPolicyChunks; ++c) mbar_init(&s_bar[c], 1);
        mbar_init(&s_told, 1);
        if (C > 1) mbar_expect_tx(&s_told, (unsigned)(C * kWarps * sizeof(float2)));
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_failed = 0;
    }
    const float w = __ldg(a.weight + row);
    const long long y = target_of(a, row);
    const bool live = w != 0.f && y >= 0 && y < a.V;

    // Vectors of the row: 16-byte pieces of memory, the first and the last of which may reach over the row's ends
    // (into the same 16 bytes as one of its elements; those values are not used).  This block has vectors [v0, v0 + nv)
    // of it, elements [e_first, e_last); of its vectors [lo, hi) lie wholly inside the row.
    const int before = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
    const int vectors = (before + a.V + N - 1) / N;
    const int v0 = rank * a.slice, nv = max(min(a.slice, vectors - v0), 0);
    const int e_first = max(v0 * N - before, 0), e_last = min((v0 + nv) * N - before, a.V);
    const int lo = (rank == 0 && before) ? 1 : 0, hi = max(min(nv, (before + a.V) / N - v0), lo);
    T *gv = g - before + (long long)v0 * N;                       // where this block's vectors go, if they are aligned there
    const bool same = a.grad && ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(x)) & 15u) == 0;
    const T *sx = reinterpret_cast<const T *>(s_row) + before - v0 * N;   // element e of the row, for e in [e_first, e_last)

    if (live) {
        __syncthreads();                                          // barriers initialised
        const int per = a.chunk, chunks = (nv + per - 1) / per;    // chunk c is in buffer c % kPolicyChunks
        auto fetch = [&](int c) {
            const unsigned bytes = (unsigned)(min(per, nv - c * per) * 16);
            const unsigned char *src = reinterpret_cast<const unsigned char *>(x - before) + ((size_t)v0 + (size_t)c * per) * 16;
            mbar_expect_tx(&s_bar[c % kPolicyChunks], bytes);
            bulk_load(s_row + (c % kPolicyChunks) * per, src, bytes, &s_bar[c % kPolicyChunks]);
        };
        if (tid == 0)
            for (int c = 0; c < min(chunks, kPolicyChunks); ++c) fetch(c);
        if (C > 1) cluster_arrive_relaxed();                      // this block's s_stats may be written
        const float xy = to_float(x[y]);                          // before it is written over (grad may be logits): see below
        const float old = __ldg(a.old_logp + row), A = __ldg(a.advantage + row);
        const float ref = a.ref_logp ? __ldg(a.ref_logp + row) : 0.f;

        float m = -FLT_MAX, s = 0.f;
        const float k = a.log2e_t, rest = a.log2e_t_rest;
        const int head = min((lo + v0) * N - before, e_last), tail = max((hi + v0) * N - before, head);   // whole vectors: elements [head, tail)
        int landed = 0, issued = min(chunks, kPolicyChunks), bad = 0;   // chunks whose copies this thread has waited for, has started (thread 0)
        for (int c = 0; c < chunks && !bad; ++c) {
            if (!mbar_wait_bounded(&s_bar[c % kPolicyChunks], (c / kPolicyChunks) & 1, a.spin)) {
                bad = 1;
            } else {
                landed = c + 1;
                const uint4 *v = s_row + (c % kPolicyChunks) * per - (size_t)c * per;                     // v[i]: vector i of the slice
                const int stop = min(hi, (c + 1) * per);
                int i = max(lo, c * per) + tid;
                for (; i + (kTake - 1) * kThreads < stop; i += kTake * kThreads) take<T, kTake, kThreads>(v + i, k, rest, m, s);
                for (; i < stop; i += kThreads) take<T, 1, kThreads>(v + i, k, rest, m, s);
                // the row's ends, element by element
                const T *ve = reinterpret_cast<const T *>(v) + before - v0 * N;
                if (c == 0 && tid < head - e_first) merge(m, s, to_float(ve[e_first + tid]), 1.f, k);
                if (c == chunks - 1 && tid >= 32 && tid - 32 < e_last - tail) merge(m, s, to_float(ve[tail + tid - 32]), 1.f, k);
            }
            if (chunks > kPolicyChunks) {                         // the ring: the chunk's buffer is free
                bad = __syncthreads_or(bad);
                if (tid == 0 && !bad && c + kPolicyChunks < chunks) {
                    fetch(c + kPolicyChunks);
                    issued = c + kPolicyChunks + 1;
                }
            }
        }
        if (bad) {                                                // the row becomes NaN
            s = __int_as_float(0x7fc00000);
            s_failed = 1;
            a.hdr->failed = 1;
        }
        warp_merge(m, s, k);
        bool told = true;
        if (C > 1) {                                              // every warp's pair goes to every block of the cluster
            cluster_wait();                                       // the other blocks have started
            // The block that holds the target's logit may write over it once it has all pairs, so a pair must not leave before the
            // read of xy in its warp has come back.  The vote makes it wait: what is sent depends on every lane's xy (which,
            // if it is NaN, makes the row NaN in any case).
            if (__any_sync(0xffffffffu, isnan(xy))) s = __int_as_float(0x7fc00000);
            if (lane < C) cluster_send2(cluster_map(&s_stats[rank * kWarps + warp], lane), m, s, cluster_map(&s_told, lane));
            // a block stays until it has been told by all, so nobody writes to one that has left
            told = mbar_wait_bounded(&s_told, 0, kSpinLimit);
        } else {
            if (lane == 0) s_stats[warp] = make_float2(m, s);
            __syncthreads();
        }
        m = lane < C * kWarps ? s_stats[lane].x : -FLT_MAX;
        s = lane < C * kWarps ? s_stats[lane].y : 0.f;
        warp_merge(m, s, k);                                      // the same bits in every warp
        if (!told) {
            s = __int_as_float(0x7fc00000);
            a.hdr->failed = 1;
        }

        const RowTerms r = row_terms(a, (xy - m) * a.inv_t - logf(s), old, ref, A);
        if (rank == 0 && tid == 0) put_terms(a, row, r.lp, w * r.loss, w * r.kl, r.clipped ? w : 0.f);

        if (a.grad) {
            const float c = w * r.slope * a.inv_t, cn = -c / s, near = a.log2e_t_near;
            auto entry = [&](int e) {
                const float f = exp2_fast((to_float(sx[e]) - m) * near) * cn;
                g[e] = from_float<T>(e == y ? f + c : f);
            };
            if (same) {
                uint4 *out = reinterpret_cast<uint4 *>(gv);
#pragma unroll 4
                for (int i = lo + tid; i < hi; i += kThreads) __stcs(out + i, slope_vector<T>(s_row[i], near, m, cn));
                if (tid < head - e_first) entry(e_first + tid);
                else if (tid >= 32 && tid - 32 < e_last - tail) entry(tail + tid - 32);
                const int at = (int)y + before - v0 * N;          // the target's place in the slice: written over by the
                if (at >= lo * N && at < hi * N && (at / N - lo) % kThreads == tid) entry((int)y);   // thread that wrote its vector
            } else {
                for (int e = e_first + tid; e < e_last; e += kThreads) entry(e);
            }
        }
        if (s_failed && tid == 0)                                 // copies still under way land before the block leaves
            for (int c = landed; c < issued; ++c) mbar_wait_bounded(&s_bar[c % kPolicyChunks], (c / kPolicyChunks) & 1, kSpinLimit);
    } else {
        if (rank == 0 && tid == 0) put_terms(a, row, 0.f, 0.f, 0.f, 0.f);
        if (a.grad) {
            const T zero = from_float<T>(0.f);
            if (same) {
                uint4 *out = reinterpret_cast<uint4 *>(gv);
                for (int i = lo + tid; i < hi; i += kThreads) __stcs(out + i, make_uint4(0, 0, 0, 0));
                const int head = min((lo + v0) * N - before, e_last), tail = max((hi + v0) * N - before, head);
                if (tid < head - e_first) g[e_first + tid] = zero;
                else if (tid >= 32 && tid - 32 < e_last - tail) g[tail + tid - 32] = zero;
            } else {
                for (int e = e_first + tid; e < e_last; e += kThreads) g[e] = zero;
            }
        }
    }
    let_next_start();
}

// ---------------------------------------------------------------- short rows
// Rows of up to 32 kHold vectors: a warp holds a row in registers, kHold vectors a lane, and takes another one when it
// is done.  A block's start, its copies and its barriers would take longer than such a row.
constexpr int kShortThreads = 128;

template <typename T, int kHold>
__global__ void __launch_bounds__(kShortThreads, kHold == 8 ? 4 : 8) policy_short_kernel(const PolicyArgs a) {
    constexpr int N = Vec16<T>::N, kPairs = N / 2;
    const int lane = threadIdx.x & 31;
    const float k = a.log2e_t;
    const long long stride = (long long)gridDim.x * (kShortThreads / 32);
    long long row_l = (long long)blockIdx.x * (kShortThreads / 32) + (threadIdx.x >> 5);
    float w_next = row_l < a.T ? __ldg(a.weight + row_l) : 0.f;
    long long y_next = row_l < a.T ? target_of(a, (int)row_l) : -1;
    for (; row_l < a.T; row_l += stride) {
        const int row = (int)row_l;
        const float w = w_next;
        const long long y = y_next;
        if (row_l + stride < a.T) {                               // the next row's, ahead of this one's work
            w_next = __ldg(a.weight + row_l + stride);
            y_next = target_of(a, (int)(row_l + stride));
        }
        const T *x = static_cast<const T *>(a.logits) + (long long)row * a.ld;
        T *g = static_cast<T *>(a.grad) + (long long)row * a.ld_grad;
        const bool live = w != 0.f && y >= 0 && y < a.V;
        const int before = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T)), vectors = (before + a.V + N - 1) / N;
        const bool same = a.grad && ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(x)) & 15u) == 0;
        const uint4 *xv = reinterpret_cast<const uint4 *>(x - before);
        // vector i of the gradient; the ends of the row, and rows that are not aligned as the logits' are, element by element
        auto put = [&](int i, const float2 (&f)[kPairs]) {
            const int e = i * N - before;
            if (same && e >= 0 && e + N <= a.V) {
                __stcs(reinterpret_cast<uint4 *>(g + e), Vec16<T>::put(f));
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (e + j >= 0 && e + j < a.V) g[e + j] = from_float<T>((j & 1) ? f[j / 2].y : f[j / 2].x);
            }
        };
        if (!live) {
            if (lane == 0) put_terms(a, row, 0.f, 0.f, 0.f, 0.f);
            if (a.grad) {
                float2 zero[kPairs];
#pragma unroll
                for (int j = 0; j < kPairs; ++j) zero[j] = make_float2(0.f, 0.f);
                for (int i = lane; i < vectors; i += 32) put(i, zero);
            }
            continue;
        }
        uint4 v[kHold];
#pragma unroll
        for (int h = 0; h < kHold; ++h) {
            const int i = lane + 32 * h;
            v[h] = i < vectors ? __ldcs(xv + i) : make_uint4(0, 0, 0, 0);
        }
        const float xy = to_float(x[y]), old = __ldg(a.old_logp + row), A = __ldg(a.advantage + row), ref = a.ref_logp ? __ldg(a.ref_logp + row) : 0.f;
        // what is outside the row counts as -inf
        const uint4 none = Vec16<T>::nothing();
        float m = -FLT_MAX, s = 0.f;
#pragma unroll
        for (int h = 0; h < kHold; ++h) {
            const int i = lane + 32 * h, e = i * N - before;
            if (i >= vectors) {
                v[h] = none;
            } else if (e < 0 || e + N > a.V) {
                float2 f[kPairs];
                Vec16<T>::get(v[h], f);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (e + j < 0 || e + j >= a.V) ((j & 1) ? f[j / 2].y : f[j / 2].x) = __int_as_float(0xff800000);
                v[h] = Vec16<T>::put(f);
            }
            float2 f[kPairs];
            Vec16<T>::get(v[h], f);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) m = fmaxf(fmaxf(m, f[j].x), f[j].y);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
        for (int h = 0; h < kHold; ++h) {
            float2 f[kPairs], sum = make_float2(0.f, 0.f);
            Vec16<T>::get(v[h], f);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                const float2 t = scaled2(f[j], m, k, a.log2e_t_rest);
                sum = add2(sum, make_float2(exp2_fast(t.x), exp2_fast(t.y)));
            }
            s += sum.x + sum.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        const RowTerms r = row_terms(a, (xy - m) * a.inv_t - logf(s), old, ref, A);
        if (lane == 0) put_terms(a, row, r.lp, w * r.loss, w * r.kl, r.clipped ? w : 0.f);
        if (a.grad) {
            const float c = w * r.slope * a.inv_t, cn = -c / s, near = a.log2e_t_near;
            const int at = (int)y + before;
            __syncwarp();                                         // every lane has its xy before one writes over it (grad may be logits)
#pragma unroll
            for (int h = 0; h < kHold; ++h) {
                const int i = lane + 32 * h;
                if (i >= vectors) break;
                float2 f[kPairs];
                Vec16<T>::get(v[h], f);
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    const float2 t = mul2(add2(f[j], both(-m)), both(near));
                    f[j] = mul2(make_float2(exp2_fast(t.x), exp2_fast(t.y)), both(cn));
                }
                if (at / N == i) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (at % N == j) ((j & 1) ? f[j / 2].y : f[j / 2].x) += c;
                }
                put(i, f);
            }
        }
    }
    let_next_start();
}

}  // namespace
