// Clipped policy loss with a KL term from logits: loss, log-probabilities and the logits' gradient.
#pragma once
#include "local_common.cuh"

namespace {

// One row of logits x[V] (bf16 or fp32), target y, z = x / temperature:
//   lse = log sum_v exp z_v;  lp = z_y - lse;  q = exp(lp - old)
//   L   = -min(q A, clip(q, lo, hi) A) + kl_coef (exp(ref - lp) - (ref - lp) - 1)
//   s   = dL/dlp = -[not clipped] q A + kl_coef (1 - exp(ref - lp))
//   dx_v = w s / temperature ([v = y] - exp(z_v - lse))
// The gradient needs the row's statistics and the row again.  A cluster of 1 to 8 blocks keeps the
// row in its shared memory between the two, so that the row is read once and its gradient written
// once: the pass is bound by those bytes.  Each block copies its slice in with bulk asynchronous
// copies (up to kPolicyChunks, each with its own mbarrier, so that the first is used while the last is
// under way), forms a running maximum and sum per thread, and the blocks exchange one pair of numbers.
// Exponentials are base 2: e_v = 2^((x_v - max) log2e / temperature), with the difference formed first
// so that rows of the type's lowest value, and -inf entries, need no special case.

constexpr int kPolicyThreads = 256;
constexpr int kPolicyChunks = 4;
constexpr int kPolicyMaxCluster = 8;

struct PolicyHeader {           // first bytes of the workspace; all zero before the first call
    int status;                 // dppf_status of the last call
    unsigned done;              // rows finished in this call; back at 0 when the call ends
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
    int chunk;                  // ... and that a bulk copy brings
    int spin;
    float clip_lo, clip_hi, kl_coef, log2e_t, inv_t;
};

template <typename T> struct Vec16;      // the elements of a 16-byte vector, in pairs
template <> struct Vec16<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(uint4 u, float2 *x) {
        x[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
        x[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
    }
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

// Running maximum m and sum s = sum 2^((x - m) k) of a thread, over G vectors at once.
template <typename T, int G>
__device__ __forceinline__ void take(const uint4 *v, float k, float &m, float &s) {
    constexpr int kPairs = Vec16<T>::N / 2 * G;
    float2 x[kPairs];
#pragma unroll
    for (int i = 0; i < G; ++i) Vec16<T>::get(v[i * kPolicyThreads], x + i * (Vec16<T>::N / 2));
    float top = m;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) top = fmaxf(fmaxf(top, x[i].x), x[i].y);
    s *= exp2_fast((m - top) * k);
    m = top;
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const float2 t = mul2(add2(x[i], both(-top)), both(k));
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

// Fixed-order sum of the rows' terms by the last block to finish.
__device__ __forceinline__ void policy_finish(const PolicyArgs &a, double *s_red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int k = 0; k < 3; ++k) {
        const float *t = a.terms + (size_t)k * a.T;
        double sum = 0.0;
#pragma unroll 4
        for (int i = threadIdx.x; i < a.T; i += kPolicyThreads) sum += (double)__ldcg(t + i);
        sum = warp_sum(sum);
        if (lane == 0) s_red[warp] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            double all = 0.0;
            for (int w = 0; w < kPolicyThreads / 32; ++w) all += s_red[w];
            a.sums[k] = (float)all;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.hdr->status = __ldcg(&a.hdr->failed) ? DPPF_ERR_TIMEOUT : DPPF_OK;
        a.hdr->failed = 0;
    }
}

template <typename T>
__global__ void __launch_bounds__(kPolicyThreads) policy_kernel(const PolicyArgs a) {
    constexpr int N = Vec16<T>::N, kTake = 4;
    extern __shared__ __align__(128) uint4 s_row[];              // this block's slice, as aligned in the row
    __shared__ unsigned long long s_bar[kPolicyChunks];
    __shared__ float2 s_stats[kPolicyMaxCluster];                // one entry from each block of the cluster
    __shared__ float2 s_warp[kPolicyThreads / 32];
    __shared__ double s_red[kPolicyThreads / 32];
    __shared__ int s_failed, s_last;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = (int)cluster_size(), rank = (int)cluster_rank();
    const int row = blockIdx.x / C;
    const T *x = static_cast<const T *>(a.logits) + (long long)row * a.ld;
    T *g = static_cast<T *>(a.grad) + (long long)row * a.ld_grad;

    if (tid == 0) {
        for (int c = 0; c < kPolicyChunks; ++c) mbar_init(&s_bar[c], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_failed = 0;
        s_last = 0;
    }
    const float w = __ldg(a.weight + row);
    const long long y = a.targets64 ? __ldg(static_cast<const long long *>(a.targets) + row)
                                    : (long long)__ldg(static_cast<const int *>(a.targets) + row);
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

    auto count_row = [&](float lp, float loss, float kl, float part) {   // by one thread of the cluster
        a.logp[row] = lp;
        a.terms[row] = loss;
        a.terms[(size_t)a.T + row] = kl;
        a.terms[2 * (size_t)a.T + row] = part;
        __threadfence();
        s_last = atomicInc(&a.hdr->done, (unsigned)a.T - 1u) == (unsigned)a.T - 1u;
        __threadfence();
    };

    if (live) {
        __syncthreads();                                          // barriers initialised
        const int per = a.chunk;
        if (tid == 0) {
            const unsigned char *src = reinterpret_cast<const unsigned char *>(x - before) + (size_t)v0 * 16;
            for (int c = 0; c * per < nv; ++c) {
                const unsigned bytes = (unsigned)(min(per, nv - c * per) * 16);
                mbar_expect_tx(&s_bar[c], bytes);
                bulk_load(s_row + c * per, src + (size_t)c * per * 16, bytes, &s_bar[c]);
            }
        }
        if (C > 1) cluster_arrive_relaxed();                      // this block's s_stats may be written
        const float xy = to_float(x[y]);                          // before any block writes (grad may be logits)
        const float old = __ldg(a.old_logp + row), A = __ldg(a.advantage + row);
        const float ref = a.ref_logp ? __ldg(a.ref_logp + row) : 0.f;

        float m = -FLT_MAX, s = 0.f;
        const float k = a.log2e_t;
        int bad = 0;
        for (int c = 0; c * per < nv; ++c) {
            if (!mbar_wait_bounded(&s_bar[c], 0, a.spin)) { bad = 1; break; }
            const int stop = min(hi, (c + 1) * per);
            int i = max(lo, c * per) + tid;
            for (; i + (kTake - 1) * kPolicyThreads < stop; i += kTake * kPolicyThreads) take<T, kTake>(s_row + i, k, m, s);
            for (; i < stop; i += kPolicyThreads) take<T, 1>(s_row + i, k, m, s);
        }
        if (!bad) {                                               // the row's ends, element by element
            const int head = min(lo * N + v0 * N - before, e_last), tail = max(hi * N + v0 * N - before, head);
            int e = -1;
            if (tid < head - e_first) e = e_first + tid;
            else if (tid >= 32 && tid - 32 < e_last - tail) e = tail + tid - 32;
            if (e >= 0) merge(m, s, to_float(sx[e]), 1.f, k);
        } else {                                                  // the row becomes NaN; seen by the last block
            s = __int_as_float(0x7fc00000);
            s_failed = 1;
            atomicExch(&a.hdr->failed, 1);
            __threadfence();
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            merge(m, s, __shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o), k);
        if (lane == 0) s_warp[warp] = make_float2(m, s);
        __syncthreads();
        m = s_warp[0].x; s = s_warp[0].y;
#pragma unroll
        for (int i = 1; i < kPolicyThreads / 32; ++i) merge(m, s, s_warp[i].x, s_warp[i].y, k);
        if (C > 1) {
            cluster_wait();                                       // the other blocks have started
            if (tid < C) cluster_store2(cluster_map(&s_stats[rank], tid), m, s);
            if (warp == 0) cluster_arrive();
            else cluster_arrive_relaxed();
            cluster_wait();
            m = s_stats[0].x; s = s_stats[0].y;
            for (int i = 1; i < C; ++i) merge(m, s, s_stats[i].x, s_stats[i].y, k);
        }

        const float lp = (xy - m) * a.inv_t - logf(s);
        const float q = expf(lp - old);
        const bool clipped = (A > 0.f && q > a.clip_hi) || (A < 0.f && q < a.clip_lo);
        const float qc = fminf(fmaxf(q, a.clip_lo), a.clip_hi);
        float loss = 0.f, slope = 0.f, kl = 0.f;
        if (A != 0.f) {
            loss = clipped ? -qc * A : -q * A;
            slope = clipped ? 0.f : -q * A;
        }
        if (a.ref_logp) {
            const float gap = ref - lp, eg = expm1f(gap);
            kl = eg - gap;
            loss += a.kl_coef * kl;
            slope -= a.kl_coef * eg;
        }
        // before the gradient's stores, which a fence would wait for
        if (rank == 0 && tid == 0) count_row(lp, w * loss, w * kl, clipped ? w : 0.f);

        if (a.grad) {
            const float c = w * slope * a.inv_t, cn = -c / s;
            auto entry = [&](int e) {
                const float f = exp2_fast((to_float(sx[e]) - m) * k) * cn;
                g[e] = from_float<T>(e == y ? f + c : f);
            };
            if (same) {
                uint4 *out = reinterpret_cast<uint4 *>(gv);
#pragma unroll 4
                for (int i = lo + tid; i < hi; i += kPolicyThreads) __stcs(out + i, slope_vector<T>(s_row[i], k, m, cn));
                const int head = min(lo * N + v0 * N - before, e_last), tail = max(hi * N + v0 * N - before, head);
                if (tid < head - e_first) entry(e_first + tid);
                else if (tid >= 32 && tid - 32 < e_last - tail) entry(tail + tid - 32);
                const int at = (int)y + before - v0 * N;          // the target's place in the slice: written over by the
                if (at >= lo * N && at < hi * N && (at / N - lo) % kPolicyThreads == tid) entry((int)y);   // thread that wrote its vector
            } else {
                for (int e = e_first + tid; e < e_last; e += kPolicyThreads) entry(e);
            }
        }
        if (s_failed && tid == 0)                                 // copies still under way land before the block leaves
            for (int c = 0; c * per < nv; ++c) mbar_wait_bounded(&s_bar[c], 0, kSpinLimit);
    } else {
        __syncthreads();                                          // s_last is initialised
        if (rank == 0 && tid == 0) count_row(0.f, 0.f, 0.f, 0.f);
        if (a.grad) {
            const T zero = from_float<T>(0.f);
            if (same) {
                uint4 *out = reinterpret_cast<uint4 *>(gv);
                for (int i = lo + tid; i < hi; i += kPolicyThreads) __stcs(out + i, make_uint4(0, 0, 0, 0));
                const int head = min(lo * N + v0 * N - before, e_last), tail = max(hi * N + v0 * N - before, head);
                if (tid < head - e_first) g[e_first + tid] = zero;
                else if (tid >= 32 && tid - 32 < e_last - tail) g[tail + tid - 32] = zero;
            } else {
                for (int e = e_first + tid; e < e_last; e += kPolicyThreads) g[e] = zero;
            }
        }
    }

    if (rank != 0) return;
    __syncthreads();
    if (s_last) policy_finish(a, s_red);
}

}  // namespace
