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
constexpr int kPolicyChunks = 8;
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
    int spin;
    float clip_lo, clip_hi, kl_coef, log2e_t, inv_t;
};

template <typename T> struct Vec16;      // the elements of a 16-byte vector
template <> struct Vec16<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(uint4 u, float (&x)[4]) {
        x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
template <> struct Vec16<bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(uint4 u, float (&x)[8]) {
        x[0] = bf16_low(u.x); x[1] = bf16_high(u.x); x[2] = bf16_low(u.y); x[3] = bf16_high(u.y);
        x[4] = bf16_low(u.z); x[5] = bf16_high(u.z); x[6] = bf16_low(u.w); x[7] = bf16_high(u.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&x)[8]) {
        return make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    }
};

// (m, s) stands for s 2^(m k); the maxima start at -FLT_MAX, so differences never are inf - inf
// unless the row holds +inf or NaN.
__device__ __forceinline__ void merge(float &m, float &s, float m2, float s2, float k) {
    const float top = fmaxf(m, m2);
    s = s * exp2_fast((m - top) * k) + s2 * exp2_fast((m2 - top) * k);
    m = top;
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
    constexpr int N = Vec16<T>::N;
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
    }
    const float w = __ldg(a.weight + row);
    const long long y = a.targets64 ? __ldg(static_cast<const long long *>(a.targets) + row)
                                    : (long long)__ldg(static_cast<const int *>(a.targets) + row);
    const bool live = w != 0.f && y >= 0 && y < a.V;

    // Vectors of the row: 16-byte pieces of memory, the first and the last of which may reach over
    // the row's ends (into the same 16 bytes as one of its elements; those values are not used).
    const int before = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
    const int vectors = (before + a.V + N - 1) / N;
    const int v0 = rank * a.slice, v1 = min(v0 + a.slice, vectors), nv = max(v1 - v0, 0);
    const int e_first = max(v0 * N - before, 0), e_last = min(v1 * N - before, a.V);   // elements [e_first, e_last)
    const bool same = a.grad && ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(x)) & 15u) == 0;

    float term[3] = {0.f, 0.f, 0.f}, lp = 0.f;
    if (live) {
        __syncthreads();                                          // barriers initialised
        const int per = (a.slice + kPolicyChunks - 1) / kPolicyChunks;
        if (tid == 0) {
            const unsigned char *src = reinterpret_cast<const unsigned char *>(x - before) + (size_t)v0 * 16;
            for (int c = 0; c * per < nv; ++c) {
                const unsigned bytes = (unsigned)(min(per, nv - c * per) * 16);
                mbar_expect_tx(&s_bar[c], bytes);
                bulk_load(s_row + c * per, src + (size_t)c * per * 16, bytes, &s_bar[c]);
            }
        }
        if (C > 1) cluster_arrive();                              // this block's s_stats may be written
        const float xy = to_float(x[y]);                          // before any block writes (grad may be logits)
        const float old = __ldg(a.old_logp + row), A = __ldg(a.advantage + row);
        const float ref = a.ref_logp ? __ldg(a.ref_logp + row) : 0.f;

        float m = -FLT_MAX, s = 0.f;
        const float k = a.log2e_t;
        int bad = 0;
        for (int c = 0; c * per < nv; ++c) {
            if (!mbar_wait_bounded(&s_bar[c], 0, a.spin)) { bad = 1; break; }
            const int stop = min(nv, (c + 1) * per);
            for (int i = c * per + tid; i < stop; i += kPolicyThreads) {
                float f[N];
                Vec16<T>::get(s_row[i], f);
                const int e = (v0 + i) * N - before;
                if (e < 0 || e + N > a.V) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (e + j < 0 || e + j >= a.V) f[j] = __int_as_float(0xff800000);
                }
                float top = m;
#pragma unroll
                for (int j = 0; j < N; ++j) top = fmaxf(top, f[j]);
                s *= exp2_fast((m - top) * k);
                m = top;
#pragma unroll
                for (int j = 0; j < N; ++j) s += exp2_fast((f[j] - m) * k);
            }
        }
        if (bad) {                                                // the row becomes NaN; seen by the last block
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
        for (int i = 1; i < kPolicyThreads / 32; ++i) merge(m, s, s_warp[i].x, s_warp[i].y, k);
        if (C > 1) {
            cluster_wait();                                       // the other blocks have started
            if (tid < C) cluster_store2(cluster_map(&s_stats[rank], tid), m, s);
            cluster_arrive();
            cluster_wait();
            m = s_stats[0].x; s = s_stats[0].y;
            for (int i = 1; i < C; ++i) merge(m, s, s_stats[i].x, s_stats[i].y, k);
        }

        lp = (xy - m) * a.inv_t - logf(s);
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
        term[0] = w * loss;
        term[1] = w * kl;
        term[2] = clipped ? w : 0.f;

        if (a.grad) {
            const float c = w * slope * a.inv_t, cn = -c / s;
            const int yv = (int)((y + before) / N) - v0, yj = (int)((y + before) % N);   // the target's place in the slice
            if (same) {
                for (int i = tid; i < nv; i += kPolicyThreads) {
                    float f[N];
                    Vec16<T>::get(s_row[i], f);
#pragma unroll
                    for (int j = 0; j < N; ++j) f[j] = exp2_fast((f[j] - m) * k) * cn;
                    if (i == yv) {
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            if (j == yj) f[j] += c;
                    }
                    const int e = (v0 + i) * N - before;
                    if (e >= 0 && e + N <= a.V) {
                        __stcs(reinterpret_cast<uint4 *>(g + e), Vec16<T>::put(f));
                    } else {
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            if (e + j >= 0 && e + j < a.V) g[e + j] = from_float<T>(f[j]);
                    }
                }
            } else {
                const T *sx = reinterpret_cast<const T *>(s_row) + before - v0 * N;
                for (int e = e_first + tid; e < e_last; e += kPolicyThreads) {
                    float f = exp2_fast((to_float(sx[e]) - m) * k) * cn;
                    if (e == y) f += c;
                    g[e] = from_float<T>(f);
                }
            }
        }
        if (s_failed && tid == 0)                                 // copies still under way land before the block leaves
            for (int c = 0; c * per < nv; ++c) mbar_wait_bounded(&s_bar[c], 0, kSpinLimit);
    } else if (a.grad) {
        if (same) {
            for (int i = tid; i < nv; i += kPolicyThreads) {
                const int e = (v0 + i) * N - before;
                if (e >= 0 && e + N <= a.V) {
                    __stcs(reinterpret_cast<uint4 *>(g + e), make_uint4(0, 0, 0, 0));
                } else {
                    for (int j = 0; j < N; ++j)
                        if (e + j >= 0 && e + j < a.V) g[e + j] = from_float<T>(0.f);
                }
            }
        } else {
            for (int e = e_first + tid; e < e_last; e += kPolicyThreads) g[e] = from_float<T>(0.f);
        }
    }

    if (rank != 0) return;
    __syncthreads();
    if (tid == 0) {
        a.logp[row] = lp;
        for (int i = 0; i < 3; ++i) a.terms[(size_t)i * a.T + row] = term[i];
        __threadfence();
        s_last = atomicInc(&a.hdr->done, (unsigned)a.T - 1u) == (unsigned)a.T - 1u;
        __threadfence();
    }
    __syncthreads();
    if (s_last) policy_finish(a, s_red);
}

}  // namespace
