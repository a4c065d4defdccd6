// Layer norm after a residual addition, and its gradient with the weight's and bias's.
//
//   h = x + branch (rounded to x's type);  mu = mean h;  r = (mean (h - mu)^2 + eps)^-1/2;  y = (h - mu) r w + b
//   u = w dy;  xh = (h - mu) r;  dx = r (u - mean u - xh mean(u xh)) + dsum;  dw = sum_t dy xh;  db = sum_t dy
//
// Both are bound by memory: a row is read once, stays in registers (sixteen elements a thread) for the statistics, the second
// moment taken about the mean, and is written once.  (Of a bf16 row alone 32 elements a thread, 64 bytes, as of an fp32 one: 8,192 x 8,192 86 -> 72 us,
// 40,000 x 768 37 -> 32; an fp32 row with 32, or a branch beside it, 123 -> 126.)  Rows of up to 512 elements take a warp or, shorter ones, a part of one (a power of two of
// lanes), longer ones a block; above
// kNormRow elements (kNormGradRow for the gradient) a block walks the row several times, the later ones from L2.
//
// The gradient's blocks stay: each walks rows blockIdx.x, + gridDim.x, ... and keeps its columns' sums of dy xh and dy in registers;
// they go to the workspace once a block, and a second launch adds the blocks' sums in block order.  No atomics: the sums' order
// depends on T and H alone.
//
// Measured on a B200 (copy rate 6.54 TB/s): 16,384 x 4,096, fp32 stream plus a bf16 branch to bf16, 123 us (6.55 TB/s); its gradient with the
// stream's, 164 us (5.7 TB/s): reads and writes mixed, half of the warps resident (64 registers).  bf16 rows without a stream are bound by
// latency: 8,192 x 8,192 72 us (3.7 TB/s), the gradient with the stream's 148.  Tried and lost: blocks that stay for several rows and read
// ahead (123 -> 130 us; 8,192 x 8,192 bf16 70), weights held in registers (gradient 167 -> 217), eight elements a thread forward (123 -> 131).
#pragma once
#include "local_common.cuh"

namespace {

constexpr int kNormElements = 16;                         // of a row in one thread
constexpr int kNormWarpRow = 32 * kNormElements;          // longest row of a warp
constexpr int kNormRow = 1024 * kNormElements;            // longest row that a block holds
constexpr int kNormGradElements = 8;                     // the gradient's, of rows of blocks: the columns' sums lie beside them
constexpr int kNormGradRow = 1024 * kNormGradElements;    // longest row that a block holds so
constexpr int kNormWarps = 8;                             // rows side by side in a block, a warp each
constexpr int kNormWideThreads = 512;
constexpr int kNormJoinThreads = 1024;

// Eight fp32 in one access of 32 bytes (as two of 16 a warp's accesses touch every 32-byte sector twice); else as everywhere.
template <typename T, int N, bool kOnce = true>
__device__ __forceinline__ void load_row(const T *p, float (&f)[N]) {
    if constexpr (N == 8 && sizeof(T) == 4) {
        if constexpr (kOnce)
            asm volatile("ld.global.cs.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]) : "l"(p) : "memory");
        else
            asm volatile("ld.global.cg.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]) : "l"(p) : "memory");
    } else {
        load_vec<T, N, kOnce>(p, f);
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_row(T *p, const float (&f)[N]) {
    if constexpr (N == 8 && sizeof(T) == 4)
        asm volatile("st.global.cs.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                     ::"f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]), "l"(p) : "memory");
    else
        store_vec<T, N>(p, f);
}

struct NormArgs {
    const void *x, *branch, *weight, *bias;
    void *sum, *out;
    float *mean, *rstd;
    long long ld_x, ld_branch, ld_sum, ld_out, T;
    int H, groups;               // groups: of N elements
    int lanes;                   // of a row within a warp
    int branch32, weight32;      // fp32 (else bf16)
    float eps;
};

struct NormGradArgs {
    const void *dy, *x, *weight, *dsum;
    const float *mean, *rstd;
    void *dx, *dweight, *dbias;
    float *part;                 // [blocks][2][H]
    long long ld_dy, ld_x, ld_dsum, ld_dx, T;
    int H, groups, lanes, blocks;
    int weight32, grad32, add;   // types of the weight and of its gradient; add to the gradients
    float inv_h;
};

// N elements of an array whose type is known at run time.
template <int N>
__device__ __forceinline__ void load_either(const void *p, int is32, long long at, float (&f)[N]) {
    if (is32) load_row<float, N>(static_cast<const float *>(p) + at, f);
    else load_row<bf16, N>(static_cast<const bf16 *>(p) + at, f);
}
// The same of a weight or bias, which every row reads again: through the first-level cache (from the second it was several times a
// bf16 row's own traffic: 40,000 x 768 38 us, 26 so).
template <int N>
__device__ __forceinline__ void load_weight(const void *p, int is32, int at, float (&f)[N]) {
    constexpr int kWords = N < 4 ? N : 4;
    if (is32) {
        const float *q = static_cast<const float *>(p) + at;
        using W = typename Words<kWords>::type;
#pragma unroll
        for (int i = 0; i < N / kWords; ++i) {
            const W w = __ldg(reinterpret_cast<const W *>(q) + i);
            memcpy(&f[i * kWords], &w, sizeof(W));
        }
    } else if constexpr (N == 1) {
        f[0] = to_float(__ldg(static_cast<const bf16 *>(p) + at));
    } else {
        using W = typename Words<N / 2>::type;
        const W w = __ldg(reinterpret_cast<const W *>(static_cast<const bf16 *>(p) + at));
        unsigned u[N / 2];
        memcpy(u, &w, sizeof(W));
#pragma unroll
        for (int i = 0; i < N / 2; ++i) { f[2 * i] = bf16_low(u[i]); f[2 * i + 1] = bf16_high(u[i]); }
    }
}

// Sums of K values over the threads of a row: `lanes` of a warp, or the block.  `s` is used by one call in two (the caller alternates), so
// that one barrier is enough.
template <bool kWarp, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*s)[32], int lanes = 32) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (!kWarp || o < lanes)
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if constexpr (!kWarp) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) s[k][warp] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = lane < warps ? s[k][lane] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
    }
}

template <typename TX, typename TO, int N, int E, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kNormWarps * 32 : E > kNormElements ? 512 : 1024) norm_kernel(const __grid_constant__ NormArgs a) {
    constexpr int G = E / N;
    __shared__ float s_sum[2][1][32];
    const int L = kWarp ? a.lanes : blockDim.x, t = kWarp ? threadIdx.x & (L - 1) : threadIdx.x;
    long long row = kWarp ? (long long)blockIdx.x * (kNormWarps * 32 / L) + threadIdx.x / L : blockIdx.x;
    const bool mine = row < a.T;
    if (!mine) row = a.T - 1;                                    // a warp's parts go on together: these write nothing
    const TX *x = static_cast<const TX *>(a.x) + row * a.ld_x;
    float h[G][N], sum[1] = {0.f};
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int at = g * L + t;
        if (at < a.groups) load_row<TX, N>(x + (long long)at * N, h[g]);
        else
#pragma unroll
            for (int i = 0; i < N; ++i) h[g][i] = 0.f;
    }
    if (a.branch && mine) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int at = g * L + t;
            if (at >= a.groups) continue;
            float b[N];
            load_either<N>(a.branch, a.branch32, row * a.ld_branch + (long long)at * N, b);
#pragma unroll
            for (int i = 0; i < N; ++i) h[g][i] = to_float(from_float<TX>(h[g][i] + b[i]));
            store_row<TX, N>(static_cast<TX *>(a.sum) + row * a.ld_sum + (long long)at * N, h[g]);
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[0] += h[g][i];
    row_sums<kWarp, 1>(sum, s_sum[0], L);
    const float mean = sum[0] / (float)a.H;
    sum[0] = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g)
        if (g * L + t < a.groups)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                h[g][i] -= mean;
                sum[0] = fmaf(h[g][i], h[g][i], sum[0]);
            }
    row_sums<kWarp, 1>(sum, s_sum[1], L);
    const float rstd = 1.0f / sqrtf(sum[0] / (float)a.H + a.eps);
    if (!mine) return;
    if (t == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int at = g * L + t;
        if (at >= a.groups) continue;
        float w[N], b[N];
        load_weight<N>(a.weight, a.weight32, at * N, w);
        if (a.bias) load_weight<N>(a.bias, a.weight32, at * N, b);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = h[g][i] * rstd;
            h[g][i] = a.bias ? fmaf(y, w[i], b[i]) : y * w[i];
        }
        store_row<TO, N>(static_cast<TO *>(a.out) + row * a.ld_out + (long long)at * N, h[g]);
    }
}

// Rows longer than a block holds: h is formed (and written) in the first walk and read again in two more.
template <typename TX, typename TO, int N>
__global__ void __launch_bounds__(kNormWideThreads) norm_wide_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float s_sum[2][1][32];
    const long long row = blockIdx.x;
    const TX *x = static_cast<const TX *>(a.x) + row * a.ld_x;
    float sum[1] = {0.f};
    for (int at = threadIdx.x; at < a.groups; at += kNormWideThreads) {
        float h[N];
        load_row<TX, N, false>(x + (long long)at * N, h);
        if (a.branch) {
            float b[N];
            load_either<N>(a.branch, a.branch32, row * a.ld_branch + (long long)at * N, b);
#pragma unroll
            for (int i = 0; i < N; ++i) h[i] = to_float(from_float<TX>(h[i] + b[i]));
            store_row<TX, N>(static_cast<TX *>(a.sum) + row * a.ld_sum + (long long)at * N, h);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) sum[0] += h[i];
    }
    row_sums<false, 1>(sum, s_sum[0]);
    const float mean = sum[0] / (float)a.H;
    const TX *from = a.branch ? static_cast<const TX *>(a.sum) + row * a.ld_sum : x;     // each thread reads what it wrote itself
    sum[0] = 0.f;
    for (int at = threadIdx.x; at < a.groups; at += kNormWideThreads) {
        float h[N];
        load_row<TX, N, false>(from + (long long)at * N, h);
#pragma unroll
        for (int i = 0; i < N; ++i) sum[0] = fmaf(h[i] - mean, h[i] - mean, sum[0]);
    }
    row_sums<false, 1>(sum, s_sum[1]);
    const float rstd = 1.0f / sqrtf(sum[0] / (float)a.H + a.eps);
    if (threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
    for (int at = threadIdx.x; at < a.groups; at += kNormWideThreads) {
        float h[N], w[N], b[N];
        load_row<TX, N>(from + (long long)at * N, h);
        load_weight<N>(a.weight, a.weight32, at * N, w);
        if (a.bias) load_weight<N>(a.bias, a.weight32, at * N, b);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = (h[i] - mean) * rstd;
            h[i] = a.bias ? fmaf(y, w[i], b[i]) : y * w[i];
        }
        store_row<TO, N>(static_cast<TO *>(a.out) + row * a.ld_out + (long long)at * N, h);
    }
}

// ---------------------------------------------------------------- gradient

// dx of N elements
template <typename TX, int N>
__device__ __forceinline__ void norm_dx(const NormGradArgs &a, long long row, int at, const float (&u)[N], const float (&xh)[N], const float (&dsum)[N], float rstd, float mu, float mx) {
    float d[N];
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = fmaf(rstd, u[i] - mu - xh[i] * mx, dsum[i]);
    store_row<TX, N>(static_cast<TX *>(a.dx) + row * a.ld_dx + (long long)at * N, d);
}

// Block `b` writes its columns' sums; threads that share columns (the warps of a block with a warp a row) add theirs in warp order.
template <int N, int E, bool kWarp>
__device__ __forceinline__ void put_sums(const NormGradArgs &a, int L, int t, float (&dw)[E / N][N], float (&db)[E / N][N]) {
    constexpr int G = E / N;
    float *part = a.part + (long long)blockIdx.x * 2 * a.H;
    if constexpr (kWarp) {
        __shared__ float s_all[2][kNormWarpRow];
        for (int o = L; o < 32; o *= 2)                          // the rows side by side in a warp
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dw[g][i] += __shfl_xor_sync(0xffffffffu, dw[g][i], o);
                    db[g][i] += __shfl_xor_sync(0xffffffffu, db[g][i], o);
                }
        const int warp = threadIdx.x >> 5;
        for (int w = 0; w < kNormWarps; ++w) {
            if (warp == w && (threadIdx.x & 31) < L)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const int at = g * L + t;
                    if (at < a.groups)
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const int c = at * N + i;
                            s_all[0][c] = (w ? s_all[0][c] : 0.f) + dw[g][i];
                            s_all[1][c] = (w ? s_all[1][c] : 0.f) + db[g][i];
                        }
                }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < a.H; c += kNormWarps * 32) {
            __stcg(part + c, s_all[0][c]);
            __stcg(part + a.H + c, s_all[1][c]);
        }
    } else {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int at = g * L + t;
            if (at < a.groups)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    __stcg(part + at * N + i, dw[g][i]);
                    __stcg(part + a.H + at * N + i, db[g][i]);
                }
        }
    }
}

template <typename TX, typename TO, int N, int E, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kNormWarps * 32 : 1024, kWarp ? 2 : 1) norm_grad_kernel(const __grid_constant__ NormGradArgs a) {
    constexpr int G = E / N;
    __shared__ float s_sum[2][2][32];
    const int L = kWarp ? a.lanes : blockDim.x, t = kWarp ? threadIdx.x & (L - 1) : threadIdx.x;
    float dw[G][N], db[G][N];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < N; ++i) dw[g][i] = db[g][i] = 0.f;
    const long long step = kWarp ? (long long)gridDim.x * (kNormWarps * 32 / L) : gridDim.x;
    long long row = kWarp ? (long long)blockIdx.x * (kNormWarps * 32 / L) + threadIdx.x / L : blockIdx.x;
    int odd = 0;
    // a warp's parts go on together: those past the last row add zeros and write nothing
    for (long long all = kWarp ? row - threadIdx.x % 32 / L : row; all < a.T; all += step, row += step) {
        const bool mine = row < a.T;
        float u[G][N], xh[G][N], more[G][N], sums[2] = {0.f, 0.f};
        const float mean = mine ? a.mean[row] : 0.f, rstd = mine ? a.rstd[row] : 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int at = g * L + t;
            if (mine && at < a.groups) {
                load_row<TO, N>(static_cast<const TO *>(a.dy) + row * a.ld_dy + (long long)at * N, u[g]);
                load_row<TX, N>(static_cast<const TX *>(a.x) + row * a.ld_x + (long long)at * N, xh[g]);
                if (a.dsum) load_row<TX, N>(static_cast<const TX *>(a.dsum) + row * a.ld_dsum + (long long)at * N, more[g]);
                else
#pragma unroll
                    for (int i = 0; i < N; ++i) more[g][i] = 0.f;
            }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int at = g * L + t;
            if (!mine || at >= a.groups) continue;
            float w[N];
            load_weight<N>(a.weight, a.weight32, at * N, w);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                xh[g][i] = (xh[g][i] - mean) * rstd;
                dw[g][i] = fmaf(u[g][i], xh[g][i], dw[g][i]);
                db[g][i] += u[g][i];
                u[g][i] *= w[i];
                sums[0] += u[g][i];
                sums[1] = fmaf(u[g][i], xh[g][i], sums[1]);
            }
        }
        row_sums<kWarp, 2>(sums, s_sum[odd], L);
        odd ^= 1;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int at = g * L + t;
            if (mine && at < a.groups) norm_dx<TX, N>(a, row, at, u[g], xh[g], more[g], rstd, sums[0] * a.inv_h, sums[1] * a.inv_h);
        }
    }
    put_sums<N, E, kWarp>(a, L, t, dw, db);
    let_next_start();
}

// Longer rows: the columns' sums first (dx may replace dy), a block for a stretch of columns and every gridDim.y-th row, then dx.
template <typename TX, typename TO, int N>
__global__ void __launch_bounds__(kNormWideThreads) norm_grad_columns_kernel(const __grid_constant__ NormGradArgs a) {
    const int at = blockIdx.x * kNormWideThreads + threadIdx.x;
    if (at >= a.groups) return;
    float dw[N], db[N];
#pragma unroll
    for (int i = 0; i < N; ++i) dw[i] = db[i] = 0.f;
    for (long long row = blockIdx.y; row < a.T; row += gridDim.y) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float dy[N], x[N];
        load_row<TO, N, false>(static_cast<const TO *>(a.dy) + row * a.ld_dy + (long long)at * N, dy);
        load_row<TX, N, false>(static_cast<const TX *>(a.x) + row * a.ld_x + (long long)at * N, x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            dw[i] = fmaf(dy[i], (x[i] - mean) * rstd, dw[i]);
            db[i] += dy[i];
        }
    }
    float *part = a.part + (long long)blockIdx.y * 2 * a.H + (long long)at * N;
#pragma unroll
    for (int i = 0; i < N; ++i) { __stcg(part + i, dw[i]); __stcg(part + a.H + i, db[i]); }
}

template <typename TX, typename TO, int N>
__global__ void __launch_bounds__(kNormWideThreads) norm_grad_wide_kernel(const __grid_constant__ NormGradArgs a) {
    __shared__ float s_sum[2][32];
    const long long row = blockIdx.x;
    const float mean = a.mean[row], rstd = a.rstd[row];
    const TO *dy = static_cast<const TO *>(a.dy) + row * a.ld_dy;
    const TX *x = static_cast<const TX *>(a.x) + row * a.ld_x;
    float sums[2] = {0.f, 0.f}, u[N], xh[N], w[N];
    auto load = [&](int at) {
        load_row<TO, N, false>(dy + (long long)at * N, u);
        load_row<TX, N, false>(x + (long long)at * N, xh);
        load_weight<N>(a.weight, a.weight32, at * N, w);
#pragma unroll
        for (int i = 0; i < N; ++i) { xh[i] = (xh[i] - mean) * rstd; u[i] *= w[i]; }
    };
    for (int at = threadIdx.x; at < a.groups; at += kNormWideThreads) {
        load(at);
#pragma unroll
        for (int i = 0; i < N; ++i) { sums[0] += u[i]; sums[1] = fmaf(u[i], xh[i], sums[1]); }
    }
    row_sums<false, 2>(sums, s_sum);
    for (int at = threadIdx.x; at < a.groups; at += kNormWideThreads) {
        float more[N];
        load(at);
        if (a.dsum) load_row<TX, N>(static_cast<const TX *>(a.dsum) + row * a.ld_dsum + (long long)at * N, more);
        else
#pragma unroll
            for (int i = 0; i < N; ++i) more[i] = 0.f;
        norm_dx<TX, N>(a, row, at, u, xh, more, rstd, sums[0] * a.inv_h, sums[1] * a.inv_h);
    }
}

// The blocks' sums, added in block order by 32 threads a column (every 32nd block each; with eight it took 10 us for 296 blocks of 4,096 columns) and
// then those 32.
// blockIdx.y: 0 the weight's gradient, 1 the bias's.
__global__ void __launch_bounds__(kNormJoinThreads) norm_join_kernel(const __grid_constant__ NormGradArgs a) {
    constexpr int kParts = kNormJoinThreads / 32;
    __shared__ float s_part[kParts][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    wait_for_previous();
    float sum = 0.f;
    if (c < a.H) {
        const float *p = a.part + (long long)blockIdx.y * a.H + c;
#pragma unroll 8
        for (int b = part; b < a.blocks; b += kParts) sum += __ldcg(p + (long long)b * 2 * a.H);
    }
    s_part[part][lane] = sum;
    __syncthreads();
    if (part || c >= a.H) return;
    sum = s_part[0][lane];
#pragma unroll
    for (int k = 1; k < kParts; ++k) sum += s_part[k][lane];
    void *to = blockIdx.y ? a.dbias : a.dweight;
    if (a.grad32) {
        float *d = static_cast<float *>(to) + c;
        *d = a.add ? *d + sum : sum;
    } else {
        bf16 *d = static_cast<bf16 *>(to) + c;
        *d = from_float<bf16>(a.add ? to_float(*d) + sum : sum);
    }
}

}  // namespace
