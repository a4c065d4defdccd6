// Rotary positions: pairs of a head's elements turned by position * frequency, all heads of a token alike.
//
//   a = position * frequency_i;   (x1, x2) -> scale (x1 cos a - x2 sin a, x2 cos a + x1 sin a);   inverse: by -a
//
// Bound by memory: every element is read and written once.  A block takes some tokens: its threads compute their angles once, in
// 64 bits (an fp32 product is off by half a radian at position 10^7), put cosine and sine in shared memory, and then walk the
// tokens' heads, N pairs a thread at a time.  16,384 tokens of 40 heads of 128, bf16 in place: 55 us (6.0 TB/s, of a copy rate of 6.5);
// with pairs side by side 63.  The table is as small as that (8 KB) so that eight blocks fit an SM: 61 us with 32 KB.
#pragma once
#include "local_common.cuh"

namespace {

constexpr int kRotaryThreads = 256;
constexpr int kRotaryMaxTokens = 16;          // of a block
constexpr int kRotaryTable = 1024;            // cosines (and as many sines) that a block holds

struct RotaryArgs {
    const void *x;
    void *out;
    const void *positions;
    const double *frequencies;
    long long ld_x, head_x, ld_out, head_out, T;
    int heads, D, half;          // half: pairs that are turned
    int tokens;                  // of a block
    int turn_groups, rest_groups;   // of a head: N pairs each; N elements each that are copied (0 in place)
    int positions64, inverse;
    float scale;
};

template <int N>
__device__ __forceinline__ void table_load(const float *p, float (&f)[N]) {      // starts are multiples of N
    if constexpr (N >= 4)
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(p + i);
            f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
        }
    else if constexpr (N == 2) {
        const float2 v = *reinterpret_cast<const float2 *>(p);
        f[0] = v.x; f[1] = v.y;
    } else {
        f[0] = p[0];
    }
}

template <typename T, int N, bool kInterleaved>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const __grid_constant__ RotaryArgs a) {
    __shared__ __align__(16) float s_cos[kRotaryTable], s_sin[kRotaryTable];
    const long long first = (long long)blockIdx.x * a.tokens;
    const int tokens = (int)min((long long)a.tokens, a.T - first);
    for (int i = threadIdx.x; i < tokens * a.half; i += kRotaryThreads) {
        const int t = i / a.half;
        const double p = a.positions64 ? (double)static_cast<const long long *>(a.positions)[first + t] : (double)static_cast<const int *>(a.positions)[first + t];
        double turns = p * a.frequencies[i - t * a.half] * 0.15915494309189535;      // 1 / (2 pi)
        turns -= rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        s_cos[i] = c * a.scale;
        s_sin[i] = (a.inverse ? -s : s) * a.scale;
    }
    __syncthreads();
    const int each = a.turn_groups + a.rest_groups, row = a.heads * each;
    for (int i = threadIdx.x; i < tokens * row; i += kRotaryThreads) {
        const int t = i / row, in_row = i - t * row, head = in_row / each, g = in_row - head * each;
        const T *x = static_cast<const T *>(a.x) + (first + t) * a.ld_x + head * a.head_x;
        T *out = static_cast<T *>(a.out) + (first + t) * a.ld_out + head * a.head_out;
        if (g >= a.turn_groups) {
            const int at = 2 * a.half + (g - a.turn_groups) * N;
            float v[N];
            load_vec<T, N>(x + at, v);
            store_vec<T, N>(out + at, v);
            continue;
        }
        float cs[N], sn[N];
        table_load(s_cos + t * a.half + g * N, cs);
        table_load(s_sin + t * a.half + g * N, sn);
        if constexpr (kInterleaved) {
            float v[2 * N];
            if constexpr (N == 1) { v[0] = to_float(x[2 * g]); v[1] = to_float(x[2 * g + 1]); }   // a pair may lie across its boundary
            else load_vec<T, 2 * N>(x + 2 * g * N, v);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float p = v[2 * k], q = v[2 * k + 1];
                v[2 * k] = p * cs[k] - q * sn[k];
                v[2 * k + 1] = q * cs[k] + p * sn[k];
            }
            if constexpr (N == 1) { out[2 * g] = from_float<T>(v[0]); out[2 * g + 1] = from_float<T>(v[1]); }
            else store_vec<T, 2 * N>(out + 2 * g * N, v);
        } else {
            float p[N], q[N], r[N];
            load_vec<T, N>(x + g * N, p);
            load_vec<T, N>(x + a.half + g * N, q);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                r[k] = p[k] * cs[k] - q[k] * sn[k];
                q[k] = q[k] * cs[k] + p[k] * sn[k];
            }
            store_vec<T, N>(out + g * N, r);
            store_vec<T, N>(out + a.half + g * N, q);
        }
    }
}

}  // namespace
