// Shared pieces of the kernels around a worker's local step on a language model (embedding, policy
// loss, AdamW over many tensors): element types, vectors of eight elements, cluster accesses.
#pragma once
#include "chunk_ring.cuh"
#include <cuda_bf16.h>
#include <cfloat>

namespace {

using bf16 = __nv_bfloat16;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float x) { return __float2bfloat16_rn(x); }

// ---------------------------------------------------------------- N consecutive elements as fp32
// N * sizeof(T) bytes in as few accesses as its alignment to min(16, N * sizeof(T)) bytes allows.
// kOnce: the data is not read again soon (streaming loads; stores always are).

__device__ __forceinline__ float bf16_low(unsigned u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_high(unsigned u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ unsigned bf16_pair(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<unsigned *>(&h);
}

template <int N> struct Words;                       // N 32-bit words
template <> struct Words<1> { using type = unsigned; };
template <> struct Words<2> { using type = uint2; };
template <> struct Words<4> { using type = uint4; };

template <typename T, int N, bool kOnce = true>
__device__ __forceinline__ void load_vec(const T *p, float (&f)[N]) {
    if constexpr (N == 1) {
        f[0] = to_float(kOnce ? __ldcs(p) : __ldcg(p));
    } else {
        constexpr int kWords = N * (int)sizeof(T) / 4, kPer = kWords < 4 ? kWords : 4;
        using W = typename Words<kPer>::type;
        unsigned u[kWords];
#pragma unroll
        for (int i = 0; i < kWords / kPer; ++i) {
            const W w = kOnce ? __ldcs(reinterpret_cast<const W *>(p) + i) : __ldcg(reinterpret_cast<const W *>(p) + i);
            memcpy(&u[i * kPer], &w, sizeof(W));
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = __uint_as_float(u[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) { f[2 * i] = bf16_low(u[i]); f[2 * i + 1] = bf16_high(u[i]); }
        }
    }
}

template <typename T, int N>
__device__ __forceinline__ void store_vec(T *p, const float (&f)[N]) {
    if constexpr (N == 1) {
        __stcs(p, from_float<T>(f[0]));
    } else {
        constexpr int kWords = N * (int)sizeof(T) / 4, kPer = kWords < 4 ? kWords : 4;
        using W = typename Words<kPer>::type;
        unsigned u[kWords];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) u[i] = __float_as_uint(f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) u[i] = bf16_pair(f[2 * i], f[2 * i + 1]);
        }
#pragma unroll
        for (int i = 0; i < kWords / kPer; ++i) {
            W w;
            memcpy(&w, &u[i * kPer], sizeof(W));
            __stcs(reinterpret_cast<W *>(p) + i, w);
        }
    }
}

// ---------------------------------------------------------------- two fp32 operations in one instruction
// Each result is rounded by itself.  A packed sum that follows a packed product was seen to come out as a fused
// multiply-add, in spite of .rn: where the product has to be rounded first, the sum is written as two scalar ones.

__device__ __forceinline__ unsigned long long pack2(float2 a) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y));
    return r;
}
__device__ __forceinline__ float2 unpack2(unsigned long long a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(a)), "l"(pack2(b)));
    return unpack2(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(a)), "l"(pack2(b)));
    return unpack2(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pack2(a)), "l"(pack2(b)), "l"(pack2(c)));
    return unpack2(r);
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// ---------------------------------------------------------------- clusters

__device__ __forceinline__ unsigned cluster_rank() {
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned cluster_size() {
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// Arrival of a thread that has written nothing the others are to see: no fence.
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// Shared-memory address of the same variable in another block of the cluster.
__device__ __forceinline__ unsigned cluster_map(const void *p, unsigned rank) {
    unsigned a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    return a;
}
// Asynchronous store of a pair to an address of the cluster's shared memory, counted (8 bytes) on the mbarrier `bar` of the
// same block: who waits for that sees the pair, and no fence is needed.
__device__ __forceinline__ void cluster_send2(unsigned a, float x, float y, unsigned bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(a), "f"(x), "f"(y), "r"(bar) : "memory");
}

// ---------------------------------------------------------------- launches that follow one another
// The dependent launch may be scheduled from here on; it waits for this one's end before it reads.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {   // 2 ulp; results below 2^-126 are 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace
