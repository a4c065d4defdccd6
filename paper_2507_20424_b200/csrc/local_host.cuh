// Host side that the operators of a worker's local step share: devices, launches, checks of arguments.
#pragma once
#include "dppf.h"
#include <cuda_runtime.h>
#include <atomic>
#include <climits>
#include <cmath>
#include <cstdint>
#include <initializer_list>

namespace dppf_internal {
int first_pass_polls();          // poll budgets set by dppf_debug_set_poll_limits
int later_pass_polls();
}

namespace {

constexpr int kMaxDevices = 64;

inline int current_device() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return -1;
    return dev;
}

inline int multiprocessors(int dev) {
    static std::atomic<int> known[kMaxDevices];
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return -1;
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// Dynamic shared memory above 48 KB has to be allowed once per kernel and device.
template <typename K>
bool allow_smem(K kernel, int dev, std::atomic<int> *done, int bytes) {
    if (done[dev].load(std::memory_order_relaxed)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done[dev].store(1, std::memory_order_relaxed);
    return true;
}

inline int launched() { return cudaGetLastError() == cudaSuccess ? DPPF_OK : DPPF_ERR_CUDA; }

// A launch that may be set up while the one before it in the stream still runs (its kernel waits by itself).
template <typename... P, typename... A>
bool launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess;
}

inline bool all_finite(std::initializer_list<float> vals) {
    for (float f : vals)
        if (!std::isfinite(f)) return false;
    return true;
}

inline bool ranges_meet(const void *a, size_t abytes, const void *b, size_t bbytes) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return a && b && abytes && bbytes && pa < pb + bbytes && pb < pa + abytes;
}

inline bool known_type(int t) { return t == DPPF_FLOAT32 || t == DPPF_BFLOAT16; }
inline size_t type_bytes(int t) { return t == DPPF_FLOAT32 ? 4 : 2; }
inline bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Bytes from the first element of row 0 to the last one of row rows - 1.
inline size_t matrix_bytes(int64_t rows, int64_t cols, int64_t ld, int type) {
    return rows > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * type_bytes(type) : 0;
}

constexpr int64_t kMaxLd = (int64_t)1 << 40;

// Rows of a matrix start on 16-byte boundaries.
inline bool rows_on_16(const void *p, int64_t ld, int type) { return aligned_to(p, 16) && (size_t)ld * type_bytes(type) % 16 == 0; }

// Heads of packed rows: element i of head h of token t at p[t * ld + h * head + i].
struct HeadRows {
    const void *p;
    int64_t ld, head, T;
    int heads, D, type;

    int64_t width() const { return (heads - 1) * head + D; }                        // of a token's heads, from the first to the last
    bool by_token() const { return ld >= width() && head >= (heads > 1 ? D : 0); }
    // No element lies on another: a token's heads side by side within its row, or a head's tokens within its block.
    bool apart() const {
        if (ld < 0 || head < 0 || ld > kMaxLd || head > kMaxLd) return false;
        return by_token() || (ld >= D && head >= (T - 1) * ld + D);
    }
    size_t bytes() const { return T > 0 ? (size_t)((T - 1) * ld + width()) * type_bytes(type) : 0; }
    // Whether an element of one may be an element of the other.  Heads of the same rows, as queries and keys of one product have
    // them, are told apart by their columns.
    bool meets(const HeadRows &o) const {
        if (!ranges_meet(p, bytes(), o.p, o.bytes())) return false;
        if (type == o.type && ld == o.ld && by_token() && o.by_token()) {
            const int64_t row = ld * (int64_t)type_bytes(type), w = width() * (int64_t)type_bytes(type), ow = o.width() * (int64_t)type_bytes(type);
            int64_t gap = (int64_t)(reinterpret_cast<intptr_t>(o.p) - reinterpret_cast<intptr_t>(p)) % row;
            if (gap < 0) gap += row;
            return !(gap >= w && gap + ow <= row);
        }
        return true;
    }
};

inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace
