// Tensor cores of sm_100a as the attention kernels use them: tiles of 128 rows brought in by tensor copies, products issued by one
// thread with their sums in tensor memory, and bounded waits.
//
// Shared memory: a tile of 128 rows by 64 or 128 bf16 columns lies as one or two blocks of 64 columns (kBlockBytes each), a row of
// a block in 128 bytes, 16-byte pieces swizzled within 1,024 bytes (the copies' 128-byte swizzle).  As an operand whose rows are
// its M or N index ("rows") a step of 16 columns is 32 bytes further on; as one whose rows are summed over ("columns": M or N
// is the tile's column) a step of 16 rows is 2,048 bytes further on and the next 64 columns are a block further on.
// Tensor memory: 128 lanes (rows of a product) of 512 32-bit columns; a warp reaches the 32 lanes of its number modulo 4.
#pragma once
#include "local_common.cuh"
#include <cuda.h>

namespace {

constexpr int kTile = 128;                       // rows of a tile
constexpr unsigned kBlockBytes = kTile * 128;    // 64 columns of bf16

// ---------------------------------------------------------------- waits
// Every wait is bounded; the first that gives up makes all others of the block give up soon.

struct Waits {
    volatile int *dead;      // shared, one for the block
    int limit;
    __device__ __forceinline__ bool later(unsigned long long *bar, unsigned parity) const {
#pragma unroll 1
        for (int i = 0; i < limit; ++i) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((i & 63) == 63 && *dead) return false;
        }
        *dead = 1;
        return false;
    }
    // The first look is apart from the loop: one that finds the phase done costs some 40 cycles, the loop's 150.
    __device__ __forceinline__ bool operator()(unsigned long long *bar, unsigned parity) const {
        if (__builtin_expect(limit > 0 && mbar_try_wait(bar, parity), 1)) return true;
        return later(bar, parity);
    }
    // by a whole warp, which goes on together
    __device__ __forceinline__ bool together(unsigned long long *bar, unsigned parity) const {
        if (__builtin_expect(__all_sync(0xffffffffu, limit > 0 && mbar_try_wait(bar, parity)), 1)) return true;
        return __all_sync(0xffffffffu, later(bar, parity));
    }
};

__device__ __forceinline__ void mbar_arrive(unsigned long long *bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// Registers of a warpgroup's threads from here on.  A block starts with kThreads times as many as it was compiled for; what one
// warpgroup gives up another may take, never more than that in all.
template <int kRegisters> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegisters)); }
template <int kRegisters> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegisters)); }

// Barrier `id` (1 .. 15) of `threads` threads.
__device__ __forceinline__ void group_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// ---------------------------------------------------------------- copies

// Box at (column, head, row) of a tensor [rows][heads][columns]; what lies outside the tensor is zero.  column * 2 is a multiple of 16.
__device__ __forceinline__ void tensor_load(unsigned dst, const CUtensorMap *map, int column, int head, int row, unsigned long long *bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(column), "r"(head), "r"(row), "r"(smem_addr(bar)) : "memory");
}
// A tile: its blocks of 64 columns, announced to `bar` by the caller.
template <int kBlocks>
__device__ __forceinline__ void tile_load(unsigned dst, const CUtensorMap *map, int head, int row, unsigned long long *bar) {
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) tensor_load(dst + c * kBlockBytes, map, 64 * c, head, row, bar);
}
// Rows first .. 127 of a tile become zeros (a warp): rows of other sequences must not reach a sum over rows, where 0 times NaN is NaN.
template <int kBlocks>
__device__ __forceinline__ void zero_rows(unsigned tile, int first) {
    const int lane = threadIdx.x & 31, pieces = (kTile - first) * 8;
#pragma unroll
    for (int c = 0; c < kBlocks; ++c)
        for (int i = lane; i < pieces; i += 32)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + c * kBlockBytes + first * 128 + i * 16), "r"(0) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the products read through the asynchronous proxy
    __syncwarp();
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// Where the 16-byte piece `piece` (eight columns) of row r lies in a tile.
__device__ __forceinline__ unsigned piece_at(unsigned tile, int r, int piece) { return tile + (piece >> 3) * kBlockBytes + r * 128 + (((piece & 7) ^ (r & 7)) << 4); }

// Sixteen words of row r of a tile: its columns [32 part, 32 part + 32).
__device__ __forceinline__ void tile_row(unsigned tile, int r, int part, unsigned (&u)[16]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int piece = part * 4 + c;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(u[4 * c]), "=r"(u[4 * c + 1]), "=r"(u[4 * c + 2]), "=r"(u[4 * c + 3])
                     : "r"(piece_at(tile, r, piece)) : "memory");
    }
}

// ---------------------------------------------------------------- products
// An instruction's operands lie in uniform registers.  Values that the compiler knows to be the same in all lanes stay there; of
// others it moves every one over before each instruction, which held the products up (about 100 cycles an instruction, of 64).
// So what they are formed from passes through uniform(), and their thread is the one that elect() names.

__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ unsigned uniform(unsigned x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ bool elect() {                            // true in one lane of the warp, always the same
    unsigned is;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(is));
    return is != 0;
}

__device__ __forceinline__ unsigned long long operand(unsigned addr, unsigned leading_bytes) {
    // bits 0-13 address / 16, 16-29 leading offset / 16, 32-45 stride of eight rows / 16, 46-48 one, 61-63 128-byte swizzle
    return (unsigned long long)((addr & 0x3ffff) >> 4) | (unsigned long long)(leading_bytes >> 4) << 16 | (unsigned long long)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ unsigned long long operand_rows(unsigned tile) { return operand(tile, 16); }
__device__ __forceinline__ unsigned long long operand_columns(unsigned tile) { return operand(tile, kBlockBytes); }

// Instruction descriptor: fp32 sums, bf16 operands, M = 128, N a multiple of 16; kColumns: the second operand's rows are summed over.
template <int N, bool kColumns>
__device__ __forceinline__ constexpr unsigned product_kind() {
    return 1u << 4 | 1u << 7 | 1u << 10 | (kColumns ? 1u << 16 : 0u) | (unsigned)(N >> 3) << 17 | (unsigned)(kTile >> 4) << 24;
}
// d[128, N] (+)= a b over 16 elements; one thread.
__device__ __forceinline__ void product16(unsigned d, unsigned long long a, unsigned long long b, unsigned kind, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"((unsigned)add) : "memory");
}
// The same with the first operand in tensor memory.
__device__ __forceinline__ void product16_tmem(unsigned d, unsigned a, unsigned long long b, unsigned kind, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(kind), "r"((unsigned)add) : "memory");
}
// d[128, 128] = rows of tile a times rows of tile b, summed over the first 16 kSteps columns.
template <int kSteps>
__device__ __forceinline__ void product_rows(unsigned d, unsigned a, unsigned b) {
    const unsigned long long da = operand_rows(a), db = operand_rows(b);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const unsigned at = ((k / 4) * kBlockBytes + (k % 4) * 32) >> 4;
        product16(d, da + at, db + at, product_kind<kTile, false>(), k > 0);
    }
}
// The same with a's rows in tensor memory, 16 columns in eight there.
template <int kSteps>
__device__ __forceinline__ void product_rows_tmem(unsigned d, unsigned a, unsigned b) {
    const unsigned long long db = operand_rows(b);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) product16_tmem(d, a + 8 * k, db + (((k / 4) * kBlockBytes + (k % 4) * 32) >> 4), product_kind<kTile, false>(), k > 0);
}
// d[128, 16 kSteps] (+)= p[128, 64] times rows [64 half, 64 half + 64) of tile b, summed over them.  p: bf16 pairs in 32 columns of tensor
// memory.
template <int kSteps>
__device__ __forceinline__ void product_columns(unsigned d, unsigned p, unsigned b, int half, bool add) {
    const unsigned long long db = operand_columns(b + half * 8192);
#pragma unroll
    for (int k = 0; k < 4; ++k) product16_tmem(d, p + k * 8, db + ((k * 2048) >> 4), product_kind<16 * kSteps, true>(), add || k > 0);
}
// Arrives on `bar` when all products that this thread has issued are done.
__device__ __forceinline__ void products_done(unsigned long long *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// ---------------------------------------------------------------- tensor memory

__device__ __forceinline__ void tmem_alloc(unsigned *where, int columns) {      // a warp; waits for other blocks' columns
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(where)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(unsigned at, int columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

#define DPPF_R4(v, i) "=f"(v[i]), "=f"(v[i + 1]), "=f"(v[i + 2]), "=f"(v[i + 3])
#define DPPF_R16(v, i) DPPF_R4(v, i), DPPF_R4(v, i + 4), DPPF_R4(v, i + 8), DPPF_R4(v, i + 12)
#define DPPF_M4(v, i) "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3])
#define DPPF_M16(v, i) DPPF_M4(v, i), DPPF_M4(v, i + 4), DPPF_M4(v, i + 8), DPPF_M4(v, i + 12)
#define DPPF_U4(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3])
#define DPPF_U16(v, i) DPPF_U4(v, i), DPPF_U4(v, i + 4), DPPF_U4(v, i + 8), DPPF_U4(v, i + 12)

// 32 columns of the thread's lane; the values are there after tmem_loaded(v).
__device__ __forceinline__ void tmem_load32(unsigned at, float (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
                 "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : DPPF_R16(v, 0), DPPF_R16(v, 16) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_loaded(float (&v)[32]) {       // waits for all loads before it; ties v's uses to the wait
    asm volatile("tcgen05.wait::ld.sync.aligned;" : DPPF_M16(v, 0), DPPF_M16(v, 16)::"memory");
}
__device__ __forceinline__ void tmem_load16(unsigned at, float (&v)[16]) {          // 16 columns, waited for
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
                 "tcgen05.wait::ld.sync.aligned;"
                 : DPPF_R16(v, 0) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store16(unsigned at, const unsigned (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(at), DPPF_U16(v, 0) : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

}  // namespace
