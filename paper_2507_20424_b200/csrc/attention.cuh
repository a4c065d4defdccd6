// Attention within packed sequences: the plan of a batch, the forward kernel and the two of the gradient.
//
// A batch of B sequences is T packed rows; sequence b is rows [starts[b], starts[b + 1]).  The plan, made once a batch on the
// device, lists its tiles of 128 rows (and of 256), the longest work first; rows of no sequence are tiles of their own, whose
// outputs are zeros.
#pragma once
#include "tensor_core.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ---------------------------------------------------------------- the plan

constexpr int kPlanThreads = 1024;
constexpr int kPlanBins = 2048;
constexpr unsigned kPlanMagic = 0x4450504cu;
enum { kByQuery, kByQuery2, kByKey, kPlanLists };     // tiles of 128 rows by work of a query tile; of 256; of 128 by work of a key tile

struct PlanHeader {          // first bytes of the plan
    int status;              // dppf_status seen by the kernels
    unsigned magic;
    int tiles[kPlanLists];
    int T, B;                // what the lists' places go by
};
__device__ __forceinline__ bool is_plan(const PlanHeader *h, long long T, int B) { return h->magic == kPlanMagic && h->T == T && h->B == B; }
struct PlanTile { int row, rows, begin, end; };       // first row, rows of this tile; its sequence's rows (begin == end: no sequence)

__device__ __forceinline__ PlanTile uniform(const PlanTile &t) { return {uniform(t.row), uniform(t.rows), uniform(t.begin), uniform(t.end)}; }

struct PlanArgs {
    const void *starts;
    PlanHeader *hdr;
    int *bounds, *count;     // [B + 1] each: starts in order and within [0, T]; tiles before sequence b
    PlanTile *list[kPlanLists];
    long long T;
    int B, starts64, most[kPlanLists];
};

__device__ __forceinline__ int plan_scan(int v, int *s_warp, bool sum) {        // inclusive sum or maximum over the block
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v = sum ? v + u : max(v, u);
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int w = s_warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int u = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w = sum ? w + u : max(w, u);
        }
        s_warp[lane] = w;
    }
    __syncthreads();
    return warp == 0 ? v : sum ? v + s_warp[warp - 1] : max(v, s_warp[warp - 1]);
}

// One block.  The order within a list is that of a counting sort by work (atomics within a bin: tiles of equal work in any order,
// which no result depends on).
__global__ void __launch_bounds__(kPlanThreads) attention_plan_kernel(const __grid_constant__ PlanArgs a) {
    __shared__ int s_warp[32], s_bin[kPlanBins], s_carry;
    const int tid = threadIdx.x;
    // starts that fall back or lie outside [0, T] are pulled into order: no tile reaches beyond the rows, none overlaps another
    if (tid == 0) s_carry = 0;
    __syncthreads();
    for (int b0 = 0; b0 <= a.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        long long v = 0;
        if (b <= a.B) v = a.starts64 ? static_cast<const long long *>(a.starts)[b] : (long long)static_cast<const int *>(a.starts)[b];
        const int m = max(plan_scan((int)max(0LL, min(v, a.T)), s_warp, false), s_carry);
        if (b <= a.B) a.bounds[b] = m;
        __syncthreads();
        if (tid == kPlanThreads - 1) s_carry = m;
        __syncthreads();
    }
    const int first = a.bounds[0], last = a.bounds[a.B], T = (int)a.T;
    for (int list = 0; list < kPlanLists; ++list) {
        const int size = list == kByQuery2 ? 2 * kTile : kTile;
        __syncthreads();
        if (tid == 0) s_carry = 0;
        for (int i = tid; i < kPlanBins; i += kPlanThreads) s_bin[i] = 0;
        __syncthreads();
        for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
            const int b = b0 + tid, n = b < a.B ? (a.bounds[b + 1] - a.bounds[b] + size - 1) / size : 0;
            const int sum = plan_scan(n, s_warp, true) + s_carry;
            if (b < a.B) a.count[b + 1] = sum;
            __syncthreads();
            if (tid == kPlanThreads - 1) s_carry = sum;
            __syncthreads();
        }
        if (tid == 0) a.count[0] = 0;
        __syncthreads();
        const int tiles = s_carry, before = (first + size - 1) / size, after = (T - last + size - 1) / size;
        auto tile = [&](int i) {                                     // i-th tile: sequences', then the rows of none
            PlanTile t;
            if (i < tiles) {
                int lo = 0, hi = a.B - 1;                            // the sequence whose tiles i is among
                while (lo < hi) {
                    const int mid = (lo + hi + 1) / 2;
                    if (a.count[mid] <= i) lo = mid;
                    else hi = mid - 1;
                }
                t.begin = a.bounds[lo];
                t.end = a.bounds[lo + 1];
                t.row = t.begin + (i - a.count[lo]) * size;
                t.rows = min(size, t.end - t.row);
            } else {
                i -= tiles;
                t.begin = t.end = 0;
                t.row = i < before ? i * size : last + (i - before) * size;
                t.rows = min(size, (i < before ? first : T) - t.row);
            }
            return t;
        };
        auto bin = [&](const PlanTile &t) {                          // most work first
            const int work = t.begin == t.end ? 0 : 1 + (list == kByKey ? t.end - t.row : t.row - t.begin) / kTile;
            return kPlanBins - 1 - min(work, kPlanBins - 1);
        };
        const int all = min(tiles + before + after, a.most[list]);
        for (int i = tid; i < all; i += kPlanThreads) atomicAdd(&s_bin[bin(tile(i))], 1);
        __syncthreads();
        const int x = s_bin[2 * tid], y = s_bin[2 * tid + 1], sum = plan_scan(x + y, s_warp, true);
        s_bin[2 * tid] = sum - x - y;
        s_bin[2 * tid + 1] = sum - y;
        __syncthreads();
        for (int i = tid; i < all; i += kPlanThreads) {
            const PlanTile t = tile(i);
            a.list[list][atomicAdd(&s_bin[bin(t)], 1)] = t;
        }
        if (tid == 0) a.hdr->tiles[list] = all;
    }
    if (tid == 0) {
        a.hdr->status = DPPF_OK;
        a.hdr->T = T;
        a.hdr->B = a.B;
        a.hdr->magic = kPlanMagic;
    }
}
static_assert(kPlanBins == 2 * kPlanThreads, "a thread scans two bins");

// ---------------------------------------------------------------- forward

struct AttentionArgs {
    CUtensorMap q, k, v;
    PlanHeader *hdr;
    const PlanTile *tiles;
    bf16 *out;
    float *lse;                  // [heads][T]
    long long ld_out, head_out, T;
    int list, share, D, B;       // share: query heads of a key head
    int by_head, units;          // the two slots of a block: two heads of a tile of 128 rows, or the halves of one of 256; blocks of a tile
    int causal, window;          // window 0: none
    float scale2;                // scale * log2 e
    int spin;
};

constexpr float kRise = 0x1p20f, kRiseLog2 = 20.0f;      // exponentials relative to a maximum taken earlier
constexpr int kForwardThreads = 384;       // two warpgroups of a slot each, one of copies and products
// Of the 168 registers a thread that a block of 384 starts with: a row of scores stays in a softmax thread's.
constexpr int kSoftmaxRegisters = 208, kControlRegisters = 88;
static_assert(256 * kSoftmaxRegisters + 128 * kControlRegisters <= kForwardThreads * 168, "no more registers than the block has");
template <int kSteps>
struct ForwardShape {
    static constexpr int kBlocks = (kSteps + 3) / 4;
    static constexpr unsigned kTileBytes = kBlocks * kBlockBytes;
    static constexpr int kStages = kBlocks == 2 ? 2 : 4;                 // of a tile of keys and one of values
    static constexpr int kPolynomial = kBlocks == 2 ? 8 : 4;             // one in so many exponentials is a polynomial
    static constexpr unsigned kSmem = (2 + 2 * kStages) * kTileBytes + 2 * kBlockBytes + 1024;      // and half a tile of results a slot
};

// 32 columns of a row, from column 32 part on, times `by` as bf16 into a tile that no product or copy needs any more.
__device__ __forceinline__ void put_row(unsigned tile, int r, int part, const float (&v)[32], float by) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float *f = v + 8 * c;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece_at(tile, r, part * 4 + c)), "r"(bf16_pair(f[0] * by, f[1] * by)), "r"(bf16_pair(f[2] * by, f[3] * by)),
                     "r"(bf16_pair(f[4] * by, f[5] * by)), "r"(bf16_pair(f[6] * by, f[7] * by)) : "memory");
    }
}
// A warp's 32 rows of a tile, from row r0 on, to memory: kPieces pieces of 16 bytes from `first` on, those of a row by lanes side by side (a
// row a thread took 4,000 cycles for what takes 1,000 so).  out: row 0 of the tile; rows: how many of the tile are to be written.
template <int kPieces>
__device__ __forceinline__ void store_rows(unsigned tile, int r0, int first, bf16 *out, long long ld, int rows, int D) {
    constexpr int kRows = 32 / kPieces;
    const int lane = threadIdx.x & 31, piece = first + lane % kPieces;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 32; i += kRows) {
        const int r = r0 + i + lane / kPieces;
        if (r < rows && piece * 8 < D) {
            uint4 u;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(piece_at(tile, r, piece)) : "memory");
            *reinterpret_cast<uint4 *>(out + r * ld + piece * 8) = u;
        }
    }
}
// Rows [0, rows) of a head: value `fill` (0 or NaN) in all columns; threads tid of n.
__device__ __forceinline__ void fill_rows(bf16 *p, long long ld, int rows, int D, float fill, int tid, int n) {
    const unsigned u = bf16_pair(fill, fill);
    for (int i = tid; i < rows * (D / 8); i += n) {
        const int r = i / (D / 8), c = i - r * (D / 8);
        *reinterpret_cast<uint4 *>(p + r * ld + c * 8) = make_uint4(u, u, u, u);
    }
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}

// 2^x of two numbers on the multiply-add pipes, for a part of the exponentials: the special function unit gives 16 a cycle and SM,
// as many as the products of a tile ask for in their time.  x = n + f with n whole and |f| <= 1/2: the fp32 sum x + 1.5 2^23 + 127 ends in
// n + 127, the exponent field of 2^n, and a polynomial of degree 4 (least relative error with p(0) = 1 on the interval: 2.9e-6, far below the 2^-8 of
// the bf16 result) gives 2^f, its last step with f and 1 times 2^n.  x <= -127 gives 0 and NaN stays NaN (an addition to the polynomial's exponent
// field made it a finite number; that was 2 % faster in the gradient of heads of 64, up to 1 % elsewhere).  x above 127.5 gives any
// number: the forward kernel looks for those, the gradient's are masked.
__device__ __forceinline__ float2 exp2_polynomial(float2 x) {
    const float kRound = 12582912.0f + 127.0f;
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(-127.0f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(-127.0f));
    const float2 t = add2(x, both(kRound)), n = add2(t, both(-kRound)), f = fma2(n, both(-1.0f), x);
    const float2 s = make_float2(__int_as_float(__float_as_int(t.x) << 23), __int_as_float(__float_as_int(t.y) << 23)), fs = mul2(f, s);
    float2 p = fma2(f, both(0.009582852944731712f), both(0.055906426161527634f));
    p = fma2(p, f, both(0.24024099111557007f));
    p = fma2(p, f, both(0.6931241750717163f));
    return fma2(p, fs, s);
}

// A row of NaN, where a wait gave up (copies may still be on their way to the tiles).
__device__ __forceinline__ void spoil_row(bf16 *row, int D) {
    const unsigned u = 0x7fc07fc0u;
    for (int c = 0; c < D; c += 8) *reinterpret_cast<uint4 *>(row + c) = make_uint4(u, u, u, u);
}

// S = scale q k^T over the keys that a query sees; out = softmax(S) v; lse = log sum exp S.
// One pass over the keys with a running maximum and sum.  A block has two slots of 128 queries that share their keys and values:
// while one slot's warpgroup takes the exponentials of its scores (a row a thread), the tensor cores work for the other.
// Scores and output sums stay in tensor memory; the probabilities replace the scores there as bf16, the first operand of the second product.
// A block stays for several tiles: the next one's copies and first products run while this one's results are written.  Tiles come
// sorted by work; a round of them is dealt out forwards, the next backwards, so that every block gets about the same.
//
// Rounded to fewer bits: the probabilities, to bf16 for the second product (relative to about the largest; the sum that they are divided by is of
// the fp32 values), and the result.  What bounds it: a slot's chain of scores (512 cycles of the tensor cores), copy to registers (110), exponentials
// (1,700: 128 a thread, a part on the multiply-add pipes) and the second product (512), two of which run by turns: about 3,200 cycles for two
// tiles of 128 x 128 x 128, 2,048 of them products.  Measured on a B200: 16,384 tokens in four sequences, 16 heads of 128 on four
// key heads, all keys 456 us (1,205 TFLOP/s; with a key head each 531); 8,192 tokens in six documents, 32 heads on eight, causal 273 us (1,079 TFLOP/s); in
// runs of seconds the 1,000 W limit makes that 311.
// Tried and lost: one maximum a tile before the exponentials (3 to 5 %), two threads a row (10 %), a warp for each slot's products (10 %),
// products from registers that the compiler does not know to be uniform (25 %).

struct ForwardItem {             // a tile of queries, two slots: rows [row, row + rows) of a head, key blocks [lo, hi) counted from the sequence's begin
    PlanTile t;
    int head0, kv_head, lo[2], hi[2], first, last, slots;
    bool by_head;
    __device__ __forceinline__ ForwardItem(const AttentionArgs &a, const PlanTile &tile, int unit) : t(tile), by_head(a.by_head) {
        head0 = by_head ? 2 * unit : unit;
        kv_head = head0 / a.share;
        slots = by_head || t.rows > kTile ? 2 : 1;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            lo[s] = a.window ? max(0, row(s) - a.window + 1 - t.begin) / kTile : 0;
            hi[s] = ((a.causal ? min(t.end, row(s) + kTile) : t.end) - t.begin + kTile - 1) / kTile;
        }
        first = slots == 2 ? min(lo[0], lo[1]) : lo[0];
        last = slots == 2 ? max(hi[0], hi[1]) : hi[0];
    }
    __device__ __forceinline__ bool idle() const { return t.begin == t.end; }                                  // rows of no sequence
    __device__ __forceinline__ int row(int s) const { return by_head ? t.row : t.row + s * kTile; }
    __device__ __forceinline__ int rows(int s) const { return by_head ? t.rows : min(kTile, t.rows - s * kTile); }
    __device__ __forceinline__ int head(int s) const { return by_head ? head0 + s : head0; }
    __device__ __forceinline__ int key0(int j) const { return t.begin + j * kTile; }
};

// The items of this block, in order; the plan is read an item ahead.
struct ForwardItems {
    const PlanTile *tiles;
    unsigned total, units, round, at;
    PlanTile ahead;
    __device__ __forceinline__ unsigned index(unsigned r) const { return r * gridDim.x + (r & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x); }
    __device__ __forceinline__ explicit ForwardItems(const AttentionArgs &a) : tiles(a.tiles), total(uniform((unsigned)a.hdr->tiles[a.list]) * (unsigned)a.units), units(a.units), round(0), at(index(0)) {
        if (at < total) ahead = tiles[at / units];
    }
    __device__ __forceinline__ bool there() const { return at < total; }
    __device__ __forceinline__ ForwardItem take(const AttentionArgs &a) {
        const PlanTile t = uniform(ahead);
        const int unit = (int)(at % units);
        at = index(++round);
        if (at < total) ahead = tiles[at / units];
        return ForwardItem(a, t, unit);
    }
};

template <int kSteps>
__global__ void __launch_bounds__(kForwardThreads, 1) attention_kernel(const __grid_constant__ AttentionArgs a) {
    using Shape = ForwardShape<kSteps>;
    constexpr int kBlocks = Shape::kBlocks;
    constexpr int kStages = Shape::kStages, kPolynomial = Shape::kPolynomial;
    constexpr unsigned kTileBytes = Shape::kTileBytes;
    constexpr int kColumns = 512;
    extern __shared__ unsigned char smem_raw[];
    __shared__ unsigned long long q_full[2], q_free[2], k_full[kStages], v_full[kStages], v_ready[kStages], empty[kStages], s_full[2], p_half[2], p_full[2], o_full[2], o_free[2], drained;
    __shared__ unsigned s_tmem;
    __shared__ volatile int s_dead;
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    if (tid < 3) prefetch_map(tid == 0 ? &a.q : tid == 1 ? &a.k : &a.v);
    if (!is_plan(a.hdr, a.T, a.B)) {                 // not a plan of these rows and sequences
        if (blockIdx.x == 0 && tid == 0) a.hdr->status = DPPF_ERR_WORKSPACE;
        return;
    }
    const unsigned smem = (smem_addr(smem_raw) + 1023) & ~1023u, s_q = smem, s_kv = smem + 2 * kTileBytes, s_out = s_kv + 2 * kStages * kTileBytes;
    const Waits wait{&s_dead, a.spin};
    if (tid == 0) {
        for (int s = 0; s < 2; ++s) {
            for (unsigned long long *bar : {&q_full[s], &q_free[s], &s_full[s], &o_full[s]}) mbar_init(bar, 1);
            for (unsigned long long *bar : {&p_half[s], &p_full[s], &o_free[s]}) mbar_init(bar, 128);
        }
        for (int i = 0; i < kStages; ++i)
            for (unsigned long long *bar : {&k_full[i], &v_full[i], &v_ready[i], &empty[i]}) mbar_init(bar, 1);
        mbar_init(&drained, 1);
        s_dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) tmem_alloc(&s_tmem, kColumns);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = uniform(s_tmem);                               // scores of slot s at 128 s, its output at 256 + 128 s

    // Phases are counted on from item to item: q_full, q_free, o_full, o_free by the slot's items, s_full, p_half, p_full by its tiles of keys,
    // the stages by all tiles of keys.
    if (warp >= 8) {
        give_registers<kControlRegisters>();
        if (warp == 8) {
            // ---- copies
            unsigned pairs = 0, items[2] = {0, 0};
            bool ok = true;
            for (ForwardItems all(a); ok && all.there();) {
                const ForwardItem it = all.take(a);
                if (it.idle()) continue;
                if (elect()) {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
                        if (ok && s < it.slots) ok = items[s] == 0 || wait(&q_free[s], (items[s] - 1) & 1);
                    for (int j = it.first; ok && j < it.last; ++j) {
                        const unsigned st = pairs % kStages;
                        ok = pairs < kStages || wait(&empty[st], (pairs / kStages - 1) & 1);
                        if (!ok) break;
                        auto query = [&](int s) {
                            mbar_expect_tx(&q_full[s], kTileBytes);
                            tile_load<kBlocks>(s_q + s * kTileBytes, &a.q, it.head(s), it.row(s), &q_full[s]);
                            ++items[s];
                        };
                        if (j == it.first) query(0);
                        mbar_expect_tx(&k_full[st], kTileBytes);
                        tile_load<kBlocks>(s_kv + 2 * st * kTileBytes, &a.k, it.kv_head, it.key0(j), &k_full[st]);
                        if (j == it.first && it.slots == 2) query(1);
                        mbar_expect_tx(&v_full[st], kTileBytes);
                        tile_load<kBlocks>(s_kv + (2 * st + 1) * kTileBytes, &a.v, it.kv_head, it.key0(j), &v_full[st]);
                        ++pairs;
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
            }
            if (elect()) {                                               // the copies in flight land before the block leaves
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (items[s]) mbar_wait_bounded(&q_full[s], (items[s] - 1) & 1, kSpinLimit);
                for (unsigned i = pairs > kStages ? pairs - kStages : 0; i < pairs; ++i) {
                    mbar_wait_bounded(&k_full[i % kStages], (i / kStages) & 1, kSpinLimit);
                    mbar_wait_bounded(&v_full[i % kStages], (i / kStages) & 1, kSpinLimit);
                }
            }
        } else if (warp == 9) {
            // ---- products: of one slot the probabilities times the values of tile j, then the scores of tile j + 1; then of the other
            const bool leader = elect();
            unsigned pairs = 0, item_phase = 0, tile_phase = 0, later = 0;          // bit s: of slot s; later: the slot had an item before
            bool ok = true;
            for (ForwardItems all(a); ok && all.there();) {
                const ForwardItem it = all.take(a);
                if (it.idle()) continue;
                const int slots = it.slots, lo0 = it.lo[0], hi0 = it.hi[0], lo1 = it.lo[1], hi1 = it.hi[1], lo = it.first, hi = it.last;
                ok = wait.together(&q_full[0], item_phase & 1) && (slots == 1 || wait.together(&q_full[1], item_phase >> 1 & 1));
                for (int j = lo - 1; ok && j < hi; ++j) {
                    const unsigned n = pairs + (unsigned)(j - lo), st = n % kStages, to = (n + 1) % kStages;     // n is used from j = lo on
                    const unsigned tile = s_kv + (2 * st + 1) * kTileBytes;
                    ok = (j < lo || wait.together(&v_ready[st], (n / kStages) & 1)) && (j + 1 >= hi || wait.together(&k_full[to], ((n + 1) / kStages) & 1));
#pragma unroll 1
                    for (int s = 0; ok && s < slots; ++s) {
                        const int first = s ? lo1 : lo0, end = s ? hi1 : hi0;
                        const unsigned S = tmem + s * 128, O = tmem + 256 + s * 128;
                        if (j >= first && j < end) {
                            ok = wait.together(&p_half[s], tile_phase >> s & 1) && (j > first || !(later >> s & 1) || wait.together(&o_free[s], (item_phase >> s & 1) ^ 1));
                            if (!ok) break;
                            tmem_fence_after();
                            if (leader) product_columns<kSteps>(O, S, tile, 0, j > first);
                            ok = wait.together(&p_full[s], tile_phase >> s & 1);
                            if (!ok) break;
                            tmem_fence_after();
                            if (leader) {
                                product_columns<kSteps>(O, S + 32, tile, 1, true);
                                if (j + 1 == end) products_done(&o_full[s]);
                            }
                            tile_phase ^= 1u << s;
                        }
                        if (j >= lo && s + 1 == slots && leader) products_done(&empty[st]);
                        if (j + 1 >= first && j + 1 < end && leader) {
                            product_rows<kSteps>(S, s_q + s * kTileBytes, s_kv + 2 * to * kTileBytes);
                            products_done(&s_full[s]);
                            if (j + 2 == end) products_done(&q_free[s]);
                        }
                    }
                }
                pairs += (unsigned)(hi - lo);
                item_phase ^= slots == 2 ? 3u : 1u;
                later |= slots == 2 ? 3u : 1u;
            }
            if (leader) {                                               // nothing is in flight when the block leaves
                products_done(&drained);
                mbar_wait_bounded(&drained, 0, kSpinLimit);
            }
        } else if (warp == 10) {
            // ---- values as they arrive: rows of other sequences must not reach a sum.  Every tile passes here, so that the warp cannot be
            // a phase behind.
            unsigned pairs = 0;
            bool ok = true;
            for (ForwardItems all(a); ok && all.there();) {
                const ForwardItem it = all.take(a);
                if (it.idle()) continue;
                for (int j = it.first; j < it.last; ++j, ++pairs) {
                    const unsigned st = pairs % kStages;
                    if (!(ok = wait.together(&v_full[st], (pairs / kStages) & 1))) break;
                    const int there = it.t.end - it.key0(j);
                    if (there < kTile) zero_rows<kBlocks>(s_kv + (2 * st + 1) * kTileBytes, there);
                    if (lane == 0) mbar_arrive(&v_ready[st]);
                }
            }
        }
    } else {
        // ---- softmax: a row a thread
        take_registers<kSoftmaxRegisters>();
        const int s = warp >> 2, r = tid & 127;
        const unsigned lanes = (unsigned)(warp & 3) << 21, S = tmem + lanes + s * 128, O = tmem + lanes + 256 + s * 128;
        unsigned items = 0, tiles = 0;
        bool ok = true;
        for (ForwardItems all(a); all.there();) {
            const ForwardItem it = all.take(a);
            const PlanTile &t = it.t;
            if (it.idle()) {
                for (int h = 0; h < (it.by_head ? 2 : 1); ++h) {
                    fill_rows(a.out + (long long)t.row * a.ld_out + (it.head0 + h) * a.head_out, a.ld_out, t.rows, a.D, 0.f, tid, 256);
                    for (int i = tid; i < t.rows; i += 256) a.lse[(it.head0 + h) * a.T + t.row + i] = -INFINITY;
                }
                continue;
            }
            if (s >= it.slots) continue;
            const int slot_row = it.row(s), row = slot_row + r, first = s ? it.lo[1] : it.lo[0], last = s ? it.hi[1] : it.hi[0];
            const bool mine = r < it.rows(s);
            // keys [see_lo, see_hi) of this row
            const int see_lo = a.window ? max(t.begin, row - a.window + 1) : t.begin, see_hi = a.causal ? min(t.end, row + 1) : t.end;
            float top = -INFINITY, sum = 0.f;                            // of the scaled scores, in powers of two
            for (int j = first; ok && j < last; ++j, ++tiles) {
                ok = wait.together(&s_full[s], tiles & 1);
                if (!ok) break;
                tmem_fence_after();
                float v[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_load32(S + c * 32, v[c]);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_loaded(v[c]);
                const int key0 = it.key0(j);
                // blocks that every row of the tile sees whole need no masks
                const bool whole = (a.causal ? slot_row + 1 : t.end) >= key0 + kTile && (!a.window || slot_row + kTile - a.window <= key0) && key0 + kTile <= t.end;
                if (!whole) {
                    const int from = see_lo - key0, to = see_hi - key0;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c * 32 + i < from || c * 32 + i >= to) v[c][i] = -INFINITY;
                }
                unsigned p[2][16];
                auto exponentials = [&](int c, float2 &sums, unsigned (&to)[16], float &high) {      // of 32 columns
                    const float2 by = both(a.scale2), off = both(top == -INFINITY ? 0.f : -top);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float2 e = fma2(make_float2(v[c][2 * i], v[c][2 * i + 1]), by, off);
                        if (i % kPolynomial == 3) { high = max3(high, e.x, e.y); e = exp2_polynomial(e); }
                        else { e.x = exp2_fast(e.x); e.y = exp2_fast(e.y); }
                        sums = add2(sums, e);
                        to[i] = bf16_pair(e.x, e.y);
                    }
                };
                // The sums stay relative to the maximum of the first tile until an exponential would be above kRise, which is rare: fp32 and
                // bf16 keep their relative precision up to 2^127, and the sum of the values, up to kRise times the keys times the largest
                // of them, stays below that for values of up to 2^107 / keys.  (At 2^60 in place of 2^20 that was 2^67 / keys; the times are
                // the same.)  So no maximum is taken of what the first half's sum tells: it is at least the largest of them.  (A polynomial's
                // argument above 127.5 would come out as any number: those are looked at.)
                float2 sums = make_float2(0.f, 0.f);
                float high = -INFINITY;                                      // of the second half, and of the first's polynomials
                if (j > first) {
                    exponentials(0, sums, p[0], high);
                    exponentials(1, sums, p[1], high);
                }
                float m[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 32; i += 2)
#pragma unroll
                    for (int c = 0; c < 2; ++c) m[c] = max3(m[c], v[c + 2][i], v[c + 2][i + 1]);
                const float most = fmaxf(m[0], m[1]) * a.scale2;
                const bool grow = top == -INFINITY || sums.x + sums.y > kRise || fmaxf(high, most - top) > kRiseLog2;
                if (j == first || __any_sync(0xffffffffu, grow)) {
#pragma unroll
                    for (int i = 0; i < 32; i += 2)
#pragma unroll
                        for (int c = 0; c < 2; ++c) m[c] = max3(m[c], v[c][i], v[c][i + 1]);
                    // a row that does not ask for it keeps its own: no row's bits depend on another's
                    const float now = j == first || grow ? fmaxf(m[0], m[1]) * a.scale2 : -INFINITY;
                    if (j > first) {
                        const float f = now > top ? exp2_fast(top - now) : 1.0f;
                        sum *= f;
                        for (int c = 0; c < 4 * kBlocks; ++c) {
                            float o[16];
                            unsigned u[16];
                            tmem_load16(O + c * 16, o);
#pragma unroll
                            for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(o[i] * f);
                            tmem_store16(O + c * 16, u);
                        }
                    }
                    top = fmaxf(top, now);
                    sums = make_float2(0.f, 0.f);
                    exponentials(0, sums, p[0], high);
                    exponentials(1, sums, p[1], high);
                }
                tmem_store16(S, p[0]);
                tmem_store16(S + 16, p[1]);
                tmem_stored();
                tmem_fence_before();
                mbar_arrive(&p_half[s]);
                exponentials(2, sums, p[0], high);
                tmem_store16(S + 32, p[0]);
                exponentials(3, sums, p[1], high);
                tmem_store16(S + 48, p[1]);
                sum += sums.x + sums.y;
                tmem_stored();
                tmem_fence_before();
                mbar_arrive(&p_full[s]);
            }
            ok = ok && wait.together(&o_full[s], items & 1);
            ++items;
            tmem_fence_after();
            bf16 *out = a.out + (long long)slot_row * a.ld_out + it.head(s) * a.head_out;
            if (mine) a.lse[it.head(s) * a.T + row] = ok ? (top + log2f(sum)) * kLn2 : __int_as_float(0x7fc00000);
            if (!ok) {                                                   // this item's rows and those of all that follow
                if (mine) spoil_row(out + r * a.ld_out, a.D);
                continue;
            }
            const float by = sum > 0.f || sum != sum ? 1.0f / sum : 0.f;
            float o[2 * kBlocks][32];
#pragma unroll
            for (int c = 0; c < 2 * kBlocks; ++c) tmem_load32(O + c * 32, o[c]);
#pragma unroll
            for (int c = 0; c < 2 * kBlocks; ++c) tmem_loaded(o[c]);
            tmem_fence_before();
            mbar_arrive(&o_free[s]);
            const unsigned tile = s_out + s * kBlockBytes;               // 64 columns at a time
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) {
                put_row(tile, r, 0, o[2 * c], by);
                put_row(tile, r, 1, o[2 * c + 1], by);
                store_rows<8>(tile, r & ~31, 0, out + 64 * c, a.ld_out, it.rows(s), a.D - 64 * c);
                __syncwarp();
            }
        }
        tmem_fence_before();
    }
    __syncthreads();
    tmem_fence_after();
    if (warp == 9) tmem_free(tmem, kColumns);
    if (tid == 0 && s_dead) a.hdr->status = DPPF_ERR_TIMEOUT;
}

// ---------------------------------------------------------------- gradient
//   P = exp(S - lse);  D_i = do_i . o_i;  dP = do v^T;  dS = P (dP - D);  dq = scale dS k;  dk = scale dS^T q;  dv = P^T do
// Two kernels, each of which forms S and dP anew: one goes over the keys for a tile of queries (D and dq), one over the queries and the heads
// that share a key head for a tile of keys (dk, dv).  Seven products in place of the five that a single kernel needs, whose
// sums of dq would be additions in memory by many blocks, in another order each time; here every sum has one owner and one order.

struct AttentionGradArgs {
    CUtensorMap q, k, v, grad_out, out;
    PlanHeader *hdr;
    const PlanTile *query_tiles, *key_tiles;
    const float *lse;
    float *delta;                // [heads][T]
    bf16 *dq, *dk, *dv;
    long long ld_dq, head_dq, ld_dk, head_dk, ld_dv, head_dv, T;
    float *part;                 // [splits][2][kv_heads][T][D]: dv and dk (without scale) of a part of the heads that share a key head
    int heads, kv_heads, share, splits, D, B;
    int causal, window;
    float scale, scale2;
    int spin_query, spin;        // polls of a wait in the kernel over the keys, for a tile of queries, and in the other
};

constexpr int kGradThreads = 384;          // two warpgroups that halve a tile's columns, one of copies and products

// Sixteen pairs of 32 values as bf16.
__device__ __forceinline__ void put_pairs(unsigned at, const float (&v)[32]) {
    unsigned u[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    tmem_store16(at, u);
}

// v = 2^(v by + off(i)) for pairs i; a third of them by polynomial.
template <typename Off>
__device__ __forceinline__ void probabilities(float (&v)[32], float2 by, Off off) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float2 e = fma2(make_float2(v[2 * i], v[2 * i + 1]), by, off(i));
        if (i % 3 == 2) e = exp2_polynomial(e);
        else { e.x = exp2_fast(e.x); e.y = exp2_fast(e.y); }
        v[2 * i] = e.x;
        v[2 * i + 1] = e.y;
    }
}
// v *= d + off(i) for pairs i
template <typename Off>
__device__ __forceinline__ void times_difference(float (&v)[32], const float (&d)[32], Off off) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float2 e = mul2(make_float2(v[2 * i], v[2 * i + 1]), add2(make_float2(d[2 * i], d[2 * i + 1]), off(i)));
        v[2 * i] = e.x;
        v[2 * i + 1] = e.y;
    }
}

template <int kSteps>
struct QueryGradShape {
    static constexpr int kBlocks = (kSteps + 3) / 4;
    static constexpr bool kApart = kSteps <= 6;              // dS has a place of its own in tensor memory
    static constexpr int kKeys = 3, kValues = 2;             // stages: a tile of keys is needed until dq has it, one of values until dP has it
    static constexpr unsigned kSmem = (2 + kKeys + kValues) * kBlocks * kBlockBytes + 1024;
};

// dq of a tile of queries, and D.  The tile's queries and grad_out lie in tensor memory, too: with both operands of a product in shared
// memory its reads take all of that memory's bandwidth, and the copies' writes come on top.  A thread takes half a row of scores to registers at
// once, so that the products of the next tile of keys can replace them while it takes the exponentials.  With heads of up to 96 there is room
// for dS beside dP, and the next dP comes as early; else it waits for the products with dS, whose place it takes.
template <int kSteps>
__global__ void __launch_bounds__(kGradThreads, 1) attention_grad_query_kernel(const __grid_constant__ AttentionGradArgs a) {
    using Shape = QueryGradShape<kSteps>;
    constexpr int kBlocks = Shape::kBlocks;
    constexpr int kKeys = Shape::kKeys, kValues = Shape::kValues, kColumns = 512;
    constexpr bool kApart = Shape::kApart;
    constexpr unsigned kTileBytes = kBlocks * kBlockBytes;
    extern __shared__ unsigned char smem_raw[];
    __shared__ unsigned long long q_full, o_read, rows_ready, k_full[kKeys], k_empty[kKeys], v_full[kValues], v_empty[kValues], s_full, s_free, dp_full, dp_free, ds_full, o_full, k_fixed, drained;
    __shared__ float s_delta[kTile];
    __shared__ unsigned s_tmem;
    __shared__ volatile int s_dead;
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    const int head = (int)(blockIdx.x % a.heads), kv_head = head / a.share;
    const unsigned index = blockIdx.x / a.heads;
    if (tid < 5) prefetch_map(tid == 0 ? &a.q : tid == 1 ? &a.grad_out : tid == 2 ? &a.k : tid == 3 ? &a.out : &a.v);
    if (!is_plan(a.hdr, a.T, a.B)) {
        if (blockIdx.x == 0 && tid == 0) a.hdr->status = DPPF_ERR_WORKSPACE;
        return;
    }
    if (index >= (unsigned)a.hdr->tiles[kByQuery]) return;
    const PlanTile t = uniform(a.query_tiles[index]);
    if (t.begin == t.end) {
        fill_rows(a.dq + (long long)t.row * a.ld_dq + head * a.head_dq, a.ld_dq, t.rows, a.D, 0.f, tid, kGradThreads);
        return;
    }
    const int lo = a.window ? max(0, t.row - a.window + 1 - t.begin) / kTile : 0;
    const int hi = ((a.causal ? min(t.end, t.row + kTile) : t.end) - t.begin + kTile - 1) / kTile, n = hi - lo;
    const unsigned smem = (smem_addr(smem_raw) + 1023) & ~1023u, s_q = smem, s_do = s_q + kTileBytes, s_k = s_do + kTileBytes, s_v = s_k + kKeys * kTileBytes, s_out = s_k + (kKeys - 1) * kTileBytes;   // the tile's output where the third tile of keys will be
    const Waits wait{&s_dead, a.spin_query};

    if (tid == 0) {
        for (unsigned long long *bar : {&q_full, &s_full, &dp_full, &o_full, &k_fixed, &drained}) mbar_init(bar, 1);
        for (unsigned long long *bar : {&rows_ready, &s_free, &dp_free, &ds_full}) mbar_init(bar, 256);
        mbar_init(&o_read, 128);
        for (int i = 0; i < kKeys; ++i) { mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 1); }
        for (int i = 0; i < kValues; ++i) { mbar_init(&v_full[i], 1); mbar_init(&v_empty[i], 1); }
        s_dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) tmem_alloc(&s_tmem, kColumns);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = uniform(s_tmem), DP = tmem + 128, DQ = tmem + 256, Q = DQ + 16 * kSteps, DO = Q + 8 * kSteps;      // scores at 0
    const unsigned DS = kApart ? tmem + 448 : DP;                        // a half of 64 columns as pairs in 32: side by side, or in front of what it comes from
    constexpr int kHalf = kApart ? 32 : 64;

    const int there = t.end - (t.begin + (hi - 1) * kTile);              // rows of the last tile that are the sequence's
    if (warp == 8) {
        int keys = 0, values = 0;
        if (elect()) {
            mbar_expect_tx(&q_full, 3 * kTileBytes);
            tile_load<kBlocks>(s_q, &a.q, head, t.row, &q_full);
            tile_load<kBlocks>(s_do, &a.grad_out, head, t.row, &q_full);
            tile_load<kBlocks>(s_out, &a.out, head, t.row, &q_full);
            for (int j = 0; j < n; ++j) {
                const int sk = j % kKeys, sv = j % kValues, row = t.begin + (lo + j) * kTile;
                if (j == kKeys - 1 && !wait(&o_read, 0)) break;
                if (j >= kKeys && !wait(&k_empty[sk], (j / kKeys - 1) & 1)) break;
                mbar_expect_tx(&k_full[sk], kTileBytes);
                tile_load<kBlocks>(s_k + sk * kTileBytes, &a.k, kv_head, row, &k_full[sk]);
                ++keys;
                if (j >= kValues && !wait(&v_empty[sv], (j / kValues - 1) & 1)) break;
                mbar_expect_tx(&v_full[sv], kTileBytes);
                tile_load<kBlocks>(s_v + sv * kTileBytes, &a.v, kv_head, row, &v_full[sv]);
                ++values;
            }
        }
        keys = __reduce_max_sync(0xffffffffu, keys);                     // the elected lane's
        values = __reduce_max_sync(0xffffffffu, values);
        if (there < kTile && keys == n) {                                // keys of other sequences must not reach a sum
            const int st = (n - 1) % kKeys;
            if (wait.together(&k_full[st], ((n - 1) / kKeys) & 1)) zero_rows<kBlocks>(s_k + st * kTileBytes, there);
            if (lane == 0) mbar_arrive(&k_fixed);
        }
        if (lane == 0) {                                                 // the copies in flight land before the block leaves
            mbar_wait_bounded(&q_full, 0, kSpinLimit);
            for (int i = max(0, keys - kKeys); i < keys; ++i) mbar_wait_bounded(&k_full[i % kKeys], (i / kKeys) & 1, kSpinLimit);
            for (int i = max(0, values - kValues); i < values; ++i) mbar_wait_bounded(&v_full[i % kValues], (i / kValues) & 1, kSpinLimit);
        }
    } else if (warp == 9) {
        // A wait behind products that were just issued returns when they have begun, and what it holds up leaves the tensor cores idle
        // for some 200 cycles: so the waits stand together, in front of the scores, and only that for dS lies between the products.
        auto arrived = [&](int j) { return wait.together(&k_full[j % kKeys], (j / kKeys) & 1) && wait.together(&v_full[j % kValues], (j / kValues) & 1); };
        auto scores = [&](int j) {
            product_rows_tmem<kSteps>(tmem, Q, s_k + j % kKeys * kTileBytes);
            products_done(&s_full);
        };
        auto dps = [&](int j) {
            product_rows_tmem<kSteps>(DP, DO, s_v + j % kValues * kTileBytes);
            products_done(&dp_full);
            products_done(&v_empty[j % kValues]);
        };
        bool ok = wait.together(&rows_ready, 0) && arrived(0);
        tmem_fence_after();
        if (ok && elect()) { scores(0); dps(0); }
        for (int j = 0; ok && j < n; ++j) {
            const bool more = j + 1 < n;
            ok = more ? arrived(j + 1) && wait.together(&s_free, j & 1) : there >= kTile || wait.together(&k_fixed, 0);
            if (!ok) break;
            tmem_fence_after();
            if (more && elect()) scores(j + 1);
            if (kApart && more) {
                ok = wait.together(&dp_free, j & 1);
                if (!ok) break;
                tmem_fence_after();
                if (elect()) dps(j + 1);
            }
            ok = wait.together(&ds_full, j & 1);
            if (!ok) break;
            tmem_fence_after();
            if (elect()) {
                product_columns<kSteps>(DQ, DS, s_k + j % kKeys * kTileBytes, 0, j > 0);
                product_columns<kSteps>(DQ, DS + kHalf, s_k + j % kKeys * kTileBytes, 1, true);
                if (!kApart && more) dps(j + 1);
                products_done(&k_empty[j % kKeys]);
                if (!more) products_done(&o_full);
            }
        }
        if (elect()) {
            products_done(&drained);
            mbar_wait_bounded(&drained, 0, kSpinLimit);
        }
    } else if (warp < 8) {
        const int half = warp >> 2, r = tid & 127, row = t.row + r;
        const bool mine = r < t.rows;
        const unsigned lanes = (unsigned)(warp & 3) << 21;
        // queries and grad_out go on to tensor memory, a row a thread, one of them a warpgroup; that of grad_out forms D
        const float lse2 = mine ? a.lse[head * a.T + row] * kLog2e : 0.f;
        bool ok = wait.together(&q_full, 0);
        float delta = 0.f;
#pragma unroll
        for (int c = 0; c < kSteps / 2; ++c) {
            unsigned u[16];
            tile_row(half ? s_do : s_q, r, c, u);
            tmem_store16((half ? DO : Q) + lanes + 16 * c, u);
            if (half) {
                unsigned o[16];
                tile_row(s_out, r, c, o);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    delta = fmaf(bf16_low(o[i]), bf16_low(u[i]), delta);
                    delta = fmaf(bf16_high(o[i]), bf16_high(u[i]), delta);
                }
            }
        }
        if (half) mbar_arrive(&o_read);
        tmem_stored();
        tmem_fence_before();
        mbar_arrive(&rows_ready);
        if (half) {
            if (!ok) delta = __int_as_float(0x7fc00000);                 // of tiles that did not come: the other kernel must not take it for D
            s_delta[r] = delta;
            if (mine) a.delta[head * a.T + row] = delta;
        }
        group_sync(1, 256);
        delta = s_delta[r];
        const int see_lo = a.window ? max(t.begin, row - a.window + 1) : t.begin, see_hi = a.causal ? min(t.end, row + 1) : t.end;
        for (int j = 0; ok && j < n; ++j) {
            const int key0 = t.begin + (lo + j) * kTile + 64 * half;
            const bool whole = (a.causal ? t.row + 1 : t.end) >= key0 + 64 && (!a.window || t.row + kTile - a.window <= key0) && key0 + 64 <= t.end;
            const int from = see_lo - key0, to = see_hi - key0;
            ok = wait.together(&s_full, j & 1);
            if (!ok) break;
            tmem_fence_after();
            float p[2][32], d[32];
#pragma unroll
            for (int c = 0; c < 2; ++c) tmem_load32(tmem + lanes + 64 * half + 32 * c, p[c]);
#pragma unroll
            for (int c = 0; c < 2; ++c) tmem_loaded(p[c]);
            tmem_fence_before();
            mbar_arrive(&s_free);
#pragma unroll
            for (int c = 0; c < 2; ++c) probabilities(p[c], both(a.scale2), [&](int) { return both(-lse2); });
            ok = wait.together(&dp_full, j & 1);
            if (!ok) break;
            tmem_fence_after();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                tmem_load32(DP + lanes + 64 * half + 32 * c, d);
                tmem_loaded(d);
                if (kApart && c) {
                    tmem_fence_before();
                    mbar_arrive(&dp_free);
                }
                times_difference(p[c], d, [&](int) { return both(-delta); });
            }
            if (!whole)                                                  // a select: what is masked may be NaN
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c * 32 + i < from || c * 32 + i >= to) p[c][i] = 0.f;
            if (kApart && j > 0) {                                       // the products with the dS before are done
                ok = wait.together(&k_empty[(j - 1) % kKeys], ((j - 1) / kKeys) & 1);
                if (!ok) break;
                tmem_fence_after();
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) put_pairs(DS + lanes + kHalf * half + 16 * c, p[c]);
            tmem_stored();
            tmem_fence_before();
            mbar_arrive(&ds_full);
        }
        ok = ok && wait.together(&o_full, 0);
        tmem_fence_after();
        bf16 *dq = a.dq + (long long)t.row * a.ld_dq + head * a.head_dq;
        if (ok) {
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) {
                float o[32];
                tmem_load32(DQ + lanes + (half * kBlocks + c) * 32, o);
                tmem_loaded(o);
                put_row(s_q, r, half * kBlocks + c, o, a.scale);
            }
            store_rows<4 * kBlocks>(s_q, r & ~31, half * 4 * kBlocks, dq, a.ld_dq, t.rows, a.D);
        } else if (mine) {
            spoil_row(dq + r * a.ld_dq, a.D);
        }
        tmem_fence_before();
    }
    __syncthreads();
    tmem_fence_after();
    if (warp == 9) tmem_free(tmem, kColumns);
    if (tid == 0 && s_dead) a.hdr->status = DPPF_ERR_TIMEOUT;
}

template <int kSteps>
struct KeyGradShape {
    static constexpr int kBlocks = (kSteps + 3) / 4;
    static constexpr bool kApart = kSteps <= 6;              // the probabilities have a place of their own in tensor memory
    static constexpr int kQueries = 3, kOuts = 2;            // stages: a tile of queries is asked for before the one before it is done with
    static constexpr unsigned kTiles = (2 + kQueries + kOuts) * kBlocks * kBlockBytes;
    static constexpr unsigned kSmem = kTiles + 2 * 2 * kTile * 4;        // and lse and D of two tiles of queries
};

// dk and dv of a tile of keys: a row of the transposed scores is a key.  Scores and dP take turns: while the exponentials of one
// tile are taken, the tensor cores form dk and dP, and dv and the next scores while dS is.  With heads of up to 96 there is room for
// the probabilities beside the scores, and the next scores come as soon as a thread has its half row in registers.
template <int kSteps>
__global__ void __launch_bounds__(kGradThreads, 1) attention_grad_key_kernel(const __grid_constant__ AttentionGradArgs a) {
    using Shape = KeyGradShape<kSteps>;
    constexpr int kBlocks = Shape::kBlocks;
    constexpr int kQueries = Shape::kQueries, kOuts = Shape::kOuts, kColumns = 512;
    constexpr bool kApart = Shape::kApart;
    constexpr unsigned kTileBytes = kBlocks * kBlockBytes;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ unsigned long long kv_full, q_full[kQueries], q_ready[kQueries], q_empty[kQueries], do_full[kOuts], do_ready[kOuts], do_empty[kOuts], stat_full[2], s_full, s_free, dp_full, p_full, ds_full, o_full, drained;
    __shared__ unsigned s_tmem;
    __shared__ volatile int s_dead;
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    const int unit = (int)(blockIdx.x % (a.kv_heads * a.splits)), kv_head = unit / a.splits, split = unit % a.splits;
    const unsigned index = blockIdx.x / (a.kv_heads * a.splits);
    if (tid < 4) prefetch_map(tid == 0 ? &a.k : tid == 1 ? &a.q : tid == 2 ? &a.v : &a.grad_out);
    if (!is_plan(a.hdr, a.T, a.B) || index >= (unsigned)a.hdr->tiles[kByKey]) return;      // the status is the first kernel's
    const PlanTile t = uniform(a.key_tiles[index]);
    auto part_row = [&](int which, int row) { return a.part + (((long long)(split * 2 + which) * a.kv_heads + kv_head) * a.T + row) * a.D; };
    if (t.begin == t.end) {
        if (a.splits > 1) {
            for (int which = 0; which < 2; ++which)
                for (int i = tid; i < t.rows * a.D; i += kGradThreads) part_row(which, t.row)[i] = 0.f;
            return;
        }
        fill_rows(a.dk + (long long)t.row * a.ld_dk + kv_head * a.head_dk, a.ld_dk, t.rows, a.D, 0.f, tid, kGradThreads);
        fill_rows(a.dv + (long long)t.row * a.ld_dv + kv_head * a.head_dv, a.ld_dv, t.rows, a.D, 0.f, tid, kGradThreads);
        return;
    }
    // blocks of queries [lo, hi) that see any of these keys, of each head in turn
    const int lo = a.causal ? (t.row - t.begin) / kTile : 0;
    const int hi = ((a.window ? (int)min((long long)t.end, (long long)t.row + t.rows - 1 + a.window) : t.end) - t.begin + kTile - 1) / kTile;
    const int head0 = kv_head * a.share + split * a.share / a.splits, heads = kv_head * a.share + (split + 1) * a.share / a.splits - head0;
    const int each = hi - lo, n = each * heads;
    const unsigned s_k = smem_addr(smem_raw), s_v = s_k + kTileBytes, s_q = s_v + kTileBytes, s_do = s_q + kQueries * kTileBytes;
    float (*s_stat)[2][kTile] = reinterpret_cast<float (*)[2][kTile]>(smem_raw + Shape::kTiles);      // lse in powers of two, and D, of a tile of queries
    const Waits wait{&s_dead, a.spin};

    if (tid == 0) {
        for (unsigned long long *bar : {&kv_full, &s_full, &dp_full, &o_full, &drained}) mbar_init(bar, 1);
        mbar_init(&p_full, 256);
        mbar_init(&s_free, 256);
        mbar_init(&ds_full, 256);
        for (int i = 0; i < kQueries; ++i) { mbar_init(&q_full[i], 1); mbar_init(&q_ready[i], 1); mbar_init(&q_empty[i], 1); }
        for (int i = 0; i < kOuts; ++i) { mbar_init(&do_full[i], 1); mbar_init(&do_ready[i], 1); mbar_init(&do_empty[i], 1); mbar_init(&stat_full[i], 32); }
        s_dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) tmem_alloc(&s_tmem, kColumns);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = uniform(s_tmem), DP = tmem + 128, DV = tmem + 256, DK = DV + 16 * kSteps;     // scores at 0
    const unsigned P = kApart ? tmem + 448 : tmem;                       // a half of 64 columns as pairs in 32
    constexpr int kHalf = kApart ? 32 : 64;

    auto head_of = [&](int i) { return head0 + i / each; };
    auto row_of = [&](int i) { return t.begin + (lo + i % each) * kTile; };
    if (warp == 8) {
        // ---- copies
        if (elect()) {
            int queries = 0, outs = 0;
            mbar_expect_tx(&kv_full, 2 * kTileBytes);
            tile_load<kBlocks>(s_k, &a.k, kv_head, t.row, &kv_full);
            tile_load<kBlocks>(s_v, &a.v, kv_head, t.row, &kv_full);
            for (int i = 0; i < n; ++i) {
                const int sq = i % kQueries, so = i % kOuts, head = head_of(i), row = row_of(i);
                if (i >= kQueries && !wait(&q_empty[sq], (i / kQueries - 1) & 1)) break;
                mbar_expect_tx(&q_full[sq], kTileBytes);
                tile_load<kBlocks>(s_q + sq * kTileBytes, &a.q, head, row, &q_full[sq]);
                ++queries;
                if (i >= kOuts && !wait(&do_empty[so], (i / kOuts - 1) & 1)) break;
                mbar_expect_tx(&do_full[so], kTileBytes);
                tile_load<kBlocks>(s_do + so * kTileBytes, &a.grad_out, head, row, &do_full[so]);
                ++outs;
            }
            mbar_wait_bounded(&kv_full, 0, kSpinLimit);                  // the copies in flight land before the block leaves
            for (int i = max(0, queries - kQueries); i < queries; ++i) mbar_wait_bounded(&q_full[i % kQueries], (i / kQueries) & 1, kSpinLimit);
            for (int i = max(0, outs - kOuts); i < outs; ++i) mbar_wait_bounded(&do_full[i % kOuts], (i / kOuts) & 1, kSpinLimit);
        }
    } else if (warp == 9) {
        // ---- products
        auto queries = [&](int i) { return wait.together(&q_ready[i % kQueries], (i / kQueries) & 1); };
        auto outs = [&](int i) { return wait.together(&do_ready[i % kOuts], (i / kOuts) & 1); };
        auto scores = [&](int i) {
            product_rows<kSteps>(tmem, s_k, s_q + i % kQueries * kTileBytes);
            products_done(&s_full);
        };
        auto dps = [&](int i) {
            product_rows<kSteps>(DP, s_v, s_do + i % kOuts * kTileBytes);
            products_done(&dp_full);
        };
        bool ok = wait.together(&kv_full, 0) && queries(0) && outs(0);
        if (ok && elect()) { scores(0); dps(0); }
        for (int i = 0; ok && i < n; ++i) {
            const unsigned tile_do = s_do + i % kOuts * kTileBytes, tile_q = s_q + i % kQueries * kTileBytes;
            const bool more = i + 1 < n;
            ok = !more || queries(i + 1);
            if (kApart && more) {
                ok = ok && wait.together(&s_free, i & 1);
                tmem_fence_after();
                if (ok && elect()) scores(i + 1);
            }
            ok = ok && wait.together(&p_full, i & 1);
            if (!ok) break;
            tmem_fence_after();
            if (elect()) {
                product_columns<kSteps>(DV, P, tile_do, 0, i > 0);
                product_columns<kSteps>(DV, P + kHalf, tile_do, 1, true);
                products_done(&do_empty[i % kOuts]);
                if (!kApart && more) scores(i + 1);
            }
            ok = (!more || outs(i + 1)) && wait.together(&ds_full, i & 1);
            if (!ok) break;
            tmem_fence_after();
            if (elect()) {
                product_columns<kSteps>(DK, DP, tile_q, 0, i > 0);
                product_columns<kSteps>(DK, DP + 64, tile_q, 1, true);
                if (more) dps(i + 1);
                products_done(&q_empty[i % kQueries]);
                if (!more) products_done(&o_full);
            }
        }
        if (elect()) {
            products_done(&drained);
            mbar_wait_bounded(&drained, 0, kSpinLimit);
        }
    } else if (warp >= 10) {
        // ---- tiles as they arrive: rows of other sequences must not reach a sum.  One warp for the queries, one for grad_out and for lse
        // and D, which it reads a tile ahead.  Every tile passes here, so that neither warp can be a phase behind.
        const bool queries = warp == 10;
        const int stages = queries ? kQueries : kOuts;
        float lse[4], delta[4];
        auto read = [&](int i) {
            const int row = row_of(i);
            const long long at = head_of(i) * a.T + row;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bool is = row + lane + 32 * k < t.end;
                lse[k] = is ? __ldcg(a.lse + at + lane + 32 * k) : 0.f;
                delta[k] = is ? __ldcg(a.delta + at + lane + 32 * k) : 0.f;
            }
        };
        if (!queries) read(0);
        bool ok = true;
        for (int i = 0; ok && i < n; ++i) {
            const int st = i % stages, there = t.end - row_of(i);
            if (!queries) {
                // those of two tiles before are done with when its products with dS are
                if (i >= 2 && !(ok = wait.together(&q_empty[(i - 2) % kQueries], ((i - 2) / kQueries) & 1))) break;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    s_stat[i & 1][0][lane + 32 * k] = -kLog2e * lse[k];
                    s_stat[i & 1][1][lane + 32 * k] = -delta[k];
                }
                mbar_arrive(&stat_full[i & 1]);
                if (i + 1 < n) read(i + 1);
            }
            if (!(ok = wait.together(queries ? &q_full[st] : &do_full[st], (i / stages) & 1))) break;
            if (there < kTile) zero_rows<kBlocks>((queries ? s_q : s_do) + st * kTileBytes, there);
            if (lane == 0) mbar_arrive(queries ? &q_ready[st] : &do_ready[st]);
        }
    } else if (warp < 8) {
        const int half = warp >> 2, r = tid & 127, key = t.row + r;
        const unsigned lanes = (unsigned)(warp & 3) << 21;
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int q0 = row_of(i) + 64 * half;
            const bool whole = q0 + 64 <= t.end && (!a.causal || q0 >= t.row + kTile - 1) && (!a.window || q0 + 63 < t.row + a.window);
            const int from = a.causal ? key - q0 : 0, to = (a.window ? (int)min((long long)t.end, (long long)key + a.window) : t.end) - q0;
            ok = wait.together(&s_full, i & 1) && wait.together(&stat_full[i & 1], (i >> 1) & 1);
            if (!ok) break;
            tmem_fence_after();
            float p[2][32], d[32];
#pragma unroll
            for (int c = 0; c < 2; ++c) tmem_load32(tmem + lanes + 64 * half + 32 * c, p[c]);
#pragma unroll
            for (int c = 0; c < 2; ++c) tmem_loaded(p[c]);
            if (kApart) {
                tmem_fence_before();
                mbar_arrive(&s_free);
            }
            const float4 *lse2 = reinterpret_cast<const float4 *>(&s_stat[i & 1][0][64 * half]), *delta = reinterpret_cast<const float4 *>(&s_stat[i & 1][1][64 * half]);
            auto pair_of = [](const float4 *p, int k) { const float4 f = p[k / 2]; return k % 2 ? make_float2(f.z, f.w) : make_float2(f.x, f.y); };
#pragma unroll
            for (int c = 0; c < 2; ++c) probabilities(p[c], both(a.scale2), [&](int k) { return pair_of(lse2, c * 16 + k); });
            if (!whole)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (c * 32 + k < from || c * 32 + k >= to) p[c][k] = 0.f;
            if (kApart && i > 0) {                                       // the products with the probabilities before are done
                ok = wait.together(&do_empty[(i - 1) % kOuts], ((i - 1) / kOuts) & 1);
                if (!ok) break;
                tmem_fence_after();
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) put_pairs(P + lanes + kHalf * half + 16 * c, p[c]);
            tmem_stored();
            tmem_fence_before();
            mbar_arrive(&p_full);
            ok = wait.together(&dp_full, i & 1);
            if (!ok) break;
            tmem_fence_after();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                tmem_load32(DP + lanes + 64 * half + 32 * c, d);
                tmem_loaded(d);
                times_difference(p[c], d, [&](int k) { return pair_of(delta, c * 16 + k); });
            }
            if (!whole)                                                  // a select: what is masked may be NaN
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (c * 32 + k < from || c * 32 + k >= to) p[c][k] = 0.f;
#pragma unroll
            for (int c = 0; c < 2; ++c) put_pairs(DP + lanes + 64 * half + 16 * c, p[c]);
            tmem_stored();
            tmem_fence_before();
            mbar_arrive(&ds_full);
        }
        ok = ok && wait.together(&o_full, 0);
        tmem_fence_after();
        const long long ld = half ? a.ld_dk : a.ld_dv;
        bf16 *to = (half ? a.dk + kv_head * a.head_dk : a.dv + kv_head * a.head_dv) + t.row * ld;
        if (a.splits > 1) {
            float *part = part_row(half, key);
            for (int c = 0; c < 2 * kBlocks; ++c) {
                float o[32];
                if (ok) {
                    tmem_load32((half ? DK : DV) + lanes + c * 32, o);
                    tmem_loaded(o);
                }
                if (r < t.rows)
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        if (c * 32 + i < a.D) *reinterpret_cast<float4 *>(part + c * 32 + i) = ok ? make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]) : make_float4(NAN, NAN, NAN, NAN);
            }
        } else if (ok) {
            const unsigned tile = half ? s_k : s_v;                      // all products are done
#pragma unroll
            for (int c = 0; c < 2 * kBlocks; ++c) {
                float o[32];
                tmem_load32((half ? DK : DV) + lanes + c * 32, o);
                tmem_loaded(o);
                put_row(tile, r, c, o, half ? a.scale : 1.0f);
            }
            store_rows<8 * kBlocks>(tile, r & ~31, 0, to, ld, t.rows, a.D);
        } else if (r < t.rows) {
            spoil_row(to + r * ld, a.D);
        }
        tmem_fence_before();
    }
    __syncthreads();
    tmem_fence_after();
    if (warp == 9) tmem_free(tmem, kColumns);
    if (tid == 0 && s_dead) a.hdr->status = DPPF_ERR_TIMEOUT;
}

// The parts of dk and dv, added in order, eight columns of a row a thread.  blockIdx.y: 0 dv, 1 dk.
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads) attention_grad_join_kernel(const __grid_constant__ AttentionGradArgs a) {
    const int pieces = a.D / 8, which = blockIdx.y;
    const long long rows = a.kv_heads * a.T, i = (long long)blockIdx.x * kJoinThreads + threadIdx.x;
    if (!is_plan(a.hdr, a.T, a.B) || i >= rows * pieces) return;
    const long long at = i / pieces, kv_head = at / a.T, row = at - kv_head * a.T;
    const int piece = (int)(i - at * pieces);
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.f;
    for (int s = 0; s < a.splits; ++s) {
        const float4 *p = reinterpret_cast<const float4 *>(a.part + ((s * 2 + which) * rows + at) * a.D + piece * 8);
        const float4 x = __ldcs(p), y = __ldcs(p + 1);
        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
        v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
    }
    const float by = which ? a.scale : 1.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= by;
    bf16 *to = which ? a.dk + row * a.ld_dk + kv_head * a.head_dk : a.dv + row * a.ld_dv + kv_head * a.head_dv;
    store_vec<bf16, 8>(to + piece * 8, v);
}

}  // namespace
