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
    int T;
};
struct PlanTile { int row, rows, begin, end; };       // first row, rows of this tile; its sequence's rows (begin == end: no sequence)

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
    int list, heads, share, D;   // share: query heads of a key head
    int by_head, units;          // the two slots of a block: two heads of a tile of 128 rows, or the halves of one of 256; blocks of a tile
    int causal, window;          // window 0: none
    float scale, scale2;         // scale * log2 e
    int spin;
};

constexpr int kForwardThreads = 384;       // two warpgroups of a slot each, one of copies and products
template <int kBlocks>
struct ForwardShape {
    static constexpr unsigned kTileBytes = kBlocks * kBlockBytes;
    static constexpr int kStages = kBlocks == 2 ? 4 : 6;                 // of keys and values in turn
    static constexpr unsigned kSmem = (2 + kStages) * kTileBytes + 1024;
};

// Eight bf16 columns a store, those below D, of 32 columns from `at` on.
__device__ __forceinline__ void put_columns(bf16 *row, int at, int D, const float (&v)[32], float by) {
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        if (at + i < D) {
            uint4 u;
            u.x = bf16_pair(v[i] * by, v[i + 1] * by);
            u.y = bf16_pair(v[i + 2] * by, v[i + 3] * by);
            u.z = bf16_pair(v[i + 4] * by, v[i + 5] * by);
            u.w = bf16_pair(v[i + 6] * by, v[i + 7] * by);
            *reinterpret_cast<uint4 *>(row + at + i) = u;
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

// S = scale q k^T over the keys that a query sees; out = softmax(S) v; lse = log sum exp S.
// One pass over the keys with a running maximum and sum.  A block has two slots of 128 queries that share their keys and values:
// while one slot's warpgroup takes the exponentials of its scores (a row a thread), the tensor cores work for the other.
// Scores and output sums stay in tensor memory; the probabilities replace the scores there as bf16, the first operand of the second product.
template <int kBlocks>
__global__ void __launch_bounds__(kForwardThreads, 1) attention_kernel(const __grid_constant__ AttentionArgs a) {
    using Shape = ForwardShape<kBlocks>;
    constexpr int kStages = Shape::kStages;
    constexpr unsigned kTileBytes = Shape::kTileBytes;
    constexpr int kColumns = 512;
    extern __shared__ unsigned char smem_raw[];
    __shared__ unsigned long long q_full[2], kv_full[kStages], kv_empty[kStages], s_full[2], p_full[2], o_full[2], drained;
    __shared__ unsigned s_tmem;
    __shared__ volatile int s_dead;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned unit = blockIdx.x % a.units, index = blockIdx.x / a.units;
    if (a.hdr->magic != kPlanMagic || a.hdr->T != a.T) {                 // not a plan of these rows
        if (blockIdx.x == 0 && tid == 0) a.hdr->status = DPPF_ERR_WORKSPACE;
        return;
    }
    if (index >= (unsigned)a.hdr->tiles[a.list]) return;
    const PlanTile t = a.tiles[index];
    // slots: query rows [row, row + rows) of a head
    const int head0 = a.by_head ? 2 * unit : unit, kv_head = head0 / a.share;
    auto slot_row = [&](int s) { return a.by_head ? t.row : t.row + s * kTile; };
    auto slot_rows = [&](int s) { return a.by_head ? t.rows : min(kTile, t.rows - s * kTile); };
    auto slot_head = [&](int s) { return a.by_head ? head0 + s : head0; };
    if (t.begin == t.end) {                                              // rows of no sequence
        for (int s = 0; s < (a.by_head ? 2 : 1); ++s) {
            fill_rows(a.out + (long long)t.row * a.ld_out + (head0 + s) * a.head_out, a.ld_out, t.rows, a.D, 0.f, tid, kForwardThreads);
            for (int i = tid; i < t.rows; i += kForwardThreads) a.lse[(head0 + s) * a.T + t.row + i] = -INFINITY;
        }
        return;
    }
    // key blocks [lo, hi) of a slot, counted from the sequence's begin; the blocks that both need come in once
    auto block_lo = [&](int s) { return a.window ? max(0, slot_row(s) - a.window + 1 - t.begin) / kTile : 0; };
    auto block_hi = [&](int s) { return slot_rows(s) <= 0 ? 0 : ((a.causal ? min(t.end, slot_row(s) + kTile) : t.end) - t.begin + kTile - 1) / kTile; };
    const int lo0 = block_lo(0), hi0 = block_hi(0), hi1 = block_hi(1), lo1 = hi1 ? block_lo(1) : 0;
    const int lo = hi1 ? min(lo0, lo1) : lo0, hi = max(hi0, hi1);
    const unsigned smem = (smem_addr(smem_raw) + 1023) & ~1023u, s_q = smem, s_kv = smem + 2 * kTileBytes;
    const Waits wait{&s_dead, a.spin};

    if (tid == 0) {
        for (int s = 0; s < 2; ++s) { mbar_init(&q_full[s], 1); mbar_init(&s_full[s], 1); mbar_init(&p_full[s], 128); mbar_init(&o_full[s], 1); }
        for (int i = 0; i < kStages; ++i) { mbar_init(&kv_full[i], 1); mbar_init(&kv_empty[i], 1); }
        mbar_init(&drained, 1);
        s_dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) tmem_alloc(&s_tmem, kColumns);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = s_tmem;                                        // scores of slot s at 128 s, its output at 256 + 128 s

    if (warp == 8) {
        // ---- copies
        if (lane == 0) {
            unsigned issued = 0;
            bool ok = true;
            auto load = [&](const CUtensorMap *map, int block) {
                const unsigned st = issued % kStages;
                ok = ok && (issued < kStages || wait(&kv_empty[st], (issued / kStages - 1) & 1));
                if (!ok) return;
                mbar_expect_tx(&kv_full[st], kTileBytes);
                tile_load<kBlocks>(s_kv + st * kTileBytes, map, kv_head, t.begin + block * kTile, &kv_full[st]);
                ++issued;
            };
            for (int s = 0; s < (hi1 ? 2 : 1); ++s) {
                mbar_expect_tx(&q_full[s], kTileBytes);
                tile_load<kBlocks>(s_q + s * kTileBytes, &a.q, slot_head(s), slot_row(s), &q_full[s]);
                if (s == 0) load(&a.k, lo);
            }
            load(&a.v, lo);
            for (int j = lo + 1; j < hi; ++j) { load(&a.k, j); load(&a.v, j); }
            // the copies in flight land before the block leaves
            for (int s = 0; s < (hi1 ? 2 : 1); ++s) mbar_wait_bounded(&q_full[s], 0, kSpinLimit);
            for (unsigned i = issued > kStages ? issued - kStages : 0; i < issued; ++i) mbar_wait_bounded(&kv_full[i % kStages], (i / kStages) & 1, kSpinLimit);
        }
    } else if (warp == 9) {
        // ---- products, issued by lane 0; the warp waits together
        auto full = [&](int n) { return wait.together(&kv_full[n % kStages], (n / kStages) & 1); };
        auto active = [&](int s, int j) { return s == 0 ? j >= lo0 && j < hi0 : j >= lo1 && j < hi1; };
        auto scores = [&](int s, int j) {
            if (lane == 0) {
                product_rows<kBlocks>(tmem + s * 128, s_q + s * kTileBytes, s_kv + (2 * (j - lo)) % kStages * kTileBytes);
                products_done(&s_full[s]);
            }
        };
        bool ok = wait.together(&q_full[0], 0) && (!hi1 || wait.together(&q_full[1], 0)) && full(0);
        if (ok) {
            for (int s = 0; s < 2; ++s)
                if (active(s, lo)) scores(s, lo);
            if (lane == 0) products_done(&kv_empty[0]);
        }
        for (int j = lo; ok && j < hi; ++j) {
            const int nv = 2 * (j - lo) + 1, nk = nv + 1;
            const unsigned tile = s_kv + nv % kStages * kTileBytes;
            ok = full(nv);
            if (!ok) break;
            const int there = t.end - (t.begin + j * kTile);
            if (there < kTile) zero_rows<kBlocks>(tile, there);
            if (j + 1 < hi && !(ok = full(nk))) break;
            for (int s = 0; s < 2; ++s) {
                if (active(s, j)) {
                    ok = wait.together(&p_full[s], (j - (s ? lo1 : lo0)) & 1);
                    if (!ok) break;
                    tmem_fence_after();
                    if (lane == 0) {
                        product_columns<kBlocks>(tmem + 256 + s * 128, tmem + s * 128, tmem + s * 128 + 32, tile, j > (s ? lo1 : lo0));
                        if (j + 1 == (s ? hi1 : hi0)) products_done(&o_full[s]);
                    }
                }
                if (active(s, j + 1)) scores(s, j + 1);
            }
            if (ok && lane == 0) {
                products_done(&kv_empty[nv % kStages]);
                if (j + 1 < hi) products_done(&kv_empty[nk % kStages]);
            }
        }
        if (lane == 0) {                                                 // nothing is in flight when the block leaves
            products_done(&drained);
            mbar_wait_bounded(&drained, 0, kSpinLimit);
        }
    } else if (warp < 8) {
        // ---- softmax: a row a thread
        const int s = warp >> 2, r = tid & 127, row = slot_row(s) + r;
        const int first = s ? lo1 : lo0, last = s ? hi1 : hi0;
        const unsigned lanes = (unsigned)(warp & 3) << 21, S = tmem + lanes + s * 128, O = tmem + lanes + 256 + s * 128;
        // keys [see_lo, see_hi) of this row
        const int see_lo = a.window ? max(t.begin, row - a.window + 1) : t.begin, see_hi = a.causal ? min(t.end, row + 1) : t.end;
        float top = -INFINITY, sum = 0.f;                                // of the scaled scores, in powers of two
        bool ok = true;
        for (int j = first; j < last; ++j) {
            ok = wait.together(&s_full[s], (j - first) & 1);
            if (!ok) break;
            tmem_fence_after();
            float v[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_load32(S + c * 32, v[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_loaded(v[c]);
            const int key0 = t.begin + j * kTile;
            // blocks that every row of the tile sees whole need no masks
            const bool whole = (a.causal ? slot_row(s) + 1 : t.end) >= key0 + kTile && (!a.window || slot_row(s) + kTile - a.window <= key0) && key0 + kTile <= t.end;
            if (!whole) {
                const int from = see_lo - key0, to = see_hi - key0;
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c * 32 + i < from || c * 32 + i >= to) v[c][i] = -INFINITY;
            }
            float m[4] = {v[0][0], v[1][0], v[2][0], v[3][0]};
#pragma unroll
            for (int i = 1; i < 32; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) m[c] = fmaxf(m[c], v[c][i]);
            const float now = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) * a.scale2;
            // The sums stay relative to an older maximum until one is 2^8 above it: then no exponential is above 2^8, and fp32 sums
            // of bf16 products lose nothing.
            const bool grow = now > top + 8.0f || top == -INFINITY;
            if (j > first && __any_sync(0xffffffffu, grow && now > top)) {
                const float f = grow && now > top ? exp2_fast(top - now) : 1.0f;
                sum *= f;
                for (int c = 0; c < 2 * kBlocks; ++c) {
                    float o[32];
                    tmem_load32(O + c * 32, o);
                    tmem_loaded(o);
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] *= f;
                    tmem_store32(O + c * 32, o);
                }
            }
            if (grow && now > top) top = now;
            const float2 by = both(a.scale2), off = both(top == -INFINITY ? 0.f : -top);
            float2 sums = make_float2(0.f, 0.f);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                unsigned p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float2 e = fma2(make_float2(v[c][2 * i], v[c][2 * i + 1]), by, off);
                    e.x = exp2_fast(e.x);
                    e.y = exp2_fast(e.y);
                    sums = add2(sums, e);
                    p[i] = bf16_pair(e.x, e.y);
                }
                tmem_store16(S + c * 16, p);
            }
            sum += sums.x + sums.y;
            tmem_stored();
            tmem_fence_before();
            mbar_arrive(&p_full[s]);
        }
        if (last > first) {
            ok = ok && wait.together(&o_full[s], 0);
            tmem_fence_after();
            const bool mine = r < slot_rows(s);
            const float by = ok ? (sum > 0.f || sum != sum ? 1.0f / sum : 0.f) : __int_as_float(0x7fc00000);
            bf16 *out = a.out + (long long)row * a.ld_out + slot_head(s) * a.head_out;
            for (int c = 0; c < 2 * kBlocks; ++c) {
                float o[32];
                tmem_load32(O + c * 32, o);
                tmem_loaded(o);
                if (mine) put_columns(out, c * 32, a.D, o, by);
            }
            if (mine) a.lse[slot_head(s) * a.T + row] = ok ? (top + log2f(sum)) * kLn2 : __int_as_float(0x7fc00000);
        }
        tmem_fence_before();
    }
    __syncthreads();
    tmem_fence_after();
    if (warp == 9) tmem_free(tmem, kColumns);
    if (tid == 0 && s_dead) a.hdr->status = DPPF_ERR_TIMEOUT;
}

}  // namespace
