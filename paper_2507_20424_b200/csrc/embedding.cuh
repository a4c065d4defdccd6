// Embedding lookup with a scale, and its gradient by sorted tokens.
#pragma once
#include "local_common.cuh"

namespace {

// ---------------------------------------------------------------- lookup
// out[t] = scale * table[id_t], zeros where id_t is outside [0, V).  One fp32 product, rounded once.
// Bound by the bytes of the distinct rows and of the output.

struct LookupArgs {
    const void *table, *ids;
    void *out;
    long long ld_table, ld_out;   // elements
    long long T, V;
    int groups;                   // groups of N elements in a row (the last may be short)
    int H, ids64;
    unsigned rows_per_block;
    float scale;
};

__device__ __forceinline__ long long read_id(const void *ids, int ids64, long long i) {
    return ids64 ? __ldg(static_cast<const long long *>(ids) + i) : (long long)__ldg(static_cast<const int *>(ids) + i);
}

constexpr int kLookupThreads = 256;

// A block takes rows_per_block rows; its threads walk the groups of those rows in memory order.
// N = 8 needs rows of both tensors that start on 16-byte boundaries and H % 8 == 0, N = 1 takes anything.
template <typename TW, typename TO, int N>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(const LookupArgs a) {
    const long long t0 = (long long)blockIdx.x * a.rows_per_block;
    const unsigned rows = (unsigned)min((long long)a.rows_per_block, a.T - t0);
    const unsigned total = rows * (unsigned)a.groups;
    for (unsigned i = threadIdx.x; i < total; i += kLookupThreads) {
        const unsigned r = i / (unsigned)a.groups, j = (i - r * (unsigned)a.groups) * N;
        const long long t = t0 + r, id = read_id(a.ids, a.ids64, t);
        float f[N];
        if (id >= 0 && id < a.V) {
            load_vec<TW, N>(static_cast<const TW *>(a.table) + id * a.ld_table + j, f);
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] *= a.scale;
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = 0.f;
        }
        store_vec<TO, N>(static_cast<TO *>(a.out) + t * a.ld_out + j, f);
    }
}

// ---------------------------------------------------------------- gradient: order of the tokens
// dtable[v] = scale * sum over t with id_t = v of dout[t].  The tokens are sorted by id, stably, so
// that equal ids stand together and each sum runs in token order: the result is the same from run to
// run, with no atomics on floating numbers.
//
// Sort: least significant digit first, digits of up to 9 bits, by ONE cluster of up to 8 blocks
// (two passes for any vocabulary up to 262,143).  Every warp owns a stretch of the input; it counts
// its digits in a histogram of its own in shared memory, a prefix sum over (digit, block, warp) turns
// the counts into first places, and the warp walks its stretch again and places each element:
// rank within 32 elements by match, then the warp's running place.  Ids outside [0, V) get the key V
// and end up last.  The other blocks of the launch write the zeros of a gradient that is written whole.

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigitBits = 9;
constexpr int kBins = 1 << kDigitBits;
constexpr int kSortMaxCluster = 8;

struct SortArgs {
    const void *ids;
    int ids64;
    long long V;
    unsigned T;
    unsigned *key[2], *pos[2];   // workspace: two buffers; the result is in buffer passes & 1
    int passes, bits;            // digits and their width
    // zero fill (rows of dtable), none if zero == null
    void *zero;
    long long zero_ld;           // bytes
    long long zero_width;        // bytes of a row
    int zero_vec;                // rows start on 16-byte boundaries and are a multiple of 16 bytes wide
};

__device__ __forceinline__ void fill_zero(const SortArgs &a, long long block, long long blocks) {
    unsigned char *base = static_cast<unsigned char *>(a.zero);
    if (a.zero_vec) {
        const long long w = a.zero_width / 16;
        if (a.zero_ld == a.zero_width) {                                     // one stretch
            for (long long i = block * kSortThreads + threadIdx.x; i < w * a.V; i += blocks * kSortThreads)
                __stcs(reinterpret_cast<uint4 *>(base) + i, make_uint4(0, 0, 0, 0));
        } else {
            for (long long v = block; v < a.V; v += blocks)
                for (long long i = threadIdx.x; i < w; i += kSortThreads)
                    __stcs(reinterpret_cast<uint4 *>(base + v * a.zero_ld) + i, make_uint4(0, 0, 0, 0));
        }
    } else {                                                                  // 2 bytes divide every element type
        const long long w = a.zero_width / 2;
        for (long long v = block; v < a.V; v += blocks)
            for (long long i = threadIdx.x; i < w; i += kSortThreads)
                reinterpret_cast<unsigned short *>(base + v * a.zero_ld)[i] = 0;
    }
}

__device__ __forceinline__ unsigned sort_key(const SortArgs &a, int pass, unsigned i) {
    if (pass > 0) return __ldcg(a.key[pass & 1] + i);
    const long long id = read_id(a.ids, a.ids64, i);
    return (unsigned)((id < 0 || id >= a.V) ? a.V : id);
}

__global__ void __launch_bounds__(kSortThreads) embedding_sort_kernel(const SortArgs a) {
    extern __shared__ unsigned s_hist[];                      // [kSortWarps][bins]
    __shared__ unsigned s_total[kBins], s_scan[kSortWarps];
    const int C = (int)cluster_size(), rank = (int)cluster_rank();
    if ((int)blockIdx.x >= C) {
        fill_zero(a, (long long)blockIdx.x - C, (long long)gridDim.x - C);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bins = 1 << a.bits;
    const unsigned mask = (unsigned)bins - 1u;
    const unsigned warps = (unsigned)C * kSortWarps;
    const unsigned stretch = ((a.T + warps - 1) / warps + 31u) & ~31u;
    const unsigned long long from = (unsigned long long)(rank * kSortWarps + warp) * stretch;
    const unsigned i0 = (unsigned)min(from, (unsigned long long)a.T);
    const unsigned i1 = (unsigned)min(from + stretch, (unsigned long long)a.T);
    unsigned *hist = s_hist + warp * bins;

    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.bits;
        for (int b = lane; b < bins; b += 32) hist[b] = 0;
        __syncwarp();
#pragma unroll 4
        for (unsigned i = i0 + lane; i < i1; i += 32) atomicAdd(&hist[(sort_key(a, pass, i) >> shift) & mask], 1u);
        __syncthreads();
        unsigned run = 0;                                     // elements of this block with digit tid
        if (tid < bins) {
            for (int w = 0; w < kSortWarps; ++w) {
                const unsigned c = s_hist[w * bins + tid];
                s_hist[w * bins + tid] = run;
                run += c;
            }
            s_total[tid] = run;
        }
        if (C > 1) { cluster_arrive(); cluster_wait(); }
        unsigned all = run, lower = 0;                        // ... of the cluster; of the blocks before this one
        if (C > 1 && tid < bins) {
            all = 0;
            for (int r = 0; r < C; ++r) {
                const unsigned c = cluster_load(cluster_map(&s_total[tid], r));
                if (r < rank) lower += c;
                all += c;
            }
        }
        unsigned incl = all;                                  // prefix sum over the digits
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned n = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += n;
        }
        if (lane == 31) s_scan[warp] = incl;
        __syncthreads();
        if (tid < bins) {
            unsigned first = incl - all + lower;
            for (int w = 0; w < warp; ++w) first += s_scan[w];
            for (int w = 0; w < kSortWarps; ++w) s_hist[w * bins + tid] += first;
        }
        __syncthreads();
        unsigned *key_out = a.key[(pass + 1) & 1], *pos_out = a.pos[(pass + 1) & 1];
        for (unsigned i = i0; i < i1; i += 32) {
            const bool in = i + lane < i1;
            const unsigned key = in ? sort_key(a, pass, i + lane) : 0u;
            const unsigned pos = !in ? 0u : pass > 0 ? __ldcg(a.pos[pass & 1] + i + lane) : i + lane;
            const unsigned digit = in ? (key >> shift) & mask : 0xffffffffu;
            const unsigned peers = __match_any_sync(0xffffffffu, digit);
            unsigned place = 0;
            if (in) place = hist[digit] + __popc(peers & ((1u << lane) - 1u));
            __syncwarp();
            if (in && lane == 31 - __clz(peers)) hist[digit] = place + 1;
            __syncwarp();
            if (in) {
                __stcg(key_out + place, key);
                __stcg(pos_out + place, pos);
            }
        }
        __threadfence();                                      // the next pass reads what other blocks wrote
        if (C > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient: sums over equal ids
// The sorted tokens are cut into tiles of `tile` places.  A thread owns N columns of one tile and
// walks its places, with the rows' loads ahead of the sums.  An id whose tokens all lie in the tile
// is written at once; the part of one that reaches over a tile's end goes to the workspace (at most
// two a tile: the first id's and the last id's), and a second launch adds such parts in tile order.

constexpr int kReduceThreads = 256;

struct ReduceArgs {
    const unsigned *key, *pos;
    const void *dout;
    void *dtable;
    float *part;                 // [tiles][2][H]: 0 an id that came in from the tile before, 1 one that starts here and goes on
    long long ld_dout, ld_dtable;
    unsigned T, V;
    int H, groups, tile, tiles;
    int row_threads;             // threads side by side on one tile's columns (power of two)
    int add;
    float scale;
};

template <typename TW, int N>
__device__ __forceinline__ void write_row(const ReduceArgs &a, unsigned v, int j, float (&acc)[N]) {
    TW *p = static_cast<TW *>(a.dtable) + (long long)v * a.ld_dtable + j;
    if (a.add) {
        float f[N];
        load_vec<TW, N>(p, f);
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] = fmaf(acc[k], a.scale, f[k]);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] *= a.scale;
    }
    store_vec<TW, N>(p, acc);
}

template <typename TG, typename TW, int N>
__global__ void __launch_bounds__(kReduceThreads) embedding_reduce_kernel(const ReduceArgs a) {
    constexpr int kAhead = 8;
    const int sub = threadIdx.x / a.row_threads, col = threadIdx.x - sub * a.row_threads;
    const int tile = blockIdx.x * (kReduceThreads / a.row_threads) + sub;
    const int grp = blockIdx.y * a.row_threads + col;
    if (tile >= a.tiles || grp >= a.groups) return;
    const int j = grp * N;
    const unsigned i0 = (unsigned)tile * a.tile, i1 = min(i0 + a.tile, a.T);
    const unsigned none = 0xffffffffu;
    const unsigned before = i0 ? __ldg(a.key + i0 - 1) : none;
    const unsigned after = i1 < a.T ? __ldg(a.key + i1) : none;
    unsigned cur = __ldg(a.key + i0);
    bool open = cur == before;                               // the current id came in from the tile before
    float acc[N];
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] = 0.f;
    auto flush = [&](bool goes_on) {
        if (cur >= a.V) return;
        if (open || goes_on)
            store_vec<float, N>(a.part + ((size_t)tile * 2 + (open ? 0 : 1)) * a.H + j, acc);
        else
            write_row<TW, N>(a, cur, j, acc);
    };
    for (unsigned i = i0; i < i1; i += kAhead) {
        unsigned key[kAhead];
        float f[kAhead][N];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            key[u] = i + u < i1 ? __ldg(a.key + i + u) : none;
            if (key[u] < a.V) {
                const unsigned t = __ldg(a.pos + i + u);
                load_vec<TG, N>(static_cast<const TG *>(a.dout) + (long long)t * a.ld_dout + j, f[u]);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) f[u][k] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= i1) break;
            if (key[u] != cur) {
                flush(false);
                cur = key[u];
                open = false;
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] += f[u][k];
        }
    }
    flush(cur == after);
}

// One thread group per tile: if an id starts in the tile and goes on, its parts are added up here.
template <typename TW, int N>
__global__ void __launch_bounds__(kReduceThreads) embedding_join_kernel(const ReduceArgs a) {
    const int sub = threadIdx.x / a.row_threads, col = threadIdx.x - sub * a.row_threads;
    const int tile = blockIdx.x * (kReduceThreads / a.row_threads) + sub;
    const int grp = blockIdx.y * a.row_threads + col;
    if (tile + 1 >= a.tiles || grp >= a.groups) return;
    const unsigned i0 = (unsigned)tile * a.tile, i1 = i0 + a.tile;
    const unsigned v = __ldg(a.key + i1 - 1);
    if (v >= a.V || __ldg(a.key + i1) != v) return;          // nothing goes on
    if (__ldg(a.key + i0) == v && i0 && __ldg(a.key + i0 - 1) == v) return;   // it started before this tile
    // tiles reached: places up to the last one with id v
    unsigned lo = i1, hi = a.T;                              // key[lo] == v; first place past v is in (lo, hi]
    while (hi - lo > 1) {
        const unsigned mid = lo + (hi - lo) / 2;
        if (__ldg(a.key + mid) == v) lo = mid; else hi = mid;
    }
    const int last = (int)(lo / (unsigned)a.tile);
    const int j = grp * N;
    float acc[N], f[N];
    load_vec<float, N>(a.part + ((size_t)tile * 2 + 1) * a.H + j, acc);
#pragma unroll 4
    for (int t = tile + 1; t <= last; ++t) {
        load_vec<float, N>(a.part + (size_t)t * 2 * a.H + j, f);
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] += f[k];
    }
    write_row<TW, N>(a, v, j, acc);
}

}  // namespace
