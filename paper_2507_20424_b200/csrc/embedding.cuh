// Embedding lookup with a scale, and its gradient by sorted tokens.
#pragma once
#include "local_common.cuh"

namespace {

// ---------------------------------------------------------------- lookup
// out[t] = scale * table[id_t], zeros where id_t is outside [0, V).  The fp32 product, rounded to out's type.
// Bound by the bytes of the distinct rows and of the output.

struct LookupArgs {
    const void *table, *ids;
    void *out;
    long long ld_table, ld_out;   // elements
    long long T, V;
    int groups;                   // groups of N elements in a row
    int H, ids64;
    unsigned rows_per_block;
    float scale;
};

__device__ __forceinline__ long long read_id(const void *ids, int ids64, long long i) {
    return ids64 ? __ldg(static_cast<const long long *>(ids) + i) : (long long)__ldg(static_cast<const int *>(ids) + i);
}

constexpr int kLookupThreads = 256;

// A block takes rows_per_block rows; its threads walk the groups of those rows in memory order, kLookupAhead at a time.
// N elements are 16 bytes of the output (16,384 rows of 1,024 from fp32 to bf16: 8 elements 11.9 us, 4 14.2; 26,214 of 5,120 from
// bf16 to fp32: 4 elements 104 us, 8 130) where rows of both tensors start on 16-byte boundaries and H allows it; 4 and 2 need rows
// on boundaries of so many elements and such an H, 1 takes anything.
// Groups that a thread has under way, for the same two: 2 at full occupancy (32 registers) 11.9 and 104 us; 1 11.9 and 107; 4 at half
// the occupancy 13.2 and 120, at full occupancy, out of registers, 25.6 and 116.
constexpr int kLookupAhead = 2;

template <typename TW, typename TO, int N>
__global__ void __launch_bounds__(kLookupThreads, 8) lookup_kernel(const LookupArgs a) {
    constexpr int kAhead = kLookupAhead;
    const long long t0 = (long long)blockIdx.x * a.rows_per_block;
    const unsigned rows = (unsigned)min((long long)a.rows_per_block, a.T - t0);
    const unsigned total = rows * (unsigned)a.groups;
    for (unsigned i0 = threadIdx.x; i0 < total; i0 += kLookupThreads * kAhead) {
        long long id[kAhead];
        unsigned r[kAhead], j[kAhead];
        float f[kAhead][N];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const unsigned i = i0 + u * kLookupThreads;
            r[u] = i / (unsigned)a.groups;
            j[u] = (i - r[u] * (unsigned)a.groups) * N;
            id[u] = i < total ? read_id(a.ids, a.ids64, t0 + r[u]) : -1;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (id[u] >= 0 && id[u] < a.V) {
                load_vec<TW, N, false>(static_cast<const TW *>(a.table) + id[u] * a.ld_table + j[u], f[u]);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) f[u][k] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i0 + u * kLookupThreads >= total) break;
            if (id[u] >= 0 && id[u] < a.V) {
#pragma unroll
                for (int k = 0; k < N; ++k) f[u][k] *= a.scale;
            }
            store_vec<TO, N>(static_cast<TO *>(a.out) + (t0 + r[u]) * a.ld_out + j[u], f[u]);
        }
    }
}

// ---------------------------------------------------------------- gradient
// dtable[v] = scale * sum over t with id_t = v of dout[t].  The tokens are sorted by id, stably, so that equal ids stand
// together.  A sum runs in token order within a part (a tile, or a warp's stretch of few tokens); how a long sum's parts are added
// depends on the ids and sizes alone: the result is the same from run to run, and no order of atomics matters.
// The launches (count, place per digit, sums and zeros, joins) are each set up while the one before ends; up to
// kFewTokens tokens take a single launch that sorts in every block.

struct GradArgs {
    const void *ids;
    int ids64;
    unsigned T, V;
    const void *dout;
    void *dtable;
    long long ld_dout, ld_dtable;   // elements
    int H, add;
    float scale;
    uint2 *order0, *order1;      // workspace: (key, token) in order; the sort's result is in buffer passes & 1
    unsigned *hist;              // [3][kSortBlocks][kBins]: a digit's counts, the next one's, the one's after that, in turn
    int passes, bits;            // digits and their width
    int sort_blocks;
    unsigned chunk;              // tokens of a block of the sort, a multiple of kSortThreads
    int zero_vec;                // rows of dtable start on 16-byte boundaries and are a multiple of 16 bytes wide
    // rows of a gradient that is written whole: the last early_rows are zeroed by spare blocks of the sort's launches,
    // the late_rows before them (where their ids do not occur) beside the joins, the others beside the sums
    unsigned early_rows, late_rows;
    int zero_blocks, late_blocks;   // blocks that write zeros, beside the sums and beside the joins
    int zero_rows;               // rows that each of them looks after at a time
    // sums
    float *part;                 // [tiles][2][H]: 0 an id that came in from the tile before, 1 one that starts here and goes on
    int groups, tile, tiles;
    int row_threads;             // threads side by side on one tile's columns
    int tile_blocks;             // blocks side by side over the tiles
};

__device__ __forceinline__ unsigned token_key(const GradArgs &a, unsigned i) {
    const long long id = read_id(a.ids, a.ids64, i);
    return (id < 0 || id >= (long long)a.V) ? a.V : (unsigned)id;
}

// Zeros to row v, by `threads` threads of which this is `rank`.
template <typename TW>
__device__ __forceinline__ void zero_row(const GradArgs &a, long long v, int rank, int threads) {
    TW *p = static_cast<TW *>(a.dtable) + v * a.ld_dtable;
    if (a.zero_vec) {
        const int w = a.H * (int)sizeof(TW) / 16;
        for (int i = rank; i < w; i += threads) __stcs(reinterpret_cast<uint4 *>(p) + i, make_uint4(0, 0, 0, 0));
    } else {
        for (int i = rank; i < a.H; i += threads) p[i] = from_float<TW>(0.f);
    }
}

// ---------------------------------------------------------------- gradient: order of the tokens
// Least significant digit first, digits of up to 9 bits (two for any vocabulary up to 262,143).  A block owns a chunk of the
// sequence and a warp a stretch of the chunk.  The first launch counts each chunk's digits.  A launch per
// digit then places: a block reads all chunks' counts, so that it knows where each of its digits begins, counts per
// warp in shared memory, and its warps walk their stretches: rank within 32 elements by match, then the warp's running
// place.  As an element is placed, its next digit is counted for the chunk that it moves to (whole
// numbers: any order).  Ids outside [0, V) get the key V and end up last.

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigitBits = 9;
constexpr int kBins = 1 << kDigitBits;
constexpr int kSortBlocks = 128;     // at most
constexpr int kSortHold = 4;         // elements a lane keeps in registers between counting and placing
constexpr int kCountGroups = kSortThreads / (kBins / 4);
constexpr size_t kPlaceSmem = (size_t)(kSortWarps + 2 * kCountGroups) * kBins * sizeof(unsigned);

__device__ __forceinline__ unsigned *counts_of(const GradArgs &a, int pass) { return a.hist + (size_t)(pass % 3) * kSortBlocks * kBins; }

__global__ void __launch_bounds__(kSortThreads) embedding_count_kernel(const GradArgs a) {
    __shared__ unsigned s_count[kBins];
    let_next_start();
    const unsigned mask = (1u << a.bits) - 1u;
    for (int b = threadIdx.x; b < kBins; b += kSortThreads) s_count[b] = 0;
    __syncthreads();
    const unsigned long long end = min((unsigned long long)(blockIdx.x + 1) * a.chunk, (unsigned long long)a.T);
    for (unsigned long long i = (unsigned long long)blockIdx.x * a.chunk + threadIdx.x; i < end; i += kSortThreads)
        atomicAdd(&s_count[token_key(a, (unsigned)i) & mask], 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kSortThreads) {
        counts_of(a, 0)[(size_t)blockIdx.x * kBins + b] = s_count[b];
        counts_of(a, 1)[(size_t)blockIdx.x * kBins + b] = 0;
    }
}

template <typename TW>
__global__ void __launch_bounds__(kSortThreads) embedding_place_kernel(const GradArgs a, int pass) {
    extern __shared__ unsigned s_hist[];                      // [kSortWarps][kBins], then [kCountGroups][kBins] twice
    __shared__ unsigned s_scan[kSortWarps];
    unsigned *s_all = s_hist + kSortWarps * kBins, *s_lower = s_all + kCountGroups * kBins;
    let_next_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if ((int)blockIdx.x >= a.sort_blocks) {                   // nothing else in this sequence of launches touches the table yet
        const long long from = (long long)a.V - a.early_rows + (long long)a.early_rows * pass / a.passes, to = (long long)a.V - a.early_rows + (long long)a.early_rows * (pass + 1) / a.passes;
        for (long long v = from + (long long)(blockIdx.x - a.sort_blocks) * kSortWarps + warp; v < to; v += (long long)(gridDim.x - a.sort_blocks) * kSortWarps)
            zero_row<TW>(a, v, lane, 32);
        return;
    }
    unsigned *hist = s_hist + warp * kBins;
    for (int b = lane; b < kBins; b += 32) hist[b] = 0;
    __syncwarp();                                             // the zeros, before any lane counts into them
    wait_for_previous();

    const int shift = pass * a.bits;
    const unsigned mask = (1u << a.bits) - 1u;
    const bool more = pass + 1 < a.passes;
    const uint2 *in_order = (pass & 1) ? a.order1 : a.order0;
    uint2 *out_order = (pass & 1) ? a.order0 : a.order1;
    const unsigned *counts = counts_of(a, pass);
    unsigned *next_counts = counts_of(a, pass + 1);
    if (more && tid < kBins) counts_of(a, pass + 2)[(size_t)blockIdx.x * kBins + tid] = 0;
    const unsigned stretch = a.chunk / kSortWarps;            // a multiple of 32
    const unsigned long long from = (unsigned long long)blockIdx.x * a.chunk + (unsigned long long)warp * stretch;
    const unsigned i0 = (unsigned)min(from, (unsigned long long)a.T), i1 = (unsigned)min(from + stretch, (unsigned long long)a.T);
    auto element = [&](unsigned i) { return pass == 0 ? make_uint2(token_key(a, i), i) : __ldcg(in_order + i); };   // (key, token)

    uint2 held[kSortHold];                                    // the first elements of the stretch
#pragma unroll
    for (int u = 0; u < kSortHold; ++u) {
        const unsigned i = i0 + u * 32 + lane;
        held[u] = i < i1 ? element(i) : make_uint2(0, 0);
    }
    {                                                         // four digits a thread, the chunks in kCountGroups turns
        const int q = tid % (kBins / 4), turn = tid / (kBins / 4);
        uint4 all = make_uint4(0, 0, 0, 0), lower = all;
#pragma unroll 8
        for (int c = turn; c < a.sort_blocks; c += kCountGroups) {
            const uint4 n = __ldcg(reinterpret_cast<const uint4 *>(counts + (size_t)c * kBins) + q);
            all.x += n.x; all.y += n.y; all.z += n.z; all.w += n.w;
            if (c < (int)blockIdx.x) { lower.x += n.x; lower.y += n.y; lower.z += n.z; lower.w += n.w; }
        }
        reinterpret_cast<uint4 *>(s_all + turn * kBins)[q] = all;
        reinterpret_cast<uint4 *>(s_lower + turn * kBins)[q] = lower;
    }
#pragma unroll
    for (int u = 0; u < kSortHold; ++u)
        if (i0 + u * 32 + lane < i1) atomicAdd(&hist[(held[u].x >> shift) & mask], 1u);
    for (unsigned i = i0 + 32 * kSortHold + lane; i < i1; i += 32) atomicAdd(&hist[(element(i).x >> shift) & mask], 1u);
    __syncthreads();
    unsigned all = 0, first = 0;                              // elements of digit tid; where this block's begin
    if (tid < kBins) {
#pragma unroll
        for (int g = 0; g < kCountGroups; ++g) { all += s_all[g * kBins + tid]; first += s_lower[g * kBins + tid]; }
    }
    unsigned incl = all;                                      // prefix sum over the digits
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned n = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += n;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    if (tid < kBins) {
        first += incl - all;
        for (int w = 0; w < warp; ++w) first += s_scan[w];
        unsigned count[kSortWarps];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) count[w] = s_hist[w * kBins + tid];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            s_hist[w * kBins + tid] = first;
            first += count[w];
        }
    }
    __syncthreads();
    auto place = [&](bool in, uint2 e) {
        const unsigned digit = in ? (e.x >> shift) & mask : 0xffffffffu;
        const unsigned peers = __match_any_sync(0xffffffffu, digit);
        unsigned at = 0;
        if (in) at = hist[digit] + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
        if (in && lane == 31 - __clz(peers)) hist[digit] = at + 1;
        __syncwarp();
        if (in) {
            __stcg(out_order + at, e);
            if (more) atomicAdd(next_counts + (size_t)(at / a.chunk) * kBins + ((e.x >> (shift + a.bits)) & mask), 1u);
        }
    };
#pragma unroll
    for (int u = 0; u < kSortHold; ++u)
        if (i0 + u * 32 < i1) place(i0 + u * 32 + lane < i1, held[u]);
    for (unsigned i = i0 + 32 * kSortHold; i < i1; i += 32) {
        const bool in = i + lane < i1;
        place(in, in ? element(i + lane) : make_uint2(0, 0));
    }
}

// ---------------------------------------------------------------- gradient: sums over equal ids
// The sorted tokens are cut into tiles of `tile` places.  A thread owns N columns of one tile and walks its
// places, kAhead rows under way.  An id that starts in a tile and ends in it or in the next is added up and
// written by the thread of the tile where it starts (the next tile passes over it).  Of a longer one every tile leaves
// its part in the workspace, and the last launch adds the parts.

constexpr int kReduceThreads = 256;
constexpr int kMaxTile = 32;
constexpr int kMinRowThreads = 8;

// N elements as they are stored
template <typename T, int N> struct Stored { unsigned w[N * sizeof(T) >= 4 ? N * sizeof(T) / 4 : 1]; };
template <typename T, int N>
__device__ __forceinline__ Stored<T, N> load_stored(const T *p) {
    Stored<T, N> r;
    if constexpr (N == 1 && sizeof(T) == 2) {
        r.w[0] = __ldcs(reinterpret_cast<const unsigned short *>(p));
    } else {
        constexpr int kWords = N * (int)sizeof(T) / 4, kPer = kWords < 4 ? kWords : 4;
        using W = typename Words<kPer>::type;
#pragma unroll
        for (int i = 0; i < kWords / kPer; ++i) {
            const W w = __ldcs(reinterpret_cast<const W *>(p) + i);
            memcpy(&r.w[i * kPer], &w, sizeof(W));
        }
    }
    return r;
}
template <int N> __device__ __forceinline__ float element_of(const Stored<float, N> &r, int k) { return __uint_as_float(r.w[k]); }
template <int N> __device__ __forceinline__ float element_of(const Stored<bf16, N> &r, int k) { return (k & 1) ? bf16_high(r.w[k / 2]) : bf16_low(r.w[k / 2]); }

// dtable[v] = scale * acc, or += that.  Every element has one writer in a launch, so adding to fp32 in memory (one
// rounding, nothing waits for the old value) depends on no order.
template <typename TW, int N>
__device__ __forceinline__ void finish_row(const GradArgs &a, unsigned v, int j, const float (&acc)[N]) {
    TW *p = static_cast<TW *>(a.dtable) + (long long)v * a.ld_dtable + j;
    float f[N];
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = acc[k] * a.scale;
    if (!a.add) {
        store_vec<TW, N>(p, f);
    } else if constexpr (sizeof(TW) == 4) {
        if constexpr (N >= 4) {
#pragma unroll
            for (int k = 0; k < N; k += 4)
                asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p + k), "f"(f[k]), "f"(f[k + 1]), "f"(f[k + 2]), "f"(f[k + 3]) : "memory");
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) atomicAdd(reinterpret_cast<float *>(p) + k, f[k]);
        }
    } else {
        float old[N];
        load_vec<TW, N>(p, old);
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] += old[k];
        store_vec<TW, N>(p, f);
    }
}

// Zeros to the rows of ids that do not occur, zero_rows at a time: the sorted keys between the rows' bounds tell which.
constexpr int kMaxZeroRows = 1024;

// First place in the sorted keys that is not below v, by a warp, 33 stretches at a time.
__device__ __forceinline__ unsigned lower_bound(const uint2 *order, unsigned T, long long v, int lane) {
    unsigned lo = 0, hi = T;                                 // places before lo are below v, places from hi on are not
    while (lo < hi) {
        const unsigned step = (hi - lo + 32) / 33;
        const unsigned long long at = (unsigned long long)lo + (unsigned long long)step * (lane + 1) - 1;
        const int below = __popc(__ballot_sync(0xffffffffu, at < hi && (long long)__ldcg(&order[at < hi ? at : lo].x) < v));
        const unsigned end = (unsigned)min((unsigned long long)hi, (unsigned long long)lo + (unsigned long long)step * (below + 1) - 1);
        lo += step * below;
        hi = max(lo, end);
    }
    return lo;
}

template <typename TW>
__device__ __forceinline__ void zero_absent(const GradArgs &a, const uint2 *order, long long begin, long long end, int block, int blocks) {
    __shared__ unsigned s_seen[kMaxZeroRows / 32], s_from, s_to;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int threads = blockDim.x;
    for (long long v0 = begin + (long long)block * a.zero_rows; v0 < end; v0 += (long long)blocks * a.zero_rows) {
        const int rows = (int)min((long long)a.zero_rows, end - v0);
        if (tid < kMaxZeroRows / 32) s_seen[tid] = 0;
        if (warp < 2) {
            const unsigned at = lower_bound(order, a.T, warp ? v0 + rows : v0, lane);
            if (lane == 0) (warp ? s_to : s_from) = at;
        }
        __syncthreads();
        for (unsigned i = s_from + tid; i < s_to; i += threads) {
            const int r = (int)(__ldcg(&order[i].x) - v0);
            if (!((s_seen[r >> 5] >> (r & 31)) & 1u)) atomicOr(&s_seen[r >> 5], 1u << (r & 31));
        }
        __syncthreads();
        for (int r = warp; r < rows; r += threads / 32)
            if (!((s_seen[r >> 5] >> (r & 31)) & 1u)) zero_row<TW>(a, v0 + r, lane, 32);
        __syncthreads();
    }
}

template <typename TG, typename TW, int N>
__global__ void __launch_bounds__(kReduceThreads, 4) embedding_reduce_kernel(const GradArgs a) {
    constexpr int kAhead = N * sizeof(TG) == 32 ? 4 : 8;
    constexpr int kMost = kReduceThreads / kMinRowThreads * kMaxTile;
    __shared__ unsigned s_key[kMost + 2 * kMaxTile + 2], s_pos[kMost + kMaxTile];
    let_next_start();
    wait_for_previous();
    // the blocks that write zeros are spread evenly among the others
    const long long zeros_before = (long long)blockIdx.x * a.zero_blocks / gridDim.x;
    if ((long long)(blockIdx.x + 1) * a.zero_blocks / gridDim.x > zeros_before) {
        zero_absent<TW>(a, (a.passes & 1) ? a.order1 : a.order0, 0, (long long)a.V - a.early_rows - a.late_rows, (int)zeros_before, a.zero_blocks);
        return;
    }
    const int block = (int)(blockIdx.x - zeros_before), block_x = block % a.tile_blocks, block_y = block / a.tile_blocks;
    const int subs = kReduceThreads / a.row_threads;
    const int sub = threadIdx.x / a.row_threads, col = threadIdx.x - sub * a.row_threads;
    const uint2 *order = (a.passes & 1) ? a.order1 : a.order0;
    // keys of the places from one tile (and one) before this block's to one after it; V + 1 where there is none
    const int span = subs * a.tile;
    const long long base = (long long)block_x * span;
    for (int i = threadIdx.x; i < span + 2 * a.tile + 2; i += kReduceThreads) {
        const long long at = base + i - a.tile - 1;
        const uint2 e = at >= 0 && at < (long long)a.T ? __ldcg(order + at) : make_uint2(a.V + 1, 0);
        s_key[i] = e.x;
        if (i > a.tile && i - a.tile - 1 < span + a.tile) s_pos[i - a.tile - 1] = e.y;
    }
    __syncthreads();
    const int tile = block_x * subs + sub;
    const int grp = block_y * a.row_threads + col;
    if (sub >= subs || tile >= a.tiles || grp >= a.groups) return;
    const int j = grp * N, L = a.tile;
    const unsigned *key = s_key + sub * L + L + 1, *pos = s_pos + sub * L;        // key[-L - 1] .. key[2 L]
    int i = 0, n = (int)min((long long)L, (long long)a.T - (long long)tile * L);
    bool came = key[0] == key[-1];                           // the current id came in, and is a long one
    if (came && key[-L - 1] != key[0] && key[L] != key[0]) { // not so long: the tile before has it
        while (i < n && key[i] == key[-1]) ++i;
        came = false;
    }
    const bool goes_on = key[n - 1] == key[n];
    bool leaves = goes_on;                                   // the last id goes on as a long one
    if (goes_on && key[-1] != key[n - 1] && key[2 * L] != key[n - 1]) {
        const unsigned v = key[n - 1];
        while (key[n] == v) ++n;
        leaves = false;
    }
    float acc[N];
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] = 0.f;
    const TG *dout = static_cast<const TG *>(a.dout) + j;
    for (; i < n; i += kAhead) {
        Stored<TG, N> f[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < n && key[i + u] < a.V) f[u] = load_stored<TG, N>(dout + (long long)pos[i + u] * a.ld_dout);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= n || key[i + u] >= a.V) break;      // ids outside [0, V) are last
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] += element_of<N>(f[u], k);
            if (key[i + u] != key[i + u + 1]) {              // the id's last token
                if (came) store_vec<float, N>(a.part + (size_t)tile * 2 * a.H + j, acc);
                else finish_row<TW, N>(a, key[i + u], j, acc);
                came = false;
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] = 0.f;
            }
        }
    }
    if (leaves && key[n - 1] < a.V) store_vec<float, N>(a.part + ((size_t)tile * 2 + (came ? 0 : 1)) * a.H + j, acc);
}

// A block looks through kJoinTiles tiles for long ids that start in one of them and adds each one's parts over 32 N columns,
// several ids side by side: its warps are dealt out among them (1, 2, 4 or 8 an id, by how many long ids start in these tiles), a
// warp adds every so manieth part, in tile order, and the warps' sums are added in theirs.
constexpr int kJoinTiles = 32;
constexpr int kJoinThreads = 256;
constexpr int kJoinWarps = kJoinThreads / 32;

template <typename TW, int N>
__global__ void __launch_bounds__(kJoinThreads, 3) embedding_join_kernel(const GradArgs a) {
    __shared__ float s_sum[kJoinWarps][32 * N];
    wait_for_previous();
    const uint2 *order = (a.passes & 1) ? a.order1 : a.order0;
    const int join_blocks = (int)gridDim.x - a.late_blocks;
    if ((int)blockIdx.x >= join_blocks) {
        const long long end = (long long)a.V - a.early_rows;
        zero_absent<TW>(a, order, end - a.late_rows, end, (int)blockIdx.x - join_blocks, a.late_blocks);
        return;
    }
    const int tile_groups = (a.tiles + kJoinTiles - 1) / kJoinTiles, block_x = blockIdx.x % tile_groups, block_y = blockIdx.x / tile_groups;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int j = (block_y * 32 + lane) * N;
    const bool in = j < a.H;
    const int mine = block_x * kJoinTiles + lane;            // every warp looks at the same tiles
    auto first_key = [&](long long tile) {                   // of a tile; V + 1 past the last
        return tile < a.tiles ? __ldcg(&order[tile * a.tile].x) : a.V + 1;
    };
    unsigned v = a.V + 1;
    bool starts = false;                                     // a long id starts in this lane's tile: it reaches the tile after the next
    if (mine + 2 < a.tiles) {
        v = first_key(mine + 1);
        const unsigned i0 = (unsigned)mine * a.tile, last = __ldcg(&order[i0 + a.tile - 1].x), before = i0 ? __ldcg(&order[i0 - 1].x) : a.V + 1;
        starts = v < a.V && last == v && before != v && first_key((long long)mine + 2) == v;
    }
    const unsigned found = __ballot_sync(0xffffffffu, starts);
    for (int done = 0; done < __popc(found); done += kJoinWarps) {
        const int ids = min(__popc(found) - done, kJoinWarps), share = ids > 4 ? 1 : ids > 2 ? 2 : ids > 1 ? 4 : 8;   // warps an id
        const int mine_of = warp / share, sub = warp % share;
        const bool busy = mine_of < ids;
        unsigned id = a.V;
        float acc[N];
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] = 0.f;
        if (busy) {
            const int from = (int)__fns(found, 0, done + mine_of + 1), tile = block_x * kJoinTiles + from;
            id = __shfl_sync(0xffffffffu, v, from);
            for (int p0 = sub;; p0 += 32 * share) {          // parts p0, p0 + share, ...: as many as begin with the id
                const int p = p0 + share * lane;
                const int count = __popc(__ballot_sync(0xffffffffu, p == 0 || first_key((long long)tile + p) == id));
                if (in) {
#pragma unroll 8
                    for (int q = 0; q < count; ++q) {
                        float f[N];
                        const int part = p0 + share * q;
                        load_vec<float, N>(a.part + ((size_t)(tile + part) * 2 + (part == 0 ? 1 : 0)) * a.H + j, f);
#pragma unroll
                        for (int k = 0; k < N; ++k) acc[k] += f[k];
                    }
                }
                if (count < 32) break;
            }
#pragma unroll
            for (int k = 0; k < N; ++k) s_sum[warp][k * 32 + lane] = acc[k];
        }
        __syncthreads();
        if (busy && sub == 0 && in) {
            for (int w = 1; w < share; ++w) {
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] += s_sum[warp + w][k * 32 + lane];
            }
            finish_row<TW, N>(a, id, j, acc);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient: few tokens
// One launch, no workspace.  Every block sorts all the tokens in shared memory (each thread counts the tokens that
// come before its own).  The first column_blocks blocks take 32 N columns each: their warps walk equal
// stretches of the sorted tokens, and an id that reaches over a stretch's end is added up by the warp where it starts, from
// the parts that the others leave in shared memory.  The other blocks write zeros to the rows of ids that do not occur.

constexpr int kFewTokens = 512;
constexpr int kFewThreads = 1024;
constexpr int kFewWarps = kFewThreads / 32;

template <typename TG, typename TW, int N>
__global__ void __launch_bounds__(kFewThreads) embedding_few_kernel(const GradArgs a) {
    __shared__ __align__(16) unsigned s_id[kFewTokens];
    __shared__ unsigned s_key[kFewTokens + 2], s_pos[kFewTokens];
    __shared__ float s_part[kFewWarps][32 * N];              // sum of the id that a warp's stretch begins with, if it came in
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned T = a.T;
    const int column_blocks = (int)gridDim.x - a.zero_blocks;
    unsigned mine = a.V;
    if ((unsigned)tid < T) mine = token_key(a, tid);
    if (tid < kFewTokens) s_id[tid] = (unsigned)tid < T ? mine : 0xffffffffu;     // past the end: above every key
    if (tid == 0) { s_key[0] = a.V + 1; s_key[T + 1] = a.V + 1; }
    __syncthreads();
    if ((int)blockIdx.x >= column_blocks) {
        // rows [v0, v1) of this block, 1024 at a time: which of them occur?
        __shared__ unsigned s_seen[32];
        const long long per = ((long long)a.V + a.zero_blocks - 1) / a.zero_blocks;
        const long long v0 = per * ((int)blockIdx.x - column_blocks), v1 = min(v0 + per, (long long)a.V);
        for (long long v = v0; v < v1; v += 1024) {
            const int rows = (int)min(1024LL, v1 - v);
            if (tid < 32) s_seen[tid] = 0;
            __syncthreads();
            if ((unsigned)tid < T && mine >= v && mine < v + rows) atomicOr(&s_seen[(mine - v) >> 5], 1u << ((mine - v) & 31));
            __syncthreads();
            for (int r = warp; r < rows; r += kFewWarps)
                if (!((s_seen[r >> 5] >> (r & 31)) & 1u)) zero_row<TW>(a, v + r, lane, 32);
            __syncthreads();
        }
        return;
    }
    if (warp * 32 < (int)T) {
        // tokens before this warp's count if their id is not above, those after it if it is below; the warp's own by position
        unsigned place = 0;
        const uint4 *ids4 = reinterpret_cast<const uint4 *>(s_id);
#pragma unroll 4
        for (int i = 0; i < warp * 8; ++i) {
            const uint4 u = ids4[i];
            place += (u.x <= mine) + (u.y <= mine) + (u.z <= mine) + (u.w <= mine);
        }
#pragma unroll 4
        for (int i = warp * 8 + 8; i < ((int)T + 3) / 4; ++i) {
            const uint4 u = ids4[i];
            place += (u.x < mine) + (u.y < mine) + (u.z < mine) + (u.w < mine);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const unsigned u = __shfl_sync(0xffffffffu, mine, i);
            place += (i < lane ? u <= mine : u < mine) && warp * 32 + i < (int)T;
        }
        if ((unsigned)tid < T) {
            s_key[place + 1] = mine;
            s_pos[place] = tid;
        }
    }
    __syncthreads();
    const unsigned *key = s_key + 1;                         // key[-1] .. key[T]
    const unsigned each = (T + kFewWarps - 1) / kFewWarps;
    const unsigned from = min(warp * each, T), to = min(from + each, T);
    const int j = (blockIdx.x * 32 + lane) * N;
    const bool in = j < a.H;
    constexpr int kAhead = N * sizeof(TG) == 32 ? 4 : 8;
    float acc[N];
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] = 0.f;
    bool open = from < to && from > 0 && key[from] == key[(int)from - 1];
    for (unsigned i = from; i < to; i += kAhead) {
        Stored<TG, N> f[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (in && i + u < to && key[i + u] < a.V) f[u] = load_stored<TG, N>(static_cast<const TG *>(a.dout) + (long long)s_pos[i + u] * a.ld_dout + j);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= to || key[i + u] >= a.V) break;
            if (in) {
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] += element_of<N>(f[u], k);
            }
            const bool ends = key[i + u] != key[i + u + 1];
            if ((ends || i + u + 1 == to) && open) {         // (a part of) an id that came in
#pragma unroll
                for (int k = 0; k < N; ++k) s_part[warp][k * 32 + lane] = acc[k];
                open = false;
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] = 0.f;
            } else if (ends) {
                if (in) finish_row<TW, N>(a, key[i + u], j, acc);
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] = 0.f;
            }
        }
    }
    __syncthreads();
    // an id that starts in this stretch and goes on
    if (from < to && in && key[to - 1] < a.V && key[to - 1] == key[to]) {
        const unsigned v = key[to - 1];
        if (from > 0 && key[from] == v && key[(int)from - 1] == v) return;       // it came in itself
        for (int w = warp + 1; w < kFewWarps && w * each < T && key[w * each] == v; ++w) {
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] += s_part[w][k * 32 + lane];
        }
        finish_row<TW, N>(a, v, j, acc);
    }
}

}  // namespace
