// Operators of a worker's local step on a language model: host side and C ABI (include/dppf.h).
//   local_common.cuh   element types, vectors of eight elements, cluster accesses
//   embedding.cuh      lookup with a scale; the table's gradient by sorted tokens
//   policy_loss.cuh    clipped policy loss with a KL term, forward and backward, from logits
//   local_host.cuh     devices, launches, checks of arguments
//   adamw_tensors.cuh  AdamW over many tensors, optimiser state in fp32 or in 8 bits
#include "dppf.h"

#include <limits>

#include "adamw_tensors.cuh"
#include "embedding.cuh"
#include "local_host.cuh"
#include "policy_loss.cuh"

namespace {

// ---------------------------------------------------------------- embedding

// Elements that a thread moves at a time: `wide` (16 bytes of a type), 4, 2 or 1, as row starts and width of both matrices allow.
int group_width(int H, int wide, const void *p, int64_t ldp, int tp, const void *q, int64_t ldq, int tq) {
    for (const int n : {wide, 4, 2}) {
        auto fits = [&](const void *x, int64_t ld, int type) {
            const size_t boundary = n * type_bytes(type) < 16 ? n * type_bytes(type) : 16;
            return aligned_to(x, boundary) && (size_t)ld * type_bytes(type) % boundary == 0;
        };
        if (H % n == 0 && fits(p, ldp, tp) && fits(q, ldq, tq)) return n;
    }
    return 1;
}

template <typename TW, typename TO>
int launch_lookup(LookupArgs a, int n, int sms, cudaStream_t s) {
    a.groups = a.H / n;
    // two rounds of a thread's groups, at least one row a block
    long long rows = (2LL * kLookupAhead * kLookupThreads) / a.groups;
    if (rows < 1) rows = 1;
    // short lookups: fewer rows a block, so that four blocks an SM share the work
    while (rows > 1 && (a.T + rows - 1) / rows < 4LL * sms) rows = (rows + 1) / 2;
    a.rows_per_block = (unsigned)rows;
    const long long grid = (a.T + rows - 1) / rows;
    if (grid > INT_MAX) return DPPF_ERR_INVALID_ARG;
    constexpr int kWide = 16 / sizeof(TO);
    if (n == kWide) lookup_kernel<TW, TO, kWide><<<(unsigned)grid, kLookupThreads, 0, s>>>(a);
    else if (n == 4) lookup_kernel<TW, TO, 4><<<(unsigned)grid, kLookupThreads, 0, s>>>(a);
    else if (n == 2) lookup_kernel<TW, TO, 2><<<(unsigned)grid, kLookupThreads, 0, s>>>(a);
    else lookup_kernel<TW, TO, 1><<<(unsigned)grid, kLookupThreads, 0, s>>>(a);
    return launched();
}

// Places of the sorted tokens that a thread walks: long enough that few sums are split, short enough that about
// 2,000 threads an SM are at work, each on one of a row's `groups` (8 to 32).  The SMs are a B200's 148 whatever the device: the
// workspace is laid out by this, and its size is asked for without one.
int reduce_tile(int64_t T, int groups) {
    const double rows = (double)T * groups / (148.0 * 2048.0);
    int tile = 8;
    while (tile < kMaxTile && tile < rows) tile *= 2;
    return tile;
}

struct EmbeddingLayout {
    size_t order[2], hist, part, total;
};
EmbeddingLayout embedding_layout(int64_t T, int H) {
    EmbeddingLayout l;
    size_t at = 0;
    for (int i = 0; i < 2; ++i) { l.order[i] = at; at += round256((size_t)T * sizeof(uint2)); }
    l.hist = at;
    at += (size_t)3 * kSortBlocks * kBins * 4;
    l.part = at;
    const int64_t tile = reduce_tile(T, (H + 7) / 8);             // of the widest groups: the others' are no shorter
    at += round256((size_t)((T + tile - 1) / tile) * 2 * (size_t)H * 4);
    l.total = at;
    return l;
}

// Bytes of zeros written at a time by a block, beside a digit's launch of the sort and beside the joins
constexpr long long kZeroBytes = 65536, kEarlyBytes = 32LL << 20, kLateBytes = 40LL << 20;

std::atomic<int> g_place_ready[2][kMaxDevices];

// Threads side by side on a row's groups: a whole part of them that leaves the fewest of a block's threads idle.
// Rows of 50 groups in 50 threads, tiles by the groups that a row has: 91,096 tokens of 200 fp32 44 us (in 64 threads
// and tiles by the width 55); of 473 groups, one element each, 20,011 tokens 37 us (44).
int row_threads(int groups) {
    int best = kMinRowThreads;
    double used = 0.0;
    for (int parts = (groups + kReduceThreads - 1) / kReduceThreads, i = 0; i < 8; ++parts, ++i) {
        const int n = (groups + parts - 1) / parts;
        if (n < kMinRowThreads) break;
        const double share = (double)groups * (kReduceThreads / n) / ((double)kReduceThreads * parts);
        if (share > used * 1.05) { best = n; used = share; }
    }
    return best;
}

template <typename TG, typename TW, int N>
int launch_grad(GradArgs a, int dev, int sms, cudaStream_t s) {
    a.groups = a.H / N;
    const long long row_bytes = (long long)a.H * (int)sizeof(TW), zero_bytes = a.add ? 0 : (long long)a.V * row_bytes;
    if (a.T <= kFewTokens) {
        const int column_blocks = (a.groups + 31) / 32;
        a.zero_blocks = (int)((zero_bytes + 65535) / 65536 < 2LL * sms ? (zero_bytes + 65535) / 65536 : 2LL * sms);
        embedding_few_kernel<TG, TW, N><<<column_blocks + a.zero_blocks, kFewThreads, 0, s>>>(a);
        return launched();
    }
    if (!allow_smem(embedding_place_kernel<TW>, dev, g_place_ready[sizeof(TW) == 4 ? 0 : 1], (int)kPlaceSmem)) return DPPF_ERR_CUDA;
    const long long per = ((long long)a.T + kSortBlocks - 1) / kSortBlocks;
    a.chunk = (unsigned)((per + kSortThreads - 1) / kSortThreads * kSortThreads);
    a.sort_blocks = (int)(((long long)a.T + a.chunk - 1) / a.chunk);
    // zeros (V rows): what SMs without a part in the sort can write meanwhile, what fits beside the joins, the rest
    const int spare = zero_bytes && a.sort_blocks < 2 * sms ? 2 * sms - a.sort_blocks : 0;
    a.zero_rows = (int)(kZeroBytes / row_bytes < 1 ? 1 : kZeroBytes / row_bytes > kMaxZeroRows ? kMaxZeroRows : kZeroBytes / row_bytes);
    if (zero_bytes) {
        auto rows_of = [&](long long bytes, long long most) { return bytes / row_bytes < most ? bytes / row_bytes : most; };
        a.early_rows = spare ? (unsigned)rows_of(kEarlyBytes * a.passes, a.V) : 0;
        a.late_rows = (unsigned)rows_of(kLateBytes, (long long)a.V - a.early_rows);
        auto blocks_of = [&](long long rows) { const long long n = (rows + a.zero_rows - 1) / a.zero_rows; return (int)(n < 16LL * sms ? n : 16LL * sms); };
        a.zero_blocks = blocks_of((long long)a.V - a.early_rows - a.late_rows);
        a.late_blocks = blocks_of(a.late_rows);
    }
    embedding_count_kernel<<<a.sort_blocks, kSortThreads, 0, s>>>(a);
    bool ok = cudaPeekAtLastError() == cudaSuccess;
    for (int pass = 0; pass < a.passes; ++pass)
        ok = ok && launch_after(embedding_place_kernel<TW>, dim3((unsigned)(a.sort_blocks + spare)), kSortThreads, kPlaceSmem, s, a, pass);
    a.tile = reduce_tile(a.T, a.groups);
    a.tiles = (int)(((long long)a.T + a.tile - 1) / a.tile);
    a.row_threads = row_threads(a.groups);
    const int subs = kReduceThreads / a.row_threads;
    a.tile_blocks = (a.tiles + subs - 1) / subs;
    const long long blocks = (long long)a.tile_blocks * ((a.groups + a.row_threads - 1) / a.row_threads);
    if (blocks + a.zero_blocks > INT_MAX) return DPPF_ERR_INVALID_ARG;
    ok = ok && launch_after(embedding_reduce_kernel<TG, TW, N>, dim3((unsigned)(blocks + a.zero_blocks)), kReduceThreads, 0, s, a);
    const long long joins = (long long)((a.tiles + kJoinTiles - 1) / kJoinTiles) * ((a.groups + 31) / 32) + a.late_blocks;
    if (joins > INT_MAX) return DPPF_ERR_INVALID_ARG;
    ok = ok && launch_after(embedding_join_kernel<TW, N>, dim3((unsigned)joins), kJoinThreads, 0, s, a);
    if (!ok) { cudaGetLastError(); return DPPF_ERR_CUDA; }
    return DPPF_OK;
}
template <typename TG, typename TW>
int launch_grad_width(const GradArgs &a, int n, int dev, int sms, cudaStream_t s) {
    constexpr int kWide = 16 / sizeof(TG);
    return n == kWide ? launch_grad<TG, TW, kWide>(a, dev, sms, s) : n == 4 ? launch_grad<TG, TW, 4>(a, dev, sms, s) : n == 2 ? launch_grad<TG, TW, 2>(a, dev, sms, s) : launch_grad<TG, TW, 1>(a, dev, sms, s);
}

// ---------------------------------------------------------------- policy loss

constexpr size_t kPolicyHeaderBytes = 256;
constexpr int kPolicySliceMax = 200 * 1024;        // shared memory of one block's slice at most
// Six blocks and more fit an SM: some load while others write.  4,096 x 131,072 bf16, a quarter masked, in slices of 32 KB: 319 us,
// of 64 KB: 345 us; with 64 threads a block (slices of 32 KB) 352.
constexpr int kPolicySliceGood = 36 * 1024;

// Rows up to this size go to blocks of 64 threads (with a gradient, a quarter masked): 8,000 x 8,192 bf16 47 us (128 threads: 51),
// 10,000 x 4,096 37 (47); for rows of 32 KB 128 threads are quicker (8,000 x 16,384: 83 us, 90).
constexpr int kPolicyShortSlice = 24 * 1024;

std::atomic<int> g_policy_ready[2][kMaxDevices];

template <typename T>
int launch_policy(PolicyArgs a, int dev, cudaStream_t s) {
    std::atomic<int> *ready = g_policy_ready[sizeof(T) == 4 ? 0 : 1];
    if (!allow_smem(policy_kernel<T, kPolicyThreads>, dev, ready, kPolicySliceMax)) return DPPF_ERR_CUDA;
    const int sms = multiprocessors(dev);
    if (sms < 0) return DPPF_ERR_CUDA;
    // 16-byte vectors that a row spans: one more if rows may start inside one
    const int vectors = (int)(((size_t)a.V * sizeof(T) + 15) / 16) + (rows_on_16(a.logits, a.ld, sizeof(T) == 4 ? DPPF_FLOAT32 : DPPF_BFLOAT16) ? 0 : 1);
    if (vectors <= 8 * 32) {
        auto kernel = vectors <= 2 * 32 ? policy_short_kernel<T, 2> : vectors <= 4 * 32 ? policy_short_kernel<T, 4> : policy_short_kernel<T, 8>;
        const long long blocks = ((long long)a.T + kShortThreads / 32 - 1) / (kShortThreads / 32), most = 16LL * sms;
        kernel<<<(unsigned)(blocks < most ? blocks : most), kShortThreads, 0, s>>>(a);
        if (cudaPeekAtLastError() != cudaSuccess || !launch_after(policy_finish_kernel, dim3(3), kFinishThreads, 0, s, a)) { cudaGetLastError(); return DPPF_ERR_CUDA; }
        return DPPF_OK;
    }
    int C = 1;
    auto slice_bytes = [&](int c) { return (vectors + c - 1) / c * 16; };
    while (a.grad && C < kPolicyMaxCluster && slice_bytes(C) > kPolicySliceGood) C *= 2;
    // few rows: split them further while SMs are idle and a slice stays above 8 KB; rows that are only read also while
    // there are fewer than 8 blocks an SM and a slice stays above 16 KB (388 x 187,236 bf16: 36 us, 41 with 2)
    while (C < kPolicyMaxCluster && (((long long)a.T * C < 2LL * sms && slice_bytes(C) > 16 * 1024) ||
                                     (!a.grad && (long long)a.T * C < 8LL * sms && slice_bytes(C) > 32 * 1024))) C *= 2;
    a.slice = (vectors + C - 1) / C;
    // a slice in four chunks, in whole rounds of the block's threads; a longer one goes through the ring if it is not kept
    const bool shorter = C == 1 && a.slice * 16 <= kPolicyShortSlice;
    const int threads = shorter ? kPolicyShortThreads : kPolicyThreads;
    a.chunk = (a.slice + kPolicyChunks * threads - 1) / (kPolicyChunks * threads) * threads;
    if (!a.grad && a.chunk > kPolicyRing) a.chunk = kPolicyRing;
    const int held = a.slice < kPolicyChunks * a.chunk ? a.slice : kPolicyChunks * a.chunk;
    if (held * 16 > kPolicySliceMax) return DPPF_ERR_INVALID_ARG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.T * (unsigned)C);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)held * 16;
    cfg.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)C;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = C > 1 ? 1 : 0;                                // a cluster of one starts slower than a plain block
    if (cudaLaunchKernelEx(&cfg, shorter ? policy_kernel<T, kPolicyShortThreads> : policy_kernel<T, kPolicyThreads>, a) != cudaSuccess || !launch_after(policy_finish_kernel, dim3(3), kFinishThreads, 0, s, a)) {
        cudaGetLastError();
        return DPPF_ERR_CUDA;
    }
    return DPPF_OK;
}

// ---------------------------------------------------------------- AdamW over many tensors

int64_t units_of(int64_t n) { return (n + kStateBlock - 1) / kStateBlock; }

template <typename TP, typename TG, int kBits, int kEntries>
int launch_tensors(TensorTable<kEntries> &tab, int sms, cudaStream_t s) {
    constexpr int kBlocks = TensorShape<TP, TG, kBits>::kBlocks;
    const long long most = (long long)sms * kBlocks;                 // blocks that are resident
    tab.groups = 0;
    if (kBits == 8) {
        auto groups_of = [](const TensorEntry &e) { return codes_on_8(e) ? (int)(e.n / (kStateBlock * kGroup)) : 0; };
        long long groups = 0;
        for (int k = 0; k < tab.n; ++k) groups += groups_of(tab.e[k]);
        const bool grouped = groups >= most * kTensorWarps;          // every warp gets one
        tab.units = 0;
        for (int k = 0; k < tab.n; ++k) {
            TensorEntry &e = tab.e[k];
            const int mine = grouped ? groups_of(e) : 0;
            e.first_unit = tab.units;
            e.first_group = tab.groups;
            tab.units += (int)units_of(e.n) - mine * kGroup;
            tab.groups += mine;
        }
    }
    const long long warps = (long long)tab.units + tab.groups, blocks = (warps + kTensorWarps - 1) / kTensorWarps;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    if (kBits == 32 || sqrt2_is_enough(tab.args.eps, tab.args.inv_sqrt_bc2)) adamw_tensors_kernel<TP, TG, kBits, false, kEntries><<<grid, kTensorThreads, 0, s>>>(tab);
    else adamw_tensors_kernel<TP, TG, kBits, kBits == 8, kEntries><<<grid, kTensorThreads, 0, s>>>(tab);
    return launched();
}
template <int kEntries>
int launch_tensors_types(TensorTable<kEntries> &tab, int tp, int tg, int bits, int sms, cudaStream_t s) {
#define DPPF_TENSORS(P, G) \
    return bits == 8 ? launch_tensors<P, G, 8, kEntries>(tab, sms, s) : launch_tensors<P, G, 32, kEntries>(tab, sms, s)
    if (tp == DPPF_FLOAT32 && tg == DPPF_FLOAT32) DPPF_TENSORS(float, float);
    if (tp == DPPF_FLOAT32) DPPF_TENSORS(float, bf16);
    if (tg == DPPF_FLOAT32) DPPF_TENSORS(bf16, float);
    DPPF_TENSORS(bf16, bf16);
#undef DPPF_TENSORS
}

struct TensorScalars {
    const float *grad_scale;
    AdamArgs args;
    float b1, lr, wd;
    unsigned seed_term;
    int tp, tg, bits;
};

// Elements (0 .. 255) by which units have to begin before the tensor so that they lie on multiples of their own size (else
// of 16 bytes) in the parameter, the gradient and both fp32 moments; -1 if no number does.
int common_lead(const dppf_tensor &t, int tp, int tg) {
    const void *p[4] = {t.param, t.grad, t.exp_avg, t.exp_avg_sq};
    const int type[4] = {tp, tg, DPPF_FLOAT32, DPPF_FLOAT32};
    auto at = [&](int i) { return reinterpret_cast<uintptr_t>(p[i]) / type_bytes(type[i]); };   // in elements
    auto fits = [&](uintptr_t lead, bool units) {
        for (int i = 0; i < 4; ++i)
            if ((at(i) - lead) % (units ? kStateBlock : 16 / type_bytes(type[i])) != 0) return false;
        return true;
    };
    const uintptr_t lead = at(0) % kStateBlock, small = at(tp == DPPF_BFLOAT16 ? 0 : tg == DPPF_BFLOAT16 ? 1 : 2) % 8;
    return fits(lead, true) ? (int)lead : fits(small, false) ? (int)small : -1;
}

// Tensors [first, last) as one launch, or as many as the table and the unit count allow.
template <int kEntries>
int launch_table(const dppf_tensor *ts, int first, int last, const TensorScalars &p, int sms, cudaStream_t s) {
    TensorTable<kEntries> tab;
    tab.grad_scale = p.grad_scale;
    tab.args = p.args;
    tab.b1 = p.b1;
    tab.seed_term = p.seed_term;
    int k = first;
    while (k < last) {
        tab.n = 0;
        int64_t units = 0;
        for (; k < last && tab.n < kEntries; ++k) {
            const dppf_tensor &t = ts[k];
            if (t.numel == 0) continue;
            const int lead = p.bits == 8 ? 0 : common_lead(t, p.tp, p.tg);
            const int64_t more = units_of(t.numel + (lead > 0 ? lead : 0));
            if (units + more > INT_MAX / 2 && tab.n) break;
            TensorEntry &e = tab.e[tab.n++];
            e.param = t.param; e.grad = t.grad; e.m = t.exp_avg; e.v = t.exp_avg_sq;
            e.m_scale = t.exp_avg_scale; e.v_scale = t.exp_avg_sq_scale;
            e.n = t.numel;
            e.decay = (float)(1.0 - (double)p.lr * (double)p.wd * (double)t.decay);
            e.first_unit = (int)units;
            e.lead = lead;
            units += more;
        }
        if (tab.n == 0) break;
        tab.units = (int)units;
        const int rc = launch_tensors_types<kEntries>(tab, p.tp, p.tg, p.bits, sms, s);
        if (rc != DPPF_OK) return rc;
    }
    return DPPF_OK;
}

}  // namespace

extern "C" {

int dppf_embedding(const void *table, int table_type, int64_t V, int H, int64_t ld_table, const void *ids, int id_bits, int64_t T,
                   float scale, void *out, int out_type, int64_t ld_out, void *cuda_stream) {
    if (!known_type(table_type) || !known_type(out_type) || (id_bits != 32 && id_bits != 64)) return DPPF_ERR_INVALID_ARG;
    if (V < 1 || V > INT_MAX - 1 || H < 1 || H > DPPF_MAX_WIDTH || T < 0 || T > INT_MAX || ld_table < H || ld_out < H || ld_table > kMaxLd || ld_out > kMaxLd ||
        !std::isfinite(scale))
        return DPPF_ERR_INVALID_ARG;
    if (T == 0) return DPPF_OK;
    if (!table || !ids || !out) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(table, type_bytes(table_type)) || !aligned_to(out, type_bytes(out_type)) || !aligned_to(ids, id_bits / 8)) return DPPF_ERR_ALIGNMENT;
    const size_t out_bytes = matrix_bytes(T, H, ld_out, out_type);
    if (ranges_meet(out, out_bytes, table, matrix_bytes(V, H, ld_table, table_type)) || ranges_meet(out, out_bytes, ids, (size_t)T * (id_bits / 8)))
        return DPPF_ERR_INVALID_ARG;
    const int dev = current_device(), sms = dev < 0 ? -1 : multiprocessors(dev);
    if (sms < 0) return DPPF_ERR_CUDA;
    LookupArgs a;
    a.table = table; a.ids = ids; a.out = out;
    a.ld_table = ld_table; a.ld_out = ld_out; a.T = T; a.V = V; a.H = H; a.ids64 = id_bits == 64;
    a.scale = scale;
    const int n = group_width(H, out_type == DPPF_BFLOAT16 ? 8 : 4, table, ld_table, table_type, out, ld_out, out_type);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (table_type == DPPF_FLOAT32) return out_type == DPPF_FLOAT32 ? launch_lookup<float, float>(a, n, sms, s) : launch_lookup<float, bf16>(a, n, sms, s);
    return out_type == DPPF_FLOAT32 ? launch_lookup<bf16, float>(a, n, sms, s) : launch_lookup<bf16, bf16>(a, n, sms, s);
}

size_t dppf_embedding_workspace_bytes(int64_t T, int H) {
    if (T < 1 || T > INT_MAX || H < 1 || H > DPPF_MAX_WIDTH) return 0;
    return embedding_layout(T, H).total;
}

int dppf_embedding_grad(const void *grad_out, int out_type, int64_t ld_out, const void *ids, int id_bits, int64_t T, float scale,
                        void *grad_table, int table_type, int64_t V, int H, int64_t ld_table, int accumulate, void *ws,
                        size_t ws_bytes, void *cuda_stream) {
    if (!known_type(table_type) || !known_type(out_type) || (id_bits != 32 && id_bits != 64)) return DPPF_ERR_INVALID_ARG;
    if (V < 1 || V > INT_MAX - 1 || H < 1 || H > DPPF_MAX_WIDTH || T < 0 || T > INT_MAX || ld_table < H || ld_out < H || ld_table > kMaxLd || ld_out > kMaxLd ||
        !std::isfinite(scale))
        return DPPF_ERR_INVALID_ARG;
    if (!grad_table) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(grad_table, type_bytes(table_type))) return DPPF_ERR_ALIGNMENT;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (T == 0) {
        if (accumulate) return DPPF_OK;
        return cudaMemset2DAsync(grad_table, (size_t)ld_table * type_bytes(table_type), 0, (size_t)H * type_bytes(table_type), (size_t)V, s) == cudaSuccess
                   ? DPPF_OK : DPPF_ERR_CUDA;
    }
    if (!grad_out || !ids || !ws) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(grad_out, type_bytes(out_type)) || !aligned_to(ids, id_bits / 8) || !aligned_to(ws, 128)) return DPPF_ERR_ALIGNMENT;
    const EmbeddingLayout l = embedding_layout(T, H);
    if (ws_bytes < l.total) return DPPF_ERR_WORKSPACE;
    const size_t table_bytes = matrix_bytes(V, H, ld_table, table_type), out_bytes = matrix_bytes(T, H, ld_out, out_type), id_bytes = (size_t)T * (id_bits / 8);
    if (ranges_meet(grad_table, table_bytes, grad_out, out_bytes) || ranges_meet(grad_table, table_bytes, ids, id_bytes) ||
        ranges_meet(ws, l.total, grad_table, table_bytes) || ranges_meet(ws, l.total, grad_out, out_bytes) || ranges_meet(ws, l.total, ids, id_bytes))
        return DPPF_ERR_INVALID_ARG;
    const int dev = current_device();
    if (dev < 0) return DPPF_ERR_CUDA;
    const int sms = multiprocessors(dev);
    if (sms < 0) return DPPF_ERR_CUDA;
    GradArgs a = {};
    a.ids = ids; a.ids64 = id_bits == 64;
    a.T = (unsigned)T; a.V = (unsigned)V; a.H = H;
    a.dout = grad_out; a.dtable = grad_table;
    a.ld_dout = ld_out; a.ld_dtable = ld_table;
    a.add = accumulate ? 1 : 0;
    a.scale = scale;
    unsigned char *base = static_cast<unsigned char *>(ws);
    a.order0 = reinterpret_cast<uint2 *>(base + l.order[0]);
    a.order1 = reinterpret_cast<uint2 *>(base + l.order[1]);
    a.hist = reinterpret_cast<unsigned *>(base + l.hist);
    a.part = reinterpret_cast<float *>(base + l.part);
    int bits = 1;
    while (((int64_t)1 << bits) <= V) ++bits;                    // keys 0 .. V
    a.passes = (bits + kDigitBits - 1) / kDigitBits;
    a.bits = (bits + a.passes - 1) / a.passes;
    a.zero_vec = rows_on_16(grad_table, ld_table, table_type) && (size_t)H * type_bytes(table_type) % 16 == 0;
    const int n = group_width(H, out_type == DPPF_BFLOAT16 ? 8 : 4, grad_out, ld_out, out_type, grad_table, ld_table, table_type);
    if (out_type == DPPF_FLOAT32)
        return table_type == DPPF_FLOAT32 ? launch_grad_width<float, float>(a, n, dev, sms, s) : launch_grad_width<float, bf16>(a, n, dev, sms, s);
    return table_type == DPPF_FLOAT32 ? launch_grad_width<bf16, float>(a, n, dev, sms, s) : launch_grad_width<bf16, bf16>(a, n, dev, sms, s);
}

size_t dppf_policy_workspace_bytes(int64_t T) {
    if (T < 1 || T > DPPF_MAX_POLICY_TOKENS) return 0;
    return kPolicyHeaderBytes + round256((size_t)T * 3 * sizeof(float));
}

int dppf_policy_loss(const void *logits, int type, int64_t T, int V, int64_t ld, const void *targets, int target_bits,
                     const float *old_logp, const float *ref_logp, const float *advantage, const float *weight, float clip_low,
                     float clip_high, float kl_coef, float temperature, float *sums_out, float *logp_out, void *grad_logits,
                     int64_t ld_grad, void *ws, size_t ws_bytes, void *cuda_stream) {
    if (!known_type(type) || (target_bits != 32 && target_bits != 64)) return DPPF_ERR_INVALID_ARG;
    if (T < 1 || T > DPPF_MAX_POLICY_TOKENS || V < 1 || V > DPPF_MAX_VOCABULARY || ld < V || ld > kMaxLd) return DPPF_ERR_INVALID_ARG;
    if (grad_logits && (ld_grad < V || ld_grad > kMaxLd)) return DPPF_ERR_INVALID_ARG;
    if (!all_finite({clip_low, clip_high, kl_coef, temperature}) || clip_low < 0.f || clip_low > 1.f || clip_high < 0.f || !(temperature > 0.f) ||
        1.4426950408889634 / (double)temperature > (double)FLT_MAX)         // neither that nor 1 / temperature is an fp32 number
        return DPPF_ERR_INVALID_ARG;
    if (!logits || !targets || !old_logp || !advantage || !weight || !sums_out || !logp_out || !ws) return DPPF_ERR_INVALID_ARG;
    if (kl_coef != 0.f && !ref_logp) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(logits, type_bytes(type)) || !aligned_to(grad_logits, type_bytes(type)) || !aligned_to(targets, target_bits / 8) || !aligned_to(ws, 128) ||
        !aligned_to(old_logp, 4) || !aligned_to(ref_logp, 4) || !aligned_to(advantage, 4) || !aligned_to(weight, 4) || !aligned_to(sums_out, 4) ||
        !aligned_to(logp_out, 4))
        return DPPF_ERR_ALIGNMENT;
    const size_t need = dppf_policy_workspace_bytes(T);
    if (ws_bytes < need) return DPPF_ERR_WORKSPACE;
    const size_t in_bytes = matrix_bytes(T, V, ld, type), grad_bytes = grad_logits ? matrix_bytes(T, V, ld_grad, type) : 0, row = (size_t)T * 4;
    const bool in_place = grad_logits == logits && ld_grad == ld;
    if (!in_place && ranges_meet(grad_logits, grad_bytes, logits, in_bytes)) return DPPF_ERR_INVALID_ARG;
    struct Range { const void *p; size_t n; };
    const Range written[] = {{grad_logits, grad_bytes}, {logp_out, row}, {sums_out, 12}, {ws, need}};
    const Range read[] = {{targets, (size_t)T * (target_bits / 8)}, {old_logp, row}, {ref_logp, row}, {advantage, row}, {weight, row}};
    for (int i = 0; i < 4; ++i) {
        for (const Range &r : read)
            if (ranges_meet(written[i].p, written[i].n, r.p, r.n)) return DPPF_ERR_INVALID_ARG;
        for (int k = 0; k < i; ++k)
            if (ranges_meet(written[i].p, written[i].n, written[k].p, written[k].n)) return DPPF_ERR_INVALID_ARG;
        if (i > 0 && ranges_meet(written[i].p, written[i].n, logits, in_bytes)) return DPPF_ERR_INVALID_ARG;
    }
    const int dev = current_device();
    if (dev < 0) return DPPF_ERR_CUDA;
    PolicyArgs a;
    a.logits = logits; a.grad = grad_logits; a.ld = ld; a.ld_grad = ld_grad;
    a.targets = targets; a.targets64 = target_bits == 64;
    a.old_logp = old_logp; a.ref_logp = ref_logp; a.advantage = advantage; a.weight = weight;
    a.logp = logp_out; a.sums = sums_out;
    a.hdr = reinterpret_cast<PolicyHeader *>(ws);
    a.terms = reinterpret_cast<float *>(static_cast<unsigned char *>(ws) + kPolicyHeaderBytes);
    a.T = (int)T; a.V = V; a.slice = 0;
    a.spin = dppf_internal::first_pass_polls();
    a.clip_lo = (float)(1.0 - (double)clip_low);
    a.clip_hi = (float)(1.0 + (double)clip_high);
    a.kl_coef = kl_coef;
    const double log2e_t = 1.4426950408889634 / (double)temperature;
    a.log2e_t = a.log2e_t_near = (float)log2e_t;
    if ((double)a.log2e_t >= log2e_t) a.log2e_t = std::nextafterf(a.log2e_t, 0.f);
    a.log2e_t_rest = (float)(log2e_t - (double)a.log2e_t);
    if (a.log2e_t_rest == 0.f) a.log2e_t_rest = std::numeric_limits<float>::denorm_min();   // 0 * -inf would be NaN
    a.inv_t = (float)(1.0 / (double)temperature);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return type == DPPF_FLOAT32 ? launch_policy<float>(a, dev, s) : launch_policy<bf16>(a, dev, s);
}

int dppf_adamw_tensors(const dppf_tensor *tensors_host, int n_tensors, int param_type, int grad_type, int state_bits, float lr,
                       float beta1, float beta2, float eps, float weight_decay, int step, const float *grad_scale, uint32_t seed,
                       void *cuda_stream) {
    if (n_tensors < 0 || (n_tensors && !tensors_host) || !known_type(param_type) || !known_type(grad_type) || (state_bits != 8 && state_bits != 32))
        return DPPF_ERR_INVALID_ARG;
    if (!all_finite({lr, beta1, beta2, eps, weight_decay}) || step < 1) return DPPF_ERR_INVALID_ARG;
    if (!(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f)) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(grad_scale, 4)) return DPPF_ERR_ALIGNMENT;
    int present = 0;
    for (int k = 0; k < n_tensors; ++k) {
        const dppf_tensor &t = tensors_host[k];
        if (t.numel < 0 || t.numel > ((int64_t)1 << 37) || !std::isfinite(t.decay)) return DPPF_ERR_INVALID_ARG;
        if (t.numel == 0) continue;
        ++present;
        const size_t n = (size_t)t.numel, scales = state_bits == 8 ? (n + kStateBlock - 1) / kStateBlock * 4 : 0;
        if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq) return DPPF_ERR_INVALID_ARG;
        if (state_bits == 8 && (!t.exp_avg_scale || !t.exp_avg_sq_scale)) return DPPF_ERR_INVALID_ARG;
        if (!aligned_to(t.param, type_bytes(param_type)) || !aligned_to(t.grad, type_bytes(grad_type))) return DPPF_ERR_ALIGNMENT;
        if (state_bits == 32 ? !aligned_to(t.exp_avg, 4) || !aligned_to(t.exp_avg_sq, 4) : !aligned_to(t.exp_avg_scale, 4) || !aligned_to(t.exp_avg_sq_scale, 4))
            return DPPF_ERR_ALIGNMENT;
        const size_t state = n * (size_t)(state_bits / 8);
        const void *p[6] = {t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale};
        const size_t b[6] = {n * type_bytes(param_type), n * type_bytes(grad_type), state, state, scales, scales};
        for (int i = 0; i < 6; ++i)
            for (int j = 0; j < i; ++j)
                if (ranges_meet(p[i], b[i], p[j], b[j])) return DPPF_ERR_INVALID_ARG;
    }
    if (present == 0) return DPPF_OK;
    const int dev = current_device();
    const int sms = dev < 0 ? -1 : multiprocessors(dev);
    if (sms < 0) return DPPF_ERR_CUDA;
    TensorScalars p;
    p.grad_scale = grad_scale;
    const double bc1 = 1.0 - std::pow((double)beta1, (double)step), bc2 = 1.0 - std::pow((double)beta2, (double)step);
    p.args.m1 = p.args.m2 = nullptr;
    p.args.g = nullptr;
    p.args.decay = 0.f;                                          // each tensor's own
    p.args.one_minus_b1 = (float)(1.0 - (double)beta1);
    p.args.b2 = beta2;
    p.args.one_minus_b2 = (float)(1.0 - (double)beta2);
    p.args.step_size = (float)((double)lr / bc1);
    p.args.inv_sqrt_bc2 = (float)(1.0 / std::sqrt(bc2));
    p.args.eps = eps;
    p.b1 = beta1; p.lr = lr; p.wd = weight_decay;
    p.seed_term = seed * 0x9e3779b9u;
    p.tp = param_type; p.tg = grad_type; p.bits = state_bits;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (present <= kSmallTable) return launch_table<kSmallTable>(tensors_host, 0, n_tensors, p, sms, s);
    return launch_table<kLargeTable>(tensors_host, 0, n_tensors, p, sms, s);
}

}  // extern "C"
