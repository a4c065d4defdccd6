// Attention within packed sequences: host side and C ABI (include/dppf.h).
//   tensor_core.cuh    tensor copies, products with sums in tensor memory, bounded waits
//   attention.cuh      the plan of a batch and the kernels
//   local_host.cuh     devices, launches, checks of arguments
#include "dppf.h"

#include "attention.cuh"
#include "local_host.cuh"
#include <algorithm>

namespace {

constexpr int64_t kMaxStride = (int64_t)1 << 38;

struct PlanLayout {
    int most[kPlanLists];
    size_t bounds, count, list[kPlanLists], total;
};
PlanLayout plan_layout(int64_t T, int64_t B) {
    PlanLayout l;
    size_t at = 256;
    l.bounds = at;
    at += round256((size_t)(B + 1) * sizeof(int));
    l.count = at;
    at += round256((size_t)(B + 1) * sizeof(int));
    for (int i = 0; i < kPlanLists; ++i) {
        const int64_t size = i == kByQuery2 ? 2 * kTile : kTile;
        l.most[i] = (int)(T / size + (B < T ? B : T) + 4);       // a part of a tile for each sequence that is not empty, and at both ends
        l.list[i] = at;
        at += round256((size_t)l.most[i] * sizeof(PlanTile));
    }
    l.total = at;
    return l;
}
bool plan_shape(int64_t T, int64_t B) { return T >= 0 && T <= DPPF_MAX_ATTENTION_TOKENS && B >= 1 && B <= DPPF_MAX_SEQUENCES; }

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static std::atomic<void *> known;
    void *fn = known.load(std::memory_order_relaxed);
    if (!fn) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
        known.store(fn, std::memory_order_relaxed);
    }
    return reinterpret_cast<EncodeTiled>(fn);
}
// The heads as a tensor [T][heads][D], copied in boxes of 128 rows by 64 columns of a head.
bool heads_map(CUtensorMap *map, const HeadRows &h) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)h.D, (cuuint64_t)h.heads, (cuuint64_t)h.T};
    const cuuint64_t strides[2] = {(cuuint64_t)(h.heads > 1 ? h.head : h.D) * 2, (cuuint64_t)h.ld * 2};     // a single head's may be 0
    const cuuint32_t box[3] = {64, 1, kTile}, one[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(h.p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows of heads as the kernels take them: bf16, strides and starts on 16 bytes.
bool heads_aligned(const HeadRows &h) { return aligned_to(h.p, 16) && h.ld % 8 == 0 && h.head % 8 == 0; }
bool heads_strides(const HeadRows &h) { return h.ld <= kMaxStride && h.head <= kMaxStride && h.apart(); }

struct AttentionShape {
    int64_t T, B;
    int heads, kv_heads, D, causal, window;
    float scale;
    bool fine() const {
        return plan_shape(T, B) && heads >= 1 && heads <= DPPF_MAX_HEADS && kv_heads >= 1 && heads % kv_heads == 0 && D >= 8 && D <= DPPF_MAX_ATTENTION_WIDTH && D % 8 == 0 &&
               (causal == 0 || causal == 1) && window >= 0 && (window == 0 || causal) && std::isfinite((float)((double)scale * 1.4426950408889634)) && scale > 0.f;
    }
};

std::atomic<int> g_forward_ready[3][kMaxDevices];

template <int kSteps>
int launch_attention(const AttentionArgs &a, long long blocks, int dev, cudaStream_t s) {
    constexpr int kSmem = (int)ForwardShape<kSteps>::kSmem;
    if (!allow_smem(attention_kernel<kSteps>, dev, g_forward_ready[kSteps / 2 - 2], kSmem)) return DPPF_ERR_CUDA;
    const int sms = multiprocessors(dev);
    if (sms < 0) return DPPF_ERR_CUDA;
    attention_kernel<kSteps><<<(unsigned)(blocks < sms ? blocks : sms), kForwardThreads, kSmem, s>>>(a);
    return launched();
}

// Parts that the heads of a key head are dealt out to: where tiles of keys are fewer than the SMs (148, whatever the device: the workspace
// is laid out by this, and its size is asked for without one), as many as give each SM one, and no more than there are heads.
int grad_splits(int64_t T, int kv_heads, int share) {
    const int64_t tiles = (T + kTile - 1) / kTile * kv_heads, want = (148 + tiles - 1) / tiles;
    return (int)(tiles >= 148 ? 1 : want < share ? want : share);
}
// Rows of parts at most: of splits kv_heads T, with splits kv_heads <= heads, and splits tiles < 148 + tiles where there are parts at all.
int64_t grad_part_rows(int64_t T, int heads) { return T * heads < 2 * 148 * kTile ? T * heads : 2 * 148 * kTile; }

std::atomic<int> g_query_ready[3][kMaxDevices], g_key_ready[3][kMaxDevices];

template <int kSteps>
int launch_attention_grad(const AttentionGradArgs &a, long long query_blocks, long long key_blocks, int dev, cudaStream_t s) {
    constexpr int kQuerySmem = (int)QueryGradShape<kSteps>::kSmem, kKeySmem = (int)KeyGradShape<kSteps>::kSmem;
    if (!allow_smem(attention_grad_query_kernel<kSteps>, dev, g_query_ready[kSteps / 2 - 2], kQuerySmem) || !allow_smem(attention_grad_key_kernel<kSteps>, dev, g_key_ready[kSteps / 2 - 2], kKeySmem))
        return DPPF_ERR_CUDA;
    attention_grad_query_kernel<kSteps><<<(unsigned)query_blocks, kGradThreads, kQuerySmem, s>>>(a);
    if (cudaPeekAtLastError() == cudaSuccess) attention_grad_key_kernel<kSteps><<<(unsigned)key_blocks, kGradThreads, kKeySmem, s>>>(a);
    if (a.splits > 1 && cudaPeekAtLastError() == cudaSuccess) {
        const long long pieces = a.kv_heads * a.T * (a.D / 8);
        attention_grad_join_kernel<<<dim3((unsigned)((pieces + kJoinThreads - 1) / kJoinThreads), 2), kJoinThreads, 0, s>>>(a);
    }
    return launched();
}

}  // namespace

extern "C" {

size_t dppf_attention_plan_bytes(int64_t T, int64_t B) { return plan_shape(T, B) ? plan_layout(T, B).total : 0; }

int dppf_attention_plan(const void *starts, int start_bits, int64_t T, int64_t B, void *plan, size_t plan_bytes, void *cuda_stream) {
    if ((start_bits != 32 && start_bits != 64) || !plan_shape(T, B) || !starts || !plan) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(starts, start_bits / 8) || !aligned_to(plan, 128)) return DPPF_ERR_ALIGNMENT;
    const PlanLayout l = plan_layout(T, B);
    if (plan_bytes < l.total) return DPPF_ERR_WORKSPACE;
    if (ranges_meet(starts, (size_t)(B + 1) * (start_bits / 8), plan, l.total)) return DPPF_ERR_INVALID_ARG;
    unsigned char *base = static_cast<unsigned char *>(plan);
    PlanArgs a = {};
    a.starts = starts; a.starts64 = start_bits == 64; a.T = T; a.B = (int)B;
    a.hdr = reinterpret_cast<PlanHeader *>(base);
    a.bounds = reinterpret_cast<int *>(base + l.bounds);
    a.count = reinterpret_cast<int *>(base + l.count);
    for (int i = 0; i < kPlanLists; ++i) {
        a.list[i] = reinterpret_cast<PlanTile *>(base + l.list[i]);
        a.most[i] = l.most[i];
    }
    attention_plan_kernel<<<1, kPlanThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    return launched();
}

int dppf_attention(const void *q, int64_t ld_q, int64_t head_q, const void *k, int64_t ld_k, int64_t head_k, const void *v, int64_t ld_v, int64_t head_v,
                   int64_t T, int64_t B, int heads, int kv_heads, int D, int causal, int window, float scale, void *out, int64_t ld_out, int64_t head_out,
                   float *lse_out, void *plan, size_t plan_bytes, void *cuda_stream) {
    const AttentionShape shape = {T, B, heads, kv_heads, D, causal, window, scale};
    if (!shape.fine()) return DPPF_ERR_INVALID_ARG;
    if (T == 0) return DPPF_OK;
    const HeadRows hq = {q, ld_q, head_q, T, heads, D, DPPF_BFLOAT16}, hk = {k, ld_k, head_k, T, kv_heads, D, DPPF_BFLOAT16}, hv = {v, ld_v, head_v, T, kv_heads, D, DPPF_BFLOAT16},
                   ho = {out, ld_out, head_out, T, heads, D, DPPF_BFLOAT16};
    if (!q || !k || !v || !out || !lse_out || !plan) return DPPF_ERR_INVALID_ARG;
    if (!heads_strides(hq) || !heads_strides(hk) || !heads_strides(hv) || !heads_strides(ho)) return DPPF_ERR_INVALID_ARG;
    if (!heads_aligned(hq) || !heads_aligned(hk) || !heads_aligned(hv) || !heads_aligned(ho) || !aligned_to(lse_out, 4) || !aligned_to(plan, 128)) return DPPF_ERR_ALIGNMENT;
    const PlanLayout l = plan_layout(T, B);
    if (plan_bytes < l.total) return DPPF_ERR_WORKSPACE;
    const size_t lse_bytes = (size_t)heads * (size_t)T * 4;
    for (const HeadRows *h : {&hq, &hk, &hv})
        if (ho.meets(*h) || ranges_meet(h->p, h->bytes(), lse_out, lse_bytes)) return DPPF_ERR_INVALID_ARG;
    if (ranges_meet(ho.p, ho.bytes(), lse_out, lse_bytes) || ranges_meet(plan, l.total, lse_out, lse_bytes) || ranges_meet(plan, l.total, ho.p, ho.bytes())) return DPPF_ERR_INVALID_ARG;
    const int dev = current_device();
    if (dev < 0) return DPPF_ERR_CUDA;
    AttentionArgs a;
    if (!heads_map(&a.q, hq) || !heads_map(&a.k, hk) || !heads_map(&a.v, hv)) return DPPF_ERR_CUDA;
    unsigned char *base = static_cast<unsigned char *>(plan);
    a.hdr = reinterpret_cast<PlanHeader *>(base);
    a.share = heads / kv_heads;
    a.by_head = a.share % 2 == 0;                 // two heads of the same keys do equal work, whatever the lengths
    a.list = a.by_head ? kByQuery : kByQuery2;
    a.units = a.by_head ? heads / 2 : heads;
    a.tiles = reinterpret_cast<const PlanTile *>(base + l.list[a.list]);
    a.out = static_cast<bf16 *>(out);
    a.lse = lse_out;
    a.ld_out = ld_out; a.head_out = head_out; a.T = T;
    a.D = D; a.B = (int)B;
    a.causal = causal; a.window = window < T ? window : 0;
    a.scale2 = (float)((double)scale * 1.4426950408889634);
    a.spin = dppf_internal::first_pass_polls();
    const long long blocks = (long long)a.units * l.most[a.list];
    if (blocks > INT_MAX) return DPPF_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    // heads as wide as 64, 96 or 128: what a product sums over, or has as columns
    return D <= 64 ? launch_attention<4>(a, blocks, dev, s) : D <= 96 ? launch_attention<6>(a, blocks, dev, s) : launch_attention<8>(a, blocks, dev, s);
}

size_t dppf_attention_workspace_bytes(int64_t T, int heads) {
    return T >= 1 && T <= DPPF_MAX_ATTENTION_TOKENS && heads >= 1 && heads <= DPPF_MAX_HEADS 
               ? round256((size_t)T * (size_t)heads * sizeof(float)) + (size_t)grad_part_rows(T, heads) * 2 * DPPF_MAX_ATTENTION_WIDTH * sizeof(float) : 0;
}

int dppf_attention_grad(const void *grad_out, int64_t ld_grad_out, int64_t head_grad_out, const void *q, int64_t ld_q, int64_t head_q, const void *k, int64_t ld_k,
                        int64_t head_k, const void *v, int64_t ld_v, int64_t head_v, const void *out, int64_t ld_out, int64_t head_out, const float *lse, int64_t T,
                        int64_t B, int heads, int kv_heads, int D, int causal, int window, float scale, void *grad_q, int64_t ld_grad_q, int64_t head_grad_q,
                        void *grad_k, int64_t ld_grad_k, int64_t head_grad_k, void *grad_v, int64_t ld_grad_v, int64_t head_grad_v, void *plan, size_t plan_bytes,
                        void *ws, size_t ws_bytes, void *cuda_stream) {
    const AttentionShape shape = {T, B, heads, kv_heads, D, causal, window, scale};
    if (!shape.fine()) return DPPF_ERR_INVALID_ARG;
    if (T == 0) return DPPF_OK;
    const HeadRows in[] = {{grad_out, ld_grad_out, head_grad_out, T, heads, D, DPPF_BFLOAT16}, {q, ld_q, head_q, T, heads, D, DPPF_BFLOAT16}, {k, ld_k, head_k, T, kv_heads, D, DPPF_BFLOAT16},
                           {v, ld_v, head_v, T, kv_heads, D, DPPF_BFLOAT16}, {out, ld_out, head_out, T, heads, D, DPPF_BFLOAT16}};
    const HeadRows written[] = {{grad_q, ld_grad_q, head_grad_q, T, heads, D, DPPF_BFLOAT16}, {grad_k, ld_grad_k, head_grad_k, T, kv_heads, D, DPPF_BFLOAT16},
                                {grad_v, ld_grad_v, head_grad_v, T, kv_heads, D, DPPF_BFLOAT16}};
    if (!lse || !plan || !ws) return DPPF_ERR_INVALID_ARG;
    for (const HeadRows &h : in)
        if (!h.p || !heads_strides(h)) return DPPF_ERR_INVALID_ARG;
    for (const HeadRows &h : written)
        if (!h.p || !heads_strides(h)) return DPPF_ERR_INVALID_ARG;
    for (const HeadRows &h : in)
        if (!heads_aligned(h)) return DPPF_ERR_ALIGNMENT;
    for (const HeadRows &h : written)
        if (!heads_aligned(h)) return DPPF_ERR_ALIGNMENT;
    if (!aligned_to(lse, 4) || !aligned_to(plan, 128) || !aligned_to(ws, 128)) return DPPF_ERR_ALIGNMENT;
    const PlanLayout l = plan_layout(T, B);
    const size_t need = dppf_attention_workspace_bytes(T, heads), lse_bytes = (size_t)heads * (size_t)T * 4;
    if (plan_bytes < l.total || ws_bytes < need) return DPPF_ERR_WORKSPACE;
    for (int i = 0; i < 3; ++i) {
        for (const HeadRows &h : in)
            if (written[i].meets(h)) return DPPF_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (written[i].meets(written[j])) return DPPF_ERR_INVALID_ARG;
        const void *p = written[i].p;
        const size_t n = written[i].bytes();
        if (ranges_meet(p, n, lse, lse_bytes) || ranges_meet(p, n, plan, l.total) || ranges_meet(p, n, ws, need)) return DPPF_ERR_INVALID_ARG;
    }
    for (const HeadRows &h : in)
        if (ranges_meet(h.p, h.bytes(), ws, need)) return DPPF_ERR_INVALID_ARG;
    if (ranges_meet(ws, need, lse, lse_bytes) || ranges_meet(ws, need, plan, l.total)) return DPPF_ERR_INVALID_ARG;
    const int dev = current_device();
    if (dev < 0) return DPPF_ERR_CUDA;
    AttentionGradArgs a;
    if (!heads_map(&a.grad_out, in[0]) || !heads_map(&a.q, in[1]) || !heads_map(&a.k, in[2]) || !heads_map(&a.v, in[3]) || !heads_map(&a.out, in[4])) return DPPF_ERR_CUDA;
    unsigned char *base = static_cast<unsigned char *>(plan);
    a.hdr = reinterpret_cast<PlanHeader *>(base);
    a.query_tiles = reinterpret_cast<const PlanTile *>(base + l.list[kByQuery]);
    a.key_tiles = reinterpret_cast<const PlanTile *>(base + l.list[kByKey]);
    a.lse = lse; a.delta = static_cast<float *>(ws);
    a.part = reinterpret_cast<float *>(static_cast<unsigned char *>(ws) + round256((size_t)T * (size_t)heads * sizeof(float)));
    a.splits = grad_splits(T, kv_heads, heads / kv_heads);
    a.dq = static_cast<bf16 *>(grad_q); a.dk = static_cast<bf16 *>(grad_k); a.dv = static_cast<bf16 *>(grad_v);
    a.ld_dq = ld_grad_q; a.head_dq = head_grad_q; a.ld_dk = ld_grad_k; a.head_dk = head_grad_k; a.ld_dv = ld_grad_v; a.head_dv = head_grad_v;
    a.T = T; a.heads = heads; a.kv_heads = kv_heads; a.share = heads / kv_heads; a.D = D; a.B = (int)B;
    a.causal = causal; a.window = window < T ? window : 0;
    a.scale = scale;
    a.scale2 = (float)((double)scale * 1.4426950408889634);
    a.spin = dppf_internal::first_pass_polls();
    a.spin_query = std::min(a.spin, dppf_internal::later_pass_polls());
    const long long query_blocks = (long long)heads * l.most[kByQuery], key_blocks = (long long)kv_heads * a.splits * l.most[kByKey];
    if (query_blocks > INT_MAX) return DPPF_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (D <= 64) return launch_attention_grad<4>(a, query_blocks, key_blocks, dev, s);
    return D <= 96 ? launch_attention_grad<6>(a, query_blocks, key_blocks, dev, s) : launch_attention_grad<8>(a, query_blocks, key_blocks, dev, s);
}

}  // extern "C"
