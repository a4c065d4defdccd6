// Operators of a transformer block in a worker's local step: host side and C ABI (include/dppf.h).
//   layer_norm.cuh     layer norm after a residual addition; its gradient
//   rotary.cuh         rotary positions and their inverse
//   local_host.cuh     devices, launches, checks of arguments
#include "dppf.h"

#include "layer_norm.cuh"
#include "local_host.cuh"
#include "rotary.cuh"

namespace {

struct Range { const void *p; size_t n; };

// ---------------------------------------------------------------- layer norm

struct NormOperand { const void *p; int64_t ld; int type; };   // ld 0: one row

// Elements that a thread moves at a time: eight, two or one, as the width and the rows' starts allow.
int norm_width(int H, std::initializer_list<NormOperand> operands) {
    for (const int n : {8, 2}) {
        bool fits = H % n == 0;
        for (const NormOperand &o : operands) {
            const size_t boundary = n * type_bytes(o.type);
            fits = fits && (!o.p || (aligned_to(o.p, boundary) && (size_t)o.ld * type_bytes(o.type) % boundary == 0));
        }
        if (fits) return n;
    }
    return 1;
}

// Threads of a block that holds a row, `each` elements a thread.
int norm_threads(int H, int each) { return ((H + each - 1) / each + 31) / 32 * 32; }

// Lanes of a warp for a row: the fewest that hold it, a power of two.
int norm_lanes(int H) {
    int lanes = 1;
    while (lanes * kNormElements < H) lanes *= 2;
    return lanes;
}

template <typename TX, typename TO, int N>
int launch_norm(NormArgs a, cudaStream_t s) {
    a.groups = a.H / N;
    a.lanes = norm_lanes(a.H);
    const int64_t side = kNormWarps * 32 / a.lanes;
    if (a.H <= kNormWarpRow) norm_kernel<TX, TO, N, kNormElements, true><<<(unsigned)((a.T + side - 1) / side), kNormWarps * 32, 0, s>>>(a);
    else if (a.H <= kNormRow && sizeof(TX) == 2 && !a.branch) norm_kernel<TX, TO, N, sizeof(TX) == 2 ? 2 * kNormElements : kNormElements, false><<<(unsigned)a.T, norm_threads(a.H, 2 * kNormElements), 0, s>>>(a);
    else if (a.H <= kNormRow) norm_kernel<TX, TO, N, kNormElements, false><<<(unsigned)a.T, norm_threads(a.H, kNormElements), 0, s>>>(a);
    else norm_wide_kernel<TX, TO, N><<<(unsigned)a.T, kNormWideThreads, 0, s>>>(a);
    return launched();
}
template <typename TX, typename TO>
int launch_norm_width(const NormArgs &a, int n, cudaStream_t s) {
    return n == 8 ? launch_norm<TX, TO, 8>(a, s) : n == 2 ? launch_norm<TX, TO, 2>(a, s) : launch_norm<TX, TO, 1>(a, s);
}

// Blocks whose columns' sums the workspace holds.  The SMs are a B200's 148 whatever the device: the size is asked for without one.
int64_t norm_grad_blocks(int64_t T, int H) {
    if (H > kNormGradRow) return T < 32 ? T : 32;                                        // rows of blocks of the columns' kernel
    const int64_t side = H <= kNormWarpRow ? kNormWarps * 32 / norm_lanes(H) : 1, rows = (T + side - 1) / side;
    const int64_t most = 148LL * (H <= kNormWarpRow ? 2 : 1024 / norm_threads(H, kNormGradElements));
    return rows < most ? rows : most;
}

template <typename TX, typename TO, int N>
int launch_norm_grad(NormGradArgs a, cudaStream_t s) {
    a.groups = a.H / N;
    a.lanes = norm_lanes(a.H);
    if (a.H <= kNormWarpRow) {
        norm_grad_kernel<TX, TO, N, kNormElements, true><<<(unsigned)a.blocks, kNormWarps * 32, 0, s>>>(a);
    } else if (a.H <= kNormGradRow) {
        norm_grad_kernel<TX, TO, N, kNormGradElements, false><<<(unsigned)a.blocks, norm_threads(a.H, kNormGradElements), 0, s>>>(a);
    } else {
        norm_grad_columns_kernel<TX, TO, N><<<dim3((unsigned)((a.groups + kNormWideThreads - 1) / kNormWideThreads), (unsigned)a.blocks), kNormWideThreads, 0, s>>>(a);
        norm_grad_wide_kernel<TX, TO, N><<<(unsigned)a.T, kNormWideThreads, 0, s>>>(a);
    }
    if (cudaPeekAtLastError() != cudaSuccess ||
        !launch_after(norm_join_kernel, dim3((unsigned)((a.H + 31) / 32), a.dbias ? 2 : 1), kNormJoinThreads, 0, s, a)) {
        cudaGetLastError();
        return DPPF_ERR_CUDA;
    }
    return DPPF_OK;
}
template <typename TX, typename TO>
int launch_norm_grad_width(const NormGradArgs &a, int n, cudaStream_t s) {
    return n == 8 ? launch_norm_grad<TX, TO, 8>(a, s) : n == 2 ? launch_norm_grad<TX, TO, 2>(a, s) : launch_norm_grad<TX, TO, 1>(a, s);
}

bool norm_shape(int64_t T, int H) { return T >= 0 && T <= INT_MAX && H >= 1 && H <= DPPF_MAX_WIDTH; }

// ---------------------------------------------------------------- rotary positions

template <typename T, int N, bool kInterleaved>
int launch_rotary(RotaryArgs a, int rest, int sms, cudaStream_t s) {
    a.turn_groups = a.half / N;
    a.rest_groups = rest / N;
    // Tokens of a block: about eight groups a thread, within the table, and four blocks an SM where there are few tokens.
    const long long groups = (long long)a.heads * (a.turn_groups + a.rest_groups);
    long long tokens = (8LL * kRotaryThreads + groups - 1) / groups;
    if (tokens > kRotaryTable / a.half) tokens = kRotaryTable / a.half;
    if (tokens > kRotaryMaxTokens) tokens = kRotaryMaxTokens;
    while (tokens > 1 && (a.T + tokens - 1) / tokens < 4LL * sms) tokens = (tokens + 1) / 2;
    a.tokens = (int)tokens;
    rotary_kernel<T, N, kInterleaved><<<(unsigned)((a.T + tokens - 1) / tokens), kRotaryThreads, 0, s>>>(a);
    return launched();
}

template <typename T>
int launch_rotary_width(const RotaryArgs &a, int rest, int sms, bool interleaved, cudaStream_t s) {
    constexpr int kWide = 16 / (int)sizeof(T);
    // elements that lie together: of a half, or of the pairs
    auto fits = [&](int n) {
        const size_t boundary = n * sizeof(T);
        const bool heads = a.heads == 1 || ((size_t)a.head_x * sizeof(T) % boundary == 0 && (size_t)a.head_out * sizeof(T) % boundary == 0);
        const int pairs = interleaved ? n / 2 : n;
        return a.half % pairs == 0 && (2 * a.half) % n == 0 && rest % pairs == 0 && aligned_to(a.x, boundary) && aligned_to(a.out, boundary) &&
               (size_t)a.ld_x * sizeof(T) % boundary == 0 && (size_t)a.ld_out * sizeof(T) % boundary == 0 && heads;
    };
    if (interleaved) {
        if (fits(kWide)) return launch_rotary<T, kWide / 2, true>(a, rest, sms, s);
        if (kWide > 4 && fits(kWide / 2)) return launch_rotary<T, (kWide > 4 ? kWide / 4 : 1), true>(a, rest, sms, s);
        return launch_rotary<T, 1, true>(a, rest, sms, s);
    }
    if (fits(kWide)) return launch_rotary<T, kWide, false>(a, rest, sms, s);
    if (fits(kWide / 2)) return launch_rotary<T, kWide / 2, false>(a, rest, sms, s);
    return launch_rotary<T, 1, false>(a, rest, sms, s);
}

}  // namespace

extern "C" {

int dppf_layer_norm(const void *x, int x_type, int64_t ld_x, const void *branch, int branch_type, int64_t ld_branch, const void *weight,
                    const void *bias, int weight_type, int64_t T, int H, float eps, void *sum_out, int64_t ld_sum, void *out, int out_type,
                    int64_t ld_out, float *mean_out, float *rstd_out, void *cuda_stream) {
    if (!known_type(x_type) || !known_type(weight_type) || !known_type(out_type) || (branch && !known_type(branch_type))) return DPPF_ERR_INVALID_ARG;
    if (!norm_shape(T, H) || !std::isfinite(eps) || eps < 0.f) return DPPF_ERR_INVALID_ARG;
    if (ld_x < H || ld_x > kMaxLd || ld_out < H || ld_out > kMaxLd || (branch && (ld_branch < H || ld_branch > kMaxLd || ld_sum < H || ld_sum > kMaxLd)))
        return DPPF_ERR_INVALID_ARG;
    if (T == 0) return DPPF_OK;
    if (!x || !weight || !out || !mean_out || !rstd_out || !branch != !sum_out) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(x, type_bytes(x_type)) || !aligned_to(weight, type_bytes(weight_type)) || !aligned_to(bias, type_bytes(weight_type)) ||
        !aligned_to(out, type_bytes(out_type)) || !aligned_to(mean_out, 4) || !aligned_to(rstd_out, 4) ||
        (branch && (!aligned_to(branch, type_bytes(branch_type)) || !aligned_to(sum_out, type_bytes(x_type)))))
        return DPPF_ERR_ALIGNMENT;
    const size_t row = (size_t)H * type_bytes(weight_type), stat = (size_t)T * 4;
    const Range in[] = {{x, matrix_bytes(T, H, ld_x, x_type)}, {branch, branch ? matrix_bytes(T, H, ld_branch, branch_type) : 0}, {weight, row}, {bias, row}};
    const Range written[] = {{out, matrix_bytes(T, H, ld_out, out_type)}, {mean_out, stat}, {rstd_out, stat}, {sum_out, branch ? matrix_bytes(T, H, ld_sum, x_type) : 0}};
    for (int i = 0; i < 4; ++i) {
        for (int k = 0; k < 4; ++k) {
            const bool same = i == 3 && k == 0 && sum_out == x && ld_sum == ld_x;        // the sum may replace x
            if (!same && ranges_meet(written[i].p, written[i].n, in[k].p, in[k].n)) return DPPF_ERR_INVALID_ARG;
        }
        for (int k = 0; k < i; ++k)
            if (ranges_meet(written[i].p, written[i].n, written[k].p, written[k].n)) return DPPF_ERR_INVALID_ARG;
    }
    NormArgs a = {};
    a.x = x; a.branch = branch; a.weight = weight; a.bias = bias;
    a.sum = sum_out; a.out = out; a.mean = mean_out; a.rstd = rstd_out;
    a.ld_x = ld_x; a.ld_branch = ld_branch; a.ld_sum = ld_sum; a.ld_out = ld_out; a.T = T; a.H = H;
    a.branch32 = branch_type == DPPF_FLOAT32; a.weight32 = weight_type == DPPF_FLOAT32;
    a.eps = eps;
    const int n = norm_width(H, {{x, ld_x, x_type}, {branch, ld_branch, branch_type}, {sum_out, ld_sum, x_type}, {out, ld_out, out_type}, {weight, 0, weight_type}, {bias, 0, weight_type}});
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (x_type == DPPF_FLOAT32) return out_type == DPPF_FLOAT32 ? launch_norm_width<float, float>(a, n, s) : launch_norm_width<float, bf16>(a, n, s);
    return out_type == DPPF_FLOAT32 ? launch_norm_width<bf16, float>(a, n, s) : launch_norm_width<bf16, bf16>(a, n, s);
}

size_t dppf_layer_norm_workspace_bytes(int64_t T, int H) {
    if (T < 1 || !norm_shape(T, H)) return 0;
    return round256((size_t)norm_grad_blocks(T, H) * 2 * (size_t)H * sizeof(float));
}

int dppf_layer_norm_grad(const void *grad_out, int out_type, int64_t ld_out, const void *x, int x_type, int64_t ld_x, const float *mean,
                         const float *rstd, const void *weight, int weight_type, int64_t T, int H, const void *grad_sum, int64_t ld_grad_sum,
                         void *grad_x, int64_t ld_grad_x, void *grad_weight, void *grad_bias, int grad_type, int accumulate, void *ws,
                         size_t ws_bytes, void *cuda_stream) {
    if (!known_type(out_type) || !known_type(x_type) || !known_type(weight_type) || !known_type(grad_type) || !norm_shape(T, H)) return DPPF_ERR_INVALID_ARG;
    if (ld_out < H || ld_out > kMaxLd || ld_x < H || ld_x > kMaxLd || ld_grad_x < H || ld_grad_x > kMaxLd || (grad_sum && (ld_grad_sum < H || ld_grad_sum > kMaxLd)))
        return DPPF_ERR_INVALID_ARG;
    if (!grad_weight) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(grad_weight, type_bytes(grad_type)) || !aligned_to(grad_bias, type_bytes(grad_type))) return DPPF_ERR_ALIGNMENT;
    const size_t grad_row = (size_t)H * type_bytes(grad_type);
    if (ranges_meet(grad_weight, grad_row, grad_bias, grad_row)) return DPPF_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (T == 0) {
        if (accumulate) return DPPF_OK;
        return cudaMemsetAsync(grad_weight, 0, grad_row, s) == cudaSuccess && (!grad_bias || cudaMemsetAsync(grad_bias, 0, grad_row, s) == cudaSuccess) ? DPPF_OK : DPPF_ERR_CUDA;
    }
    if (!grad_out || !x || !mean || !rstd || !weight || !grad_x || !ws) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(grad_out, type_bytes(out_type)) || !aligned_to(x, type_bytes(x_type)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) ||
        !aligned_to(weight, type_bytes(weight_type)) || !aligned_to(grad_sum, type_bytes(x_type)) || !aligned_to(grad_x, type_bytes(x_type)) || !aligned_to(ws, 128))
        return DPPF_ERR_ALIGNMENT;
    const size_t need = dppf_layer_norm_workspace_bytes(T, H);
    if (ws_bytes < need) return DPPF_ERR_WORKSPACE;
    const size_t stat = (size_t)T * 4;
    const Range in[] = {{grad_out, matrix_bytes(T, H, ld_out, out_type)}, {grad_sum, grad_sum ? matrix_bytes(T, H, ld_grad_sum, x_type) : 0}, {x, matrix_bytes(T, H, ld_x, x_type)},
                        {mean, stat}, {rstd, stat}, {weight, (size_t)H * type_bytes(weight_type)}};
    const Range written[] = {{grad_x, matrix_bytes(T, H, ld_grad_x, x_type)}, {grad_weight, grad_row}, {grad_bias, grad_row}, {ws, need}};
    for (int i = 0; i < 4; ++i) {
        for (int k = 0; k < 6; ++k) {
            // the gradient may replace what it is formed from, element by element
            const bool same = i == 0 && ((k == 0 && grad_x == grad_out && x_type == out_type && ld_grad_x == ld_out) || (k == 1 && grad_x == grad_sum && ld_grad_x == ld_grad_sum));
            if (!same && ranges_meet(written[i].p, written[i].n, in[k].p, in[k].n)) return DPPF_ERR_INVALID_ARG;
        }
        for (int k = 0; k < i; ++k)
            if (ranges_meet(written[i].p, written[i].n, written[k].p, written[k].n)) return DPPF_ERR_INVALID_ARG;
    }
    NormGradArgs a = {};
    a.dy = grad_out; a.x = x; a.weight = weight; a.dsum = grad_sum; a.mean = mean; a.rstd = rstd;
    a.dx = grad_x; a.dweight = grad_weight; a.dbias = grad_bias; a.part = static_cast<float *>(ws);
    a.ld_dy = ld_out; a.ld_x = ld_x; a.ld_dsum = ld_grad_sum; a.ld_dx = ld_grad_x; a.T = T; a.H = H;
    a.blocks = (int)norm_grad_blocks(T, H);
    a.weight32 = weight_type == DPPF_FLOAT32; a.grad32 = grad_type == DPPF_FLOAT32; a.add = accumulate ? 1 : 0;
    a.inv_h = (float)(1.0 / (double)H);
    const int n = norm_width(H, {{grad_out, ld_out, out_type}, {x, ld_x, x_type}, {grad_sum, ld_grad_sum, x_type}, {grad_x, ld_grad_x, x_type}, {weight, 0, weight_type}});
    if (x_type == DPPF_FLOAT32) return out_type == DPPF_FLOAT32 ? launch_norm_grad_width<float, float>(a, n, s) : launch_norm_grad_width<float, bf16>(a, n, s);
    return out_type == DPPF_FLOAT32 ? launch_norm_grad_width<bf16, float>(a, n, s) : launch_norm_grad_width<bf16, bf16>(a, n, s);
}

int dppf_rotary(const void *x, int type, int64_t ld_x, int64_t head_x, int64_t T, int heads, int D, int turned, int interleaved,
                const void *positions, int position_bits, const double *frequencies, float scale, int inverse, void *out, int64_t ld_out,
                int64_t head_out, void *cuda_stream) {
    if (!known_type(type) || (position_bits != 32 && position_bits != 64) || T < 0 || T > INT_MAX || heads < 1 || heads > DPPF_MAX_HEADS || D < 1 || D > DPPF_MAX_HEAD_WIDTH ||
        turned < 2 || turned > D || turned % 2 || !std::isfinite(scale))
        return DPPF_ERR_INVALID_ARG;
    const HeadRows hx = {x, ld_x, head_x, T, heads, D, type}, ho = {out, ld_out, head_out, T, heads, D, type};
    if (T == 0) return DPPF_OK;
    if (!x || !out || !positions || !frequencies || !hx.apart() || !ho.apart()) return DPPF_ERR_INVALID_ARG;
    if (!aligned_to(x, type_bytes(type)) || !aligned_to(out, type_bytes(type)) || !aligned_to(positions, position_bits / 8) || !aligned_to(frequencies, 8)) return DPPF_ERR_ALIGNMENT;
    const bool in_place = out == x;
    if (in_place ? (ld_out != ld_x || head_out != head_x) : ho.meets(hx)) return DPPF_ERR_INVALID_ARG;
    if (ranges_meet(out, ho.bytes(), positions, (size_t)T * (position_bits / 8)) || ranges_meet(out, ho.bytes(), frequencies, (size_t)turned / 2 * 8)) return DPPF_ERR_INVALID_ARG;
    const int dev = current_device(), sms = dev < 0 ? -1 : multiprocessors(dev);
    if (sms < 0) return DPPF_ERR_CUDA;
    RotaryArgs a = {};
    a.x = x; a.out = out; a.positions = positions; a.frequencies = frequencies;
    a.ld_x = ld_x; a.head_x = head_x; a.ld_out = ld_out; a.head_out = head_out; a.T = T;
    a.heads = heads; a.D = D; a.half = turned / 2;
    a.positions64 = position_bits == 64; a.inverse = inverse ? 1 : 0;
    a.scale = scale;
    const int rest = in_place ? 0 : D - turned;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return type == DPPF_FLOAT32 ? launch_rotary_width<float>(a, rest, sms, interleaved != 0, s) : launch_rotary_width<bf16>(a, rest, sms, interleaved != 0, s);
}

int dppf_rotary_frequencies(int turned, double base, int scaling, double factor, int64_t original_length, double *frequencies_host, float *scale_host) {
    if (turned < 2 || turned % 2 || turned > DPPF_MAX_HEAD_WIDTH || !std::isfinite(base) || !(base > 1.0) || !std::isfinite(factor) || !(factor >= 1.0) || !frequencies_host || !scale_host ||
        scaling < DPPF_POSITIONS_PLAIN || scaling > DPPF_POSITIONS_BY_PARTS || (scaling == DPPF_POSITIONS_BY_PARTS && original_length < 1))
        return DPPF_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586;
    if (scaling == DPPF_POSITIONS_STRETCHED && turned > 2) base *= std::pow(factor, (double)turned / (double)(turned - 2));
    for (int i = 0; i < turned / 2; ++i) {
        double f = std::pow(base, -2.0 * i / (double)turned);
        if (scaling == DPPF_POSITIONS_INTERPOLATED) f /= factor;
        if (scaling == DPPF_POSITIONS_BY_PARTS) {
            const double turns = (double)original_length * f / two_pi;             // over the original context
            const double keep = turns <= 1.0 ? 0.0 : turns >= 32.0 ? 1.0 : (turns - 1.0) / 31.0;
            f = (1.0 - keep) * f / factor + keep * f;
        }
        frequencies_host[i] = f;
    }
    *scale_host = scaling == DPPF_POSITIONS_BY_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return DPPF_OK;
}

}  // extern "C"
