// Cross entropy of next tokens with its gradient:
//   m = max_v l[v], s = sum_v exp(l[v] - m)
//   loss = w ((m - l[y]) + log s),  dl[v] = scale w (exp(l[v] - m) / s - [v = y])
// Rows of weight zero, or whose target is outside the vocabulary, are zeros
// whatever their logits hold.
//
// Up to kWarpVocab logits a warp holds a row in registers and reads it once;
// longer rows take a CTA, which runs over the row with a running maximum and
// sum, then once more for the gradient.
#include "tokens.cuh"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kWarpVocab = 1024, kWarpRows = 8, kRowThreads = 512;

struct LossArgs {
    const void *targets;
    const float *weight;
    float *loss;
    int64_t n;
    int type, vocab;
    float scale;
};

// The row's target (-1: the row counts for nothing) and weight.
__device__ __forceinline__ int target_of(const LossArgs &a, int64_t row, float &w) {
    const int y = load_token(a.targets, a.type, row, a.vocab);
    w = y < 0 ? 0.f : a.weight ? a.weight[row] : 1.f;
    return w == 0.f ? -1 : y;
}

// N logits per lane; lane l has l, l + 32, ...
template <typename T, int N>
__global__ void __launch_bounds__(32 * kWarpRows) loss_warp_kernel(const T *logits, T *dlogits, const LossArgs a) {
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kWarpRows + threadIdx.x / 32;
    if (row >= a.n) return;
    const T *l = logits + row * a.vocab;
    T *d = dlogits ? dlogits + row * a.vocab : nullptr;
    float w;
    const int y = target_of(a, row, w);
    if (y < 0) {
        if (lane == 0) a.loss[row] = 0.f;
        if (d)
            for (int v = lane; v < a.vocab; v += 32) d[v] = from_f32<T>(0.f);
        return;
    }
    float x[N];
    float m = -INFINITY, at = 0.f, s = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int v = j * 32 + lane;
        x[j] = v < a.vocab ? to_f32(l[v]) : -INFINITY;
        m = fmaxf(m, x[j]);
        if (v == y) at = x[j];
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
    at = __shfl_sync(kFull, at, y & 31);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        x[j] = j * 32 + lane < a.vocab ? exp_for<T>(x[j] - m) : 0.f;
        s += x[j];
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(kFull, s, o);
    if (lane == 0) a.loss[row] = w * ((m - at) + logf(s));
    if (!d) return;
    const float r = 1.f / s, c = w * a.scale;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int v = j * 32 + lane;
        if (v < a.vocab) d[v] = from_f32<T>(c * (x[j] * r - (v == y ? 1.f : 0.f)));
    }
}

// Running maximum and sum: s is relative to m.
template <typename T> __device__ __forceinline__ void join(float &m, float &s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    if (top == -INFINITY) {   // nothing yet (a NaN among the sums stays)
        s += s2;
        return;
    }
    s = s * exp_for<T>(m - top) + s2 * exp_for<T>(m2 - top);
    m = top;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) loss_row_kernel(const T *logits, T *dlogits, const LossArgs a) {
    __shared__ float sm[kRowThreads / 32], ss[kRowThreads / 32];
    pdl_wait();
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T *l = logits + row * a.vocab;
    T *d = dlogits ? dlogits + row * a.vocab : nullptr;
    float w;
    const int y = target_of(a, row, w);
    if (y < 0) {
        if (tid == 0) a.loss[row] = 0.f;
        if (d)
            for (int v = tid; v < a.vocab; v += kRowThreads) d[v] = from_f32<T>(0.f);
        return;
    }
    const float at = to_f32(l[y]);
    float m = -INFINITY, s = 0.f;
    for (int v = tid; v < a.vocab; v += kRowThreads) {
        const float x = to_f32(l[v]);
        if (x > m) {
            s = s * exp_for<T>(m - x) + 1.f;
            m = x;
        } else if (x > -INFINITY) {
            s += exp_for<T>(x - m);
        } else if (x != x) {
            s += x;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        const float m2 = __shfl_xor_sync(kFull, m, o), s2 = __shfl_xor_sync(kFull, s, o);
        join<T>(m, s, m2, s2);
    }
    if ((tid & 31) == 0) {
        sm[tid / 32] = m;
        ss[tid / 32] = s;
    }
    __syncthreads();
    m = sm[0];
    s = ss[0];
    for (int i = 1; i < kRowThreads / 32; ++i) join<T>(m, s, sm[i], ss[i]);
    if (tid == 0) a.loss[row] = w * ((m - at) + logf(s));
    if (!d) return;
    const float r = 1.f / s, c = w * a.scale;
    for (int v = tid; v < a.vocab; v += kRowThreads)
        d[v] = from_f32<T>(c * (exp_for<T>(to_f32(l[v]) - m) * r - (v == y ? 1.f : 0.f)));
}

template <typename T>
cudaError_t loss(const LossArgs &a, const void *logits, void *dlogits, cudaStream_t st) {
    const T *l = static_cast<const T *>(logits);
    T *d = static_cast<T *>(dlogits);
    if (a.vocab > kWarpVocab)
        return launch_pdl(true, loss_row_kernel<T>, dim3((unsigned)a.n), dim3(kRowThreads), 0, st, l, d, a);
    const dim3 grid((unsigned)((a.n + kWarpRows - 1) / kWarpRows));
    const auto k = a.vocab <= 256 ? loss_warp_kernel<T, 8> : loss_warp_kernel<T, kWarpVocab / 32>;
    return launch_pdl(true, k, grid, dim3(32 * kWarpRows), 0, st, l, d, a);
}

}  // namespace

cudaError_t launch_cross_entropy(const void *logits, bool bf16, const void *targets, int type, const float *weight,
                                 float scale, float *out, void *dlogits, int64_t n, int vocab, cudaStream_t s) {
    const LossArgs a{targets, weight, out, n, type, vocab, scale};
    return bf16 ? loss<__nv_bfloat16>(a, logits, dlogits, s) : loss<float>(a, logits, dlogits, s);
}

}  // namespace mbscan
