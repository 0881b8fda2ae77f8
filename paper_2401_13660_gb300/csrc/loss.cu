// Cross entropy of next tokens with its gradient:
//   m = max_v l[v], s = sum_v exp(l[v] - m)
//   loss = w ((m - l[y]) + log s),  dl[v] = scale w (exp(l[v] - m) / s - [v = y])
// Rows of weight zero, or whose target is outside the vocabulary, are zeros
// whatever their logits hold.
//
// Bound by memory: every logit read and every gradient written once. Up to
// kWarpVocab logits a warp holds a row in registers. Longer rows take a CTA (a
// cluster of them where there are few rows), which runs over the row with a
// running maximum and sum, then once more for the gradient, from L2.
#include <algorithm>

#include "cluster.cuh"
#include "tokens.cuh"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kWarpVocab = 1024, kWarpRows = 8, kRowThreads = 512, kSms = 152;

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

// The same for rows that are read anyway: no target when it counts for nothing.
struct Row {
    int y;
    float w;
};

// A row of whole 16-byte groups, G per lane (lane l has groups l, l + 32, ...); a warp takes R rows at a time.
template <typename T, int G, int R>
__global__ void __launch_bounds__(32 * kWarpRows) loss_groups_kernel(const T *logits, T *dlogits, const LossArgs a) {
    constexpr int V = kVec<T>;
    pdl_wait();
    const int lane = threadIdx.x & 31, groups = a.vocab / V;
    const int64_t row0 = ((int64_t)blockIdx.x * kWarpRows + threadIdx.x / 32) * R;
    uint4 raw[R][G];
    Row of[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool in = row0 + r < a.n;
        of[r].y = -1;
        if (in) of[r].y = target_of(a, row0 + r, of[r].w);
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (in && g * 32 + lane < groups) raw[r][g] = ld16(logits + (row0 + r) * a.vocab + (g * 32 + lane) * V);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (row0 + r >= a.n) break;
        const int y = of[r].y;
        T *d = dlogits ? dlogits + (row0 + r) * a.vocab : nullptr;
        if (y < 0) {   // whatever the logits hold
            if (lane == 0) a.loss[row0 + r] = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g)
                if (d && g * 32 + lane < groups)
                    *reinterpret_cast<uint4 *>(d + (g * 32 + lane) * V) = make_uint4(0, 0, 0, 0);
            continue;
        }
        float x[G][V];
        float m = -INFINITY, at = 0.f, s = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (g * 32 + lane < groups) {
                widen(raw[r][g], x[g]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) x[g][j] = -INFINITY;
            }
            const int hit = y - (g * 32 + lane) * V;   // 0 .. V-1: the target is in this group
#pragma unroll
            for (int j = 0; j < V; ++j) {
                m = fmaxf(m, x[g][j]);
                if (hit == j) at = x[g][j];
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
        at = __shfl_sync(kFull, at, y / V & 31);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const bool in = g * 32 + lane < groups;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[g][j] = in ? exp_for<T>(x[g][j] - m) : 0.f;
                s += x[g][j];
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(kFull, s, o);
        const float w = of[r].w, c = w * a.scale, k = c / s;
        if (lane == 0) a.loss[row0 + r] = w * ((m - at) + logf(s));
        if (!d) continue;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (g * 32 + lane >= groups) break;
            const int hit = y - (g * 32 + lane) * V;
            float o[V];
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = hit == j ? fmaf(x[g][j], k, -c) : x[g][j] * k;
            st16(d + (g * 32 + lane) * V, o);
        }
    }
}

// Rows that are no whole groups. N logits per lane; lane l has l, l + 32, ...
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
    float x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = j * 32 + lane < a.vocab ? to_f32(l[j * 32 + lane]) : -INFINITY;
    if (y < 0) {
        if (lane == 0) a.loss[row] = 0.f;
        if (d)
            for (int v = lane; v < a.vocab; v += 32) d[v] = from_f32<T>(0.f);
        return;
    }
    float m = -INFINITY, at = 0.f, s = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        m = fmaxf(m, x[j]);
        if (j * 32 + lane == y) at = x[j];
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
    const float c = w * a.scale, k = c / s;
    if (lane == 0) a.loss[row] = w * ((m - at) + logf(s));
    if (!d) return;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int v = j * 32 + lane;
        if (v < a.vocab) d[v] = from_f32<T>(v == y ? fmaf(x[j], k, -c) : x[j] * k);
    }
}

// Running maximum m and sum s of exp(x - m); nothing yet: m = -inf, s = 0. A NaN stays in s.
struct Running {
    float m = -INFINITY, s = 0.f;
    template <typename T, int N> __device__ __forceinline__ void add(const float (&x)[N]) {
        float top = m;
#pragma unroll
        for (int j = 0; j < N; ++j) top = fmaxf(top, x[j]);
        const float ref = top == -INFINITY ? 0.f : top;   // masked logits only, so far: exp(-inf) = 0
        s *= exp_for<T>(m - ref);
#pragma unroll
        for (int j = 0; j < N; ++j) s += exp_for<T>(x[j] - ref);
        m = top;
    }
    template <typename T> __device__ __forceinline__ void join(float m2, float s2) {
        const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
        s = s * exp_for<T>(m - ref) + s2 * exp_for<T>(m2 - ref);
        m = top;
    }
};

// A row per cluster of C CTAs: each takes a contiguous part of the row's whole 16-byte groups, the first and the last
// also the elements before and behind them (rows of odd length begin at any element).
constexpr int kAhead = 4;   // groups loaded at once by a thread
template <typename T, int C>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(kRowThreads) loss_row_kernel(const T *logits, T *dlogits,
                                                                                       const LossArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float sm[kRowThreads / 32], ss[kRowThreads / 32], mine[2];
    pdl_wait();
    const int tid = threadIdx.x, part = blockIdx.x % C;
    const int64_t row = blockIdx.x / C;
    const T *l = logits + row * a.vocab;
    T *d = dlogits ? dlogits + row * a.vocab : nullptr;
    const int head = min((int)((16u - ((uint32_t)(row * a.vocab * (int64_t)sizeof(T)) & 15u) & 15u) / sizeof(T)), a.vocab);
    const int groups = (a.vocab - head) / V, tail = head + groups * V;
    const int g0 = (int)((int64_t)groups * part / C), g1 = (int)((int64_t)groups * (part + 1) / C);
    // the odd elements: one per thread at most
    int odd = -1;
    if (part == 0 && tid < head) odd = tid;
    if (part == C - 1 && tid >= 32 && tid - 32 < a.vocab - tail) odd = tail + tid - 32;
    float w;
    const int y = target_of(a, row, w);
    if (y < 0) {   // uniform in the cluster
        if (tid == 0 && part == 0) a.loss[row] = 0.f;
        if (!d) return;
        if (odd >= 0) d[odd] = from_f32<T>(0.f);
        for (int g = g0 + tid; g < g1; g += kRowThreads)
            *reinterpret_cast<uint4 *>(d + head + (int64_t)g * V) = make_uint4(0, 0, 0, 0);
        return;
    }
    const float at = to_f32(l[y]);
    const float own = odd >= 0 ? to_f32(l[odd]) : -INFINITY;
    Running run;
    if (odd >= 0) {
        const float x[1] = {own};
        run.add<T>(x);
    }
    for (int g = g0 + tid; g < g1; g += kAhead * kRowThreads) {
        uint4 raw[kAhead];
        float x[kAhead * V];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (g + k * kRowThreads < g1) raw[k] = ld16(l + head + (int64_t)(g + k * kRowThreads) * V);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float v[V];
            widen(raw[k], v);
#pragma unroll
            for (int j = 0; j < V; ++j) x[k * V + j] = g + k * kRowThreads < g1 ? v[j] : -INFINITY;
        }
        run.add<T>(x);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        const float m2 = __shfl_xor_sync(kFull, run.m, o), s2 = __shfl_xor_sync(kFull, run.s, o);
        run.join<T>(m2, s2);
    }
    if ((tid & 31) == 0) {
        sm[tid / 32] = run.m;
        ss[tid / 32] = run.s;
    }
    __syncthreads();
    run.m = sm[0];
    run.s = ss[0];
#pragma unroll
    for (int i = 1; i < kRowThreads / 32; ++i) run.join<T>(sm[i], ss[i]);
    if constexpr (C > 1) {
        if (tid == 0) {
            mine[0] = run.m;
            mine[1] = run.s;
        }
        cluster_arrive();
        cluster_wait();
        Running all;
#pragma unroll
        for (int i = 0; i < C; ++i) all.join<T>(cluster_load(&mine[0], i), cluster_load(&mine[1], i));
        run = all;
        cluster_arrive();   // has read the others'; waited for at the end
    }
    const float c = w * a.scale, k = c / run.s, m = run.m;
    if (tid == 0 && part == 0) a.loss[row] = w * ((m - at) + logf(run.s));
    if (d) {
        const auto grad = [&](float x, int v) {
            const float e = exp_for<T>(x - m);
            return v == y ? fmaf(e, k, -c) : e * k;
        };
        if (odd >= 0) d[odd] = from_f32<T>(grad(own, odd));
        for (int g = g0 + tid; g < g1; g += kAhead * kRowThreads) {
            uint4 raw[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                if (g + q * kRowThreads < g1) raw[q] = ld16(l + head + (int64_t)(g + q * kRowThreads) * V);
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                if (g + q * kRowThreads >= g1) break;
                const int v0 = head + (g + q * kRowThreads) * V;
                float v[V];
                widen(raw[q], v);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = grad(v[j], v0 + j);
                st16(d + v0, v);
            }
        }
    }
    if constexpr (C > 1) cluster_wait();
}

template <typename T>
cudaError_t loss(const LossArgs &a, const void *logits, void *dlogits, cudaStream_t st) {
    const T *l = static_cast<const T *>(logits);
    T *d = static_cast<T *>(dlogits);
    const auto run = [&](auto kernel, int64_t ctas, int threads) {
        return launch_pdl(true, kernel, dim3((unsigned)ctas), dim3(threads), 0, st, l, d, a);
    };
    if (a.vocab > kWarpVocab) {
        // CTAs of a row: as many as there are SMs for, each with two groups per thread at least
        int c = 1;
        while (c < 8 && a.n * c * 2 <= kSms && a.vocab / kVec<T> >= 4 * c * kRowThreads) c *= 2;
        return run(c == 1   ? loss_row_kernel<T, 1>
                   : c == 2 ? loss_row_kernel<T, 2>
                   : c == 4 ? loss_row_kernel<T, 4>
                            : loss_row_kernel<T, 8>,
                   a.n * c, kRowThreads);
    }
    const auto warps = [&](auto kernel, int rows) {
        return run(kernel, (a.n + kWarpRows * rows - 1) / (kWarpRows * rows), 32 * kWarpRows);
    };
    if (a.vocab % kVec<T> != 0) {
        if (a.vocab <= 256) return warps(loss_warp_kernel<T, 8>, 1);
        return warps(loss_warp_kernel<T, kWarpVocab / 32>, 1);
    }
    constexpr int kMost = kWarpVocab / 32 / kVec<T>;   // groups of a lane: 4 (bf16), 8 (fp32)
    const int groups = (a.vocab / kVec<T> + 31) / 32;
    if (groups <= kMost / 4) return warps(loss_groups_kernel<T, kMost / 4, 2>, 2);
    if (groups <= kMost / 2) return warps(loss_groups_kernel<T, kMost / 2, 1>, 1);
    return warps(loss_groups_kernel<T, kMost, 1>, 1);
}

}  // namespace

cudaError_t launch_cross_entropy(const void *logits, bool bf16, const void *targets, int type, const float *weight,
                                 float scale, float *out, void *dlogits, int64_t n, int vocab, cudaStream_t s) {
    const LossArgs a{targets, weight, out, n, type, vocab, scale};
    return bf16 ? loss<__nv_bfloat16>(a, logits, dlogits, s) : loss<float>(a, logits, dlogits, s);
}

}  // namespace mbscan
