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
#include "pairs.cuh"
#include "tokens.cuh"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kWarpVocab = 1024, kSms = 152;
// Warps of a CTA. 65536 x 256 bf16, eight lanes to a row: 1, 2, 4, 8 11.5, 11.4, 11.5, 12.1 us; a whole warp to a row, two
// rows side by side 14.3; warps that stay and fetch rows ahead 19.
constexpr int kWarpRows = 2;
// Threads of a row that is read twice, and the 16-byte groups that each loads at once: 32 elements, and two CTAs per SM
// (64 registers). 1003 x 32001 fp32 44 us; with plainer exponentials 512 threads and 16, 32, 64 elements took 51, 43, 51,
// 256 or 1024 threads 47 to 55. Rows that are read once keep 8 groups for each of 128 or 256 threads: 3000 x 5001 fp32 30 us,
// read twice 47; 1000 x 16000 bf16 18.4, read twice 19.6 (with everything in L2 13.0 and 15.2).
constexpr int kRowThreads = 512, kOnceGroups = 8;
// CTAs per SM that the registers of a row that is read once leave room for (fp32: 768 threads of 80 registers; of the 86 that
// the compiler would take 5 CTAs of 128 or 2 of 256 fit: 3000 x 5001 37 us instead of 30).
template <typename T, int kThreads> constexpr int kOnceCtas = sizeof(T) == 4 ? 768 / kThreads : 1;
template <typename T, bool kOnce> constexpr int kAhead = kOnce ? kOnceGroups : 32 / kVec<T>;

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

// e^x for x = l - m <= 0 on the SFU, within (1.5 |x| + 4) 2^-24 relative: for bf16 logits, whose gradient is rounded to
// 2^-9, and for sums that join others, where what is far below the maximum weighs as little as its error does.
__device__ __forceinline__ float exp_sfu(float x) { return ex2(x * kLog2e); }
// e^x of the logits: of fp32 ones to the precision of their gradient, down to e^-150 = 0 (masked).
template <typename T> __device__ __forceinline__ float2 exp2_of(float2 l, float2 minus_m) {
    const float2 c = add2(l, minus_m);
    if constexpr (sizeof(T) == 4) return exp_carried(make_float2(max_nan(c.x, -150.f), max_nan(c.y, -150.f)));
    const float2 t = mul2(c, splat(kLog2e));
    return make_float2(ex2(t.x), ex2(t.y));
}
template <typename T> __device__ __forceinline__ float exp_of(float x) {
    if constexpr (sizeof(T) == 4) return exp_carried(max_nan(x, -150.f));
    return exp_sfu(x);
}
// w scale / s, the factor of a row's gradient.
template <typename T> __device__ __forceinline__ float factor(float c, float s) {
    if constexpr (sizeof(T) == 4) return c / s;
    return __fdividef(c, s);
}

// A 16-byte group as pairs.
template <typename T> constexpr int kPairs = kVec<T> / 2;
template <typename T> __device__ __forceinline__ void to_pairs(const uint4 &q, float2 (&v)[kPairs<T>]) {
    float f[kVec<T>];
    widen(q, f);
#pragma unroll
    for (int j = 0; j < kPairs<T>; ++j) v[j] = make_float2(f[2 * j], f[2 * j + 1]);
}
template <typename T> __device__ __forceinline__ uint4 from_pairs(const float2 (&v)[kPairs<T>]) {
    float f[kVec<T>];
#pragma unroll
    for (int j = 0; j < kPairs<T>; ++j) {
        f[2 * j] = v[j].x;
        f[2 * j + 1] = v[j].y;
    }
    return narrow(f);
}
// A group of masked logits (-inf): neither the maximum nor a sum changes by it.
template <typename T> __device__ __forceinline__ uint4 masked() {
    const unsigned w = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    return make_uint4(w, w, w, w);
}

// Rows of whole 16-byte groups: L lanes to a row, 32 / L rows to a warp, so that what a row needs once (its target, the
// steps of its sums, the logarithm) is done for several at a time; G groups per lane (lane l of them: l, l + L, ...).
template <typename T, int L, int G>
__global__ void __launch_bounds__(32 * kWarpRows) loss_groups_kernel(const T *logits, T *dlogits, const LossArgs a) {
    constexpr int V = kVec<T>, P = kPairs<T>;
    pdl_wait();
    const int lane = threadIdx.x % L, groups = a.vocab / V;
    const int64_t row = ((int64_t)blockIdx.x * (32 * kWarpRows) + threadIdx.x) / L;
    const bool in = row < a.n;
    const int64_t base = row * a.vocab;
    uint4 raw[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
        raw[g] = in && g * L + lane < groups ? ld16(logits + base + (g * L + lane) * V) : masked<T>();
    float w = 0.f, at = 0.f;
    const int y = in ? target_of(a, row, w) : -1;   // -1: the row counts for nothing, whatever its logits hold
    if (y >= 0) at = to_f32(logits[base + y]);
    float2 x[G][P];
    float m = -INFINITY;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        to_pairs<T>(raw[g], x[g]);
#pragma unroll
        for (int j = 0; j < P; ++j) m = fmaxf(m, fmaxf(x[g][j].x, x[g][j].y));
    }
#pragma unroll
    for (int o = L / 2; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
    float2 sum = splat(0.f);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            x[g][j] = exp2_of<T>(x[g][j], splat(-m));
            sum = add2(sum, x[g][j]);
        }
    float s = sum.x + sum.y;
#pragma unroll
    for (int o = L / 2; o > 0; o /= 2) s += __shfl_xor_sync(kFull, s, o);
    if (!in) return;
    const float c = w * a.scale, k = factor<T>(c, s);
    if (lane == 0) a.loss[row] = y >= 0 ? w * ((m - at) + logf(s)) : 0.f;
    if (!dlogits) return;
    T *d = dlogits + base;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        if (g * L + lane >= groups) break;
#pragma unroll
        for (int j = 0; j < P; ++j) x[g][j] = mul2(x[g][j], splat(k));
        uint4 q = from_pairs<T>(x[g]);
        if (y < 0) q = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(d + (g * L + lane) * V) = q;
    }
    // over what this lane has just stored
    if (y >= 0 && y / V % L == lane) d[y] = from_f32<T>(fmaf(exp_of<T>(at - m), k, -c));
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
        x[j] = exp_of<T>(x[j] - m);
        s += x[j];
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(kFull, s, o);
    const float c = w * a.scale, k = factor<T>(c, s);
    if (lane == 0) a.loss[row] = w * ((m - at) + logf(s));
    if (!d) return;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int v = j * 32 + lane;
        if (v < a.vocab) d[v] = from_f32<T>(v == y ? fmaf(x[j], k, -c) : x[j] * k);
    }
}

// Running maximum m and sum s of exp(x - m); nothing yet: m = -inf, s = 0. A NaN stays in s.
template <typename T> struct Running {
    float m = -INFINITY, s = 0.f;
    // masked logits only, so far: their exp(-inf - 0) = 0
    static __device__ __forceinline__ float reference(float top) { return top == -INFINITY ? 0.f : top; }
    template <int N> __device__ __forceinline__ void add(const float2 (&x)[N]) {
        float top = m;
#pragma unroll
        for (int j = 0; j < N; ++j) top = fmaxf(top, fmaxf(x[j].x, x[j].y));
        const float ref = reference(top);
        float2 sum = make_float2(s * exp_sfu(m - ref), 0.f);
#pragma unroll
        for (int j = 0; j < N; ++j) sum = add2(sum, exp2_of<T>(x[j], splat(-ref)));
        s = sum.x + sum.y;
        m = top;
    }
    __device__ __forceinline__ void join(float m2, float s2) {
        const float top = fmaxf(m, m2), ref = reference(top);
        s = s * exp_sfu(m - ref) + s2 * exp_sfu(m2 - ref);
        m = top;
    }
};

// A row per cluster of C CTAs: each takes a contiguous part of the row's whole 16-byte groups, the first and the last
// also the elements before and behind them (rows of odd length begin at any element). With kOnce a thread's groups, at
// most kOnceGroups, stay in its registers for the gradient.
template <typename T, int kThreads, int C, bool kOnce>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(kThreads, kOnce ? kOnceCtas<T, kThreads> : 2)
    loss_row_kernel(const T *logits, T *dlogits, const LossArgs a) {
    constexpr int V = kVec<T>, P = kPairs<T>;
    __shared__ float sm[kThreads / 32], ss[kThreads / 32], mine[2];
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
        for (int g = g0 + tid; g < g1; g += kThreads)
            *reinterpret_cast<uint4 *>(d + head + (int64_t)g * V) = make_uint4(0, 0, 0, 0);
        return;
    }
    const float at = to_f32(l[y]);
    const float own = odd >= 0 ? to_f32(l[odd]) : -INFINITY;
    Running<T> run;
    {
        const float2 x[1] = {make_float2(own, -INFINITY)};
        run.add(x);
    }
    uint4 raw[kAhead<T, kOnce>];
    for (int g = g0 + tid; g < g1; g += kAhead<T, kOnce> * kThreads) {
        float2 x[kAhead<T, kOnce> * P];
#pragma unroll
        for (int k = 0; k < kAhead<T, kOnce>; ++k)
            raw[k] = g + k * kThreads < g1 ? ld16(l + head + (int64_t)(g + k * kThreads) * V) : masked<T>();
#pragma unroll
        for (int k = 0; k < kAhead<T, kOnce>; ++k) {
            float2 v[P];
            to_pairs<T>(raw[k], v);
#pragma unroll
            for (int j = 0; j < P; ++j) x[k * P + j] = v[j];
        }
        run.add(x);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        const float m2 = __shfl_xor_sync(kFull, run.m, o), s2 = __shfl_xor_sync(kFull, run.s, o);
        run.join(m2, s2);
    }
    if ((tid & 31) == 0) {
        sm[tid / 32] = run.m;
        ss[tid / 32] = run.s;
    }
    __syncthreads();
    run.m = sm[0];
    run.s = ss[0];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) run.join(sm[i], ss[i]);
    if constexpr (C > 1) {
        if (tid == 0) {
            mine[0] = run.m;
            mine[1] = run.s;
        }
        cluster_arrive();
        cluster_wait();
        Running<T> all;
#pragma unroll
        for (int i = 0; i < C; ++i) all.join(cluster_load(&mine[0], i), cluster_load(&mine[1], i));
        run = all;
        cluster_arrive();   // has read the others'; waited for at the end
    }
    const float c = w * a.scale, k = factor<T>(c, run.s), m = run.m;
    if (tid == 0 && part == 0) a.loss[row] = w * ((m - at) + logf(run.s));
    if (d) {
        const T hot = from_f32<T>(fmaf(exp_of<T>(at - m), k, -c));
        if (odd >= 0) d[odd] = odd == y ? hot : from_f32<T>(exp_of<T>(own - m) * k);
        for (int g = g0 + tid; g < g1; g += kAhead<T, kOnce> * kThreads) {
#pragma unroll
            for (int q = 0; q < kAhead<T, kOnce>; ++q)
                if (!kOnce && g + q * kThreads < g1) raw[q] = ld16(l + head + (int64_t)(g + q * kThreads) * V);
#pragma unroll
            for (int q = 0; q < kAhead<T, kOnce>; ++q) {
                if (g + q * kThreads >= g1) break;
                const int v0 = head + (g + q * kThreads) * V;
                float2 v[P];
                to_pairs<T>(raw[q], v);
#pragma unroll
                for (int j = 0; j < P; ++j) v[j] = mul2(exp2_of<T>(v[j], splat(-m)), splat(k));
                *reinterpret_cast<uint4 *>(d + v0) = from_pairs<T>(v);
                if (y >= v0 && y < v0 + V) d[y] = hot;   // over what this thread has just stored
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
        // Rows of up to kOnceGroups groups for each of 128 (256) threads are read once. Longer ones take 512, and where there
        // are SMs for it several CTAs, each with two groups per thread at least.
        const int groups = a.vocab / kVec<T>;
        if (groups <= 128 * kOnceGroups) return run(loss_row_kernel<T, 128, 1, true>, a.n, 128);
        if (groups <= 256 * kOnceGroups) return run(loss_row_kernel<T, 256, 1, true>, a.n, 256);
        int c = 1;
        while (c < 8 && a.n * c * 2 <= kSms && groups >= 4 * c * kRowThreads) c *= 2;
        return run(c == 1   ? loss_row_kernel<T, kRowThreads, 1, false>
                   : c == 2 ? loss_row_kernel<T, kRowThreads, 2, false>
                   : c == 4 ? loss_row_kernel<T, kRowThreads, 4, false>
                            : loss_row_kernel<T, kRowThreads, 8, false>,
                   a.n * c, kRowThreads);
    }
    const auto warps = [&](auto kernel, int rows) {   // of so many rows each
        return run(kernel, (a.n + kWarpRows * rows - 1) / (kWarpRows * rows), 32 * kWarpRows);
    };
    if (a.vocab % kVec<T> != 0)
        return warps(a.vocab <= 256 ? loss_warp_kernel<T, 8> : loss_warp_kernel<T, kWarpVocab / 32>, 1);
    // four groups a lane, as many lanes as that takes (fp32 above 512: eight)
    const int groups = a.vocab / kVec<T>;
    if (groups <= 32) return warps(loss_groups_kernel<T, 8, 4>, 4);
    if (groups <= 64) return warps(loss_groups_kernel<T, 16, 4>, 2);
    if (groups <= 128) return warps(loss_groups_kernel<T, 32, 4>, 1);
    return warps(loss_groups_kernel<T, 32, kWarpVocab / 32 / kVec<T>>, 1);
}

}  // namespace

cudaError_t launch_cross_entropy(const void *logits, bool bf16, const void *targets, int type, const float *weight,
                                 float scale, float *out, void *dlogits, int64_t n, int vocab, cudaStream_t s) {
    const LossArgs a{targets, weight, out, n, type, vocab, scale};
    return bf16 ? loss<__nv_bfloat16>(a, logits, dlogits, s) : loss<float>(a, logits, dlogits, s);
}

}  // namespace mbscan
