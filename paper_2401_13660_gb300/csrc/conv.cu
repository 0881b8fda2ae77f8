// The causal depthwise convolution (kernel 4) with SiLU over a span, and its
// gradients (Table 6 "Pre-SSM 1D convolution").
//
// With u[-3 .. -1] the window carried into the span (zeros without one) and
// u[t] = x[t], per channel:
//   p[t] = b + sum_k w[k] u[t-3+k],  out[t] = p sigmoid(p),  window out = u[L-3 .. L-1]
//   g[t] = dout[t] s (1 + p (1 - s)), s = sigmoid(p[t])          (p is formed again)
//   du[i] = sum_k w[k] g[i+3-k] over 0 <= i+3-k < L, plus the window-out gradient for i >= L-3
//   dw[k] = sum_t g[t] u[t-3+k],  db = sum_t g[t]
//
// A thread owns one 16-byte group of channels over a chunk of consecutive steps
// and keeps the last inputs (and gradients) in registers, so each input is read
// once but for the three steps around a chunk's ends. A CTA holds tx groups x
// ty chunks.
#include <algorithm>

#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kThreads = 256;

// How a span is cut: chunks of `rows` steps (at least 4, so that only a row's
// first chunk reads the window in), tx channel groups and ty chunks per CTA.
struct Cut {
    int rows, tx, ty;
    int64_t groups, chunks, items, gx, gy;   // chunks of a batch row; items = batch * chunks; CTAs = gx * gy
};

Cut cut_span(int64_t batch, int64_t L, int64_t width, int vec, int least) {
    Cut c{};
    c.groups = width / vec;
    c.tx = 1;
    while (c.tx < 32 && c.tx < c.groups) c.tx *= 2;
    c.ty = kThreads / c.tx;
    c.rows = 64;
    const int64_t want = 152 * 1024;   // threads
    while (c.rows > least && batch * ((L + c.rows - 1) / c.rows) * c.groups < want) c.rows /= 2;
    c.chunks = L > 0 ? (L + c.rows - 1) / c.rows : 1;   // an empty span still moves its window
    c.items = batch * c.chunks;
    c.gx = (c.groups + c.tx - 1) / c.tx;
    c.gy = (c.items + c.ty - 1) / c.ty;
    return c;
}

struct ConvShape {
    int64_t L, width, x_stride, dx_stride, groups, chunks, items;
    int rows, tx, gx;
};

template <typename T>
__device__ __forceinline__ void load_weights(const float *w, const float *bias, int64_t d0, float (&wv)[4][kVec<T>],
                                             float (&bv)[kVec<T>]) {
#pragma unroll
    for (int j = 0; j < kVec<T>; ++j) {
        const float4 q = gld4(w + 4 * (d0 + j));
        wv[0][j] = q.x; wv[1][j] = q.y; wv[2][j] = q.z; wv[3][j] = q.w;
        bv[j] = 0.f;
    }
    if (bias) ldf(bias + d0, bv);
}

// u[i] of batch row b for i >= -3.
template <typename T>
__device__ __forceinline__ void load_u(const T *x, const T *state, const ConvShape &s, int64_t b, int64_t i, int64_t d0,
                                       float (&v)[kVec<T>]) {
    if (i >= 0) {
        widen(ld16(x + (b * s.L + i) * s.x_stride + d0), v);
    } else if (state) {
        widen(ld16(state + (b * 3 + 3 + i) * s.width + d0), v);
    } else {
#pragma unroll
        for (int j = 0; j < kVec<T>; ++j) v[j] = 0.f;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) conv_kernel(const T *x, const T *state, const float *w, const float *bias,
                                                        T *out, T *state_out, const ConvShape s) {
    constexpr int V = kVec<T>;
    pdl_wait();
    const int64_t by = blockIdx.x / s.gx, bx = blockIdx.x - by * s.gx;
    const int64_t group = bx * s.tx + threadIdx.x % s.tx;
    const int64_t item = by * (kThreads / s.tx) + threadIdx.x / s.tx;
    if (group >= s.groups || item >= s.items) return;
    const int64_t b = item / s.chunks, chunk = item - b * s.chunks, d0 = group * V;
    const int64_t t0 = chunk * s.rows, t1 = min(t0 + s.rows, s.L);
    float wv[4][V], bv[V], u[4][V];
    load_weights<T>(w, bias, d0, wv, bv);
#pragma unroll
    for (int k = 0; k < 3; ++k) load_u(x, state, s, b, t0 - 3 + k, d0, u[k]);
    for (int64_t t = t0; t < t1; ++t) {
        load_u(x, state, s, b, t, d0, u[3]);
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float p = bv[j];
#pragma unroll
            for (int k = 0; k < 4; ++k) p = fmaf(wv[k][j], u[k][j], p);
            o[j] = __fdividef(p, 1.f + exp_for<T>(-p));
#pragma unroll
            for (int k = 0; k < 3; ++k) u[k][j] = u[k + 1][j];
        }
        st16(out + (b * s.L + t) * s.width + d0, o);
    }
    // The first chunk's thread has read the window in, so it may be written over now.
    if (chunk == 0 && state_out) {
        float v[3][V];
#pragma unroll
        for (int k = 0; k < 3; ++k) load_u(x, state, s, b, s.L - 3 + k, d0, v[k]);
#pragma unroll
        for (int k = 0; k < 3; ++k) st16(state_out + (b * 3 + k) * s.width + d0, v[k]);
    }
}

// Gradients. part [gy][5][width]: sums of dw[0..3] and db over the CTA's chunks.
template <typename T>
__global__ void __launch_bounds__(kThreads) conv_backward_kernel(const T *x, const T *state, const float *w,
                                                                 const float *bias, const T *dout, const T *dstate_out,
                                                                 T *dx, T *dstate, float *part, const ConvShape s) {
    constexpr int V = kVec<T>;
    __shared__ float red[kThreads * V];
    pdl_wait();
    const int64_t by = blockIdx.x / s.gx, bx = blockIdx.x - by * s.gx;
    const int ty = kThreads / s.tx;
    const int64_t group = bx * s.tx + threadIdx.x % s.tx;
    const int64_t item = by * ty + threadIdx.x / s.tx;
    float acc[5][V];
#pragma unroll
    for (int k = 0; k < 5; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[k][j] = 0.f;
    const int64_t d0 = group * V;
    if (group < s.groups && item < s.items) {
        const int64_t b = item / s.chunks, chunk = item - b * s.chunks;
        const int64_t t0 = chunk * s.rows, t1 = min(t0 + s.rows, s.L);
        float wv[4][V], bv[V], u[4][V], g[4][V];   // g[k] = g[t-3+k]
        load_weights<T>(w, bias, d0, wv, bv);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            load_u(x, state, s, b, t0 - 3 + k, d0, u[k]);
#pragma unroll
            for (int j = 0; j < V; ++j) g[k][j] = 0.f;
        }
        for (int64_t t = t0; t < t1 + 3; ++t) {
            if (t < s.L) {
                float go[V];
                load_u(x, state, s, b, t, d0, u[3]);
                widen(ld16(dout + (b * s.L + t) * s.width + d0), go);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float p = bv[j];
#pragma unroll
                    for (int k = 0; k < 4; ++k) p = fmaf(wv[k][j], u[k][j], p);
                    const float sg = __fdividef(1.f, 1.f + exp_for<T>(-p));
                    g[3][j] = go[j] * (sg * fmaf(p, 1.f - sg, 1.f));
                    if (t < t1) {   // the steps after belong to the next chunk
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[k][j] = fmaf(g[3][j], u[k][j], acc[k][j]);
                        acc[4][j] += g[3][j];
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) g[3][j] = 0.f;
            }
            // du[t-3] is complete; those before the chunk belong to the chunk before
            const int64_t i = t - 3;
            if (i >= t0 || (chunk == 0 && dstate)) {
                float du[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float v = 0.f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) v = fmaf(wv[k][j], g[3 - k][j], v);
                    du[j] = v;
                }
                if (dstate_out && i >= s.L - 3) {
                    float e[V];
                    widen(ld16(dstate_out + (b * 3 + i - (s.L - 3)) * s.width + d0), e);
#pragma unroll
                    for (int j = 0; j < V; ++j) du[j] += e[j];
                }
                if (i >= 0) st16(dx + (b * s.L + i) * s.dx_stride + d0, du);
                else st16(dstate + (b * 3 + 3 + i) * s.width + d0, du);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    u[k][j] = u[k + 1][j];
                    g[k][j] = g[k + 1][j];
                }
        }
    }
    // sum over the CTA's chunks, in their order
#pragma unroll
    for (int k = 0; k < 5; ++k) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) red[threadIdx.x * V + j] = acc[k][j];
        __syncthreads();
        for (int c = threadIdx.x; c < s.tx * V; c += kThreads) {
            if (bx * s.tx * V + c >= s.width) break;
            float sum = 0.f;
            for (int y = 0; y < ty; ++y) sum += red[y * s.tx * V + c];
            part[(by * 5 + k) * s.width + bx * s.tx * V + c] = sum;
        }
    }
}

constexpr int kSumCols = 32, kSumRows = 8;

// dw, dbias: the partial sums added in their order (each of kSumRows strands, then the strands).
__global__ void __launch_bounds__(kSumCols *kSumRows) conv_sum_kernel(const float *part, int64_t parts, int64_t width,
                                                                      float *dw, float *dbias) {
    __shared__ float red[kSumRows][kSumCols];
    pdl_wait();
    const int col = threadIdx.x % kSumCols, row = threadIdx.x / kSumCols;
    const int64_t c = (int64_t)blockIdx.x * kSumCols + col;   // k * width + channel
    float sum = 0.f;
    if (c < 5 * width)
        for (int64_t i = row; i < parts; i += kSumRows) sum += part[i * 5 * width + c];
    red[row][col] = sum;
    __syncthreads();
    if (row == 0 && c < 5 * width) {
#pragma unroll
        for (int r = 1; r < kSumRows; ++r) sum += red[r][col];
        const int64_t k = c / width, d = c - k * width;
        if (k < 4) dw[4 * d + k] = sum;
        else if (dbias) dbias[d] = sum;
    }
}

ConvShape shape_of(const ConvParams &p, const Cut &c) {
    ConvShape s{};
    s.L = p.seqlen; s.width = p.width; s.x_stride = p.x_stride; s.dx_stride = p.dx_stride;
    s.groups = c.groups; s.chunks = c.chunks; s.items = c.items;
    s.rows = c.rows; s.tx = c.tx; s.gx = (int)c.gx;
    return s;
}

template <typename T> cudaError_t forward(const ConvParams &p, cudaStream_t st) {
    const Cut c = cut_span(p.batch, p.seqlen, p.width, kVec<T>, 4);
    return launch_pdl(true, conv_kernel<T>, dim3((unsigned)(c.gx * c.gy)), dim3(kThreads), 0, st,
                      static_cast<const T *>(p.x), static_cast<const T *>(p.state), p.w, p.bias,
                      static_cast<T *>(p.out), static_cast<T *>(p.state_out), shape_of(p, c));
}

template <typename T> cudaError_t backward(const ConvParams &p, float *part, cudaStream_t st) {
    const Cut c = cut_span(p.batch, p.seqlen, p.width, kVec<T>, 8);
    cudaError_t e = cudaSuccess;
    if (c.gy > 0)   // without batch rows the sums are zeros
        e = launch_pdl(true, conv_backward_kernel<T>, dim3((unsigned)(c.gx * c.gy)), dim3(kThreads), 0, st,
                   static_cast<const T *>(p.x), static_cast<const T *>(p.state), p.w, p.bias,
                   static_cast<const T *>(p.dout), static_cast<const T *>(p.dstate_out), static_cast<T *>(p.dx),
                   static_cast<T *>(p.dstate), part, shape_of(p, c));
    if (e != cudaSuccess) return e;
    return launch_pdl(true, conv_sum_kernel, dim3((unsigned)((5 * p.width + kSumCols - 1) / kSumCols)),
                      dim3(kSumCols * kSumRows), 0, st, static_cast<const float *>(part), c.gy, p.width, p.dw, p.dbias);
}

}  // namespace

size_t conv_backward_scratch(int64_t batch, int64_t seqlen, int64_t width) {
    int64_t gy = 0;
    for (int vec : {4, 8}) gy = std::max(gy, cut_span(batch, seqlen, width, vec, 8).gy);
    return (size_t)(gy * 5 * width) * sizeof(float);
}

cudaError_t launch_conv(const ConvParams &p, bool bf16, cudaStream_t s) {
    return bf16 ? forward<__nv_bfloat16>(p, s) : forward<float>(p, s);
}

cudaError_t launch_conv_backward(const ConvParams &p, bool bf16, float *part, cudaStream_t s) {
    return bf16 ? backward<__nv_bfloat16>(p, part, s) : backward<float>(p, part, s);
}

}  // namespace mbscan
