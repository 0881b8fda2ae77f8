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
// Both are bound by memory (2 and 3 elements moved for about 12 and 32
// operations). A thread owns one 16-byte group of channels over a chunk of
// consecutive steps and keeps the last inputs (and gradients) in registers, so
// each input is read once but for the three steps around a chunk's ends. Its
// rows come through a ring of asynchronous copies in shared memory that no other
// thread reads: the bytes in flight that the memory needs (over 100 KB per SM)
// would not fit in registers, and nothing is synchronised. A CTA holds tx groups
// x ty chunks; the chunks' length is what fills the SMs' CTA slots evenly.
#include <algorithm>

#include "pairs.cuh"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kSms = 152;
constexpr int kStage = 4;   // rows per stage of the ring (the taps' registers go around once in a stage)
// Stages: 8 x 8192 x 2048 bf16, backward, with 2, 3, 4: 138, 131, 129 us; fp32 3 x 1003 x 1544: 14.9, 15.2, 16.2.
template <typename T> constexpr int kStages = sizeof(T) == 2 ? 4 : 3;
template <typename T> constexpr int kGroup = 16 / (int)sizeof(T);   // channels of a thread
constexpr int kFwdThreads = 256, kFwdCtas = 2, kBwdThreads = 128;
template <typename T> constexpr int kBwdCtas = sizeof(T) == 2 ? 2 : 3;   // by their registers (234 and 144)
// Steps of a chunk at most, where there are enough of them. 8 x 8192 x 2048 bf16, forward with 24, 32, 48, 64, 96:
// 89, 85, 84, 85, 90 us; backward (sums to hand over) with 64, 128, 192, 256: 148, 139, 134, 129.
constexpr int kFwdLongest = 48, kBwdLongest = 256;

// How a span is cut: chunks of `rows` steps (at least 4, so that only a row's
// first chunk reads the window in), tx channel groups and ty chunks per CTA.
struct Cut {
    int rows, tx, ty;
    int64_t groups, chunks, items, gx, gy;   // chunks of a batch row; items = batch * chunks; CTAs = gx * gy
};

Cut cut_span(int64_t batch, int64_t L, int64_t width, int vec, int threads, int ctas, int longest) {
    Cut c{};
    c.groups = width / vec;
    c.tx = 1;
    while (c.tx < 32 && c.tx < c.groups) c.tx *= 2;
    c.ty = threads / c.tx;
    c.gx = (c.groups + c.tx - 1) / c.tx;
    int64_t rows = L;
    for (int64_t waves = 1; waves <= 32; ++waves) {   // of CTAs: as few as keep chunks short
        const int64_t chunks = (int64_t)kSms * ctas * waves / c.gx * c.ty / (batch > 0 ? batch : 1);
        rows = chunks > 0 ? (L + chunks - 1) / chunks : L;
        if (rows <= longest) break;
    }
    rows = std::max<int64_t>((rows + kStage - 1) / kStage * kStage, kStage);
    c.rows = (int)rows;
    c.chunks = L > 0 ? (L + rows - 1) / rows : 1;   // an empty span still moves its window
    c.items = batch * c.chunks;
    c.gy = (c.items + c.ty - 1) / c.ty;
    return c;
}

template <typename T> Cut cut_backward(int64_t batch, int64_t L, int64_t width) {
    return cut_span(batch, L, width, kGroup<T>, kBwdThreads, kBwdCtas<T>, kBwdLongest);
}

struct ConvShape {
    int64_t L, width, x_stride, dx_stride, groups, chunks, items;
    int rows, tx, gx;
};

// 2^64 sigmoid(p) of a pair, as 1 / (2^-64 + 2^-64 e^-p): the SFU's reciprocal flushes results below 2^-126, where
// p sigmoid(p) is a normal number still (p = -88: -5e-37). e^-p of the accuracy that T wants.
constexpr float kDown = 0x1p-64f;
__device__ __forceinline__ float2 sigmoid_of(float2 e) {
    const float2 q = fma2(e, splat(kDown), splat(kDown));
    return make_float2(rcp(q.x), rcp(q.y));
}
template <typename T> __device__ __forceinline__ float2 sigmoid2(float2 p);
template <> __device__ __forceinline__ float2 sigmoid2<__nv_bfloat16>(float2 p) {
    const float2 a = mul2(p, splat(-kLog2e));
    return sigmoid_of(make_float2(ex2(a.x), ex2(a.y)));
}
// fp32: within 2^-21 relative. Beyond +-100 the result is 1 or 0 to the last bit.
template <> __device__ __forceinline__ float2 sigmoid2<float>(float2 p) {
    const float2 c = make_float2(fminf(fmaxf(p.x, -100.f), 100.f), fminf(fmaxf(p.y, -100.f), 100.f));
    return sigmoid_of(exp_carried(make_float2(-c.x, -c.y)));
}

// A 16-byte group as pairs of channels.
template <typename T> __device__ __forceinline__ void to_pairs(const uint4 &q, float2 (&v)[kGroup<T> / 2]) {
    float f[kGroup<T>];
    widen(q, f);
#pragma unroll
    for (int j = 0; j < kGroup<T> / 2; ++j) v[j] = make_float2(f[2 * j], f[2 * j + 1]);
}
template <typename T> __device__ __forceinline__ void put_pairs(T *p, const float2 (&v)[kGroup<T> / 2]) {
    float f[kGroup<T>];
#pragma unroll
    for (int j = 0; j < kGroup<T> / 2; ++j) {
        f[2 * j] = v[j].x;
        f[2 * j + 1] = v[j].y;
    }
    st16(p, f);
}

template <int P>
__device__ __forceinline__ void load_weights(const float *w, const float *bias, int64_t d0, float2 (&wv)[4][P],
                                             float2 (&bv)[P]) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const float4 q = gld4(w + 4 * (d0 + 2 * j)), r = gld4(w + 4 * (d0 + 2 * j + 1));
        wv[0][j] = make_float2(q.x, r.x);
        wv[1][j] = make_float2(q.y, r.y);
        wv[2][j] = make_float2(q.z, r.z);
        wv[3][j] = make_float2(q.w, r.w);
        bv[j] = bias ? gld2(bias + d0 + 2 * j) : make_float2(0.f, 0.f);
    }
}

// u[i] of batch row b for i >= -3, as it lies in memory.
template <typename T>
__device__ __forceinline__ uint4 load_u(const T *x, const T *state, const ConvShape &s, int64_t b, int64_t i, int64_t d0) {
    if (i >= 0) return ld16(x + (b * s.L + i) * s.x_stride + d0);
    if (state) return ld16(state + (b * 3 + 3 + i) * s.width + d0);
    return make_uint4(0, 0, 0, 0);
}

template <typename T>
__global__ void __launch_bounds__(kFwdThreads, kFwdCtas)
    conv_kernel(const T *x, const T *state, const float *w, const float *bias, T *out, T *state_out, const ConvShape s) {
    constexpr int V = kGroup<T>, P = V / 2;
    extern __shared__ uint4 smem[];   // [kStages<T> * kStage][kFwdThreads]
    pdl_wait();
    const int64_t by = blockIdx.x / s.gx, bx = blockIdx.x - by * s.gx;
    const int64_t group = bx * s.tx + threadIdx.x % s.tx;
    const int64_t item = by * (kFwdThreads / s.tx) + threadIdx.x / s.tx;
    if (group >= s.groups || item >= s.items) return;
    const int64_t b = (uint32_t)item / (uint32_t)s.chunks;   // at most 2^28 items
    const int64_t chunk = item - b * s.chunks, d0 = group * V;
    const int64_t t0 = chunk * s.rows;
    const int n = (int)min((int64_t)s.rows, s.L - t0);
    uint4 *mine = smem + threadIdx.x;
    const T *src = x + (b * s.L + t0) * s.x_stride + d0;
    int slot = 0;
    const auto issue = [&](int r) {   // stage of the rows from r on
        if (r + kStage <= n) {
#pragma unroll
            for (int j = 0; j < kStage; ++j) copy16(mine + (slot + j) * kFwdThreads, src + j * s.x_stride);
        } else {
#pragma unroll
            for (int j = 0; j < kStage - 1; ++j)
                if (r + j < n) copy16(mine + (slot + j) * kFwdThreads, src + j * s.x_stride);
        }
        src += kStage * s.x_stride;
        copy_commit();
        slot = (slot + kStage) % (kStages<T> * kStage);
    };
#pragma unroll
    for (int k = 0; k < kStages<T> - 1; ++k) issue(k * kStage);
    float2 wv[4][P], bv[P], u[4][P];
    load_weights(w, bias, d0, wv, bv);
#pragma unroll
    for (int k = 0; k < 3; ++k) to_pairs<T>(load_u<T>(x, state, s, b, t0 - 3 + k, d0), u[k]);
    T *dst = out + (b * s.L + t0) * s.width + d0;
    const auto row = [&](int j) {
        to_pairs<T>(mine[(slot + j) * kFwdThreads], u[(j + 3) & 3]);
        float2 o[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float2 p = bv[i];
#pragma unroll
            for (int k = 0; k < 4; ++k) p = fma2(wv[k][i], u[(j + k) & 3][i], p);
            o[i] = mul2(p, mul2(sigmoid2<T>(p), splat(kDown)));
        }
        put_pairs<T>(dst, o);
        dst += s.width;
    };
    for (int r = 0; r < n; r += kStage) {
        issue(r + (kStages<T> - 1) * kStage);   // into the slots read in the round before
        copy_wait<kStages<T> - 1>();
        if (r + kStage <= n) {
#pragma unroll
            for (int j = 0; j < kStage; ++j) row(j);
        } else {
#pragma unroll
            for (int j = 0; j < kStage - 1; ++j)
                if (r + j < n) row(j);
        }
    }
    // The first chunk's thread has read the window in, so it may be written over now.
    if (chunk == 0 && state_out) {
        uint4 v[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) v[k] = load_u<T>(x, state, s, b, s.L - 3 + k, d0);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4 *>(state_out + (b * 3 + k) * s.width + d0) = v[k];
    }
}

// Gradients. part [gy][5][width]: sums of dw[0..3] and db over the CTA's chunks.
template <typename T>
__global__ void __launch_bounds__(kBwdThreads, kBwdCtas<T>)
    conv_backward_kernel(const T *x, const T *state, const float *w, const float *bias, const T *dout, const T *dstate_out,
                         T *dx, T *dstate, float *part, const ConvShape s) {
    constexpr int V = kGroup<T>, P = V / 2;
    extern __shared__ uint4 smem[];   // [kStages<T> * kStage][x, dout][kBwdThreads]
    pdl_wait();
    const int64_t by = blockIdx.x / s.gx, bx = blockIdx.x - by * s.gx;
    const int ty = kBwdThreads / s.tx;
    const int64_t group = bx * s.tx + threadIdx.x % s.tx;
    const int64_t item = by * ty + threadIdx.x / s.tx;
    float2 acc[5][P];
#pragma unroll
    for (int k = 0; k < 5; ++k)
#pragma unroll
        for (int i = 0; i < P; ++i) acc[k][i] = splat(0.f);
    if (group < s.groups && item < s.items) {
        const int64_t b = (uint32_t)item / (uint32_t)s.chunks;   // at most 2^28 items
        const int64_t chunk = item - b * s.chunks, d0 = group * V;
        const int64_t t0 = chunk * s.rows;
        const int n = (int)min((int64_t)s.rows, s.L - t0);        // steps of the chunk
        const int m = (int)min((int64_t)s.rows + 3, s.L - t0);    // and of the three after it
        uint4 *mine = smem + threadIdx.x;
        const T *xs = x + (b * s.L + t0) * s.x_stride + d0, *gs = dout + (b * s.L + t0) * s.width + d0;
        int slot = 0;
        const auto issue = [&](int r) {
            const auto one = [&](int j) {
                copy16(mine + 2 * (slot + j) * kBwdThreads, xs + j * s.x_stride);
                copy16(mine + (2 * (slot + j) + 1) * kBwdThreads, gs + j * s.width);
            };
            if (r + kStage <= m) {
#pragma unroll
                for (int j = 0; j < kStage; ++j) one(j);
            } else {
#pragma unroll
                for (int j = 0; j < kStage - 1; ++j)
                    if (r + j < m) one(j);
            }
            xs += kStage * s.x_stride;
            gs += kStage * s.width;
            copy_commit();
            slot = (slot + kStage) % (kStages<T> * kStage);
        };
#pragma unroll
        for (int k = 0; k < kStages<T> - 1; ++k) issue(k * kStage);
        float2 wv[4][P], bv[P], u[4][P], g[4][P];   // step t in u, g[(t + 3) & 3]
        load_weights(w, bias, d0, wv, bv);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            to_pairs<T>(load_u<T>(x, state, s, b, t0 - 3 + k, d0), u[k]);
#pragma unroll
            for (int i = 0; i < P; ++i) g[k][i] = splat(0.f);
        }
        T *dst = dx + (b * s.L + t0 - 3) * s.dx_stride + d0;   // of du[t-3]
        const auto grad = [&](int j) {   // g of the step in slot j
            float2 go[P];
            to_pairs<T>(mine[2 * (slot + j) * kBwdThreads], u[(j + 3) & 3]);
            to_pairs<T>(mine[(2 * (slot + j) + 1) * kBwdThreads], go);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float2 p = bv[i];
#pragma unroll
                for (int k = 0; k < 4; ++k) p = fma2(wv[k][i], u[(j + k) & 3][i], p);
                const float2 sg = sigmoid2<T>(p);
                const float2 h = fma2(p, fma2(sg, splat(-kDown * kDown), splat(kDown)), splat(kDown));   // 2^-64 (1 + p (1 - s))
                g[(j + 3) & 3][i] = mul2(go[i], mul2(sg, h));
            }
        };
        const auto sums = [&](int j) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[k][i] = fma2(g[(j + 3) & 3][i], u[(j + k) & 3][i], acc[k][i]);
                acc[4][i] = add2(acc[4][i], g[(j + 3) & 3][i]);
            }
        };
        const auto du_of = [&](int j, float2 (&du)[P]) {   // du[t-3]: complete with g[t]
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float2 v = mul2(wv[0][i], g[(j + 3) & 3][i]);
#pragma unroll
                for (int k = 1; k < 4; ++k) v = fma2(wv[k][i], g[(j + 3 - k) & 3][i], v);
                du[i] = v;
            }
        };
        for (int r = 0; r < n + 3; r += kStage) {
            issue(r + (kStages<T> - 1) * kStage);
            copy_wait<kStages<T> - 1>();
            if (r >= 3 && r + kStage <= n) {   // in the middle of the chunk
#pragma unroll
                for (int j = 0; j < kStage; ++j) {
                    float2 du[P];
                    grad(j);
                    sums(j);
                    du_of(j, du);
                    put_pairs<T>(dst, du);
                    dst += s.dx_stride;
                }
                continue;
            }
#pragma unroll
            for (int j = 0; j < kStage; ++j) {
                if (r + j < m) {
                    grad(j);
                    if (r + j < n) sums(j);   // the steps after belong to the next chunk
                } else {
#pragma unroll
                    for (int i = 0; i < P; ++i) g[(j + 3) & 3][i] = splat(0.f);
                }
                // what lies before the chunk belongs to the chunk before
                if (r + j < n + 3 && (r + j >= 3 || (chunk == 0 && dstate))) {
                    float2 du[P];
                    du_of(j, du);
                    const int64_t at = t0 + r + j - s.L;   // >= 0: u[t-3] is in the window out
                    if (at >= 0 && dstate_out) {
                        float2 e[P];
                        to_pairs<T>(ld16(dstate_out + (b * 3 + at) * s.width + d0), e);
#pragma unroll
                        for (int i = 0; i < P; ++i) du[i] = add2(du[i], e[i]);
                    }
                    if (r + j >= 3) put_pairs<T>(dst, du);
                    else put_pairs<T>(dstate + (b * 3 + r + j) * s.width + d0, du);
                }
                dst += s.dx_stride;
            }
        }
    }
    // Sum over the CTA's chunks, in their order. Rows of tx + 4 floats let the sums read channels (8 or 4 rows apart)
    // without bank conflicts; narrow ones (narrow inputs) stay tight, so that ty * 5 * V of them fit in the ring.
    copy_wait<0>();
    __syncthreads();   // the ring is free
    float *red = reinterpret_cast<float *>(smem);   // [ty][5][V][pitch]
    const int pitch = s.tx >= 8 ? s.tx + 4 : s.tx;
    {
        float *mine = red + threadIdx.x / s.tx * (5 * V * pitch) + threadIdx.x % s.tx;
#pragma unroll
        for (int k = 0; k < 5; ++k)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                mine[(k * V + 2 * i) * pitch] = acc[k][i].x;
                mine[(k * V + 2 * i + 1) * pitch] = acc[k][i].y;
            }
    }
    __syncthreads();
    const int64_t c0 = bx * s.tx * V;
    for (int c = threadIdx.x; c < s.tx * V; c += kBwdThreads) {
        if (c0 + c >= s.width) break;
#pragma unroll
        for (int k = 0; k < 5; ++k) {
            const float *at = red + (k * V + c % V) * pitch + c / V;
            float sum = 0.f;
            for (int y = 0; y < ty; ++y) sum += at[y * (5 * V * pitch)];
            part[(by * 5 + k) * s.width + c0 + c] = sum;
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

// Dynamic shared memory beyond 48 KB has to be asked for, on the device that the launch goes to (here: at every call).
template <typename K> cudaError_t allow_smem(K kernel, size_t bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T> cudaError_t forward(const ConvParams &p, cudaStream_t st) {
    const Cut c = cut_span(p.batch, p.seqlen, p.width, kGroup<T>, kFwdThreads, kFwdCtas, kFwdLongest);
    constexpr size_t smem = (size_t)kStages<T> * kStage * kFwdThreads * 16;
    if (const cudaError_t e = allow_smem(conv_kernel<T>, smem); e != cudaSuccess) return e;
    return launch_pdl(true, conv_kernel<T>, dim3((unsigned)(c.gx * c.gy)), dim3(kFwdThreads), smem, st,
                      static_cast<const T *>(p.x), static_cast<const T *>(p.state), p.w, p.bias,
                      static_cast<T *>(p.out), static_cast<T *>(p.state_out), shape_of(p, c));
}

template <typename T> cudaError_t backward(const ConvParams &p, float *part, cudaStream_t st) {
    const Cut c = cut_backward<T>(p.batch, p.seqlen, p.width);
    constexpr size_t smem = (size_t)kStages<T> * kStage * 2 * kBwdThreads * 16;
    static_assert(smem >= kBwdThreads * 5 * kGroup<T> * 3 / 2 * sizeof(float), "room for the sums: a pitch is at most 3/2 tx");
    if (c.gy > 0) {   // without batch rows the sums are zeros
        cudaError_t e = allow_smem(conv_backward_kernel<T>, smem);
        if (e == cudaSuccess)
            e = launch_pdl(true, conv_backward_kernel<T>, dim3((unsigned)(c.gx * c.gy)), dim3(kBwdThreads), smem, st,
                           static_cast<const T *>(p.x), static_cast<const T *>(p.state), p.w, p.bias,
                           static_cast<const T *>(p.dout), static_cast<const T *>(p.dstate_out), static_cast<T *>(p.dx),
                           static_cast<T *>(p.dstate), part, shape_of(p, c));
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(true, conv_sum_kernel, dim3((unsigned)((5 * p.width + kSumCols - 1) / kSumCols)),
                      dim3(kSumCols * kSumRows), 0, st, static_cast<const float *>(part), c.gy, p.width, p.dw, p.dbias);
}

}  // namespace

size_t conv_backward_scratch(int64_t batch, int64_t seqlen, int64_t width) {
    const int64_t gy =
        std::max(cut_backward<float>(batch, seqlen, width).gy, cut_backward<__nv_bfloat16>(batch, seqlen, width).gy);
    return (size_t)(gy * 5 * width) * sizeof(float);
}

cudaError_t launch_conv(const ConvParams &p, bool bf16, cudaStream_t s) {
    return bf16 ? forward<__nv_bfloat16>(p, s) : forward<float>(p, s);
}

cudaError_t launch_conv_backward(const ConvParams &p, bool bf16, float *part, cudaStream_t s) {
    return bf16 ? backward<__nv_bfloat16>(p, part, s) : backward<float>(p, part, s);
}

}  // namespace mbscan
