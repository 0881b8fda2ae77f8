// Norm over all the tensors of a model and clipping by it:
//   norm = sqrt(sum of g^2),  out = g * (max_norm < norm < inf ? max_norm / norm : 1)
//
// The tensors' addresses and sizes travel in the kernel's parameters (nothing
// is copied to the GPU or kept there), kListMax at a time. A launch cuts its
// tensors' elements, laid end to end in units of kUnit, into one equal range
// per CTA. Squares are summed in fp32 per thread and in 64 bits from there on,
// in an order that depends on the sizes only.
#include <algorithm>

#include "../../include/mbscan.h"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kThreads = 512, kUnit = 4096, kCtas = 2 * 152;
constexpr int kListMax = 960, kListSmall = 100;   // of 32 KB (4 KB) of kernel parameters

struct Entry {
    const void *in;
    void *out;
    int64_t numel;
    uint32_t first;   // unit
    uint32_t flags;   // kInBf16 | kOutBf16 | kWide (both 16-byte aligned)
};
enum { kInBf16 = 1, kOutBf16 = 2, kWide = 4 };

template <int N> struct List {
    int count;
    uint32_t units;
    Entry e[N];
};

// The entry that unit u lies in.
template <int N> __device__ __forceinline__ int find(const List<N> &l, uint32_t u) {
    int lo = 0, hi = l.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (l.e[mid].first <= u) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Sums of squares that overflow or vanish in fp32 are kept apart, scaled by
// 2^-150 and 2^150: those of groups whose largest element is above 2^50 or below 2^-50.
struct Squares {
    float mid = 0.f, big = 0.f, small = 0.f;
    template <int N> __device__ __forceinline__ void add(const float (&v)[N]) {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) top = fmaxf(top, fabsf(v[j]));
        if (top > 0x1p50f) {
#pragma unroll
            for (int j = 0; j < N; ++j) big = fmaf(v[j] * 0x1p-75f, v[j] * 0x1p-75f, big);
        } else if (top < 0x1p-50f && top > 0.f) {
#pragma unroll
            for (int j = 0; j < N; ++j) small = fmaf(v[j] * 0x1p75f, v[j] * 0x1p75f, small);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) mid = fmaf(v[j], v[j], mid);
        }
    }
    __device__ __forceinline__ double total() const {
        return (double)mid + (double)big * 0x1p150 + (double)small * 0x1p-150;
    }
};

template <typename T> __device__ __forceinline__ void sum_range(const Entry &e, int64_t lo, int64_t hi, Squares &q) {
    const T *p = static_cast<const T *>(e.in);
    if (e.flags & kWide) {
        const int64_t whole = lo + (hi - lo) / kVec<T> * kVec<T>;
        for (int64_t i = lo + threadIdx.x * kVec<T>; i < whole; i += kThreads * kVec<T>) {
            float v[kVec<T>];
            widen(ld16(p + i), v);
            q.add(v);
        }
        lo = whole;
    }
    for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
        const float v[1] = {to_f32(p[i])};
        q.add(v);
    }
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double red[kThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(kFull, v, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) v += red[i];
    __syncthreads();
    return v;
}

// slots [kCtas]: the CTAs' sums; the first launch of a call sets them, later ones add to them.
template <int N>
__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ List<N> l, double *slots, bool first) {
    pdl_wait();
    const uint32_t u0 = (uint32_t)((uint64_t)l.units * blockIdx.x / gridDim.x);
    const uint32_t u1 = (uint32_t)((uint64_t)l.units * (blockIdx.x + 1) / gridDim.x);
    Squares q;
    if (u0 < u1) {
        for (int k = find(l, u0); k < l.count && l.e[k].first < u1; ++k) {
            const Entry &e = l.e[k];
            const int64_t lo = u0 > e.first ? (int64_t)(u0 - e.first) * kUnit : 0;
            const int64_t hi = min((int64_t)(u1 - e.first) * kUnit, e.numel);
            if (e.flags & kInBf16) sum_range<__nv_bfloat16>(e, lo, hi, q);
            else sum_range<float>(e, lo, hi, q);
        }
    }
    const double sum = block_sum(q.total());
    if (threadIdx.x == 0) slots[blockIdx.x] = (first ? 0.0 : slots[blockIdx.x]) + sum;
}

__global__ void __launch_bounds__(kThreads) norm_finish_kernel(const double *slots, float *norm) {
    pdl_wait();
    const double sum = block_sum(threadIdx.x < kCtas ? slots[threadIdx.x] : 0.0);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

template <typename T, typename O> __device__ __forceinline__ void clip_range(const Entry &e, int64_t lo, int64_t hi, float c) {
    const T *p = static_cast<const T *>(e.in);
    O *o = static_cast<O *>(e.out);
    if (e.flags & kWide) {
        constexpr int V = kVec<T> < kVec<O> ? kVec<O> : kVec<T>;   // 8 if either is bf16
        const int64_t whole = lo + (hi - lo) / V * V;
        for (int64_t i = lo + threadIdx.x * V; i < whole; i += kThreads * V) {
            float v[V];
#pragma unroll
            for (int j = 0; j < V; j += kVec<T>) {
                float x[kVec<T>];
                widen(ld16(p + i + j), x);
#pragma unroll
                for (int k = 0; k < kVec<T>; ++k) v[j + k] = x[k] * c;
            }
#pragma unroll
            for (int j = 0; j < V; j += kVec<O>) {
                float x[kVec<O>];
#pragma unroll
                for (int k = 0; k < kVec<O>; ++k) x[k] = v[j + k];
                st16(o + i + j, x);
            }
        }
        lo = whole;
    }
    for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) o[i] = from_f32<O>(to_f32(p[i]) * c);
}

template <int N>
__global__ void __launch_bounds__(kThreads) clip_kernel(const __grid_constant__ List<N> l, const float *norm, float max_norm,
                                                        bool in_place) {
    pdl_wait();
    const float n = *norm;
    const float c = n > max_norm && n < INFINITY ? max_norm / n : 1.f;
    if (in_place && c == 1.f) return;
    const uint32_t u0 = (uint32_t)((uint64_t)l.units * blockIdx.x / gridDim.x);
    const uint32_t u1 = (uint32_t)((uint64_t)l.units * (blockIdx.x + 1) / gridDim.x);
    if (u0 >= u1) return;
    for (int k = find(l, u0); k < l.count && l.e[k].first < u1; ++k) {
        const Entry &e = l.e[k];
        const int64_t lo = u0 > e.first ? (int64_t)(u0 - e.first) * kUnit : 0;
        const int64_t hi = min((int64_t)(u1 - e.first) * kUnit, e.numel);
        switch (e.flags & (kInBf16 | kOutBf16)) {
            case 0: clip_range<float, float>(e, lo, hi, c); break;
            case kInBf16: clip_range<__nv_bfloat16, float>(e, lo, hi, c); break;
            case kOutBf16: clip_range<float, __nv_bfloat16>(e, lo, hi, c); break;
            default: clip_range<__nv_bfloat16, __nv_bfloat16>(e, lo, hi, c); break;
        }
    }
}

// Fill a list from tensors i .. of `in` (and `out`, or null); returns how many fitted.
template <int N> int64_t fill(List<N> &l, const mb_tensor *in, const mb_tensor *out, int64_t i, int64_t count) {
    l.count = 0;
    l.units = 0;
    int64_t k = i;
    for (; k < count && l.count < N; ++k) {
        if (in[k].numel == 0) continue;
        const int64_t units = (in[k].numel + kUnit - 1) / kUnit;
        if (l.units + units > 0x7fffffff) break;
        const void *o = out ? out[k].data : in[k].data;
        Entry &e = l.e[l.count++];
        e.in = in[k].data;
        e.out = const_cast<void *>(o);
        e.numel = in[k].numel;
        e.first = l.units;
        e.flags = (in[k].dtype == MB_BF16 ? kInBf16 : 0) | ((out ? out : in)[k].dtype == MB_BF16 ? kOutBf16 : 0) |
                  (((reinterpret_cast<uintptr_t>(e.in) | reinterpret_cast<uintptr_t>(o)) & 15u) == 0 ? kWide : 0);
        l.units += (uint32_t)units;
    }
    return k;
}

template <int N, typename F>
cudaError_t each_list(const mb_tensor *in, const mb_tensor *out, int64_t count, const F &launch) {
    List<N> l;
    int64_t i = 0;
    do {
        i = fill(l, in, out, i, count);
        const cudaError_t e = launch(l, std::min<uint32_t>(l.units, kCtas));
        if (e != cudaSuccess) return e;
    } while (i < count);
    return cudaSuccess;
}

template <int N> cudaError_t norm_of(const mb_tensor *in, int64_t count, double *slots, cudaStream_t s) {
    bool first = true;
    return each_list<N>(in, nullptr, count, [&](const List<N> &l, uint32_t) {
        const bool f = first;
        first = false;
        return launch_pdl(true, norm_kernel<N>, dim3(kCtas), dim3(kThreads), 0, s, l, slots, f);
    });
}

template <int N>
cudaError_t clip_of(const mb_tensor *in, const mb_tensor *out, int64_t count, const float *norm, float max_norm,
                    cudaStream_t s) {
    return each_list<N>(in, out, count, [&](const List<N> &l, uint32_t ctas) {
        if (ctas == 0) return cudaSuccess;
        return launch_pdl(true, clip_kernel<N>, dim3(ctas), dim3(kThreads), 0, s, l, norm, max_norm, out == nullptr);
    });
}

}  // namespace

size_t grad_norm_scratch() { return kCtas * sizeof(double); }

cudaError_t launch_grad_norm(const mb_tensor *in, int64_t count, float *norm, void *scratch, cudaStream_t s) {
    double *slots = static_cast<double *>(scratch);
    const cudaError_t e = count <= kListSmall ? norm_of<kListSmall>(in, count, slots, s) : norm_of<kListMax>(in, count, slots, s);
    if (e != cudaSuccess) return e;
    return launch_pdl(true, norm_finish_kernel, dim3(1), dim3(kThreads), 0, s, static_cast<const double *>(slots), norm);
}

cudaError_t launch_grad_clip(const mb_tensor *in, const mb_tensor *out, int64_t count, const float *norm, float max_norm,
                             cudaStream_t s) {
    return count <= kListSmall ? clip_of<kListSmall>(in, out, count, norm, max_norm, s)
                               : clip_of<kListMax>(in, out, count, norm, max_norm, s);
}

}  // namespace mbscan
