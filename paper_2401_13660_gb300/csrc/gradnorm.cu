// Norm over all the tensors of a model and clipping by it:
//   norm = sqrt(sum of g^2),  out = g * (max_norm < norm < inf ? max_norm / norm : 1)
//
// The tensors' addresses and sizes travel in the kernel's parameters (nothing
// is copied to the GPU or kept there), kListMax at a time. A launch cuts its
// tensors into units of kUnit elements, of which each CTA takes an equal range.
// Squares are summed in fp32 within a warp and in 64 bits from there on (by a few
// threads: the GPU adds about two doubles per SM and clock), in an order that
// depends on the sizes only; the last CTA to arrive adds the CTAs' sums. Bound by
// memory: the gradients are read once for the norm, read and written to clip. The
// 353M-sized model (0.70 GB, into 1.41 GB): norm 114 us, 6.2 TB/s, and clip 360 us,
// 5.9 TB/s, whether loads are 4 or 8 deep, in registers or in rings of
// asynchronous copies, by 1, 2, 3 or 4 CTAs per SM.
#include <algorithm>

#include "../../include/mbscan.h"
#include "tma.cuh"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kUnit = 4096, kCtasPerSm = 2, kCtas = 152 * kCtasPerSm;
constexpr int kAhead = 4, kClipAhead = 2;   // groups loaded at once by a thread (4 to clip spill)
constexpr int kListMax = 960, kListSmall = 100;   // in 32 KB (4 KB) of kernel parameters

struct Entry {
    const void *in;
    void *out;
    int64_t numel;
    uint32_t first;   // unit
    uint32_t flags;   // kInBf16 | kOutBf16 | kWide (both 16-byte aligned)
};
enum { kInBf16 = 1, kOutBf16 = 2, kWide = 4 };

template <int N> struct List {
    int count, ctas;
    uint32_t units;
    uint16_t start[kCtas];   // the entry that a CTA's first unit lies in (searched on the GPU: ten dependent loads)
    Entry e[N];
};

template <int N> __host__ __device__ __forceinline__ uint32_t first_unit(const List<N> &l, int cta) {
    return (uint32_t)((uint64_t)l.units * (uint32_t)cta / (uint32_t)l.ctas);
}

// The CTA's part of the list, an equal range of units: f(entry, first element, end) for each tensor in it. (Units dealt
// out in turn, each CTA walking the whole list: the 353M-sized model 498 us instead of 484, with 8 CTAs per SM 627.)
template <int N, typename F> __device__ __forceinline__ void each_part(const List<N> &l, const F &f) {
    const uint32_t u0 = first_unit(l, blockIdx.x), u1 = first_unit(l, blockIdx.x + 1);
    if (u0 >= u1) return;
    for (int k = l.start[blockIdx.x]; k < l.count && l.e[k].first < u1; ++k) {
        const Entry &e = l.e[k];
        f(e, u0 > e.first ? (int64_t)(u0 - e.first) * kUnit : 0, min((int64_t)(u1 - e.first) * kUnit, e.numel));
    }
}

// Sums of squares that overflow or vanish in fp32 are kept apart, scaled by
// 2^-150 and 2^150: those of groups whose largest element is above 2^50 or below 2^-50.
// The others join their sum with its rounding error carried along (a thread adds thousands of groups in a large model:
// without it the norm of 350M elements was off by 1.2e-6).
struct Squares {
    float mid = 0.f, lost = 0.f, big = 0.f, small = 0.f;
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
            float group;
            if constexpr (N == 1) {
                group = v[0] * v[0];
            } else {
                float2 pair = mul2(make_float2(v[0], v[1]), make_float2(v[0], v[1]));
#pragma unroll
                for (int j = 2; j < N; j += 2) pair = fma2(make_float2(v[j], v[j + 1]), make_float2(v[j], v[j + 1]), pair);
                group = pair.x + pair.y;
            }
            const float term = group - lost, sum = mid + term;
            lost = (sum - mid) - term;
            mid = sum;
        }
    }
    // The warp's sum (lane 0 has it).
    __device__ __forceinline__ double warp_total() {
        float m = mid - lost;
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            m += __shfl_down_sync(kFull, m, o);
            big += __shfl_down_sync(kFull, big, o);
            small += __shfl_down_sync(kFull, small, o);
        }
        return (threadIdx.x & 31) == 0 ? (double)m + (double)big * 0x1p150 + (double)small * 0x1p-150 : 0.0;
    }
};

template <typename T> __device__ __forceinline__ void sum_range(const Entry &e, int64_t lo, int64_t hi, Squares &q) {
    constexpr int V = kVec<T>;
    const T *p = static_cast<const T *>(e.in);
    int64_t i = lo + threadIdx.x;
    if (e.flags & kWide) {
        const int64_t whole = lo + (hi - lo) / V * V;
        i = lo + threadIdx.x * V;
        for (; i + (kAhead - 1) * kThreads * V < whole; i += kAhead * kThreads * V) {
            uint4 raw[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) raw[k] = ld16(p + i + k * kThreads * V);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                float v[V];
                widen(raw[k], v);
                q.add(v);
            }
        }
        for (; i < whole; i += kThreads * V) {
            float v[V];
            widen(ld16(p + i), v);
            q.add(v);
        }
        i = whole + threadIdx.x;
    }
    for (; i < hi; i += kThreads) {
        const float v[1] = {to_f32(p[i])};
        q.add(v);
    }
}

// slots [kCtas]: the CTAs' sums; the first launch of a call sets them, later ones add to them. With `norm` (the last
// launch) the last CTA to arrive adds them up and leaves `arrived` at zero again.
template <int N>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) norm_kernel(const __grid_constant__ List<N> l, double *slots, bool first,
                                                           int *arrived, float *norm) {
    __shared__ double red[kWarps];
    __shared__ bool last;
    pdl_wait();
    Squares q;
    each_part(l, [&](const Entry &e, int64_t lo, int64_t hi) {
        if (e.flags & kInBf16) sum_range<__nv_bfloat16>(e, lo, hi, q);
        else sum_range<float>(e, lo, hi, q);
    });
    pdl_trigger();   // clipping may set up
    const int lane = threadIdx.x & 31;
    const double mine = q.warp_total();
    if (lane == 0) red[threadIdx.x / 32] = mine;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    double sum = lane < kWarps ? red[lane] : 0.0;
#pragma unroll
    for (int o = kWarps / 2; o > 0; o /= 2) sum += __shfl_down_sync(kFull, sum, o);
    if (lane == 0) {
        slots[blockIdx.x] = (first ? 0.0 : slots[blockIdx.x]) + sum;
        __threadfence();   // the sum, before its count
        last = norm && atomicAdd(arrived, 1) == (int)gridDim.x - 1;
        __threadfence();   // the count, before the others' sums
    }
    __syncwarp();
    if (!last) return;
    sum = 0.0;
    for (int i = lane; i < (int)gridDim.x; i += 32) sum += __ldcg(slots + i);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) sum += __shfl_down_sync(kFull, sum, o);
    if (lane == 0) {
        *norm = (float)sqrt(sum);
        *arrived = 0;
    }
}

// V consecutive elements, 8 or 16 bytes of them.
template <int V> __device__ __forceinline__ void load_some(const float *p, float (&v)[V]) { ldf(p, v); }
__device__ __forceinline__ void load_some(const __nv_bfloat16 *p, float (&v)[8]) { widen(ld16(p), v); }
__device__ __forceinline__ void load_some(const __nv_bfloat16 *p, float (&v)[4]) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    v[0] = __uint_as_float(u.x << 16);
    v[1] = __uint_as_float(u.x & 0xffff0000u);
    v[2] = __uint_as_float(u.y << 16);
    v[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ void store_some(float *p, const float (&v)[4]) { st16(p, v); }
__device__ __forceinline__ void store_some(__nv_bfloat16 *p, const float (&v)[8]) { st16(p, v); }
__device__ __forceinline__ void store_some(__nv_bfloat16 *p, const float (&v)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2 *>(p) =
        make_uint2(*reinterpret_cast<const unsigned *>(&a), *reinterpret_cast<const unsigned *>(&b));
}

// Elements [lo, hi) times c. A thread's group is 16 bytes of the wider type, so that a warp's stores are whole.
template <typename T, typename O> __device__ __forceinline__ void clip_range(const Entry &e, int64_t lo, int64_t hi, float c) {
    const T *p = static_cast<const T *>(e.in);
    O *o = static_cast<O *>(e.out);
    int64_t i = lo + threadIdx.x;
    if (e.flags & kWide) {
        constexpr int V = sizeof(T) > sizeof(O) ? kVec<T> : kVec<O>, kStep = kThreads * V;
        const int64_t whole = lo + (hi - lo) / V * V;
        for (i = lo + threadIdx.x * V; i < whole; i += kClipAhead * kStep) {
            float v[kClipAhead][V];
#pragma unroll
            for (int a = 0; a < kClipAhead; ++a)
                if (i + a * kStep < whole) load_some(p + i + a * kStep, v[a]);
#pragma unroll
            for (int a = 0; a < kClipAhead; ++a) {
                if (i + a * kStep >= whole) break;
#pragma unroll
                for (int j = 0; j < V; ++j) v[a][j] *= c;
                store_some(o + i + a * kStep, v[a]);
            }
        }
        i = whole + threadIdx.x;
    }
    for (; i < hi; i += kThreads) o[i] = from_f32<O>(to_f32(p[i]) * c);
}

template <int N>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) clip_kernel(const __grid_constant__ List<N> l, const float *norm, float max_norm,
                                                        bool in_place) {
    pdl_wait();
    const float n = *norm;
    const float c = n > max_norm && n < INFINITY ? max_norm / n : 1.f;
    if (in_place && c == 1.f) return;
    each_part(l, [&](const Entry &e, int64_t lo, int64_t hi) {
        switch (e.flags & (kInBf16 | kOutBf16)) {
            case 0: clip_range<float, float>(e, lo, hi, c); break;
            case kInBf16: clip_range<__nv_bfloat16, float>(e, lo, hi, c); break;
            case kOutBf16: clip_range<float, __nv_bfloat16>(e, lo, hi, c); break;
            default: clip_range<__nv_bfloat16, __nv_bfloat16>(e, lo, hi, c); break;
        }
    });
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

// Cut a filled list into the parts of `ctas` CTAs.
template <int N> void cut(List<N> &l, unsigned ctas) {
    l.ctas = (int)ctas;
    for (int c = 0, k = 0; c < l.ctas; ++c) {
        while (k + 1 < l.count && l.e[k + 1].first <= first_unit(l, c)) ++k;
        l.start[c] = (uint16_t)k;
    }
}

template <int N, typename F>
cudaError_t each_list(const mb_tensor *in, const mb_tensor *out, int64_t count, const F &launch) {
    List<N> l{};
    int64_t i = 0;
    do {
        i = fill(l, in, out, i, count);
        const cudaError_t e = launch(l, i >= count);
        if (e != cudaSuccess) return e;
    } while (i < count);
    return cudaSuccess;
}

unsigned ctas_for(uint32_t units) { return std::max(std::min<uint32_t>(units, kCtas), 1u); }

template <int N>
cudaError_t norm_of(const mb_tensor *in, int64_t count, double *slots, int *arrived, float *norm, cudaStream_t s) {
    bool first = true;
    return each_list<N>(in, nullptr, count, [&](List<N> &l, bool last) {
        const bool f = first;
        first = false;
        cut(l, f && last ? ctas_for(l.units) : kCtas);   // several launches: each with all the slots
        return launch_pdl(true, norm_kernel<N>, dim3(l.ctas), dim3(kThreads), 0, s, l, slots, f, arrived,
                          last ? norm : nullptr);
    });
}

template <int N>
cudaError_t clip_of(const mb_tensor *in, const mb_tensor *out, int64_t count, const float *norm, float max_norm,
                    cudaStream_t s) {
    return each_list<N>(in, out, count, [&](List<N> &l, bool) {
        if (l.units == 0) return cudaSuccess;
        cut(l, ctas_for(l.units));
        return launch_pdl(true, clip_kernel<N>, dim3(l.ctas), dim3(kThreads), 0, s, l, norm, max_norm, out == nullptr);
    });
}

}  // namespace

size_t grad_norm_scratch() { return kCtas * sizeof(double); }

cudaError_t launch_grad_norm(const mb_tensor *in, int64_t count, float *norm, StatusBlock *status, void *scratch,
                             cudaStream_t s) {
    double *slots = static_cast<double *>(scratch);
    int *arrived = reinterpret_cast<int *>(reinterpret_cast<char *>(status) + kStatusBytes / 2);   // zero between calls
    return count <= kListSmall ? norm_of<kListSmall>(in, count, slots, arrived, norm, s)
                               : norm_of<kListMax>(in, count, slots, arrived, norm, s);
}

cudaError_t launch_grad_clip(const mb_tensor *in, const mb_tensor *out, int64_t count, const float *norm, float max_norm,
                             cudaStream_t s) {
    return count <= kListSmall ? clip_of<kListSmall>(in, out, count, norm, max_norm, s)
                               : clip_of<kListMax>(in, out, count, norm, max_norm, s);
}

}  // namespace mbscan
