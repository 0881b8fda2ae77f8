// 8-bit values with block scales, for projections whose products run in 8 bits
// (matmul.cu). A block of 128 consecutive columns (of one row: activations; of
// 128 rows: weights) shares a power of two, so that the largest value it holds
// fits e4m3's range (448 = 1.75 * 2^8):
//   E = the smallest integer >= -126 with max |x| <= 448 * 2^E   (0 where the block is all zeros)
//   q = e4m3(x * 2^-E), to nearest, ties to even; scale byte E + 127
// A power of two costs no accuracy where e4m3 is normal (the product x * 2^-E
// is exact), and the tensor cores apply it to their products themselves. NaN
// and infinities become NaN and take no part in the maximum, so that the rest
// of their block keeps its values and the error shows in what is computed from
// them.
//
// All of these are streaming kernels bound by memory: a warp takes a block at a
// time, four columns a lane (16-byte loads of fp32, 8 of bf16, 4-byte stores),
// and finds the block's maximum in one integer reduction (the bits of
// non-negative floats are ordered as they are).
#include <cuda_fp8.h>

#include "common.cuh"
#include "pairs.cuh"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kBlock = kQuantBlock;
constexpr int kWord = 4;   // blocks whose scales share a 32-bit word

__device__ __forceinline__ float4 load4(const float *p) { return gld4(p); }
// Four elements as they are in memory, and widened.
__device__ __forceinline__ float4 raw4(const float *p) { return gld4(p); }
__device__ __forceinline__ uint2 raw4(const __nv_bfloat16 *p) { return *reinterpret_cast<const uint2 *>(p); }
__device__ __forceinline__ float4 wide(const float4 &v) { return v; }
__device__ __forceinline__ float4 wide(const uint2 &u) {
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u));
}
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p) { return wide(raw4(p)); }

// The bits of |x|, 0 for what is not finite.
__device__ __forceinline__ unsigned magnitude(float x) {
    const unsigned b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}
__device__ __forceinline__ unsigned magnitude(const float4 &v) {
    return max(max(magnitude(v.x), magnitude(v.y)), max(magnitude(v.z), magnitude(v.w)));
}

// E of a block from the bits of its largest magnitude m * 2^k, 1 <= m < 2: k - 8 for m <= 1.75, else k - 7
// (fp32's own subnormals end at the lower limit). Of elements times 2^lift: E + lift.
__device__ __forceinline__ int block_exponent(unsigned top, int lift = 0) {
    if (top == 0u) return lift;
    const int k = (int)(top >> 23) - 127;
    return max((top & 0x7fffffu) > 0x600000u ? k - 7 : k - 8, lift - 126);
}
__device__ __forceinline__ int ilog(float x) { return (int)(__float_as_uint(x) >> 23 & 255u) - 127; }   // of a normal number
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }   // -126 <= e <= 127

// Four values times 2^-E as e4m3, the first in the lowest byte.
__device__ __forceinline__ unsigned round4(float2 a, float2 b, float inv) {   // no infinities
    a = mul2(a, splat(inv));
    b = mul2(b, splat(inv));
    return __nv_cvt_float2_to_fp8x2(a, __NV_SATFINITE, __NV_E4M3) |
           (unsigned)__nv_cvt_float2_to_fp8x2(b, __NV_SATFINITE, __NV_E4M3) << 16;
}
__device__ __forceinline__ float finite(float x) { return fabsf(x) <= 3.402823466e38f ? x : __uint_as_float(0x7fffffffu); }
__device__ __forceinline__ unsigned round4(const float4 &v, float inv) {
    return round4(make_float2(finite(v.x), finite(v.y)), make_float2(finite(v.z), finite(v.w)), inv);
}

// ---- the norm's arithmetic: the 8-bit value is the one nearest to the norm itself (with plain fp32 one element in 10^5
// falls on the other side of a border between two, a step of up to an eighth of its value). The sum of squares carries its
// rounding errors along; elements are formed in fp32, and only where that is too near to a border, in a block of a thousand,
// with their errors too, and where fp32's range may not hold what that takes, with their exponents apart.

struct Sum {   // hi + lo
    float hi, lo;
};
__device__ __forceinline__ Sum plus(Sum a, Sum b) {
    const float t = a.hi + b.hi, bb = t - a.hi;
    return {t, (a.hi - (t - bb)) + (b.hi - bb) + (a.lo + b.lo)};
}
// Adds the squares of two values to two sums.
__device__ __forceinline__ void add_squares(float2 &hi, float2 &lo, float2 v) {
    const float2 p = mul2(v, v), minus = splat(-1.f);
    const float2 e = fma2(v, v, mul2(p, minus));
    const float2 t = add2(hi, p), b = fma2(hi, minus, t);
    const float2 err = add2(fma2(fma2(b, minus, t), minus, hi), fma2(b, minus, p));
    hi = t;
    lo = add2(lo, add2(err, e));
}
// What is formed is the norm times 2^kLift: v * rstd is 2^15.5 at the most (the root of the width), and 2^-165 is no subnormal
// then, nor is its rounding error. No more than a constant, so that nothing waits for it.
constexpr int kLift = 64;

// 2^lift / sqrt(total / width + eps): a step of Newton's iteration gives the lower part.
__device__ __forceinline__ Sum rstd_of(Sum total, float width, float eps, int lift) {
    const float q = __fdiv_rn(total.hi, width);
    const float ql = __fdiv_rn(fmaf(-q, width, total.hi) + total.lo, width);
    const Sum x = plus({q, ql}, {eps, 0.f});
    const float r = rsqrtf(x.hi), p = r * r, pe = fmaf(r, r, -p);
    const float t = fmaf(-x.lo, p, fmaf(-x.hi, pe, fmaf(-x.hi, p, 1.f)));
    return {r * exp2i(lift), x.hi > 0.f && x.hi <= 3.402823466e38f ? exp2i(lift - 1) * r * t : 0.f};
}
// v * rstd * g, with the last bit set where that is not exact (rounding to odd): rounded again, to fewer bits, it gives what
// the product itself would. What is beyond fp32 is NaN.
__device__ __forceinline__ float odd(float q, float lo) {
    const float t = __fadd_rz(q, lo);
    return t - q != lo ? __uint_as_float(__float_as_uint(t) | 1u) : t;
}
__device__ __forceinline__ float2 normalized(float2 v, float2 g, Sum rstd) {
    const float2 minus = splat(-1.f), p = mul2(v, splat(rstd.hi));
    const float2 pe = fma2(v, splat(rstd.lo), fma2(v, splat(rstd.hi), mul2(p, minus)));
    const float2 q = mul2(p, g);
    const float2 lo = fma2(pe, g, fma2(p, g, mul2(q, minus)));
    return make_float2(odd(q.x, lo.x), odd(q.y, lo.y));
}

__device__ __forceinline__ unsigned warp_max(unsigned v) { return __reduce_max_sync(kFull, v); }

// The same with exponents apart, where fp32's range does not hold all of it: t 2^n, 1 <= |t| < 8 (or t is zero, or NaN).
struct Apart {
    float t;
    int n;
};
__device__ __forceinline__ Apart apart(float x) {   // 1 <= |t| < 2, but of zero and what is no number
    const bool low = fabsf(x) < 0x1p-126f;
    const unsigned b = __float_as_uint(low ? x * 0x1p64f : x), e = b >> 23 & 255u;
    if (e == 0u || e == 255u) return {x, 0};
    return {__uint_as_float((b & 0x807fffffu) | 0x3f800000u), (int)e - (low ? 127 + 64 : 127)};
}
__device__ __forceinline__ Apart normalized(float v, float g, Sum rstd, int n) {   // rstd times 2^n, 1 <= rstd.hi < 2
    const Apart a = apart(v), b = apart(g);
    const float p = a.t * rstd.hi, pe = fmaf(a.t, rstd.lo, fmaf(a.t, rstd.hi, -p));
    const float q = p * b.t;
    const Apart y = {odd(q, fmaf(pe, b.t, fmaf(p, b.t, -q))), a.n + b.n + n};
    return y.n + ilog(y.t) > 127 ? Apart{__uint_as_float(0x7fffffffu), 0} : y;   // beyond fp32
}
// The order of magnitudes as that of whole numbers: exponent + kLowest, 23 bits of the mantissa; what is below is 1, what is
// no number 0.
constexpr int kLowest = 161;
__device__ __forceinline__ unsigned magnitude(const Apart &y) {
    const unsigned b = magnitude(y.t);
    const int e = y.n + ilog(y.t) + kLowest;
    return b == 0u ? 0u : e > 0 ? (unsigned)e << 23 | (b & 0x7fffffu) : 1u;
}
// Bytes and E of a block of such values.
__device__ __forceinline__ uint2 round_apart(const Apart (&y)[4]) {
    const unsigned most = warp_max(max(max(magnitude(y[0]), magnitude(y[1])), max(magnitude(y[2]), magnitude(y[3]))));
    const int k = (int)(most >> 23) - kLowest;
    const int e = most == 0u ? 0 : max((most & 0x7fffffu) > 0x600000u ? k - 7 : k - 8, -126);
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = y[i].t * exp2i(min(max(y[i].n - e, -126), 127));
    return make_uint2(round4(make_float2(f[0], f[1]), make_float2(f[2], f[3]), 1.f), (unsigned)e);
}

// rstd of a row, times 2^lift, from every thread's sums of squares. One warp adds those of many up: every one would take its turn.
__device__ __forceinline__ Sum row_rstd(Sum *red, float2 hi, float2 lo, float width, float eps, int lift) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    Sum ss = plus({hi.x, lo.x}, {hi.y, lo.y});
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss = plus(ss, {__shfl_xor_sync(kFull, ss.hi, o), __shfl_xor_sync(kFull, ss.lo, o)});
    if (warps == 1) return rstd_of(ss, width, eps, lift);
    __syncthreads();
    if (lane == 0) red[warp] = ss;
    __syncthreads();
    if (warp == 0) {
        ss = lane < warps ? red[lane] : Sum{0.f, 0.f};
#pragma unroll 1
        for (int o = warps > 16 ? 16 : warps > 8 ? 8 : warps > 4 ? 4 : warps > 2 ? 2 : 1; o > 0; o >>= 1)
            ss = plus(ss, {__shfl_xor_sync(kFull, ss.hi, o), __shfl_xor_sync(kFull, ss.lo, o)});
        __syncwarp();
        if (lane == 0) red[0] = rstd_of(ss, width, eps, lift);
    }
    __syncthreads();
    return red[0];
}

// residual[row] += add[row] (when given); q, scales = the 8-bit form of residual[row] * w / sqrt(mean residual[row]^2 + eps).
// One CTA per row: warp i takes the words (four blocks) i, i + warps, ..., or single blocks with kPer = 1 (few rows:
// latency counts, and a row spread over four times the warps is there sooner). The first kPer blocks of a warp stay in
// registers between the sum of squares and the rounding; wider rows are read again.
template <typename T, int kPer>
__global__ void __launch_bounds__(kPer == 1 ? 1024 : 512, 1) rmsnorm_q8_kernel(const T *addend, float *residual, const float *w, float eps,
                                                                            uint8_t *q, uint8_t *scales, int width, int stride,
                                                                            bool early) {
    __shared__ Sum red[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int64_t row = blockIdx.x;
    float *r = residual + row * width;
    const T *a = addend ? addend + row * width : nullptr;
    const int step = warps * kPer;
    float4 kept[kPer];
    float2 hi = make_float2(0.f, 0.f), lo = hi;
    if (early) pdl_trigger();
    pdl_wait();
    for (int b0 = warp * kPer; b0 < stride; b0 += step) {
        float4 v[kPer], d[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int c = (b0 + j) * kBlock + 4 * lane;
            v[j] = c < width ? load4(r + c) : make_float4(0.f, 0.f, 0.f, 0.f);
            if (a && c < width) d[j] = load4(a + c);
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int c = (b0 + j) * kBlock + 4 * lane;
            if (a && c < width) {
                v[j].x += d[j].x; v[j].y += d[j].y; v[j].z += d[j].z; v[j].w += d[j].w;
                *reinterpret_cast<float4 *>(r + c) = v[j];
            }
            add_squares(hi, lo, make_float2(v[j].x, v[j].y));
            add_squares(hi, lo, make_float2(v[j].z, v[j].w));
            if (b0 < step) kept[j] = v[j];
        }
    }
    Sum rstd = row_rstd(red, hi, lo, (float)width, eps, kLift);
    // squares beyond fp32's range, or lost below it: the row again times a power of two
    const int up = !(rstd.hi >= exp2i(kLift - 62)) ? -80 : rstd.hi > exp2i(kLift + 50) ? 96 : 0;
    if (up != 0) {
        const float scale = exp2i(up);
        hi = lo = make_float2(0.f, 0.f);
        for (int b0 = warp * kPer; b0 < stride; b0 += step) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int c = (b0 + j) * kBlock + 4 * lane;
                const float4 v = b0 < step ? kept[j] : c < width ? load4(r + c) : make_float4(0.f, 0.f, 0.f, 0.f);
                add_squares(hi, lo, make_float2(v.x * scale, v.y * scale));
                add_squares(hi, lo, make_float2(v.z * scale, v.w * scale));
            }
        }
        rstd = row_rstd(red, hi, lo, (float)width, eps * scale * scale, 0);
    }
    const float near = rstd.hi + rstd.lo;
    constexpr unsigned kLeast = (unsigned)(127 + kLift - 17) << 23;
    bool again = up != 0;   // what fp32 may not hold all of, nor in a row that was taken times a power of two
    for (int b0 = warp * kPer; b0 < stride; b0 += step) {
        unsigned word = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int c = (b0 + j) * kBlock + 4 * lane;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f), g = v;
            if (c < width) {
                v = b0 < step ? kept[j] : load4(r + c);
                g = load4(w + c);
            }
            // within 2^-22 of the norm: times 1 - 2^-21 and 1 + 2^-21 it is rounded to the same value, or it is near a border
            const float2 v0 = make_float2(v.x, v.y), v1 = make_float2(v.z, v.w), g0 = make_float2(g.x, g.y), g1 = make_float2(g.z, g.w);
            float2 y0 = mul2(mul2(v0, splat(near)), g0), y1 = mul2(mul2(v1, splat(near)), g1);
            float top = fmaxf(fmaxf(fabsf(y0.x), fabsf(y0.y)), fmaxf(fabsf(y1.x), fabsf(y1.y)));   // passes NaN over
            const unsigned most = warp_max(__float_as_uint(top));
            int e = block_exponent(most, kLift);
            const float inv = exp2i(-e);
            unsigned bytes = round4(y0, y1, inv * (1.f - 0x1p-21f));
            const bool border = bytes != round4(y0, y1, inv * (1.f + 0x1p-21f)) || ((most + 8u) & 0x7fffffu) - 0x600000u <= 16u;
            // Where the largest value is 2^-17 or more, what is not rounded to zero is above 2^-37, so v * rstd above 2^-165
            // whatever the weights are. Below that, and beyond 2^64, fp32 may not hold what it takes. (Zeros are zeros, or
            // below 2^-213.)
            again = again || (most != 0u && (most < kLeast || most >= 0x7f7ffff0u));
            if (__any_sync(kFull, border) && most != 0u) {
                y0 = normalized(v0, g0, rstd);
                y1 = normalized(v1, g1, rstd);
                top = fmaxf(fmaxf(fabsf(y0.x), fabsf(y0.y)), fmaxf(fabsf(y1.x), fabsf(y1.y)));
                e = block_exponent(warp_max(magnitude(top)), kLift);
                bytes = round4(y0, y1, exp2i(-e));
            }
            if (c < width) *reinterpret_cast<unsigned *>(q + row * width + c) = bytes;
            word |= (unsigned)(e - kLift + 127) << (8 * j);
        }
        if (lane == 0) {
            if (kPer == 1) scales[row * stride + b0] = (uint8_t)word;
            else *reinterpret_cast<unsigned *>(scales + row * stride + b0) = word;
        }
    }
    if (!again) return;
    // This warp's blocks once more (down here: in the loop, never run, this costs 256 x 2304 0.1 us). rstd.hi is normal, or
    // the row has an infinity, or NaN.
    const int n = rstd.hi >= 0x1p-126f && rstd.hi <= 0x1p126f ? ilog(rstd.hi) : 0;
    const Sum r1 = {rstd.hi * exp2i(-n), rstd.lo * exp2i(-n)};
    const int to = n + (up != 0 ? up : -kLift);
#pragma unroll 1
    for (int b0 = warp * kPer; b0 < stride; b0 += step) {
#pragma unroll 1
        for (int j = 0; j < kPer; ++j) {
            const int c = (b0 + j) * kBlock + 4 * lane;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f), g = v;
            if (c < width) {
                v = load4(r + c);
                g = load4(w + c);
            }
            const Apart y[4] = {normalized(v.x, g.x, r1, to), normalized(v.y, g.y, r1, to), normalized(v.z, g.z, r1, to),
                                normalized(v.w, g.w, r1, to)};
            const uint2 u = round_apart(y);
            if (c < width) *reinterpret_cast<unsigned *>(q + row * width + c) = u.x;
            if (lane == 0) scales[row * stride + b0 + j] = (uint8_t)(u.y + 127u);
        }
    }
}

constexpr int kQuantThreads = 256;

// Rows of x, a warp to two words of scales (512 columns each), which may be of different rows.
template <typename T>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const T *x, int64_t x_stride, uint8_t *q, uint8_t *scales,
                                                                     int64_t rows, int width, int stride, int each, bool early) {
    using Raw = decltype(raw4(static_cast<const T *>(nullptr)));
    constexpr int kEach = 2;
    const int lane = threadIdx.x & 31, words = stride / kWord;
    const int64_t tasks = rows * words, first = ((int64_t)blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5)) * each;
    if (early) pdl_trigger();
    pdl_wait();
    Raw v[kEach][kWord];
#pragma unroll
    for (int t = 0; t < kEach; ++t) {
        const int64_t row = (first + t) / words;
        const int b0 = (int)(first + t - row * words) * kWord;
#pragma unroll
        for (int j = 0; j < kWord; ++j) {
            const int c = (b0 + j) * kBlock + 4 * lane;
            v[t][j] = t < each && first + t < tasks && c < width ? raw4(x + row * x_stride + c) : Raw{};
        }
    }
#pragma unroll
    for (int t = 0; t < kEach; ++t) {
        if (t >= each || first + t >= tasks) return;
        const int64_t row = (first + t) / words;
        const int b0 = (int)(first + t - row * words) * kWord;
        unsigned word = 0;
#pragma unroll
        for (int j = 0; j < kWord; ++j) {
            const int c = (b0 + j) * kBlock + 4 * lane;
            const float4 f = wide(v[t][j]);
            const int e = block_exponent(warp_max(magnitude(f)));
            if (c < width) *reinterpret_cast<unsigned *>(q + row * width + c) = round4(f, exp2i(-e));
            word |= (unsigned)(e + 127) << (8 * j);
        }
        if (lane == 0) *reinterpret_cast<unsigned *>(scales + row * stride + b0) = word;
    }
}

// 128 x 128 blocks, one CTA each; it keeps its 64 values a thread in registers until the block's maximum is known. There is
// a CTA for every byte of a row of scales: the bytes behind the last block become those of blocks of zeros.
template <typename T>
__global__ void __launch_bounds__(kQuantThreads) quantize_blocks_kernel(const T *x, int64_t x_stride, uint8_t *q, uint8_t *scales,
                                                                       int64_t rows, int width, int stride) {
    using Raw = decltype(raw4(static_cast<const T *>(nullptr)));
    constexpr int kWarps = kQuantThreads / 32, kRows = kBlock / kWarps;
    __shared__ unsigned red[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t down = blockIdx.x / stride, row0 = down * kBlock + warp;
    const int across = (int)(blockIdx.x - down * stride), c = across * kBlock + 4 * lane;
    pdl_wait();
    Raw v[kRows];
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        v[i] = row0 + i * kWarps < rows && c < width ? raw4(x + (row0 + i * kWarps) * x_stride + c) : Raw{};
#pragma unroll
    for (int i = 0; i < kRows; ++i) top = max(top, magnitude(wide(v[i])));
    top = warp_max(top);
    if (lane == 0) red[warp] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWarps; ++i) top = max(top, red[i]);
    const int e = block_exponent(top);
    const float inv = exp2i(-e);
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (row0 + i * kWarps < rows && c < width)
            *reinterpret_cast<unsigned *>(q + (row0 + i * kWarps) * width + c) = round4(wide(v[i]), inv);
    if (threadIdx.x == 0) scales[blockIdx.x] = (uint8_t)(e + 127);
}

// The values that q and its scales stand for, 16 columns a thread.
template <typename T>
__global__ void __launch_bounds__(kQuantThreads) dequantize_kernel(const uint8_t *q, const uint8_t *scales, int shift, T *out,
                                                                  int64_t rows, int width, int stride, bool early) {
    const int groups = width / 16;
    const int64_t i = (int64_t)blockIdx.x * kQuantThreads + threadIdx.x;
    if (early) pdl_trigger();
    pdl_wait();
    if (i >= rows * groups) return;
    const int64_t row = i / groups;
    const int c = (int)(i - row * groups) * 16;
    const uint4 u = ld16(q + row * width + c);
    const unsigned s = scales[(row >> shift) * stride + c / kBlock];
    // 2^(s - 127): byte 0 is 2^-127, subnormal, and 255 no number
    const float f = s == 255u ? __uint_as_float(0x7fffffffu) : s == 0u ? __uint_as_float(1u << 22) : __uint_as_float(s << 23);
    const unsigned word[4] = {u.x, u.y, u.z, u.w};
    float v[16];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const __nv_fp8x2_storage_t two = (__nv_fp8x2_storage_t)(word[j / 2] >> (16 * (j & 1)));
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3);   // exact
        const float2 p = __half22float2(__half2(h));
        v[2 * j] = p.x * f;
        v[2 * j + 1] = p.y * f;
    }
    T *o = out + row * width + c;
#pragma unroll
    for (int j = 0; j < 16; j += kVec<T>) {
        float g[kVec<T>];
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k) g[k] = v[j + k];
        st16(o + j, g);
    }
}

// Whether a grid leaves room for the next kernel's CTAs (see pdl_trigger's comment).
bool leaves_room(int64_t ctas) { return ctas <= 2 * (int64_t)device_sms(); }

unsigned ctas(int64_t n) { return (unsigned)((n + kQuantThreads - 1) / kQuantThreads); }

template <typename T>
cudaError_t norm(const void *add, float *residual, const float *w, float eps, uint8_t *q, uint8_t *scales, int64_t rows,
                 int width, cudaStream_t s) {
    const int stride = (int)quant_stride(width);
    // few rows: a warp to a block; many: a warp to four (65536 x 1024: 128 us; eight 140, two 134)
    const bool few = rows <= 4 * (int64_t)device_sms();
    const int per = few ? 1 : kWord, most = few ? 32 : 16;
    const int warps = (stride + per - 1) / per < most ? (stride + per - 1) / per : most;
    const auto kern = few ? rmsnorm_q8_kernel<T, 1> : rmsnorm_q8_kernel<T, kWord>;
    return launch_pdl(true, kern, dim3((unsigned)rows), dim3(32 * warps), 0, s, static_cast<const T *>(add), residual, w, eps, q,
                      scales, width, stride, leaves_room(rows));
}

template <typename T>
cudaError_t quantize(const void *x, int64_t x_stride, bool blocks, uint8_t *q, uint8_t *scales, int64_t rows, int width,
                     cudaStream_t s) {
    const int stride = (int)quant_stride(width);
    if (!blocks) {
        const int64_t tasks = rows * (stride / kWord);
        const int each = tasks * 32 > 2048 * (int64_t)device_sms() ? 2 : 1;   // a warp's, where they fill the GPU
        const unsigned grid = ctas((tasks + each - 1) / each * 32);
        return launch_pdl(true, quantize_rows_kernel<T>, dim3(grid), dim3(kQuantThreads), 0, s, static_cast<const T *>(x), x_stride,
                          q, scales, rows, width, stride, each, leaves_room(grid));
    }
    const int64_t down = (rows + kBlock - 1) / kBlock;
    return launch_pdl(true, quantize_blocks_kernel<T>, dim3((unsigned)(down * stride)), dim3(kQuantThreads), 0, s,
                      static_cast<const T *>(x), x_stride, q, scales, rows, width, stride);
}

}  // namespace

cudaError_t launch_rmsnorm_q8(const void *add, bool bf16, float *residual, const float *w, float eps, uint8_t *q,
                              uint8_t *scales, int64_t rows, int64_t width, cudaStream_t s) {
    return bf16 ? norm<__nv_bfloat16>(add, residual, w, eps, q, scales, rows, (int)width, s)
                : norm<float>(add, residual, w, eps, q, scales, rows, (int)width, s);
}

cudaError_t launch_quantize(const void *x, bool bf16, int64_t x_stride, bool blocks, uint8_t *q, uint8_t *scales, int64_t rows,
                            int64_t width, cudaStream_t s) {
    return bf16 ? quantize<__nv_bfloat16>(x, x_stride, blocks, q, scales, rows, (int)width, s)
                : quantize<float>(x, x_stride, blocks, q, scales, rows, (int)width, s);
}

cudaError_t launch_dequantize(const uint8_t *q, const uint8_t *scales, bool blocks, void *out, bool bf16, int64_t rows,
                              int64_t width, cudaStream_t s) {
    const int stride = (int)quant_stride(width), shift = blocks ? 7 : 0;
    const dim3 grid(ctas(rows * (width / 16))), block(kQuantThreads);
    const bool early = leaves_room(grid.x);
    if (bf16)
        return launch_pdl(true, dequantize_kernel<__nv_bfloat16>, grid, block, 0, s, q, scales, shift,
                          static_cast<__nv_bfloat16 *>(out), rows, (int)width, stride, early);
    return launch_pdl(true, dequantize_kernel<float>, grid, block, 0, s, q, scales, shift, static_cast<float *>(out), rows,
                      (int)width, stride, early);
}

}  // namespace mbscan
