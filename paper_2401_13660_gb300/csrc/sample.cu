// Draws from next-token distributions. For a row of logits l with temperature T, weights w_i = exp((l_i - max) / T),
// tokens in the order of falling logits (of equal ones, the lower index first):
//   1. the first top_k of them;
//   2. of these, those before which there is less than top_p of their mass;
//   3. of these, those with w_i >= min_p;
//   the token: the first, by index, up to which there is more than u of the mass that is left.
//
// Every comparison is of integers. A weight is held as a whole number of units of 2^-shift (shift = 62 - log2 of the
// vocabulary: sums of a row fit 62 bits), so sums do not depend on their order, atomics included, and products with top_p
// and u are taken exactly. A weight itself is within 2^-31 of its value and one unit (weight()): a draw differs from
// that of exact arithmetic where u falls that near to a border.
//
// Rows of up to 256 tokens (bytes): one warp, eight tokens a lane, sorted in registers. Longer rows: a CTA, or a
// cluster of them where rows are few, which keeps the row in shared memory, finds where top_k and top_p end by histograms of
// counts and masses over the distance to the maximum, and sorts out the one bin that holds the end.
#include "../../include/mbscan.h"
#include "cluster.cuh"
#include "common.cuh"
#include "pairs.cuh"
#include "vec.cuh"

#include <math.h>

namespace mbscan {
namespace {

typedef unsigned long long u64;

// ---- weights

// 2^(-j / 256) in units of 2^-62.
struct Powers {
    u64 v[256];
};
constexpr Powers make_powers() {
    // 2^(-1/256) by eight square roots of 1/2 (Newton's iteration), its powers by products: a few units of 2^-52 off
    double r = 0.5;
    for (int i = 0; i < 8; ++i) {
        double s = 1.0;
        for (int k = 0; k < 60; ++k) s = 0.5 * (s + r / s);
        r = s;
    }
    Powers p{};
    double x = 1.0;
    for (int j = 0; j < 256; ++j) {
        p.v[j] = (u64)(x * 4611686018427387904.0);
        x *= r;
    }
    return p;
}
__device__ const Powers kPowers = make_powers();

// What turns logits into weights: log2(e) / T as a sum of two floats, the row's maximum.
struct Scale {
    float hi, lo, top;
    int drop;   // 62 - shift
};
__device__ __forceinline__ Scale make_scale(float temperature, float top, int drop) {
    constexpr float kHi = 1.4426950408889634f, kLo = (float)(1.4426950408889634074 - (double)kHi);
    const bool flat = !(temperature < 1e30f);
    Scale s;
    const float t = fmaxf(temperature, 0x1p-127f);   // log2(e) / T within fp32
    s.hi = flat ? 0.f : __fdiv_rn(kHi, t);
    s.lo = flat ? 0.f : __fdiv_rn(fmaf(-s.hi, t, kHi) + kLo, t);
    s.top = flat ? 0.f : top;
    s.drop = drop;
    return s;
}

// Two weights, 2^-y for y = (top - l) log2(e) / T. y is formed as a sum of two floats (the difference and the product with
// their rounding errors); it is split at multiples of 1/256 (P. T. P. Tang's table method, 1989), and what is left, |r| < 1/500,
// goes through the series of exp to the third power: the error is that of r's rounding, 2^-9 2^-24, and of the units of 2^-32
// in which the power's correction is taken. Whole numbers are made by adding 1.5 * 2^23, which leaves them in the low bits
// (conversions have a quarter of the rate), everything in fp32 is done on pairs. Logits that are masked give no number.
constexpr float kMagic = 12582912.f;
constexpr int kMagicBits = 0x4b400000;

__device__ __forceinline__ u64 power(float m, float t, int drop, const u64 *powers) {
    const int i = __float_as_int(m);
    const u64 p = powers[i & 255];
    const u64 w = p + (u64)((long long)(int)(p >> 32) * (2 * (__float_as_int(t) - kMagicBits)));
    return w >> min(drop + ((i - kMagicBits) >> 8), 63);   // w < 2^63
}
__device__ __forceinline__ void weights(const Scale &s, float2 l, const u64 *powers, u64 &w0, u64 &w1) {
    const float2 minus = splat(-1.f), top = splat(s.top), hi = splat(s.hi);
    const float2 d = fma2(l, minus, top);
    const float2 b = add2(d, splat(-s.top));
    const float2 e = fma2(add2(l, b), minus, fma2(fma2(b, minus, d), minus, top));   // top - l = d + e, where that is finite
    float2 y = mul2(d, hi);
    const float2 rest = fma2(d, splat(s.lo), fma2(e, hi, fma2(d, hi, mul2(d, splat(-s.hi)))));
    y = make_float2(fminf(y.x, 100.f), fminf(y.y, 100.f));   // nothing is left then
    const float2 m = fma2(y, splat(256.f), splat(kMagic));
    const float2 x = mul2(add2(fma2(add2(m, splat(-kMagic)), splat(-1.f / 256.f), y), rest), splat(-0.6931471805599453f));
    const float2 em = fma2(mul2(x, x), fma2(x, splat(1.f / 6.f), splat(0.5f)), x);   // |em| < 2^-9
    const float2 t = fma2(em, splat(2147483648.f), splat(kMagic));
    w0 = power(m.x, t.x, s.drop, powers);
    w1 = power(m.y, t.y, s.drop, powers);
}
// One, where few are wanted.
__device__ __noinline__ u64 weight_of(float hi, float lo, float top, int drop, float l, const u64 *powers) {
    u64 w, same;
    weights(Scale{hi, lo, top, drop}, make_float2(l, l), powers, w, same);
    return w;
}
__device__ __forceinline__ u64 weight(const Scale &s, float l, const u64 *powers) {
    return weight_of(s.hi, s.lo, s.top, s.drop, l, powers);
}

// ---- logits

// A logit as it counts: NaN as -inf, +inf as the type's largest finite number.
template <typename T> __device__ __forceinline__ float clean(float l) {
    const float most = sizeof(T) == 2 ? __uint_as_float(0x7f7f0000u) : __uint_as_float(0x7f7fffffu);
    return fminf(fmaxf(l, __uint_as_float(0xff800000u)), most);
}
// The order of floats (-0 as 0) as that of unsigned numbers.
__device__ __forceinline__ unsigned key_of(float l) {
    const unsigned b = __float_as_uint(l + 0.f);
    return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(unsigned k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr unsigned kMasked = 0x007fffffu;   // of -inf: tokens that are never drawn are no larger

// ---- a row's settings

struct Settings {
    u64 u;             // 2^64 u
    u64 p;             // 2^64 top_p
    u64 least;         // min_p in units of weights
    float temperature;
    int k;             // 0: all
    bool greedy, nucleus;
};
__device__ __forceinline__ u64 fraction(float f) {   // 2^64 f, f in [0, 1)
    return f > 0.f ? __float2ull_rd(f * 18446744073709551616.f) : 0;
}
__device__ __forceinline__ Settings settings_of(const SampleParams &a, int64_t row, int drop) {
    Settings s;
    const float u = a.u[row];
    s.u = u < 1.f ? fraction(u) : u >= 1.f ? ~0ull : 0;   // no number: 0
    s.temperature = a.temperature ? a.temperature[row] : 1.f;
    s.greedy = !(s.temperature > 0.f);
    const int k = a.top_k ? a.top_k[row] : 0;
    s.k = k > 0 && k < a.vocab ? k : 0;
    const float p = a.top_p ? a.top_p[row] : 1.f;
    s.nucleus = p < 1.f;
    s.p = s.nucleus ? fraction(p) : 0;
    const float m = a.min_p ? a.min_p[row] : 0.f;
    s.least = m > 0.f ? __float2ull_ru(fminf(m, 1.f) * __uint_as_float((unsigned)(127 + 62 - drop) << 23)) : 0;
    return s;
}
// The mass that a nucleus of `total` must reach: top_p total, rounded up, at least one unit.
__device__ __forceinline__ u64 nucleus_mass(u64 p, u64 total) {
    const u64 t = __umul64hi(p, total) + (p * total != 0);
    return t ? t : 1;
}

__device__ __forceinline__ void put(const SampleParams &a, int64_t row, int token, u64 w, u64 total) {
    if (a.wide) static_cast<long long *>(a.tokens)[row] = token;
    else static_cast<int *>(a.tokens)[row] = token;
    if (a.prob) a.prob[row] = token < 0 ? 0.f : __fdiv_rn(__ull2float_rn(w), __ull2float_rn(total));
}

__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
__device__ __forceinline__ u64 warp_before(u64 v, int lane) {   // sum over the lanes before
    u64 s = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const u64 t = __shfl_up_sync(kFull, s, o);
        if (lane >= o) s += t;
    }
    return s - v;
}

// ---- rows of up to 256 tokens

constexpr int kShort = 256, kEach = kShort / 32;

template <typename K> __device__ __forceinline__ void exchange(K &a, K &b, bool down) {
    const K hi = a > b ? a : b, lo = a > b ? b : a;
    a = down ? hi : lo;
    b = down ? lo : hi;
}
// Falling order over the warp, position 8 * lane + j.
template <int kSize, int kStep, typename K> __device__ __forceinline__ void merge_step(K (&v)[kEach], int lane) {
    const bool falls = kSize == kShort || (lane & (kSize / kEach)) == 0;   // stretches of kSize <= 8: by the position in them
    if constexpr (kStep >= kEach) {
        const bool larger = falls == ((lane & (kStep / kEach)) == 0);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const K o = __shfl_xor_sync(kFull, v[j], kStep / kEach);
            v[j] = (v[j] > o) == larger ? v[j] : o;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if ((j & kStep) == 0) exchange(v[j], v[j | kStep], kSize < kEach ? (j & kSize) == 0 : falls);
    }
    if constexpr (kStep > 1) merge_step<kSize, kStep / 2>(v, lane);
}
template <int kSize = 2, typename K> __device__ __forceinline__ void sort256(K (&v)[kEach], int lane) {
    merge_step<kSize, kSize / 2>(v, lane);
    if constexpr (kSize < kShort) sort256<kSize * 2>(v, lane);
}

template <typename T>
__global__ void __launch_bounds__(256) sample_short_kernel(const __grid_constant__ SampleParams a, int drop, bool early) {
    __shared__ u64 powers[256];
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < 256; i += blockDim.x) powers[i] = kPowers.v[i];
    if (early) pdl_trigger();
    pdl_wait();
    __syncthreads();
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (row >= a.n) return;
    const T *l = static_cast<const T *>(a.logits) + row * a.vocab;
    unsigned key[kEach];
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = kEach * lane + j;
        key[j] = i < a.vocab ? key_of(clean<T>(to_f32(l[i]))) : 0u;
        top = max(top, key[j]);
    }
    top = __reduce_max_sync(kFull, top);
    if (top <= kMasked) {   // nothing to draw
        if (lane == 0) put(a, row, -1, 0, 1);
        return;
    }
    const Settings st = settings_of(a, row, drop);
    if (st.greedy) {
        int at = kShort;
#pragma unroll
        for (int j = kEach - 1; j >= 0; --j) at = key[j] == top ? kEach * lane + j : at;
        at = __reduce_min_sync(kFull, at);
        if (lane == 0) put(a, row, at, 1, 1);
        return;
    }
    const Scale sc = make_scale(st.temperature, of_key(top), drop);
    // the tokens that stay: of larger keys than the last one's, and the first `equals` of those that have it
    unsigned last = kMasked;
    int equals = 0;
    if (st.k || st.nucleus) {
        unsigned c[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) c[j] = key[j];
        sort256(c, lane);
        u64 w[kEach], mine = 0;
#pragma unroll
        for (int j = 0; j < kEach; j += 2) {
            weights(sc, make_float2(of_key(c[j]), of_key(c[j + 1])), powers, w[j], w[j + 1]);
            if (c[j] <= kMasked || (st.k && kEach * lane + j >= st.k)) w[j] = 0;
            if (c[j + 1] <= kMasked || (st.k && kEach * lane + j + 1 >= st.k)) w[j + 1] = 0;
            mine += w[j] + w[j + 1];
        }
        u64 before = warp_before(mine, lane);
        const u64 total = __shfl_sync(kFull, before + mine, 31);
        const u64 reach = st.nucleus ? nucleus_mass(st.p, total) : ~0ull;
        int kept = 0;   // a prefix of the sorted tokens
        last = ~0u;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const bool stays = c[j] > kMasked && (!st.k || kEach * lane + j < st.k) && before < reach;
            kept += stays;
            last = stays ? min(last, c[j]) : last;
            before += w[j];
        }
        kept = __reduce_add_sync(kFull, kept);
        last = __reduce_min_sync(kFull, last);
        int above = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) above += c[j] > last;
        equals = kept - __reduce_add_sync(kFull, above);
    }
    int alike = 0;   // of the equal ones, those of lower lanes
#pragma unroll
    for (int j = 0; j < kEach; ++j) alike += key[j] == last;
    {
        const int own = alike;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int v = __shfl_up_sync(kFull, alike, o);
            if (lane >= o) alike += v;
        }
        alike -= own;
    }
    u64 w[kEach], mine = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (j % 2 == 0) weights(sc, make_float2(of_key(key[j]), of_key(key[j + 1])), powers, w[j], w[j + 1]);
        const bool in = key[j] > last || (key[j] == last && alike < equals);
        alike += key[j] == last;
        if (!in || w[j] < st.least) w[j] = 0;
        mine += w[j];
    }
    u64 upto = warp_before(mine, lane);
    const u64 total = __shfl_sync(kFull, upto + mine, 31);
    const u64 t = __umul64hi(st.u, total);   // the first token with more than this up to it
    int at = -1;
    u64 got = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (upto <= t && upto + w[j] > t) {
            at = kEach * lane + j;
            got = w[j];
        }
        upto += w[j];
    }
    if (at >= 0) put(a, row, at, got, total);   // one lane's
}

// ---- longer rows

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;          // of the distance to the maximum, kPerOctave to a factor of two
constexpr float kPerOctave = 32.f;
constexpr int kList = kThreads;      // tokens that are ranked one against the other
constexpr int kHead = 256;           // tokens among which a row is finished at once
constexpr int kMaxCtas = 8;          // of a row

struct alignas(16) Shared {
    u64 powers[256];
    unsigned low[kBins], high[kBins];   // masses of the bins; counts in `low` alone
    u64 warp[kWarps];
    u64 slot[2][kMaxCtas];
    u64 list[kList], head[kHead];       // tokens (place) of the bin that holds the end, and of those before it
    u64 weight[kList];
    u64 found_before, last;
    int found, length, ahead, length_full, ahead_full;
};

// The shared memory of the long rows' kernels: Shared, then the CTA's part of the row.
extern __shared__ __align__(16) unsigned char g_row[];

// Logit and index of a token, larger for what comes first.
__device__ __forceinline__ u64 place(float l, int i) { return (u64)key_of(l) << 32 | (unsigned)~i; }
__device__ __forceinline__ float logit_at(u64 place) { return of_key((unsigned)(place >> 32)); }
__device__ __forceinline__ int index_at(u64 place) { return (int)~(unsigned)place; }

// The CTAs of a row: one, or a cluster whose CTAs hold consecutive parts of it.
template <bool kCluster> struct Team {
    Shared &sh;
    int rank, size, phase = 0;

    __device__ __forceinline__ void sync() const {
        if (kCluster) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
    }
    // Sum over the CTA.
    __device__ u64 block_sum(u64 v) const {
        v = warp_sum(v);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5] = v;
        __syncthreads();
        u64 s = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) s += sh.warp[i];
        return s;
    }
    // One number of each CTA, known to all its threads, to every CTA. Two sets of slots take turns: a CTA that is at the
    // next exchange but one has seen every other leave this one.
    __device__ const u64 *exchange(u64 mine) {
        u64 *const slot = sh.slot[phase];
        phase ^= 1;
        if (kCluster) {
            if ((int)threadIdx.x < size)
                asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_address(&slot[rank], threadIdx.x)), "l"(mine) : "memory");
        } else if (threadIdx.x == 0) {
            slot[0] = mine;
        }
        sync();
        return slot;
    }
    __device__ u64 sum(u64 mine, u64 &before) {   // over the CTAs, and over those before
        const u64 *slot = exchange(mine);
        u64 s = 0;
        before = 0;
#pragma unroll 1
        for (int i = 0; i < size; ++i) {
            if (i == rank) before = s;
            s += slot[i];
        }
        return s;
    }
    __device__ __forceinline__ unsigned peek(const unsigned *p, int cta) const {
        return kCluster ? (unsigned)cluster_load(reinterpret_cast<const int *>(p), cta) : *p;
    }
    __device__ __forceinline__ int peek(const int *p, int cta) const { return kCluster ? cluster_load(p, cta) : *p; }
    // A token to a list of the first CTA, as long as that has room; a list that was seen full is left alone (`full`: the
    // places of one length would be handed out one after the other, to thousands of tokens in vain).
    __device__ __forceinline__ void append(int *length, u64 *list, int room, u64 v, int *full) const {
        if (*const_cast<volatile int *>(full)) return;
        int at;
        if (kCluster) {
            asm volatile("atom.shared::cluster.add.s32 %0, [%1], 1;" : "=r"(at) : "r"(cluster_address(length, 0)) : "memory");
            if (at < room) asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_address(&list[at], 0)), "l"(v) : "memory");
        } else {
            at = atomicAdd(length, 1);
            if (at < room) list[at] = v;
        }
        if (at >= room) *const_cast<volatile int *>(full) = 1;
    }
    __device__ __forceinline__ void tell(u64 *p, u64 v) const {   // the same place of every CTA, by one thread
#pragma unroll 1
        for (int i = 0; i < size; ++i)
            if (kCluster) asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_address(p, i)), "l"(v) : "memory");
            else *p = v;
    }
    __device__ __forceinline__ void tell(int *p, int v) const {
#pragma unroll 1
        for (int i = 0; i < size; ++i)
            if (kCluster) asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(cluster_address(p, i)), "r"(v) : "memory");
            else *p = v;
    }

    // The bin in which the running sum of the histogram's masses (counts) reaches `goal`, and the sum before it: found,
    // found_before. Every CTA has filled its own `bins` bins (and all have met since); each adds up an equal share of them
    // over all CTAs.
    template <bool kMass> __device__ void find_bin(int bins, u64 goal) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        const int share = bins / size, each = (share + kThreads - 1) / kThreads;   // at most 4
        u64 v[kBins / kThreads], mine = 0;
#pragma unroll
        for (int j = 0; j < kBins / kThreads; ++j) {
            const int b = threadIdx.x * each + j;
            v[j] = 0;
            if (j < each && b < share) {
                unsigned low[kMaxCtas], high[kMaxCtas];   // all on their way at once
#pragma unroll
                for (int i = 0; i < (kCluster ? kMaxCtas : 1); ++i)
                    if (i < size) {
                        low[i] = peek(&sh.low[rank * share + b], i);
                        high[i] = kMass ? peek(&sh.high[rank * share + b], i) : 0u;
                    }
#pragma unroll
                for (int i = 0; i < (kCluster ? kMaxCtas : 1); ++i)
                    if (i < size) v[j] += ((u64)high[i] << 32) + low[i];
            }
            mine += v[j];
        }
        u64 before = warp_before(mine, lane);
        if (lane == 31) sh.warp[warp] = before + mine;
        __syncthreads();
        u64 all = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
            if (i < warp) before += sh.warp[i];
            all += sh.warp[i];
        }
        u64 ahead;
        sum(all, ahead);
        before += ahead;
        if (before < goal && before + mine >= goal) {
#pragma unroll
            for (int j = 0; j < kBins / kThreads; ++j) {
                if (before < goal && before + v[j] >= goal) {
                    tell(&sh.found, rank * share + (int)threadIdx.x * each + j);
                    tell(&sh.found_before, before);
                }
                before += v[j];
            }
        }
        sync();
    }
};

// The logits of this CTA's part of a row, in 16-byte groups as they lie in memory: in shared memory as they count, or
// where they are (rows that do not fit). What a group holds beyond the row is masked.
template <typename T, bool kKept> struct Row {
    static constexpr int kPer = kVec<T>;
    const T *l;
    int vocab, offset;     // the first group starts `offset` elements before the row
    int g0, g1;            // this CTA's groups
    // the tokens that are left: those not behind the last one
    float last = -INFINITY;
    int last_index = -1;

    __device__ __forceinline__ int index(int g) const { return g * kPer - offset; }
    __device__ __forceinline__ float from_memory(int i) const {
        return i >= 0 && i < vocab ? clean<T>(to_f32(l[i])) : __uint_as_float(0xff800000u);
    }
    __device__ __forceinline__ float at(int g, int j) const {
        if (kKept) return to_f32(reinterpret_cast<const T *>(g_row + sizeof(Shared))[(g - g0) * kPer + j]);
        return from_memory(index(g) + j);
    }
    __device__ __forceinline__ void load(int g, float (&f)[kPer]) const {
        if (kKept) {
            widen(reinterpret_cast<const uint4 *>(g_row + sizeof(Shared))[g - g0], f);
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) f[j] = from_memory(index(g) + j);
        }
    }
    __device__ __forceinline__ bool in(float v, int i) const { return v > last || (v == last && i <= last_index); }
    // f(logits, first index) of this thread's groups that may hold tokens that are left: no other is as large as the last
    template <typename F> __device__ __forceinline__ void groups(F &&f) const {
#pragma unroll 1
        for (int g = g0 + (int)threadIdx.x; g < g1; g += kThreads) {
            float v[kPer];
            load(g, v);
            float most = v[0];
#pragma unroll
            for (int j = 1; j < kPer; ++j) most = fmaxf(most, v[j]);
            if (most >= last) f(v, index(g));
        }
    }
    // f(logit, index), one after the other, of the tokens that are left of groups a, a + step, ... < b
    template <typename F> __device__ __forceinline__ void each(int a, int b, int step, F &&f) const {
#pragma unroll 1
        for (int g = a; g < b; g += step) {
            float v[kPer];
            unsigned some = 0;
            load(g, v);
#pragma unroll
            for (int j = 0; j < kPer; ++j) some |= in(v[j], index(g) + j) ? 1u << j : 0u;
#pragma unroll 1
            for (; some; some &= some - 1) {
                const int j = __ffs(some) - 1;
                f(at(g, j), index(g) + j);
            }
        }
    }
    template <typename F> __device__ __forceinline__ void each(F &&f) const { each(g0 + (int)threadIdx.x, g1, kThreads, f); }
};

__device__ __forceinline__ void add_mass(Shared &sh, int b, u64 w) {   // 64 bits by two atomics of 32
    const unsigned lo = (unsigned)w;
    const unsigned was = atomicAdd(&sh.low[b], lo);
    const unsigned hi = (unsigned)(w >> 32) + (was + lo < was ? 1u : 0u);
    if (hi) atomicAdd(&sh.high[b], hi);
}
template <bool kMass> __device__ __forceinline__ void clear_bins(Shared &sh, int bins) {
    for (int b = threadIdx.x; b < bins; b += kThreads) {
        sh.low[b] = 0;
        if (kMass) sh.high[b] = 0;
    }
    __syncthreads();
}
// Never falls as l does.
__device__ __forceinline__ int bin_of(const Scale &sc, float l) {
    return __float_as_int(fmaf(fminf((sc.top - l) * sc.hi, (kBins - 1) / kPerOctave), kPerOctave, kMagic)) - kMagicBits;
}

// The end of a row whose tokens in question are few: `size` of them, this thread's first kHead places. They are the
// likeliest of the row, and more than are kept. total: the mass that top_p is of; 0: that of the top_k among these.
__device__ void finish(Shared &sh, const SampleParams &a, int64_t r, const Settings &st, const Scale &sc, int size, u64 total,
                       int ahead) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kUsed = kHead / 32;
    const bool mine = tid < size;
    const u64 at = mine ? (tid < ahead ? sh.head[tid] : sh.list[tid - ahead]) : 0;
    u64 w = mine ? weight(sc, logit_at(at), sh.powers) : 0;
    __syncthreads();
    if (mine) {
        sh.list[tid] = at;
        sh.weight[tid] = w;
    }
    __syncthreads();
    int rank = 0;
    u64 before = 0;
    if (mine) {
#pragma unroll 4
        for (int j = 0; j < size; ++j)
            if (sh.list[j] > at) {
                ++rank;
                before += sh.weight[j];
            }
    }
    const auto sum_of = [&](u64 v) {
        v = warp_sum(v);
        if (lane == 0) sh.warp[warp] = v;
        __syncthreads();
        u64 s = 0;
#pragma unroll
        for (int i = 0; i < kUsed; ++i) s += sh.warp[i];
        return s;
    };
    bool stays = mine;
    if (total == 0) {
        stays = mine && rank < st.k;
        total = sum_of(stays ? w : 0);
    }
    if (st.nucleus) stays = stays && before < nucleus_mass(st.p, total);
    if (!stays || w < st.least) w = 0;
    __syncthreads();
    if (mine) sh.weight[tid] = w;
    total = sum_of(w);
    const u64 t = __umul64hi(st.u, total);
    if (w == 0) return;
    u64 upto = 0;
#pragma unroll 4
    for (int j = 0; j < size; ++j)
        if ((unsigned)sh.list[j] > (unsigned)at) upto += sh.weight[j];   // lower indexes
    if (upto <= t && upto + w > t) put(a, r, index_at(at), w, total);
}

// Narrows the row to the tokens before which the sum of masses (counts) is below the goal: `goal_of` the sum over all that
// are left by now. Nothing changes where the sum does not reach the goal. False: the row is finished.
template <bool kMass, bool kCluster, typename T, bool kKept, typename G>
__device__ bool cut(Team<kCluster> &team, Row<T, kKept> &row, const SampleParams &a, int64_t r, const Settings &st, const Scale &sc,
                    G &&goal_of) {
    constexpr int kPer = kVec<T>;
    Shared &sh = team.sh;
    if (threadIdx.x == 0) sh.length = sh.ahead = sh.length_full = sh.ahead_full = 0;
    clear_bins<kMass>(sh, kBins);
    u64 sum = 0;
    row.groups([&](const float (&v)[kPer], int i) {
#pragma unroll
        for (int j = 0; j < kPer; j += 2) {
            const bool in0 = row.in(v[j], i + j), in1 = row.in(v[j + 1], i + j + 1);
            if (kMass) {
                u64 w0, w1;
                weights(sc, make_float2(v[j], v[j + 1]), sh.powers, w0, w1);
                if (in0) add_mass(sh, bin_of(sc, v[j]), w0);
                if (in1) add_mass(sh, bin_of(sc, v[j + 1]), w1);
                sum += (in0 ? w0 : 0) + (in1 ? w1 : 0);
            } else {
                if (in0) atomicAdd(&sh.low[bin_of(sc, v[j])], 1u);
                if (in1) atomicAdd(&sh.low[bin_of(sc, v[j + 1])], 1u);
                sum += (in0 ? 1 : 0) + (in1 ? 1 : 0);
            }
        }
    });
    u64 before;
    const u64 total = team.sum(team.block_sum(sum), before), goal = goal_of(total);
    if (total < goal) return true;
    team.template find_bin<kMass>(kBins, goal);
    const int bin = sh.found;
    before = sh.found_before;
    if (!kMass && before > kHead && threadIdx.x == 0) sh.ahead_full = sh.ahead = kHead + 1;   // not to be finished at once
    if (!kMass) __syncthreads();
    unsigned prefix = 0, known = 0;   // bits of the key that the tokens looked at share
    for (;;) {
        // the tokens in question, to the first CTA, and those before them
        row.groups([&](const float (&v)[kPer], int i) {
            unsigned some = 0;
            const int least = known == 0 && !*const_cast<volatile int *>(&sh.ahead_full) ? 0 : bin;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int b = bin_of(sc, v[j]);
                some |= b >= least && b <= bin && row.in(v[j], i + j) ? 1u << j : 0u;
            }
#pragma unroll 1
            for (; some; some &= some - 1) {
                const int j = __ffs(some) - 1;
                const float l = row.at((i + j + row.offset) / kPer, j);
                if (bin_of(sc, l) < bin) {
                    team.append(&sh.ahead, sh.head, kHead, place(l, i + j), &sh.ahead_full);
                } else if ((key_of(l) & known) == prefix) {
                    team.append(&sh.length, sh.list, kList, place(l, i + j), &sh.length_full);
                }
            }
        });
        team.sync();
        const int size = team.peek(&sh.length, 0), ahead = team.peek(&sh.ahead, 0);
        if (known == 0 && ahead + size <= kHead) {
            if (kCluster) team.sync();   // all have seen that
            if (team.rank == 0) finish(sh, a, r, st, sc, ahead + size, kMass ? total : 0, ahead);
            return false;
        }
        if (size <= kList) {
            // each against all others; the last that stays is the one at which the sum reaches the goal
            if (team.rank == 0) {
                const u64 at = (int)threadIdx.x < size ? sh.list[threadIdx.x] : 0;
                if (kMass) {
                    if (at) sh.weight[threadIdx.x] = weight(sc, logit_at(at), sh.powers);
                    __syncthreads();
                }
                if (at) {
                    u64 mine = before;
#pragma unroll 4
                    for (int j = 0; j < size; ++j)
                        if (sh.list[j] > at) mine += kMass ? sh.weight[j] : 1;
                    const u64 w = kMass ? sh.weight[threadIdx.x] : 1;
                    if (mine < goal && mine + w >= goal) team.tell(&sh.last, at);
                }
            }
            break;
        }
        if (known == 0xffffffffu) {   // all the same: the first of them by index
            const float l = of_key(prefix);
            const u64 w = kMass ? weight(sc, l, sh.powers) : 1;
            const u64 want = (goal - before + w - 1) / w;   // w > 0: the sum reaches the goal among them
            // a stretch of groups to a thread; the one that holds it token by token
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
            const int stretch = (row.g1 - row.g0 + kThreads - 1) / kThreads, first = row.g0 + (int)threadIdx.x * stretch;
            const int end = min(row.g1, first + stretch);
            u64 mine = 0;
            row.each(first, end, 1, [&](float o, int) { mine += o == l; });
            u64 upto = warp_before(mine, lane), ahead_of;
            __syncthreads();
            if (lane == 31) sh.warp[warp] = upto + mine;
            __syncthreads();
            u64 all = 0;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
                if (i < warp) upto += sh.warp[i];
                all += sh.warp[i];
            }
            team.sum(all, ahead_of);
            upto += ahead_of;
            if (upto < want && upto + mine >= want)
                row.each(first, end, 1, [&](float o, int i) {
                    if (o == l && ++upto == want) team.tell(&sh.last, place(l, i));
                });
            break;
        }
        // too many: those that share the next eight bits of the key
        team.sync();   // all have seen the length
        const int shift = known == 0 ? 24 : known == 0xff000000u ? 16 : known == 0xffff0000u ? 8 : 0;
        if (threadIdx.x == 0) sh.length = sh.ahead = sh.length_full = sh.ahead_full = 0;
        clear_bins<kMass>(sh, 256);
        row.each([&](float l, int) {
            if (bin_of(sc, l) != bin || (key_of(l) & known) != prefix) return;
            const int b = (int)(255u - (key_of(l) >> shift & 255u));
            if (kMass) add_mass(sh, b, weight(sc, l, sh.powers));
            else atomicAdd(&sh.low[b], 1u);
        });
        team.sync();
        team.template find_bin<kMass>(256, goal - before);
        before += sh.found_before;
        prefix |= (255u - (unsigned)sh.found) << shift;
        known |= 255u << shift;
    }
    team.sync();
    row.last = logit_at(sh.last);
    row.last_index = index_at(sh.last);
    return true;
}

template <typename T, bool kCluster, bool kKept>
__global__ void __launch_bounds__(kThreads, 2) sample_long_kernel(const __grid_constant__ SampleParams a, int drop, int ctas,
                                                                  bool early) {
    Shared &sh = *reinterpret_cast<Shared *>(g_row);
    if (kCluster) cluster_arrive();   // everybody is there before the first exchange
    constexpr int kPer = kVec<T>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < 256; i += kThreads) sh.powers[i] = kPowers.v[i];
    if (early) pdl_trigger();
    pdl_wait();
    const int64_t r = blockIdx.x / (unsigned)ctas;
    Team<kCluster> team{sh, (int)(blockIdx.x % (unsigned)ctas), ctas};
    Row<T, kKept> row;
    row.l = static_cast<const T *>(a.logits) + r * a.vocab;
    row.vocab = a.vocab;
    row.offset = (int)(reinterpret_cast<uintptr_t>(row.l) & 15) / (int)sizeof(T);
    const int groups = (row.offset + a.vocab + kPer - 1) / kPer;
    row.g0 = (int)((int64_t)groups * team.rank / ctas);
    row.g1 = (int)((int64_t)groups * (team.rank + 1) / ctas);
    uint4 *const copy = reinterpret_cast<uint4 *>(g_row + sizeof(Shared));
    float top = __uint_as_float(0xff800000u);
    const auto take = [&](int g, const float (&f)[kPer]) {
        if (kKept) copy[g - row.g0] = narrow(f);
#pragma unroll
        for (int j = 0; j < kPer; ++j) top = fmaxf(top, f[j]);
    };
    // the whole groups of the row, and the two that may be cut
    const int whole0 = (row.offset + kPer - 1) / kPer, whole1 = (row.offset + a.vocab) / kPer;
#pragma unroll 4
    for (int g = max(row.g0, whole0) + (int)threadIdx.x; g < min(row.g1, whole1); g += kThreads) {
        float f[kPer];
        widen(ld16(row.l + row.index(g)), f);
#pragma unroll
        for (int j = 0; j < kPer; ++j) f[j] = clean<T>(f[j]);
        take(g, f);
    }
    if (threadIdx.x < 2) {
        const int g = threadIdx.x == 0 ? 0 : groups - 1;
        if (g >= row.g0 && g < row.g1 && (g < whole0 || g >= whole1)) {
            float f[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) f[j] = row.from_memory(row.index(g) + j);
            take(g, f);
        }
    }
    {
        const unsigned k = __reduce_max_sync(kFull, key_of(top));
        if (lane == 0) sh.warp[warp] = k;
        __syncthreads();
        u64 best = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) best = max(best, sh.warp[i]);
        if (kCluster) cluster_wait();
        const u64 *slot = team.exchange(best);
#pragma unroll 1
        for (int i = 0; i < ctas; ++i) best = max(best, slot[i]);
        top = of_key((unsigned)best);
    }
    if (!(top > __uint_as_float(0xff800000u))) {
        if (team.rank == 0 && threadIdx.x == 0) put(a, r, -1, 0, 1);
        return;
    }
    const Settings st = settings_of(a, r, drop);
    if (st.greedy || st.k == 1) {
        int at = 0x7fffffff;
        row.each([&](float l, int i) { at = l == top ? min(at, i) : at; });
        at = __reduce_min_sync(kFull, at);
        __syncthreads();
        if (lane == 0) sh.warp[warp] = (u64)at;
        __syncthreads();
        u64 first = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) first = min(first, sh.warp[i]);
        const u64 *slot = team.exchange(first);
#pragma unroll 1
        for (int i = 0; i < ctas; ++i) first = min(first, slot[i]);
        if (team.rank == 0 && threadIdx.x == 0) put(a, r, (int)first, 1, 1);
        return;
    }
    const Scale sc = make_scale(st.temperature, top, drop);
    if (st.k && !cut<false>(team, row, a, r, st, sc, [&](u64) { return (u64)st.k; })) return;
    if (st.nucleus && !cut<true>(team, row, a, r, st, sc, [&](u64 total) { return nucleus_mass(st.p, total); })) return;
    // the draw: the CTA, then the warp that holds the token (by a stretch of groups each), then by groups of 32 lanes
    const auto left = [&](float l) -> u64 {
        const u64 w = weight(sc, l, sh.powers);
        return w >= st.least ? w : 0;
    };
    int g0 = row.g0, g1 = row.g1;
    u64 t = 0, total = 0;
#pragma unroll 1
    for (int level = 0; level < 2; ++level) {
        const int stretch = (g1 - g0 + kThreads - 1) / kThreads * 32, b0 = g0 + warp * stretch, b1 = min(g1, b0 + stretch);
        u64 sum = 0;
#pragma unroll 1
        for (int c = b0; c < b1; c += 32) {
            const int g = min(c + lane, b1 - 1);
            float v[kPer];
            row.load(g, v);
            unsigned some = 0;
#pragma unroll
            for (int j = 0; j < kPer; ++j) some |= c + lane < b1 && row.in(v[j], row.index(g) + j) ? 1u << j : 0u;
            // all of the group, or one after the other where no lane has many (a group of eight costs three of these)
            if (__any_sync(kFull, __popc(some) * 3 > kPer)) {
#pragma unroll
                for (int j = 0; j < kPer; j += 2) {
                    u64 w0, w1;
                    weights(sc, make_float2(v[j], v[j + 1]), sh.powers, w0, w1);
                    sum += (some >> j & 1u && w0 >= st.least ? w0 : 0) + (some >> j & 2u && w1 >= st.least ? w1 : 0);
                }
            } else {
                for (; some; some &= some - 1) sum += left(row.at(g, __ffs(some) - 1));
            }
        }
        sum = warp_sum(sum);
        __syncthreads();
        if (lane == 0) sh.warp[warp] = sum;
        __syncthreads();
        if (level == 0) {
            u64 mine = 0, before;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) mine += sh.warp[i];
            total = team.sum(mine, before);
            t = __umul64hi(st.u, total);
            if (t < before || t >= before + mine) return;   // another CTA's
            t -= before;
        }
        int at = 0;
        for (; at < kWarps - 1 && sh.warp[at] <= t; ++at) t -= sh.warp[at];
        g0 += at * stretch;
        g1 = min(g1, g0 + stretch);
    }
    if (warp != 0) return;
#pragma unroll 1
    for (int c = g0; c < g1; c += 32) {
        u64 mine = 0;
        row.each(c + lane, min(g1, c + lane + 1), 1, [&](float l, int) { mine += left(l); });
        u64 upto = warp_before(mine, lane);
        const u64 sum = __shfl_sync(kFull, upto + mine, 31);
        if (upto <= t && upto + mine > t)
            row.each(c + lane, c + lane + 1, 1, [&](float l, int i) {
                const u64 w = left(l);
                if (upto <= t && upto + w > t) put(a, r, i, w, total);
                upto += w;
            });
        if (sum > t) break;
        t -= sum;
    }
}

template <typename T> cudaError_t launch(const SampleParams &p, cudaStream_t s) {
    int bits = 0;
    while (((int64_t)1 << bits) < p.vocab) ++bits;
    const DeviceLimits *lim = device_limits();
    if (!lim) return cudaErrorInvalidDevice;
    if (p.vocab <= kShort) {
        const int warps = p.n <= 4 * (int64_t)lim->sms ? 2 : 8;
        return launch_pdl(true, sample_short_kernel<T>, dim3((unsigned)((p.n + warps - 1) / warps)), dim3(32 * warps), 0, s, p,
                          bits, p.n <= 4 * (int64_t)lim->sms);
    }
    // CTAs of a row: as many as leave each of them 2048 tokens and the GPU two to an SM, or as its logits need
    constexpr int kPer = kVec<T>;
    const auto bytes = [&](int ctas) { return sizeof(Shared) + ((size_t)p.vocab / kPer / ctas + 3) * 16; };
    int ctas = 1;
    while (ctas < kMaxCtas && (bytes(ctas) > lim->smem_optin ||
                               (p.n * ctas <= (int64_t)lim->sms && p.vocab >= 4096 * ctas)))
        ctas *= 2;
    const bool keep = bytes(ctas) <= lim->smem_optin;
    const auto kern = !keep      ? sample_long_kernel<T, true, false>
                      : ctas > 1 ? sample_long_kernel<T, true, true>
                                 : sample_long_kernel<T, false, true>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)lim->smem_optin);
    if (e != cudaSuccess) return e;
    if (p.n > INT32_MAX / ctas) return cudaErrorInvalidValue;
    return launch_cluster(true, kern, dim3((unsigned)(p.n * ctas)), dim3(kThreads), ctas, keep ? bytes(ctas) : sizeof(Shared), s, p,
                          bits, ctas, p.n * ctas <= lim->sms);
}

}  // namespace

cudaError_t launch_sample(const SampleParams &p, bool bf16, cudaStream_t s) {
    return bf16 ? launch<__nv_bfloat16>(p, s) : launch<float>(p, s);
}

}  // namespace mbscan
