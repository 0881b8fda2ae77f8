// Draws from next-token distributions. For a row of logits l with temperature T, weights w_i = exp((l_i - max) / T),
// tokens in the order of falling logits (of equal ones, the lower index first):
//   1. the first top_k of them;
//   2. of these, those before which there is less than top_p of their mass;
//   3. of these, those with w_i >= min_p;
//   the token: the first, by index, up to which there is more than u of the mass that is left.
//
// Every comparison is of integers. A weight is held as a whole number of units of 2^-shift (shift = 62 - log2 of the
// vocabulary: sums of a row fit 62 bits), so sums do not depend on their order, atomics included, and products with top_p
// and u are taken exactly. A weight itself is within 2^-32 of its value (weight()): a draw differs from that of exact
// arithmetic where u falls that near to a border.
//
// Rows of up to 256 tokens (bytes): one warp, eight tokens a lane, sorted in registers. Longer rows: one CTA, which keeps
// the row in shared memory, finds where top_k and top_p end by histograms of counts and masses over the distance to the
// maximum, and sorts out the one bin that holds the end.
#include "../../include/mbscan.h"
#include "common.cuh"
#include "vec.cuh"

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
    Scale s;
    s.hi = fminf(__fdiv_rn(kHi, temperature), 3.402823466e38f);
    s.lo = s.hi < 1e38f && s.hi > 1e-30f ? (fmaf(-s.hi, temperature, kHi) + kLo) / temperature : 0.f;
    s.top = top;
    s.drop = drop;
    return s;
}
// (top - l) log2(e) / T, without its lower part: never falls as l does.
__device__ __forceinline__ float distance(const Scale &s, float l) { return fminf(s.top - l, 3.402823466e38f) * s.hi; }

// 2^-y for y = (top - l) log2(e) / T. y is formed as a sum of two floats (the difference and the product with their
// rounding errors); it is split at multiples of 1/256 (P. T. P. Tang's table method, 1989), and what is left, |r| < 1/500, goes
// through the series of exp to the third power: the error is that of r's rounding, 2^-9 2^-24.
__device__ __forceinline__ u64 weight(const Scale &s, float l, const u64 *powers) {
    const float d = s.top - l;
    const float b = d - s.top;
    float e = (s.top - (d - b)) - (l + b);          // top - l = d + e
    const bool huge = !(d <= 3.402823466e38f);
    const float d1 = huge ? 3.402823466e38f : d;
    e = huge ? 0.f : e;
    const float y = d1 * s.hi;
    if (!(y < 100.f)) return 0;
    const float ylo = fmaf(d1, s.lo, fmaf(e, s.hi, fmaf(d1, s.hi, -y)));
    const int i = __float2int_rn(y * 256.f);
    const float r = fmaf((float)i, -1.f / 256.f, y) + ylo;
    const float x = r * -0.6931471805599453f;
    const float em = fmaf(x * x, fmaf(x, 1.f / 6.f, 0.5f), x);
    const u64 p = powers[i & 255];
    const long long c = __float2ll_rn((float)(unsigned)(p >> 32) * 4294967296.f * em);
    const int drop = s.drop + (i >> 8);
    return drop < 64 ? (p + (u64)c) >> drop : 0;
}

// ---- logits

// A logit as it counts: NaN as -inf, +inf as the type's largest finite number, -0 as 0.
template <typename T> __device__ __forceinline__ float clean(float l) {
    const float most = sizeof(T) == 2 ? __uint_as_float(0x7f7f0000u) : __uint_as_float(0x7f7fffffu);
    return l == l ? fminf(l, most) + 0.f : __uint_as_float(0xff800000u);
}
// The order of floats as that of unsigned numbers.
__device__ __forceinline__ unsigned key_of(float l) {
    const unsigned b = __float_as_uint(l);
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
template <typename K> __device__ __forceinline__ void sort256(K (&v)[kEach], int lane) {
#pragma unroll
    for (int size = 2; size <= kShort; size *= 2) {
#pragma unroll
        for (int step = size / 2; step > 0; step /= 2) {
            if (step >= kEach) {
                const bool down = (lane & (size / kEach)) == 0 || size == kShort;
                const bool first = (lane & (step / kEach)) == 0;
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    const K o = __shfl_xor_sync(kFull, v[j], step / kEach);
                    v[j] = (v[j] > o) == (down == first) ? v[j] : o;
                }
            } else {
#pragma unroll
                for (int j = 0; j < kEach; ++j)
                    if ((j & step) == 0)
                        exchange(v[j], v[j | step], size < kEach ? (j & size) == 0 : (lane & (size / kEach)) == 0 || size == kShort);
            }
        }
    }
}

// Logit and index in one number, larger for what comes first: 16 + 8 bits of bf16 logits, 32 + 8 of fp32 ones.
__device__ __forceinline__ unsigned pack(__nv_bfloat16, unsigned key, int i) { return key >> 16 << 8 | (unsigned)(255 - i); }
__device__ __forceinline__ unsigned unpack(__nv_bfloat16, unsigned c) { return c >> 8 << 16 | (c & 0x800000u ? 0u : 0xffffu); }
__device__ __forceinline__ u64 pack(float, unsigned key, int i) { return (u64)key << 8 | (unsigned)(255 - i); }
__device__ __forceinline__ unsigned unpack(float, u64 c) { return (unsigned)(c >> 8); }

template <typename T>
__global__ void __launch_bounds__(256) sample_short_kernel(const __grid_constant__ SampleParams a, int drop, bool early) {
    using K = decltype(pack(T{}, 0u, 0));
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
    K last = 0;   // of the tokens that stay
    if (st.k || st.nucleus) {
        K c[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) c[j] = pack(T{}, key[j], kEach * lane + j);
        sort256(c, lane);
        u64 w[kEach], mine = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const unsigned k = unpack(T{}, c[j]);
            w[j] = k > kMasked && (!st.k || kEach * lane + j < st.k) ? weight(sc, of_key(k), powers) : 0;
            mine += w[j];
        }
        u64 before = warp_before(mine, lane);
        const u64 total = __shfl_sync(kFull, before + mine, 31);
        const u64 reach = st.nucleus ? nucleus_mass(st.p, total) : ~0ull;
        int kept = 0;   // a prefix of the sorted tokens
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const unsigned k = unpack(T{}, c[j]);
            kept += k > kMasked && (!st.k || kEach * lane + j < st.k) && before < reach;
            before += w[j];
        }
        kept = __reduce_add_sync(kFull, kept);
        K mine_last = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) mine_last = ((kept - 1) & (kEach - 1)) == j ? c[j] : mine_last;
        last = __shfl_sync(kFull, mine_last, (kept - 1) / kEach);
    }
    u64 w[kEach], mine = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const bool in = key[j] > kMasked && pack(T{}, key[j], kEach * lane + j) >= last;
        w[j] = in ? weight(sc, of_key(key[j]), powers) : 0;
        if (w[j] < st.least) w[j] = 0;
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
constexpr int kList = 1024;          // tokens that are ranked one against the other

struct alignas(16) Shared {
    u64 powers[256];
    u64 mass[kBins];
    unsigned count[kBins];
    u64 warp_mass[kWarps];
    unsigned warp_count[kWarps];
    unsigned list_key[kList];
    int list_index[kList];
    u64 list_weight[kList];
    u64 found_mass;
    unsigned found_count, length, last_key;
    int found, last_index;
};

// A row's logits: where they are, and the tokens that are left of it, those of (key, index) not behind the last one.
template <typename T> struct Row {
    const T *l;
    int vocab;
    unsigned last_key = kMasked + 1;
    int last_index = 0x7fffffff;
    __device__ __forceinline__ unsigned key(int i) const { return key_of(clean<T>(to_f32(l[i]))); }
    __device__ __forceinline__ bool in(unsigned k, int i) const { return k > last_key || (k == last_key && i <= last_index); }
};

__device__ __forceinline__ void add64(u64 *p, u64 v) { atomicAdd(p, v); }

// Prefix sums of the histogram's first `bins` (a multiple of kThreads, or fewer) by every thread of the CTA: finds the bin
// in which the running sum of counts (of masses) reaches `goal`, the sum before it and what it holds.
template <bool kMass> __device__ void find_bin(Shared &sh, int bins, u64 goal) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, each = (bins + kThreads - 1) / kThreads;
    u64 mine = 0;
    __syncthreads();
    for (int j = 0; j < each; ++j) {
        const int b = threadIdx.x * each + j;
        if (b < bins) mine += kMass ? sh.mass[b] : sh.count[b];
    }
    u64 before = warp_before(mine, lane);
    if (lane == 31) sh.warp_mass[warp] = before + mine;
    __syncthreads();
    for (int i = 0; i < warp; ++i) before += sh.warp_mass[i];
    if (before < goal && before + mine >= goal)
        for (int j = 0; j < each; ++j) {
            const int b = threadIdx.x * each + j;
            const u64 v = b < bins ? (kMass ? sh.mass[b] : sh.count[b]) : 0;
            if (before < goal && before + v >= goal) {
                sh.found = b;
                sh.found_mass = before;
                sh.found_count = sh.count[b];
            }
            before += v;
        }
    __syncthreads();
}

// Sum over the CTA.
__device__ u64 block_sum(Shared &sh, u64 v) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.warp_mass[threadIdx.x >> 5] = v;
    __syncthreads();
    u64 s = 0;
    for (int i = 0; i < kWarps; ++i) s += sh.warp_mass[i];
    return s;
}

// The last token that stays where tokens stay as long as the sum of counts (kMass: of masses) before them is below `goal`.
// The histograms are of the row's tokens that are left by now; their sum reaches the goal. Narrows the row.
template <bool kMass, typename T>
__device__ void cut(Shared &sh, Row<T> &row, const Scale &sc, u64 goal) {
    find_bin<kMass>(sh, kBins, goal);
    const int bin = sh.found;
    u64 before = sh.found_mass;
    unsigned size = sh.found_count;
    const auto bin_of = [&](unsigned k) { return (int)fminf(distance(sc, of_key(k)) * kPerOctave, (float)(kBins - 1)); };
    unsigned prefix = 0, known = 0;   // bits of the key that the tokens looked at share
    // as long as they are many: by the next eight bits
    while (size > kList && known != 0xffffffffu) {
        const int shift = known == 0 ? 24 : known == 0xff000000u ? 16 : known == 0xffff0000u ? 8 : 0;
        __syncthreads();
        for (int b = threadIdx.x; b < 256; b += kThreads) {
            sh.mass[b] = 0;
            sh.count[b] = 0;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < row.vocab; i += kThreads) {
            const unsigned k = row.key(i);
            if (!row.in(k, i) || (k & known) != prefix || bin_of(k) != bin) continue;
            const unsigned b = 255u - (k >> shift & 255u);
            atomicAdd(&sh.count[b], 1u);
            if (kMass) add64(&sh.mass[b], weight(sc, of_key(k), sh.powers));
        }
        __syncthreads();
        find_bin<kMass>(sh, 256, goal - before);
        before += sh.found_mass;
        size = sh.found_count;
        prefix |= (255u - (unsigned)sh.found) << shift;
        known |= 255u << shift;
    }
    __syncthreads();
    if (size > kList) {   // all the same: the first of them by index
        const u64 w = kMass ? weight(sc, of_key(prefix), sh.powers) : 1;
        const u64 want = w ? (goal - before + w - 1) / w : size;   // at least 1: the goal is not reached before
        // a stretch of indexes to a warp, and the one that holds it token by token
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        const int stretch = (row.vocab + kThreads - 1) / kThreads * 32, i0 = warp * stretch, i1 = min(row.vocab, i0 + stretch);
        unsigned n = 0;
        for (int i = i0 + lane; i < i1; i += 32) {
            const unsigned k = row.key(i);
            n += k == prefix && row.in(k, i);
        }
        n = __reduce_add_sync(kFull, n);
        if (lane == 0) sh.warp_count[warp] = n;
        __syncthreads();
        u64 at = 0;
        for (int i = 0; i < warp; ++i) at += sh.warp_count[i];
        if (at < want && at + n >= want)
            for (int c = i0; c < i1; c += 32) {
                const unsigned k = c + lane < i1 ? row.key(c + lane) : 0u;
                const unsigned here = __ballot_sync(kFull, k == prefix && row.in(k, c + lane));
                const u64 mine = at + __popc(here & (0xffffffffu >> (31 - lane)));
                if (mine == want && (here >> lane & 1u)) {
                    sh.last_key = prefix;
                    sh.last_index = c + lane;
                }
                at += __popc(here);
            }
        __syncthreads();
        row.last_key = sh.last_key;
        row.last_index = sh.last_index;
        return;
    }
    if (threadIdx.x == 0) sh.length = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < row.vocab; i += kThreads) {
        const unsigned k = row.key(i);
        if (!row.in(k, i) || (k & known) != prefix || bin_of(k) != bin) continue;
        const unsigned at = atomicAdd(&sh.length, 1u);
        sh.list_key[at] = k;
        sh.list_index[at] = i;
        if (kMass) sh.list_weight[at] = weight(sc, of_key(k), sh.powers);
    }
    __syncthreads();
    // each against all others; the last that stays is the one at which the sum reaches the goal
    for (unsigned i = threadIdx.x; i < size; i += kThreads) {
        const unsigned k = sh.list_key[i];
        const int at = sh.list_index[i];
        u64 sum = before;
        for (unsigned j = 0; j < size; ++j) {
            const unsigned o = sh.list_key[j];
            if (o > k || (o == k && sh.list_index[j] < at)) sum += kMass ? sh.list_weight[j] : 1;
        }
        const u64 w = kMass ? sh.list_weight[i] : 1;
        if (sum < goal && sum + w >= goal) {
            sh.last_key = k;
            sh.last_index = at;
        }
    }
    __syncthreads();
    row.last_key = sh.last_key;
    row.last_index = sh.last_index;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_long_kernel(const __grid_constant__ SampleParams a, int drop, bool keep, bool early) {
    extern __shared__ __align__(16) unsigned char dyn[];
    Shared &sh = *reinterpret_cast<Shared *>(dyn);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < 256; i += kThreads) sh.powers[i] = kPowers.v[i];
    if (early) pdl_trigger();
    pdl_wait();
    const int64_t r = blockIdx.x;
    Row<T> row;
    row.l = static_cast<const T *>(a.logits) + r * a.vocab;
    row.vocab = a.vocab;
    // the row to shared memory, as it lies in its 16-byte groups
    const T *src = row.l;
    constexpr int kPer = kVec<T>;
    const int head = (int)((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / (int)sizeof(T);
    const int h = min(head, a.vocab), groups = (a.vocab - h) / kPer, tail = h + groups * kPer;
    T *copy = reinterpret_cast<T *>(dyn + sizeof(Shared)) + (kPer - head) % kPer;
    unsigned top = 0;
    const auto take = [&](int i) {
        const T v = src[i];
        if (keep) copy[i] = v;
        top = max(top, key_of(clean<T>(to_f32(v))));
    };
    if ((int)threadIdx.x < h) take(threadIdx.x);
    for (int i = tail + threadIdx.x; i < a.vocab; i += kThreads) take(i);
#pragma unroll 4
    for (int i = threadIdx.x; i < groups; i += kThreads) {
        const uint4 u = ld16(src + h + i * kPer);
        if (keep) *reinterpret_cast<uint4 *>(copy + h + i * kPer) = u;
        float f[kPer];
        widen(u, f);
#pragma unroll
        for (int j = 0; j < kPer; ++j) top = max(top, key_of(clean<T>(f[j])));
    }
    if (keep) row.l = copy;
    top = __reduce_max_sync(kFull, top);
    if (lane == 0) sh.warp_count[warp] = top;
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) top = max(top, sh.warp_count[i]);
    if (top <= kMasked) {
        if (threadIdx.x == 0) put(a, r, -1, 0, 1);
        return;
    }
    const Settings st = settings_of(a, r, drop);
    const float m = of_key(top);
    if (st.greedy || st.k == 1) {
        if (threadIdx.x == 0) sh.found = 0x7fffffff;
        __syncthreads();
        for (int i = threadIdx.x; i < row.vocab; i += kThreads)
            if (row.key(i) == top) {
                atomicMin(&sh.found, i);
                break;
            }
        __syncthreads();
        if (threadIdx.x == 0) put(a, r, sh.found, 1, 1);
        return;
    }
    const Scale sc = make_scale(st.temperature, m, drop);
    const auto histograms = [&](bool masses) {
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            sh.count[b] = 0;
            sh.mass[b] = 0;
        }
        __syncthreads();
        u64 sum = 0;
        for (int i = threadIdx.x; i < row.vocab; i += kThreads) {
            const unsigned k = row.key(i);
            if (!row.in(k, i)) continue;
            const float l = of_key(k);
            const int b = (int)fminf(distance(sc, l) * kPerOctave, (float)(kBins - 1));
            atomicAdd(&sh.count[b], 1u);
            if (masses) {
                const u64 w = weight(sc, l, sh.powers);
                if (w) add64(&sh.mass[b], w);
                sum += w;
            }
        }
        return block_sum(sh, sum);
    };
    if (st.k) {
        histograms(false);
        u64 alive = 0;
        for (int b = threadIdx.x; b < kBins; b += kThreads) alive += sh.count[b];
        if (block_sum(sh, alive) > (u64)st.k) cut<false>(sh, row, sc, st.k);
    }
    if (st.nucleus) {
        const u64 total = histograms(true);
        cut<true>(sh, row, sc, nucleus_mass(st.p, total));
    }
    // the draw: a stretch of indexes to a warp; the one that holds the token again, a sixteenth to a warp; then by one warp
    int i0 = 0, i1 = row.vocab;
    u64 t = 0, total = 0;
    const auto left = [&](int i) -> u64 {
        const unsigned k = row.key(i);
        if (!row.in(k, i)) return 0;
        const u64 w = weight(sc, of_key(k), sh.powers);
        return w >= st.least ? w : 0;
    };
    for (int level = 0; level < 2; ++level) {
        const int stretch = ((i1 - i0 + kThreads - 1) / kThreads) * 32, b0 = i0 + warp * stretch, b1 = min(i1, b0 + stretch);
        u64 sum = 0;
        for (int i = b0 + lane; i < b1; i += 32) sum += left(i);
        sum = warp_sum(sum);
        __syncthreads();
        if (lane == 0) sh.warp_mass[warp] = sum;
        __syncthreads();
        if (level == 0) {
            for (int i = 0; i < kWarps; ++i) total += sh.warp_mass[i];
            t = __umul64hi(st.u, total);
        }
        int at = 0;
        for (; at < kWarps - 1 && sh.warp_mass[at] <= t; ++at) t -= sh.warp_mass[at];
        i0 += at * stretch;
        i1 = min(i1, i0 + stretch);
    }
    if (warp == 0)
        for (int c = i0; c < i1; c += 32) {
            const u64 w = c + lane < i1 ? left(c + lane) : 0;
            const u64 before = warp_before(w, lane);
            if (before <= t && before + w > t) put(a, r, c + lane, w, total);
            const u64 sum = __shfl_sync(kFull, before + w, 31);
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
    const size_t row = ((size_t)p.vocab * sizeof(T) + 31) / 16 * 16;
    const bool keep = sizeof(Shared) + row <= lim->smem_optin;
    const cudaError_t e = cudaFuncSetAttribute(sample_long_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)lim->smem_optin);
    if (e != cudaSuccess) return e;
    return launch_pdl(true, sample_long_kernel<T>, dim3((unsigned)p.n), dim3(kThreads), sizeof(Shared) + (keep ? row : 0), s, p,
                      bits, keep, p.n <= lim->sms);
}

}  // namespace

cudaError_t launch_sample(const SampleParams &p, bool bf16, cudaStream_t s) {
    return bf16 ? launch<__nv_bfloat16>(p, s) : launch<float>(p, s);
}

}  // namespace mbscan
