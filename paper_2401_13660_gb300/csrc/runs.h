// Runs of equal values in sorted keys that are cut into pieces of equal length,
// looked up by a whole warp. `vote(f)` gives a bit for each lane l whose f(l)
// holds (a ballot; all else is the same in every lane), `vote(f, g, b, c)` both
// at once, `key(i)` is the i-th key. No CUDA in here: the host compiles it too, with keys that check their index.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define MB_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define MB_HOST_DEVICE inline
#endif

namespace mbscan {

MB_HOST_DEVICE int bits_set(unsigned v) {
#ifdef __CUDA_ARCH__
    return __popc(v);
#else
    return __builtin_popcount(v);
#endif
}
MB_HOST_DEVICE int lowest_bit(unsigned v) {   // of v != 0
#ifdef __CUDA_ARCH__
    return __ffs(v) - 1;
#else
    return __builtin_ctz(v);
#endif
}

// The first q of [lo, hi) for which `from(q)` (a sorted key) is at least k, or hi.
template <typename Vote, typename From>
MB_HOST_DEVICE int64_t first_at(const Vote &vote, int64_t lo, int64_t hi, int k, const From &from) {
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32;
        const int below = bits_set(vote([&](int lane) {   // a prefix of the lanes
            const int64_t at = lo + step * lane;
            return at < hi && from(at) < k;
        }));
        if (below == 0) break;
        hi = hi < lo + step * below ? hi : lo + step * below;
        lo = lo + step * (below - 1) + 1;
    }
    return lo;
}

// Of piece p, keys [p * piece, (p + 1) * piece) of n: the pieces where the run of its first key begins and where that of
// its last key ends. A CTA of many short pieces also goes over some behind the last one: nothing runs there, and no key
// is looked up (their missing first key equals none, so the search would go back past the beginning).
struct RunEnds {
    int64_t begin, end;
};
template <typename Vote, typename Key>
MB_HOST_DEVICE RunEnds run_ends(const Vote &vote, const Key &key, int64_t n, int64_t piece, int64_t pieces, int64_t p) {
    if (p >= pieces) return {p, p};
    const auto key_at = [&](int64_t i) { return i >= 0 && i < n ? key(i) : -1; };
    const int64_t q0 = p * piece, q1 = q0 + piece;
    const int enters = key_at(q0), leaves = key_at(q1 - 1);
    unsigned b, f;   // both at once: the keys' loads overlap
    vote([&](int lane) { return key_at(q0 - 1 - lane * piece) != enters; },
         [&](int lane) { return key_at(q1 + lane * piece) != leaves; }, b, f);
    RunEnds r = {p - (b ? lowest_bit(b) : 32), p + (f ? lowest_bit(f) : 32)};
    if (!b) r.begin = first_at(vote, 0, r.begin, enters, [&](int64_t q) { return key((q + 1) * piece - 1); });
    if (leaves < 0) r.end = p;   // the last piece, cut short
    else if (!f) r.end = first_at(vote, r.end + 1, pieces, leaves + 1, [&](int64_t q) { return key(q * piece); }) - 1;
    return r;
}

}  // namespace mbscan
