// Embedding lookup with scaling, and the table's gradient by sorted tokens.
//
//   out[i] = scale * table[tokens[i]]                      (zeros where the token is outside the table)
//   dtable[v] (+)= scale * sum_{i: tokens[i] = v} dout[i]
//
// Both are bound by memory: out is written, dout read once.
//
// The gradient first sorts the token positions by token (stable, so that every
// sum has one order), then adds the rows of dout in that order. The sorted
// positions are cut into pieces: a run of equal tokens inside one piece is
// written at once, one that spans pieces leaves a partial sum in each, and the
// last to arrive adds them up in their order. So a token of a third of the text
// costs no more than a rare one, and the result depends on the inputs alone.
#include <algorithm>

#include "cluster.cuh"
#include "runs.h"
#include "tokens.cuh"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kThreads = 256, kSms = 152;

// Four elements, widened.
__device__ __forceinline__ void ld4(const float *p, float (&v)[4]) { ldf(p, v); }
__device__ __forceinline__ void ld4(const __nv_bfloat16 *p, float (&v)[4]) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    v[0] = __uint_as_float(u.x << 16);
    v[1] = __uint_as_float(u.x & 0xffff0000u);
    v[2] = __uint_as_float(u.y << 16);
    v[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ void st4(float *p, const float (&v)[4]) { stf(p, v); }
__device__ __forceinline__ void st4(__nv_bfloat16 *p, const float (&v)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2 *>(p) =
        make_uint2(*reinterpret_cast<const unsigned *>(&a), *reinterpret_cast<const unsigned *>(&b));
}

// CTA (block of rows, column tile): each thread four columns of kRows rows, the tokens loaded first.
constexpr int kRows = 4;
struct LookupArgs {
    const void *tokens;
    int type, vocab, tx;   // tx threads side by side in a row
    float scale;
    int64_t n, width;
};

template <typename T, typename O>
__global__ void __launch_bounds__(kThreads) embed_kernel(const T *table, O *out, const LookupArgs a) {
    pdl_wait();
    const int64_t c = ((int64_t)blockIdx.y * a.tx + threadIdx.x % a.tx) * 4;
    if (c >= a.width) return;
    const int ty = kThreads / a.tx;
    const int64_t row = (int64_t)blockIdx.x * ty * kRows + threadIdx.x / a.tx;
    int tok[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) tok[k] = row + k * ty < a.n ? load_token(a.tokens, a.type, row + k * ty, a.vocab) : -1;
    float v[kRows][4];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        if (tok[k] >= 0) ld4(table + tok[k] * a.width + c, v[k]);
        else v[k][0] = v[k][1] = v[k][2] = v[k][3] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        if (row + k * ty >= a.n) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] = tok[k] >= 0 ? v[k][j] * a.scale : 0.f;
        st4(out + (row + k * ty) * a.width + c, v[k]);
    }
}

// ---- sort: one cluster of kSortCtas CTAs, a stable counting sort per 8 bits
// of the key. CTA c owns the c-th slice of the items. In a pass it counts the
// digits of its slice, learns from the other CTAs' counts (shared memory of the
// cluster) where its items of each digit go, then ranks the slice tile by tile,
// puts the tile in order in shared memory and writes it out run by run (straight
// from the registers, 65536 tokens took 22 us: scattered stores from 8 SMs). A
// slice of one tile (up to 131072 tokens in all) is ranked and counted in one go.
// 65536 tokens: 10 us, 16 CTAs; 8 CTAs 13 us.
// Tokens outside the table are dropped in the first pass; as many keys at the
// end become `vocab`.
constexpr int kSortCtas = 16, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortItems = 8;
constexpr int kTile = kSortThreads * kSortItems, kDigits = 256;

struct SortShared {
    int warp[kSortWarps][kDigits];   // a tile's digits by warp, then how many are in the warps before
    int part[4][kDigits];
    int total[kDigits], first[kDigits];   // of the tile: items of a digit, where they begin in its order
    int count[kDigits];                   // of the slice; read by the cluster
    int next[kDigits];                    // where the slice's next item of a digit goes
    int scan[2][kDigits / 32];
    int key[kTile];                       // the tile in order
    uint16_t from[kTile];                 // place in the tile
};
static_assert(kTile <= 65536, "places are 16 bits");

// Lanes whose digit (0 .. 255, or 256) is this lane's: by votes (8192 items of a CTA 2.5 us; __match_any_sync 7.2).
__device__ __forceinline__ unsigned lanes_with(int digit) {
    const bool item = digit < kDigits;
    const unsigned items = __ballot_sync(kFull, item);
    unsigned same = item ? items : ~items;
#pragma unroll
    for (int bit = 0; bit < 8; ++bit) {
        const int set = digit >> bit & 1;
        same &= ~(__ballot_sync(kFull, set) ^ (unsigned)-set);
    }
    return same;
}
// Inclusive sum over a warp.
__device__ __forceinline__ int warp_scan(int v) {
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int up = __shfl_up_sync(kFull, v, o);
        if ((threadIdx.x & 31) >= o) v += up;
    }
    return v;
}

struct SortArgs {
    const void *tokens;
    int type, vocab, passes;
    int64_t n;
    int *keys[2], *perm[2];   // the sorted keys and positions end in [passes & 1]
    int *arrived;             // cleared, for the sums
    int64_t counters;
};

__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads, 1) sort_kernel(const SortArgs a) {
    extern __shared__ uint4 smem[];
    SortShared &sh = *reinterpret_cast<SortShared *>(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
    int64_t items = a.n;   // of the pass
    pdl_trigger();   // few CTAs: the sums' may set up meanwhile
    pdl_wait();
    for (int64_t i = (int64_t)cta * kSortThreads + tid; i < a.counters; i += kSortCtas * kSortThreads) a.arrived[i] = 0;
    for (int pass = 0; pass < a.passes; ++pass) {
        const int *keys = pass & 1 ? a.keys[1] : a.keys[0], *perm = pass & 1 ? a.perm[1] : a.perm[0];
        int *keys_out = pass & 1 ? a.keys[0] : a.keys[1], *perm_out = pass & 1 ? a.perm[0] : a.perm[1];
        const int shift = 8 * pass;
        const int64_t per = (items + kSortCtas - 1) / kSortCtas;
        const int64_t lo = min(per * cta, items), hi = min(lo + per, items);
        const bool one_tile = per <= kTile;
        const int each = one_tile ? (int)((per + kSortThreads - 1) / kSortThreads) : kSortItems;   // items of a thread

        int key[kSortItems], rank[kSortItems];   // -1: no item
        const auto place = [&](int j) { return (warp * each + j) * 32 + lane; };
        const auto load_all = [&](int64_t base, auto get) {   // the type is asked for once, so that the loads overlap
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                const int64_t i = base + place(j);
                key[j] = j < each && i < hi ? get(i) : -1;
            }
        };
        const auto load = [&](int64_t base) {
            const auto valid = [&](int64_t t) { return t >= 0 && t < a.vocab ? (int)t : -1; };
            if (pass > 0) load_all(base, [&](int64_t i) { return __ldcg(keys + i); });
            else if (a.type == MB_TOKEN_U8)
                load_all(base, [&](int64_t i) { return valid(static_cast<const uint8_t *>(a.tokens)[i]); });
            else if (a.type == MB_TOKEN_I32)
                load_all(base, [&](int64_t i) { return valid(static_cast<const int32_t *>(a.tokens)[i]); });
            else
                load_all(base, [&](int64_t i) { return valid(static_cast<const int64_t *>(a.tokens)[i]); });
        };
        const auto digit_of = [&](int k) { return k >= 0 ? k >> shift & 255 : kDigits; };
        // The loaded tile: rank[] within the digit and warp, sh.warp the digit's items in the warps before, sh.total.
        const auto rank_tile = [&]() {
            for (int d = tid; d < kSortWarps * kDigits / 4; d += kSortThreads)
                reinterpret_cast<int4 *>(sh.warp)[d] = make_int4(0, 0, 0, 0);
            unsigned same[kSortItems];
#pragma unroll
            for (int j = 0; j < kSortItems; ++j)
                if (j < each) same[j] = lanes_with(digit_of(key[j]));
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                if (j >= each) break;
                const int digit = digit_of(key[j]);
                const int before = __popc(same[j] & ((1u << lane) - 1));
                const int old = digit < kDigits ? sh.warp[warp][digit] : 0;
                __syncwarp();
                if (digit < kDigits && before == 0) sh.warp[warp][digit] = old + __popc(same[j]);
                __syncwarp();
                rank[j] = old + before;
            }
            __syncthreads();
            const int d = tid % kDigits, quarter = tid / kDigits;   // 8 warps' counts each
            int c[kSortWarps / 4], sum = 0;
#pragma unroll
            for (int w = 0; w < kSortWarps / 4; ++w) {
                c[w] = sh.warp[quarter * (kSortWarps / 4) + w][d];
                sum += c[w];
            }
            sh.part[quarter][d] = sum;
            __syncthreads();
            int at = 0;
            for (int q = 0; q < quarter; ++q) at += sh.part[q][d];
            if (quarter == 3) sh.total[d] = at + sum;
#pragma unroll
            for (int w = 0; w < kSortWarps / 4; ++w) {
                sh.warp[quarter * (kSortWarps / 4) + w][d] = at;
                at += c[w];
            }
            __syncthreads();
        };
        const auto scatter = [&](int64_t base) {
            int incl = 0;
            if (tid < kDigits) {
                incl = warp_scan(sh.total[tid]);
                if (lane == 31) sh.scan[1][warp] = incl;
            }
            __syncthreads();
            int many = 0;   // items of the tile
            for (int w = 0; w < kDigits / 32; ++w) {
                incl += w < warp ? sh.scan[1][w] : 0;
                many += sh.scan[1][w];
            }
            if (tid < kDigits) sh.first[tid] = incl - sh.total[tid];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                if (j >= each || key[j] < 0) continue;
                const int digit = digit_of(key[j]), to = sh.first[digit] + sh.warp[warp][digit] + rank[j];
                sh.key[to] = key[j];
                sh.from[to] = (uint16_t)place(j);
            }
            __syncthreads();
#pragma unroll 4
            for (int i = tid; i < many; i += kSortThreads) {
                const int k = sh.key[i], digit = digit_of(k), to = sh.next[digit] + i - sh.first[digit];
                const int64_t from = base + sh.from[i];
                keys_out[to] = k;
                perm_out[to] = pass > 0 ? __ldcg(perm + from) : (int)from;
            }
        };

        if (one_tile) {
            load(lo);
            rank_tile();
            if (tid < kDigits) sh.count[tid] = sh.total[tid];
        } else {
            if (tid < kDigits) sh.count[tid] = 0;
            __syncthreads();
            for (int64_t base = lo; base < hi; base += kTile) {
                load(base);
#pragma unroll
                for (int j = 0; j < kSortItems; ++j) {
                    const int digit = digit_of(key[j]);
                    const unsigned same = lanes_with(digit);
                    if (digit < kDigits && lane == __ffs(same) - 1) atomicAdd(&sh.count[digit], __popc(same));
                }
            }
        }
        cluster_arrive();
        cluster_wait();   // every CTA's counts are there
        if (tid < kDigits) {
            int before = 0, total = 0;   // of this digit: in the CTAs before, in all
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) {
                const int v = cluster_load(&sh.count[tid], c);
                before += c < cta ? v : 0;
                total += v;
            }
            const int incl = warp_scan(total);   // of the digits up to this one
            if (lane == 31) sh.scan[0][warp] = incl;
            sh.next[tid] = incl - total + before;
        }
        __syncthreads();
        const bool last = pass + 1 == a.passes;
        if (last) cluster_arrive();   // has read the others' counts
        int lower = 0, all = 0;
        for (int w = 0; w < kDigits / 32; ++w) {
            lower += w < warp ? sh.scan[0][w] : 0;
            all += sh.scan[0][w];
        }
        items = all;
        if (tid < kDigits) sh.next[tid] += lower;
        __syncthreads();
        if (one_tile) {
            scatter(lo);
        } else {
            for (int64_t base = lo; base < hi; base += kTile) {
                load(base);
                rank_tile();
                scatter(base);
                __syncthreads();
                if (tid < kDigits) sh.next[tid] += sh.total[tid];
                __syncthreads();
            }
        }
        if (!last) cluster_arrive();
        cluster_wait();   // the pass's output is visible to the cluster; after the last: nobody reads these counts any more
    }
    int *keys = a.passes & 1 ? a.keys[1] : a.keys[0];
    for (int64_t i = items + (int64_t)cta * kSortThreads + tid; i < a.n; i += kSortCtas * kSortThreads) keys[i] = a.vocab;
}

// ---- sums of the sorted rows
// A thread's rows come through a ring of asynchronous copies of its own, kSumStages stages of four rows. 65536 x 1024
// fp32 in all, pieces for so many CTAs of 256 threads per SM: with 3 stages 2 57.3 us, 3 60.4; with 2 stages 3 58.3, 4
// 59.3, 8 67.7; with 4 stages 2 58.0; 128 threads 59.8 to 61; eight rows at a time in registers 64.
constexpr int kSumThreads = 256, kSumCtas = 3, kSumStage = 4, kSumStages = 3;
constexpr int kPieceCtas = 2;   // per SM; the third's room is for CTAs that clear
constexpr int kMostTy = kSumThreads / 4, kMostRows = 1024, kLongest = 320;   // pieces, positions of a CTA; positions of a piece

struct SumArgs {
    const int *keys, *perm;   // sorted
    int64_t n, width, pieces;
    int vocab, accumulate, piece;
    int tx;                    // threads side by side in a row; kSumThreads / tx pieces per CTA
    int64_t sum_blocks;        // CTAs of the sums; the ones behind them clear rows
    float scale;
    float *dtable;
    float *part;    // [pieces][2][width]: of the run that enters a piece, of the one that leaves it
    int *arrived;   // [pieces][column tiles]: partial sums there of the run that begins in a piece; zeros
};

template <int V> __device__ __forceinline__ void put_row(const SumArgs &a, int key, int64_t c, const float (&acc)[V]) {
    float v[V];
    float *row = a.dtable + key * a.width + c;
    if (a.accumulate) {
        ldf(row, v);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = fmaf(acc[j], a.scale, v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = acc[j] * a.scale;
    }
    stf(row, v);
}

// The lanes of this warp for which f holds.
struct Votes {
    template <typename F> __device__ __forceinline__ unsigned operator()(const F &f) const {
        return __ballot_sync(kFull, f((int)(threadIdx.x & 31)));
    }
    template <typename F, typename G> __device__ __forceinline__ void operator()(const F &f, const G &g, unsigned &b, unsigned &c) const {
        const bool x = f((int)(threadIdx.x & 31)), y = g((int)(threadIdx.x & 31));
        b = __ballot_sync(kFull, x);
        c = __ballot_sync(kFull, y);
    }
};

// Clear the row of a token that does not occur (a warp).
__device__ __forceinline__ void clear_row(const SumArgs &a, int64_t v) {
    const int64_t at = first_at(Votes{}, 0, a.n, (int)v, [&](int64_t i) { return a.keys[i]; });
    if (at < a.n && a.keys[at] == v) return;
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t c = (threadIdx.x & 31) * 4; c < a.width; c += 128) stf(a.dtable + v * a.width + c, zero);
}

// CTA (kSumThreads / tx pieces, column tile): a 16-byte group of columns per thread. Whoever brings the last partial sum
// of a run that spans pieces adds them up, in the order of the pieces (a kernel of its own for that took 12 us).
// The CTAs behind clear the rows of tokens that do not occur, beside the sums: an SM stores 54 GB/s, so all of them are
// wanted (cleared beside the sort by 96 SMs, 32001 x 1792 took 45 us before the sums could begin).
template <typename T>
__global__ void __launch_bounds__(kSumThreads, kSumCtas) embed_sum_kernel(const T *dout, const SumArgs a) {
    constexpr int V = kVec<T>;
    extern __shared__ uint4 smem[];   // [kSumStages * kSumStage][kSumThreads]
    __shared__ int keys_of[kMostRows + 2 * kMostTy], perm_of[kMostRows];
    __shared__ int64_t begin_of[kMostTy], end_of[kMostTy];   // pieces where the run that enters begins, that leaves ends
    __shared__ int joins[kMostTy];                           // bit 0, 1: this CTA joins the one that enters, leaves
    pdl_wait();
    if (blockIdx.x >= a.sum_blocks) {
        const int64_t v = ((int64_t)blockIdx.x - a.sum_blocks) * (kSumThreads / 32) + threadIdx.x / 32;
        if (v < a.vocab && blockIdx.y == 0) clear_row(a, v);
        return;
    }
    const int ty = kSumThreads / a.tx, x = threadIdx.x % a.tx, y = threadIdx.x / a.tx;
    const int64_t piece0 = blockIdx.x * (int64_t)ty, piece = piece0 + y, p0 = piece * a.piece;
    const int64_t c = ((int64_t)blockIdx.y * a.tx + x) * V;
    const int count = (int)max((int64_t)0, min((int64_t)a.piece, a.n - p0));
    int *keys = keys_of + y * (a.piece + 2), *perm = perm_of + y * a.piece;
    const auto key_at = [&](int64_t i) { return i >= 0 && i < a.n ? a.keys[i] : -1; };
    for (int i = x; i < count + 2; i += a.tx) keys[i] = key_at(p0 + i - 1);   // and the neighbours' keys
    for (int i = x; i < count; i += a.tx) perm[i] = a.perm[p0 + i];
    __syncthreads();
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    const bool active = c < a.width;
    int m = active ? count : 0;   // tokens outside the table sort last: without them
    if (m > 0 && keys[m] >= a.vocab) {
        int lo = 0;   // the first of them lies in [lo, m]
        while (lo < m) {
            const int mid = (lo + m) / 2;
            if (keys[mid + 1] < a.vocab) lo = mid + 1;
            else m = mid;
        }
    }
    uint4 *mine = smem + threadIdx.x;
    const T *column = dout + c;
    int slot = 0;
    const auto issue = [&](int r) {
#pragma unroll
        for (int j = 0; j < kSumStage; ++j)
            if (r + j < m) copy16(mine + (slot + j) * kSumThreads, column + perm[r + j] * a.width);
        copy_commit();
        slot = (slot + kSumStage) % (kSumStages * kSumStage);
    };
#pragma unroll
    for (int k = 0; k < kSumStages - 1; ++k) issue(k * kSumStage);
    const int lane = threadIdx.x & 31;
    // while the first rows are on their way, a warp per piece finds where the runs at its ends lie
    for (int g = threadIdx.x / 32; g < ty; g += kSumThreads / 32) {
        const RunEnds r = run_ends(Votes{}, [&](int64_t i) { return a.keys[i]; }, a.n, a.piece, a.pieces, piece0 + g);
        if (lane == 0) {
            begin_of[g] = r.begin;
            end_of[g] = r.end;
        }
    }
    bool whole = keys[1] != keys[0];   // the run began here
    for (int r = 0; r < m; r += kSumStage) {
        issue(r + (kSumStages - 1) * kSumStage);   // into the slots read in the round before
        copy_wait<kSumStages - 1>();
#pragma unroll
        for (int j = 0; j < kSumStage; ++j) {
            if (r + j >= m) break;
            const int i = r + j, key = keys[i + 1];
            float v[V];
            widen(mine[(slot + j) * kSumThreads], v);
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += v[e];
            const bool ends = keys[i + 2] != key;
            if (ends || i + 1 == count) {
                if (whole && ends) put_row(a, key, c, acc);
                else stf(a.part + (piece * 2 + (whole ? 1 : 0)) * a.width + c, acc);
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = 0.f;
                whole = true;
            }
        }
    }
    // the runs that enter (from begin_of) and that leave (to end_of); one that does both is counted as entering
    const int first = keys[1], last = keys[count];   // of an empty piece: -1
    const bool enters = count > 0 && first < a.vocab && keys[0] == first;
    const bool through = enters && first == last;
    const bool leaves = count > 0 && last < a.vocab && keys[count + 1] == last && !through;
    __threadfence();   // the partial sums, before their counts
    __syncthreads();
    if (x == 0) {
        int join = 0;
        const int64_t tiles = gridDim.y, tile = blockIdx.y;
        if (enters) {
            const int64_t begin = begin_of[y], end = through ? end_of[y] : piece;
            if (atomicAdd(a.arrived + begin * tiles + tile, 1) == (int)(end - begin)) join |= 1;
        }
        if (leaves && atomicAdd(a.arrived + piece * tiles + tile, 1) == (int)(end_of[y] - piece)) join |= 2;
        joins[y] = join;
        __threadfence();   // the counts, before the others' partial sums
    }
    __syncthreads();
    for (int side = 0; side < 2; ++side) {
        if (!active || !(joins[y] >> side & 1)) continue;
        const int64_t begin = side == 0 ? begin_of[y] : piece, end = side == 0 && !through ? piece : end_of[y];
        const auto add = [&](const float *p) {
            float v[V];
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const float4 q = __ldcg(reinterpret_cast<const float4 *>(p + j));   // other SMs wrote them
                v[j] = q.x; v[j + 1] = q.y; v[j + 2] = q.z; v[j + 3] = q.w;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += v[j];
        };
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
        add(a.part + (begin * 2 + 1) * a.width + c);
#pragma unroll(64 / V)
        for (int64_t q = begin + 1; q <= end; ++q) add(a.part + q * 2 * a.width + c);
        put_row(a, side == 0 ? first : last, c, acc);
    }
}

int threads_for(int64_t groups, int most) {   // a power of two, at least 4
    int tx = 4;
    while (tx < most && tx < groups) tx *= 2;
    return tx;
}

template <typename T, typename O>
cudaError_t lookup(const LookupArgs &a, const void *table, void *out, cudaStream_t s) {
    const int64_t rows = (int64_t)kThreads / a.tx * kRows;
    const dim3 grid((unsigned)((a.n + rows - 1) / rows), (unsigned)((a.width / 4 + a.tx - 1) / a.tx));
    return launch_pdl(true, embed_kernel<T, O>, grid, dim3(kThreads), 0, s, static_cast<const T *>(table),
                      static_cast<O *>(out), a);
}

int64_t round256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// How the sums are cut: into equal pieces for kPieceCtas CTAs per SM, of 16 positions at least (few tokens: more CTAs) and
// kLongest at most; no more than kMostRows positions in a CTA.
struct Pieces {
    int piece, tx;
    int64_t pieces, tiles;
};
Pieces cut_rows(int64_t n, int64_t width, int vec) {
    Pieces c{};
    c.tx = threads_for(width / vec, kSumThreads);
    c.tiles = (width / vec + c.tx - 1) / c.tx;
    const int64_t ty = kSumThreads / c.tx, slots = std::max<int64_t>(kSms * kPieceCtas / c.tiles, 1) * ty;
    const int64_t piece = (n + slots - 1) / slots;
    c.piece = (int)std::min<int64_t>(std::max<int64_t>(piece, 16), std::min<int64_t>(kLongest, kMostRows / ty));
    c.pieces = (n + c.piece - 1) / c.piece;
    return c;
}

// Scratch: keys and positions twice, arrived, part (room for either type, which are cut differently).
struct Scratch {
    int64_t each, arrived, part;   // bytes
};
Scratch scratch_for(int64_t n, int64_t width) {
    const Pieces f = cut_rows(n, width, kVec<float>), h = cut_rows(n, width, kVec<__nv_bfloat16>);
    return Scratch{round256(n * 4), round256(std::max(f.pieces * f.tiles, h.pieces * h.tiles) * 4),
                   std::max(f.pieces, h.pieces) * 2 * width * 4};
}

}  // namespace

cudaError_t launch_embed(const void *tokens, int type, const void *table, bool table_bf16, float scale, void *out,
                         bool out_bf16, int64_t n, int vocab, int64_t width, cudaStream_t s) {
    using B = __nv_bfloat16;
    const LookupArgs a{tokens, type, vocab, threads_for(width / 4, kThreads), scale, n, width};
    const auto f = table_bf16 ? (out_bf16 ? lookup<B, B> : lookup<B, float>)
                              : (out_bf16 ? lookup<float, B> : lookup<float, float>);
    return f(a, table, out, s);
}

size_t embed_backward_scratch(int64_t n, int64_t width) {
    const Scratch s = scratch_for(n, width);
    return (size_t)(4 * s.each + s.arrived + s.part);
}

cudaError_t launch_embed_backward(const void *tokens, int type, const void *dout, bool bf16, float scale, bool accumulate,
                                  float *dtable, int64_t n, int vocab, int64_t width, void *scratch, cudaStream_t s) {
    char *base = static_cast<char *>(scratch);
    const Scratch room = scratch_for(n, width);
    const Pieces cut = cut_rows(n, width, bf16 ? kVec<__nv_bfloat16> : kVec<float>);
    SortArgs so{};
    so.tokens = tokens; so.type = type; so.vocab = vocab; so.n = n;
    for (int i = 0; i < 2; ++i) {
        so.keys[i] = reinterpret_cast<int *>(base + i * room.each);
        so.perm[i] = reinterpret_cast<int *>(base + (2 + i) * room.each);
    }
    so.passes = 1;
    while (so.passes < 4 && (int64_t)(vocab - 1) >> (8 * so.passes)) ++so.passes;
    so.arrived = reinterpret_cast<int *>(base + 4 * room.each);
    so.counters = cut.pieces * cut.tiles;
    if (n > 0) {
        cudaError_t e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared));
        if (e == cudaSuccess) e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e == cudaSuccess)
            e = launch_pdl(true, sort_kernel, dim3(kSortCtas), dim3(kSortThreads), sizeof(SortShared), s, so);
        if (e != cudaSuccess) return e;
    }
    SumArgs a{};
    a.keys = so.keys[so.passes & 1]; a.perm = so.perm[so.passes & 1];
    a.n = n; a.width = width; a.piece = cut.piece; a.pieces = cut.pieces; a.tx = cut.tx;
    a.vocab = vocab; a.accumulate = accumulate; a.scale = scale;
    a.dtable = dtable;
    a.part = reinterpret_cast<float *>(base + 4 * room.each + room.arrived);
    a.arrived = so.arrived;
    a.sum_blocks = (a.pieces * a.tx + kSumThreads - 1) / kSumThreads;
    const int64_t clear_blocks = accumulate ? 0 : ((int64_t)vocab + kSumThreads / 32 - 1) / (kSumThreads / 32);
    const dim3 grid((unsigned)(a.sum_blocks + clear_blocks), (unsigned)cut.tiles);
    if (grid.x == 0) return cudaSuccess;   // no tokens, nothing to clear
    const auto sum = [&](auto kernel, auto *rows) {
        constexpr size_t smem = (size_t)kSumStages * kSumStage * kSumThreads * 16;
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        return e != cudaSuccess ? e : launch_pdl(true, kernel, grid, dim3(kSumThreads), smem, s, rows, a);
    };
    return bf16 ? sum(embed_sum_kernel<__nv_bfloat16>, static_cast<const __nv_bfloat16 *>(dout))
                : sum(embed_sum_kernel<float>, static_cast<const float *>(dout));
}

}  // namespace mbscan
