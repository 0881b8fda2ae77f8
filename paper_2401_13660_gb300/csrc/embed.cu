// Embedding lookup with scaling, and the table's gradient by sorted tokens.
//
//   out[i] = scale * table[tokens[i]]                      (zeros where the token is outside the table)
//   dtable[v] (+)= scale * sum_{i: tokens[i] = v} dout[i]
//
// The gradient first sorts the token positions by token (stable, so that every
// sum has one order), then adds the rows of dout in that order: runs of equal
// tokens are cut into pieces of kPiece positions, a run inside one piece is
// written at once, one that spans pieces leaves a partial sum in each, which a
// last kernel adds up. No atomics: the result depends on the inputs alone.
#include <algorithm>

#include "tokens.cuh"
#include "vec.cuh"

namespace mbscan {
namespace {

constexpr int kThreads = 256;

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

// One thread per four elements of out.
template <typename T, typename O>
__global__ void __launch_bounds__(kThreads) embed_kernel(const void *tokens, int type, const T *table, float scale, O *out,
                                                         int64_t n, int vocab, int64_t width) {
    pdl_wait();
    const int64_t groups = width / 4;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n * groups; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / groups, c = (i - row * groups) * 4;
        const int tok = load_token(tokens, type, row, vocab);
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (tok >= 0) {
            ld4(table + tok * width + c, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= scale;
        }
        st4(out + row * width + c, v);
    }
}

// ---- sort: one cluster of kSortCtas CTAs, a stable counting sort per 8 bits
// of the key. CTA c owns the c-th slice of the items. A pass counts the slice's
// digits, learns from the other CTAs' counts (shared memory of the cluster)
// where its items of each digit begin, then ranks the slice tile by tile.
// Tokens outside the table are dropped in the first pass; as many keys at the
// end become `vocab`.
constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortItems = 4;
constexpr int kTile = kSortThreads * kSortItems, kDigits = 256;

struct SortShared {
    int count[kDigits];               // this CTA's digits in the pass; read by the cluster
    int next[kDigits];                // where its next item of a digit goes
    int warp[kSortWarps][kDigits];    // a tile's digits by warp, then where each warp's begin
    int scan[kDigits / 32];
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_load(const int *p, int cta) {   // *p of that CTA's shared memory
    uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(cta));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(r) : "memory");
    return v;
}

struct SortArgs {
    const void *tokens;
    int type, vocab, passes;
    int64_t n;
    int *keys[2], *perm[2];   // the sorted keys and positions end in [passes & 1]
};

__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads) sort_kernel(const SortArgs a) {
    __shared__ SortShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
    int64_t items = a.n;   // of the pass
    pdl_wait();
    for (int pass = 0; pass < a.passes; ++pass) {
        const int64_t per = (items + kSortCtas - 1) / kSortCtas;
        const int64_t lo = min(per * cta, items), hi = min(lo + per, items);
        const int *keys = a.keys[pass & 1], *perm = a.perm[pass & 1];
        int *keys_out = a.keys[~pass & 1], *perm_out = a.perm[~pass & 1];
        const int shift = 8 * pass;
        auto key_at = [&](int64_t i) {   // -1: none
            if (i >= hi) return -1;
            return pass > 0 ? __ldcg(keys + i) : load_token(a.tokens, a.type, i, a.vocab);
        };
        if (tid < kDigits) sh.count[tid] = 0;
        __syncthreads();
        for (int64_t base = lo; base < hi; base += kSortThreads) {
            const int key = key_at(base + tid), digit = key >= 0 ? key >> shift & 255 : kDigits;
            const unsigned same = __match_any_sync(kFull, digit);
            if (digit < kDigits && lane == __ffs(same) - 1) atomicAdd(&sh.count[digit], __popc(same));
        }
        cluster_sync();   // every CTA's counts are there (and its output of the pass before)
        if (tid < kDigits) {
            int before = 0, total = 0;   // of this digit: in the CTAs before, in all
            for (int c = 0; c < kSortCtas; ++c) {
                const int v = cluster_load(&sh.count[tid], c);
                if (c < cta) before += v;
                total += v;
            }
            int incl = total;   // of the digits up to this one
            for (int o = 1; o < 32; o *= 2) {
                const int up = __shfl_up_sync(kFull, incl, o);
                if (lane >= o) incl += up;
            }
            if (lane == 31) sh.scan[warp] = incl;
            sh.next[tid] = incl - total + before;
        }
        cluster_sync();   // nobody reads these counts any more
        if (tid < kDigits) {
            int lower = 0;
            for (int w = 0; w < warp; ++w) lower += sh.scan[w];
            sh.next[tid] += lower;
        }
        items = 0;
        for (int w = 0; w < kDigits / 32; ++w) items += sh.scan[w];
        for (int64_t base = lo; base < hi; base += kTile) {
            for (int d = tid; d < kSortWarps * kDigits; d += kSortThreads) (&sh.warp[0][0])[d] = 0;
            __syncthreads();
            int key[kSortItems], rank[kSortItems];
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) key[j] = key_at(base + (warp * kSortItems + j) * 32 + lane);
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                const int digit = key[j] >= 0 ? key[j] >> shift & 255 : kDigits;
                const unsigned same = __match_any_sync(kFull, digit);
                const int leader = __ffs(same) - 1;
                int old = 0;
                if (digit < kDigits && lane == leader) {
                    old = sh.warp[warp][digit];
                    sh.warp[warp][digit] = old + __popc(same);
                }
                __syncwarp();
                rank[j] = __shfl_sync(kFull, old, leader) + __popc(same & ((1u << lane) - 1));
            }
            __syncthreads();
            if (tid < kDigits) {
                int at = sh.next[tid];
                for (int w = 0; w < kSortWarps; ++w) {
                    const int c = sh.warp[w][tid];
                    sh.warp[w][tid] = at;
                    at += c;
                }
                sh.next[tid] = at;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                if (key[j] < 0) continue;
                const int64_t i = base + (warp * kSortItems + j) * 32 + lane;
                const int to = sh.warp[warp][key[j] >> shift & 255] + rank[j];
                keys_out[to] = key[j];
                perm_out[to] = pass > 0 ? __ldcg(perm + i) : (int)i;
            }
            __syncthreads();
        }
        cluster_sync();   // the pass's output is visible to the cluster
    }
    int *keys = a.keys[a.passes & 1];
    for (int64_t i = items + (int64_t)cta * kSortThreads + tid; i < a.n; i += kSortCtas * kSortThreads) keys[i] = a.vocab;
}

// ---- sums of the sorted rows
constexpr int kPiece = 64, kSumThreads = 128;

struct SumArgs {
    const int *keys, *perm;   // sorted
    int64_t n, width, pieces;
    int vocab, accumulate;
    float scale;
    float *dtable;
    float *part;   // [pieces][2][width]: of the run that enters a piece, of the one that leaves it
};

__device__ __forceinline__ void put_row(const SumArgs &a, int key, int64_t c, const float (&acc)[4]) {
    float v[4] = {acc[0] * a.scale, acc[1] * a.scale, acc[2] * a.scale, acc[3] * a.scale};
    float *row = a.dtable + key * a.width + c;
    if (a.accumulate) {
        float old[4];
        ldf(row, old);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += old[j];
    }
    stf(row, v);
}

// CTA (piece, column tile): four columns per thread.
template <typename T>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const T *dout, const SumArgs a) {
    __shared__ int keys[kPiece + 2], perm[kPiece];
    pdl_wait();
    const int64_t p0 = blockIdx.x * (int64_t)kPiece;
    const int64_t c = ((int64_t)blockIdx.y * kSumThreads + threadIdx.x) * 4;
    const int count = (int)min((int64_t)kPiece, a.n - p0);
    for (int i = threadIdx.x; i < count + 2; i += kSumThreads) {   // and the neighbours' keys, -1 where there is none
        const int64_t at = p0 + i - 1;
        keys[i] = at >= 0 && at < a.n ? a.keys[at] : -1;
    }
    for (int i = threadIdx.x; i < count; i += kSumThreads) perm[i] = a.perm[p0 + i];
    __syncthreads();
    if (c >= a.width) return;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    bool whole = keys[1] != keys[0];   // the run began here
    for (int i = 0; i < count; ++i) {
        const int key = keys[i + 1];
        if (key >= a.vocab) break;   // tokens outside the table, sorted last
        float v[4];
        ld4(dout + perm[i] * a.width + c, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += v[j];
        const bool last = i + 1 == count;
        if (last || keys[i + 2] != key) {
            const bool ends = keys[i + 2] != key;
            if (whole && ends) put_row(a, key, c, acc);
            else stf(a.part + (blockIdx.x * 2 + (whole ? 1 : 0)) * a.width + c, acc);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = 0.f;
            whole = true;
        }
    }
}

// Rows of tokens that do not occur: zeros (one warp a row).
__global__ void __launch_bounds__(kThreads) embed_zero_kernel(const SumArgs a) {
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t v = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (v >= a.vocab) return;
    int64_t lo = 0, hi = a.n;   // the first position whose key is >= v lies in [lo, hi]
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32, at = lo + step * lane;
        const unsigned below = __ballot_sync(kFull, at < hi && a.keys[at] < v);
        const int k = __popc(below);   // the lanes below form a prefix
        if (k == 0) break;             // keys[lo] >= v
        const int64_t new_lo = lo + step * (k - 1) + 1;
        hi = min(hi, lo + step * k);
        lo = new_lo;
    }
    if (lo < a.n && a.keys[lo] == v) return;
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t c = lane * 4; c < a.width; c += 128) stf(a.dtable + v * a.width + c, zero);
}

// Runs over several pieces: CTA (piece where the run begins, column tile) adds their partial sums in order.
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(const SumArgs a) {
    pdl_wait();
    const int64_t p0 = blockIdx.x * (int64_t)kPiece, p1 = p0 + kPiece;
    if (p1 >= a.n) return;
    const int key = a.keys[p1 - 1];
    if (key >= a.vocab || a.keys[p1] != key) return;                 // no run leaves the piece
    if (a.keys[p0] == key && p0 > 0 && a.keys[p0 - 1] == key) return;   // it began before
    const int64_t c = ((int64_t)blockIdx.y * kSumThreads + threadIdx.x) * 4;
    if (c >= a.width) return;
    float acc[4];
    ldf(a.part + (blockIdx.x * 2 + 1) * a.width + c, acc);
    for (int64_t q = blockIdx.x + 1; q < a.pieces && a.keys[q * kPiece] == key; ++q) {
        float v[4];
        ldf(a.part + q * 2 * a.width + c, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += v[j];
    }
    put_row(a, key, c, acc);
}

template <typename T, typename O>
cudaError_t lookup(const void *tokens, int type, const void *table, float scale, void *out, int64_t n, int vocab,
                   int64_t width, cudaStream_t s) {
    const int64_t blocks = (n * (width / 4) + kThreads - 1) / kThreads;
    return launch_pdl(true, embed_kernel<T, O>, dim3((unsigned)std::min<int64_t>(blocks, 152 * 64)), dim3(kThreads), 0, s,
                      tokens, type, static_cast<const T *>(table), scale, static_cast<O *>(out), n, vocab, width);
}

int64_t round256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

cudaError_t launch_embed(const void *tokens, int type, const void *table, bool table_bf16, float scale, void *out,
                         bool out_bf16, int64_t n, int vocab, int64_t width, cudaStream_t s) {
    using B = __nv_bfloat16;
    const auto f = table_bf16 ? (out_bf16 ? lookup<B, B> : lookup<B, float>)
                              : (out_bf16 ? lookup<float, B> : lookup<float, float>);
    return f(tokens, type, table, scale, out, n, vocab, width, s);
}

size_t embed_backward_scratch(int64_t n, int64_t width) {
    const int64_t pieces = (n + kPiece - 1) / kPiece;
    return (size_t)(4 * round256(n * 4) + pieces * 2 * width * 4);
}

cudaError_t launch_embed_backward(const void *tokens, int type, const void *dout, bool bf16, float scale, bool accumulate,
                                  float *dtable, int64_t n, int vocab, int64_t width, void *scratch, cudaStream_t s) {
    char *base = static_cast<char *>(scratch);
    const int64_t each = round256(n * 4);
    SortArgs so{};
    so.tokens = tokens; so.type = type; so.vocab = vocab; so.n = n;
    for (int i = 0; i < 2; ++i) {
        so.keys[i] = reinterpret_cast<int *>(base + i * each);
        so.perm[i] = reinterpret_cast<int *>(base + (2 + i) * each);
    }
    so.passes = 1;
    while (so.passes < 4 && (int64_t)(vocab - 1) >> (8 * so.passes)) ++so.passes;
    SumArgs a{};
    a.keys = so.keys[so.passes & 1]; a.perm = so.perm[so.passes & 1];
    a.n = n; a.width = width; a.pieces = (n + kPiece - 1) / kPiece;
    a.vocab = vocab; a.accumulate = accumulate; a.scale = scale;
    a.dtable = dtable;
    a.part = reinterpret_cast<float *>(base + 4 * each);
    cudaError_t e = cudaSuccess;
    const dim3 grid((unsigned)a.pieces, (unsigned)((width / 4 + kSumThreads - 1) / kSumThreads));
    if (n > 0) {
        e = launch_pdl(true, sort_kernel, dim3(kSortCtas), dim3(kSortThreads), 0, s, so);
        if (e != cudaSuccess) return e;
    }
    if (!accumulate) {
        e = launch_pdl(true, embed_zero_kernel, dim3((unsigned)((vocab + kThreads / 32 - 1) / (kThreads / 32))),
                       dim3(kThreads), 0, s, a);
        if (e != cudaSuccess) return e;
    }
    if (n == 0) return e;
    if (bf16)
        e = launch_pdl(true, embed_sum_kernel<__nv_bfloat16>, grid, dim3(kSumThreads), 0, s,
                       static_cast<const __nv_bfloat16 *>(dout), a);
    else
        e = launch_pdl(true, embed_sum_kernel<float>, grid, dim3(kSumThreads), 0, s, static_cast<const float *>(dout), a);
    if (e != cudaSuccess || a.pieces < 2) return e;
    return launch_pdl(true, embed_join_kernel, grid, dim3(kSumThreads), 0, s, a);
}

}  // namespace mbscan
