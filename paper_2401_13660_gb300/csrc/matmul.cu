// Product of 8-bit matrices with block scales (quant.cu) on the fifth-generation tensor cores:
//   out[m, n] = sum_b 2^(sa[m, b] + sw[n / 128, b] - 254) sum_{k in block b} a[m, k] w[n, k]
// The scales are powers of two, so the tensor core applies them to its own products (block-scaled tcgen05.mma; its scale
// granularity is 32 columns, a block of 128 is four instructions with the same scale), and the sum over all blocks stays in
// fp32 in tensor memory: no pass over partial sums.
//
// The weights are the instruction's A operand (128 output features in the 128 lanes), the rows of a its B operand (16 to
// 224 of them, the columns of the sum in tensor memory): one row costs an eighth of a tile then, not 127 idle lanes, and a
// decode step streams each weight through one tile.
//
// Twelve warps: one issues the TMA copies of both operands into a ring of stages (128 to 512 columns of the sum each,
// 128-byte swizzle), one the products, two lay out scales for the tensor core (512 columns' worth at a time: the four scales of a
// word go to one column of tensor memory), and eight move finished sums to global memory while the next tile's products run
// into the other half of tensor memory. CTAs take tiles in turn. Where tiles are few, a cluster of CTAs shares each tile's
// sum, every one over part of it; each gets the others' parts of its share of the rows into its shared memory and adds them up
// in the order of the ranks, so that a result is the same in every run.
#include "../../include/mbscan.h"
#include "cluster.cuh"
#include "common.cuh"
#include "matmul_plan.h"
#include "umma.cuh"

#include <atomic>

namespace mbscan {
namespace {

constexpr int kThreads = 128 + 128 * kGroups;

// Column and row of a tile.
struct Place {
    int feature, row;
};
__device__ __forceinline__ Place place_of(const Tiles &t, int tile) {
    if (t.band == 1) return {tile % t.features, tile / t.features};
    const int many = t.band * t.features, b = tile / many, in = tile - b * many;
    const int height = min(t.band, t.rows - b * t.band);
    return {in / height, b * t.band + in % height};
}

struct Args {
    CUtensorMap a, w, out;
    MatmulParams p;
    Tiles t;
    int stride;               // bytes between rows of scales
};

struct Barriers {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t scales_full[kSlots], scales_empty[kSlots];
    uint64_t sum_full[2], sum_empty[2];
    uint64_t drained;   // of a CTA whose waits gave up: the products it had issued
    uint32_t tmem;
};

// A place in a ring of `size`, and how often it has been round.
struct Ring {
    int at = 0;
    uint32_t round = 0;
    __device__ __forceinline__ void next(int size) {
        if (++at == size) {
            at = 0;
            round ^= 1;
        }
    }
};

template <typename T> __device__ __forceinline__ T *out_at(const MatmulParams &p, int64_t row, int64_t n) {
    const int64_t part = n / p.part;
    return static_cast<T *>(p.out) + (part * p.rows + row) * p.part + (n - part * p.part);
}

// Four lanes' four words turned: word j of lane i is lane j's word i.
__device__ __forceinline__ void transpose4(uint32_t *v, int lane) {
#pragma unroll
    for (int d = 1; d <= 2; d *= 2) {
        const bool odd = lane & d;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j & d) continue;
            const uint32_t got = __shfl_xor_sync(~0u, odd ? v[j] : v[j + d], d);
            v[j] = odd ? got : v[j];
            v[j + d] = odd ? v[j + d] : got;
        }
    }
}
__device__ __forceinline__ uint32_t bf16_pair(uint32_t lo, uint32_t hi) {   // of the bits of two floats
    const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ void store4(float *p, const float4 &v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, const float4 &v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const unsigned *>(&a), *reinterpret_cast<const unsigned *>(&b));
}

// Among the four warps of a group that moves sums (after mbar_wait_group: all of them are there, or none).
__device__ __forceinline__ void group_sync(int group) { asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory"); }

// kCtas: 1, or 2: a pair of CTAs shares a tile of 256 features, each with its 128 features and half of the rows.
template <typename T, int kCtas>
__global__ void __launch_bounds__(kThreads, 2) matmul_q8_kernel(const __grid_constant__ Args g) {
    extern __shared__ unsigned char dyn[];
    __shared__ Barriers bar;
    unsigned char *const smem = dyn + ((1024u - (smem_u32(dyn) & 1023u)) & 1023u);
    const Tiles t = g.t;   // in registers: a wait would have them read again
    constexpr int kWide = kCtas * kFeatures;
    const int mine = t.height / kCtas;   // rows that this CTA loads
    const int deep = kCtas == 2 ? 1 : t.deep;
    const uint32_t unit_bytes = (uint32_t)(kFeatures + mine) * kK, stage_bytes = deep * unit_bytes;
    unsigned char *const scales = smem + t.ring;
    // 1024-byte aligned (swizzled); of a CTA's only tile, where the ring was
    T *const chunks = reinterpret_cast<T *>(t.sums == 1 ? smem : scales + kSlots * kSlotBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int half = kCtas == 2 ? (int)(blockIdx.x & 1u) : 0;
    const int rank = kCtas == 2 ? 0 : (int)(blockIdx.x % (unsigned)t.split);
    const int team = kCtas == 2 ? 2 : t.split;
    const int first = (int)(blockIdx.x / (unsigned)team), step = (int)(gridDim.x / (unsigned)team), tiles = t.features * t.rows;
    // this CTA's blocks of the sum: whole stages but for the last
    const int units = (t.blocks + deep - 1) / deep;
    const int k0 = units * rank / t.split * deep, k1 = min(t.blocks, units * (rank + 1) / t.split * deep);
    // a barrier of the CTA that issues the products
    const auto lead = [&](uint64_t *b) { return cluster_address(b, 0); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < t.stages; ++i) {
            mbar_init(&bar.full[i], 1);
            mbar_init(&bar.empty[i], 1);
        }
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(&bar.scales_full[i], kCtas);
            mbar_init(&bar.scales_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bar.sum_full[i], 1);
            mbar_init(&bar.sum_empty[i], 4 * kGroups * kCtas);
        }
        mbar_init(&bar.drained, 1);
        fence_mbar_init();
        for (const CUtensorMap *m : {&g.a, &g.w, &g.out}) tma_prefetch_map(m);
    }
    if (warp == 0) tmem_alloc<kCtas>(&bar.tmem, t.columns);
    tmem_fence_before();
    __syncthreads();
    if (kCtas == 2) {   // the other's barriers are there
        cluster_arrive();
        cluster_wait();
    }
    tmem_fence_after();
    const uint32_t tmem = bar.tmem, tmem_scales = tmem + t.sums * t.height;
    pdl_wait();

    bool ok = true;
    if (warp == 0) {
        Ring r;
        int issued = 0;
        for (int tile = first; tile < tiles && ok; tile += step) {
            const Place at_tile = place_of(t, tile);
            const int n0 = at_tile.feature * kWide + half * kFeatures, m0 = at_tile.row * t.height + half * mine;
            for (int k = k0; k < k1; k += deep, ++issued, r.next(t.stages)) {
                uint64_t *const full = &bar.full[r.at];
                if (!(ok = __all_sync(kFull, mbar_wait(&bar.empty[r.at], r.round ^ 1)))) break;
                unsigned char *at = smem + (uint32_t)r.at * stage_bytes;
                const int end = min(k1, k + deep);
                if (elect_one()) {
                    if (half == 0) mbar_arrive_expect_tx(full, (uint32_t)(end - k) * kCtas * unit_bytes);
                    const uint32_t to = kCtas == 2 ? lead(full) : 0u;
#pragma unroll 1
                    for (int u = k; u < end; ++u, at += unit_bytes)
                        if (kCtas == 1) {
                            tma_load_2d(at, &g.w, full, u * kK, n0);
                            tma_load_2d(at + kFeatures * kK, &g.a, full, u * kK, m0);
                        } else {
                            tma_load_2d_pair(at, &g.w, to, u * kK, n0);
                            tma_load_2d_pair(at + kFeatures * kK, &g.a, to, u * kK, m0);
                        }
                }
            }
        }
        // a failed CTA must not end with copies in flight (those of a pair arrive at the first of them)
        for (int i = issued > t.stages ? issued - t.stages : 0; !ok && half == 0 && i < issued; ++i)
            if (!mbar_wait(&bar.full[i % t.stages], i / t.stages & 1)) break;
    } else if (warp == 1 && half == 0) {
        const auto wait = [](uint64_t *b, uint32_t parity) {
            return (bool)__all_sync(kFull, kCtas == 1 ? mbar_wait(b, parity) : mbar_wait_cluster(b, parity));
        };
        const uint64_t desc = umma_desc_128(smem_u32(smem)), desc_scales = umma_desc_rows16(smem_u32(scales));
        const uint32_t word0 = umma_word_q8(kWide, t.height, 0);
        Ring r, slot, sums;   // stages; slots of scales; the two sums
        uint32_t set = 0;
        for (int tile = first; tile < tiles && ok; tile += step, sums.next(t.sums)) {
            const uint32_t sum = tmem + sums.at * t.height;
            if (!(ok = wait(&bar.sum_empty[sums.at], sums.round ^ 1))) break;
            tmem_fence_after();
            for (int k = k0; k < k1; k += deep, r.next(t.stages)) {
                const uint32_t tmem_w = tmem_scales + set * kScaleColumns, tmem_a = tmem_w + 4;
                // a stage's blocks are of one word of scales; whether it begins, or ends, with this slot
                const int end = min(k1, k + deep);
                const bool begins = k == k0 || k % 4 == 0, ends = end == k1 || end % 4 == 0;
                if (begins && !(ok = wait(&bar.scales_full[slot.at], slot.round))) break;
                if (!(ok = __all_sync(kFull, mbar_wait(&bar.full[r.at], r.round)))) break;
                tmem_fence_after();
                uint64_t dw = desc + (uint32_t)r.at * (stage_bytes >> 4);
                const uint64_t ds = desc_scales + (uint32_t)slot.at * (kSlotBytes >> 4);
                if (elect_one()) {
                    if (begins) {
                        tmem_copy_scales<kCtas>(tmem_w, ds);
                        tmem_copy_scales<kCtas>(tmem_a, ds + (512 >> 4));
                        if (t.height > 128) tmem_copy_scales<kCtas>(tmem_a + 4, ds + (1024 >> 4));
                    }
#pragma unroll 1
                    for (int u = k; u < end; ++u, dw += unit_bytes >> 4) {
                        const uint64_t da = dw + (kFeatures * kK >> 4);
                        const uint32_t word = word0 | (uint32_t)(u & 3) << 4 | (uint32_t)(u & 3) << 29;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            umma_q8<kCtas>(sum, dw + 2 * j, da + 2 * j, word, tmem_w, tmem_a, u > k0 || j > 0);
                    }
                    umma_commit<kCtas>(&bar.empty[r.at]);
                    if (ends) umma_commit<kCtas>(&bar.scales_empty[slot.at]);
                    if (end == k1) umma_commit<kCtas>(&bar.sum_full[sums.at]);
                }
                if (ends) {
                    slot.next(kSlots);
                    set ^= 1;
                }
            }
        }
        if (!ok) {   // tensor memory and the ring stay until what was issued is done
            if (elect_one()) umma_commit<kCtas>(&bar.drained);
            wait(&bar.drained, 0);
        }
    } else if (warp == 2 || warp == 3) {   // words in turn
        int group = 0;
        const int blocks = (int)((g.p.n_out + kFeatures - 1) / kFeatures);
        for (int tile = first; tile < tiles && ok; tile += step) {
            const Place at_tile = place_of(t, tile);
            const int block = at_tile.feature * kCtas + half, m0 = at_tile.row * t.height;
            for (int q = k0 / 4; q <= (k1 - 1) / 4; ++q, ++group) {
                const int slot = group % kSlots;
                if ((group & 1) != warp - 2) continue;
                if (!(ok = __all_sync(kFull, mbar_wait(&bar.scales_empty[slot], (group / kSlots & 1) ^ 1)))) break;
                const uint32_t w = block < blocks ? *reinterpret_cast<const uint32_t *>(g.p.w_scales + (int64_t)block * g.stride + 4 * q)
                                                  : 0x7f7f7f7fu;
                uint4 *at = reinterpret_cast<uint4 *>(scales + slot * kSlotBytes);
                at[lane] = make_uint4(w, w, w, w);
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int64_t row = m0 + 128 * part + 32 * j + lane;
                        v[j] = row < g.p.rows ? *reinterpret_cast<const uint32_t *>(g.p.a_scales + row * g.stride + 4 * q) : 0x7f7f7f7fu;
                    }
                    at[32 + 32 * part + lane] = make_uint4(v[0], v[1], v[2], v[3]);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (kCtas == 1) mbar_arrive(&bar.scales_full[slot]);
                    else mbar_arrive_cluster(lead(&bar.scales_full[slot]));
                }
            }
        }
    } else if (warp >= 4) {
        const int feature = warp % 4 * 32 + lane, group = warp / 4 - 1;
        const bool leads = threadIdx.x % 128 == 0;
        T *const held = chunks + group * t.held * (kChunk * kFeatures);
        // bf16: two halves of 64 features, rows of 128 bytes, their 16-byte pieces swizzled by the row
        const int row = lane % 8;
        const uint32_t mine_at = warp % 4 / 2 * (kChunk * 128) + row * 128 + ((warp % 2 * 4 + lane / 8) ^ row) * 16;
        Ring sums;
        for (int tile = first; tile < tiles && ok; tile += step, sums.next(t.sums)) {
            const Place at_tile = place_of(t, tile);
            const int n0 = at_tile.feature * kWide + half * kFeatures, m0 = at_tile.row * t.height;
            if (kCtas == 1 && t.split > 1) {   // a part of a sum: below
                ok = __all_sync(kFull, mbar_wait(&bar.sum_full[sums.at], sums.round));
                break;
            }
            if (leads) bulk_wait_read_all();   // what was held before has been read
            if (!(ok = mbar_wait_group(&bar.sum_full[sums.at], sums.round, 1 + group))) break;
            tmem_fence_after();
            const uint32_t sum = tmem + sums.at * t.height + ((uint32_t)(warp % 4) * 32 << 16);
            const int rows = n0 >= g.p.n_out ? 0 : (int)(g.p.rows - m0 < t.height ? g.p.rows - m0 : t.height);
            const int part = n0 / (int)g.p.part, x = n0 - part * (int)g.p.part;
            // the sum has been read by this warp: before its stores, which take longer than the products may wait
            const auto sum_read = [&] {
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (kCtas == 1) mbar_arrive(&bar.sum_empty[sums.at]);
                    else mbar_arrive_cluster_relaxed(lead(&bar.sum_empty[sums.at]));
                }
            };
            for (int c0 = group * kChunk; c0 < rows; c0 += t.held * kGroups * kChunk) {
                const int c1 = min(rows, c0 + t.held * kGroups * kChunk);
                if (c0 != group * kChunk) {   // as above
                    if (leads) bulk_wait_read_all();
                    group_sync(group);
                }
                T *chunk = held;
                for (int c = c0; c < c1; c += kGroups * kChunk, chunk += kChunk * kFeatures) {
                    uint32_t v0[16], v1[16];
                    if (sizeof(T) == 2) {
                        tmem_load_fragments(sum + c, v0);
                        tmem_load_fragments(sum + c + (16 << 16), v1);
                    } else {
                        tmem_load16(sum + c, v0);
                        tmem_load16(sum + c + 16, v1);   // a tile of 16 rows: columns that are not used
                    }
                    tmem_load_wait(v0);
                    tmem_load_wait(v1);
                    if (sizeof(T) == 2) {
                        const uint32_t at = smem_u32(chunk) + mine_at;
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            stsm_x4_trans(at + q * 1024, bf16_pair(v0[4 * q], v0[4 * q + 1]), bf16_pair(v0[4 * q + 2], v0[4 * q + 3]),
                                          bf16_pair(v1[4 * q], v1[4 * q + 1]), bf16_pair(v1[4 * q + 2], v1[4 * q + 3]));
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            chunk[j * kFeatures + feature] = from_f32<T>(__uint_as_float(v0[j]));
                            chunk[(16 + j) * kFeatures + feature] = from_f32<T>(__uint_as_float(v1[j]));
                        }
                    }
                }
                if (c0 + t.held * kGroups * kChunk >= rows) sum_read();
                fence_proxy_async_smem();
                group_sync(group);
                if (leads) {
                    constexpr int kStore = sizeof(T) == 2 ? 64 : 128;   // features
                    chunk = held;
                    for (int c = c0; c < c1; c += kGroups * kChunk, chunk += kChunk * kFeatures)
#pragma unroll
                        for (int f = 0; f < kFeatures; f += kStore)
                            if (n0 + f < g.p.n_out) tma_store_3d(&g.out, chunk + f * kChunk, x + f, m0 + c, part);
                    bulk_commit();
                }
            }
            if (group * kChunk >= rows) sum_read();   // nothing of it is this group's
        }
        if (leads) bulk_wait_read_all();   // shared memory stays until its stores have read it
    }
    pdl_trigger();   // not before: the next kernel's CTAs beside this one cost 1 x 1024 x 4096 0.5 us
    if (!ok) report(g.p.status, MB_ERR_TIMEOUT, blockIdx.x);
    __syncthreads();
    if (kCtas == 1 && t.split > 1) {
        // Every CTA has an equal share of the rows, gets all parts of them where its ring was, once all are done with their
        // rings, and adds them up in the order of the ranks. Sent, 16 bytes to a lane, 64 x 4608 x 2304 takes 7.4 us and
        // 1 x 2048 x 1024 4.7; fetched from where each CTA had put its parts down, 8.0 and 5.0 (128 rows of a tile: 10.5,
        // 10.4).
        cluster_arrive();
        const Place at_tile = place_of(t, first);
        const int64_t m0 = (int64_t)at_tile.row * t.height;
        const int each = t.height / t.split, n0 = at_tile.feature * kFeatures;
        const int feature = warp % 4 * 32 + lane / 4 * 4, rows = (int)(g.p.rows - m0 < t.height ? g.p.rows - m0 : t.height);
        const uint32_t sum = tmem + ((uint32_t)(warp % 4) * 32 << 16);
        const int part = (65535 + each) / each;   // of a row below 224, row * part >> 16 is row / each
        cluster_wait();
        if (warp >= 4) {
            tmem_fence_after();
            for (int c = (warp / 4 - 1) * 16; c < rows; c += kGroups * 16) {
                uint32_t v[16];
                tmem_load16(sum + c, v);
                tmem_load_wait(v);
#pragma unroll
                for (int q = 0; q < 16; q += 4) {
                    transpose4(v + q, lane);
                    const int row = c + q + lane % 4, to = row * part >> 16;
                    const uint32_t at = cluster_address(smem, to) + ((rank * each + row - to * each) * kFeatures + feature) * 4;
                    if (row < rows)
                        asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[q]), "r"(v[q + 1]),
                                     "r"(v[q + 2]), "r"(v[q + 3])
                                     : "memory");
                }
            }
        }
        cluster_arrive();
        cluster_wait();
        const float4 *parts = reinterpret_cast<const float4 *>(smem);
        for (int i = threadIdx.x; i < each * 32; i += kThreads) {
            const int64_t m = m0 + rank * each + i / 32, n = n0 + i % 32 * 4;
            if (m >= g.p.rows || n >= g.p.n_out) continue;
            float4 v = parts[i];
#pragma unroll 1
            for (int s = 1; s < t.split; ++s) {
                const float4 o = parts[s * each * 32 + i];
                v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
            }
            store4(out_at<T>(g.p, m, n), v);
        }
    }
    if (kCtas == 2) {   // nobody ends while the other's products and arrivals are under way
        cluster_arrive();
        cluster_wait();
    }
    if (warp == 0) tmem_free<kCtas>(tmem, t.columns);
}

static_assert(sizeof(Barriers) <= kBarrierBytes, "beside the dynamic shared memory");
static_assert(kK == kQuantBlock, "a block of the sum has one scale");

// Clusters of so many CTAs that fit the current device with all the shared memory they can have; 0 where they cannot be
// launched or the device does not say. Asked once: a product takes the same form in every call.
int full_clusters(int size) {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices][kMaxSplit + 1];   // the answer and one, 0: not asked yet
    int dev = 0, n = 0;
    const DeviceLimits *lim = device_limits();
    if (!lim || cudaGetDevice(&dev) != cudaSuccess || dev >= kDevices) return 0;
    if ((n = known[dev][size].load(std::memory_order_relaxed)) > 0) return n - 1;
    const auto kern = matmul_q8_kernel<__nv_bfloat16, 1>;
    const int smem = (int)(lim->smem_optin - kBarrierBytes);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(size * lim->sms));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 0) {
        cudaGetLastError();   // not a later call's
        n = 0;
    }
    known[dev][size].store(n + 1, std::memory_order_relaxed);
    return n;
}

}  // namespace

bool plan_matmul_here(int64_t rows, int64_t n_out, int64_t width, bool out_bf16, MatmulPlan *plan) {
    const DeviceLimits *lim = device_limits();
    if (!lim) return false;
    *plan = plan_matmul(rows, n_out, width, out_bf16, {lim->sms, lim->smem_sm, lim->smem_reserved, lim->smem_optin}, full_clusters);
    return true;
}

cudaError_t launch_matmul_q8(const MatmulParams &p, bool out_bf16, cudaStream_t s) {
    MatmulPlan plan;
    if (!plan_matmul_here(p.rows, p.n_out, p.width, out_bf16, &plan)) return cudaErrorInvalidDevice;
    Args g;
    g.p = p;
    g.stride = (int)quant_stride(p.width);
    g.t = plan.t;
    const Tiles &t = g.t;
    const uint64_t wd[2] = {(uint64_t)p.width, (uint64_t)p.n_out}, ad[2] = {(uint64_t)p.width, (uint64_t)p.rows};
    const uint64_t st[1] = {(uint64_t)p.width};
    const uint32_t wb[2] = {kK, kFeatures}, ab[2] = {kK, (uint32_t)(t.height / plan.ctas)};
    if (!encode_tmap(&g.w, p.w, 1, 2, wd, st, wb, 128) || !encode_tmap(&g.a, p.a, 1, 2, ad, st, ab, 128))
        return cudaErrorInvalidValue;
    const int es = out_bf16 ? 2 : 4;
    const uint64_t od[3] = {(uint64_t)p.part, (uint64_t)p.rows, (uint64_t)(p.n_out / p.part)};
    const uint64_t os[2] = {(uint64_t)(p.part * es), (uint64_t)(p.rows * p.part * es)};
    const uint32_t ob[3] = {out_bf16 ? 64u : 128u, kChunk, 1};
    if (!encode_tmap(&g.out, p.out, es, 3, od, os, ob, out_bf16 ? 128 : 0)) return cudaErrorInvalidValue;
    const bool pair = plan.ctas == 2;
    const auto kern = pair ? (out_bf16 ? matmul_q8_kernel<__nv_bfloat16, 2> : matmul_q8_kernel<float, 2>)
                           : (out_bf16 ? matmul_q8_kernel<__nv_bfloat16, 1> : matmul_q8_kernel<float, 1>);
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)(device_limits()->smem_optin - kBarrierBytes));
    if (e != cudaSuccess) return e;
    return launch_cluster(true, kern, dim3((unsigned)(plan.teams * plan.team)), dim3(kThreads), plan.team, plan.smem, s, g);
}

}  // namespace mbscan
