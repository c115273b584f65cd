// Product of codes for many tokens: y[t][n] = s_t s_n (sum_k a[t][k] w[n][k] + z_t c_n), 8-bit operands.
//
// Bound by the tensor cores.  A pair of CTAs (cta_group::2) shares a tile of 256 tokens by 256 channels: each CTA has 128 tokens on the lanes
// of its tensor memory and loads them and half of the channels, so that an SM reads 64 bytes of operands a cycle for 8192 products
// instead of 96.  Two accumulators: the epilogue of a tile runs under the products of the next.  One CTA to an SM; pairs take every
// (gridDim / 2)-th tile, in bands of 8 tiles of tokens, so that tiles in flight share operands in L2.
//
// Packed operands are spread to bytes before (spread_kernel), in the caller's workspace.
#pragma once

#include "perq_mm_few.cuh"

namespace perq_mm {

constexpr int MANY_TOKENS = 256, MANY_CHANNELS = 256;      // of a tile; either half is a CTA's to load
constexpr uint32_t MANY_HALF = 128 * 128;                   // bytes of 128 rows by 128 codes
constexpr uint32_t MANY_STAGE = 2 * MANY_HALF;
constexpr int MANY_STAGES = 6;
constexpr int MANY_BAND = 8;
constexpr int MANY_THREADS = 256;                           // loads, products, two idle, four of the epilogue

struct ManyParams {
    const float *a_scales, *w_scales;
    const int32_t *w_sums, *offsets;
    void *out;
    int32_t T, N, E;
    int32_t n_tiles, steps;
    int32_t shift, asym, out_type;
    int32_t wide;                // 32 bytes of results can be stored at once
    uint32_t idesc;
};

struct ManySmem {
    static constexpr uint32_t bars = MANY_STAGES * MANY_STAGE;            // full, empty; accumulators full, empty
    static constexpr uint32_t slot = bars + 16 * MANY_STAGES + 32;
    static constexpr uint32_t scales = slot + 16;                         // [2][256] of the channels' scales, [2][256] of their sums
    static constexpr uint32_t first = scales + 4 * 4 * MANY_CHANNELS;     // [E + 1]
};

struct ManyItem {
    int32_t expert, t0, t_end, n0;
};
// Tiles of an expert (or of the call) in bands of MANY_BAND tiles of tokens, tokens first inside a band.
__device__ __forceinline__ ManyItem many_item(const ManyParams &p, const int32_t *first, uint32_t item)
{
    ManyItem it;
    uint32_t tiles, local;
    int32_t begin = 0;
    it.expert = 0;
    it.t_end = p.T;
    if (p.offsets == nullptr) {
        tiles = (uint32_t)(p.T + MANY_TOKENS - 1) / MANY_TOKENS;
        local = item;
    } else {
        int lo = 0, hi = p.E;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((uint32_t)first[mid] * (uint32_t)p.n_tiles <= item) lo = mid; else hi = mid;
        }
        tiles = (uint32_t)(first[lo + 1] - first[lo]);
        local = item - (uint32_t)first[lo] * (uint32_t)p.n_tiles;
        it.expert = lo;
        begin = min(max(__ldg(p.offsets + lo), 0), p.T);
        it.t_end = min(max(__ldg(p.offsets + lo + 1), 0), p.T);
    }
    const uint32_t band = local / (MANY_BAND * (uint32_t)p.n_tiles), in = local - band * MANY_BAND * (uint32_t)p.n_tiles;
    const uint32_t height = min((uint32_t)MANY_BAND, tiles - band * MANY_BAND), n = in / height;
    it.t0 = begin + (int32_t)(band * MANY_BAND + in - n * height) * MANY_TOKENS;
    it.n0 = (int32_t)n * MANY_CHANNELS;
    return it;
}

// A load of the pair: its bytes count at the leading CTA's barrier (the same offset; bit 24 of the address is the CTA of the pair).
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar & 0xfeffffffu) : "memory");
}
// The products issued so far, at the barriers of both CTAs.
__device__ __forceinline__ void commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, int32_t (&u)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
                   "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]),
                   "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]),
                   "=r"(u[30]), "=r"(u[31])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void store_wide(void *dst, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

__global__ void __launch_bounds__(MANY_THREADS, 1)
many_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap a_map, const ManyParams p)
{
    extern __shared__ unsigned char raw[];
    unsigned char *const smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t rank = cluster_rank();
    int32_t *const first = reinterpret_cast<int32_t *>(smem + ManySmem::first);
    const uint32_t full = base + ManySmem::bars, empty = full + 8 * MANY_STAGES, d_full = empty + 8 * MANY_STAGES, d_empty = d_full + 16;
    if (tid == 0) {
        prefetch_map(&w_map);
        prefetch_map(&a_map);
        for (int i = 0; i < MANY_STAGES; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(d_full + 8 * i, 1);
            mbar_init(d_empty + 8 * i, 8);               // the epilogue warps of both CTAs
        }
        mbar_init_fence();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + ManySmem::slot), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    griddep_wait();
    griddep_launch();
    if (warp == 2 && p.offsets != nullptr) count_tiles(p.offsets, p.E, p.T, MANY_TOKENS, first, lane);
    tmem_fence_before();
    __syncthreads();
    cluster_sync();                                          // (both CTAs' barriers are there)
    tmem_fence_after();

    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(smem + ManySmem::slot);
    const uint32_t token_tiles = p.offsets ? (uint32_t)first[p.E] : (uint32_t)(p.T + MANY_TOKENS - 1) / MANY_TOKENS;
    const uint32_t items = token_tiles * (uint32_t)p.n_tiles, begin = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    auto give_up = [&]() { atomicOr(&g_error, ERROR_MANY); };

    if (warp == 0) {
        if (lane == 0) {
            uint32_t n = 0;
            bool ok = true;
            for (uint32_t item = begin; item < items && ok; item += pairs) {
                const ManyItem it = many_item(p, first, item);
                const int w_row = it.expert * p.N + it.n0 + (int)rank * 128, a_row = it.t0 + (int)rank * 128;
                for (int k = 0; k < p.steps; ++k, ++n) {
                    const uint32_t s = n % MANY_STAGES, bar = full + 8 * s, to = base + s * MANY_STAGE;
                    if (n >= MANY_STAGES && !mbar_wait(empty + 8 * s, (n / MANY_STAGES - 1u) & 1u)) { give_up(); ok = false; break; }
                    if (rank == 0) mbar_expect_tx(bar, 2 * MANY_STAGE);      // both CTAs' loads
                    tma_load_pair(to, &a_map, k * 128, a_row, bar);
                    tma_load_pair(to + MANY_HALF, &w_map, k * 128, w_row, bar);
                }
            }
            // nothing is in flight when the pair ends, also after a wait that ran out (both CTAs' loads count at the first one's barriers)
            if (rank == 0)
                for (uint32_t i = n > MANY_STAGES ? n - MANY_STAGES : 0u; i < n; ++i) (void)mbar_wait(full + 8 * (i % MANY_STAGES), (i / MANY_STAGES) & 1u);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            uint32_t n = 0, j = 0;
            bool ok = true;
            for (uint32_t item = begin; item < items; item += pairs, ++j) {
                const uint32_t b = j & 1u, d = tmem + b * MANY_CHANNELS;
                if (j >= 2 && !mbar_wait(d_empty + 8 * b, ((j >> 1) - 1u) & 1u)) ok = false;
                tmem_fence_after();
                for (int k = 0; k < p.steps && ok; ++k, ++n) {
                    const uint32_t s = n % MANY_STAGES;
                    ok = mbar_wait(full + 8 * s, (n / MANY_STAGES) & 1u);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t a = operand_lo(base + s * MANY_STAGE), w = operand_lo(base + s * MANY_STAGE + MANY_HALF);
#pragma unroll
                    for (int i = 0; i < 4; ++i) product<2>(d, a + 2 * i, w + 2 * i, p.idesc, k > 0 || i > 0);
                    commit_pair(empty + 8 * s);
                }
                if (!ok) { give_up(); break; }
                commit_pair(d_full + 8 * b);
            }
            for (uint32_t i = j > 2 ? j - 2 : 0u; i < j; ++i) (void)mbar_wait(d_full + 8 * (i & 1u), (i >> 1) & 1u);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // (a wait that ran out ends no warp's part: the four go on to the barriers that they share, without waiting or storing)
        const int q = warp & 3, st = tid - 128;
        uint32_t j = 0;
        bool ok = true;
        for (uint32_t item = begin; item < items; item += pairs, ++j) {
            const uint32_t b = j & 1u;
            const ManyItem it = many_item(p, first, item);
            float *const scale = reinterpret_cast<float *>(smem + ManySmem::scales) + b * MANY_CHANNELS, *const sums = scale + 2 * MANY_CHANNELS;
            // (the scales of the tile before last are read no more: all four warps have met since)
            for (int i = st; i < MANY_CHANNELS; i += 128) {
                const int n = it.n0 + i;
                const size_t channel = (size_t)it.expert * (size_t)p.N + (size_t)min(n, p.N - 1);
                scale[i] = __ldg(p.w_scales + channel);
                sums[i] = p.asym ? (float)__ldg(p.w_sums + channel) : 0.0f;
            }
            const int t = it.t0 + (int)rank * 128 + q * 32 + lane;
            const bool mine = t < it.t_end;
            const TokenScale ts = token_scale(p.a_scales, p.asym, min(t, p.T - 1));
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (ok && !mbar_wait(d_full + 8 * b, (j >> 1) & 1u)) { give_up(); ok = false; }
            tmem_fence_after();
            const uint32_t from = tmem + b * MANY_CHANNELS + ((uint32_t)(q * 32) << 16);
            const size_t row = (size_t)t * (size_t)p.N;
            for (int c = 0; c < MANY_CHANNELS && it.n0 + c < p.N; c += 32) {
                int32_t u[32];
                tmem_load32(from + c, u);
                if (!mine || !ok) continue;
                float y[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = scaled(u[i], p.shift, ts.s, scale[c + i], ts.z, sums[c + i]);
                const size_t at = row + (size_t)(it.n0 + c);
                if (p.wide && it.n0 + c + 32 <= p.N) {
                    uint32_t w[8];
                    if (p.out_type == OUT_F32) {
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(y[8 * h + i]);
                            store_wide(static_cast<float *>(p.out) + at + 8 * h, w);
                        }
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) w[i] = pack_two(p.out_type, y[16 * h + 2 * i], y[16 * h + 2 * i + 1]);
                            store_wide(static_cast<uint16_t *>(p.out) + at + 16 * h, w);
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (it.n0 + c + i < p.N) store_one(p.out, p.out_type, at + i, y[i]);
                }
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(d_empty + 8 * b, 0);
        }
    }

    tmem_fence_before();
    __syncthreads();
    cluster_sync();                                          // (neither leaves while the other may arrive at its barriers or use its operands)
    if (warp == 1) {
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Packed rows to bytes, 16 times the codes, in their order.  Of grouped weights only the experts that have rows.
struct SpreadParams {
    const uint4 *src;
    uint4 *dst;
    const int32_t *offsets;      // (weights of experts)
    long long chunks;            // of 16 packed bytes
    long long per_expert;
    int32_t T;
};
__global__ void __launch_bounds__(256) spread_kernel(const SpreadParams p)
{
    griddep_wait();
    griddep_launch();
    for (long long i = (long long)blockIdx.x * 256 + (int)threadIdx.x; i < p.chunks; i += (long long)gridDim.x * 256) {
        if (p.offsets != nullptr) {
            const int e = (int)(i / p.per_expert);
            if (min(max(__ldg(p.offsets + e), 0), p.T) >= min(max(__ldg(p.offsets + e + 1), 0), p.T)) continue;
        }
        const uint4 v = __ldg(p.src + i);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t x[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t lo = codes_lo(w[k]), hi = codes_hi(w[k]);
            x[2 * k] = __byte_perm(lo, hi, 0x5140);
            x[2 * k + 1] = __byte_perm(lo, hi, 0x7362);
        }
        p.dst[2 * i] = make_uint4(x[0], x[1], x[2], x[3]);
        p.dst[2 * i + 1] = make_uint4(x[4], x[5], x[6], x[7]);
    }
}

}  // namespace perq_mm
