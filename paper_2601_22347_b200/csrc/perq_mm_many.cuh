// Product of codes for many tokens: y[t][n] = s_t s_n (sum_k a[t][k] w[n][k] + z_t c_n), 8-bit operands.
//
// Bound by the tensor cores.  A pair of CTAs (cta_group::2) shares a tile of 256 tokens by 256 (or 128) channels: each CTA has 128 tokens on the lanes
// of its tensor memory and loads them and half of the channels, so that an SM reads 64 bytes of operands a cycle for 8192 products
// instead of 96.  Two accumulators: the epilogue of a tile, by eight warps, runs under the products of the next.  One CTA to an SM; pairs take every
// (gridDim / 2)-th tile, in bands of 8 tiles of tokens, so that tiles in flight share operands in L2.
//
// Packed operands are spread to bytes before (spread_kernel), in the caller's workspace.
#pragma once

#include "perq_mm_few.cuh"

namespace perq_mm {

constexpr int MANY_TOKENS = 256;                            // of a tile; either half is a CTA's to load
constexpr uint32_t MANY_HALF = 128 * 128;                   // bytes of its 128 tokens by 128 codes
constexpr int MANY_BAND = 8;
constexpr int MANY_THREADS = 384;                           // warps: loads, products, two idle, eight of the epilogue
constexpr int MANY_ROOM = 17;                               // words of a lane's 16 results on their way to whole rows

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

// CHANNELS of a tile: 256 or 128.
template <int CHANNELS>
struct Many {
    static constexpr uint32_t stage = MANY_HALF + CHANNELS / 2 * 128;
    static constexpr int stages = CHANNELS == 256 ? 6 : 8;
    static constexpr uint32_t bars = stages * stage;                      // full, empty; accumulators full, empty
    static constexpr uint32_t slot = bars + 16 * stages + 32;
    static constexpr uint32_t scales = slot + 16;                         // [2][CHANNELS] of the channels' scales, [2][CHANNELS] of their sums
    static constexpr uint32_t rows = scales + 4 * 4 * CHANNELS;           // [8][32][MANY_ROOM] of the epilogue's warps
    static constexpr uint32_t first = rows + 8 * 32 * MANY_ROOM * 4;      // [E + 1]
};

struct ManyItem {
    int32_t expert, t0, t_end, n0;
};
// Tiles of an expert (or of the call) in bands of MANY_BAND tiles of tokens, tokens first inside a band.
template <int CHANNELS>
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
    it.n0 = (int32_t)n * CHANNELS;
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
__device__ __forceinline__ void store_wide(void *dst, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

template <int CHANNELS>
__global__ void __launch_bounds__(MANY_THREADS, 1)
many_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ ManyParams p)
{
    using K = Many<CHANNELS>;
    constexpr uint32_t STAGES = K::stages;
    extern __shared__ unsigned char raw[];
    unsigned char *const smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t rank = cluster_rank();
    int32_t *const first = reinterpret_cast<int32_t *>(smem + K::first);
    const uint32_t full = base + K::bars, empty = full + 8 * STAGES, d_full = empty + 8 * STAGES, d_empty = d_full + 16;
    if (tid == 0) {
        prefetch_map(&w_map);
        prefetch_map(&a_map);
        for (uint32_t i = 0; i < STAGES; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(d_full + 8 * i, 1);
            mbar_init(d_empty + 8 * i, 16);              // the epilogue warps of both CTAs
        }
        mbar_init_fence();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + K::slot), "r"(2u * CHANNELS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    griddep_wait();
    griddep_launch();
    if (warp == 2 && p.offsets != nullptr) count_tiles(p.offsets, p.E, p.T, MANY_TOKENS, first, lane);
    tmem_fence_before();
    __syncthreads();
    cluster_sync();                                          // (both CTAs' barriers are there)
    tmem_fence_after();

    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(smem + K::slot);
    const uint32_t token_tiles = p.offsets ? (uint32_t)first[p.E] : (uint32_t)(p.T + MANY_TOKENS - 1) / MANY_TOKENS;
    const uint32_t items = token_tiles * (uint32_t)p.n_tiles, begin = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    auto give_up = [&]() { atomicOr(&g_error, ERROR_MANY); };

    if (warp == 0) {
        if (lane == 0) {
            uint32_t n = 0;
            bool ok = true;
            for (uint32_t item = begin; item < items && ok; item += pairs) {
                const ManyItem it = many_item<CHANNELS>(p, first, item);
                const int w_row = it.expert * p.N + it.n0 + (int)rank * (CHANNELS / 2), a_row = it.t0 + (int)rank * 128;
                for (int k = 0; k < p.steps; ++k, ++n) {
                    const uint32_t s = n % STAGES, bar = full + 8 * s, to = base + s * K::stage;
                    if (n >= STAGES && !mbar_wait(empty + 8 * s, (n / STAGES - 1u) & 1u)) { give_up(); ok = false; break; }
                    if (rank == 0) mbar_expect_tx(bar, 2 * K::stage);      // both CTAs' loads
                    tma_load_pair(to, &a_map, k * 128, a_row, bar);
                    tma_load_pair(to + MANY_HALF, &w_map, k * 128, w_row, bar);
                }
            }
            // nothing is in flight when the pair ends, also after a wait that ran out (both CTAs' loads count at the first one's barriers)
            if (rank == 0)
                for (uint32_t i = n > STAGES ? n - STAGES : 0u; i < n; ++i) (void)mbar_wait(full + 8 * (i % STAGES), (i / STAGES) & 1u);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            uint32_t n = 0, j = 0;
            bool ok = true;
            for (uint32_t item = begin; item < items; item += pairs, ++j) {
                const uint32_t b = j & 1u, d = tmem + b * CHANNELS;
                if (j >= 2 && !mbar_wait(d_empty + 8 * b, ((j >> 1) - 1u) & 1u)) ok = false;
                tmem_fence_after();
                for (int k = 0; k < p.steps && ok; ++k, ++n) {
                    const uint32_t s = n % STAGES;
                    ok = mbar_wait(full + 8 * s, (n / STAGES) & 1u);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t a = operand_lo(base + s * K::stage), w = operand_lo(base + s * K::stage + MANY_HALF);
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
        // (a wait that ran out ends no warp's part: the eight go on to the barriers that they share, without waiting or storing)
        const int q = warp & 3, half = (warp - 4) >> 2, st = tid - 128;
        const int c_begin = half * (CHANNELS / 2), c_end = c_begin + CHANNELS / 2;
        const uint32_t room = base + K::rows + (uint32_t)((warp - 4) * 32 * MANY_ROOM) * 4u;
        uint32_t j = 0;
        bool ok = true;
        for (uint32_t item = begin; item < items; item += pairs, ++j) {
            const uint32_t b = j & 1u;
            const ManyItem it = many_item<CHANNELS>(p, first, item);
            const uint32_t scale = base + K::scales + b * CHANNELS * 4u, sums = scale + 2u * CHANNELS * 4u;
            // (the scales of the tile before last are read no more: all eight warps have met since)
            for (int i = st; i < CHANNELS; i += 256) {
                const size_t channel = (size_t)it.expert * (size_t)p.N + (size_t)min(it.n0 + i, p.N - 1);
                sts32(scale + 4u * (uint32_t)i, __float_as_uint(__ldg(p.w_scales + channel)));
                if (p.asym) sts32(sums + 4u * (uint32_t)i, __float_as_uint((float)__ldg(p.w_sums + channel)));
            }
            const int t = it.t0 + (int)rank * 128 + q * 32 + lane;
            const bool mine = t < it.t_end;
            const TokenScale ts = token_scale(p.a_scales, p.asym, min(t, p.T - 1));
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (ok && !mbar_wait(d_full + 8 * b, (j >> 1) & 1u)) { give_up(); ok = false; }
            tmem_fence_after();
            const uint32_t from = tmem + b * CHANNELS + ((uint32_t)(q * 32) << 16);
            const size_t row = (size_t)t * (size_t)p.N;
            const int rows = min(32, it.t_end - (t - lane));         // of this warp
            for (int c = c_begin; c < c_end && it.n0 + c < p.N && rows > 0 && ok; c += 16) {
                int32_t u[16];
                tmem_load16(from + c, u);
                float y[16];
                float4 s_n[4], c_n[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 v = lds128(scale + 4u * (uint32_t)c + 16u * i), z = p.asym ? lds128(sums + 4u * (uint32_t)c + 16u * i) : make_uint4(0, 0, 0, 0);
                    s_n[i] = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
                    c_n[i] = make_float4(__uint_as_float(z.x), __uint_as_float(z.y), __uint_as_float(z.z), __uint_as_float(z.w));
                }
                tmem_wait(u);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[4 * i] = scaled(u[4 * i], p.shift, ts.s, s_n[i].x, ts.z, c_n[i].x);
                    y[4 * i + 1] = scaled(u[4 * i + 1], p.shift, ts.s, s_n[i].y, ts.z, c_n[i].y);
                    y[4 * i + 2] = scaled(u[4 * i + 2], p.shift, ts.s, s_n[i].z, ts.z, c_n[i].z);
                    y[4 * i + 3] = scaled(u[4 * i + 3], p.shift, ts.s, s_n[i].w, ts.z, c_n[i].w);
                }
                const size_t at = row + (size_t)(it.n0 + c);
                uint32_t w[8];
                if (p.wide && it.n0 + c + 16 <= p.N) {
                    if (p.out_type == OUT_F32) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(y[8 * h + i]);
                            if (mine) store_wide(static_cast<float *>(p.out) + at + 8 * h, w);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = pack_two(p.out_type, y[2 * i], y[2 * i + 1]);
                        if (mine) store_wide(static_cast<uint16_t *>(p.out) + at, w);
                    }
                } else {
                    // rows that cannot be stored 32 bytes at a time go through shared memory: 16 lanes then store adjacent results
#pragma unroll
                    for (int i = 0; i < 16; ++i) sts32(room + (uint32_t)(lane * MANY_ROOM + i) * 4u, __float_as_uint(y[i]));
                    __syncwarp();
                    const int n = it.n0 + c + (lane & 15);
                    for (int r = lane >> 4; r < rows; r += 2) {
                        float v;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(room + (uint32_t)(r * MANY_ROOM + (lane & 15)) * 4u) : "memory");
                        if (n < p.N) store_one(p.out, p.out_type, (size_t)(t - lane + r) * (size_t)p.N + (size_t)n, v);
                    }
                    __syncwarp();
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
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2u * CHANNELS) : "memory");
    }
}

// Packed rows to bytes, 16 times the codes, in their order: tokens (blockIdx.y == 0, where they are packed), and the weights of every expert
// that has rows, which the product reads next, from L2 where they fit.  The tokens are read for 4 chunks of 16 bytes at once.
struct SpreadParams {
    const uint4 *tokens, *weights;
    uint4 *tokens_out, *weights_out;
    const int32_t *offsets;
    long long token_chunks, expert_chunks;       // of 16 packed bytes
    int32_t T;
};
__global__ void __launch_bounds__(256) spread_kernel(const SpreadParams p)
{
    griddep_wait();
    griddep_launch();
    const bool tokens = p.tokens != nullptr && blockIdx.y == 0;
    const int expert = (int)blockIdx.y - (p.tokens != nullptr ? 1 : 0);
    if (!tokens && p.offsets != nullptr &&
        min(max(__ldg(p.offsets + expert), 0), p.T) >= min(max(__ldg(p.offsets + expert + 1), 0), p.T)) return;
    const uint4 *const src = tokens ? p.tokens : p.weights + (size_t)expert * (size_t)p.expert_chunks;
    uint4 *const dst = tokens ? p.tokens_out : p.weights_out + 2 * (size_t)expert * (size_t)p.expert_chunks;
    const long long n = tokens ? p.token_chunks : p.expert_chunks, step = (long long)gridDim.x * 256;
    for (long long i0 = (long long)blockIdx.x * 256 + (int)threadIdx.x; i0 < n; i0 += 4 * step) {
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i0 + k * step < n) v[k] = __ldg(src + i0 + k * step);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i0 + k * step >= n) break;
            const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
            uint32_t x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = codes_lo(w[i]), hi = codes_hi(w[i]);
                x[2 * i] = __byte_perm(lo, hi, 0x5140);
                x[2 * i + 1] = __byte_perm(lo, hi, 0x7362);
            }
            store_wide(dst + 2 * (i0 + k * step), x);
        }
    }
}

}  // namespace perq_mm
