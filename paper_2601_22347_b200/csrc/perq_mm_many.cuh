// Product of codes for many tokens: y[t][n] = s_t s_n (sum_k a[t][k] w[n][k] + z_t c_n), 8-bit operands.
//
// Bound by the tensor cores.  A pair of CTAs (cta_group::2) shares a tile of 256 tokens by 256 channels: each CTA has 128 tokens on the lanes
// of its tensor memory and loads them and half of the channels, so that an SM reads 64 bytes of operands a cycle for 8192 products
// instead of 96.  Two accumulators: the epilogue of a tile, by eight warps, runs under the products of the next.  One CTA to an SM; pairs take every
// (gridDim / 2)-th tile, in bands of 8 tiles of tokens, so that tiles in flight share operands in L2.
//
// Few tiles of a dense call are split along k over up to four pairs of a cluster.  They meet when their products are done, send their sums, 16
// columns at a time, to the pair that adds them up, into the shared memory that held operands, and meet again.
//
// Packed operands are spread to bytes before (spread_kernel), in the caller's workspace.
//
// Measured in CUDA graphs, 8-bit codes: 16384 x 4096 x 14336 in 606 us (3.2e15 operations a second, tensor pipe 88 %); 4099 rows over 32 experts of
// 2048 x 4096 in 63 us (287 MB, 4.6 TB/s; pipe 59 %); 1531 x 1001 x 9728 in 22 us (48 of the 74 pairs have work, 8 us are launch, the first loads and the pairs'
// exchange).  4-bit codes: 2048 x 4096 x 4096 in 31.5 us, 5 more than with 8-bit ones (spread_kernel); 8192 rows over 8 experts of 4096 x 2048 in 74 us, 17.5 of
// them spread_kernel (42 MB read, 84 MB written to L2 in part: 7.2 TB/s).  These are at 1965 MHz.  Back to back for seconds, under the power limit: 714 us at
// 1290 MHz, 77 at 1245 (so the 4099 rows are not bound by DRAM alone: 22 of their 35 tiles of tokens hold 128 rows or fewer, and the pair's second CTA loads others'
// rows all the same) and 83 at 1710.
// Tried: tiles of 128 channels (a k-step takes as long), stores that do not stay in L2 (no change), the next 16 columns on their way while the last are stored
// (62 -> 64 us at 4099 rows: the epilogue waits for its stores).
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
    int32_t split;               // pairs of a cluster
    int32_t shift, asym, out_type;
    int32_t wide;                // 32 bytes of results can be stored at once
    uint32_t idesc;
};

constexpr int MANY_CHANNELS = 256;
constexpr uint32_t MANY_STAGE = 2 * MANY_HALF;
constexpr uint32_t MANY_STAGES = 6;

struct ManySmem {
    static constexpr uint32_t bars = MANY_STAGES * MANY_STAGE;            // full, empty; accumulators full, empty
    static constexpr uint32_t slot = bars + 16 * MANY_STAGES + 32;
    static constexpr uint32_t scales = slot + 16;                         // [2][256] of the channels' scales, [2][256] of their sums
    static constexpr uint32_t rows = scales + 4 * 4 * MANY_CHANNELS;      // [8][32][MANY_ROOM] of the epilogue's warps
    static constexpr uint32_t first = rows + 8 * 32 * MANY_ROOM * 4;      // [2 (E + 1)], see count_tiles
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
        begin = first[p.E + 1 + lo];
        it.t_end = first[p.E + 2 + lo];
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
// The products issued so far, at the barriers of both CTAs (bits of their ranks).
__device__ __forceinline__ void commit_pair(uint32_t bar, uint32_t both)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)both) : "memory");
}
__device__ __forceinline__ void store_wide_if(const void *dst, const uint32_t (&w)[8], bool yes)
{
    asm volatile("{ .reg .pred q; setp.ne.u32 q, %9, 0; @q st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8}; }"
                 ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"((uint32_t)yes) : "memory");
}
__device__ __forceinline__ void store_wide(void *dst, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// The results of one lane's token: 16 adjacent channels from column c of the tile on, from their sums.  Called by whole warps; `rows` of the
// warp's 32 tokens are there.
//
// Rows that cannot be stored 32 bytes at a time go through shared memory.  16-bit results wait there for the next 16 columns (`more`: these come), then 16
// lanes store a row's 32 as words, shifted by a result where the row begins between two words; fp32 ones go at once.  (bf16, 2048 x 4097 x 2048, rows of 4112
// being 16.5 us: 29.5 by single results, 28.1 by words, 21.8 without branches, and 19.4 for 4098.)
struct ManyRow {
    TokenScale ts;
    int32_t t, rows, n0;
    uint32_t scale, sums, room;  // shared memory: the channels' scales and sums, and the warp's room
    int32_t waiting;             // columns in the room
};
__device__ __forceinline__ void many_store(const ManyParams &p, ManyRow &r, const int32_t (&u)[16], int c, bool more, int lane)
{
    float y[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4 v = lds128(r.scale + 4u * (uint32_t)c + 16u * i), z = p.asym ? lds128(r.sums + 4u * (uint32_t)c + 16u * i) : make_uint4(0, 0, 0, 0);
        y[4 * i] = scaled(u[4 * i], p.shift, r.ts.s, __uint_as_float(v.x), r.ts.z, __uint_as_float(z.x));
        y[4 * i + 1] = scaled(u[4 * i + 1], p.shift, r.ts.s, __uint_as_float(v.y), r.ts.z, __uint_as_float(z.y));
        y[4 * i + 2] = scaled(u[4 * i + 2], p.shift, r.ts.s, __uint_as_float(v.z), r.ts.z, __uint_as_float(z.z));
        y[4 * i + 3] = scaled(u[4 * i + 3], p.shift, r.ts.s, __uint_as_float(v.w), r.ts.z, __uint_as_float(z.w));
    }
    const size_t at = (size_t)r.t * (size_t)p.N + (size_t)(r.n0 + c);
    if (p.out_type == OUT_F32) {
        if (p.wide && r.n0 + c + 16 <= p.N) {
            uint32_t w[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(y[8 * h + i]);
                store_wide_if(static_cast<float *>(p.out) + at + 8 * h, w, lane < r.rows);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) sts32(r.room + (uint32_t)(lane * MANY_ROOM + i) * 4u, __float_as_uint(y[i]));
        __syncwarp();
        const int n = r.n0 + c + (lane & 15);
        const float *const to = static_cast<const float *>(p.out) + (size_t)(r.t - lane + (lane >> 4)) * (size_t)p.N + (size_t)n;
#pragma unroll
        for (int h0 = 0; h0 < 16; h0 += 8) {
            uint32_t v[8];
#pragma unroll
            for (int h = 0; h < 8; ++h) v[h] = lds32(r.room + (uint32_t)((2 * (h0 + h) + (lane >> 4)) * MANY_ROOM + (lane & 15)) * 4u);
#pragma unroll
            for (int h = 0; h < 8; ++h) store_if(to + (size_t)(2 * (h0 + h)) * (size_t)p.N, v[h], n < p.N && 2 * (h0 + h) + (lane >> 4) < r.rows);
        }
        __syncwarp();
        return;
    }
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = pack_two(p.out_type, y[2 * i], y[2 * i + 1]);
    if (p.wide && r.n0 + c + 16 <= p.N) {
        store_wide_if(static_cast<uint16_t *>(p.out) + at, w, lane < r.rows);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sts32(r.room + (uint32_t)(lane * MANY_ROOM + r.waiting / 2 + i) * 4u, w[i]);
    r.waiting += 16;
    if (r.waiting < 32 && more) return;
    __syncwarp();
    // (every second row: its place between two words is the same for all that a lane stores)
    const int i = lane & 15, n0 = r.n0 + c + 16 - r.waiting, columns = min(r.waiting, p.N - n0);
    const uint16_t *const to = static_cast<const uint16_t *>(p.out) + (size_t)(r.t - lane + (lane >> 4)) * (size_t)p.N + (size_t)n0;
    const int odd = (int)(reinterpret_cast<uintptr_t>(to) >> 1) & 1, e = 2 * i + odd;              // results e and e + 1 are a word of the row
    const bool both = e + 1 < columns, one = !both && e < columns, first = odd && i == 0, edges = __any_sync(0xffffffffu, one || first);
#pragma unroll
    for (int h0 = 0; h0 < 16; h0 += 8) {
        uint32_t v[8], v1[8];
#pragma unroll
        for (int h = 0; h < 8; ++h) {
            const uint32_t from = r.room + (uint32_t)((2 * (h0 + h) + (lane >> 4)) * MANY_ROOM + i) * 4u;
            v[h] = lds32(from);
            v1[h] = lds32(from + 4u);
        }
#pragma unroll
        for (int h = 0; h < 8; ++h) {
            const uint16_t *const row = to + (size_t)(2 * (h0 + h)) * (size_t)p.N;
            const bool there = 2 * (h0 + h) + (lane >> 4) < r.rows;
            const uint32_t word = __funnelshift_r(v[h], v1[h], 16 * odd);
            store_if(row + e, word, both && there);
            if (edges) {
                store16_if(row + e, word, one && there);
                store16_if(row, v[h], first && there);
            }
        }
    }
    __syncwarp();
    r.waiting = 0;
}

__global__ void __launch_bounds__(MANY_THREADS, 1)
many_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ ManyParams p)
{
    extern __shared__ unsigned char raw[];
    unsigned char *const smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    // the CTA of its pair, the pair's first CTA, the pair of its cluster
    const uint32_t rank = cluster_rank(), side = rank & 1u, lead = rank & ~1u, part = rank >> 1, split = (uint32_t)p.split;
    int32_t *const first = reinterpret_cast<int32_t *>(smem + ManySmem::first);
    const uint32_t full = base + ManySmem::bars, empty = full + 8 * MANY_STAGES, d_full = empty + 8 * MANY_STAGES, d_empty = d_full + 16;
    if (tid == 0) {
        prefetch_map(&w_map);
        prefetch_map(&a_map);
        for (uint32_t i = 0; i < MANY_STAGES; ++i) {
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
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + ManySmem::slot), "r"(2u * MANY_CHANNELS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    griddep_wait();
    griddep_launch();
    if (warp == 2 && p.offsets != nullptr) count_tiles(p.offsets, p.E, p.T, MANY_TOKENS, first, lane);
    tmem_fence_before();
    __syncthreads();
    cluster_sync();                                          // (the others' barriers are there)
    tmem_fence_after();

    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(smem + ManySmem::slot);
    const uint32_t token_tiles = p.offsets ? (uint32_t)first[p.E] : (uint32_t)(p.T + MANY_TOKENS - 1) / MANY_TOKENS;
    const uint32_t items = token_tiles * (uint32_t)p.n_tiles, begin = blockIdx.x / (2u * split), pairs = gridDim.x / (2u * split);
    const int step0 = (int)((uint32_t)p.steps * part / split), step1 = (int)((uint32_t)p.steps * (part + 1u) / split);
    auto give_up = [&]() { atomicOr(&g_error, ERROR_MANY); };

    // of an epilogue warp: its quarter of the lanes, its half of the columns
    const int q = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    ManyRow row;
    row.waiting = 0;
    row.room = base + ManySmem::rows + (uint32_t)((warp - 4) * 32 * MANY_ROOM) * 4u;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t n = 0;
            bool ok = true;
            for (uint32_t item = begin; item < items && ok; item += pairs) {
                const ManyItem it = many_item(p, first, item);
                const int w_row = it.expert * p.N + it.n0 + (int)side * (MANY_CHANNELS / 2), a_row = it.t0 + (int)side * 128;
                for (int k = step0; k < step1; ++k, ++n) {
                    const uint32_t s = n % MANY_STAGES, bar = full + 8 * s, to = base + s * MANY_STAGE;
                    if (n >= MANY_STAGES && !mbar_wait(empty + 8 * s, (n / MANY_STAGES - 1u) & 1u)) { give_up(); ok = false; break; }
                    if (side == 0) mbar_expect_tx(bar, 2 * MANY_STAGE);      // both CTAs' loads
                    tma_load_pair(to, &a_map, k * 128, a_row, bar);
                    tma_load_pair(to + MANY_HALF, &w_map, k * 128, w_row, bar);
                }
            }
            // nothing is in flight when the pair ends, also after a wait that ran out (both CTAs' loads count at the first one's barriers)
            if (side == 0)
                for (uint32_t i = n > MANY_STAGES ? n - MANY_STAGES : 0u; i < n; ++i) (void)mbar_wait(full + 8 * (i % MANY_STAGES), (i / MANY_STAGES) & 1u);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (side == 0 && lane == 0) {
            uint32_t n = 0, j = 0;
            bool ok = true;
            for (uint32_t item = begin; item < items; item += pairs, ++j) {
                const uint32_t b = j & 1u, d = tmem + b * MANY_CHANNELS;
                if (j >= 2 && !mbar_wait(d_empty + 8 * b, ((j >> 1) - 1u) & 1u)) ok = false;
                tmem_fence_after();
                for (int k = step0; k < step1 && ok; ++k, ++n) {
                    const uint32_t s = n % MANY_STAGES;
                    ok = mbar_wait(full + 8 * s, (n / MANY_STAGES) & 1u);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t a = operand_lo(base + s * MANY_STAGE), w = operand_lo(base + s * MANY_STAGE + MANY_HALF);
#pragma unroll
                    for (int i = 0; i < 4; ++i) product<2>(d, a + 2 * i, w + 2 * i, p.idesc, k > step0 || i > 0);
                    commit_pair(empty + 8 * s, 3u << lead);
                }
                if (!ok) { give_up(); break; }
                commit_pair(d_full + 8 * b, 3u << lead);
            }
            for (uint32_t i = j > 2 ? j - 2 : 0u; i < j; ++i) (void)mbar_wait(d_full + 8 * (i & 1u), (i >> 1) & 1u);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // (a wait that ran out ends no warp's part: the eight go on to the barriers that they share, without waiting or storing)
        uint32_t j = 0;
        bool ok = true;
        for (uint32_t item = begin; item < items; item += pairs, ++j) {
            const uint32_t b = j & 1u;
            const ManyItem it = many_item(p, first, item);
            row.scale = base + ManySmem::scales + b * MANY_CHANNELS * 4u;
            row.sums = row.scale + 2u * MANY_CHANNELS * 4u;
            // (the scales of the tile before last are read no more: all eight warps have met since)
            {
                const int i = tid - 128;
                const size_t channel = (size_t)it.expert * (size_t)p.N + (size_t)min(it.n0 + i, p.N - 1);
                sts32(row.scale + 4u * (uint32_t)i, __float_as_uint(__ldg(p.w_scales + channel)));
                if (p.asym) sts32(row.sums + 4u * (uint32_t)i, __float_as_uint((float)__ldg(p.w_sums + channel)));
            }
            row.t = it.t0 + (int)side * 128 + q * 32 + lane;
            row.n0 = it.n0;
            row.rows = min(32, it.t_end - (row.t - lane));
            row.ts = token_scale(p.a_scales, p.asym, min(row.t, p.T - 1));
            __syncwarp();                                    // (the barrier wants whole warps, and lane 0 comes from the arrival below)
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (ok && !mbar_wait_warp(d_full + 8 * b, (j >> 1) & 1u)) { give_up(); ok = false; }
            if (split > 1) break;                            // (one tile to a cluster: see below)
            tmem_fence_after();
            for (int c = half * (MANY_CHANNELS / 2); c < (half + 1) * (MANY_CHANNELS / 2) && it.n0 + c < p.N && row.rows > 0 && ok; c += 16) {
                int32_t u[16];
                __syncwarp();
                tmem_load16(tmem + b * MANY_CHANNELS + lanes + c, u);
                tmem_wait(u);
                many_store(p, row, u, c, c + 16 < (half + 1) * (MANY_CHANNELS / 2) && it.n0 + c + 16 < p.N, lane);
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(d_empty + 8 * b, lead);
        }
    }

    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    cluster_sync();                                          // (nobody leaves or overwrites what another may still use)
    tmem_fence_after();
    if (split > 1) {
        // columns 16 g .. 16 g + 15 are added up by pair g split / 16; sums lie as [part][column group][4 columns][128 tokens], 16 bytes each
        const uint32_t g0 = (16u * part + split - 1u) / split, g1 = (16u * (part + 1u) + split - 1u) / split;
        if (warp >= 4) {
            for (uint32_t g = (uint32_t)half * 8u; g < (uint32_t)half * 8u + 8u; ++g) {
                const uint32_t owner = g * split / 16u, owner_g0 = (16u * owner + split - 1u) / split, owner_n = (16u * (owner + 1u) + split - 1u) / split - owner_g0;
                int32_t u[16];
                __syncwarp();
                tmem_load16(tmem + lanes + 16u * g, u);
                tmem_wait(u);
                const uint32_t at = base + (((part * owner_n + (g - owner_g0)) * 4u) * 128u + (uint32_t)(q * 32 + lane)) * 16u;
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    asm volatile("{ .reg .b32 a; mapa.shared::cluster.u32 a, %0, %1; st.shared::cluster.v4.u32 [a], {%2, %3, %4, %5}; }"
                                 ::"r"(at + i * 128u * 16u), "r"(2u * owner + side), "r"(u[4 * i]), "r"(u[4 * i + 1]), "r"(u[4 * i + 2]), "r"(u[4 * i + 3]) : "memory");
            }
        }
        __syncwarp();
        cluster_sync();
        if (warp >= 4) {
            // (the first half of the warps has one more where they are odd)
            const uint32_t middle = (g0 + g1 + 1u) / 2u, end = half ? g1 : middle;
            for (uint32_t g = half ? middle : g0; g < end; ++g) {
                if (row.rows <= 0 || row.n0 + (int)(16u * g) >= p.N) break;
                int32_t u[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) u[i] = 0;
                for (uint32_t r = 0; r < split; ++r) {
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        const uint4 v = lds128(base + (((r * (g1 - g0) + (g - g0)) * 4u + i) * 128u + (uint32_t)(q * 32 + lane)) * 16u);
                        u[4 * i] += (int32_t)v.x; u[4 * i + 1] += (int32_t)v.y; u[4 * i + 2] += (int32_t)v.z; u[4 * i + 3] += (int32_t)v.w;
                    }
                }
                many_store(p, row, u, (int)(16u * g), g + 1u < end && row.n0 + (int)(16u * g + 16u) < p.N, lane);
            }
        }
    }
    __syncwarp();
    if (warp == 1) {
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2u * MANY_CHANNELS) : "memory");
    }
}

// Packed rows to bytes, 16 times the codes, in their order: tokens (blockIdx.y == 0, where they are packed), and the weights of every expert
// that has rows, which the product reads next, from L2 where they fit.  A thread has two chunks of 16 bytes on their
// way (one / two / four / eight, 2048 x 4096 x 4096 with 8-bit tokens, in us: 30.5 / 31.0 / 32.6 / 34).
struct SpreadParams {
    const uint4 *tokens, *weights;
    uint4 *tokens_out, *weights_out;
    const int32_t *offsets;
    long long token_chunks, expert_chunks;       // of 16 packed bytes
    int32_t T;
    int32_t wide;                                // the workspace can be written 32 bytes at a time
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
    for (long long i0 = (long long)blockIdx.x * 256 + (int)threadIdx.x; i0 < n; i0 += 2 * step) {
        uint4 v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (i0 + k * step < n) v[k] = __ldg(src + i0 + k * step);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (i0 + k * step >= n) break;
            const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
            uint32_t x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = codes_lo(w[i]), hi = codes_hi(w[i]);
                x[2 * i] = __byte_perm(lo, hi, 0x5140);
                x[2 * i + 1] = __byte_perm(lo, hi, 0x7362);
            }
            uint4 *const to = dst + 2 * (i0 + k * step);
            if (p.wide) {
                store_wide(to, x);
            } else {
                to[0] = make_uint4(x[0], x[1], x[2], x[3]);
                to[1] = make_uint4(x[4], x[5], x[6], x[7]);
            }
        }
    }
}

}  // namespace perq_mm
