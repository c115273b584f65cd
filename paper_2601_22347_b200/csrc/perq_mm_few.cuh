// Product of codes for few tokens (or few to an expert): y[t][n] = s_t s_n (sum_k a[t][k] w[n][k] + z_t c_n).
//
// Such calls are bound by reading the weights once, so a tile is 128 weight channels on the lanes of tensor memory by NT = 16 .. 128
// tokens as its columns: one token wastes columns of the tensor core, which has time, and not weights.  A warp loads k-steps by TMA into a
// ring; one issues the products.  4-bit codes lie packed in the ring, 256 to a step, and two teams of four warps spread them to bytes, each every second
// step: weights into tensor memory, a row to a lane, where the tensor core takes its first operand from (through shared memory they would move
// six times their bytes there, 13.0 us for 1 x 4096 x 14336), tokens into operand tiles in shared memory.  Where both operands are packed a tile has
// the even codes of a step or the odd ones (the sum does not mind, as long as both operands have it), where only one is, its halves in their
// order.  The accumulator is 32-bit integers, so sums are exact and the same however they are split.
//
// Few tiles are split along k over the CTAs of a cluster.  Every CTA sends its partial sums to the one that adds them up and stores their
// results, through distributed shared memory: no workspace, no atomics and no second launch.  Where half of an SM's tensor memory and half of its
// shared memory (three loads) are enough, two CTAs share it, so that the next call's set-up runs under this one.  (Every plan takes more than a third
// of the shared memory and, with more than half of the columns, more than two thirds: CTAs that meet on an SM never wait for each other's tensor memory,
// also those of two calls at once.)
//
// Measured in CUDA graphs, weights not in L2: 1 x 4096 x 14336, both packed, 9.9 us, 16 x 14336 x 4096 with 8-bit tokens 10.8 us (29.4 MB, 2.7 .. 3.0 TB/s:
// 4 .. 5 us are launch, the first loads' way and the cluster's sums; the 16 tokens' 112 tiles in two parts are 224 CTAs on 296 places), 64 rows over 32 experts of
// 2048 x 4096 28 us (118 MB, 4.2 TB/s; 448 tiles on 296 CTAs: 76 % busy), 500 over 8 of 2048 x 2048 11.4 us (15.6 with a branch to each result).
//
// Grouped calls (offsets): expert e has rows offsets[e] .. offsets[e + 1].  Every CTA counts the tiles of all experts itself and
// takes every gridDim-th one; experts without rows have none, so their weights are not read.
#pragma once

#include "perq_mm_ptx.cuh"

namespace perq_mm {

constexpr int FEW_ROWS = 128;                 // weight channels of a tile
constexpr int FEW_TEAM = 4;                   // warps of each of two teams that spread packed codes
constexpr uint32_t FEW_TILE = FEW_ROWS * 128; // bytes of 128 channels by 128 codes

struct FewParams {
    const float *a_scales, *w_scales;
    const int32_t *w_sums, *offsets;
    void *out;
    int32_t T, N, E;
    int32_t nt;                  // tokens of a tile
    int32_t n_tiles;             // tiles of N
    int32_t steps;               // k-steps
    int32_t split;               // CTAs of the cluster
    int32_t shift, asym;
    int32_t out_type;
    uint32_t idesc;
    uint32_t loads, spreads;     // stages of the two rings
    uint32_t w_bytes, a_bytes;   // of a load
    uint32_t spread_bytes;       // of a spread stage in shared memory (the tokens)
    uint32_t tmem_cols;          // two accumulators, and the spread weights
    int32_t log2_share;          // four columns each: how many a CTA of the cluster adds up (with fewer fours than CTAs, the first ones one each)
    uint32_t off_spread, off_sums, off_bars, off_first;
};

template <bool W4, bool A4>
struct Few {
    static constexpr bool packed = W4 || A4;
    static constexpr int tiles = packed ? 2 : 1;                              // of 128 codes in a k-step
    static constexpr int step_codes = 128 * tiles;
    static constexpr int epilogue = packed ? 4 + 2 * FEW_TEAM : 4;            // first of four warps
    static constexpr int threads = (epilogue + 4) * 32;
};

// Where a tile's tokens and channels are.
struct FewItem {
    int32_t expert, t0, t_end, n0;
};
__device__ __forceinline__ FewItem few_item(const FewParams &p, const int32_t *first, uint32_t item)
{
    FewItem it;
    if (p.offsets == nullptr) {
        const uint32_t tiles = (uint32_t)(p.T + p.nt - 1) / (uint32_t)p.nt, n = item / tiles;
        it.expert = 0;
        it.t0 = (int32_t)(item - n * tiles) * p.nt;
        it.t_end = p.T;
        it.n0 = (int32_t)n * FEW_ROWS;
        return it;
    }
    // the expert whose tiles begin at or before this one: first[e] tiles of tokens lie before expert e
    int lo = 0, hi = p.E;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((uint32_t)first[mid] * (uint32_t)p.n_tiles <= item) lo = mid; else hi = mid;
    }
    const uint32_t tiles = (uint32_t)(first[lo + 1] - first[lo]), local = item - (uint32_t)first[lo] * (uint32_t)p.n_tiles, n = local / tiles;
    it.expert = lo;
    it.t0 = first[p.E + 1 + lo] + (int32_t)(local - n * tiles) * p.nt;
    it.t_end = first[p.E + 2 + lo];
    it.n0 = (int32_t)n * FEW_ROWS;
    return it;
}

// first[e]: tiles of tokens of the experts before e, and behind these E + 1 numbers the offsets, by one warp.  Offsets outside 0 .. T are taken into
// it, and one below an earlier one counts as that: an expert never has rows of another, and the tiles are no more than the host counts on.
__device__ __forceinline__ void count_tiles(const int32_t *offsets, int E, int32_t T, int32_t nt, int32_t *first, int lane)
{
    int32_t *const at = first + E + 1;
    int32_t most = 0;
    for (int e0 = 0; e0 <= E; e0 += 32) {
        const int e = e0 + lane;
        int32_t v = e <= E ? min(max(__ldg(offsets + e), 0), T) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) v = max(v, __shfl_up_sync(0xffffffffu, v, o));
        v = max(v, most);
        if (e <= E) at[e] = v;
        most = __shfl_sync(0xffffffffu, v, 31);
    }
    __syncwarp();
    int32_t before = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
        const int e = e0 + lane;
        const int32_t n = e < E ? (at[e + 1] - at[e] + nt - 1) / nt : 0;
        int32_t sum = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        if (e < E) first[e] = before + sum - n;
        before += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) first[E] = before;
}

// A word, or its low half, where `yes`; without a branch.
__device__ __forceinline__ void store_if(const void *dst, uint32_t v, bool yes)
{
    asm volatile("{ .reg .pred q; setp.ne.u32 q, %2, 0; @q st.global.b32 [%0], %1; }" ::"l"(dst), "r"(v), "r"((uint32_t)yes) : "memory");
}
__device__ __forceinline__ void store16_if(const void *dst, uint32_t v, bool yes)
{
    asm volatile("{ .reg .pred q; setp.ne.u32 q, %2, 0; @q st.global.b16 [%0], %1; }" ::"l"(dst), "h"((uint16_t)v), "r"((uint32_t)yes) : "memory");
}

// A result, where `yes`.
template <bool F32>
__device__ __forceinline__ void store_one(void *out, int type, size_t at, float v, bool yes)
{
    if (F32) {
        store_if(static_cast<float *>(out) + at, __float_as_uint(v), yes);
    } else {
        uint16_t bf, h;
        asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(bf) : "f"(v));
        asm("cvt.rn.f16.f32 %0, %1;" : "=h"(h) : "f"(v));
        store16_if(static_cast<uint16_t *>(out) + at, type == OUT_BF16 ? bf : h, yes);
    }
}
// Two results in one register, the first in its low half.
__device__ __forceinline__ uint32_t pack_two(int type, float a, float b)
{
    uint32_t r;
    if (type == OUT_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

struct TokenScale {
    float s, z;
};
__device__ __forceinline__ TokenScale token_scale(const float *scales, int asym, int32_t t)
{
    TokenScale r;
    r.s = __ldg(scales + (asym ? 2 * (size_t)t : (size_t)t));
    r.z = asym ? __ldg(scales + 2 * (size_t)t + 1) : 0.0f;
    return r;
}

// Packed rows of 128 bytes (256 codes) with 128-byte swizzle become two operand tiles.  BOTH: the even codes and the odd ones, in their places; else the
// first and second half, in their order.  Tokens, by a team; eight lanes have a row's chunks and write eight groups of banks (in their
// order the second half's odd chunks come first, for that).
template <bool BOTH>
__device__ __forceinline__ void spread_tokens(uint32_t src, uint32_t dst, uint32_t tile, int rows, int tid)
{
    for (int i = tid; i < rows * 8; i += FEW_TEAM * 32) {
        const uint32_t r = (uint32_t)i >> 3, c = (uint32_t)i & 7u;
        const uint4 v = lds128(src + operand_at(r, c));
        const uint4 lo = make_uint4(codes_lo(v.x), codes_lo(v.y), codes_lo(v.z), codes_lo(v.w));
        const uint4 hi = make_uint4(codes_hi(v.x), codes_hi(v.y), codes_hi(v.z), codes_hi(v.w));
        if (BOTH) {
            const uint32_t at = dst + operand_at(r, c);
            sts128(at, lo);
            sts128(at + tile, hi);
        } else {
            const uint4 x = make_uint4(__byte_perm(lo.x, hi.x, 0x5140), __byte_perm(lo.x, hi.x, 0x7362), __byte_perm(lo.y, hi.y, 0x5140),
                                       __byte_perm(lo.y, hi.y, 0x7362));
            const uint4 y = make_uint4(__byte_perm(lo.z, hi.z, 0x5140), __byte_perm(lo.z, hi.z, 0x7362), __byte_perm(lo.w, hi.w, 0x5140),
                                       __byte_perm(lo.w, hi.w, 0x7362));
            const uint32_t to = dst + (c >> 2) * tile, k = 2u * (c & 3u);
            const bool second = (c >> 2) != 0u;
            sts128(to + operand_at(r, second ? k + 1u : k), second ? y : x);
            sts128(to + operand_at(r, second ? k : k + 1u), second ? x : y);
        }
    }
}
// Weights, a row to a lane: 32 columns of tensor memory to a tile.
template <bool BOTH>
__device__ __forceinline__ void spread_weights(uint32_t src, uint32_t columns, int row)
{
#pragma unroll
    for (int g = 0; g < 8; g += 4) {
        uint32_t w[16];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint4 v = lds128(src + operand_at((uint32_t)row, (uint32_t)(g + c)));
            w[4 * c] = v.x; w[4 * c + 1] = v.y; w[4 * c + 2] = v.z; w[4 * c + 3] = v.w;
        }
        uint32_t x[16];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (BOTH) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = half ? codes_hi(w[i]) : codes_lo(w[i]);
                tmem_store16(columns + 32 * half + 4 * g, x);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t lo = codes_lo(w[8 * half + i]), hi = codes_hi(w[8 * half + i]);
                    x[2 * i] = __byte_perm(lo, hi, 0x5140);
                    x[2 * i + 1] = __byte_perm(lo, hi, 0x7362);
                }
                tmem_store16(columns + 8 * g + 16 * half, x);
            }
        }
    }
}

// Places in a ring: stage and the parity of its phase.
struct Ring {
    uint32_t n, stage, parity;
    __device__ __forceinline__ explicit Ring(uint32_t stages, uint32_t first_parity = 0u) : n(stages), stage(0u), parity(first_parity) {}
    __device__ __forceinline__ void next()
    {
        if (++stage == n) {
            stage = 0u;
            parity ^= 1u;
        }
    }
};

template <bool W4, bool A4>
__global__ void __launch_bounds__(Few<W4, A4>::threads, Few<W4, A4>::packed ? 2 : 4)
few_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ FewParams p)
{
    using K = Few<W4, A4>;
    extern __shared__ unsigned char raw[];
    unsigned char *const smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    int32_t *const first = reinterpret_cast<int32_t *>(smem + p.off_first);           // [2 (E + 1)], see count_tiles
    volatile uint32_t *const slot = reinterpret_cast<volatile uint32_t *>(smem + p.off_bars);
    // barriers: loads full and empty, spread full and empty, accumulators full and empty (two)
    const uint32_t l_full = base + p.off_bars + 16, l_empty = l_full + 8 * p.loads, s_full = l_empty + 8 * p.loads, s_empty = s_full + 8 * p.spreads,
                   d_full = s_empty + 8 * p.spreads, d_empty = d_full + 16;
    const uint32_t rank = p.split > 1 ? cluster_rank() : 0u;
    const uint32_t clusters = gridDim.x / (uint32_t)p.split, begin = blockIdx.x / (uint32_t)p.split;
    const uint32_t step0 = (uint32_t)p.steps * rank / (uint32_t)p.split, step1 = (uint32_t)p.steps * (rank + 1u) / (uint32_t)p.split;
    const uint32_t a_tile = (uint32_t)p.nt * 128u, load_bytes = p.w_bytes + p.a_bytes;
    auto load_at = [&](uint32_t s) { return base + s * load_bytes; };
    auto spread_at = [&](uint32_t s) { return base + p.off_spread + s * p.spread_bytes; };
    auto weights_at = [&](uint32_t tmem, uint32_t s) { return tmem + 2u * (uint32_t)p.nt + s * 64u; };
    auto give_up = [&]() { atomicOr(&g_error, ERROR_FEW); };
    auto load = [&](const FewItem &it, uint32_t k, uint32_t s) {
        const uint32_t to = load_at(s), bar = l_full + 8 * s;
        const int w_row = it.expert * p.N + it.n0;
        mbar_expect_tx(bar, load_bytes);
        if (W4) tma_load(to, &w_map, (int)(k * 128u), w_row, bar);
        else
            for (int h = 0; h < K::tiles; ++h) tma_load(to + h * FEW_TILE, &w_map, (int)(k * K::step_codes + h * 128u), w_row, bar);
        if (A4) tma_load(to + p.w_bytes, &a_map, (int)(k * 128u), it.t0, bar);
        else
            for (int h = 0; h < K::tiles; ++h) tma_load(to + p.w_bytes + h * a_tile, &a_map, (int)(k * K::step_codes + h * 128u), it.t0, bar);
    };

    uint32_t early = 0;                                      // k-steps of the first tile that are loaded before anything else is set up
    if (warp == 0) {
        if (lane == 0) {
            prefetch_map(&w_map);
            prefetch_map(&a_map);
            for (uint32_t i = 0; i < p.loads; ++i) {
                mbar_init(l_full + 8 * i, 1);
                // let go by the warps that spread it and, where an operand is used as it was loaded, by the tensor core
                mbar_init(l_empty + 8 * i, (K::packed ? FEW_TEAM : 0) + (W4 && A4 ? 0 : 1));
            }
            mbar_init_fence();
            griddep_wait();
            if (p.offsets == nullptr) {
                const FewItem it = few_item(p, first, begin);
                for (; early < p.loads && step0 + early < step1; ++early) load(it, step0 + early, early);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + p.off_bars), "r"(p.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (warp == 3 && lane == 0) {
        for (uint32_t i = 0; i < p.spreads; ++i) {
            mbar_init(s_full + 8 * i, FEW_TEAM);
            mbar_init(s_empty + 8 * i, 1);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            mbar_init(d_full + 8 * i, 1);
            mbar_init(d_empty + 8 * i, 4);
        }
        mbar_init_fence();
    }
    griddep_wait();
    griddep_launch();
    if (warp == 2 && p.offsets != nullptr) count_tiles(p.offsets, p.E, p.T, p.nt, first, lane);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (p.split > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");        // (this CTA's shared memory is there)

    const uint32_t tmem = *slot;
    const uint32_t token_tiles = p.offsets ? (uint32_t)first[p.E] : (uint32_t)(p.T + p.nt - 1) / (uint32_t)p.nt;
    const uint32_t items = token_tiles * (uint32_t)p.n_tiles;

    if (warp == 0) {
        if (lane == 0) {
            Ring r(p.loads, 1u);
            uint32_t n = 0;
            bool ok = true;
            for (uint32_t item = begin; item < items && ok; item += clusters) {
                const FewItem it = few_item(p, first, item);
                for (uint32_t k = step0; k < step1; ++k, ++n, r.next()) {
                    if (n < early) continue;
                    if (!mbar_wait(l_empty + 8 * r.stage, r.parity)) { give_up(); ok = false; break; }
                    load(it, k, r.stage);
                }
            }
            // nothing is in flight when the CTA ends, also after a wait that ran out
            for (uint32_t i = n > p.loads ? n - p.loads : 0u; i < n; ++i) (void)mbar_wait(l_full + 8 * (i % p.loads), (i / p.loads) & 1u);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            Ring r(p.loads), u(p.spreads);
            uint32_t j = 0;
            bool ok = true;
            for (uint32_t item = begin; item < items; item += clusters, ++j) {
                const uint32_t b = j & 1u;
                if (j >= 2 && !mbar_wait(d_empty + 8 * b, ((j >> 1) - 1u) & 1u)) ok = false;
                const uint32_t d = tmem + b * (uint32_t)p.nt;
                tmem_fence_after();
                for (uint32_t k = step0; k < step1; ++k, r.next()) {
                    ok = ok && (K::packed ? mbar_wait(s_full + 8 * u.stage, u.parity) : mbar_wait(l_full + 8 * r.stage, r.parity));
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t w = W4 ? weights_at(tmem, u.stage) : load_at(r.stage), a = A4 ? spread_at(u.stage) : load_at(r.stage) + p.w_bytes;
#pragma unroll
                    for (int h = 0; h < K::tiles; ++h) {
                        const uint32_t ad = operand_lo(a + h * a_tile), wd = operand_lo(w + h * FEW_TILE);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (W4) product_from_tmem(d, w + 32 * h + 8 * i, ad + 2 * i, p.idesc, k > step0 || h > 0 || i > 0);
                            else product<1>(d, wd + 2 * i, ad + 2 * i, p.idesc, k > step0 || h > 0 || i > 0);
                        }
                    }
                    if (!(W4 && A4)) commit(l_empty + 8 * r.stage);
                    if (K::packed) {
                        commit(s_empty + 8 * u.stage);
                        u.next();
                    }
                }
                if (!ok) { give_up(); break; }
                commit(d_full + 8 * b);
            }
            // (products in flight end before tensor memory is given back)
            for (uint32_t i = j > 2 ? j - 2 : 0u; i < j; ++i) (void)mbar_wait(d_full + 8 * (i & 1u), (i >> 1) & 1u);
        }
        __syncwarp();
    } else if (K::packed && warp >= 4 && warp < 4 + 2 * FEW_TEAM) {
        const int team = (warp - 4) / FEW_TEAM, st = tid - 128 - team * FEW_TEAM * 32;
        Ring r(p.loads), u(p.spreads, 1u);
        uint32_t n = 0;
        bool ok = true;
        for (uint32_t item = begin; item < items && ok; item += clusters) {
            for (uint32_t k = step0; k < step1; ++k, ++n, r.next(), u.next()) {
                if ((n & 1u) != (uint32_t)team) continue;
                ok = mbar_wait_warp(l_full + 8 * r.stage, r.parity) && mbar_wait_warp(s_empty + 8 * u.stage, u.parity);
                if (!ok) { give_up(); break; }
                const uint32_t from = load_at(r.stage);
                if (A4) {
                    spread_tokens<W4 && A4>(from + p.w_bytes, spread_at(u.stage), a_tile, p.nt, st);
                    fence_async_smem();
                    __syncwarp();
                }
                if (W4) {
                    tmem_fence_after();
                    spread_weights<W4 && A4>(from, weights_at(tmem, u.stage) + ((uint32_t)((warp & 3) * 32) << 16), (warp & 3) * 32 + lane);
                    tmem_store_wait();
                    tmem_fence_before();
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(s_full + 8 * u.stage);
                    mbar_arrive(l_empty + 8 * r.stage);
                }
            }
        }
    } else if (warp >= K::epilogue) {
        const int q = warp & 3;
        uint32_t j = 0;
        if (p.split > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        for (uint32_t item = begin; item < items; item += clusters, ++j) {
            const uint32_t b = j & 1u;
            const FewItem it = few_item(p, first, item);
            const int n = it.n0 + q * 32 + lane, columns = min(p.nt, it.t_end - it.t0);
            const bool mine = n < p.N;
            float s_n = 0.0f, c_n = 0.0f;
            if (p.split == 1) {
                const size_t channel = (size_t)it.expert * (size_t)p.N + (size_t)min(n, p.N - 1);
                s_n = __ldg(p.w_scales + channel);
                c_n = p.asym ? (float)__ldg(p.w_sums + channel) : 0.0f;
            }
            if (!mbar_wait_warp(d_full + 8 * b, (j >> 1) & 1u)) { give_up(); break; }
            tmem_fence_after();
            const uint32_t from = tmem + b * (uint32_t)p.nt + ((uint32_t)(q * 32) << 16);
            TokenScale ts = {0.0f, 0.0f};
            for (int c = 0; c < columns; c += 16) {
                int32_t u[16];
                __syncwarp();
                tmem_load16(from + c, u);
                if (p.split > 1) {                          // partial sums, four columns of a channel at a time: to the CTA that adds them up
                    tmem_wait(u);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        if (c + i < columns) {
                            const uint32_t four = (uint32_t)(c + i) >> 2, owner = four >> p.log2_share;
                            const uint32_t at = base + p.off_sums + (((rank << p.log2_share) + (four & ((1u << p.log2_share) - 1u))) * FEW_ROWS + (uint32_t)(q * 32 + lane)) * 16u;
                            asm volatile("{ .reg .b32 a; mapa.shared::cluster.u32 a, %0, %1; st.shared::cluster.v4.u32 [a], {%2, %3, %4, %5}; }"
                                         ::"r"(at), "r"(owner), "r"(u[i]), "r"(u[i + 1]), "r"(u[i + 2]), "r"(u[i + 3]) : "memory");
                        }
                    }
                } else {
                    if ((c & 16) == 0) ts = token_scale(p.a_scales, p.asym, min(it.t0 + c + lane, p.T - 1));      // of 32 tokens, one to a lane
                    tmem_wait(u);
                    float y[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        y[i] = scaled(u[i], p.shift, __shfl_sync(0xffffffffu, ts.s, (c & 16) + i), s_n, __shfl_sync(0xffffffffu, ts.z, (c & 16) + i), c_n);
                    const size_t at = (size_t)(it.t0 + c) * (size_t)p.N + (size_t)n;
                    if (p.out_type == OUT_F32) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) store_one<true>(p.out, p.out_type, at + (size_t)i * (size_t)p.N, y[i], mine && c + i < columns);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) store_one<false>(p.out, p.out_type, at + (size_t)i * (size_t)p.N, y[i], mine && c + i < columns);
                    }
                }
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(d_empty + 8 * b);
        }
    }
    __syncwarp();
    tmem_fence_before();
    if (p.split == 1) {
        __syncthreads();
    } else {
        // every CTA of the cluster adds up a share of the tile's tokens, a thread four tokens of a channel
        if (warp < K::epilogue) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        const bool any = begin < items;
        FewItem it = {0, 0, 0, 0};
        if (any) it = few_item(p, first, begin);
        const int share = 1 << p.log2_share, row = tid & (FEW_ROWS - 1), n = it.n0 + row;
        int four = tid / FEW_ROWS;
        auto token_of = [&](int f) { return it.t0 + (((int)rank << p.log2_share) + f) * 4; };
        auto here = [&](int f) { return any && n < p.N && f < share && (int)rank * share + f < p.nt / 4 && token_of(f) < it.t_end; };
        float s_n = 0.0f, c_n = 0.0f;
        TokenScale ts[4];
        if (here(four)) {                                    // (on their way while the others' sums arrive)
            const size_t channel = (size_t)it.expert * (size_t)p.N + (size_t)n;
            s_n = __ldg(p.w_scales + channel);
            c_n = p.asym ? (float)__ldg(p.w_sums + channel) : 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) ts[e] = token_scale(p.a_scales, p.asym, min(token_of(four) + e, it.t_end - 1));
        }
        cluster_sync();
        while (here(four)) {
            int32_t v[4] = {0, 0, 0, 0};
            for (int r = 0; r < p.split; ++r) {
                const uint4 u = lds128(base + p.off_sums + (uint32_t)((((r << p.log2_share) + four) * FEW_ROWS + row) * 16));
                v[0] += (int32_t)u.x; v[1] += (int32_t)u.y; v[2] += (int32_t)u.z; v[3] += (int32_t)u.w;
            }
            const int t = token_of(four);
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = scaled(v[e], p.shift, ts[e].s, s_n, ts[e].z, c_n);
            const size_t at = (size_t)t * (size_t)p.N + (size_t)n;
            if (p.out_type == OUT_F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) store_one<true>(p.out, p.out_type, at + (size_t)e * (size_t)p.N, y[e], t + e < it.t_end);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) store_one<false>(p.out, p.out_type, at + (size_t)e * (size_t)p.N, y[e], t + e < it.t_end);
            }
            four += K::threads / FEW_ROWS;
            if (!here(four)) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) ts[e] = token_scale(p.a_scales, p.asym, min(token_of(four) + e, it.t_end - 1));
        }
    }
    __syncwarp();
    if (warp == 1) {
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.tmem_cols) : "memory");
    }
}

}  // namespace perq_mm
