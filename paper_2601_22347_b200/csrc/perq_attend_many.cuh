// Attention over the 8-bit cache for many queries to a sequence: prompts and chunks of them, on the fifth-generation tensor cores.
//
// A CTA has 256 rows (pairs of a token and one of the `group` heads of queries to a head of keys), two tiles of 128, and goes over the keys they see, 128 at a time.  Four warps
// bring codes in, make them fp16 (exactly) and lay them down as operands, keys and values in turn, in a ring; one thread issues the products: S = Q K^T into tensor memory, then O += P V with P
// from tensor memory and V's rows as they are (its channels run along N).  Either tile has four warps of its own, a row to a thread: the row's maximum, P = 2^(x + log2 s_v - m)
// rounded to fp16 over the columns where S was, and the probabilities' sum.  The products of one tile run under the other's exponentials.  O stays in tensor memory; m moves, and
// O with it, only when something is over 2^8 times larger.
//
// Bound by the tensor cores and the exponentials alike: 128 x 128 x 128 products twice are 1024 cycles, the tile's 16384 exponentials as many.
#pragma once

#include "perq_attend_few.cuh"

namespace perq_kv {

constexpr int MANY_ROWS = 256, MANY_KEYS = 128, MANY_THREADS = 512;
// (perq_attend_few's rows go up to this; both sides measured beside launch_attention)
enum : unsigned int { ERROR_ATTEND = 1u << 7 };

struct ManyParams {
    AttendParams a;
    float *partial;                           // [item][split][256][D + 2], where the keys of an item are split over CTAs
    int32_t split;
};

template <int D>
struct Many {
    static constexpr uint32_t tile = 128u * D * 2u;                    // bytes of 128 rows of fp16
    static constexpr uint32_t half = 128u * 128u;                      // of 64 channels of them
    static constexpr uint32_t stages = D == 128 ? 5 : 8;
    static constexpr uint32_t off_ring = 2u * tile, off_steps = off_ring + stages * tile;
    static constexpr uint32_t off_bars = off_steps + 8u * 8u * 16u;
    static constexpr uint32_t bars = 2u * stages + 8u + 2u + 2u + 2u + 2u + 1u;   // full, empty; steps; Q, S, P, O of each tile; the end
    static constexpr uint32_t off_slot = off_bars + 8u * bars, bytes = off_slot + 16u + 1024u;
    static constexpr uint32_t columns = 512u;                          // S0, S1, O0, O1
    static constexpr uint32_t o_column = 256u;
};

// kind::f16, fp16 operands, fp32 sums; values' channels run along N (the second operand's rows are keys).
__host__ __device__ constexpr uint32_t f16_desc(int m, int n, bool second_transposed)
{
    return (1u << 4) | ((uint32_t)second_transposed << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void product_f16(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{ .reg .pred p; .reg .b64 a, b; setp.ne.b32 p, %4, 0; mov.b64 a, {%1, %5}; mov.b64 b, {%2, %5}; "
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p; }"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(perq_mm::OPERAND_HI) : "memory");
}
__device__ __forceinline__ void product_f16_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{ .reg .pred p; .reg .b64 b; setp.ne.b32 p, %4, 0; mov.b64 b, {%2, %5}; "
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p; }"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(perq_mm::OPERAND_HI) : "memory");
}
// A tile of [128 rows][64 channels] halves: as an operand whose rows are M or N, and as one whose rows are K (64 channels of N, then those a half further on).
__device__ __forceinline__ uint32_t rows_operand(uint32_t addr) { return ((addr >> 4) & 0x3fffu) | (1u << 16); }
template <int D>
__device__ __forceinline__ uint32_t keys_operand(uint32_t addr) { return ((addr >> 4) & 0x3fffu) | ((Many<D>::half >> 4) << 16); }

#define PERQ_R8(v, i) "=f"(v[i]), "=f"(v[i + 1]), "=f"(v[i + 2]), "=f"(v[i + 3]), "=f"(v[i + 4]), "=f"(v[i + 5]), "=f"(v[i + 6]), "=f"(v[i + 7])
// 32 columns of this warp's 32 lanes; they are there after loads_wait.
__device__ __forceinline__ void tmem_load32(uint32_t at, float (&v)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : PERQ_R8(v, 0), PERQ_R8(v, 8), PERQ_R8(v, 16), PERQ_R8(v, 24) : "r"(at) : "memory");
}
#undef PERQ_R8
#define PERQ_W8(v, i) "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]), "+f"(v[i + 6]), "+f"(v[i + 7])
__device__ __forceinline__ void loads_wait(float (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : PERQ_W8(v, 0), PERQ_W8(v, 8), PERQ_W8(v, 16), PERQ_W8(v, 24) :: "memory");
}
__device__ __forceinline__ void loads_there(float (&v)[32])            // (after a loads_wait that came later)
{
    asm volatile("" : PERQ_W8(v, 0), PERQ_W8(v, 8), PERQ_W8(v, 16), PERQ_W8(v, 24) :: "memory");
}
#undef PERQ_W8
#define PERQ_O8(v, i) "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]), "f"(v[i + 3]), "f"(v[i + 4]), "f"(v[i + 5]), "f"(v[i + 6]), "f"(v[i + 7])
__device__ __forceinline__ void tmem_store32(uint32_t at, const float (&v)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
                 :: PERQ_O8(v, 0), PERQ_O8(v, 8), PERQ_O8(v, 16), PERQ_O8(v, 24), "r"(at) : "memory");
}
#undef PERQ_O8

typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair_of(float x, float y)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void pair_split(Pair p, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p)); }
__device__ __forceinline__ Pair pair_fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Pair pair_add(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max_of3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// What a CTA works on.
struct ManyItem {
    int32_t sequence, head, row0, rows;       // rows of the sequence's (token, head) pairs
    int32_t begin, first;                     // its rows of the call, and the position of the first
    int32_t sunk, low, tiles;                 // tiles of keys: 0 .. sunk - 1, then from `low` on
    int32_t number;                           // of the item: where its parts lie
};
__device__ __forceinline__ int many_tiles(const AttendParams &p, const Rows &r)
{
    const long long rows = (long long)min(r.n, p.most) * p.group;
    return rows > p.few_rows ? (int)((rows + MANY_ROWS - 1) / MANY_ROWS) : 0;
}
// The number-th tile of rows of the call (head by head, a sequence's last first: those see most).  Called by all threads of the CTA.
template <int THREADS_>
__device__ __forceinline__ ManyItem many_item(const AttendParams &p, int number)
{
    __shared__ int32_t sums[THREADS_ / 32];
    __shared__ ManyItem found;
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5, head = number % p.heads, tile = number / p.heads;
    if (tid == 0) found.rows = 0;
    for (int base = 0, before = 0; base < p.q.S; base += THREADS_) {
        Rows r = {0, 0, 0};
        int c = 0;
        if (base + tid < p.q.S) {
            r = rows_of(p.q, base + tid);
            c = many_tiles(p, r);
        }
        int sum = c;
#pragma unroll
        for (int l = 1; l < 32; l *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, sum, l);
            if (lane >= l) sum += v;
        }
        if (lane == 31) sums[warp] = sum;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < THREADS_ / 32; ++w) {
            if (w < warp) sum += sums[w];
            all += sums[w];
        }
        const int at = tile - (before + sum - c);
        if (at >= 0 && at < c) {
            ManyItem it;
            const int tokens = min(r.n, p.most);
            it.sequence = base + tid;
            it.head = head;
            it.row0 = (c - 1 - at) * MANY_ROWS;
            it.rows = min(MANY_ROWS, tokens * p.group - it.row0);
            it.begin = r.begin;
            it.first = r.length - r.n;
            const int position0 = it.first + it.row0 / p.group, position1 = it.first + (it.row0 + it.rows - 1) / p.group;
            it.low = p.window > 0 ? max(position0 - p.window + 1, 0) / MANY_KEYS : 0;
            const int end = max(position1 + 1, 0);
            it.sunk = min((min(p.sinks, end) + MANY_KEYS - 1) / MANY_KEYS, it.low);
            it.tiles = it.sunk + (end + MANY_KEYS - 1) / MANY_KEYS - it.low;
            it.number = number;
            found = it;
        }
        before += all;
        __syncthreads();
        if (before > tile) break;
    }
    __syncthreads();
    return found;
}

template <int D>
__device__ __forceinline__ float *many_part(const ManyParams &p, int number, int part)
{
    return p.partial + ((size_t)number * (size_t)p.split + (size_t)part) * (size_t)(MANY_ROWS * (D + 2));
}

template <int D, bool FINE>                   // FINE: pages of 16 tokens
__global__ void __launch_bounds__(MANY_THREADS, 1) many_kernel(const __grid_constant__ ManyParams p)
{
    using K = Many<D>;
    using namespace perq_mm;
    extern __shared__ __align__(128) unsigned char smem[];
    const uint32_t base = (smem_u32(smem) + 1023u) & ~1023u;
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    griddep_wait();
    griddep_launch();
    const int part = (int)(blockIdx.x % (unsigned)p.split);
    const ManyItem it = many_item<MANY_THREADS>(p.a, (int)(blockIdx.x / (unsigned)p.split));
    if (it.rows <= 0) return;
    const int tile0 = (int)((long long)it.tiles * part / p.split), tile1 = (int)((long long)it.tiles * (part + 1) / p.split), tiles = tile1 - tile0;
    const bool two = it.rows > 128;
    const uint32_t full = base + K::off_bars, empty = full + 8u * K::stages, steps_full = empty + 8u * K::stages, q_full = steps_full + 64u, s_full = q_full + 16u,
                   p_full = s_full + 16u, o_full = p_full + 16u, end = o_full + 16u, slot = base + K::off_slot, steps = base + K::off_steps;
    if (tid == 0) {
        for (uint32_t i = 0; i < K::stages; ++i) {
            mbar_init(full + 8u * i, 4);                               // a warp that brings codes in, each
            mbar_init(empty + 8u * i, 1);
        }
        for (uint32_t i = 0; i < 8; ++i) mbar_init(steps_full + 8u * i, 1);
        for (uint32_t i = 0; i < 2; ++i) {
            mbar_init(q_full + 8u * i, 4);
            mbar_init(s_full + 8u * i, 1);
            mbar_init(p_full + 8u * i, 4);
            mbar_init(o_full + 8u * i, 1);
        }
        mbar_init(end, 1);
        mbar_init_fence();
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(K::columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = lds32(slot);
    auto give_up = [&]() { atomicOr(&g_error, ERROR_ATTEND); };
    auto key_of = [&](int tile) { return (tile < it.sunk ? tile : tile - it.sunk + it.low) * MANY_KEYS; };

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const int t = warp >> 2, thread = tid & 127, row = t * 128 + thread;
        const bool there = row < it.rows;
        const int token = (it.row0 + min(row, it.rows - 1)) / p.a.group, h = it.row0 + min(row, it.rows - 1) - token * p.a.group;
        const int position = it.first + token;
        const size_t all_heads = (size_t)p.a.heads * (size_t)p.a.group, of_row = (size_t)it.head * (size_t)p.a.group + (size_t)h;
        float factor;
        if (t == 0 || two) {
            // the row, rotated, scaled to 1 .. 2 by a power of two, fp16
            float v[D], most = 0.0f;
            const uint4 *const from = reinterpret_cast<const uint4 *>(p.a.x + (size_t)(it.begin + token) * (size_t)p.a.stride + of_row * D);
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const uint4 w = there ? __ldg(from + c) : make_uint4(0, 0, 0, 0);
                const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[8 * c + 2 * k] = from16(x[k] & 0xffffu, p.a.f16 != 0);
                    v[8 * c + 2 * k + 1] = from16(x[k] >> 16, p.a.f16 != 0);
                }
            }
#pragma unroll
            for (int l = 0; (1 << l) < D; ++l)
                if (l < p.a.log2b) {
#pragma unroll
                    for (int i = 0; i < D; ++i)
                        if ((i & (1 << l)) == 0) {
                            const float x = v[i], y = v[i + (1 << l)];
                            v[i] = x + y;
                            v[i + (1 << l)] = x - y;
                        }
                }
#pragma unroll
            for (int i = 0; i < D; ++i) most = fmaxf(most, fabsf(v[i]));
            const int e = min(max((int)(__float_as_uint(most) >> 23), 1), 253);
            float down = __uint_as_float((uint32_t)(254 - e) << 23);
            factor = __uint_as_float((uint32_t)e << 23) * fabsf(p.a.scale);
            if (p.a.scale < 0.0f) down = -down;                        // (a page's largest logit is that of its largest S)
            const uint32_t to = base + (uint32_t)t * K::tile + (uint32_t)thread * 128u;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                uint4 w;
                w.x = half2_of(v[8 * c] * down, v[8 * c + 1] * down);
                w.y = half2_of(v[8 * c + 2] * down, v[8 * c + 3] * down);
                w.z = half2_of(v[8 * c + 4] * down, v[8 * c + 5] * down);
                w.w = half2_of(v[8 * c + 6] * down, v[8 * c + 7] * down);
                sts128(to + (uint32_t)(c / 8) * K::half + (uint32_t)(((c ^ thread) & 7) * 16), w);
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full + 8u * (uint32_t)t);

            const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_at = tmem + (uint32_t)t * 128u + lanes, o_at = tmem + K::o_column + (uint32_t)t * 128u + lanes;
            // rows of this warp: all keys of a tile from `seen_low` on (or of the first tokens) up to seen_high are seen by all of them
            const int row_first = it.row0 + t * 128 + (warp & 3) * 32, row_last = it.row0 + it.rows - 1;
            const int low_position = it.first + min(row_first, row_last) / p.a.group, high_position = it.first + min(row_first + 31, row_last) / p.a.group;
            float m = -INFINITY, l = 0.0f;
            bool ok = true;
            for (int j = 0; j < tiles; ++j) {
                const int key = key_of(tile0 + j);
                if (!mbar_wait_warp(steps_full + 8u * (uint32_t)(j & 7), (uint32_t)(j >> 3) & 1u) || !mbar_wait_warp(s_full + 8u * (uint32_t)t, (uint32_t)j & 1u)) {
                    ok = false;
                    break;
                }
                tmem_fence_after();
                float s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_load32(s_at + 32u * c, s[c]);
                const uint32_t at = steps + (uint32_t)(j & 7) * 128u;
                constexpr int G = FINE ? 8 : 4, W = 128 / G;
                // of a page's columns: the factor of S, log2 s_v, 1 / s_v
                auto step_of = [&](int g) { return lds128(at + (uint32_t)(g * (8 / G)) * 16u); };
                loads_wait(s[0]);
                loads_there(s[1]);
                loads_there(s[2]);
                loads_there(s[3]);
                const bool whole = key + MANY_KEYS - 1 <= low_position && (p.a.window <= 0 || key > high_position - p.a.window || key + MANY_KEYS <= p.a.sinks);
                float most_x = -INFINITY;
                if (!whole) {
                    // logits now, so that what is not seen can be left out whatever its step is
                    const int last = position - key, window_low = p.a.window > 0 ? last - p.a.window : -1, sunk = p.a.sinks - key;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const uint4 w = step_of(g);
                        const float f = factor * __uint_as_float(w.x), b = __uint_as_float(w.y);
#pragma unroll
                        for (int i = g * W; i < (g + 1) * W; ++i) {
                            const float x = i <= last && (i > window_low || i < sunk) ? fmaf(s[i / 32][i % 32], f, b) : -INFINITY;
                            s[i / 32][i % 32] = x;
                            most_x = fmaxf(most_x, x);
                        }
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const uint4 w = step_of(g);
                        float top = -INFINITY;
#pragma unroll
                        for (int i = g * W; i < (g + 1) * W; i += 2) top = max_of3(top, s[i / 32][i % 32], s[i / 32][i % 32 + 1]);
                        most_x = fmaxf(most_x, fmaf(top, factor * __uint_as_float(w.x), __uint_as_float(w.y)));
                    }
                }
                if (__any_sync(0xffffffffu, most_x - m > 8.0f)) {
                    const float next = fmaxf(m, most_x), alpha = next == -INFINITY ? 1.0f : exp2_of(m - next);
                    m = next;
                    l *= alpha;
                    if (j > 0) {
                        if (!mbar_wait_warp(o_full + 8u * (uint32_t)t, (uint32_t)(j - 1) & 1u)) {
                            ok = false;
                            break;
                        }
                        tmem_fence_after();
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            float o[32];
                            tmem_load32(o_at + 32u * c, o);
                            loads_wait(o);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] *= alpha;
                            tmem_store32(o_at + 32u * c, o);
                        }
                    }
                }
                const float reference = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int g = c * G / 4; g < (c + 1) * G / 4; ++g) {
                        const uint4 step = step_of(g);
                        const float f = whole ? factor * __uint_as_float(step.x) : 1.0f, b = (whole ? __uint_as_float(step.y) : 0.0f) - reference;
                        const Pair ff = pair_of(f, f), bb = pair_of(b, b);
                        Pair sum = pair_of(0.0f, 0.0f);
#pragma unroll
                        for (int i = 0; i < W; i += 2) {
                            const int k = (g * W + i) % 32;
                            float x, y;
                            pair_split(pair_fma(pair_of(s[c][k], s[c][k + 1]), ff, bb), x, y);
                            x = exp2_of(x);
                            y = exp2_of(y);
                            sum = pair_add(sum, pair_of(x, y));
                            w[k / 2] = half2_of(x, y);
                        }
                        float x, y;
                        pair_split(sum, x, y);
                        x += y;
                        if (x != 0.0f) l = fmaf(x, __uint_as_float(step.z), l);        // (a step that is not finite stays with the rows that see it)
                    }
                    tmem_store16(s_at + 16u * c, w);
                }
                tmem_store_wait();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8u * (uint32_t)t);
            }
            if (ok && tiles > 0 && !mbar_wait_warp(o_full + 8u * (uint32_t)t, (uint32_t)(tiles - 1) & 1u)) ok = false;
            if (!ok) {
                give_up();
            } else {
                tmem_fence_after();
                const float r = p.split > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
                float *const to_part = p.split > 1 ? many_part<D>(p, it.number, part) + (size_t)row * D : nullptr;
                const size_t to_out = ((size_t)(it.begin + token) * all_heads + of_row) * D;
                if (p.split > 1) {
                    float *const ends = many_part<D>(p, it.number, part) + MANY_ROWS * D;
                    ends[row] = m;
                    ends[MANY_ROWS + row] = l;
                }
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    float o[32];
                    if (tiles > 0) {
                        tmem_load32(o_at + 32u * c, o);
                        loads_wait(o);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0.0f;
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] *= r;
                    if (!there) continue;
                    if (p.split > 1) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4 *>(to_part + 32 * c + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    } else if (p.a.out_type == OUT_F32) {
                        float *const to_f = static_cast<float *>(p.a.out) + to_out + 32 * c;
#pragma unroll
                        for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4 *>(to_f + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    } else {
                        const bool f16 = p.a.out_type == OUT_F16;
                        uint16_t *const to_h = static_cast<uint16_t *>(p.a.out) + to_out + 32 * c;
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4 *>(to_h + i) = make_uint4(pack16(o[i], o[i + 1], f16), pack16(o[i + 2], o[i + 3], f16), pack16(o[i + 4], o[i + 5], f16),
                                                                              pack16(o[i + 6], o[i + 7], f16));
                    }
                }
            }
        }
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // codes of a tile to fp16: a thread has 16 channels of every (128 / rows a pass)-th key
        constexpr int chunks = D / 16, passes = chunks, rows_a_pass = 128 / chunks;      // (128 threads, 128 * chunks pieces)
        const int thread = tid - 256, chunk = thread % chunks, row0 = thread / chunks;
        const int32_t *const table = p.a.q.pages + (size_t)it.sequence * (size_t)p.a.q.width;
        const int log2page = p.a.q.page, group = lane & 7;
        // of a tile, lanes 0 .. 7: the pages of its eight groups of 16 keys
        auto pages_of = [&](int j) {
            const int key = key_of(tile0 + j) + 16 * group;
            return j < tiles ? min(max(__ldg(table + min(key >> log2page, p.a.q.width - 1)), 0), p.a.q.n_pages - 1) : 0;
        };
        uint4 raw[passes];
        auto load = [&](int i, int j, int32_t pages, const int8_t *codes) {
            if (j >= tiles) return;
            const int key0 = key_of(tile0 + j), row = row0 + i * rows_a_pass, page = __shfl_sync(0xffffffffu, pages, (row >> 4) & 7);
            const size_t at = ((((size_t)page * (size_t)p.a.heads + (size_t)it.head) << log2page) + (size_t)((key0 + row) & ((1 << log2page) - 1))) * D + (size_t)(chunk * 16);
            raw[i] = __ldg(reinterpret_cast<const uint4 *>(codes + at));
        };
        int32_t pages = pages_of(0);
#pragma unroll
        for (int i = 0; i < passes; ++i) load(i, 0, pages, p.a.k_codes);
        bool ok = true;
        uint32_t n = 0;                                                // pieces of the ring so far
        for (int j = 0; j < tiles && ok; ++j) {
            const int32_t next = pages_of(j + 1);
            if (warp == 8) {
                const size_t block = (size_t)pages * (size_t)p.a.heads + (size_t)it.head;
                const float ks = __ldg(p.a.k_steps + block), vs = __ldg(p.a.v_steps + block);
                const bool none = vs < 0x1p-64f;
                if (lane < 8)
                    sts128(steps + (uint32_t)(j & 7) * 128u + (uint32_t)lane * 16u,
                           make_uint4(__float_as_uint(ks), __float_as_uint(none ? -64.0f : log2_of(vs)), __float_as_uint(none ? 0x1p64f : 1.0f / vs), 0u));
            }
#pragma unroll
            for (int kind = 0; kind < 2; ++kind, ++n) {
                const uint32_t s = n % K::stages, to = base + K::off_ring + s * K::tile;
                if (n >= K::stages && !mbar_wait_warp(empty + 8u * s, (n / K::stages - 1u) & 1u)) {
                    ok = false;
                    break;
                }
                if (kind == 0 && warp == 8) {
                    // (at most five tiles ahead of the rows' warps, as many as the ring holds)
                    __syncwarp();
                    if (lane == 0) mbar_arrive(steps_full + 8u * (uint32_t)(j & 7));
                }
#pragma unroll
                for (int i = 0; i < passes; ++i) {
                    const uint32_t row = (uint32_t)(row0 + i * rows_a_pass);
                    const uint32_t x[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                    uint4 o[2];
                    uint32_t *const w = reinterpret_cast<uint32_t *>(o);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        w[2 * k] = codes_f16(__byte_perm(x[k], 0u, 0x4140));             // codes 0 and 1, 2 and 3
                        w[2 * k + 1] = codes_f16(__byte_perm(x[k], 0u, 0x4342));
                    }
                    if (kind == 0) load(i, j, pages, p.a.v_codes); else load(i, j + 1, next, p.a.k_codes);
                    // (the second half's threads write their second 16 bytes first: eight threads then meet no conflict)
                    const uint32_t at = to + (uint32_t)(chunk / 4) * K::half + row * 128u, c = 2u * (uint32_t)(chunk & 3), flip = (uint32_t)(chunk / 4) & 1u;
                    sts128(at + (((c + flip) ^ row) & 7u) * 16u, flip ? o[1] : o[0]);
                    sts128(at + (((c + 1u - flip) ^ row) & 7u) * 16u, flip ? o[0] : o[1]);
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(full + 8u * s);
            }
            pages = next;
        }
        if (!ok) give_up();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 12 && lane == 0 && tiles > 0) {
            const uint32_t qk = f16_desc(128, 128, false), pv = f16_desc(128, D, true);
            bool ok = true;
            uint32_t n = 0;
            auto logits = [&](uint32_t t, uint32_t s) {
                const uint32_t a = rows_operand(base + t * K::tile), b = rows_operand(base + K::off_ring + s * K::tile);
#pragma unroll
                for (uint32_t k = 0; k < D / 16; ++k) {
                    const uint32_t at = (k / 4u) * (K::half >> 4) + (k % 4u) * 2u;
                    product_f16(tmem + t * 128u, a + at, b + at, qk, k > 0);
                }
                commit(s_full + 8u * t);
            };
            auto outputs = [&](uint32_t t, uint32_t s, bool more) {
                const uint32_t b = keys_operand<D>(base + K::off_ring + s * K::tile);
#pragma unroll
                for (uint32_t k = 0; k < MANY_KEYS / 16; ++k) product_f16_tmem(tmem + K::o_column + t * 128u, tmem + t * 128u + 8u * k, b + k * 128u, pv, more || k > 0);
                commit(o_full + 8u * t);
            };
            auto wait_for = [&](uint32_t bar, uint32_t parity) {
                if (ok && !mbar_wait(bar, parity)) ok = false;
                tmem_fence_after();
                return ok;
            };
            auto piece = [&](uint32_t i) { return wait_for(full + 8u * (i % K::stages), (i / K::stages) & 1u); };
            if (wait_for(q_full, 0) && (!two || wait_for(q_full + 8u, 0)) && piece(0)) {
                logits(0, 0);
                if (two) logits(1, 0);
                commit(empty);
                n = 1;
                for (int j = 0; j < tiles && ok; ++j, n += 2) {
                    const bool more = j + 1 < tiles;
                    const uint32_t sv = n % K::stages, sk = (n + 1) % K::stages;
                    if (!piece(n) || !wait_for(p_full, (uint32_t)j & 1u)) break;
                    outputs(0, sv, j > 0);
                    if (more) {
                        if (!piece(n + 1)) break;
                        logits(0, sk);
                    }
                    if (two) {
                        if (!wait_for(p_full + 8u, (uint32_t)j & 1u)) break;
                        outputs(1, sv, j > 0);
                        if (more) logits(1, sk);
                    }
                    commit(empty + 8u * sv);
                    if (more) commit(empty + 8u * sk);
                }
            }
            if (!ok) give_up();
            // nothing is in flight when the CTA ends
            commit(end);
            (void)mbar_wait(end, 0);
        }
        __syncwarp();
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(K::columns) : "memory");
}

// Rows whose keys were split: blockIdx.x is an item, blockIdx.y a quarter of its rows.
template <int D>
__global__ void __launch_bounds__(THREADS) many_join_kernel(const __grid_constant__ ManyParams p)
{
    griddep_wait();
    griddep_launch();
    const ManyItem it = many_item<THREADS>(p.a, (int)blockIdx.x);
    const int row_begin = (int)blockIdx.y * (MANY_ROWS / 4), row_end = min(row_begin + MANY_ROWS / 4, it.rows);
    for (int k = (int)threadIdx.x; k < (row_end - row_begin) * (D / 4); k += THREADS) {
        const int row = row_begin + k / (D / 4), channel = k % (D / 4) * 4;
        float m = -INFINITY, l = 0.0f;
        for (int c = 0; c < p.split; ++c) m = fmaxf(m, many_part<D>(p, it.number, c)[MANY_ROWS * D + row]);
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int c = 0; c < p.split; ++c) {
            const float *const from = many_part<D>(p, it.number, c);
            const float mc = from[MANY_ROWS * D + row], a = mc == -INFINITY ? (m == -INFINITY ? 1.0f : 0.0f) : exp2_of(mc - m);
            const float4 x = *reinterpret_cast<const float4 *>(from + (size_t)row * D + channel);
            l = fmaf(a, from[MANY_ROWS * D + MANY_ROWS + row], l);
            v.x = fmaf(a, x.x, v.x); v.y = fmaf(a, x.y, v.y); v.z = fmaf(a, x.z, v.z); v.w = fmaf(a, x.w, v.w);
        }
        const float r = l == 0.0f ? 0.0f : 1.0f / l;
        const int token = (it.row0 + row) / p.a.group, h = it.row0 + row - token * p.a.group;
        store_out4<D>(p.a, ((size_t)(it.begin + token) * (size_t)(p.a.heads * p.a.group) + (size_t)(it.head * p.a.group + h)) * D + (size_t)channel,
                      make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
    }
}

}  // namespace perq_kv
