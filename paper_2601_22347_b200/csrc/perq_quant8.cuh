// Rows of bf16 to 8-bit codes with one scale each: gather, block rotation, code = rne(127 u / max |u|), and sums of codes.
//
// u = H x' is the unnormalised rotation (+-1 sums), so s = max|u| / (127 sqrt b).  A lane holds 16 adjacent channels of its row: the first
// four butterfly stages are lane-local, up to five more (b = 512) exchange with lanes of the same warp.  Bound by memory: 3 bytes
// an element, each read and written once; the next rows' loads are in flight while a row is rotated.
//
// Codes are those of exact arithmetic.  A stage rounds each value to within 2^-24 of itself, an error vector of at most 2^-24 |v|, and
// the stages after it are orthogonal but for the factor that they give v itself: log2(b) of them lose |u32 - u| <= log2(b) 2^-24 |u|_2
// <= E max|u| over the block, E = log2(b) sqrt(b) 2^-24.  The row's maximum is summed again in fp64 wherever |u32| is within 2 E of the
// largest.  A quotient q = 127 u / max is off by 127 E (block's max) / max for u, and by |q| times E for the maximum and 3 roundings: by
// the block's largest quotient times 2 E + 6 2^-24 in all.  Elements that lie that close to the border between two codes are summed
// again in fp64 (b = 32, gaussian values: 1.8 of a row of 4096; with outliers, next to none outside their blocks).
#pragma once

#include "perq_mm_ptx.cuh"

namespace perq_q8 {

using perq_mm::griddep_launch;
using perq_mm::griddep_wait;

constexpr int LANE_ELEMS = 16;                // channels of a lane in one piece of a row
constexpr int WARP_ELEMS = 32 * LANE_ELEMS;
constexpr int MAX_LOG2B = 9;
constexpr int MAX_THREADS = 1024;
constexpr int STAGES = 3;                     // rows of a group of warps in shared memory: one is read, the others are on their way

struct Params {
    const uint16_t *x;
    const int32_t *perm;
    int8_t *codes;
    float *scales;
    long long T;
    int32_t d;
    int32_t warps;               // to a row
    int32_t rows;                // of a CTA at a time
    float near_max;              // 1 - 2 E, and a little: |u32| from here on may be the maximum
    float doubt;                 // a block's largest quotient times this: how far its quotients may be off
    double inv_scale;            // 1 / (127 sqrt b)
};

// What the warps of a row agree on.
struct alignas(128) RowShared {
    unsigned long long top[2];   // exact maximum, the bits of a positive double; rows take turns
    unsigned long long full[4];  // barriers of the stages
    float part[32];              // warps' maxima
};

__device__ __forceinline__ void row_barrier(int id, int warps)
{
    if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory");
}

// Two fp32 values in one register pair, added and multiplied at once.
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair_of(float x, float y)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void split(Pair p, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p)); }
__device__ __forceinline__ Pair pair_add(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair pair_fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float max3(float m, Pair v)
{
    float x, y, r;
    split(v, x, y);
    asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float warp_max(float v)       // (not negative)
{
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}

// The butterflies of blocks of 2^LOG2B channels (0: none) over a warp's 512.
template <int LOG2B>
__device__ __forceinline__ void rotate(Pair (&u)[LANE_ELEMS / 2], const uint32_t (&raw)[8], int lane)
{
    const Pair neg = pair_of(-1.0f, -1.0f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = __uint_as_float(raw[i] << 16), b = __uint_as_float(raw[i] & 0xffff0000u);
        u[i] = LOG2B == 0 ? pair_of(a, b) : pair_of(a + b, a - b);
    }
    if (LOG2B == 0) return;
#pragma unroll
    for (int h = 1; h < LANE_ELEMS / 2; h *= 2) {
#pragma unroll
        for (int i = 0; i < LANE_ELEMS / 2; ++i) {
            if ((i & h) == 0) {
                const Pair a = u[i], b = u[i + h];
                u[i] = pair_add(a, b);
                u[i + h] = pair_fma(b, neg, a);
            }
        }
    }
#pragma unroll
    for (int m = 1; m < 1 << (LOG2B > 4 ? LOG2B - 4 : 0); m *= 2) {
        const float s = (lane & m) ? -1.0f : 1.0f;
        const Pair ss = pair_of(s, s);
#pragma unroll
        for (int i = 0; i < LANE_ELEMS / 2; ++i) {
            float x, y;
            split(u[i], x, y);
            u[i] = pair_fma(ss, u[i], pair_of(__shfl_xor_sync(0xffffffffu, x, m), __shfl_xor_sync(0xffffffffu, y, m)));      // (s u exact: one rounding)
        }
    }
}

// In fp64, output i of this lane's block (or the channel itself without a rotation): every lane of the block calls with its 16 inputs.
template <int LOG2B>
__device__ __forceinline__ double exact_output(const uint32_t (&raw)[8], int i, int lane)
{
    constexpr int lanes = LOG2B > 4 ? 1 << (LOG2B - 4) : 1;
    const int k0 = (lane & (lanes - 1)) * LANE_ELEMS;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};                // (four chains: half of the time here is waiting for sums)
    // bit j: the sign of input k0 + j, the parity of i & (k0 + j)
    const uint32_t signs = ((i & 1) ? 0xaaaau : 0u) ^ ((i & 2) ? 0xccccu : 0u) ^ ((i & 4) ? 0xf0f0u : 0u) ^ ((i & 8) ? 0xff00u : 0u) ^ ((__popc(i & k0) & 1) ? 0xffffu : 0u);
#pragma unroll
    for (int j = 0; j < LANE_ELEMS; ++j) {
        const uint32_t w = raw[j >> 1];
        const uint32_t f = (j & 1) ? (w & 0xffff0000u) : (w << 16);
        if (LOG2B == 0) {
            if (j == i) sum[0] = (double)__uint_as_float(f);
        } else {
            sum[j & 3] += (double)__uint_as_float(f ^ ((signs << (31 - j)) & 0x80000000u));
        }
    }
    double s = (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
    for (int m = 1; m < lanes; m *= 2) s += __shfl_xor_sync(0xffffffffu, s, m);
    return s;
}

// Calls f(element, exact output) for each element in `mask` of every lane; the lanes of a block take them one after another.
template <int LOG2B, typename F>
__device__ __forceinline__ void each_exact(uint32_t mask, const uint32_t (&raw)[8], int lane, F f)
{
    constexpr int lanes = LOG2B > 4 ? 1 << (LOG2B - 4) : 1;
    const uint32_t block = (lanes == 32 ? 0xffffffffu : (1u << lanes) - 1u) << (lane & ~(lanes - 1));
    while (true) {
        const uint32_t any = __ballot_sync(0xffffffffu, mask != 0u);
        if (any == 0u) return;
        const uint32_t mine = any & block;
        const int lead = mine ? __ffs((int)mine) - 1 : lane, e = mask ? __ffs((int)mask) - 1 : 0;
        const int i = __shfl_sync(0xffffffffu, (lane & (lanes - 1)) * LANE_ELEMS + e, lead);
        const double u = exact_output<LOG2B>(raw, i, lane);
        if (mask != 0u && lane == lead) {
            f(e, u);
            mask &= mask - 1u;
        }
    }
}

// Threads of a CTA at most, and CTAs to an SM that registers have to leave room for: rows of up to 4096, 10240 and 32768 channels.
template <int SIZE>
struct Size {
    static constexpr int threads = SIZE == 0 ? 256 : SIZE == 1 ? 640 : MAX_THREADS;
    static constexpr int ctas = SIZE == 0 ? 4 : SIZE == 1 ? 1 : 1;
};

// PIECES of 16 channels to a lane, 512 to a warp; PERM: the row is gathered from its stage.
template <int LOG2B, int SIZE, int PIECES, bool PERM>
__global__ void __launch_bounds__(Size<SIZE>::threads, Size<SIZE>::ctas) quant8_kernel(const Params p)
{
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int group = warp / p.warps, w = warp - group * p.warps, bar = 1 + group;
    const bool lead = w == 0 && lane == 0;
    RowShared *const row = reinterpret_cast<RowShared *>(smem) + group;
    const uint32_t row_bytes = (uint32_t)p.d * 2u, stages = perq_mm::smem_u32(smem) + (uint32_t)sizeof(RowShared) * (uint32_t)p.rows + (uint32_t)group * STAGES * row_bytes;
    const uint32_t full = perq_mm::smem_u32(row->full);
    if (lead) {
        for (int i = 0; i < STAGES; ++i) perq_mm::mbar_init(full + 8 * i, 1);
        perq_mm::mbar_init_fence();
        row->top[0] = 0ull;
    }
    row_barrier(bar, p.warps);
    griddep_wait();
    griddep_launch();
    const long long step = (long long)gridDim.x * p.rows;
    long long t = (long long)blockIdx.x * p.rows + group;
    const uint16_t *ahead = p.x + (size_t)t * (size_t)p.d;            // the next row to load
    long long t_ahead = t;
    uint32_t s_ahead = 0;
    auto load = [&]() {
        if (t_ahead < p.T) {
            perq_mm::mbar_expect_tx(full + 8 * s_ahead, row_bytes);
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(stages + s_ahead * row_bytes), "l"(ahead), "r"(row_bytes), "r"(full + 8 * s_ahead) : "memory");
        }
        t_ahead += step;
        ahead += (size_t)step * (size_t)p.d;
        s_ahead = s_ahead + 1 == STAGES ? 0 : s_ahead + 1;
    };
    if (lead)
        for (int i = 0; i < STAGES - 1; ++i) load();
    const int c0 = w * WARP_ELEMS + lane * LANE_ELEMS, per_piece = p.warps * WARP_ELEMS;        // this lane's first channel, and from piece to piece
    uint32_t from[PERM ? PIECES : 1][8];                 // PERM: pairs of channels
    if (PERM) {
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                from[k][i] = 0u;
                if (c0 + k * per_piece < p.d) {
                    const int32_t *const q = p.perm + c0 + k * per_piece + 2 * i;
                    from[k][i] = (uint32_t)min(max(__ldg(q), 0), p.d - 1) | ((uint32_t)min(max(__ldg(q + 1), 0), p.d - 1) << 16);
                }
            }
    }
    uint32_t s = 0, phase = 0;
    int turn = 0;
    for (; t < p.T; t += step, turn ^= 1) {
        const uint32_t stage = stages + s * row_bytes;
        if (!perq_mm::mbar_wait(full + 8 * s, phase)) atomicOr(&perq_mm::g_error, perq_mm::ERROR_ROWS);       // (its codes are wrong then)
        // this lane's 16 channels
        auto inputs = [&](int k, uint32_t (&raw)[8]) {
            const bool valid = c0 + k * per_piece < p.d;
            if (PERM) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint16_t lo = 0, hi = 0;
                    if (valid) {
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(lo) : "r"(stage + 2u * (from[PERM ? k : 0][i] & 0xffffu)));
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(hi) : "r"(stage + 2u * (from[PERM ? k : 0][i] >> 16)));
                    }
                    raw[i] = (uint32_t)lo | ((uint32_t)hi << 16);
                }
            } else {
                const uint32_t at = stage + 2u * (uint32_t)(c0 + k * per_piece);
                const uint4 a = valid ? perq_mm::lds128(at) : make_uint4(0, 0, 0, 0), b = valid ? perq_mm::lds128(at + 16) : make_uint4(0, 0, 0, 0);
                raw[0] = a.x; raw[1] = a.y; raw[2] = a.z; raw[3] = a.w;
                raw[4] = b.x; raw[5] = b.y; raw[6] = b.z; raw[7] = b.w;
            }
        };
        Pair u[PIECES][LANE_ELEMS / 2];
        float block[PIECES], top = 0.0f;                 // largest of the lane's block, of the warp
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            uint32_t raw[8];
            inputs(k, raw);
            rotate<LOG2B>(u[k], raw, lane);
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < LANE_ELEMS / 2; ++i) m = max3(m, u[k][i]);
#pragma unroll
            for (int l = 1; l < 1 << (LOG2B > 4 ? LOG2B - 4 : 0); l *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, l));
            block[k] = m;
            top = fmaxf(top, m);
        }
        top = warp_max(top);
        float all = top;
        if (p.warps > 1) {
            if (lane == 0) row->part[w] = top;
            row_barrier(bar, p.warps);
            all = warp_max(lane < p.warps ? row->part[lane] : 0.0f);
        } else {
            __syncwarp();                                // (row->top is cleared, the row before is done with)
        }
        // every warp is past the row before: its stage is loaded again, and the other turn's maximum cleared
        if (lead) {
            load();
            row->top[turn ^ 1] = 0ull;
        }
        const float near = all * p.near_max;
        if (top >= near && all > 0.0f) {
            double best = 0.0;
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                uint32_t mask = 0u, raw[8];
                if (block[k] >= near) {
#pragma unroll
                    for (int i = 0; i < LANE_ELEMS / 2; ++i) {
                        float x, y;
                        split(u[k][i], x, y);
                        mask |= (fabsf(x) >= near ? 1u << (2 * i) : 0u) | (fabsf(y) >= near ? 2u << (2 * i) : 0u);
                    }
                }
                if (!__any_sync(0xffffffffu, mask != 0u)) continue;
                inputs(k, raw);
                each_exact<LOG2B>(mask, raw, lane, [&](int, double v) { best = fmax(best, fabs(v)); });
            }
            if (best > 0.0) atomicMax(&row->top[turn], (unsigned long long)__double_as_longlong(best));
        }
        row_barrier(bar, p.warps);
        const double exact = __longlong_as_double((long long)*reinterpret_cast<volatile unsigned long long *>(&row->top[turn]));
        if (lead) p.scales[t] = (float)(exact * p.inv_scale);
        // Rows so small that 127 / max overflows are settled element by element.
        const bool tiny = !(all > 0x1p-120f);
        const float ratio = tiny ? 0.0f : 127.0f / all;
        const Pair rr = pair_of(ratio, ratio), magic = pair_of(12582912.0f, 12582912.0f), neg = pair_of(-1.0f, -1.0f);     // 1.5 2^23: the low byte of the sum is the code
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            uint32_t code[4];
            float off = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const Pair g = pair_fma(u[k][2 * c], rr, magic), h = pair_fma(u[k][2 * c + 1], rr, magic);
                off = max3(off, pair_fma(u[k][2 * c], rr, pair_fma(g, neg, magic)));
                off = max3(off, pair_fma(u[k][2 * c + 1], rr, pair_fma(h, neg, magic)));
                const uint32_t lo = __byte_perm((uint32_t)g, (uint32_t)(g >> 32), 0x0040), hi = __byte_perm((uint32_t)h, (uint32_t)(h >> 32), 0x0040);
                code[c] = __byte_perm(lo, hi, 0x5410);
            }
            const float doubt = 0.5f - 0x1p-23f - block[k] * ratio * p.doubt;
            const bool some = off >= doubt || (tiny && all > 0.0f);
            if (__any_sync(0xffffffffu, some)) {
                uint32_t mask = 0u, raw[8];
                if (some) {
#pragma unroll
                    for (int i = 0; i < LANE_ELEMS / 2; ++i) {
                        float x, y;
                        split(pair_fma(u[k][i], rr, pair_fma(pair_fma(u[k][i], rr, magic), neg, magic)), x, y);
                        mask |= (tiny || fabsf(x) >= doubt ? 1u << (2 * i) : 0u) | (tiny || fabsf(y) >= doubt ? 2u << (2 * i) : 0u);
                    }
                }
                inputs(k, raw);
                each_exact<LOG2B>(mask, raw, lane, [&](int e, double v) {
                    const uint32_t q = (uint32_t)__double2int_rn(127.0 * v / exact) & 0xffu;
                    const uint32_t keep = ~(0xffu << ((e & 3) * 8)), put = q << ((e & 3) * 8);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if ((e >> 2) == c) code[c] = (code[c] & keep) | put;
                });
            }
            if (c0 + k * per_piece < p.d)
                *reinterpret_cast<uint4 *>(p.codes + (size_t)t * (size_t)p.d + (c0 + k * per_piece)) = make_uint4(code[0], code[1], code[2], code[3]);
        }
        if (++s == STAGES) {
            s = 0;
            phase ^= 1u;
        }
    }
}

// sums[r] = sum of the codes of row r, a warp to a row.
struct SumParams {
    const void *codes;
    int32_t *sums;
    long long rows;
    int32_t chunks;              // of 16 bytes to a row
    int32_t packed;
};
__global__ void __launch_bounds__(256) code_sums_kernel(const SumParams p)
{
    griddep_wait();
    griddep_launch();
    const int lane = (int)threadIdx.x & 31;
    const long long r = (long long)blockIdx.x * 8 + ((int)threadIdx.x >> 5);
    if (r >= p.rows) return;
    const uint4 *src = reinterpret_cast<const uint4 *>(p.codes) + (size_t)r * (size_t)p.chunks;
    int32_t s = 0;
    for (int c = lane; c < p.chunks; c += 32) {
        const uint4 v = __ldg(src + c);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p.packed) {                              // 16 times the codes, in their signed places
                s = __dp4a((int)perq_mm::codes_lo(w[i]), 0x01010101, s);
                s = __dp4a((int)perq_mm::codes_hi(w[i]), 0x01010101, s);
            } else {
                s = __dp4a((int)w[i], 0x01010101, s);
            }
        }
    }
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    if (lane == 0) p.sums[r] = p.packed ? s >> 4 : s;
}

}  // namespace perq_q8
