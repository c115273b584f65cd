// Rows of bf16 to 8-bit codes with one scale each: gather, block rotation, code = rne(127 u / max |u|), and sums of codes.
//
// u = H x' is the unnormalised rotation (+-1 sums), so s = max|u| / (127 sqrt b).  A lane holds 16 adjacent channels of its row: the first
// four butterfly stages are lane-local, up to five more (b = 512) exchange with lanes of the same warp.  Bound by memory: 3 bytes
// an element, each read and written once; the next row's loads are in flight while a row is rotated.
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

struct Params {
    const uint16_t *x;
    const int32_t *perm;
    int8_t *codes;
    float *scales;
    long long T;
    int32_t d, log2b;
    int32_t warps;               // to a row
    int32_t rows;                // of a CTA at a time
    float near_max;              // 1 - 2 E, and a little: |u32| from here on may be the maximum
    float doubt;                 // a block's largest quotient times this: how far its quotients may be off
    double inv_scale;            // 1 / (127 sqrt b)
};

// What the warps of a row agree on.
struct alignas(16) RowShared {
    unsigned long long top[2];   // exact maximum, the bits of a positive double; rows take turns
    float part[32];              // warps' maxima
};

__device__ __forceinline__ void row_barrier(int id, int warps)
{
    if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory");
}

__device__ __forceinline__ void load_piece(uint32_t (&raw)[8], const uint16_t *src, bool valid)
{
    if (valid) {
        const uint4 a = __ldg(reinterpret_cast<const uint4 *>(src)), b = __ldg(reinterpret_cast<const uint4 *>(src) + 1);
        raw[0] = a.x; raw[1] = a.y; raw[2] = a.z; raw[3] = a.w;
        raw[4] = b.x; raw[5] = b.y; raw[6] = b.z; raw[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i] = 0u;
    }
}

// Two values that are added and multiplied at once.
struct __align__(8) Pair {
    float x, y;
};
__device__ __forceinline__ Pair pair_add(Pair a, Pair b)
{
    Pair r;
    asm("{ .reg .b64 p, q, s; mov.b64 p, {%2, %3}; mov.b64 q, {%4, %5}; add.rn.f32x2 s, p, q; mov.b64 {%0, %1}, s; }"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ Pair pair_fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("{ .reg .b64 p, q, s, t; mov.b64 p, {%2, %3}; mov.b64 q, {%4, %5}; mov.b64 s, {%6, %7}; fma.rn.f32x2 t, p, q, s; mov.b64 {%0, %1}, t; }"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float max3(float m, Pair v) { return fmaxf(fmaxf(m, fabsf(v.x)), fabsf(v.y)); }
__device__ __forceinline__ float warp_max(float v)       // (not negative)
{
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}

// The butterflies of blocks of 2^log2b channels (0: none) over a warp's 512.
__device__ __forceinline__ void rotate(Pair (&u)[LANE_ELEMS / 2], int log2b, int lane)
{
    if (log2b == 0) return;
    const Pair neg = {-1.0f, -1.0f};
#pragma unroll
    for (int i = 0; i < LANE_ELEMS / 2; ++i) {
        const float a = u[i].x, b = u[i].y;
        u[i].x = a + b;
        u[i].y = a - b;
    }
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
    for (int m = 1; m < 1 << (log2b - 4); m *= 2) {
        const float s = (lane & m) ? -1.0f : 1.0f;
        const Pair ss = {s, s};
#pragma unroll
        for (int i = 0; i < LANE_ELEMS / 2; ++i) {
            const Pair v = {__shfl_xor_sync(0xffffffffu, u[i].x, m), __shfl_xor_sync(0xffffffffu, u[i].y, m)};
            u[i] = pair_fma(ss, u[i], v);                // (s u exact: one rounding)
        }
    }
}

// In fp64, output i of this lane's block (or the channel itself without a rotation): every lane of the block calls with its 16 inputs.
__device__ __forceinline__ double exact_output(const uint32_t (&raw)[8], int i, int log2b, int lane)
{
    const int lanes = log2b > 4 ? 1 << (log2b - 4) : 1, k0 = (lane & (lanes - 1)) * LANE_ELEMS;
    double s = 0.0;
    // bit j: the sign of input k0 + j, the parity of i & (k0 + j)
    const uint32_t signs = ((i & 1) ? 0xaaaau : 0u) ^ ((i & 2) ? 0xccccu : 0u) ^ ((i & 4) ? 0xf0f0u : 0u) ^ ((i & 8) ? 0xff00u : 0u) ^ ((__popc(i & k0) & 1) ? 0xffffu : 0u);
#pragma unroll
    for (int j = 0; j < LANE_ELEMS; ++j) {
        const uint32_t w = raw[j >> 1];
        const uint32_t f = (j & 1) ? (w & 0xffff0000u) : (w << 16);
        if (log2b == 0) {
            if (j == i) s = (double)__uint_as_float(f);
        } else {
            s += (double)__uint_as_float(f ^ ((signs << (31 - j)) & 0x80000000u));
        }
    }
    for (int m = 1; m < lanes; m *= 2) s += __shfl_xor_sync(0xffffffffu, s, m);
    return s;
}

// Calls f(element, exact output) for each element in `mask` of every lane; the lanes of a block take them one after another.
template <typename F>
__device__ __forceinline__ void each_exact(uint32_t mask, const uint32_t (&raw)[8], int log2b, int lane, F f)
{
    const int lanes = log2b > 4 ? 1 << (log2b - 4) : 1;
    const uint32_t block = (lanes == 32 ? 0xffffffffu : (1u << lanes) - 1u) << (lane & ~(lanes - 1));
    while (true) {
        const uint32_t any = __ballot_sync(0xffffffffu, mask != 0u);
        if (any == 0u) return;
        const uint32_t mine = any & block;
        const int lead = mine ? __ffs((int)mine) - 1 : lane, e = mask ? __ffs((int)mask) - 1 : 0;
        const int i = __shfl_sync(0xffffffffu, (lane & (lanes - 1)) * LANE_ELEMS + e, lead);
        const double u = exact_output(raw, i, log2b, lane);
        if (mask != 0u && lane == lead) {
            f(e, u);
            mask &= mask - 1u;
        }
    }
}

// PIECES of 16 channels to a lane, 512 to a warp; PERM: the row is gathered through shared memory.
template <int PIECES, bool PERM>
__global__ void __launch_bounds__(MAX_THREADS, 1) quant8_kernel(const Params p)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int group = warp / p.warps, w = warp - group * p.warps, bar = 1 + group;
    RowShared *const row = reinterpret_cast<RowShared *>(smem) + group;
    uint16_t *const staged = reinterpret_cast<uint16_t *>(smem + sizeof(RowShared) * (size_t)p.rows) + (size_t)group * (size_t)p.d;
    int at[PIECES];
    bool valid[PIECES];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        at[k] = (k * p.warps + w) * WARP_ELEMS + lane * LANE_ELEMS;
        valid[k] = at[k] < p.d;
    }
    griddep_wait();
    griddep_launch();
    uint32_t from[PIECES][8];                            // PERM: pairs of channels
    if (PERM) {
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                from[k][i] = 0u;
                if (valid[k]) {
                    const uint32_t a = (uint32_t)min(max(__ldg(p.perm + at[k] + 2 * i), 0), p.d - 1);
                    const uint32_t b = (uint32_t)min(max(__ldg(p.perm + at[k] + 2 * i + 1), 0), p.d - 1);
                    from[k][i] = a | (b << 16);
                }
            }
    }
    const long long step = (long long)gridDim.x * p.rows;
    long long t = (long long)blockIdx.x * p.rows + group;
    uint32_t next[PIECES][8];
    if (t < p.T) {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) load_piece(next[k], p.x + (size_t)t * (size_t)p.d + at[k], valid[k]);
    }
    if (w == 0 && lane == 0) row->top[0] = 0ull;
    const int block_lanes = p.log2b > 4 ? 1 << (p.log2b - 4) : 1;
    int turn = 0;
    for (; t < p.T; t += step, turn ^= 1) {
        uint32_t raw[PIECES][8];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (PERM && valid[k]) {
                uint4 *const dst = reinterpret_cast<uint4 *>(staged + at[k]);
                dst[0] = make_uint4(next[k][0], next[k][1], next[k][2], next[k][3]);
                dst[1] = make_uint4(next[k][4], next[k][5], next[k][6], next[k][7]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[k][i] = next[k][i];
        }
        if (PERM) {
            row_barrier(bar, p.warps);
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    raw[k][i] = valid[k] ? (uint32_t)staged[from[k][i] & 0xffffu] | ((uint32_t)staged[from[k][i] >> 16] << 16) : 0u;
        }
        if (t + step < p.T) {
#pragma unroll
            for (int k = 0; k < PIECES; ++k) load_piece(next[k], p.x + (size_t)(t + step) * (size_t)p.d + at[k], valid[k]);
        }
        Pair u[PIECES][LANE_ELEMS / 2];
        float block[PIECES], top = 0.0f;                 // largest of the lane's block, of the warp
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) u[k][i] = {__uint_as_float(raw[k][i] << 16), __uint_as_float(raw[k][i] & 0xffff0000u)};
            rotate(u[k], p.log2b, lane);
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < LANE_ELEMS / 2; ++i) m = max3(m, u[k][i]);
            for (int l = 1; l < block_lanes; l *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, l));
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
            __syncwarp();                                // (row->top is cleared)
        }
        // (the other turn's maximum: every warp is past the row that had it)
        if (w == 0 && lane == 0) row->top[turn ^ 1] = 0ull;
        const float near = all * p.near_max;
        if (top >= near && all > 0.0f) {
            double best = 0.0;
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                uint32_t mask = 0u;
                if (block[k] >= near) {
#pragma unroll
                    for (int i = 0; i < LANE_ELEMS / 2; ++i) mask |= (fabsf(u[k][i].x) >= near ? 1u << (2 * i) : 0u) | (fabsf(u[k][i].y) >= near ? 2u << (2 * i) : 0u);
                }
                each_exact(mask, raw[k], p.log2b, lane, [&](int, double v) { best = fmax(best, fabs(v)); });
            }
            if (best > 0.0) atomicMax(&row->top[turn], (unsigned long long)__double_as_longlong(best));
        }
        row_barrier(bar, p.warps);
        const double exact = __longlong_as_double((long long)*reinterpret_cast<volatile unsigned long long *>(&row->top[turn]));
        if (w == 0 && lane == 0) p.scales[t] = (float)(exact * p.inv_scale);
        // Rows so small that 127 / max overflows are settled element by element.
        const bool tiny = !(all > 0x1p-120f);
        const float ratio = tiny ? 0.0f : 127.0f / all;
        const Pair rr = {ratio, ratio}, magic = {12582912.0f, 12582912.0f}, neg = {-1.0f, -1.0f};     // 1.5 2^23: the low byte of the sum is the code
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            uint32_t code[4];
            float off = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const Pair g = pair_fma(u[k][2 * c], rr, magic), h = pair_fma(u[k][2 * c + 1], rr, magic);
                off = max3(off, pair_fma(u[k][2 * c], rr, pair_fma(g, neg, magic)));
                off = max3(off, pair_fma(u[k][2 * c + 1], rr, pair_fma(h, neg, magic)));
                const uint32_t lo = __byte_perm(__float_as_uint(g.x), __float_as_uint(g.y), 0x0040);
                const uint32_t hi = __byte_perm(__float_as_uint(h.x), __float_as_uint(h.y), 0x0040);
                code[c] = __byte_perm(lo, hi, 0x5410);
            }
            const float doubt = 0.5f - 0x1p-23f - block[k] * ratio * p.doubt;
            const bool some = off >= doubt || (tiny && all > 0.0f);
            if (__any_sync(0xffffffffu, some)) {
                uint32_t mask = 0u;
                if (some) {
#pragma unroll
                    for (int i = 0; i < LANE_ELEMS / 2; ++i) {
                        const Pair g = pair_fma(pair_fma(u[k][i], rr, magic), neg, magic), q = pair_fma(u[k][i], rr, g);
                        mask |= (tiny || fabsf(q.x) >= doubt ? 1u << (2 * i) : 0u) | (tiny || fabsf(q.y) >= doubt ? 2u << (2 * i) : 0u);
                    }
                }
                each_exact(mask, raw[k], p.log2b, lane, [&](int e, double v) {
                    const uint32_t q = (uint32_t)__double2int_rn(127.0 * v / exact) & 0xffu;
                    const uint32_t keep = ~(0xffu << ((e & 3) * 8)), put = q << ((e & 3) * 8);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if ((e >> 2) == c) code[c] = (code[c] & keep) | put;
                });
            }
            if (valid[k]) *reinterpret_cast<uint4 *>(p.codes + (size_t)t * (size_t)p.d + at[k]) = make_uint4(code[0], code[1], code[2], code[3]);
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
