// Rows of bf16 to 8-bit codes with one scale each: gather, block rotation, code = rne(127 u / max |u|), and sums of codes.
//
// u = H x' is the unnormalised rotation (+-1 sums), so s = max|u| / (127 sqrt b).  A lane holds 16 adjacent channels of its row: the first
// four butterfly stages are lane-local, up to five more (b = 512) exchange with lanes of the same warp.  Bound by memory: 3 bytes
// an element, each read and written once; the next row's loads are in flight while a row is rotated.
//
// Codes are those of exact arithmetic.  A stage rounds each value to within 2^-24 of itself, an error vector of at most 2^-24 |v|, and
// the stages after it are orthogonal but for the factor that they give v itself: log2(b) of them lose |u32 - u| <= log2(b) 2^-24 |u|_2
// <= E max|u|, E = log2(b) sqrt(b) 2^-24.  The row's maximum is summed again in fp64 wherever |u32| is within 2 E of the largest, and so is
// every element whose quotient lies that close to the border between two codes (E = 0 without a rotation: then only the fp32 quotient
// is in doubt).  b = 32, gaussian values: 1.8 elements of a row of 4096.
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
    float doubt;                 // |quotient - code| from here on may round the other way
    double inv_scale;            // 1 / (127 sqrt b)
};

// What the warps of a row agree on.
struct alignas(16) RowShared {
    unsigned long long top;      // exact maximum, the bits of a positive double
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

// The butterflies of blocks of 2^log2b channels (0: none) over a warp's 512.
__device__ __forceinline__ void rotate(float (&u)[LANE_ELEMS], int log2b, int lane)
{
    if (log2b == 0) return;
#pragma unroll
    for (int h = 1; h < LANE_ELEMS; h *= 2) {
#pragma unroll
        for (int i = 0; i < LANE_ELEMS; ++i) {
            if ((i & h) == 0) {
                const float a = u[i], b = u[i + h];
                u[i] = a + b;
                u[i + h] = a - b;
            }
        }
    }
    for (int m = 1; m < 1 << (log2b - 4); m *= 2) {
        const float s = (lane & m) ? -1.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < LANE_ELEMS; ++i) {
            const float v = __shfl_xor_sync(0xffffffffu, u[i], m);
            u[i] = fmaf(s, u[i], v);                     // (s u exact: one rounding)
        }
    }
}

// In fp64, output i of this lane's block (or the channel itself without a rotation): every lane of the block calls with its 16 inputs.
__device__ __forceinline__ double exact_output(const uint32_t (&raw)[8], int i, int log2b, int lane)
{
    const int lanes = log2b > 4 ? 1 << (log2b - 4) : 1, k0 = (lane & (lanes - 1)) * LANE_ELEMS;
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < LANE_ELEMS; ++j) {
        const uint32_t w = raw[j >> 1];
        const uint32_t f = (j & 1) ? (w & 0xffff0000u) : (w << 16);
        if (log2b == 0) {
            if (j == i) s = (double)__uint_as_float(f);
        } else {
            const uint32_t sign = (uint32_t)(__popc(i & (k0 + j)) & 1) << 31;
            s += (double)__uint_as_float(f ^ sign);
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
    for (; t < p.T; t += step) {
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
        if (w == 0 && lane == 0) row->top = 0ull;
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
        float u[PIECES][LANE_ELEMS], top = 0.0f;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[k][2 * i] = __uint_as_float(raw[k][i] << 16);
                u[k][2 * i + 1] = __uint_as_float(raw[k][i] & 0xffff0000u);
            }
            rotate(u[k], p.log2b, lane);
#pragma unroll
            for (int i = 0; i < LANE_ELEMS; ++i) top = fmaxf(top, fabsf(u[k][i]));
        }
#pragma unroll
        for (int m = 16; m >= 1; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
        float all = top;
        if (p.warps > 1) {
            if (lane == 0) row->part[w] = top;
            row_barrier(bar, p.warps);
            all = lane < p.warps ? row->part[lane] : 0.0f;
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, m));
        } else {
            __syncwarp();                                // (row->top is cleared)
        }
        // the exact maximum
        const float near = all * p.near_max;
        if (top >= near && all > 0.0f) {
            double best = 0.0;
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                uint32_t mask = 0u;
#pragma unroll
                for (int i = 0; i < LANE_ELEMS; ++i) mask |= (fabsf(u[k][i]) >= near ? 1u : 0u) << i;
                each_exact(mask, raw[k], p.log2b, lane, [&](int, double v) { best = fmax(best, fabs(v)); });
            }
            if (best > 0.0) atomicMax(&row->top, (unsigned long long)__double_as_longlong(best));
        }
        row_barrier(bar, p.warps);
        const double exact = __longlong_as_double((long long)row->top);
        if (w == 0 && lane == 0) p.scales[t] = (float)(exact * p.inv_scale);
        // |quotients| <= 127 (1 + 2 E).  Rows so small that 127 / max overflows are settled element by element.
        const float r = 127.0f / all;
        const bool tiny = !(all > 0x1p-120f);
        const float ratio = tiny ? 0.0f : r;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            uint32_t code[4];
            float off = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float g[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    g[i] = fmaf(u[k][4 * c + i], ratio, 12582912.0f);              // 1.5 2^23: the low byte is the code
                    off = fmaxf(off, fabsf(fmaf(u[k][4 * c + i], ratio, 12582912.0f - g[i])));
                }
                const uint32_t lo = __byte_perm(__float_as_uint(g[0]), __float_as_uint(g[1]), 0x0040);
                const uint32_t hi = __byte_perm(__float_as_uint(g[2]), __float_as_uint(g[3]), 0x0040);
                code[c] = __byte_perm(lo, hi, 0x5410);
            }
            const bool some = off >= p.doubt || (tiny && all > 0.0f);
            if (__any_sync(0xffffffffu, some)) {
                uint32_t mask = 0u;
                if (some) {
#pragma unroll
                    for (int i = 0; i < LANE_ELEMS; ++i) {
                        const float q = fmaf(u[k][i], ratio, 12582912.0f) - 12582912.0f;
                        mask |= (tiny || fabsf(fmaf(u[k][i], ratio, -q)) >= p.doubt ? 1u : 0u) << i;
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
        // (part and top are written again by the next row: after its first barrier that all have passed, or here)
        row_barrier(bar, p.warps);
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
