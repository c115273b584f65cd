// Rows of bf16 to 8-bit codes with one scale each: gather, block rotation, code = rne(127 u / max |u|), and sums of codes.
//
// u = H x' is the unnormalised rotation (+-1 sums), so s = max|u| / (127 sqrt b).  A lane holds 16 adjacent channels of its row, bits 0 .. 3 of
// their index, and lanes bits 4 .. 8.  The tensor cores take bits 0, 1, 4 and 5 (mma.sync m16n8k16 on the bf16 values as they are stored: the
// fragments of its first operand and of its results are then the same lane's channels, and the second operand is a Hadamard matrix, with
// zeros where a bit is not of the block), packed fp32 butterflies bits 2 and 3, exchanges with other lanes bits 6 .. 8 of longer blocks.  Bound by
// memory: 3 bytes an element, each read and written once; the next rows' loads are in flight while a row is rotated.
//
// Codes are those of exact arithmetic.  The tensor core cuts 16 terms toward zero at 2^(e-25), e the exponent of the largest, and the sum to fp32: with
// terms no larger than the largest output of their n (Parseval), it loses at most 8 + 2 units of 2^-24 of that (12 are counted).  A butterfly adds half
// a unit of rounding and up to doubles what was lost before; no value on the way exceeds the block's largest output.  In all |u32 - u| <= E max|u| over the
// block, E = (13 b / n - 1) 2^-24 with n = min(16, b / 4).  The row's maximum is summed again in fp64 wherever |u32| is within 2 E of the largest.
// A quotient q = 127 u / max is off by 127 E (block's max) / max for u, and by |q| times E for the maximum, a unit for its reciprocal (at most 2^-23 of it, for
// maxima up to 2^126) and 3 roundings: by the block's largest quotient times 2 E + 9 2^-24 in all.  Elements that lie that close to the border between two codes are summed again in fp64
// (b = 32, gaussian values: 3 of a row of 4096; with outliers, next to none outside their blocks).
//
// Such places are rare, so a warp only notes them and settles them sixteen rows at a time, 32 / (b / 16) at once, from the inputs in global memory; it stores
// the rows' scales and mends codes.  (16384 x 4096, b = 32, 4 warps to a row, earlier: exact sums as they came up 70 us, by a warp of its own 60 .. 88 us.)  A warp
// has up to four pieces of 512 channels of a row in registers.  Rows of up to 2048 need no barrier; the warps of longer ones meet at one barrier
// a row and two for every sixteen.
//
// Measured in CUDA graphs, rows with outliers: 16384 x 4096, b = 32, 41.0 us (201 MB, 4.9 TB/s), 1531 x 9728, b = 128, permuted, 27.8 us (45 MB, 1.6 TB/s: two-byte
// gathers from shared memory and their latency at 15 warps, 5 us of settling), one row of 4096 3.7 us.  Gaussian rows, with more codes in doubt: 51 and 39 us.
#pragma once

#include "perq_mm_ptx.cuh"

namespace perq_q8 {

using perq_mm::griddep_launch;
using perq_mm::griddep_wait;

constexpr int LANE_ELEMS = 16;                // channels of a lane in one piece of a row
constexpr int WARP_ELEMS = 32 * LANE_ELEMS;
constexpr int MAX_LOG2B = 9;
constexpr int MAX_WARPS = 32;                 // of a CTA
constexpr int STAGES = 2;                     // rows of a group of warps in shared memory: one is read, the next is on its way
constexpr int BATCH = 16;                     // rows that are settled together
constexpr int NOTES = 64;                     // of a warp, batch and kind; more: everything that it has of these rows is settled

// Warps of a CTA, by the pieces that each holds (120 and 64 registers to a thread; four pieces in 96 registers: 42 -> 48 .. 70 us for 16384 x 4096).
__host__ __device__ constexpr int cta_warps(int pieces) { return pieces == 4 ? 16 : 32; }

struct Params {
    const uint16_t *x;
    const int32_t *perm;
    int8_t *codes;
    float *scales;
    long long T;
    int32_t d;
    int32_t warps;               // to a row
    int32_t rows;                // of a CTA at a time, a group of warps each
    float near_max;              // 1 - 2 E, and a little: |u32| from here on may be the maximum
    float doubt;                 // a block's largest quotient times this: how far its quotients may be off
    double inv_scale;            // 1 / (127 sqrt b)
};

struct Group {
    unsigned long long full[STAGES];                                  // barriers: the row is there
    unsigned long long top[BATCH];                                    // exact maxima, their bits
};
struct Notes {
    uint32_t count[2];
    uint32_t note[2][NOTES];                                          // row of the batch << 16 | channel: what may be the maximum, codes in doubt
};
struct alignas(128) Shared {
    Group group[MAX_WARPS];
    Notes notes[MAX_WARPS];
    float part[2][MAX_WARPS];                                         // warps' maxima; rows take turns
};
enum { NOTE_MAX = 0, NOTE_CODE = 1 };

// The warps of a row.  (Up to eight rows of a CTA have several: a barrier each, by constants, because a CTA that names one by a register holds all.)
__device__ __forceinline__ void row_barrier(int group, int warps)
{
    const int threads = warps * 32;
    __syncwarp();
    if (warps == 1) return;
    switch (group) {
    case 0: asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); break;
    case 1: asm volatile("bar.sync 2, %0;" ::"r"(threads) : "memory"); break;
    case 2: asm volatile("bar.sync 3, %0;" ::"r"(threads) : "memory"); break;
    case 3: asm volatile("bar.sync 4, %0;" ::"r"(threads) : "memory"); break;
    case 4: asm volatile("bar.sync 5, %0;" ::"r"(threads) : "memory"); break;
    case 5: asm volatile("bar.sync 6, %0;" ::"r"(threads) : "memory"); break;
    case 6: asm volatile("bar.sync 7, %0;" ::"r"(threads) : "memory"); break;
    default: asm volatile("bar.sync 8, %0;" ::"r"(threads) : "memory"); break;
    }
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
// (maxima are NaN where anything is: a row that is not finite is not lost)
__device__ __forceinline__ float max3(float m, Pair v)
{
    float x, y, r;
    split(v, x, y);
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float max2(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max(float v)       // (not negative; max2's NaN is above infinity as a number of bits)
{
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}

// Second operands: Hadamard matrices over the bits e, q, h of a channel (0; 4 and 5; 1), h of the outputs 0 and 1.  This lane's k are
// 2 (lane % 4) + {0, 1} and 8 more, its n is lane / 4; k and n are e + 2 q + 8 h and e + 2 q.
struct Hadamard {
    uint32_t k[2][2];
};
template <int LOG2B>
__device__ __forceinline__ Hadamard hadamard_operand(int lane)
{
    constexpr int inside = LOG2B == 4 ? 0 : LOG2B == 5 ? 1 : 3;      // bits of q that are the block's
    Hadamard m;
    const int q = lane & 3, n = lane >> 2, qn = n >> 1, en = n & 1;
    const bool zero = ((q ^ qn) & ~inside) != 0;
#pragma unroll
    for (int hn = 0; hn < 2; ++hn)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t w = 0u;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int odd = ((e & en) + __popc(q & qn & inside) + (h & hn)) & 1;
                w |= (odd ? 0xbf80u : 0x3f80u) << (16 * e);
            }
            m.k[hn][h] = zero ? 0u : w;
        }
    return m;
}
__device__ __forceinline__ void mma_rows(Pair &lo, Pair &hi, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    float c[4];
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    lo = pair_of(c[0], c[1]);
    hi = pair_of(c[2], c[3]);
}

// Blocks of 2^LOG2B channels (0: none) over a warp's 512.
template <int LOG2B>
__device__ __forceinline__ void rotate(Pair (&u)[LANE_ELEMS / 2], const uint32_t (&raw)[8], const Hadamard &m, int lane)
{
    if (LOG2B == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = pair_of(__uint_as_float(raw[i] << 16), __uint_as_float(raw[i] & 0xffff0000u));
        return;
    }
    const Pair neg = pair_of(-1.0f, -1.0f);
#pragma unroll
    for (int i = 0; i < 8; i += 4)
#pragma unroll
        for (int h = 0; h < 2; ++h) mma_rows(u[i + h], u[i + 2 + h], raw[i], raw[i + 2], raw[i + 1], raw[i + 3], m.k[h][0], m.k[h][1]);
#pragma unroll
    for (int h = 2; h < LANE_ELEMS / 2; h *= 2) {
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
    for (int l = 4; l < 1 << (LOG2B > 4 ? LOG2B - 4 : 0); l *= 2) {
        const float s = (lane & l) ? -1.0f : 1.0f;
        const Pair ss = pair_of(s, s);
#pragma unroll
        for (int i = 0; i < LANE_ELEMS / 2; ++i) {
            float x, y;
            split(u[i], x, y);
            u[i] = pair_fma(ss, u[i], pair_of(__shfl_xor_sync(0xffffffffu, x, l), __shfl_xor_sync(0xffffffffu, y, l)));      // (s u exact: one rounding)
        }
    }
}

// Notes the elements in `mask` of a lane whose first channel is c.
__device__ __forceinline__ void note(Notes *notes, int kind, uint32_t mask, uint32_t row, int c)
{
    while (mask != 0u) {
        const int e = __ffs((int)mask) - 1;
        mask &= mask - 1u;
        const uint32_t at = atomicAdd(&notes->count[kind], 1u);
        if (at < NOTES) notes->note[kind][at] = (row << 16) | (uint32_t)(c + e);
    }
}

// Notes what is in doubt of a lane's 16 outputs: quotients from `limit` on away from their codes (0: all; 1: none), outputs from `near` on; NaN always.  (Inside the
// unrolled loop over the pieces this was half of its instructions, and twice its time.)
__device__ __noinline__ void note_lane(Notes *notes, Pair u0, Pair u1, Pair u2, Pair u3, Pair u4, Pair u5, Pair u6, Pair u7, float ratio, float limit, float near,
                                       uint32_t row, int c)
{
    const Pair u[8] = {u0, u1, u2, u3, u4, u5, u6, u7}, rr = pair_of(ratio, ratio), magic = pair_of(12582912.0f, 12582912.0f), neg = pair_of(-1.0f, -1.0f);
    uint32_t codes = 0u, most = 0u;
#pragma unroll
    for (int j = 0; j < LANE_ELEMS / 2; ++j) {
        float x, y, v, w;
        split(u[j], v, w);
        split(pair_fma(u[j], rr, pair_fma(pair_fma(u[j], rr, magic), neg, magic)), x, y);
        codes |= (fabsf(x) < limit ? 0u : 1u << (2 * j)) | (fabsf(y) < limit ? 0u : 2u << (2 * j));
        most |= (fabsf(v) < near ? 0u : 1u << (2 * j)) | (fabsf(w) < near ? 0u : 2u << (2 * j));
    }
    note(notes, NOTE_CODE, codes, row, c);
    note(notes, NOTE_MAX, most, row, c);
}

// 16 adjacent channels of a row as the rotation takes them, raw pairs.  table: places in the row, in bytes (PERM).
template <bool PERM>
__device__ __forceinline__ void inputs16(uint32_t (&raw)[8], const uint16_t *row, uint32_t table, int k0)
{
    if (PERM) {
        const uint4 a = perq_mm::lds128(table + 2u * (uint32_t)k0), b = perq_mm::lds128(table + 2u * (uint32_t)k0 + 16u);
        const uint32_t at[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        const unsigned char *const bytes = reinterpret_cast<const unsigned char *>(row);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            raw[j] = (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(bytes + (at[j] & 0xffffu))) |
                     ((uint32_t)__ldg(reinterpret_cast<const uint16_t *>(bytes + (at[j] >> 16))) << 16);
    } else {
        const uint4 a = __ldg(reinterpret_cast<const uint4 *>(row + k0)), b = __ldg(reinterpret_cast<const uint4 *>(row + k0) + 1);
        raw[0] = a.x; raw[1] = a.y; raw[2] = a.z; raw[3] = a.w;
        raw[4] = b.x; raw[5] = b.y; raw[6] = b.z; raw[7] = b.w;
    }
}

// n noted places, 32 / (b / 16) at a time, b / 16 lanes to a place (at least one), 16 inputs each: f(row, channel, exact output) is called by the
// first of them.
template <int LOG2B, bool PERM, typename R, typename F>
__device__ __forceinline__ void settle_places(const uint32_t *places, uint32_t n, uint32_t table, int lane, R row_of, F f)
{
    constexpr int lanes = LOG2B > 4 ? 1 << (LOG2B - 4) : 1, at_once = 32 / lanes;
    for (uint32_t i0 = 0; i0 < n; i0 += at_once) {
        const uint32_t i = i0 + (uint32_t)lane / lanes;
        const bool mine = i < n;
        const uint32_t place = places[mine ? i : 0];
        const int c = (int)(place & 0xffffu), k0 = c / (lanes * LANE_ELEMS) * (lanes * LANE_ELEMS) + (lane & (lanes - 1)) * LANE_ELEMS;
        uint32_t raw[8];
        inputs16<PERM>(raw, row_of(place >> 16), table, k0);
        double sum[4] = {0.0, 0.0, 0.0, 0.0};                // (four chains: most of the time here is waiting for sums)
        // bit j: the sign of input k0 + j, the parity of c & (k0 + j) inside the block
        const uint32_t signs = ((c & 1) ? 0xaaaau : 0u) ^ ((c & 2) ? 0xccccu : 0u) ^ ((c & 4) ? 0xf0f0u : 0u) ^ ((c & 8) ? 0xff00u : 0u) ^
                               ((__popc(c & k0 & ((1 << LOG2B) - 1)) & 1) ? 0xffffu : 0u);
#pragma unroll
        for (int j = 0; j < LANE_ELEMS; ++j) {
            const uint32_t v = (j & 1) ? (raw[j >> 1] & 0xffff0000u) : (raw[j >> 1] << 16);
            if (LOG2B == 0) {
                if (j == (c & 15)) sum[0] = (double)__uint_as_float(v);
            } else {
                sum[j & 3] += (double)__uint_as_float(v ^ ((signs << (31 - j)) & 0x80000000u));
            }
        }
        double u = (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
        for (int m = 1; m < lanes; m *= 2) u += __shfl_xor_sync(0xffffffffu, u, m);
        if (mine && (lane & (lanes - 1)) == 0) f(place >> 16, c, u);
        __syncwarp();
    }
}

// n blocks in fp64, 32 / (b / 16) at a time, b / 16 lanes to a block (at least one), 16 channels each.  place_of(i): row of the batch << 16 | a channel
// of block i (past the row: none); f(row, channel, outputs) is called by every lane that has some, with its first channel.
template <int LOG2B, bool PERM, typename P, typename R, typename F>
__device__ __forceinline__ void settle_blocks(const Params &p, uint32_t n, uint32_t table, int lane, P place_of, R row_of, F f)
{
    constexpr int lanes = LOG2B > 4 ? 1 << (LOG2B - 4) : 1, at_once = 32 / lanes;
    for (uint32_t i0 = 0; i0 < n; i0 += at_once) {
        const uint32_t i = i0 + (uint32_t)lane / lanes;
        uint32_t place = i < n ? place_of(i) : 0u;
        const bool mine = i < n && (int)(place & 0xffffu) < p.d;
        if (!mine) place = 0u;
        const int c = (int)(place & 0xffffu) / (lanes * LANE_ELEMS) * (lanes * LANE_ELEMS) + (lane & (lanes - 1)) * LANE_ELEMS;
        uint32_t raw[8];
        inputs16<PERM>(raw, row_of(place >> 16), table, c);
        double v[LANE_ELEMS];
#pragma unroll
        for (int j = 0; j < LANE_ELEMS; ++j) v[j] = (double)__uint_as_float((j & 1) ? (raw[j >> 1] & 0xffff0000u) : (raw[j >> 1] << 16));
        if (LOG2B > 0) {
#pragma unroll
            for (int h = 1; h < LANE_ELEMS; h *= 2)
#pragma unroll
                for (int j = 0; j < LANE_ELEMS; ++j)
                    if ((j & h) == 0) {
                        const double a = v[j], b = v[j + h];
                        v[j] = a + b;
                        v[j + h] = a - b;
                    }
            for (int l = 1; l < lanes; l *= 2)
#pragma unroll
                for (int j = 0; j < LANE_ELEMS; ++j) {
                    const double w = __shfl_xor_sync(0xffffffffu, v[j], l);
                    v[j] = (lane & l) ? w - v[j] : v[j] + w;
                }
        }
        __syncwarp();
        if (mine) f(place >> 16, c, v);
    }
}
// The bits of |v|, which are ordered as the numbers are, with NaN above infinity.
__device__ __forceinline__ unsigned long long size_bits(double v) { return (unsigned long long)__double_as_longlong(v) & 0x7fffffffffffffffull; }
__device__ __forceinline__ unsigned long long largest(const double (&v)[LANE_ELEMS])
{
    unsigned long long m = 0ull;
#pragma unroll
    for (int j = 0; j < LANE_ELEMS; ++j) m = max(m, size_bits(v[j]));
    return m;
}
// A row's maximum that codes can be counted from; where it is not, they are 0.
__device__ __forceinline__ bool counts(double top) { return top > 0.0 && top < __longlong_as_double(0x7ff0000000000000ll); }
// rne(127 v / top) by the reciprocal, off by less than 2^-44: where that could matter, and on borders, by the quotient.
__device__ __forceinline__ void store_codes(int8_t *to, const double (&v)[LANE_ELEMS], double top)
{
    const bool some = counts(top);
    const double r = some ? 127.0 / top : 0.0;
    uint32_t code[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < LANE_ELEMS; ++j) {
        const double t = some ? v[j] * r : 0.0;
        int q = __double2int_rn(t);
        if (fabs(t - (double)q) > 0.5 - 0x1p-40) q = __double2int_rn(127.0 * v[j] / top);
        code[j >> 2] |= ((uint32_t)q & 0xffu) << (8 * (j & 3));
    }
    *reinterpret_cast<uint4 *>(to) = make_uint4(code[0], code[1], code[2], code[3]);
}


// A warp's share of the rows of a batch, row t0 + r * step the r-th.
template <int LOG2B, int PIECES, bool PERM>
__device__ __noinline__ void settle_batch(const Params &p, Group *group, Notes *notes, uint32_t table, long long t0, long long step, uint32_t rows, int g, int w, int lane)
{
    __syncwarp();
    const uint32_t n_max = *reinterpret_cast<volatile uint32_t *>(&notes->count[NOTE_MAX]), n_code = *reinterpret_cast<volatile uint32_t *>(&notes->count[NOTE_CODE]);
    const bool all = n_max > NOTES || n_code > NOTES;                 // everything that it has of all rows
    auto row_of = [&](uint32_t r) { return p.x + (size_t)(t0 + r * step) * (size_t)p.d; };
    auto raise = [&](uint32_t r, unsigned long long m) {
        if (m != 0ull) atomicMax(&group->top[r], m);
    };
    auto top_of = [&](uint32_t r) { return __longlong_as_double((long long)*reinterpret_cast<volatile unsigned long long *>(&group->top[r])); };
    constexpr uint32_t block = LOG2B > 4 ? 1u << LOG2B : LANE_ELEMS, blocks = WARP_ELEMS / block * PIECES;
    auto own = [&](uint32_t k) {
        const uint32_t r = k / blocks, j = k % blocks * block;
        return (r << 16) | ((j / WARP_ELEMS * (uint32_t)p.warps + (uint32_t)w) * WARP_ELEMS + j % WARP_ELEMS);
    };
    if (all) settle_blocks<LOG2B, PERM>(p, rows * blocks, table, lane, own, row_of, [&](uint32_t r, int, const double (&v)[LANE_ELEMS]) { raise(r, largest(v)); });
    else settle_places<LOG2B, PERM>(notes->note[NOTE_MAX], n_max, table, lane, row_of, [&](uint32_t r, int, double u) { raise(r, size_bits(u)); });
    row_barrier(g, p.warps);
    if (all)
        settle_blocks<LOG2B, PERM>(p, rows * blocks, table, lane, own, row_of, [&](uint32_t r, int c, const double (&v)[LANE_ELEMS]) {
            store_codes(p.codes + (size_t)(t0 + r * step) * (size_t)p.d + c, v, top_of(r));
        });
    else
        settle_places<LOG2B, PERM>(notes->note[NOTE_CODE], n_code, table, lane, row_of, [&](uint32_t r, int c, double u) {
            const double top = top_of(r);
            p.codes[(size_t)(t0 + r * step) * (size_t)p.d + c] = counts(top) ? (int8_t)__double2int_rn(127.0 * u / top) : (int8_t)0;
        });
    __syncwarp();
    if (w == 0 && lane < (int)rows) p.scales[t0 + lane * step] = (float)(top_of((uint32_t)lane) * p.inv_scale);
    row_barrier(g, p.warps);
    if (w == 0 && lane < BATCH) group->top[lane] = 0ull;              // (read and raised again after the next row's barrier)
    if (lane < 2) notes->count[lane] = 0u;
    __syncwarp();
}

// PIECES of 16 channels to a lane, 512 to a warp; PERM: the row is gathered from its stage.
template <int LOG2B, int PIECES, bool PERM>
__global__ void __launch_bounds__(cta_warps(PIECES) * 32, 1) quant8_kernel(const __grid_constant__ Params p)
{
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    Shared *const sh = reinterpret_cast<Shared *>(smem);
    const uint32_t row_bytes = (uint32_t)p.d * 2u, table = perq_mm::smem_u32(smem) + (uint32_t)sizeof(Shared);
    const int g = warp / p.warps, w = warp - g * p.warps;
    Group *const group = &sh->group[g];
    Notes *const notes = &sh->notes[warp];
    const uint32_t full = perq_mm::smem_u32(group->full), ring = table + (PERM ? (row_bytes + 127u) & ~127u : 0u) + (uint32_t)(g * STAGES) * row_bytes;
    if (w == 0 && lane == 0) {
        for (int i = 0; i < STAGES; ++i) perq_mm::mbar_init(full + 8 * i, 1);
        perq_mm::mbar_init_fence();
        for (int i = 0; i < BATCH; ++i) group->top[i] = 0ull;
    }
    if (lane < 2) notes->count[lane] = 0u;
    griddep_wait();
    griddep_launch();
    if (PERM) {                                          // places in the row, in bytes
        for (int c = 2 * tid; c < p.d; c += 2 * (int)blockDim.x) {
            const uint32_t a = (uint32_t)min(max(__ldg(p.perm + c), 0), p.d - 1), b = (uint32_t)min(max(__ldg(p.perm + c + 1), 0), p.d - 1);
            perq_mm::sts32(table + 2u * (uint32_t)c, 2u * a | (b << 17));
        }
    }
    __syncthreads();
    const long long step = (long long)gridDim.x * p.rows, first = (long long)blockIdx.x * p.rows + g;
    const uint32_t steps = first < p.T ? (uint32_t)((p.T - first + step - 1) / step) : 0u;
    const int c0 = w * WARP_ELEMS + lane * LANE_ELEMS, per_piece = p.warps * WARP_ELEMS;        // this lane's first channel, and from piece to piece
    auto load = [&](uint32_t i) {
        if (i < steps) {
            const uint32_t s = i % STAGES;
            perq_mm::mbar_expect_tx(full + 8 * s, row_bytes);
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(ring + s * row_bytes), "l"(p.x + (size_t)(first + (long long)i * step) * (size_t)p.d), "r"(row_bytes), "r"(full + 8 * s) : "memory");
        }
    };
    if (w == 0 && lane == 0)
        for (uint32_t i = 0; i < STAGES; ++i) load(i);
    const Hadamard matrix = hadamard_operand<LOG2B>(lane);
    const Pair magic = pair_of(12582912.0f, 12582912.0f), neg = pair_of(-1.0f, -1.0f);          // 1.5 2^23: the low byte of a sum with it is the code
    constexpr int block_lanes = LOG2B > 4 ? 1 << (LOG2B - 4) : 1;
    bool alive = true;
    for (uint32_t i = 0; i < steps; ++i) {
        // (a wait that ran out: what follows is wrong, and is not waited for)
        if (alive && !perq_mm::mbar_wait_warp(full + 8 * (i % STAGES), (i / STAGES) & 1u)) {
            alive = false;
            if (lane == 0) atomicOr(&perq_mm::g_error, perq_mm::ERROR_ROWS);
        }
        const uint32_t row = ring + i % STAGES * row_bytes;
        Pair u[PIECES][LANE_ELEMS / 2];
        float block[PIECES], top = 0.0f;                 // largest of the lane's block, of the warp
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const bool valid = c0 + k * per_piece < p.d;
            const uint32_t at = (PERM ? table : row) + 2u * (uint32_t)(c0 + k * per_piece);
            const uint4 a = valid ? perq_mm::lds128(at) : make_uint4(0, 0, 0, 0), b = valid ? perq_mm::lds128(at + 16) : make_uint4(0, 0, 0, 0);
            uint32_t raw[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            if (PERM) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint16_t lo, hi;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(lo) : "r"(row + (raw[j] & 0xffffu)));
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(hi) : "r"(row + (raw[j] >> 16)));
                    raw[j] = valid ? (uint32_t)lo | ((uint32_t)hi << 16) : 0u;
                }
            }
            __syncwarp();
            rotate<LOG2B>(u[k], raw, matrix, lane);
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < LANE_ELEMS / 2; ++j) m = max3(m, u[k][j]);
#pragma unroll
            for (int l = 1; l < block_lanes; l *= 2) m = max2(m, __shfl_xor_sync(0xffffffffu, m, l));
            block[k] = m;
            top = max2(top, m);
        }
        top = warp_max(top);
        float all = top;
        if (p.warps > 1) {
            if (lane == 0) sh->part[i & 1u][warp] = top;
            row_barrier(g, p.warps);
            all = warp_max(lane < p.warps ? sh->part[i & 1u][g * p.warps + lane] : 0.0f);
        } else {
            __syncwarp();
        }
        if (w == 0 && lane == 0) load(i + STAGES);       // (all of the row's warps have read it)
        // Rows so small that 127 / max overflows, or so large that 1 / max is no normal number (a unit of it is then more than 2^-23 of it), are settled
        // block by block, and so are those whose sums are not finite.
        // (One comparison of bits, which also finds NaN: 16384 x 4096, b = 32, 41.9 us with two of numbers, 41.0 so.)
        const bool odd = __float_as_uint(all) - (__float_as_uint(0x1p-120f) + 1u) >= __float_as_uint(0x1p126f) - __float_as_uint(0x1p-120f);
        float ratio;
        asm("rcp.approx.f32 %0, %1;" : "=f"(ratio) : "f"(all));          // (off by a unit at most)
        ratio = odd ? 0.0f : 127.0f * ratio;
        const Pair rr = pair_of(ratio, ratio);
        const float near = odd ? (all != 0.0f ? 0.0f : 1.0f) : all * p.near_max;
        int8_t *const out = p.codes + (size_t)(first + (long long)i * step) * (size_t)p.d + c0;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            uint32_t code[4];
            float off = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const Pair x = pair_fma(u[k][2 * c], rr, magic), y = pair_fma(u[k][2 * c + 1], rr, magic);
                off = max3(off, pair_fma(u[k][2 * c], rr, pair_fma(x, neg, magic)));
                off = max3(off, pair_fma(u[k][2 * c + 1], rr, pair_fma(y, neg, magic)));
                const uint32_t lo = __byte_perm((uint32_t)x, (uint32_t)(x >> 32), 0x0040), hi = __byte_perm((uint32_t)y, (uint32_t)(y >> 32), 0x0040);
                code[c] = __byte_perm(lo, hi, 0x5410);
            }
            if (c0 + k * per_piece < p.d) {
                *reinterpret_cast<uint4 *>(out + k * per_piece) = make_uint4(code[0], code[1], code[2], code[3]);
                const bool doubt = off >= 0.5f - 0x1p-23f - block[k] * ratio * p.doubt;
                if (doubt || !(block[k] < near)) {
                    note_lane(notes, u[k][0], u[k][1], u[k][2], u[k][3], u[k][4], u[k][5], u[k][6], u[k][7], ratio, odd ? 0.0f : doubt ? 0.5f - 0x1p-23f - block[k] * ratio * p.doubt : 1.0f,
                              near, i % BATCH, c0 + k * per_piece);
                }
            }
        }
        if (i % BATCH == BATCH - 1 || i + 1 == steps)
            settle_batch<LOG2B, PIECES, PERM>(p, group, notes, table, first + (long long)(i / BATCH * BATCH) * step, step, i % BATCH + 1u, g, w, lane);
    }
    // (nothing is in flight when the CTA ends, also after a wait that ran out)
    if (!alive && w == 0 && lane == 0)
        for (uint32_t i = steps > STAGES ? steps - STAGES : 0u; i < steps; ++i) (void)perq_mm::mbar_wait(full + 8 * (i % STAGES), (i / STAGES) & 1u);
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
