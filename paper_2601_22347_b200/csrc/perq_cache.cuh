// An 8-bit cache of keys and values in pages: writing (rotation of the keys, a step for each page and head) and reading back.
//
// A block is `page` tokens of one head, int8 [page][D], with one fp32 step s.  New rows y (keys: rotated) give a = max |y| and s' = fp32(a / 127); s is s', or the
// larger of s' and the block's step where earlier tokens stay in it.  code = rne(y / s), and earlier codes become rne(code s_old / s) where s has grown: the
// cache costs one read of a block's codes more only when its largest value changes.
//
// A new element is read once (2 bytes) and written once (1 byte).  A lane holds 16 adjacent channels of a token, so that a block of b channels is a butterfly of four stages in registers and up to
// three exchanges between lanes.  Eight or sixteen warps share a block of a prompt and keep its rotated values in registers over the barrier that its maximum needs; blocks of up to 2048
// elements have a warp each.  For few tokens a warp has a block of its own and a lane four channels: what is met for the first time is most of such a call, and that is a quarter of the code.
// Four prompts of up to 4096 tokens, 8 heads of 128, pages of 128: 31 us, 61 MB at 1.9 TB/s.  Bound by what a block's steps wait for one after another, at two blocks to an SM (all registers):
// finding it 1.9 us, reading 1.5, the maximum's barrier 0.5, settling it 0.9 to 1.7, codes 1.1.  256 sequences' next tokens 12.6 us where no step grows: a chain
// of sequence, page, step, tokens and exact maximum, each from memory.  Where steps grow a warp has a page's earlier codes to round again, 16 bytes to a lane at a time, one load after another: 45 us with pages of 64
// whose slots are spread, 71 with pages of 128 (one token: 15 and 14; in the last slot 26 and 47).  In use, a step of the block of slot k grows in about one of k + 1 calls.
//
// Codes are those of exact arithmetic.  A butterfly of L = log2 b stages rounds each sum L times, so |u32 - u| <= L 2^-24 sum |x|, and sum |x| <= sqrt b |x|_2 =
// |u|_2 <= sqrt b max |u| over the rotation's block: E = 1.01 L sqrt b 2^-24 of its largest (b = 128: 4.8e-6).  What may be the block's maximum (within 2 E of the largest in
// fp32) is summed again in fp64, and so is an element whose quotient lies within 127 (E + 2^-21) of the border between two codes (b = 128: one in 800), by the
// lanes that hold its rotation's block.
#pragma once

#include "perq_mm_ptx.cuh"

namespace perq_kv {

using perq_mm::griddep_launch;
using perq_mm::griddep_wait;

constexpr int THREADS = 256;
constexpr int LANE = 16;                      // channels of a lane

// The sequences of a call.
struct Sequences {
    const int32_t *offsets, *lengths, *pages;
    int32_t T, S, width, n_pages, page;       // (page: its log2)
};
struct Rows {
    int32_t begin, n;                         // rows of the call
    int32_t length;                           // tokens, these included
};
// What the host never looks at is taken into its range here: wrong numbers, never a fault.
__device__ __forceinline__ Rows rows_of(const Sequences &q, int i)
{
    Rows r;
    r.begin = min(max(*(q.offsets + i), 0), q.T);
    r.n = max(min(max(*(q.offsets + i + 1), 0), q.T) - r.begin, 0);
    r.length = (int32_t)min((long long)max(*(q.lengths + i), 0), (long long)q.width << q.page);
    return r;
}
// Blocks that a sequence's rows fall into; rows at positions below 0 (fewer tokens than rows) into none.
__device__ __forceinline__ int blocks_of(const Sequences &q, const Rows &r)
{
    const int first = max(r.length - r.n, 0);
    return r.length > first ? ((r.length - 1) >> q.page) - (first >> q.page) + 1 : 0;
}

// A lane's C channels, two to a word.
template <int C>
__device__ __forceinline__ void unpack(float (&u)[C], const uint32_t (&w)[C / 2], bool f16)
{
    if (f16) {
#pragma unroll
        for (int i = 0; i < C / 2; ++i)
            asm("{ .reg .b16 x, y; mov.b32 {x, y}, %2; cvt.f32.f16 %0, x; cvt.f32.f16 %1, y; }" : "=f"(u[2 * i]), "=f"(u[2 * i + 1]) : "r"(w[i]));
    } else {
#pragma unroll
        for (int i = 0; i < C / 2; ++i) {
            u[2 * i] = __uint_as_float(w[i] << 16);
            u[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
__device__ __forceinline__ void unpack(float (&u)[LANE], const uint4 &lo, const uint4 &hi, bool f16)
{
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    unpack<LANE>(u, w, f16);
}
// Times the Hadamard matrix of blocks of 2^log2b channels (0: none), without its factor.
template <int C>
__device__ __forceinline__ void rotate(float (&u)[C], int log2b, int lane)
{
    if (log2b == 0) return;
#pragma unroll
    for (int h = 1; h < C; h *= 2)
#pragma unroll
        for (int i = 0; i < C; ++i)
            if ((i & h) == 0) {
                const float a = u[i], b = u[i + h];
                u[i] = a + b;
                u[i + h] = a - b;
            }
#pragma unroll 1
    for (int l = 1; l < (1 << log2b) / C; l *= 2) {
        const float s = (lane & l) ? -1.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < C; ++i) u[i] = fmaf(s, u[i], __shfl_xor_sync(0xffffffffu, u[i], l));      // (s u exact: one rounding)
    }
}

// rne(y / s) for |y / s| < 2^31, exactly: the quotient's nearest whole number, mended by what is left.  y has to have 53 - 32 bits to spare, or no ties.
__device__ __forceinline__ int exact_code(double y, float s)
{
    const double w = (double)s;
    double n = rint(y / w);
    const double left = fma(-n, w, y), twice = 2.0 * fabs(left);
    if (twice > w || (twice == w && fmod(n, 2.0) != 0.0)) n += left > 0.0 ? 1.0 : -1.0;
    return (int)fmin(fmax(n, -127.0), 127.0);
}

struct WriteParams {
    Sequences q;
    const uint16_t *x[2];                     // keys, values: [T] rows of heads * D, row strides
    long long stride[2];
    int8_t *codes[2];                         // [n_pages, heads, page, D]
    float *steps[2];                          // [n_pages, heads]
    int32_t heads, f16;
    int32_t log2b;                            // of the keys
    int32_t parts;                            // CTAs to a page's blocks, for all heads' keys and values
};

struct Place {
    int32_t row, slot, n;                     // its rows of the call, and their first place in the block
    int32_t entry;                            // its place in the sequence's row of the table, read when it is wanted
    int32_t sequence;
};
// Which sequence's which page the number-th block is.  Called by all threads of the CTA.
template <int SIZE>
__device__ __forceinline__ Place find_block(const Sequences &q, int number)
{
    __shared__ int32_t sums[SIZE / 32];
    __shared__ Place found;
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto place_of = [&](int i, const Rows &r, int at) {
        const int first = r.length - r.n, index = (max(first, 0) >> q.page) + at, from = max(index << q.page, max(first, 0));
        Place p;
        p.row = r.begin + (from - first);
        p.slot = from - (index << q.page);
        p.n = min((index + 1) << q.page, r.length) - from;
        p.entry = index;
        p.sequence = i;
        return p;
    };
    if (q.S <= 32) {
        // (every warp for itself)
        Rows r = {0, 0, 0};
        int c = 0;
        if (lane < q.S) {
            r = rows_of(q, lane);
            c = blocks_of(q, r);
        }
        int sum = c;
#pragma unroll
        for (int l = 1; l < 32; l *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, sum, l);
            if (lane >= l) sum += v;
        }
        const int at = number - (sum - c);
        const unsigned here = __ballot_sync(0xffffffffu, at >= 0 && at < c);
        Place p = {0, 0, 0, 0, 0};
        if (here == 0u) return p;
        if (at >= 0 && at < c) p = place_of(lane, r, at);
        const int owner = __ffs(here) - 1;
        p.row = __shfl_sync(0xffffffffu, p.row, owner);
        p.slot = __shfl_sync(0xffffffffu, p.slot, owner);
        p.n = __shfl_sync(0xffffffffu, p.n, owner);
        p.entry = __shfl_sync(0xffffffffu, p.entry, owner);
        p.sequence = owner;
        return p;
    }
    if (tid == 0) found.n = 0;
    for (int base = 0, before = 0; base < q.S; base += SIZE) {
        Rows r = {0, 0, 0};
        int c = 0;
        if (base + tid < q.S) {
            r = rows_of(q, base + tid);
            c = blocks_of(q, r);
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
        for (int w = 0; w < SIZE / 32; ++w) {
            if (w < warp) sum += sums[w];
            all += sums[w];
        }
        const int at = number - (before + sum - c);
        if (at >= 0 && at < c) {
            found = place_of(base + tid, r, at);
        }
        before += all;
        __syncthreads();
        if (before > number) break;
    }
    __syncthreads();
    return found;
}

// WARPS warps have a block (8 or 16: the CTA's; 1: a block of each), `tokens` of it at a time, of which each lane keeps HELD lots of C channels.  ALL: those are all that there can be.
// (C is 16 for prompts.  For few tokens it is 4: instructions that are met for the first time are most of such a call, and a quarter of them is unrolled.)
template <int D, int WARPS, int HELD, int C>
struct Write {
    static constexpr int lanes = D / C;                                // to a token
    static constexpr int threads = WARPS == 16 ? 512 : THREADS;
    static constexpr int tokens = WARPS * 32 / lanes;
};

template <int D, int WARPS, int HELD, int C, bool ALL>
__global__ void __launch_bounds__(WARPS == 16 ? 512 : THREADS, HELD == 4 || WARPS == 16 ? 2 : 4) write_kernel(const __grid_constant__ WriteParams p)
{
    using K = Write<D, WARPS, HELD, C>;
    __shared__ float part[K::threads / 32];
    __shared__ unsigned long long exact[K::threads / 32];
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5;
    griddep_wait();
    griddep_launch();
    const int number = (int)(blockIdx.x / (unsigned)p.parts), in = (int)(blockIdx.x % (unsigned)p.parts);
    const Place at = find_block<K::threads>(p.q, number);
    if (at.n <= 0) return;
    // (on its way while the tokens are read and rotated)
    const int page = *(p.q.pages + (size_t)at.sequence * (size_t)p.q.width + (size_t)at.entry);
    const int item = WARPS == 1 ? in * (K::threads / 32) + warp : in;
    if (item >= 2 * p.heads) return;                                   // (whole warps, and then no barrier follows)
    const int kind = item >= p.heads ? 1 : 0, head = item - kind * p.heads, log2b = kind ? 0 : p.log2b;
    const bool f16 = p.f16 != 0;
    const uint16_t *const x = p.x[kind] + (size_t)at.row * (size_t)p.stride[kind] + (size_t)head * D;
    const int share = WARPS == 1 ? lane : tid, mine = share / K::lanes, channel = (share % K::lanes) * C;
    const int lots = (at.n + K::tokens - 1) / K::tokens;
    const bool held = ALL || lots <= HELD;                             // (else every pass reads and rotates again)
    auto load = [&](int lot, float (&u)[C]) {
        const int t = lot * K::tokens + mine;
        uint32_t w[C / 2] = {};
        if (t < at.n) {
            const uint16_t *const from = x + (size_t)t * (size_t)p.stride[kind] + channel;
            if constexpr (C == 16) {
                const uint4 lo = *reinterpret_cast<const uint4 *>(from), hi = *(reinterpret_cast<const uint4 *>(from) + 1);
                w[0] = lo.x; w[1] = lo.y; w[2] = lo.z; w[3] = lo.w; w[4] = hi.x; w[5] = hi.y; w[6] = hi.z; w[7] = hi.w;
            } else {
                const uint2 lo = *reinterpret_cast<const uint2 *>(from);
                w[0] = lo.x; w[1] = lo.y;
            }
        }
        unpack<C>(u, w, f16);
    };
    // The lanes' elements that have a bit in `want` (C of a lot, lots from lot0 on) are summed again in fp64, by the lanes that have their token: take(lot, i, u) gets each.
    auto settle = [&](int lot0, unsigned long long want, auto &&take) {
        for (unsigned asked = __ballot_sync(0xffffffffu, want != 0ull); asked != 0u; asked = __ballot_sync(0xffffffffu, want != 0ull)) {
            const unsigned group = ((K::lanes == 32 ? 0xffffffffu : ((1u << (K::lanes & 31)) - 1u) << (lane & ~(K::lanes - 1)))) & asked;
            const int leader = group ? __ffs(group) - 1 : lane, bit = want ? __ffsll((long long)want) - 1 : 0;
            const int lot = lot0 + __shfl_sync(0xffffffffu, bit / C, leader);
            const unsigned e = (unsigned)__shfl_sync(0xffffffffu, channel + bit % C, leader) & ((1u << log2b) - 1u);
            float v[C];
            load(lot, v);
            double sum = 0.0;
            // (other rotations' blocks of the token add up what nobody reads)
#pragma unroll
            for (int k = 0; k < C; ++k) sum += __popc(e & (unsigned)(channel + k)) & 1 ? -(double)v[k] : (double)v[k];
            for (int l = 1; l < (1 << log2b) / C; l *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, l);
            if (log2b == 0) {
#pragma unroll
                for (int k = 0; k < C; ++k)
                    if (k == bit % C) sum = (double)v[k];
            }
            if (leader == lane && want != 0ull) {
                take(lot, bit % C, sum);
                want &= want - 1ull;
            }
        }
    };

    // 1. the largest of the block
    float u[HELD][C], top = 0.0f, tops[HELD];
    for (int lot0 = 0; lot0 < lots; lot0 += HELD) {
#pragma unroll
        for (int h = 0; h < HELD; ++h)
            if (lot0 + h < lots) load(lot0 + h, u[h]);
#pragma unroll
        for (int h = 0; h < HELD; ++h)
            if (lot0 + h < lots) {
                rotate(u[h], log2b, lane);
                tops[h] = 0.0f;
#pragma unroll
                for (int i = 0; i < C; i += 2) asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(tops[h]) : "f"(fabsf(u[h][i])), "f"(fabsf(u[h][i + 1])));
                asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(tops[h]));
            }
        if (ALL) break;
    }
    if (page < 0 || page >= p.q.n_pages) return;                       // (the whole block's: no barrier is missed)
    const size_t block = (size_t)page * (size_t)p.heads + (size_t)head;
    int8_t *const codes = p.codes[kind] + (block << p.q.page) * (size_t)D;
    float *const step = p.steps[kind] + block;
    const float before = at.slot > 0 ? *step : 0.0f;
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
    if (WARPS > 1) {
        if (lane == 0) {
            part[warp] = top;
            exact[warp] = 0ull;
        }
        __syncthreads();
        top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(part[lane % WARPS])));
    }
    const double wide_root = (log2b & 1 ? 1.4142135623730951 : 1.0) * (double)(1 << (log2b >> 1));        // sqrt b
    const float root = (float)wide_root;
    const float e = log2b == 0 ? 0.0f : 1.01f * (float)log2b * root * 0x1p-24f;
    // Far from the ends of fp32, or everything is summed in fp64.
    const bool plain = top < 0x1p100f && top > 0x1p-80f;
    double a = (double)top;
    if (top != 0.0f && log2b != 0) {
        const float near = plain ? top * (1.0f - 2.0f * e - 0x1p-22f) : -1.0f;
        unsigned long long most = 0ull;
        for (int lot0 = 0; lot0 < lots; lot0 += HELD) {
            unsigned long long want = 0ull;
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                if (lot0 + h >= lots) break;
                if (!held) {
                    load(lot0 + h, u[h]);
                    rotate(u[h], log2b, lane);
                }
                if ((!held || !(tops[h] < near)) && (lot0 + h) * K::tokens + mine < at.n) {
                    unsigned bits = 0u;
#pragma unroll
                    for (int i = 0; i < C; ++i) bits |= !(fabsf(u[h][i]) < near) ? 1u << i : 0u;
                    want |= (unsigned long long)bits << (C * h);
                }
            }
            settle(lot0, want, [&](int, int, double y) { most = max(most, (unsigned long long)__double_as_longlong(fabs(y))); });
            if (ALL) break;
        }
        // (numbers of bits, as none is negative: the upper halves' largest, then the lower ones' of those that have it)
        auto largest = [](unsigned long long v) {
            const unsigned high = __reduce_max_sync(0xffffffffu, (unsigned)(v >> 32));
            return (unsigned long long)high << 32 | __reduce_max_sync(0xffffffffu, (unsigned)(v >> 32) == high ? (unsigned)v : 0u);
        };
        most = largest(most);
        if (WARPS > 1) {
            if (lane == 0) exact[warp] = most;
            __syncthreads();
            most = largest(exact[lane % WARPS]);
        }
        a = __longlong_as_double((long long)most);
    }
    // a / sqrt b / 127: by a product that is off by 2^-51 at most, unless that could decide how it is rounded to fp32 (or fp32's ends are near).  Divisions in fp64 are 60 instructions each.
    const double about = a * (1.0 / 127.0) * (log2b & 1 ? 0.70710678118654752 : 1.0) * __longlong_as_double((long long)(1023 - (log2b >> 1)) << 52);
    const uint32_t rest = (uint32_t)__double_as_longlong(about) & 0x1fffffffu;
    float s = plain && rest - 0x0ffffff0u > 0x20u ? (float)about : (float)(a / wide_root / 127.0);
    if (before > s || before != before) s = before;
    const bool finite = fabsf(s) <= 3.4028235e38f, none = !finite || s == 0.0f;

    // 2. codes
    const float inverse = 1.0f / (s * root);                           // (off by 3 2^-24, and a quotient by one more)
    // (a value of s is at least that of the largest / 127, so |u| inverse stays below 127 and a little)
    const bool quick = plain && s > 0x1p-100f;
    const float sure = quick ? 0.5f - 127.5f * (e + 0x1p-21f) : -1.0f;
    for (int lot0 = 0; lot0 < lots; lot0 += HELD) {
        unsigned long long doubt = 0ull;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            if (lot0 + h >= lots) break;
            if (!held) {
                load(lot0 + h, u[h]);
                rotate(u[h], log2b, lane);
            }
            uint32_t c[C];
            float far = 0.0f;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const float q = u[h][i] * inverse, t = q + 12582912.0f;
                u[h][i] = q - (t - 12582912.0f);
                c[i] = __float_as_uint(t);
            }
#pragma unroll
            for (int i = 0; i < C; i += 2) asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(far) : "f"(fabsf(u[h][i])), "f"(fabsf(u[h][i + 1])));
            const int t = (lot0 + h) * K::tokens + mine;
            if (!(far <= sure) && !none && t < at.n) {
                unsigned bits = 0u;
#pragma unroll
                for (int i = 0; i < C; ++i) bits |= !(fabsf(u[h][i]) <= sure) ? 1u << i : 0u;
                doubt |= (unsigned long long)bits << (C * h);
            }
            uint32_t w[C / 4];
#pragma unroll
            for (int i = 0; i < C / 4; ++i)
                w[i] = none ? 0u : __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0040), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0040), 0x5410);
            int8_t *const to = codes + (size_t)(at.slot + t) * D + channel;
            if (t < at.n) {
                if constexpr (C == 16) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
                else *reinterpret_cast<uint32_t *>(to) = w[0];
            }
        }
        // (bytes of what this lane has just stored)
        settle(lot0, doubt, [&](int lot, int i, double y) { codes[(size_t)(at.slot + lot * K::tokens + mine) * D + channel + i] = (int8_t)exact_code(y / wide_root, s); });
        if (ALL) break;
    }
    // 3. earlier codes, where the step has grown
    if (at.slot > 0 && !(s == before)) {
        const float ratio = before / s;
        const bool fast = before > 0x1p-80f && s < 0x1p100f;
        // (16 codes to a lane)
        for (int k = share; k < at.slot * (D / 16); k += WARPS * 32) {
            uint4 *const to = reinterpret_cast<uint4 *>(codes) + k;
            uint4 old = *to;
            uint32_t *const w = reinterpret_cast<uint32_t *>(&old);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t r = 0u;
#pragma unroll 1
                for (int b = 0; b < 32; b += 8) {
                    const int code = (int)(int8_t)(w[i] >> b);
                    const float q = (float)code * ratio, n = rintf(q);
                    int v = (int)n;
                    if (!fast || fabsf(q - n) > 0.5f - 128.0f * 0x1p-22f) v = none ? 0 : exact_code((double)code * (double)before, s);
                    r |= (uint32_t)(uint8_t)v << b;
                }
                w[i] = none ? 0u : r;
            }
            *to = old;
        }
    }
    if ((WARPS == 1 ? lane : tid) == 0) *step = s;
}

// ------------------------------------------------------------------------------------------------------ reading back
constexpr int READ_TOKENS = 32;               // of a CTA
constexpr int READ_AHEAD = 4;

struct ReadParams {
    Sequences q;
    const int8_t *codes[2];
    const float *steps[2];
    void *out[2];                             // [T, heads, D]
    int32_t heads, out_type, log2b;
};

__device__ __forceinline__ uint32_t pack16(float x, float y, bool f16)
{
    uint32_t r;
    if (f16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
}

// 32 bytes: in one store where they lie on a multiple of 32, so that no sector is written in halves.
__device__ __forceinline__ void store32(void *to, const uint32_t *w, bool wide)
{
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else {
        static_cast<uint4 *>(to)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        static_cast<uint4 *>(to)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// A lane has 16 channels of a token and head; blockIdx.y: keys, values.  The sequence of a row is looked for once a token.  Bound by instructions where keys are rotated (eight sequences of up
// to 4096 tokens, blocks of 128, 5.0 TB/s without the rotation): 3 exchanges of 16 words each, 64 sums.  Conversions of codes run beside that on a pipe of their own; by permuted bytes and a
// subtraction they cost the one that is wanted (31 -> 42 us), and so do sums of two in one integer (36).
template <int D>
__global__ void __launch_bounds__(THREADS) read_kernel(const __grid_constant__ ReadParams p)
{
    constexpr int lanes = D / LANE;
    __shared__ int32_t place[READ_TOKENS], slot[READ_TOKENS];
    griddep_wait();
    griddep_launch();
    const int tid = (int)threadIdx.x, lane = tid & 31, row0 = (int)blockIdx.x * READ_TOKENS, kind = (int)blockIdx.y;
    if (tid < READ_TOKENS) {
        // the last sequence that begins at or before the row (offsets do not decrease)
        const int row = row0 + tid;
        int lo = 0, hi = p.q.S;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (*(p.q.offsets + mid) <= row) lo = mid; else hi = mid;
        }
        const Rows r = rows_of(p.q, lo);
        int at = -2;                                                   // not a row of any sequence: left as it is
        slot[tid] = 0;
        if (row >= r.begin && row < r.begin + r.n) {
            const int position = r.length - r.n + (row - r.begin);
            at = position < 0 ? -1 : *(p.q.pages + (size_t)lo * (size_t)p.q.width + (size_t)(position >> p.q.page));
            if (at < 0 || at >= p.q.n_pages) at = -1;                  // (zeros)
            slot[tid] = position & ((1 << p.q.page) - 1);
        }
        place[tid] = at;
    }
    __syncthreads();
    const int tokens = min(READ_TOKENS, p.q.T - row0), items = tokens * p.heads * lanes, log2b = kind ? 0 : p.log2b;
    const float factor = 1.0f / sqrtf((float)(1 << log2b));
    const bool wide = (reinterpret_cast<size_t>(p.out[kind]) & 31u) == 0u;
    for (int i0 = 0; i0 < items; i0 += READ_AHEAD * THREADS) {
        // (all that is read is on its way before the first of it is used)
        uint4 v[READ_AHEAD];
        float s[READ_AHEAD];
        int page[READ_AHEAD];
#pragma unroll
        for (int a = 0; a < READ_AHEAD; ++a) {
            const int i = i0 + a * THREADS + tid, t = min(i / lanes / p.heads, tokens - 1), head = i / lanes % p.heads, channel = i % lanes * LANE;
            page[a] = i < items ? place[t] : -2;
            v[a] = make_uint4(0, 0, 0, 0);
            s[a] = 0.0f;
            if (page[a] >= 0) {
                const size_t block = (size_t)page[a] * (size_t)p.heads + (size_t)head;
                v[a] = *reinterpret_cast<const uint4 *>(p.codes[kind] + ((block << p.q.page) + (size_t)slot[t]) * D + channel);
                s[a] = *(p.steps[kind] + block);
            }
        }
#pragma unroll
        for (int a = 0; a < READ_AHEAD; ++a) {
            if (i0 + a * THREADS >= items) break;
            float u[LANE];
            const uint32_t w[4] = {v[a].x, v[a].y, v[a].z, v[a].w};
#pragma unroll
            for (int k = 0; k < LANE; ++k) u[k] = (float)(int8_t)(w[k / 4] >> (8 * (k % 4)));
            rotate(u, log2b, lane);                                    // (whole numbers below 2^14: exact)
#pragma unroll
            for (int k = 0; k < LANE; ++k) u[k] *= s[a] * factor;
            if (page[a] == -2) continue;
            // (rows are dense: the i-th 16 channels from the CTA's first row on)
            const size_t at = ((size_t)row0 * (size_t)(p.heads * lanes) + (size_t)(i0 + a * THREADS + tid)) * LANE;
            if (p.out_type == perq_mm::OUT_F32) {
                float *const to = static_cast<float *>(p.out[kind]) + at;
                uint32_t o[LANE];
#pragma unroll
                for (int k = 0; k < LANE; ++k) o[k] = __float_as_uint(u[k]);
                store32(to, o, wide);
                store32(to + 8, o + 8, wide);
            } else {
                uint32_t o[LANE / 2];
#pragma unroll
                for (int k = 0; k < LANE / 2; ++k) o[k] = pack16(u[2 * k], u[2 * k + 1], p.out_type == perq_mm::OUT_F16);
                store32(static_cast<uint16_t *>(p.out[kind]) + at, o, wide);
            }
        }
    }
}

}  // namespace perq_kv
