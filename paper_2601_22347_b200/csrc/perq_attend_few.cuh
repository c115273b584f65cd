// Attention over the 8-bit cache for few queries to a sequence: decode steps and drafted tokens.
//
// Bound by memory: the visible codes of a (sequence, head of keys) are read once for all queries that share it.  Rows are pairs of a new token and one of the `group`
// heads of queries that share a head of keys; a unit of work is 16 keys for a tile of 8 or 16 rows.  The CTAs take equal shares of all units, whatever the lengths are
// (they are known on the device only), and a share's eight warps take its units in turn.  A row whose units belong to several CTAs is put together by join_kernel, in a
// fixed order.
//
// Keys (then, transposed, values) are the first operand of mma.sync, rows the second, so that eight rows cost no more than they have to.  The order of the
// channels inside a product is free: a lane takes 16 adjacent codes of its keys as they lie in memory, and of its values 16 adjacent channels of four keys.  A warp has a ring of its own
// in shared memory, filled by tensor copies whose 128-byte swizzle, with odd keys taken four further on (key_in), keeps its 16-byte reads free of conflicts.  (Copies of 16 bytes by every
// lane ended at 4.6 TB/s, also with nothing done to what they brought: 64 sequences of up to 12000 tokens 228 us.)
//
// Logits: keys' codes stay 8-bit integers (m16n8k32).  A query becomes 128 hi + lo of two 8-bit integers, its largest channel 16256, so it is off by 2^-15 of that at most, and S = sum
// (128 hi + lo) code is exact.  (Codes to fp16 instead: 80 instructions for 16 keys of 128 channels; these products take 8 of the 8 cycles that an fp16 one takes too.)
// Values' codes become fp16 exactly: code ^ 0x80 in the low bits of 1024, minus 1152.
//
// 64 sequences of up to 12000 tokens, 8 heads of 128 with 4 of queries each: 181 us, 5.8 TB/s of 6.5.  32 sequences of up to 5 tokens, 4 heads of 64 with 8 of queries each, a window of 4096:
// 60 us, 1.1 TB/s; there a sequence has one to three tiles of 16 rows, each of which goes over its keys again (from L2), at 440 instructions a unit in all (64 sequences: 360), and a CTA's
// share of 223 units crosses tiles, whose queries and results cost some microseconds each.
//
// y = s_k f S + log2 s_v - m, base 2, with f the row's factor and m its reference.  Values' steps go into the exponent: P = 2^y, so that fp16 P meet exact codes and no row's
// sums mix steps; the sum of probabilities adds P / s_v in fp32.  m is 7 below the largest so far and is only moved when something is over 2^15 (P_MOST: fp16 ends at 2^16), so that P has all of
// fp16's range: off by 2^-11 of itself (half a last place), or by half of fp16's smallest step, 2^-25, which is 2^-32 of the row's largest.  (With m at the largest that was 2^-25 of it: beside keys
// whose values are zero, those of 2^-22.4 of their probability gave a result off by 1 %, those of 2^-27.7 nothing.)  Values' steps below 2^-64 (of zeros) count as 2^-64.
#pragma once

#include "perq_cache.cuh"

namespace perq_kv {

constexpr int FEW_WARPS = THREADS / 32;
constexpr int FEW_KEYS = 16;                  // of a unit
// Exponents of the largest P when a reference is set, and of the largest that there may be before it is moved.
constexpr float P_LIFT = 7.0f, P_MOST = 15.0f;
// Set in perq_mm's error word when a bounded wait ran out.
enum : unsigned int { ERROR_ATTEND = 1u << 7 };

struct AttendParams {
    Sequences q;
    const uint16_t *x;                        // queries: [T] rows of heads * group * D, row stride
    long long stride;
    const int8_t *k_codes, *v_codes;
    const float *k_steps, *v_steps;
    void *out;                                // [T, heads * group, D]
    float *partial;                           // of shares: [2 * CTAs][rows][D + 2]
    int32_t heads, group;
    int32_t most;                             // rows of a sequence that are looked at
    int32_t few_rows;                         // sequences of up to so many (token, head) rows are the kernel's for few queries, the others the one's for many
    int32_t window, sinks, log2b, f16, out_type;
    float scale;                              // of logits, times log2 e / sqrt b
};

// Row g of a product's first operand is this key of eight, so that rows next to each other differ in bit 2 of their place, and even rows hold even keys.
__device__ __forceinline__ int key_in(int g) { return g ^ ((g & 1) << 2); }
// Where 16 bytes lie in rows of D with their copies' swizzle (of 128 or 64 bytes).
template <int D>
__device__ __forceinline__ uint32_t swizzled(int row, int chunk)
{
    return (uint32_t)(row * D + (D == 128 ? (chunk ^ row) & 7 : (chunk ^ (row >> 1)) & 3) * 16);
}
__device__ __forceinline__ float exp2_of(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float log2_of(float x)
{
    float r;
    asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) { return pack16(lo, hi, true); }
// Two codes in bytes 0 and 2 as fp16.
__device__ __forceinline__ uint32_t codes_f16(uint32_t w)
{
    uint32_t r;
    asm("{ .reg .b32 t; lop3.b32 t, %1, 0x00ff00ff, 0x64806480, 0x6a; sub.rn.f16x2 %0, t, %2; }" : "=r"(r) : "r"(w), "r"(0x64806480u));
    return r;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_i8(int32_t (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) { return perq_mm::lds128(at); }
__device__ __forceinline__ uint2 lds64(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}

// The units of a sequence's tiles: groups of keys 0 .. sunk - 1, then from `low` on.
struct Units {
    Rows r;
    int32_t tokens;                           // rows that are looked at
    int32_t sunk, low, count;                 // groups of a tile; at least one, so that rows that see nothing are written
    int32_t tiles;                            // of rows, each once for every head of keys
};
template <int ROWS>
__device__ __forceinline__ Units units_of(const AttendParams &p, int i)
{
    Units u;
    u.r = rows_of(p.q, i);
    u.tokens = min(u.r.n, p.most);
    const long long rows = (long long)u.tokens * p.group;
    u.tiles = rows <= p.few_rows ? ((int)rows + ROWS - 1) / ROWS : 0;
    const int first = u.r.length - u.r.n, end = max(min(u.r.length, first + u.tokens), 0);
    u.low = p.window > 0 ? max(first - p.window + 1, 0) / FEW_KEYS : 0;
    u.sunk = min((min(p.sinks, end) + FEW_KEYS - 1) / FEW_KEYS, u.low);
    u.count = max(u.sunk + (end + FEW_KEYS - 1) / FEW_KEYS - u.low, 1);
    return u;
}

struct Share {
    long long all, per;                       // units of the call, and of a CTA
};
struct Found {
    int32_t sequence;
    long long begin;                          // its first unit
};
// The units of all sequences, and the sequence of unit `per * number` (none: S).  Called by all threads of the CTA; up to 32 sequences are looked at by every warp for itself.
template <int ROWS>
__device__ __forceinline__ Share share_units(const AttendParams &p, int number, int ctas, Found &f)
{
    if (p.q.S <= 32) {
        const int lane = (int)threadIdx.x & 31;
        long long mine = 0;
        if (lane < p.q.S) {
            const Units u = units_of<ROWS>(p, lane);
            mine = (long long)u.tiles * u.count * p.heads;
        }
        long long up_to = mine;
#pragma unroll
        for (int l = 1; l < 32; l *= 2) {
            const long long v = __shfl_up_sync(0xffffffffu, up_to, l);
            if (lane >= l) up_to += v;
        }
        Share s;
        s.all = __shfl_sync(0xffffffffu, up_to, 31);
        s.per = max((s.all + ctas - 1) / ctas, (long long)FEW_WARPS);
        const long long unit = s.per * number, begin = up_to - mine;
        const unsigned here = __ballot_sync(0xffffffffu, unit >= begin && unit < up_to);
        f.sequence = here ? __ffs(here) - 1 : p.q.S;
        f.begin = __shfl_sync(0xffffffffu, begin, here ? __ffs(here) - 1 : 0);
        return s;
    }
    __shared__ long long sums[FEW_WARPS];
    __shared__ Found found;
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long units = 0;
    auto mine = [&](int i) {
        if (i >= p.q.S) return 0ll;
        const Units u = units_of<ROWS>(p, i);
        return (long long)u.tiles * u.count * p.heads;
    };
    auto total = [&](long long c, long long &up_to) {                  // over the CTA; of the threads up to this one
        up_to = c;
#pragma unroll
        for (int l = 1; l < 32; l *= 2) {
            const long long v = __shfl_up_sync(0xffffffffu, up_to, l);
            if (lane >= l) up_to += v;
        }
        if (lane == 31) sums[warp] = up_to;
        __syncthreads();
        long long all = 0;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) {
            if (w < warp) up_to += sums[w];
            all += sums[w];
        }
        __syncthreads();
        return all;
    };
    long long c0 = 0, up0 = 0;
    for (int base = 0; base < p.q.S; base += THREADS) {
        long long up_to;
        const long long c = mine(base + tid), all = total(c, up_to);
        if (base == 0) {
            c0 = c;
            up0 = up_to;
        }
        units += all;
    }
    Share s;
    s.all = units;
    // (a share of at least a unit for each warp)
    s.per = max((units + ctas - 1) / ctas, (long long)FEW_WARPS);
    const long long unit = s.per * number;
    if (tid == 0) found.sequence = p.q.S;
    __syncthreads();
    if (unit < units) {
        long long before = 0;
        for (int base = 0; base < p.q.S && before <= unit; base += THREADS) {
            long long c = c0, up_to = up0, all;
            if (p.q.S > THREADS) {
                c = mine(base + tid);
                all = total(c, up_to);
            } else {
                all = units;
            }
            const long long begin = before + up_to - c;
            if (unit >= begin && unit < begin + c) {
                found.sequence = base + tid;
                found.begin = begin;
            }
            before += all;
        }
    }
    __syncthreads();
    f = found;
    __syncthreads();
    return s;
}

template <int D, int NT>
struct Few {
    static constexpr int rows = 8 * NT;
    static constexpr int parts = D / 64;                               // 16-byte parts of a key to a lane
    static constexpr int v_bytes = D / 8;                              // of a value
    static constexpr int k_lane = 2 * parts * 16, lane_bytes = k_lane + 4 * v_bytes;
    static constexpr int stages = D == 64 ? 6 : NT == 1 ? 3 : 6;          // units of a warp that are on their way or read
    static constexpr int stage = 32 * lane_bytes, ring = FEW_WARPS * stages * stage;               // keys, values
    static constexpr int off_q = ring, off_factor = off_q + 2 * rows * D, off_top = off_factor + rows * 4, off_sum = off_top + FEW_WARPS * rows * 4,
                         off_bars = off_sum + FEW_WARPS * rows * 4, bytes = off_bars + FEW_WARPS * stages * 8 + 1024;
    static_assert(FEW_WARPS * rows * D * 4 <= ring, "the warps' sums lie where the copies did");
};

// Where a share's results lie: sums [rows][D], then the largest and the sum of probabilities of each row.
template <int D, int NT>
__device__ __forceinline__ float *share_result(const AttendParams &p, int number, bool from_start)
{
    return p.partial + (size_t)(2 * number + (from_start ? 1 : 0)) * (size_t)(8 * NT * (D + 2));
}

template <int D>
__device__ __forceinline__ void store_out4(const AttendParams &p, size_t at, float4 v)
{
    if (p.out_type == perq_mm::OUT_F32) {
        *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at) = v;
    } else {
        const bool f16 = p.out_type == perq_mm::OUT_F16;
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + at) = make_uint2(pack16(v.x, v.y, f16), pack16(v.z, v.w, f16));
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(THREADS, NT == 1 || D == 64 ? 2 : 1) few_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ AttendParams p)
{
    using K = Few<D, NT>;
    extern __shared__ __align__(128) unsigned char raw[];
    unsigned char *const smem = raw + ((1024u - (perq_mm::smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t base = perq_mm::smem_u32(smem);
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, q = lane & 3;
    int8_t *const q_room = reinterpret_cast<int8_t *>(smem + K::off_q);
    float *const factor = reinterpret_cast<float *>(smem + K::off_factor), *const tops = reinterpret_cast<float *>(smem + K::off_top),
          *const totals = reinterpret_cast<float *>(smem + K::off_sum), *const sums = reinterpret_cast<float *>(smem);
    const uint32_t mine = base + (uint32_t)(warp * K::stages * K::stage), bars = base + K::off_bars + (uint32_t)(warp * K::stages * 8);
    if (lane == 0) {
        perq_mm::prefetch_map(&k_map);
        perq_mm::prefetch_map(&v_map);
        for (uint32_t k = 0; k < K::stages; ++k) perq_mm::mbar_init(bars + 8u * k, 1);
        perq_mm::mbar_init_fence();
    }
    __syncwarp();
    griddep_wait();
    griddep_launch();
    Found f;
    const Share share = share_units<K::rows>(p, (int)blockIdx.x, (int)gridDim.x, f);
    long long unit = share.per * (long long)blockIdx.x;
    const long long unit_end = min(unit + share.per, share.all);
    int i = f.sequence;
    long long begin = f.begin;
    // this lane's places in a unit: 16 channels of a key (and of the one eight further on), channels of four keys' values
    uint32_t k_at[K::parts], v_at[2];
#pragma unroll
    for (int c = 0; c < K::parts; ++c) k_at[c] = swizzled<D>(key_in(g), q + 4 * c);
#pragma unroll
    for (int r = 0; r < 2; ++r) v_at[r] = 16u * D + (D == 128 ? swizzled<D>(key_in(2 * q + r), g) : swizzled<D>(key_in(2 * q + r), g / 2) + (uint32_t)(g & 1) * 8u);
    int slot_in = 0, slot = 0;                                         // of the ring: what is issued, and what is read, next
    uint32_t parity = 0u;                                              // of the ring's barriers, for what is read
    bool ok = true;

    while (unit < unit_end && i < p.q.S) {
        // the tile of this unit
        const Units u = units_of<K::rows>(p, i);
        const long long of_sequence = (long long)u.tiles * u.count * p.heads;
        if (unit >= begin + of_sequence) {
            begin += of_sequence;
            // (the next one with rows: a padded batch has many without)
            for (++i; i < p.q.S; i += 32) {
                const unsigned some = __ballot_sync(0xffffffffu, i + lane < p.q.S && units_of<K::rows>(p, min(i + lane, p.q.S - 1)).tiles > 0);
                if (some != 0u) {
                    i += __ffs(some) - 1;
                    break;
                }
            }
            continue;
        }
        const int number = (int)((unit - begin) / u.count), head = number / u.tiles, row0 = (number - head * u.tiles) * K::rows;
        const long long tile_begin = begin + (long long)number * u.count;
        const int l0 = (int)(unit - tile_begin), l1 = (int)min((long long)u.count, unit_end - tile_begin), rows = min(K::rows, u.tokens * p.group - row0);
        const int first = u.r.length - u.r.n;                          // position of the sequence's first row
        const int low_position = first + row0 / p.group, high_position = first + (row0 + rows - 1) / p.group;
        const int32_t *const table = p.q.pages + (size_t)i * (size_t)p.q.width;
        auto key_of = [&](int l) { return (l < u.sunk ? l : l - u.sunk + u.low) * FEW_KEYS; };
        // of 32 units of this warp, one to a lane: pages, s_k, log2 s_v, 1 / s_v
        const int units = l1 - l0 > warp ? (l1 - l0 - warp + FEW_WARPS - 1) / FEW_WARPS : 0;
        int next_page = 0, later_page = 0;
        float next_step[3] = {0.0f, 0.0f, 0.0f}, step[3] = {0.0f, 0.0f, 0.0f};
        auto fetch = [&](int batch) {
            const int n = batch * 32 + lane, l = l0 + warp + n * FEW_WARPS;
            if (n < units) {
                later_page = min(max(*(table + min(key_of(l) >> p.q.page, p.q.width - 1)), 0), p.q.n_pages - 1);
                const size_t block = (size_t)later_page * (size_t)p.heads + (size_t)head;
                const float vs = *(p.v_steps + block);
                next_step[0] = *(p.k_steps + block);
                next_step[1] = vs < 0x1p-64f ? -64.0f : log2_of(vs);
                next_step[2] = vs < 0x1p-64f ? 0x1p64f : 1.0f / vs;
            }
        };
        auto issue = [&](int n) {
            if (n < units) {
                const int its_page = __shfl_sync(0xffffffffu, next_page, n & 31), key = key_of(l0 + warp + n * FEW_WARPS);
                if (lane == 0) {
                    const uint32_t to = mine + (uint32_t)slot_in * K::stage, bar = bars + 8u * (uint32_t)slot_in;
                    const int line = ((its_page * p.heads + head) << p.q.page) + (key & ((1 << p.q.page) - 1));
                    perq_mm::mbar_expect_tx(bar, K::stage);
                    perq_mm::tma_load(to, &k_map, 0, line, bar);
                    perq_mm::tma_load(to + 16u * D, &v_map, 0, line, bar);
                }
                slot_in = slot_in + 1 == K::stages ? 0 : slot_in + 1;
            }
        };
        fetch(0);
        next_page = later_page;
#pragma unroll
        for (int n = 0; n < K::stages - 1; ++n) issue(n);

        // queries: rotated, then 128 hi + lo with the largest channel 16256
        {
            constexpr int lanes = D / LANE;
            const int row = min(tid / lanes, K::rows - 1), channel = tid % lanes * LANE;
            uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
            if (tid / lanes < rows) {
                const int token = (row0 + row) / p.group, h = (row0 + row) - token * p.group;
                const uint4 *const from = reinterpret_cast<const uint4 *>(p.x + (size_t)(u.r.begin + token) * (size_t)p.stride + (size_t)(head * p.group + h) * D + channel);
                lo = *from;
                hi = *(from + 1);
            }
            float v[LANE], top = 0.0f;
            unpack(v, lo, hi, p.f16 != 0);
            // (by 2^-8 first, which is exact for bf16's smallest too, so that sums of 128 channels do not pass fp32's largest)
#pragma unroll
            for (int k = 0; k < LANE; ++k) v[k] *= 0x1p-8f;
            rotate(v, p.log2b, lane);
#pragma unroll
            for (int k = 0; k < LANE; ++k) asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(fabsf(v[k])));
#pragma unroll
            for (int l = 1; l < lanes; l *= 2) asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(__shfl_xor_sync(0xffffffffu, top, l)));
            // (by a power of two first, so that no reciprocal leaves the range; a row that is not finite has a factor that is not)
            const int e = min(max((int)(__float_as_uint(top) >> 23), 1), 253);
            const float down = __uint_as_float((uint32_t)(254 - e) << 23), scaled = top * down, up = scaled > 0.0f ? 16256.0f / scaled : 0.0f;
            if (tid / lanes < K::rows) {
                uint32_t w[2][4] = {};
#pragma unroll
                for (int k = 0; k < LANE; ++k) {
                    const int n = __float2int_rn(v[k] * down * up), high = (n + 64) >> 7;
                    w[0][k / 4] |= (uint32_t)(uint8_t)high << (8 * (k % 4));
                    w[1][k / 4] |= (uint32_t)(uint8_t)(n - 128 * high) << (8 * (k % 4));
                }
#pragma unroll
                for (int plane = 0; plane < 2; ++plane)
                    *reinterpret_cast<uint4 *>(q_room + (plane * K::rows + row) * D + channel) = make_uint4(w[plane][0], w[plane][1], w[plane][2], w[plane][3]);
                if (channel == 0) factor[row] = scaled * (256.0f / 16256.0f) * __uint_as_float((uint32_t)e << 23) * p.scale;
            }
        }
        __syncthreads();
        uint32_t qb[NT][2][4 * K::parts];                              // [tile][hi, lo]
        float row_factor[NT][2];
        int position[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int plane = 0; plane < 2; ++plane)
#pragma unroll
                for (int c = 0; c < K::parts; ++c) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(q_room + (plane * K::rows + t * 8 + g) * D + 16 * (q + 4 * c));
                    qb[t][plane][4 * c] = w.x; qb[t][plane][4 * c + 1] = w.y; qb[t][plane][4 * c + 2] = w.z; qb[t][plane][4 * c + 3] = w.w;
                }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int row = t * 8 + 2 * q + c;
                row_factor[t][c] = factor[row];
                position[t][c] = row < rows ? first + (row0 + row) / p.group : -1;
            }
        }
        float o[NT][D / 16][4], top[NT][2], total[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][j][e] = 0.0f;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                top[t][c] = -INFINITY;
                total[t][c] = 0.0f;
            }
        }

        for (int n = 0; n < units; ++n) {
            if ((n & 31) == 0) {
#pragma unroll
                for (int k = 0; k < 3; ++k) step[k] = next_step[k];
            }
            // (of the next 32 units, well before the first of them is issued)
            if ((n & 31) == 16) fetch((n >> 5) + 1);
            if ((n & 31) == 33 - K::stages) next_page = later_page;
            __syncwarp();                                              // (all lanes have read what lay where the next copy goes)
            issue(n + K::stages - 1);
            if (!perq_mm::mbar_wait_warp(bars + 8u * (uint32_t)slot, parity)) ok = false;
            const uint32_t at = mine + (uint32_t)slot * K::stage;
            slot = slot + 1 == K::stages ? 0 : slot + 1;
            parity ^= slot == 0 ? 1u : 0u;
            if (!ok) continue;                                         // (the other copies are waited for all the same)
            const float ks = __shfl_sync(0xffffffffu, step[0], n & 31), log_step = __shfl_sync(0xffffffffu, step[1], n & 31), inverse = __shfl_sync(0xffffffffu, step[2], n & 31);
            int32_t acc[NT][2][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][0][e] = acc[t][1][e] = 0;
            // (all that is read of the unit is on its way before the first of it is used)
            uint4 x[K::parts], y[K::parts];
#pragma unroll
            for (int c = 0; c < K::parts; ++c) {
                x[c] = lds128(at + k_at[c]);
                y[c] = lds128(at + k_at[c] + 8u * D);
            }
            uint32_t v[4][D / 32];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (D == 128) {
                    const uint4 w = lds128(at + v_at[r & 1] + (uint32_t)(r >> 1) * 8u * D);
                    v[r][0] = w.x; v[r][1] = w.y; v[r][2] = w.z; v[r][3] = w.w;
                } else {
                    const uint2 w = lds64(at + v_at[r & 1] + (uint32_t)(r >> 1) * 8u * D);
                    v[r][0] = w.x; v[r][1] = w.y;
                }
            }
#pragma unroll
            for (int c = 0; c < K::parts; ++c)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int plane = 0; plane < 2; ++plane) {
                        mma_i8(acc[t][plane], x[c].x, y[c].x, x[c].y, y[c].y, qb[t][plane][4 * c], qb[t][plane][4 * c + 1]);
                        mma_i8(acc[t][plane], x[c].z, y[c].z, x[c].w, y[c].w, qb[t][plane][4 * c + 2], qb[t][plane][4 * c + 3]);
                    }
            const int key = key_of(l0 + warp + n * FEW_WARPS);
            const bool edge = key + FEW_KEYS - 1 > low_position || (p.window > 0 && key <= high_position - p.window && key + FEW_KEYS > p.sinks);
            float s[NT][4], over = -INFINITY;
            auto exponents = [&]() {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const float ff[2] = {row_factor[t][0] * ks, row_factor[t][1] * ks};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int c = e & 1;
                        // (two steps, so that the largest, which the reference was made of, is no further from it than it was then, however large both are)
                        s[t][e] = fmaf((float)(128 * acc[t][0][e] + acc[t][1][e]), ff[c], log_step) - top[t][c];
                        if (edge) {
                            const int j = key + key_in(g) + 8 * (e >> 1), at_row = position[t][c];
                            if (j > at_row || (p.window > 0 && j <= at_row - p.window && j >= p.sinks)) s[t][e] = -INFINITY;
                        }
                        over = fmaxf(over, s[t][e]);
                    }
                }
            };
            exponents();
            // (a row that has seen nothing has the reference -inf, so everything is over)
            if (__any_sync(0xffffffffu, over > P_MOST)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        // logits without the reference
                        const float ff = row_factor[t][c] * ks;
                        float m = -INFINITY;
#pragma unroll
                        for (int e = c; e < 4; e += 2)
                            if (s[t][e] != -INFINITY) m = fmaxf(m, fmaf((float)(128 * acc[t][0][e] + acc[t][1][e]), ff, log_step));
#pragma unroll
                        for (int l = 4; l < 32; l *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, l));
                        m = fmaxf(m - P_LIFT, top[t][c]);
                        const float alpha = m == -INFINITY ? 1.0f : exp2_of(top[t][c] - m);
                        top[t][c] = m;
                        total[t][c] *= alpha;
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) {
                            o[t][j][c] *= alpha;
                            o[t][j][c + 2] *= alpha;
                        }
                    }
                exponents();
            }
            uint32_t pb[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][e] = exp2_of(s[t][e]);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float sum = s[t][c] + s[t][c + 2];
                    if (sum != 0.0f) total[t][c] = fmaf(sum, inverse, total[t][c]);          // (a step that is not finite stays with the rows that see it)
                }
                pb[t][0] = transposed(half2_of(s[t][0], s[t][1]));
                pb[t][1] = transposed(half2_of(s[t][2], s[t][3]));
            }
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                constexpr uint32_t pick[4] = {0x0400u, 0x0501u, 0x0602u, 0x0703u};
                const int w = j / 2, b = 2 * (j % 2);
                const uint32_t a0 = codes_f16(__byte_perm(v[0][w], v[1][w], pick[b])), a1 = codes_f16(__byte_perm(v[0][w], v[1][w], pick[b + 1]));
                const uint32_t a2 = codes_f16(__byte_perm(v[2][w], v[3][w], pick[b])), a3 = codes_f16(__byte_perm(v[2][w], v[3][w], pick[b + 1]));
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_f16(o[t][j], a0, a1, a2, a3, pb[t][0], pb[t][1]);
            }
        }
        if (!ok && lane == 0) atomicOr(&perq_mm::g_error, ERROR_ATTEND);

        // the warps' results become one
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int l = 4; l < 32; l *= 2) total[t][c] += __shfl_xor_sync(0xffffffffu, total[t][c], l);
                if (g == 0) {
                    tops[warp * K::rows + t * 8 + 2 * q + c] = top[t][c];
                    totals[warp * K::rows + t * 8 + 2 * q + c] = total[t][c];
                }
            }
        __syncthreads();
        // (a lane has channels (D / 8) g + 2 j and one more of rows 2 q and 2 q + 1)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float *const to = sums + ((size_t)warp * K::rows + (size_t)(t * 8 + 2 * q + c)) * D + g * K::v_bytes;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) *reinterpret_cast<float2 *>(to + 2 * j) = make_float2(o[t][j][c], o[t][j][c + 2]);
            }
        __syncthreads();
        const bool whole_row = l0 == 0 && l1 == u.count;
        float *const result = share_result<D, NT>(p, (int)blockIdx.x, l0 == 0);
        for (int k = tid; k < K::rows * D / 4; k += THREADS) {
            const int row = k / (D / 4), channel = k % (D / 4) * 4;
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int w = 0; w < FEW_WARPS; ++w) m = fmaxf(m, tops[w * K::rows + row]);
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < FEW_WARPS; ++w) {
                const float mw = tops[w * K::rows + row], a = mw == -INFINITY ? (m == -INFINITY ? 1.0f : 0.0f) : exp2_of(mw - m);
                const float4 x = *reinterpret_cast<const float4 *>(sums + ((size_t)w * K::rows + (size_t)row) * D + channel);
                l = fmaf(a, totals[w * K::rows + row], l);
                v.x = fmaf(a, x.x, v.x); v.y = fmaf(a, x.y, v.y); v.z = fmaf(a, x.z, v.z); v.w = fmaf(a, x.w, v.w);
            }
            if (whole_row) {
                if (row >= rows) continue;
                const float r = l == 0.0f ? 0.0f : 1.0f / l;
                const int token = (row0 + row) / p.group, h = (row0 + row) - token * p.group;
                store_out4<D>(p, ((size_t)(u.r.begin + token) * (size_t)(p.heads * p.group) + (size_t)(head * p.group + h)) * D + (size_t)channel,
                              make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
            } else {
                *reinterpret_cast<float4 *>(result + row * D + channel) = v;
                if (channel == 0) {
                    result[K::rows * D + row] = m;
                    result[K::rows * D + K::rows + row] = l;
                }
            }
        }
        perq_mm::fence_async_smem();                                   // (before the next tile's copies)
        __syncthreads();
        unit = tile_begin + l1;
    }
}

// Results of parts of a row's keys, weighted: 4 rows of `parts` results, whose sums lie at `sums_of(part)` (row, then channels), and their references and probabilities at `ends_of(part)`
// ([row], [row + stride]).  `finish(row, channel, v)` gets four channels of a row.  Called by all threads of the CTA, which has 4 * parts + 4 floats and 16 * THREADS bytes of shared memory
// at `room`.  Loads of eight parts are on their way at once: one after another they were most of the time (a token behind 1000: 8.9 us, two behind 130000 16).
constexpr int JOIN_ROWS = 4;
template <int D, typename Sums, typename Ends, typename Finish>
__device__ __forceinline__ void join_rows(float *room, int parts, int stride, const Sums &sums_of, const Ends &ends_of, const Finish &finish)
{
    constexpr int items = JOIN_ROWS * D / 4, lots = THREADS / items;   // of four channels; threads to one
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5;
    float *const weights = room + 4 * THREADS, *const inverse = weights + JOIN_ROWS * parts;
    if (warp < JOIN_ROWS) {
        float m = -INFINITY, l = 0.0f;
        for (int c = lane; c < parts; c += 32) {
            const float x = ends_of(c)[warp];
            weights[c * JOIN_ROWS + warp] = x;
            m = fmaxf(m, x);
        }
#pragma unroll
        for (int k = 16; k > 0; k /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
        for (int c = lane; c < parts; c += 32) {
            const float x = weights[c * JOIN_ROWS + warp], a = x == -INFINITY ? (m == -INFINITY ? 1.0f : 0.0f) : exp2_of(x - m);
            weights[c * JOIN_ROWS + warp] = a;
            l = fmaf(a, ends_of(c)[stride + warp], l);
        }
#pragma unroll
        for (int k = 16; k > 0; k /= 2) l += __shfl_xor_sync(0xffffffffu, l, k);
        if (lane == 0) inverse[warp] = l == 0.0f ? 0.0f : 1.0f / l;
    }
    __syncthreads();
    const int item = tid % items, lot = tid / items, row = item / (D / 4), channel = item % (D / 4) * 4;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int c0 = lot; c0 < parts; c0 += 8 * lots) {
        float4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = c0 + k * lots;
            x[k] = c < parts ? *reinterpret_cast<const float4 *>(sums_of(c) + row * D + channel) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = c0 + k * lots;
            const float a = c < parts ? weights[c * JOIN_ROWS + row] : 0.0f;
            v.x = fmaf(a, x[k].x, v.x); v.y = fmaf(a, x[k].y, v.y); v.z = fmaf(a, x[k].z, v.z); v.w = fmaf(a, x[k].w, v.w);
        }
    }
    float4 *const others = reinterpret_cast<float4 *>(room);
    others[tid] = v;
    __syncthreads();
    if (lot == 0) {
#pragma unroll
        for (int k = 1; k < lots; ++k) {
            const float4 x = others[item + k * items];
            v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        }
        const float r = inverse[row];
        finish(row, channel, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
    }
}
inline size_t join_bytes(int parts) { return (size_t)(4 * THREADS + JOIN_ROWS * parts + JOIN_ROWS) * 4; }

// Tiles whose units several CTAs had: CTA (b, y) puts four rows of the one together that its boundary, between shares b and b + 1, is the first to cut.
template <int D, int NT>
__global__ void __launch_bounds__(THREADS) join_kernel(const __grid_constant__ AttendParams p, int ctas)
{
    using K = Few<D, NT>;
    extern __shared__ __align__(16) float room[];
    // (what the sequences are is read before the wait: the kernel before this one let it start after its own wait, so whatever made them has ended, and it writes none of it)
    Found f;
    const Share share = share_units<K::rows>(p, (int)blockIdx.x + 1, ctas, f);
    griddep_wait();
    griddep_launch();
    const long long boundary = share.per * (long long)(blockIdx.x + 1);
    if (boundary >= share.all) return;
    const Units u = units_of<K::rows>(p, f.sequence);
    const int number = (int)((boundary - f.begin) / u.count), head = number / u.tiles, row0 = (number - head * u.tiles) * K::rows + (int)blockIdx.y * JOIN_ROWS;
    const long long tile_begin = f.begin + (long long)number * u.count, tile_end = tile_begin + u.count;
    if (tile_begin == boundary || tile_begin < boundary - share.per) return;
    const int rows = u.tokens * p.group - row0, c0 = (int)blockIdx.x, c1 = (int)((tile_end - 1) / share.per);
    if (rows <= 0) return;
    auto result_of = [&](int c) { return share_result<D, NT>(p, c0 + c, c == 0) + (int)blockIdx.y * JOIN_ROWS * D; };
    join_rows<D>(room, c1 - c0 + 1, K::rows, result_of, [&](int c) { return share_result<D, NT>(p, c0 + c, c == 0) + K::rows * D + (int)blockIdx.y * JOIN_ROWS; },
                 [&](int row, int channel, float4 v) {
                     if (row >= rows) return;
                     const int token = (row0 + row) / p.group, h = (row0 + row) - token * p.group;
                     store_out4<D>(p, ((size_t)(u.r.begin + token) * (size_t)(p.heads * p.group) + (size_t)(head * p.group + h)) * D + (size_t)channel, v);
                 });
}

}  // namespace perq_kv
