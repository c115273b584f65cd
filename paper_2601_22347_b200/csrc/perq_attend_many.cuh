// Attention over the 8-bit cache for many queries to a sequence: prompts and chunks of them, on the fifth-generation tensor cores.
//
// A work is 256 rows (pairs of a token and one of the `group` heads of queries to a head of keys), two tiles of 128, over the keys they see, 128 at a time.  Bulk copies bring codes in, a page
// at a time, keys and values in turn; four warps make them fp16 (exactly: code ^ 0x80 in the low bits of 1024, minus 1152) and lay them down as operands, in a ring; one warp issues the
// products: S = Q K^T into tensor memory, then O += P V with P from tensor memory and V's rows as they are (its channels run along N).  Either tile has four warps of its own, a row to a
// thread, which take 64 keys at a time: their maximum, P = 2^(x + log2 s_v - m) rounded to fp16 over the columns where S was, and the probabilities' sum in fp32.  S has room for 64 keys
// twice, so the products with the last 64 and for the next run under the exponentials of these.  O stays in tensor memory; m, which is 7 below the largest so far, moves, and O with it, only
// when something is over 2^15 (as in the kernel for few queries).  A CTA takes the work of others that have not begun (next_cta), and its loads and conversions run ahead into it.
//
// Floors: 4 D operations a pair of a row and a key it sees, at the tensor cores' rate.  From a graph, chunks of up to 512 tokens behind 16000, 32 heads of 128: 284 us, 833 TFLOP/s of 1667; two prompts of
// up to 8192 272, 835 (in calls on inputs in turn 302 and 286).  No unit bounds it: a step of 64 keys of both tiles takes about 2000 cycles, and the products or the exponentials 1024 each.  With
// something left out, the chunks' and the prompts' times are less by: exponentials 6 and 9 %, codes to fp16 6 and 6, maxima nothing, sums nothing, exponentials with products 17 and 14, exponentials with
// maxima and sums 11 and 12, these with reading S and the products too 21 and 24.  So three quarters are what is left then: the steps' waits for one another, P to tensor memory, codes to fp16, loads.
// (64 registers of S to a thread leave no room for the next step's beside them; ptxas spills 28 bytes at D = 128.)
// What did not help: two threads to a row and 128 keys (the same); the maximum of P instead of S, with a second try where it was too large (349 -> 399 us); the
// next S read under the exponentials (303 -> 326, registers); sleeping waits (+4 %); one exponential in four on the multiply-add pipe (310, in eight 298); heads in the inner order (+3 %).
#pragma once

#include "perq_attend_few.cuh"

namespace perq_kv {

constexpr int CODES_WARP = 8, MMA_WARP = 12, LOAD_WARP = 13; // warps: 8 of the rows, 4 that make codes fp16, the products', the loads', 2 idle
constexpr int MANY_ROWS = 256, MANY_KEYS = 128, MANY_THREADS = 512;

struct ManyParams {
    AttendParams a;
    float *partial;                           // [item][split][256][D + 2], where the keys of an item are split over CTAs
    int32_t split;
};

template <int D>
struct Many {
    static constexpr uint32_t tile = 128u * D * 2u, raw = 128u * D;    // bytes of 128 rows of fp16, of codes
    static constexpr uint32_t half = 128u * 128u;                      // of 64 channels of the former
    static constexpr uint32_t stages = D == 128 ? 4 : 8, raw_stages = D == 128 ? 2 : 4;
    static constexpr uint32_t off_ring = 2u * tile, off_raw = off_ring + stages * tile, off_steps = off_raw + raw_stages * raw;
    static constexpr uint32_t off_bars = off_steps + 8u * 8u * 16u;
    static constexpr uint32_t bars = 2u * stages + 2u * raw_stages + 8u + 2u + 4u + 4u + 2u + 2u + 2u + 4u + 1u + 1u;   // operands, codes: full, empty; steps; Q, S and P (twice), O, all of O, results of each tile; works; the next one; the end
    static constexpr uint32_t off_slot = (off_bars + 8u * bars + 15u) & ~15u, off_next = off_slot + 16u, bytes = off_next + 16u + 1024u;
    static constexpr uint32_t columns = 512u;                          // S0, S1, O0, O1
    static constexpr uint32_t o_column = 256u;
};

// kind::f16, fp16 operands, fp32 sums; values' channels run along N (the second operand's rows are keys).
__host__ __device__ constexpr uint32_t f16_desc(int m, int n, bool second_transposed)
{
    return (1u << 4) | ((uint32_t)second_transposed << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// Waits of whole warps for barriers that only this CTA's threads and copies arrive at.
__device__ __forceinline__ bool cta_poll(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0u;
}
__device__ __forceinline__ bool cta_wait_warp(uint32_t bar, uint32_t parity)
{
    bool done = cta_poll(bar, parity);
    for (uint32_t i = 0; i < perq_mm::WAIT_POLLS && !done; ++i) done = cta_poll(bar, parity);
    return __all_sync(0xffffffffu, done);
}
// By whole warps, of which one lane issues: what describes a product then stays in uniform registers.  (A lane of its own, with the warps that compute exponentials on the
// same scheduler: 380 cycles to an instruction of 64.)
__device__ __forceinline__ void product_f16(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{ .reg .pred p, q; .reg .b64 a, b; setp.ne.b32 p, %4, 0; mov.b64 a, {%1, %5}; mov.b64 b, {%2, %5}; elect.sync _|q, 0xffffffff; "
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p; }"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(perq_mm::OPERAND_HI) : "memory");
}
__device__ __forceinline__ void product_f16_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{ .reg .pred p, q; .reg .b64 b; setp.ne.b32 p, %4, 0; mov.b64 b, {%2, %5}; elect.sync _|q, 0xffffffff; "
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p; }"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(perq_mm::OPERAND_HI) : "memory");
}
__device__ __forceinline__ void commit_one(uint32_t bar)
{
    asm volatile("{ .reg .pred q; elect.sync _|q, 0xffffffff; @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(bar) : "memory");
}
// A tile of [128 rows][64 channels] halves: as an operand whose rows are M or N, and as one whose rows are K (64 channels of N, then those a half further on).
__device__ __forceinline__ uint32_t rows_operand(uint32_t addr) { return ((addr >> 4) & 0x3fffu) | (1u << 16); }
template <int D>
__device__ __forceinline__ uint32_t keys_operand(uint32_t addr) { return ((addr >> 4) & 0x3fffu) | ((Many<D>::half >> 4) << 16); }

// For two barriers, polled before either answer is looked at.
__device__ __forceinline__ bool cta_wait_warp(uint32_t bar, uint32_t parity, uint32_t bar1, uint32_t parity1)
{
    const bool done = cta_poll(bar, parity), done1 = cta_poll(bar1, parity1);
    if (__all_sync(0xffffffffu, done && done1)) return true;
    return cta_wait_warp(bar, parity) && cta_wait_warp(bar1, parity1);
}
// 2^x on the multiply-add pipe, for x up to 100: 2^(x - n) with n the nearest whole number by its Taylor polynomial of degree 5 (off by (ln2 / 2)^6 / 6! = 2.4e-6), times 2^n.  One in
// eight exponentials is taken so, because the others are what two warps of a scheduler wait for (16 a cycle and SM): chunks behind long contexts 310 -> 298 us; one in four 310.  Below -125: 0.
// (NaN need not stay NaN: rows that have one carry it in their sum.)
__device__ __forceinline__ float exp2_fma(float x)
{
    const float t = x + 12582912.0f, f = x - (t - 12582912.0f);
    float r = fmaf(f, 1.3333558e-3f, 9.6181291e-3f);
    r = fmaf(r, f, 5.5504109e-2f);
    r = fmaf(r, f, 2.4022651e-1f);
    r = fmaf(r, f, 6.9314718e-1f);
    r = fmaf(r, f, 1.0f);
    r = __int_as_float(__float_as_int(r) + (__float_as_int(t) << 23));
    return x < -125.0f ? 0.0f : r;
}
// The index of a CTA of the grid that has not begun and does not any more, as this one takes its work; -1: there is none left.  (The device gives them out in order, so CTAs that are done
// early take more; every gridDim-th work to a CTA instead: two prompts of up to 8192 tokens 340 us, 301 with a CTA to a work.)
__device__ __forceinline__ int next_cta(uint32_t room, uint32_t bar, uint32_t parity, int lane, bool &ok)
{
    if (lane == 0) {
        perq_mm::mbar_expect_tx(bar, 16u);
        asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(room), "r"(bar) : "memory");
    }
    __syncwarp();
    ok = cta_wait_warp(bar, parity);
    if (!ok) return -1;
    uint32_t yes, x, y, z;           // (y and z are 0)
    asm volatile("{ .reg .b128 h; .reg .pred p; ld.shared.b128 h, [%4]; clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h; selp.u32 %0, 1, 0, p; mov.u32 %1, 0; mov.u32 %2, 0; "
                 "mov.u32 %3, 0; @p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, %2, %3, _}, h; }"
                 : "=r"(yes), "=r"(x), "=r"(y), "=r"(z) : "r"(room) : "memory");
    perq_mm::fence_async_smem();                                       // (the next answer is written where this one was)
    __syncwarp();
    return yes ? (int)(x + y + z) : -1;
}
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t minus_1152(uint32_t v)
{
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0x64806480u));
    return r;
}
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

// Two fp32 values in one register pair, added and multiplied at once.
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
    int32_t part, tile0, count;               // where the keys are split: this CTA's part of the tiles
    int32_t number;                           // of the item: where its parts lie
};
__device__ __forceinline__ int many_tiles(const AttendParams &p, const Rows &r)
{
    const long long rows = (long long)min(r.n, p.most) * p.group;
    return rows > p.few_rows ? (int)((rows + MANY_ROWS - 1) / MANY_ROWS) : 0;
}
// The number-th tile of rows of the call, head by head and a sequence's last tile first: those see most.  Up to 32 sequences also go by the most that they see, so that the CTAs that
// come last have little to do (four chunks of 226 to 478 tokens behind 5.7 to 12.7 thousand: 382 us in their own order).  By one warp.
__device__ __forceinline__ ManyItem many_item(const AttendParams &p, int number, int lane)
{
    const int head = number % p.heads, tile = number / p.heads;
    ManyItem it;
    it.rows = 0;
    for (int base = 0, before = 0; base < p.q.S && before <= tile; base += 32) {
        Rows r = {0, 0, 0};
        int c = 0;
        if (base + lane < p.q.S) {
            r = rows_of(p.q, base + lane);
            c = many_tiles(p, r);
        }
        const int seen = p.window > 0 ? min(r.length, p.window + r.n) : r.length;
        int first = 0, all = 0;
#pragma unroll
        for (int l = 0; l < 32; ++l) {
            const int cl = __shfl_sync(0xffffffffu, c, l), sl = __shfl_sync(0xffffffffu, seen, l);
            all += cl;
            if (p.q.S <= 32 ? sl > seen || (sl == seen && l < lane) : l < lane) first += cl;
        }
        const int at = tile - before - first;
        const unsigned mine = __ballot_sync(0xffffffffu, at >= 0 && at < c);
        if (mine != 0u) {
            const int tokens = min(r.n, p.most);
            it.sequence = base + lane;
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
            const int owner = __ffs(mine) - 1;
            int *const words = reinterpret_cast<int *>(&it);
#pragma unroll
            for (int i = 0; i < (int)(sizeof(ManyItem) / sizeof(int)); ++i) words[i] = __shfl_sync(0xffffffffu, words[i], owner);
            return it;
        }
        before += all;
    }
    return it;
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
    __shared__ ManyItem found[2];
    const uint32_t full = base + K::off_bars, empty = full + 8u * K::stages, raw_full = empty + 8u * K::stages, raw_empty = raw_full + 8u * K::raw_stages,
                   steps_full = raw_empty + 8u * K::raw_stages, q_full = steps_full + 64u, s_full = q_full + 16u, p_full = s_full + 32u, o_full = p_full + 32u, o_done = o_full + 16u,
                   stored = o_done + 16u, work_full = stored + 16u, work_empty = work_full + 16u, next_full = work_empty + 16u, end = next_full + 8u, slot = base + K::off_slot, steps = base + K::off_steps;
    if (tid == 0) {
        for (uint32_t i = 0; i < K::stages; ++i) {
            mbar_init(full + 8u * i, 4);                               // the warps that make codes fp16
            mbar_init(empty + 8u * i, 1);
        }
        for (uint32_t i = 0; i < K::raw_stages; ++i) {
            mbar_init(raw_full + 8u * i, 1);
            mbar_init(raw_empty + 8u * i, 4);
        }
        for (uint32_t i = 0; i < 8; ++i) mbar_init(steps_full + 8u * i, 1);
        for (uint32_t i = 0; i < 2; ++i) {
            mbar_init(q_full + 8u * i, 4);
            mbar_init(o_full + 8u * i, 1);
            mbar_init(o_done + 8u * i, 1);
            mbar_init(stored + 8u * i, 4);
            mbar_init(work_full + 8u * i, 1);
            mbar_init(work_empty + 8u * i, MMA_WARP + 1);             // all that read it
        }
        for (uint32_t i = 0; i < 4; ++i) {
            mbar_init(s_full + 8u * i, 1);
            mbar_init(p_full + 8u * i, 4);
        }
        mbar_init(next_full, 1);
        mbar_init(end, 1);
        mbar_init_fence();
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(K::columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = lds32(slot);
    auto give_up = [&]() { atomicOr(&g_error, ERROR_ATTEND); };
    auto key_of = [](const ManyItem &it, int tile) { return (tile < it.sunk ? tile : tile - it.sunk + it.low) * MANY_KEYS; };
    // The number-th work of this CTA, which the loads' warp looks for ahead; rows of 0: there are no more.
    auto work_of = [&](uint32_t number, ManyItem &it) {
        if (!cta_wait_warp(work_full + 8u * (number & 1u), (number >> 1) & 1u)) {
            if (lane == 0) give_up();
            return false;
        }
        it = found[number & 1u];
        __syncwarp();
        if (lane == 0) mbar_arrive(work_empty + 8u * (number & 1u));
        return it.rows > 0;
    };

    if (warp < CODES_WARP) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");          // (of 128 at launch: 2 x 176 + 80 + 80 = 4 x 128)
        const int t = warp >> 2, row = t * 128 + (tid & 127);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, o_at = tmem + K::o_column + (uint32_t)t * 128u + lanes;
        ManyItem it;
        bool ok = true;
        uint32_t mine = 0u, j0 = 0u, done = 0u;                        // of this tile of rows: works, tiles of keys, works with some, so far
        uint32_t global0 = 0u, next0 = 0u;                             // tiles of keys of the CTA before this work, and behind it
        for (uint32_t work = 0; ok && work_of(work, it); ++work) {
            global0 = next0;
            next0 += (uint32_t)it.count;
            if (t * 128 >= it.rows) continue;
            const int tile0 = it.tile0, tiles = it.count, position = it.first + (it.row0 + min(row, it.rows - 1)) / p.a.group;
            // (the four warps' rows of queries lie where others' results did)
            if (mine > 0 && !cta_wait_warp(stored + 8u * (uint32_t)t, (mine - 1u) & 1u)) {
                ok = false;
                break;
            }
            ++mine;
            // Queries: 32 rows to a warp, 16 channels to a lane; a row's largest is scaled to 1 .. 2 by a power of two, then it is rotated and rounded to fp16.
            // (A row to a thread: 12 us of loads that touch 32 rows each.)
            float factor = 0.0f, l = 0.0f;                             // (l: of probabilities)
            if (tiles > 0) {
                constexpr int wide = D / LANE, at_once = 32 / wide;    // lanes of a row, rows at once
                const int in = lane / wide, channel = lane % wide * LANE, first_row = (warp & 3) * 32;
#pragma unroll 1
                for (int k0 = 0; k0 < 32 / at_once; k0 += 4) {
                    uint4 lo[4], hi[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = t * 128 + first_row + (k0 + k) * at_once + in, its_token = (it.row0 + r) / p.a.group, its_head = it.row0 + r - its_token * p.a.group;
                        lo[k] = hi[k] = make_uint4(0, 0, 0, 0);
                        if (r < it.rows) {
                            const uint4 *const from = reinterpret_cast<const uint4 *>(p.a.x + (size_t)(it.begin + its_token) * (size_t)p.a.stride +
                                                                                      (size_t)(it.head * p.a.group + its_head) * D + channel);
                            lo[k] = *from;
                            hi[k] = *(from + 1);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float v[LANE], most = 0.0f;
                        unpack(v, lo[k], hi[k], p.a.f16 != 0);
#pragma unroll
                        for (int i = 0; i < LANE; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(fabsf(v[i])));
#pragma unroll
                        for (int k1 = 1; k1 < wide; k1 *= 2) asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(__shfl_xor_sync(0xffffffffu, most, k1)));
                        const int e = min(max((int)(__float_as_uint(most) >> 23), 1), 253);
                        // (with the sign of the logits' scale, as a page's largest logit has to be that of its largest S)
                        const float down = copysignf(__uint_as_float((uint32_t)(254 - e) << 23), p.a.scale);
#pragma unroll
                        for (int i = 0; i < LANE; ++i) v[i] *= down;
                        rotate(v, p.a.log2b, lane);
                        const uint32_t r = (uint32_t)(first_row + (k0 + k) * at_once + in), c = (uint32_t)(channel % 64) / 8u;
                        const uint32_t to = base + (uint32_t)t * K::tile + (uint32_t)(channel / 64) * K::half + r * 128u;
                        sts128(to + ((c ^ r) & 7u) * 16u, make_uint4(half2_of(v[0], v[1]), half2_of(v[2], v[3]), half2_of(v[4], v[5]), half2_of(v[6], v[7])));
                        sts128(to + (((c + 1u) ^ r) & 7u) * 16u, make_uint4(half2_of(v[8], v[9]), half2_of(v[10], v[11]), half2_of(v[12], v[13]), half2_of(v[14], v[15])));
                        // (the lane of the row has its factor.  A query that is not finite makes the sum of probabilities NaN, unless the row sees nothing)
                        const float top = __shfl_sync(0xffffffffu, most, (lane % at_once) * wide);
                        if (lane / at_once == k0 + k) {
                            factor = fminf(__uint_as_float(min(max(__float_as_uint(top) >> 23, 1u), 253u) << 23) * fabsf(p.a.scale), 3.4028235e38f);
                            if (!(top <= 3.4028235e38f) && position >= 0) l = __uint_as_float(0x7fffffffu);
                        }
                    }
                }
            }
            if (tiles > 0) {
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full + 8u * (uint32_t)t);
            }

            // rows of this warp: all of a tile's keys that its rows have in common
            const int row_first = it.row0 + t * 128 + (warp & 3) * 32, row_last = it.row0 + it.rows - 1;
            const int low_position = it.first + min(row_first, row_last) / p.a.group, high_position = it.first + min(row_first + 31, row_last) / p.a.group;
            float m = -INFINITY;
            float limit = P_MOST;                                      // (of the warp: none where m is far from 0)
            for (int u = 0; u < 2 * tiles; ++u) {
                const int side = u & 1, key = key_of(it, tile0 + (u >> 1)) + 64 * side;
                const uint32_t j = j0 + (uint32_t)(u >> 1), global = global0 + (uint32_t)(u >> 1);
                const uint32_t s_at = tmem + (uint32_t)(t * 128 + side * 64) + lanes, buffer = 8u * (uint32_t)(2 * t + side);
                if (!cta_wait_warp(steps_full + 8u * (global & 7u), (global >> 3) & 1u, s_full + buffer, j & 1u)) {
                    ok = false;
                    break;
                }
                tmem_fence_after();
                float s[2][32];
                tmem_load32(s_at, s[0]);
                tmem_load32(s_at + 32u, s[1]);
                constexpr int G = FINE ? 4 : 2, W = 64 / G;
                // of a page's columns: the factor of S (at least 2^-120, so that what is not seen stays -inf: |S| < 2^23), log2 s_v, 1 / s_v
                const uint32_t at = steps + (global & 7u) * 128u + (uint32_t)side * 64u;
                float f[G], b[G], inverse[G];
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const uint4 w = lds128(at + (uint32_t)(g * (4 / G)) * 16u);
                    f[g] = fmaxf(factor * __uint_as_float(w.x), 0x1p-120f);
                    b[g] = __uint_as_float(w.y);
                    inverse[g] = __uint_as_float(w.z);
                    if (w.w != 0u) {
                        // a step that is not finite: so is what sees one of its keys
                        const int k0 = key + g * W, k1 = min(k0 + W - 1, position);
                        if (k0 <= position && (p.a.window <= 0 || k1 > position - p.a.window || k0 < p.a.sinks)) l = __uint_as_float(0x7fffffffu);
                    }
                }
                loads_wait(s[0]);
                loads_there(s[1]);
                if (key + 63 > low_position || (p.a.window > 0 && key <= high_position - p.a.window && key + 64 > p.a.sinks)) {
                    // what this row does not see, a bit each
                    const int last = position - key, low = p.a.window > 0 ? last - p.a.window : -1, sunk = p.a.sinks - key;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const uint32_t seen = bits_below(last + 1 - 32 * c) & (~bits_below(low + 1 - 32 * c) | (p.a.window > 0 ? bits_below(sunk - 32 * c) : 0u));
#pragma unroll
                        for (int i = 0; i < 32; ++i) s[c][i] = seen & (1u << i) ? s[c][i] : -INFINITY;
                    }
                }
                float most_x = -INFINITY;
                {
                    // (chains of their own, as each step of one waits for the last)
                    float top[4];
#pragma unroll
                    for (int g = 0; g < 4; ++g) top[g] = fmaxf(s[g / 2][16 * (g % 2)], s[g / 2][16 * (g % 2) + 1]);
#pragma unroll
                    for (int i = 2; i < 16; i += 2)
#pragma unroll
                        for (int g = 0; g < 4; ++g) top[g] = max_of3(top[g], s[g / 2][16 * (g % 2) + i], s[g / 2][16 * (g % 2) + i + 1]);
#pragma unroll
                    for (int g = 0; g < G; ++g) most_x = fmaxf(most_x, fmaf(FINE ? top[g] : fmaxf(top[2 * g % 4], top[(2 * g + 1) % 4]), f[g], b[g]));
                }
                if (__any_sync(0xffffffffu, most_x - m > limit)) {
                    const float next = fmaxf(m, most_x - P_LIFT), alpha = next == -INFINITY ? 1.0f : exp2_of(m - next);
                    m = next;
                    limit = __any_sync(0xffffffffu, fabsf(m) > 0x1p16f && m != -INFINITY) ? -INFINITY : P_MOST;
                    l *= alpha;
                    if (u > 0) {
                        if (!cta_wait_warp(o_full + 8u * (uint32_t)t, (uint32_t)(u - 1) & 1u)) {
                            ok = false;
                            break;
                        }
                        tmem_fence_after();
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) {
                            int32_t o[16];
                            uint32_t w[16];
                            tmem_load16(o_at + 16u * c, o);
                            tmem_wait(o);
#pragma unroll
                            for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(__int_as_float(o[i]) * alpha);
                            tmem_store16(o_at + 16u * c, w);
                        }
                    }
                    if (limit != P_MOST) {
                        // In one step b - m is rounded first, by up to 2^-24 of m: not what the largest is over it, if that is no small part of 1.  So here in two.
                        const float reference = m == -INFINITY ? 0.0f : m;
#pragma unroll
                        for (int g = 0; g < G; ++g) {
#pragma unroll
                            for (int i = g * W; i < (g + 1) * W; ++i) s[i / 32][i % 32] = fmaf(s[i / 32][i % 32], f[g], b[g]) - reference;
                            f[g] = 1.0f;
                            b[g] = reference;
                        }
                    }
                }
                const float reference = m == -INFINITY ? 0.0f : m;
                // (exponentials of 32 columns in place, then their sums: a warp that takes them as they come waits for each)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
#pragma unroll
                    for (int g = 0; g < G / 2; ++g) {
                        const float shift = b[c * G / 2 + g] - reference;
                        const Pair ff = pair_of(f[c * G / 2 + g], f[c * G / 2 + g]), bb = pair_of(shift, shift);
#pragma unroll
                        for (int i = g * W; i < (g + 1) * W; i += 2) {
                            pair_split(pair_fma(pair_of(s[c][i], s[c][i + 1]), ff, bb), s[c][i], s[c][i + 1]);
                            s[c][i] = exp2_of(s[c][i]);
                            s[c][i + 1] = i % 8 == 6 ? exp2_fma(s[c][i + 1]) : exp2_of(s[c][i + 1]);
                        }
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 32; i += 2) w[i / 2] = half2_of(s[c][i], s[c][i + 1]);
                    tmem_store16(s_at + 16u * c, w);
#pragma unroll
                    for (int g = 0; g < G / 2; ++g) {
                        Pair sum[2] = {pair_of(s[c][g * W], s[c][g * W + 1]), pair_of(s[c][g * W + 2], s[c][g * W + 3])};
#pragma unroll
                        for (int i = g * W + 4; i < (g + 1) * W; i += 4) {
                            sum[0] = pair_add(sum[0], pair_of(s[c][i], s[c][i + 1]));
                            sum[1] = pair_add(sum[1], pair_of(s[c][i + 2], s[c][i + 3]));
                        }
                        float x, y;
                        pair_split(pair_add(sum[0], sum[1]), x, y);
                        l = fmaf(x + y, inverse[c * G / 2 + g], l);
                    }
                }
                tmem_store_wait();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + buffer);
            }
            if (tiles > 0) {
                if (ok && !cta_wait_warp(o_done + 8u * (uint32_t)t, done & 1u)) ok = false;
                tmem_fence_after();
                j0 += (uint32_t)tiles;
                ++done;
            }
            if (ok) {
                const float r = p.split > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
                const bool f16 = p.a.out_type == OUT_F16;
                if (p.split > 1) {
                    float *const ends = many_part<D>(p, it.number, it.part) + MANY_ROWS * D;
                    ends[row] = m;
                    ends[MANY_ROWS + row] = l;
                }
                // Results go through shared memory, where the queries were, as many bytes of every row at a time as its queries had, so that rows are stored whole.
                constexpr int line_bytes = 2 * D;
                const uint32_t room = base + (uint32_t)t * K::tile + (uint32_t)((warp & 3) * 32 * line_bytes);
                auto to_rows = [&](const uint32_t (&w)[4], int chunk) {
                    sts128(room + (uint32_t)(lane * line_bytes + ((chunk ^ lane) & 7) * 16 + (chunk & 8) * 16), make_uint4(w[0], w[1], w[2], w[3]));
                };
                auto store_rows = [&](auto &&address) {
                    __syncwarp();
                    constexpr int wide = line_bytes / 16, at_once = 32 / wide;
#pragma unroll 4
                    for (int k = 0; k < 32 / at_once; ++k) {
                        const int line = k * at_once + lane / wide, chunk = lane % wide, r = t * 128 + (warp & 3) * 32 + line;
                        const uint4 w = lds128(room + (uint32_t)(line * line_bytes + ((chunk ^ line) & 7) * 16 + (chunk & 8) * 16));
                        if (r < it.rows) *reinterpret_cast<uint4 *>(address(r) + chunk * 16) = w;
                    }
                    __syncwarp();
                };
                auto out_row = [&](int r, int bytes) {                 // of the results
                    const int pairs = it.row0 + r, its_token = pairs / p.a.group, its_head = pairs - its_token * p.a.group;
                    return static_cast<char *>(p.a.out) +
                           ((size_t)(it.begin + its_token) * ((size_t)p.a.heads * (size_t)p.a.group) + (size_t)(it.head * p.a.group + its_head)) * (size_t)(D * bytes);
                };
                const bool wide = p.split > 1 || p.a.out_type == OUT_F32;
                constexpr int per = D / 32;                            // 16 fp32 columns each, to a line
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    int32_t u[16];
                    if (tiles > 0) {
                        tmem_load16(o_at + 16u * c, u);
                        tmem_wait(u);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) u[i] = 0;
                    }
                    float o[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = __int_as_float(u[i]) * r;
                    if (wide) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t w[4] = {__float_as_uint(o[4 * i]), __float_as_uint(o[4 * i + 1]), __float_as_uint(o[4 * i + 2]), __float_as_uint(o[4 * i + 3])};
                            to_rows(w, 4 * (c % per) + i);
                        }
                        if (c % per == per - 1) {
                            if (p.split > 1) {
                                char *const to = reinterpret_cast<char *>(many_part<D>(p, it.number, it.part) + 16 * (c - per + 1));
                                store_rows([&](int r) { return to + (size_t)r * (4 * D); });
                            } else {
                                store_rows([&](int r) { return out_row(r, 4) + 64 * (c - per + 1); });
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t w[4] = {pack16(o[8 * i], o[8 * i + 1], f16), pack16(o[8 * i + 2], o[8 * i + 3], f16), pack16(o[8 * i + 4], o[8 * i + 5], f16),
                                                   pack16(o[8 * i + 6], o[8 * i + 7], f16)};
                            to_rows(w, 2 * c + i);
                        }
                    }
                }
                if (!wide) store_rows([&](int r) { return out_row(r, 2); });
                if (lane == 0) mbar_arrive(stored + 8u * (uint32_t)t);
            }
        }
        if (!ok && lane == 0) give_up();
    } else if (warp < MMA_WARP) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        // Codes to fp16.  A thread has 16 channels of one key in 32; eight threads have 64 channels each of two keys next to each other, for D = 128 the lower 64 of one and the
        // upper 64 of the other, so that neither reads nor stores meet a conflict.
        constexpr uint32_t halves = D / 64;
        const uint32_t thread = (uint32_t)(tid - 32 * CODES_WARP), quad = thread & 3u, row = thread >> 2, odd = halves == 2 ? row & 1u : 0u;
        const uint32_t to0 = row * 128u + (((2u * quad) ^ row) & 7u) * 16u, to1 = row * 128u + (((2u * quad + 1u) ^ row) & 7u) * 16u;
        bool ok = true;
        ManyItem it;
        uint32_t n = 0;                                                // pieces so far
        for (uint32_t work = 0; ok && work_of(work, it); ++work)
        for (const uint32_t n_end = n + 2u * (uint32_t)it.count; n < n_end; ++n) {
            const uint32_t s = n % K::stages, r = n % K::raw_stages, to = base + K::off_ring + s * K::tile, from = base + K::off_raw + r * K::raw + row * D + quad * 16u;
            if (!cta_wait_warp(raw_full + 8u * r, (n / K::raw_stages) & 1u) || (n >= K::stages && !cta_wait_warp(empty + 8u * s, (n / K::stages - 1u) & 1u))) {
                ok = false;
                break;
            }
#pragma unroll
            for (uint32_t h = 0; h < halves; ++h) {
                const uint32_t half = h ^ odd, source = from + half * 64u, target = to + half * K::half;
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint4 raw = lds128(source + i * (32u * D));
                    const uint32_t x[4] = {raw.x, raw.y, raw.z, raw.w};
                    uint32_t w[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t y = x[k] ^ 0x80808080u;         // codes 0 and 1, 2 and 3 in the low bits of 1024, minus 1152
                        w[2 * k] = minus_1152(__byte_perm(y, 0x64646464u, 0x4140));
                        w[2 * k + 1] = minus_1152(__byte_perm(y, 0x64646464u, 0x4342));
                    }
                    sts128(target + to0 + i * 4096u, make_uint4(w[0], w[1], w[2], w[3]));
                    sts128(target + to1 + i * 4096u, make_uint4(w[4], w[5], w[6], w[7]));
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(full + 8u * s);
                mbar_arrive(raw_empty + 8u * r);
            }
        }
        if (!ok && lane == 0) give_up();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (warp == MMA_WARP) {
            const uint32_t qk = f16_desc(128, 64, false), pv = f16_desc(128, D, true);
            bool ok = true;
            // S of 64 keys (half h of a tile of keys) for a tile of rows, and O of them
            auto logits = [&](uint32_t t, uint32_t h, uint32_t s) {
                const uint32_t a = rows_operand(base + t * K::tile), b = rows_operand(base + K::off_ring + s * K::tile + h * 8192u), d = tmem + t * 128u + h * 64u;
#pragma unroll
                for (uint32_t k = 0; k < D / 16; ++k) {
                    const uint32_t at = (k / 4u) * (K::half >> 4) + (k % 4u) * 2u;
                    product_f16(d, a + at, b + at, qk, k > 0);
                }
                commit_one(s_full + 8u * (2u * t + h));
            };
            auto outputs = [&](uint32_t t, uint32_t h, uint32_t s, bool more) {
                const uint32_t a = tmem + t * 128u + h * 64u, b = keys_operand<D>(base + K::off_ring + s * K::tile + h * 8192u), d = tmem + K::o_column + t * 128u;
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) product_f16_tmem(d, a + 8u * k, b + k * 128u, pv, more || k > 0);
                commit_one(o_full + 8u * t);
            };
            auto wait_for = [&](uint32_t bar, uint32_t parity) {
                if (ok && !cta_wait_warp(bar, parity)) ok = false;
                tmem_fence_after();
                return ok;
            };
            auto piece = [&](uint32_t i) { return wait_for(full + 8u * (i % K::stages), (i / K::stages) & 1u); };
            ManyItem it;
            uint32_t n = 0, j0[2] = {0u, 0u}, done[2] = {0u, 0u};      // pieces; of each tile of rows: tiles of keys, and works with some, so far
            for (uint32_t work = 0; ok && work_of(work, it); ++work) {
                const int tiles = it.count;
                const uint32_t row_tiles = it.rows > 128 ? 2u : 1u;
                if (tiles == 0) continue;
                for (uint32_t t = 0; t < row_tiles && ok; ++t) {
                    if (!wait_for(q_full + 8u * t, done[t] & 1u) || (t == 0 && !piece(n))) break;
                    logits(t, 0, n % K::stages);
                    logits(t, 1, n % K::stages);
                }
                if (!ok) break;
                commit_one(empty + 8u * (n % K::stages));
                ++n;
                for (int j = 0; j < tiles && ok; ++j, n += 2) {
                    const bool more = j + 1 < tiles;
                    const uint32_t sv = n % K::stages, sk = (n + 1) % K::stages;
                    if (!piece(n)) break;
                    for (uint32_t h = 0; h < 2 && ok; ++h)
                        for (uint32_t t = 0; t < row_tiles && ok; ++t) {
                            if (!wait_for(p_full + 8u * (2u * t + h), (j0[t] + (uint32_t)j) & 1u)) break;
                            outputs(t, h, sv, j > 0 || h > 0);
                            if (more) {
                                if (h == 0 && t == 0 && !piece(n + 1)) break;
                                logits(t, h, sk);
                            } else if (h == 1) {
                                commit_one(o_done + 8u * t);
                            }
                        }
                    commit_one(empty + 8u * sv);
                    if (more) commit_one(empty + 8u * sk);
                }
                --n;                                                   // (the last tile has no keys behind it)
                for (uint32_t t = 0; t < row_tiles; ++t) {
                    j0[t] += (uint32_t)tiles;
                    ++done[t];
                }
            }
            if (!ok && lane == 0) give_up();
            // nothing is in flight when the CTA ends
            commit_one(end);
            (void)cta_wait_warp(end, 0);
        }
        if (warp == LOAD_WARP) {
            // a lane to a page of a tile (eight at most): its codes and steps
            const int log2page = p.a.q.page, each = min(1 << log2page, MANY_KEYS), copies = MANY_KEYS / each;
            bool ok = true;
            uint32_t n = 0, global = 0;                                // pieces, and tiles of keys, so far
            int index = (int)blockIdx.x;
            for (uint32_t work = 0; ok; ++work) {
                if (work > 0) {
                    index = next_cta(base + K::off_next, next_full, (work - 1u) & 1u, lane, ok);
                    if (!ok) break;
                }
                ManyItem it;
                it.rows = 0;
                if (index >= 0) it = many_item(p.a, index / p.split, lane);
                it.part = index >= 0 ? index % p.split : 0;
                it.tile0 = (int)((long long)it.tiles * it.part / p.split);
                it.count = (int)((long long)it.tiles * (it.part + 1) / p.split) - it.tile0;
                if (work >= 2 && !cta_wait_warp(work_empty + 8u * (work & 1u), (work / 2u - 1u) & 1u)) {
                    ok = false;
                    break;
                }
                if (lane == 0) {
                    found[work & 1u] = it;
                    mbar_arrive(work_full + 8u * (work & 1u));
                }
                __syncwarp();
                if (it.rows <= 0) break;
                const int32_t *const table = p.a.q.pages + (size_t)it.sequence * (size_t)p.a.q.width;
                auto page_of = [&](int j) {
                    const int key = key_of(it, it.tile0 + j) + lane * each;
                    return lane < copies && j < it.count ? min(max(*(table + min(key >> log2page, p.a.q.width - 1)), 0), p.a.q.n_pages - 1) : 0;
                };
                int page = page_of(0);
                for (int j = 0; j < it.count && ok; ++j, ++global) {
                    const int next = page_of(j + 1);
                    const size_t block = (size_t)page * (size_t)p.a.heads + (size_t)it.head;
                    const float ks = *(p.a.k_steps + block), vs = *(p.a.v_steps + block);
                    for (int kind = 0; kind < 2; ++kind, ++n) {
                        const uint32_t r = n % K::raw_stages, bar = raw_full + 8u * r;
                        if (n >= K::raw_stages && !cta_wait_warp(raw_empty + 8u * r, (n / K::raw_stages - 1u) & 1u)) {
                            ok = false;
                            break;
                        }
                        if (lane == 0) mbar_expect_tx(bar, K::raw);
                        __syncwarp();
                        if (lane < copies)
                            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                         ::"r"(base + K::off_raw + r * K::raw + (uint32_t)(lane * each * D)),
                                         "l"((kind ? p.a.v_codes : p.a.k_codes) + ((block << log2page) * (size_t)D)), "r"((uint32_t)(each * D)), "r"(bar) : "memory");
                    }
                    if (!ok) break;
                    // of 16 keys each: s_k, log2 s_v, 1 / s_v, and whether one of them is not finite, which the rows' warps see to
                    const int mine = (lane & 7) * 16 / each;
                    const float k = __shfl_sync(0xffffffffu, ks, mine), v = __shfl_sync(0xffffffffu, vs, mine);
                    const bool bad = !(fabsf(k) <= 0x1p126f && fabsf(v) <= 0x1p126f), none = bad || v < 0x1p-64f;
                    if (lane < 8)
                        sts128(steps + (global & 7u) * 128u + (uint32_t)lane * 16u,
                               make_uint4(__float_as_uint(bad ? 0.0f : k), __float_as_uint(none ? -64.0f : log2_of(v)), __float_as_uint(none ? 0x1p64f : 1.0f / v),
                                          (uint32_t)bad));
                    __syncwarp();
                    if (lane == 0) mbar_arrive(steps_full + 8u * (global & 7u));
                    page = next;
                }
            }
            if (!ok && lane == 0) give_up();
            // nothing is in flight when the CTA ends
            for (uint32_t i = n > K::raw_stages ? n - K::raw_stages : 0u; i < n; ++i) (void)cta_wait_warp(raw_full + 8u * (i % K::raw_stages), (i / K::raw_stages) & 1u);
        }
        __syncwarp();
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(K::columns) : "memory");
}

// Rows whose keys were split: blockIdx.x is an item, blockIdx.y a part of its rows.  A thread has four channels of a row at a time, and AHEAD parts of them on their way (two where there are no
// more: bound by instructions and latency, 23.5 -> 19.8 us for two parts each of 200 items of 256 rows, all from memory).
constexpr int MANY_JOIN = 8;
template <int D, int AHEAD>
__device__ __forceinline__ void join_many(const ManyParams &p, const ManyItem &it)
{
    const int row_begin = (int)blockIdx.y * (MANY_ROWS / MANY_JOIN), row_end = min(row_begin + MANY_ROWS / MANY_JOIN, it.rows);
    const float *const parts = many_part<D>(p, it.number, 0);
    constexpr size_t each = (size_t)MANY_ROWS * (D + 2);
#pragma unroll 2
    for (int k = (int)threadIdx.x; k < (row_end - row_begin) * (D / 4); k += THREADS) {
        const int row = row_begin + k / (D / 4), channel = k % (D / 4) * 4;
        float m = -INFINITY, l = 0.0f;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int c0 = 0; c0 < p.split; c0 += AHEAD) {
            float4 x[AHEAD];
            float xm[AHEAD], xl[AHEAD], next = m;
#pragma unroll
            for (int c = 0; c < AHEAD; ++c) {
                const float *const from = parts + (size_t)min(c0 + c, p.split - 1) * each;
                x[c] = *reinterpret_cast<const float4 *>(from + (size_t)row * D + channel);
                xm[c] = c0 + c < p.split ? from[(size_t)MANY_ROWS * D + row] : -INFINITY;
                xl[c] = from[(size_t)MANY_ROWS * D + MANY_ROWS + row];
            }
#pragma unroll
            for (int c = 0; c < AHEAD; ++c) next = fmaxf(next, xm[c]);
            const float before = m == -INFINITY ? 0.0f : exp2_of(m - next);
            v.x *= before; v.y *= before; v.z *= before; v.w *= before;
            l *= before;
#pragma unroll
            for (int c = 0; c < AHEAD; ++c) {
                // (a part that has seen nothing, or nothing but what is not finite, which stays)
                const float a = xm[c] == -INFINITY ? (c0 + c < p.split && xl[c] != xl[c] ? 1.0f : 0.0f) : exp2_of(xm[c] - next);
                l = fmaf(a, xl[c], l);
                v.x = fmaf(a, x[c].x, v.x); v.y = fmaf(a, x[c].y, v.y); v.z = fmaf(a, x[c].z, v.z); v.w = fmaf(a, x[c].w, v.w);
            }
            m = next;
        }
        const float r = l == 0.0f ? 0.0f : 1.0f / l;
        const int token = (it.row0 + row) / p.a.group, h = it.row0 + row - token * p.a.group;
        store_out4<D>(p.a, ((size_t)(it.begin + token) * (size_t)(p.a.heads * p.a.group) + (size_t)(it.head * p.a.group + h)) * D + (size_t)channel,
                      make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
    }
}
template <int D>
__global__ void __launch_bounds__(THREADS) many_join_kernel(const __grid_constant__ ManyParams p)
{
    __shared__ ManyItem found;
    if (threadIdx.x < 32) {
        const ManyItem it = many_item(p.a, (int)blockIdx.x, (int)threadIdx.x);        // (before the wait, as in join_kernel)
        if (threadIdx.x == 0) found = it;
    }
    __syncthreads();
    griddep_wait();
    griddep_launch();
    const ManyItem it = found;
    if (p.split == 2) join_many<D, 2>(p, it);
    else join_many<D, 4>(p, it);
}

}  // namespace perq_kv
