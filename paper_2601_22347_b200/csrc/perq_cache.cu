// C ABI of the 8-bit cache (writing, reading back) and of the attention over it: argument checks, choice of kernel, launches.
// Nothing here allocates device memory or synchronises.
#include "perq.h"

#include <algorithm>
#include <cmath>
#include <cstring>

#include "perq_attend_many.cuh"
#include "perq_host.cuh"

namespace {

using namespace perq_kv;

// Programmatic stream serialization as everywhere in the library.
template <typename... P>
int launch(void (*kernel)(P...), long long grid, int threads, size_t smem, cudaStream_t st, int grid_y, const P &...p)
{
    if (int rc = allow_smem(kernel, smem)) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid, (unsigned)grid_y);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, p...) != cudaSuccess) {
        (void)cudaGetLastError();
        return PERQ_ERR_CUDA;
    }
    return PERQ_OK;
}

int check_cache(int64_t T, int32_t S, int32_t heads, int32_t D, int32_t b, int32_t page, int64_t n_pages, int32_t width)
{
    if (T < 0 || T > (1 << 30) || S < 0 || S > PERQ_MAX_SEQUENCES || heads < 1 || heads > PERQ_MAX_HEADS || (D != 64 && D != 128)) return PERQ_ERR_SHAPE;
    if (!is_pow2(page) || page < 16 || page > 128 || n_pages < 1 || n_pages > INT32_MAX || n_pages * page * heads > INT32_MAX || width < 1 || (int64_t)width * page > (1 << 30)) return PERQ_ERR_SHAPE;
    if (!is_pow2(b) || (b != 1 && b < 16) || b > D) return PERQ_ERR_BLOCK;
    return PERQ_OK;
}
bool row_stride(int64_t stride, int64_t channels) { return stride >= channels && stride % 8 == 0; }
int check_pointers(const void *const *p, int n)
{
    for (int i = 0; i < n; ++i)
        if (!p[i]) return PERQ_ERR_NULL;
    for (int i = 0; i < n; ++i)
        if (!aligned16(p[i])) return PERQ_ERR_ALIGN;
    return PERQ_OK;
}

Sequences sequences(const int32_t *offsets, const int32_t *lengths, const int32_t *pages, int64_t T, int32_t S, int32_t width, int64_t n_pages, int32_t page)
{
    Sequences q;
    q.offsets = offsets;
    q.lengths = lengths;
    q.pages = pages;
    q.T = (int32_t)T;
    q.S = S;
    q.width = width;
    q.n_pages = (int32_t)n_pages;
    q.page = ilog2(page);
    return q;
}

template <int D>
int launch_write(WriteParams &p, int page, cudaStream_t st)
{
    // Blocks that rows can fall into: n rows reach into at most n / page + 2, and into no more than n.
    const int64_t blocks = std::min<int64_t>(p.q.T, p.q.T / page + 2ll * p.q.S);
    const bool few = p.q.T <= 8ll * p.q.S;
    const bool one = few || page * D <= 2048;                          // a warp to a block
    p.parts = one ? (2 * p.heads + THREADS / 32 - 1) / (THREADS / 32) : 2 * p.heads;
    const int64_t grid = blocks * p.parts;
    if (grid >= (1ll << 31)) return PERQ_ERR_SHAPE;
    if (few) return launch(write_kernel<D, 1, 1, 4, false>, grid, THREADS, 0, st, 1, p);
    if (one) return launch(write_kernel<D, 1, 4, 16, true>, grid, THREADS, 0, st, 1, p);
    switch (page * D / 4096) {
    case 1: return launch(write_kernel<D, 8, 1, 16, true>, grid, THREADS, 0, st, 1, p);
    case 2: return launch(write_kernel<D, 8, 2, 16, true>, grid, THREADS, 0, st, 1, p);
    default: return launch(write_kernel<D, 16, 2, 16, true>, grid, 512, 0, st, 1, p);
    }
}

// How many CTAs share the units of few queries: what is resident at once.
int few_ctas(int sms, int nt, int D) { return nt == 1 || D == 64 ? 2 * sms : sms; }

// Codes as rows of D bytes, in boxes of a unit's keys.
template <int D>
bool codes_map(CUtensorMap *map, const void *codes, const AttendParams &p)
{
    TensorMapEncode encode = tensor_map_encode();
    if (encode == nullptr) return false;
    const cuuint64_t dims[2] = {D, ((cuuint64_t)p.q.n_pages * (cuuint64_t)p.heads) << p.q.page}, strides[1] = {D};
    const cuuint32_t size[2] = {D, FEW_KEYS}, step[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(codes), dims, strides, size, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int NT>
int launch_few(const AttendParams &p, int sms, cudaStream_t st)
{
    const int ctas = few_ctas(sms, NT, D);
    CUtensorMap k, v;
    if (!codes_map<D>(&k, p.k_codes, p) || !codes_map<D>(&v, p.v_codes, p)) return PERQ_ERR_CUDA;
    if (int rc = launch(few_kernel<D, NT>, ctas, THREADS, Few<D, NT>::bytes, st, 1, k, v, p)) return rc;
    return launch(join_kernel<D, NT>, ctas - 1, THREADS, join_bytes(ctas), st, 8 * NT / JOIN_ROWS, p, ctas);
}

// Rows (of tokens and heads) of a sequence up to which the kernel for few queries takes it.  32 sequences of 8000 tokens, 8 heads of 128 with 4 of queries each, few against many: 16 rows 131 and 209 us,
// 32 rows 247 and 213, 48 rows 362 and 213; two sequences: 32 rows 30 and 37, 48 rows 37 and 37, 64 rows 43 and 39 (behind 500 tokens: 12 and 18, 18 and 18, 18 and 20).  Heads of 64: 32 rows 157 and
// 182, 48 rows 226 and 182; two sequences 27 and 25, 31 and 25.
constexpr int FEW_ROWS = 32, BOTH_ROWS = 64;
constexpr int MANY_PIECES = 4;               // to an SM, of tiles of rows whose keys are split

// CTAs to the keys of a tile of rows.  Few items leave SMs without work, or, with contexts of different lengths, one SM with much more than another; every piece costs as much as four and a half
// tiles of keys for its queries and results, and joining them two.  With items alike the call takes whole rounds of pieces, with different ones the CTAs take them as they come: the mean of
// both is what is compared.  (Two sequences of 16 tokens behind 8000, 8 heads of 128 with 4 of queries each, in 1, 4, 9 and 15 pieces: 105, 42, 39 and 54 us, 9 are taken; of 64 tokens 138, 56, 45
// and 64, 9 too; eight of 16 in 1, 2 and 4: 108, 72 and 81, 2.)  How many keys there are is guessed from the table's width, and how many items from all rows: a prompt of 300 tokens 21 us, 50 with
// a table for 131072; a chunk of 512 behind 16000 163, 244 beside 15 decode steps and 367 beside 63.
int many_split(const AttendParams &p, long long most_items, long long items, int sms)
{
    long long keys = (long long)p.q.width << p.q.page;
    if (p.window > 0) keys = std::min(keys, (long long)p.window + p.sinks + std::min(p.q.T, p.most) + 2 * MANY_KEYS);
    const long long tiles = (keys + MANY_KEYS - 1) / MANY_KEYS, limit = std::min<long long>(std::min<long long>(MANY_PIECES * sms / most_items, 16), tiles);
    int best = 1;
    double least = 0.0;
    for (int s = 1; s == 1 || s <= limit; ++s) {
        const double rounds = (double)items * s / sms, cost = 0.5 * (std::ceil(rounds) + rounds + 0.5) * (4.5 + (double)tiles / s) + (s > 1 ? 2.0 : 0.0);
        if (s > 1 && cost >= least) continue;
        best = s;
        least = cost;
    }
    return best;
}

template <int D>
int launch_many(const AttendParams &a, int sms, cudaStream_t st)
{
    ManyParams p;
    std::memset(&p, 0, sizeof(p));
    p.a = a;
    p.partial = a.partial;
    // (n sequences of more than a.few_rows rows each have at most rows / 256 + n tiles, and there are no more of them than fit into the rows; if they are alike, so many have them)
    const long long rows = (long long)a.q.T * a.group, n = std::min<long long>(a.q.S, rows / (a.few_rows + 1)), each = (rows + n - 1) / n;
    const long long items = (rows / MANY_ROWS + n) * a.heads;
    p.split = many_split(a, items, n * ((each + MANY_ROWS - 1) / MANY_ROWS) * a.heads, sms);
    if (items * p.split >= (1ll << 31)) return PERQ_ERR_SHAPE;
    if (int rc = launch(a.q.page == 4 ? many_kernel<D, true> : many_kernel<D, false>, items * p.split, MANY_THREADS, Many<D>::bytes, st, 1, p)) return rc;
    return p.split > 1 ? launch(many_join_kernel<D>, items, THREADS, 0, st, MANY_JOIN, p) : PERQ_OK;
}

template <int D>
int launch_attention(AttendParams &p, int sms, cudaStream_t st)
{
    const int64_t most = std::min<int64_t>(p.q.T, p.most), rows = most * p.group;
    if (rows <= 8) return launch_few<D, 1>(p, sms, st);
    // Up to 64 rows one kernel takes all sequences, by the mean of their rows (32 sequences of up to 5 tokens and 8 heads, 1 to 4 of them by one kernel and 5 by the other: 113 us, 63 by the first).
    if (rows <= FEW_ROWS || (rows <= BOTH_ROWS && p.q.T * (int64_t)p.group <= (int64_t)FEW_ROWS * p.q.S)) return launch_few<D, 2>(p, sms, st);
    // Beyond, the kernel for many takes them all if the shortest has more than FEW_ROWS where every row of the call is one's and the others have `most`; that saves two launches: two sequences of
    // 256 rows behind 500 tokens 27 -> 23 us.  (Queries of a sequence with few rows are then rounded as the others' are.)
    p.few_rows = rows <= BOTH_ROWS || (p.q.T - (p.q.S - 1) * most) * p.group > FEW_ROWS ? 0 : FEW_ROWS;
    if (p.few_rows > 0)
        if (int rc = launch_few<D, 2>(p, sms, st)) return rc;
    return launch_many<D>(p, sms, st);
}

}  // namespace

cudaError_t perq_kv_read_error(unsigned int *flags) { return cudaMemcpyFromSymbol(flags, perq_mm::g_error, sizeof *flags); }
cudaError_t perq_kv_clear_error()
{
    const unsigned int zero = 0;
    return cudaMemcpyToSymbol(perq_mm::g_error, &zero, sizeof zero);
}

extern "C" {

int perq_cache_write_i8(const void *k, const void *v, int32_t in_type, int64_t k_stride, int64_t v_stride, const int32_t *offsets, const int32_t *lengths,
                        const int32_t *pages, int64_t T, int32_t S, int32_t heads, int32_t D, int32_t b, int32_t page, int64_t n_pages, int32_t width,
                        void *k_codes, float *k_steps, void *v_codes, float *v_steps, void *stream)
{
    if (int rc = check_cache(T, S, heads, D, b, page, n_pages, width)) return rc;
    if (!row_stride(k_stride, (int64_t)heads * D) || !row_stride(v_stride, (int64_t)heads * D)) return PERQ_ERR_SHAPE;
    if (in_type != PERQ_OUT_BF16 && in_type != PERQ_OUT_F16) return PERQ_ERR_FMT;
    if (T == 0 || S == 0) return PERQ_OK;
    const void *const all[] = {k, v, offsets, lengths, pages, k_codes, k_steps, v_codes, v_steps};
    if (int rc = check_pointers(all, 9)) return rc;
    WriteParams p;
    std::memset(&p, 0, sizeof(p));
    p.q = sequences(offsets, lengths, pages, T, S, width, n_pages, page);
    p.x[0] = static_cast<const uint16_t *>(k);
    p.x[1] = static_cast<const uint16_t *>(v);
    p.stride[0] = k_stride;
    p.stride[1] = v_stride;
    p.codes[0] = static_cast<int8_t *>(k_codes);
    p.codes[1] = static_cast<int8_t *>(v_codes);
    p.steps[0] = k_steps;
    p.steps[1] = v_steps;
    p.heads = heads;
    p.f16 = in_type == PERQ_OUT_F16;
    p.log2b = ilog2(b);
    return D == 64 ? launch_write<64>(p, page, static_cast<cudaStream_t>(stream)) : launch_write<128>(p, page, static_cast<cudaStream_t>(stream));
}

int perq_cache_read_i8(const void *k_codes, const float *k_steps, const void *v_codes, const float *v_steps, const int32_t *offsets, const int32_t *lengths,
                       const int32_t *pages, int64_t T, int32_t S, int32_t heads, int32_t D, int32_t b, int32_t page, int64_t n_pages, int32_t width, void *k,
                       void *v, int32_t out_type, void *stream)
{
    if (int rc = check_cache(T, S, heads, D, b, page, n_pages, width)) return rc;
    if (out_type < PERQ_OUT_BF16 || out_type > PERQ_OUT_F32) return PERQ_ERR_FMT;
    if (T == 0 || S == 0) return PERQ_OK;
    const void *const all[] = {k, v, offsets, lengths, pages, k_codes, k_steps, v_codes, v_steps};
    if (int rc = check_pointers(all, 9)) return rc;
    ReadParams p;
    std::memset(&p, 0, sizeof(p));
    p.q = sequences(offsets, lengths, pages, T, S, width, n_pages, page);
    p.codes[0] = static_cast<const int8_t *>(k_codes);
    p.codes[1] = static_cast<const int8_t *>(v_codes);
    p.steps[0] = k_steps;
    p.steps[1] = v_steps;
    p.out[0] = k;
    p.out[1] = v;
    p.heads = heads;
    p.out_type = out_type;
    p.log2b = ilog2(b);
    const long long grid = (T + READ_TOKENS - 1) / READ_TOKENS;
    return launch(D == 64 ? read_kernel<64> : read_kernel<128>, grid, THREADS, 0, static_cast<cudaStream_t>(stream), 2, p);
}

int perq_attention_i8_workspace_bytes(int64_t T, int32_t S, int32_t heads, int32_t group, int32_t D, int32_t most, size_t *bytes)
{
    if (int rc = check_cache(T, S, heads, D, 1, 16, 1, 1)) return rc;
    if (group < 1 || (int64_t)heads * group > PERQ_MAX_HEADS || most < 1) return PERQ_ERR_SHAPE;
    if (!bytes) return PERQ_ERR_NULL;
    int sms = sm_count();
    if (sms <= 0) sms = 148;                                           // (no device, no launch: sizes are answered for a B200)
    const int64_t rows = std::min<int64_t>(T, most) * group;
    const size_t few = std::max((size_t)few_ctas(sms, 1, D) * 8, (size_t)few_ctas(sms, 2, D) * 16) * 2, many = rows > FEW_ROWS ? (size_t)MANY_PIECES * (size_t)sms * MANY_ROWS : 0;
    *bytes = T == 0 || S == 0 ? 0 : std::max(few, many) * (size_t)(D + 2) * 4;
    return PERQ_OK;
}

int perq_attention_i8(const void *q, int32_t in_type, int64_t q_stride, const void *k_codes, const float *k_steps, const void *v_codes, const float *v_steps,
                      const int32_t *offsets, const int32_t *lengths, const int32_t *pages, int64_t T, int32_t S, int32_t heads, int32_t group, int32_t D,
                      int32_t b, int32_t page, int64_t n_pages, int32_t width, int32_t most, float scale, int32_t window, int32_t sinks, void *out,
                      int32_t out_type, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_cache(T, S, heads, D, b, page, n_pages, width)) return rc;
    if (group < 1 || (int64_t)heads * group > PERQ_MAX_HEADS || !row_stride(q_stride, (int64_t)heads * group * D) || most < 1 || window < 0 || sinks < 0 || !std::isfinite(scale)) return PERQ_ERR_SHAPE;
    if ((in_type != PERQ_OUT_BF16 && in_type != PERQ_OUT_F16) || out_type < PERQ_OUT_BF16 || out_type > PERQ_OUT_F32) return PERQ_ERR_FMT;
    if (T == 0 || S == 0) return PERQ_OK;
    const void *const all[] = {q, k_codes, k_steps, v_codes, v_steps, offsets, lengths, pages, out};
    if (int rc = check_pointers(all, 9)) return rc;
    size_t need = 0;
    if (int rc = perq_attention_i8_workspace_bytes(T, S, heads, group, D, most, &need)) return rc;
    if (need > 0 && (!workspace || workspace_bytes < need)) return PERQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return PERQ_ERR_ALIGN;
    const int sms = sm_count();
    if (sms <= 0) return PERQ_ERR_CUDA;
    AttendParams p;
    std::memset(&p, 0, sizeof(p));
    p.q = sequences(offsets, lengths, pages, T, S, width, n_pages, page);
    p.x = static_cast<const uint16_t *>(q);
    p.stride = q_stride;
    p.k_codes = static_cast<const int8_t *>(k_codes);
    p.v_codes = static_cast<const int8_t *>(v_codes);
    p.k_steps = k_steps;
    p.v_steps = v_steps;
    p.out = out;
    p.partial = static_cast<float *>(workspace);
    p.heads = heads;
    p.group = group;
    p.most = most;
    p.few_rows = INT32_MAX;
    p.window = std::min(window, 1 << 30);
    p.sinks = std::min(sinks, 1 << 30);
    p.log2b = ilog2(b);
    p.f16 = in_type == PERQ_OUT_F16;
    p.out_type = out_type;
    p.scale = scale * (1.4426950408889634f / std::sqrt((float)b));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return D == 64 ? launch_attention<64>(p, sms, st) : launch_attention<128>(p, sms, st);
}

}  // extern "C"
