// C ABI of the 8-bit linear layers (rows to 8-bit codes, products of codes): argument checks, choice of kernel, tensor maps, launches.
// Nothing here allocates device memory or synchronises, except where perq.h says so.
#include "perq.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <tuple>

#include "perq_host.cuh"
#include "perq_mm_many.cuh"
#include "perq_quant8.cuh"

namespace {

// Whether a format's codes lie two to a byte.
inline bool is_packed(int32_t fmt) { return fmt != PERQ_FMT_INT8; }

// Codes [rows, d] in boxes of `box` rows by 128 bytes, as operands (128-byte swizzle).
bool codes_map(CUtensorMap *map, const void *codes, bool packed, uint64_t rows, int d, int box)
{
    TensorMapEncode encode = tensor_map_encode();
    if (encode == nullptr) return false;
    const uint64_t bytes = packed ? (uint64_t)d / 2 : (uint64_t)d;
    const cuuint64_t dims[2] = {bytes, rows}, strides[1] = {bytes};
    const cuuint32_t size[2] = {128, (cuuint32_t)box}, step[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(codes), dims, strides, size, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Programmatic stream serialization as everywhere in the library, and clusters.
template <typename P>
int launch_product(void (*kernel)(CUtensorMap, CUtensorMap, P), unsigned grid, int threads, size_t smem, int cluster, cudaStream_t st, const CUtensorMap &w,
                   const CUtensorMap &a, const P &p)
{
    if (int rc = allow_smem(kernel, smem)) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, w, a, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return PERQ_ERR_CUDA;
    }
    return PERQ_OK;
}

// Clusters of a kernel that the device holds at once (0: it cannot say), asked once for a kernel, device, size and shared memory.
std::mutex g_clusters_mutex;
std::map<std::tuple<const void *, int, int, size_t>, int> g_clusters;

template <typename K>
int max_clusters(K kernel, int threads, size_t smem, int size)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    std::lock_guard<std::mutex> lock(g_clusters_mutex);
    const auto key = std::make_tuple(reinterpret_cast<const void *>(kernel), dev, size, smem);
    const auto known = g_clusters.find(key);
    if (known != g_clusters.end()) return known->second;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)size);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (allow_smem(kernel, smem) != PERQ_OK || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        n = 0;
    }
    g_clusters[key] = n;
    return n;
}

// A product: dense ones are grouped ones of one expert that has all rows.
struct Product {
    const void *a, *w;
    const float *a_scales, *w_scales;
    const int32_t *w_sums, *offsets;
    void *out;
    int64_t T;
    int32_t N, d, E, a_fmt, w_fmt, out_type;
};

template <bool W4, bool A4>
int launch_few(const Product &m, cudaStream_t st)
{
    using K = perq_mm::Few<W4, A4>;
    const int sms = sm_count();
    if (sms <= 0) return PERQ_ERR_CUDA;
    perq_mm::FewParams p;
    std::memset(&p, 0, sizeof(p));
    // columns for the tokens of a call, or for a little more than an expert has on average
    const int64_t want = m.offsets ? std::min<int64_t>(m.T, (m.T * 3 / 2 + m.E - 1) / m.E) : m.T;
    p.nt = want <= 16 ? 16 : want <= 32 ? 32 : want <= 64 ? 64 : 128;
    p.n_tiles = (m.N + perq_mm::FEW_ROWS - 1) / perq_mm::FEW_ROWS;
    p.steps = (m.d + K::step_codes - 1) / K::step_codes;
    // at most as many tiles of tokens as there are experts with rows, and full ones
    const int64_t token_tiles = m.offsets ? std::min<int64_t>(m.E, m.T) + m.T / p.nt : (m.T + p.nt - 1) / p.nt;
    const int64_t items = token_tiles * p.n_tiles;
    if (items >= (1ll << 31)) return PERQ_ERR_SHAPE;
    p.w_bytes = (W4 ? 1 : K::tiles) * perq_mm::FEW_TILE;
    p.a_bytes = (A4 ? 1 : K::tiles) * (uint32_t)p.nt * 128u;
    p.spread_bytes = A4 ? 2u * (uint32_t)p.nt * 128u : 0u;
    p.spreads = K::packed ? 3 : 0;
    p.tmem_cols = 32;
    while (p.tmem_cols < 2u * (uint32_t)p.nt + (W4 ? 64u * p.spreads : 0u)) p.tmem_cols *= 2;
    const uint32_t load = p.w_bytes + p.a_bytes, tail = 16 + 16 * (12 + 4) + 32 + 8 * (m.offsets ? (uint32_t)m.E + 1 : 1);
    // The split that fills the SMs, as far as its clusters fit on the device at once, and room for its sums.  Two CTAs to an SM where there are enough for
    // that, tensor memory has room for both and the ring is then long enough.
    uint32_t sums = 0;
    int per_sm = p.tmem_cols <= 256 ? 2 : 1;
    for (;; per_sm = 1) {
        auto loads = [&]() {
            sums = p.split > 1 ? (uint32_t)std::max(p.nt / 4, p.split) * perq_mm::FEW_ROWS * 16u : 0u;
            return (uint32_t)std::max(0, std::min(12, ((int)(kMaxSmem / per_sm) - 2048 - (int)(tail + sums + p.spreads * p.spread_bytes)) / (int)load));
        };
        p.split = 1;
        while (p.split < 8 && items * p.split * 2 <= (int64_t)sms * per_sm && p.split * 2 <= p.steps) p.split *= 2;
        while (per_sm == 1 && p.split > 2 && items > max_clusters(perq_mm::few_kernel<W4, A4>, K::threads, kMaxSmem / per_sm - 8192, p.split)) p.split /= 2;
        p.loads = loads();
        if (per_sm == 2 && p.loads >= 3) break;
        if (per_sm == 2) continue;
        if (p.loads < 2 && p.spreads > 2) {              // (8-bit weights with 128 packed tokens are 48 KB a step)
            p.spreads = 2;
            p.loads = loads();
        }
        if (p.loads < 2 && p.split > 1) {
            p.split = 1;
            p.loads = loads();
        }
        break;
    }
    p.log2_share = ilog2(std::max(1, p.nt / 4 / p.split));
    if (p.loads < 2) return PERQ_ERR_SHAPE;              // (no shape of these kernels)
    p.off_spread = p.loads * load;
    p.off_sums = p.off_spread + p.spreads * p.spread_bytes;
    p.off_bars = p.off_sums + sums;
    p.off_first = p.off_bars + 16 + 16 * (p.loads + p.spreads) + 32;
    const size_t smem = 1024 + p.off_first + 8 * (m.offsets ? (size_t)m.E + 1 : 1);
    p.a_scales = m.a_scales;
    p.w_scales = m.w_scales;
    p.w_sums = m.w_sums;
    p.offsets = m.offsets;
    p.out = m.out;
    p.T = (int32_t)m.T;
    p.N = m.N;
    p.E = m.E;
    p.asym = m.a_fmt == PERQ_FMT_INT4_ASYM;
    p.shift = (W4 ? 4 : 0) + (A4 ? 4 : 0);
    p.out_type = m.out_type;
    p.idesc = perq_mm::product_desc(true, !p.asym, perq_mm::FEW_ROWS, p.nt);
    CUtensorMap w, a;
    if (!codes_map(&w, m.w, W4, (uint64_t)m.E * (uint64_t)m.N, m.d, perq_mm::FEW_ROWS) || !codes_map(&a, m.a, A4, (uint64_t)m.T, m.d, p.nt)) return PERQ_ERR_CUDA;
    const int64_t clusters = p.split > 1 ? items : std::min<int64_t>(items, (int64_t)sms * per_sm);
    return launch_product(perq_mm::few_kernel<W4, A4>, (unsigned)(clusters * p.split), K::threads, smem, p.split, st, w, a, p);
}

// Programmatic stream serialization, without clusters.
template <typename P>
int launch_plain(void (*kernel)(P), long long grid, int threads, size_t smem, cudaStream_t st, const P &p, int grid_y = 1)
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
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return PERQ_ERR_CUDA;
    }
    return PERQ_OK;
}

// What a dense product of more than 64 tokens takes in either kernel, us, from their k-steps (both sides measured, model in brackets).
//   few: tiles of 128 x 128, a round of them on all SMs after another; a k-step, 128 codes of 8 bits or 256 with a packed operand, is 0.27, 0.54 (4-bit
//     weights) or 1.1 us (4-bit tokens only, spread beside 8-bit weights that fill the ring)
//   many: tiles of 256 x 256, 0.27 us for 128 codes, split over pairs where that fits; packed operands are spread first, 0.365 us for a million codes, most of it
//     under the launch
// 8-bit codes, few / many: 512 x 4096 x 4096 14.3 [14.8] / 13.7 [13.7], 128 x 14336 x 4096 15.7 [14.8] / 17.1 [16.0], 1400 x 1024 x 9728 25.6 [26.7] / 20.6 [19.7],
//   1100 x 2048 x 4096 14.2 [14.8] / 16.0 [16.0], 1024 x 1024 x 2048 9.3 [8.4] / 10.4 [11.7]
// 4-bit weights: 512 x 4096 x 4096 14.6 [14.2] / 18.2 [17.3], 768 x 4096 x 4096 23.5 [23.5] / 19.9 [20.0], 768 x 8192 x 4096 33.0 [32.7] / 34.6 [34.8],
//   256 x 14336 x 4096 24.2 / 29.1, 640 x 4096 x 14336 64 [67] / 54
// 4-bit tokens, 8-bit weights: 512 x 4096 x 4096 19.8 [23] / 16.4 [16.2], 1024 x 1024 x 2048 10.1 [10.0] / 12.1 [14.2]
double few_time(const Product &m, int sms)
{
    const bool w4 = is_packed(m.w_fmt), packed = w4 || is_packed(m.a_fmt);
    const int64_t tiles = (m.T + 127) / 128 * ((m.N + 127) / 128), steps = packed ? (m.d + 255) / 256 : (m.d + 127) / 128;
    int64_t split = 1;
    while (split < 8 && tiles * split * 2 <= sms * (packed ? 1 : 2) && split * 2 <= steps) split *= 2;
    const int64_t rounds = (tiles * split + sms - 1) / sms;
    return 5.0 + (double)rounds * ((double)steps / (double)split * (w4 ? 0.54 : packed ? 1.1 : 0.27) + 0.6);
}
double many_time(const Product &m, int sms)
{
    const int64_t items = (m.T + 255) / 256 * ((m.N + 255) / 256), steps = (m.d + 127) / 128, pairs = std::max(1, sms / 2);
    int64_t split = 4;
    while (split > 1 && (steps < 24 || items * split > sms * 7 / 16)) --split;
    const double codes = 1e-6 * m.d * ((is_packed(m.a_fmt) ? (double)m.T : 0.0) + (is_packed(m.w_fmt) ? (double)m.N : 0.0));
    return (split > 1 ? 9.4 : 7.4) + 0.27 * (double)((items * split + pairs - 1) / pairs * steps) / (double)split + (codes > 0.0 ? std::max(2.5, 0.365 * codes - 3.3) : 0.0);
}

// Whether the kernel for many tokens is the better one.  Grouped calls, by the rows to an expert (us, CUDA graphs, few / many):
//   8-bit codes: 64 51 / 60 (32 experts of 2048 x 4096), 96 61.1 / 61.1 and 21.5 / 21.3 (8 of 4096 x 2048), 100 15.5 / 14.4 (8 of 2048 x 2048), 128 26 / 22
//   4-bit weights: 512 50.8 / 54.0 (8 of 4096 x 2048), 43.7 / 55.7 (4 of 4096 x 4096), 768 72.6 / 66.4, 40.1 / 41.5 (8 of 2048 x 2048), 1024 89 / 74
//   4-bit tokens, 8-bit weights: 64 25.4 / 21.3 (8 of 4096 x 2048), 128 35 / 22
bool many_is_better(const Product &m, int sms)
{
    if (m.offsets) return m.T >= (is_packed(m.w_fmt) ? 768 : is_packed(m.a_fmt) ? 64 : 96) * (int64_t)m.E;
    if (sms <= 0) sms = 148;                             // (no device, no launch: sizes are answered for a B200)
    return m.T > 64 && many_time(m, sms) < few_time(m, sms);
}

// Pairs of CTAs that share a tile along k: as many as there is room for.  (One / two / four pairs: 256 x 4096 x 4096 15.0 / 12.9, 512 x 1024 x 4096
// 14.9 / 12.5 / 11.9, 1536 x 1024 x 9728 28 / 21; with sixteen steps in all it loses: 1024 x 2048 x 2048 10.5 / 11.3.)
int many_split(const Product &m, int64_t items, int steps, size_t smem)
{
    if (m.offsets || steps < 24) return 1;
    for (int split = 4; split > 1; --split)
        if (items <= max_clusters(perq_mm::many_kernel, perq_mm::MANY_THREADS, smem, 2 * split)) return split;
    return 1;
}

// What the kernel for many tokens wants of the workspace: packed operands as bytes, tokens first.
struct ManySpace {
    size_t tokens, weights;
};
ManySpace many_space(const Product &m)
{
    auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
    return {is_packed(m.a_fmt) ? up((size_t)m.T * (size_t)m.d) : 0, is_packed(m.w_fmt) ? up((size_t)m.E * (size_t)m.N * (size_t)m.d) : 0};
}

int launch_many(const Product &m, unsigned char *workspace, int sms, cudaStream_t st)
{
    const ManySpace space = many_space(m);
    const void *tokens = space.tokens ? workspace : m.a, *weights = space.weights ? workspace + space.tokens : m.w;
    if (space.tokens || space.weights) {
        perq_mm::SpreadParams p;
        std::memset(&p, 0, sizeof(p));
        if (space.tokens) {
            p.tokens = static_cast<const uint4 *>(m.a);
            p.tokens_out = reinterpret_cast<uint4 *>(workspace);
            p.token_chunks = (long long)m.T * m.d / 32;
        }
        if (space.weights) {
            p.weights = static_cast<const uint4 *>(m.w);
            p.weights_out = reinterpret_cast<uint4 *>(workspace + space.tokens);
            p.expert_chunks = (long long)m.N * m.d / 32;
            p.offsets = m.offsets;
        }
        p.T = (int32_t)m.T;
        p.wide = (reinterpret_cast<uintptr_t>(workspace) & 31u) == 0;            // (the weights' part begins a multiple of 256 bytes behind)
        const int parts = (space.tokens ? 1 : 0) + (space.weights ? m.E : 0);
        const long long most = std::max(p.token_chunks, p.expert_chunks), ctas = std::min<long long>((most + 511) / 512, std::max(1, 16 * sms / parts));
        if (int rc = launch_plain(perq_mm::spread_kernel, ctas, 256, 0, st, p, parts)) return rc;
    }
    perq_mm::ManyParams p;
    std::memset(&p, 0, sizeof(p));
    p.a_scales = m.a_scales;
    p.w_scales = m.w_scales;
    p.w_sums = m.w_sums;
    p.offsets = m.offsets;
    p.out = m.out;
    p.T = (int32_t)m.T;
    p.N = m.N;
    p.E = m.E;
    p.n_tiles = (m.N + perq_mm::MANY_CHANNELS - 1) / perq_mm::MANY_CHANNELS;
    p.steps = (m.d + 127) / 128;
    p.asym = m.a_fmt == PERQ_FMT_INT4_ASYM;
    p.shift = (space.tokens ? 4 : 0) + (space.weights ? 4 : 0);
    p.out_type = m.out_type;
    p.wide = (size_t)m.N * (m.out_type == PERQ_OUT_F32 ? 4 : 2) % 32 == 0 && (reinterpret_cast<uintptr_t>(m.out) & 31u) == 0;
    p.idesc = perq_mm::product_desc(!p.asym, true, perq_mm::MANY_TOKENS, perq_mm::MANY_CHANNELS);
    const int64_t token_tiles = m.offsets ? std::min<int64_t>(m.E, m.T) + m.T / perq_mm::MANY_TOKENS : (m.T + perq_mm::MANY_TOKENS - 1) / perq_mm::MANY_TOKENS;
    const int64_t items = token_tiles * p.n_tiles;
    if (items >= (1ll << 31)) return PERQ_ERR_SHAPE;
    CUtensorMap w, a;
    if (!codes_map(&w, weights, false, (uint64_t)m.E * (uint64_t)m.N, m.d, perq_mm::MANY_CHANNELS / 2) || !codes_map(&a, tokens, false, (uint64_t)m.T, m.d, 128)) return PERQ_ERR_CUDA;
    const size_t smem = 1024 + perq_mm::ManySmem::first + 8 * (m.offsets ? (size_t)m.E + 1 : 1);
    p.split = many_split(m, items, p.steps, smem);
    const int64_t clusters = p.split > 1 ? items : std::min<int64_t>(items, sms / 2);
    return launch_product(perq_mm::many_kernel, (unsigned)(2 * p.split * clusters), perq_mm::MANY_THREADS, smem, 2 * p.split, st, w, a, p);
}

int check_product(const Product &m)
{
    if (m.T < 0 || m.T > (1 << 30) || m.N <= 0 || m.N > PERQ_MAX_N || m.d <= 0 || m.d % 32 != 0 || m.d > PERQ_MAX_D) return PERQ_ERR_SHAPE;
    if (m.E < 1 || m.E > PERQ_MAX_EXPERTS || (int64_t)m.E * m.N > (1ll << 30)) return PERQ_ERR_SHAPE;
    if (m.a_fmt != PERQ_FMT_INT8 && m.a_fmt != PERQ_FMT_INT4 && m.a_fmt != PERQ_FMT_INT4_ASYM) return PERQ_ERR_FMT;
    if (m.w_fmt != PERQ_FMT_INT8 && m.w_fmt != PERQ_FMT_INT4) return PERQ_ERR_FMT;
    if (m.out_type < PERQ_OUT_BF16 || m.out_type > PERQ_OUT_F32) return PERQ_ERR_FMT;
    return PERQ_OK;
}

size_t product_workspace(const Product &m)
{
    const int sms = sm_count();
    if (m.T == 0 || !many_is_better(m, sms)) return 0;
    const ManySpace space = many_space(m);
    return space.tokens + space.weights;
}

// A workspace for m.T tokens that serves fewer too.  Which dense calls go to the kernel for many tokens is no matter of tokens alone (in 4-bit codes of
// 4096 x 4096 1024 tokens do, 1025 to 1152 do not), so the largest tile of 128 tokens is looked for that has such calls.  The first call of a tile is the
// likeliest: the other kernel takes as long for all of them, and this one no less for more.  (From above, so it is found at once for most large calls; 10 ns a
// tile where it is not.)
size_t workspace_up_to(Product m)
{
    const int sms = sm_count();
    const int64_t T = m.T;
    auto space = [&]() {
        const ManySpace s = many_space(m);
        return s.tokens + s.weights;
    };
    if (T == 0 || space() == 0) return 0;
    if (m.offsets || T <= 64) return many_is_better(m, sms) ? space() : 0;
    for (int64_t first = (T - 1) / 128 * 128 + 1; first > 0; first -= 128) {
        m.T = std::max<int64_t>(first, 65);                  // (64 and fewer go to the other kernel)
        if (many_is_better(m, sms)) {
            m.T = std::min(T, first + 127);
            return space();
        }
    }
    return 0;
}

int run_product(const Product &m, void *workspace, size_t workspace_bytes, cudaStream_t st)
{
    if (!m.a || !m.a_scales || !m.w || !m.w_scales || !m.out || (m.a_fmt == PERQ_FMT_INT4_ASYM && !m.w_sums)) return PERQ_ERR_NULL;
    const size_t need = product_workspace(m);
    if (need > 0 && (!workspace || workspace_bytes < need)) return PERQ_ERR_WORKSPACE;
    if (!aligned16(m.a) || !aligned16(m.a_scales) || !aligned16(m.w) || !aligned16(m.w_scales) || !aligned16(m.w_sums) || !aligned16(m.out) ||
        !aligned16(m.offsets) || !aligned16(workspace))
        return PERQ_ERR_ALIGN;
    const int sms = sm_count();
    if (sms <= 0) return PERQ_ERR_CUDA;
    if (many_is_better(m, sms)) return launch_many(m, static_cast<unsigned char *>(workspace), sms, st);
    const bool w4 = is_packed(m.w_fmt), a4 = is_packed(m.a_fmt);
    if (w4) return a4 ? launch_few<true, true>(m, st) : launch_few<true, false>(m, st);
    return a4 ? launch_few<false, true>(m, st) : launch_few<false, false>(m, st);
}

template <int LOG2B>
int launch_quant8_b(const perq_q8::Params &p, int pieces, long long grid, int threads, size_t smem, cudaStream_t st)
{
    using namespace perq_q8;
    switch (pieces) {
    case 1: return launch_plain(p.perm ? quant8_kernel<LOG2B, 1, true> : quant8_kernel<LOG2B, 1, false>, grid, threads, smem, st, p);
    case 2: return launch_plain(p.perm ? quant8_kernel<LOG2B, 2, true> : quant8_kernel<LOG2B, 2, false>, grid, threads, smem, st, p);
    default: return launch_plain(p.perm ? quant8_kernel<LOG2B, 4, true> : quant8_kernel<LOG2B, 4, false>, grid, threads, smem, st, p);
    }
}

int launch_quant8(const void *x, const int32_t *perm, int64_t T, int32_t d, int32_t b, void *codes, float *scales, cudaStream_t st)
{
    using namespace perq_q8;
    const int sms = sm_count();
    if (sms <= 0) return PERQ_ERR_CUDA;
    Params p;
    std::memset(&p, 0, sizeof(p));
    p.x = static_cast<const uint16_t *>(x);
    p.perm = perm;
    p.codes = static_cast<int8_t *>(codes);
    p.scales = scales;
    p.T = T;
    p.d = d;
    const int log2b = ilog2(b);
    const int all = (d + WARP_ELEMS - 1) / WARP_ELEMS;
    // Pieces of a row to a warp: a row costs a warp a fixed part, so four, but few permuted rows, whose warps gather, are better spread (us for one / two / four,
    // gaussian values: 16384 x 4096, b = 32, 174 / 103 / 51, 1531 x 9728, b = 128, 56 / 31 / 25, 148 x 4096 5.3 / 5.0 / 5.0, 1 x 4096 4.3 / 4.4 / 4.4; permuted 1 x 4096
    // 5.6 / 5.9 / 6.8, 148 6.8 / 6.6 / 7.6, 300 7.7 / 7.5 / 7.5, 1531 x 9728 63 / 46 / 39).
    const int pieces = all == 1 || (perm && T <= sms && all <= cta_warps(1)) ? 1 : all == 2 ? 2 : 4;
    p.warps = (all + pieces - 1) / pieces;
    const size_t fixed = sizeof(Shared) + (perm ? ((size_t)d * 2 + 127) / 128 * 128 : 0), row = (size_t)STAGES * (size_t)d * 2;
    int rows = (int)std::min<size_t>((size_t)(cta_warps(pieces) / p.warps), (kMaxSmem - fixed) / row);
    if (p.warps > 1) rows = std::min(rows, 8);               // (a barrier each)
    p.rows = (int)std::min<int64_t>(rows, std::max<int64_t>(1, (T + sms - 1) / sms));
    if (p.rows < 1) return PERQ_ERR_SHAPE;                   // (no width up to PERQ_MAX_D)
    const double e = b == 1 ? 0.0 : (13.0 * b / std::min(16, b / 4) - 1.0) * 0x1p-24;
    p.near_max = (float)(1.0 - 2.0 * e - 0x1p-22);
    p.doubt = (float)(1.001 * (2.0 * e + 9.0 * 0x1p-24));
    p.inv_scale = 1.0 / (127.0 * std::sqrt((double)b));
    const int threads = p.rows * p.warps * 32;
    const size_t smem = fixed + (size_t)p.rows * row;
    const long long grid = std::min<long long>((T + p.rows - 1) / p.rows, sms);
    switch (log2b) {
    case 0: return launch_quant8_b<0>(p, pieces, grid, threads, smem, st);
    case 4: return launch_quant8_b<4>(p, pieces, grid, threads, smem, st);
    case 5: return launch_quant8_b<5>(p, pieces, grid, threads, smem, st);
    case 6: return launch_quant8_b<6>(p, pieces, grid, threads, smem, st);
    case 7: return launch_quant8_b<7>(p, pieces, grid, threads, smem, st);
    case 8: return launch_quant8_b<8>(p, pieces, grid, threads, smem, st);
    default: return launch_quant8_b<9>(p, pieces, grid, threads, smem, st);
    }
}

}  // namespace

cudaError_t perq_mm_read_error(unsigned int *flags) { return cudaMemcpyFromSymbol(flags, perq_mm::g_error, sizeof *flags); }
cudaError_t perq_mm_clear_error()
{
    const unsigned int zero = 0;
    return cudaMemcpyToSymbol(perq_mm::g_error, &zero, sizeof zero);
}

extern "C" {

int perq_rotate_quantize_i8(const void *x, const int32_t *perm, int64_t T, int32_t d, int32_t b, void *out_codes, float *out_scales, void *stream)
{
    if (T < 0 || d <= 0 || d % 32 != 0 || d > PERQ_MAX_D) return PERQ_ERR_SHAPE;
    if (!is_pow2(b) || (b != 1 && b < 16) || b > d || d % b != 0) return PERQ_ERR_BLOCK;
    if (b > 1 << perq_q8::MAX_LOG2B) return PERQ_ERR_UNSUPPORTED;
    if (T == 0) return PERQ_OK;
    if (!x || !out_codes || !out_scales) return PERQ_ERR_NULL;
    if (!aligned16(x) || !aligned16(perm) || !aligned16(out_codes) || !aligned16(out_scales)) return PERQ_ERR_ALIGN;
    return launch_quant8(x, perm, T, d, b, out_codes, out_scales, static_cast<cudaStream_t>(stream));
}

int perq_code_sums(const void *codes, int32_t fmt, int64_t rows, int32_t d, int32_t *sums, void *stream)
{
    if (rows < 0 || rows > (1ll << 30) || d <= 0 || d % 32 != 0 || d > PERQ_MAX_D) return PERQ_ERR_SHAPE;
    if (fmt != PERQ_FMT_INT8 && fmt != PERQ_FMT_INT4) return PERQ_ERR_FMT;
    if (rows == 0) return PERQ_OK;
    if (!codes || !sums) return PERQ_ERR_NULL;
    if (!aligned16(codes) || !aligned16(sums)) return PERQ_ERR_ALIGN;
    perq_q8::SumParams p;
    p.codes = codes;
    p.sums = sums;
    p.rows = rows;
    p.packed = is_packed(fmt);
    p.chunks = d / (p.packed ? 32 : 16);
    return launch_plain(perq_q8::code_sums_kernel, (rows + 7) / 8, 256, 0, static_cast<cudaStream_t>(stream), p);
}

int perq_matmul_i8_workspace_bytes(int64_t T, int32_t N, int32_t d, int32_t a_fmt, int32_t w_fmt, size_t *bytes)
{
    const Product m = {nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, T, N, d, 1, a_fmt, w_fmt, PERQ_OUT_BF16};
    if (int rc = check_product(m)) return rc;
    if (!bytes) return PERQ_ERR_NULL;
    *bytes = workspace_up_to(m);
    return PERQ_OK;
}

int perq_matmul_i8(const void *a_codes, const float *a_scales, int32_t a_fmt, const void *w_codes, const float *w_scales, int32_t w_fmt, const int32_t *w_sums,
                   int64_t T, int32_t N, int32_t d, void *out, int32_t out_type, void *workspace, size_t workspace_bytes, void *stream)
{
    const Product m = {a_codes, w_codes, a_scales, w_scales, w_sums, nullptr, out, T, N, d, 1, a_fmt, w_fmt, out_type};
    if (int rc = check_product(m)) return rc;
    if (T == 0) return PERQ_OK;
    return run_product(m, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

int perq_grouped_matmul_i8_workspace_bytes(int64_t T, int32_t E, int32_t N, int32_t d, int32_t a_fmt, int32_t w_fmt, size_t *bytes)
{
    // (offsets only says that there are some)
    const Product m = {nullptr, nullptr, nullptr, nullptr, nullptr, reinterpret_cast<const int32_t *>(16), nullptr, T, N, d, E, a_fmt, w_fmt, PERQ_OUT_BF16};
    if (int rc = check_product(m)) return rc;
    if (!bytes) return PERQ_ERR_NULL;
    *bytes = workspace_up_to(m);
    return PERQ_OK;
}

int perq_grouped_matmul_i8(const void *a_codes, const float *a_scales, int32_t a_fmt, const void *w_codes, const float *w_scales, int32_t w_fmt,
                           const int32_t *w_sums, const int32_t *offsets, int64_t T, int32_t E, int32_t N, int32_t d, void *out, int32_t out_type, void *workspace,
                           size_t workspace_bytes, void *stream)
{
    const Product m = {a_codes, w_codes, a_scales, w_scales, w_sums, offsets, out, T, N, d, E, a_fmt, w_fmt, out_type};
    if (int rc = check_product(m)) return rc;
    if (T == 0) return PERQ_OK;
    if (!offsets) return PERQ_ERR_NULL;
    return run_product(m, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
