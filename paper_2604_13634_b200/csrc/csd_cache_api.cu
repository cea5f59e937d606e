// C ABI of the decode-pass operators: rotary positions, the paged cache, attention over it (declared in include/csd.h).
#include <atomic>
#include <climits>
#include <cmath>
#include <cstring>

#include "../../include/csd.h"
#include "csd_host.h"
#include "csd_attention.cuh"
#include "csd_pages.cuh"
#include "csd_rope.cuh"

using namespace csd;

namespace {

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// A launch that may begin beside the end of what is before it on the stream (the kernels wait themselves before they touch
// global memory).
template <typename... P, typename... A>
csd_status_t launch(void (*kernel)(P...), dim3 grid, unsigned int threads, size_t smem, cudaStream_t st, const A &...args)
{
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) {
        (void)cudaGetLastError();
        return CSD_ERR_CUDA;
    }
    return CSD_OK;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// ---- rotary positions ---------------------------------------------------------------------------

bool rope_ok(const csd_rope_t *r, int D)
{
    return r->steps && r->rot >= 2 && r->rot % 2 == 0 && r->rot <= D &&
           (r->layout == CSD_ROPE_HALF || r->layout == CSD_ROPE_INTERLEAVED) && std::isfinite(r->magnitude);
}

// How a head's row is cut.  Units of 16 bytes' worth of pairs where rot divides into them; single 16-byte vectors where the row does; else pair by pair.
enum class Cut { kUnits, kVectors, kPairs };

Cut cut_of(int P, int rot, int D, bool vectors)
{
    if (!vectors || D % P != 0 || D / P > rope::kThreads) return Cut::kPairs;
    return rot % (2 * P) == 0 ? Cut::kUnits : Cut::kVectors;
}

int units_of(Cut cut, int P, int rot, int D)
{
    if (cut == Cut::kVectors) return D / P;
    if (cut == Cut::kPairs) P = 1;
    return rot / (2 * P) + (D - rot + 2 * P - 1) / (2 * P);
}

// Blocks of whole tokens where they fit, blocks of a token's groups of heads where one takes more; false: too many.
bool place_tokens(long long tokens, long long groups, int units, rope::Places &at, dim3 &grid)
{
    const long long per_token = groups * units;
    if (tokens > INT_MAX - rope::kThreads || per_token > INT_MAX) return false;      // the last block's tokens are counted past the end
    at.n_tokens = static_cast<int>(tokens);
    at.per_token = static_cast<int>(per_token);
    at.tokens = per_token >= rope::kThreads ? 1 : rope::kThreads / at.per_token;
    at.groups = rope::kThreads / units;
    const long long taken = at.groups > 0 ? static_cast<long long>(at.groups) * units : rope::kThreads;
    const long long rows = at.tokens > 1 ? 1 : (per_token + taken - 1) / taken;
    if (rows > 65535) return false;
    grid = dim3(static_cast<unsigned int>((tokens + at.tokens - 1) / at.tokens), static_cast<unsigned int>(rows));
    return true;
}

int groups_of(int heads) { return (heads - 1) / rope::kHeads + 1; }         // (of any positive count: a sum could pass 31 bits)

template <typename T>
csd_status_t run_rope(rope::RopeParams p, csd_rope_layout_t layout, cudaStream_t st)
{
    constexpr int P = 16 / static_cast<int>(sizeof(T));
    const long long all = p.xb | p.xs | p.xh | p.yb | p.ys | p.yh;
    const Cut cut = cut_of(P, p.turn.rot, p.D, all % P == 0 && aligned16(p.x) && aligned16(p.y));
    p.units = units_of(cut, P, p.turn.rot, p.D);
    dim3 grid;
    if (!place_tokens(static_cast<long long>(p.B) * p.S, groups_of(p.H), p.units, p.at, grid)) return CSD_ERR_UNSUPPORTED;
    const bool half = layout == CSD_ROPE_HALF;
    auto go = [&](auto kernel) { return launch(kernel, grid, rope::kThreads, 0, st, p); };
    if (cut == Cut::kUnits) return go(half ? rope::rope_kernel<T, P, true, false> : rope::rope_kernel<T, P, false, false>);
    if (cut == Cut::kVectors) return go(half ? rope::rope_kernel<T, P, true, true> : rope::rope_kernel<T, P, false, true>);
    return go(half ? rope::rope_kernel<T, 1, true, false> : rope::rope_kernel<T, 1, false, false>);
}

template <typename T>
csd_status_t run_append(rope::AppendParams p, csd_rope_layout_t layout, cudaStream_t st)
{
    constexpr int P = 8;
    const long long all = p.qb | p.qt | p.qh | p.kb | p.kt | p.kh | p.vb | p.vt | p.vh;
    const Cut cut = cut_of(P, p.turn.rot, p.D, all % P == 0 && aligned16(p.q) && aligned16(p.k) && aligned16(p.v) && aligned16(p.q_out));
    p.units = units_of(cut, P, p.turn.rot, p.D);
    p.q_groups = groups_of(p.Hq);
    p.kv_groups = groups_of(p.Hkv);
    dim3 grid;
    if (!place_tokens(static_cast<long long>(p.B) * p.T, p.q_groups + 2ll * p.kv_groups, p.units, p.at, grid)) return CSD_ERR_UNSUPPORTED;
    const bool half = layout == CSD_ROPE_HALF;
    auto go = [&](auto kernel) { return launch(kernel, grid, rope::kThreads, 0, st, p); };
    if (cut == Cut::kUnits) return go(half ? rope::rope_append_kernel<T, P, true, false> : rope::rope_append_kernel<T, P, false, false>);
    if (cut == Cut::kVectors) return go(half ? rope::rope_append_kernel<T, P, true, true> : rope::rope_append_kernel<T, P, false, true>);
    return go(half ? rope::rope_append_kernel<T, 1, true, false> : rope::rope_append_kernel<T, 1, false, false>);
}

// ---- the cache ----------------------------------------------------------------------------------

constexpr int kStatusWords = 64;                     // flags, page copies wanted, reserved

bool cache_shape_ok(int rows, int max_pages, int n_pages)
{
    return rows > 0 && rows <= CSD_CACHE_MAX_ROWS && max_pages > 0 && n_pages > 0 && n_pages <= (1 << 28) &&
           static_cast<long long>(rows) * (max_pages + 1ll) <= (1ll << 31) - 1;
}

csd_cache_layout_t meta_layout(int rows, int max_pages, int n_pages)
{
    csd_cache_layout_t l;
    size_t at = 0;
    auto take = [&](size_t words) {
        const size_t o = at;
        at = align_up(at + words * 4, 256);
        return o;
    };
    l.flags = take(kStatusWords);
    l.lens = take(static_cast<size_t>(rows));
    l.granted = take(static_cast<size_t>(rows));
    l.table = take(static_cast<size_t>(rows) * max_pages);
    l.refs = take(static_cast<size_t>(n_pages));
    l.free_bits = take((static_cast<size_t>(n_pages) + 31) / 32);
    l.total = at;
    return l;
}

struct ScratchLayout {
    size_t moves, list, staged, total;
};

ScratchLayout scratch_layout(int rows, int max_pages, int n_pages)
{
    ScratchLayout s;
    // a copy per row (extend) or per second page (compact), and one word more
    const size_t pairs = static_cast<size_t>(rows > n_pages / 2 ? rows : n_pages / 2) + 1;
    s.moves = 0;
    s.list = align_up(pairs * 8, 256);
    s.staged = s.list + align_up(static_cast<size_t>(n_pages) * 4, 256);
    s.total = s.staged + align_up(static_cast<size_t>(rows) * (max_pages + 1) * 4, 256);
    return s;
}

csd_status_t check_cache(const csd_cache_t *c)
{
    if (!c || !c->k || !c->v || !c->meta || !c->scratch) return CSD_ERR_INVALID_ARG;
    if (c->dtype != CSD_BF16 && c->dtype != CSD_F16) return c->dtype == CSD_F32 ? CSD_ERR_UNSUPPORTED : CSD_ERR_INVALID_ARG;
    if (c->layers <= 0 || c->n_pages <= 0 || c->heads <= 0 || c->dim <= 0 || c->rows <= 0 || c->max_pages <= 0) return CSD_ERR_INVALID_ARG;
    if (c->page_size < 8 || c->page_size > 256 || (c->page_size & (c->page_size - 1)) != 0) return CSD_ERR_UNSUPPORTED;
    if (c->dim % 8 != 0 || c->dim > 256 || c->heads > 4096) return CSD_ERR_UNSUPPORTED;
    // (a copy of a page has a row of the grid for every layer's keys and values; its pieces are counted in 31 bits)
    const long long pieces = (static_cast<long long>(c->heads) * c->page_size * c->dim * 2 + pages::kCopyBytes - 1) / pages::kCopyBytes;
    if (c->layers > 32767 || (c->rows > c->n_pages / 2 ? c->rows : c->n_pages / 2) * pieces > INT_MAX) return CSD_ERR_UNSUPPORTED;
    if (!cache_shape_ok(c->rows, c->max_pages, c->n_pages) || static_cast<long long>(c->max_pages) * c->page_size > (1ll << 30)) return CSD_ERR_UNSUPPORTED;
    if (!aligned16(c->k) || !aligned16(c->v)) return CSD_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(c->meta) & 255u) || (reinterpret_cast<uintptr_t>(c->scratch) & 255u)) return CSD_ERR_INVALID_ARG;
    const int64_t page = static_cast<int64_t>(c->heads) * c->page_size * c->dim;
    const bool heads_outside = c->stride_token == c->dim && c->stride_head == static_cast<int64_t>(c->page_size) * c->dim;
    const bool tokens_outside = c->stride_head == c->dim && c->stride_token == static_cast<int64_t>(c->heads) * c->dim;
    // (with one head or eight-token pages the two orders can coincide; either reading is then the same memory)
    const bool one_head = c->heads == 1 && c->stride_token == c->dim;
    if (!heads_outside && !tokens_outside && !one_head) return CSD_ERR_INVALID_ARG;
    if (c->stride_page < page || c->stride_page % 8 != 0 || c->stride_page > (1ll << 36)) return CSD_ERR_INVALID_ARG;
    if (c->layers > 1) {
        if (c->stride_layer % 8 != 0 || c->stride_layer > (1ll << 40)) return CSD_ERR_INVALID_ARG;
        const bool layers_outside = c->stride_layer >= (c->n_pages - 1ll) * c->stride_page + page;
        const bool pages_outside = c->stride_layer >= page && c->stride_page >= (c->layers - 1ll) * c->stride_layer + page;
        if (!layers_outside && !pages_outside) return CSD_ERR_INVALID_ARG;
    }
    return CSD_OK;
}

pages::View view_of(const csd_cache_t *c)
{
    const csd_cache_layout_t l = meta_layout(c->rows, c->max_pages, c->n_pages);
    const ScratchLayout s = scratch_layout(c->rows, c->max_pages, c->n_pages);
    char *m = static_cast<char *>(c->meta), *x = static_cast<char *>(c->scratch);
    pages::View v;
    v.rows = c->rows;
    v.max_pages = c->max_pages;
    v.n_pages = c->n_pages;
    v.page_size = c->page_size;
    v.page_shift = 0;
    while ((1 << v.page_shift) < c->page_size) ++v.page_shift;
    v.words = (c->n_pages + 31) / 32;
    v.flags = reinterpret_cast<unsigned int *>(m + l.flags);
    v.n_moves = reinterpret_cast<int *>(m + l.flags) + 1;
    v.lens = reinterpret_cast<int *>(m + l.lens);
    v.granted = reinterpret_cast<int *>(m + l.granted);
    v.table = reinterpret_cast<int *>(m + l.table);
    v.refs = reinterpret_cast<int *>(m + l.refs);
    v.free_bits = reinterpret_cast<unsigned int *>(m + l.free_bits);
    v.moves = reinterpret_cast<int *>(x + s.moves);
    v.list = reinterpret_cast<int *>(x + s.list);
    v.staged = reinterpret_cast<int *>(x + s.staged);
    return v;
}

// The copies that the bookkeeping launch before has listed; at most `most` pages.
csd_status_t copy_pages(const csd_cache_t *c, const pages::View &v, long long most, cudaStream_t st)
{
    pages::CopyParams p;
    p.k = static_cast<char *>(c->k);
    p.v = static_cast<char *>(c->v);
    p.layer_bytes = c->stride_layer * 2;
    p.page_stride_bytes = c->stride_page * 2;
    p.page_bytes = c->heads * c->page_size * c->dim * 2;
    p.layers = c->layers;
    p.pieces = (p.page_bytes + pages::kCopyBytes - 1) / pages::kCopyBytes;
    p.n_moves = v.n_moves;
    p.moves = v.moves;
    const long long per_block = pages::kCopyThreads / 32, planes = 2ll * p.layers;
    long long blocks = (most * p.pieces + per_block - 1) / per_block;
    const long long cap = (static_cast<long long>(host::multiprocessors()) * 8 + planes - 1) / planes;
    if (blocks > cap) blocks = cap;
    if (blocks < 1) return CSD_OK;
    return launch(pages::pages_copy_kernel, dim3(static_cast<unsigned int>(blocks), static_cast<unsigned int>(planes)), pages::kCopyThreads, 0, st, p);
}

// ---- attention ----------------------------------------------------------------------------------

constexpr int kMaxDevices = 64;
constexpr int kSmemPerSm = 228 * 1024, kSmemReserved = 1024, kSmemStatic = 1024;     // per block: the system's, and the kernel's own

struct AttentionPlan {
    int rows, row_tiles, tile_rows, dp, grid, stages, smem, run_cost, q_buffers;
    size_t splits_off, parts_off, total;
};

int attention_grid(int blocks_per_sm)
{
    const int g = host::multiprocessors() * blocks_per_sm;
    return g < attention::kMaxGrid ? g : attention::kMaxGrid;
}

template <typename C>
AttentionPlan attention_plan(int rows, int B)
{
    AttentionPlan a;
    a.rows = rows;
    a.tile_rows = C::kRows;
    a.dp = C::DP;
    a.row_tiles = (rows + C::kRows - 1) / C::kRows;
    a.grid = attention_grid(C::kBlocksPerSm);
    a.run_cost = 2;      // measured: 2 to 3 of 64-element tiles, no difference from 1 to 3 beyond
    const int limit = kSmemPerSm / C::kBlocksPerSm - kSmemReserved - kSmemStatic;
    const int fixed = 1024 + C::kQBytes + C::kMlBytes + (B + 1) * 4;
    a.stages = (limit - fixed) / C::kStageBytes;
    if (a.stages > attention::kMaxStages) a.stages = attention::kMaxStages;
    a.smem = fixed + a.stages * C::kStageBytes;
    a.splits_off = 0;
    a.parts_off = align_up(static_cast<size_t>(a.grid) * sizeof(attention::Split), 256);
    a.total = a.parts_off + static_cast<size_t>(2) * a.grid * C::kSlotFloats * 4;
    return a;
}

template <typename T, typename F>
auto with_config(int dim, F f)
{
    using attention::Config;
    if (dim <= 64) return f(Config<T, 64, 2, 2>());
    if (dim <= 128) return f(Config<T, 128, 1, 2>());
    return f(Config<T, 256, 1, 1>());
}

// Which kernel: up to 16 query rows per (row, key head) fit the register tiles of the mma.sync kernel (97 us where the other takes 107,
// 16 query rows of 128 elements); beyond, the tensor-memory kernel, with row tiles of at most 128 (105 us against 156 with 20 rows).
bool attention_uses_tc(int rows) { return rows > 16; }

// Two blocks per SM while their accumulators fit in half of the tensor memory each (128 + dim columns of 512).
int tc_blocks(int dim) { return dim <= 128 ? 2 : 1; }

// Products of 64 rows: a warp of the softmax then has 16 query rows, not 32.  On a cool GPU that is 0 to 2 % faster, but the products
// draw less, and kept busy for a second the clock stays higher.  Busy, 64 rows against 128: 243 us and 262 for 128 rows of 500 to 4000 in
// pages of 16 (36 query rows of 128 elements), 258 and 269 (64), 113 and 120 for 32 ragged rows up to 8191 (30); 131 and 140 (32 query rows
// of 256 elements); with 64 elements in pages of 64 tokens 144 and 152 (32), but 159 and 158 (48, cool 160 and 144) and 165 and 161 (64,
// cool 163 and 147), where twice the warps' work counts; in pages of 16 the loads hide the difference (169 and 170 with 32).
bool tc_products_of_64(int tile_rows, int dim) { return tile_rows <= (dim <= 64 ? 32 : 64); }

AttentionPlan attention_tc_plan(int rows, int dim, int B)
{
    AttentionPlan a;
    a.rows = rows;
    a.dp = dim <= 64 ? 64 : (dim <= 128 ? 128 : 256);
    a.grid = attention_grid(tc_blocks(dim));
    a.run_cost = a.dp == 64 ? 8 : (a.dp == 128 ? 4 : 2);      // about 5 us: 240 us at 2, 228 at 4, 231 at 6 for 1024 units of 8 to 63 tiles
    const int halves = (dim + 63) / 64, slot = halves * attention::kTcTile * 128;
    const int limit = kSmemPerSm / tc_blocks(dim) - kSmemReserved - kSmemStatic;
    // The kernel's waits want four slots at least: two sets of query rows give way to one for them, and where tables of thousands
    // of rows leave little, a row tile holds fewer query rows.
    for (int most = 128;; most /= 2) {
        a.row_tiles = (rows + most - 1) / most;
        a.tile_rows = ((rows + a.row_tiles - 1) / a.row_tiles + 7) / 8 * 8;
        a.row_tiles = (rows + a.tile_rows - 1) / a.tile_rows;
        for (a.q_buffers = 2; a.q_buffers >= 1; --a.q_buffers) {
            const int fixed = 1024 + a.q_buffers * halves * a.tile_rows * 128 + (B + 1) * 4;
            a.stages = (limit - fixed) / slot;
            if (a.stages > attention::kTcMaxSlots) a.stages = attention::kTcMaxSlots;
            a.smem = fixed + a.stages * slot;
            if (a.stages >= 4) break;
        }
        if (a.stages >= 4 || most == 16) break;
    }
    a.splits_off = 0;
    a.parts_off = align_up(static_cast<size_t>(a.grid) * sizeof(attention::Split), 256);
    a.total = a.parts_off + static_cast<size_t>(2) * a.grid * a.tile_rows * (a.dp + 2) * 4;
    return a;
}

AttentionPlan attention_plan_of(int T, int group, int dim, int B)
{
    if (attention_uses_tc(T * group)) return attention_tc_plan(T * group, dim, B);
    return with_config<__nv_bfloat16>(dim, [&](auto cfg) { return attention_plan<decltype(cfg)>(T * group, B); });
}

bool attention_shape_ok(int rows, int T, int q_heads, int heads, int dim)
{
    if (rows <= 0 || rows > CSD_CACHE_MAX_ROWS || T <= 0 || T > CSD_MAX_K + 1 || heads <= 0 || heads > 4096 || q_heads <= 0 || q_heads > (1 << 16) ||
        q_heads % heads != 0 || dim <= 0 || dim > 256 || dim % 8 != 0)
        return false;
    return static_cast<long long>(rows) * T * q_heads <= (1ll << 27);
}

// A layer's keys or values as [n_pages, heads, page_size, dim] with boxes of 64 elements x box_rows places, 128-byte swizzle.  L2 fetches
// of 128 bytes: with 256 a head of 64 elements whose tokens lie apart pulls its neighbour in as well, which another block wants
// at another time (135 us against 99 for 583 MB; no difference for 128 elements).
bool make_pool_map(CUtensorMap *map, const csd_cache_t *c, const void *pool, int layer, int box_rows)
{
    const host::EncodeTiledFn fn = host::encode_tiled();
    if (!fn) return false;
    char *base = static_cast<char *>(const_cast<void *>(pool)) + layer * c->stride_layer * 2;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(c->dim), static_cast<cuuint64_t>(c->page_size), static_cast<cuuint64_t>(c->heads),
                                static_cast<cuuint64_t>(c->n_pages)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(c->stride_token) * 2, static_cast<cuuint64_t>(c->stride_head) * 2,
                                   static_cast<cuuint64_t>(c->stride_page) * 2};
    const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(box_rows), 1, 1};
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    return fn(map, c->dtype == CSD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, strides, box, ones,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Lets a kernel use the shared memory it wants, once per device; `split_regs` is what its warpgroups must find at launch, in
// registers per thread summed over `groups` of them (a larger share than there is would be waited for).
template <typename K>
bool kernel_ready(K kernel, std::atomic<bool> (&done)[kMaxDevices], int smem, int groups, int split_regs)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
        (void)cudaGetLastError();
        return false;
    }
    if (done[dev].load()) return true;
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, kernel) != cudaSuccess || attr.numRegs * groups < split_regs ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    done[dev].store(true);
    return true;
}

// Common to both kernels: the plan's numbers, and what is known of the units before the lengths are read.
void fill_plan(attention::Params &p, const AttentionPlan &a, char *ws)
{
    p.rows = a.rows;
    p.row_tiles = a.row_tiles;
    p.n_stages = a.stages;
    p.run_cost = a.run_cost;
    p.by_unit = static_cast<long long>(p.B) * p.Hkv * a.row_tiles <= a.grid ? 1 : 0;
    p.splits = reinterpret_cast<attention::Split *>(ws + a.splits_off);
    p.parts = reinterpret_cast<float *>(ws + a.parts_off);
}

template <typename T, int DP>
csd_status_t launch_join(const attention::Params &p, const AttentionPlan &a, cudaStream_t st)
{
    const int most = a.rows < a.tile_rows ? a.rows : a.tile_rows;
    const unsigned int units = static_cast<unsigned int>(p.by_unit ? p.B * p.Hkv * a.row_tiles : a.grid);
    // a block per row where a unit may have 32 parts or more (8 units of 37: 90.1 us against 91.5 with four rows to a block, 40.0
    // against 41.6 with 72 rows; with four: 39.3 against 41.3 for 16 units of 18, 28.0 against 29.8 for 256, 206 against 212 for 1024)
    if (a.grid >= 32ll * units)
        return launch(attention::attention_join_kernel<T, DP, 1>, dim3(units, static_cast<unsigned int>(most)), attention::kJoinThreads, 0, st, p, a.tile_rows);
    return launch(attention::attention_join_kernel<T, DP, 4>, dim3(units, static_cast<unsigned int>((most + 3) / 4)), attention::kJoinThreads, 0, st, p, a.tile_rows);
}

template <typename C>
csd_status_t run_attention(attention::Params p, const csd_cache_t *cache, int layer, char *ws, cudaStream_t st)
{
    static std::atomic<bool> ready[kMaxDevices];
    if (!kernel_ready(attention::attention_kernel<C>, ready, kSmemPerSm / C::kBlocksPerSm - kSmemReserved - kSmemStatic, C::kGroups,
                      C::kMoveRegs ? C::kConsumerRegs * (C::kGroups - 1) + C::kProducerRegs : 0))
        return CSD_ERR_CUDA;
    const AttentionPlan a = attention_plan<C>(p.T * p.group, p.B);
    fill_plan(p, a, ws);
    p.box_rows = cache->page_size < C::kTile ? cache->page_size : C::kTile;
    CUtensorMap map_k, map_v;
    if (!make_pool_map(&map_k, cache, cache->k, layer, p.box_rows) || !make_pool_map(&map_v, cache, cache->v, layer, p.box_rows)) return CSD_ERR_CUDA;
    const csd_status_t rc = launch(attention::attention_kernel<C>, dim3(static_cast<unsigned int>(a.grid)), C::kThreads, static_cast<size_t>(a.smem), st, map_k, map_v, p);
    return rc != CSD_OK ? rc : launch_join<typename C::T, C::DP>(p, a, st);
}

template <typename T, int kBlocks, int kM>
csd_status_t run_attention_tc(attention::Params p, const AttentionPlan &a, const csd_cache_t *cache, int layer, char *ws, cudaStream_t st)
{
    static std::atomic<bool> ready[kMaxDevices];
    if (!kernel_ready(attention::attention_tc_kernel<T, kBlocks, kM>, ready, kSmemPerSm / kBlocks - kSmemReserved - kSmemStatic, 1, 0)) return CSD_ERR_CUDA;
    fill_plan(p, a, ws);
    p.tile_rows = a.tile_rows;
    p.q_buffers = a.q_buffers;
    p.part_stride = a.dp;
    p.halves = (p.D + 63) / 64;
    p.d16 = (p.D + 15) / 16 * 16;
    p.box_rows = cache->page_size < attention::kTcTile ? cache->page_size : attention::kTcTile;
    p.k_pool = static_cast<char *>(cache->k) + layer * cache->stride_layer * 2;
    p.v_pool = static_cast<char *>(cache->v) + layer * cache->stride_layer * 2;
    p.pool_page = cache->stride_page;
    p.pool_head = cache->stride_head;
    p.pool_token = cache->stride_token;
    CUtensorMap map_k, map_v;
    if (!make_pool_map(&map_k, cache, cache->k, layer, p.box_rows) || !make_pool_map(&map_v, cache, cache->v, layer, p.box_rows)) return CSD_ERR_CUDA;
    const csd_status_t rc = launch(attention::attention_tc_kernel<T, kBlocks, kM>, dim3(static_cast<unsigned int>(a.grid)), attention::kTcThreads,
                                   static_cast<size_t>(a.smem), st, map_k, map_v, p);
    if (rc != CSD_OK) return rc;
    if (a.dp == 64) return launch_join<T, 64>(p, a, st);
    if (a.dp == 128) return launch_join<T, 128>(p, a, st);
    return launch_join<T, 256>(p, a, st);
}

template <typename T>
csd_status_t run_attention_any(const attention::Params &p, const csd_cache_t *cache, int layer, char *ws, cudaStream_t st)
{
    if (attention_uses_tc(p.T * p.group)) {
        const AttentionPlan a = attention_tc_plan(p.T * p.group, p.D, p.B);
        if (tc_products_of_64(a.tile_rows, p.D))
            return tc_blocks(p.D) == 2 ? run_attention_tc<T, 2, 64>(p, a, cache, layer, ws, st) : run_attention_tc<T, 1, 64>(p, a, cache, layer, ws, st);
        return tc_blocks(p.D) == 2 ? run_attention_tc<T, 2, 128>(p, a, cache, layer, ws, st) : run_attention_tc<T, 1, 128>(p, a, cache, layer, ws, st);
    }
    return with_config<T>(p.D, [&](auto cfg) { return run_attention<decltype(cfg)>(p, cache, layer, ws, st); });
}

}  // namespace

extern "C" {

csd_status_t csd_rope_steps(int rot, double base, csd_rope_scaling_t scaling, double factor, double original_len, double low,
                            double high, uint64_t *steps, float *magnitude)
{
    if (!steps || !magnitude || rot < 2 || rot % 2 != 0 || rot > 65536) return CSD_ERR_INVALID_ARG;
    if (!(base > 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor)) return CSD_ERR_INVALID_ARG;
    if (scaling < CSD_ROPE_PLAIN || scaling > CSD_ROPE_YARN) return CSD_ERR_INVALID_ARG;
    if (scaling >= CSD_ROPE_PARTS &&
        (!(original_len > 0.0) || !std::isfinite(original_len) || !(low > 0.0) || !(high > low) || !std::isfinite(high)))
        return CSD_ERR_INVALID_ARG;
    const double two_pi = 2.0 * 3.14159265358979323846;
    const double b = scaling == CSD_ROPE_BASE && rot > 2 ? base * std::pow(factor, rot / (rot - 2.0)) : base;
    double from = 0.0, to = 0.0;                     // pairs between which the blend of YARN goes
    if (scaling == CSD_ROPE_YARN) {
        from = std::floor(rot * std::log(original_len / (high * two_pi)) / (2.0 * std::log(base)));
        to = std::ceil(rot * std::log(original_len / (low * two_pi)) / (2.0 * std::log(base)));
        if (from < 0.0) from = 0.0;
        if (to > rot - 1.0) to = rot - 1.0;
        if (to - from < 0.001) to = from + 0.001;
    }
    for (int i = 0; i < rot / 2; ++i) {
        double th = std::pow(b, -2.0 * i / rot), keep = 1.0;
        if (scaling == CSD_ROPE_LINEAR) keep = 0.0;
        if (scaling == CSD_ROPE_PARTS) keep = (original_len * th / two_pi - low) / (high - low);
        if (scaling == CSD_ROPE_YARN) keep = 1.0 - (i - from) / (to - from);
        keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
        if (scaling != CSD_ROPE_PLAIN && scaling != CSD_ROPE_BASE) th = th * keep + th / factor * (1.0 - keep);
        steps[i] = static_cast<uint64_t>(std::nearbyint(th / two_pi * 18446744073709551616.0));    // below 2^62
    }
    *magnitude = scaling == CSD_ROPE_YARN ? static_cast<float>(0.1 * std::log(factor) + 1.0) : 1.0f;
    return CSD_OK;
}

csd_status_t csd_rope(const void *x, void *y, csd_dtype_t dtype, int B, int S, int H, int D, int64_t x_stride_b, int64_t x_stride_s,
                      int64_t x_stride_h, int64_t y_stride_b, int64_t y_stride_s, int64_t y_stride_h, const int32_t *positions,
                      int64_t pos_stride_b, int64_t pos_stride_s, const csd_rope_t *rope, int inverse, void *stream)
{
    if (!rope || B < 0 || S < 0 || H < 0 || D <= 0 || !rope_ok(rope, D)) return CSD_ERR_INVALID_ARG;
    if (dtype != CSD_F32 && dtype != CSD_BF16 && dtype != CSD_F16) return CSD_ERR_INVALID_ARG;
    if (rope->rot > rope::kMaxRot) return CSD_ERR_UNSUPPORTED;
    if (B == 0 || S == 0 || H == 0) return CSD_OK;
    if (!x || !y || !positions) return CSD_ERR_INVALID_ARG;
    host::other_work_enqueued();
    rope::RopeParams p;
    std::memset(&p, 0, sizeof p);
    p.x = x;
    p.y = y;
    p.B = B; p.S = S; p.H = H; p.D = D;
    p.xb = x_stride_b; p.xs = x_stride_s; p.xh = x_stride_h;
    p.yb = y_stride_b; p.ys = y_stride_s; p.yh = y_stride_h;
    p.positions = positions;
    p.pb = pos_stride_b; p.ps = pos_stride_s;
    p.turn.steps = reinterpret_cast<const unsigned long long *>(rope->steps);
    p.turn.rot = rope->rot;
    p.turn.magnitude = rope->magnitude;
    p.inverse = inverse;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == CSD_F32) return run_rope<float>(p, rope->layout, st);
    if (dtype == CSD_BF16) return run_rope<__nv_bfloat16>(p, rope->layout, st);
    return run_rope<__half>(p, rope->layout, st);
}

csd_status_t csd_rope_append(const void *q, int64_t q_stride_b, int64_t q_stride_t, int64_t q_stride_h, int q_heads, const void *k,
                             int64_t k_stride_b, int64_t k_stride_t, int64_t k_stride_h, const void *v, int64_t v_stride_b,
                             int64_t v_stride_t, int64_t v_stride_h, void *q_out, int T, const csd_cache_t *cache, int layer,
                             const csd_rope_t *rope, const int32_t *n_new, void *stream)
{
    const csd_status_t ok = check_cache(cache);
    if (ok != CSD_OK) return ok;
    if (!q || !k || !v || !q_out || T <= 0 || q_heads <= 0 || layer < 0 || layer >= cache->layers) return CSD_ERR_INVALID_ARG;
    if (rope && !rope_ok(rope, cache->dim)) return CSD_ERR_INVALID_ARG;
    host::other_work_enqueued();
    const pages::View pv = view_of(cache);
    rope::AppendParams p;
    std::memset(&p, 0, sizeof p);
    p.q = q; p.k = k; p.v = v;
    p.q_out = q_out;
    p.k_pool = static_cast<char *>(cache->k) + layer * cache->stride_layer * 2;
    p.v_pool = static_cast<char *>(cache->v) + layer * cache->stride_layer * 2;
    p.B = cache->rows; p.T = T; p.Hq = q_heads; p.Hkv = cache->heads; p.D = cache->dim;
    p.qb = q_stride_b; p.qt = q_stride_t; p.qh = q_stride_h;
    p.kb = k_stride_b; p.kt = k_stride_t; p.kh = k_stride_h;
    p.vb = v_stride_b; p.vt = v_stride_t; p.vh = v_stride_h;
    p.pool_page = cache->stride_page; p.pool_head = cache->stride_head; p.pool_token = cache->stride_token;
    p.page_shift = pv.page_shift;
    p.n_pages = cache->n_pages;
    p.max_pages = cache->max_pages;
    p.table = pv.table; p.lens = pv.lens; p.n_new = n_new;
    p.flags = pv.flags;
    if (rope) {
        p.turn.steps = reinterpret_cast<const unsigned long long *>(rope->steps);
        p.turn.rot = rope->rot;
        p.turn.magnitude = rope->magnitude;
    }
    const csd_rope_layout_t layout = rope ? rope->layout : CSD_ROPE_HALF;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cache->dtype == CSD_BF16 ? run_append<__nv_bfloat16>(p, layout, st) : run_append<__half>(p, layout, st);
}

size_t csd_cache_meta_bytes(int rows, int max_pages, int n_pages)
{
    return cache_shape_ok(rows, max_pages, n_pages) ? meta_layout(rows, max_pages, n_pages).total : 0;
}

csd_status_t csd_cache_meta_layout(int rows, int max_pages, int n_pages, csd_cache_layout_t *out)
{
    if (!out || !cache_shape_ok(rows, max_pages, n_pages)) return CSD_ERR_INVALID_ARG;
    *out = meta_layout(rows, max_pages, n_pages);
    return CSD_OK;
}

size_t csd_cache_scratch_bytes(int rows, int max_pages, int n_pages)
{
    return cache_shape_ok(rows, max_pages, n_pages) ? scratch_layout(rows, max_pages, n_pages).total : 0;
}

csd_status_t csd_cache_rebuild(const csd_cache_t *cache, void *stream)
{
    const csd_status_t ok = check_cache(cache);
    if (ok != CSD_OK) return ok;
    host::other_work_enqueued();
    const pages::View v = view_of(cache);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemsetAsync(v.flags, 0, kStatusWords * 4, st) != cudaSuccess ||
        cudaMemsetAsync(v.refs, 0, static_cast<size_t>(cache->n_pages) * 4, st) != cudaSuccess) {
        (void)cudaGetLastError();
        return CSD_ERR_CUDA;
    }
    const csd_status_t rc = launch(pages::rebuild_count_kernel, dim3(static_cast<unsigned int>(v.rows)), pages::kRowThreads, 0, st, v);
    if (rc != CSD_OK) return rc;
    return launch(pages::rebuild_bits_kernel, dim3(static_cast<unsigned int>((v.n_pages + pages::kRowThreads - 1) / pages::kRowThreads)), pages::kRowThreads, 0, st, v);
}

csd_status_t csd_cache_extend(const csd_cache_t *cache, int T, const int32_t *n_new, void *stream)
{
    const csd_status_t ok = check_cache(cache);
    if (ok != CSD_OK) return ok;
    if (T < 0) return CSD_ERR_INVALID_ARG;
    host::other_work_enqueued();
    const pages::View v = view_of(cache);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const csd_status_t rc = launch(pages::extend_kernel, dim3(1), pages::kBlock, 0, st, v, n_new, T);
    return rc != CSD_OK ? rc : copy_pages(cache, v, cache->rows, st);
}

static csd_status_t shorten(const csd_cache_t *cache, const int32_t *new_lens, const int32_t *accept_len, void *stream)
{
    const csd_status_t ok = check_cache(cache);
    if (ok != CSD_OK) return ok;
    if (!new_lens && !accept_len) return CSD_ERR_INVALID_ARG;
    host::other_work_enqueued();
    const pages::View v = view_of(cache);
    return launch(pages::truncate_kernel, dim3(static_cast<unsigned int>(v.rows)), pages::kRowThreads, 0, static_cast<cudaStream_t>(stream), v, new_lens, accept_len);
}

csd_status_t csd_cache_truncate(const csd_cache_t *cache, const int32_t *new_lens, void *stream) { return shorten(cache, new_lens, nullptr, stream); }

csd_status_t csd_cache_commit(const csd_cache_t *cache, const int32_t *accept_len, void *stream) { return shorten(cache, nullptr, accept_len, stream); }

csd_status_t csd_cache_fork(const csd_cache_t *cache, const int32_t *parent, void *stream)
{
    const csd_status_t ok = check_cache(cache);
    if (ok != CSD_OK) return ok;
    if (!parent) return CSD_ERR_INVALID_ARG;
    host::other_work_enqueued();
    const pages::View v = view_of(cache);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const csd_status_t rc = launch(pages::fork_stage_kernel, dim3(static_cast<unsigned int>(v.rows)), pages::kRowThreads, 0, st, v, parent);
    return rc != CSD_OK ? rc : launch(pages::fork_commit_kernel, dim3(static_cast<unsigned int>(v.rows)), pages::kRowThreads, 0, st, v, parent);
}

csd_status_t csd_cache_compact(const csd_cache_t *cache, void *stream)
{
    const csd_status_t ok = check_cache(cache);
    if (ok != CSD_OK) return ok;
    host::other_work_enqueued();
    const pages::View v = view_of(cache);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    csd_status_t rc = launch(pages::compact_kernel, dim3(1), pages::kBlock, 0, st, v);
    if (rc == CSD_OK) rc = launch(pages::rename_kernel, dim3(static_cast<unsigned int>(v.rows)), pages::kRowThreads, 0, st, v);
    return rc != CSD_OK ? rc : copy_pages(cache, v, cache->n_pages / 2, st);
}

size_t csd_attention_workspace_bytes(int rows, int T, int q_heads, int heads, int dim)
{
    if (!attention_shape_ok(rows, T, q_heads, heads, dim)) return 0;
    return attention_plan_of(T, q_heads / heads, dim, rows).total;
}

csd_status_t csd_attention(const void *q, int64_t q_stride_b, int64_t q_stride_t, int64_t q_stride_h, int T, int q_heads,
                           const csd_cache_t *cache, int layer, float scale, const int32_t *n_new, void *out, float *lse,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    const csd_status_t ok = check_cache(cache);
    if (ok != CSD_OK) return ok;
    if (!q || !out || !workspace || T <= 0 || q_heads <= 0 || layer < 0 || layer >= cache->layers || !std::isfinite(scale)) return CSD_ERR_INVALID_ARG;
    if (!attention_shape_ok(cache->rows, T, q_heads, cache->heads, cache->dim)) return CSD_ERR_UNSUPPORTED;
    const AttentionPlan plan = attention_plan_of(T, q_heads / cache->heads, cache->dim, cache->rows);
    // positions are counted in 31 bits: tiles of 64 places at least, and what a unit costs beside its tiles
    const double row_positions = (static_cast<double>(cache->max_pages) * cache->page_size + 63) / 64 + plan.run_cost;
    if (row_positions * cache->rows * cache->heads * plan.row_tiles >= 2147483648.0) return CSD_ERR_UNSUPPORTED;
    const size_t need = plan.total;
    if (!aligned16(q) || !aligned16(out) || (q_stride_b | q_stride_t | q_stride_h) % 8 != 0) return CSD_ERR_INVALID_ARG;
    if (workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return CSD_ERR_WORKSPACE;
    host::other_work_enqueued();
    const pages::View pv = view_of(cache);
    attention::Params p;
    std::memset(&p, 0, sizeof p);
    p.q = q;
    p.out = out;
    p.lse = lse;
    p.B = cache->rows; p.T = T; p.Hq = q_heads; p.Hkv = cache->heads; p.D = cache->dim; p.group = q_heads / cache->heads;
    p.qb = q_stride_b; p.qt = q_stride_t; p.qh = q_stride_h;
    p.page_shift = pv.page_shift;
    p.n_pages = cache->n_pages;
    p.max_pages = cache->max_pages;
    p.table = pv.table; p.lens = pv.lens; p.n_new = n_new;
    p.flags = pv.flags;
    p.scale_log2 = scale * kLog2e;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    return cache->dtype == CSD_BF16 ? run_attention_any<__nv_bfloat16>(p, cache, layer, ws, st) : run_attention_any<__half>(p, cache, layer, ws, st);
}

}  // extern "C"
