// Host side of the calls on the paged key-value cache (sttm_cache_append, sttm_cache_attend,
// sttm_cache_evict): argument checks, workspace layout, launches.
#include "../../include/sttm.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <utility>

#include "sttm_cache_append.cuh"
#include "sttm_cache_attend.cuh"
#include "sttm_cache_evict.cuh"
#include "sttm_host.cuh"

namespace {

using namespace sttm;

// Launch with programmatic stream serialization (see launch_after in sttm_api.cu); `cluster` > 1: that many
// blocks to a cluster.
template <typename... KArgs, typename... Args>
sttm_status launch(void (*kernel)(KArgs...), long long grid, unsigned block, size_t smem, unsigned cluster, void* stream,
                   Args&&... args) {
    if (grid < 1 || grid > INT_MAX) return STTM_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(std::forward<Args>(args))...) == cudaSuccess ? STTM_OK : STTM_ERR_CUDA;
}

// raises a kernel's limit on dynamic shared memory once per device
sttm_status allow_smem(const void* kernel, size_t bytes, size_t (&allowed)[kMaxDevices]) {
    const int dev = device_slot();
    if (dev < 0) return STTM_ERR_UNSUPPORTED;
    if (allowed[dev] >= bytes) return STTM_OK;
    STTM_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    allowed[dev] = bytes;
    return STTM_OK;
}

// Slots of a row at most: the kernels count them in 32 bits and step up to sm_count() * 4096 beyond the last
// (148 multiprocessors: 606208).
constexpr int kMaxSlots = INT_MAX - (1 << 20);

bool multiple_of_8(long long v) { return v % 8 == 0; }
// is any of these arrays of 4-byte numbers (or NULL) at an address that is no multiple of 4?
template <typename... P>
bool odd_address(const P*... p) { return (((uintptr_t)p | ...) & 3) != 0; }

// Do rows of `len` numbers, `seq` elements from one sequence to the next and `head` from one of its heads to the next, share any?
// (One axis has to lie inside the other's stride; the stride of an axis of length one says nothing.)
bool rows_overlap(long long seq, long long head, int seqs, int heads, int len) {
    if (seqs == 1 && heads == 1) return false;
    if (seqs == 1 || heads == 1) return (heads == 1 ? seq : head) < len;
    const long long inner = std::min(seq, head), outer = std::max(seq, head), last = (seq < head ? seqs : heads) - 1;
    return inner < len || outer < len || (outer - len) / last < inner;
}

sttm_status check_cache(const sttm_cache* c) {
    if (c == nullptr || c->k == nullptr || c->v == nullptr || c->table == nullptr) return STTM_ERR_ARG;
    if (c->pages < 1 || c->heads < 1 || c->page < 1 || c->seqs < 1 || c->table_width < 1 || c->dim < 1) return STTM_ERR_ARG;
    if (c->dtype != STTM_BF16 && c->dtype != STTM_F16) return STTM_ERR_UNSUPPORTED;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256) return STTM_ERR_UNSUPPORTED;
    if (c->page % 8 != 0 || c->pages > INT_MAX - 1) return STTM_ERR_UNSUPPORTED;
    if ((long long)c->table_width * c->page > INT_MAX || (long long)c->seqs * c->heads > INT_MAX / 64) return STTM_ERR_UNSUPPORTED;
    if (misaligned(c->k, 16) || misaligned(c->v, 16) || odd_address(c->table)) return STTM_ERR_ARG;
    // (the stride of an axis of length one is never used)
    if ((c->pages > 1 && !multiple_of_8(c->page_stride)) || (c->heads > 1 && !multiple_of_8(c->head_stride)) || !multiple_of_8(c->slot_stride))
        return STTM_ERR_ARG;
    if (c->slot_stride < c->dim || (c->heads > 1 && c->head_stride < c->dim) || (c->pages > 1 && c->page_stride < c->dim)) return STTM_ERR_ARG;
    if (c->seqs > 1 && c->table_stride < c->table_width) return STTM_ERR_ARG;
    return STTM_OK;
}

CacheView view_of(const sttm_cache* c) {
    CacheView v;
    v.k = (uint16_t*)c->k;
    v.v = (uint16_t*)c->v;
    v.pages = c->pages;
    v.page_stride = c->pages > 1 ? c->page_stride : 0;
    v.head_stride = c->heads > 1 ? c->head_stride : 0;
    v.slot_stride = c->slot_stride;
    v.table = c->table;
    v.table_stride = c->table_stride;
    v.table_width = c->table_width;
    v.heads = c->heads;
    v.page = c->page;
    v.seqs = c->seqs;
    return v;
}

// a call of `f` with the element type as a value and the channels as a constant
template <typename F>
sttm_status by_type(const sttm_cache* c, F&& f) {
    auto dims = [&](auto tag) -> sttm_status {
        if (c->dim == 64) return f(tag, std::integral_constant<int, 64>());
        if (c->dim == 128) return f(tag, std::integral_constant<int, 128>());
        return f(tag, std::integral_constant<int, 256>());
    };
    return c->dtype == STTM_BF16 ? dims(__nv_bfloat16()) : dims(__half());
}

// Keys (or values) as [page][head][64-channel half][slot][64 channels]: a box of `box` slots and all channels
// lands in shared memory half by half, rows of 128 bytes under the 128-byte swizzle.
sttm_status make_cache_map(const sttm_cache* c, void* base, int box, CUtensorMap* map) {
    const EncodeTiledFn encode = tensor_map_encoder();
    if (encode == nullptr) return STTM_ERR_CUDA;
    const cuuint64_t inner = (cuuint64_t)c->slot_stride * 2;
    const cuuint64_t dims[5] = {64, (cuuint64_t)c->page, (cuuint64_t)(c->dim / 64), (cuuint64_t)c->heads, (cuuint64_t)c->pages};
    const cuuint64_t strides[4] = {inner, 128, c->heads > 1 ? (cuuint64_t)c->head_stride * 2 : inner,
                                   c->pages > 1 ? (cuuint64_t)c->page_stride * 2 : inner};
    const cuuint32_t shape[5] = {64, (cuuint32_t)box, (cuuint32_t)(c->dim / 64), 1, 1}, ones[5] = {1, 1, 1, 1, 1};
    const CUresult r = encode(map, c->dtype == STTM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5,
                              base, dims, strides, shape, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? STTM_OK : STTM_ERR_UNSUPPORTED;      // (a stride beyond what a tensor map holds)
}

// Rows go to clusters (one launch, no parts in memory) up to so many tiles per CTA; beyond, equal shares spread them over
// more SMs.  Clusters / shares in us, 128 channels, seven heads per KV head, more caches in turn than L2 holds:
//   tiles per CTA              4             6             8            12
//   1 row, 16 CTAs         9.8 /  9.7   11.6 / 10.4   12.8 / 11.7   16.2 / 14.1
//   4 rows, 16 CTAs       11.3 / 12.7   12.7 / 13.9   13.9 / 14.0   16.7 / 16.1
//   8 rows, 16 CTAs       13.0 / 14.1   14.9 / 16.3   16.4 / 17.6   20.0 / 20.2
//   16 rows, 8 CTAs       12.6 / 14.2                 15.8 / 17.6   19.5 / 20.2
//   32 rows, 4 CTAs       12.2 / 13.8                 15.3 / 17.2
// The edge lies at 4 tiles for one row, at 8 for four, and beyond 12 from eight rows on; six is between.  Where the rows alone
// occupy half of the GPU's CTAs, a CTA takes a row up to kWholeTiles tiles: 256 rows of 512 slots 18.2 us against 22.5, of 1024 29.5
// against 33.7, of 4096 85.5 against 90.7; with scores 24.4 / 28.3, 41.9 / 42.0, and from there on shares win (1536: 57.4 / 54.9),
// so 16 tiles.  With scores only the latter: a cluster's few threads take longer over the scores than the
// launch that spares them.
constexpr int kClusterTiles = 6, kWholeTiles = 16;

// Clusters of `size` CTAs with an SM each (attention over 256 channels, the selection of an eviction) that the GPU holds at once.
// Fewer than its SMs over `size`, since a cluster lies in one group of SMs whose number it need not divide: 15 of 8 CTAs, 33 of 4,
// 74 of 2 on 148 SMs.  (Two CTAs to an SM leave room: 14 clusters of 16, 33 of 8.)
int resident_clusters(int size) {
    static int cached[kMaxDevices][kAttMaxCluster + 1] = {};
    const int dev = device_slot();
    if (dev < 0) return sm_count() / size;
    int& n = cached[dev][size];
    if (n == 0) {
        const auto kernel = k_cache_attend<__nv_bfloat16, 256, 16>;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)size);
        cfg.blockDim = dim3(kAttThreads);
        cfg.dynamicSmemBytes = attend_stages(256) * (size_t)kAttStage + attend_fixed_bytes<256, 16>();
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = (unsigned)size;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        static size_t allowed[kMaxDevices] = {};
        if (allow_smem((const void*)kernel, cfg.dynamicSmemBytes, allowed) != STTM_OK ||
            cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1)
            n = sm_count() / size;
    }
    return n;
}

struct AttendPlan {
    int cluster;                  // see AttendArgs
    long long tiles;              // upper bound over all rows
    int row_tiles, grid_limit;
    long long join_blocks, join_grid;   // k_cache_join's blocks that join rows, and all
    int chunks;                   // blocks per row that update scores
    size_t rows, stats, partial, logits, total;
};

sttm_status plan_attend(const sttm_cache* c, const sttm_attend_params* p, AttendPlan* pl) {
    sttm_status s = check_cache(c);
    if (s != STTM_OK) return s;
    if (p == nullptr || p->q_heads < 1 || p->q_heads % c->heads != 0 || p->max_len < 1) return STTM_ERR_ARG;
    if ((long long)p->max_len > (long long)c->table_width * c->page) return STTM_ERR_ARG;
    const int group = p->q_heads / c->heads;
    if (group > 64 || p->max_len > kMaxSlots) return STTM_ERR_UNSUPPORTED;
    const long long rows = (long long)c->seqs * c->heads;
    const int tile = attend_tile(c->dim);
    pl->row_tiles = (p->max_len + tile - 1) / tile;
    pl->tiles = rows * pl->row_tiles;
    if (pl->tiles > INT_MAX / 2) return STTM_ERR_UNSUPPORTED;
    pl->grid_limit = sm_count() * (c->dim == 256 ? 1 : 2);
    // The largest cluster that leaves every CTA a tile and, over all rows, an SM.  16 CTAs want 8 SMs of one GPC, or 16
    // where an SM holds one CTA: there 8 have to do, and fewer where the rows' clusters would not be resident at once (16 rows
    // of 1024 slots took 23.0 us in clusters of 8, in two goes; 14.7 in shares).
    const int most = c->dim == 256 ? 8 : kAttMaxCluster;
    int size = 1;
    while (size < most && size < pl->row_tiles && rows * size * 2 <= sm_count()) size *= 2;
    if (c->dim == 256)
        while (size > 1 && rows > resident_clusters(size)) size /= 2;
    const bool many = rows * 2 > pl->grid_limit;
    pl->cluster = pl->row_tiles <= size * (many ? kWholeTiles : kClusterTiles) && (many || p->scores == nullptr) ? size : 0;
    // blocks per row that update scores: one go each while all of them are resident at once
    pl->join_blocks = rows * group;
    pl->chunks = (int)std::min<long long>((p->max_len + kScoreSlots - 1) / kScoreSlots,
                                          std::max<long long>(1, (long long)sm_count() * 8 / rows));
    pl->join_grid = pl->join_blocks + (p->scores ? rows * pl->chunks : 0);
    if (!pl->cluster && pl->join_grid > INT_MAX) return STTM_ERR_UNSUPPORTED;       // (before the first kernel runs)
    const long long parts = pl->cluster ? (pl->cluster == 1 ? rows : 0) : std::min<long long>(pl->grid_limit, pl->tiles) + rows;
    pl->rows = 0;
    pl->stats = align_up((size_t)rows * sizeof(int4));
    pl->partial = pl->stats + align_up((size_t)parts * group * sizeof(float2));
    pl->logits = pl->partial + (pl->cluster ? 0 : align_up((size_t)parts * group * c->dim * 4));
    pl->total = pl->logits + (p->scores ? align_up((size_t)pl->tiles * group * tile * 4) : 0);
    return STTM_OK;
}

template <typename T, int DIM, int ROWS>
sttm_status launch_attend(const AttendArgs& a, const AttendPlan& pl, const CUtensorMap& mk, const CUtensorMap& mv, void* stream) {
    static size_t allowed[kMaxDevices] = {};
    const size_t smem = a.stages * kAttStage + attend_fixed_bytes<DIM, ROWS>();
    sttm_status s = allow_smem((const void*)k_cache_attend<T, DIM, ROWS>, smem, allowed);
    if (s != STTM_OK) return s;
    if (pl.cluster > 8) {
        static bool large[kMaxDevices] = {};
        const int dev = device_slot();
        if (!large[dev]) STTM_CUDA_TRY(cudaFuncSetAttribute(k_cache_attend<T, DIM, ROWS>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        large[dev] = true;
    }
    const long long rows = (long long)a.seqs * a.heads;
    const long long grid = pl.cluster ? rows * pl.cluster : std::min<long long>(pl.grid_limit, pl.tiles);
    return launch(k_cache_attend<T, DIM, ROWS>, grid, kAttThreads, smem, (unsigned)pl.cluster, stream, a, mk, mv);
}

}  // namespace

extern "C" {

sttm_status sttm_cache_append(const sttm_cache* cache, const sttm_append_params* p, void* stream) {
    sttm_status s = check_cache(cache);
    if (s != STTM_OK) return s;
    if (p == nullptr || p->row_offsets == nullptr || p->rows < 0 || p->q_heads < 0) return STTM_ERR_ARG;
    if (p->new_lengths != nullptr && p->new_lengths == p->lengths) return STTM_ERR_ARG;
    if (misaligned(p->row_offsets, 8) || odd_address(p->lengths, p->new_lengths, p->inv_freq, p->device_status, (const int32_t*)p->positions))
        return STTM_ERR_ARG;
    if (p->rot < 0 || p->rot > cache->dim || p->rot % 16 != 0) return STTM_ERR_ARG;
    if (p->rows > 0) {
        if (p->k == nullptr || p->v == nullptr || (p->q_heads > 0 && (p->q == nullptr || p->q_out == nullptr))) return STTM_ERR_ARG;
        if (p->rot > 0 && (p->positions == nullptr || p->inv_freq == nullptr)) return STTM_ERR_ARG;
        if (misaligned(p->k, 16) || misaligned(p->v, 16) || (p->q_heads > 0 && (misaligned(p->q, 16) || misaligned(p->q_out, 16))))
            return STTM_ERR_ARG;
        if (!multiple_of_8(p->k_row) || !multiple_of_8(p->k_head) || !multiple_of_8(p->v_row) || !multiple_of_8(p->v_head))
            return STTM_ERR_ARG;
        if (p->q_heads > 0 && (!multiple_of_8(p->q_row) || !multiple_of_8(p->q_head))) return STTM_ERR_ARG;
        if ((p->q_norm && misaligned(p->q_norm, 16)) || (p->k_norm && misaligned(p->k_norm, 16))) return STTM_ERR_ARG;
    }
    if (p->axes != 1 && p->axes != 3) return STTM_ERR_ARG;
    if (p->axes == 3 && p->rot > 0) {
        if (p->sections[0] < 0 || p->sections[1] < 0 || p->sections[2] < 0) return STTM_ERR_ARG;
        if ((long long)p->sections[0] + p->sections[1] + p->sections[2] != p->rot / 2) return STTM_ERR_ARG;
    }
    AppendArgs a = {};
    a.c = view_of(cache);
    a.q = (const uint16_t*)p->q;
    a.k = (const uint16_t*)p->k;
    a.v = (const uint16_t*)p->v;
    a.q_row = p->q_row; a.q_head = p->q_head;
    a.k_row = p->k_row; a.k_head = p->k_head;
    a.v_row = p->v_row; a.v_head = p->v_head;
    a.q_out = (uint16_t*)p->q_out;
    a.rows = p->rows;
    a.q_heads = p->q_heads;
    a.row_offsets = (const long long*)p->row_offsets;
    a.lengths = p->lengths;
    a.new_lengths = p->new_lengths;
    a.positions = p->positions;
    a.positions_f32 = p->positions_f32;
    a.axis_stride = p->axes == 3 ? p->axis_stride : 0;
    a.sec0 = p->axes == 3 ? p->sections[0] : p->rot / 2;
    a.sec1 = p->axes == 3 ? p->sections[0] + p->sections[1] : p->rot / 2;
    a.inv_freq = p->inv_freq;
    a.rot = p->rot;
    a.q_norm = p->q_norm;
    a.k_norm = p->k_norm;
    a.eps = p->eps;
    a.status = p->device_status;
    // warps per row: one once the rows fill the GPU, else one per step of a row's heads
    const int per_step = 32 / (cache->dim / 16), steps = (p->q_heads + per_step - 1) / per_step + 2 * ((cache->heads + per_step - 1) / per_step);
    const long long wanted = (long long)sm_count() * 32;
    a.parts = (int)std::min<long long>(steps, std::max<long long>(1, wanted / std::max<long long>(1, p->rows)));
    const long long grid = std::max<long long>(1, (p->rows * a.parts + kAppendWarps - 1) / kAppendWarps);
    return by_type(cache, [&](auto tag, auto dim) {
        using T = decltype(tag);
        constexpr int D = decltype(dim)::value;
        return p->interleaved ? launch(k_cache_append<T, D, true>, grid, kAppendWarps * 32, 0, 0, stream, a)
                              : launch(k_cache_append<T, D, false>, grid, kAppendWarps * 32, 0, 0, stream, a);
    });
}

size_t sttm_attend_workspace_bytes(const sttm_cache* cache, const sttm_attend_params* p) {
    AttendPlan pl;
    return plan_attend(cache, p, &pl) == STTM_OK ? pl.total : 0;
}

sttm_status sttm_cache_attend(const sttm_cache* cache, const sttm_attend_params* p, void* ws, size_t ws_bytes, void* stream) {
    AttendPlan pl;
    sttm_status s = plan_attend(cache, p, &pl);
    if (s != STTM_OK) return s;
    if (p->q == nullptr || p->out == nullptr || p->lengths == nullptr || ws == nullptr) return STTM_ERR_ARG;
    if (misaligned(p->q, 16) || misaligned(p->out, 16) || misaligned(ws, 256)) return STTM_ERR_ARG;
    if (odd_address(p->lengths, p->scores, p->lse, p->device_status)) return STTM_ERR_ARG;
    if (p->scores != nullptr && rows_overlap(p->score_seq, p->score_head, cache->seqs, cache->heads, p->max_len)) return STTM_ERR_ARG;
    if (!multiple_of_8(p->q_seq) || !multiple_of_8(p->q_head) || !std::isfinite(p->scale)) return STTM_ERR_ARG;
    if (p->mask != nullptr && cache->seqs > 1 && p->mask_stride < p->max_len) return STTM_ERR_ARG;
    if (ws_bytes < pl.total) return STTM_ERR_WORKSPACE;
    char* w = (char*)ws;
    AttendArgs a = {};
    a.table = cache->table;
    a.table_stride = cache->table_stride;
    a.pages = cache->pages;
    a.heads = cache->heads;
    a.page = cache->page;
    a.seqs = cache->seqs;
    a.group = p->q_heads / cache->heads;
    // slots per copy: the largest power of two that divides a page, at most a tile
    a.tile = attend_tile(cache->dim);
    a.box = std::min(cache->page & -cache->page, a.tile);
    a.max_len = p->max_len;
    a.cluster = pl.cluster;
    a.q = (const uint16_t*)p->q;
    a.q_seq = p->q_seq;
    a.q_head = p->q_head;
    a.lengths = p->lengths;
    a.mask = p->mask;
    a.mask_stride = p->mask_stride;
    a.scale_log2 = (float)((double)p->scale * 1.4426950408889634);
    a.out = (uint16_t*)p->out;
    a.lse = p->lse;
    a.status = p->device_status;
    a.rows = (int4*)(w + pl.rows);
    a.stats = (float2*)(w + pl.stats);
    a.partial = (float*)(w + pl.partial);
    a.logits = p->scores ? (float*)(w + pl.logits) : nullptr;
    a.scores = p->scores;
    a.score_seq = p->score_seq;
    a.score_head = p->score_head;
    a.decay = p->decay;
    CUtensorMap mk, mv;
    if ((s = make_cache_map(cache, cache->k, a.box, &mk)) != STTM_OK) return s;
    if ((s = make_cache_map(cache, cache->v, a.box, &mv)) != STTM_OK) return s;
    return by_type(cache, [&](auto tag, auto dim) {
        using T = decltype(tag);
        constexpr int D = decltype(dim)::value;
        a.stages = attend_stages(D);
        sttm_status r = a.group <= 8 ? launch_attend<T, D, 8>(a, pl, mk, mv, stream) : launch_attend<T, D, 16>(a, pl, mk, mv, stream);
        if (r != STTM_OK || pl.cluster) return r;
        return launch(k_cache_join<T, D>, pl.join_grid, kJoinThreads, 0, 0, stream, a, (int)pl.join_blocks, pl.chunks);
    });
}

sttm_status sttm_cache_evict(const sttm_cache* src, const sttm_cache* dst, const sttm_evict_params* p, void* stream) {
    sttm_status s = check_cache(src);
    if (s != STTM_OK) return s;
    if ((s = check_cache(dst)) != STTM_OK) return s;
    if (p == nullptr || p->lengths == nullptr || p->keep == nullptr || p->scores == nullptr || p->new_lengths == nullptr ||
        p->kept == nullptr || p->new_scores == nullptr)
        return STTM_ERR_ARG;
    if (src->heads != dst->heads || src->dim != dst->dim || src->dtype != dst->dtype || src->seqs != dst->seqs) return STTM_ERR_ARG;
    if (p->max_len < 1 || (long long)p->max_len > (long long)src->table_width * src->page || p->kept_width < 1) return STTM_ERR_ARG;
    if (p->first < 0 || p->last < 0) return STTM_ERR_ARG;
    if (p->max_len > kMaxSlots || p->kept_width > kMaxSlots) return STTM_ERR_UNSUPPORTED;
    if (odd_address(p->lengths, p->keep, p->scores, p->new_lengths, p->kept, p->new_scores, p->device_status)) return STTM_ERR_ARG;
    if (p->new_lengths == p->lengths || p->new_lengths == p->keep || p->new_scores == p->scores) return STTM_ERR_ARG;
    EvictArgs a = {};
    a.src = view_of(src);
    a.dst = view_of(dst);
    a.lengths = p->lengths;
    a.keep = p->keep;
    a.max_len = p->max_len;
    a.first = p->first;
    a.last = p->last;
    a.kept_width = p->kept_width;
    a.scores = p->scores;
    a.score_seq = p->score_seq;
    a.score_head = p->score_head;
    a.new_lengths = p->new_lengths;
    a.kept = p->kept;
    a.new_scores = p->new_scores;
    a.status = p->device_status;
    const long long rows = (long long)src->seqs * src->heads;
    // CTAs per row: as few as hold its keys (more would only meet at more barriers), but more while the rows
    // leave SMs idle and all their clusters are resident at once (16 rows of 55788 slots: 31.3 us in clusters of 8, in two goes, against
    // 20.6 in clusters of 4; 15 rows in clusters of 8 19.2)
    int size = 1;
    while (size < kSelMaxCluster && ((long long)size * kSelThreads * kSelMaxKeys < p->max_len ||
                                     (rows * size * 2 <= sm_count() && rows <= resident_clusters(size * 2) &&
                                      (long long)size * kSelThreads * 3 < p->max_len)))
        size *= 2;
    const long long per_thread = ((long long)p->max_len + (long long)size * kSelThreads - 1) / ((long long)size * kSelThreads);
    auto select = [&](auto kpt) -> sttm_status {
        constexpr int KPT = decltype(kpt)::value;
        static size_t allowed[kMaxDevices] = {};
        const size_t smem = KPT * kSelThreads * 4;
        sttm_status r = allow_smem((const void*)k_cache_select<KPT>, smem, allowed);
        return r != STTM_OK ? r : launch(k_cache_select<KPT>, rows * size, kSelThreads, smem, (unsigned)size, stream, a);
    };
    s = per_thread <= 3 ? select(std::integral_constant<int, 3>()) : per_thread <= 9 ? select(std::integral_constant<int, 9>())
      : per_thread <= 17 ? select(std::integral_constant<int, 17>()) : per_thread <= 25 ? select(std::integral_constant<int, 25>())
      : per_thread <= kSelMaxKeys ? select(std::integral_constant<int, kSelMaxKeys>())
                                  : launch(k_cache_select_long, rows * size, kSelThreads, 0, (unsigned)size, stream, a);
    if (s != STTM_OK) return s;
    return by_type(src, [&](auto, auto dim) {
        constexpr int D = decltype(dim)::value;
        const int per_go = kMoveWords * kMoveThreads / (D / 4);     // slots a block has in flight
        const long long go = (p->kept_width + per_go - 1) / per_go, fill = std::max<long long>(1, (long long)sm_count() * 32 / rows);
        const int chunks = (int)std::min(go, fill);
        return launch(k_cache_move<D>, rows * chunks, kMoveThreads, 0, 0, stream, a, chunks);
    });
}

}  // extern "C"
