// Host side of sttm_prefix_attend: argument checks, workspace layout, launches.
#include "../../include/sttm.h"

#include <algorithm>
#include <cmath>

#include "sttm_cache_host.cuh"
#include "sttm_prefix.cuh"

namespace {

using namespace sttm;

struct PrefixPlan {
    long long grid, join_grid;
    int join_rows;                              // per block
    size_t entries, of, stats, partial, total;  // byte offsets in the workspace, and its size
};

sttm_status plan_prefix(const sttm_cache* prefix, const sttm_cache* own, const sttm_prefix_params* p, PrefixPlan* pl) {
    sttm_status s = check_cache(prefix);
    if (s != STTM_OK) return s;
    if (own != nullptr && (s = check_cache(own)) != STTM_OK) return s;
    if (p == nullptr || p->rows < 0 || p->seqs < 1 || p->q_heads < 1 || p->q_heads % prefix->heads != 0) return STTM_ERR_ARG;
    if (own != nullptr && (own->heads != prefix->heads || own->dim != prefix->dim || own->dtype != prefix->dtype || own->seqs != p->seqs))
        return STTM_ERR_ARG;
    if (p->seq_offsets == nullptr && prefix->seqs != 1) return STTM_ERR_ARG;
    if (p->max_prefix < 1 || (long long)p->max_prefix > (long long)prefix->table_width * prefix->page) return STTM_ERR_ARG;
    if (own != nullptr && (p->max_own < 1 || (long long)p->max_own > (long long)own->table_width * own->page)) return STTM_ERR_ARG;
    const int group = p->q_heads / prefix->heads;
    if (group > 64 || p->max_prefix > kMaxSlots || (own != nullptr && p->max_own > kMaxSlots)) return STTM_ERR_UNSUPPORTED;
    if (p->rows > INT_MAX - 256 || p->seqs > INT_MAX / 2 || prefix->seqs > INT_MAX / 2) return STTM_ERR_UNSUPPORTED;
    pl->grid = std::min(sm_count(), kJoinParts / 2);
    const long long heads = p->rows * p->q_heads;
    // Few rows have many pieces each, and leave SMs idle unless several blocks share them; many rows keep every SM busy with 32
    // rows to a block, which reads each piece's statistics once.  Measured, 8 rows against 32: 56 rows x heads 14.9 us against
    // 17.5, 448 37.7 against 52.1; 4900 52.0 against 36.7, 6144 128 against 112, 21364 709 against 637.
    pl->join_rows = heads <= pl->grid * 32 ? 8 : 32;
    pl->join_grid = (p->rows * group + pl->join_rows - 1) / pl->join_rows * prefix->heads * prefix_join_split(prefix->dim, pl->join_rows);
    if (heads > INT_MAX) return STTM_ERR_UNSUPPORTED;
    // every row once per kind of entry, and every CTA's pieces in a stretch of their own
    const long long rows = pl->grid * 256 + heads * (own != nullptr ? 2 : 1);
    pl->entries = 256;
    pl->of = pl->entries + align_up(((size_t)prefix->seqs + (own != nullptr ? own->seqs : 0)) * sizeof(PrefixEntry));
    pl->stats = pl->of + 2 * align_up((size_t)p->rows * 4);
    pl->partial = pl->stats + align_up((size_t)rows * sizeof(float2));
    pl->total = pl->partial + align_up((size_t)rows * prefix->dim * 4);
    return STTM_OK;
}

// Keys (or values) as [page][head][64-channel part][slot][64 channels], a copy taking `box` slots of one part: rows of 128
// bytes under the 128-byte swizzle.
sttm_status make_part_map(const sttm_cache* c, void* base, int box, CUtensorMap* map) {
    const EncodeTiledFn encode = tensor_map_encoder();
    if (encode == nullptr) return STTM_ERR_CUDA;
    const cuuint64_t inner = (cuuint64_t)c->slot_stride * 2;
    const cuuint64_t dims[5] = {64, (cuuint64_t)c->page, (cuuint64_t)(c->dim / 64), (cuuint64_t)c->heads, (cuuint64_t)c->pages};
    const cuuint64_t strides[4] = {inner, 128, c->heads > 1 ? (cuuint64_t)c->head_stride * 2 : inner,
                                   c->pages > 1 ? (cuuint64_t)c->page_stride * 2 : inner};
    const cuuint32_t shape[5] = {64, (cuuint32_t)box, 1, 1, 1}, ones[5] = {1, 1, 1, 1, 1};
    const CUresult r = encode(map, c->dtype == STTM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5,
                              base, dims, strides, shape, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? STTM_OK : STTM_ERR_UNSUPPORTED;
}

// Queries as [row][64-channel part][head][64 channels], a copy taking one part of `tokens` rows' heads of one KV head.
sttm_status make_query_map(const sttm_cache* c, const sttm_prefix_params* p, int group, int tokens, CUtensorMap* map) {
    const EncodeTiledFn encode = tensor_map_encoder();
    if (encode == nullptr) return STTM_ERR_CUDA;
    const cuuint64_t dims[4] = {64, (cuuint64_t)p->q_heads, (cuuint64_t)(c->dim / 64), (cuuint64_t)p->rows};
    const cuuint64_t head = p->q_heads > 1 ? (cuuint64_t)p->q_head * 2 : 128;
    const cuuint64_t strides[3] = {head, 128, p->rows > 1 ? (cuuint64_t)p->q_row * 2 : head};
    const cuuint32_t box[4] = {64, (cuuint32_t)group, 1, (cuuint32_t)tokens}, ones[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, c->dtype == STTM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                              const_cast<void*>(p->q), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? STTM_OK : STTM_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

size_t sttm_prefix_workspace_bytes(const sttm_cache* prefix, const sttm_cache* own, const sttm_prefix_params* p) {
    PrefixPlan pl;
    return plan_prefix(prefix, own, p, &pl) == STTM_OK ? pl.total : 0;
}

sttm_status sttm_prefix_attend(const sttm_cache* prefix, const sttm_cache* own, const sttm_prefix_params* p, void* ws, size_t ws_bytes,
                               void* stream) {
    PrefixPlan pl;
    sttm_status s = plan_prefix(prefix, own, p, &pl);
    if (s != STTM_OK) return s;
    if (p->row_offsets == nullptr || p->prefix_lengths == nullptr || (own != nullptr && p->lengths == nullptr) || ws == nullptr) return STTM_ERR_ARG;
    if (misaligned(p->row_offsets, 8) || odd_address(p->seq_offsets, p->prefix_lengths, p->lengths, p->lse, p->device_status) || misaligned(ws, 256))
        return STTM_ERR_ARG;
    if (!std::isfinite(p->scale) || !(p->scale > 0.0f)) return STTM_ERR_ARG;
    if (p->rows > 0) {
        if (p->q == nullptr || p->out == nullptr || misaligned(p->q, 16) || misaligned(p->out, 16)) return STTM_ERR_ARG;
        if ((p->rows > 1 && (!multiple_of_8(p->q_row) || p->q_row < prefix->dim || p->q_row > LLONG_MAX / 8 / p->rows)) ||
            (p->q_heads > 1 && (!multiple_of_8(p->q_head) || p->q_head < prefix->dim || p->q_head > LLONG_MAX / 8 / p->q_heads)))
            return STTM_ERR_ARG;
    }
    if (ws_bytes < pl.total) return STTM_ERR_WORKSPACE;
    if (p->rows == 0) return STTM_OK;
    // (out may lie where q does: the first kernel has read it by then)
    const long long heads = p->rows * p->q_heads;
    const Span out = {p->out, heads * prefix->dim * 2}, lse = {p->lse, heads * 4}, space = {ws, (long long)pl.total}, status = {p->device_status, 4};
    const Span q = {p->q, ((p->rows > 1 ? (p->rows - 1) * p->q_row : 0) + (p->q_heads > 1 ? (p->q_heads - 1) * p->q_head : 0) + prefix->dim) * 2};
    const Span offsets = {p->row_offsets, (p->seqs + 1ll) * 8}, seq_offsets = {p->seq_offsets, (prefix->seqs + 1ll) * 4};
    const Span shared = {p->prefix_lengths, prefix->seqs * 4ll}, own_slots = {own != nullptr ? p->lengths : nullptr, p->seqs * 4ll};
    if (overlaps_any(out, lse, offsets, seq_offsets, shared, own_slots, status) || overlaps_any(lse, offsets, seq_offsets, shared, own_slots, status) ||
        overlaps_any(space, out, lse, q, offsets, seq_offsets, shared, own_slots, status))
        return STTM_ERR_ARG;
    char* w = (char*)ws;
    PrefixArgs a = {};
    a.prefix = view_of(prefix);
    a.own = own != nullptr ? view_of(own) : CacheView{};
    a.rows = p->rows;
    a.q_heads = p->q_heads;
    a.group = p->q_heads / prefix->heads;
    a.block_tokens = 128 / a.group;
    a.seqs = p->seqs;
    a.row_offsets = (const long long*)p->row_offsets;
    a.seq_offsets = p->seq_offsets;
    a.prefix_lengths = p->prefix_lengths;
    a.lengths = p->lengths;
    a.max_prefix = p->max_prefix;
    a.max_own = p->max_own;
    a.scale_log2 = (float)((double)p->scale * 1.4426950408889634);
    a.out = (uint16_t*)p->out;
    a.lse = p->lse;
    a.status = p->device_status;
    a.head = (PrefixHead*)w;
    a.entries = (PrefixEntry*)(w + pl.entries);
    a.prefix_of = (int32_t*)(w + pl.of);
    a.own_of = (int32_t*)(w + pl.of + align_up((size_t)p->rows * 4));
    a.stats = (float2*)(w + pl.stats);
    a.partial = (float*)(w + pl.partial);
    return by_type(prefix, [&](auto tag, auto dim) -> sttm_status {
        using T = decltype(tag);
        constexpr int D = decltype(dim)::value;
        PrefixMaps maps;
        sttm_status r = make_query_map(prefix, p, a.group, a.block_tokens, &maps.q);
        for (int i = 0; i < 2 && r == STTM_OK; i++) {
            const sttm_cache* c = i && own != nullptr ? own : prefix;
            a.page_box[i] = std::min(c->page & -c->page, PrefixShape<D>::SLOTS);
            if ((r = make_part_map(c, c->k, a.page_box[i], &maps.k[i])) == STTM_OK) r = make_part_map(c, c->v, a.page_box[i], &maps.v[i]);
        }
        if (r != STTM_OK) return r;
        auto attend = [&](auto fine) -> sttm_status {
            constexpr bool FINE = decltype(fine)::value;
            static size_t allowed[kMaxDevices] = {};
            const sttm_status f = allow_smem((const void*)k_prefix_attend<T, D, FINE>, PrefixShape<D>::SMEM, allowed);
            return f != STTM_OK ? f : launch(k_prefix_attend<T, D, FINE>, pl.grid, PrefixShape<D>::THREADS, PrefixShape<D>::SMEM, 0, stream, a, maps);
        };
        if ((r = p->fine ? attend(std::true_type()) : attend(std::false_type())) != STTM_OK) return r;
        return pl.join_rows == 8 ? launch(k_prefix_join<T, D, 8>, pl.join_grid, kPrefixJoinThreads, 0, 0, stream, a)
                                 : launch(k_prefix_join<T, D, 32>, pl.join_grid, kPrefixJoinThreads, 0, 0, stream, a);
    });
}

}  // extern "C"
