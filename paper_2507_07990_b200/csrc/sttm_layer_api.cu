// Host side of a decoder layer's calls (sttm_block_norm, sttm_quantize_rows, sttm_quant_matmul): argument checks, choice of the
// kernel's form, launches.
#include "../../include/sttm.h"

#include <algorithm>
#include <cmath>

#include "sttm_block_norm.cuh"
#include "sttm_cache_host.cuh"
#include "sttm_quant_matmul.cuh"

namespace {

using namespace sttm;

bool known_type(int dtype) { return dtype == STTM_BF16 || dtype == STTM_F16 || dtype == STTM_F32; }

// a call of `f` with the element type as a value
template <typename F>
sttm_status by_element(int dtype, F&& f) {
    return dtype == STTM_BF16 ? f(__nv_bfloat16()) : dtype == STTM_F16 ? f(__half()) : f(0.0f);
}

// Many rows: a warp each out of shared memory, where that holds six or more and there are four or more to each of the rows that a warp has on its way (1 to 4
// slots).  One slot: 55724 rows of 3584 bf16, both norms and a gate, 280 us against 305 in blocks; 15630 of 1157 fp16 with gates of their own 49 against
// 92; but 5278 rows of 3584, 2.4 a warp, 35 against 28.  Four slots (both norms, L2 cold): 56832 rows of 256 bf16, 16 a warp, 37 against 43, 28416 22.5 against
// 26; below the rule the two are even (14208 rows of 512, 4 a warp, 20.5 both; 7104 14.3 both).
// Else a block each: short rows a warp, few rows the fewest threads that hold one with one chunk (of 16 bytes, or of one element where rows do not
// fill whole 16-byte words) each, two of fp32, eight single elements (one row of 3584: 4.1 us on its own, with four chunks a thread 5.9); more rows
// than the GPU takes at once four chunks a thread (5278 rows: 28 us, with one 35).
template <typename T, int VEC, bool QUANTIZE>
sttm_status launch_rows(const NormArgs& a, void* stream) {
    RowsShape shape;
    const int arrays = a.gate_rows != nullptr ? 3 : 2, weights = (a.post_norm != nullptr) + (a.gate != nullptr) + (a.pre_norm != nullptr);
    shape.pitch = (uint32_t)align_up((size_t)a.dim * sizeof(T) + (VEC == 1 ? 32 : 0), 128);
    shape.weights = (uint32_t)align_up((size_t)a.dim * 4, 128);
    const int fit = ((int)kRowsSmem - 1024 - weights * (int)shape.weights) / (int)(arrays * shape.pitch + 8);
    shape.warps = std::max(1, std::min(fit, kRowsWarps));
    shape.slots = std::min(4, fit / shape.warps);
    if (fit >= 6 && a.dim >= 64 && a.rows >= 4ll * shape.warps * shape.slots * sm_count()) {
        static size_t allowed[kMaxDevices] = {};
        const sttm_status s = allow_smem((const void*)k_norm_rows<T, VEC, QUANTIZE>, kRowsSmem, allowed);
        if (s != STTM_OK) return s;
        const size_t smem = (size_t)shape.warps * shape.slots * arrays * shape.pitch + align_up((size_t)shape.warps * shape.slots * 8, 128) + weights * shape.weights;
        const long long grid = std::min<long long>((a.rows + shape.warps - 1) / shape.warps, sm_count());
        return launch(k_norm_rows<T, VEC, QUANTIZE>, grid, shape.warps * 32, smem, 0, stream, a, shape);
    }
    auto go = [&](auto tpr, auto nch) -> sttm_status {
        constexpr int TPR = decltype(tpr)::value, N = decltype(nch)::value, BLOCK = norm_block(TPR), PER = BLOCK / TPR;
        const long long grid = (a.rows + PER - 1) / PER;
        if constexpr (QUANTIZE) return launch(k_quantize_rows<T, VEC, TPR, N>, grid, BLOCK, 0, 0, stream, a);
        else return launch(k_block_norm<T, VEC, TPR, N>, grid, BLOCK, 0, 0, stream, a);
    };
    constexpr int NCH = VEC == 1 ? 8 : VEC == 4 ? 2 : 1;
    const std::integral_constant<int, NCH> nch{};
    const int per_thread = NCH * VEC;
    if constexpr (VEC > 1) {
        const std::integral_constant<int, 32 / VEC> four{};
        if (a.dim <= 1024) return go(std::integral_constant<int, 32>(), four);
        if (a.rows > 2ll * sm_count() && a.dim <= 4096) return go(std::integral_constant<int, 128>(), four);
        if (a.rows > 2ll * sm_count() && a.dim <= 8192) return go(std::integral_constant<int, 256>(), four);
    }
    if (a.dim <= 32 * per_thread) return go(std::integral_constant<int, 32>(), nch);
    if (a.dim <= 128 * per_thread) return go(std::integral_constant<int, 128>(), nch);
    if (a.dim <= 256 * per_thread) return go(std::integral_constant<int, 256>(), nch);
    if (a.dim <= 512 * per_thread) return go(std::integral_constant<int, 512>(), nch);
    if (a.dim <= 1024 * per_thread) return go(std::integral_constant<int, 1024>(), nch);
    // (the inner widths of gated blocks, 18944 or 29568 for instance: 5278 gated bf16 rows 171 and 230 us, beside 139 for 16384; one row 5.8 and 6.6)
    if constexpr (QUANTIZE && VEC > 1)
        if (a.dim > kNormMaxDim) return go(std::integral_constant<int, 1024>(), std::integral_constant<int, 4 * NCH>());
    return go(std::integral_constant<int, 1024>(), std::integral_constant<int, 2 * NCH>());
}

struct MatmulPlan {
    bool swap;                    // weights are the 128-row operand
    int nt, cluster, stages;
    long long a_tiles, b_tiles, grid;
};

// Clusters of `size` CTAs, two to an SM, that the GPU holds at once: fewer than its SMs allow (33 of 8, 71 of 4 on 148 SMs), since a cluster lies in
// one group of SMs.
int matmul_clusters(int size) {
    static int cached[kMaxDevices][9] = {};
    const int dev = device_slot();
    if (dev < 0) return sm_count() * 2 / size;
    int n = cached[dev][size];
    if (n == 0) {                                               // (two threads at once find the same)
        const auto kernel = k_quant_matmul<__nv_bfloat16, 16>;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)size);
        cfg.blockDim = dim3(kMatThreads);
        cfg.dynamicSmemBytes = kMatSmem;
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = (unsigned)size;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        static size_t allowed[kMaxDevices] = {};
        if (allow_smem((const void*)kernel, kMatSmem, allowed) != STTM_OK || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
            (void)cudaGetLastError();                           // (not for the next call on this thread to find)
            n = sm_count() * 2 / size;
        }
        cached[dev][size] = n;
    }
    return n;
}

// Few tokens take 16, 32 or 64 columns beside 128 weights.  More than 64 do so too (several tiles of 64) while two CTAs or more can share a tile's inner axis;
// beyond, the kernel for pairs.  us, products alone, weights out of HBM, few tokens' kernel / pairs':
//   inner x outer     tokens 64      128       256       300       400
//   3584 x 4608      8.7 / 17.5  11.1 / 18  13.3 / 18  16.4 / 17.5 17.5 / 17.2
//   14336 x 3584    13.9 / 41    18.7 / 41  27.5 / 41  29.0 / 41   46.2 / 40
//   3584 x 28672    27.8 / 30    30.9 / 32
//   1024 x 1024      5.0 / 8.0    5.0 / 8.7  5.6 / 8.7  5.8 / 8.8   6.1 / 8.8
// A cluster shares the inner axis as widely as all clusters are resident at once (36 tiles in clusters of 8, of which 33 fit: 10.6 us, of 4: 6.7) and leaves every
// CTA two steps.
MatmulPlan plan_matmul(const sttm_matmul_params* p) {
    MatmulPlan pl;
    const int blocks = (p->inner + kMatK - 1) / kMatK, sms = sm_count();
    pl.nt = p->rows <= 16 ? 16 : p->rows <= 32 ? 32 : 64;
    pl.a_tiles = ((long long)p->outer + 127) / 128;
    pl.b_tiles = (p->rows + pl.nt - 1) / pl.nt;
    long long tiles = pl.a_tiles * pl.b_tiles;
    pl.swap = p->rows <= 64 || tiles <= sms;
    if (!pl.swap) {
        pl.a_tiles = (p->rows + 255) / 256;
        pl.b_tiles = ((long long)p->outer + 255) / 256;
        tiles = pl.a_tiles * pl.b_tiles;
        pl.nt = 256;
        pl.cluster = 2;
        pl.stages = kPairStages;
        pl.grid = 2 * std::min<long long>(tiles, sms / 2);
        return pl;
    }
    pl.stages = std::min(kMatMaxStages, (int)((kMatSmem - matmul_fixed_bytes()) / matmul_slot(pl.nt)));
    pl.cluster = 1;
    while (pl.cluster < 8 && blocks >= 4 * pl.cluster && tiles <= matmul_clusters(2 * pl.cluster)) pl.cluster *= 2;
    pl.grid = pl.cluster > 1 ? tiles * pl.cluster : std::min<long long>(tiles, 2ll * sms);
    return pl;
}

sttm_status make_rows_map(const void* base, long long rows, int inner, long long row_bytes, int box_rows, CUtensorMap* map) {
    const EncodeTiledFn encode = tensor_map_encoder();
    if (encode == nullptr) return STTM_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)row_bytes};
    const cuuint32_t box[2] = {kMatK, (cuuint32_t)box_rows}, ones[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? STTM_OK : STTM_ERR_UNSUPPORTED;
}

template <typename T, int NT>
sttm_status launch_matmul(const MatmulArgs& a, const MatmulPlan& pl, const CUtensorMap& ma, const CUtensorMap& mb, void* stream) {
    static size_t allowed[kMaxDevices] = {};
    const size_t smem = (size_t)pl.stages * matmul_slot(NT) + matmul_fixed_bytes();
    const sttm_status s = allow_smem((const void*)k_quant_matmul<T, NT>, smem, allowed);
    return s != STTM_OK ? s : launch(k_quant_matmul<T, NT>, pl.grid, kMatThreads, smem, pl.cluster > 1 ? pl.cluster : 0, stream, a, ma, mb);
}

// `rows` rows of `width` bytes, `row` bytes apart
struct RowsAt {
    const void* at;
    long long row, width;
};
Span span_of(const RowsAt& a, long long rows) { return {a.at, (rows - 1) * a.row + a.width}; }
bool share_memory(const RowsAt& a, const RowsAt& b, long long rows) { return overlap(span_of(a, rows), span_of(b, rows)); }
bool in_place(const RowsAt& a, const RowsAt& b, long long rows) { return a.at == b.at && a.width == b.width && (a.row == b.row || rows == 1); }

}  // namespace

extern "C" {

sttm_status sttm_block_norm(const sttm_norm_params* p, void* stream) {
    if (p == nullptr || p->rows < 0 || p->dim < 1 || !known_type(p->dtype)) return STTM_ERR_ARG;
    if (p->dim > kNormMaxDim || p->rows > INT_MAX) return STTM_ERR_UNSUPPORTED;
    if (!std::isfinite(p->residual_scale) || !(p->eps >= 0.0f)) return STTM_ERR_ARG;
    if (p->rows == 0) return STTM_OK;
    if (p->x == nullptr || (p->sum == nullptr && p->out == nullptr && p->q == nullptr) || (p->q == nullptr) != (p->q_scale == nullptr)) return STTM_ERR_ARG;
    const long long e = p->dtype == STTM_F32 ? 4 : 2, width = p->dim * e;
    const void* const in[3] = {p->x, p->residual, p->gate_rows};
    const long long in_row[3] = {p->x_row, p->residual_row, p->gate_row};
    const void* const out[3] = {p->sum, p->out, p->q};
    const long long out_row[3] = {p->sum_row, p->out_row, p->q_row};
    bool wide = p->dim % (16 / e) == 0;
    for (int i = 0; i < 3; i++) {
        if (in[i] != nullptr && ((p->rows > 1 && (in_row[i] < p->dim || in_row[i] > LLONG_MAX / 4 / p->rows)) || misaligned(in[i], e))) return STTM_ERR_ARG;
        if (out[i] != nullptr && ((p->rows > 1 && (out_row[i] < p->dim || out_row[i] > LLONG_MAX / 4 / p->rows)) || (i < 2 && misaligned(out[i], e)))) return STTM_ERR_ARG;
        wide = wide && (in[i] == nullptr || (!misaligned(in[i], 16) && (p->rows == 1 || in_row[i] * e % 16 == 0)));
        wide = wide && (out[i] == nullptr || i == 2 || (!misaligned(out[i], 16) && (p->rows == 1 || out_row[i] * e % 16 == 0)));
    }
    if (odd_address(p->post_norm, p->gate, p->pre_norm, p->q_scale, p->device_status)) return STTM_ERR_ARG;
    const uintptr_t weights = (uintptr_t)p->post_norm | (uintptr_t)p->gate | (uintptr_t)p->pre_norm;
    wide = wide && weights % 16 == 0 && (p->q == nullptr || (!misaligned(p->q, 8) && (p->rows == 1 || p->q_row % 8 == 0)));
    const Span post = {p->post_norm, p->dim * 4ll}, gate = {p->gate, p->dim * 4ll}, pre = {p->pre_norm, p->dim * 4ll};
    const Span scales = {p->q_scale, p->rows * 4}, status = {p->device_status, 4};
    if (overlaps_any(scales, post, gate, pre, status)) return STTM_ERR_ARG;
    for (int o = 0; o < 3; o++) {
        const RowsAt to = o < 2 ? RowsAt{out[o], out_row[o] * e, width} : RowsAt{p->q, p->q_row, p->dim};
        if (overlaps_any(span_of(to, p->rows), post, gate, pre, scales, status)) return STTM_ERR_ARG;
        for (int i = 0; i < 3; i++) {
            const RowsAt from = {in[i], in_row[i] * e, width};
            if ((share_memory(to, from, p->rows) && !in_place(to, from, p->rows)) || overlap(scales, span_of(from, p->rows))) return STTM_ERR_ARG;
        }
        for (int u = 0; u < o; u++)
            if (share_memory(to, {out[u], out_row[u] * e, width}, p->rows)) return STTM_ERR_ARG;
    }
    NormArgs a = {};
    a.x = p->x; a.residual = p->residual; a.gate_rows = p->gate_rows;
    a.x_row = p->x_row; a.residual_row = p->residual_row; a.gate_row = p->gate_row;
    a.post_norm = p->post_norm; a.gate = p->gate; a.pre_norm = p->pre_norm;
    a.residual_scale = p->residual_scale;
    a.eps = p->eps;
    a.sum = p->sum; a.out = p->out;
    a.sum_row = p->sum_row; a.out_row = p->out_row;
    a.q = p->q; a.q_row = p->q_row; a.q_scale = p->q_scale;
    a.status = p->device_status;
    a.rows = p->rows;
    a.dim = p->dim;
    return by_element(p->dtype, [&](auto tag) {
        using T = decltype(tag);
        return wide ? launch_rows<T, 16 / sizeof(T), false>(a, stream) : launch_rows<T, 1, false>(a, stream);
    });
}

sttm_status sttm_quantize_rows(const sttm_quantize_params* p, void* stream) {
    if (p == nullptr || p->rows < 0 || p->dim < 1 || !known_type(p->dtype)) return STTM_ERR_ARG;
    const long long e = p->dtype == STTM_F32 ? 4 : 2, in = p->gated ? 2ll * p->dim : p->dim;
    if (p->dim > kQuantizeMaxDim || (p->dim > kNormMaxDim && p->dim % (16 / e) != 0) || p->rows > INT_MAX) return STTM_ERR_UNSUPPORTED;
    if (p->rows == 0) return STTM_OK;
    if (p->x == nullptr || p->q == nullptr || p->scale == nullptr || odd_address(p->scale, p->device_status)) return STTM_ERR_ARG;
    if (misaligned(p->x, e) || (p->rows > 1 && (p->x_row < in || p->q_row < p->dim || p->x_row > LLONG_MAX / 4 / p->rows || p->q_row > LLONG_MAX / 4 / p->rows)))
        return STTM_ERR_ARG;
    const Span x = span_of({p->x, p->x_row * e, in * e}, p->rows), q = span_of({p->q, p->q_row, p->dim}, p->rows), scales = {p->scale, p->rows * 4};
    if (overlaps_any(q, x, scales, Span{p->device_status, 4}) || overlaps_any(scales, x, Span{p->device_status, 4})) return STTM_ERR_ARG;
    const bool wide = p->dim % (16 / e) == 0 && !misaligned(p->x, 16) && !misaligned(p->q, 8) && (p->rows == 1 || (p->x_row * e % 16 == 0 && p->q_row % 8 == 0));
    if (p->dim > kNormMaxDim && !wide) return STTM_ERR_UNSUPPORTED;
    NormArgs a = {};
    a.x = p->x; a.x_row = p->x_row;
    a.q = p->q; a.q_row = p->q_row; a.q_scale = p->scale;
    a.status = p->device_status;
    a.rows = p->rows;
    a.dim = p->dim;
    a.gated = p->gated != 0;
    return by_element(p->dtype, [&](auto tag) {
        using T = decltype(tag);
        return wide ? launch_rows<T, 16 / sizeof(T), true>(a, stream) : launch_rows<T, 1, true>(a, stream);
    });
}

sttm_status sttm_quant_matmul(const sttm_matmul_params* p, void* stream) {
    if (p == nullptr || p->rows < 0 || p->inner < 1 || p->outer < 1 || !known_type(p->out_dtype)) return STTM_ERR_ARG;
    if (p->inner > 131056 || p->rows > INT_MAX) return STTM_ERR_UNSUPPORTED;
    if (p->w == nullptr || p->w_scale == nullptr || misaligned(p->w, 16) || p->w_row % 16 != 0 || p->w_row < p->inner || p->w_row > LLONG_MAX / 4 / p->outer)
        return STTM_ERR_ARG;
    if (odd_address(p->x_scale, p->w_scale, p->bias, p->device_status)) return STTM_ERR_ARG;
    if (p->rows == 0) return STTM_OK;
    if (p->x == nullptr || p->x_scale == nullptr || p->out == nullptr || misaligned(p->x, 16) || p->x_row % 16 != 0 || p->x_row < p->inner ||
        p->x_row > LLONG_MAX / 4 / p->rows)
        return STTM_ERR_ARG;
    const int e = p->out_dtype == STTM_F32 ? 4 : 2;
    if (misaligned(p->out, e) || (p->rows > 1 && (p->out_row < p->outer || p->out_row > LLONG_MAX / 4 / p->rows))) return STTM_ERR_ARG;
    if (overlaps_any(span_of({p->out, p->out_row * e, (long long)p->outer * e}, p->rows), span_of({p->x, p->x_row, p->inner}, p->rows),
                     span_of({p->w, p->w_row, p->inner}, p->outer), Span{p->x_scale, p->rows * 4}, Span{p->w_scale, p->outer * 4ll},
                     Span{p->bias, p->outer * 4ll}, Span{p->device_status, 4}))
        return STTM_ERR_ARG;
    const MatmulPlan pl = plan_matmul(p);
    if (pl.a_tiles * pl.b_tiles > INT_MAX / 8) return STTM_ERR_UNSUPPORTED;
    MatmulArgs a = {};
    a.x_scale = p->x_scale; a.w_scale = p->w_scale; a.bias = p->bias;
    a.out = p->out;
    a.out_row = p->out_row;
    a.rows = p->rows;
    a.outer = p->outer;
    a.blocks = (p->inner + kMatK - 1) / kMatK;
    a.a_tiles = (int)pl.a_tiles; a.b_tiles = (int)pl.b_tiles;
    a.cluster = pl.cluster;
    a.stages = (uint32_t)pl.stages;
    a.status = p->device_status;
    a.wide = !misaligned(p->out, 16) && (p->rows == 1 || p->out_row * e % 16 == 0);
    CUtensorMap mx, mw;
    sttm_status s;
    if ((s = make_rows_map(p->x, p->rows, p->inner, p->x_row, pl.swap ? pl.nt : 128, &mx)) != STTM_OK) return s;
    if ((s = make_rows_map(p->w, p->outer, p->inner, p->w_row, 128, &mw)) != STTM_OK) return s;
    return by_element(p->out_dtype, [&](auto tag) -> sttm_status {
        using T = decltype(tag);
        if (!pl.swap) {
            static size_t allowed[kMaxDevices] = {};
            const sttm_status r = allow_smem((const void*)k_quant_matmul_pair<T>, kPairSmem, allowed);
            return r != STTM_OK ? r : launch(k_quant_matmul_pair<T>, pl.grid, kMatThreads, kPairSmem, 2, stream, a, mx, mw);
        }
        switch (pl.nt) {
            case 16: return launch_matmul<T, 16>(a, pl, mw, mx, stream);
            case 32: return launch_matmul<T, 32>(a, pl, mw, mx, stream);
            default: return launch_matmul<T, 64>(a, pl, mw, mx, stream);
        }
    });
}

}  // extern "C"
