// Attention of new tokens of several sequences over a prefix that they share and over their own slots (sttm_prefix_attend).
//
// With G query heads per KV head, the new tokens of all sequences of a prefix are rows (token, query head of the group) of one
// matrix per KV head, and the prefix is read once for all of them:
//     S = Q K^T,  P = exp2(c S - c m),  O = P V,  l = row sums of P,          c = scale * log2(e)
// on the tensor cores (tcgen05): 128 rows and a tile of kv slots at a time, S and O in tensor memory.  A thread owns a row: it
// takes the row's logits out of tensor memory, forms the weights and puts them back as 16-bit operand of the second product.  The
// reference m of the exponentials follows the row's maximum only when that has risen by more than 2^8, so O is
// rarely rescaled; weights of up to 2^8 lose nothing in 32-bit sums.  Weights enter the product in the cache's type, rounded once (half a
// step of it, as the output is: errors against 64 bits are 1.4 times those of the output's rounding alone); their sum l is taken before that
// rounding, in 32 bits.  With FINE they enter as the rounded weight and what it leaves, two numbers that hold 16 bits of it (22 in fp16) as in
// sttm_cache_attend, in the two halves of the place that the logits leave, and two products add up: 16 questions of 53 to 42 tokens on 55724 slots
// 797 us instead of 608 (with the join), one answer token each 40.1 instead of 37.2.
//
// Two row blocks of 128 are in work at a time (of one block, alternate tiles), so that the products of one run beside the
// exponentials of the other: four warps per block, three that copy (queries, then key and value tiles through a ring) and one
// that issues the products.  256-channel heads fill tensor memory with one O: there one block's tiles alternate between two
// places for S.
//
// Work is cut into equal shares of steps over all CTAs whatever the lengths are (which the host does not know): entries are the prefixes
// and then the sequences' own slots; an entry has an item per KV head and block of rows, an item a step per tile of slots and
// kPieceSteps for what it costs besides (queries in, O out).  What a CTA has of an item is a piece: O, l and m of its rows go to
// memory, and k_prefix_join puts a row's pieces together.  One of the copy warps works the pieces out for the others.
//
// Measured (bf16, 28 / 4 heads of 128): 16 questions of 53 to 42 tokens on 55724 slots 0.53 ms at full clocks, 0.61 to 0.64 at the power limit; the first
// kernel alone 516 to 537 us (1140 to 1180 TFLOP/s, the tensor cores busy 69 % of the time, the special-function units 66 %); one answer token
// each 37 us, 3.1 TB/s (tiles at HBM's rate, then 7 us of start and end and 7 of the join).
#pragma once

#include <climits>

#include "sttm_cache.cuh"

namespace sttm {

struct PrefixArgs {
    CacheView prefix, own;        // own.seqs = 0: no own slots
    int page_box[2];              // slots per tensor copy (prefix, own)
    long long rows;
    int q_heads, group;
    int block_tokens;             // tokens in 128 rows: 128 / group
    int seqs;
    const long long* row_offsets;
    const int32_t* seq_offsets;   // or null: one prefix
    const int32_t *prefix_lengths, *lengths;
    int max_prefix, max_own;
    float scale_log2;
    uint16_t* out;
    float* lse;
    int32_t* status;
    struct PrefixHead* head;      // workspace
    struct PrefixEntry* entries;
    int32_t *own_of, *prefix_of;  // [rows] a token's entries
    float2* stats;                // per stored row: m (times c, in powers of two) and l
    float* partial;               // O of the stored rows: per block of rows [dim / 4][rows][4]
};

struct PrefixHead {
    long long total, share;       // steps (-1: bad offsets), steps per CTA
};
struct PrefixEntry {
    long long step0, row0;        // steps and stored rows before it
    long long first;              // its first token
    int tokens, len, units;       // units: steps per item
    int blocks;                   // row blocks per KV head (pairs of 128 rows, or one block whose tiles alternate)
};

constexpr int kPieces = 4;                                      // worked out ahead

template <int DIM>
struct PrefixShape {
    static constexpr int SLOTS = DIM == 256 ? 64 : 128;         // per tile
    static constexpr int SETS = DIM == 256 ? 1 : 2;             // row blocks in work
    static constexpr int HALVES = DIM / 64;                     // 64-channel parts of 128 bytes per row
    static constexpr int TILE = SLOTS * DIM * 2, QBLOCK = 128 * DIM * 2;
    static constexpr int RING = DIM == 64 ? 10 : 5;
    static constexpr int THREADS = SETS * 128 + 128;            // softmax warps, one that issues the products, three that copy
    static constexpr uint32_t O_COL = 256;                      // S at columns 0 and 128, O from here on
    static constexpr int BARS = 2 + 2 * RING + 8 + 2 * kPieces;
    static constexpr size_t SMEM = (size_t)SETS * QBLOCK + (size_t)RING * TILE + BARS * 8 + 16 + 64 * 8 + 128 * 8 + 1024;
    static constexpr int STORE = SETS * 128;                    // stored rows of a piece at most
};

// weights of fp16 caches are taken 2^4 larger, to use more of that type's range
template <typename T>
constexpr float kWeightBias = 0.0f;
template <>
constexpr float kWeightBias<__half> = 4.0f;

constexpr float kLazyRise = 8.0f;                               // powers of two
constexpr int kPieceSteps = 3;
constexpr int kCopyWarps = 3;

// ---- entries ----

template <int DIM>
__device__ __forceinline__ PrefixEntry prefix_entry(const PrefixArgs& a, int e, int32_t& bits) {
    using Shape = PrefixShape<DIM>;
    PrefixEntry r;
    const int P = a.prefix.seqs;
    long long lo, hi;
    int len, most;
    if (e < P) {
        int s0 = 0, s1 = a.seqs;
        if (a.seq_offsets != nullptr) {
            s0 = a.seq_offsets[e];
            s1 = a.seq_offsets[e + 1];
            if (s0 < 0 || s1 < s0 || s1 > a.seqs) {
                bits |= kStatusArg;
                s0 = s1 = 0;
            }
        }
        lo = a.row_offsets[s0];
        hi = a.row_offsets[s1];
        len = a.prefix_lengths[e];
        most = a.max_prefix;
    } else {
        lo = a.row_offsets[e - P];
        hi = a.row_offsets[e - P + 1];
        len = a.lengths[e - P];
        most = a.max_own;
    }
    if (lo < 0 || hi < lo) {
        bits |= kStatusArg;
        lo = hi = 0;
    }
    if (hi > a.rows) {
        bits |= kStatusCapacity;
        hi = a.rows;
        lo = min(lo, hi);
    }
    if (len > most) {
        bits |= kStatusCapacity;
        len = most;
    }
    r.first = lo;
    r.tokens = (int)(hi - lo);
    r.len = max(len, 0);
    r.units = r.len > 0 ? (r.len + Shape::SLOTS - 1) / Shape::SLOTS + kPieceSteps : 0;
    const int per = r.tokens <= a.block_tokens ? a.block_tokens : Shape::SETS * a.block_tokens;
    r.blocks = (r.tokens + per - 1) / per;
    r.step0 = r.row0 = 0;
    return r;
}
// two sets take alternate tiles of one block of rows
template <int DIM>
__device__ __forceinline__ bool alternates(const PrefixArgs& a, const PrefixEntry& e) { return PrefixShape<DIM>::SETS == 1 || e.tokens <= a.block_tokens; }
__device__ __forceinline__ long long steps_of(const PrefixArgs& a, const PrefixEntry& e) { return (long long)a.prefix.heads * e.blocks * e.units; }
__device__ __forceinline__ long long rows_of(const PrefixArgs& a, const PrefixEntry& e) { return e.units ? (long long)a.q_heads * e.tokens : 0; }

// (a division in 64 bits takes some hundred instructions)
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

__device__ __forceinline__ long long warp_scan(long long v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const long long u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// What a CTA has of an item, as one warp works it out for the others, in shared memory (every warp for itself, with the walk's state in the
// softmax warps' registers: 16 questions on 55724 slots 659 us against 630, 96 answers on 6 videos 125 against 116).
struct Piece {
    long long first, store;       // the entry's first token; stored row of the piece's first
    int tokens, len;              // of the entry
    int u0, u1;                   // tiles
    int head, block, at;          // at: entry
    bool own, pair, there;        // pair: two blocks of rows, else one, of whose tiles the sets take every other; there: not behind the last
    __device__ __forceinline__ int tiles() const { return u1 - u0; }
    // rows (token, query head) of a set's block, and the first of them in memory
    __device__ __forceinline__ int set_rows(const PrefixArgs& a, int set) const {
        return min(a.block_tokens, max(0, tokens - (block * (pair ? 2 : 1) + set) * a.block_tokens)) * a.group;
    }
    __device__ __forceinline__ long long set_store(const PrefixArgs& a, int set) const { return store + set * a.block_tokens * a.group; }
};

template <int DIM>
struct PieceWalk {
    PrefixEntry e;
    int at;
    long long step, end;
    __device__ __forceinline__ Piece next(const PrefixArgs& a) {
        Piece p;
        p.there = step < end;
        if (!p.there) return p;
        int32_t bits = 0;
        while (step >= e.step0 + steps_of(a, e)) {
            const long long s = e.step0 + steps_of(a, e), r = e.row0 + rows_of(a, e);
            e = prefix_entry<DIM>(a, ++at, bits);
            e.step0 = s;
            e.row0 = r;
        }
        const long long in = step - e.step0;
        const int item = (int)quotient(in, e.units);
        const int from = (int)(in - (long long)item * e.units), to = (int)min((long long)e.units, from + (end - step));
        step += to - from;
        p.first = e.first;
        p.tokens = e.tokens;
        p.len = e.len;
        p.at = at;
        p.own = at >= a.prefix.seqs;
        p.pair = !alternates<DIM>(a, e);
        p.u0 = max(0, from - kPieceSteps);
        p.u1 = max(0, to - kPieceSteps);
        p.head = item / e.blocks;
        p.block = item - p.head * e.blocks;
        const int per = (p.pair ? 2 : 1) * a.block_tokens;
        if (p.own) {
            // tiles behind the last slot that the block's last token sees hold nothing for it
            const int last = min(e.tokens, (p.block + 1) * per), seen = max(0, e.len - e.tokens + last);
            p.u1 = max(p.u0, min(p.u1, (seen + PrefixShape<DIM>::SLOTS - 1) / PrefixShape<DIM>::SLOTS));
        }
        p.store = (long long)blockIdx.x * PrefixShape<DIM>::STORE + e.row0 + ((long long)p.head * e.tokens + (long long)p.block * per) * a.group;
        return p;
    }
};

// ---- products ----

// instruction descriptor of tcgen05.mma kind::f16 with M = 128 (see kTcIdesc): type of A and B, N, B with its N axis contiguous
template <typename T>
__host__ __device__ constexpr uint32_t attend_idesc(int n, bool b_by_n) {
    const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
    return (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)b_by_n << 16) | ((uint32_t)(n / 8) << 17) | (8u << 24);
}
// (The descriptors of a warp's products differ in their low words alone.  The instruction wants them in uniform registers: moving
// there what the compiler takes for a value of one thread costs more than the product, see one_value.)
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "mov.b64 da, {%1, %2};\n\t"
        "mov.b64 db, {%3, %4};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
// A in tensor memory
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Operand whose row axis (channels) is contiguous, 128-byte swizzle: groups of eight slots 1024 bytes apart, 64-channel
// parts `part` bytes apart.
__device__ __forceinline__ uint64_t operand_by_n(uint32_t addr, uint32_t part) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(part >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t taddr, const uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]),
          "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]),
          "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// loads of 32 columns that are on their way until tmem_wait_load; what they bring is used after tmem_loaded
__device__ __forceinline__ void tmem_load32(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
          "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
          "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_loaded(uint32_t (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        asm volatile("" : "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7]));
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void copy_queries(uint32_t dst, const CUtensorMap* map, int head, int half, int row, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(head), "r"(half), "r"(row), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void copy_slots(uint32_t dst, const CUtensorMap* map, int place, int half, int head, int page, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(place), "r"(half), "r"(head), "r"(page), "r"(bar)
        : "memory");
}

// 32 channels of a row: four at a time, those of one set's rows beside each other, so that a warp writes whole stretches
__device__ __forceinline__ void store32(float4* to, int rows, const uint32_t (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 8; i++)
        to[i * rows] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
}

struct PrefixMaps {
    CUtensorMap q, k[2], v[2];    // prefix, own
};

template <typename T, int DIM, bool FINE>
__global__ void __launch_bounds__(PrefixShape<DIM>::THREADS, 1)
k_prefix_attend(const __grid_constant__ PrefixArgs a, const __grid_constant__ PrefixMaps maps) {
    using Shape = PrefixShape<DIM>;
    constexpr int SLOTS = Shape::SLOTS, SETS = Shape::SETS, HALVES = Shape::HALVES, RING = Shape::RING, TILE = Shape::TILE;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t qmem = smem_u32(smem), ring = qmem + SETS * Shape::QBLOCK;
    unsigned char* rest = smem + SETS * Shape::QBLOCK + RING * TILE;
    const uint32_t q_full = smem_u32(rest), q_empty = q_full + 8, full = q_full + 16, empty = full + 8 * RING;
    const uint32_t s_full = empty + 8 * RING, p_half = s_full + 16, p_full = p_half + 16, o_full = p_full + 16;
    const uint32_t piece_full = o_full + 16, piece_empty = piece_full + 8 * kPieces;
    uint32_t* tmem_word = reinterpret_cast<uint32_t*>(rest + Shape::BARS * 8);
    long long* scan = reinterpret_cast<long long*>(rest + Shape::BARS * 8 + 16);        // [64]
    Piece* const pieces = reinterpret_cast<Piece*>(scan);       // [kPieces], once the shares are known
    static_assert(sizeof(Piece) * kPieces <= 40 * sizeof(long long) && sizeof(PieceWalk<DIM>) <= 16 * sizeof(long long), "scan's places");
    float2* stat = reinterpret_cast<float2*>(scan + 64);        // [128] m and l of a row in the second set

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int COPY_WARP = SETS * 4, MMA_WARP = COPY_WARP + 1, WARPS = Shape::THREADS / 32;
    if (tid == 0) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        for (int s = 0; s < RING; s++) {
            mbar_init(full + 8 * s, kCopyWarps);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(s_full + 8 * b, 1);
            mbar_init(p_half + 8 * b, 4);
            mbar_init(p_full + 8 * b, 4);
            mbar_init(o_full + 8 * b, 1);
        }
        for (int i = 0; i < kPieces; i++) {
            mbar_init(piece_full + 8 * i, 1);
            mbar_init(piece_empty + 8 * i, WARPS - 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == COPY_WARP && lane < 5) {                        // (the maps are parameters: no kernel before writes them)
        const CUtensorMap* const map[5] = {&maps.q, &maps.k[0], &maps.v[0], &maps.k[1], &maps.v[1]};
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(lane == 0 ? map[0] : lane == 1 ? map[1] : lane == 2 ? map[2] : lane == 3 ? map[3] : map[4])) : "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_word)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_word);
    wait_for_prior_kernel();
    let_next_kernel_start();

    // ---- shares: the sum of all entries' steps, and the entry in which this CTA's first step lies ----
    const int entries = a.prefix.seqs + a.own.seqs;
    int32_t bits = 0;
    PrefixEntry x = {};                                         // this thread's entry of a go, with what is before it
    long long steps = 0, rows = 0;                              // of the goes so far
    auto go_through = [&](int e0) {
        const int e = e0 + tid;
        x = PrefixEntry{};
        if (e < entries) x = prefix_entry<DIM>(a, e, bits);
        const long long s = steps_of(a, x), r = rows_of(a, x);
        long long si = s, ri = r;
        const int busy = min(WARPS, (entries - e0 + 31) / 32);  // warps that have entries
        if (warp < busy) {
            si = warp_scan(s, lane);
            ri = warp_scan(r, lane);
        }
        if (e0 > 0) __syncthreads();                            // (scan has been read)
        if (lane == 31) {
            scan[warp] = si;
            scan[16 + warp] = ri;
        }
        const int bad = __syncthreads_or(bits & kStatusArg);
        x.step0 = steps + si - s;
        x.row0 = rows + ri - r;
        for (int w = 0; w < busy; w++) {
            const long long sw = scan[w], rw = scan[16 + w];
            if (w < warp) {
                x.step0 += sw;
                x.row0 += rw;
            }
            steps += sw;
            rows += rw;
        }
        return bad;
    };
    // (the entries' own offsets are looked at with them; without own slots those inside a prefix are no entry's)
    if (a.own.seqs == 0)
        for (int b = tid; b < a.seqs; b += Shape::THREADS)
            if (a.row_offsets[b + 1] < a.row_offsets[b]) bits |= kStatusArg;
    int bad = 0;
    for (int e0 = 0; e0 < entries; e0 += Shape::THREADS) bad |= go_through(e0);
    if (blockIdx.x == 0 && bits) raise_status(a.status, bits);
    const long long total = bad ? 0 : steps, share = quotient(total + gridDim.x - 1, gridDim.x);
    if (blockIdx.x == 0 && tid == 0) *a.head = PrefixHead{bad ? -1 : total, share};
    PieceWalk<DIM> walk;                                        // (without work of its own it stays where it is)
    walk.step = min(total, (long long)blockIdx.x * share);
    walk.end = min(total, walk.step + share);
    PieceWalk<DIM>* const start = reinterpret_cast<PieceWalk<DIM>*>(scan + 40);
    if (tid == 0) {
        start->step = walk.step;
        start->end = walk.end;
    }
    if (total > 0) {
        const bool once = entries <= Shape::THREADS;            // x is still there
        steps = rows = 0;
        for (int e0 = 0; e0 < entries; e0 += Shape::THREADS) {
            if (!once) {
                __syncthreads();
                go_through(e0);
            }
            const int e = e0 + tid;
            if (e < entries && x.step0 <= walk.step && walk.step < x.step0 + steps_of(a, x)) {
                start->e = x;
                start->at = e;
            }
            if (blockIdx.x == 0 && e < entries) a.entries[e] = x;
            // The tokens' entries, shared between the CTAs, all of which go through all entries for it.  (One CTA's thread per entry instead, with the
            // others stopping at their first step: 390 questions of 50 tokens 442 us against 96, 3200 of one token 208 against 148.)
            if (e < entries && x.units > 0)
                for (long long i = blockIdx.x; i < x.tokens; i += gridDim.x) (e < a.prefix.seqs ? a.prefix_of : a.own_of)[x.first + i] = e;
        }
    }
    __syncthreads();
    walk = *start;

    // 384 threads are launched with 168 registers each (64512).  The softmax warps hold a row of 128 logits: they take 208, for
    // which the third warpgroup goes down to 88 (128 * 88 + 256 * 208 = 64512).
    bool timed_out = false;
    // The last copy warp (it has the fewest boxes of a tile) works out the pieces, one ahead of its own copies, and puts them into shared memory.
    auto publish = [&](int i) -> bool {
        const Piece next = walk.next(a);
        if (i >= kPieces && !mbar_wait_near(piece_empty + 8 * (i % kPieces), i / kPieces - 1, timed_out)) return false;
        if (lane == 0) {
            pieces[i % kPieces] = next;
            mbar_arrive(piece_full + 8 * (i % kPieces));
        }
        __syncwarp();
        return true;
    };
    auto there_is = [&](int i) -> bool { return mbar_wait_near(piece_full + 8 * (i % kPieces), i / kPieces, timed_out) && pieces[i % kPieces].there; };
    auto done_with = [&](int i) {
        __syncwarp();
        if (lane == 0) mbar_arrive(piece_empty + 8 * (i % kPieces));
    };
    if (warp >= COPY_WARP) {
        if constexpr (SETS == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp != MMA_WARP) {
        // ------------------------------------- copies -------------------------------------
        // Issuing a tensor copy keeps a warp busy for some 80 cycles whatever its size, and small pages make many of them: the
        // boxes of a tile (a box of slots, 64 channels) are shared between three warps, one box to a lane.
        const int part = warp == COPY_WARP ? 0 : warp - MMA_WARP;
        int n = 0, p = 0;                                       // ring slots and pieces with tiles taken up so far
        const bool walks = part == kCopyWarps - 1;
        if (walks) publish(0);
        for (int i = 0; there_is(i) && (!walks || publish(i + 1)); i++) {
            const Piece now = pieces[i % kPieces];
            if (!walks) done_with(i);
            const int tiles = now.tiles();
            if (tiles == 0) continue;
            const bool pair = now.pair;
            const int own = now.own;
            const CacheView& c = own ? a.own : a.prefix;
            const int box = a.page_box[own], page_slots = c.page, pages = (int)c.pages;
            const int32_t* table = c.table + (own ? now.at - a.prefix.seqs : now.at) * c.table_stride;
            const int at = lane * kCopyWarps + part, in_tile = at / HALVES * box, half = at % HALVES;
            const bool copies = in_tile < SLOTS;
            // Page and place in it of this lane's box, by the tile's number modulo four; looked up two tiles ahead.  (-1: the box lies
            // behind the last slot.  It is not copied: logits there are masked, values cleared.  `pages`, beyond the pool: zeros.)
            int page[4], place[4];
            const int slot0 = now.u0 * SLOTS + in_tile, by_pages = SLOTS / page_slots, by_slots = SLOTS % page_slots;
            int left = now.len - slot0, stretch = slot0 / page_slots, spot = slot0 - stretch * page_slots;     // of the tile looked up next
            auto look_up = [&](int& pg, int& pl) {
                pg = -1;
                pl = spot;
                if (copies && left > 0) {
                    pg = table[stretch];
                    if (pg < 0) pg = INT_MAX;
                }
                left -= SLOTS;
                stretch += by_pages;
                spot += by_slots;
                if (spot >= page_slots) {
                    spot -= page_slots;
                    stretch++;
                }
            };
            const uint32_t to = ring + half * (SLOTS * 128) + in_tile * 128;
            auto copy = [&](const CUtensorMap* map, int pg, int pl) -> bool {
                const int s = n % RING;
                if (n >= RING && !mbar_wait_near(empty + 8 * s, n / RING - 1, timed_out)) return false;
                const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, pg >= 0));
                if (lane == 0) mbar_expect_tx(full + 8 * s, boxes * box * 128);
                __syncwarp();
                if (pg >= 0) {
                    if (pg >= pages) {
                        raise_status(a.status, kStatusArg);
                        pg = pages;
                    }
                    copy_slots(to + s * TILE, map, pl, half, now.head, pg, full + 8 * s);
                }
                n++;
                return true;
            };
            look_up(page[0], place[0]);
            look_up(page[1], place[1]);
            if (walks) {
                if (p > 0 && !mbar_wait_near(q_empty, p - 1, timed_out)) break;
                if (lane == 0) {
                    const int sets = pair ? 2 : 1, q_bytes = a.block_tokens * a.group * 128;
                    mbar_expect_tx(q_full, sets * HALVES * q_bytes);
                    for (int t = 0; t < sets; t++)
                        for (int h = 0; h < HALVES; h++)
                            copy_queries(qmem + t * Shape::QBLOCK + h * (128 * 128), &maps.q, now.head * a.group, h,
                                         (int)(now.first + (long long)(now.block * sets + t) * a.block_tokens), q_full);
                }
                __syncwarp();
                p++;
            }
            // In the order in which the products want them, K0 V0 K1 V1 ..., or K0 K1 V0 K2 V1 ... where tiles alternate: keys of tile j,
            // values of the tile one or two before.
            const int behind = pair ? 1 : 2;
            bool ok = true;
            for (int j0 = 0; ok && j0 < tiles + behind; j0 += 4) {
#pragma unroll
                for (int u = 0; u < 4; u++) {
                    const int j = j0 + u;
                    if (ok && j >= behind && j < tiles + behind)
                        ok = pair ? copy(&maps.v[own], page[(u + 3) & 3], place[(u + 3) & 3]) : copy(&maps.v[own], page[(u + 2) & 3], place[(u + 2) & 3]);
                    if (ok && j < tiles) ok = copy(&maps.k[own], page[u], place[u]);
                    look_up(page[(u + 2) & 3], place[(u + 2) & 3]);
                }
            }
            if (!ok) break;
        }
        // the CTA must not end with copies in flight
        for (int i = max(0, n - RING); i < n; i++) {
            bool late = false;
            mbar_wait_sleep(full + 8 * (i % RING), i / RING, late);
            timed_out |= late;
        }
        if (p > 0) {
            bool late = false;
            mbar_wait_sleep(q_full, p - 1, late);
            timed_out |= late;
        }
        } else {
        // ------------------------------------- products -------------------------------------
        // Step x of a piece: tile x / 2 for set x % 2, or tile x where tiles alternate.  First the logits of steps 0 and 1, then the
        // values of step x and the logits of step x + 2: those of one set run while the other's exponentials are formed.  Between two
        // products this warp's own instructions, one dependent on the other, are time in which the tensor cores idle: ring slots are
        // counted up as they are taken (in the order in which the copies fill them), addresses are ready before the waits.
        int p = 0;                                              // pieces
        uint32_t slot = 0, turn = 0, weights_turn[2] = {0, 0};  // ring slot taken next; parities of its, and of the weights', next wait
        const uint32_t q_lo = one_value((uint32_t)tc_operand(qmem)), ring_lo = one_value((uint32_t)tc_operand(ring));
        const uint32_t ring_by_n = one_value((uint32_t)operand_by_n(ring, SLOTS * 128)), tm = one_value(tmem), bars = one_value(smem_u32(rest));
        const uint32_t o_full_u = bars + (o_full - q_full), s_full_u = bars + (s_full - q_full), empty_u = bars + (empty - q_full);
        auto take = [&](uint32_t& taken) -> bool {
            taken = slot;
            const bool ok = mbar_wait_near(full + 8 * slot, turn, timed_out);
            if (++slot == RING) {
                slot = 0;
                turn ^= 1;
            }
            return ok;
        };
        for (int i = 0; there_is(i); i++) {
            const Piece now = pieces[i % kPieces];
            done_with(i);
            const int tiles = now.tiles();
            if (tiles == 0) continue;
            const bool pair = now.pair;
            // logits of set (place) b
            auto logits = [&](auto place, int set, uint32_t k_slot, bool frees, bool last) {
                constexpr int b = decltype(place)::value;
                const uint32_t at = one_value(k_slot), a_lo = q_lo + (SETS == 2 && set ? Shape::QBLOCK / 16 : 0), b_lo = ring_lo + at * (TILE / 16);
                if (elected()) {
#pragma unroll
                    for (int k = 0; k < DIM / 16; k++)
                        mma_ss(tm + b * 128, a_lo + (k >> 2) * (128 * 128 / 16) + (k & 3) * 2, kOperandHigh, b_lo + (k >> 2) * (SLOTS * 128 / 16) + (k & 3) * 2,
                               kOperandHigh, attend_idesc<T>(SLOTS, false), k > 0);
                    tc_commit(s_full_u + 8 * b);
                    if (frees) tc_commit(empty_u + 8 * at);
                    if (last) tc_commit(bars + 8);              // q_empty
                }
                __syncwarp();
            };
            // weights of place b times the values
            auto values = [&](auto place, uint32_t v_slot, bool more, bool frees) -> bool {
                constexpr int b = decltype(place)::value, set = SETS == 2 ? b : 0;
                const uint32_t at = one_value(v_slot), v_lo = ring_by_n + at * (TILE / 16), d = tm + Shape::O_COL + set * DIM;
                if (!mbar_wait_near(p_half + 8 * b, weights_turn[b], timed_out)) return false;
                tc_fence_after();
                if (elected()) {
#pragma unroll
                    for (int k = 0; k < SLOTS / 32; k++) {
                        mma_ts(d, tm + b * 128 + k * 8, v_lo + k * (2048 / 16), kOperandHigh, attend_idesc<T>(DIM, true), k > 0 ? 1 : more);
                        if (FINE) mma_ts(d, tm + b * 128 + 64 + k * 8, v_lo + k * (2048 / 16), kOperandHigh, attend_idesc<T>(DIM, true), 1);
                    }
                }
                __syncwarp();
                if (!mbar_wait_near(p_full + 8 * b, weights_turn[b], timed_out)) return false;
                weights_turn[b] ^= 1;
                tc_fence_after();
                if (elected()) {
#pragma unroll
                    for (int k = SLOTS / 32; k < SLOTS / 16; k++) {
                        mma_ts(d, tm + b * 128 + k * 8, v_lo + k * (2048 / 16), kOperandHigh, attend_idesc<T>(DIM, true), 1);
                        if (FINE) mma_ts(d, tm + b * 128 + 64 + k * 8, v_lo + k * (2048 / 16), kOperandHigh, attend_idesc<T>(DIM, true), 1);
                    }
                    tc_commit(o_full_u + 8 * set);
                    if (frees) tc_commit(empty_u + 8 * at);
                }
                __syncwarp();
                return true;
            };
            // What lies behind the last slot may be anything: 0 times it must be 0.
            auto clear_tail = [&](int j, uint32_t v_slot) {
                const int there = now.len - (now.u0 + j) * SLOTS;
                if (j + 1 < tiles || there >= SLOTS) return;
                for (int w = lane; w < (SLOTS - there) * 8 * HALVES; w += 32) {
                    const int h = w / ((SLOTS - there) * 8), u = w - h * (SLOTS - there) * 8;
                    *reinterpret_cast<uint4*>(smem + SETS * Shape::QBLOCK + v_slot * TILE + h * (SLOTS * 128) + there * 128 + u * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async_smem();
                __syncwarp();
            };
            const std::integral_constant<int, 0> zero{};
            const std::integral_constant<int, 1> one{};
            uint32_t ks = 0, vs = 0;
            if (!mbar_wait_near(q_full, p, timed_out) || !take(ks)) break;
            p++;
            bool ok = true;
            if (pair) {
                logits(zero, 0, ks, false, false);
                logits(one, 1, ks, true, tiles == 1);
#pragma unroll 1
                for (int j = 0; j < tiles; j++) {
                    const bool more = j + 1 < tiles;
                    if (!(ok = take(vs))) break;
                    clear_tail(j, vs);
                    if (!(ok = values(zero, vs, j > 0, false))) break;
                    if (more) {
                        if (!(ok = take(ks))) break;
                        logits(zero, 0, ks, false, false);
                    }
                    if (!(ok = values(one, vs, j > 0, true))) break;
                    if (more) logits(one, 1, ks, true, j + 2 == tiles);
                }
            } else {
                logits(zero, 0, ks, true, tiles == 1);
                if (tiles > 1) {
                    if (!take(ks)) break;
                    logits(one, 0, ks, true, tiles == 2);
                }
#pragma unroll 1
                for (int j = 0; j < tiles; j += 2) {
                    if (!(ok = take(vs))) break;
                    clear_tail(j, vs);
                    if (!(ok = values(zero, vs, j > 0, true))) break;
                    if (j + 2 < tiles) {
                        if (!(ok = take(ks))) break;
                        logits(zero, 0, ks, true, j + 3 == tiles);
                    }
                    if (j + 1 < tiles) {
                        if (!(ok = take(vs))) break;
                        clear_tail(j + 1, vs);
                        if (!(ok = values(one, vs, SETS == 1 || j > 0, true))) break;
                        if (j + 3 < tiles) {
                            if (!(ok = take(ks))) break;
                            logits(one, 0, ks, true, j + 4 == tiles);
                        }
                    }
                }
            }
            if (!ok) break;
        }
        }
    } else {
        // ------------------------------------- softmax -------------------------------------
        if constexpr (SETS == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int set = warp >> 2, row = 32 * (warp & 3) + lane;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t o_at = tmem + lanes + Shape::O_COL + set * DIM;
        const int tok = row / a.group;
        int s_uses0 = 0, s_uses1 = 0, o_uses = 0;               // logits taken from either place, products into O
        int at = 0;                                             // piece
        for (; there_is(at); at++) {
            const Piece& now = pieces[at % kPieces];
            const bool pair = now.pair;
            const int tiles = now.tiles(), token = (now.block * (pair ? 2 : 1) + (pair ? set : 0)) * a.block_tokens + tok;
            const bool there = tok < a.block_tokens && token < now.tokens;
            // slots that this row sees, of the piece's
            const int limit = (now.own ? min(now.len, now.len - now.tokens + token + 1) : now.len) - now.u0 * SLOTS;
            float m = -INFINITY, l = 0.0f;
            const int steps = pair ? 2 * tiles : tiles;
            bool first = true;
            for (int x = SETS == 2 ? set : 0; x < steps; x += SETS) {
                const int j = pair ? x >> 1 : x, b = x & 1;
                const uint32_t s_at = tmem + lanes + b * 128;
                if (!mbar_wait_near(s_full + 8 * b, b ? s_uses1++ : s_uses0++, timed_out)) break;
                tc_fence_after();
                uint32_t v[SLOTS / 32][32];
#pragma unroll
                for (int i = 0; i < SLOTS / 32; i++) tmem_load32(s_at + 32 * i, v[i]);
                tmem_wait_load();
#pragma unroll
                for (int i = 0; i < SLOTS / 32; i++) tmem_loaded(v[i]);
                const int left = limit - j * SLOTS;             // slots of this tile that the row sees
                if (__any_sync(0xffffffffu, left < SLOTS)) {
#pragma unroll
                    for (int i = 0; i < SLOTS; i++)
                        if (i >= left) v[i / 32][i % 32] = 0xff800000u;
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < SLOTS; i += 2) {
                    float& t = top[(i >> 1) & 3];
                    t = max3(t, __uint_as_float(v[i / 32][i % 32]), __uint_as_float(v[i / 32][i % 32 + 1]));
                }
                const float tile_top = max3(max3(top[0], top[1], top[2]), top[3], top[3]);
                const bool rise = (tile_top - m) * a.scale_log2 > kLazyRise;     // (not for -inf after -inf)
                float factor = 1.0f;
                if (rise) {
                    factor = exp2_fast((m - tile_top) * a.scale_log2);
                    m = tile_top;
                }
                if (!first && __any_sync(0xffffffffu, rise)) {
                    if (!mbar_wait_near(o_full + 8 * set, o_uses - 1, timed_out)) break;
                    tc_fence_after();
                    l *= factor;
#pragma unroll 1
                    for (int i = 0; i < DIM; i += 32) {
                        uint32_t o[32];
                        tc_load32(o_at + i, o);
#pragma unroll
                        for (int k = 0; k < 32; k++) o[k] = __float_as_uint(__uint_as_float(o[k]) * factor);
                        tmem_store32(o_at + i, o);
                    }
                }
                first = false;
                // (a NaN among the logits makes the row NaN)
                const float base = tile_top != tile_top ? tile_top : m == -INFINITY ? 0.0f : kWeightBias<T> - m * a.scale_log2;
                const uint64_t scale2 = both(a.scale_log2, a.scale_log2), base2 = both(base, base);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < SLOTS / 32; i++) {
                    uint32_t w[16], left_over[16];
#pragma unroll
                    for (int k = 0; k < 16; k++) {
                        const uint64_t e = fma2(both(__uint_as_float(v[i][2 * k]), __uint_as_float(v[i][2 * k + 1])), scale2, base2);
                        float p0, p1;
                        apart(e, p0, p1);
                        p0 = exp2_fast(p0);
                        p1 = exp2_fast(p1);
                        sum[k & 1] = add2(sum[k & 1], both(p0, p1));
                        w[k] = Pair<T>::pack(p0, p1);
                        if constexpr (FINE) {
                            const float2 rounded = Pair<T>::split(w[k]);
                            left_over[k] = Pair<T>::pack(p0 - rounded.x, p1 - rounded.y);       // (the differences are exact)
                        }
                    }
                    tmem_store16(s_at + 16 * i, w);
                    if constexpr (FINE) tmem_store16(s_at + 64 + 16 * i, left_over);
                    if (i + 1 == SLOTS / 64) {                  // the product begins with the first half of the weights
                        tmem_wait_store();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(p_half + 8 * b);
                        __syncwarp();
                    }
                }
                float s0, s1;
                apart(add2(sum[0], sum[1]), s0, s1);
                l += s0 + s1;
                tmem_wait_store();
                tc_fence_before();
                __syncwarp();
                // With two places for one block's logits the product before may still run: it is waited for here, since a wait for this
                // tile's, by its parity, would take that of two tiles before for it.
                if (SETS == 1 && o_uses > 0 && !mbar_wait_near(o_full + 8 * set, o_uses - 1, timed_out)) break;
                if (lane == 0) mbar_arrive(p_full + 8 * b);
                o_uses++;
            }
            if (timed_out) break;
            // this piece's O, l and m
            if (!first && !mbar_wait_near(o_full + 8 * set, o_uses - 1, timed_out)) break;
            tc_fence_after();
            const int rows = now.set_rows(a, pair ? set : 0);
            const long long store = now.set_store(a, pair ? set : 0);
            float4* const to = reinterpret_cast<float4*>(a.partial + store * DIM) + row;
            if (SETS == 2 && !pair && tiles > 1) {
                // both sets have a part of the same rows, in the same lanes: each puts half of the channels together
                if (set == 1) stat[row] = make_float2(m, l);
                named_sync(1, 256);
                float f0 = 0.0f, f1 = 0.0f;
                if (set == 0) {
                    const float2 other = stat[row];
                    const float most = fmaxf(m, other.x);
                    f0 = m == -INFINITY ? 0.0f : exp2_fast((m - most) * a.scale_log2);
                    f1 = other.x == -INFINITY ? 0.0f : exp2_fast((other.x - most) * a.scale_log2);
                    // (without a maximum l is 0, or NaN: logits that are all NaN have none, and have to reach the output)
                    l = (m == -INFINITY ? l : f0 * l) + (other.x == -INFINITY ? other.y : f1 * other.y);
                    m = most;
                    stat[row] = make_float2(f0, f1);
                }
                named_sync(1, 256);
                if (set == 1) {
                    f0 = stat[row].x;
                    f1 = stat[row].y;
                }
#pragma unroll 1
                for (int i = set * (DIM / 2); i < (set + 1) * (DIM / 2); i += 32) {
                    uint32_t o[32], u[32];
                    tmem_load32(tmem + lanes + Shape::O_COL + i, o);
                    tmem_load32(tmem + lanes + Shape::O_COL + DIM + i, u);
                    tmem_wait_load();
                    tmem_loaded(o);
                    tmem_loaded(u);
#pragma unroll
                    for (int k = 0; k < 32; k++) o[k] = __float_as_uint(f0 * __uint_as_float(o[k]) + f1 * __uint_as_float(u[k]));
                    if (there) store32(to + (i / 4) * rows, rows, o);
                    __syncwarp();                               // (the next load is one for the whole warp)
                }
                tc_fence_before();
                named_sync(1, 256);                             // before either set's O is begun again
            } else if (!first) {
#pragma unroll 1
                for (int i = 0; i < DIM; i += 32) {
                    uint32_t o[32];
                    tc_load32(o_at + i, o);
                    if (there) store32(to + (i / 4) * rows, rows, o);
                    __syncwarp();
                }
                tc_fence_before();
            }
            if (there && (pair || set == 0)) a.stats[store + row] = make_float2(m == -INFINITY ? -INFINITY : m * a.scale_log2 - kWeightBias<T>, l);
            done_with(at);
        }
        // A warp whose wait ran out has left a piece before the barriers at which the sets meet, or does not learn of the pieces to come: the
        // others wait for it there.
        if (SETS == 2 && timed_out) {
            walk = *start;
            for (int i = 0;; i++) {
                const Piece now = walk.next(a);
                if (!now.there) break;
                if (i >= at && !now.pair && now.tiles() > 1)
                    for (int k = 0; k < 3; k++) named_sync(1, 256);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == MMA_WARP) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
    if (timed_out) raise_status(a.status, kStatusWaitTimeout);
}

// ---- pieces of a row to its output ----

constexpr int kPrefixJoinThreads = 256;
constexpr int kJoinParts = 320;                                 // pieces of a row at most: two entries' over all CTAs

// A block puts ROWS rows (token, query head of one KV head) together: 32, or, where rows are few and their pieces many, 8, and then eight chunks
// of four channels of them, the pieces shared between four groups of threads.  First a part of a warp per row finds the row's pieces and
// their weights; then a thread takes four channels of a row, rows beside each other as the pieces store them.  Dependent reads bound it: a token's
// entries, where they lie, m and l, O.
__host__ __device__ constexpr int prefix_join_split(int dim, int rows) { return rows == 8 ? dim / 32 : 1; }     // blocks per rows

template <typename T, int DIM, int ROWS>
__global__ void __launch_bounds__(kPrefixJoinThreads) k_prefix_join(const __grid_constant__ PrefixArgs a) {
    constexpr int LANES = kPrefixJoinThreads / ROWS;            // per row
    struct Row {
        const float4* from[2];    // the row's first four channels in its first piece
        int parts[2], rows[2];    // pieces; rows of the block that they lie in
        float inv, top;
    };
    __shared__ Row found[ROWS];
    __shared__ float weights[ROWS][kJoinParts + 1];             // (rows in different banks)
    wait_for_prior_kernel();
    let_next_kernel_start();
    const uint32_t per_kv = (uint32_t)a.rows * a.group, blocks = (per_kv + ROWS - 1) / ROWS;       // (below 2^31)
    constexpr uint32_t SPLIT = prefix_join_split(DIM, ROWS);
    const uint32_t split = blockIdx.x % SPLIT, at_block = blockIdx.x / SPLIT;
    const uint32_t kv = at_block / blocks, row0 = (at_block - kv * blocks) * ROWS;
    {
        const int k = threadIdx.x / LANES, lane = threadIdx.x % LANES;
        const uint32_t token = (row0 + k) / (uint32_t)a.group;
        const int g = (int)(row0 + k - token * a.group);
        Row r = {};
        // (a token of no sequence, or without a prefix, finds rubbish in the tables: an entry whose tokens it is not among)
        const bool there = row0 + k < per_kv;
        const int of[2] = {there ? a.prefix_of[token] : -1, there && a.own.seqs > 0 ? a.own_of[token] : -1};
        const bool used = there && token >= a.row_offsets[0] && token < a.row_offsets[a.seqs];
        const PrefixHead head = *a.head;
        long long at[2] = {0, 0};                               // stored row of the first piece
#pragma unroll
        for (int which = 0; which < 2; which++) {
            const bool fits = used && head.total > 0 && of[which] >= (which ? a.prefix.seqs : 0) && of[which] < a.prefix.seqs + (which ? a.own.seqs : 0);
            if (!fits) continue;
            const PrefixEntry e = a.entries[of[which]];
            if (e.units == 0 || token < e.first || token >= e.first + e.tokens) continue;
            const int in = (int)(token - e.first), set = in / a.block_tokens, block = alternates<DIM>(a, e) ? set : set >> 1;
            const long long s0 = e.step0 + ((long long)kv * e.blocks + block) * e.units;
            const long long c0 = quotient(s0, head.share), c1 = quotient(s0 + e.units - 1, head.share);
            const long long first = c0 * PrefixShape<DIM>::STORE + e.row0 + ((long long)kv * e.tokens + (long long)set * a.block_tokens) * a.group;
            const int row = (in - set * a.block_tokens) * a.group + g;
            at[which] = first + row;
            r.from[which] = reinterpret_cast<const float4*>(a.partial + first * DIM) + row;
            r.rows[which] = min(a.block_tokens, e.tokens - set * a.block_tokens) * a.group;
            r.parts[which] = (int)(c1 - c0) + 1;
        }
        const int n = r.parts[0] + r.parts[1];
        auto stat = [&](int i) {
            return i >= n ? make_float2(-INFINITY, 0.0f)
                          : a.stats[i < r.parts[0] ? at[0] + (long long)i * PrefixShape<DIM>::STORE : at[1] + (long long)(i - r.parts[0]) * PrefixShape<DIM>::STORE];
        };
        const float2 mine = stat(lane);                         // (all of them, unless the row is cut into more than LANES)
        r.top = mine.x;
        for (int i = lane + LANES; i < n; i += LANES) r.top = fmaxf(r.top, stat(i).x);
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) r.top = fmaxf(r.top, __shfl_xor_sync(0xffffffffu, r.top, o));
        float total = 0.0f;
        for (int i = lane; i < n; i += LANES) {
            const float2 s = i < LANES ? mine : stat(i);
            const float weight = s.x == -INFINITY ? 0.0f : exp2f(s.x - r.top);
            weights[k][i] = weight;
            total += weight * s.y;
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        r.inv = total == 0.0f ? 0.0f : 1.0f / total;
        if (!used || head.total < 0) r.parts[0] = -1;           // (bad offsets: nothing is written)
        if (lane == 0) {
            found[k] = r;
            if (r.parts[0] >= 0 && a.lse != nullptr && split == 0)
                a.lse[(long long)token * a.q_heads + kv * a.group + g] = total == 0.0f ? -INFINITY : (r.top + log2f(total)) * 0.69314718055994531f;
        }
    }
    __syncthreads();
    const int k = threadIdx.x % ROWS;
    const Row r = found[k];
    const int n = r.parts[0] < 0 ? 0 : r.parts[0] + r.parts[1];
    const uint32_t token = (row0 + k) / (uint32_t)a.group;
    uint16_t* const out = a.out + ((long long)token * a.q_heads + kv * a.group + (row0 + k - token * a.group)) * DIM;
    if constexpr (ROWS == 8) {
        constexpr int GROUPS = 4, AHEAD = 10;
        __shared__ float4 parked[GROUPS - 1][64];
        const int group = threadIdx.x / 64, chunk = split * 8 + threadIdx.x / 8 % 8;
        const float4 *const from0 = r.from[0] + (long long)chunk * r.rows[0], *const from1 = r.from[1] + (long long)chunk * r.rows[1];
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (int i0 = group; i0 < n; i0 += GROUPS * AHEAD) {
            float4 o[AHEAD];
            float f[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const int i = i0 + u * GROUPS;
                f[u] = i < n ? weights[k][i] : 0.0f;
                // (a piece without tiles has the weight 0: it stored no O)
                o[u] = *(f[u] == 0.0f         ? reinterpret_cast<const float4*>(a.partial)
                         : i >= r.parts[0] ? from1 + (long long)(i - r.parts[0]) * (PrefixShape<DIM>::STORE * (DIM / 4))
                                             : from0 + (long long)i * (PrefixShape<DIM>::STORE * (DIM / 4)));
            }
#pragma unroll
            for (int u = 0; u < AHEAD; u++)
                if (f[u] != 0.0f) {
                    acc.x += f[u] * o[u].x;
                    acc.y += f[u] * o[u].y;
                    acc.z += f[u] * o[u].z;
                    acc.w += f[u] * o[u].w;
                }
        }
        if (group > 0) parked[group - 1][threadIdx.x % 64] = acc;
        __syncthreads();
        if (group > 0 || r.parts[0] < 0) return;
#pragma unroll
        for (int g = 0; g < GROUPS - 1; g++) {
            const float4 o = parked[g][threadIdx.x];
            acc.x += o.x;
            acc.y += o.y;
            acc.z += o.z;
            acc.w += o.w;
        }
        *reinterpret_cast<uint2*>(out + chunk * 4) = make_uint2(Pair<T>::pack(acc.x * r.inv, acc.y * r.inv), Pair<T>::pack(acc.z * r.inv, acc.w * r.inv));
        return;
    }
    if (r.parts[0] < 0) return;
    // CHUNKS chunks of four channels of AHEAD pieces are on their way at a time
    constexpr int CHUNKS = DIM / 4 > LANES ? (DIM / 4 / LANES < 4 ? DIM / 4 / LANES : 4) : 1, AHEAD = 16 / CHUNKS;
#pragma unroll 1
    for (int chunk = threadIdx.x / ROWS; chunk < DIM / 4; chunk += LANES * CHUNKS) {
        const float4 *const from0 = r.from[0] + (long long)chunk * r.rows[0], *const from1 = r.from[1] + (long long)chunk * r.rows[1];
        float4 acc[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) acc[c] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (int i0 = 0; i0 < n; i0 += AHEAD) {
            float4 o[AHEAD][CHUNKS];
            float f[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const int i = i0 + u;
                f[u] = i < n ? weights[k][i] : 0.0f;
                const bool own = i >= r.parts[0];
                // (a piece without tiles has the weight 0: it stored no O)
                const float4* const from = f[u] == 0.0f ? reinterpret_cast<const float4*>(a.partial)
                                           : own        ? from1 + (long long)(i - r.parts[0]) * (PrefixShape<DIM>::STORE * (DIM / 4))
                                                        : from0 + (long long)i * (PrefixShape<DIM>::STORE * (DIM / 4));
                const int next = f[u] == 0.0f ? 0 : LANES * (own ? r.rows[1] : r.rows[0]);
#pragma unroll
                for (int c = 0; c < CHUNKS; c++) o[u][c] = from[c * next];
            }
#pragma unroll
            for (int u = 0; u < AHEAD; u++)
                if (f[u] != 0.0f)
#pragma unroll
                    for (int c = 0; c < CHUNKS; c++) {
                        acc[c].x += f[u] * o[u][c].x;
                        acc[c].y += f[u] * o[u][c].y;
                        acc[c].z += f[u] * o[u][c].z;
                        acc[c].w += f[u] * o[u][c].w;
                    }
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; c++)
            *reinterpret_cast<uint2*>(out + (chunk + c * LANES) * 4) =
                make_uint2(Pair<T>::pack(acc[c].x * r.inv, acc[c].y * r.inv), Pair<T>::pack(acc[c].z * r.inv, acc[c].w * r.inv));
    }
}

}  // namespace sttm
