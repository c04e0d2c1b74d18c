// Attention of drafted trees over a paged KV cache.
//  o[t][h] = sum_r softmax_r(scale q . K[r]) V[r] over the cached rows of the token's sequence and the drafted rows its bits name.
// One pass over the rows with the running maximum and sum; long sequences divided among workgroups, whose records (maximum, sum, columns) a second launch joins.
//  * All queries on a KV head (tokens times heads of the group) share its rows: 16 or 32 of them are the columns of a wave's products.  Few queries (single tokens, short
//    drafts) are bound by the stream of rows, many by the matrix cores and the exponentials; there is a kernel for either.
//  * Both products transposed: S^T = K Q^T with the rows of K as they lie in memory, then O^T = V^T P^T.  A lane then holds the scores of ONE query
//    (column lane % 32), 16 of a block's 32 rows, so maximum, sum and rescaling need no other lane but the one 32 further; and its probabilities are the B operand of the
//    second product as they stand, for rows 4 (lane / 32) + 0..3 (+ 8) of every 16: the A operand takes V's rows in that order.
//  * K and V go from memory straight into LDS, a tile ahead.  Eight rows in a row lie in one page (pages are powers of two from 8 rows on), so page numbers are
//    looked up through the scalar cache, and an address is a wave-uniform base plus a lane's fixed offset.
//  * The maximum is only moved, and the sums rescaled, when a probability would exceed the largest so far by a factor (TreeRange): fp32 sums hold those as well as ones up to 1.
//  * Probabilities that become binary16 numbers are relative to the maximum times 2^12, which the quotient with their sum cancels: rows far below the maximum, which may be
//    many (behind a first token that takes nearly everything, say), would else be subnormal numbers of few bits, or zero from 2^-25 of the largest on.
//  * fp32 queries: Q (scaled by a power of two per query) and P as two binary16 numbers each, 22 bits, two products into one accumulator.  16-bit queries: P as two numbers of
//    the type where few queries wait for the rows anyway, rounded to one where many make the products the bound.
//  * Tiles with drafted rows, rows past the end or rows whose page is absent are special: scores are masked by selection, and V's rows that nobody sees are
//    zeroed in LDS (zero times what they hold need not be zero).  A drafted row that somebody sees and another does not may hold infinities or NaN: such elements are
//    zeroed for the product and added to the sums of those that see them in the end.
// Measured, with the join: one token behind 512 rows (32 / 8 heads of 128, fp32) 9.7 to 11.4 us, behind 30001 (64 / 8) 27.0: 4.6 TB/s, 5.1 within its launch, of which 3.5 us pass
// before rows arrive; 16 sequences of one token behind 4100 (40 / 8, f16) 44.7: 5.2; 12 tokens behind 8192 (32 / 8, fp32) 21.2; 8 x 63 behind 6000 (64 / 8, bf16) 100: 730 TFLOP/s
// within its launch of 1174 that a large product reaches, fp32 160.
#include <atomic>
#include <cstddef>
#include <type_traits>

#include "paged_common.h"

namespace prima {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef short s4v __attribute__((ext_vector_type(4)));

constexpr int TREE_MAX_RANGES = 256;
constexpr int TREE_STEP = 64;        // rows that ranges are multiples of
constexpr int TREE_REC = 4;          // a record: (maximum, sum, -, -), D columns

// Of the probabilities that enter the products as numbers of type C, in powers of two: LIFT is what the largest score so far has, DEFER how far above it one may be before the
// maximum is moved.  Binary16 ends below 2^16; 2^3 is passed by hardly any score behind the first tile's (N(0, 1) scores: maxima of 64 and 6000 are 2.4 and 3.8).  bfloat16 has fp32's range.
template <class C>
struct TreeRange {
    static constexpr float LIFT = 12.f, DEFER = 3.f;
};
template <>
struct TreeRange<BF16> {
    static constexpr float LIFT = 0.f, DEFER = 8.f;
};

struct TreeAttnArgs {
    PagedArgs p;
    const void *q;
    void *o;
    float *part;  // the ranges' records
    int64_t ldq, ldo;
    float scale;  // times log2 e
    int Hq, G;        // G: query heads of a KV head
    unsigned inverse; // 2^32 / G, rounded up (G > 1)
    int tile_q;       // queries of a workgroup
    int order[PRIMA_PAGED_MAX_SEQS];       // sequences, the longest first
    int work0[PRIMA_PAGED_MAX_SEQS + 1];   // first workgroup of every sequence in that order, and their number
    int ranges[PRIMA_PAGED_MAX_SEQS];      // of a sequence
    int range_rows[PRIMA_PAGED_MAX_SEQS];  // of a sequence's ranges (the last may have fewer)
    int rec0[PRIMA_PAGED_MAX_SEQS];        // records in front of a sequence's, for one head (sequences of one range have none)
};

template <int D, int NR>
struct TreeShape {
    static constexpr int NK = 8 / NR;               // waves that share queries
    static constexpr int BLOCKS = NR == 8 ? 2 : 1;  // blocks of 32 rows a wave takes of a tile
    static constexpr int ROWS = 32 * BLOCKS * NK;   // of a tile: 64, or 128
    static constexpr int SLOTS = ROWS == 64 ? 3 : 2; // places for tiles of K (V)
    static constexpr int TILE = ROWS * D;           // elements of K (V) in a tile
    static constexpr size_t RING = 2 * SLOTS * TILE * 2;
    static constexpr size_t JOIN = NK == 1 ? 0 : 8 * 32 * (D + 4) * 4 + 2 * 8 * 32 * 4;
    static constexpr size_t LDS = RING > JOIN ? RING : JOIN;
};

template <class C>
__device__ __forceinline__ f16v tree_mfma(u4v a, u4v b, f16v c);
template <>
__device__ __forceinline__ f16v tree_mfma<F16>(u4v a, u4v b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f16v tree_mfma<BF16>(u4v a, u4v b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

// whether a 16-bit number is infinite or NaN
template <class C>
__device__ __forceinline__ bool odd16(unsigned v)
{
    constexpr unsigned E = sizeof(C) && __is_same(C, BF16) ? 0x7f80u : 0x7c00u;
    return (v & E) == E;
}
template <class C>
__device__ __forceinline__ float widen16(unsigned v)
{
    if (__is_same(C, BF16)) return __builtin_bit_cast(float, v << 16);
    return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<unsigned short>(v)));
}

// eight 16-bit numbers: whether one is infinite or NaN; those replaced by zero
template <class C>
__device__ __forceinline__ bool odd8(u4v v)
{
    bool r = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) r = r || odd16<C>(v[e] & 0xffffu) || odd16<C>(v[e] >> 16);
    return r;
}
template <class C>
__device__ __forceinline__ u4v without_odd(u4v v)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (odd16<C>(v[e] & 0xffffu)) v[e] &= 0xffff0000u;
        if (odd16<C>(v[e] >> 16)) v[e] &= 0xffffu;
    }
    return v;
}
// The power of two that brings a query's largest element under 2^12, where the low parts stay normal numbers
__device__ __forceinline__ int tree_query_scale(float most)
{
    int ex = 0;
    if (most > 0.f && most < INFINITY) frexpf(most, &ex); // most < 2^ex
    return min(max(12 - ex, -116), 100);
}
__device__ __forceinline__ void split8(const float (&v)[8], float s, u4v &hi, u4v &lo)
{
    h8 h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = v[e] * s;
        h[e] = static_cast<_Float16>(x);
        l[e] = static_cast<_Float16>(x - static_cast<float>(h[e]));
    }
    hi = __builtin_bit_cast(u4v, h);
    lo = __builtin_bit_cast(u4v, l);
}

// The token of query q of a KV head (query q is head q % G of token q / G); q G < 2^32
__device__ __forceinline__ int tree_token(const TreeAttnArgs &a, int q) { return a.G == 1 ? q : static_cast<int>(__umulhi(static_cast<unsigned>(q), a.inverse)); }

// A workgroup's sequence, KV head, queries and rows.  A sequence's workgroups: ranges times heads, eight at a time, and of each eight the tiles of queries one after the other: workgroups
// that read the same rows are a multiple of eight apart, on one chiplet and at one time, and every chiplet has as many (with tiles that only some sequences have as a dimension of the
// grid some had more than compute units: 156 us instead of 104 for eight sequences of up to 40 fp32 tokens behind 4000 rows).
struct TreeWork {
    int b, past, tok0, n_tok, kvh, q_tile, tiles, range, ranges, row0, row1, rec0;
};
__device__ __forceinline__ TreeWork tree_work(const TreeAttnArgs &a, int lane)
{
    TreeWork w;
    int at = 0;
    w.b = 0;
    if (a.p.n_seqs > 1) {
        const int end = lane < a.p.n_seqs ? arg_int<offsetof(TreeAttnArgs, work0)>(lane + 1) : INT32_MAX;
        at = __builtin_popcountll(__ballot(end <= static_cast<int>(blockIdx.x)));
        w.b = arg_int<offsetof(TreeAttnArgs, order)>(at);
    }
    const int work0 = arg_int<offsetof(TreeAttnArgs, work0)>(at), n = arg_int<offsetof(TreeAttnArgs, work0)>(at + 1) - work0;
    w.ranges = arg_int<offsetof(TreeAttnArgs, ranges)>(w.b);
    w.past = arg_int<offsetof(TreeAttnArgs, p.n_past)>(w.b);
    w.tok0 = arg_int<offsetof(TreeAttnArgs, p.tok0)>(w.b);
    w.n_tok = arg_int<offsetof(TreeAttnArgs, p.tok0)>(w.b + 1) - w.tok0;
    w.rec0 = arg_int<offsetof(TreeAttnArgs, rec0)>(w.b);
    const int each = arg_int<offsetof(TreeAttnArgs, range_rows)>(w.b), Hkv = a.p.Hkv, units = w.ranges * Hkv;
    int unit = blockIdx.x - work0;
    w.q_tile = 0;
    w.tiles = 1;
    if (n > units) {
        w.tiles = n / units;
        const int eight = unit / (8 * w.tiles), in = unit - eight * 8 * w.tiles, of = min(8, units - 8 * eight);
        w.q_tile = of == 8 ? in >> 3 : in / of;
        unit = 8 * eight + in - w.q_tile * of;
    }
    w.range = (Hkv & (Hkv - 1)) == 0 ? unit >> __builtin_ctz(Hkv) : unit / Hkv;
    w.kvh = unit - w.range * Hkv;
    w.row0 = w.range * each;
    w.row1 = w.row0 + min(each, w.past + w.n_tok - w.row0); // (the last range's end need not be a 32-bit number)
    return w;
}

// Columns d .. d + 3 of query q of the sequence's on the head, as numerators under 2^mx, with their denominator: to the output, or to the range's record
template <class TA, int D>
__device__ __forceinline__ void tree_put(const TreeAttnArgs &a, const TreeWork &w, int kvh, int q, int d, float mx, float sum, f4v v)
{
    const int t = tree_token(a, q), h = kvh * a.G + q - t * a.G;
    if (w.ranges == 1) {
        const float r = sum == 0.f ? 0.f : 1.f / sum;
        typedef TA TA4 __attribute__((ext_vector_type(4)));
        TA4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = static_cast<TA>(sum == 0.f ? 0.f : v[e] * r);
        *reinterpret_cast<TA4 *>(static_cast<TA *>(a.o) + static_cast<int64_t>(w.tok0 + t) * a.ldo + h * D + d) = o;
        return;
    }
    float *rec = a.part + (static_cast<int64_t>(w.rec0) * a.Hq + (static_cast<int64_t>(t) * a.Hq + h) * w.ranges + w.range) * (TREE_REC + D);
    if (d == 0) *reinterpret_cast<float2 *>(rec) = make_float2(mx, sum);
    *reinterpret_cast<f4v *>(rec + TREE_REC + d) = v;
}

// A sequence's row of the table, through the scalar cache (nothing writes it while the kernel runs), its entry for a group of eight rows (requested early, looked at late), and what
// page that is (-1: none)
typedef const __attribute__((address_space(4))) int32_t TreeTable;
__device__ __forceinline__ TreeTable *tree_table(const TreeAttnArgs &a, int b) { return (TreeTable *)(a.p.table + static_cast<int64_t>(b) * a.p.table_stride); }
__device__ __forceinline__ int tree_entry(const TreeAttnArgs &a, TreeTable *table, int row, int row1) { return table[min(row, row1 - 1) >> a.p.page_shift]; }
__device__ __forceinline__ int tree_page(const TreeAttnArgs &a, int entry, int row, int row1)
{
    return row < row1 && static_cast<unsigned>(entry) < static_cast<unsigned>(a.p.n_pages) ? entry : -1;
}

// row r of a head; null: it has no page
__device__ __forceinline__ const uint16_t *tree_row(const TreeAttnArgs &a, const uint16_t *pool, TreeTable *table, int kvh, int r)
{
    const int id = table[r >> a.p.page_shift];
    if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.p.n_pages)) return nullptr;
    return pool + kvh * a.p.head_stride + id * a.p.page_stride + (r & ((1 << a.p.page_shift) - 1)) * a.p.row_stride;
}

template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// In each group of 16 lanes, lane i names four consecutive 16-bit numbers and receives, of those named by lanes i / 4 + 4 r, the one at position i % 4.
__device__ __forceinline__ s4v read_transposed(unsigned lds_at)
{
    typedef __attribute__((address_space(3))) s4v Quad;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((Quad *)(static_cast<uintptr_t>(lds_at)));
}

// Where a row's 16-byte chunks lie in LDS: chunk c at c xor swizzle, so that 256 bytes read at once meet in no bank: of K (sixteen rows, one chunk), and of V by
// the transposing reads (four rows and four chunks for blocks of 32 queries, eight rows and two chunks for 16).
template <int D>
__device__ __forceinline__ int swizzle_k(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
template <int D>
__device__ __forceinline__ int swizzle_v32(int row) { return D == 128 ? 4 * (row & 3) : 2 * row & 4; }
template <int D>
__device__ __forceinline__ int swizzle_v16(int row) { return D == 128 ? 2 * (row & 7) : row & 6; }

// 16 bytes a lane from a wave-uniform base plus the lane's byte offset straight into LDS (dma16 with a scalar base)
template <bool NT>
__device__ __forceinline__ void dma16_at(const void *uniform, unsigned lane_offset, uint32_t lds_addr)
{
    const uint64_t u = reinterpret_cast<uintptr_t>(uniform); // (said to be in scalar registers once more, wherever the compiler has it)
    const uint64_t base = static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(u >> 32)))) << 32 |
                          static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(u)));
    if (NT) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" : : "v"(lane_offset), "s"(base), "s"(lds_addr) : "memory");
    else asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(lane_offset), "s"(base), "s"(lds_addr) : "memory");
}

// ---- more queries: bound by the matrix cores and the exponentials ----
// Eight waves: NR blocks of 32 queries, and 8 / NR waves that take different rows of a tile for the same queries.  All waves bring a part of each tile, two tiles
// ahead.  A wave alternates between products (the outputs of one tile, then the scores of the next) and exponentials; waves 0..3 and 4..7, which share the
// SIMDs in pairs, are half a tile apart, so that one's products run beside the other's exponentials.  A barrier ends each half.  (Left to drift with one barrier a
// tile they take turns worse: 119 us against 108.)  A half of 64 rows and 256 queries takes 1740 cycles: 1024 of the matrix cores, 1024 of reads from LDS beside them (products
// alone 1500), the other four waves' exponentials 1340; the card's power holds the clock at 2.04 GHz meanwhile.
template <class A, class C, int D, int NR>
__global__ void __launch_bounds__(512, 2) tree_wide_kernel(TreeAttnArgs a)
{
    typedef TreeShape<D, NR> Shape;
    typedef typename A::type TA;
    constexpr bool SPLIT = __is_same(A, F32);
    constexpr int NK = Shape::NK, BLOCKS = Shape::BLOCKS, ROWS = Shape::ROWS, SLOTS = Shape::SLOTS, TILE = Shape::TILE;
    constexpr int STEPS = D / 16, DB = D / 32, CH = D / 8; // CH: 16-byte chunks of a row
    constexpr int RPI = 64 / CH, MINE = ROWS / 8, NI = MINE / RPI, GROUPS = MINE / 8; // rows of a request, rows and requests of a wave, its groups of eight rows
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ __align__(8) uint8_t notes[4][8]; // by tile % 4 and wave: its groups without a page
    __shared__ int odd_rows;                     // there are drafted rows with infinities or NaN
    request_args<sizeof(a)>();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int G = a.G;
    const TreeWork w = tree_work(a, lane);
    const int kvh = w.kvh, past = w.past, row0 = w.row0, row1 = w.row1, q_first = w.q_tile * a.tile_q, n_q = min(w.n_tok * G, q_first + a.tile_q);
    const int n_tiles = (row1 - row0 + ROWS - 1) / ROWS, plain = min(past, row1); // plain: rows in front of it are cached ones of this range
    const int wr = wave % NR, wk = wave / NR;
    const bool idle = q_first + 32 * wr >= n_q; // only brings rows for the others (eight sequences of 20 bf16 tokens of 64 / 8 heads behind 6000 rows 61.0 -> 52.3 us)

    // ---- pages: the table's entries of the first tiles, then the queries, are requested before anything is waited for ----
    const int first_row = row0 + wave * MINE;
    TreeTable *const table = tree_table(a, w.b);
    struct Entries { int id[GROUPS]; };
    auto look_up = [&](int i) __attribute__((always_inline)) { // of the wave's groups of eight rows of tile i
        Entries r;
#pragma unroll
        for (int y = 0; y < GROUPS; ++y) r.id[y] = tree_entry(a, table, first_row + ROWS * i + 8 * y, row1);
        return r;
    };
    const Entries entries0 = look_up(0), entries1 = look_up(1), entries2 = look_up(2);

    // ---- queries: lane (col, half) holds elements 16 x + 8 half .. + 7 of its query ----
    const int qi = q_first + 32 * wr + col;
    const bool q_ok = qi < n_q;
    const int q_t = q_ok ? tree_token(a, qi) : 0, q_h = kvh * G + (q_ok ? qi - q_t * G : 0);
    u4v qh[STEPS], ql[SPLIT ? STEPS : 1];
    float qv[SPLIT ? STEPS : 1][8];
    {
        const TA *qp = static_cast<const TA *>(a.q) + static_cast<int64_t>(w.tok0 + q_t) * a.ldq + q_h * D + 8 * half;
#pragma unroll
        for (int x = 0; x < STEPS; ++x) {
            if constexpr (SPLIT) A::load8(qp + 16 * x, qv[x]);
            else qh[x] = *reinterpret_cast<const u4v *>(qp + 16 * x);
        }
    }
    uint64_t bits = ~0ull >> (63 - q_t); // drafted rows the query sees
    if (a.p.tree) bits = a.p.tree[w.tok0 + q_t];
    bool hole = false;
    for (int e = (row0 >> a.p.page_shift) + threadIdx.x; e <= (row1 - 1) >> a.p.page_shift; e += 512)
        hole |= static_cast<unsigned>(a.p.table[static_cast<int64_t>(w.b) * a.p.table_stride + e]) >= static_cast<unsigned>(a.p.n_pages);
    const bool holes = __builtin_amdgcn_readfirstlane(__syncthreads_or(hole)) != 0;

    // ---- this wave's part of a tile into LDS: 1 KiB, RPI rows, a request ----
    // Where the wave's groups of a tile lie in the pool, in elements; bad: bits of those that have no page (then at the same rows of page 0)
    const int page_mask = (1 << a.p.page_shift) - 1;
    struct Place { int64_t at[GROUPS]; int bad; };
    auto place = [&](int i, const Entries &entries) __attribute__((always_inline)) {
        Place r;
        r.bad = 0;
#pragma unroll
        for (int y = 0; y < GROUPS; ++y) {
            const int row = first_row + ROWS * i + 8 * y, id = tree_page(a, entries.id[y], row, row1);
            r.at[y] = max(id, 0) * a.p.page_stride + static_cast<int64_t>(row & page_mask) * a.p.row_stride;
            if (holes) r.bad |= (id < 0) << y;
        }
        return r;
    };
    uint16_t *const ring = reinterpret_cast<uint16_t *>(smem); // [K, V][SLOTS][ROWS][D]
    const int in_row = lane / CH, in_chunk = lane % CH;
    const uint16_t *const Kh = a.p.K + kvh * a.p.head_stride, *const Vh = a.p.V + kvh * a.p.head_stride;
    // a lane's byte offsets from a request's first row; V's are the same for all requests
    unsigned k_lane[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) k_lane[j] = 2 * (in_row * static_cast<int>(a.p.row_stride) + 8 * (in_chunk ^ swizzle_k<D>(wave * MINE + RPI * j + in_row)));
    const unsigned v_lane = 2 * (in_row * static_cast<int>(a.p.row_stride) + 8 * (in_chunk ^ swizzle_v32<D>(in_row)));
    auto request = [&](int slot, const Place &pl, int which) __attribute__((always_inline)) {
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address(ring + (SLOTS * which + slot) * TILE + wave * MINE * D));
#pragma unroll
        for (int j = 0; j < NI; ++j) dma16_at<false>((which ? Vh : Kh) + pl.at[RPI * j / 8] + RPI * j % 8 * a.p.row_stride, which ? v_lane : k_lane[j], to + 2 * RPI * j * D);
    };
    // Rows without a page are rare: only a range that has some (holes) keeps notes of them, for everybody, of this wave's groups
    auto note_absent = [&](int i, const Place &pl) __attribute__((always_inline)) {
        if (holes && lane == 0) notes[i & 3][wave] = static_cast<uint8_t>(pl.bad);
    };
    // V of tile i, this wave's part, is in LDS: rows that nobody sees are zeroed, and so are infinities and NaN of drafted rows, which are added in the end
    auto mend_v = [&](int i, int slot) __attribute__((always_inline)) {
        const int tile = row0 + ROWS * i;
        if (tile + ROWS <= plain && !holes) return;
        const int bad = holes ? __builtin_amdgcn_readfirstlane(notes[i & 3][wave]) : 0;
        uint16_t *const Vw = ring + (SLOTS + slot) * TILE;
        bool odd = false;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int r = wave * MINE + RPI * j + in_row;
            u4v *at = reinterpret_cast<u4v *>(Vw + r * D + 8 * in_chunk);
            if (tile + r >= row1 || (bad >> (RPI * j >> 3) & 1)) *at = u4v{0, 0, 0, 0};
            else if (tile + r >= past && odd8<C>(*at)) {
                *at = without_odd<C>(*at);
                odd = true;
            }
        }
        if (odd) odd_rows = 1;
    };
    if (threadIdx.x == 0) odd_rows = 0;
    // Issued so far and from here on: K of tiles up to k + SLOTS - 1 and V up to k + SLOTS - 2 when tile k's scores are about to be formed
    Place next; // of the next tile whose V is to be requested
    {
        const Place p0 = place(0, entries0);
        next = place(1, entries1);
        request(0, p0, 0);
        request(0, p0, 1);
        note_absent(0, p0);
        if (n_tiles > 1) {
            request(1, next, 0);
            note_absent(1, next);
            if (SLOTS == 3) request(1, next, 1);
        }
        if (SLOTS == 3) {
            next = place(2, entries2);
            if (n_tiles > 2) {
                request(2, next, 0);
                note_absent(2, next);
            }
        }
    }
    Entries behind = SLOTS == 3 ? look_up(3) : entries2; // of tile k + SLOTS
    if (!q_ok) bits = 0;
    bits &= ~0ull >> (64 - w.n_tok);

    float f = a.scale;
    if constexpr (SPLIT) {
        float most = 0.f;
#pragma unroll
        for (int x = 0; x < STEPS; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(qv[x][e]));
        const int up = tree_query_scale(max_across_32(most));
        const float s = ldexpf(1.f, up);
        f *= ldexpf(1.f, -up);
#pragma unroll
        for (int x = 0; x < STEPS; ++x) split8(qv[x], s, qh[x], ql[x]);
    }

    float m = -INFINITY, mf = 0.f, l = 0.f; // maximum of the scores before f, m f - LIFT (0: there is none yet), this lane's half of the sum
    f16v acc[DB], s[BLOCKS];
#pragma unroll
    for (int x = 0; x < DB; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[x][i] = 0.f;
    u4v ph[BLOCKS][2], pl[BLOCKS][2];

    // where a lane reads: K of row (32-row block) + col; V, transposing, rows 4 half + col % 16 / 4 (+ 8, 16, 24), elements 16 (col / 16) + 4 (col % 4) of
    // every 32 (a lane gets, of four rows, the element at its own place: 16 (col / 16) + col % 16)
    const int vrow = 4 * half + ((lane & 15) >> 2);
    unsigned vat[DB]; // byte offsets in a block
#pragma unroll
    for (int x = 0; x < DB; ++x) {
        const int c = (4 * x + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swizzle_v32<D>(vrow);
        vat[x] = vrow * 2 * D + c * 16 + (lane & 1) * 8;
    }
    auto is_gone = [&](uint64_t note, int group) __attribute__((always_inline)) { return (note >> (8 * (group / GROUPS) + group % GROUPS) & 1) != 0; };

    // Operands are read from LDS AHEAD products before their own (left to itself the compiler reads each right in front of its product and waits for it: 1450
    // cycles for outputs and 1050 for scores of 512 cycles of products each).
    constexpr int AHEAD = 4; // (6 or 8: no faster)
    static_assert(AHEAD <= BLOCKS * STEPS && AHEAD <= BLOCKS * 2 * DB);
    u4v v[AHEAD];
    auto v_operand = [&](int slot, int n) __attribute__((always_inline)) { // 32 columns of 16 rows
        typedef short s8v __attribute__((ext_vector_type(8)));
        const unsigned at = lds_address(ring + (SLOTS + slot) * TILE + wk * BLOCKS * 32 * D) + vat[n % DB] + (n / DB) * 16 * 2 * D;
        return __builtin_bit_cast(u4v, (s8v)__builtin_shufflevector(read_transposed(at), read_transposed(at + 8 * 2 * D), 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto k_operand = [&](int slot, int n) __attribute__((always_inline)) { // 16 columns of 32 rows
        return *reinterpret_cast<const u4v *>(ring + slot * TILE + (wk * BLOCKS * 32 + n % BLOCKS * 32 + col) * D + 8 * ((2 * (n / BLOCKS) + half) ^ swizzle_k<D>(col)));
    };
    // ---- outputs of the tile in `slot`, transposed: register e of acc[x] is column 32 x + 8 (e / 4) + 4 half + e % 4 of the query's; behind them the first
    // operands of the scores of the next one (if there is none: of what lies there, for nothing) ----
    auto outputs = [&](int slot, int slot1) __attribute__((always_inline)) {
        constexpr int N = BLOCKS * 2 * DB;
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) v[n] = v_operand(slot, n);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            __builtin_amdgcn_sched_barrier(0);
            acc[n % DB] = tree_mfma<C>(v[n % AHEAD], ph[n / DB / 2][n / DB % 2], acc[n % DB]);
            if constexpr (SPLIT) acc[n % DB] = tree_mfma<C>(v[n % AHEAD], pl[n / DB / 2][n / DB % 2], acc[n % DB]);
            v[n % AHEAD] = n + AHEAD < N ? v_operand(slot, n + AHEAD) : k_operand(slot1, n + AHEAD - N);
        }
    };
    // ---- scores of the tile in `slot`: register e of s[k] is row 8 (e / 4) + 4 half + e % 4 of the block; operand n is in v[(n + FIRST) % AHEAD] ----
    auto scores = [&](int slot, auto first) __attribute__((always_inline)) {
        constexpr int FIRST = decltype(first)::value, N = STEPS * BLOCKS;
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[k][e] = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            u4v &op = v[(n + FIRST) % AHEAD];
            __builtin_amdgcn_sched_barrier(0);
            s[n % BLOCKS] = tree_mfma<C>(op, qh[n / BLOCKS], s[n % BLOCKS]);
            if constexpr (SPLIT) s[n % BLOCKS] = tree_mfma<C>(op, ql[n / BLOCKS], s[n % BLOCKS]);
            if (n + AHEAD < N) op = k_operand(slot, n + AHEAD);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // ---- probabilities of tile i ----
    auto probabilities = [&](int i) __attribute__((always_inline)) {
        const int tile = row0 + ROWS * i;
        const bool special = tile + ROWS > plain || holes;
        const uint64_t note = holes ? *reinterpret_cast<const uint64_t *>(notes[i & 3]) : 0; // wave v's from bit 8 v on
        uint32_t sees[BLOCKS]; // rows of the block that the query sees
        if (special) {
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k) {
                const int first = tile + 32 * (wk * BLOCKS + k), d = first - past; // d: drafted index of the block's first row
                uint32_t rows = row1 >= first + 32 ? 0xffffffffu : (row1 <= first ? 0u : (1u << (row1 - first)) - 1);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    if (is_gone(note, (wk * BLOCKS + k) * 4 + y)) rows &= ~(0xffu << 8 * y);
                const uint32_t cached = d >= 0 ? 0u : (d <= -32 ? 0xffffffffu : (1u << -d) - 1);
                const uint32_t draft = d >= 64 ? 0u : (d >= 0 ? static_cast<uint32_t>(bits >> d) : (d <= -32 ? 0u : static_cast<uint32_t>(bits << -d)));
                sees[k] = (cached | draft) & rows;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[k][e] = sees[k] >> (8 * (e / 4) + e % 4 + 4 * half) & 1 ? s[k][e] : -INFINITY;
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[k][e]);
        top = max_across_32(top);
        // (nothing to see yet: mf is 0 and the first score there is moves it, whatever it is)
        if (__ballot(m == -INFINITY ? top > m : fmaf(top, f, -mf) > TreeRange<C>::LIFT + TreeRange<C>::DEFER) != 0) {
            const float mn = fmaxf(m, top), mnf = mn == -INFINITY ? 0.f : fmaf(mn, f, -TreeRange<C>::LIFT);
            const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mf - mnf); // (nothing so far: the sums are 0)
            l *= corr;
#pragma unroll
            for (int x = 0; x < DB; ++x) acc[x] *= corr;
            m = mn;
            mf = mnf;
        }
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[k][e] = __builtin_amdgcn_exp2f(fmaf(s[k][e], f, -mf));
        if (special) {
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[k][e] = sees[k] >> (8 * (e / 4) + e % 4 + 4 * half) & 1 ? s[k][e] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) {
#pragma unroll
            for (int e = 0; e < 16; ++e) l += s[k][e];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                // 16-bit queries: probabilities rounded to the cache's type, as the output is in the end: its error against 64 bits is 1.4 times that of the output's rounding alone
                // (2.34e-3 of the rms instead of 1.66e-3 in bf16, 2.9e-4 instead of 2.1e-4 in f16).  Two numbers, as with fp32 queries, leave that alone but are half as many
                // products again: 8 x 63 bf16 tokens behind 6000 rows 99 -> 127 us, 8 x 20 51 -> 62.
                if constexpr (__is_same(C, BF16)) {
                    b8 hi;
#pragma unroll
                    for (int e = 0; e < 8; ++e) hi[e] = static_cast<__bf16>(s[k][8 * y + e]);
                    ph[k][y] = __builtin_bit_cast(u4v, hi);
                } else {
                    h8 hi, lo;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        hi[e] = static_cast<_Float16>(s[k][8 * y + e]);
                        if constexpr (SPLIT) lo[e] = static_cast<_Float16>(s[k][8 * y + e] - static_cast<float>(hi[e]));
                    }
                    ph[k][y] = __builtin_bit_cast(u4v, hi);
                    if constexpr (SPLIT) pl[k][y] = __builtin_bit_cast(u4v, lo);
                }
            }
        }
    };
    // What has to be there at the end of half 2 k + 1: K of tile k + 1 and V of tile k, this wave's parts
    auto arrived = [&](int k, int slot) __attribute__((always_inline)) {
        if constexpr (SLOTS == 3) {
            if (k + 2 < n_tiles) wait_loads<2 * NI>();
            else if (k + 1 < n_tiles) wait_loads<NI>();
            else wait_loads<0>();
        } else wait_loads<0>();
        mend_v(k, slot);
    };

    // ---- Halves 2 k and 2 k + 1, with a barrier behind each: for waves 0..3 products (outputs of tile k - 1, scores of tile k) and exponentials of tile k, for waves
    // 4..7, one barrier behind, exponentials of tile k - 1 and products. ----
    const int late = wave >> 2;
    // K of tile 0 (oldest) has to be there; V of tile 0 and what follows it may be on its way
    if constexpr (SLOTS == 3) {
        if (n_tiles > 2) wait_loads<4 * NI>();
        else if (n_tiles > 1) wait_loads<3 * NI>();
        else wait_loads<NI>();
    } else {
        if (n_tiles > 1) wait_loads<2 * NI>();
        else wait_loads<NI>();
    }
    __syncthreads();
    auto slot_of = [&](int slot, int d) __attribute__((always_inline)) { return slot + d >= SLOTS ? slot + d - SLOTS : slot + d; };
    // In half 2 k (waves 4..7) or 2 k + 1, k > 0, slot: of tile k.  Places that everybody has left: K of tile k - 1, V of tile k - 2
    auto refill = [&](int k, int slot) __attribute__((always_inline)) {
        if (k + SLOTS - 2 < n_tiles) request(slot_of(slot, SLOTS - 2), next, 1);
        if (k + SLOTS - 1 < n_tiles) {
            next = place(k + SLOTS - 1, behind);
            request(slot_of(slot, SLOTS - 1), next, 0);
            note_absent(k + SLOTS - 1, next);
        }
        behind = look_up(k + SLOTS);
    };
    if (late) __syncthreads();
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) v[n] = k_operand(0, n);
    if (!idle) scores(0, std::integral_constant<int, 0>());
    if (late) arrived(0, 0);
    __syncthreads();
    for (int k = 0, slot = 0; k < n_tiles; ++k) {
        const int slot1 = slot_of(slot, 1);
        if (late || k > 0) refill(k + late, late ? slot1 : slot); // (in front of the exponentials either way: the products' half is the longer one)
        if (!idle) probabilities(k);
        if (!late) arrived(k, slot);
        __syncthreads();
        __builtin_amdgcn_s_setprio(1);
        if (!idle) outputs(slot, slot1);
        if (k + 1 < n_tiles) {
            if (!idle) scores(slot1, std::integral_constant<int, BLOCKS * 2 * DB % AHEAD>());
            __builtin_amdgcn_s_setprio(0);
            if (late) arrived(k + 1, slot1);
        }
        __syncthreads();
        slot = slot1;
    }
    if (!late) __syncthreads();
    l = add_across_32(l);
    if (m == -INFINITY) mf = -INFINITY;
    if (odd_rows) { // infinities and NaN of drafted rows, out of memory, to the sums of the queries that see them
        for (int r = max(past, row0); r < row1; ++r) {
            if ((r - row0) % ROWS / (32 * BLOCKS) != wk || !(bits >> (r - past) & 1)) continue; // (another wave's row)
            const uint16_t *v = tree_row(a, a.p.V, table, kvh, r);
            if (!v) continue;
            for (int x = 0; x < DB; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const unsigned u = v[32 * x + 8 * (e / 4) + 4 * half + e % 4];
                    const float add = odd16<C>(u) ? widen16<C>(u) : 0.f;
#pragma unroll
                    for (int y = 0; y < DB; ++y)
                        if (y == x) acc[y][e] += add;
                }
        }
    }
    if constexpr (NK == 1) {
        if (q_ok)
#pragma unroll
            for (int x = 0; x < DB; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    tree_put<TA, D>(a, w, kvh, qi, 32 * x + 8 * y + 4 * half, mf, l, f4v{acc[x][4 * y], acc[x][4 * y + 1], acc[x][4 * y + 2], acc[x][4 * y + 3]});
    } else {
        // the waves that share queries meet in LDS
        constexpr int LD = D + 4;
        float *os = reinterpret_cast<float *>(smem), *ms = os + 8 * 32 * LD, *ls = ms + 8 * 32; // [wave][32][LD], [wave][32]
        __syncthreads();
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y)
                *reinterpret_cast<f4v *>(os + (wave * 32 + col) * LD + 32 * x + 8 * y + 4 * half) = f4v{acc[x][4 * y], acc[x][4 * y + 1], acc[x][4 * y + 2], acc[x][4 * y + 3]};
        if (half == 0) {
            ms[wave * 32 + col] = mf;
            ls[wave * 32 + col] = l;
        }
        __syncthreads();
        const int n = n_q - q_first;
        for (int idx = threadIdx.x; idx < n * (D / 4); idx += 512) {
            const int i = idx / (D / 4), d = (idx - i * (D / 4)) * 4;
            float mx = -INFINITY, sum = 0.f;
            f4v v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NK; ++k) mx = fmaxf(mx, ms[32 * NR * k + i]);
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const int at = 32 * NR * k + i;
                const float e = ms[at] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms[at] - mx);
                sum += ls[at] * e;
                v += *reinterpret_cast<const f4v *>(os + at * LD + d) * e;
            }
            tree_put<TA, D>(a, w, kvh, q_first + i, d, mx, sum, v);
        }
    }
}

// ---- up to 64 queries on a KV head: bound by the stream of rows ----
// Four waves, each with tiles of 16 rows of its own (rows 16 w + 64 i of the range), NQ blocks of 16 queries; no barrier before the end.  K and V of a tile are
// requested apart, each two tiles ahead into the place its predecessor but one has left, so that three of the four are always on their way.
template <class A, int D, int NQ>
struct TreeNarrow {
    static constexpr int TILE = 16 * D;                       // elements of K (V) in a tile
    static constexpr size_t RING = 4 * 4 * TILE * 2;          // [wave][K, K, V, V][16][D]
    static constexpr size_t QUERIES = 16 * NQ * D * sizeof(typename A::type);
    static constexpr size_t JOIN = 4 * 16 * NQ * (D + 4) * 4 + 2 * 4 * 16 * NQ * 4;
    static constexpr size_t LDS = RING + QUERIES > JOIN ? RING + QUERIES : JOIN;
};

template <class C>
__device__ __forceinline__ f4v tree_mfma16(u4v a, u4v b, f4v c)
{
    if constexpr (__is_same(C, BF16)) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
template <class C>
__device__ __forceinline__ f4v tree_mfma16_half(s4v a, s4v b, f4v c)
{
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    if constexpr (__is_same(C, BF16)) return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(h4, a), __builtin_bit_cast(h4, b), c, 0, 0, 0);
}

// Probabilities as two numbers of type C, whatever the queries' type: the stream of rows hides the second product (us, rounded once / in two: 16 sequences of one f16 token behind 4100 rows
// 44.2 / 44.7, one behind 30001 26.4 / 26.9, 36 of 4 bf16 tokens behind 3000 72.3 / 74.9).  The first is cut off, not rounded, and the second is above zero where the probability is: an
// infinity in V then stays one.
template <class C>
__device__ __forceinline__ void split_probabilities(const float (&p)[4], s4v &hi, s4v &lo)
{
    typedef typename C::type C4 __attribute__((ext_vector_type(4)));
    C4 l;
    if constexpr (__is_same(C, BF16)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const unsigned cut = __builtin_bit_cast(unsigned, p[r]) & 0xffff0000u;
            hi[r] = static_cast<short>(cut >> 16);
            l[r] = static_cast<__bf16>(fmaxf(p[r] - __builtin_bit_cast(float, cut), p[r] * 0x1p-24f));
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            typedef short s2v __attribute__((ext_vector_type(2)));
            const auto cut = __builtin_amdgcn_cvt_pkrtz(p[r], p[r + 1]);
            const s2v bits = __builtin_bit_cast(s2v, cut); // (of the pair: the compiler takes the first for either of its elements)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                hi[r + e] = bits[e];
                l[r + e] = static_cast<_Float16>(__builtin_amdgcn_fmed3f(p[r + e] - static_cast<float>(cut[e]), 0x1p-24f, p[r + e])); // (2^-24: the least binary16 number)
            }
        }
    }
    lo = __builtin_bit_cast(s4v, l);
}

template <class A, class C, int D, int NQ>
__global__ void __launch_bounds__(256, 2) tree_narrow_kernel(TreeAttnArgs a)
{
    typedef typename A::type TA;
    constexpr bool SPLIT = __is_same(A, F32);
    constexpr int STEPS = D / 32, DB = D / 16, CH = D / 8, RPI = 64 / CH, NI = 16 / RPI, TILE = 16 * D; // NI: requests for K (V) of a tile
    extern __shared__ __align__(16) uint8_t smem[];
    request_args<sizeof(a)>();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    const int G = a.G;
    const TreeWork wk = tree_work(a, lane);
    const int kvh = wk.kvh;
    const int past = wk.past, n_tok = wk.n_tok, tok0 = wk.tok0, n_q = n_tok * G, row1 = wk.row1;
    const int n_tiles = (row1 - wk.row0 - 16 * wave + 63) >> 6; // of this wave (below 1: none)
    const int q_first = wk.q_tile * 16 * NQ;
    const bool shared = wk.tiles > 1; // others read the rows too

    // ---- pages of the wave's tiles (two times eight rows): the table's entries of the first, then the queries, are requested before anything is waited for ----
    TreeTable *const table = tree_table(a, wk.b);
    const int first_row = wk.row0 + 16 * wave;
    struct Entries { int id[2]; };
    auto look_up = [&](int i) __attribute__((always_inline)) { // of tile i
        Entries r;
#pragma unroll
        for (int y = 0; y < 2; ++y) r.id[y] = tree_entry(a, table, first_row + 64 * i + 8 * y, row1);
        return r;
    };
    auto pages_of = [&](int i, const Entries &entries) __attribute__((always_inline)) { // -1: there is none
        Entries r;
#pragma unroll
        for (int y = 0; y < 2; ++y) r.id[y] = tree_page(a, entries.id[y], first_row + 64 * i + 8 * y, row1);
        return r;
    };
    const Entries entries0 = look_up(0), entries1 = look_up(1);
    Entries behind = look_up(2); // of tile i + 2

    // ---- queries: brought once for the four waves, 1 KiB at a time, chunk c of query q at c xor the low bits of q (each wave reading them from memory by itself in
    // the products' order took 5800 cycles for 32 fp32 queries: 16-byte pieces of 16 rows, four times) ----
    constexpr int QCH = D * static_cast<int>(sizeof(TA)) / 16, QI = 16 * NQ * QCH / 64 / 4; // chunks of a query, a wave's requests
    uint8_t *const qs = smem + TreeNarrow<A, D, NQ>::RING;
    uint64_t bits[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int qi = q_first + 16 * n + col, t = qi < n_q ? tree_token(a, qi) : 0;
        bits[n] = ~0ull >> (63 - t);
        if (a.p.tree) bits[n] = a.p.tree[tok0 + t];
    }
    static_assert(QI >= 1 || QCH * 16 * NQ == 128);
    if (QI >= 1 || wave < 2) {
#pragma unroll
        for (int j = 0; j < (QI >= 1 ? QI : 1); ++j) {
            const int at = (wave * (QI >= 1 ? QI : 1) + j) * 64 + lane, q = at / QCH, c = at % QCH ^ (q & (QCH < 16 ? 7 : 15));
            const int qi = min(q_first + q, n_q - 1), t = tree_token(a, qi);
            const TA *src = static_cast<const TA *>(a.q) + static_cast<int64_t>(tok0 + t) * a.ldq + (kvh * G + qi - t * G) * D;
            dma16<false>(reinterpret_cast<const uint8_t *>(src) + 16 * c, __builtin_amdgcn_readfirstlane(lds_address(qs) + (at - lane) * 16));
        }
    }

    // ---- what a wave requests: 1 KiB, RPI rows, at a time ----
    const int in_row = lane / CH, in_chunk = lane % CH, page_mask = (1 << a.p.page_shift) - 1;
    uint16_t *const ring = reinterpret_cast<uint16_t *>(smem) + wave * 4 * TILE;
    const uint16_t *const Kh = a.p.K + kvh * a.p.head_stride, *const Vh = a.p.V + kvh * a.p.head_stride;
    unsigned lane_at[2][NI]; // byte offsets from a request's first row
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int row = RPI * j + in_row, at = in_row * static_cast<int>(a.p.row_stride);
        lane_at[0][j] = 2 * (at + 8 * (in_chunk ^ swizzle_k<D>(row)));
        lane_at[1][j] = 2 * (at + 8 * (in_chunk ^ swizzle_v16<D>(row)));
    }
    // K (which 0) or V of tile i, whose pages are `pg`
    auto request = [&](int i, const Entries &pg, int which) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // what its place held has been read
        const uint32_t to = lds_address(ring + (2 * which + (i & 1)) * TILE);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int r = RPI * j;
            // (rows of an absent page: those of page 0)
            const int64_t at = max(pg.id[r >> 3], 0) * a.p.page_stride + static_cast<int64_t>((first_row + 64 * i + r) & page_mask) * a.p.row_stride;
            if (shared) dma16_at<false>((which ? Vh : Kh) + at, lane_at[which][j], __builtin_amdgcn_readfirstlane(to + 2 * r * D));
            else dma16_at<true>((which ? Vh : Kh) + at, lane_at[which][j], __builtin_amdgcn_readfirstlane(to + 2 * r * D));
        }
    };
    // The queries and the bits are waited for here, about as long as the table: the compiler, which does not know of the requests, would have the bits wait for all
#pragma unroll
    for (int n = 0; n < NQ; ++n) asm volatile("s_waitcnt vmcnt(0)" : "+v"(bits[n]) : : "memory");
    Entries now = pages_of(0, entries0), next = pages_of(1, entries1);
    if (n_tiles > 0) {
        request(0, now, 0);
        request(0, now, 1);
    }
    if (n_tiles > 1) {
        request(1, next, 0);
        request(1, next, 1);
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) bits[n] = q_first + 16 * n + col < n_q ? bits[n] & (~0ull >> (64 - n_tok)) : 0;

    // lane (col, g) holds elements 32 x + 8 g .. + 7 of query 16 n + col
    __syncthreads();
    u4v qh[NQ][STEPS], ql[NQ][SPLIT ? STEPS : 1];
    float f[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const uint8_t *const q = qs + (16 * n + col) * QCH * 16;
        f[n] = a.scale;
        if constexpr (SPLIT) {
            float v[STEPS][8], most = 0.f;
#pragma unroll
            for (int x = 0; x < STEPS; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const f4v part = *reinterpret_cast<const f4v *>(q + 16 * ((8 * x + 2 * g + y) ^ col));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[x][4 * y + e] = part[e];
                        most = fmaxf(most, fabsf(part[e]));
                    }
                }
            const int up = tree_query_scale(max_across_32(max_across_16(most)));
            const float s = ldexpf(1.f, up);
            f[n] *= ldexpf(1.f, -up);
#pragma unroll
            for (int x = 0; x < STEPS; ++x) split8(v[x], s, qh[n][x], ql[n][x]);
        } else {
#pragma unroll
            for (int x = 0; x < STEPS; ++x) qh[n][x] = *reinterpret_cast<const u4v *>(q + 16 * ((4 * x + g) ^ (col & (QCH < 16 ? 7 : 15))));
        }
    }

    bool odd = false; // this lane has met infinities or NaN in drafted rows
    float m[NQ], mf[NQ], l[NQ]; // maximum of the scores before f, m f - LIFT (0: there is none yet), this lane's quarter of the sum
    f4v acc[NQ][DB];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = -INFINITY;
        mf[n] = l[n] = 0.f;
#pragma unroll
        for (int x = 0; x < DB; ++x) acc[n][x] = f4v{0.f, 0.f, 0.f, 0.f};
    }
    // transposing reads of V: rows 4 g + col / 4, elements 4 (col % 4) of every 16 (a lane gets, of four rows, the element at its own column)
    const int vrow = 4 * g + (col >> 2);

    for (int i = 0; i < n_tiles; ++i) {
        const int tile = first_row + 64 * i;
        const bool special = tile + 16 > past || now.id[0] < 0 || now.id[1] < 0;
        if (i + 1 < n_tiles) wait_loads<3 * NI>();
        else wait_loads<NI>();
        const uint16_t *const Kt = ring + (i & 1) * TILE;
        uint16_t *const Vt = ring + (2 + (i & 1)) * TILE;
        // ---- scores: register r is row 4 g + r ----
        f4v s[NQ];
        u4v kv[STEPS];
#pragma unroll
        for (int x = 0; x < STEPS; ++x) kv[x] = *reinterpret_cast<const u4v *>(Kt + col * D + 8 * ((4 * x + g) ^ swizzle_k<D>(col)));
        __builtin_amdgcn_sched_barrier(0); // (all reads before the first product)
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < STEPS; ++x)
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                s[n] = tree_mfma16<C>(kv[x], qh[n][x], s[n]);
                if constexpr (SPLIT) s[n] = tree_mfma16<C>(kv[x], ql[n][x], s[n]);
            }
        const Entries after = pages_of(i + 2, behind);
        if (i + 2 < n_tiles) request(i + 2, after, 0);
        uint32_t rows = 0xffffu; // of the tile that exist
        uint32_t sees[NQ];
        if (special) {
            rows = row1 >= tile + 16 ? 0xffffu : (1u << (row1 - tile)) - 1;
            if (now.id[0] < 0) rows &= 0xff00u;
            if (now.id[1] < 0) rows &= 0x00ffu;
            const int d = tile - past; // drafted index of the tile's first row
            const uint32_t cached = d >= 0 ? 0u : (d <= -16 ? 0xffffu : (1u << -d) - 1);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const uint32_t draft = d >= 64 ? 0u : (d >= 0 ? static_cast<uint32_t>(bits[n] >> d) : (d <= -16 ? 0u : static_cast<uint32_t>(bits[n] << -d)));
                sees[n] = (cached | draft) & rows;
#pragma unroll
                for (int r = 0; r < 4; ++r) s[n][r] = sees[n] >> (4 * g + r) & 1 ? s[n][r] : -INFINITY;
            }
        }
        s4v ph[NQ], pl[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const float top = max_across_32(max_across_16(fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3]))));
            // (nothing to see yet: mf is 0 and the first score there is moves it, whatever it is)
            if (__ballot(m[n] == -INFINITY ? top > m[n] : fmaf(top, f[n], -mf[n]) > TreeRange<C>::LIFT + TreeRange<C>::DEFER) != 0) {
                const float mn = fmaxf(m[n], top), mnf = mn == -INFINITY ? 0.f : fmaf(mn, f[n], -TreeRange<C>::LIFT);
                const float corr = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mf[n] - mnf); // (nothing so far: the sums are 0)
                l[n] *= corr;
#pragma unroll
                for (int x = 0; x < DB; ++x) acc[n][x] *= corr;
                m[n] = mn;
                mf[n] = mnf;
            }
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], f[n], -mf[n]));
                if (special) p[r] = sees[n] >> (4 * g + r) & 1 ? p[r] : 0.f;
                l[n] += p[r];
            }
            split_probabilities<C>(p, ph[n], pl[n]);
        }
        if (i + 2 < n_tiles) wait_loads<3 * NI>();
        else if (i + 1 < n_tiles) wait_loads<2 * NI>();
        else wait_loads<0>();
        if (special) { // V's rows that nobody sees are zeroed, and so are infinities and NaN of drafted rows, which are added in the end
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int r = RPI * j + in_row;
                u4v *at = reinterpret_cast<u4v *>(Vt + r * D + 8 * in_chunk);
                if (!(rows >> r & 1)) *at = u4v{0, 0, 0, 0};
                else if (tile + r >= past && odd8<C>(*at)) {
                    *at = without_odd<C>(*at);
                    odd = true;
                }
            }
        }
        // ---- outputs, transposed: register e is column 16 x + 4 g + e of the query's ----
        const unsigned vbase = lds_address(Vt) + vrow * 2 * D + (lane & 1) * 8;
        s4v v[DB];
#pragma unroll
        for (int x = 0; x < DB; ++x) v[x] = read_transposed(vbase + ((2 * x + ((lane & 3) >> 1)) ^ swizzle_v16<D>(vrow)) * 16);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                acc[n][x] = tree_mfma16_half<C>(v[x], ph[n], acc[n][x]);
                acc[n][x] = tree_mfma16_half<C>(v[x], pl[n], acc[n][x]);
            }
        if (i + 2 < n_tiles) request(i + 2, after, 1);
        now = next;
        next = after;
        behind = look_up(i + 3);
    }

    if (__ballot(odd) != 0) { // infinities and NaN of this wave's drafted rows, out of memory, to the sums of the queries that see them
        for (int i = 0; i < n_tiles; ++i)
            for (int r = max(past, first_row + 64 * i); r < min(row1, first_row + 64 * i + 16); ++r) {
                const uint16_t *v = tree_row(a, a.p.V, table, kvh, r);
                if (!v) continue;
                for (int x = 0; x < DB; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned u = v[16 * x + 4 * g + e];
#pragma unroll
                        for (int n = 0; n < NQ; ++n) {
                            const float add = odd16<C>(u) && (bits[n] >> (r - past) & 1) ? widen16<C>(u) : 0.f;
#pragma unroll
                            for (int y = 0; y < DB; ++y)
                                if (y == x) acc[n][y][e] += add;
                        }
                    }
            }
    }
    // ---- the waves meet in LDS ----
    constexpr int LD = D + 4, ALL = 4 * NQ * 16;
    float *const os = reinterpret_cast<float *>(smem), *const ms = os + ALL * LD, *const ls = ms + ALL; // [wave][16 NQ][LD], [wave][16 NQ]
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int at = (wave * NQ + n) * 16 + col;
#pragma unroll
        for (int x = 0; x < DB; ++x) *reinterpret_cast<f4v *>(os + at * LD + 16 * x + 4 * g) = acc[n][x];
        const float sum = add_across_32(add_across_16(l[n]));
        if (g == 0) {
            ms[at] = m[n] == -INFINITY ? -INFINITY : mf[n];
            ls[at] = sum;
        }
    }
    __syncthreads();
    const int nq = min(16 * NQ, n_q - q_first);
    for (int idx = threadIdx.x; idx < nq * (D / 4); idx += 256) {
        const int q = idx / (D / 4), d = (idx - q * (D / 4)) * 4;
        float mx = -INFINITY, den = 0.f;
        f4v v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ms[w * 16 * NQ + q]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float mw = ms[w * 16 * NQ + q], e = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mx);
            den += ls[w * 16 * NQ + q] * e;
            v += *reinterpret_cast<const f4v *>(os + (w * 16 * NQ + q) * LD + d) * e;
        }
        tree_put<TA, D>(a, wk, kvh, q_first + q, d, mx, den, v);
    }
}

// The ranges' records of one query joined: a workgroup a query, four columns a thread, 1024 / D ranges at a time, EARLY times that requested at once.
template <class A, int D, int EARLY>
__global__ void __launch_bounds__(256) tree_join_kernel(TreeAttnArgs a)
{
    typedef typename A::type TA;
    constexpr int COLS = D / 4, AT_ONCE = 256 / COLS;
    __shared__ float weight[TREE_MAX_RANGES], most[4], sums[4];
    __shared__ f4v shares[256];
    const int t = blockIdx.y, h = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int b = 0;
    if (a.p.n_seqs > 1) {
        const int end = lane < a.p.n_seqs ? arg_int<offsetof(TreeAttnArgs, p.tok0)>(lane + 1) : INT32_MAX;
        b = __builtin_popcountll(__ballot(end <= t));
    }
    const int ranges = arg_int<offsetof(TreeAttnArgs, ranges)>(b);
    if (ranges == 1) return; // written by the range itself
    const float *rec = a.part + (static_cast<int64_t>(arg_int<offsetof(TreeAttnArgs, rec0)>(b)) * a.Hq +
                                 (static_cast<int64_t>(t - arg_int<offsetof(TreeAttnArgs, p.tok0)>(b)) * a.Hq + h) * ranges) * (TREE_REC + D);
    // the thread's first columns are on their way while the weights are formed
    const int c = threadIdx.x % COLS, r0 = threadIdx.x / COLS;
    f4v early[EARLY];
#pragma unroll
    for (int k = 0; k < EARLY; ++k) early[k] = *reinterpret_cast<const f4v *>(rec + min(r0 + k * AT_ONCE, ranges - 1) * (TREE_REC + D) + TREE_REC + 4 * c);
#pragma unroll
    for (int k = 0; k < EARLY; ++k)
        if (r0 + k * AT_ONCE >= ranges) early[k] = f4v{0.f, 0.f, 0.f, 0.f}; // (the last once more, as nothing)
    const bool mine = static_cast<int>(threadIdx.x) < ranges;
    const float2 ml = mine ? *reinterpret_cast<const float2 *>(rec + threadIdx.x * (TREE_REC + D)) : make_float2(-INFINITY, 0.f);
    const float wm = wave_max(ml.x);
    if (lane == 0) most[wave] = wm;
    __syncthreads();
    const float mx = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
    const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - mx);
    weight[threadIdx.x] = w; // (0 past the last)
    const float ws = wave_sum(ml.y * w);
    if (lane == 0) sums[wave] = ws;
    __syncthreads();
    f4v v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < EARLY; ++k) v += early[k] * weight[r0 + k * AT_ONCE];
#pragma unroll 4
    for (int r = r0 + EARLY * AT_ONCE; r < ranges; r += AT_ONCE) v += *reinterpret_cast<const f4v *>(rec + r * (TREE_REC + D) + TREE_REC + 4 * c) * weight[r];
    shares[threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.x >= COLS) return;
#pragma unroll
    for (int k = 1; k < AT_ONCE; ++k) v += shares[threadIdx.x + k * COLS];
    const float sum = sums[0] + sums[1] + sums[2] + sums[3], r = sum == 0.f ? 0.f : 1.f / sum;
    typedef TA TA4 __attribute__((ext_vector_type(4)));
    TA4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = static_cast<TA>(sum == 0.f ? 0.f : v[e] * r);
    *reinterpret_cast<TA4 *>(static_cast<TA *>(a.o) + t * a.ldo + h * D + 4 * c) = o;
}

// The same for up to FEW ranges: 1024 / D queries of a token a workgroup, all records of one requested at once.
template <class A, int D, int FEW>
__global__ void __launch_bounds__(256) tree_join_few_kernel(TreeAttnArgs a)
{
    typedef typename A::type TA;
    constexpr int COLS = D / 4, QUERIES = 256 / COLS;
    const int t = blockIdx.y, lane = threadIdx.x & 63, c = threadIdx.x % COLS, h = blockIdx.x * QUERIES + threadIdx.x / COLS;
    int b = 0;
    if (a.p.n_seqs > 1) {
        const int end = lane < a.p.n_seqs ? arg_int<offsetof(TreeAttnArgs, p.tok0)>(lane + 1) : INT32_MAX;
        b = __builtin_popcountll(__ballot(end <= t));
    }
    const int ranges = arg_int<offsetof(TreeAttnArgs, ranges)>(b);
    if (ranges == 1 || h >= a.Hq) return;
    const float *rec = a.part + (static_cast<int64_t>(arg_int<offsetof(TreeAttnArgs, rec0)>(b)) * a.Hq +
                                 (static_cast<int64_t>(t - arg_int<offsetof(TreeAttnArgs, p.tok0)>(b)) * a.Hq + h) * ranges) * (TREE_REC + D);
    float2 ml[FEW];
    f4v v[FEW];
#pragma unroll
    for (int r = 0; r < FEW; ++r) {
        const float *at = rec + min(r, ranges - 1) * (TREE_REC + D); // (past the last: once more, as nothing)
        ml[r] = *reinterpret_cast<const float2 *>(at);
        v[r] = *reinterpret_cast<const f4v *>(at + TREE_REC + 4 * c);
    }
#pragma unroll
    for (int r = 0; r < FEW; ++r)
        if (r >= ranges) {
            ml[r].x = -INFINITY;
            v[r] = f4v{0.f, 0.f, 0.f, 0.f};
        }
    float mx = ml[0].x, sum = 0.f;
#pragma unroll
    for (int r = 1; r < FEW; ++r) mx = fmaxf(mx, ml[r].x);
    f4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < FEW; ++r) {
        const float w = ml[r].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[r].x - mx);
        sum += ml[r].y * w;
        o += v[r] * w;
    }
    const float r = sum == 0.f ? 0.f : 1.f / sum;
    typedef TA TA4 __attribute__((ext_vector_type(4)));
    TA4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = static_cast<TA>(sum == 0.f ? 0.f : o[e] * r);
    *reinterpret_cast<TA4 *>(static_cast<TA *>(a.o) + t * a.ldo + h * D + 4 * c) = w;
}

// How a step is shared out.
struct TreePlan {
    int narrow, wide, groups; // blocks of 16 queries of the narrow kernel or of 32 of the wide one (0: the other); workgroups
    int most;                 // ranges of a sequence
    size_t bytes;                      // of records
};

static TreePlan tree_plan(const PagedArgs &p, int Hq, int D, bool split, TreeAttnArgs &a) // split: fp32 queries
{
    TreePlan r{};
    const int G = Hq / p.Hkv;
    int most_tok = 0, most_rows = 1;
    int64_t pieces = 0, work = 0, pieces_64 = 0, pieces_128 = 0, work_256 = 0; // 32 (64, 128) queries on a KV head; rows of each of these (of 256)
    for (int b = 0; b < p.n_seqs; ++b) {
        const int n = p.tok0[b + 1] - p.tok0[b];
        if (n == 0) continue;
        if (n > most_tok) most_tok = n;
        if (p.n_past[b] + n > most_rows) most_rows = p.n_past[b] + n;
        const int64_t tiles = static_cast<int64_t>((n * G + 31) / 32) * p.Hkv;
        pieces += tiles;
        work += tiles * (p.n_past[b] + n);
        pieces_64 += static_cast<int64_t>((n * G + 63) / 64) * p.Hkv;
        pieces_128 += static_cast<int64_t>((n * G + 127) / 128) * p.Hkv;
        work_256 += static_cast<int64_t>((n * G + 255) / 256) * p.Hkv * (p.n_past[b] + n);
    }
    if (most_tok == 0) return r;
    const int most_q = most_tok * G, places_narrow = 512, places_wide = 256; // workgroups that run at once
    // More than 32 queries on a head: the narrow kernel brings the rows once for every 32 of them, the wide one up to 256, but with eight waves and barriers.
    // us, narrow / wide, one sequence, 8 KV heads: 48 fp32 queries behind 1000 rows 13.2 / 17.5, 8192: 21.2 / 22.7, 16000: 27.0 / 24.9; 96: 4000 19.4 / 21.1,
    // 8192 25.3 / 25.0; 504 bf16 queries 1000: 19.3 / 19.3, 4000: 39.2 / 26.5; eight sequences of 48 fp32 queries behind 1000: 20.9 / 21.8, 2000: 24.8 / 24.0.
    // And up to 64 queries of more sequences than the wide kernel has places for, behind few rows: 64 of 8 fp32 tokens, 64 / 8 heads, behind 200 rows 29.4 / 35.9, 500 44.9 / 50.4,
    // 1000 73.4 / 66.9 (bf16 25.1 / 27.8, 40.8 / 39.4, 62.3 / 56.3); 41 of 16, 32 / 8 heads, behind 119 20.7 / 27.3.
    if (most_q <= 32 || (pieces <= places_narrow && work <= 200000) || (most_q <= 64 && pieces_64 > places_wide && work <= 512 * pieces)) r.narrow = most_q <= 16 ? 1 : 2;
    // More than 128: eight waves of queries, which bring the rows half as often as four and another four for other rows; four where the ranges of eight would be short (660 rows and
    // fewer) and their records many, unless they are more than run at once, and for fp32 queries, for which eight leave registers short.  us, four / eight, 64 / 8 heads: one sequence of
    // 20 bf16 tokens behind 8000 rows 22.8 / 25.8, 32000 50.7 / 47.2, 63 behind 4000 26.4 / 31.2, eight of 63 behind 1000 33.1 / 34.9, 4000 83.6 / 75.9, 16 of 40 behind 1000 46.9 / 38.3;
    // fp32, when it had eight, 27.1 / 32.4, 64.0 / 70.9, 32.8 / 38.3, 41.8 / 47.0, 113 / 117, 60.4 / 58.9.
    else r.wide = most_q <= 64 ? 2 : (most_q <= 128 || split || (work_256 <= 660 * places_wide && pieces_128 <= places_wide) ? 4 : 8);
    const int tile_q = r.narrow ? 16 * r.narrow : 32 * r.wide;
    const int q_tiles = (most_q + tile_q - 1) / tile_q;
    a.tile_q = r.narrow ? tile_q : 32 * ((most_q + 32 * q_tiles - 1) / (32 * q_tiles)); // evenly: blocks of 32 that no queries are left for cost little
    auto tiles_of = [&](int tok) { return (tok * G + a.tile_q - 1) / a.tile_q; };
    // Ranges as short as give every compute unit its two workgroups (narrow) or its one in one round; up to 256 rows undivided: joining ranges takes a launch.
    // (One token, 32 / 8 heads, us, undivided / divided: 200 rows 9.5 / 11.0, 300: 10.7 / 11.6, 500: 14.2 / 12.4.)
    const int places = r.narrow ? places_narrow : places_wide;
    auto count = [&](int rows) {
        int64_t n = 0;
        for (int b = 0; b < p.n_seqs; ++b) {
            const int tok = p.tok0[b + 1] - p.tok0[b];
            if (tok) n += (static_cast<int64_t>(p.n_past[b]) + tok + rows - 1) / rows * tiles_of(tok);
        }
        return n * p.Hkv;
    };
    int lo = 1, hi = (most_rows + TREE_STEP - 1) / TREE_STEP; // steps of a range: the fewest that fit
    const int least = static_cast<int>((static_cast<int64_t>(most_rows) + TREE_STEP * TREE_MAX_RANGES - 1) / (TREE_STEP * TREE_MAX_RANGES));
    if (lo < least) lo = least;
    if (most_rows <= 256) lo = hi;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (count(mid * TREE_STEP) <= places) hi = mid;
        else lo = mid + 1;
    }
    int rec = 0;
    for (int b = 0; b < p.n_seqs; ++b) {
        const int tok = p.tok0[b + 1] - p.tok0[b];
        int n = 0;
        if (tok) { // evenly: as many ranges of as many steps as there need to be
            const int steps = (p.n_past[b] + tok + TREE_STEP - 1) / TREE_STEP, parts = (steps + lo - 1) / lo, each = (steps + parts - 1) / parts;
            n = (steps + each - 1) / each;
            a.range_rows[b] = each * TREE_STEP;
        }
        a.ranges[b] = n;
        a.rec0[b] = rec;
        if (n > r.most) r.most = n;
        if (n > 1) rec += tok * n;
    }
    // Where workgroups are more than run at once the short ones come last (34 sequences of 1330 to 1994 rows, 19 bf16 tokens, 64 / 8 heads: 101.6 -> 85.4 us, 36 of 4 behind 3000 79.4 -> 72.6)
    int rows_of[PRIMA_PAGED_MAX_SEQS];
    for (int b = 0; b < p.n_seqs; ++b) {
        const int rows = a.ranges[b] ? a.range_rows[b] : 0;
        int at = b;
        for (; at > 0 && rows_of[at - 1] < rows; --at) {
            rows_of[at] = rows_of[at - 1];
            a.order[at] = a.order[at - 1];
        }
        rows_of[at] = rows;
        a.order[at] = b;
    }
    for (int i = 0; i < p.n_seqs; ++i) {
        const int b = a.order[i];
        a.work0[i] = r.groups;
        r.groups += a.ranges[b] * p.Hkv * tiles_of(p.tok0[b + 1] - p.tok0[b]);
    }
    a.work0[p.n_seqs] = r.groups;
    r.bytes = round_up(static_cast<size_t>(rec) * Hq * (TREE_REC + D) * sizeof(float), 256);
    return r;
}

// The kernels' dynamic LDS may pass 64 KiB: all of them are told on the first call, whichever it launches, so that a step of other lengths, heads or types may be captured after it.
template <class A, class C, int D>
static bool tree_attributes()
{
    auto set = [](auto kernel, size_t lds) {
        return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds)) == hipSuccess;
    };
    bool ok = set(tree_narrow_kernel<A, C, D, 1>, TreeNarrow<A, D, 1>::LDS) && set(tree_narrow_kernel<A, C, D, 2>, TreeNarrow<A, D, 2>::LDS) &&
              set(tree_wide_kernel<A, C, D, 2>, TreeShape<D, 2>::LDS) && set(tree_wide_kernel<A, C, D, 4>, TreeShape<D, 4>::LDS);
    if constexpr (!__is_same(A, F32)) ok = ok && set(tree_wide_kernel<A, C, D, 8>, TreeShape<D, 8>::LDS); // (no plan has it with fp32 queries)
    return ok;
}
static bool tree_attributes_set()
{
    static std::atomic<bool> done{false};
    if (!done) // set twice by two threads at worst: the attribute calls are idempotent
        done = tree_attributes<F32, F16, 128>() && tree_attributes<F16, F16, 128>() && tree_attributes<BF16, BF16, 128>() && tree_attributes<F32, F16, 64>() &&
               tree_attributes<F16, F16, 64>() && tree_attributes<BF16, BF16, 64>();
    return done;
}

template <class A, class C, int D, int NQ>
static void launch_tree_narrow(const TreeAttnArgs &a, dim3 grid, hipStream_t st)
{
    hipLaunchKernelGGL((tree_narrow_kernel<A, C, D, NQ>), grid, dim3(256), (TreeNarrow<A, D, NQ>::LDS), st, a);
}
template <class A, class C, int D, int NR>
static void launch_tree_wide(const TreeAttnArgs &a, dim3 grid, hipStream_t st)
{
    hipLaunchKernelGGL((tree_wide_kernel<A, C, D, NR>), grid, dim3(512), (TreeShape<D, NR>::LDS), st, a);
}

template <class A, class C, int D>
static prima_status launch_tree_attn(const TreeAttnArgs &a, const TreePlan &r, hipStream_t st)
{
    const dim3 grid(r.groups);
    if (!tree_attributes_set()) return PRIMA_E_DEVICE;
    if (r.narrow == 1) launch_tree_narrow<A, C, D, 1>(a, grid, st);
    else if (r.narrow == 2) launch_tree_narrow<A, C, D, 2>(a, grid, st);
    else if (r.wide == 2) launch_tree_wide<A, C, D, 2>(a, grid, st);
    else if (r.wide == 4) launch_tree_wide<A, C, D, 4>(a, grid, st);
    else if constexpr (!__is_same(A, F32)) launch_tree_wide<A, C, D, 8>(a, grid, st);
    else return PRIMA_E_DEVICE; // (no plan has it)
    if (r.most < 2) return last_launch_status();
    constexpr int few = 1024 / D; // queries of a workgroup
    const dim3 groups((a.Hq + few - 1) / few, paged_tokens(a.p));
    if (r.most <= 2) hipLaunchKernelGGL((tree_join_few_kernel<A, D, 2>), groups, dim3(256), 0, st, a);
    else if (r.most <= 4) hipLaunchKernelGGL((tree_join_few_kernel<A, D, 4>), groups, dim3(256), 0, st, a);
    else if (r.most <= 8) hipLaunchKernelGGL((tree_join_few_kernel<A, D, 8>), groups, dim3(256), 0, st, a);
    // (us, four / eight times 1024 / D ranges at once: 59 ranges 27.7 / 26.7, 32: 20.9 / 21.2)
    else if (r.most <= 4 * few) hipLaunchKernelGGL((tree_join_kernel<A, D, 4>), dim3(a.Hq, paged_tokens(a.p)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((tree_join_kernel<A, D, 8>), dim3(a.Hq, paged_tokens(a.p)), dim3(256), 0, st, a);
    return last_launch_status();
}

// (64 tokens of at most 1024 heads: tree_token)
static bool tree_heads_ok(int Hq, int Hkv) { return Hq >= 1 && Hq <= 65535 && Hq % Hkv == 0 && Hq / Hkv <= 1024; }

template <int D>
static prima_status launch_tree_attn(const TreeAttnArgs &a, const TreePlan &r, int dtype, int cache, hipStream_t st)
{
    if (cache == PRIMA_DT_BF16) return launch_tree_attn<BF16, BF16, D>(a, r, st);
    if (dtype == PRIMA_DT_F16) return launch_tree_attn<F16, F16, D>(a, r, st);
    return launch_tree_attn<F32, F16, D>(a, r, st);
}

} // namespace prima

using namespace prima;

extern "C" {

size_t prima_tree_attn_workspace_bytes(const prima_kv_pages *pages, const prima_paged_step *step, int32_t n_q_heads)
{
    TreeAttnArgs a{};
    if (paged_args(pages, step, a.p) != PRIMA_OK || !tree_heads_ok(n_q_heads, a.p.Hkv)) return 0;
    const size_t split = tree_plan(a.p, n_q_heads, pages->head_dim, true, a).bytes, whole = tree_plan(a.p, n_q_heads, pages->head_dim, false, a).bytes;
    const size_t most = split > whole ? split : whole; // (whatever the queries' type)
    return most > 256 ? most : 256;                    // (none are needed: some all the same, since 0 is what a refusal gives and the call takes no null pointer)
}

prima_status prima_tree_attn_plan(const prima_kv_pages *pages, const prima_paged_step *step, int32_t n_q_heads, int32_t dtype, int32_t *few, int32_t *many,
                                  int32_t *ranges, int32_t *range_rows)
{
    if (!few || !many || !ranges || !range_rows) return PRIMA_E_NULL;
    TreeAttnArgs a{};
    const prima_status s = paged_args(pages, step, a.p);
    if (s != PRIMA_OK) return s;
    if (!act_dtype_ok(*pages, dtype) || !tree_heads_ok(n_q_heads, a.p.Hkv)) return PRIMA_E_SHAPE;
    const TreePlan r = tree_plan(a.p, n_q_heads, pages->head_dim, dtype == PRIMA_DT_F32, a);
    *few = r.narrow;
    *many = r.wide;
    for (int b = 0; b < a.p.n_seqs; ++b) {
        ranges[b] = a.ranges[b];
        range_rows[b] = a.range_rows[b];
    }
    return PRIMA_OK;
}

prima_status prima_tree_attn(const prima_kv_pages *pages, const prima_paged_step *step, int32_t n_q_heads, int32_t dtype, const void *q, int64_t ldq,
                             float scale, void *o, int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!q || !o || !workspace) return PRIMA_E_NULL;
    TreeAttnArgs a{};
    const prima_status s = paged_args(pages, step, a.p);
    if (s != PRIMA_OK) return s;
    if (!act_dtype_ok(*pages, dtype) || !tree_heads_ok(n_q_heads, a.p.Hkv)) return PRIMA_E_SHAPE;
    const int D = pages->head_dim;
    const int64_t qd = static_cast<int64_t>(n_q_heads) * D;
    if (ldq < qd || ldo < qd) return PRIMA_E_SHAPE;
    if (!(scale > 0.f && scale <= 1e6f)) return PRIMA_E_RANGE;
    const int unit = dtype == PRIMA_DT_F32 ? 4 : 8; // elements of 16 bytes
    if (!aligned(q, 16) || !aligned(o, 16) || ldq % unit || ldo % unit || !aligned(workspace, 256)) return PRIMA_E_ALIGN;
    const TreePlan r = tree_plan(a.p, n_q_heads, D, dtype == PRIMA_DT_F32, a);
    if (workspace_bytes < r.bytes) return PRIMA_E_WORKSPACE;
    if (r.groups == 0) return PRIMA_OK;
    a.q = q; a.o = o; a.ldq = ldq; a.ldo = ldo; a.scale = scale * 1.44269504088896340736f; a.Hq = n_q_heads;
    a.G = n_q_heads / a.p.Hkv;
    a.inverse = 0xffffffffu / static_cast<unsigned>(a.G) + 1;
    a.part = static_cast<float *>(workspace);
    if (D == 128) return launch_tree_attn<128>(a, r, dtype, pages->dtype, static_cast<hipStream_t>(hip_stream));
    return launch_tree_attn<64>(a, r, dtype, pages->dtype, static_cast<hipStream_t>(hip_stream));
}

} // extern "C"
