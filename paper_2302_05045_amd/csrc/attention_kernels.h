// Softmax attention over packed sequences and its backward pass, which recomputes the probabilities: what lies between the QKV
// projection and the output projection of a transformer layer.  Per sequence and head
//   S = scale Q K^T with the masked places at -inf,  lse = log sum exp S,  P = exp(S - lse),  O = P V
//   delta = rowsum(dO O),  dV = P^T dO,  dP = dO V^T,  dS = P (dP - delta),  dQ = scale dS K,  dK = scale dS^T Q
// No matrix of scores exists in memory: the forward pass keeps lse, one number a row, and the backward pass forms S again.
//
// Bound by the matrix units (fp16 products, fp32 sums), with the LDS reads of their operands and, in the softmax, the vector ALU close
// behind.  What the kernels share:
//  - A wave owns 32 rows of one side (queries; keys for dK, dV) whose operands stay in its registers; the other side comes
//    in tiles of 64 rows through LDS, two tiles in turn, copied past the registers while the other is multiplied.
//  - Scores are formed transposed where the wave owns queries: S^T = K Q^T puts a query into a lane's column, so the softmax is a
//    maximum and a sum over a lane's own registers and one exchange between the wave's halves.  An accumulator register holds rows
//    8 (i / 4) + 4 half + i % 4 of the block: eight of them in a row are, as they are, the operand of the next product over 16 of
//    those rows, as long as the other operand is read in the same order -- and the transposing LDS read takes any four rows.
//    So P and dS go from one product to the next without leaving the registers.
//  - A tile's LDS rows are 128 or 256 bytes; 16-byte piece c of row r lies at c ^ swizzle(r), which spreads both kinds of read, 16
//    rows by one piece and 4 rows by 64 bytes, over all banks.
//  - Workgroups of a head go to one of the 8 XCDs, where they share its other side in the L2 (pick()).
// P and dS are rounded to fp16 for the products they enter, as Q, K, V and dO are: 2^-11 of themselves; statistics and all sums are fp32.  (fp32 products
// have a sixteenth of the rate.)  delta is fp32, of out as memory has it, rounded: an error no larger than that of dS.  dS is rounded without the scale
// that dQ and dK take at the end: with 2^-3 or less in it, the dS of thousands of keys, 2^-10 and less where dO is near 1, would be among fp16's
// subnormal numbers and lose bits, for a range above 65504 in which a loss scale is too large anyway.
// dQ and dK, dV are formed by two kernels, each of which forms S and dP: 7 products for the 5 that one kernel would need, but every
// sum has one owner and one order, so the same call gives the same bits (with additions to dQ in memory it would not).
#pragma once

#include "common.h"
#include "lds_copy.h"

namespace samo {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kAttnThreads = 256, kWaveRows = 32, kTileRows = 64;
constexpr int kOwnRows = kAttnThreads / 64 * kWaveRows;           // 128
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// KS: steps of 16 that a head's dim takes; 32 x 32 blocks, bytes of an LDS row, 16-byte pieces of one, bytes of a tile.
constexpr int blocks_of(int ks) { return (ks + 1) / 2; }
constexpr int pitch_of(int ks) { return ks <= 4 ? 128 : 256; }
constexpr int tile_bytes(int ks) { return kTileRows * pitch_of(ks); }

template <int PITCH>
__device__ __forceinline__ int swizzle(int row)
{
    return PITCH == 256 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
}

// A sequence's rows of one operand, at one head.
struct Rows {
    const _Float16 *base;
    int64_t stride;          // elements from row to row
    int count, dim;
};

// A wave's share, one of four, of the tiles of one operand.
template <int KS>
struct Tiles {
    static constexpr int PITCH = pitch_of(KS), kPieces = PITCH / 16, kRowsPer = 64 / kPieces, kCopies = kTileRows / kRowsPer / 4;
    Rows R;
    bool plain;                                              // whole tiles by a scalar address and these:
    unsigned offset[kCopies];                                // of the lane's piece from the tile's first row
    __device__ __forceinline__ static int copy_of(int i) { return (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3) * kCopies + i; }
    __device__ __forceinline__ static int row_of(int i) { return copy_of(i) * kRowsPer + (int)(threadIdx.x & 63) / kPieces; }
    __device__ __forceinline__ static int piece_of(int i) { return (int)(threadIdx.x & 63) % kPieces ^ swizzle<PITCH>(row_of(i)); }
    __device__ __forceinline__ explicit Tiles(const Rows &rows) : R(rows)
    {
        // A dim of whole steps reads no piece behind it into a product that counts; rows less than 2^24 elements apart keep the offsets in 32 bits.
        plain = R.dim == 16 * KS && R.stride < 1 << 24;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) offset[i] = (unsigned)row_of(i) * (unsigned)R.stride * 2 + (piece_of(i) * 8 < R.dim ? piece_of(i) * 16 : 0);
    }
    // rows first .. first + 63 to LDS; what is behind the rows is zero, and behind the dim where it counts
    __device__ __forceinline__ void bring(int first, unsigned lds_at) const
    {
        if (plain && first + kTileRows <= R.count) {
            const unsigned char *base = uniform(reinterpret_cast<const unsigned char *>(R.base + (int64_t)first * R.stride));
#pragma unroll
            for (int i = 0; i < kCopies; ++i) dma16_from(base, offset[i], lds_at + copy_of(i) * 1024);
            return;
        }
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int row = first + row_of(i), piece = piece_of(i);
            const bool there = row < R.count && piece * 8 < R.dim;
            dma16(there ? static_cast<const void *>(R.base + (int64_t)row * R.stride + piece * 8) : zero_row, lds_at + copy_of(i) * 1024);
        }
    }
};

// A tile copied by one wave: its kWhole instructions.
template <int KS>
struct OwnTiles {
    static constexpr int PITCH = pitch_of(KS), kPieces = PITCH / 16, kRowsPer = 64 / kPieces, kWhole = kTileRows / kRowsPer;
    Rows R;
    __device__ __forceinline__ void bring(int first, unsigned lds_at) const
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kWhole; ++i) {
            const int in_tile = i * kRowsPer + lane / kPieces, row = first + in_tile, piece = lane % kPieces ^ swizzle<PITCH>(in_tile);
            const bool there = row < R.count && piece * 8 < R.dim;
            dma16(there ? static_cast<const void *>(R.base + (int64_t)row * R.stride + piece * 8) : zero_row, lds_at + i * 1024);
        }
    }
};

// Operand with the tile's rows as its rows (32 of them from row 32 block) and 16 columns from 16 ks.
template <int PITCH>
__device__ __forceinline__ half8 read_rows(const unsigned char *tile, int block, int ks)
{
    const int lane = threadIdx.x & 63, row = lane & 31;
    return *reinterpret_cast<const half8 *>(tile + (block * 32 + row) * PITCH + (((2 * ks + (lane >> 5)) ^ swizzle<PITCH>(row)) << 4));
}

// Operand with the tile's columns 32 db .. as its rows, over the tile's rows 16 step .. in the order an accumulator holds them.
template <int PITCH>
__device__ __forceinline__ half8 read_columns(const unsigned char *tile, int step, int db)
{
    const int lane = threadIdx.x & 63, i = lane & 15, half = lane >> 5;
    const int piece = 4 * db + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
    const int row = 4 * half + (i >> 2);                       // and row + 8
    const unsigned char *at = tile + step * 16 * PITCH + (i & 1) * 8;
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS short4v *)(LDS_AS unsigned char *)(at + row * PITCH + ((piece ^ swizzle<PITCH>(row)) << 4)));
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (LDS_AS short4v *)(LDS_AS unsigned char *)(at + (row + 8) * PITCH + ((piece ^ swizzle<PITCH>(row + 8)) << 4)));
    const short8v q = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(half8, q);
}

// The wave's own rows as operand columns, straight from memory: row (lane & 31), 8 elements of every step's 16.
template <int KS>
__device__ __forceinline__ void load_own(const Rows &R, int first, half8 (&own)[KS])
{
    const int lane = threadIdx.x & 63, row = first + (lane & 31), half = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int col = 16 * ks + 8 * half;
        half8 x = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row < R.count && col < R.dim) x = *reinterpret_cast<const half8 *>(R.base + (int64_t)row * R.stride + col);
        own[ks] = x;
    }
}

// The same of a row that the lane names.
template <int KS>
__device__ __forceinline__ void load_row(const _Float16 *row, bool there, int dim, half8 (&own)[KS])
{
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int col = 16 * ks + 8 * half;
        half8 x = {0, 0, 0, 0, 0, 0, 0, 0};
        if (there && col < dim) x = *reinterpret_cast<const half8 *>(row + col);
        own[ks] = x;
    }
}

// x of the other half of the wave, lane by lane.
__device__ __forceinline__ float other_half(float x)
{
    const auto two = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? two[0] : two[1]);
}

__device__ __forceinline__ half8 to_half8(const f32x16 &x, int at)
{
    half8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)x[at + e];
    return h;
}

// Row of a 32 x 32 accumulator's register i.
__device__ __forceinline__ int acc_row(int i) { return 8 * (i >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (i & 3); }

// Column (lane & 31) of a transposed result, times factor, as row `row` of a tensor.
template <int DB>
__device__ __forceinline__ void store_own(_Float16 *base, int64_t stride, int row, int count, int dim, const f32x16 (&acc)[DB], float factor)
{
    if (row >= count) return;
    _Float16 *to = base + (int64_t)row * stride;
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * db + 8 * g + 4 * half;
            if (d >= dim) continue;
            half4 h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = (_Float16)(acc[db][4 * g + e] * factor);
            *reinterpret_cast<half4 *>(to + d) = h;
        }
}

template <int N>
__device__ __forceinline__ void clear(f32x16 (&acc)[N])
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
}

// One sequence: where its rows begin and how many there are, inside the tensors whatever the tables hold.
struct Sequence {
    int64_t q0, k0;
    int q_len, k_len;
};
__device__ __forceinline__ void bounds_of(const int32_t *start, int b, int64_t tokens, int64_t &first, int &len)
{
    int64_t lo = 0, hi = tokens;
    if (start) {
        lo = start[b];
        hi = start[b + 1];
        lo = lo < 0 ? 0 : lo > tokens ? tokens : lo;
        hi = hi < lo ? lo : hi > tokens ? tokens : hi;
    }
    first = lo;
    len = (int)(hi - lo);
}
__device__ __forceinline__ Sequence sequence_of(const AttnArgs &A, int b)
{
    Sequence s;
    bounds_of(A.q_start, b, A.q_tokens, s.q0, s.q_len);
    bounds_of(A.k_start, b, A.k_tokens, s.k0, s.k_len);
    return s;
}

// Of a launch's work: a sequence, a head, 128 of its own rows, and a part of what they are multiplied with.
struct Place {
    int b, head, tile, part;
    int64_t slot;                            // of the part's sums
};
__device__ __forceinline__ Place place_of(int of_head, int tile, int part, const AttnArgs &A)
{
    const int head = of_head / A.batch;
    return {of_head - head * A.batch, head, tile, part, ((int64_t)of_head * A.tiles + tile) * A.splits + part};
}
// The workgroup's place.  The tiles that see the most go first, of all heads and sequences, so that a launch ends with short workgroups.  An XCD gets
// the same heads of every tile, whose other side stays in its L2, or, where few heads and sequences do not divide evenly among
// the XCDs, what comes next.  All tiles of a head together / this, us on one card, forward and backward: 8192 causal tokens in 4
// sequences, 32 heads of 64, 122 and 378 / 100 and 317; of 80 163 and 509 / 140 and 481; in one sequence, 32 heads of 128 on 8, 608 and 2094 / 598 and 2052.
__device__ __host__ inline int heads_an_xcd(int all) { return all % 8 == 0 || all >= 64 ? (all + 7) / 8 : 0; }       // 0: what comes next
__device__ __forceinline__ bool pick(const AttnArgs &A, int heads, Place &p)
{
    const int all = A.batch * heads, share = heads_an_xcd(all), xcd = (int)(blockIdx.x & 7), local = (int)(blockIdx.x >> 3) / A.splits;
    const int n = share ? 0 : local * 8 + xcd, turn = share ? local / share : n / all;
    const int of_head = share ? xcd * share + local - turn * share : n - turn * all;
    if (turn >= A.tiles || of_head >= all) return false;
    p = place_of(of_head, A.tiles - 1 - turn, (int)(blockIdx.x >> 3) % A.splits, A);
    return true;
}

// Where a wave of a workgroup leaves the sums of its 32 rows, as they lie in its registers: part by part, and within a part wave by wave.
template <int DB>
__device__ __forceinline__ f32x4 *sums_of(float *parts, int64_t slot, int wave) { return reinterpret_cast<f32x4 *>(parts) + (slot * 4 + wave) * (DB * 256) + (threadIdx.x & 63); }
template <int DB>
__device__ __forceinline__ void leave(float *parts, int64_t slot, int wave, int row, int count, const f32x16 (&acc)[DB])
{
    if (row >= count) return;
    f32x4 *to = sums_of<DB>(parts, slot, wave);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) to[(4 * db + g) * 64] = f32x4{acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
}

// Which keys a query sees: first_key(query) .. end_key(query) - 1, all of them without `causal`; and which queries see a key.
template <bool KEYS>                          // whether there may be first keys that every query sees
struct Mask {
    bool causal;
    int shift, window, q_len, k_len;         // window 2^30: none
    int first;                               // those keys; 0 but with causal
    __device__ __forceinline__ bool early(int key) const { return KEYS && key < first; }
    __device__ __forceinline__ int first_key(int query) const { return causal ? query + shift - window + 1 : 0; }
    __device__ __forceinline__ int end_key(int query) const { return causal ? min(query + shift + 1, k_len) : k_len; }
    __device__ __forceinline__ int first_query(int key) const { return causal && !early(key) ? key - shift : 0; }
    __device__ __forceinline__ int end_query(int key) const { return causal && !early(key) ? min(key - shift + window, q_len) : q_len; }
    // whether all of / any of a block of queries and keys (first and last of each) are seen
    __device__ __forceinline__ bool all(int q0, int q1, int k0, int k1) const
    {
        return k1 < k_len && (!causal || early(k1) || (k1 <= q0 + shift && k0 > q1 + shift - window));
    }
    __device__ __forceinline__ bool any(int q0, int q1, int k0, int k1) const
    {
        return !causal || early(k0) || (k0 <= q1 + shift && k1 > q0 + shift - window);
    }
};
// The numbers from .. end - 1 by one comparison.
struct Span {
    int from;
    unsigned count;
    __device__ __forceinline__ Span(int first, int end) : from(first), count(end > first ? (unsigned)(end - first) : 0u) {}
    __device__ __forceinline__ bool holds(int x) const { return (unsigned)(x - from) < count; }
};
template <bool KEYS>
__device__ __forceinline__ Mask<KEYS> mask_of(const AttnArgs &A, const Sequence &s, int b)
{
    Mask<KEYS> m;
    m.first = KEYS && A.causal && A.form.first_keys ? min(max(A.form.first_keys[b], 0), s.k_len) : 0;
    m.causal = A.causal != 0;
    m.shift = s.k_len - s.q_len;
    m.window = A.window > 0 ? min(A.window, 1 << 30) : 1 << 30;
    m.q_len = s.q_len;
    m.k_len = s.k_len;
    return m;
}

// A part's share of the tiles of keys that any of the queries q0 .. q1 sees: those of the first keys, then from what the window leaves on.
template <bool KEYS>
struct KeyTiles {
    int first, end;                          // the first tile's first row, and what lies behind the last one's rows or begins
    int head, near;                          // the end of the first keys' tiles, and where the others begin
    int from, count;                         // of all tiles, those of the part
    __device__ __forceinline__ KeyTiles(const AttnArgs &A, const Mask<KEYS> &M, int q0, int q1, int part)
    {
        first = 0;
        end = M.k_len;
        if (M.causal) {
            const int last = q1 + M.shift + 1, begin = q0 + M.shift - M.window + 1;
            end = last < end ? last : end;
            first = begin > 0 ? begin / kTileRows * kTileRows : 0;
        }
        head = near = 0;
        if (KEYS) {
            head = (M.first + kTileRows - 1) / kTileRows * kTileRows;
            near = max(first, head);
            end = max(end, M.first);
        }
        const int heads = KEYS ? head / kTileRows : 0, begin = KEYS ? near : first;
        const int tiles = heads + (end > begin ? (end - begin + kTileRows - 1) / kTileRows : 0), each = (tiles + A.splits - 1) / A.splits;
        from = min(tiles, part * each);
        const int to = min(tiles, from + each);
        count = to - from;
        if (KEYS) {
            first = from < heads ? from * kTileRows : near + (from - heads) * kTileRows;
            end = from == to ? first : to <= heads ? to * kTileRows : near + (to - heads) * kTileRows;
        } else {
            first += from * kTileRows;
            end = min(end, first + each * kTileRows);
        }
    }
    __device__ __forceinline__ int at(int n) const       // the first row of the part's nth tile, where there may be first keys
    {
        const int heads = head / kTileRows, i = from + n;
        return i < heads ? i * kTileRows : near + (i - heads) * kTileRows;
    }
    __device__ __forceinline__ int after(int k0) const { return KEYS && k0 + kTileRows == head ? near : k0 + kTileRows; }
};

// Scores of another form (SCORED): z = cap tanh(x / cap) + bias(d), x the scaled product.  All of it in units of `unit` and log 2: a product, or its tanh,
// and a bias are added and enter the exponent by the same multiplication as a plain product.  Slopes without a cap are what the matrix instructions
// start from, so that they cost the making of 16 registers; with one, and of a table (late), the bias is added to what they leave.  Biases of a block of queries and keys, whose
// distances are those of its diagonals, come in four kinds:
//   kSame    one number, where all distances have one bucket: nothing to do for an element (most blocks of long sequences)
//   kLinear  a slope, the block on one side of the diagonal and kNear or more from it: one multiplication and addition for each element.  The line begins
//            at most 63 distances from an element's, so that its rounding is that of a bias of twice the size at most
//   kAcross  a slope, the block nearer: one more, and each bias by itself, exact on the diagonal whatever the slope
//   kLaid    buckets that differ: the wave works out its diagonals' biases, a lane each, and lays them into LDS
// The table's columns and borders live in the wave's lanes: the bucket of a distance that the lanes agree on is the number of set bits of a comparison.
constexpr int kMaxBuckets = SAMO_ATTENTION_MAX_BUCKETS;
enum { kSame, kLinear, kAcross, kLaid };
constexpr int kNear = 64;
// Where a row's largest score so far, in log 2, is beyond this, its product with `unit` is off by more than 2^-8 and the exponents are taken from the
// difference of the scores (slopes only: a table's biases are below 2^17 in log 2, a cap's scores below 2^9).
constexpr float kFarScore = 0x1p16f;
// Which parts there are, kernels of their own: none (kKeys: but the first keys), one, two; kAll: slopes and a table, with a cap or without.  With one kernel
// for the last three, both passes, us: 8192 tokens in 4, 32 heads of 128 on 8, cap and slopes 1313 and 1114; 16 heads of 64, cap and 32 buckets 385 and 331.
enum { kPlain, kKeys, kCap, kSlope, kTable, kCapSlope, kCapTable, kAll };
constexpr bool has_cap(int form) { return form == kCap || form >= kCapSlope; }
constexpr bool has_slope(int form) { return form == kSlope || form == kCapSlope || form == kAll; }
constexpr bool has_table(int form) { return form == kTable || form >= kCapTable; }
// Biases of a table alone are found while the products are under way and added to them, not what they start from: both passes, us, before / behind,
// 8192 tokens in 4, 32 buckets: 16 heads of 64 277 / 273, 32 of 128 on 8 830 / 820, capped 958 / 944.  (A token of 3 sequences, attention_few_kernel: 16.4 / 17.0, so before.)
constexpr bool late(int form) { return has_table(form) && !has_slope(form); }
constexpr bool packs(int form) { return form != kPlain && !has_table(form); }
struct Bias {
    int kind, column;                        // column: of all the block's pairs, the second half behind kMaxBuckets; -1 where they differ
    int sign;                                // kAcross: of the distance from row to row
    int diagonal;                            // where they differ: of the lane's diagonal, row - column + 31 (blocks of 32 rows)
    float same, step, base;                  // kSame; kLinear: from row to row, and at the lane's first; kAcross: the slope, and the lane's first distance
};
__device__ __forceinline__ float of_lane(float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(4 * lane, __builtin_bit_cast(int, x))); }
template <int FORM>
struct Form {
    static constexpr bool kCapped = has_cap(FORM), kSloped = has_slope(FORM), kTabled = has_table(FORM), kBiased = kSloped || kTabled, tabled = kTabled;
    bool capped = kCapped, two_sided = false;
    float unit, slope = 0.f;
    float c0, c1, c2, c3, small, into;       // the tanh's polynomial of a product, the largest product that it is for, and scale / cap
    int border = kFar;                       // lane l: where bucket l + 1 begins
    int single = 0;                          // the first buckets that are one distance each
    float past = 0.f, ahead = 0.f;           // lane l: the bias of bucket l, and where the key lies behind
    __device__ __forceinline__ Form(const AttnArgs &A, int head)
    {
        const int lane = threadIdx.x & 63;
        const AttnForm &F = A.form;
        if (FORM == kAll) capped = F.cap > 0.f;
        unit = (capped ? F.cap : A.scale) * kLog2e;
        if constexpr (kCapped) {
            into = capped ? A.scale / F.cap : 0.f;
            const float square = into * into;
            c0 = 0.999999464f * into;
            c1 = -0.333263189f * into * square;
            c2 = 0.131902963f * into * square * square;
            c3 = -0.0444022268f * into * square * square * square;
            small = into > 0x1p-17f && into < 0x1p17f ? kSmall / into : -1.f;       // where into^7 and what it is multiplied with are numbers
        }
        const float of_bias = capped ? 1.f / F.cap : 1.f / A.scale;
        if constexpr (kSloped) slope = F.slopes[head] * of_bias;
        if constexpr (kTabled) {
            two_sided = F.two_sided != 0;
            const int columns = two_sided ? 2 * F.buckets : F.buckets;
            const _Float16 *table = F.table + (int64_t)head * columns;
            border = lane < F.buckets - 1 ? min(max(F.borders[lane], 0), kFar) : kFar;
            single = __builtin_ctzll(~__ballot(border == lane + 1));
            past = lane < F.buckets ? (float)table[lane] * of_bias : 0.f;
            ahead = two_sided && lane < F.buckets ? (float)table[F.buckets + lane] * of_bias : 0.f;
        }
    }
    static constexpr int kFar = 1 << 30;     // behind every distance
    __device__ __forceinline__ int away(int d) const { return two_sided ? abs(d) : max(d, 0); }      // a distance as the buckets count it
    __device__ __forceinline__ int bucket(int away) const { return __builtin_popcountll(__ballot(border <= away)); }
    // tanh(t) of t = scale x / cap, two ways.  For |t| up to kSmall t times a polynomial in t^2, the one of its degree whose largest relative error is least
    // (5.5e-7; found by exchange), in powers of x: five instructions.  Anywhere: sign (1 - e) / (1 + e), e = exp(-2 |t|), within 2^-22: 9, two of
    // them slow.  By the block, whose largest |x| is looked for.
    static constexpr float kSmall = 0.5f;
    __device__ __forceinline__ f32x16 tanhs(f32x16 s) const
    {
        float most = fabsf(s[0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, fabsf(s[i]));
        if (!__ballot(most > small)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float u = s[i] * s[i];
                s[i] *= fmaf(fmaf(fmaf(c3, u, c2), u, c1), u, c0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(fabsf(s[i]) * (-2.f * kLog2e * into));
                s[i] = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), s[i]);
            }
        }
        return s;
    }
    // The biases of a block of ROWS rows and 32 columns, d = base + SIGN (row - column).  Several columns may have the same distances (pack): `own` is the
    // lane's in row 0, and the last column's lies `span` from base.
    template <int ROWS, int SIGN>
    __device__ __forceinline__ Bias plan(float *room, int base) const { return plan<ROWS, SIGN>(room, base, base - SIGN * (int)(threadIdx.x & 31), 31); }
    template <int ROWS, int SIGN>
    __device__ __forceinline__ Bias plan(float *room, int base, int own, int span) const
    {
        Bias b = {kSame, -1, 0, -1, 0.f, 0.f, 0.f};
        if constexpr (kBiased) laying<ROWS, SIGN>(b, room, base, own, span);
        return b;
    }
    template <int ROWS, int SIGN>
    __device__ __forceinline__ void laying(Bias &b, float *room, int base, int own, int span) const
    {
        const int lane = threadIdx.x & 63, lo = SIGN > 0 ? base - span : base - (ROWS - 1), hi = SIGN > 0 ? base + ROWS - 1 : base + span;
        int b0 = 0, b1 = 0;
        if (tabled) {
            const bool one_side = !two_sided || lo >= 0 || hi < 0, behind = two_sided && hi < 0;
            b0 = bucket(behind ? -hi : max(lo, 0));
            b1 = bucket(two_sided ? max(-lo, hi) : max(hi, 0));
            if (one_side && b0 == b1) {
                b.column = behind ? kMaxBuckets + b0 : b0;
                if (!kSloped) {
                    b.same = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, behind ? ahead : past), b0));
                    return;
                }
            }
        } else {
            if constexpr (kSloped) {
                const float first = (float)(own + SIGN * 4 * (lane >> 5));
                const bool one_side = lo >= kNear || hi <= -kNear;
                const float down = one_side && lo < 0 ? slope : -slope;
                b.kind = one_side ? kLinear : kAcross;
                b.step = one_side ? SIGN * down : down;
                b.base = one_side ? down * first : first;
                b.sign = SIGN;
            }
            return;
        }
        b.kind = kLaid;
#pragma unroll
        for (int part = 0; part < (ROWS + 31 + 63) / 64; ++part) {
            const int e = part * 64 + lane, d = base + SIGN * (e - 31), n = away(d);
            float bias = kSloped ? -slope * fabsf((float)d) : 0.f;
            if (tabled) {
                int at = max(b0, min(n, single));
                for (int i = max(b0, single); i < b1; ++i) at += n >= __builtin_amdgcn_readlane(border, i);
                bias += of_lane(past, at);
                if (two_sided) {
                    const float behind = of_lane(ahead, at), before = bias;
                    bias = d < 0 ? behind + (kSloped ? -slope * fabsf((float)d) : 0.f) : before;
                }
                if (part == 0) b.diagonal = two_sided && d < 0 ? kMaxBuckets + at : at;
            }
            if (e < ROWS + 31) room[e] = bias;
        }
        __builtin_amdgcn_wave_barrier();
    }
    // Those of rows 32 block .. (not kSame), as an accumulator holds them.
    __device__ __forceinline__ f32x16 biases(const Bias &b, const float *room, int block) const
    {
        f32x16 x = {};
        const float *at = room + 31 + 32 * block - (int)(threadIdx.x & 31);
        if (kSloped && b.kind == kLinear) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = fmaf(b.step, (float)(32 * block + 8 * (i >> 2) + (i & 3)), b.base);
        } else if (kSloped && b.kind == kAcross) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = b.step * fabsf(b.base + b.sign * (float)(32 * block + 8 * (i >> 2) + (i & 3)));
        } else if constexpr (kTabled) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = at[acc_row(i)];
        }
        return x;
    }
    // What the products' sums start from, and what becomes of them.
    __device__ __forceinline__ bool starts(const Bias &b) const { return kBiased && b.kind != kSame && !capped; }
    __device__ __forceinline__ f32x16 with_bias(f32x16 s, const Bias &b, const float *room, int block) const
    {
        if constexpr (kBiased) {
            if (b.kind == kSame) return s;
            if (kSloped && b.kind == kLinear) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] += fmaf(b.step, (float)(32 * block + 8 * (i >> 2) + (i & 3)), b.base);
            } else if (kSloped && b.kind == kAcross) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = fmaf(b.step, fabsf(b.base + b.sign * (float)(32 * block + 8 * (i >> 2) + (i & 3))), s[i]);
            } else if constexpr (kTabled) {
                const float *at = room + 31 + 32 * block - (int)(threadIdx.x & 31);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] += at[acc_row(i)];
            }
        }
        return s;
    }
};
constexpr int kBiasRoom = 96;                // floats of a wave's biases

// Scores of rows whose largest is far from zero as differences from it, and what is to be taken off them then.  Other rows of the wave stay as they are.
__device__ __forceinline__ void from_top(f32x16 (&s)[2], float top, float &against)
{
    const bool far = fabsf(against) > kFarScore;
    if (!__ballot(far)) return;
    top = far ? top : 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] -= top;
    against = far ? 0.f : against;
}

// Waves to a SIMD that the registers of the forms' kernels leave room for, forward and dQ.  Heads of 33 to 64: three, without a spilled register but in dQ of a
// cap with a table (2 of 168); dQ of 32 buckets, 8 x 1024 in both directions, 12 heads of 64, 84 us with two and 68 with three (768 workgroups are one
// round then); four would spill in the forward pass (4093 tokens in 7, 16 heads, both passes 109 us with three there, 113 with four).
enum { kForward, kDq, kDkv };
constexpr int waves_of(int ks, int form) { return form == kPlain || form == kAll || ks > 4 ? 2 : ks == 2 && !has_table(form) ? 4 : 3; }
struct NoForm {};
template <int FORM>
__device__ __forceinline__ auto form_of(const AttnArgs &A, int head)
{
    if constexpr (FORM != kPlain) return Form<FORM>(A, head);
    else return NoForm{};
}

__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int step = 32; step > 0; step >>= 1) x += __shfl_xor(x, step);
    return x;
}
// x of the lanes up to this one that have its column, added; lanes of a column are neighbours.
template <int CONTROL, int ROWS>
__device__ __forceinline__ void scan_step(float &x, int column)
{
    const float other = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, ROWS, 0xf, false));
    x += __builtin_amdgcn_update_dpp(-1, column, CONTROL, ROWS, 0xf, false) == column ? other : 0.f;
}
__device__ __forceinline__ float scan_of_column(float x, int column)
{
    scan_step<0x111, 0xf>(x, column);        // one lane to the right within rows of 16, two, four, eight
    scan_step<0x112, 0xf>(x, column);
    scan_step<0x114, 0xf>(x, column);
    scan_step<0x118, 0xf>(x, column);
    scan_step<0x142, 0xa>(x, column);        // a row's last lane to the next row; the second row's to the third and fourth
    scan_step<0x143, 0xc>(x, column);
    return x;
}

// The table's gradient: lane l holds the sums of dS over the pairs of bucket l so far.  A block whose pairs have one column adds to its lanes' own sums, which meet
// when the column changes.  Of another one the diagonals are added: half of its rows at a time go to LDS, each shifted by its number, so that a
// diagonal is a column; rows keep their places, and what is beside them zero.  A scan over the lanes of a bucket's diagonals leaves its sum in their last.
constexpr int kSkewed = 47, kSkewRoom = 16 * kSkewed;
struct BucketSums {
    float past = 0.f, ahead = 0.f, run = 0.f;
    int column = 0;
    __device__ __forceinline__ void start(float *room) const
    {
        for (int i = threadIdx.x & 63; i < kSkewRoom; i += 64) room[i] = 0.f;
        __builtin_amdgcn_wave_barrier();
    }
    __device__ __forceinline__ void flush()
    {
        const float sum = wave_sum(run);
        const int lane = threadIdx.x & 63;
        past += lane == column ? sum : 0.f;
        ahead += lane + kMaxBuckets == column ? sum : 0.f;
        run = 0.f;
    }
    template <int FORM>
    __device__ __forceinline__ void add(const Form<FORM> &F, const f32x16 &ds, const Bias &b, float *room, int base)       // d = base - row + column
    {
        const int lane = threadIdx.x & 63;
        if (b.column >= 0) {
            if (b.column != column) {
                flush();
                column = b.column;
            }
            float some[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 16; ++i) some[i & 3] += ds[i];
            run += (some[0] + some[1]) + (some[2] + some[3]);
            return;
        }
        const int half = lane >> 5, col = min(lane, kSkewed - 1);
        float *to = room + 4 * half * (kSkewed + 1) + 31 - (lane & 31);
        float diagonal[2];
#pragma unroll
        for (int part = 0; part < 2; ++part) {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[(8 * (i >> 2) + (i & 3)) * (kSkewed + 1)] = ds[8 * part + i];
            __builtin_amdgcn_wave_barrier();
            float some[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int row = 0; row < 16; ++row) some[row & 3] += room[row * kSkewed + col];
            __builtin_amdgcn_wave_barrier();
            diagonal[part] = lane < kSkewed ? (some[0] + some[1]) + (some[2] + some[3]) : 0.f;
        }
        const float second = of_lane(diagonal[1], lane - 16);
        const float sums = scan_of_column(diagonal[0] + (lane >= 16 ? second : 0.f), b.diagonal);     // lane: row - column + 31
        const int zero = base + 31;                                                       // the lane of distance 0
        const int before = __shfl_up(F.border, 1), begin = lane == 0 ? 0 : before, end = F.border;       // of the lane's bucket
        auto last_of = [&](int from, int to) {                                            // the sum of lanes from .. to
            to = min(to, 62);
            const float sum = of_lane(sums, to);
            return max(from, 0) <= to ? sum : 0.f;
        };
        if (zero >= 0 || !F.two_sided) past += last_of(zero - end + 1, lane == 0 && !F.two_sided ? 62 : zero - begin);
        if (zero < 62 && F.two_sided) ahead += last_of(zero + max(begin, 1), zero + end - 1);
    }
    // all waves' sums, one float a column
    template <int FORM>
    __device__ __forceinline__ void leave(const Form<FORM> &F, int buckets, float (*meeting)[2 * kMaxBuckets], float *to)
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, columns = F.two_sided ? 2 * buckets : buckets;
        flush();
        if (lane < buckets) {
            meeting[wave][lane] = past;
            if (F.two_sided) meeting[wave][buckets + lane] = ahead;
        }
        __syncthreads();
        if ((int)threadIdx.x < columns) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kAttnThreads / 64; ++w) sum += meeting[w][threadIdx.x];
            to[threadIdx.x] = sum;
        }
    }
};

// The forward pass.  Four waves of 32 queries: with two tiles of keys and values in LDS two workgroups fit a compute unit up to heads of 128, which is
// what covers the copies' latency and the softmax of one by the products of the other.  8192 causal tokens, 32 heads of 128 on 8: 595 us,
// 920 TFLOP/s, bound by the chip's power (zeros: 1230); two sequences of 4096, not causal, 935; 4 x 2048 causal, 32 heads of 80:
// 140 to 153 us by card, 600 (80 is padded to 96 in the second product; 17 tiles a workgroup pay for its start and for what lies behind the diagonal in two).
template <int KS, int FORM>
__global__ void __launch_bounds__(kAttnThreads, waves_of(KS, FORM)) attention_kernel(const AttnArgs A)
{
    constexpr bool SCORED = FORM != kPlain, kCapped = has_cap(FORM), kTabled = has_table(FORM), kSloped = has_slope(FORM), kBiased = kTabled || kSloped, kLate = late(FORM);
    constexpr int DB = blocks_of(KS), PITCH = pitch_of(KS), kTile = tile_bytes(KS);
    __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTile];       // K, V; two tiles each
    __shared__ float biases[kTabled ? kAttnThreads / 64 : 1][kBiasRoom];
    // Few queries of heads that share keys: a tile's rows are pack heads of each query, so that a tile of keys is read and multiplied once for all of them
    // (one token of 5 sequences behind 4001, 32 heads of 128 on 8: 30 us head by head, 20 so, 15 by attention_few_kernel).
    constexpr bool kPacks = packs(FORM);
    const int pack = kPacks ? A.pack : 1;
    Place at;
    if (!pick(A, pack > 1 ? A.kv_heads : A.heads, at)) return;
    const int b = at.b, tile = at.tile;
    const Sequence seq = sequence_of(A, b);
    const int rows = seq.q_len * pack;
    if (tile * kOwnRows >= rows) return;
    const Mask<SCORED> M = mask_of<SCORED>(A, seq, b);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int first_row = tile * kOwnRows, last_row = min(first_row + kOwnRows, rows) - 1;
    const int w_row = first_row + wave * kWaveRows, w_end = min(w_row + kWaveRows, rows) - 1, row = w_row + (lane & 31);
    int q_first = first_row, q_last = last_row, w_first = w_row, w_last = w_end;       // the queries; of the wave: none where last < first
    int query = row, head = at.head, kv = head / A.group;
    if (pack > 1) {
        q_first = first_row / pack;
        q_last = last_row / pack;
        w_first = w_row / pack;
        w_last = w_end < w_row ? w_first - 1 : w_end / pack;
        query = row / pack;
        kv = at.head;
        head = kv * pack + row - query * pack;
    }
    const Tiles<KS> K(Rows{A.k + seq.k0 * A.k_row + kv * A.k_head, A.k_row, seq.k_len, A.dim});
    const Tiles<KS> V(Rows{A.v + seq.k0 * A.v_row + kv * A.v_head, A.v_row, seq.k_len, A.dim});
    const KeyTiles<SCORED> tiles(A, M, q_first, q_last, at.part);
    const unsigned lds_at = (unsigned)(size_t)(LDS_AS unsigned char *)lds;

    if (tiles.first < tiles.end) {
        K.bring(tiles.first, lds_at);
        V.bring(tiles.first, lds_at + 2 * kTile);
    }
    half8 own[KS];
    if (pack > 1) load_row<KS>(A.q + (seq.q0 + query) * A.q_row + head * A.q_head, row < rows, A.dim, own);
    else load_own<KS>(Rows{A.q + seq.q0 * A.q_row + head * A.q_head, A.q_row, seq.q_len, A.dim}, w_first, own);
    const Span seen(M.first_key(query), M.end_key(query));
    f32x16 out[DB];
    clear(out);
    [[maybe_unused]] const auto form = form_of<FORM>(A, head);
    float c = A.scale * kLog2e;
    if constexpr (SCORED) c = form.unit;
    float top = -INFINITY, sum = 0.f;                        // top: what the exponents are taken against, within 8 of the largest so far
    int buffer = 0;
    for (int k0 = tiles.first; k0 < tiles.end; k0 = tiles.after(k0), buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        meet();                                              // the tile is there, and the other one has been read by every wave
        if (tiles.after(k0) < tiles.end) {
            K.bring(tiles.after(k0), lds_at + (buffer ^ 1) * kTile);
            V.bring(tiles.after(k0), lds_at + (2 + (buffer ^ 1)) * kTile);
        }
        if (w_last < w_first || !M.any(w_first, w_last, k0, k0 + kTileRows - 1)) continue;
        const unsigned char *kt = lds + buffer * kTile, *vt = lds + (2 + buffer) * kTile;
        f32x16 s[2];
        clear(s);
        [[maybe_unused]] Bias bias = {kSame, -1, 0, -1, 0.f, 0.f, 0.f};
        if constexpr (kBiased && !kLate) {
            const int base = w_first + M.shift - k0;
            if (kPacks && pack > 1) bias = form.template plan<kTileRows, -1>(nullptr, base, query + M.shift - k0, (w_row + kWaveRows - 1) / pack - w_first);
            else bias = form.template plan<kTileRows, -1>(biases[kTabled ? wave : 0], base);
            if (form.starts(bias)) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) s[kb] = form.biases(bias, biases[kTabled ? wave : 0], kb);
            }
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(kt, kb, ks), own[ks], s[kb], 0, 0, 0);
        if constexpr (kLate) bias = form.template plan<kTileRows, -1>(biases[wave], w_first + M.shift - k0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            if constexpr (kCapped)
                if (form.capped) s[kb] = form.tanhs(s[kb]);
            if constexpr (kBiased)
                if (kLate || form.capped) s[kb] = form.with_bias(s[kb], bias, biases[kTabled ? wave : 0], kb);
        }
        if (!M.all(w_first, w_last, k0, k0 + kTileRows - 1)) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][i] = seen.holds(k0 + 32 * kb + acc_row(i)) || M.early(k0 + 32 * kb + acc_row(i)) ? s[kb][i] : -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) most = fmaxf(most, s[i >> 4][i & 15]);
        most = fmaxf(most, other_half(most));
        if constexpr (kBiased) most += bias.same;
        // Only where a row's largest score passes what its exponents are taken against by 2^8 are the sums so far brought down: P stays
        // below 2^8 otherwise, which fp16 holds as well as numbers below 1.
        if (__ballot(kSloped ? (most - top) * c > 8.f : most * c > top * c + 8.f)) {
            const float next = fmaxf(top, most);
            const float down = next == top ? 1.f : __builtin_amdgcn_exp2f((top - next) * c);
            top = next;
            sum *= down;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) out[db][i] *= down;
        }
        float against = top == -INFINITY ? 0.f : top * c;    // a row that has seen no key yet
        if constexpr (kBiased) against -= bias.same * c;
        if constexpr (kSloped) from_top(s, top, against);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[kb][i] = __builtin_amdgcn_exp2f(fmaf(s[kb][i], c, -against));
                sum += s[kb][i];
            }
#pragma unroll
        for (int step = 0; step < 4; ++step) {
            const half8 p = to_half8(s[step >> 1], 8 * (step & 1));
#pragma unroll
            for (int db = 0; db < DB; ++db) out[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_columns<PITCH>(vt, step, db), p, out[db], 0, 0, 0);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    sum += other_half(sum);
    if (A.splits > 1) {
        leave<DB>(A.parts, at.slot, wave, row, rows, out);
        if (lane < 32) A.part_stats[(at.slot * 4 + wave) * 32 + lane] = f32x2{top * c, sum};
        return;
    }
    const float factor = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;      // a row that sees no key: zero; NaN stays
    if (pack > 1) store_own<DB>(A.out + (seq.q0 + query) * A.out_row + head * A.out_head, 0, row < rows ? 0 : 1, 1, A.dim, out, factor);
    else store_own<DB>(A.out + seq.q0 * A.out_row + head * A.out_head, A.out_row, query, seq.q_len, A.dim, out, factor);
    if (lane < 32 && row < rows) A.lse[(int64_t)head * A.q_tokens + seq.q0 + query] = sum == 0.f ? -INFINITY : (SCORED ? top * c * kLn2 : top * A.scale) + __logf(sum);
}

// The forward pass of at most 32 rows: a token, or a few, of one sequence, with the heads that share their keys (pack).  The four waves of a workgroup have
// the same rows and every fourth tile of the part's keys each, which they copy for themselves, multiply and wait for by themselves: with
// rows for one wave alone it is the chain of a tile (copy, product, softmax, product) that takes the time, and here four go on at once.  The next tile's
// keys are under way from the first product on, its values from the second.  The waves' sums meet in LDS, the parts' in attention_join_kernel.
template <int KS, int FORM>
__global__ void __launch_bounds__(kAttnThreads) attention_few_kernel(const AttnArgs A)
{
    constexpr bool kCapped = has_cap(FORM), kTabled = has_table(FORM), kSloped = has_slope(FORM), kBiased = kTabled || kSloped;
    constexpr bool kPacks = packs(FORM);
    constexpr int DB = blocks_of(KS), PITCH = pitch_of(KS), kTile = tile_bytes(KS), kWaves = kAttnThreads / 64;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kWaves][2 * kTile];            // a wave's K, V
    __shared__ float biases[kTabled ? kWaves : 1][kBiasRoom];
    __shared__ f32x2 stats[kWaves][kWaveRows];
    static_assert(DB * 4096 <= 2 * kTile && DB <= kWaves, "a wave's sums lie where its tiles were, and a wave joins 32 dims");
    const int pack = kPacks ? A.pack : 1;
    Place at;
    if (!pick(A, pack > 1 ? A.kv_heads : A.heads, at)) return;
    const Sequence seq = sequence_of(A, at.b);
    const int rows = seq.q_len * pack;
    if (rows == 0) return;
    const Mask<true> M = mask_of<true>(A, seq, at.b);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, row = lane & 31, query = row / pack;
    const int kv = pack > 1 ? at.head : at.head / A.group, head = pack > 1 ? kv * pack + row - query * pack : at.head, last = (rows - 1) / pack;
    const OwnTiles<KS> K = {Rows{A.k + seq.k0 * A.k_row + kv * A.k_head, A.k_row, seq.k_len, A.dim}};
    const OwnTiles<KS> V = {Rows{A.v + seq.k0 * A.v_row + kv * A.v_head, A.v_row, seq.k_len, A.dim}};
    const KeyTiles<true> tiles(A, M, 0, last, at.part);
    const unsigned char *kt = lds[wave], *vt = kt + kTile;
    const unsigned lds_at = (unsigned)(size_t)(LDS_AS unsigned char *)lds + wave * 2 * kTile;
    half8 own[KS];
    load_row<KS>(A.q + (seq.q0 + query) * A.q_row + head * A.q_head, row < rows, A.dim, own);
    const auto form = form_of<FORM>(A, head < A.heads ? head : A.heads - 1);
    if (wave < tiles.count) {
        K.bring(tiles.at(wave), lds_at);
        V.bring(tiles.at(wave), lds_at + kTile);
    }
    const Span seen(M.first_key(query), M.end_key(query));
    const float c = form.unit;
    f32x16 out[DB];
    clear(out);
    float top = -INFINITY, sum = 0.f;
    for (int n = wave; n < tiles.count; n += kWaves) {
        const int k0 = tiles.at(n);
        const bool more = n + kWaves < tiles.count;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(OwnTiles<KS>::kWhole) : "memory");       // but for the values, which were asked for last
        f32x16 s[2];
        clear(s);
        [[maybe_unused]] Bias bias = {kSame, -1, 0, -1, 0.f, 0.f, 0.f};
        if constexpr (kBiased) {
            const int base = M.shift - k0;
            if (pack > 1) bias = form.template plan<kTileRows, -1>(nullptr, base, query + base, (kWaveRows - 1) / pack);
            else bias = form.template plan<kTileRows, -1>(biases[kTabled ? wave : 0], base);
            if (form.starts(bias)) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) s[kb] = form.biases(bias, biases[kTabled ? wave : 0], kb);
            }
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(kt, kb, ks), own[ks], s[kb], 0, 0, 0);
        if (more) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                             // the keys have been read
            K.bring(tiles.at(n + kWaves), lds_at);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            if constexpr (kCapped)
                if (form.capped) s[kb] = form.tanhs(s[kb]);
            if constexpr (kBiased)
                if (form.capped) s[kb] = form.with_bias(s[kb], bias, biases[kTabled ? wave : 0], kb);
        }
        if (!M.all(0, last, k0, k0 + kTileRows - 1)) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][i] = seen.holds(k0 + 32 * kb + acc_row(i)) || M.early(k0 + 32 * kb + acc_row(i)) ? s[kb][i] : -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) most = fmaxf(most, s[i >> 4][i & 15]);
        most = fmaxf(most, other_half(most));
        if constexpr (kBiased) most += bias.same;
        const float next = fmaxf(top, most), down = next == top ? 1.f : __builtin_amdgcn_exp2f((top - next) * c);
        top = next;
        sum *= down;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) out[db][i] *= down;
        float against = top == -INFINITY ? 0.f : top * c;
        if constexpr (kBiased) against -= bias.same * c;
        if constexpr (kSloped) from_top(s, top, against);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[kb][i] = __builtin_amdgcn_exp2f(fmaf(s[kb][i], c, -against));
                sum += s[kb][i];
            }
        if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(OwnTiles<KS>::kWhole) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int step = 0; step < 4; ++step) {
            const half8 p = to_half8(s[step >> 1], 8 * (step & 1));
#pragma unroll
            for (int db = 0; db < DB; ++db) out[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_columns<PITCH>(vt, step, db), p, out[db], 0, 0, 0);
        }
        if (more) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            V.bring(tiles.at(n + kWaves), lds_at + kTile);
        }
    }
    sum += other_half(sum);
    if (lane < kWaveRows) stats[wave][lane] = f32x2{top * c, sum};
    f32x4 *mine = reinterpret_cast<f32x4 *>(lds[wave]) + lane;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) mine[(4 * db + g) * 64] = f32x4{out[db][4 * g], out[db][4 * g + 1], out[db][4 * g + 2], out[db][4 * g + 3]};
    __syncthreads();
    if (wave >= DB) return;
    // 32 dims of all rows: the waves' sums, weighed by how far their exponents were taken down
    f32x16 all[1];
    clear(all);
    top = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = stats[w][row][1] != 0.f ? fmaxf(top, stats[w][row][0]) : top;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const f32x2 stat = stats[w][row];
        const float weight = stat[1] != 0.f ? __builtin_amdgcn_exp2f(stat[0] - top) : 0.f;
        sum = fmaf(stat[1], weight, sum);
        const f32x4 *from = reinterpret_cast<const f32x4 *>(lds[w]) + 4 * wave * 64 + lane;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 x = from[g * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) all[0][4 * g + e] = fmaf(x[e], weight, all[0][4 * g + e]);
        }
    }
    if (row >= rows) return;
    if (A.splits > 1) {
        f32x4 *to = sums_of<DB>(A.parts, at.slot, 0) + 4 * wave * 64;
#pragma unroll
        for (int g = 0; g < 4; ++g) to[g * 64] = f32x4{all[0][4 * g], all[0][4 * g + 1], all[0][4 * g + 2], all[0][4 * g + 3]};
        if (wave == 0 && lane < kWaveRows) A.part_stats[at.slot * 4 * kWaveRows + lane] = f32x2{top, sum};
        return;
    }
    const float factor = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    store_own<1>(A.out + (seq.q0 + query) * A.out_row + head * A.out_head + 32 * wave, 0, 0, 1, A.dim - 32 * wave, all, factor);
    if (wave == 0 && lane < kWaveRows) A.lse[(int64_t)head * A.q_tokens + seq.q0 + query] = sum == 0.f ? -INFINITY : top * kLn2 + __logf(sum);
}

// dQ, and delta on the way: three products a tile.  delta is formed from out as it was stored, since one of more bits would be twice its bytes in both passes.
// Its error is the same for all keys of a query, and adds most where they are few and to a table's sums of dz (0.0004 of the whole; one rounding is 0.0002).
// 8192 causal tokens, 32 heads of 128 on 8: 825 us, 1000 TFLOP/s; 4 x 2048, 32 heads of 80: 180 us.
template <int KS, int FORM>
__global__ void __launch_bounds__(kAttnThreads, waves_of(KS, FORM)) attention_dq_kernel(const AttnArgs A)
{
    constexpr bool SCORED = FORM != kPlain, kCapped = has_cap(FORM), kTabled = has_table(FORM), kBiased = kTabled || has_slope(FORM), kLate = late(FORM);
    constexpr int DB = blocks_of(KS), PITCH = pitch_of(KS), kTile = tile_bytes(KS);
    __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTile];
    __shared__ float biases[kTabled ? kAttnThreads / 64 : 1][kBiasRoom];
    __shared__ float skewed[kTabled ? kAttnThreads / 64 : 1][kSkewRoom];
    __shared__ float meeting[kTabled ? kAttnThreads / 64 : 1][2 * kMaxBuckets];
    Place at;
    if (!pick(A, A.heads, at)) return;
    const int b = at.b, head = at.head, tile = at.tile;
    const Sequence seq = sequence_of(A, b);
    const int columns = kTabled ? (A.form.two_sided ? 2 : 1) * A.form.buckets : 0;
    if (tile * kOwnRows >= seq.q_len) {                      // nothing to the table's gradient
        if (kTabled && A.form.dtable_parts && (int)threadIdx.x < columns) A.form.dtable_parts[at.slot * columns + threadIdx.x] = 0.f;
        return;
    }
    const Mask<SCORED> M = mask_of<SCORED>(A, seq, b);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int q_first = tile * kOwnRows, q_last = min(q_first + kOwnRows, seq.q_len) - 1;
    const int w_first = q_first + wave * kWaveRows, w_last = min(w_first + kWaveRows, seq.q_len) - 1;
    const int query = w_first + (lane & 31);
    const int kv = head / A.group;
    const Rows Q = {A.q + seq.q0 * A.q_row + head * A.q_head, A.q_row, seq.q_len, A.dim};
    const Tiles<KS> K(Rows{A.k + seq.k0 * A.k_row + kv * A.k_head, A.k_row, seq.k_len, A.dim});
    const Tiles<KS> V(Rows{A.v + seq.k0 * A.v_row + kv * A.v_head, A.v_row, seq.k_len, A.dim});
    const Rows DO = {A.dout + seq.q0 * A.dout_row + head * A.dout_head, A.dout_row, seq.q_len, A.dim};
    const Rows O = {A.out + seq.q0 * A.out_row + head * A.out_head, A.out_row, seq.q_len, A.dim};
    const KeyTiles<SCORED> tiles(A, M, q_first, q_last, at.part);
    const unsigned lds_at = (unsigned)(size_t)(LDS_AS unsigned char *)lds;
    if (tiles.first < tiles.end) {
        K.bring(tiles.first, lds_at);
        V.bring(tiles.first, lds_at + 2 * kTile);
    }
    half8 own[KS], down[KS];
    load_own<KS>(Q, w_first, own);
    load_own<KS>(DO, w_first, down);
    float delta = 0.f;
    {
        half8 o[KS];
        load_own<KS>(O, w_first, o);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)o[ks][e], (float)down[ks][e], delta);
        delta += other_half(delta);
    }
    const int64_t stat = (int64_t)head * A.q_tokens + seq.q0 + query;
    [[maybe_unused]] const auto form = form_of<FORM>(A, head);
    [[maybe_unused]] BucketSums buckets;
    if constexpr (kTabled)
        if (A.form.dtable_parts) buckets.start(skewed[wave]);
    float c = A.scale * kLog2e;
    if constexpr (SCORED) c = form.unit;
    float lse = SCORED ? INFINITY : 0.f;                     // behind the rows P is zero, whatever the bias: the table's sums run over all lanes
    if (query < seq.q_len) {
        lse = A.lse[stat] * kLog2e;
        if (lane < 32 && at.part == 0) A.delta[stat] = delta;
    }
    const Span seen(M.first_key(query), M.end_key(query));
    f32x16 acc[DB];
    clear(acc);
    int buffer = 0;
    for (int k0 = tiles.first; k0 < tiles.end; k0 = tiles.after(k0), buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        meet();
        if (tiles.after(k0) < tiles.end) {
            K.bring(tiles.after(k0), lds_at + (buffer ^ 1) * kTile);
            V.bring(tiles.after(k0), lds_at + (2 + (buffer ^ 1)) * kTile);
        }
        const unsigned char *kt = lds + buffer * kTile, *vt = lds + (2 + buffer) * kTile;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const int k1 = k0 + 32 * kb;
            if (k1 >= seq.k_len || w_last < w_first || !M.any(w_first, w_last, k1, k1 + 31)) continue;
            f32x16 s[1], dp[1];
            clear(s);
            clear(dp);
            [[maybe_unused]] Bias bias = {kSame, -1, 0, -1, 0.f, 0.f, 0.f};
            float less = lse;
            if constexpr (kBiased && !kLate) {
                bias = form.template plan<32, -1>(biases[kTabled ? wave : 0], w_first + M.shift - k1);
                if (form.starts(bias)) s[0] = form.biases(bias, biases[kTabled ? wave : 0], 0);
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(kt, kb, ks), own[ks], s[0], 0, 0, 0);
                dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(vt, kb, ks), down[ks], dp[0], 0, 0, 0);
            }
            [[maybe_unused]] f32x16 t;
            if constexpr (kLate) bias = form.template plan<32, -1>(biases[wave], w_first + M.shift - k1);
            if constexpr (kCapped)
                if (form.capped) s[0] = t = form.tanhs(s[0]);
            if constexpr (kBiased) {
                if (kLate || form.capped) s[0] = form.with_bias(s[0], bias, biases[kTabled ? wave : 0], 0);
                less = fmaf(-bias.same, c, lse);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] = __builtin_amdgcn_exp2f(fmaf(s[0][i], c, -less)) * (dp[0][i] - delta);
            if (!M.all(w_first, w_last, k1, k1 + 31)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[0][i] = seen.holds(k1 + acc_row(i)) || M.early(k1 + acc_row(i)) ? s[0][i] : 0.f;
            }
            if constexpr (kTabled)
                if (A.form.dtable_parts) buckets.add(form, s[0], bias, skewed[wave], w_first + M.shift - k1);
            if constexpr (kCapped)
                if (form.capped) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[0][i] *= fmaf(-t[i], t[i], 1.f);
                }
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                const half8 ds = to_half8(s[0], 8 * step);
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_columns<PITCH>(kt, 2 * kb + step, db), ds, acc[db], 0, 0, 0);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (kTabled) {
        if (A.form.dtable_parts) buckets.leave(form, A.form.buckets, meeting, A.form.dtable_parts + at.slot * columns);
    }
    if (A.splits > 1) leave<DB>(A.parts, at.slot, wave, query, seq.q_len, acc);
    else store_own<DB>(A.dq + seq.q0 * A.dq_row + head * A.dq_head, A.dq_row, query, seq.q_len, A.dim, acc, A.scale);
}

// lse, or delta, of the 64 queries of a tile to LDS, by one wave; what is behind the rows as `behind`.
__device__ __forceinline__ void copy_stats(const float *from, int first, int count, const float *behind, unsigned lds_at)
{
    const int at = first + (threadIdx.x & 63);
    const float *p = at < count ? from + at : behind;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(p), "s"(lds_at) : "memory");
}
__device__ const float infinite_lse[1] = {INFINITY};         // a probability of zero

// dK and dV: 128 keys to a workgroup, 32 to a wave; the queries of every head that shares the keys come by.  With SIDES = 2 a wave and the one four behind it
// have the same keys, one takes the first 32 queries of every tile and the other the last, and their sums meet in LDS at the end: a workgroup's time
// counts as much as the device's, under a causal mask the first keys are seen by every query (8192 tokens, 32 heads of 128, 8 of keys: with
// four waves the longest of 512 workgroups took 1.8 ms by itself; the whole backward pass 2414 -> 2090 us).
// Four products a tile: 1220 us for those 8192 tokens, 900 TFLOP/s; 4 x 2048, 32 heads of 80 (one wave to its keys): 240 us.
// Two waves to a SIMD have 256 registers each.  Heads of more than 96 fill half of them with their sums: there the rows of V stay in LDS, from where
// they are read for every block.
// So do the rows of K where the scores are of another form, which takes registers of its own: 8192 tokens in 4, 32 heads of 128 on 8, both passes, us, with K in
// registers / in LDS: slopes 753 / 734, capped 860 / 827, 32 buckets 909 / 799, capped with slopes 1114 (in part spilled) / 828.
// What still spills: a cap with a table 1 or 2 registers of heads of 65 to 80, 10 (6 where two waves share) of 81 to 96, 2 of more; a cap with slopes 1, all
// three 2 and 6 of 81 to 96; dQ of all three 6 of heads above 96.
template <int KS, int SIDES, int FORM>
__global__ void __launch_bounds__(SIDES * kAttnThreads, 2) attention_dkv_kernel(const AttnArgs A)
{
    constexpr bool SCORED = FORM != kPlain, kCapped = has_cap(FORM), kTabled = has_table(FORM), kBiased = kTabled || has_slope(FORM), kLate = late(FORM);
    constexpr bool kWide = KS > 6, kLean = kWide && FORM != kPlain;
    constexpr int DB = blocks_of(KS), PITCH = pitch_of(KS), kTile = tile_bytes(KS);
    __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTile + (kWide + kLean) * kOwnRows * PITCH];       // Q, dO; two tiles each; V, K
    __shared__ __attribute__((aligned(16))) float stats[2][2][kTileRows];         // lse, delta
    __shared__ float biases[kTabled ? SIDES * kAttnThreads / 64 : 1][kBiasRoom];
    Place at;
    if (!pick(A, A.kv_heads, at)) return;
    const int b = at.b, kv = at.head, tile = A.tiles - 1 - at.tile;        // the first keys are seen by the most queries
    const Sequence seq = sequence_of(A, b);
    if (tile * kOwnRows >= seq.k_len) return;
    const Mask<SCORED> M = mask_of<SCORED>(A, seq, b);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, side = wave >> 2;
    const int k_first = tile * kOwnRows, k_last = min(k_first + kOwnRows, seq.k_len) - 1;
    const int w_first = k_first + (wave & 3) * kWaveRows, w_last = min(w_first + kWaveRows, seq.k_len) - 1;
    const int key = w_first + (lane & 31);
    const Rows K = {A.k + seq.k0 * A.k_row + kv * A.k_head, A.k_row, seq.k_len, A.dim};
    const Rows V = {A.v + seq.k0 * A.v_row + kv * A.v_head, A.v_row, seq.k_len, A.dim};
    // Q and lse come by waves 0-3, dO and delta by 4-7 where there are such
    struct Coming {
        Tiles<KS> tiles;
        const _Float16 *base;
        int64_t apart;
        const float *stats, *behind;
    };
    auto coming_of = [&](int what) {
        const _Float16 *base = what ? A.dout + seq.q0 * A.dout_row : A.q + seq.q0 * A.q_row;
        return Coming{Tiles<KS>(Rows{base, what ? A.dout_row : A.q_row, seq.q_len, A.dim}), base, what ? A.dout_head : A.q_head,
                      (what ? A.delta : A.lse) + seq.q0, what ? reinterpret_cast<const float *>(zero_row) : infinite_lse};
    };
    Coming first_operand = coming_of(side), second_operand = coming_of(1);
    // the queries that see any of the workgroup's keys
    int q_first = 0, q_end = seq.q_len;
    if (M.causal && !M.early(k_first)) {
        const int begin = k_first - M.shift;
        q_first = begin > 0 ? begin / kTileRows * kTileRows : 0;
        const int64_t end = (int64_t)k_last - M.shift + M.window;
        q_end = end < q_end ? (int)(end > 0 ? end : 0) : q_end;
    }
    const int tiles = q_end > q_first ? (q_end - q_first + kTileRows - 1) / kTileRows : 0;
    // a part's share of the tiles of all heads
    const int all = tiles * A.group, each = (all + A.splits - 1) / A.splits, from = min(all, at.part * each), count = min(all - from, each);
    int shared = tiles ? from / tiles : 0, t = from - shared * tiles;
    const unsigned lds_at = (unsigned)(size_t)(LDS_AS unsigned char *)lds, stats_at = (unsigned)(size_t)(LDS_AS unsigned char *)stats;
    auto bring_one = [&](Coming &c, int what, int shared, int t, int buffer) {
        const int head = kv * A.group + shared, first = q_first + t * kTileRows;
        c.tiles.R.base = c.base + head * c.apart;
        c.tiles.bring(first, lds_at + (2 * what + buffer) * kTile);
        if ((wave & 3) == 0) copy_stats(c.stats + (int64_t)head * A.q_tokens, first, seq.q_len, c.behind, stats_at + (buffer * 2 + what) * kTileRows * 4);
    };
    auto bring = [&](int shared, int t, int buffer) {
        bring_one(first_operand, side, shared, t, buffer);
        if (SIDES == 1) bring_one(second_operand, 1, shared, t, buffer);
    };
    if (kWide)
        for (int part = side; part < 2; part += SIDES) {
            Tiles<KS>(V).bring(k_first + part * kTileRows, lds_at + 4 * kTile + part * kTileRows * PITCH);
            if (kLean) Tiles<KS>(K).bring(k_first + part * kTileRows, lds_at + 4 * kTile + (kOwnRows + part * kTileRows) * PITCH);
        }
    if (count > 0) bring(shared, t, 0);
    half8 own[kLean ? 1 : KS], ownv[kWide ? 1 : KS];
    if constexpr (!kLean) load_own<KS>(K, w_first, own);
    if constexpr (!kWide) load_own<KS>(V, w_first, ownv);
    const unsigned char *v_rows = lds + 4 * kTile + (wave & 3) * kWaveRows * PITCH, *k_rows = v_rows + kOwnRows * PITCH;
    const Span seen(M.first_query(key), M.end_query(key));
    f32x16 dk[DB], dv[DB];
    clear(dk);
    clear(dv);
    // P's exponents by the group's first head; the form of another is taken when its queries come
    [[maybe_unused]] auto form = form_of<FORM>(A, kv * A.group + min(shared, A.group - 1));
    float c = A.scale * kLog2e;
    if constexpr (SCORED) c = form.unit;
    int buffer = 0;
    for (int n = 0; n < count; ++n, buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        meet();
        const int q0 = q_first + t * kTileRows;
        if (SCORED && t == 0 && n > 0) form = form_of<FORM>(A, kv * A.group + shared);
        if (++t == tiles) {
            t = 0;
            ++shared;
        }
        if (n + 1 < count) bring(shared, t, buffer ^ 1);
        const unsigned char *qt = lds + buffer * kTile, *dot = lds + (2 + buffer) * kTile;
#pragma unroll
        for (int part = 0; part < 2 / SIDES; ++part) {
            const int qb = SIDES == 2 ? side : part;
            const int q1 = q0 + 32 * qb;
            if (q1 >= seq.q_len || w_last < w_first || !M.any(q1, q1 + 31, w_first, w_last)) continue;
            f32x16 s[1], dp[1];
            clear(s);
            clear(dp);
            [[maybe_unused]] Bias bias = {kSame, -1, 0, -1, 0.f, 0.f, 0.f};
            [[maybe_unused]] float more = 0.f;
            if constexpr (kBiased && !kLate) {
                bias = form.template plan<32, 1>(biases[kTabled ? wave : 0], q1 + M.shift - w_first);
                if (form.starts(bias)) s[0] = form.biases(bias, biases[kTabled ? wave : 0], 0);
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const half8 k = kLean ? read_rows<PITCH>(k_rows, 0, ks) : own[kLean ? 0 : ks];
                s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(qt, qb, ks), k, s[0], 0, 0, 0);
                const half8 v = kWide ? read_rows<PITCH>(v_rows, 0, ks) : ownv[kWide ? 0 : ks];
                dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(dot, qb, ks), v, dp[0], 0, 0, 0);
            }
            if constexpr (kLate) {
                bias = form.template plan<32, 1>(biases[wave], q1 + M.shift - w_first);
                if constexpr (!kCapped) s[0] = form.with_bias(s[0], bias, biases[wave], 0);
            }
            if constexpr (kBiased) more = bias.same * c;
            if constexpr (kCapped)
                if (form.capped) {                           // dP - delta, times the cap's slope
                    s[0] = form.tanhs(s[0]);
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 delta = *reinterpret_cast<const f32x4 *>(&stats[buffer][1][32 * qb + 8 * g + 4 * (lane >> 5)]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int i = 4 * g + e;
                            dp[0][i] = (dp[0][i] - delta[e]) * fmaf(-s[0][i], s[0][i], 1.f);
                        }
                    }
                    if constexpr (kBiased) s[0] = form.with_bias(s[0], bias, biases[kTabled ? wave : 0], 0);
                }
            [[maybe_unused]] bool reduced = false;           // whether delta has been taken off
            if constexpr (kCapped) reduced = form.capped;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int at = 32 * qb + 8 * g + 4 * (lane >> 5);
                const f32x4 lse = *reinterpret_cast<const f32x4 *>(&stats[buffer][0][at]), delta = *reinterpret_cast<const f32x4 *>(&stats[buffer][1][at]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * g + e;
                    s[0][i] = __builtin_amdgcn_exp2f(fmaf(s[0][i], c, kBiased ? fmaf(-lse[e], kLog2e, more) : -lse[e] * kLog2e));
                    dp[0][i] = s[0][i] * (kCapped && reduced ? dp[0][i] : dp[0][i] - delta[e]);
                }
            }
            if (!M.all(q1, q1 + 31, w_first, w_last)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool on = seen.holds(q1 + acc_row(i));
                    s[0][i] = on ? s[0][i] : 0.f;
                    dp[0][i] = on ? dp[0][i] : 0.f;
                }
            }
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                const half8 p = to_half8(s[0], 8 * step), ds = to_half8(dp[0], 8 * step);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_columns<PITCH>(dot, 2 * qb + step, db), p, dv[db], 0, 0, 0);
                    dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_columns<PITCH>(qt, 2 * qb + step, db), ds, dk[db], 0, 0, 0);
                }
            }
        }
    }
    if constexpr (SIDES == 2) {
        // a wave of the first four keeps dK and the one behind it dV: each gets the other's sums of it, kPart blocks of dims at a time
        constexpr int kPart = 4 * kTile / (8 * 4096);
        f32x4 *meeting = reinterpret_cast<f32x4 *>(lds) + lane;
        auto give = [&](const f32x16 (&acc)[DB], int first) {
#pragma unroll
            for (int i = 0; i < kPart && first + i < DB; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    meeting[(((wave ^ 4) * kPart + i) * 4 + g) * 64] = f32x4{acc[first + i][4 * g], acc[first + i][4 * g + 1], acc[first + i][4 * g + 2], acc[first + i][4 * g + 3]};
        };
        auto take = [&](f32x16 (&acc)[DB], int first) {
#pragma unroll
            for (int i = 0; i < kPart && first + i < DB; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 other = meeting[((wave * kPart + i) * 4 + g) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[first + i][4 * g + e] += other[e];
                }
        };
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int first = 0; first < DB; first += kPart) {
            __syncthreads();
            if (side) give(dk, first);
            else give(dv, first);
            __syncthreads();
            if (side) take(dv, first);
            else take(dk, first);
        }
    }
    if (A.splits > 1) {                                      // dK's sums, then dV's
        if (SIDES == 1 || side) leave<DB>(A.parts, 2 * at.slot + 1, wave & 3, key, seq.k_len, dv);
        if (SIDES == 1 || !side) leave<DB>(A.parts, 2 * at.slot, wave & 3, key, seq.k_len, dk);
        return;
    }
    if (SIDES == 1 || side) store_own<DB>(A.dv + seq.k0 * A.dv_row + kv * A.dv_head, A.dv_row, key, seq.k_len, A.dim, dv, 1.f);
    if (SIDES == 1 || !side) store_own<DB>(A.dk + seq.k0 * A.dk_row + kv * A.dk_head, A.dk_row, key, seq.k_len, A.dim, dk, A.scale);
}

// The workgroups of dK and dV from which a wave has its keys for itself; below, where the longest workgroup is what the call waits for, two share them.
// Whole backward pass of heads of 64, one wave / two, us: 32 workgroups, 512 tokens of 8 heads 31 / 29; 256, 2048 of 16 heads 76 / 75; 512,
// two times 2048 of 16 heads 111 / 103; 512, 16384 of 16 heads on 4 2108 / 2204; 1024, 8192 in 16 sequences of 16 heads 73 / 86; 2048, 8192 of 32
// heads 1064 / 1132.  Of 80: 1024 workgroups 94 / 113, 2048 1395 / 1495, but 512 long ones 3651 / 2935; of 96 101 / 120, 1506 / 1584, 3947 / 3105.
// Heads of more than 96 always share: V's rows in LDS leave room for one workgroup.
constexpr int one_side_from(int dim) { return dim <= 64 ? 512 : dim <= 96 ? 1024 : INT32_MAX; }

// An XCD's workgroups, as pick() deals them; heads and sequences are fewer than 2^31 together.
int64_t places_of(int64_t all, int64_t tiles)
{
    const int share = heads_an_xcd((int)all);
    return share ? share * tiles : ceil_div(all * tiles, 8);
}

// The kernel of a launch, without what joins its parts.
template <int KS, int FORM>
hipError_t launch_dim(int which, const AttnArgs &a, int64_t items, hipStream_t s)
{
    const dim3 grid((unsigned)(places_of(items / a.tiles, a.tiles) * a.splits * 8));
    if constexpr (FORM != kPlain)
        if (which == kForward && a.few) {
            hipLaunchKernelGGL((attention_few_kernel<KS, FORM>), grid, dim3(kAttnThreads), 0, s, a);
            return hipGetLastError();
        }
    if (which == kForward) hipLaunchKernelGGL((attention_kernel<KS, FORM>), grid, dim3(kAttnThreads), 0, s, a);
    else if (which == kDq) hipLaunchKernelGGL((attention_dq_kernel<KS, FORM>), grid, dim3(kAttnThreads), 0, s, a);
    else if (KS <= 6 && items * a.splits >= one_side_from(a.dim))
        hipLaunchKernelGGL((attention_dkv_kernel<KS, KS <= 6 ? 1 : 2, FORM>), grid, dim3(kAttnThreads), 0, s, a);
    else hipLaunchKernelGGL((attention_dkv_kernel<KS, 2, FORM>), grid, dim3(2 * kAttnThreads), 0, s, a);
    return hipGetLastError();
}

template <int FORM>
hipError_t launch_form(int which, const AttnArgs &a, int64_t items, hipStream_t s)
{
    switch ((a.dim + 15) / 16) {                             // padded: a kernel for each of the sizes in use, and the next one up for the others
    case 1: case 2: return launch_dim<2, FORM>(which, a, items, s);
    case 3: case 4: return launch_dim<4, FORM>(which, a, items, s);
    case 5: return launch_dim<5, FORM>(which, a, items, s);
    case 6: return launch_dim<6, FORM>(which, a, items, s);
    default: return launch_dim<8, FORM>(which, a, items, s);
    }
}

}  // namespace
}  // namespace samo
