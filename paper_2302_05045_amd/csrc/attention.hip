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

// A part's share of the tiles first .. end: whole tiles of 64, in order.
__device__ __forceinline__ void share_of(const AttnArgs &A, int part, int &first, int &end)
{
    const int tiles = end > first ? (end - first + kTileRows - 1) / kTileRows : 0, each = (tiles + A.splits - 1) / A.splits;
    first += min(tiles, part * each) * kTileRows;
    end = min(end, first + each * kTileRows);
}

// Which keys a query sees: first_key(query) .. end_key(query) - 1, all of them without `causal`; and which queries see a key.
struct Mask {
    bool causal;
    int shift, window, q_len, k_len;         // window 2^30: none
    __device__ __forceinline__ int first_key(int query) const { return causal ? query + shift - window + 1 : 0; }
    __device__ __forceinline__ int end_key(int query) const { return causal ? min(query + shift + 1, k_len) : k_len; }
    __device__ __forceinline__ int first_query(int key) const { return causal ? key - shift : 0; }
    __device__ __forceinline__ int end_query(int key) const { return causal ? min(key - shift + window, q_len) : q_len; }
    // whether all of / any of a block of queries and keys (first and last of each) are seen
    __device__ __forceinline__ bool all(int q0, int q1, int k0, int k1) const { return k1 < k_len && (!causal || (k1 <= q0 + shift && k0 > q1 + shift - window)); }
    __device__ __forceinline__ bool any(int q0, int q1, int k0, int k1) const { return !causal || (k0 <= q1 + shift && k1 > q0 + shift - window); }
};
// The numbers from .. end - 1 by one comparison.
struct Span {
    int from;
    unsigned count;
    __device__ __forceinline__ Span(int first, int end) : from(first), count(end > first ? (unsigned)(end - first) : 0u) {}
    __device__ __forceinline__ bool holds(int x) const { return (unsigned)(x - from) < count; }
};
__device__ __forceinline__ Mask mask_of(const AttnArgs &A, const Sequence &s)
{
    Mask m;
    m.causal = A.causal != 0;
    m.shift = s.k_len - s.q_len;
    m.window = A.window > 0 ? min(A.window, 1 << 30) : 1 << 30;
    m.q_len = s.q_len;
    m.k_len = s.k_len;
    return m;
}

// The tiles of keys that any of the queries q0 .. q1 sees: [first, end) in rows, first a multiple of the tile.
__device__ __forceinline__ void key_range(const Mask &M, int q0, int q1, int k_len, int &first, int &end)
{
    first = 0;
    end = k_len;
    if (M.causal) {
        const int last = q1 + M.shift + 1, begin = q0 + M.shift - M.window + 1;
        end = last < end ? last : end;
        first = begin > 0 ? begin / kTileRows * kTileRows : 0;
    }
}

// The forward pass.  Four waves of 32 queries: with two tiles of keys and values in LDS two workgroups fit a compute unit up to heads of 128, which is
// what covers the copies' latency and the softmax of one by the products of the other.  8192 causal tokens, 32 heads of 128 on 8: 595 us,
// 920 TFLOP/s, bound by the chip's power (zeros: 1230); two sequences of 4096, not causal, 935; 4 x 2048 causal, 32 heads of 80:
// 140 to 153 us by card, 600 (80 is padded to 96 in the second product; 17 tiles a workgroup pay for its start and for what lies behind the diagonal in two).
template <int KS>
__global__ void __launch_bounds__(kAttnThreads, 2) attention_kernel(const AttnArgs A)
{
    constexpr int DB = blocks_of(KS), PITCH = pitch_of(KS), kTile = tile_bytes(KS);
    __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTile];       // K, V; two tiles each
    Place at;
    if (!pick(A, A.heads, at)) return;
    const int b = at.b, head = at.head, tile = at.tile;
    const Sequence seq = sequence_of(A, b);
    if (tile * kOwnRows >= seq.q_len) return;
    const Mask M = mask_of(A, seq);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int q_first = tile * kOwnRows, q_last = min(q_first + kOwnRows, seq.q_len) - 1;
    const int w_first = q_first + wave * kWaveRows, w_last = min(w_first + kWaveRows, seq.q_len) - 1;   // of the wave; none where last < first
    const int query = w_first + (lane & 31);
    const int kv = head / A.group;
    const Rows Q = {A.q + seq.q0 * A.q_row + head * A.q_head, A.q_row, seq.q_len, A.dim};
    const Tiles<KS> K(Rows{A.k + seq.k0 * A.k_row + kv * A.k_head, A.k_row, seq.k_len, A.dim});
    const Tiles<KS> V(Rows{A.v + seq.k0 * A.v_row + kv * A.v_head, A.v_row, seq.k_len, A.dim});
    int k_first, k_end;
    key_range(M, q_first, q_last, seq.k_len, k_first, k_end);
    share_of(A, at.part, k_first, k_end);
    const unsigned lds_at = (unsigned)(size_t)(LDS_AS unsigned char *)lds;

    if (k_first < k_end) {
        K.bring(k_first, lds_at);
        V.bring(k_first, lds_at + 2 * kTile);
    }
    half8 own[KS];
    load_own<KS>(Q, w_first, own);
    const Span seen(M.first_key(query), M.end_key(query));
    f32x16 out[DB];
    clear(out);
    const float c = A.scale * kLog2e;
    float top = -INFINITY, sum = 0.f;                        // top: what the exponents are taken against, within 8 of the largest so far
    int buffer = 0;
    for (int k0 = k_first; k0 < k_end; k0 += kTileRows, buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        meet();                                              // the tile is there, and the other one has been read by every wave
        if (k0 + kTileRows < k_end) {
            K.bring(k0 + kTileRows, lds_at + (buffer ^ 1) * kTile);
            V.bring(k0 + kTileRows, lds_at + (2 + (buffer ^ 1)) * kTile);
        }
        if (w_last < w_first || !M.any(w_first, w_last, k0, k0 + kTileRows - 1)) continue;
        const unsigned char *kt = lds + buffer * kTile, *vt = lds + (2 + buffer) * kTile;
        f32x16 s[2];
        clear(s);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(kt, kb, ks), own[ks], s[kb], 0, 0, 0);
        if (!M.all(w_first, w_last, k0, k0 + kTileRows - 1)) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][i] = seen.holds(k0 + 32 * kb + acc_row(i)) ? s[kb][i] : -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) most = fmaxf(most, s[i >> 4][i & 15]);
        most = fmaxf(most, other_half(most));
        // Only where a row's largest score passes what its exponents are taken against by 2^8 are the sums so far brought down: P stays
        // below 2^8 otherwise, which fp16 holds as well as numbers below 1.
        if (__ballot(most * c > top * c + 8.f)) {
            const float next = fmaxf(top, most);
            const float down = next == top ? 1.f : __builtin_amdgcn_exp2f((top - next) * c);
            top = next;
            sum *= down;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) out[db][i] *= down;
        }
        const float against = top == -INFINITY ? 0.f : top * c;       // a row that has seen no key yet
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
        leave<DB>(A.parts, at.slot, wave, query, seq.q_len, out);
        if (lane < 32) A.part_stats[(at.slot * 4 + wave) * 32 + lane] = f32x2{top * c, sum};
        return;
    }
    const float factor = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;      // a row that sees no key: zero; NaN stays
    store_own<DB>(A.out + seq.q0 * A.out_row + head * A.out_head, A.out_row, query, seq.q_len, A.dim, out, factor);
    if (lane < 32 && query < seq.q_len) A.lse[(int64_t)head * A.q_tokens + seq.q0 + query] = sum == 0.f ? -INFINITY : top * A.scale + __logf(sum);
}

// dQ, and delta on the way: three products a tile.  8192 causal tokens, 32 heads of 128 on 8: 825 us, 1000 TFLOP/s; 4 x 2048, 32 heads of 80: 180 us.
template <int KS>
__global__ void __launch_bounds__(kAttnThreads, 2) attention_dq_kernel(const AttnArgs A)
{
    constexpr int DB = blocks_of(KS), PITCH = pitch_of(KS), kTile = tile_bytes(KS);
    __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTile];
    Place at;
    if (!pick(A, A.heads, at)) return;
    const int b = at.b, head = at.head, tile = at.tile;
    const Sequence seq = sequence_of(A, b);
    if (tile * kOwnRows >= seq.q_len) return;
    const Mask M = mask_of(A, seq);
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
    int k_first, k_end;
    key_range(M, q_first, q_last, seq.k_len, k_first, k_end);
    share_of(A, at.part, k_first, k_end);
    const unsigned lds_at = (unsigned)(size_t)(LDS_AS unsigned char *)lds;
    if (k_first < k_end) {
        K.bring(k_first, lds_at);
        V.bring(k_first, lds_at + 2 * kTile);
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
    const float c = A.scale * kLog2e;
    float lse = 0.f;
    if (query < seq.q_len) {
        lse = A.lse[stat] * kLog2e;
        if (lane < 32 && at.part == 0) A.delta[stat] = delta;
    }
    const Span seen(M.first_key(query), M.end_key(query));
    f32x16 acc[DB];
    clear(acc);
    int buffer = 0;
    for (int k0 = k_first; k0 < k_end; k0 += kTileRows, buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        meet();
        if (k0 + kTileRows < k_end) {
            K.bring(k0 + kTileRows, lds_at + (buffer ^ 1) * kTile);
            V.bring(k0 + kTileRows, lds_at + (2 + (buffer ^ 1)) * kTile);
        }
        const unsigned char *kt = lds + buffer * kTile, *vt = lds + (2 + buffer) * kTile;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const int k1 = k0 + 32 * kb;
            if (k1 >= seq.k_len || w_last < w_first || !M.any(w_first, w_last, k1, k1 + 31)) continue;
            f32x16 s[1], dp[1];
            clear(s);
            clear(dp);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(kt, kb, ks), own[ks], s[0], 0, 0, 0);
                dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(vt, kb, ks), down[ks], dp[0], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] = __builtin_amdgcn_exp2f(fmaf(s[0][i], c, -lse)) * (dp[0][i] - delta);
            if (!M.all(w_first, w_last, k1, k1 + 31)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[0][i] = seen.holds(k1 + acc_row(i)) ? s[0][i] : 0.f;
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
template <int KS, int SIDES>
__global__ void __launch_bounds__(SIDES * kAttnThreads, 2) attention_dkv_kernel(const AttnArgs A)
{
    constexpr bool kWide = KS > 6;
    constexpr int DB = blocks_of(KS), PITCH = pitch_of(KS), kTile = tile_bytes(KS);
    __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTile + (kWide ? kOwnRows * PITCH : 0)];       // Q, dO; two tiles each; V
    __shared__ __attribute__((aligned(16))) float stats[2][2][kTileRows];         // lse, delta
    Place at;
    if (!pick(A, A.kv_heads, at)) return;
    const int b = at.b, kv = at.head, tile = A.tiles - 1 - at.tile;        // the first keys are seen by the most queries
    const Sequence seq = sequence_of(A, b);
    if (tile * kOwnRows >= seq.k_len) return;
    const Mask M = mask_of(A, seq);
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
    if (M.causal) {
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
        for (int part = side; part < 2; part += SIDES) Tiles<KS>(V).bring(k_first + part * kTileRows, lds_at + 4 * kTile + part * kTileRows * PITCH);
    if (count > 0) bring(shared, t, 0);
    half8 own[KS], ownv[kWide ? 1 : KS];
    load_own<KS>(K, w_first, own);
    if constexpr (!kWide) load_own<KS>(V, w_first, ownv);
    const unsigned char *v_rows = lds + 4 * kTile + (wave & 3) * kWaveRows * PITCH;
    const Span seen(M.first_query(key), M.end_query(key));
    f32x16 dk[DB], dv[DB];
    clear(dk);
    clear(dv);
    const float c = A.scale * kLog2e;
    int buffer = 0;
    for (int n = 0; n < count; ++n, buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        meet();
        const int q0 = q_first + t * kTileRows;
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
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(qt, qb, ks), own[ks], s[0], 0, 0, 0);
                const half8 v = kWide ? read_rows<PITCH>(v_rows, 0, ks) : ownv[kWide ? 0 : ks];
                dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_rows<PITCH>(dot, qb, ks), v, dp[0], 0, 0, 0);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int at = 32 * qb + 8 * g + 4 * (lane >> 5);
                const f32x4 lse = *reinterpret_cast<const f32x4 *>(&stats[buffer][0][at]), delta = *reinterpret_cast<const f32x4 *>(&stats[buffer][1][at]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * g + e;
                    s[0][i] = __builtin_amdgcn_exp2f(fmaf(s[0][i], c, -lse[e] * kLog2e));
                    dp[0][i] = s[0][i] * (dp[0][i] - delta[e]);
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

// Whole rows from the sums of their parts, added in order: a wave has 32 rows, and 32 dims of them, as the kernel that left them had.
// Parts of out are weighed by how far their exponents were taken down; one that has seen no key is not read.
enum { kForward, kDq, kDkv };
template <int DB, int WHICH>
__global__ void __launch_bounds__(DB * 64) attention_join_kernel(const AttnArgs A)
{
    constexpr int kTensors = WHICH == kDkv ? 2 : 1;
    const int rows = (int)(blockIdx.x & 3), db = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, tensor = (int)blockIdx.y;
    const int item = (int)(blockIdx.x >> 2);
    const Place at = place_of(item / A.tiles, item % A.tiles, 0, A);
    const Sequence seq = sequence_of(A, at.b);
    const int count = WHICH == kDkv ? seq.k_len : seq.q_len, row = (WHICH == kDkv ? A.tiles - 1 - at.tile : at.tile) * kOwnRows + rows * kWaveRows + (lane & 31);
    if (row >= count) return;
    f32x16 acc[1];
    clear(acc);
    float top = -INFINITY, sum = 0.f;
    if (WHICH == kForward)
        for (int part = 0; part < A.splits; ++part) {
            const f32x2 stat = A.part_stats[((at.slot + part) * 4 + rows) * 32 + (lane & 31)];
            if (stat[1] != 0.f) top = fmaxf(top, stat[0]);
        }
    for (int part = 0; part < A.splits; ++part) {
        float weight = 1.f;
        if (WHICH == kForward) {
            const f32x2 stat = A.part_stats[((at.slot + part) * 4 + rows) * 32 + (lane & 31)];
            if (stat[1] == 0.f) continue;
            weight = __builtin_amdgcn_exp2f(stat[0] - top);
            sum = fmaf(stat[1], weight, sum);
        }
        const f32x4 *from = sums_of<DB>(A.parts, (at.slot + part) * kTensors + tensor, rows) + 4 * db * 64;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 x = from[g * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[0][4 * g + e] = fmaf(x[e], weight, acc[0][4 * g + e]);
        }
    }
    _Float16 *to;
    int64_t stride;
    float factor = A.scale;
    if (WHICH == kForward) {
        to = A.out + seq.q0 * A.out_row + at.head * A.out_head;
        stride = A.out_row;
        factor = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
        if (db == 0 && lane < 32) A.lse[(int64_t)at.head * A.q_tokens + seq.q0 + row] = sum == 0.f ? -INFINITY : top * kLn2 + __logf(sum);
    } else if (WHICH == kDq) {
        to = A.dq + seq.q0 * A.dq_row + at.head * A.dq_head;
        stride = A.dq_row;
    } else if (tensor == 0) {
        to = A.dk + seq.k0 * A.dk_row + at.head * A.dk_head;
        stride = A.dk_row;
    } else {
        to = A.dv + seq.k0 * A.dv_row + at.head * A.dv_head;
        stride = A.dv_row;
        factor = 1.f;
    }
    store_own<1>(to + 32 * db, stride, row, count, A.dim - 32 * db, acc, factor);
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

template <int KS>
hipError_t launch_dim(int which, const AttnArgs &a, int64_t items, hipStream_t s)
{
    constexpr int DB = blocks_of(KS);
    const dim3 grid((unsigned)(places_of(items / a.tiles, a.tiles) * a.splits * 8)), joins((unsigned)(items * 4), which == kDkv ? 2 : 1);
    if (which == kForward) hipLaunchKernelGGL((attention_kernel<KS>), grid, dim3(kAttnThreads), 0, s, a);
    else if (which == kDq) hipLaunchKernelGGL((attention_dq_kernel<KS>), grid, dim3(kAttnThreads), 0, s, a);
    else if (KS <= 6 && items * a.splits >= one_side_from(a.dim))
        hipLaunchKernelGGL((attention_dkv_kernel<KS, KS <= 6 ? 1 : 2>), grid, dim3(kAttnThreads), 0, s, a);
    else hipLaunchKernelGGL((attention_dkv_kernel<KS, 2>), grid, dim3(2 * kAttnThreads), 0, s, a);
    if (a.splits > 1) {
        if (hipError_t e = hipGetLastError()) return e;
        if (which == kForward) hipLaunchKernelGGL((attention_join_kernel<DB, kForward>), joins, dim3(DB * 64), 0, s, a);
        else if (which == kDq) hipLaunchKernelGGL((attention_join_kernel<DB, kDq>), joins, dim3(DB * 64), 0, s, a);
        else hipLaunchKernelGGL((attention_join_kernel<DB, kDkv>), joins, dim3(DB * 64), 0, s, a);
    }
    return hipGetLastError();
}

int64_t items_of(int which, const AttnArgs &a)
{
    return (int64_t)a.batch * (which == kDkv ? a.kv_heads : a.heads) * ceil_div(which == kDkv ? a.max_k : a.max_q, kOwnRows);
}

int blocks_of_dim(int dim) { return dim <= 32 ? 1 : dim <= 64 ? 2 : dim <= 96 ? 3 : 4; }

// Bytes of the sums that a launch leaves: 128 rows of fp32 a part, and the softmax's two numbers a row.
int64_t sums_bytes(int which, const AttnArgs &a, int splits)
{
    if (splits <= 1) return 0;
    const int64_t slots = items_of(which, a) * splits;
    return slots * kOwnRows * (which == kForward ? 32 * 4 * blocks_of_dim(a.dim) + 8 : (which == kDkv ? 2 : 1) * 32 * 4 * blocks_of_dim(a.dim));
}

// What a launch costs with its keys (for dK and dV: queries) in so many parts, us.  A workgroup works through tiles of 64; the device's share of all of them,
// and as the launch ends half the longest workgroup besides; the longest one by itself; and for parts a second kernel and the sums, written and read.
// A tile by itself takes 1.25 us with heads of 64 and 1.5 with 128, 1.4 and 2.3 where two workgroups share a compute unit; the backward pass's
// a quarter more.  Measured against the parts taken, whole calls, us: one token behind 8191, 32 heads of 128 on 8, 181 with one part, 36 with 8, 33 with 16;
// 2000 tokens in 3 sequences behind 3000 each, 16 heads of 64, 72 and 57 with three; 4096 tokens, 8 heads of 128, 89 and 59 with three; 1024 tokens of
// 16 heads of 96 23 and 25 with two, which it takes; 2048 in 4 sequences, 16 heads of 64, 13 and 23 with two; one token each behind 8 contexts of 2048, 32 heads of
// 128, 62, 50 with two and 57 with four.
// Where every workgroup has as much to do, the rounds that they take count whole.
double launch_us(int which, const AttnArgs &a, int64_t items, int splits)
{
    const bool dkv = which == kDkv, one_side = dkv && items * splits >= one_side_from(a.dim);
    const double q = (double)a.q_tokens / a.batch, k = (double)a.k_tokens / a.batch;
    double longest = dkv ? q : k, mean = 1.0;
    if (a.window) longest = std::min(longest, (double)a.window + kOwnRows);
    else if (a.causal) mean = 1.0 - 0.5 * std::min(1.0, q / std::max(k, 1.0));
    longest = std::ceil(longest / kTileRows) * (dkv ? a.group : 1);
    const double own = std::min((double)items, (double)(dkv ? a.kv_heads : a.heads) * ((double)(dkv ? a.k_tokens : a.q_tokens) / kOwnRows + a.batch));
    const double alone = (1.0 + 0.004 * a.dim) * (which == kForward ? 1.0 : 1.25), shared = (0.57 + 0.0133 * a.dim) * (which == kForward ? 1.0 : 1.25);
    const double rows = std::min(1.0, (double)(dkv ? a.max_k : a.max_q) / kOwnRows);
    const double all = own * longest * mean / compute_units() * (dkv && !one_side ? alone : shared / 2);
    const double part = std::ceil(longest / splits), slots = compute_units() * (dkv && !one_side ? 1.0 : 2.0);
    double us = std::max(alone * part, all + alone * part / 2);
    if (mean > 0.95)                                         // workgroups alike: whole rounds of them
        us = std::ceil(own * splits / slots) * part * ((dkv && !one_side) || own * splits <= compute_units() ? alone : shared);
    return splits > 1 ? us + 4.5 + 0.5 * splits + (double)sums_bytes(which, a, splits) * rows * 2 / 5e6 : us;
}

// The parts a launch is split into.
int splits_of(int which, const AttnArgs &a)
{
    constexpr int kMost = 16, kSlots = 2048;
    const int64_t items = items_of(which, a), forced = knob(SAMO_KNOB_ATTENTION_SPLIT, -1);
    if (items == 0) return 1;
    if (forced > 0) return (int)std::max<int64_t>(1, std::min<int64_t>({kMost, forced, (1 << 21) / items}));       // a launch holds 2^23 workgroups and more
    // Two rounds of the device are even enough: the longest workgroups come first (8192 tokens, 32 heads of 128, 8 of keys: forward 574 us as they are and 660
    // in two parts, backward 1983 and 2107).
    if (items >= (which == kDkv && a.dim > 64 ? 2 : 4) * compute_units()) return 1;
    int best = 1;
    double least = launch_us(which, a, items, 1);
    if (least < 12.0) return 1;                              // two parts take six of them, and five for the second kernel
    for (int splits = 2; splits <= kMost && items * splits <= kSlots; ++splits) {
        const double us = launch_us(which, a, items, splits);
        if (us < least) {
            least = us;
            best = splits;
        }
    }
    return best;
}

hipError_t launch(int which, AttnArgs a, size_t bytes, hipStream_t s)
{
    a.tiles = (int)ceil_div(which == kDkv ? a.max_k : a.max_q, kOwnRows);
    const int64_t items = items_of(which, a);
    if (items == 0) return hipSuccess;
    a.splits = splits_of(which, a);
    if (!a.parts || (size_t)sums_bytes(which, a, a.splits) > bytes) a.splits = 1;
    a.part_stats = reinterpret_cast<f32x2 *>(a.parts + items * a.splits * kOwnRows * 32 * blocks_of_dim(a.dim));
    switch ((a.dim + 15) / 16) {                             // padded: a kernel for each of the sizes in use, and the next one up for the others
    case 1: case 2: return launch_dim<2>(which, a, items, s);
    case 3: case 4: return launch_dim<4>(which, a, items, s);
    case 5: return launch_dim<5>(which, a, items, s);
    case 6: return launch_dim<6>(which, a, items, s);
    default: return launch_dim<8>(which, a, items, s);
    }
}

}  // namespace

// The runtime counts a launch's threads in 32 bits: fewer than 2^24 workgroups, of dK and dV where two waves share the keys of so many 2^23.  (Launches in
// parts are far smaller.)
bool attention_fits(const samo_attention_desc &d, bool backward)
{
    for (int which = backward ? kDq : kForward; which <= (backward ? kDkv : kForward); ++which) {
        const int64_t all = (int64_t)d.batch * (which == kDkv ? d.kv_heads : d.heads), tiles = ceil_div(which == kDkv ? d.max_k : d.max_q, kOwnRows);
        const int64_t most = UINT32_MAX / (kAttnThreads * (which == kDkv && one_side_from(d.dim) == INT32_MAX ? 2 : 1));
        if (tiles > 0 && (all > most || places_of(all, tiles) > most / 8)) return false;
    }
    return true;
}

int64_t attention_sums_bytes(const AttnArgs &a, bool backward)
{
    if (!backward) return sums_bytes(kForward, a, splits_of(kForward, a));
    return std::max(sums_bytes(kDq, a, splits_of(kDq, a)), sums_bytes(kDkv, a, splits_of(kDkv, a)));
}

hipError_t launch_attention(const AttnArgs &a, size_t bytes, hipStream_t s) { return launch(kForward, a, bytes, s); }

hipError_t launch_attention_backward(const AttnArgs &a, size_t bytes, hipStream_t s)
{
    if (hipError_t e = launch(kDq, a, bytes, s)) return e;   // delta first: the other kernel reads it
    return launch(kDkv, a, bytes, s);
}

}  // namespace samo
