// The gated feed-forward block's up-projections, activation and product in one kernel, and its backward pass.  With X of tokens x in
// and two weight matrices of ffn x in, dense fp16 with explicit zeros as the expansion leaves them (Section III-C):
//   G = X Wg^T,  U = X Wu^T,  h = act(G) U
//   dG = dh U act'(G),  dU = dh act(G),  dX = dG Wg + dU Wu          (dWg = dG^T X and dWu = dU^T X are samo_wgrad_gather's)
// Products of fp16 with fp32 sums; G and U are rounded once to fp16 where they are kept for the backward pass, h is formed from the sums.  dG and dU are formed
// in fp32 from those and rounded to fp16: the weight gradients take them as fp16, and dX's products, which fp32 would make 16 times as slow, the same numbers.
//
// Bound by the matrix units from a few hundred tokens on, by the weights' bytes below.
//  - glu_kernel: a tile of 256 tokens by 128 features of both G and U (128 by 128, 64 or 32 for calls of few tiles), which so meet in one
//    wave's registers: the epilogue multiplies them and neither has to exist in memory.
//  - glu_dx_kernel: the same loop over both products of dX, one after the other along the summation: dG and dU against Wg and Wu.
//    Few tiles split the summation (glu_dx_shape), their fp32 sums meet in a workspace and are added in order.
//  - glu_pointwise_kernel: dG and dU, elementwise.
//  - glu_skinny_kernel: up to 32 tokens; the weights go past LDS straight into the matrix instructions, once.
// The tile loop: eight waves, a ring of stages of 32 or 64 along the summation in LDS, copied past the registers; the two waves
// of a SIMD are half a stage apart, so that one's multiplications cover the other's reads and copies.  An operand whose summation index is
// adjacent in memory (X, W in G and U, dG, dU) is kept in rows of 64 or 128 bytes; the one whose
// other index is (W in dX) as it comes, read with the transposing LDS read.
#include "common.h"
#include "lds_copy.h"

namespace samo {
namespace {

constexpr int kGluThreads = 512, kColumnPitch = 1024 + 32;

// A tile shape: a wave has AB x BB blocks of 16 x 16, AB of the weights' side and BB of the tokens'; the waves are 2 x 4.  So 64 BB tokens by
// 32 AB rows of weights (half of them G's, half U's) or, in dX, 32 AB columns; a stage is STEPS steps of 32 along the summation.
template <int AB, int BB, int STEPS, bool COLUMNS>
struct Shape {
    static constexpr int kTokens = 64 * BB, kSide = 32 * AB, kDeep = 32 * STEPS;
    static constexpr int kCopiesA = AB * STEPS / 2, kCopiesB = BB * STEPS;    // of a wave and stage: waves 0-3 bring the weights' panel, 4-7 the tokens'
    static constexpr int kMost = kCopiesA > kCopiesB ? kCopiesA : kCopiesB;
    static constexpr int kPanelA = 4 * kCopiesA * (COLUMNS ? kColumnPitch : 1024), kPanelB = 4 * kCopiesB * 1024;
    static constexpr int kStage = kPanelA + kPanelB;
    static constexpr int kRing = 160 * 1024 / kStage < 6 ? 160 * 1024 / kStage : 6;
    static_assert(kRing >= 3, "two stages on their way while one is multiplied");
    // A panel of an operand whose summation index is adjacent in memory: rows of 64 STEPS bytes, a copy brings 16 / STEPS of them: the lane's row, and
    // its 16-byte piece of it.  Rows of 64 bytes keep their pieces' order: a quarter of a wave's read (lanes 0-3, 12-15, 20-27 and so on) meets half of
    // the banks twice, which does not show, where orders that meet every bank once make the copies slower (8192 tokens, 4096 x 10928, us
    // forward and dX: 1238 and 1237; piece ^ row / 2 1245 and 1286; another one 1294 and 1273).  Rows of 128 are swizzled.
    static constexpr int kPieces = 4 * STEPS;
    __device__ __forceinline__ static int swizzle(int row) { return STEPS == 1 ? 0 : row >> 1 & 7; }
    __device__ __forceinline__ static int row_of(int n) { return n * (16 / STEPS) + (int)(threadIdx.x & 63) / kPieces; }
    __device__ __forceinline__ static int piece_of(int row) { return (int)(threadIdx.x & 63) % kPieces ^ swizzle(row); }
    __device__ __forceinline__ static half8 read_row(const unsigned char *panel, int row0, int step)
    {
        const int lane = threadIdx.x & 63, row = row0 + (lane & 15);
        return *reinterpret_cast<const half8 *>(panel + row * (64 * STEPS) + (((4 * step + (lane >> 4)) ^ swizzle(row)) << 4));
    }
    // Column panel: a copy's 1 KiB is an LDS row of 2 (kSide 256) or 4 (128) rows of the matrix, 512 or 256 bytes each; 2 AB LDS rows are a step.  Row 8 g + e
    // of a step is in LDS row and place such that the transposing read of four rows finds them in four LDS rows, whose pitch spreads them
    // over the banks, and its second one four in the next place.
    static constexpr int kPlaces = 512 / kSide, kPlaceBytes = 2 * kSide, kPlaceLanes = kSide / 8;
    __device__ __forceinline__ static half8 read_column(const unsigned char *panel, int col0, int step)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4, e = (lane >> 2) & 3;
        const int row = kPlaces == 2 ? 4 * g + e : 4 * (g & 1) + e, place = kPlaces == 2 ? 0 : 2 * (g >> 1);
        return read_fragment(panel + (step * 2 * AB + row) * kColumnPitch + place * kPlaceBytes + (lane & 3) * 8 + col0 * 2, kPlaceBytes);
    }
    // the matrix row, of the stage's, that a lane of copy n brings
    __device__ __forceinline__ static int column_row_of(int n)
    {
        const int place = (int)(threadIdx.x & 63) / kPlaceLanes, step = n / (2 * AB), m = n % (2 * AB);
        return 32 * step + (kPlaces == 2 ? 8 * (m >> 2) + 4 * place + (m & 3) : 8 * (2 * (place >> 1) + (m >> 2)) + 4 * (place & 1) + (m & 3));
    }
};

template <int ACT>
__device__ __forceinline__ float activation(float z, float &slope)
{
    if (ACT == SAMO_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __expf(-z));
        slope = s * fmaf(z, 1.f - s, 1.f);
        return z * s;
    }
    if (ACT == SAMO_ACT_GELU) {
        // the complementary error function by Abramowitz & Stegun, 7.1.26: 1.5e-7
        const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f)), e = __expf(-x * x);
        const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        const float tail = 0.5f * poly * e, c = z < 0.f ? tail : 1.f - tail;
        slope = fmaf(z * 0.39894228040143268f, e, c);
        return z * c;
    }
    if (ACT == SAMO_ACT_GELU_TANH) {
        // z (1 + tanh y) / 2 = z sigmoid(2 y)
        const float y2 = 1.5957691216057308f * z * fmaf(0.044715f * z, z, 1.f);
        const float s = __builtin_amdgcn_rcpf(1.f + __expf(-y2));
        slope = s * fmaf(z * (1.f - s), 1.5957691216057308f * fmaf(3.f * 0.044715f * z, z, 1.f), 1.f);
        return z * s;
    }
    slope = z > 0.f ? 1.f : 0.f;
    return z > 0.f ? z : (z <= 0.f ? 0.f : z);               // NaN stays
}

// G as it is kept for the backward pass, which has relu's slope from its sign: a positive sum that rounds to zero stays the smallest positive number, so
// that both passes are on the same side of zero.
template <int ACT>
__device__ __forceinline__ _Float16 kept_gate(float g)
{
    return (_Float16)(ACT == SAMO_ACT_RELU && g > 0.f ? fmaxf(g, 0x1p-24f) : g);
}

// Waits until at most `younger` stages' copies of this wave, PER each, are outstanding, and every LDS read has returned.
template <int PER, int MOST>
__device__ __forceinline__ void wait_copies(int younger)
{
    if constexpr (MOST > 0) {
        if (younger < MOST) return wait_copies<PER, MOST - 1>(younger);
    }
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PER * MOST) : "memory");
}

// acc += the wave's AB x BB blocks of 16 x 16 over stages 0 .. stages - 1; copy(s, i, lds) issues the wave's copy i of stage s.
// Waves 0-3 and 4-7 are half a stage apart (b(i): barriers of all eight waves):
//   waves 0-3:  b(0) fetch 0  b(1) multiply 0  b(2) fetch 1  b(3) multiply 1 ...
//   waves 4-7:  b(0)          b(1) fetch 0     b(2) multiply 0  b(3) fetch 1 ...
// fetch s reads the stage's fragments and issues the copies of stage s + R - 1, R the ring's stages, into the place of stage s - 1, which waves
// 4-7, the later ones, have read before b(2s).  Stage s + 1 is read from b(2s + 2) on: every wave waits for its own copies of it before that
// barrier, when those of stages s + 2 .. s + R - 1 are the only younger ones.
template <int AB, int BB, int STEPS, bool COLUMNS, typename Copy>
__device__ __forceinline__ void multiply_stages(int stages, const Copy &copy, unsigned char *lds, int a_at, int b_at, f32x4 (&acc)[BB][AB])
{
    typedef Shape<AB, BB, STEPS, COLUMNS> S;
    constexpr int R = S::kRing, kMost = S::kMost;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave >> 2;
    const int mine = group ? S::kCopiesB : S::kCopiesA;
    const unsigned lds_at = (unsigned)(size_t)(LDS_AS unsigned char *)lds;
    auto wait = [&](int younger) {
        if (S::kCopiesA == S::kCopiesB || group == 0) wait_copies<S::kCopiesA, R - 2>(younger);
        else wait_copies<S::kCopiesB, R - 2>(younger);
    };
#pragma unroll
    for (int b = 0; b < BB; ++b)
#pragma unroll
        for (int a = 0; a < AB; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[b][a][r] = 0.f;
    for (int s = 0; s < R - 1 && s < stages; ++s)
#pragma unroll
        for (int i = 0; i < kMost; ++i)
            if (i < mine) copy(s, i, lds_at + s * S::kStage);
    wait(min(stages, R - 1) - 1);
    meet();
    if (group == 1) meet();
    int slot = 0;
    for (int s = 0; s < stages; ++s) {
        const unsigned char *cur = lds + slot * S::kStage;
        const unsigned dst = lds_at + (slot == 0 ? R - 1 : slot - 1) * S::kStage;
        const bool more = s + R - 1 < stages;
        auto next = [&](int i) {
            __builtin_amdgcn_sched_barrier(0);               // the copies stay spread between the LDS reads
            if (more && i < mine) copy(s + R - 1, i, dst);
            __builtin_amdgcn_sched_barrier(0);
        };
        half8 fa[STEPS][AB], fb[STEPS][BB];
        constexpr int kReads = STEPS * (AB + BB);
        int sent = 0;                                        // (known to the compiler at every place)
#pragma unroll
        for (int n = 0; n < kReads; ++n) {
            const int k = n / (AB + BB), m = n % (AB + BB);
            if (m < BB) fb[k][m] = S::read_row(cur + S::kPanelA, b_at + 16 * m, k);
            else if constexpr (COLUMNS) fa[k][m - BB] = S::read_column(cur, a_at + 16 * (m - BB), k);
            else fa[k][m - BB] = S::read_row(cur, a_at + 16 * (m - BB), k);
            if (sent < kMost && (n + 1) * kMost >= (sent + 1) * kReads - kReads / 2) next(sent++);
        }
        const int left = min(stages - 2 - s, R - 2);         // stages behind the next one that are on their way
        if (group == 0) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        else wait(left);
        __builtin_amdgcn_sched_barrier(0);
        meet();
        __builtin_amdgcn_s_setprio(1);                       // the multiplying wave first: the other one's reads fit in between
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int q = 0; q < AB * BB; ++q) {              // consecutive instructions share an operand
                const int a = q / BB, b = (a & 1) ? BB - 1 - q % BB : q % BB;
                acc[b][a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[k][a], fb[k][b], acc[b][a], 0, 0, 0);
            }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        if (group == 0) wait(left);
        meet();
        slot = slot == R - 1 ? 0 : slot + 1;
    }
    if (group == 0) meet();
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}

// Workgroups are dealt to the 8 XCDs in contiguous runs of tiles; a run goes down four tiles of tokens before it goes across, so that what an
// XCD holds at a time shares panels in its L2.
__device__ __forceinline__ bool pick_tile(int tiles_t, int tiles_f, int copies, int &tt, int &tf, int &part)
{
    const int tiles = tiles_t * tiles_f, items = tiles * copies, per_xcd = (items + 7) / 8;
    const int item = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || item >= items) return false;
    part = item / tiles;
    const int tile = item - part * tiles, group = tile / (4 * tiles_f), in_group = tile - group * 4 * tiles_f;
    const int deep = min(4, tiles_t - 4 * group);
    tf = in_group / deep;
    tt = 4 * group + in_group - tf * deep;
    return true;
}

// G, U and h.  8192 tokens, 4096 x 10928: 1214 us, 1210 TFLOP/s, bound by the chip's power; 2048, 2560 x 6832: 157 us, 910 (432 tiles in two rounds of
// the compute units); 1003, 1024 x 2736: 26 us (176 tiles, fewer than there are compute units).
template <int AB, int BB, int STEPS, int ACT>
__global__ void __launch_bounds__(kGluThreads, 2) glu_kernel(const GluArgs A)
{
    typedef Shape<AB, BB, STEPS, false> S;
    constexpr int kFeatures = S::kSide / 2, kHalf = kFeatures / 2;     // of the tile, and of a wave: of G and of U
    __shared__ __attribute__((aligned(1024))) unsigned char lds[S::kRing * S::kStage];
    int tt, tf, part;
    if (!pick_tile(A.tiles_t, A.tiles_f, 1, tt, tf, part)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t t0 = (int64_t)tt * S::kTokens;
    const int f0 = tf * kFeatures;
    const int64_t row_bytes = (int64_t)A.in * 2;
    // waves 0-3 copy the weights' panel, rows of G and of U in turn as the waves take them, 4-7 that of X.  What lies behind the last row is the last
    // row again: it ends in results that are not stored.
    const bool weights = wave < 4;
    constexpr int kMost = S::kMost, kDeep = S::kDeep;
    const int mine = weights ? S::kCopiesA : S::kCopiesB, n0 = (wave & 3) * mine;
    const unsigned char *next[kMost];                        // the lane's piece of the next stage, copy by copy
    int deep[kMost];                                         // and where along the summation, in a stage
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int row = S::row_of(n0 + i);
        const int64_t f = min(f0 + row / (2 * kHalf) * kHalf + row % kHalf, A.ffn - 1), t = min(t0 + row, A.tokens - 1);
        const _Float16 *m = !weights ? A.x : (n0 + i) * (16 / STEPS) / kHalf & 1 ? A.w_up : A.w_gate;
        next[i] = reinterpret_cast<const unsigned char *>(m) + (weights ? f : t) * row_bytes + S::piece_of(row) * 16;
        deep[i] = S::piece_of(row) * 8;
    }
    const unsigned to = (weights ? 0 : S::kPanelA) + n0 * 1024;
    auto copy = [&](int s, int i, unsigned stage) {
        dma16(s * kDeep + deep[i] < A.in ? next[i] : zero_row, stage + to + i * 1024);   // the last stage may be a part of one
        next[i] += 2 * kDeep;
    };
    f32x4 acc[BB][AB];
    const int wt = wave & 3, wf = wave >> 2;
    multiply_stages<AB, BB, STEPS, false>((A.in + kDeep - 1) / kDeep, copy, lds, wf * 2 * kHalf, wt * 16 * BB, acc);
#pragma unroll
    for (int b = 0; b < BB; ++b) {
        const int64_t t = t0 + wt * 16 * BB + 16 * b + (lane & 15);
        if (t >= A.tokens) continue;
#pragma unroll
        for (int a = 0; a < AB / 2; ++a) {
            const int f = f0 + wf * kHalf + 16 * a + 4 * (lane >> 4);
            if (f >= A.ffn) continue;
            half4 h, gate, up;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float slope;
                const float g = acc[b][a][r], u = acc[b][a + AB / 2][r];
                h[r] = (_Float16)(activation<ACT>(g, slope) * u);
                gate[r] = kept_gate<ACT>(g);
                up[r] = (_Float16)u;
            }
            const int64_t at = t * A.ffn + f;
            *reinterpret_cast<half4 *>(A.h + at) = h;
            if (A.gate) {
                *reinterpret_cast<half4 *>(A.gate + at) = gate;
                *reinterpret_cast<half4 *>(A.up + at) = up;
            }
        }
    }
}

// dX: 64 BB tokens x 32 AB columns by a workgroup, over the part of the summation that is its own.  8192 tokens, 4096 x 10928: 1304 us, 1125 TFLOP/s; 2048,
// 2560 x 6832, in three parts: 146 us, 980, and 12 for the sums.
template <int AB, int BB, int STEPS>
__global__ void __launch_bounds__(kGluThreads, 2) glu_dx_kernel(const GluArgs A)
{
    typedef Shape<AB, BB, STEPS, true> S;
    constexpr int kMost = S::kMost, kDeep = S::kDeep;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[S::kRing * S::kStage];
    int tt, ti, part;
    if (!pick_tile(A.tiles_t, A.tiles_f, A.splits, tt, ti, part)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t t0 = (int64_t)tt * S::kTokens;
    const int i0 = ti * S::kSide;
    const int of_one = (A.ffn + kDeep - 1) / kDeep;                  // stages of dG Wg, and of dU Wu
    const int first = part * A.part_stages, last = min(first + A.part_stages, 2 * of_one);
    const bool weights = wave < 4;
    const int64_t in_bytes = (int64_t)A.in * 2, ffn_bytes = (int64_t)A.ffn * 2;
    const int col = i0 + lane % S::kPlaceLanes * 8;                  // of the weights' panel; behind the last one: the first again
    const int mine = weights ? S::kCopiesA : S::kCopiesB, n0 = (wave & 3) * mine;
    int64_t offset[kMost];                                   // of the lane's piece from the operand's first element
    const unsigned char *next[kMost];                        // its place in the next stage
    int deep[kMost];                                         // and along the summation, in a stage
    const int64_t apart = weights ? kDeep * in_bytes : kDeep * 2;       // from stage to stage
    const unsigned char *one = reinterpret_cast<const unsigned char *>(weights ? A.w_gate : A.dgate);
    const unsigned char *two = reinterpret_cast<const unsigned char *>(weights ? A.w_up : A.dup);
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int row = S::row_of(n0 + i);
        offset[i] = weights ? S::column_row_of(n0 + i) * in_bytes + (col < A.in ? col : 0) * 2
                            : min(t0 + row, A.tokens - 1) * ffn_bytes + S::piece_of(row) * 16;
        deep[i] = weights ? S::column_row_of(n0 + i) : S::piece_of(row) * 8;
        next[i] = (first < of_one ? one + first * apart : two + (first - of_one) * apart) + offset[i];
    }
    const unsigned to = weights ? n0 * kColumnPitch : S::kPanelA + n0 * 1024, pitch = weights ? kColumnPitch : 1024;
    auto copy = [&](int s, int i, unsigned stage) {
        const int own = first + s, n = own >= of_one ? own - of_one : own;
        if (i == 0 && own == of_one)
#pragma unroll
            for (int j = 0; j < kMost; ++j) next[j] = two + offset[j];
        dma16(n * kDeep + deep[i] < A.ffn ? next[i] : zero_row, stage + to + i * pitch);
        next[i] += apart;
    };
    f32x4 acc[BB][AB];
    const int wt = wave & 3, wf = wave >> 2;
    multiply_stages<AB, BB, STEPS, true>(last > first ? last - first : 0, copy, lds, wf * 16 * AB, wt * 16 * BB, acc);
#pragma unroll
    for (int b = 0; b < BB; ++b) {
        const int64_t t = t0 + wt * 16 * BB + 16 * b + (lane & 15);
        if (t >= A.tokens) continue;
#pragma unroll
        for (int a = 0; a < AB; ++a) {
            const int col_out = i0 + wf * 16 * AB + 16 * a + 4 * (lane >> 4);
            if (col_out >= A.in) continue;
            const int64_t at = t * A.in + col_out;
            if (A.splits > 1) {
                *reinterpret_cast<f32x4 *>(A.partial + (int64_t)part * A.tokens * A.in + at) = acc[b][a];
                continue;
            }
            half4 x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = (_Float16)acc[b][a][r];
            *reinterpret_cast<half4 *>(A.dx + at) = x;
        }
    }
}

// The parts of dX's sums, in their order.
__global__ void __launch_bounds__(256) glu_sum_kernel(const float *partial, int splits, int64_t n, _Float16 *dx)
{
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= n) return;
    f32x4 a = *reinterpret_cast<const f32x4 *>(partial + at), b = *reinterpret_cast<const f32x4 *>(partial + at + 4);
    for (int s = 1; s < splits; ++s) {
        a += *reinterpret_cast<const f32x4 *>(partial + s * n + at);
        b += *reinterpret_cast<const f32x4 *>(partial + s * n + at + 4);
    }
    half8 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = (_Float16)a[e];
        x[4 + e] = (_Float16)b[e];
    }
    *reinterpret_cast<half8 *>(dx + at) = x;
}

// dG and dU: bound by HBM, 190 us for 8192 x 10928 (895 MB, 4.7 TB/s), 23.8 for 2048 x 6832.
template <int ACT>
__global__ void __launch_bounds__(256) glu_pointwise_kernel(const _Float16 *dh, const _Float16 *gate, const _Float16 *up, _Float16 *dgate, _Float16 *dup, int64_t n)
{
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= n) return;
    const half8 d = *reinterpret_cast<const half8 *>(dh + at), g = *reinterpret_cast<const half8 *>(gate + at), u = *reinterpret_cast<const half8 *>(up + at);
    half8 dg, du;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        // A G beyond fp16's range was kept as an infinity, where the formulas are zero times infinity: act' there is what it is at fp16's largest number
        // (0 or 1), act(-inf) is 0, and act(inf) stays infinite.
        const float kept = (float)g[e], z = fabsf(kept) == INFINITY ? copysignf(65504.f, kept) : kept, back = (float)d[e];
        float slope, a = activation<ACT>(z, slope);
        if (kept == INFINITY) a = kept;
        dg[e] = (_Float16)(back * (float)u[e] * slope);
        du[e] = (_Float16)(back * a);
    }
    *reinterpret_cast<half8 *>(dgate + at) = dg;
    *reinterpret_cast<half8 *>(dup + at) = du;
}

// Up to 16 NB tokens: a workgroup of eight waves has 16 features of G and of U, a wave every eighth 128 bytes of the rows, two steps of 32 at a time,
// the loads of kAhead such pairs on their way together.  The waves' sums are added up by halves in LDS.  Bound by the weights' bytes: 2560 x 6832
// (70 MB), one token 17.9 us, 3.9 TB/s: 427 workgroups, two on some compute units and one on others, and of a wave's two trips the second is a quarter
// full; 16 tokens 22.4, 32 28.7, where the tiles take 28.5 (and this kernel for 64 tokens 32 to 40).
constexpr int kSkinnyWaves = 8;
template <int NB, int ACT>
__global__ void __launch_bounds__(64 * kSkinnyWaves, 2) glu_skinny_kernel(const GluArgs A)
{
    constexpr int kAhead = NB == 1 ? 4 : 2, kBlocks = 2 * NB;
    __shared__ __attribute__((aligned(16))) float sums[kSkinnyWaves / 2][kBlocks][64][4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int f0 = blockIdx.x * 16, row = lane & 15, k_lane = 8 * (lane >> 4);
    const _Float16 *w[2], *x[NB];
#pragma unroll
    for (int b = 0; b < 2; ++b) w[b] = (b ? A.w_up : A.w_gate) + (int64_t)min(f0 + row, A.ffn - 1) * A.in + k_lane;
#pragma unroll
    for (int b = 0; b < NB; ++b) x[b] = A.x + min((int64_t)16 * b + row, A.tokens - 1) * A.in + k_lane;
    f32x4 acc[2][NB];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const half8 none = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int k0 = 64 * wave; k0 < A.in; k0 += 64 * kSkinnyWaves * kAhead) {
        half8 fw[2 * kAhead][2], fx[2 * kAhead][NB];
#pragma unroll
        for (int s = 0; s < 2 * kAhead; ++s) {
            const int k = k0 + 64 * kSkinnyWaves * (s / 2) + 32 * (s % 2);
            const bool there = k + k_lane < A.in;
#pragma unroll
            for (int a = 0; a < 2; ++a) fw[s][a] = there ? __builtin_nontemporal_load(reinterpret_cast<const half8 *>(w[a] + k)) : none;
#pragma unroll
            for (int b = 0; b < NB; ++b) fx[s][b] = there ? *reinterpret_cast<const half8 *>(x[b] + k) : none;
        }
#pragma unroll
        for (int s = 0; s < 2 * kAhead; ++s)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fw[s][a], fx[s][b], acc[a][b], 0, 0, 0);
    }
#pragma unroll
    for (int half = kSkinnyWaves / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int n = 0; n < kBlocks; ++n) *reinterpret_cast<f32x4 *>(sums[wave - half][n][lane]) = acc[n / NB][n % NB];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int n = 0; n < kBlocks; ++n) acc[n / NB][n % NB] += *reinterpret_cast<const f32x4 *>(sums[wave][n][lane]);
        __syncthreads();
    }
    if (wave > 0) return;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int64_t t = 16 * b + row;
        const int f = f0 + 4 * (lane >> 4);
        if (t >= A.tokens || f >= A.ffn) continue;
        half4 h, gate, up;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float slope;
            const float g = acc[0][b][r], u = acc[1][b][r];
            h[r] = (_Float16)(activation<ACT>(g, slope) * u);
            gate[r] = kept_gate<ACT>(g);
            up[r] = (_Float16)u;
        }
        const int64_t at = t * A.ffn + f;
        *reinterpret_cast<half4 *>(A.h + at) = h;
        if (A.gate) {
            *reinterpret_cast<half4 *>(A.gate + at) = gate;
            *reinterpret_cast<half4 *>(A.up + at) = up;
        }
    }
}

// The tile shapes: 64 BB tokens, 32 AB rows of weights or columns; what is around a tile's loop and a stage of it, in us with every compute
// unit at work, forward and dX.
struct TileShape {
    int tokens, side, deep;                  // of a stage
    double around, forward, dx;
};
const TileShape kShapes[] = {{256, 256, 32, 6.0, 0.87, 0.88}, {128, 256, 64, 5.0, 1.1, 1.28}, {128, 128, 64, 4.0, 0.72, 0.89}, {128, 64, 64, 4.0, 0.6, 0.0}};

// A launch's time by rounds of the compute units.
double tiles_us(const TileShape &t, double stage, int64_t tiles, double stages) { return (double)ceil_div(tiles, compute_units()) * (t.around + stage * stages); }

// The shape of a forward call's tiles.
int glu_shape(int64_t tokens, int64_t ffn, int64_t in)
{
    const int forced = knob(SAMO_KNOB_GLU_SHAPE, -1);
    if (forced >= 0 && forced < 4) return forced;
    int best = 0;
    double least = 1e300;
    for (int n = 0; n < 4; ++n) {
        const double us = tiles_us(kShapes[n], kShapes[n].forward, ceil_div(tokens, kShapes[n].tokens) * ceil_div(ffn, kShapes[n].side / 2), (double)ceil_div(in, kShapes[n].deep));
        if (us < least) {
            least = us;
            best = n;
        }
    }
    return best;
}

dim3 grid_of(int64_t items) { return dim3((unsigned)(ceil_div(items, 8) * 8)); }

template <int ACT>
hipError_t forward(GluArgs a, hipStream_t s)
{
    if (a.tokens <= kGluSkinny) {
        const dim3 grid((unsigned)ceil_div(a.ffn, 16)), block(64 * kSkinnyWaves);
        if (a.tokens <= 16) hipLaunchKernelGGL((glu_skinny_kernel<1, ACT>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((glu_skinny_kernel<2, ACT>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    const int shape = glu_shape(a.tokens, a.ffn, a.in);
    a.tiles_t = (int)ceil_div(a.tokens, kShapes[shape].tokens);
    a.tiles_f = (int)ceil_div(a.ffn, kShapes[shape].side / 2);
    const dim3 grid = grid_of((int64_t)a.tiles_t * a.tiles_f);
    if (shape == 0) hipLaunchKernelGGL((glu_kernel<8, 4, 1, ACT>), grid, dim3(kGluThreads), 0, s, a);
    else if (shape == 1) hipLaunchKernelGGL((glu_kernel<8, 2, 2, ACT>), grid, dim3(kGluThreads), 0, s, a);
    else if (shape == 2) hipLaunchKernelGGL((glu_kernel<4, 2, 2, ACT>), grid, dim3(kGluThreads), 0, s, a);
    else hipLaunchKernelGGL((glu_kernel<2, 2, 2, ACT>), grid, dim3(kGluThreads), 0, s, a);
    return hipGetLastError();
}

template <int ACT>
hipError_t pointwise(const GluArgs &a, hipStream_t s)
{
    const int64_t n = a.tokens * a.ffn;
    hipLaunchKernelGGL((glu_pointwise_kernel<ACT>), dim3((unsigned)ceil_div(n, 2048)), dim3(256), 0, s, a.dh, a.gate, a.up, a.dgate, a.dup, n);
    return hipGetLastError();
}

}  // namespace

GluShape glu_dx_shape(int64_t tokens, int64_t ffn, int64_t in, int max_splits)
{
    GluShape best;
    double least = 1e300;
    const int forced = knob(SAMO_KNOB_GLU_SHAPE, -1), forced_splits = knob(SAMO_KNOB_GLU_SPLIT, -1);
    for (int n = 0; n < 3; ++n) {
        if (forced >= 0 && forced < 3 && n != forced) continue;
        const int64_t stages = 2 * ceil_div(ffn, kShapes[n].deep), tiles = ceil_div(tokens, kShapes[n].tokens) * ceil_div(in, kShapes[n].side);
        for (int splits = 1; splits <= max_splits; ++splits) {
            const int64_t each = ceil_div(stages, splits);
            if (splits > 1 && (each < 4 || (int64_t)(splits - 1) * each >= stages)) break;
            if (forced_splits > 0 && splits > forced_splits) break;
            double us = tiles_us(kShapes[n], kShapes[n].dx, tiles * splits, (double)each);
            if (splits > 1) us += 3.0 + (double)tokens * (double)in * 8.0 * splits / 5e6;       // the sums written and read, at 5 TB/s
            if (forced_splits > 0) us = -splits;
            if (us < least) {
                least = us;
                best.shape = n;
                best.splits = splits;
                best.part_stages = (int)each;
            }
        }
    }
    return best;
}

// Whether the launches of a call can be made: the runtime counts a launch's threads in 32 bits.
bool glu_fits(int64_t tokens, int64_t in, int64_t ffn)
{
    if (tokens <= kGluSkinny) return true;
    const TileShape &t = kShapes[glu_shape(tokens, ffn, in)];
    return ceil_div(tokens, t.tokens) * ceil_div(ffn, t.side / 2) <= (int64_t)(UINT32_MAX / kGluThreads - 8);
}

bool glu_backward_fits(int64_t tokens, int64_t in, int64_t ffn, const GluShape &shape)
{
    const TileShape &t = kShapes[shape.shape];
    // eight elements to a thread in glu_pointwise_kernel, and in glu_sum_kernel
    const int64_t most = (int64_t)(UINT32_MAX - 256) * 8;
    return tokens * ffn <= most && tokens * in <= most &&
           ceil_div(tokens, t.tokens) * ceil_div(in, t.side) * shape.splits <= (int64_t)(UINT32_MAX / kGluThreads - 8);
}

hipError_t launch_glu(int act, const GluArgs &a, hipStream_t s)
{
    switch (act) {
    case SAMO_ACT_SILU: return forward<SAMO_ACT_SILU>(a, s);
    case SAMO_ACT_GELU: return forward<SAMO_ACT_GELU>(a, s);
    case SAMO_ACT_GELU_TANH: return forward<SAMO_ACT_GELU_TANH>(a, s);
    default: return forward<SAMO_ACT_RELU>(a, s);
    }
}

hipError_t launch_glu_backward(int act, GluArgs a, const GluShape &shape, hipStream_t s)
{
    hipError_t e;
    switch (act) {
    case SAMO_ACT_SILU: e = pointwise<SAMO_ACT_SILU>(a, s); break;
    case SAMO_ACT_GELU: e = pointwise<SAMO_ACT_GELU>(a, s); break;
    case SAMO_ACT_GELU_TANH: e = pointwise<SAMO_ACT_GELU_TANH>(a, s); break;
    default: e = pointwise<SAMO_ACT_RELU>(a, s);
    }
    if (e != hipSuccess || !a.dx) return e;
    const TileShape &tile = kShapes[shape.shape];
    a.tiles_t = (int)ceil_div(a.tokens, tile.tokens);
    a.tiles_f = (int)ceil_div(a.in, tile.side);
    a.splits = shape.splits;
    a.part_stages = shape.part_stages;
    const dim3 grid = grid_of((int64_t)a.tiles_t * a.tiles_f * a.splits);
    if (shape.shape == 0) hipLaunchKernelGGL((glu_dx_kernel<8, 4, 1>), grid, dim3(kGluThreads), 0, s, a);
    else if (shape.shape == 1) hipLaunchKernelGGL((glu_dx_kernel<8, 2, 2>), grid, dim3(kGluThreads), 0, s, a);
    else hipLaunchKernelGGL((glu_dx_kernel<4, 2, 2>), grid, dim3(kGluThreads), 0, s, a);
    if (hipError_t e2 = hipGetLastError()) return e2;
    if (a.splits > 1) {
        const int64_t n = a.tokens * a.in;
        hipLaunchKernelGGL(glu_sum_kernel, dim3((unsigned)ceil_div(n, 2048)), dim3(256), 0, s, a.partial, a.splits, n, a.dx);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace samo
