// Attention's launches: which kernel, in how many parts, and the kernels that join what parts have left (attention_kernels.h has the others; attention_*.hip
// those of scores of another form, a file each so that they are built side by side).
#include "attention_kernels.h"

namespace samo {
namespace {

// Whole rows from the sums of their parts, added in order: a wave has 32 rows, and 32 dims of them, as the kernel that left them had.
// Parts of out are weighed by how far their exponents were taken down; one that has seen no key does not count.  Four parts are asked for at a time, whatever
// their number; before, one after the other: a token behind 8191, 32 heads of 128 on 8 (16 parts), 33 us, now 27; two and three parts within 1 % of what they were.
template <int DB, int WHICH>
__global__ void __launch_bounds__(DB * 64) attention_join_kernel(const AttnArgs A)
{
    constexpr int kTensors = WHICH == kDkv ? 2 : 1;
    const int rows = (int)(blockIdx.x & 3), db = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, tensor = (int)blockIdx.y;
    const int item = (int)(blockIdx.x >> 2);
    const Place at = place_of(item / A.tiles, item % A.tiles, 0, A);
    const Sequence seq = sequence_of(A, at.b);
    const int pack = WHICH == kForward ? A.pack : 1;
    const int count = WHICH == kDkv ? seq.k_len : seq.q_len * pack, row = (WHICH == kDkv ? A.tiles - 1 - at.tile : at.tile) * kOwnRows + rows * kWaveRows + (lane & 31);
    // Of few rows the parts are asked for before it is known which rows there are (their memory is there for all of them): one wait less in a chain of three.
    if (WHICH == kForward && A.few ? rows > 0 : row >= count) return;
    f32x16 acc[1];
    clear(acc);
    float top = -INFINITY, sum = 0.f;
    const f32x2 *stats = A.part_stats + (at.slot * 4 + rows) * 32 + (lane & 31);
    if (WHICH == kForward)
        for (int part = 0; part < A.splits; part += 4) {
            f32x2 stat[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) stat[i] = stats[min(part + i, A.splits - 1) * 128];
#pragma unroll
            for (int i = 0; i < 4; ++i) top = stat[i][1] != 0.f ? fmaxf(top, stat[i][0]) : top;
        }
    for (int part = 0; part < A.splits; part += 4) {         // four parts' loads under way, the last ones of a part that is there
        f32x2 stat[4];
        f32x4 x[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int that = min(part + i, A.splits - 1);
            if (WHICH == kForward) stat[i] = stats[that * 128];
            const f32x4 *from = sums_of<DB>(A.parts, (at.slot + that) * kTensors + tensor, rows) + 4 * db * 64;
#pragma unroll
            for (int g = 0; g < 4; ++g) x[i][g] = from[g * 64];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool counts = part + i < A.splits && (WHICH != kForward || stat[i][1] != 0.f);
            float weight = 1.f;
            if (WHICH == kForward) {
                weight = __builtin_amdgcn_exp2f(stat[i][0] - top);
                sum = counts ? fmaf(stat[i][1], weight, sum) : sum;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[0][e] = counts ? fmaf(x[i][e >> 2][e & 3], weight, acc[0][e]) : acc[0][e];
        }
    }
    if (row >= count) return;
    const int query = pack > 1 ? row / pack : row, head = pack > 1 ? at.head * pack + row - query * pack : at.head;
    _Float16 *to;
    int64_t stride;
    float factor = A.scale;
    if (WHICH == kForward) {
        to = A.out + (seq.q0 + query) * A.out_row + head * A.out_head;
        stride = 0;
        factor = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
        if (db == 0 && lane < 32) A.lse[(int64_t)head * A.q_tokens + seq.q0 + query] = sum == 0.f ? -INFINITY : top * kLn2 + __logf(sum);
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

// The table's gradient: a head's workgroup adds what the workgroups of dQ left, in order, a column to a thread.  A chain of loads, a row of every eight each:
// 4.7 us of 7 ragged sequences, 16 heads and 32 buckets, but 9.3 of 256 sequences of 64 tokens and 55 of 256 of 512 (dQ and dK, dV: 1480).
constexpr int kTableThreads = 1024, kTableRows = kTableThreads / (2 * kMaxBuckets);
__global__ void __launch_bounds__(kTableThreads) table_gradient_kernel(const float *parts, int64_t slots, int columns, _Float16 *to)
{
    __shared__ double sums[kTableRows][2 * kMaxBuckets];
    const int column = threadIdx.x % (2 * kMaxBuckets), row = threadIdx.x / (2 * kMaxBuckets);
    double sum = 0.0;
    if (column < columns)
        for (int64_t at = row; at < slots; at += kTableRows) sum += parts[(blockIdx.x * slots + at) * columns + column];
    sums[row][column] = sum;
    __syncthreads();
    if (row > 0 || column >= columns) return;
    for (int other = 1; other < kTableRows; ++other) sum += sums[other][column];
    to[(int64_t)blockIdx.x * columns + column] = (_Float16)(float)sum;
}

// Heads whose workgroups a launch has, and their rows (pack heads of a query each, where they share them).
int64_t heads_of(int which, const AttnArgs &a) { return which == kDkv || (which == kForward && a.pack > 1) ? a.kv_heads : a.heads; }
int64_t most_rows(int which, const AttnArgs &a) { return which == kDkv ? a.max_k : which == kForward ? (int64_t)a.max_q * a.pack : a.max_q; }
int64_t items_of(int which, const AttnArgs &a) { return a.batch * heads_of(which, a) * ceil_div(most_rows(which, a), kOwnRows); }

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
// a quarter more.  Measured against the parts taken, whole calls, us: one token behind 8191, 32 heads of 128 on 8, 181 with one part, 34 with 8, 27 with 16;
// 2000 tokens in 3 sequences behind 3000 each, 16 heads of 64, 72 and 54 with three; 4096 tokens, 8 heads of 128, 90 and 57 with three; 1024 tokens of
// 16 heads of 96 23 and 25 with two, which it takes; 2048 in 4 sequences, 16 heads of 64, 13 and 23 with two; one token each behind 8 contexts of 2047, 32 heads of
// 128, 59, 50 with two and 53 with four.
// Where every workgroup has as much to do, the rounds that they take count whole.
double launch_us(int which, const AttnArgs &a, int64_t items, int splits)
{
    const bool dkv = which == kDkv, one_side = dkv && items * splits >= one_side_from(a.dim);
    const double q = (double)a.q_tokens / a.batch, k = (double)a.k_tokens / a.batch;
    double longest = dkv ? q : k, mean = 1.0;
    if (a.window) longest = std::min(longest, (double)a.window + kOwnRows);
    else if (a.causal) mean = 1.0 - 0.5 * std::min(1.0, q / std::max(k, 1.0));
    longest = std::ceil(longest / kTileRows) * (dkv ? a.group : 1);
    const double own = std::min((double)items, (double)heads_of(which, a) * ((double)(dkv ? a.k_tokens : a.q_tokens) / kOwnRows + a.batch));
    const double alone = (1.0 + 0.004 * a.dim) * (which == kForward ? 1.0 : 1.25), shared = (0.57 + 0.0133 * a.dim) * (which == kForward ? 1.0 : 1.25);
    const double rows = std::min(1.0, (double)most_rows(which, a) / kOwnRows);
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
    if (which == kForward && a.few) {                        // four tiles at once in a workgroup, a part besides for the second kernel's 5 us
        const int64_t longest = a.window ? std::min<int64_t>(a.max_k, a.window + most_rows(which, a)) : a.max_k, tiles = ceil_div(longest, kTileRows);
        const int64_t slots = compute_units() * (a.dim > 64 ? 1 : 2);
        double least = 1e30;
        for (int splits = 1; splits <= kMost && items * splits <= kSlots; ++splits) {
            const double us = 1.6 * (double)ceil_div(ceil_div(tiles, splits), 4) * (double)ceil_div(items * splits, slots) + (splits > 1 ? 5.0 + 0.15 * splits : 0.0);
            if (us < least) {
                least = us;
                best = splits;
            }
        }
        return best;
    }
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

// A form by what the call has of it.
hipError_t launch_kernel(int which, const AttnArgs &a, int64_t items, hipStream_t s)
{
    if (!a.scored) return launch_form<kPlain>(which, a, items, s);
    const bool cap = a.form.cap > 0.f, slopes = a.form.slopes != nullptr, table = a.form.table != nullptr;
    if (slopes && table) return launch_attention_all(which, a, items, s);
    if (slopes) return cap ? launch_attention_cap_slope(which, a, items, s) : launch_attention_slope(which, a, items, s);
    if (table) return cap ? launch_attention_cap_table(which, a, items, s) : launch_attention_table(which, a, items, s);
    return cap ? launch_attention_cap(which, a, items, s) : launch_attention_keys(which, a, items, s);
}

template <int DB>
void launch_join_dim(int which, const AttnArgs &a, int64_t items, hipStream_t s)
{
    const dim3 joins((unsigned)(items * 4), which == kDkv ? 2 : 1);
    if (which == kForward) hipLaunchKernelGGL((attention_join_kernel<DB, kForward>), joins, dim3(DB * 64), 0, s, a);
    else if (which == kDq) hipLaunchKernelGGL((attention_join_kernel<DB, kDq>), joins, dim3(DB * 64), 0, s, a);
    else hipLaunchKernelGGL((attention_join_kernel<DB, kDkv>), joins, dim3(DB * 64), 0, s, a);
}
hipError_t launch_join(int which, const AttnArgs &a, int64_t items, hipStream_t s)
{
    switch (blocks_of_dim(a.dim)) {
    case 1: launch_join_dim<1>(which, a, items, s); break;
    case 2: launch_join_dim<2>(which, a, items, s); break;
    case 3: launch_join_dim<3>(which, a, items, s); break;
    default: launch_join_dim<4>(which, a, items, s);
    }
    return hipGetLastError();
}

// taken: the parts that it was split into, if that is asked for.
hipError_t launch(int which, AttnArgs a, size_t bytes, hipStream_t s, int *taken = nullptr)
{
    a.tiles = (int)ceil_div(most_rows(which, a), kOwnRows);
    const int64_t items = items_of(which, a);
    if (items == 0) return hipSuccess;
    a.splits = splits_of(which, a);
    if (!a.parts || (size_t)sums_bytes(which, a, a.splits) > bytes) a.splits = 1;
    if (taken) *taken = a.splits;
    a.part_stats = reinterpret_cast<f32x2 *>(a.parts + items * a.splits * kOwnRows * 32 * blocks_of_dim(a.dim));
    if (hipError_t e = launch_kernel(which, a, items, s)) return e;
    return a.splits > 1 ? launch_join(which, a, items, s) : hipSuccess;
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

void attention_pack(AttnArgs &a)
{
    const bool one_head = !a.scored || a.form.table;         // a table's columns lie in a wave's lanes, of one head
    a.pack = one_head || (int64_t)a.max_q * a.group > kOwnRows ? 1 : a.group;
    // Up to two tiles of keys are one chain either way, and the waves' sums need no joining: 61 tokens in 9 sequences, 16 heads of 64, 6.7 us, with few 7.5.
    a.few = a.scored && most_rows(kForward, a) <= kWaveRows && a.max_k > 2 * kTileRows;
}

int64_t attention_table_bytes(const AttnArgs &a)
{
    return a.form.dtable ? items_of(kDq, a) * splits_of(kDq, a) * (a.form.two_sided ? 2 : 1) * a.form.buckets * (int64_t)sizeof(float) : 0;
}

hipError_t launch_attention_backward(const AttnArgs &a, size_t bytes, hipStream_t s)
{
    int splits = 1;
    if (hipError_t e = launch(kDq, a, bytes, s, &splits)) return e;      // delta first: the other kernel reads it
    if (a.form.dtable) {
        const int columns = (a.form.two_sided ? 2 : 1) * a.form.buckets;
        hipLaunchKernelGGL(table_gradient_kernel, dim3((unsigned)a.heads), dim3(kTableThreads), 0, s, a.form.dtable_parts,
                           items_of(kDq, a) / a.heads * splits, columns, a.form.dtable);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return launch(kDkv, a, bytes, s);
}

}  // namespace samo
