// What lies between a block's output y and the next block's input, forward and backward, a pass over the rows each: a norm behind the block, its gate and
// residual scale, the sum with the residual stream s, and the next block's norm.  With N(x) = (x - m) r, r = 1 / sqrt(mean((x - m)^2) + eps), m the
// row's mean (layer) or 0 (rms), and f = scale gate,
//   n = N(y) wy + by (or y),   s' = s + f n,   out = N(s') w + b
// and with N'(g, x) = r (g - x mean(g x) - mean(g) (layer only)) of a normed x
//   D = dnew + N'(dout w, x),   dy = N'(f D wy, yn) (or f D),
//   dw = sum dout x,  db = sum dout,  dgate = scale (wy sum D yn + by sum D) (or scale sum D y),  dwy = f sum D yn,  dby = f sum D
// Bound by HBM: forward reads s and y and writes s' and out, backward reads dout, dnew, s' and y and writes D and dy.
//
// A workgroup has a row at a time, 8 V elements of it in a thread's registers from the load to the store, and goes on to rows a grid further: the five
// vectors are loaded once, and the sums over the tokens are a thread's own columns, left to a second kernel as one row of fp32 a workgroup.
// Statistics are fp32 of fp32 values (of s' before its rounding), the variance from the differences from the mean, and meet over the row in a fixed order.
#include <algorithm>

#include "common.h"
#include "lds_copy.h"

namespace samo {
namespace {

constexpr int kNormThreads = 512, kWideThreads = 1024;

// Eight elements in a row, as they lie in memory.
template <typename T> struct Eight;
template <> struct Eight<_Float16> {
    half8 x;
    __device__ __forceinline__ float operator[](int i) const { return (float)x[i]; }
    __device__ __forceinline__ void set(int i, float v) { x[i] = (_Float16)v; }
};
template <> struct Eight<float> {
    f32x4 lo, hi;
    __device__ __forceinline__ float operator[](int i) const { return i < 4 ? lo[i] : hi[i - 4]; }
    __device__ __forceinline__ void set(int i, float v)
    {
        if (i < 4) lo[i] = v;
        else hi[i - 4] = v;
    }
};
template <typename T>
__device__ __forceinline__ Eight<T> all_of(float v)
{
    Eight<T> e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.set(i, v);
    return e;
}

// A thread's share of a row: vector v of 8 elements is the (v blockDim + thread)th.  A row is a buffer of its own, so that a thread behind its end reads
// zeros and writes nothing, without a branch and with one offset for all arrays of a type.
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
template <int V>
struct Columns {
    int hidden;
    __device__ __forceinline__ int at(int v) const { return (v * (int)blockDim.x + (int)threadIdx.x) * 8; }
    __device__ __forceinline__ bool there(int v) const { return at(v) < hidden; }
    template <typename T>
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t row_of(T *base, int64_t row) const
    {
        void *from = const_cast<void *>(static_cast<const void *>(base + row * hidden));
        return __builtin_amdgcn_make_buffer_rsrc(from, 0, base ? hidden * (int)sizeof(T) : 0, 0x27000);
    }
    // row `row` of an array, zeros of none
    __device__ __forceinline__ void load(const _Float16 *base, int64_t row, Eight<_Float16> (&to)[V]) const
    {
        const __amdgpu_buffer_rsrc_t from = row_of(base, row);
#pragma unroll
        for (int v = 0; v < V; ++v) to[v].x = __builtin_bit_cast(half8, __builtin_amdgcn_raw_buffer_load_b128(from, at(v) * 2, 0, 0));
    }
    __device__ __forceinline__ void load(const float *base, int64_t row, Eight<float> (&to)[V]) const
    {
        const __amdgpu_buffer_rsrc_t from = row_of(base, row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            to[v].lo = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, at(v) * 4, 0, 0));
            to[v].hi = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, at(v) * 4 + 16, 0, 0));
        }
    }
    __device__ __forceinline__ void vector(const _Float16 *base, Eight<_Float16> (&to)[V], float other) const
    {
        if (base) load(base, 0, to);
        else
#pragma unroll
            for (int v = 0; v < V; ++v) to[v] = all_of<_Float16>(other);
    }
    __device__ __forceinline__ void store(_Float16 *base, int64_t row, const Eight<_Float16> (&from)[V]) const
    {
        const __amdgpu_buffer_rsrc_t to = row_of(base, row);
#pragma unroll
        for (int v = 0; v < V; ++v) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, from[v].x), to, at(v) * 2, 0, 0);
    }
    __device__ __forceinline__ void store(float *base, int64_t row, const Eight<float> (&from)[V]) const
    {
        const __amdgpu_buffer_rsrc_t to = row_of(base, row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, from[v].lo), to, at(v) * 4, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, from[v].hi), to, at(v) * 4 + 16, 0, 0);
        }
    }
};

template <int CONTROL, int ROWS>
__device__ __forceinline__ float plus_lane(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, ROWS, 0xf, false));
}
// The sum over a wave, the same in all lanes.
__device__ __forceinline__ float wave_total(float x)
{
    x = plus_lane<0x111, 0xf>(x);            // one lane to the right within rows of 16, two, four, eight; rows
    x = plus_lane<0x112, 0xf>(x);
    x = plus_lane<0x114, 0xf>(x);
    x = plus_lane<0x118, 0xf>(x);
    x = plus_lane<0x142, 0xa>(x);
    x = plus_lane<0x143, 0xc>(x);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// Sums over the workgroup, the same in all threads.  Two rooms in turn: a barrier for each sum, before it is read.
template <int WAVES>
struct Totals {
    f32x4 (*room)[WAVES / 2];                // two numbers a wave, zero where there is none
    int turn;
    __device__ __forceinline__ explicit Totals(f32x4 (*r)[WAVES / 2]) : room(r), turn(0)
    {
        if (blockDim.x == 64) return;
        if (threadIdx.x < WAVES) room[threadIdx.x / (WAVES / 2)][threadIdx.x % (WAVES / 2)] = f32x4{0.f, 0.f, 0.f, 0.f};
        __syncthreads();
    }
    __device__ __forceinline__ void operator()(float &a, float &b)
    {
        a = wave_total(a);
        b = wave_total(b);
        if (blockDim.x == 64) return;
        if ((threadIdx.x & 63) == 0) {
            float *to = reinterpret_cast<float *>(room[turn]) + 2 * (threadIdx.x >> 6);
            to[0] = a;
            to[1] = b;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // not for memory, as __syncthreads() waits: the next row's loads are under way
        meet();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES / 2; ++w) {
            const f32x4 two = room[turn][w];
            a += two[0];
            b += two[1];
            a += two[2];
            b += two[3];
        }
        turn ^= 1;
    }
};

// m and r of a row whose elements behind `there` are not counted.
template <int V, int WAVES>
__device__ __forceinline__ void statistics(const float (&x)[V][8], const Columns<V> &C, bool layer, float over, float eps, Totals<WAVES> &total, float &m, float &r)
{
    float sum = 0.f, none = 0.f;
    m = 0.f;
    if (layer) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += C.there(v) ? x[v][i] : 0.f;
        total(sum, none);
        m = sum * over;
    }
    float squares = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = C.there(v) ? x[v][i] - m : 0.f;
            squares = fmaf(d, d, squares);
        }
    none = 0.f;
    total(squares, none);
    r = __builtin_amdgcn_rsqf(fmaf(squares, over, eps));
}

enum { kNoBlock, kPlainBlock, kNormedBlock };

template <typename S, int V, int THREADS, int Y>
__global__ void __launch_bounds__(THREADS) norm_kernel(const NormArgs A)
{
    __shared__ f32x4 room[2][THREADS / 128];
    Totals<THREADS / 64> total(room);
    const Columns<V> C = {A.hidden};
    const S *stream = static_cast<const S *>(A.stream);
    S *new_stream = static_cast<S *>(A.new_stream);
    const float over = 1.f / (float)A.hidden;
    const bool layer = A.layer;
    Eight<_Float16> w[V], b[V], wy[V], by[V], gate[V];
    auto vectors = [&] {
        C.vector(A.weight, w, 1.f);
        C.load(A.bias, 0, b);
        if (Y == kNormedBlock) {
            C.vector(A.y_weight, wy, 1.f);
            C.load(A.y_bias, 0, by);
        }
        if (Y != kNoBlock) C.vector(A.gate, gate, 1.f);
    };
    vectors();
    Eight<S> coming_s[V];
    Eight<_Float16> coming_y[V];
    auto bring = [&](int64_t row) {
        C.load(stream, row, coming_s);
        if (Y != kNoBlock) C.load(A.y, row, coming_y);
    };
    constexpr bool kAhead = THREADS != kWideThreads;         // a row under way while the one before it is worked on
    if (kAhead && blockIdx.x < A.tokens) bring(blockIdx.x);
    for (int64_t row = blockIdx.x; row < A.tokens; row += gridDim.x) {
        if (!kAhead) {                                       // nor are the vectors kept: there are no registers for either
            bring(row);
            vectors();
        }
        Eight<S> s[V];
        Eight<_Float16> y[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s[v] = coming_s[v];
            if (Y != kNoBlock) y[v] = coming_y[v];
        }
        if (kAhead && row + gridDim.x < A.tokens) bring(row + gridDim.x);
        float x[V][8], my = 0.f, ry = 1.f, m, r;
        if (Y != kNoBlock) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] = y[v][i];
            if (Y == kNormedBlock) statistics(x, C, layer, over, A.eps, total, my, ry);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float n = Y == kNormedBlock ? fmaf((x[v][i] - my) * ry, wy[v][i], by[v][i]) : x[v][i];
                    x[v][i] = fmaf(A.scale * gate[v][i], n, s[v][i]);
                    s[v].set(i, x[v][i]);
                }
            C.store(new_stream, row, s);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] = s[v][i];
        }
        statistics(x, C, layer, over, A.eps, total, m, r);
        Eight<_Float16> out[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) out[v].set(i, fmaf((x[v][i] - m) * r, w[v][i], b[v][i]));
        C.store(A.out, row, out);
        if (A.stats && threadIdx.x == 0) *reinterpret_cast<f32x4 *>(A.stats + 4 * row) = f32x4{my, ry, m, r};
    }
}

// The sums over the tokens that a call wants, each a row of fp32 for each workgroup: dout x, dout, D yn (D y), D.
enum { kSumOutX, kSumOut, kSumDY, kSumD, kSums };

template <typename S, int V, int THREADS, int Y, bool BIASES>
__global__ void __launch_bounds__(THREADS, THREADS == kWideThreads ? 4 : V == 1 ? 3 : 2) norm_backward_kernel(const NormArgs A)
{
    __shared__ f32x4 room[2][THREADS / 128];
    Totals<THREADS / 64> total(room);
    const Columns<V> C = {A.hidden};
    const S *stream = static_cast<const S *>(A.new_stream), *dnew = static_cast<const S *>(A.dnew);
    S *dstream = static_cast<S *>(A.dstream);
    const float over = 1.f / (float)A.hidden;
    const bool layer = A.layer;
    Eight<_Float16> w[V], wy[V], gate[V];
    auto vectors = [&] {
        C.vector(A.weight, w, 1.f);
        if (Y == kNormedBlock) C.vector(A.y_weight, wy, 1.f);
        if (Y != kNoBlock) C.vector(A.gate, gate, 1.f);
    };
    vectors();
    float sums[kSums][V][8] = {};
    const _Float16 *y_at = Y == kNormedBlock || A.of_sum[kSumDY] >= 0 ? A.y : nullptr;       // of a plain y only the gate's gradient asks
    Eight<S> coming_s[V], coming_d[V];
    Eight<_Float16> coming_dout[V], coming_y[V];
    f32x4 coming_stat;
    auto bring = [&](int64_t row) {
        C.load(A.dout, row, coming_dout);
        C.load(stream, row, coming_s);
        C.load(dnew, row, coming_d);
        if (Y != kNoBlock) C.load(y_at, row, coming_y);
        coming_stat = *reinterpret_cast<const f32x4 *>(A.stats + 4 * row);
    };
    constexpr bool kAhead = THREADS != kWideThreads;         // a row under way while the one before it is worked on
    if (kAhead && blockIdx.x < A.tokens) bring(blockIdx.x);
    for (int64_t row = blockIdx.x; row < A.tokens; row += gridDim.x) {
        if (!kAhead) {                                       // nor are the vectors kept: there are no registers for either
            bring(row);
            vectors();
        }
        Eight<S> s[V], d[V];
        Eight<_Float16> dout[V], y[V];
        const f32x4 stat = coming_stat;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s[v] = coming_s[v];
            d[v] = coming_d[v];
            dout[v] = coming_dout[v];
            if (Y != kNoBlock) y[v] = coming_y[v];
        }
        if (kAhead && row + gridDim.x < A.tokens) bring(row + gridDim.x);
        const float my = stat[0], ry = stat[1], m = stat[2], r = stat[3];
        float x[V][8], dx[V][8], gx = 0.f, g = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[v][i] = (s[v][i] - m) * r;
                dx[v][i] = dout[v][i] * w[v][i];
                gx = fmaf(dx[v][i], x[v][i], gx);            // behind the row dout is zero
                g += dx[v][i];
                sums[kSumOutX][v][i] = fmaf(dout[v][i], x[v][i], sums[kSumOutX][v][i]);
                if (BIASES) sums[kSumOut][v][i] += dout[v][i];
            }
        total(gx, g);
        gx *= over;
        g = layer ? g * over : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dx[v][i] = fmaf(r, dx[v][i] - g - x[v][i] * gx, d[v][i]);
                d[v].set(i, dx[v][i]);
            }
        C.store(dstream, row, d);
        if (Y == kNoBlock) continue;
        gx = g = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[v][i] = Y == kNormedBlock ? (y[v][i] - my) * ry : y[v][i];
                sums[kSumDY][v][i] = fmaf(dx[v][i], x[v][i], sums[kSumDY][v][i]);
                if (BIASES) sums[kSumD][v][i] += dx[v][i];
                dx[v][i] *= A.scale * gate[v][i];
                if (Y == kNormedBlock) {
                    dx[v][i] *= C.there(v) ? (float)wy[v][i] : 0.f;
                    gx = fmaf(dx[v][i], x[v][i], gx);
                    g += dx[v][i];
                }
            }
        Eight<_Float16> dy[V];
        if (Y == kNormedBlock) {
            total(gx, g);
            gx *= over;
            g = layer ? g * over : 0.f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) dy[v].set(i, Y == kNormedBlock ? ry * (dx[v][i] - g - x[v][i] * gx) : dx[v][i]);
        C.store(A.dy, row, dy);
    }
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (A.of_sum[k] < 0 || (!BIASES && (k == kSumOut || k == kSumD))) continue;
        Eight<float> mine[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) mine[v].set(i, sums[k][v][i]);
        C.store(A.partial, (int64_t)A.of_sum[k] * gridDim.x + blockIdx.x, mine);
    }
}

// The vectors' gradients from the workgroups' sums: 32 columns to a workgroup, half a wave takes every 32nd row.
constexpr int kJoinThreads = 1024, kJoinColumns = 32, kJoinRows = kJoinThreads / kJoinColumns;
__global__ void __launch_bounds__(kJoinThreads) norm_join_kernel(const NormArgs A, int rows)
{
    __shared__ float meeting[kSums][kJoinRows][kJoinColumns + 1];
    const int first = threadIdx.x / kJoinColumns, lane = threadIdx.x % kJoinColumns, column = (int)blockIdx.x * kJoinColumns + lane;
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        float sum = 0.f;
        if (A.of_sum[k] >= 0 && column < A.hidden) {
            const float *from = A.partial + (int64_t)A.of_sum[k] * rows * A.hidden + column;
            for (int row = first; row < rows; row += 8 * kJoinRows) {       // eight loads under way, the last ones of a row that is there
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = from[(int64_t)std::min(row + i * kJoinRows, rows - 1) * A.hidden];
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += row + i * kJoinRows < rows ? x[i] : 0.f;
            }
        }
        meeting[k][first][lane] = sum;
    }
    __syncthreads();
    // the sums of a column by as many lanes as there are sums
    const int k = threadIdx.x / kJoinColumns;
    if (k < kSums) {
        float sum = 0.f;
#pragma unroll
        for (int row = 0; row < kJoinRows; ++row) sum += meeting[k][row][lane];
        meeting[k][0][lane] = sum;
    }
    __syncthreads();
    if (k > 0 || column >= A.hidden) return;
    const float out_x = meeting[kSumOutX][0][lane], out = meeting[kSumOut][0][lane], dy = meeting[kSumDY][0][lane], d = meeting[kSumD][0][lane];
    const float f = A.scale * (A.gate ? (float)A.gate[column] : 1.f), wy = A.y_weight ? (float)A.y_weight[column] : 1.f, by = A.y_bias ? (float)A.y_bias[column] : 0.f;
    if (A.dweight) A.dweight[column] = (_Float16)out_x;
    if (A.dbias) A.dbias[column] = (_Float16)out;
    if (A.dgate) A.dgate[column] = (_Float16)(A.scale * (A.y_norm ? fmaf(wy, dy, by * d) : dy));
    if (A.dy_weight) A.dy_weight[column] = (_Float16)(f * dy);
    if (A.dy_bias) A.dy_bias[column] = (_Float16)(f * d);
}

// A thread has 8 elements of a row, 16 of rows of more than 4096; workgroups go on to rows a grid further.
// Backward: 8 waves a compute unit, of narrow rows 4 workgroups, at least two rows each: what covers the loads' latency with a row under way, and few enough
// to leave few rows of sums.  Both passes, rms before and after with a gate, us, at 4 / 8 / 12 waves a compute unit and more: 8192 x 4096 - / 125 / 125, 130 at 16;
// 2048 x 2560 on fp32 - / 34 / 40; 8192 x 2048 (layer, biases) - / 74 / 76, 89 at 24; 8192 x 512 27 / 30 / 35; 1003 x 1024 (layer) one row each 22, two 19.
// Wider rows: the backward kernel's sums and vectors do not fit its registers.  It spills 20 registers of rows of 4104 to 8192 on an fp32 stream with norms on
// both sides and biases; above 8192 with norms on both sides 16 and 24 (fp16, fp32), with biases 53 and 73, behind a plain block 0 and 11, 31 and 60.
// TB/s, forward and backward with the vectors' sums, rms / layer with biases: 8192 x 5120 fp16 5.2 and 4.9 / 3.4 and 4.8, fp32 5.2 and 5.2 / 4.2 and 3.3;
// 8192 x 8192 5.5 and 4.8 / 4.3 and 4.6, 5.4 and 5.2 / 5.2 and 3.7; 4096 x 16384 4.5 and 3.2 / 3.8 and 1.7, 5.3 and 3.5 / 4.5 and 2.1.
// Forward: 16 waves; of rows of 7 and 8 waves and 8 elements 4 workgroups: 8192 x 4096 125 us with 4, 131 with 2; 2048 x 8192 74 and 70; 8192 x 2560 86 with 6, 83 with 3.
struct NormShape {
    int v, threads, grid;
};
NormShape shape_of(const NormArgs &a, bool backward)
{
    NormShape s;
    s.v = a.hidden <= 8 * kNormThreads ? 1 : 2;
    s.threads = (int)ceil_div(ceil_div(a.hidden, 8 * s.v), 64) * 64;
    const int64_t waves = s.threads / 64, units = compute_units();
    int64_t most = units * (s.v == 1 && waves > 6 ? 4 : std::max<int64_t>(1, 16 / waves));
    if (backward) most = std::max(units, std::min(units * std::min<int64_t>(4, std::max<int64_t>(1, 8 / waves)), (a.tokens + 1) / 2));
    s.grid = (int)std::min(a.tokens, most);
    return s;
}

template <typename S, int V, int THREADS, int Y>
void launch_kernel(bool backward, const NormArgs &a, const NormShape &shape, hipStream_t s)
{
    const dim3 grid((unsigned)shape.grid), threads((unsigned)shape.threads);
    if (!backward) hipLaunchKernelGGL((norm_kernel<S, V, THREADS, Y>), grid, threads, 0, s, a);
    else if (a.of_sum[kSumOut] >= 0 || a.of_sum[kSumD] >= 0) hipLaunchKernelGGL((norm_backward_kernel<S, V, THREADS, Y, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((norm_backward_kernel<S, V, THREADS, Y, false>), grid, threads, 0, s, a);
}
template <typename S, int V, int THREADS>
void launch_block(bool backward, const NormArgs &a, const NormShape &shape, hipStream_t s)
{
    if (!a.y) launch_kernel<S, V, THREADS, kNoBlock>(backward, a, shape, s);
    else if (!a.y_norm) launch_kernel<S, V, THREADS, kPlainBlock>(backward, a, shape, s);
    else launch_kernel<S, V, THREADS, kNormedBlock>(backward, a, shape, s);
}
template <typename S>
void launch_stream(bool backward, const NormArgs &a, const NormShape &shape, hipStream_t s)
{
    if (shape.threads > kNormThreads) launch_block<S, 2, kWideThreads>(backward, a, shape, s);
    else if (shape.v == 2) launch_block<S, 2, kNormThreads>(backward, a, shape, s);
    else launch_block<S, 1, kNormThreads>(backward, a, shape, s);
}
hipError_t launch_rows(bool backward, const NormArgs &a, const NormShape &shape, hipStream_t s)
{
    if (shape.grid == 0) return hipSuccess;
    if (a.stream_fp32) launch_stream<float>(backward, a, shape, s);
    else launch_stream<_Float16>(backward, a, shape, s);
    return hipGetLastError();
}

// Which sums the wanted vectors need, in order; their number.
int number_sums(NormArgs &a)
{
    const bool wanted[kSums] = {a.dweight != nullptr, a.dbias != nullptr, a.dgate || a.dy_weight, a.dy_bias || (a.dgate && a.y_norm && a.y_bias)};
    int count = 0;
    for (int k = 0; k < kSums; ++k) a.of_sum[k] = wanted[k] ? count++ : -1;
    return count;
}

}  // namespace

size_t norm_workspace(NormArgs a) { return (size_t)number_sums(a) * (size_t)shape_of(a, true).grid * (size_t)a.hidden * sizeof(float); }

hipError_t launch_norm(const NormArgs &a, hipStream_t s) { return launch_rows(false, a, shape_of(a, false), s); }

hipError_t launch_norm_backward(NormArgs a, hipStream_t s)
{
    const NormShape shape = shape_of(a, true);
    const int count = number_sums(a);
    if (hipError_t e = launch_rows(true, a, shape, s)) return e;
    if (count == 0) return hipSuccess;
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)ceil_div(a.hidden, kJoinColumns)), dim3(kJoinThreads), 0, s, a, shape.grid);
    return hipGetLastError();
}

}  // namespace samo
