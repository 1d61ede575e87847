// Internal declarations shared by the translation units of libsamo (gfx950 only).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "samo.h"

namespace samo {

// Launch shapes, chosen by measurement on MI355X.  A tile workgroup (256 threads) owns a run of
// whole segments of a layer of about equal weight kTileCost, where a segment weighs kSegCost plus
// kNnzCost per kept element: at 90 % pruning that is about 4 segments (4096 dense elements, 16
// per thread — 8 or 32 per thread lose 10-15 %), 3 at 80 %, 2 at 50 %, 5-6 where nothing is kept,
// one segment per workgroup in an unpruned layer; a model that keeps under 7 % is cut with
// twice the weight (kTileCostSparse), 8-9 segments at 95 % pruning.  The weights follow the fused step's traffic
// (4 bytes per dense element, 28 per kept one) with the dense side weighted up: swept over
// (4096..16384, 8..28, 20K..64K) on the GPT shapes, this choice is within 1 % of the best at 80, 90
// and 95 % uniform pruning and 6 % ahead of fixed 4096-element tiles on row-clustered masks.  Even
// weights per workgroup keep the traffic in flight per compute unit steady whatever the local
// density (clustered masks, mixed pruned and dense layers), so one occupancy target fits all.
// Flat kernels: one 64-lane wave per workgroup with one float4 per array.
constexpr int kThreads = 256;           // index kernels: 4 wavefronts per workgroup
constexpr int kTileThreads = 256;       // tile kernels that run an optimizer step
constexpr int kExpandThreads = 128;     // expansion only: little read traffic per tile, so more, smaller workgroups
                                        // per compute unit (+15 % over 256 threads; the step kernels lose with 128)
constexpr int kSeg = SAMO_SEG_ELEMS;    // dense elements per seg_ptr entry
constexpr int64_t kTileCost = 32768;    // target weight of one tile workgroup
constexpr int64_t kTileCostSparse = 65536;   // the same for a model with less than kSparseKeep of its elements kept: the
                                        // kernels that do not read the dense gradient move too few bytes per tile there
                                        // for the workgroups a compute unit holds (measured at 95 % pruning, weights
                                        // 32K / 48K / 64K: the compressed-gradient step 0.705 / 0.754 / 0.765 of peak,
                                        // the expansion 0.716 / 0.747 / 0.765, the fused step 0.81 throughout)
constexpr int64_t kTileCostSparse32 = 49152; // ... where the dense side is fp32 (single-precision SAMO): 0.78 / 0.80 / 0.73
constexpr double kSparseKeep = 0.07;
constexpr int64_t kSegCost = 6144;      // weight of a segment's dense side (fp16 gradient lines read, fp16 weights written)
constexpr int64_t kNnzCost = 24;        // weight of a kept element (idx, p, m, v read; p, m, v written)
constexpr int64_t kTileCostMax = 98304;   // what SAMO_KNOB_TILE_COST may ask for
constexpr int kMaxTileSegs = (int)((kTileCostMax + kSegCost - 1) / kSegCost);   // of any tile: reached where nothing is kept
// The tile weight of a model (a plan, or a layer launched by itself) and the segments its heaviest
// tile can hold: the size of the workgroups' LDS image, which is requested at launch.
int knob(int which, int fallback);
inline int64_t tile_cost_for(int64_t n, int64_t nnz, bool dense_fp32)
{
    const int64_t forced = (int64_t)knob(SAMO_KNOB_TILE_COST, 0) * 1024;      // tuning aid
    if (forced >= kSegCost && forced <= kTileCostMax) return forced;
    if (n > 0 && (double)nnz < kSparseKeep * (double)n) return dense_fp32 ? kTileCostSparse32 : kTileCostSparse;
    return kTileCost;
}
inline int tile_cost_segs(int64_t cost) { return (int)((cost + kSegCost - 1) / kSegCost); }
constexpr int kFlatThreads = 64;        // flat kernels over the compressed arrays
constexpr int kChunk = 256;             // compressed elements per workgroup in the flat kernels
constexpr int kStatReduceGrid = 1024;    // workgroups of the first level of the gradient-statistics reduction
constexpr int kTileUnrollFp32 = 4;      // compressed elements in flight per thread in the single-precision tile kernel

static_assert(kMaxTileSegs >= 1 && kMaxTileSegs < 256, "the segment count of a tile record is an 8-bit field");
static_assert(kSeg % 8 == 0, "a tile is written out as whole 16-byte vectors");
static_assert(kChunk % (4 * kFlatThreads) == 0, "a chunk is whole float4 vectors per thread");

// Optimizer constants prepared on the host in double precision, rounded once to fp32.
struct AdamK {
    float lr, b1, b2, omb1, omb2, eps, wd;
    float rbc1, rbc2;   // 1 / (1 - beta^t)
    int l2, decoupled;
};
struct OptK {
    AdamK adam;
    float sgd_lr, sgd_mu, sgd_wd;
};

// Clipping / overflow guard evaluated on the device from the gradient statistics.
struct GuardK {
    const samo_grad_stats *stats;   // NULL: no guard
    float max_norm;                 // <= 0: no clipping
    int skip;                       // leave all state untouched if stats->nonfinite
};

enum { kModeDecompress = 0, kModeStep = 1 };
enum { kGradDense = 0, kGradC16 = 1, kGradC32 = 2, kGradDense32 = 3 };   // where a step / the statistics read the gradient
enum { kOptAdam = 0, kOptSgd = 1 };
enum { kOutF32 = 0, kOutF16 = 1, kOutNone = 2 };        // what the flat gather kernel writes

// Workgroup -> work record of the batched launches.  Chunk records (flat kernels): local = chunk
// index within the layer.  Tile records: local = first segment | number of segments << 24 (a
// layer has at most 2^21 segments).
struct WgRec {
    int32_t layer;
    uint32_t local;
};
constexpr int kRecSegShift = 24;

// One (sum of squares, non-finite flag) partial per workgroup of a flat launch.
struct StatPartial {
    double sum_squares;
    int64_t nonfinite;
};

// Process-wide tuning and testing knobs (samo_debug_set); `dflt` where a knob holds SAMO_KNOB_DEFAULT.
int knob(int which, int dflt);

// Up to kIndexBatchJobs index-build jobs, passed to the kernels by value (kernel argument segment).
constexpr int kIndexBatchJobs = 48;
constexpr int kFlagGroupSegs = 8;          // segments whose flag words are one group of 64 uint4 (1 KiB), a lane's four words adjacent
constexpr int kIndexSpinLimit = 1 << 20;   // about a second of polling
struct IndexBatch {
    int num;
    int wg_start[kIndexBatchJobs + 1];   // exclusive prefix of workgroups per job
    const uint8_t *mask[kIndexBatchJobs];
    int64_t n[kIndexBatchJobs];
    int32_t *idx[kIndexBatchJobs];
    int64_t cap[kIndexBatchJobs];
    int32_t *seg_ptr[kIndexBatchJobs];
    int64_t *nnz[kIndexBatchJobs];
    uint4 *flags[kIndexBatchJobs];       // NULL, or where a counting launch leaves the flag words and the fill launch reads them
    int64_t *mirror;                     // NULL, or page-locked host memory: where a counting launch puts the jobs' counts besides *nnz
    int passes;                          // 64 KiB passes a workgroup of the chained kernel makes over its block: 1, 2 or 4
    int spin_limit;                      // polls of a missing predecessor before a workgroup gives up
    int64_t *ticket;                     // the nnz of the job that owns the last workgroup: zero before the
                                         // launch, counts the workgroups as they start, final once that one ends
};
static_assert(sizeof(IndexBatch) <= 3072, "the job table must fit the kernel argument segment");

// Of `count` positions on their way to idx[at ..], how many may be stored where idx has room for cap: those
// inside [0, cap) from `at` on, none if `at` is not an offset into it.
__host__ __device__ inline int storable(int64_t cap, int64_t at, int count)
{
    if (at < 0 || at >= cap) return 0;
    return cap - at < count ? (int)(cap - at) : count;
}

// Compute units of the current device (looked up once per device; 256 if the query fails).
int compute_units();

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- launchers (each returns hipGetLastError() after enqueueing) -----------------------
hipError_t launch_index_batch(const IndexBatch &batch, hipStream_t s);
// Counting without a chain (rewrites batch.wg_start for its own kernels); flags: leaves the flag words as well.
hipError_t launch_index_count(IndexBatch &batch, bool flags, hipStream_t s);
hipError_t launch_index_fill(const IndexBatch &batch, hipStream_t s);
int64_t index_job_workgroups(int64_t n, int passes);
int64_t index_fill_workgroups(int64_t n);
int index_passes_for(int64_t mask_bytes, int compute_units);
hipError_t launch_seg_ptr_from_idx(const int32_t *idx, int64_t nnz, int64_t n, int32_t *seg_ptr,
                                   hipStream_t s);
hipError_t launch_validate(const int32_t *idx, int64_t nnz, int64_t n, const int32_t *seg_ptr,
                           int32_t *ok, hipStream_t s);

// `layers`/`recs` NULL: single-layer launch of `one`; else batched over the plan's tables.
struct LaunchSet {
    samo_layer one;
    const samo_layer *layers;
    const WgRec *recs;
    int64_t wgs;
    int segs_per_tile;   // single-layer tile launches: workgroup b owns segments [b * this, (b + 1) * this)
    float keep;          // kept fraction nnz / n of the work (plan average); steers the flat kernels' occupancy target
    float kept;          // the same of its pruned layers alone; negative: it has none
    int num_layers;      // layers of the plan
    int max_segs;        // tile launches: segments the workgroups' LDS image holds (no tile of the launch has more)
    bool backwards = false;   // tile launches of a plan: the last record first
};
// Segments per tile of a single-layer launch, from the layer's average density.
int single_layer_tile_segs(int64_t n, int64_t nnz, bool dense, bool dense_fp32);
// Up to kPlanBatchLayers layer descriptors of a plan with the starts of their tile and chunk records,
// passed to plan_write_kernel by value: the host table reaches the device without a copy.
constexpr int kPlanBatchLayers = 24;
struct PlanBatch {
    int first, count;                                 // layers [first, first + count) of the plan
    samo_layer layer[kPlanBatchLayers];
    int64_t tile_start[kPlanBatchLayers + 1];         // entry `count` is the start of layer first + count
    int64_t chunk_start[kPlanBatchLayers + 1];
};
static_assert(sizeof(PlanBatch) <= 3072, "the layer table must fit the kernel argument segment");
// Device tables of a plan inside the caller's workspace.
struct PlanTables {
    samo_layer *layers;
    int64_t *tile_start, *chunk_start;                // num_layers + 1 entries each
    WgRec *tiles, *chunks;
};
hipError_t launch_plan_write(const PlanBatch &batch, const PlanTables &t, hipStream_t s);
// Fills the tile and chunk records of every layer (reads the tables plan_write_kernel wrote and the layers' seg_ptr).
hipError_t launch_plan_records(const PlanTables &t, int num_layers, int64_t ntiles, int64_t nchunks, int64_t tile_cost,
                               hipStream_t s);
hipError_t launch_tile(int mode, int gsrc, int opt, const LaunchSet &ls, float inv_scale, const OptK &k,
                       const GuardK &guard, hipStream_t s);
hipError_t launch_tile_fp32(const LaunchSet &ls, float factor, const OptK &k, const GuardK &guard, hipStream_t s);
hipError_t launch_gather(int out, int src, const LaunchSet &ls, float inv_scale, int accumulate,
                         StatPartial *partials, hipStream_t s);
hipError_t launch_flat_step(int opt, const LaunchSet &ls, const OptK &k, const GuardK &guard, hipStream_t s);
int64_t stats_workspace_partials(int64_t gather_wgs);
hipError_t launch_stats_finalize(StatPartial *partials, int64_t gather_wgs, samo_grad_stats *out, hipStream_t s);

// Weight gradients dY^T X of up to kWgradMaxJobs linear layers, each gathered at its layer's index, in
// one launch (out_kind: kOutF32 or kOutF16; gc of that type).
constexpr int kWgradMaxJobs = SAMO_WGRAD_MAX_JOBS;
struct WgradJob {
    const _Float16 *dy;      // tokens x out
    const _Float16 *x;       // tokens x in
    int64_t tokens;
    int out, in;
    const int32_t *idx;
    const int32_t *seg_ptr;
    int64_t nnz;
    void *gc;
};
// With a workspace (wgrad_workspace bytes) the tokens of small layers are split over several workgroups.
hipError_t launch_wgrad(int out_kind, const WgradJob *jobs, int count, float inv_scale, int accumulate, void *ws,
                        size_t ws_bytes, hipStream_t s);
hipError_t wgrad_workspace(const WgradJob *jobs, int count, size_t *bytes);
// Function attributes of the weight-gradient kernels and the compute-unit count of the current device (once per device).
hipError_t wgrad_configure(int *cus);
constexpr int kMfmaRateWaves = 8;          // waves per workgroup of launch_mfma_rate, 16 MFMAs of 16 x 16 x 32 each per iteration
hipError_t launch_mfma_rate(int64_t iters, float *sink, int workgroups, hipStream_t s);

// The optimizer phase with 8-bit states (step8.hip).  A workgroup has kStep8Threads / 64 waves and takes that many segments in each
// of `rounds` rounds, of the layer `one` or, with layers set, of the one its record names with its first segment.
constexpr int kStep8Threads = 256;
constexpr int kStep8MaxRounds = 4;
struct Step8Launch {
    samo_layer8 one;
    const samo_layer8 *layers;
    const uint64_t *recs;
    int64_t wgs;
    int rounds;
    int wide;                // a layer of the launch keeps a fifth and more
};
struct Step8Args {
    AdamK adam;
    GuardK guard;
    float inv_scale;
    int from_message;        // the gradient is gc16, not g at idx
    uint32_t key;            // of the stochastic rounding: seed and step
};
constexpr int kPlan8Batch = 20;
struct Plan8Batch {
    int first, count, rounds;
    samo_layer8 layer[kPlan8Batch];
    int64_t rec_at[kPlan8Batch], recs[kPlan8Batch];   // a layer's first record and their number
};
static_assert(sizeof(Plan8Batch) <= 3072, "the layer table must fit the kernel argument segment");
hipError_t launch_plan8_write(const Plan8Batch &b, samo_layer8 *layers, void *recs, hipStream_t s);
hipError_t launch_step8(const Step8Launch &ls, bool dense, const Step8Args &a, hipStream_t s);
hipError_t launch_state8(const Step8Launch &ls, bool pack, hipStream_t s);

// Attention (attention.hip): tensors of tokens x heads x dim, a row's elements adjacent, strides in elements.
typedef float f32x2 __attribute__((ext_vector_type(2)));
struct AttnForm {                           // of the scores; all zero: scale q k
    float cap;                              // 0: none
    const float *slopes;                    // heads, NULL: none
    const _Float16 *table;                  // heads x columns, NULL: none
    const int32_t *borders;                 // buckets - 1
    int buckets, two_sided;                 // of a direction; columns: buckets, twice as many if two_sided
    const int32_t *first_keys;              // batch, NULL: none
    _Float16 *dtable;                       // NULL: not wanted
    float *dtable_parts;
};
struct AttnArgs {
    const _Float16 *q, *k, *v, *dout;
    _Float16 *out, *dq, *dk, *dv;
    float *lse, *delta;                     // heads x q_tokens
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head, dout_row, dout_head, dq_row, dq_head, dk_row, dk_head, dv_row, dv_head;
    const int32_t *q_start, *k_start;       // batch + 1 each, NULL: one sequence of all tokens
    int64_t q_tokens, k_tokens;
    int batch, heads, kv_heads, group, dim, max_q, max_k, causal, window;
    int tiles, splits;                      // of own rows a head, and parts of what they are multiplied with; set by the launch
    float scale;
    float *parts;                           // NULL: a launch is not split
    f32x2 *part_stats;
    int pack;                               // forward: heads of a query that a tile's rows hold, 1 or group
    int few;                                // forward, scored: a sequence's rows are at most 32, behind more than two tiles of keys
    int scored;                             // whether form is looked at
    AttnForm form;
};
// Whether the call's launches can be made.
bool attention_fits(const samo_attention_desc &d, bool backward);
// Bytes that a call can use at `parts`; with less a launch that would need them is not split.
int64_t attention_sums_bytes(const AttnArgs &a, bool backward);
// Sets pack and few of a scored call: group where a form's kernels can and a sequence's rows are one tile.
void attention_pack(AttnArgs &a);
// Bytes that a backward call needs at form.dtable_parts.
int64_t attention_table_bytes(const AttnArgs &a);
hipError_t launch_attention(const AttnArgs &a, size_t bytes, hipStream_t s);
hipError_t launch_attention_backward(const AttnArgs &a, size_t bytes, hipStream_t s);

// A launch's kernel for scores of another form (which: forward, dQ, dK and dV).
hipError_t launch_attention_keys(int which, const AttnArgs &a, int64_t items, hipStream_t s);
hipError_t launch_attention_cap(int which, const AttnArgs &a, int64_t items, hipStream_t s);
hipError_t launch_attention_slope(int which, const AttnArgs &a, int64_t items, hipStream_t s);
hipError_t launch_attention_table(int which, const AttnArgs &a, int64_t items, hipStream_t s);
hipError_t launch_attention_cap_slope(int which, const AttnArgs &a, int64_t items, hipStream_t s);
hipError_t launch_attention_cap_table(int which, const AttnArgs &a, int64_t items, hipStream_t s);
hipError_t launch_attention_all(int which, const AttnArgs &a, int64_t items, hipStream_t s);

// The gated feed-forward block (glu.hip).
struct GluArgs {
    const _Float16 *x, *w_gate, *w_up;      // tokens x in, ffn x in
    _Float16 *h, *gate, *up;                // tokens x ffn; gate and up NULL: not kept; read in the backward pass
    const _Float16 *dh;
    _Float16 *dgate, *dup, *dx;             // dx NULL: not wanted
    float *partial;                         // splits > 1: fp32 sums, splits x tokens x in
    int64_t tokens;
    int in, ffn;
    int tiles_t, tiles_f, splits, part_stages;
};
constexpr int kGluSkinny = 32;             // tokens up to which the weights go past LDS
constexpr int kGluMaxSplits = 16;
struct GluShape {
    int shape = 0, splits = 1, part_stages = 0;
};
// The tile shape of dX and the parts its summation is split into, at most max_splits.
GluShape glu_dx_shape(int64_t tokens, int64_t ffn, int64_t in, int max_splits);
// Whether the launches of a call, its sizes otherwise in order, can be made.
bool glu_fits(int64_t tokens, int64_t in, int64_t ffn);
bool glu_backward_fits(int64_t tokens, int64_t in, int64_t ffn, const GluShape &shape);
hipError_t launch_glu(int act, const GluArgs &a, hipStream_t s);
hipError_t launch_glu_backward(int act, GluArgs a, const GluShape &shape, hipStream_t s);

// The norms around a block (norm.hip).
struct NormArgs {
    int64_t tokens;
    int hidden, layer, y_norm, stream_fp32;
    float eps, scale;
    const void *stream;
    const _Float16 *y, *weight, *bias, *y_weight, *y_bias, *gate;     // NULL: none
    void *new_stream;                       // read in the backward pass
    _Float16 *out;
    float *stats;                           // tokens x 4, NULL: not kept
    const _Float16 *dout;
    const void *dnew;
    void *dstream;
    _Float16 *dy, *dweight, *dbias, *dy_weight, *dy_bias, *dgate;     // NULL: not wanted
    float *partial;
    int of_sum[4];                          // which row of partial a sum has; set by the launch
};
size_t norm_workspace(NormArgs a);
hipError_t launch_norm(const NormArgs &a, hipStream_t s);
hipError_t launch_norm_backward(NormArgs a, hipStream_t s);

hipError_t launch_copy(void *dst, const void *src, int64_t bytes, hipStream_t s);

}  // namespace samo
