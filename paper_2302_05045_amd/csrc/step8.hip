// The fused optimizer phase (Section III-C: compression, Adam, 16-bit copy, expansion in one pass) with Adam's two states held in
// 8 bits each: Section III-D counts 24 bytes a kept element, of which this library's fused pipeline keeps 16 (idx, p, m, v);
// with these states 10.
//
// Format.  The kept elements of one segment (1024 dense elements) form a block: m and v of a block share a power of two each, 8 bits
// of exponent.  A power of two, because scaling by it is exact: a state is rounded once when it is stored and not at all when it is
// read.  The codes:
//   m  sign, 4 bits of exponent, 3 of mantissa, subnormals: (1 + f/8) 2^(e-7) or f/8 2^-6 units; the block's largest lies in [128, 256]
//   v  5 bits of exponent, 3 of mantissa, subnormals, no sign: (1 + f/8) 2^(e-31) or f/8 2^-30 units; the largest in [1/2, 1]
// v has the wider range because Adam takes its square root: both resolve 2^-17 of the block's largest value of m and of sqrt(v).
// Codes and scales that are all zero are a state of zeros.  A block whose m or v is not finite (v: not below 2^126) has scale 255 there
// and reads as NaN, as m and v in 32 bits would.
//
// Rounding.  To nearest, an average with beta2 = 0.999 would stand still: a step moves v by less than half of the 2^-3 between two
// codes.  So it is rounded up or down by chance, with the expectation that is exact (16 random bits, a hash of seed, step
// and the element's position: the same call gives the same bits).  v > 0 is never stored as 0: the step divides by its root.
//
// Work.  A block belongs to one wave, which needs no other: it reads the segment's bounds, brings the segment's dense gradient to
// LDS as whole 16-byte vectors beside idx, p and the codes, steps its elements in registers, finds the two largest exponents (one
// packed maximum across the wave), stores codes, scales and p, and writes the dense weights from the image that takes the gradient's
// place in LDS.  Nothing waits for another wave; 16 bytes a kept element and 4 a dense one, bound by HBM.
// Unpruned layers have a kernel of their own: no idx, four consecutive elements to a lane, no image.
#include "common.h"

namespace samo {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));

#define SAMO_CONSTANT __attribute__((address_space(4)))       // memory that no launch writes while it reads it through this

constexpr int kWaves = kStep8Threads / 64;

__device__ __forceinline__ float as_float(uint32_t b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ uint32_t as_bits(float f) { return __builtin_bit_cast(uint32_t, f); }
// The bits that a block's scale adds to its elements' exponent fields: a quiet NaN's where the block is one, else none.
__device__ __forceinline__ uint32_t nan_of(uint32_t scale) { return scale == 255u ? 0x7FC00000u : 0u; }

// The codes are the leading bits of 32-bit numbers near the least normal one, where fp32's own subnormals are the format's: exponent and
// three bits of mantissa begin at bit 20, and a power of two takes them to their place (m: 2^120, v: 2^96 and the scale).  One ldexp
// does all of it, exactly in reading, with the one rounding of a value below the smallest normal number in writing.
__device__ __forceinline__ float decode_m(uint32_t code, uint32_t scale, uint32_t nan)
{
    return as_float(as_bits(ldexpf(as_float((code & 127u) << 20 | nan), (int)scale - 7)) | (code << 24 & 0x80000000u));
}
__device__ __forceinline__ float decode_v(uint32_t code, uint32_t scale, uint32_t nan) { return ldexpf(as_float(code << 20 | nan), (int)scale - 31); }

// Scale codes from the block's largest exponent fields.
__device__ __forceinline__ uint32_t scale_m(uint32_t top) { return top >= 255u ? 255u : top > 8u ? top - 7u : 1u; }
__device__ __forceinline__ uint32_t scale_v(uint32_t top) { return top >= 253u ? 255u : top + 1u; }

// Both codes of an element, m's in the low byte: the 20 bits behind a code decide with the noise's whether it is the next one.
__device__ __forceinline__ uint32_t encode(float m, float v, uint32_t sm, uint32_t sv, uint32_t noise_m, uint32_t noise_v)
{
    const uint32_t there = (sm == 255u ? 0u : 0xFFu) | (sv == 255u ? 0u : 0xFF00u);
    const uint32_t cm = ((as_bits(ldexpf(fabsf(m), 7 - (int)sm)) + noise_m) >> 20) | (as_bits(m) >> 24 & 128u);
    uint32_t cv = (as_bits(ldexpf(v, 31 - (int)sv)) + noise_v) >> 20;
    const uint32_t least = as_bits(v) < 1u ? as_bits(v) : 1u;            // v > 0 is never stored as 0
    cv = cv > least ? cv : least;
    return (cv << 8 | (cm & 255u)) & there;
}

// 32 well mixed bits of the element's number and the call's key: shifts and odd multipliers in turn (the golden ratio's digits, those of
// sqrt(2) and of sqrt(19)).
__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x = (x ^ x >> 16) * 0x9E3779B1u;
    x = (x ^ x >> 15) * 0x6A09E667u;
    x = (x ^ x >> 13) * 0x5BE0CD19u;
    return x ^ x >> 16;
}

// The largest of both halves over the wave, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t both)
{
    u16x2 a = __builtin_bit_cast(u16x2, both);
#define SAMO_MAX_STEP(ctrl, rows) \
    a = __builtin_elementwise_max(a, __builtin_bit_cast(u16x2, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, a), ctrl, rows, 0xF, false)))
    SAMO_MAX_STEP(0xB1, 0xF);                     // quad_perm 1 0 3 2
    SAMO_MAX_STEP(0x4E, 0xF);                     // quad_perm 2 3 0 1
    SAMO_MAX_STEP(0x141, 0xF);                    // row_half_mirror
    SAMO_MAX_STEP(0x140, 0xF);                    // row_mirror
    SAMO_MAX_STEP(0x142, 0xA);                    // row_bcast15 into rows 1 and 3
    SAMO_MAX_STEP(0x143, 0xC);                    // row_bcast31 into rows 2 and 3
#undef SAMO_MAX_STEP
    return (uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, a), 63);
}

// The largest |m| and v so far, as bits (those of a NaN are the largest of all), and both over the wave as exponent fields.
struct Largest {
    uint32_t m = 0, v = 0;
    __device__ __forceinline__ void take(float a, float b)
    {
        const uint32_t am = as_bits(a) & 0x7FFFFFFFu, bv = as_bits(b) & 0x7FFFFFFFu;
        m = m > am ? m : am;
        v = v > bv ? v : bv;
    }
    __device__ __forceinline__ uint32_t fields() const { return wave_max(m >> 23 | (v >> 23) << 16); }
};

// The new states, in 32 bits: each product and sum rounded by itself, so that the codes do not hang on which of them a compiler fuses.
__device__ __forceinline__ void new_states(float &m, float &v, float g, const AdamK &k)
{
#pragma clang fp contract(off)
    const float m0 = m * k.b1, m1 = g * k.omb1;
    m = m0 + m1;
    const float v0 = v * k.b2, v1 = (g * k.omb2) * g;
    v = v0 + v1;
}

__device__ __forceinline__ float new_parameter(float p, float m, float v, const AdamK &k)
{
    // The root and the quotient by the hardware's approximations (1 ulp each): the update is off by 2^-21 of itself, and the kernels, whose
    // vector ALU is nearly as busy as HBM where little is pruned, have a fifth fewer instructions.  2^-120 keeps the root's argument
    // above the subnormal numbers, which it does not take; it is the root of v that is below 2^-48 without it.
    const float root = __builtin_amdgcn_sqrtf(fmaf(v, k.rbc2, 0x1p-120f));
    const float upd = fmaf(k.decoupled ? k.wd : 0.f, p, m * k.rbc1 * __builtin_amdgcn_rcpf(root + k.eps));
    return fmaf(-k.lr, upd, p);
}

// fp32 -> fp16 of the value that is stored as the parameter (the asm keeps the conversion apart from the update's last fma).
__device__ __forceinline__ _Float16 to_half(float x)
{
    asm("" : "+v"(x));
    return (_Float16)x;
}

__device__ __forceinline__ float guard(const GuardK &gd, bool *skip)
{
    *skip = false;
    if (!gd.stats) return 1.f;
    const samo_grad_stats s = *gd.stats;
    if (gd.skip && s.nonfinite) *skip = true;
    if (gd.max_norm > 0.f) {
        const double c = (double)gd.max_norm / (sqrt(s.sum_squares) + 1e-6);
        if (c < 1.0) return (float)c;
    }
    return 1.f;
}

__device__ __forceinline__ samo_layer8 constant_layer(const samo_layer8 *layer)
{
    const SAMO_CONSTANT samo_layer8 *C = (const SAMO_CONSTANT samo_layer8 *)layer;
    samo_layer8 L;
    L.n = C->n; L.nnz = C->nnz; L.idx = C->idx; L.seg_ptr = C->seg_ptr; L.p = C->p; L.q8 = C->q8; L.s8 = C->s8; L.w = C->w; L.g = C->g;
    L.gc16 = C->gc16; L.m = C->m; L.v = C->v; L.rng_offset = C->rng_offset;
    return L;
}

// The workgroup's layer and its first segment.
__device__ __forceinline__ int64_t pick(const Step8Launch &ls, samo_layer8 *L)
{
    if (!ls.layers) {
        *L = ls.one;
        return (int64_t)blockIdx.x * kWaves * ls.rounds;
    }
    const uint64_t rec = *(const SAMO_CONSTANT uint64_t *)(ls.recs + blockIdx.x);
    *L = constant_layer(ls.layers + (uint32_t)rec);
    return (int64_t)(uint32_t)(rec >> 32);
}

// Kept elements [lo, lo + count) of the segment that the wave owns, E to a lane.
template <int E>
__device__ __forceinline__ void step_block(const samo_layer8 &L, int64_t seg, int lo, int count, _Float16 *image, bool from_message,
                                           const AdamK &k, float factor, uint32_t key)
{
    const int lane = threadIdx.x & 63;
    const uint32_t old_scale = *reinterpret_cast<const uint16_t *>(L.s8 + 2 * seg);
    const int64_t first = seg * kSeg;
    int at[E];
    float p[E], m[E], v[E];
    uint32_t code[E];
    _Float16 gm[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = lane + 64 * e;
        const bool on = i < count;
        at[e] = on ? L.idx[lo + i] : -1;
        p[e] = on ? L.p[lo + i] : 0.f;
        code[e] = on ? reinterpret_cast<const uint16_t *>(L.q8)[lo + i] : 0u;
        gm[e] = on && from_message ? __builtin_bit_cast(_Float16, L.gc16[lo + i]) : (_Float16)0.f;
    }
    const uint32_t sm_old = old_scale & 255u, sv_old = old_scale >> 8, nan_m = nan_of(sm_old), nan_v = nan_of(sv_old);
    Largest largest;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (!from_message) gm[e] = image[(at[e] - (int)first) & (kSeg - 1)];
        m[e] = v[e] = 0.f;
        if (at[e] >= 0) {
            float g = (float)gm[e] * factor;
            if (k.l2) g = fmaf(k.wd, p[e], g);
            m[e] = decode_m(code[e] & 255u, sm_old, nan_m);
            v[e] = decode_v(code[e] >> 8, sv_old, nan_v);
            new_states(m[e], v[e], g, k);
            p[e] = new_parameter(p[e], m[e], v[e], k);
        }
        largest.take(m[e], v[e]);
    }
    const uint32_t top = largest.fields();
    const uint32_t sm = scale_m(top & 0xFFFFu), sv = scale_v(top >> 16);
    // the gradient has been read: the image of the new weights takes its place (a wave's LDS accesses keep their order)
    __builtin_amdgcn_wave_barrier();
    u32x4 *vec = reinterpret_cast<u32x4 *>(image);
    vec[lane] = u32x4{0, 0, 0, 0};
    vec[lane + 64] = u32x4{0, 0, 0, 0};
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (at[e] < 0) continue;
        const int i = lo + lane + 64 * e;
        const uint32_t h = mix((L.rng_offset + (uint32_t)at[e]) ^ key);
        const uint32_t c = encode(m[e], v[e], sm, sv, ((h & 0xFFFFu) << 4) + 8u, ((h >> 16) << 4) + 8u);
        reinterpret_cast<uint16_t *>(L.q8)[i] = (uint16_t)c;
        L.p[i] = p[e];
        image[(at[e] - (int)first) & (kSeg - 1)] = to_half(p[e]);
    }
    if (lane == 0) *reinterpret_cast<uint16_t *>(L.s8 + 2 * seg) = (uint16_t)(sm | sv << 8);
}

// The same for any count: the largest exponents first, then the step, each pass four elements to a lane at a time.  (What the second
// pass reads again, the first one has left in the caches.)
__device__ __forceinline__ void step_long_block(const samo_layer8 &L, int64_t seg, int lo, int count, _Float16 *image, bool from_message,
                                             const AdamK &k, float factor, uint32_t key)
{
    const int lane = threadIdx.x & 63;
    const uint32_t old_scale = *reinterpret_cast<const uint16_t *>(L.s8 + 2 * seg);
    const int first = (int)(seg * kSeg);
    const uint32_t sm_old = old_scale & 255u, sv_old = old_scale >> 8, nan_m = nan_of(sm_old), nan_v = nan_of(sv_old);
    auto states = [&](int i, int at, float p, float &m, float &v) {
        const _Float16 gm = from_message ? __builtin_bit_cast(_Float16, L.gc16[lo + i]) : image[(at - first) & (kSeg - 1)];
        const uint32_t code = reinterpret_cast<const uint16_t *>(L.q8)[lo + i];
        float g = (float)gm * factor;
        if (k.l2) g = fmaf(k.wd, p, g);
        m = decode_m(code & 255u, sm_old, nan_m);
        v = decode_v(code >> 8, sv_old, nan_v);
        new_states(m, v, g, k);
    };
    Largest largest;
    for (int i = lane; i < count; i += 64) {
        float m, v;
        states(i, L.idx[lo + i], k.l2 ? L.p[lo + i] : 0.f, m, v);
        largest.take(m, v);
    }
    const uint32_t top = largest.fields();
    const uint32_t sm = scale_m(top & 0xFFFFu), sv = scale_v(top >> 16);
    for (int i = lane; i < count; i += 64) {
        const int at = L.idx[lo + i];
        float p = L.p[lo + i], m, v;
        states(i, at, p, m, v);
        p = new_parameter(p, m, v, k);
        const uint32_t h = mix((L.rng_offset + (uint32_t)at) ^ key);
        const uint32_t c = encode(m, v, sm, sv, ((h & 0xFFFFu) << 4) + 8u, ((h >> 16) << 4) + 8u);
        reinterpret_cast<uint16_t *>(L.q8)[lo + i] = (uint16_t)c;
        L.p[lo + i] = p;
    }
    __builtin_amdgcn_wave_barrier();
    u32x4 *vec = reinterpret_cast<u32x4 *>(image);
    vec[lane] = u32x4{0, 0, 0, 0};
    vec[lane + 64] = u32x4{0, 0, 0, 0};
    __builtin_amdgcn_wave_barrier();
    for (int i = lane; i < count; i += 64) image[(L.idx[lo + i] - first) & (kSeg - 1)] = to_half(L.p[lo + i]);
    if (lane == 0) *reinterpret_cast<uint16_t *>(L.s8 + 2 * seg) = (uint16_t)(sm | sv << 8);
}

// The segment's dense gradient to LDS; the last segment of a layer may be a part of one.
__device__ __forceinline__ void bring_gradient(const uint16_t *g, int64_t n, int64_t seg, _Float16 *image)
{
    const int lane = threadIdx.x & 63;
    const int64_t first = seg * kSeg;
    if (first + kSeg <= n) {
        const u32x4 *from = reinterpret_cast<const u32x4 *>(g + first);
        const u32x4 a = __builtin_nontemporal_load(from + lane), b = __builtin_nontemporal_load(from + lane + 64);
        reinterpret_cast<u32x4 *>(image)[lane] = a;
        reinterpret_cast<u32x4 *>(image)[lane + 64] = b;
        return;
    }
    for (int i = lane; i < (int)(n - first); i += 64) image[i] = __builtin_bit_cast(_Float16, g[first + i]);
}

__device__ __forceinline__ void store_image(uint16_t *w, int64_t n, int64_t seg, const _Float16 *image)
{
    const int lane = threadIdx.x & 63;
    const int64_t first = seg * kSeg;
    if (first + kSeg <= n) {
        const u32x4 *vec = reinterpret_cast<const u32x4 *>(image);
        u32x4 *to = reinterpret_cast<u32x4 *>(w + first);
        __builtin_nontemporal_store(vec[lane], to + lane);
        __builtin_nontemporal_store(vec[lane + 64], to + lane + 64);
        return;
    }
    for (int i = lane; i < (int)(n - first); i += 64) w[first + i] = __builtin_bit_cast(uint16_t, image[i]);
}

// The bounds of a group's segments in the compressed arrays, one to a lane: lane i holds the first entry of segment group + i, inside
// the arrays whatever the table holds.
__device__ __forceinline__ int group_bounds(const samo_layer8 &L, int64_t group, int64_t segments, int rounds)
{
    const int lane = threadIdx.x & 63;
    const int64_t at = group + lane < segments ? group + lane : segments;
    if (lane > kWaves * rounds) return 0;
    if (!L.seg_ptr) return (int)(at * kSeg < L.n ? at * kSeg : L.n);
    const int bound = L.seg_ptr[at];
    return bound < 0 ? 0 : bound > (int)L.nnz ? (int)L.nnz : bound;
}

// WIDE: for layers that keep a fifth and more, whose blocks pass 256 elements: twice the registers, four workgroups to a compute unit.  Bound by HBM: 24
// blocks of the 350M shape, 10 % kept, 273 to 325 us by card (5.2 to 6.2 TB/s); 400 M elements, 25 % kept 595 us, 50 % 885 (5.4).
template <bool WIDE>
__global__ void __launch_bounds__(kStep8Threads, WIDE ? 4 : 6) step8_pruned_kernel(const Step8Launch ls, const Step8Args A)
{
    __shared__ __attribute__((aligned(16))) _Float16 images[kWaves][kSeg];
    bool skip;
    const float factor = A.inv_scale * guard(A.guard, &skip);
    if (skip) return;
    samo_layer8 L;
    const int64_t group = pick(ls, &L);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t segments = (L.n + kSeg - 1) / kSeg;
    _Float16 *image = images[wave];
    const int bound = group_bounds(L, group, segments, ls.rounds);
    for (int r = 0; r < ls.rounds; ++r) {
        const int mine = r * kWaves + wave;
        const int64_t seg = group + mine;
        if (seg >= segments) break;
        if (!A.from_message) bring_gradient(L.g, L.n, seg, image);
        __builtin_amdgcn_wave_barrier();
        const int lo = __builtin_amdgcn_readlane(bound, mine);
        int count = __builtin_amdgcn_readlane(bound, mine + 1) - lo;
        count = count < 0 ? 0 : count > kSeg ? kSeg : count;
        if (count <= 128) step_block<2>(L, seg, lo, count, image, A.from_message, A.adam, factor, A.key);
        else if (count <= 256) step_block<4>(L, seg, lo, count, image, A.from_message, A.adam, factor, A.key);
        else if (WIDE && count <= 512) step_block<8>(L, seg, lo, count, image, A.from_message, A.adam, factor, A.key);
        else if (WIDE) step_block<16>(L, seg, lo, count, image, A.from_message, A.adam, factor, A.key);
        else step_long_block(L, seg, lo, count, image, A.from_message, A.adam, factor, A.key);
        __builtin_amdgcn_wave_barrier();
        store_image(L.w, L.n, seg, image);
        __builtin_amdgcn_wave_barrier();
    }
}

// Unpruned layers: position = entry; a lane has eight consecutive elements of either half of the segment.  206 M elements: 527 to 606 us by card, 6.3 to 5.4
// TB/s.
__global__ void __launch_bounds__(kStep8Threads, 4) step8_dense_kernel(const Step8Launch ls, const Step8Args A)
{
    bool skip;
    const float factor = A.inv_scale * guard(A.guard, &skip);
    if (skip) return;
    samo_layer8 L;
    const int64_t seg = pick(ls, &L) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (seg * kSeg >= L.n) return;
    const int64_t first = seg * kSeg;
    const int count = L.n - first < kSeg ? (int)(L.n - first) : kSeg;
    const bool full = count == kSeg;
    const uint16_t *grad = (A.from_message ? L.gc16 : L.g) + first;
    float *params = L.p + first;
    uint16_t *codes = reinterpret_cast<uint16_t *>(L.q8) + first, *weights = L.w + first;
    const uint32_t old_scale = *reinterpret_cast<const uint16_t *>(L.s8 + 2 * seg);
    const uint32_t sm_old = old_scale & 255u, sv_old = old_scale >> 8, nan_m = nan_of(sm_old), nan_v = nan_of(sv_old);
    float p[16], m[16], v[16];
    uint32_t g2[8], c2[8];                                   // two 16-bit values each
    auto place = [&](int e) { return full ? (e >> 3) * 512 + 8 * lane + (e & 7) : lane + 64 * e; };
    if (full) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 gg = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(grad + 512 * j) + lane);
            const u32x4 cc = *(reinterpret_cast<const u32x4 *>(codes + 512 * j) + lane);
            const f32x4 pa = *reinterpret_cast<const f32x4 *>(params + 512 * j + 8 * lane), pb = *reinterpret_cast<const f32x4 *>(params + 512 * j + 8 * lane + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                g2[4 * j + e] = gg[e];
                c2[4 * j + e] = cc[e];
                p[8 * j + e] = pa[e];
                p[8 * j + 4 + e] = pb[e];
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const int i = place(e), i2 = place(e + 1);
            g2[e / 2] = (i < count ? grad[i] : 0u) | (uint32_t)(i2 < count ? grad[i2] : 0u) << 16;
            c2[e / 2] = (i < count ? codes[i] : 0u) | (uint32_t)(i2 < count ? codes[i2] : 0u) << 16;
            p[e] = i < count ? params[i] : 0.f;
            p[e + 1] = i2 < count ? params[i2] : 0.f;
        }
    }
    Largest largest;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t code = c2[e / 2] >> (e & 1) * 16;
        float g = (float)__builtin_bit_cast(_Float16, (uint16_t)(g2[e / 2] >> (e & 1) * 16)) * factor;
        if (A.adam.l2) g = fmaf(A.adam.wd, p[e], g);
        m[e] = decode_m(code & 255u, sm_old, nan_m);
        v[e] = decode_v(code >> 8 & 255u, sv_old, nan_v);
        new_states(m[e], v[e], g, A.adam);
        if (!full && place(e) >= count) m[e] = v[e] = 0.f;
        p[e] = new_parameter(p[e], m[e], v[e], A.adam);
        largest.take(m[e], v[e]);
    }
    const uint32_t top = largest.fields();
    const uint32_t sm = scale_m(top & 0xFFFFu), sv = scale_v(top >> 16);
    uint32_t w2[8];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t h = mix((L.rng_offset + (uint32_t)(first + place(e))) ^ A.key);
        const uint32_t c = encode(m[e], v[e], sm, sv, ((h & 0xFFFFu) << 4) + 8u, ((h >> 16) << 4) + 8u);
        const uint32_t w = __builtin_bit_cast(uint16_t, to_half(p[e]));
        c2[e / 2] = (e & 1) ? c2[e / 2] | c << 16 : c;
        w2[e / 2] = (e & 1) ? w2[e / 2] | w << 16 : w;
    }
    if (full) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            *reinterpret_cast<f32x4 *>(params + 512 * j + 8 * lane) = f32x4{p[8 * j], p[8 * j + 1], p[8 * j + 2], p[8 * j + 3]};
            *reinterpret_cast<f32x4 *>(params + 512 * j + 8 * lane + 4) = f32x4{p[8 * j + 4], p[8 * j + 5], p[8 * j + 6], p[8 * j + 7]};
            *(reinterpret_cast<u32x4 *>(codes + 512 * j) + lane) = u32x4{c2[4 * j], c2[4 * j + 1], c2[4 * j + 2], c2[4 * j + 3]};
            __builtin_nontemporal_store(u32x4{w2[4 * j], w2[4 * j + 1], w2[4 * j + 2], w2[4 * j + 3]}, reinterpret_cast<u32x4 *>(weights + 512 * j) + lane);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = place(e);
            if (i >= count) continue;
            params[i] = p[e];
            codes[i] = (uint16_t)(c2[e / 2] >> (e & 1) * 16);
            weights[i] = (uint16_t)(w2[e / 2] >> (e & 1) * 16);
        }
    }
    if (lane == 0) *reinterpret_cast<uint16_t *>(L.s8 + 2 * seg) = (uint16_t)(sm | sv << 8);
}

// m and v in 32 bits from the codes; a wave to a segment, whose first 128 elements are asked for before the last round's are stored.  10 % kept of 400 M elements
// 93 us, 4.3 TB/s (a segment's 102 elements are short rows), 50 % 568, 3.5; 206 M unpruned 356 to 382.
__global__ void __launch_bounds__(kStep8Threads) unpack8_kernel(const Step8Launch ls)
{
    samo_layer8 L;
    const int64_t group = pick(ls, &L);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t segments = (L.n + kSeg - 1) / kSeg;
    const uint16_t *codes = reinterpret_cast<const uint16_t *>(L.q8);
    if (!L.seg_ptr) {                                        // a whole segment: eight elements to a lane and half
        const int64_t seg = group + wave;
        if (seg >= segments) return;
        const uint32_t scale = *reinterpret_cast<const uint16_t *>(L.s8 + 2 * seg);
        const uint32_t sm = scale & 255u, sv = scale >> 8, nan_m = nan_of(sm), nan_v = nan_of(sv);
        const int64_t first = seg * kSeg;
        if (first + kSeg <= L.n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t at = first + 256 * j + 4 * lane;
                const u32x2 two = *reinterpret_cast<const u32x2 *>(codes + at);
                f32x4 m, v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t code = two[e / 2] >> (e & 1) * 16;
                    m[e] = decode_m(code & 255u, sm, nan_m);
                    v[e] = decode_v(code >> 8 & 255u, sv, nan_v);
                }
                __builtin_nontemporal_store(m, reinterpret_cast<f32x4 *>(L.m + at));
                __builtin_nontemporal_store(v, reinterpret_cast<f32x4 *>(L.v + at));
            }
            return;
        }
        for (int64_t i = first + lane; i < L.n; i += 64) {
            const uint32_t code = codes[i];
            L.m[i] = decode_m(code & 255u, sm, nan_m);
            L.v[i] = decode_v(code >> 8, sv, nan_v);
        }
        return;
    }
    const int bound = group_bounds(L, group, segments, ls.rounds);
    const uint32_t scales = lane < kWaves * ls.rounds && group + lane < segments ? *reinterpret_cast<const uint16_t *>(L.s8 + 2 * (group + lane)) : 0u;
    constexpr int kAhead = 2;
    uint32_t code[kStep8MaxRounds][kAhead];
#pragma unroll
    for (int r = 0; r < kStep8MaxRounds; ++r) {              // everything of ordinary segments is asked for at once
        const int mine = r * kWaves + wave;
        const int lo = __builtin_amdgcn_readlane(bound, mine), hi = __builtin_amdgcn_readlane(bound, mine + 1);
#pragma unroll
        for (int e = 0; e < kAhead; ++e) code[r][e] = r < ls.rounds && lo + lane + 64 * e < hi ? codes[lo + lane + 64 * e] : 0u;
    }
#pragma unroll
    for (int r = 0; r < kStep8MaxRounds; ++r) {
        if (r >= ls.rounds) break;
        const int mine = r * kWaves + wave;
        const int lo = __builtin_amdgcn_readlane(bound, mine), hi = __builtin_amdgcn_readlane(bound, mine + 1);
        const uint32_t scale = (uint32_t)__builtin_amdgcn_readlane((int)scales, mine);
        const uint32_t sm = scale & 255u, sv = scale >> 8, nan_m = nan_of(sm), nan_v = nan_of(sv);
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int i = lo + lane + 64 * e;
            if (i >= hi) continue;
            L.m[i] = decode_m(code[r][e] & 255u, sm, nan_m);
            L.v[i] = decode_v(code[r][e] >> 8, sv, nan_v);
        }
        for (int i = lo + lane + 64 * kAhead; i < hi; i += 64) {
            const uint32_t c = codes[i];
            L.m[i] = decode_m(c & 255u, sm, nan_m);
            L.v[i] = decode_v(c >> 8, sv, nan_v);
        }
    }
}

// The codes from m and v, rounded to nearest; a wave to a segment, read twice.  Not on a step's path: 10 % kept of 400 M elements 139 us, 2.9 TB/s, 50 % 582, 3.5.
__global__ void __launch_bounds__(kStep8Threads) pack8_kernel(const Step8Launch ls)
{
    samo_layer8 L;
    const int64_t group = pick(ls, &L);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t segments = (L.n + kSeg - 1) / kSeg;
    const int bound = group_bounds(L, group, segments, ls.rounds);
    uint16_t *codes = reinterpret_cast<uint16_t *>(L.q8);
    for (int r = 0; r < ls.rounds; ++r) {
        const int mine = r * kWaves + wave;
        const int64_t seg = group + mine;
        if (seg >= segments) break;
        const int lo = __builtin_amdgcn_readlane(bound, mine), hi = __builtin_amdgcn_readlane(bound, mine + 1);
        Largest largest;
        for (int i = lo + lane; i < hi; i += 64) largest.take(L.m[i], L.v[i]);
        const uint32_t top = largest.fields();
        const uint32_t sm = scale_m(top & 0xFFFFu), sv = scale_v(top >> 16);
        for (int i = lo + lane; i < hi; i += 64) codes[i] = (uint16_t)encode(L.m[i], L.v[i], sm, sv, 1u << 19, 1u << 19);
        if (lane == 0) *reinterpret_cast<uint16_t *>(L.s8 + 2 * seg) = (uint16_t)(sm | sv << 8);
    }
}

// A few layers of a plan and the records of theirs: where the layer's first one goes, and how many segments it stands for.
__global__ void __launch_bounds__(256) plan8_write_kernel(const Plan8Batch B, samo_layer8 *layers, uint2 *recs)
{
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (t < B.count) layers[B.first + t] = B.layer[t];
    int j = 0;
    int64_t before = 0;
    while (j < B.count && t >= before + B.recs[j]) before += B.recs[j++];
    if (j < B.count) recs[B.rec_at[j] + (t - before)] = make_uint2((uint32_t)(B.first + j), (uint32_t)((t - before) * kWaves * (B.layer[j].seg_ptr ? B.rounds : 1)));
}

}  // namespace

hipError_t launch_plan8_write(const Plan8Batch &b, samo_layer8 *layers, void *recs, hipStream_t s)
{
    int64_t threads = b.count;
    int64_t total = 0;
    for (int j = 0; j < b.count; ++j) total += b.recs[j];
    if (total > threads) threads = total;
    if (threads == 0) return hipSuccess;
    hipLaunchKernelGGL(plan8_write_kernel, dim3((unsigned)ceil_div(threads, 256)), dim3(256), 0, s, b, layers, static_cast<uint2 *>(recs));
    return hipGetLastError();
}

hipError_t launch_step8(const Step8Launch &ls, bool dense, const Step8Args &a, hipStream_t s)
{
    if (ls.wgs <= 0) return hipSuccess;
    if (dense) hipLaunchKernelGGL(step8_dense_kernel, dim3((unsigned)ls.wgs), dim3(kStep8Threads), 0, s, ls, a);
    else if (ls.wide) hipLaunchKernelGGL(step8_pruned_kernel<true>, dim3((unsigned)ls.wgs), dim3(kStep8Threads), 0, s, ls, a);
    else hipLaunchKernelGGL(step8_pruned_kernel<false>, dim3((unsigned)ls.wgs), dim3(kStep8Threads), 0, s, ls, a);
    return hipGetLastError();
}

hipError_t launch_state8(const Step8Launch &ls, bool pack, hipStream_t s)
{
    if (ls.wgs <= 0) return hipSuccess;
    if (pack) hipLaunchKernelGGL(pack8_kernel, dim3((unsigned)ls.wgs), dim3(kStep8Threads), 0, s, ls);
    else hipLaunchKernelGGL(unpack8_kernel, dim3((unsigned)ls.wgs), dim3(kStep8Threads), 0, s, ls);
    return hipGetLastError();
}

}  // namespace samo
