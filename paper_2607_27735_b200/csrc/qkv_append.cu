// From a projection's output to the cache in one launch: RMS norm of every head of Q and K, rotation by the row's position,
// Q rounded to bf16 for the attention calls, K and V written to their slots in the form the cache has.
//
//   y = x / sqrt(mean(x^2) + eps) * w;  (y_i, y_j) <- (y_i cos - y_j sin, y_j cos + y_i sin)  for the pairs of the position
//
// Bound by memory: every element is read and written once.  A head of a row is D / 8 neighbouring lanes with 16 bytes
// each, so the norm is a few shuffles, and a pair (i, i + rot / 2) is one more; everything between the load and
// the one rounding at the end is fp32 in registers.
//
// A cache with a scale for each page (SPEC_KV_FP8_E4M3_PAGE) takes a second launch: the rows that a call brings for one page are
// a run of neighbours, whose largest value decides the page's scale before any of them can be stored.  The first launch leaves
// every row's own scale, a power of two, as one byte for each head; the second has the largest of a run's and
// writes the rows.  K is normed and turned twice for that, and in a large call K and V come from memory twice: the first launch
// streams Q through L2 in between (16382 rows of the 32B shape: the second one reads 71 MB, all of K, V and the angles).  Tried in its place: a block for each
// run, with the rows held in registers or staged in shared memory between the largest value and the store.  That has too few
// runs to fill the SMs and a longer chain for each (16382 rows of the 32B shape 176 to 290 us, 2250 rows on 128-token pages 51 to 57;
// so 131 and 25).
// Measured (device): 72 rows of the 8B shape, page scales 5.6 us, both launches chains of latencies; 8195 rows of
// the 8B shape into bf16 44.2 us, 4.6 TB/s; with page scales 16382 rows of the 32B shape 131 us, 3.4 TB/s of the least bytes: K, V
// and their angles are taken twice, and both launches fill two thirds of the issue slots.
// Scales are powers of two: a floating-point byte loses nothing by that but a binade of range, and the rows already in the page
// are rescaled without a second rounding (other than to subnormals) when the scale has to grow.
#include "chained.cuh"
#include "spec_common.cuh"

namespace spec {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kAhead = 4;                 // heads that a lane has in flight
enum Cache { kBf16, kHead8, kPage8 };

struct AppendArgs {
    KvView kv;
    __nv_bfloat16 *k16, *v16;  // the cache, for writing
    uint8_t *k8, *v8;
    float *k_scale, *v_scale;  // per page (written) or per head (read)
    const __nv_bfloat16 *q, *k, *v;
    int64_t q_layer, q_row, k_layer, k_row, v_layer, v_row;
    int n_rows;
    const int32_t* positions;
    const int32_t* slots;
    const __nv_bfloat16 *q_weight, *k_weight;
    float eps;
    const float* cos_sin;
    int max_pos, rot, interleaved;
    __nv_bfloat16* q_out;
    int* status;
    int heads_per_warp, q_parts, kv_parts, row_blocks;  // row part: warps that share a row's Q heads, its K and V heads; its blocks
    uint8_t* need;  // page scales: [K, V][n_layers][n_rows][n_kv_heads in eights] exponents of the rows' own scales
};

__device__ __forceinline__ void unpack(const uint4& w, float (&x)[8])
{
    x[0] = bf16_lo(w.x), x[1] = bf16_hi(w.x), x[2] = bf16_lo(w.y), x[3] = bf16_hi(w.y);
    x[4] = bf16_lo(w.z), x[5] = bf16_hi(w.z), x[6] = bf16_lo(w.w), x[7] = bf16_hi(w.w);
}
__device__ __forceinline__ uint4 pack(const float (&x)[8])
{
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint2 pack_e4m3(const float (&x)[8])
{
    return make_uint2(e4m3x2(x[0], x[1]) | (e4m3x2(x[2], x[3]) << 16), e4m3x2(x[4], x[5]) | (e4m3x2(x[6], x[7]) << 16));
}

// Norm, weight and rotation of a lane's eight elements x as one form, y_i = r (a_i x_i + b_i x'_i) with x' the partners of the
// pairs and r the head's 1 / rms: a and b hold the weights times the cosines and sines and serve every head of a row.
struct Turn {
    float a[8], b[8];
    int off;    // lanes to the partner's lane (0: in the lane itself, or not turned)
    bool on;    // the lane's elements are turned
};
template <int D>
__device__ __forceinline__ Turn load_turn(const AppendArgs& p, const __nv_bfloat16* weight, int layer, const float* row, int l)
{
    Turn t;
    const int e0 = 8 * l, half = p.rot / 2, lane = threadIdx.x & 31;
    float g[8];
    if (weight) {
        unpack(*reinterpret_cast<const uint4*>(weight + (int64_t)layer * D + e0), g);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) t.a[i] = g[i], t.b[i] = 0.f;
    t.off = 0;
    t.on = p.cos_sin != nullptr && e0 < p.rot;
    if (p.cos_sin == nullptr) return t;
    if (p.interleaved) {
        if (t.on) {
            const float4 c = __ldcg(reinterpret_cast<const float4*>(row + e0 / 2)), s = __ldcg(reinterpret_cast<const float4*>(row + half + e0 / 2));
            const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                t.a[2 * i] = g[2 * i] * cc[i];
                t.b[2 * i] = -g[2 * i + 1] * ss[i];
                t.a[2 * i + 1] = g[2 * i + 1] * cc[i];
                t.b[2 * i + 1] = g[2 * i] * ss[i];
            }
        }
        return t;
    }
    const bool second = e0 >= half;
    if (t.on) t.off = second ? -half / 8 : half / 8;
    float gp[8];  // the partners' weights
#pragma unroll
    for (int i = 0; i < 8; ++i) gp[i] = __shfl_sync(0xffffffffu, g[i], lane + t.off);
    if (t.on) {
        const float4* c = reinterpret_cast<const float4*>(row + (second ? e0 - half : e0));
        const float4* n = reinterpret_cast<const float4*>(row + half + (second ? e0 - half : e0));
        const float4 c0 = __ldcg(c), c1 = __ldcg(c + 1), s0 = __ldcg(n), s1 = __ldcg(n + 1);
        const float cc[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, ss[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t.a[i] = g[i] * cc[i];
            t.b[i] = second ? gp[i] * ss[i] : -gp[i] * ss[i];
        }
    }
    return t;
}

// The head's 1 / rms, on each of its lanes (1 without a norm); every lane of the warp takes part.
template <int D>
__device__ __forceinline__ float head_norm(const AppendArgs& p, const uint4& w, bool norm)
{
    if (!norm) return 1.f;
    float x[8], ss = 0.f;
    unpack(w, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int o = D / 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    return rsqrtf(ss * (1.f / D) + p.eps);
}
// Eight elements of a head, normed and turned.
__device__ __forceinline__ void turned(const AppendArgs& p, const Turn& t, const uint4& w, float r, float (&y)[8])
{
    const int lane = threadIdx.x & 31;
    float x[8];
    unpack(w, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = t.a[i] * x[i];
    if (p.cos_sin) {
        float v[8];
        if (p.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x[i ^ 1];
        } else {
            unpack(make_uint4(__shfl_sync(0xffffffffu, w.x, lane + t.off), __shfl_sync(0xffffffffu, w.y, lane + t.off),
                              __shfl_sync(0xffffffffu, w.z, lane + t.off), __shfl_sync(0xffffffffu, w.w, lane + t.off)), v);
        }
        if (t.on) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(t.b[i], v[i], y[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] *= r;
}

// x / s.  A power of two has an exact reciprocal; the division of any other scale is done as one.
__device__ __forceinline__ void scale_down(float (&x)[8], float s)
{
    if ((__float_as_uint(s) & 0x7fffffu) == 0 && s >= 1.1754944e-38f && s <= 4.2535296e37f) {
        const float f = 1.f / s;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= f;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] / s;
    }
}

__host__ __device__ constexpr int eights(int n) { return (n + 7) & ~7; }

// Biased exponent of the smallest power of two s with amax <= 448 s, at least that of 2^-64 (448 = 1.75 * 2^8).
constexpr int kLeastExp = 127 - 64;
__device__ __forceinline__ int pow2_exp(float amax)
{
    const uint32_t u = __float_as_uint(fminf(amax, 3.3895314e38f));  // (an infinity counts as the largest bf16 number)
    return max((int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), kLeastExp);
}
// Leaves the exponent of the scale that a head's elements, r times y, need (every lane of the head takes part).  The largest of the
// rounded products is the product of the largest; what is no number asks for nothing.
template <int D>
__device__ __forceinline__ void leave_need(uint8_t* dst, const float (&y)[8], float r, int l)
{
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(y[e]));
    const uint32_t lanes = (D == 128 ? 0xffffu : 0xffu) << ((threadIdx.x & 31) / (D / 8) * (D / 8));
#pragma unroll
    for (int o = D / 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(lanes, amax, o));
    if (l == 0) *dst = (uint8_t)pow2_exp(fmaxf(amax * r, 0.f));
}

__device__ __forceinline__ void store_head8(uint8_t* dst, float (&y)[8], const float* scale, int at)
{
    if (scale) scale_down(y, scale[at]);
    *reinterpret_cast<uint2*>(dst) = pack_e4m3(y);
}

// Whether a row is to be written; a position or a slot out of range is reported.
__device__ __forceinline__ bool row_ok(const AppendArgs& a, int i, int slot, int& pos)
{
    const int there = a.cos_sin ? a.positions[i] : 0;
    pos = 0;
    if (slot < 0) return false;  // padding
    bool ok = slot < (int64_t)a.kv.n_pages * a.kv.page_size;
    if (a.cos_sin) {
        pos = there;
        ok = ok && pos >= 0 && pos < a.max_pos;
    }
    if (!ok) {
        set_status(a.status, SPEC_ERR_BAD_INDEX);
        pos = 0;
    }
    return ok;
}

// Batches of heads on their way to the lanes that asked for them: one in registers, or (AHEAD) two in shared memory, the next one under
// the arithmetic of the last, with no register held (in registers: 104 of them, two blocks on an SM, no gain).  A lane reads back what it
// has copied itself.  Three batches take so much of the L1's memory that it is slower (8195 rows into bf16 44.2 -> 49.4 us).
template <bool AHEAD>
struct Stage;
template <>
struct Stage<false> {
    uint4 in[kAhead];
    __device__ __forceinline__ Stage(int, int) {}
    __device__ __forceinline__ void fetch(int, int j, const __nv_bfloat16* src, bool on)
    {
        in[j] = on ? __ldcg(reinterpret_cast<const uint4*>(src)) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void end_batch() {}
    __device__ __forceinline__ void arrived() {}
    __device__ __forceinline__ uint4 get(int, int j, bool) const { return in[j]; }
};
template <>
struct Stage<true> {
    uint4* mine;
    __device__ __forceinline__ Stage(int warp, int lane)
    {
        __shared__ uint4 all[kWarps * 2 * kAhead * 32];
        mine = all + warp * 2 * kAhead * 32 + lane;
    }
    __device__ __forceinline__ void fetch(int t, int j, const __nv_bfloat16* src, bool on)
    {
        if (on)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(mine + ((t & 1) * kAhead + j) * 32)),
                         "l"(src) : "memory");
    }
    __device__ __forceinline__ void end_batch() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    // all batches but the last one asked for are there
    __device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
    __device__ __forceinline__ uint4 get(int t, int j, bool on) const { return on ? mine[((t & 1) * kAhead + j) * 32] : make_uint4(0, 0, 0, 0); }
};

// Q heads of every row, and K and V heads where a row needs nothing of its neighbours.  A warp takes heads [first, first + per)
// of Q, or of K and then V, of one row.
// (80 registers where few warps are there anyway: 1100 rows of the 8B shape into 8 bits 12.6 -> 10.6 us)
template <int D, int CACHE, bool AHEAD>
__global__ void __launch_bounds__(kThreads, AHEAD ? 4 : 3) qkv_append_kernel(const __grid_constant__ AppendArgs a)
{
    stream_wait();
    constexpr int LPH = D / 8, HPI = 32 / LPH;  // lanes of a head, heads of a load instruction
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPH, sub = lane / LPH;
    const unsigned item = blockIdx.x * kWarps + warp, parts = (unsigned)(a.q_parts + a.kv_parts);
    if (item >= (unsigned)a.n_rows * parts) return;
    const int i = (int)(item / parts), part = (int)(item - (unsigned)i * parts), layer = blockIdx.y;
    const int64_t lr = (int64_t)layer * a.n_rows + i;
    const bool is_q = part < a.q_parts;
    const int H = is_q ? a.kv.n_q_heads : a.kv.n_kv_heads;
    const int first = (is_q ? part : part - a.q_parts) * a.heads_per_warp, end = min(H, first + a.heads_per_warp);
    // batches of kAhead * HPI heads: of Q, or of K and then of V (one of each, but for AHEAD)
    const int batches = AHEAD ? (end - first + kAhead * HPI - 1) / (kAhead * HPI) : 1, n_batches = is_q ? batches : 2 * batches;
    Stage<AHEAD> stage(warp, lane);
    const __nv_bfloat16* const src0 = is_q ? a.q + layer * a.q_layer + i * a.q_row : a.k + layer * a.k_layer + i * a.k_row;
    const __nv_bfloat16* const src1 = a.v + layer * a.v_layer + i * a.v_row;
    auto request = [&](int t) {
        const __nv_bfloat16* src = t < batches ? src0 : src1;
        const int h0 = first + (t < batches ? t : t - batches) * kAhead * HPI + sub;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = h0 + j * HPI;
            stage.fetch(t, j, src + h * D + 8 * l, t < n_batches && h < end);
        }
        stage.end_batch();
    };
    request(0);  // (on its way while the row's place and angles are looked up)
    if (AHEAD) request(1);
    const int slot = a.slots[i];
    int pos;
    const bool ok = row_ok(a, i, slot, pos);
    const int64_t need_row = eights(a.kv.n_kv_heads), need_all = (int64_t)a.kv.n_layers * a.n_rows * need_row;
    uint8_t* need = a.need + lr * need_row;
    if (!ok) {
        if (CACHE == kPage8 && !is_q)  // a row that is left out asks its run for nothing
            for (int h = first + lane; h < end; h += 32) need[h] = need[h + need_all] = 0;
        return;
    }
    const int page = slot / a.kv.page_size, in_page = slot - page * a.kv.page_size;
    const int64_t at = layer * a.kv.layer_stride + page * a.kv.page_stride + in_page * a.kv.slot_stride + 8 * l;
    const __nv_bfloat16* weight = is_q ? a.q_weight : a.k_weight;
    const Turn turn = load_turn<D>(a, weight, layer, a.cos_sin + (int64_t)pos * a.rot, l);
    for (int t = 0; t < batches; ++t) {
        const int h0 = first + t * kAhead * HPI;
        stage.arrived();
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (h0 + j * HPI >= end) break;  // the same for the whole warp
            const int h = h0 + j * HPI + sub;
            const uint4 w = stage.get(t, j, h < end);
            float y[8];
            const float rms = head_norm<D>(a, w, weight != nullptr);
            turned(a, turn, w, CACHE == kPage8 && !is_q ? 1.f : rms, y);
            if (h >= end) continue;
            if (is_q) *reinterpret_cast<uint4*>(a.q_out + (lr * a.kv.n_q_heads + h) * D + 8 * l) = pack(y);
            else if (CACHE == kBf16) *reinterpret_cast<uint4*>(a.k16 + at + h * a.kv.head_stride) = pack(y);
            else if (CACHE == kHead8) store_head8(a.k8 + at + h * a.kv.head_stride, y, a.k_scale, layer * a.kv.n_kv_heads + h);
            else leave_need<D>(need + h, y, rms, l);
        }
        if (AHEAD) request(t + 2);
    }
    if (is_q) return;
    need += need_all;
    for (int t = batches; t < n_batches; ++t) {
        const int h0 = first + (t - batches) * kAhead * HPI;
        if (!AHEAD) request(t);
        stage.arrived();
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (h0 + j * HPI >= end) break;
            const int h = h0 + j * HPI + sub;
            const uint4 w = stage.get(t, j, h < end);
            if (h >= end) continue;
            if (CACHE == kBf16) {
                *reinterpret_cast<uint4*>(a.v16 + at + h * a.kv.head_stride) = w;
            } else {
                float y[8];
                unpack(w, y);
                if (CACHE == kHead8) store_head8(a.v8 + at + h * a.kv.head_stride, y, a.v_scale, layer * a.kv.n_kv_heads + h);
                else leave_need<D>(need + h, y, 1.f, l);
            }
        }
        if (AHEAD) request(t + 2);
    }
}

// Rows [0, n) of a page, this lane's eight bytes of each, times f.
__device__ __forceinline__ void rescale(uint8_t* row, int64_t slot_stride, int n, float f)
{
    constexpr int kRows = 8;  // in flight: one warp reads the page of a single token's call (a call whose pages all grow: 12.1 us, four rows 13.9)
    for (int r0 = 0; r0 < n; r0 += kRows) {
        uint2 b[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (r0 + r < n) b[r] = *reinterpret_cast<const uint2*>(row + (r0 + r) * slot_stride);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (r0 + r >= n) break;
            const float2 x0 = e4m3x2_to_float2((uint16_t)b[r].x), x1 = e4m3x2_to_float2((uint16_t)(b[r].x >> 16));
            const float2 x2 = e4m3x2_to_float2((uint16_t)b[r].y), x3 = e4m3x2_to_float2((uint16_t)(b[r].y >> 16));
            const float x[8] = {x0.x * f, x0.y * f, x1.x * f, x1.y * f, x2.x * f, x2.y * f, x3.x * f, x3.y * f};
            *reinterpret_cast<uint2*>(row + (r0 + r) * slot_stride) = pack_e4m3(x);
        }
    }
}

// The second launch for a cache with page scales: a warp takes some heads of K, then of V, of one row.  It finds the extent of the
// row's run from the neighbours' slots and the run's scale from their bytes; the warp of a run's first row stores the scale
// and rescales the slots before it where the scale has grown.  (A scale that is read while that warp stores it is the old or the
// new one: either gives the same larger of itself and the run's.)  What comes before the wait is older than the first
// launch, which lets this one go only when all before it is complete; it is read from L2.
template <int D, bool AHEAD>
__global__ void __launch_bounds__(kThreads, AHEAD ? 4 : 3) append_pages_kernel(const __grid_constant__ AppendArgs a)
{
    constexpr int LPH = D / 8, HPI = 32 / LPH;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPH, sub = lane / LPH;
    const unsigned item = blockIdx.x * kWarps + warp, parts = (unsigned)a.kv_parts;
    const bool some = item < (unsigned)a.n_rows * parts;
    const int i = some ? (int)(item / parts) : 0, part = some ? (int)(item - (unsigned)i * parts) : 0, layer = blockIdx.y;
    const int H = a.kv.n_kv_heads, N = a.n_rows, ps = a.kv.page_size;
    const int head0 = part * a.heads_per_warp, end = min(H, head0 + a.heads_per_warp);
    const int slot = some ? __ldcg(a.slots + i) : -1;
    int pos = a.cos_sin && some ? __ldcg(a.positions + i) : 0;
    const bool in_cache = slot >= 0 && slot < (int64_t)a.kv.n_pages * ps, ok = in_cache && pos >= 0 && (!a.cos_sin || pos < a.max_pos);
    Stage<AHEAD> stage(warp, lane);
    auto request = [&](int x) {  // 0: K's heads, 1: V's
        const __nv_bfloat16* src = x == 0 ? a.k + layer * a.k_layer + i * a.k_row : a.v + layer * a.v_layer + i * a.v_row;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = head0 + j * HPI + sub;
            stage.fetch(x, j, src + h * D + 8 * l, ok && h < end);
        }
        stage.end_batch();
    };
    request(0);
    if (AHEAD) request(1);
    const Turn turn = load_turn<D>(a, a.k_weight, layer, a.cos_sin + (int64_t)(ok ? pos : 0) * a.rot, l);
    const int page = in_cache ? slot / ps : 0, s = in_cache ? slot - page * ps : 0;
    int before = 0, after = 0;  // rows of the run before and behind this one
    if (in_cache) {
        for (const int most = min(s, i); before < most;) {
            const int t = before + 1 + lane;
            const uint32_t stop = ~__ballot_sync(0xffffffffu, t <= most && __ldcg(a.slots + i - t) == slot - t);
            before += stop ? __ffs((int)stop) - 1 : 32;
            if (stop) break;
        }
        for (const int most = min(ps - 1 - s, N - 1 - i); after < most;) {
            const int t = after + 1 + lane;
            const uint32_t stop = ~__ballot_sync(0xffffffffu, t <= most && __ldcg(a.slots + i + t) == slot + t);
            after += stop ? __ffs((int)stop) - 1 : 32;
            if (stop) break;
        }
    }
    stream_wait();
    if (!in_cache) return;
    const int first = s - before;  // the run's first slot in the page
    const int64_t base = layer * a.kv.layer_stride + page * a.kv.page_stride + 8 * l;
    const int64_t scale_at = ((int64_t)layer * a.kv.n_pages + page) * H;

    // the warp's heads are of one group of eight: the largest bytes of the run's rows, K and V, and the scales as they are
    const int64_t need_row = eights(H), need_all = (int64_t)a.kv.n_layers * N * need_row;
    const uint8_t* need = a.need + ((int64_t)layer * N + i - before) * need_row + (head0 & ~7);
    uint2 nk = make_uint2(0, 0), nv = nk;
    for (int r = lane; r <= before + after; r += 32) {
        const uint2 x = __ldcg(reinterpret_cast<const uint2*>(need + r * need_row)), y = __ldcg(reinterpret_cast<const uint2*>(need + r * need_row + need_all));
        nk = make_uint2(__vmaxu4(nk.x, x.x), __vmaxu4(nk.y, x.y));
        nv = make_uint2(__vmaxu4(nv.x, y.x), __vmaxu4(nv.y, y.y));
    }
    float old_k[kAhead], old_v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int h = head0 + j * HPI + sub;
        old_k[j] = old_v[j] = 0.f;
        if (h < end && first > 0) {
            old_k[j] = __ldcg(a.k_scale + scale_at + h);
            old_v[j] = __ldcg(a.v_scale + scale_at + h);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        nk = make_uint2(__vmaxu4(nk.x, __shfl_xor_sync(0xffffffffu, nk.x, o)), __vmaxu4(nk.y, __shfl_xor_sync(0xffffffffu, nk.y, o)));
        nv = make_uint2(__vmaxu4(nv.x, __shfl_xor_sync(0xffffffffu, nv.x, o)), __vmaxu4(nv.y, __shfl_xor_sync(0xffffffffu, nv.y, o)));
    }
    stage.arrived();
    // the run's scale for a head; its first row's warp stores it, and keeps by how much the slots before the run have to shrink
    auto scale_of = [&](const uint2& most, float& was, float* scales, int h) -> float {
        const float old = was > 0.f && was < __builtin_huge_valf() ? was : 0.f;
        const uint32_t e = ((h & 4 ? most.y : most.x) >> (8 * (h & 3))) & 0xffu;
        const float now = fmaxf(old, __uint_as_float(max(e, (uint32_t)kLeastExp) << 23));
        const bool mine = before == 0 && h < end && (e != 0 || first > 0);  // (0: all rows are left out, and the page does not start anew)
        if (mine && l == 0) scales[scale_at + h] = now;
        was = mine && now > old && first > 0 ? old / now : 1.f;
        return now;
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        if (head0 + j * HPI >= end) break;  // the same for the whole warp
        const int h = head0 + j * HPI + sub;
        const float now = scale_of(nk, old_k[j], a.k_scale, h);
        const uint4 w = stage.get(0, j, ok && h < end);
        float y[8];
        turned(a, turn, w, head_norm<D>(a, w, a.k_weight != nullptr), y);
        scale_down(y, now);
        if (ok && h < end) *reinterpret_cast<uint2*>(a.k8 + base + s * a.kv.slot_stride + h * a.kv.head_stride) = pack_e4m3(y);
    }
    if (AHEAD) stage.end_batch();
    else request(1);
    stage.arrived();
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        if (head0 + j * HPI >= end) break;
        const int h = head0 + j * HPI + sub;
        const float now = scale_of(nv, old_v[j], a.v_scale, h);
        float y[8];
        unpack(stage.get(1, j, ok && h < end), y);
        scale_down(y, now);
        if (ok && h < end) *reinterpret_cast<uint2*>(a.v8 + base + s * a.kv.slot_stride + h * a.kv.head_stride) = pack_e4m3(y);
    }
    if (before > 0 || first == 0) return;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int h = head0 + j * HPI + sub;
        if (h >= end) break;
        if (old_k[j] != 1.f) rescale(a.k8 + base + h * a.kv.head_stride, a.kv.slot_stride, first, old_k[j]);
        if (old_v[j] != 1.f) rescale(a.v8 + base + h * a.kv.head_stride, a.kv.slot_stride, first, old_v[j]);
    }
}

template <int D, int CACHE>
int launch(AppendArgs a, cudaStream_t stream)
{
    constexpr int HPI = 32 / (D / 8);
    const int Hq = a.q ? a.kv.n_q_heads : 0, Hk = a.kv.n_kv_heads;
    const int64_t rows = (int64_t)a.kv.n_layers * a.n_rows;
    // few rows: a warp per load instruction, so that the call is one trip to memory; more than two waves of warps with a batch each:
    // all heads of Q, or of K and V, whose angles and weights are fetched once, and each batch under the arithmetic of the one before
    // (8B shape into bf16, a batch each and whole rows: 1300 rows 10.2 and 12.5 us, 1700 15.0 and 14.0, 6000 42.8 and 35.2)
    a.heads_per_warp = kAhead * HPI;
    const int64_t batches = rows * ((Hq + kAhead * HPI - 1) / (kAhead * HPI) + (Hk + kAhead * HPI - 1) / (kAhead * HPI));
    if (rows * (Hq + 2 * Hk) <= 8L * sm_count() * kWarps * HPI) a.heads_per_warp = HPI;
    else if (batches > 2 * 3L * sm_count() * kWarps) a.heads_per_warp = 1 << 20;
    a.q_parts = (Hq + a.heads_per_warp - 1) / a.heads_per_warp;
    a.kv_parts = (Hk + a.heads_per_warp - 1) / a.heads_per_warp;
    // (page scales: the second launch has two to eight heads a warp, of one group of eight, and a lane's all in flight)
    const int page_heads = a.heads_per_warp > 8 ? 8 : a.heads_per_warp, page_parts = (Hk + page_heads - 1) / page_heads;
    if (a.kv.n_layers > 65535 || (int64_t)a.n_rows * (a.q_parts + a.kv_parts) > INT32_MAX ||
        (CACHE == kPage8 && (int64_t)a.n_rows * page_parts > INT32_MAX))
        return SPEC_ERR_UNSUPPORTED_SHAPE;
    const unsigned all = (unsigned)(((int64_t)a.n_rows * (a.q_parts + a.kv_parts) + kWarps - 1) / kWarps);
    const int rc = launch_chained(a.heads_per_warp > kAhead * HPI ? qkv_append_kernel<D, CACHE, true> : qkv_append_kernel<D, CACHE, false>,
                                  dim3(all, (unsigned)a.kv.n_layers), dim3(kThreads), 0, 1, stream, a);
    if (rc != SPEC_OK || CACHE != kPage8) return rc;
    a.heads_per_warp = page_heads;
    a.kv_parts = page_parts;
    const unsigned again = (unsigned)(((int64_t)a.n_rows * a.kv_parts + kWarps - 1) / kWarps);
    // more than a wave of warps: V on its way with K, through shared memory (which fewer rows would pay for with
    // the carve-out's change behind another kernel: 72 rows 5.9 -> 8.3 us)
    return launch_chained(rows * a.kv_parts > 4L * sm_count() * kWarps ? append_pages_kernel<D, true> : append_pages_kernel<D, false>,
                          dim3(again, (unsigned)a.kv.n_layers), dim3(kThreads), 0, 1, stream, a);
}

template <int D>
int launch_cache(const AppendArgs& a, cudaStream_t stream)
{
    if (!a.kv.fp8) return launch<D, kBf16>(a, stream);
    return a.kv.page_scale ? launch<D, kPage8>(a, stream) : launch<D, kHead8>(a, stream);
}

}  // namespace

// The status word; with page scales a byte for every row and head of K and V behind it.
size_t append_workspace(const KvView& kv, int64_t n_rows)
{
    return kStatusBytes + (kv.page_scale ? (size_t)(2 * kv.n_layers * n_rows * eights(kv.n_kv_heads)) : 0);
}

int qkv_append_launch(const QkvRows& r, const KvView& kv, int32_t n_rows, const int32_t* positions, const int32_t* slots,
                      const void* q_weight, const void* k_weight, float eps, const float* cos_sin, int max_pos, int rot,
                      int interleaved, void* q_out, void* workspace, cudaStream_t stream)
{
    AppendArgs a = {};
    a.kv = kv;
    a.k16 = const_cast<__nv_bfloat16*>(kv.k);
    a.v16 = const_cast<__nv_bfloat16*>(kv.v);
    a.k8 = const_cast<uint8_t*>(kv.k8);
    a.v8 = const_cast<uint8_t*>(kv.v8);
    a.k_scale = const_cast<float*>(kv.k_scale);
    a.v_scale = const_cast<float*>(kv.v_scale);
    a.q = static_cast<const __nv_bfloat16*>(r.q), a.q_layer = r.q_layer, a.q_row = r.q_row;
    a.k = static_cast<const __nv_bfloat16*>(r.k), a.k_layer = r.k_layer, a.k_row = r.k_row;
    a.v = static_cast<const __nv_bfloat16*>(r.v), a.v_layer = r.v_layer, a.v_row = r.v_row;
    a.n_rows = n_rows;
    a.positions = positions;
    a.slots = slots;
    a.q_weight = static_cast<const __nv_bfloat16*>(q_weight);
    a.k_weight = static_cast<const __nv_bfloat16*>(k_weight);
    a.eps = eps;
    a.cos_sin = cos_sin;
    a.max_pos = max_pos;
    a.rot = rot;
    a.interleaved = interleaved;
    a.q_out = static_cast<__nv_bfloat16*>(q_out);
    a.status = static_cast<int*>(workspace);
    a.need = static_cast<uint8_t*>(workspace) + kStatusBytes;
    return kv.head_dim == 128 ? launch_cache<128>(a, stream) : launch_cache<64>(a, stream);
}

}  // namespace spec
