// From a projection's output to the cache in one launch: RMS norm of every head of Q and K, rotation by the row's position,
// Q rounded to bf16 for the attention calls, K and V written to their slots in the form the cache has.
//
//   y = x / sqrt(mean(x^2) + eps) * w;  (y_i, y_j) <- (y_i cos - y_j sin, y_j cos + y_i sin)  for the pairs of the position
//
// Bound by memory: every element is read and written once.  A head of a row is D / 8 neighbouring lanes with 16 bytes
// each, so the norm is a few shuffles, and a pair (i, i + rot / 2) is one more; everything between the load and
// the one rounding at the end is fp32 in registers.
//
// A cache with a scale for each page (SPEC_KV_FP8_E4M3_PAGE) is written a page at a time: the rows that a call brings for
// one page are a run of neighbours, whose largest value decides the page's scale before any of them is stored.  Scales
// are powers of two: a floating-point byte loses nothing by that but a binade of range, and the rows already in the page
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
    int window;                         // page part: rows in which a block looks for the beginnings of runs, at most 32
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
__device__ __forceinline__ Turn load_turn(const AppendArgs& p, const __nv_bfloat16* weight, int layer, int pos, int l)
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
    const float* row = p.cos_sin + (int64_t)pos * p.rot;
    if (p.interleaved) {
        if (t.on) {
            const float4 c = *reinterpret_cast<const float4*>(row + e0 / 2), s = *reinterpret_cast<const float4*>(row + half + e0 / 2);
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
        const float4 c0 = c[0], c1 = c[1], s0 = n[0], s1 = n[1];
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

// Q heads of every row, and K and V heads where a row needs nothing of its neighbours.  A warp takes heads [first, first + per)
// of Q, or of K and then V, of one row.
template <int D, int CACHE>
__device__ __forceinline__ void row_part(const AppendArgs& a, int block)
{
    constexpr int LPH = D / 8, HPI = 32 / LPH;  // lanes of a head, heads of a load instruction
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPH, sub = lane / LPH;
    const int64_t item = (int64_t)block * (blockDim.x / 32) + warp;
    const int64_t rows = (int64_t)a.kv.n_layers * a.n_rows;
    const int parts = a.q_parts + a.kv_parts;
    if (item >= rows * parts) return;
    const int64_t lr = item / parts;
    const int part = (int)(item - lr * parts), layer = (int)(lr / a.n_rows), i = (int)(lr - (int64_t)layer * a.n_rows);
    const bool is_q = part < a.q_parts;
    const int H = is_q ? a.kv.n_q_heads : a.kv.n_kv_heads;
    const int first = (is_q ? part : part - a.q_parts) * a.heads_per_warp, end = min(H, first + a.heads_per_warp);
    uint4 in[kAhead];
    auto request = [&](const __nv_bfloat16* src, int h0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = h0 + j * HPI + sub;
            in[j] = h < end ? *reinterpret_cast<const uint4*>(src + h * D + 8 * l) : make_uint4(0, 0, 0, 0);
        }
    };
    const __nv_bfloat16* src = is_q ? a.q + layer * a.q_layer + i * a.q_row : a.k + layer * a.k_layer + i * a.k_row;
    request(src, first);  // (on its way while the row's place and angles are looked up)
    const int slot = a.slots[i];
    int pos;
    if (!row_ok(a, i, slot, pos)) return;
    const int page = slot / a.kv.page_size, in_page = slot - page * a.kv.page_size;
    const int64_t at = layer * a.kv.layer_stride + page * a.kv.page_stride + in_page * a.kv.slot_stride + 8 * l;
    const __nv_bfloat16* weight = is_q ? a.q_weight : a.k_weight;
    const Turn turn = load_turn<D>(a, weight, layer, pos, l);
    for (int h0 = first; h0 < end; h0 += kAhead * HPI) {
        if (h0 != first) request(src, h0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (h0 + j * HPI >= end) break;  // the same for the whole warp
            const int h = h0 + j * HPI + sub;
            float y[8];
            turned(a, turn, in[j], head_norm<D>(a, in[j], weight != nullptr), y);
            if (h >= end) continue;
            if (is_q) *reinterpret_cast<uint4*>(a.q_out + (lr * a.kv.n_q_heads + h) * D + 8 * l) = pack(y);
            else if (CACHE == kBf16) *reinterpret_cast<uint4*>(a.k16 + at + h * a.kv.head_stride) = pack(y);
            else if (CACHE == kHead8) store_head8(a.k8 + at + h * a.kv.head_stride, y, a.k_scale, layer * a.kv.n_kv_heads + h);
        }
    }
    if (is_q || CACHE == kPage8) return;
    src = a.v + layer * a.v_layer + i * a.v_row;
    for (int h0 = first; h0 < end; h0 += kAhead * HPI) {
        request(src, h0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = h0 + j * HPI + sub;
            if (h >= end) continue;
            if (CACHE == kBf16) {
                *reinterpret_cast<uint4*>(a.v16 + at + h * a.kv.head_stride) = in[j];
            } else {
                float y[8];
                unpack(in[j], y);
                store_head8(a.v8 + at + h * a.kv.head_stride, y, a.v_scale, layer * a.kv.n_kv_heads + h);
            }
        }
    }
}

// The smallest power of two s with amax <= 448 s, at least 2^-64 (448 = 1.75 * 2^8).
__device__ __forceinline__ float pow2_scale(float amax)
{
    const uint32_t u = __float_as_uint(fminf(amax, 3.3895314e38f));  // (an infinity counts as the largest bf16 number)
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);  // biased exponent of the scale
    return __uint_as_float((uint32_t)max(e, 127 - 64) << 23);
}

// K or V rows of a head, page by page: a block looks for the beginnings of runs in a window of rows.
template <int D>
__device__ __forceinline__ void page_part(const AppendArgs& a, int block)
{
    constexpr int LPH = D / 8, RPI = 32 / LPH;  // lanes of a row, rows of a warp's load
    constexpr int kHeld = 2;                    // rows of a lane that stay in registers between the largest value and the store
    __shared__ float amax_s[2][kThreads / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n_warps = blockDim.x / 32, step = n_warps * RPI;
    const int l = lane % LPH, sub = lane / LPH;
    const int N = a.n_rows, ps = a.kv.page_size, H = a.kv.n_kv_heads;
    const int windows = (N + a.window - 1) / a.window;
    const bool is_k = block % 2 == 0;
    const int win = block / 2 % windows, h = (block / 2 / windows) % H, layer = block / 2 / (windows * H);
    const __nv_bfloat16* src = is_k ? a.k + layer * a.k_layer + h * D + 8 * l : a.v + layer * a.v_layer + h * D + 8 * l;
    const int64_t src_row = is_k ? a.k_row : a.v_row;
    uint8_t* dst = (is_k ? a.k8 : a.v8) + layer * a.kv.layer_stride + h * a.kv.head_stride + 8 * l;
    float* scales = (is_k ? a.k_scale : a.v_scale) + (int64_t)layer * a.kv.n_pages * H + h;
    const bool norm = is_k && a.k_weight;
    int buf = 0;

    // the beginnings of runs among the window's rows, a row per lane (every warp for itself)
    const int mine = win * a.window + lane;
    int slot_l = -1;
    bool begins = false;
    if (lane < a.window && mine < N) {
        slot_l = a.slots[mine];
        begins = slot_l >= 0 && slot_l < (int64_t)a.kv.n_pages * ps;
        if (slot_l >= 0 && !begins && warp == 0) set_status(a.status, SPEC_ERR_BAD_INDEX);
        if (begins && mine > 0 && slot_l % ps != 0 && a.slots[mine - 1] == slot_l - 1) begins = false;
    }
    for (uint32_t left = __ballot_sync(0xffffffffu, begins); left; left &= left - 1) {
        const int which = __ffs((int)left) - 1, i = win * a.window + which, slot = __shfl_sync(0xffffffffu, slot_l, which);
        const int page = slot / ps, first = slot - page * ps;
        int n = 1;  // rows of the run
        const int most = min(N - i, ps - first);
        while (n < most) {
            const bool next = n + lane < most && a.slots[i + n + lane] == slot + n + lane;
            const uint32_t end = ~__ballot_sync(0xffffffffu, next);
            n += end ? __ffs((int)end) - 1 : 32;
            if (end) break;
        }
        // one row's bits, and whether it is written (zeros where not)
        auto fetch = [&](int r, int& pos, uint4& in) -> bool {
            pos = 0;
            in = make_uint4(0, 0, 0, 0);
            const bool ok = r < n && row_ok(a, i + r, slot + r, pos);
            if (ok) in = *reinterpret_cast<const uint4*>(src + (i + r) * src_row);
            return ok;
        };
        auto finish = [&](int pos, const uint4& in, float (&y)[8]) {
            if (is_k) {  // (the same for the whole block)
                const Turn t = load_turn<D>(a, a.k_weight, layer, pos, l);
                turned(a, t, in, head_norm<D>(a, in, norm), y);
            } else {
                unpack(in, y);
            }
        };
        const float was = scales[(int64_t)page * H];
        const float old = first > 0 && was > 0.f && was < __builtin_huge_valf() ? was : 0.f;
        const bool held = n <= kHeld * step;
        float y[kHeld][8], amax = 0.f;
        bool ok[kHeld];
        // rows r0 + j * step of this lane: their bits all requested, then finished one after the other
        auto batch = [&](int r0) {
            uint4 in[kHeld];
            int pos[kHeld];
#pragma unroll
            for (int j = 0; j < kHeld; ++j) ok[j] = fetch(r0 + j * step + warp * RPI + sub, pos[j], in[j]);
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                if (r0 + j * step < n) finish(pos[j], in[j], y[j]);  // (the same for the whole block)
        };
        for (int r0 = 0; r0 < n; r0 += kHeld * step) {
            batch(r0);
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                if (r0 + j * step < n)
#pragma unroll
                    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(y[j][e]));
        }
        amax = warp_max(amax);
        if (lane == 0) amax_s[buf][warp] = amax;
        __syncthreads();
        for (int j = 0; j < n_warps; ++j) amax = fmaxf(amax, amax_s[buf][j]);
        buf ^= 1;  // (the next run's values; the barrier after them is behind everybody's reads of these)
        const float now = fmaxf(old, pow2_scale(amax));
        if (tid == 0) scales[(int64_t)page * H] = now;
        uint8_t* rows = dst + page * a.kv.page_stride;
        if (now > old) {
            const float f = old / now;
            for (int r = warp * RPI + sub; r < first; r += step) {
                uint8_t* p = rows + r * a.kv.slot_stride;
                const uint2 b = *reinterpret_cast<const uint2*>(p);
                const float2 x0 = e4m3x2_to_float2((uint16_t)b.x), x1 = e4m3x2_to_float2((uint16_t)(b.x >> 16));
                const float2 x2 = e4m3x2_to_float2((uint16_t)b.y), x3 = e4m3x2_to_float2((uint16_t)(b.y >> 16));
                const float x[8] = {x0.x * f, x0.y * f, x1.x * f, x1.y * f, x2.x * f, x2.y * f, x3.x * f, x3.y * f};
                *reinterpret_cast<uint2*>(p) = pack_e4m3(x);
            }
        }
        for (int r0 = 0; r0 < n; r0 += kHeld * step) {
            if (!held) batch(r0);
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                if (!ok[j]) continue;
                scale_down(y[j], now);
                *reinterpret_cast<uint2*>(rows + (first + r0 + j * step + warp * RPI + sub) * a.kv.slot_stride) = pack_e4m3(y[j]);
            }
        }
    }
}

template <int D, int CACHE>
__global__ void __launch_bounds__(kThreads, 4) qkv_append_kernel(const __grid_constant__ AppendArgs a)
{
    stream_wait();
    if ((int)blockIdx.x < a.row_blocks) row_part<D, CACHE>(a, blockIdx.x);
    else if (CACHE == kPage8) page_part<D>(a, blockIdx.x - a.row_blocks);
}

template <int D, int CACHE>
int launch(AppendArgs a, cudaStream_t stream)
{
    constexpr int HPI = 32 / (D / 8);
    const int Hq = a.q ? a.kv.n_q_heads : 0, Hk = CACHE == kPage8 ? 0 : a.kv.n_kv_heads;
    const int64_t rows = (int64_t)a.kv.n_layers * a.n_rows;
    int threads = kThreads;
    int64_t row_blocks = 0, page_blocks = 0;
    // few rows: a warp per load instruction, so that the call is one trip to memory; many: all heads of Q, or of K and V, whose
    // angles and weights are fetched once
    a.heads_per_warp = kAhead * HPI;
    if (rows * (Hq + 2 * Hk) <= 8L * sm_count() * kWarps * HPI) a.heads_per_warp = HPI;
    else if (rows >= 8L * sm_count() * kWarps) a.heads_per_warp = 1 << 20;
    a.q_parts = (Hq + a.heads_per_warp - 1) / a.heads_per_warp;
    a.kv_parts = (Hk + a.heads_per_warp - 1) / a.heads_per_warp;
    if (CACHE == kPage8) {
        // Warps of a run: as many as give the SMs sixteen each, and have rows.  Blocks that find no run's beginning cost
        // their launch, so a block looks through more rows the more there are.
        const int64_t problems = 2ll * a.kv.n_layers * a.kv.n_kv_heads, len = a.n_rows < a.kv.page_size ? a.n_rows : a.kv.page_size;
        const int64_t runs = problems * ((a.n_rows + a.kv.page_size - 1) / a.kv.page_size);
        threads = 32;
        while (threads < kThreads && runs * threads < 16ll * 32 * sm_count() && len * D / 8 > threads) threads *= 2;
        int64_t w = (problems * a.n_rows + 8191) / 8192;
        a.window = (int)(w < 1 ? 1 : (w > 32 ? 32 : w));
        page_blocks = problems * ((a.n_rows + a.window - 1) / a.window);
    }
    row_blocks = (rows * (a.q_parts + a.kv_parts) * 32 + threads - 1) / threads;
    if (row_blocks + page_blocks > 0x7fffffff) return SPEC_ERR_UNSUPPORTED_SHAPE;
    if (row_blocks + page_blocks == 0) return SPEC_OK;
    a.row_blocks = (int)row_blocks;
    return launch_chained(qkv_append_kernel<D, CACHE>, dim3((unsigned)(row_blocks + page_blocks)), dim3(threads), 0, 1, stream, a);
}

template <int D>
int launch_cache(const AppendArgs& a, cudaStream_t stream)
{
    if (!a.kv.fp8) return launch<D, kBf16>(a, stream);
    return a.kv.page_scale ? launch<D, kPage8>(a, stream) : launch<D, kHead8>(a, stream);
}

}  // namespace

size_t append_workspace() { return kStatusBytes; }

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
    return kv.head_dim == 128 ? launch_cache<128>(a, stream) : launch_cache<64>(a, stream);
}

}  // namespace spec
