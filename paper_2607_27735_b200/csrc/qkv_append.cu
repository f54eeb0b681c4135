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
    int heads_per_warp, row_blocks;  // row part: heads of a row that a warp takes; blocks of that part
    int window;                      // page part: rows in which a block looks for the beginnings of runs
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

// What a lane needs to turn its eight elements of a head at one position.
struct Turn {
    float c[8], s[8];  // interleaved: the first four of each
    int off;           // lanes to the partner (0: not turned)
    bool second;       // this lane has the second elements of its pairs
};
template <int D>
__device__ __forceinline__ Turn load_turn(const AppendArgs& a, int pos, int l)
{
    Turn t;
    const int e0 = 8 * l, half = a.rot / 2;
    t.off = 0;
    t.second = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) t.c[i] = 1.f, t.s[i] = 0.f;
    if (!a.cos_sin || e0 >= a.rot) return t;
    const float* row = a.cos_sin + (int64_t)pos * a.rot;
    if (a.interleaved) {
        const float4 c = *reinterpret_cast<const float4*>(row + e0 / 2), s = *reinterpret_cast<const float4*>(row + half + e0 / 2);
        t.c[0] = c.x, t.c[1] = c.y, t.c[2] = c.z, t.c[3] = c.w;
        t.s[0] = s.x, t.s[1] = s.y, t.s[2] = s.z, t.s[3] = s.w;
        return t;
    }
    t.second = e0 >= half;
    t.off = t.second ? -half / 8 : half / 8;
    const float4* p = reinterpret_cast<const float4*>(row + (t.second ? e0 - half : e0));
    const float4* n = reinterpret_cast<const float4*>(row + half + (t.second ? e0 - half : e0));
    const float4 c0 = p[0], c1 = p[1], s0 = n[0], s1 = n[1];
    t.c[0] = c0.x, t.c[1] = c0.y, t.c[2] = c0.z, t.c[3] = c0.w, t.c[4] = c1.x, t.c[5] = c1.y, t.c[6] = c1.z, t.c[7] = c1.w;
    t.s[0] = s0.x, t.s[1] = s0.y, t.s[2] = s0.z, t.s[3] = s0.w, t.s[4] = s1.x, t.s[5] = s1.y, t.s[6] = s1.z, t.s[7] = s1.w;
    return t;
}

// Norm (w: this lane's eight weights, null without one) and rotation of a head; every lane of the warp takes part.
template <int D>
__device__ __forceinline__ void norm_turn(const AppendArgs& a, float (&x)[8], const uint4* w, bool norm, const Turn& t, bool turn)
{
    constexpr int LPH = D / 8;
    const int lane = threadIdx.x & 31;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (norm) {
        float g[8];
        unpack(*w, g);
        const float r = rsqrtf(ss * (1.f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * g[i];
    }
    if (a.cos_sin == nullptr) return;
    if (a.interleaved) {
        if (turn) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float u = x[2 * i], v = x[2 * i + 1];
                x[2 * i] = u * t.c[i] - v * t.s[i];
                x[2 * i + 1] = v * t.c[i] + u * t.s[i];
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = __shfl_sync(0xffffffffu, x[i], lane + t.off);
        if (turn && t.off) x[i] = t.second ? x[i] * t.c[i] + y * t.s[i] : x[i] * t.c[i] - y * t.s[i];
    }
}

// Whether a row is to be written; a position or a slot out of range is reported.
__device__ __forceinline__ bool row_ok(const AppendArgs& a, int i, int slot, int& pos)
{
    pos = 0;
    if (slot < 0) return false;  // padding
    bool ok = slot < (int64_t)a.kv.n_pages * a.kv.page_size;
    if (a.cos_sin) {
        pos = a.positions[i];
        ok = ok && pos >= 0 && pos < a.max_pos;
    }
    if (!ok) {
        set_status(a.status, SPEC_ERR_BAD_INDEX);
        pos = 0;
    }
    return ok;
}

// Q heads of every row, and K and V heads where a row needs nothing of its neighbours.
template <int D, int CACHE>
__device__ __forceinline__ void row_part(const AppendArgs& a, int block)
{
    constexpr int LPH = D / 8, HPI = 32 / LPH;  // lanes of a head, heads of a load instruction
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPH, sub = lane / LPH;
    const int Hq = a.q ? a.kv.n_q_heads : 0, Hk = CACHE == kPage8 ? 0 : a.kv.n_kv_heads, H = Hq + 2 * Hk;
    const int parts = (H + a.heads_per_warp - 1) / a.heads_per_warp;
    const int64_t item = (int64_t)block * kWarps + warp;
    const int64_t rows = (int64_t)a.kv.n_layers * a.n_rows;
    if (item >= rows * parts) return;
    const int64_t lr = item / parts;
    const int part = (int)(item - lr * parts), layer = (int)(lr / a.n_rows), i = (int)(lr - (int64_t)layer * a.n_rows);
    const int slot = a.slots[i];
    int pos;
    if (!row_ok(a, i, slot, pos)) return;
    const Turn turn = load_turn<D>(a, pos, l);
    const bool turns = a.cos_sin != nullptr && 8 * l < a.rot;
    uint4 wq = make_uint4(0, 0, 0, 0), wk = wq;
    if (a.q_weight && Hq) wq = *reinterpret_cast<const uint4*>(a.q_weight + (int64_t)layer * D + 8 * l);
    if (a.k_weight && Hk) wk = *reinterpret_cast<const uint4*>(a.k_weight + (int64_t)layer * D + 8 * l);
    const int page = slot / a.kv.page_size, in_page = slot - page * a.kv.page_size;
    const int64_t at = layer * a.kv.layer_stride + page * a.kv.page_stride + in_page * a.kv.slot_stride + 8 * l;
    const __nv_bfloat16* q = a.q + layer * a.q_layer + i * a.q_row + 8 * l;
    const __nv_bfloat16* k = a.k + layer * a.k_layer + i * a.k_row + 8 * l;
    const __nv_bfloat16* v = a.v + layer * a.v_layer + i * a.v_row + 8 * l;
    __nv_bfloat16* out = a.q_out + ((int64_t)layer * a.n_rows + i) * a.kv.n_q_heads * D + 8 * l;
    const int h1 = min(H, (part + 1) * a.heads_per_warp);
    for (int h0 = part * a.heads_per_warp; h0 < h1; h0 += kAhead * HPI) {
        uint4 in[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = h0 + j * HPI + sub;
            in[j] = make_uint4(0, 0, 0, 0);
            if (h < h1)
                in[j] = *reinterpret_cast<const uint4*>(h < Hq ? q + h * D : (h < Hq + Hk ? k + (h - Hq) * D : v + (h - Hq - Hk) * D));
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (h0 + j * HPI >= h1) break;  // the same for the whole warp
            const int h = h0 + j * HPI + sub;
            const bool is_q = h < Hq, is_k = !is_q && h < Hq + Hk;
            float x[8];
            unpack(in[j], x);
            const uint4 w = is_q ? wq : wk;
            norm_turn<D>(a, x, &w, is_q ? a.q_weight != nullptr : is_k && a.k_weight != nullptr, turn, turns && (is_q || is_k));
            if (h >= h1) continue;
            if (is_q) {
                *reinterpret_cast<uint4*>(out + h * D) = pack(x);
            } else if (CACHE == kBf16) {
                const int g = h - Hq - (is_k ? 0 : Hk);
                *reinterpret_cast<uint4*>((is_k ? a.k16 : a.v16) + at + g * a.kv.head_stride) = pack(x);
            } else if (CACHE == kHead8) {
                const int g = h - Hq - (is_k ? 0 : Hk);
                const float* sc = is_k ? a.k_scale : a.v_scale;
                if (sc) {
                    const float s = sc[(int64_t)layer * a.kv.n_kv_heads + g];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] / s;
                }
                *reinterpret_cast<uint2*>((is_k ? a.k8 : a.v8) + at + g * a.kv.head_stride) = pack_e4m3(x);
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

// K (first half of the block) and V (second half) rows of a page and head, run by run.
template <int D>
__device__ __forceinline__ void page_part(const AppendArgs& a, int block)
{
    constexpr int LPH = D / 8, RPI = 32 / LPH;  // lanes of a row, rows of a warp's load
    constexpr int kTeam = kThreads / 2, kStep = kTeam / 32 * RPI;  // threads of a team, rows that it takes at a time
    __shared__ float amax_s[2][2][kTeam / 32];  // [buffer][team][warp]
    const int team = threadIdx.x / kTeam, tid = threadIdx.x % kTeam, warp = tid >> 5, lane = tid & 31;
    const int l = lane % LPH, sub = lane / LPH;
    const int N = a.n_rows, ps = a.kv.page_size, H = a.kv.n_kv_heads;
    const int windows = (N + a.window - 1) / a.window;
    const int win = block % windows, h = (block / windows) % H, layer = block / (windows * H);
    const bool is_k = team == 0;
    const __nv_bfloat16* src = is_k ? a.k + layer * a.k_layer + h * D + 8 * l : a.v + layer * a.v_layer + h * D + 8 * l;
    const int64_t src_row = is_k ? a.k_row : a.v_row;
    uint8_t* dst = (is_k ? a.k8 : a.v8) + layer * a.kv.layer_stride + h * a.kv.head_stride + 8 * l;
    float* scales = (is_k ? a.k_scale : a.v_scale) + (int64_t)layer * a.kv.n_pages * H + h;
    const bool norm = is_k && a.k_weight, turns = is_k && a.cos_sin != nullptr && 8 * l < a.rot;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (norm) w = *reinterpret_cast<const uint4*>(a.k_weight + (int64_t)layer * D + 8 * l);
    int buf = 0;

    for (int i = win * a.window; i < min(N, (win + 1) * a.window); ++i) {
        const int slot = a.slots[i];
        if (slot < 0) continue;
        if (slot >= (int64_t)a.kv.n_pages * ps) {
            if (threadIdx.x == 0) set_status(a.status, SPEC_ERR_BAD_INDEX);
            continue;
        }
        const int page = slot / ps, first = slot - page * ps;
        if (i > 0 && first > 0 && a.slots[i - 1] == slot - 1) continue;  // inside a run
        int n = 1;  // rows of the run
        const int most = min(N - i, ps - first);
        while (n < most) {
            const bool next = n + lane < most && a.slots[i + n + lane] == slot + n + lane;
            const uint32_t end = ~__ballot_sync(0xffffffffu, next);
            n += end ? __ffs((int)end) - 1 : 32;
            if (end) break;
        }
        // one row's eight elements of this lane; zeros where the row is not written
        auto row = [&](int r, float (&x)[8]) -> bool {
            int pos = 0;
            bool ok = r < n;
            uint4 in = make_uint4(0, 0, 0, 0);
            if (ok) ok = row_ok(a, i + r, slot + r, pos);
            if (ok) in = *reinterpret_cast<const uint4*>(src + (i + r) * src_row);
            unpack(in, x);
            if (is_k) {  // (the same for the whole warp)
                const Turn t = load_turn<D>(a, pos, l);
                norm_turn<D>(a, x, &w, norm, t, turns);
            }
            return ok;
        };
        float amax = 0.f;
        for (int r0 = 0; r0 < n; r0 += kStep) {
            float x[8];
            row(r0 + warp * RPI + sub, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
        }
        amax = warp_max(amax);
        const float was = scales[(int64_t)page * H];
        const float old = first > 0 && was > 0.f && was < __builtin_huge_valf() ? was : 0.f;
        if (lane == 0) amax_s[buf][team][warp] = amax;
        if (is_k) asm volatile("bar.sync 1, %0;" ::"n"(kTeam) : "memory");
        else asm volatile("bar.sync 2, %0;" ::"n"(kTeam) : "memory");
#pragma unroll
        for (int j = 0; j < kTeam / 32; ++j) amax = fmaxf(amax, amax_s[buf][team][j]);
        buf ^= 1;
        const float now = fmaxf(old, pow2_scale(amax));
        if (tid == 0) scales[(int64_t)page * H] = now;
        uint8_t* rows = dst + page * a.kv.page_stride;
        if (now > old) {
            const float f = old / now;
            for (int r = warp * RPI + sub; r < first; r += kStep) {
                uint8_t* p = rows + r * a.kv.slot_stride;
                const uint2 b = *reinterpret_cast<const uint2*>(p);
                const float2 x0 = e4m3x2_to_float2((uint16_t)b.x), x1 = e4m3x2_to_float2((uint16_t)(b.x >> 16));
                const float2 x2 = e4m3x2_to_float2((uint16_t)b.y), x3 = e4m3x2_to_float2((uint16_t)(b.y >> 16));
                const float x[8] = {x0.x * f, x0.y * f, x1.x * f, x1.y * f, x2.x * f, x2.y * f, x3.x * f, x3.y * f};
                *reinterpret_cast<uint2*>(p) = pack_e4m3(x);
            }
        }
        for (int r0 = 0; r0 < n; r0 += kStep) {
            const int r = r0 + warp * RPI + sub;
            float x[8];
            const bool ok = row(r, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] / now;
            if (ok) *reinterpret_cast<uint2*>(rows + (first + r) * a.kv.slot_stride) = pack_e4m3(x);
        }
    }
}

template <int D, int CACHE>
__global__ void __launch_bounds__(kThreads) qkv_append_kernel(const __grid_constant__ AppendArgs a)
{
    stream_wait();
    if ((int)blockIdx.x < a.row_blocks) row_part<D, CACHE>(a, blockIdx.x);
    else if (CACHE == kPage8) page_part<D>(a, blockIdx.x - a.row_blocks);
}

template <int D, int CACHE>
int launch(AppendArgs a, cudaStream_t stream)
{
    constexpr int HPI = 32 / (D / 8);
    const int H = (a.q ? a.kv.n_q_heads : 0) + (CACHE == kPage8 ? 0 : 2 * a.kv.n_kv_heads);
    const int64_t rows = (int64_t)a.kv.n_layers * a.n_rows;
    int64_t row_blocks = 0, page_blocks = 0;
    a.heads_per_warp = kAhead * HPI;
    if (H) {
        // few rows: a warp per load instruction, so that the call is one trip to memory; many: whole rows, whose angles
        // are fetched once
        if (rows * H <= 8L * sm_count() * kWarps * HPI) a.heads_per_warp = HPI;
        else if (rows >= 8L * sm_count() * kWarps) a.heads_per_warp = (H + kAhead * HPI - 1) / (kAhead * HPI) * (kAhead * HPI);
        const int parts = (H + a.heads_per_warp - 1) / a.heads_per_warp;
        row_blocks = (rows * parts + kWarps - 1) / kWarps;
    }
    if (CACHE == kPage8) {
        const int64_t problems = (int64_t)a.kv.n_layers * a.kv.n_kv_heads;
        int64_t w = (problems * a.n_rows + 4095) / 4096;
        a.window = (int)(w < 1 ? 1 : (w > 32 ? 32 : w));
        page_blocks = problems * ((a.n_rows + a.window - 1) / a.window);
    }
    if (row_blocks + page_blocks > 0x7fffffff) return SPEC_ERR_UNSUPPORTED_SHAPE;
    a.row_blocks = (int)row_blocks;
    return launch_chained(qkv_append_kernel<D, CACHE>, dim3((unsigned)(row_blocks + page_blocks)), dim3(kThreads), 0, 1, stream, a);
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
