// Sampled drafts: probabilities of logits rows, and the acceptance of drafted tokens against them (the verification stage of
// "The Draft-Verification Paradigm" when tokens are drawn, not taken greedily).
//
// probs_kernel: p = softmax(z / T) row by row, fp32.  Bound by memory: 2 or 4 bytes in and 4 out per logit.  A row is
// split over a cluster of CTAs that keep their shares in shared memory between the sum and the store: the logits are read
// from memory once (576 bf16 rows of 128256: 95 us, 4.7 TB/s of 443 MB; read twice, through L2, they took 193).  What is
// left: a CTA loads, sums and stores one after the other, and six on an SM overlap no better.
//
// accept_kernel: drafted token x of row i is accepted iff all before it were and u_i q_i(x) < p_i(x); the first
// rejected row m is replaced by a draw from max(p_m - q_m, 0), or, with all accepted, from p_m, by inverting the
// cumulative sum at u_last times its total.  Only the drafted tokens' probabilities and one row pair per sequence are
// read.  The sums are in 64 bits (the difference of two fp32 numbers is exact there): the token is a whole number
// that an error of 1e-7 in a sum over 1e5 tokens would change every few dozen draws.  64 sequences, eight drafts, 128256
// tokens: 20.2 us for 66 MB with 39 % of the issue slots in use: a warp asks for its next vectors only when it has added up
// the last ones, and the second walk spills 136 bytes.  (64-bit sums by integer additions of scaled values: 25.6.)
#include <cooperative_groups.h>

#include "chained.cuh"
#include "draft_common.cuh"
#include "spec_common.cuh"

namespace cg = cooperative_groups;

namespace spec {

namespace {

// A cluster's exchange by stores: every CTA leaves its part in the shared memory of all, and nobody reads another CTA's, so
// one barrier does, and none before the end.  The first half of a barrier at the start of a kernel says that a CTA is there.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

constexpr float kInf = __builtin_huge_valf();
constexpr int kMaxCtas = 8;  // CTAs of a cluster

// ---- probabilities --------------------------------------------------------------------------

// 2^x by the hardware's approximation, within two units in the last place: one instruction for each of a row's logits, twice.
// Against 64 bits probabilities come out 0.8 to 1.3e-7 off, those of elementary fp32 operations 0.7 to 2.7e-7.  In the sums, which are
// at least 1, results below 2^-126 are flushed; probabilities keep them.
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float ex2_subnormal(float x)  // keeps results below 2^-126
{
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct Part {      // of a set of logits z: the largest, sum of e^((z - m) / T), the first place that holds m
    float m, s;
    int at;
};
__device__ __forceinline__ Part merge(const Part& a, const Part& b, float c)
{
    Part r;
    r.m = fmaxf(a.m, b.m);
    // (an empty part, or one of masked logits only, has m = -inf and s = 0)
    const float fa = a.m == r.m ? 1.f : ex2((a.m - r.m) * c), fb = b.m == r.m ? 1.f : ex2((b.m - r.m) * c);
    r.s = a.s * fa + b.s * fb;
    r.at = a.m > b.m ? a.at : (b.m > a.m ? b.at : min(a.at, b.at));
    return r;
}
__device__ __forceinline__ Part merge_lanes(Part p, float c, int lanes)
{
    for (int o = lanes / 2; o > 0; o >>= 1)
        p = merge(p, Part{__shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
                          __shfl_xor_sync(0xffffffffu, p.at, o)}, c);
    return p;
}

// Eight logits from the bits of a 16-byte (bf16) or two 16-byte (fp32) vectors.
template <int DT>
struct Vec {
    uint4 w[DT == 1 ? 1 : 2];
    __device__ __forceinline__ void unpack(float (&z)[8]) const
    {
        if (DT == 1) {
            z[0] = bf16_lo(w[0].x), z[1] = bf16_hi(w[0].x), z[2] = bf16_lo(w[0].y), z[3] = bf16_hi(w[0].y);
            z[4] = bf16_lo(w[0].z), z[5] = bf16_hi(w[0].z), z[6] = bf16_lo(w[0].w), z[7] = bf16_hi(w[0].w);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                z[4 * i] = __uint_as_float(w[i % (DT == 1 ? 1 : 2)].x), z[4 * i + 1] = __uint_as_float(w[i % (DT == 1 ? 1 : 2)].y);
                z[4 * i + 2] = __uint_as_float(w[i % (DT == 1 ? 1 : 2)].z), z[4 * i + 3] = __uint_as_float(w[i % (DT == 1 ? 1 : 2)].w);
            }
        }
    }
};
template <int DT>
__device__ __forceinline__ float load1(const void* row, int64_t at)
{
    return DT == 1 ? __bfloat162float(static_cast<const __nv_bfloat16*>(row)[at]) : static_cast<const float*>(row)[at];
}
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kProbThreads = 256, kProbWarps = kProbThreads / 32;

// One cluster (gridDim.x CTAs) per row.  STAGED: a thread copies its groups of eight logits to shared memory (asynchronously, all in
// flight at once, no registers held) and walks them three times there: largest, sum, store; a CTA's 32 KB at a 128 K
// vocabulary in bf16 leave room for six CTAs on an SM, whose loads, exchanges and stores overlap.  Else (a share beyond shared
// memory) it walks them in global memory, where the second and third visit find them in L2.
// Exponentials are 2^((z - m) c), c = log2 e / T: the difference first, so that its error does not grow with |m|.
// A row's first `head` logits, up to its first 16-byte boundary, and its last few after the whole groups are one per thread
// of the first and of the last CTA.
template <int DT, bool STAGED>
__global__ void __launch_bounds__(kProbThreads, 6)
probs_kernel(const void* logits, int vocab, int64_t row_stride, const float* temperature, float* probs, int64_t out_stride)
{
    extern __shared__ __align__(16) uint8_t stage_s[];
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ Part warp_part[kProbWarps];
    __shared__ Part cta_part[kMaxCtas], row_part;
    constexpr int ES = DT == 1 ? 2 : 4, NW = DT == 1 ? 1 : 2;
    const int CS = gridDim.x, rank = blockIdx.x, row = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (CS > 1) cluster_arrive();
    stream_wait();
    const char* base = static_cast<const char*>(logits) + (int64_t)row * row_stride * ES;
    float* out = probs + (int64_t)row * out_stride;

    const int head = min(vocab, (int)((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15) / ES);
    const int groups = (vocab - head) / 8, tail = vocab - head - 8 * groups;
    const int g_per = (groups + CS - 1) / CS;
    const int g0 = min(groups, rank * g_per), g1 = min(groups, g0 + g_per);
    const uint4* src = reinterpret_cast<const uint4*>(base + head * ES);
    uint4* stage = reinterpret_cast<uint4*>(stage_s);  // (a thread reads back only what it has copied itself)
    if (STAGED) {
        for (int g = g0 + tid; g < g1; g += kProbThreads)
#pragma unroll
            for (int i = 0; i < NW; ++i)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(stage + (g - g0) * NW + i)),
                             "l"(src + (int64_t)g * NW + i) : "memory");
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    const float t = temperature ? temperature[row] : 1.f;
    const bool greedy = t <= 0.f;
    const float c = greedy ? kLog2e : fminf(1.f / t, 1e30f) * kLog2e;  // (so small a t leaves the largest logits only, as 1 / t = inf would not)
    const int single = rank == 0 && tid < head ? tid : (rank == CS - 1 && tid >= 16 && tid - 16 < tail ? head + 8 * groups + tid - 16 : -1);
    const float z1 = single >= 0 ? load1<DT>(base, single) : -kInf;
    if (STAGED) asm volatile("cp.async.wait_group 0;" ::: "memory");
    auto fetch = [&](int g) -> Vec<DT> {
        Vec<DT> v;
#pragma unroll
        for (int i = 0; i < NW; ++i) v.w[i] = STAGED ? stage[(g - g0) * NW + i] : __ldcg(src + (int64_t)g * NW + i);
        return v;
    };

    Part mine{z1, 0.f, 0x7fffffff};
    for (int g = g0 + tid; g < g1; g += kProbThreads) {
        float z[8];
        fetch(g).unpack(z);
#pragma unroll
        for (int i = 0; i < 8; ++i) mine.m = fmaxf(mine.m, z[i]);
    }
    if (!(mine.m > -kInf)) mine.m = -kInf;  // (a NaN alone)
    const float ref = mine.m == -kInf ? 0.f : mine.m;
    if (greedy) {
        if (mine.m > -kInf) {
            if (z1 == mine.m) mine.at = single;
            for (int g = g0 + tid; g < g1; g += kProbThreads) {
                float z[8];
                fetch(g).unpack(z);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (z[i] == mine.m) mine.at = min(mine.at, head + 8 * g + i);
            }
        }
    } else {
        float s = ex2((z1 - ref) * c);
        for (int g = g0 + tid; g < g1; g += kProbThreads) {
            float z[8];
            fetch(g).unpack(z);
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = ex2((z[i] - ref) * c);
            s += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        }
        mine.s = s;
    }
    // warp, CTA, cluster, in a fixed order
    mine = merge_lanes(mine, c, 32);
    if (lane == 0) warp_part[warp] = mine;
    __syncthreads();
    if (CS > 1) cluster_wait();
    if (warp == 0) {
        Part p = lane < kProbWarps ? warp_part[lane] : Part{-kInf, 0.f, 0x7fffffff};
        p = merge_lanes(p, c, kProbWarps);  // (on each of the first lanes)
        if (CS == 1 && lane == 0) row_part = p;
        if (CS > 1 && lane < CS) *cluster.map_shared_rank(&cta_part[rank], lane) = p;
        __syncwarp();
    }
    if (CS > 1) {
        cluster_arrive();
        cluster_wait();
        if (warp == 0) {
            Part p{-kInf, 0.f, 0x7fffffff};
            if (lane < CS) p = cta_part[lane];
            p = merge_lanes(p, c, kMaxCtas);
            if (lane == 0) row_part = p;
        }
    }
    __syncthreads();
    const Part all = row_part;

    const bool vec = (reinterpret_cast<uintptr_t>(out + head) & 15) == 0;
    const bool none = all.m == -kInf && all.s == 0.f;  // nothing is left of the row
    const float inv_s = none ? 0.f : 1.f / all.s, top = all.m == -kInf ? 0.f : all.m;
    if (single >= 0) out[single] = greedy ? (single == all.at ? 1.f : 0.f) : ex2_subnormal((z1 - top) * c) * inv_s;
    for (int g = g0 + tid; g < g1; g += kProbThreads) {
        const int at = head + 8 * g;
        float z[8];
        fetch(g).unpack(z);
        if (greedy) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = at + i == all.at ? 1.f : 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = (z[i] - top) * c;
            const float least = fminf(fminf(fminf(z[0], z[1]), fminf(z[2], z[3])), fminf(fminf(z[4], z[5]), fminf(z[6], z[7])));
            if (least < -125.f) {  // results below 2^-126: four instructions more each
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = ex2_subnormal(z[i]) * inv_s;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = ex2(z[i]) * inv_s;
            }
        }
        if (vec) {
            __stcs(reinterpret_cast<float4*>(out + at), make_float4(z[0], z[1], z[2], z[3]));
            __stcs(reinterpret_cast<float4*>(out + at) + 1, make_float4(z[4], z[5], z[6], z[7]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) out[at + i] = z[i];
        }
    }
}

template <int DT, bool STAGED>
int launch_probs(int cs, int n_rows, int64_t smem, cudaStream_t stream, const void* logits, int vocab, int64_t row_stride,
                 const float* temperature, float* probs, int64_t out_stride)
{
    auto kern = probs_kernel<DT, STAGED>;
    if (smem && !draft::opt_in_smem(reinterpret_cast<const void*>(kern), (size_t)smem)) return SPEC_ERR_CUDA;
    return launch_chained(kern, dim3(cs, n_rows), dim3(kProbThreads), (size_t)smem, cs, stream, logits, vocab, row_stride, temperature, probs,
                          out_stride);
}

template <int DT>
int probs_of(const void* logits, int n_rows, int vocab, int64_t row_stride, const float* temperature, float* probs,
             int64_t out_stride, cudaStream_t stream)
{
    // CTAs of a row: as few as keep a share within 40 KB, so that five or more share an SM (six at 32 KB, 128 K tokens in bf16); more
    // while the rows alone leave SMs idle and every thread has a few groups
    constexpr int kGroup = DT == 1 ? 16 : 32;
    constexpr int kShare = 40 * 1024, kMost = 200 * 1024;
    const int groups = vocab / 8 + 1;
    int cs = 1;
    while (cs < kMaxCtas && (int64_t)((groups + cs - 1) / cs) * kGroup > kShare) cs *= 2;
    while (cs < kMaxCtas && (long)n_rows * cs * 2 <= 2L * sm_count() && groups >= 4 * cs * kProbThreads) cs *= 2;
    const int64_t share = (int64_t)((groups + cs - 1) / cs) * kGroup;
    if (share > kMost)
        return launch_probs<DT, false>(cs, n_rows, 0, stream, logits, vocab, row_stride, temperature, probs, out_stride);
    return launch_probs<DT, true>(cs, n_rows, share, stream, logits, vocab, row_stride, temperature, probs, out_stride);
}

// ---- acceptance -----------------------------------------------------------------------------

constexpr int kChunk = 128;  // tokens that a warp takes at a time, four neighbours per lane

__device__ __forceinline__ double warp_sum_f64(double x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

struct AcceptArgs {
    const float* p;
    int64_t p_batch, p_row;
    const float* q;  // null: every drafted token was taken with probability 1
    int64_t q_batch, q_row;
    const int32_t* draft;
    const int32_t* n_draft;
    const float* u;
    int batch, k, vocab;
    int32_t* n_accepted;
    int32_t* next_token;
};

// One cluster per sequence; every warp has a contiguous share of the vocabulary.
template <int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) accept_sample_kernel(AcceptArgs a)
{
    constexpr int kWarps = kThreads / 32, kPerLane = kMaxCtas * kWarps / 32;  // shares of a cluster, for each lane of a warp
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ double sum_s[kMaxCtas * kWarps];  // mass of every warp's share
    __shared__ int owner_s;
    __shared__ double before_s, target_s;
    const int CS = gridDim.x, rank = blockIdx.x, b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int V = a.vocab, k = a.k;
    if (CS > 1) cluster_arrive();
    stream_wait();
    const float* u = a.u + (int64_t)b * (k + 1);

    // ---- how many drafted tokens stand: every warp for itself, 32 at a time ----
    const int nd = a.n_draft ? min(max(a.n_draft[b], 0), k) : k;
    int m = 0;
    for (int i0 = 0; i0 < nd; i0 += 32) {
        const int i = i0 + lane;
        bool ok = false;
        if (i < nd) {
            const int x = a.draft[(int64_t)b * k + i];
            if (x >= 0 && x < V) {
                const float p = fmaxf(a.p[b * a.p_batch + i * a.p_row + x], 0.f);  // (NaN as well: 0)
                const float q = a.q ? fmaxf(a.q[b * a.q_batch + i * a.q_row + x], 0.f) : 1.f;
                ok = (double)u[i] * (double)q < (double)p;  // the product of two fp32 numbers is exact in 64 bits
            }
        }
        const uint32_t wrong = ~__ballot_sync(0xffffffffu, ok);
        m = i0 + (wrong ? __ffs((int)wrong) - 1 : 32);
        if (wrong) break;
    }
    m = min(m, nd);
    const bool rejected = m < nd;
    const float* p = a.p + b * a.p_batch + m * a.p_row;
    const float* q = rejected && a.q ? a.q + b * a.q_batch + m * a.q_row : nullptr;
    int hot = rejected && !a.q ? a.draft[(int64_t)b * k + m] : -1;  // without q: the token that is taken out

    const bool vec = ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & 15) == 0;
    auto load4 = [&](const float* r, int v) -> float4 {  // four neighbouring tokens of a lane; beyond the vocabulary zeros
        if (vec && v + 4 <= V) return *reinterpret_cast<const float4*>(r + v);
        return make_float4(v < V ? r[v] : 0.f, v + 1 < V ? r[v + 1] : 0.f, v + 2 < V ? r[v + 2] : 0.f, v + 3 < V ? r[v + 3] : 0.f);
    };
    auto weight = [&](float pv, float qv, int v) -> double {  // max(p - q, 0); what is NaN or negative counts as 0
        qv = v == hot ? 1.f : fmaxf(qv, 0.f);
        return pv > qv ? (double)pv - (double)qv : 0.0;
    };

    const int chunks = (V + kChunk - 1) / kChunk, W = CS * kWarps;
    const int per = (chunks + W - 1) / W;
    const int seg = rank * kWarps + warp, c0 = min(chunks, seg * per), c1 = min(chunks, c0 + per);
    // the mass of this warp's share with q (or the token taken out), or of p alone
    auto share_sum = [&]() -> double {
        double s = 0.0;
        for (int c = c0; c < c1; c += 4) {
            float4 pv[4], qv[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = c + j < c1 ? (c + j) * kChunk + 4 * lane : V;
                pv[j] = load4(p, v);
                qv[j] = q ? load4(q, v) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = (c + j) * kChunk + 4 * lane;
                s += (weight(pv[j].x, qv[j].x, v) + weight(pv[j].y, qv[j].y, v + 1)) +
                     (weight(pv[j].z, qv[j].z, v + 2) + weight(pv[j].w, qv[j].w, v + 3));
            }
        }
        return warp_sum_f64(s);
    };
    auto exchange = [&](double s) {  // every CTA of the cluster gets the sums of all
        if (CS > 1) {
            cluster_wait();
            if (lane < CS) *cluster.map_shared_rank(&sum_s[seg], lane) = s;
            __syncwarp();
            cluster_arrive();
            cluster_wait();
        } else {
            if (lane == 0) sum_s[seg] = s;
            __syncthreads();
        }
    };
    // Which warp's share the draw falls into, and what lies before it; false if there is no mass at all.  (Warp 0 of every CTA
    // alike, a few neighbouring shares per lane.)
    auto locate = [&]() -> bool {
        if (warp == 0) {
            double x[kPerLane], mine = 0.0;
#pragma unroll
            for (int j = 0; j < kPerLane; ++j) {
                x[j] = kPerLane * lane + j < W ? sum_s[kPerLane * lane + j] : 0.0;
                mine += x[j];
            }
            double incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double t = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += t;
            }
            // (a number of 1 or more is past the total however this sum and the ones that follow are rounded)
            const double target = u[k] >= 1.f ? (double)kInf : (double)u[k] * __shfl_sync(0xffffffffu, incl, 31);
            double at = __shfl_up_sync(0xffffffffu, incl, 1), before = 0.0, before_last = 0.0;
            if (lane == 0) at = 0.0;
            int first = -1, last = -1;  // the first share that the draw does not pass, the last one with anything in it
#pragma unroll
            for (int j = 0; j < kPerLane; ++j) {
                if (x[j] > 0.0) {
                    last = kPerLane * lane + j;
                    before_last = at;
                    if (first < 0 && at + x[j] > target) {
                        first = last;
                        before = at;
                    }
                }
                at += x[j];
            }
            const uint32_t some = __ballot_sync(0xffffffffu, first >= 0), any = __ballot_sync(0xffffffffu, last >= 0);
            if (any == 0) {
                if (lane == 0) owner_s = -1;
            } else if (lane == (some ? __ffs((int)some) - 1 : 31 - __clz((int)any))) {
                owner_s = some ? first : last;
                before_s = some ? before : before_last;
                target_s = target;
            }
        }
        __syncthreads();
        return owner_s >= 0;
    };

    exchange(share_sum());
    bool mass = locate();
    if (!mass && rejected) {  // p <= q everywhere (the same on every CTA): nothing is left but p itself
        q = nullptr;
        hot = -1;
        if (CS > 1) cluster_arrive();  // everybody has read the sums
        else __syncthreads();
        exchange(share_sum());
        mass = locate();
    }
    if (rank == 0 && tid == 0) {
        a.n_accepted[b] = m;
        if (!mass) a.next_token[b] = 0;
    }
    if (mass && owner_s == seg) {
        double before = before_s;
        const double target = target_s;
        int token = -1, last = -1;
        for (int c = c0; c < c1 && token < 0; c += 4) {  // four chunks per trip to memory
            float4 pv[4], qv[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = c + j < c1 ? (c + j) * kChunk + 4 * lane : V;
                pv[j] = load4(p, v);
                qv[j] = q ? load4(q, v) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            double incl[4];  // of the lanes, chunk by chunk (four scans side by side)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = (c + j) * kChunk + 4 * lane;
                incl[j] = (weight(pv[j].x, qv[j].x, v) + weight(pv[j].y, qv[j].y, v + 1)) +
                          (weight(pv[j].z, qv[j].z, v + 2) + weight(pv[j].w, qv[j].w, v + 3));
            }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const double t = __shfl_up_sync(0xffffffffu, incl[j], o);
                    if (lane >= o) incl[j] += t;
                }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (token >= 0) break;  // the same for the whole warp
                const int v = (c + j) * kChunk + 4 * lane;
                const float pw[4] = {pv[j].x, pv[j].y, pv[j].z, pv[j].w}, qw[4] = {qv[j].x, qv[j].y, qv[j].z, qv[j].w};
                double at = __shfl_up_sync(0xffffffffu, incl[j], 1);
                at = before + (lane ? at : 0.0);
                int hit = -1, lst = -1;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double w = weight(pw[i], qw[i], v + i);
                    at += w;
                    if (w > 0.0) {
                        lst = v + i;
                        if (hit < 0 && at > target) hit = lst;
                    }
                }
                const uint32_t some = __ballot_sync(0xffffffffu, hit >= 0), any = __ballot_sync(0xffffffffu, lst >= 0);
                if (some) token = __shfl_sync(0xffffffffu, hit, __ffs((int)some) - 1);
                if (any) last = __shfl_sync(0xffffffffu, lst, 31 - __clz((int)any));
                before += __shfl_sync(0xffffffffu, incl[j], 31);
            }
        }
        // (a draw at or past the total, or between the rounding of two sums: the last token with any mass)
        if (lane == 0) a.next_token[b] = token >= 0 ? token : last;
    }
}

}  // namespace

int probs_launch(const void* logits, int dtype, int n_rows, int vocab, int64_t row_stride, const float* temperature, float* probs,
                 int64_t out_stride, cudaStream_t stream)
{
    return dtype == 1 ? probs_of<1>(logits, n_rows, vocab, row_stride, temperature, probs, out_stride, stream)
                      : probs_of<0>(logits, n_rows, vocab, row_stride, temperature, probs, out_stride, stream);
}

int accept_sample_launch(const float* p, int64_t p_batch, int64_t p_row, const float* q, int64_t q_batch, int64_t q_row,
                         const int32_t* draft, const int32_t* n_draft, const float* u, int batch, int k, int vocab,
                         int32_t* n_accepted, int32_t* next_token, cudaStream_t stream)
{
    // CTAs of a sequence: while all of them fit the SMs at once (four on each) and every warp has a few chunks; sequences that
    // would leave SMs idle even so get CTAs of 32 warps
    int cs = 1;
    while (cs < kMaxCtas && (long)batch * cs * 2 <= 4L * sm_count() && vocab >= 2 * cs * 8 * kChunk) cs *= 2;
    const AcceptArgs a{p, p_batch, p_row, q, q_batch, q_row, draft, n_draft, u, batch, k, vocab, n_accepted, next_token};
    if ((long)batch * cs <= 2L * sm_count() && (long)batch * cs > sm_count() && vocab >= 2 * cs * 16 * kChunk)
        return launch_chained(accept_sample_kernel<512>, dim3(cs, batch), dim3(512), 0, cs, stream, a);
    if ((long)batch * cs <= sm_count() && vocab >= 2 * cs * 32 * kChunk)
        return launch_chained(accept_sample_kernel<1024>, dim3(cs, batch), dim3(1024), 0, cs, stream, a);
    return launch_chained(accept_sample_kernel<256>, dim3(cs, batch), dim3(256), 0, cs, stream, a);
}

}  // namespace spec
