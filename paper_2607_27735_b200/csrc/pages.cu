// Page bookkeeping between two steps of a serving program: how many pages every sequence needs for its new length, which
// physical pages it gets from (or gives back to) a pool, and where in the cache each of the step's rows goes.
//
// With need = ceil(new_len / page_size), give = max(held - need, 0) and take = max(need - held, 0) per sequence, all
// places follow from three exclusive prefix sums over the batch: the r-th page given back goes to pool[n_free + r], the
// t-th page taken comes off the top of that stack, pool[n_free + R - 1 - t] with R = sum(give), and row i of the
// step belongs to the last sequence whose first row is at or before i.  A page that is given and taken in the same call is
// read from its former owner's table, so no thread ever waits for what another one writes: one launch, every CTA
// makes the sums for itself (a few thousand lengths at most), and the CTA that finishes last stores the new counts.
// The call is a chain of latencies (lengths -> sums -> table -> slot): nothing here is bound by bytes below some
// hundred thousand rows.  64 sequences with a round's 576 rows take 6.0 us, 256 with 75 K rows (1.6 MB) 9.2; 4.0 and 5.8 where every
// sequence holds its pages already.
#include "chained.cuh"
#include "spec_common.cuh"

namespace spec {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxSeqs = 2048;

struct Sums {
    int take, give;
    long long rows;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) { return Sums{a.take + b.take, a.give + b.give, a.rows + b.rows}; }
__device__ __forceinline__ Sums shfl_up(const Sums& s, int o)
{
    return Sums{__shfl_up_sync(0xffffffffu, s.take, o), __shfl_up_sync(0xffffffffu, s.give, o),
                __shfl_up_sync(0xffffffffu, s.rows, o)};
}

// Largest b with start[b] <= i (start[0] == 0, ascending, n entries).
__device__ __forceinline__ int owner(const int* start, int n, int i)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct PagesArgs {
    const int32_t* first_pos;
    const int32_t* new_len;
    int batch, page_size, max_pages, n_pages, max_rows;
    int32_t* table;
    int32_t* n_held;
    int32_t* pool;
    int32_t* n_free;
    int32_t* cu_rows;
    int32_t* positions;
    int32_t* slots;
    int* status;
    int* done;  // CTAs that have finished
};

__global__ void __launch_bounds__(kThreads) assign_pages_kernel(PagesArgs a)
{
    extern __shared__ int start_s[];  // [3][batch]: first page taken, first page given, first row of each sequence
    int* take0 = start_s;
    int* give0 = take0 + a.batch;
    int* row0 = give0 + a.batch;
    __shared__ Sums warp_s[kThreads / 32];
    __shared__ int bad_s, last_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) bad_s = 0;
    stream_wait_only();
    __syncthreads();

    // consecutive sequences per thread
    const int per = (a.batch + kThreads - 1) / kThreads, b0 = tid * per, b1 = min(a.batch, b0 + per);
    const int64_t cap = (int64_t)a.max_pages * a.page_size;
    Sums mine{0, 0, 0};
    bool bad = false;
    for (int b = b0; b < b1; ++b) {
        const int f = a.first_pos[b], n = a.new_len[b], held = a.n_held[b];
        if (f < 0 || n < 0 || n > cap || held < 0 || held > a.max_pages) {
            bad = true;
            break;
        }
        const int need = (int)(((int64_t)n + a.page_size - 1) / a.page_size);
        mine = mine + Sums{max(need - held, 0), max(held - need, 0), max(n - f, 0)};
    }
    if (bad) bad_s = 1;
    Sums up = mine;  // inclusive over the threads
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums y = shfl_up(up, o);
        if (lane >= o) up = up + y;
    }
    if (lane == 31) warp_s[warp] = up;
    __syncthreads();
    Sums base{0, 0, 0}, all{0, 0, 0};
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w == warp) base = all;
        all = all + warp_s[w];
    }
    const int n_free = *a.n_free;
    // the whole call or nothing: a length out of range, too few pages or too little room for the rows changes no state
    int err = SPEC_OK;
    if (bad_s || n_free < 0 || (int64_t)n_free + all.give > a.n_pages || all.rows > a.max_rows) err = SPEC_ERR_BAD_INDEX;
    else if (all.take > n_free + all.give) err = SPEC_ERR_NO_PAGES;
    if (err == SPEC_OK) {
        Sums at{base.take + up.take - mine.take, base.give + up.give - mine.give, base.rows + up.rows - mine.rows};
        for (int b = b0; b < b1; ++b) {
            take0[b] = at.take;
            give0[b] = at.give;
            row0[b] = (int)at.rows;
            const int f = a.first_pos[b], n = a.new_len[b], held = a.n_held[b];
            const int need = (int)(((int64_t)n + a.page_size - 1) / a.page_size);
            at = at + Sums{max(need - held, 0), max(held - need, 0), max(n - f, 0)};
        }
    }
    __syncthreads();

    const int64_t stride = (int64_t)gridDim.x * kThreads, i0 = (int64_t)blockIdx.x * kThreads + tid;
    const int rows = err == SPEC_OK ? (int)all.rows : 0;
    auto pages_of = [&](int b) { return (int)(((int64_t)a.new_len[b] + a.page_size - 1) / a.page_size); };
    auto given = [&](int r) -> int {  // the r-th page given back
        const int b = owner(give0, a.batch, r);
        return a.table[(int64_t)b * a.max_pages + pages_of(b) + (r - give0[b])];
    };
    auto taken = [&](int t) -> int {  // the t-th page taken
        return t < all.give ? given(all.give - 1 - t) : a.pool[n_free - 1 - (t - all.give)];
    };
    for (int64_t i = i0; i < a.max_rows; i += stride) {
        int pos = 0, slot = -1;
        if (i < rows) {
            const int b = owner(row0, a.batch, (int)i);
            pos = a.first_pos[b] + ((int)i - row0[b]);
            const int j = pos / a.page_size, held = a.n_held[b];
            const int page = j < held ? a.table[(int64_t)b * a.max_pages + j] : taken(take0[b] + (j - held));
            if ((unsigned)page < (unsigned)a.n_pages) slot = page * a.page_size + (pos - j * a.page_size);
            else set_status(a.status, SPEC_ERR_BAD_INDEX);  // a table or a pool that holds no page number there
        }
        a.positions[i] = pos;
        a.slots[i] = slot;
    }
    if (err == SPEC_OK) {
        // (entries [held, need) of a table are written, entries below held or of a sequence that gives are read; the pool is
        // read below n_free and written from there on)
        for (int64_t t = i0; t < all.take; t += stride) {
            const int b = owner(take0, a.batch, (int)t);
            a.table[(int64_t)b * a.max_pages + a.n_held[b] + ((int)t - take0[b])] = taken((int)t);
        }
        for (int64_t r = i0; r < all.give; r += stride) a.pool[n_free + r] = given((int)r);
    }
    if (blockIdx.x == 0)
        for (int b = tid; b <= a.batch; b += kThreads)
            a.cu_rows[b] = err != SPEC_OK ? 0 : (b < a.batch ? row0[b] : rows);
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        last_s = atomicAdd(a.done, 1) == (int)gridDim.x - 1;
        if (err != SPEC_OK) set_status(a.status, err);
    }
    __syncthreads();
    if (!last_s) return;
    if (tid == 0) *a.done = 0;
    if (err != SPEC_OK) return;
    for (int b = tid; b < a.batch; b += kThreads) a.n_held[b] = pages_of(b);
    if (tid == 0) *a.n_free = n_free + all.give - all.take;
}

}  // namespace

size_t pages_workspace() { return kStatusBytes + 256; }

int assign_pages_launch(const int32_t* first_pos, const int32_t* new_len, int batch, int page_size, int max_pages, int n_pages,
                        int max_rows, int32_t* table, int32_t* n_held, int32_t* pool, int32_t* n_free, int32_t* cu_rows,
                        int32_t* positions, int32_t* slots, void* workspace, cudaStream_t stream)
{
    if (batch > kMaxSeqs) return SPEC_ERR_UNSUPPORTED_SHAPE;
    PagesArgs a{first_pos, new_len, batch, page_size, max_pages, n_pages, max_rows, table, n_held, pool, n_free, cu_rows,
                positions, slots, static_cast<int*>(workspace), static_cast<int*>(workspace) + kStatusBytes / sizeof(int)};
    const int64_t items = (int64_t)max_rows + batch;
    int grid = (int)((items + 2 * kThreads - 1) / (2 * kThreads));
    if (grid > 2 * sm_count()) grid = 2 * sm_count();
    return launch_chained(assign_pages_kernel, dim3(grid < 1 ? 1 : grid), dim3(kThreads), (size_t)batch * 3 * sizeof(int), 1, stream, a);
}

}  // namespace spec
