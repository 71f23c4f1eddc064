// ec_paged_plan: pages for the new rows of every sequence of a batch, out of a stack of free ones, and a row of the pools and a position for every
// new token.
//
// With L_b rows that stay, n_b new ones and h_b pages held, sequence b wants ceil((L_b + n_b) / page) pages. Three sums over the sequences up to b
// say everything: of the new tokens (where b's tokens lie), of the pages given back (where they go on the stack), of the pages asked for
// (which of the stack's are b's, and whether there are enough). The sums are formed by one workgroup, a thread a sequence; what follows from them
// -- a page given, a page taken, a token -- is looked up by its number in the sums, so that long and short sequences cost the same.
// Bound by latency: a chain of loads, sums and stores, each behind a barrier.
#include "paged.h"

namespace ec {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;
constexpr uint32_t kPlanCap = 1u << 30;  // sums end here, beyond everything that is there, so that none wraps round

struct Plan {
    const int32_t *len_b, *new_b, *seen_b;
    int32_t *table, *held_b, *free_pages, *n_free;
    int32_t *start_b, *len_after_b, *seen_after_b, *token_start;
    int64_t* rows;
    int32_t* pos;
    int B, T, n_pages, max_pages, shift;
};

// What sequence b has and wants; -1 for len: no sequence.
struct PlanWish {
    int len, held, goal;  // goal: pages afterwards if it fits, else those of the rows that it has (at most one more than a table holds)
    uint32_t tokens;
    __device__ __forceinline__ PlanWish(const Plan& a, int b)
    {
        len = max(a.len_b[b], -1);
        held = min(max(a.held_b[b], 0), a.max_pages);
        tokens = min(max(a.new_b[b], 0), a.T + 1);
        goal = 0;
    }
    // upto: tokens up to this sequence's last
    __device__ __forceinline__ bool fit(const Plan& a, uint32_t upto)
    {
        const int64_t up = (1 << a.shift) - 1, want = ((int64_t)len + tokens + up) >> a.shift, keep = ((int64_t)len + up) >> a.shift;
        const bool fits = len >= 0 && upto <= (uint32_t)a.T && want <= a.max_pages;
        goal = len < 0 ? 0 : fits ? (int)want : (int)(keep < a.max_pages ? keep : (int64_t)a.max_pages + 1);
        return fits;
    }
};

// Least i of 0 .. n-1 with sums[i] > x (n if there is none); sums do not fall.
__device__ __forceinline__ int first_above(const uint32_t* sums, int n, uint32_t x)
{
    int lo = 0;
    while (n > 0) {
        const int half = n >> 1;
        const bool up = sums[lo + half] <= x;
        lo = up ? lo + half + 1 : lo;
        n = up ? n - half - 1 : half;
    }
    return lo;
}

// Row and position of token t, the i-th of sequence b, or of no sequence (b < 0).
__device__ __forceinline__ void plan_token(const Plan& a, uint32_t t, int b, uint32_t i, uint32_t tokens)
{
    int64_t row = -1;
    int pos = 0;
    const int start = b < 0 ? -1 : a.start_b[b];
    if (start >= 0) {
        const int slot = start + (int)i, id = a.table[(size_t)b * a.max_pages + (slot >> a.shift)];
        if ((unsigned)id < (unsigned)a.n_pages) row = ((int64_t)id << a.shift) + (slot & ((1 << a.shift) - 1));
        pos = a.seen_after_b ? (int)((uint32_t)a.seen_after_b[b] - tokens + i) : slot;
    }
    if (a.rows) a.rows[t] = row;
    if (a.pos) a.pos[t] = pos;
}

__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(Plan a)
{
    __shared__ uint32_t upto[3][kPlanMost];  // sums of new tokens, of pages given back, of pages asked for, b's own included
    __shared__ uint32_t of_wave[3][kPlanWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    uint32_t before[3] = {0, 0, 0};
    auto sum_up = [&](int which, uint32_t x) {  // over the workgroup, this thread's included, on top of the sequences before
        x = wave_scan(x);
        if (lane == kWave - 1) of_wave[which][wave] = min(x, kPlanCap);
        __syncthreads();
        uint32_t all = before[which];
        for (int w = 0; w < kPlanWaves; ++w) {
            if (w == wave) x = min(x + all, kPlanCap);
            all = min(all + of_wave[which][w], kPlanCap);
        }
        before[which] = all;
        return x;
    };
    for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        uint32_t tokens = 0, gives = 0, asks = 0;
        if (b < a.B) tokens = PlanWish(a, b).tokens;
        const uint32_t ends = sum_up(0, tokens);
        if (b < a.B) {
            PlanWish w(a, b);
            const bool fits = w.fit(a, ends);
            gives = max(w.held - w.goal, 0);
            asks = fits ? max(w.goal - w.held, 0) : 0;
        }
        gives = sum_up(1, gives);
        asks = sum_up(2, asks);
        if (b < a.B) upto[0][b] = ends, upto[1][b] = gives, upto[2][b] = asks;
        __syncthreads();
    }
    const uint32_t n_free = min(max(*a.n_free, 0), a.n_pages), there = min(n_free + before[1], (uint32_t)a.n_pages);
    auto sum_before = [&](int which, int b) { return b ? upto[which][b - 1] : 0; };
    for (uint32_t j = tid; j < before[1]; j += kPlanThreads) {  // given back, a sequence's last page first
        const int b = first_above(upto[1], a.B, j), e = min(max(a.held_b[b], 0), a.max_pages) - 1 - (int)(j - sum_before(1, b));
        int32_t* entry = a.table + (size_t)b * a.max_pages + e;
        if (n_free + j < (uint32_t)a.n_pages) a.free_pages[n_free + j] = *entry;
        *entry = -1;
    }
    __syncthreads();
    // asked for: by the sequences up to the first whose sum is more than there is
    const int refused = first_above(upto[2], a.B, there);
    const uint32_t taken = refused ? upto[2][refused - 1] : 0;
    for (uint32_t j = tid; j < taken; j += kPlanThreads) {
        const int b = first_above(upto[2], a.B, j), e = min(max(a.held_b[b], 0), a.max_pages) + (int)(j - sum_before(2, b));
        a.table[(size_t)b * a.max_pages + e] = a.free_pages[there - 1 - j];
    }
    __syncthreads();
    for (int b = tid; b < a.B; b += kPlanThreads) {
        PlanWish w(a, b);
        const bool fits = w.fit(a, upto[0][b]);
        const bool asks = fits && w.goal > w.held, granted = fits && (!asks || upto[2][b] <= there);
        const uint32_t tokens = granted ? w.tokens : 0;
        const int seen = a.seen_after_b ? a.seen_b[b] : 0;
        a.held_b[b] = asks ? (granted ? w.goal : w.held) : min(w.goal, w.held);
        a.start_b[b] = granted ? w.len : -1;
        a.len_after_b[b] = w.len + (int)tokens;
        if (a.seen_after_b) a.seen_after_b[b] = (int)((uint32_t)seen + tokens);
        a.token_start[b + 1] = (int)min(upto[0][b], (uint32_t)a.T);
    }
    if (tid == 0) {
        a.token_start[0] = 0;
        *a.n_free = (int)(there - taken);
    }
    if (!a.rows && !a.pos) return;
    __syncthreads();
    for (uint32_t t = tid; t < (uint32_t)a.T; t += kPlanThreads) {
        const int b = first_above(upto[0], a.B, t);
        const uint32_t first = b < a.B ? sum_before(0, b) : 0;
        plan_token(a, t, b < a.B ? b : -1, t - first, b < a.B ? upto[0][b] - first : 0);
    }
}

int paged_plan_dispatch(const int32_t* len_b, const int32_t* new_b, const int32_t* seen_b, int32_t* page_table, int32_t* held_b, int32_t* free_pages,
                        int32_t* n_free, int B, int T, int page_shift, int n_pages, int max_pages, int32_t* start_b, int32_t* len_after_b,
                        int32_t* seen_after_b, int32_t* token_start, int64_t* rows, int32_t* pos, hipStream_t stream)
{
    const Plan a{len_b, new_b, seen_b, page_table, held_b, free_pages, n_free, start_b, len_after_b, seen_after_b, token_start, rows, pos, B, T, n_pages,
                 max_pages, page_shift};
    hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
    return status_from_hip(hipGetLastError());
}

}  // namespace ec
