// ec_paged_plan: pages for the new rows of every sequence of a batch, out of a stack of free ones, and a row of the pools and a position for every
// new token.
//
// With L_b rows that stay, n_b new ones and h_b pages held, sequence b wants ceil((L_b + n_b) / page) pages. Three sums over the sequences up to b
// say everything: of the new tokens (where b's tokens lie), of the pages given back (where they go on the stack), of the pages asked for
// (which of the stack's are b's, and whether there are enough). The sums are formed by one workgroup, a thread a sequence; what follows from them
// -- a page given, a page taken, a token -- is looked up by its number in the sums, so that long and short sequences cost the same.
// Bound by latency: a chain of loads, sums and stores, each behind a barrier (16 sequences of a token each 4.1 us; 256 sequences with 16100 tokens 9 us, and
// 3 for the tokens' launch).
#include "paged.h"

namespace ec {

constexpr uint32_t kPlanCap = 1u << 30;  // sums end here, beyond everything that is there, so that none wraps round

constexpr int kPlanThreads = 1024, kFewThreads = 256;  // of the workgroup, and where no more sequences and no more than kFewTokens tokens are there
constexpr int kFewTokens = 512, kPlanAhead = 4;        // kPlanAhead: pages that a thread moves at a time
// Tokens up to which the one workgroup writes their rows and positions itself, 1.1 us for every 1024; more are left to a second launch, 2.3 us.
constexpr int kPlanTokens = 2048, kTokenThreads = 256, kTokensEach = 4;

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

// For every x the least i of 0 .. n-1 with sums[i] > x (n if there is none); sums do not fall. Bound by the latency of LDS, so several are sought at a time.
template <int N> __device__ __forceinline__ void first_above(const uint32_t* sums, int n, const uint32_t (&x)[N], int (&at)[N])
{
#pragma unroll
    for (int u = 0; u < N; ++u) at[u] = 0;
    for (; n > 1; n -= n / 2) {
#pragma unroll
        for (int u = 0; u < N; ++u) at[u] = sums[at[u] + n / 2 - 1] <= x[u] ? at[u] + n / 2 : at[u];
    }
#pragma unroll
    for (int u = 0; u < N; ++u) at[u] += sums[at[u]] <= x[u];
}
__device__ __forceinline__ int first_above(const uint32_t* sums, int n, uint32_t x)
{
    const uint32_t xs[1] = {x};
    int at[1];
    first_above(sums, n, xs, at);
    return at[0];
}

// Rows and positions of kTokensEach tokens from t0 on, `step` apart. ends: sums of the sequences' tokens; start(b): where its rows start, -1 if it has none in
// this step; seen(b, its tokens): what it has seen before.
template <typename Start, typename Seen>
__device__ __forceinline__ void plan_tokens(const Plan& a, const uint32_t* ends, uint32_t t0, uint32_t step, Start&& start, Seen&& seen)
{
    uint32_t t[kTokensEach];
    int b[kTokensEach], id[kTokensEach], slot[kTokensEach], pos[kTokensEach];
#pragma unroll
    for (int u = 0; u < kTokensEach; ++u) t[u] = t0 + u * step;
    first_above(ends, a.B, t, b);
#pragma unroll
    for (int u = 0; u < kTokensEach; ++u) {
        id[u] = -1, slot[u] = pos[u] = 0;
        const int s = b[u] < a.B ? start(b[u]) : -1;
        if (s < 0) continue;
        const uint32_t first = b[u] ? ends[b[u] - 1] : 0, i = t[u] - first;
        slot[u] = s + (int)i;
        id[u] = a.table[(size_t)b[u] * a.max_pages + (slot[u] >> a.shift)];
        pos[u] = a.seen_after_b ? (int)(seen(b[u], ends[b[u]] - first) + i) : slot[u];
    }
#pragma unroll
    for (int u = 0; u < kTokensEach; ++u) {
        if (t[u] >= (uint32_t)a.T) return;
        const bool page = (unsigned)id[u] < (unsigned)a.n_pages;
        if (a.rows) a.rows[t[u]] = page ? ((int64_t)id[u] << a.shift) + (slot[u] & ((1 << a.shift) - 1)) : -1;
        if (a.pos) a.pos[t[u]] = pos[u];
    }
}

template <int THREADS> __global__ __launch_bounds__(THREADS) void paged_plan_kernel(Plan a)
{
    constexpr int MOST = THREADS == kPlanThreads ? kPlanMost : THREADS, WAVES = THREADS / kWave;
    __shared__ uint32_t upto[3][MOST];  // sums of new tokens, of pages given back, of pages asked for, b's own included
    __shared__ int held[MOST];
    __shared__ uint32_t of_wave[3][WAVES];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    uint32_t before[3] = {0, 0, 0};
    auto sum_up = [&](int which, uint32_t x) {  // over the workgroup, this thread's included, on top of the sequences before
        x = wave_scan(x);
        if (lane == kWave - 1) of_wave[which][wave] = min(x, kPlanCap);
        __syncthreads();
        uint32_t all = before[which];
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) x = min(x + all, kPlanCap);
            all = min(all + of_wave[which][w], kPlanCap);
        }
        before[which] = all;
        return x;
    };
    const uint32_t n_free = min(max(*a.n_free, 0), a.n_pages);
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        const int b = b0 + tid;
        uint32_t gives = 0, asks = 0;
        PlanWish w(a, min(b, a.B - 1));
        const uint32_t ends = sum_up(0, b < a.B ? w.tokens : 0);
        if (b < a.B) {
            const bool fits = w.fit(a, ends);
            gives = max(w.held - w.goal, 0);
            asks = fits ? max(w.goal - w.held, 0) : 0;
        }
        gives = sum_up(1, gives);
        asks = sum_up(2, asks);
        if (b < a.B) upto[0][b] = ends, upto[1][b] = gives, upto[2][b] = asks, held[b] = w.held;
        __syncthreads();
    }
    const uint32_t there = min(n_free + before[1], (uint32_t)a.n_pages);
    auto sum_before = [&](int which, int b) { return b ? upto[which][b - 1] : 0; };
    // given back, a sequence's last page first
    for (uint32_t j0 = tid; j0 < before[1]; j0 += THREADS * kPlanAhead) {
        uint32_t j[kPlanAhead];
        int b[kPlanAhead];
        int32_t* entry[kPlanAhead];
        int32_t page[kPlanAhead];
#pragma unroll
        for (int u = 0; u < kPlanAhead; ++u) j[u] = min(j0 + u * THREADS, before[1] - 1);
        first_above(upto[1], a.B, j, b);
#pragma unroll
        for (int u = 0; u < kPlanAhead; ++u) {
            entry[u] = a.table + (size_t)b[u] * a.max_pages + (held[b[u]] - 1 - (int)(j[u] - sum_before(1, b[u])));
            page[u] = *entry[u];
        }
#pragma unroll
        for (int u = 0; u < kPlanAhead; ++u) {
            if (j0 + u * THREADS >= before[1]) break;
            if (n_free + j[u] < (uint32_t)a.n_pages) a.free_pages[n_free + j[u]] = page[u];
            *entry[u] = -1;
        }
    }
    __syncthreads();
    // asked for: by the sequences up to the first whose sum is more than there is
    const int refused = first_above(upto[2], a.B, there);
    const uint32_t taken = refused ? upto[2][refused - 1] : 0;
    for (uint32_t j0 = tid; j0 < taken; j0 += THREADS * kPlanAhead) {
        uint32_t j[kPlanAhead];
        int b[kPlanAhead];
        int32_t* entry[kPlanAhead];
        int32_t page[kPlanAhead];
#pragma unroll
        for (int u = 0; u < kPlanAhead; ++u) {
            j[u] = min(j0 + u * THREADS, taken - 1);
            page[u] = a.free_pages[there - 1 - j[u]];
        }
        first_above(upto[2], a.B, j, b);
#pragma unroll
        for (int u = 0; u < kPlanAhead; ++u) entry[u] = a.table + (size_t)b[u] * a.max_pages + (held[b[u]] + (int)(j[u] - sum_before(2, b[u])));
#pragma unroll
        for (int u = 0; u < kPlanAhead; ++u)
            if (j0 + u * THREADS < taken) *entry[u] = page[u];
    }
    __syncthreads();
    for (int b = tid; b < a.B; b += THREADS) {
        PlanWish w(a, b);
        const bool fits = w.fit(a, upto[0][b]);
        const bool asks = fits && w.goal > w.held, granted = fits && (!asks || upto[2][b] <= there);
        const uint32_t tokens = granted ? w.tokens : 0;
        const int seen = a.seen_after_b ? a.seen_b[b] : 0, start = granted ? w.len : -1;
        a.held_b[b] = asks ? (granted ? w.goal : w.held) : min(w.goal, w.held);
        a.start_b[b] = start;
        a.len_after_b[b] = w.len + (int)tokens;
        if (a.seen_after_b) a.seen_after_b[b] = (int)((uint32_t)seen + tokens);
        a.token_start[b + 1] = (int)min(upto[0][b], (uint32_t)a.T);
        upto[1][b] = (uint32_t)start, upto[2][b] = (uint32_t)seen;  // for the tokens
    }
    if (tid == 0) {
        a.token_start[0] = 0;
        *a.n_free = (int)(there - taken);
    }
    if ((!a.rows && !a.pos) || a.T > kPlanTokens) return;
    __syncthreads();
    for (uint32_t t0 = tid; t0 < (uint32_t)a.T; t0 += THREADS * kTokensEach)
        plan_tokens(a, upto[0], t0, THREADS, [&](int b) { return (int)upto[1][b]; }, [&](int b, uint32_t) { return upto[2][b]; });
}

// Rows and positions of many tokens.
__global__ __launch_bounds__(kTokenThreads) void paged_tokens_kernel(Plan a)
{
    __shared__ uint32_t ends[kPlanMost];  // of the sequences' tokens
    for (int b = threadIdx.x; b < a.B; b += kTokenThreads) ends[b] = (uint32_t)a.token_start[b + 1];
    __syncthreads();
    plan_tokens(a, ends, blockIdx.x * kTokensEach * kTokenThreads + threadIdx.x, kTokenThreads, [&](int b) { return a.start_b[b]; },
                [&](int b, uint32_t tokens) { return a.seen_after_b ? (uint32_t)a.seen_after_b[b] - tokens : 0; });
}

int paged_plan_dispatch(const int32_t* len_b, const int32_t* new_b, const int32_t* seen_b, int32_t* page_table, int32_t* held_b, int32_t* free_pages,
                        int32_t* n_free, int B, int T, int page_shift, int n_pages, int max_pages, int32_t* start_b, int32_t* len_after_b,
                        int32_t* seen_after_b, int32_t* token_start, int64_t* rows, int32_t* pos, hipStream_t stream)
{
    const Plan a{len_b, new_b, seen_b, page_table, held_b, free_pages, n_free, start_b, len_after_b, seen_after_b, token_start, rows, pos, B, T, n_pages,
                 max_pages, page_shift};
    if (B <= kFewThreads && T <= kFewTokens)
        hipLaunchKernelGGL(paged_plan_kernel<kFewThreads>, dim3(1), dim3(kFewThreads), 0, stream, a);
    else
        hipLaunchKernelGGL(paged_plan_kernel<kPlanThreads>, dim3(1), dim3(kPlanThreads), 0, stream, a);
    if (const int rc = status_from_hip(hipGetLastError())) return rc;
    if ((!rows && !pos) || T <= kPlanTokens) return EC_OK;
    constexpr int kEach = kTokenThreads * kTokensEach;
    hipLaunchKernelGGL(paged_tokens_kernel, dim3((T + kEach - 1) / kEach), dim3(kTokenThreads), 0, stream, a);
    return status_from_hip(hipGetLastError());
}

}  // namespace ec
