// ec_paged_store, ec_paged_evict_min: rows into the pages of their sequences, and rows out of them.
#include <algorithm>

#include "paged.h"

namespace ec {

// ------------------------------------------------------------------ store
// A workgroup per 32 rows of a (sequence, head), one more head for the positions and masses of every score group.
constexpr int kStoreRows = 32;
template <int CH>  // 16-byte chunks of a row
__global__ __launch_bounds__(256) void paged_store_kernel(const u32x4* __restrict__ k, const u32x4* __restrict__ v, const int32_t* __restrict__ pos,
                                                          const float* __restrict__ mass, Pages pages, const int32_t* __restrict__ start_b,
                                                          const int32_t* __restrict__ n_rows_b, int Hkv, int G, int T, int src_rows, u32x4* k_pages,
                                                          u32x4* v_pages, int32_t* pos_pages, float* mass_pages)
{
    const int b = blockIdx.z, head = blockIdx.y, r0 = blockIdx.x * kStoreRows;
    const int n = min(max(n_rows_b ? n_rows_b[b] : T, 0), T), start = start_b ? start_b[b] : 0;
    auto slot_of = [&](int r) {
        const int64_t s = (int64_t)start + r;
        return r < n && s >= 0 && s < pages.slots() ? (int)s : -1;
    };
    if (head < Hkv && k) {
        for (int i = threadIdx.x; i < kStoreRows * CH; i += 256) {
            const int r = r0 + i / CH, s = slot_of(r), id = s < 0 ? -1 : pages.page_of(b, s);
            if (id < 0) continue;
            const size_t from = (((size_t)b * Hkv + head) * src_rows + r) * CH + i % CH, to = pages.row(id, Hkv, head, s) * CH + i % CH;
            k_pages[to] = k[from];
            v_pages[to] = v[from];
        }
    }
    if (head == 0) {
        for (int i = threadIdx.x; i < kStoreRows * G; i += 256) {
            const int g = i / kStoreRows, r = r0 + i % kStoreRows, s = slot_of(r), id = s < 0 ? -1 : pages.page_of(b, s);
            if (id < 0) continue;
            const size_t from = ((size_t)b * G + g) * src_rows + r, to = pages.row(id, G, g, s);
            if (pos) pos_pages[to] = pos[from];
            if (mass) mass_pages[to] = mass[from];
        }
    }
}

int paged_store_dispatch(const void* k, const void* v, const int32_t* pos, const float* mass, const Pages& pages, const int32_t* start_b,
                         const int32_t* n_rows_b, int B, int Hkv, int G, int T, int src_rows, int row_bytes, void* k_pages, void* v_pages,
                         int32_t* pos_pages, float* mass_pages, hipStream_t stream)
{
    const dim3 grid((T + kStoreRows - 1) / kStoreRows, k ? Hkv : 1, B);
#define EC_STORE(CH_)                                                                                                                     \
    if (row_bytes == CH_ * 16)                                                                                                            \
        hipLaunchKernelGGL(paged_store_kernel<CH_>, grid, dim3(256), 0, stream, (const u32x4*)k, (const u32x4*)v, pos, mass, pages, start_b, \
                           n_rows_b, Hkv, G, T, src_rows, (u32x4*)k_pages, (u32x4*)v_pages, pos_pages, mass_pages)
    EC_STORE(8);
    EC_STORE(16);
    EC_STORE(32);
#undef EC_STORE
    return status_from_hip(hipGetLastError());
}

// ------------------------------------------------------------------ eviction
// A cache in pages is a set of rows: attention does not see their order, and every row carries its position.  So rows go without the others
// moving up: with m rows left, the victims below slot m are holes, the survivors at or behind it movers, as many of one as of the
// other, and the i-th hole takes the i-th mover.  Nothing that is read is written, so all moves run at once, and at most min(m, victims)
// rows move.
struct EvictGoal {
    const int32_t *len_b, *keep_b, *seen_b;
    int max_evict, protect_first, protect_recent;
    __device__ __forceinline__ int length(int b, int slots) const { return min(max(len_b[b], 0), slots); }
    __device__ __forceinline__ int victims(int b, int n) const { return min(max(n - max(keep_b[b], 0), 0), max_evict); }
};

// The order in which rows go, as an integer: fp32 order with -0 equal to +0, NaN behind +inf, protected rows (and rows on no page) last.
__device__ __forceinline__ uint32_t evict_key(float mass, bool kept)
{
    uint32_t u = __float_as_uint(mass);
    if (u == 0x80000000u) u = 0u;
    const uint32_t key = (u & 0x7fffffffu) > 0x7f800000u ? 0xfffffffeu : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return kept ? 0xffffffffu : key;
}

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave;

// Sum over the threads before this one (in lane order), and the sum over all of them in `total`.
__device__ __forceinline__ uint32_t scan_block(uint32_t x, uint32_t* sh, uint32_t& total)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    uint32_t in = x;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const uint32_t y = __shfl_up(in, off, kWave);
        if (lane >= off) in += y;
    }
    __syncthreads();
    if (lane == kWave - 1) sh[wave] = in;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) {
        if (w < wave) before += sh[w];
        total += sh[w];
    }
    return before + in - x;
}

// One workgroup per (sequence, score group): which rows go, the list of moves, and the moves of positions and masses.
__global__ __launch_bounds__(kEvictThreads) void paged_evict_select_kernel(int32_t* pos_pages, float* mass_pages, Pages pages, EvictGoal goal, int G,
                                                                           int32_t* __restrict__ counts, int2* __restrict__ moves)
{
    __shared__ uint32_t hist[256], sh[kEvictWaves], sh_prefix, sh_need;
    const int b = blockIdx.x / G, g = blockIdx.x % G, tid = threadIdx.x;
    const int n = goal.length(b, pages.slots()), gone = goal.victims(b, n), m = n - gone;
    if (gone == 0) {
        if (tid == 0) counts[blockIdx.x] = 0;
        return;
    }
    const int64_t recent = goal.protect_recent ? (int64_t)goal.seen_b[b] - goal.protect_recent : INT64_MAX;
    auto key_of = [&](int j) {
        const int id = pages.page_of(b, j);
        if (id < 0) return 0xffffffffu;
        const size_t at = pages.row(id, G, g, j);
        const int p = pos_pages ? pos_pages[at] : 0;
        return evict_key(mass_pages[at], pos_pages && (p < goal.protect_first || p >= recent));
    };
    // the gone-th smallest key, digit by digit
    uint32_t prefix = 0, need = gone;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kEvictThreads) {
            const uint32_t k = key_of(j);
            if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[k >> shift & 255], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            uint32_t d = 0;
            while (d < 255 && hist[d] < need) need -= hist[d++];
            sh_prefix = prefix | d << shift, sh_need = need;
        }
        __syncthreads();
        prefix = sh_prefix, need = sh_need;
    }
    // victims are the rows below that key and the first `need` rows that have it
    int2* list = moves + (size_t)blockIdx.x * goal.max_evict;
    uint32_t ties = 0, holes = 0, movers = 0;
    for (int j0 = 0; j0 < n; j0 += kEvictThreads) {
        const int j = j0 + tid;
        const uint32_t k = j < n ? key_of(j) : 0xffffffffu;
        const bool tie = j < n && k == prefix;
        uint32_t total;
        const uint32_t rank = ties + scan_block(tie, sh, total);
        ties += total;
        const bool victim = j < n && (k < prefix || (tie && rank < need));
        const bool hole = victim && j < m, mover = j < n && !victim && j >= m;
        const uint32_t at = scan_block((uint32_t)hole | (uint32_t)mover << 16, sh, total);
        if (hole) list[holes + (at & 0xffff)].x = j;
        if (mover) list[movers + (at >> 16)].y = j;
        holes += total & 0xffff, movers += total >> 16;
    }
    __threadfence_block();
    __syncthreads();
    holes = min(holes, movers);  // equal, unless masses change while they are read
    if (tid == 0) counts[blockIdx.x] = holes;
    for (int i = tid; i < (int)holes; i += kEvictThreads) {
        const int2 move = list[i];
        const int to = pages.page_of(b, move.x), from = pages.page_of(b, move.y);
        if (to < 0 || from < 0) continue;
        const size_t t = pages.row(to, G, g, move.x), f = pages.row(from, G, g, move.y);
        mass_pages[t] = mass_pages[f];
        if (pos_pages) pos_pages[t] = pos_pages[f];
    }
}

template <int CH>
__global__ __launch_bounds__(256) void paged_evict_move_kernel(u32x4* k_pages, u32x4* v_pages, Pages pages, int Hkv, int G, int max_evict,
                                                               const int32_t* __restrict__ counts, const int2* __restrict__ moves)
{
    constexpr int ROWS = 256 / CH;
    const int b = blockIdx.z, head = blockIdx.y >> 1, bg = b * G + (G > 1 ? head : 0), count = counts[bg];
    u32x4* rows = blockIdx.y & 1 ? v_pages : k_pages;
    const int2* list = moves + (size_t)bg * max_evict;
    for (int i = blockIdx.x * ROWS + threadIdx.x / CH; i < count; i += gridDim.x * ROWS) {
        const int2 move = list[i];
        const int to = pages.page_of(b, move.x), from = pages.page_of(b, move.y);
        if (to < 0 || from < 0) continue;
        rows[pages.row(to, Hkv, head, move.x) * CH + threadIdx.x % CH] = rows[pages.row(from, Hkv, head, move.y) * CH + threadIdx.x % CH];
    }
}

size_t paged_evict_ws(int B, int G, int max_evict)
{
    return (((size_t)B * G * 4 + 255) & ~(size_t)255) + (((size_t)B * G * max_evict * 8 + 255) & ~(size_t)255);
}

int paged_evict_dispatch(void* k_pages, void* v_pages, int32_t* pos_pages, float* mass_pages, const Pages& pages, const int32_t* len_b,
                         const int32_t* keep_b, const int32_t* seen_b, int B, int Hkv, int G, int row_bytes, int max_evict, int protect_first,
                         int protect_recent, void* ws, hipStream_t stream)
{
    int32_t* counts = static_cast<int32_t*>(ws);
    int2* moves = reinterpret_cast<int2*>(static_cast<char*>(ws) + (((size_t)B * G * 4 + 255) & ~(size_t)255));
    const EvictGoal goal{len_b, keep_b, seen_b, max_evict, protect_first, protect_recent};
    hipLaunchKernelGGL(paged_evict_select_kernel, dim3(B * G), dim3(kEvictThreads), 0, stream, pos_pages, mass_pages, pages, goal, G, counts, moves);
    if (const int rc = status_from_hip(hipGetLastError())) return rc;
    const int most = std::max(1, 4096 / (2 * Hkv * B));
#define EC_MOVE(CH_)                                                                                                                          \
    if (row_bytes == CH_ * 16)                                                                                                                \
        hipLaunchKernelGGL(paged_evict_move_kernel<CH_>, dim3(std::min((max_evict + 256 / CH_ - 1) / (256 / CH_), most), 2 * Hkv, B), dim3(256), 0, \
                           stream, (u32x4*)k_pages, (u32x4*)v_pages, pages, Hkv, G, max_evict, counts, moves)
    EC_MOVE(8);
    EC_MOVE(16);
    EC_MOVE(32);
#undef EC_MOVE
    return status_from_hip(hipGetLastError());
}

}  // namespace ec
