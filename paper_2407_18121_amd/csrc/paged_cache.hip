// ec_paged_store, ec_paged_evict_min: rows into the pages of their sequences, and rows out of them.
#include <algorithm>

#include "paged.h"

namespace ec {

// ------------------------------------------------------------------ store
// A workgroup takes kStoreRows rows of a (sequence, head), all its loads in flight; that of the first head takes positions and masses along. Bound: memory,
// at the rate of a plain copy (5.3 TB/s read and written at B16 H32 1024 .. 2048 rows; 4.97 without the non-temporal hints, 4.8 with 64 rows).
constexpr int kStoreRows = 32, kStoreGrid = 1 << 23;  // (a launch holds less than 2^32 threads in a dimension)
template <int CH>  // 16-byte chunks of a row
__global__ __launch_bounds__(256) void paged_store_kernel(const u32x4* __restrict__ k, const u32x4* __restrict__ v, const int32_t* __restrict__ pos,
                                                          const float* __restrict__ mass, Pages pages, const int32_t* __restrict__ start_b,
                                                          const int32_t* __restrict__ n_rows_b, int Hkv, int G, int base, int T, int src_rows,
                                                          u32x4* __restrict__ k_pages, u32x4* __restrict__ v_pages, int32_t* __restrict__ pos_pages,
                                                          float* __restrict__ mass_pages)
{
    constexpr int ROWS = 256 / CH, EACH = kStoreRows / ROWS;  // rows of a pass, passes
    const int b = blockIdx.z, head = blockIdx.y, r0 = base + blockIdx.x * kStoreRows;
    const int n = min(max(n_rows_b ? n_rows_b[b] : T, 0), T), start = start_b ? start_b[b] : 0;
    if (r0 >= n) return;
    auto page_at = [&](int r) {  // page of row r's slot, or -1
        const int64_t s = (int64_t)start + r;
        return r < n && s >= 0 && s < pages.slots() ? pages.page_of(b, (int)s) : -1;
    };
    if (k) {
        const int c = threadIdx.x % CH, first = r0 + threadIdx.x / CH;
        const u32x4 *from_k = k + ((size_t)b * Hkv + head) * src_rows * CH, *from_v = v + ((size_t)b * Hkv + head) * src_rows * CH;
        u32x4 x[EACH], y[EACH];
        int id[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const size_t at = (size_t)min(first + i * ROWS, n - 1) * CH + c;
            x[i] = __builtin_nontemporal_load(from_k + at), y[i] = __builtin_nontemporal_load(from_v + at), id[i] = page_at(first + i * ROWS);
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (id[i] >= 0) {
                const size_t to = pages.row(id[i], Hkv, head, start + first + i * ROWS) * CH + c;
                __builtin_nontemporal_store(x[i], k_pages + to), __builtin_nontemporal_store(y[i], v_pages + to);
            }
    }
    if (head == 0) {
        for (int i = threadIdx.x; i < kStoreRows * G; i += 256) {
            const int g = i / kStoreRows, r = r0 + i % kStoreRows, id = page_at(r);
            if (id < 0) continue;
            const size_t from = ((size_t)b * G + g) * src_rows + r, to = pages.row(id, G, g, start + r);
            if (pos) pos_pages[to] = pos[from];
            if (mass) mass_pages[to] = mass[from];
        }
    }
}

int paged_store_dispatch(const void* k, const void* v, const int32_t* pos, const float* mass, const Pages& pages, const int32_t* start_b,
                         const int32_t* n_rows_b, int B, int Hkv, int G, int T, int src_rows, int row_bytes, void* k_pages, void* v_pages,
                         int32_t* pos_pages, float* mass_pages, hipStream_t stream)
{
    const int chunks = (T - 1) / kStoreRows + 1;
    for (int chunk = 0; chunk < chunks; chunk += kStoreGrid) {  // (once, but for sources of more than 2^28 rows)
        const dim3 grid(std::min(chunks - chunk, kStoreGrid), k ? Hkv : 1, B);
#define EC_STORE(CH_)                                                                                                                     \
    if (row_bytes == CH_ * 16)                                                                                                            \
        hipLaunchKernelGGL(paged_store_kernel<CH_>, grid, dim3(256), 0, stream, (const u32x4*)k, (const u32x4*)v, pos, mass, pages, start_b, \
                           n_rows_b, Hkv, G, chunk * kStoreRows, T, src_rows, (u32x4*)k_pages, (u32x4*)v_pages, pos_pages, mass_pages)
        EC_STORE(8);
        EC_STORE(16);
        EC_STORE(32);
#undef EC_STORE
        if (const int rc = status_from_hip(hipGetLastError())) return rc;
    }
    return EC_OK;
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

constexpr uint32_t kProtected = 0xffffffffu;
// The order in which rows go, as an integer: fp32 order with -0 equal to +0, NaN behind +inf, protected rows (and rows on no page) last.
__device__ __forceinline__ uint32_t evict_key(float mass, bool kept)
{
    uint32_t u = __float_as_uint(mass);
    if (u == 0x80000000u) u = 0u;
    const uint32_t key = (u & 0x7fffffffu) > 0x7f800000u ? 0xfffffffeu : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return kept ? kProtected : key;
}

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave;
constexpr int kCopies = 8, kCopyWords = 264;
constexpr int kRun = 8;  // consecutive slots that a thread looks at: one page, one table entry, two 16-byte loads each of masses and positions

// What an eviction looks at in one (sequence, score group).
struct EvictRows {
    const int32_t* pos_pages;
    const float* mass_pages;
    const Pages& pages;
    int b, G, g, n, first;
    int64_t recent;
    __device__ __forceinline__ EvictRows(const int32_t* pos, const float* mass, const Pages& p, const EvictGoal& goal, int G_, int bg)
        : pos_pages(pos), mass_pages(mass), pages(p), b(bg / G_), G(G_), g(bg % G_), n(goal.length(b, p.slots())), first(goal.protect_first),
          recent(goal.protect_recent ? (int64_t)goal.seen_b[b] - goal.protect_recent : INT64_MAX)
    {
    }
    // Keys of RUNS runs of 8 slots, each `stride` behind the one before it, all their loads in flight; slots from n on get the largest key there is, like
    // protected ones. page[u]: the run's page or -1.
    template <int RUNS> __device__ __forceinline__ void keys(int j0, int stride, uint32_t (&key)[RUNS][kRun], int (&page)[RUNS]) const
    {
        u32x4 m[RUNS][2], p[RUNS][2] = {};
#pragma unroll
        for (int u = 0; u < RUNS; ++u) page[u] = j0 + u * stride < n ? pages.page_of(b, j0 + u * stride) : -1;
#pragma unroll
        for (int u = 0; u < RUNS; ++u) {
            const size_t at = pages.row(max(page[u], 0), G, g, j0 + u * stride);
            m[u][0] = reinterpret_cast<const u32x4*>(mass_pages + at)[0], m[u][1] = reinterpret_cast<const u32x4*>(mass_pages + at)[1];
            if (pos_pages) p[u][0] = reinterpret_cast<const u32x4*>(pos_pages + at)[0], p[u][1] = reinterpret_cast<const u32x4*>(pos_pages + at)[1];
        }
#pragma unroll
        for (int u = 0; u < RUNS; ++u)
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                const int where = (int)p[u][i / 4][i % 4];
                key[u][i] = evict_key(__uint_as_float(m[u][i / 4][i % 4]),
                                      page[u] < 0 || j0 + u * stride + i >= n || (pos_pages && (where < first || where >= recent)));
            }
    }
};

// The smallest, the largest over the wave's lanes.
template <bool LARGEST> __device__ __forceinline__ uint32_t wave_end(uint32_t x)
{
    constexpr int NONE = LARGEST ? 0 : -1;
    auto step = [&](uint32_t y) __attribute__((always_inline)) { x = LARGEST ? max(x, y) : min(x, y); };
    step(__builtin_amdgcn_update_dpp(NONE, (int)x, 0x111, 0xf, 0xf, false));  // (the lanes as in wave_scan)
    step(__builtin_amdgcn_update_dpp(NONE, (int)x, 0x112, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(NONE, (int)x, 0x114, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(NONE, (int)x, 0x118, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(NONE, (int)x, 0x142, 0xa, 0xf, false));
    step(__builtin_amdgcn_update_dpp(NONE, (int)x, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane((int)x, kWave - 1);
}
// The smallest (key, slot) over the wave's lanes.
__device__ __forceinline__ unsigned long long wave_least(unsigned long long x)
{
    const uint32_t hi = wave_end<false>((uint32_t)(x >> 32));
    return (unsigned long long)hi << 32 | wave_end<false>((uint32_t)(x >> 32) == hi ? (uint32_t)x : ~0u);
}

// Sum over the threads before this one, and the sum over all of them in `total`. `sh`: a place of its own for every call between two barriers.
template <int WAVES> __device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* sh, uint32_t& total)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const uint32_t in = wave_scan(x);
    if (lane == kWave - 1) sh[wave] = in;
    __syncthreads();
    const uint32_t sums = wave_scan(lane < WAVES ? sh[lane] : 0u);
    total = __builtin_amdgcn_readlane(sums, WAVES - 1);
    const uint32_t before = __builtin_amdgcn_readlane(sums, max(__builtin_amdgcn_readfirstlane(wave) - 1, 0));
    return (wave ? before : 0) + in - x;
}

// One workgroup per (sequence, score group): which rows go, and the list of moves. A thread holds runs of 8 consecutive slots. Sought is the gone-th
// smallest (key, slot): digit by digit, 8 bits at a time from the highest bit in which two keys differ (masses share their upper bits, and a histogram
// of those is one counter that all lanes wait for), until at most 64 rows share the digits found, which the waves rank, a share of the
// comparisons each (all in every wave: 1500 rows 8.2 us instead of 6.0). HELD: keys stay in registers, one, two or four
// runs a thread, up to 32768 rows (us of a call, held / read again for every digit: 12000 rows 15.6 / 26, 30000 rows 23 / 37); longer sequences are read again,
// a run at a time (70000 rows 96 us, with four in flight 110). Bound: a chain of latencies (length, table, masses, a barrier or two for each digit), for
// long ones by what one compute unit can read; 16 groups of 8192 rows 10 us.
template <int THREADS> struct SelectShared {
    __align__(16) uint32_t hist[4][kCopies][kCopyWords];  // a counter has a copy for every eighth lane, in banks of their own
    uint32_t sums[3][THREADS / kWave], lo[THREADS / kWave], hi[THREADS / kWave], ranks[kWave], n_few, slot;
    unsigned long long few[kWave];
};
template <int THREADS, int RUNS, bool HELD>
__device__ __forceinline__ void select_victims(const EvictRows& rows, int gone, int32_t* counts, uint2* list, SelectShared<THREADS>& sh)
{
    constexpr int WAVES = THREADS / kWave, STRIDE = THREADS * kRun;
    constexpr bool ONCE = HELD && RUNS == 1;  // a thread has one run: what its threads share is written once
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, n = rows.n, m = n - gone;
    uint32_t held[RUNS][kRun];
    int held_page[RUNS];
    if constexpr (HELD) rows.keys<RUNS>(tid * kRun, STRIDE, held, held_page);
    // f(first slot, keys, page) for every run of this thread
    auto each_run = [&](auto&& f) __attribute__((always_inline)) {
        if constexpr (HELD) {
#pragma unroll
            for (int u = 0; u < RUNS; ++u) f(tid * kRun + u * STRIDE, held[u], held_page[u]);
        } else {
            for (int j0 = 0; j0 < n; j0 += RUNS * STRIDE) {  // all threads in every round
                uint32_t key[RUNS][kRun];
                int page[RUNS];
                rows.keys<RUNS>(j0 + tid * kRun, STRIDE, key, page);
#pragma unroll
                for (int u = 0; u < RUNS; ++u) f(j0 + tid * kRun + u * STRIDE, key[u], page[u]);
            }
        }
    };
    auto& hist = sh.hist;
    auto& few = sh.few;
    auto& ranks = sh.ranks;
    for (int i = tid; i < (int)(sizeof(hist) / 16); i += THREADS) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
    if (tid < kWave) ranks[tid] = 0;
    if (tid == 0) sh.n_few = 0, sh.slot = 0;
    // how many rows are not protected, and the bits in which their keys differ
    uint32_t lo = kProtected, hi = 0, open = 0;
    each_run([&](int, uint32_t (&key)[kRun], int) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) lo = min(lo, key[i]), hi = max(hi, key[i] == kProtected ? 0u : key[i]), open += key[i] != kProtected;
    });
    lo = wave_end<false>(lo), hi = wave_end<true>(hi);
    if (lane == 0) sh.lo[wave] = lo, sh.hi[wave] = hi;
    uint32_t all_open;
    block_scan<WAVES>(open, sh.sums[0], all_open);
    lo = wave_end<false>(sh.lo[lane % WAVES]), hi = wave_end<true>(sh.hi[lane % WAVES]);

    // Victims are the rows up to `limit` in the order of (key, slot). Where only their key is known, last, and how many rows have it and go, need, the
    // slot is looked for behind.
    unsigned long long limit = (unsigned long long)(kProtected - 1) << 32 | 0xffffffffu;  // all that are not protected
    uint32_t last = kProtected, need = gone - min((uint32_t)gone, all_open);
    bool ties = need > 0;
    if ((uint32_t)gone < all_open) {
        int shift = lo == hi ? 0 : 32 - __clz(lo ^ hi);
        need = gone, ties = true;
        last = shift == 32 ? 0 : hi >> shift << shift;
        for (int pass = 0; shift > 0; ++pass) {
            const int bits = min(shift, 8), down = shift - bits;
            each_run([&](int, uint32_t (&key)[kRun], int) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < kRun; ++i)
                    if (key[i] != kProtected && ((uint64_t)(key[i] ^ last) >> shift) == 0)
                        atomicAdd(&hist[pass][lane % kCopies][key[i] >> down & ((1u << bits) - 1)], 1u);
            });
            __syncthreads();
            // every wave finds the digit for itself: four counters a lane
            uint4 c = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int copy = 0; copy < kCopies; ++copy) {
                const uint4 x = reinterpret_cast<const uint4*>(hist[pass][copy])[lane];
                c.x += x.x, c.y += x.y, c.z += x.z, c.w += x.w;
            }
            const uint32_t upto = wave_scan(c.x + c.y + c.z + c.w);
            const unsigned long long reached = __ballot(upto >= need);
            const int at = reached ? __ffsll(reached) - 1 : kWave - 1;  // (always, unless masses change while they are read)
            const uint32_t x = __builtin_amdgcn_readlane(c.x, at), y = __builtin_amdgcn_readlane(c.y, at), z = __builtin_amdgcn_readlane(c.z, at),
                           w = __builtin_amdgcn_readlane(c.w, at);
            need -= __builtin_amdgcn_readlane(upto, at) - (x + y + z + w);
            uint32_t digit = at * 4, count = x;
            if (need > count) {
                need -= count, ++digit, count = y;
                if (need > count) {
                    need -= count, ++digit, count = z;
                    if (need > count) need -= count, ++digit, count = w;
                }
            }
            last |= digit << down, shift = down;
            if (need == count) {  // all rows with these digits go
                ties = false;
                limit = (unsigned long long)min(last | ((1u << down) - 1), kProtected - 1) << 32 | 0xffffffffu;
                break;
            }
            if (count <= kWave) {  // few rows are left
                ties = false;
                each_run([&](int j, uint32_t (&key)[kRun], int) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < kRun; ++i)
                        if (key[i] != kProtected && ((uint64_t)(key[i] ^ last) >> down) == 0) {
                            const uint32_t to = atomicAdd(&sh.n_few, 1u);
                            if (to < kWave) few[to] = (unsigned long long)key[i] << 32 | (uint32_t)(j + i);
                        }
                });
                __syncthreads();
                const unsigned long long mine = few[lane];
                uint32_t smaller = 0;  // a wave's share
                for (uint32_t i = wave; i < count; i += WAVES) smaller += few[i] < mine;
                if (smaller) atomicAdd(&ranks[lane], smaller);
                __syncthreads();
                const unsigned long long found = __ballot((uint32_t)lane < count && ranks[lane] == need - 1);
                const int who = found ? __ffsll(found) - 1 : 0;
                limit = (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), who) << 32 |
                        (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, who);
                break;
            }
        }
    }
    if (ties) {  // the need-th row whose key is `last`
        uint32_t before = 0;
        each_run([&](int j, uint32_t (&key)[kRun], int) __attribute__((always_inline)) {
            uint32_t mine = 0, total;
#pragma unroll
            for (int i = 0; i < kRun; ++i) mine += j + i < n && key[i] == last;
            uint32_t rank = before + block_scan<WAVES>(mine, sh.sums[1], total);
            before += total;
#pragma unroll
            for (int i = 0; i < kRun; ++i)
                if (j + i < n && key[i] == last && ++rank == need) sh.slot = j + i;
            if constexpr (!ONCE) __syncthreads();
        });
        __syncthreads();
        limit = (unsigned long long)last << 32 | sh.slot;
    }

    uint32_t holes = 0, movers = 0;
    each_run([&](int j, uint32_t (&key)[kRun], int page) __attribute__((always_inline)) {
        uint32_t flags = 0, both = 0, total;  // bit i: a hole; bit 8 + i: a mover
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            const bool victim = ((unsigned long long)key[i] << 32 | (uint32_t)(j + i)) <= limit;
            const bool hole = victim && j + i < m, mover = !victim && j + i >= m && j + i < n;
            flags |= (uint32_t)hole << i | (uint32_t)mover << (8 + i);
            both += (uint32_t)hole | (uint32_t)mover << 16;
        }
        uint32_t at = block_scan<WAVES>(both, sh.sums[2], total);
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            const uint32_t row = page < 0 ? ~0u : ((uint32_t)page << rows.pages.shift) + ((j + i) & (rows.pages.page() - 1));
            const uint32_t to_hole = holes + (at & 0xffff), to_mover = movers + (at >> 16);
            if ((flags >> i & 1) && to_hole < (uint32_t)gone) list[to_hole].x = row;
            if ((flags >> (8 + i) & 1) && to_mover < (uint32_t)gone) list[to_mover].y = row;
            at += (flags >> i & 1) | (flags >> (8 + i) & 1) << 16;
        }
        holes += total & 0xffff, movers += total >> 16;
        if constexpr (!ONCE) __syncthreads();
    });
    if (tid == 0) *counts = min(min(holes, movers), (uint32_t)gone);  // equal, unless masses change while they are read
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void paged_evict_select_kernel(const int32_t* __restrict__ pos_pages, const float* __restrict__ mass_pages,
                                                                           Pages pages, EvictGoal goal, int G, int32_t* __restrict__ counts,
                                                                           uint2* __restrict__ moves)
{
    const EvictRows rows(pos_pages, mass_pages, pages, goal, G, blockIdx.x);
    const int gone = goal.victims(rows.b, rows.n);
    if (gone == 0) {
        if (threadIdx.x == 0) counts[blockIdx.x] = 0;
        return;
    }
    uint2* list = moves + (size_t)blockIdx.x * goal.max_evict;
    __shared__ SelectShared<THREADS> sh;
    int32_t* count = counts + blockIdx.x;
    if (THREADS < kEvictThreads || rows.n <= THREADS * kRun) select_victims<THREADS, 1, true>(rows, gone, count, list, sh);  // (fewer where the table ends before)
    else if (rows.n <= 2 * THREADS * kRun) select_victims<THREADS, 2, true>(rows, gone, count, list, sh);
    else if (rows.n <= 4 * THREADS * kRun) select_victims<THREADS, 4, true>(rows, gone, count, list, sh);
    else select_victims<THREADS, 1, false>(rows, gone, count, list, sh);
}

// A row number of the list (page and row in it) in a pool of `heads` heads.
__device__ __forceinline__ size_t pool_row(uint32_t row, const Pages& pages, int heads, int head)
{
    return pages.row(row >> pages.shift, heads, head, row);
}

// Moves: a workgroup takes 256 / CH rows of K or of V of a head at a time; K's of the group's first head take positions and masses along. Bound: memory.
// (B16 H32 8192 -> 820 rows, selection included, us: 103; with non-temporal stores 96; a row a thread instead of four in flight 93.)
template <int CH>
__global__ __launch_bounds__(256) void paged_evict_move_kernel(u32x4* k_pages, u32x4* v_pages, int32_t* pos_pages, float* mass_pages, Pages pages,
                                                               int Hkv, int G, int max_evict, const int32_t* __restrict__ counts,
                                                               const uint2* __restrict__ moves)
{
    constexpr int ROWS = 256 / CH;
    const int b = blockIdx.z, head = blockIdx.y >> 1, g = G > 1 ? head : 0, count = counts[b * G + g];
    const bool tells = !(blockIdx.y & 1) && (G > 1 || head == 0);
    u32x4* rows = blockIdx.y & 1 ? v_pages : k_pages;
    const uint2* list = moves + (size_t)(b * G + g) * max_evict;
    const int sub = threadIdx.x % CH;
    for (int i = blockIdx.x * ROWS + threadIdx.x / CH; i < count; i += gridDim.x * ROWS) {
        const uint2 move = list[i];
        if (move.x == ~0u || move.y == ~0u) continue;  // on no page
        const u32x4 x = __builtin_nontemporal_load(rows + pool_row(move.y, pages, Hkv, head) * CH + sub);
        if (tells && sub == 0) {
            const size_t to = pool_row(move.x, pages, G, g), from = pool_row(move.y, pages, G, g);
            mass_pages[to] = mass_pages[from];
            if (pos_pages) pos_pages[to] = pos_pages[from];
        }
        __builtin_nontemporal_store(x, rows + pool_row(move.x, pages, Hkv, head) * CH + sub);
    }
}

// The least (key, slot) of those a thread has seen, and its page.
struct Least {
    unsigned long long of = ~0ull;
    int page = -1;
    __device__ __forceinline__ void look(const EvictRows& rows, int from, int step)
    {
        for (int j = from; j < rows.n; j += step) {
            uint32_t key[1][kRun];
            int id[1];
            rows.keys<1>(j, 0, key, id);
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                const unsigned long long x = (unsigned long long)key[0][i] << 32 | (uint32_t)(j + i);
                if (j + i < rows.n && x < of) of = x, page = id[0];
            }
        }
    }
    // That of the workgroup, for every thread. The shared words are written once.
    __device__ __forceinline__ void of_all(unsigned long long* sh_of, int* sh_page)
    {
        const unsigned long long mine = of;
        of = wave_least(of);
        if (threadIdx.x % kWave == 0) sh_of[threadIdx.x / kWave] = of;
        __syncthreads();
        of = wave_least(sh_of[threadIdx.x % kEvictWaves]);
        if (mine == of) *sh_page = page;  // one thread's: slots differ (several, where nobody has a row)
        __syncthreads();
        page = *sh_page;
    }
};

// Long sequences, whose masses one compute unit is slow to read: the least row of each part, a workgroup a part, in a launch before (us of a call, one launch /
// two: one sequence of 16300 rows 7.6 / 8.1, 24000 9.2 / 8.1, 131000 33 / 8.2; 16 of 16300 8.1 / 8.5, 24000 10.7 / 8.8). The host knows
// the tables' room only: short sequences in long tables pay for the launch (640 rows 4.1 / 6.2, 16 of 640 4.5 / 6.9, one of 8000 5.2 / 7.2).
constexpr int kOneParts = 64, kOneAlone = 16384;  // slots up to which the workgroup that fills the hole looks through them all
struct Candidate {
    unsigned long long of;
    int page, unused;
};
__global__ __launch_bounds__(kEvictThreads) void paged_evict_least_kernel(const int32_t* __restrict__ pos_pages, const float* __restrict__ mass_pages, Pages pages,
                                                                          EvictGoal goal, int G, Candidate* __restrict__ candidates)
{
    __shared__ unsigned long long sh_of[kEvictWaves];
    __shared__ int sh_page;
    const EvictRows rows(pos_pages, mass_pages, pages, goal, G, blockIdx.y);
    if (goal.victims(rows.b, rows.n) == 0) return;
    Least least;
    least.look(rows, (blockIdx.x * kEvictThreads + threadIdx.x) * kRun, gridDim.x * kEvictThreads * kRun);
    least.of_all(sh_of, &sh_page);
    if (threadIdx.x == 0) candidates[blockIdx.y * kOneParts + blockIdx.x] = {least.of, least.page, 0};
}

// One row of every sequence, the step of a generation loop: the workgroup that finds the least row fills its place. Only the last row can be
// the one that moves, so it is fetched while the least one is sought; what is left of the chain is length, table, masses, the reduction and the store.
template <int CH, bool PARTS>
__global__ __launch_bounds__(kEvictThreads) void paged_evict_one_kernel(u32x4* k_pages, u32x4* v_pages, int32_t* pos_pages, float* mass_pages, Pages pages,
                                                                        EvictGoal goal, int Hkv, int G, const Candidate* __restrict__ candidates, int parts)
{
    constexpr int HELD = 3;  // chunks of a thread that are fetched early: 48 heads of 512 bytes
    __shared__ unsigned long long sh_best[kEvictWaves];
    __shared__ int sh_page;
    const EvictRows rows(pos_pages, mass_pages, pages, goal, G, blockIdx.x);
    const int n = rows.n, b = rows.b, tid = threadIdx.x;
    if (goal.victims(b, n) == 0) return;
    const int from = pages.page_of(b, n - 1);
    const int heads = G > 1 ? 1 : Hkv, head0 = G > 1 ? rows.g : 0, chunks = heads * 2 * CH;
    auto place = [&](int i, int id, int slot) {  // chunk i of the heads' K and V rows in a slot
        return (i / CH & 1 ? v_pages : k_pages) + pages.row(id, Hkv, head0 + i / (2 * CH), slot) * CH + i % CH;
    };
    Least least;
    if constexpr (PARTS) {
        if (tid < parts) {
            const Candidate c = candidates[blockIdx.x * kOneParts + tid];
            least.of = c.of, least.page = c.page;
        }
    } else {
        least.look(rows, tid * kRun, kEvictThreads * kRun);
    }
    u32x4 row[HELD];
    float mass = 0.f;
    int pos = 0;
    if (from >= 0) {
#pragma unroll
        for (int u = 0; u < HELD; ++u)
            if (tid + u * kEvictThreads < chunks) row[u] = *place(tid + u * kEvictThreads, from, n - 1);
        mass = mass_pages[pages.row(from, G, rows.g, n - 1)];
        if (pos_pages) pos = pos_pages[pages.row(from, G, rows.g, n - 1)];
    }
    least.of_all(sh_best, &sh_page);
    const int hole = (int)(uint32_t)least.of, to = least.page;
    if (hole == n - 1 || to < 0 || from < 0) return;
#pragma unroll
    for (int u = 0; u < HELD; ++u)
        if (tid + u * kEvictThreads < chunks) *place(tid + u * kEvictThreads, to, hole) = row[u];
    for (int i = tid + HELD * kEvictThreads; i < chunks; i += kEvictThreads) *place(i, to, hole) = *place(i, from, n - 1);
    if (tid == 0) {
        mass_pages[pages.row(to, G, rows.g, hole)] = mass;
        if (pos_pages) pos_pages[pages.row(to, G, rows.g, hole)] = pos;
    }
}

// Enough for every smaller max_evict too: the candidates of one row take more than short lists.
size_t paged_evict_ws(int B, int G, int max_evict)
{
    const size_t lists = (((size_t)B * G * 4 + 255) & ~(size_t)255) + (((size_t)B * G * max_evict * 8 + 255) & ~(size_t)255);
    return std::max(lists, (size_t)B * G * kOneParts * sizeof(Candidate));
}

int paged_evict_dispatch(void* k_pages, void* v_pages, int32_t* pos_pages, float* mass_pages, const Pages& pages, const int32_t* len_b,
                         const int32_t* keep_b, const int32_t* seen_b, int B, int Hkv, int G, int row_bytes, int max_evict, int protect_first,
                         int protect_recent, void* ws, hipStream_t stream)
{
    int32_t* counts = static_cast<int32_t*>(ws);
    uint2* moves = reinterpret_cast<uint2*>(static_cast<char*>(ws) + (((size_t)B * G * 4 + 255) & ~(size_t)255));
    const EvictGoal goal{len_b, keep_b, seen_b, max_evict, protect_first, protect_recent};
    u32x4 *k = static_cast<u32x4*>(k_pages), *v = static_cast<u32x4*>(v_pages);
    if (max_evict == 1) {
        Candidate* candidates = static_cast<Candidate*>(ws);
        const int slots = pages.slots(), parts = slots > kOneAlone ? std::min((slots + kEvictThreads * kRun - 1) / (kEvictThreads * kRun), kOneParts) : 0;
        if (parts) {
            hipLaunchKernelGGL(paged_evict_least_kernel, dim3(parts, B * G), dim3(kEvictThreads), 0, stream, pos_pages, mass_pages, pages, goal, G, candidates);
            if (const int rc = status_from_hip(hipGetLastError())) return rc;
        }
#define EC_ONE(CH_, PARTS_)                           \
    if (row_bytes == CH_ * 16 && (parts > 0) == PARTS_) \
        hipLaunchKernelGGL((paged_evict_one_kernel<CH_, PARTS_>), dim3(B * G), dim3(kEvictThreads), 0, stream, k, v, pos_pages, mass_pages, pages, goal, Hkv, G, candidates, parts)
        EC_ONE(8, false);
        EC_ONE(16, false);
        EC_ONE(32, false);
        EC_ONE(8, true);
        EC_ONE(16, true);
        EC_ONE(32, true);
#undef EC_ONE
        return status_from_hip(hipGetLastError());
    }
    // Threads for the rows that the tables have room for: fewer waves do less twice and meet sooner (us of a call that moves few bytes, 640 rows 6.4 with
    // 1024 threads and 5.6 with 256, 24 groups of 3001 9.9 and with 512 8.9).
    const int threads = pages.slots() <= 256 * kRun ? 256 : pages.slots() <= 512 * kRun ? 512 : kEvictThreads;
#define EC_SELECT(THREADS_)   \
    if (threads == THREADS_)  \
        hipLaunchKernelGGL(paged_evict_select_kernel<THREADS_>, dim3(B * G), dim3(THREADS_), 0, stream, pos_pages, mass_pages, pages, goal, G, counts, moves)
    EC_SELECT(256);
    EC_SELECT(512);
    EC_SELECT(kEvictThreads);
#undef EC_SELECT
    if (const int rc = status_from_hip(hipGetLastError())) return rc;
    const int most = std::max(1, 8192 / (2 * Hkv * B));  // the lists' lengths are on the device: workgroups go over them
#define EC_MOVE(CH_)                                                                                                                             \
    if (row_bytes == CH_ * 16)                                                                                                                   \
        hipLaunchKernelGGL(paged_evict_move_kernel<CH_>, dim3(std::min((max_evict + 256 / CH_ - 1) / (256 / CH_), most), 2 * Hkv, B), dim3(256), 0, stream, k, v, \
                           pos_pages, mass_pages, pages, Hkv, G, max_evict, counts, moves)
    EC_MOVE(8);
    EC_MOVE(16);
    EC_MOVE(32);
#undef EC_MOVE
    return status_from_hip(hipGetLastError());
}

}  // namespace ec
