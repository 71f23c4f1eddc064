// ec_paged_decode_step, ec_paged_decode_score_step: attention of one new token per sequence over a cache in pages.
//
// The rows of one (sequence, key/value head, up to 16 of its query heads), a pair, are cut into segments, one workgroup each.  A wave takes every
// WAVES-th tile of a segment's rows and keeps a running (maximum, sum, weighted V) for its 16 query heads:
//   S^T = K . Q^T      matrix instructions, so that a lane owns one query head and 4 consecutive rows of a block of 16
//   O^T += V^T . P^T   the probabilities are the second operand as they stand; V is transposed on its way out of LDS (bf16)
// Every row of K and V is read once for all query heads of its head, straight from its page into LDS; a tile is in flight while the
// one before it is used.  The new row takes part as the last row of the last tile and is stored by that tile's workgroup.
// The segments' results meet by the rule of the softmax: with M the largest of their maxima m_i, out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i.
//
// Bound by the bytes of the rows, of which the counters see 1.002 .. 1.003 times what has to be read (a large copy on this card moves 5.0 .. 5.5 TB/s):
//   bf16 D128 B16 H32/32 870 rows 39.6 us, 5.8 TB/s; one cache of 131071 rows, H40/8 89.2, 6.0; fp32 B8 H32/32 1000 rows 47.7, 5.5.
// Short caches by a chain of latencies, 8 us of B1 H32/32 640 rows: lengths and pages 0.6, first rows 1.1, a tile 0.8 and 0.5 for each further one,
// the waves' results 1.0, the ticket 0.5, the other segments' results 2.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "paged.h"
#include "tile_lds.h"

namespace ec {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
typedef __attribute__((address_space(4))) const int32_t const_i32;  // read through the scalar cache: nothing that a launch writes

constexpr int kPagedWaves = 4;         // with 2: 41.1, one long cache 110 us
constexpr int kPagedSegments = 256;  // workgroups that a launch of few pairs aims at: one a compute unit
constexpr int kWholeRounds = 3;       // a pair of so many rounds is not cut: 60, 120 rows of one sequence, H32 5.4, 5.9 us a step, joined 7.9
constexpr int kLengths = 1024;        // of a batch that are held in LDS
constexpr int kMostSegments = 256;   // of a pair, whose weights have to fit into LDS when they are joined
constexpr int kHeadBlock = 16;       // query heads of a pair, at most
constexpr float kSmallExponent = -100.f, kSmall = 0x1p-100f;  // probabilities below it are looked at apart

// The scale in base-2 units, log2(e) * scale. fp32: q takes all of it. bf16: q takes the power of two, 2^exponent, that leaves 1 .. 2 for the
// differences of scores, so that no sum leaves the range that the score itself stays in.
struct PagedScale {
    float whole, of_diff;
    int exponent;
};
static PagedScale paged_scale(float scale, int dt)
{
    const float log2 = scale * kLog2e;
    if (dt == EC_F32) return {log2, 1.f, 0};
    int n;
    const float rest = std::frexp(log2, &n);  // 0.5 .. 1
    return {log2, 2.f * rest, n - 1};
}

struct PagedStep {
    const void *q, *k_new, *v_new;
    void *k_pages, *v_pages, *out;
    int32_t* pos_pages;
    const int32_t *len_b, *new_pos_b;
    Pages pages;
    int B, H, Hkv, G;
    int group, blocks;             // query heads of a key/value head, and pairs that they make
    PagedScale scale;
    float *raw, *stats;            // of a step with masses: [B,H,slots] scores in base-2 units, [B,H,2] softmax maximum and 1 / denominator
    float* mass_pages;
    unsigned int* group_tickets;   // kMasses, of the (sequence, score group)s; zeros before and after
    unsigned int* tickets;         // of the pairs with several segments, by their first one's number; zeros before and after
    unsigned long long* partials;  // of the segments of such pairs
};

// N load instructions of consecutive rows into consecutive LDS (see load_lds_16): the instruction's offset moves both by 1 KB. The non-temporal hint
// keeps data that is read once from displacing cache lines (B16 H32 870 rows 39.0 us a step, 44.1 without; one cache of 131071 rows 89.3, 100.5).
template <int N> __device__ __forceinline__ void load_run_lds(u32x4 rsrc, uint32_t lds, const uint32_t* offset)
{
    if constexpr (N == 1)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(offset[0]), "s"(rsrc) : "memory");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %3, 0 offen nt lds\n\t"
                     "buffer_load_dwordx4 %2, %3, 0 offen offset:1024 nt lds" ::"s"(lds), "v"(offset[0]), "v"(offset[1]), "s"(rsrc) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %5, 0 offen nt lds\n\t"
                     "buffer_load_dwordx4 %2, %5, 0 offen offset:1024 nt lds\n\tbuffer_load_dwordx4 %3, %5, 0 offen offset:2048 nt lds\n\t"
                     "buffer_load_dwordx4 %4, %5, 0 offen offset:%6 nt lds"
                     ::"s"(lds), "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "s"(rsrc), "n"(3 * 1024) : "memory");
}

template <int DT, int D> struct PagedTile {
    static constexpr bool kHalf = DT == EC_BF16;
    static constexpr int kRowBytes = D * Elem<DT>::kBytes;
    static constexpr int CH = kRowBytes / 16;      // 16-byte chunks of a row
    static constexpr int RPI = kWave / CH;         // rows of a load instruction
    // Rows of a tile: 32 KB of tiles a wave and more leave a compute unit one workgroup (B16 H32 D128 870 rows 39.0 us with 16, 44.2 with 32); shorter
    // rows have the room, and 32 of them fill the matrix instruction of 32 (B8 H32 D64 1000 rows 15.4 us, 16.6 with 16)
    static constexpr int TR = kHalf && D < 128 ? 32 : 16;
    static constexpr int GROUPS = TR / 8;          // runs of 8 rows, which lie in one page
    static constexpr int IPG = 8 / RPI;            // load instructions of a run
    static constexpr int NI = GROUPS * IPG;        // of a tile of K or V
    static constexpr int BYTES = TR * kRowBytes;
    static constexpr int kResident = kPagedWaves * 4 * BYTES <= 65536 ? 2 : 1;  // workgroups that a compute unit has the LDS for
    // chunk c of row r lies at place c ^ swizzle(r): reads of 16 rows at one chunk number (K), of two chunks of 16 rows (V, bf16) and of
    // whole rows (V, fp32) meet all banks alike
    static __device__ __forceinline__ int swz_k(int r) { return CH >= 16 ? r & 15 : r >> 1 & 7; }
    static __device__ __forceinline__ int swz_v(int r) { return !kHalf ? 0 : CH >= 16 ? (r & 7) << 1 : (r >> 1 & 3) << 1; }
};

__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, kWave - 1); }

// The maximum, the sum over the lanes that share a query head (l % 16); all four get it.
__device__ __forceinline__ float head_max(float x)
{
    auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
    y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float head_sum(float x)
{
    auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

// Which segment a workgroup takes. A sequence of N rows (the new one included) has rounds of ROUND rows; a segment is at most `most` rounds
// of a pair, `most` such that a batch of few pairs has kPagedSegments segments: long sequences are cut, short ones are not. Every wave finds its
// segment for itself, a lane per sequence: no exchange between waves.
struct Segment {
    int b, n, pair, first, last, count;  // rounds first .. last-1 of the pair, which has `count` segments; b < 0: none
    int split;                           // number of the segment among those of cut pairs
    int split0;                          // and of its pair's first one
};
__device__ __forceinline__ int divided(int x, int by)  // 0 <= x < 2^24, by > 0
{
    const int q = (int)((float)x * __builtin_amdgcn_rcpf((float)by)), r = x - q * by;
    return q + (r >= by) - (r < 0);
}
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Segment segment_of(int b, int n, int pair, int seg, int rounds, int count, int split0)
{
    const int each = scalar(divided(rounds, count)), more = rounds - each * count;  // the first `more` segments have a round more
    const int first = seg * each + min(seg, more);
    return {b, n, pair, first, first + each + (seg < more), count, split0 + seg, split0};
}
// Segments that a pair of so many rounds is cut into at most. A few rounds are not cut, others as far as one round each while there are few of them (us a
// step, against segments of three rounds at least: two sequences, H8/2, fp32 D64, 374 rows 7.4 / 9.0, 758 8.3 / 9.0; bf16 D128 374 rows 8.1 / 9.5; with
// segments of one round everywhere 2550 rows 10.8, now 10.1).
__device__ __forceinline__ int most_segments(int rounds)
{
    return rounds <= kWholeRounds ? min(rounds, 1) : min(min(rounds, max(rounds / 2, 16)), kMostSegments);
}
template <int ROUND> __device__ __forceinline__ Segment find_segment(const int32_t* __restrict__ len_b, int B, int pairs, int slots, int id, int* sh_len)
{
    const int lane = threadIdx.x % kWave;
    if (B == 1) {  // nothing to look through
        const int n = ((const const_i32*)(uintptr_t)len_b)[0];
        const bool live = n >= 0 && n < slots;
        const int rounds = live ? n / ROUND + 1 : 1, count = min(max(scalar(divided(kPagedSegments, pairs)), 1), most_segments(rounds));
        const int seg = scalar(divided(id, pairs));
        if (seg >= count) return {-1, 0, 0, 0, 0, 0, 0, 0};
        const int pair = id - seg * pairs;
        return segment_of(0, live ? n : -1, pair, seg, rounds, count, pair * count);
    }
    // rows before the step, or -1 for a place without a sequence, which has one round all the same (somebody has to write its zeros)
    const bool kept = B > kWave && B <= kLengths;  // in LDS, as every wave looks through them twice
    auto rows = [&](int b) {
        const int n = b >= B ? -1 : kept ? sh_len[b] : len_b[b];
        return n >= 0 && n < slots ? n : -1;
    };
    if (kept) {
        for (int i = threadIdx.x; i < B; i += blockDim.x) sh_len[i] = len_b[i];
        __syncthreads();
    }
    auto rounds_of = [&](int b, int n) { return b >= B ? 0 : n < 0 ? 1 : n / ROUND + 1; };
    // (loops over scalars, so that all lanes are there for what passes between lanes)
    int n = -1;
    long long all = 0;
    for (int b0 = 0; b0 < B; b0 += kWave) {
        n = rows(b0 + lane);
        all += last_lane(wave_scan(rounds_of(b0 + lane, n)));
    }
    int most = (int)((all * pairs + kPagedSegments - 1) / kPagedSegments);
    // Sequences of different lengths that are cut into two or not at all leave some compute units with much and others with little: twice as many
    // segments there, as many as the chip holds at once (us a step, 256 about / 512 at most: 192 pairs of 1450 .. 2900 rows 52.0 / 45.8, 128 of 750 ..
    // 1500 22.2 / 18.8; pairs that are cut further, one length and single sequences gain nothing, and joining takes longer: 64 pairs of 2000 .. 4000 rows
    // 19.6 / 21.6, 8 of 131071 91 / 98).
    if (B <= kWave && most >= 8 && B * pairs > kPagedSegments / 3 && B * pairs <= 2 * kPagedSegments &&
        wave_max((float)rounds_of(lane, n)) * B > 1.125f * all) {
        most = (int)((all * pairs + 2 * kPagedSegments - 1) / (2 * kPagedSegments));
        while (last_lane(wave_scan(divided(rounds_of(lane, n) + most - 1, most))) * pairs > 2 * kPagedSegments) most += (most + 7) / 8;
    }
    int before = 0, cut = 0;
    for (int b0 = 0; b0 < B; b0 += kWave) {
        if (B > kWave) n = rows(b0 + lane);
        const int rounds = rounds_of(b0 + lane, n), count = min(divided(rounds + most - 1, most), most_segments(rounds));
        const int upto = wave_scan(count), cut_upto = wave_scan(count > 1 ? count : 0);
        const unsigned long long beyond = __ballot(id < before + upto * pairs);
        if (beyond) {
            const int at = __ffsll(beyond) - 1;
            const int c = __builtin_amdgcn_readlane(count, at);
            const int in = id - before - (__builtin_amdgcn_readlane(upto, at) - c) * pairs;  // number among the sequence's segments
            const int pair = scalar(divided(in, c));
            const int split0 = cut + (c > 1 ? (__builtin_amdgcn_readlane(cut_upto, at) - c) * pairs + pair * c : 0);
            return segment_of(b0 + at, __builtin_amdgcn_readlane(n, at), pair, in - pair * c, __builtin_amdgcn_readlane(rounds, at), c, split0);
        }
        before += last_lane(upto) * pairs, cut += last_lane(cut_upto) * pairs;
    }
    return {-1, 0, 0, 0, 0, 0, 0, 0};
}

constexpr int kDeviceScope = 16;  // of a buffer load
// Partial results pass between workgroups at device scope: written through and read past the caches, no fence.
__device__ __forceinline__ void put(unsigned long long* p, float x, float y)
{
    __hip_atomic_store(p, (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// What becomes of the scores: nothing; they are stored, and paged_mass_kernel adds up the masses; the last workgroup of a (sequence, score group) does.
enum { kNoScores, kScores, kMasses };
constexpr int kMassAhead = 8;  // reads in flight of a thread that adds up masses (kMasses: twice)
// What a kMasses launch takes at most: of a group pairs, slots and scores; groups of several pairs, which have tickets. It saves the host a launch, 2.5 us, and
// takes about as long (us a step, two launches / one: B1 H32/8, eight groups, 250 rows 10.7 / 10.4, 1000 11.4 / 12.1; B32 likewise 14.2 / 13.3, 34.8 / 31.2;
// B2 H8/2, one group, fp32 D64, 60 rows 8.25 / 8.2, 500 10.5 / 11.1). The scores come from beyond the caches, which one workgroup is slow at (B1
// H32, one group, 500 rows 11.9 / 13.4, 2000 rows 15 / 25), and so are many pairs at one ticket (B16 H32, one group, 60 rows 11.8 / 16.1).
constexpr int kMassPairs = 4, kMassSlots = 2048, kMassScores = 4096, kMassGroups = 512;
constexpr int kMassHeads = kMassScores / 8;  // a sequence has 8 slots at least
// 2^x; the exponential instruction gives zero where the result is subnormal, exp2f does not
__device__ __forceinline__ void weights_of(f32x4& x)
{
    const float least = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
    f32x4 p;
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(x[e]);
    if (__builtin_expect(__any(least < kSmallExponent), 0)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = exp2f(x[e]);
    }
    x = p;
}
template <int DT, int D, int EMIT>
__global__ __launch_bounds__(kPagedWaves* kWave, (PagedTile<DT, D>::kResident)) void paged_step_kernel(PagedStep a)
{
    using T = PagedTile<DT, D>;
    constexpr int WAVES = kPagedWaves, TR = T::TR, ROW = T::kRowBytes, CH = T::CH, RPI = T::RPI, NI = T::NI, ROUND = WAVES * TR;
    constexpr int KB = ROW / 64;      // 64-byte blocks of a row: what the four quarters of a wave contract together
    constexpr int OB = D / 16;        // 16-feature blocks of the output
    constexpr int PART = kHeadBlock * (D / 2 + 1);  // 8-byte words of a segment's result: (maximum, sum) of every head, then the sums
    constexpr int OROW = D + 4;       // floats of a head's sums in LDS, padded
    static_assert(kHeadBlock * OROW * 4 <= 4 * T::BYTES, "a wave's sums fit into its tiles");
    static_assert(T::TR == 16 || T::TR == 32);
    __shared__ __align__(256) unsigned char tiles[WAVES][4 * T::BYTES];  // of every wave: two tiles of K, two of V
    __shared__ float sh_m[WAVES][kHeadBlock], sh_l[WAVES][kHeadBlock];
    __shared__ unsigned int sh_ticket;
    __shared__ int sh_len[kLengths];

    const int slots = a.pages.slots();
    const Segment at = find_segment<ROUND>(a.len_b, a.B, a.Hkv * a.blocks, slots, blockIdx.x, sh_len);
    if (at.b < 0) return;
    const int hk = a.blocks == 1 ? at.pair : at.pair / a.blocks, block = at.pair - hk * a.blocks, heads = min(a.group - block * kHeadBlock, kHeadBlock);
    const int head0 = hk * a.group + block * kHeadBlock;  // first query head
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int c16 = lane % 16, quarter = lane / 16;
    const size_t out_at = ((size_t)at.b * a.H + head0) * D;  // element
    if (at.n < 0) {  // no sequence in this place
        for (int i = tid; i < heads * D; i += WAVES * kWave) {
            if constexpr (T::kHalf) static_cast<uint16_t*>(a.out)[out_at + i] = 0;
            else static_cast<float*>(a.out)[out_at + i] = 0.f;
        }
        return;
    }
    const int n = at.n;  // the new row's number
    const char* k_new = static_cast<const char*>(a.k_new) + ((size_t)at.b * a.Hkv + hk) * ROW;
    const char* v_new = static_cast<const char*>(a.v_new) + ((size_t)at.b * a.Hkv + hk) * ROW;

    // what storing the new row takes, asked for early: its page, its position, its chunk of this lane (the first CH lanes have one)
    const const_i32* table = (const const_i32*)(uintptr_t)(a.pages.table + (size_t)at.b * a.pages.max_pages);
    const int new_page = table[n >> a.pages.shift], new_pos = a.pos_pages ? ((const const_i32*)(uintptr_t)a.new_pos_b)[at.b] : 0;
    const u32x4 new_k = reinterpret_cast<const u32x4*>(k_new)[lane % CH], new_v = reinterpret_cast<const u32x4*>(v_new)[lane % CH];

    // ------------------------------------------------------------------ rows into LDS
    const uint32_t mine = __builtin_amdgcn_readfirstlane(lds_address(tiles[wave]));
    const int shift = a.pages.shift, mask = (1 << shift) - 1, end = min(n, at.last * ROUND);  // rows of the cache in the segment end there
    uint32_t k_part[2][T::IPG], v_part[T::IPG];  // a lane's place in the rows of a load instruction, K: of even and odd runs
#pragma unroll
    for (int i = 0; i < T::IPG; ++i) {
        const int r = i * RPI + lane / CH;
        k_part[0][i] = lane / CH * ROW + (lane % CH ^ T::swz_k(r)) * 16;
        k_part[1][i] = lane / CH * ROW + (lane % CH ^ T::swz_k(r + 8)) * 16;
        v_part[i] = lane / CH * ROW + (lane % CH ^ T::swz_v(r)) * 16;
    }
    // Where the runs of a tile lie in the pools, and how many bytes of them are there: none behind the segment or on no page, and what is not
    // there becomes zeros in LDS. A run in the page of the one before it needs no table entry.
    struct Ids {
        int id[T::GROUPS];
    };
    const int page_rows = 1 << shift;
    auto pages_of = [&](int row) __attribute__((always_inline)) {
        Ids ids;
#pragma unroll
        for (int u = 0; u < T::GROUPS; ++u)
            if (u == 0 || u * 8 % page_rows == 0) ids.id[u] = table[min((row + u * 8) >> shift, a.pages.max_pages - 1)];
        return ids;
    };
    struct Places {
        size_t from[T::GROUPS];
        int bytes[T::GROUPS], bad;  // bit u: run u has rows, but no page
    };
    const uint32_t head_bytes = (uint32_t)ROW << shift, page_bytes = head_bytes * (uint32_t)a.Hkv;
    auto places_of = [&](int row, const Ids& ids) __attribute__((always_inline)) {
        Places pl;
        pl.bad = 0;
        bool page = false;
#pragma unroll
        for (int u = 0; u < T::GROUPS; ++u) {
            const int r = row + u * 8, left = end - r;
            if (u == 0 || u * 8 % page_rows == 0) {
                page = (unsigned)ids.id[u] < (unsigned)a.pages.n_pages;
                pl.from[u] = (size_t)(uint32_t)(page ? ids.id[u] : 0) * page_bytes + (hk * head_bytes + (uint32_t)(r & mask) * ROW);
            } else {
                pl.from[u] = pl.from[u ? u - 1 : 0] + 8 * ROW;
            }
            pl.bytes[u] = page ? max(min(left, 8), 0) * ROW : 0;
            pl.bad |= page || left <= 0 ? 0 : 1 << u;
        }
        return pl;
    };
    auto issue_k = [&](uint32_t lds, const Places& pl) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < T::GROUPS; ++u)
            load_run_lds<T::IPG>(tile_rsrc(static_cast<const char*>(a.k_pages) + pl.from[u], pl.bytes[u]), lds + u * 8 * ROW, k_part[u & 1]);
    };
    auto issue_v = [&](uint32_t lds, const Places& pl) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < T::GROUPS; ++u)
            load_run_lds<T::IPG>(tile_rsrc(static_cast<const char*>(a.v_pages) + pl.from[u], pl.bytes[u]), lds + u * 8 * ROW, v_part);
    };
    auto issue_q = [&](uint32_t lds) __attribute__((always_inline)) {  // rows of queries like rows of K; zeros for heads that do not exist
        const char* q = static_cast<const char*>(a.q) + out_at * Elem<DT>::kBytes;
#pragma unroll
        for (int u = 0; u < kHeadBlock / 8; ++u)
            load_run_lds<T::IPG>(tile_rsrc(q + u * 8 * ROW, max(heads - u * 8, 0) * ROW), lds + u * 8 * ROW, k_part[u & 1]);
    };
    // the new row, where the tile has it: into the place that its loads left at zero
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    auto add_new = [&](uint32_t off, int row) __attribute__((always_inline)) {
        const int r = n - row;
        if (r >= 0 && r < TR) {
            if (lane < CH) {
                *(lds_u32x4*)(uintptr_t)(mine + off + r * ROW + (lane ^ T::swz_k(r)) * 16) = new_k;
                *(lds_u32x4*)(uintptr_t)(mine + 2 * T::BYTES + off + r * ROW + (lane ^ T::swz_v(r)) * 16) = new_v;
            }
            wait_lds();
        }
    };

    // ------------------------------------------------------------------ one tile after the other
    f32x4 o[OB];
#pragma unroll
    for (int i = 0; i < OB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kLowest, l = 0.f;  // l: of this lane's rows
    u32x4 qf[KB];                // this lane's head, chunks 4 kb + quarter of its query
    float of_diff = a.scale.of_diff;
    uint32_t k_at[KB], v_at[OB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) k_at[kb] = mine + c16 * ROW + ((kb * 4 + quarter) ^ T::swz_k(c16)) * 16;
#pragma unroll
    for (int i = 0; i < OB; ++i) {
        if constexpr (T::kHalf) {  // 4 features of row 4 quarter + (lane % 16) / 4: the transposing read's share
            const int r = quarter * 4 + c16 / 4;
            v_at[i] = mine + 2 * T::BYTES + r * ROW + ((i * 2 + c16 % 4 / 2) ^ T::swz_v(r)) * 16 + c16 % 2 * 8;
        } else {  // row 4 quarter + i % 4, features 64 (i / 4) + 4 c16 .. + 3
            v_at[i] = mine + 2 * T::BYTES + (quarter * 4 + i % 4) * ROW + (c16 + i / 4 * 16) * 16;
        }
    }
    constexpr int BLOCKS = TR / 16;  // of 16 rows
    [[maybe_unused]] const auto scores = __builtin_amdgcn_make_buffer_rsrc(a.raw + ((size_t)at.b * a.H + head0) * slots, 0,
                                                                           EMIT == kMasses ? heads * slots * 4 : 0, 0x00020000);

    // off: which of the two places; left: tiles with this one; later: the tile after the next, whose loads are issued once this one is in registers
    auto tile = [&](uint32_t off, int row, int bad, int left, const Places& later) __attribute__((always_inline)) {
        if (left > 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");  // all loads but the next tile's have landed
        else wait_loads();
        add_new(off, row);
        f32x4 kf[KB][BLOCKS];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t) kf[kb][t] = *(lds_f32x4*)(uintptr_t)(k_at[kb] + off + t * 16 * ROW);
        bf16x4 vh[OB][BLOCKS];  // V, bf16
        f32x4 vw[OB];           // V, fp32
#pragma unroll
        for (int i = 0; i < OB; ++i) {
            if constexpr (T::kHalf) {
#pragma unroll
                for (int t = 0; t < BLOCKS; ++t) vh[i][t] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(uintptr_t)(v_at[i] + off + t * 16 * ROW));
            } else {
                vw[i] = *(lds_f32x4*)(uintptr_t)(v_at[i] + off);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x4 s[BLOCKS];
        if constexpr (T::kHalf) {
            f32x4 part[BLOCKS][2];  // two chains
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t) part[t][0] = part[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int t = 0; t < BLOCKS; ++t)
                    part[t][kb % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[kb][t]), __builtin_bit_cast(bf16x8, qf[kb]),
                                                                             part[t][kb % 2], 0, 0, 0);
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[t][r] = part[t][0][r] + part[t][1][r];
        } else {
            f32x4 part[4];  // four chains, so that every partial sum is short
#pragma unroll
            for (int e = 0; e < 4; ++e) part[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    part[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[kb][0][e], __uint_as_float(qf[kb][e]), part[e], 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[0][r] = (part[0][r] + part[1][r]) + (part[2][r] + part[3][r]);
        }
        wait_lds();
        if (left > 2) {
            issue_k(mine + off, later);
            issue_v(mine + 2 * T::BYTES + off, later);
        }

        if (bad || row + TR > n + 1) {
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = row + t * 16 + quarter * 4 + r;
                    if (j > n || (j < n && (bad >> (t * 2 + quarter / 2) & 1))) s[t][r] = -INFINITY;
                }
        }
        if constexpr (EMIT != kNoScores) {
            if (c16 < heads) {
                float* raw = a.raw + ((size_t)at.b * a.H + head0 + c16) * slots;
#pragma unroll
                for (int t = 0; t < BLOCKS; ++t) {
                    const int j = row + t * 16 + quarter * 4;
                    f32x4 x;
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = s[t][r] * of_diff;
                    if constexpr (EMIT == kMasses) {  // written through, like the partial results
                        if (j <= n) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), scores, (c16 * slots + j) * 4, 0, kDeviceScope);
                    } else {
                        if (j <= n) *reinterpret_cast<f32x4*>(raw + j) = x;
                    }
                }
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, s[t][r]);
        const float m_new = fmaxf(m, head_max(top));
        if (__any(m_new > m)) {
            const float c = exp2f((m - m_new) * of_diff);
            l *= c;
#pragma unroll
            for (int i = 0; i < OB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] *= c;
        }
        m = m_new;
        // 2^x; the exponential instruction gives zero where the result is subnormal, exp2f does not
        float p[BLOCKS][4], sum = 0.f, least = 0.f;
#pragma unroll
        for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = (s[t][r] - m) * of_diff;
                least = fminf(least, x);
                p[t][r] = __builtin_amdgcn_exp2f(x);
            }
        bool small = __any(least < kSmallExponent && c16 < heads);
        if (__builtin_expect(small, 0)) {
            bool some = false;  // masked rows and scores of -inf, whose weight is 0 either way, are none of them
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    p[t][r] = exp2f((s[t][r] - m) * of_diff);
                    some |= p[t][r] > 0.f && p[t][r] < kSmall;
                }
            small = __any(some && c16 < heads);
        }
#pragma unroll
        for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += p[t][r];
        l += sum;

        if constexpr (T::kHalf) {
            // a probability enters as the sum of three bf16 numbers, its 24 bits cut into eights (what is left is not negative); none of those of one that
            // is not 0 is 0, so that an infinite V stays infinite: 2^-24 and 2^-25 of it at least, less than its last bit. (Two numbers, 2^-16 off: B1 H32 640 rows
            // 8.4 us, with three 8.5; B16 H32 870 rows 38.8, 39.2; two of them in one instruction of 32 rows, which their V has to be copied for: the same.)
            constexpr int PV = BLOCKS * 4;  // probabilities of a lane
            typedef __attribute__((ext_vector_type(PV))) __bf16 bf16xp;
            struct Parts {
                bf16xp of[3];
            };
            auto cut = [](float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); };
            auto split = [&](float x, int e, Parts& to) __attribute__((always_inline)) {
                const float high = cut(x), rest = x - high, middle = cut(rest);
                to.of[0][e] = (__bf16)high;
                to.of[1][e] = (__bf16)fmaxf(middle, x * 0x1p-24f);
                to.of[2][e] = (__bf16)fmaxf(rest - middle, x * 0x1p-25f);
            };
            // x + V^T . P^T of 16 features, P one of its parts
            auto multiply = [](const bf16x4(&v)[BLOCKS], const bf16xp& part, f32x4 x) __attribute__((always_inline)) {
                if constexpr (BLOCKS == 2)
                    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7), part, x, 0, 0, 0);
                else
                    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, v[0]), __builtin_bit_cast(s16x4, part), x, 0, 0, 0);
            };
            // weights whose parts would leave bf16's range, which count where V is large enough: apart, times 2^64. A row is in one of the two products
            // and weighs 0 in the other, which an infinite V does not bear: V's infinities and NaN are taken out of both, with a weight of 1.
            Parts parts;
            if (__builtin_expect(small, 0)) {
#pragma unroll
                for (int e = 0; e < PV; ++e) parts.of[0][e] = p[e / 4][e % 4] > 0.f ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll
                for (int i = 0; i < OB; ++i) {
                    bf16x4 unbounded[BLOCKS];
#pragma unroll
                    for (int t = 0; t < BLOCKS; ++t) {
                        const s16x4 v = __builtin_bit_cast(s16x4, vh[i][t]), is = (v & (short)0x7f80) == (short)0x7f80;
                        unbounded[t] = __builtin_bit_cast(bf16x4, v & is), vh[i][t] = __builtin_bit_cast(bf16x4, v & ~is);
                    }
                    o[i] = multiply(unbounded, parts.of[0], o[i]);
                }
#pragma unroll
                for (int e = 0; e < PV; ++e) {
                    float& x = p[e / 4][e % 4];
                    split(x < kSmall ? x * 0x1p64f : 0.f, e, parts);
                    x = x < kSmall ? 0.f : x;
                }
#pragma unroll
                for (int i = 0; i < OB; ++i) {
                    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int part = 0; part < 3; ++part) x = multiply(vh[i], parts.of[part], x);
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[i][r] = fmaf(x[r], 0x1p-64f, o[i][r]);
                }
            }
#pragma unroll
            for (int e = 0; e < PV; ++e) split(p[e / 4][e % 4], e, parts);
#pragma unroll
            for (int part = 0; part < 3; ++part)
#pragma unroll
                for (int i = 0; i < OB; ++i) o[i] = multiply(vh[i], parts.of[part], o[i]);
        } else {
#pragma unroll
            for (int i = 0; i < OB; ++i) {  // block i / 4 of 64 features, rows 4 quarter + i % 4
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i / 4 * 4 + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vw[i][e], p[0][i % 4], o[i / 4 * 4 + e], 0, 0, 0);
            }
        }
    };
    {
        int row = (at.first * WAVES + wave) * TR, left = at.last - at.first;  // rounds
        const Places first = places_of(row, pages_of(row));
        issue_q(mine + 3 * T::BYTES);  // the queries pass through the place of the second tile of V
        issue_k(mine, first);
        issue_v(mine + 2 * T::BYTES, first);
        Places next = places_of(row + ROUND, pages_of(row + ROUND));
        issue_k(mine + T::BYTES, next);  // (nothing, where the segment has one round)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * NI) : "memory");
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) qf[kb] = *(lds_u32x4*)(uintptr_t)(k_at[kb] + 3 * T::BYTES);
        wait_lds();
        issue_v(mine + 3 * T::BYTES, next);
        if constexpr (T::kHalf) {
            // a power of two, added to the exponents, unless that takes an element out of the range of normal numbers
            u16x2 least = {0xffff, 0xffff}, most = {0, 0};
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u16x2 x = __builtin_bit_cast(u16x2, qf[kb][e] & 0x7fff7fffu);
                    least = __builtin_elementwise_min(least, x - (u16x2){1, 1}), most = __builtin_elementwise_max(most, x);  // zeros count as large
                }
            const int lo = (min((int)least.x, (int)least.y) + 1) >> 7, hi = max((int)most.x, (int)most.y) >> 7, up = a.scale.exponent;
            if (__all((lo + up >= 1) & (hi + up <= 253) & (hi < 255))) {
                const u16x2 add = {(uint16_t)(up * 128), (uint16_t)(up * 128)};
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t word = qf[kb][e];  // (a cast of the element itself takes the vector's first)
                        const u16x2 x = __builtin_bit_cast(u16x2, word);
                        const u16x2 some = __builtin_elementwise_min(x & (u16x2){0x7fff, 0x7fff}, (u16x2){1, 1});
                        qf[kb][e] = __builtin_bit_cast(uint32_t, (u16x2)(x + some * add));
                    }
            } else {
                of_diff = a.scale.whole;
            }
        } else {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) qf[kb][e] = __float_as_uint(__uint_as_float(qf[kb][e]) * a.scale.whole);
        }
        uint32_t off = 0;
        int bad = first.bad, next_bad = next.bad;
        if (left > 2) next = places_of(row + 2 * ROUND, pages_of(row + 2 * ROUND));
        for (;; --left) {
            Ids ids;
            if (left > 3) ids = pages_of(row + 3 * ROUND);
            tile(off, row, bad, left, next);
            if (left == 1) break;
            bad = next_bad, next_bad = next.bad;
            row += ROUND, off ^= T::BYTES;
            if (left > 3) next = places_of(row + 2 * ROUND, ids);
        }
    }

    // ------------------------------------------------------------------ the waves' results together
    l = head_sum(l);
    wait_loads();  // nothing more arrives in the tiles, whose place the sums take
    if (at.last * ROUND > n && block == 0 && wave == 0) {  // the new row; nobody reads its slot in this launch
        if ((unsigned)new_page < (unsigned)a.pages.n_pages) {
            if (lane < CH) {
                const size_t to = a.pages.row(new_page, a.Hkv, hk, n) * CH + lane;
                static_cast<u32x4*>(a.k_pages)[to] = new_k;
                static_cast<u32x4*>(a.v_pages)[to] = new_v;
            }
            if (lane == 0 && a.pos_pages && (a.G > 1 || hk == 0)) a.pos_pages[a.pages.row(new_page, a.G, a.G > 1 ? hk : 0, n)] = new_pos;
        }
    }
    if (quarter == 0) sh_m[wave][c16] = m, sh_l[wave][c16] = l;
#pragma unroll
    for (int i = 0; i < OB; ++i) {
        if constexpr (T::kHalf) {
            *(lds_f32x4*)(uintptr_t)(mine + (c16 * OROW + i * 16 + quarter * 4) * 4) = o[i];
        } else {  // features 64 (i / 4) + 4 (4 quarter + r) + i % 4
            typedef __attribute__((address_space(3))) float lds_float;
#pragma unroll
            for (int r = 0; r < 4; ++r) *(lds_float*)(uintptr_t)(mine + (c16 * OROW + i / 4 * 64 + (quarter * 4 + r) * 4 + i % 4) * 4) = o[i][r];
        }
    }
    __syncthreads();
    auto write = [&](int h, int d, float x, float y) {
        if constexpr (T::kHalf)
            static_cast<uint32_t*>(a.out)[(out_at + h * D + d) / 2] = (uint32_t)f32_to_bf16(x) | (uint32_t)f32_to_bf16(y) << 16;
        else *reinterpret_cast<float2*>(static_cast<float*>(a.out) + out_at + h * D + d) = make_float2(x, y);
    };
    auto statistics = [&](int h, float top, float sum) {
        float* to = a.stats + ((size_t)at.b * a.H + head0 + h) * 2;
        if constexpr (EMIT == kMasses) put(reinterpret_cast<unsigned long long*>(to), top * of_diff, 1.f / sum);
        else if constexpr (EMIT == kScores) *reinterpret_cast<float2*>(to) = make_float2(top * of_diff, 1.f / sum);
    };
    unsigned long long* part = a.partials + (size_t)at.split * PART;
    for (int i = tid; i < heads * (D / 2); i += WAVES * kWave) {
        const int h = i / (D / 2), d = i % (D / 2) * 2;
        float top = sh_m[0][h], sum = 0.f, x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, sh_m[w][h]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float c = exp2f((sh_m[w][h] - top) * of_diff);
            const float2 v = *reinterpret_cast<const float2*>(tiles[w] + (h * OROW + d) * 4);
            sum += sh_l[w][h] * c, x += v.x * c, y += v.y * c;
        }
        if (at.count == 1) {
            write(h, d, x / sum, y / sum);
            if (d == 0) statistics(h, top, sum);
        } else {
            put(part + kHeadBlock + i, x, y);
            if (d == 0) put(part + h, top, sum);
        }
    }
    // ------------------------------------------------------------------ the masses of a group, by the last of its pairs
    auto add_masses = [&]() __attribute__((always_inline)) {
        constexpr int ROWS = WAVES * kWave, EACH = kMassSlots / ROWS;  // rows of a pass, a row a thread; four a lane where the waves share the heads
        const int g = a.G > 1 ? hk : 0, all_heads = a.H / a.G, pairs = a.G > 1 ? a.blocks : a.Hkv * a.blocks, passes = n / ROWS + 1;
        const size_t first = (size_t)at.b * a.H + g * all_heads;
        int id[EACH];  // pages and masses of this thread's rows, asked for on the way
#pragma unroll
        for (int u = 0; u < EACH; ++u) id[u] = u < passes ? a.pages.page_of(at.b, min(u * ROWS + tid, n)) : -1;
        wait_loads();  // this wave's scores and statistics are where every workgroup sees them
        float* to[EACH];
        float old[EACH];
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            to[u] = a.mass_pages + a.pages.row(max(id[u], 0), a.G, g, min(u * ROWS + tid, n));
            old[u] = u < passes ? *to[u] : 0.f;
        }
        __syncthreads();
        if (pairs > 1) {
            if (tid == 0) sh_ticket = atomicInc(a.group_tickets + at.b * a.G + g, pairs - 1);
            __syncthreads();
            if (sh_ticket != (unsigned)pairs - 1) return;
        }
        static_assert(kMassHeads * 8 + WAVES * kMassSlots * 4 <= (int)sizeof(tiles));
        float2* of = reinterpret_cast<float2*>(tiles[0]);
        float(*part)[kMassSlots] = reinterpret_cast<float(*)[kMassSlots]>(tiles[0] + kMassHeads * 8);
        const auto raw = __builtin_amdgcn_make_buffer_rsrc(a.raw + first * slots, 0, all_heads * slots * 4, 0x00020000);
        const auto stats = __builtin_amdgcn_make_buffer_rsrc(a.stats + first * 2, 0, all_heads * 8, 0x00020000);
        const int per = (all_heads + WAVES - 1) / WAVES, h0 = wave * per, heads_here = min(per, all_heads - h0);  // (none: 0 or less)
        u32x4 x[2][kMassAhead];
        int fetch_pass = 0, fetch_head = 0, pass = 0, head = 0;
        auto fetch = [&](u32x4(&to)[kMassAhead]) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < kMassAhead; ++u) {
                const int j = fetch_pass * ROWS + lane * 4;
                to[u] = __builtin_amdgcn_raw_buffer_load_b128(raw, j <= n && heads_here > 0 ? ((h0 + fetch_head) * slots + j) * 4 : 0x7ffffff0, 0, kDeviceScope);
                if (++fetch_head >= heads_here) fetch_head = 0, ++fetch_pass;
            }
        };
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        auto add = [&](const u32x4(&from)[kMassAhead]) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < kMassAhead; ++u)
                if (pass < passes) {
                    const float2 y = of[h0 + head];
                    f32x4 p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t word = from[u][e];
                        p[e] = __uint_as_float(word) - y.x;
                    }
                    weights_of(p);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] = fmaf(p[e], y.y, sum[e]);
                    if (++head >= heads_here) {
                        *reinterpret_cast<f32x4*>(part[wave] + pass * ROWS + lane * 4) = sum;
                        sum = f32x4{0.f, 0.f, 0.f, 0.f}, head = 0, ++pass;
                    }
                }
        };
        for (int h = tid; h < all_heads; h += ROWS) {
            const u32x2 y = __builtin_amdgcn_raw_buffer_load_b64(stats, h * 8, 0, kDeviceScope);
            of[h] = make_float2(__uint_as_float(y.x), __uint_as_float(y.y));
        }
        fetch(x[0]);
        fetch(x[1]);
        __syncthreads();
        if (heads_here > 0) {
            for (;;) {
                add(x[0]);
                if (pass >= passes) break;
                fetch(x[0]);
                add(x[1]);
                if (pass >= passes) break;
                fetch(x[1]);
            }
        } else {
            for (; pass < passes; ++pass) *reinterpret_cast<f32x4*>(part[wave] + pass * ROWS + lane * 4) = sum;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int j = u * ROWS + tid;
            if (j <= n && id[u] >= 0) {
                float all = part[0][j];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) all += part[w][j];
                *to[u] = (j == n ? 0.f : old[u]) + all / (float)all_heads;
            }
        }
    };
    if (at.count == 1) {
        if constexpr (EMIT == kMasses) add_masses();
        return;
    }

    // ------------------------------------------------------------------ the segments' results together, by the last to arrive
    wait_loads();  // (stores count too) this wave's partial results are where every workgroup sees them
    __syncthreads();
    if (tid == 0) sh_ticket = atomicInc(a.tickets + at.split0, at.count - 1);  // back at 0 with the last
    __syncthreads();
    if (sh_ticket != (unsigned)at.count - 1) return;
    const unsigned long long* parts = a.partials + (size_t)at.split0 * PART;
    constexpr int THREADS = WAVES * kWave, AHEAD = 8;  // loads in flight: each comes from beyond the caches (16: B1 H32 641 rows 9.7 us instead of 8.9)
    float2* weights = reinterpret_cast<float2*>(tiles[0]);  // [segment][head]: (maximum, sum), then the first is the weight
    static_assert(kMostSegments * kHeadBlock * 8 <= (int)sizeof(tiles), "all segments of a pair");
    // (segments behind the last one are behind the end of the buffer: nothing is fetched for them)
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)parts, 0, at.count * PART * 8, 0x00020000);
    u32x4 v[AHEAD];  // four sums of a head each, of as many segments
    auto fetch = [&](int i, int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, ((s0 + u) * PART + kHeadBlock + i * 2) * 8, 0, kDeviceScope);
    };
    for (int i0 = tid; i0 < max(at.count * kHeadBlock, THREADS); i0 += THREADS * AHEAD) {  // (every thread goes round once)
        u32x2 x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = i0 + u * THREADS, h = i % kHeadBlock;
            x[u] = __builtin_amdgcn_raw_buffer_load_b64(rsrc, h < heads ? (i / kHeadBlock * PART + h) * 8 : 0x7ffffff0, 0, kDeviceScope);
        }
        if (i0 == tid) fetch(tid, 0);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (i0 + u * THREADS < at.count * kHeadBlock) weights[i0 + u * THREADS] = make_float2(__uint_as_float(x[u].x), __uint_as_float(x[u].y));
    }
    __syncthreads();
    for (int h = wave; h < heads; h += WAVES) {
        float top = kLowest, sum = 0.f;
        for (int s = lane; s < at.count; s += kWave) top = fmaxf(top, weights[s * kHeadBlock + h].x);
        top = wave_max(top);
        for (int s = lane; s < at.count; s += kWave) {
            float2& x = weights[s * kHeadBlock + h];
            x.x = exp2f((x.x - top) * of_diff);
            sum += x.x * x.y;
        }
        sum = group_sum<kWave>(sum);
        if (lane == 0) {
            sh_l[0][h] = sum;
            statistics(h, top, sum);
        }
    }
    __syncthreads();
    for (int i = tid; i < heads * (D / 4); i += THREADS) {
        const int h = i / (D / 4);
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < at.count; s0 += AHEAD) {
            if (i != tid || s0) fetch(i, s0);  // the first have been asked for with the statistics
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (s0 + u < at.count) {
                    const float w = weights[(s0 + u) * kHeadBlock + h].x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = fmaf(__uint_as_float(v[u][e]), w, x[e]);
                }
        }
        const float sum = sh_l[0][h];
        write(h, i % (D / 4) * 4, x[0] / sum, x[1] / sum);
        write(h, i % (D / 4) * 4 + 2, x[2] / sum, x[3] / sum);
    }
    if constexpr (EMIT == kMasses) add_masses();
}

// mass of every row += the mean of its group's probabilities. A workgroup takes 64 rows at a time, a lane each; its four waves share the group's
// heads (eight reads of each in flight) and add up in LDS, in an order of their own: the same bits every time. Bound by latency up to some
// thousand rows, by the scores' bytes beyond: 3.5 .. 4.3 us. (Groups of few scores have no launch of their own: see kMassScores.)
constexpr int kMassRows = kWave, kMassWaves = kPagedWaves;
__global__ __launch_bounds__(kMassRows* kMassWaves) void paged_mass_kernel(const float* __restrict__ raw, const float* __restrict__ stats, float* mass_pages,
                                                                          const int32_t* __restrict__ len_b, Pages pages, int H, int G)
{
    __shared__ float part[kMassWaves][kMassRows];
    const int b = blockIdx.y / G, g = blockIdx.y % G, n = len_b[b], slots = pages.slots();
    if (n < 0 || n >= slots) return;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int heads = H / G, per = (heads + kMassWaves - 1) / kMassWaves, h0 = wave * per, h1 = min(h0 + per, heads);
    const size_t first = (size_t)b * H + g * heads;
    for (int j0 = blockIdx.x * kMassRows; j0 <= n; j0 += gridDim.x * kMassRows) {
        const int j = j0 + lane, id = pages.page_of(b, min(j, n));
        float* at = mass_pages + pages.row(max(id, 0), G, g, min(j, n));
        const float old = *at;  // on its way with the scores
        float sum = 0.f;
        for (int h = h0; h < h1; h += kMassAhead) {
            float x[kMassAhead];
#pragma unroll
            for (int u = 0; u < kMassAhead; ++u) x[u] = raw[(first + min(h + u, h1 - 1)) * slots + min(j, n)];
#pragma unroll
            for (int u = 0; u < kMassAhead; ++u)
                if (h + u < h1) {
                    const float2 of = reinterpret_cast<const float2*>(stats)[first + h + u];
                    sum = fmaf(exp2f(x[u] - of.x), of.y, sum);
                }
        }
        part[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && j <= n && id >= 0) {
            float all = part[0][lane];
#pragma unroll
            for (int w = 1; w < kMassWaves; ++w) all += part[w][lane];
            *at = (j == n ? 0.f : old) + all / (float)heads;
        }
        __syncthreads();
    }
}

// Workspace: tickets of pairs and of groups (where they lie does not hang on the call), partial results of cut pairs (a pair of r rounds is cut into less than 2 r / most segments, so there are less than twice
// kPagedSegments of them), and for EMIT scores and statistics.
static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
constexpr size_t kTicketBytes = (2 * kPagedSegments + kMassGroups) * sizeof(unsigned int);
static size_t partial_bytes(int D) { return up256((size_t)2 * kPagedSegments * kHeadBlock * (D / 2 + 1) * 8); }
size_t paged_step_ws(int B, int H, int slots, int D, bool emit)
{
    return kTicketBytes + partial_bytes(D) + (emit ? up256((size_t)B * H * slots * 4) + up256((size_t)B * H * 8) : 0);
}

template <int DT, int D> static int launch(const PagedStep& a, float* mass_pages, hipStream_t stream)
{
    constexpr int ROUND = kPagedWaves * PagedTile<DT, D>::TR;
    const long long pairs = (long long)a.B * a.Hkv * a.blocks, rounds = (a.pages.slots() + ROUND - 1) / ROUND;
    // as many workgroups as there can be segments (see find_segment); those without one leave at once
    const long long segments = a.B == 1 ? std::max<long long>(kPagedSegments, pairs) : std::max<long long>(2 * kPagedSegments, kPagedSegments + pairs);
    const dim3 grid((unsigned)std::min(segments, rounds * pairs));
    if (!mass_pages) {
        hipLaunchKernelGGL((paged_step_kernel<DT, D, kNoScores>), grid, dim3(kPagedWaves * kWave), 0, stream, a);
        return status_from_hip(hipGetLastError());
    }
    const int heads = a.H / a.G, slots = a.pages.slots();
    const int together = a.G > 1 ? a.blocks : a.Hkv * a.blocks;  // pairs of a group
    if ((together == 1 || (together <= kMassPairs && a.B * a.G <= kMassGroups)) && slots <= kMassSlots && (long long)heads * slots <= kMassScores) {
        hipLaunchKernelGGL((paged_step_kernel<DT, D, kMasses>), grid, dim3(kPagedWaves * kWave), 0, stream, a);
        return status_from_hip(hipGetLastError());
    }
    hipLaunchKernelGGL((paged_step_kernel<DT, D, kScores>), grid, dim3(kPagedWaves * kWave), 0, stream, a);
    if (const int rc = status_from_hip(hipGetLastError())) return rc;
    const int groups = a.B * a.G, most = std::max(1, 4096 / groups);  // the lengths are on the device: workgroups go over the rows
    hipLaunchKernelGGL(paged_mass_kernel, dim3(std::min((a.pages.slots() + kMassRows - 1) / kMassRows, most), groups), dim3(kMassRows * kMassWaves), 0, stream,
                       a.raw, a.stats, mass_pages, a.len_b, a.pages, a.H, a.G);
    return status_from_hip(hipGetLastError());
}

int paged_step_dispatch(const void* q, const void* k_new, const void* v_new, void* k_pages, void* v_pages, int32_t* pos_pages, float* mass_pages,
                        const Pages& pages, const int32_t* len_b, const int32_t* new_pos_b, int B, int H, int Hkv, int G, int D, float scale, int dt,
                        void* out, void* ws, hipStream_t stream)
{
    char* at = static_cast<char*>(ws);
    const PagedStep a{q, k_new, v_new, k_pages, v_pages, out, pos_pages, len_b, new_pos_b, pages, B, H, Hkv, G, H / Hkv, (H / Hkv + kHeadBlock - 1) / kHeadBlock, paged_scale(scale, dt),
                      reinterpret_cast<float*>(at + kTicketBytes + partial_bytes(D)),
                      reinterpret_cast<float*>(at + kTicketBytes + partial_bytes(D) + up256((size_t)B * H * pages.slots() * 4)),
                      mass_pages, reinterpret_cast<unsigned int*>(at) + 2 * kPagedSegments, reinterpret_cast<unsigned int*>(at),
                      reinterpret_cast<unsigned long long*>(at + kTicketBytes)};
    if (dt == EC_BF16) return D == 128 ? launch<EC_BF16, 128>(a, mass_pages, stream) : launch<EC_BF16, 64>(a, mass_pages, stream);
    return D == 128 ? launch<EC_F32, 128>(a, mass_pages, stream) : launch<EC_F32, 64>(a, mass_pages, stream);
}

}  // namespace ec
