// ec_paged_chunk_step: attention of the new tokens of every sequence, packed one after the other, over the rows that are cached in pages, their own
// among them: token i of a sequence of L rows before the step sees slots 0 .. L + i.
//
// The query heads that share a key/value head lie one after the other: row r of a (sequence, key/value head) is token r / group, head r % group of its
// query heads, so that every row of K and V that comes in serves all of them, and one token of many heads is as good a tile as many tokens
// of one head. A workgroup takes a tile of these rows and a segment of the slots that they see; where a batch has few tiles, long sequences are cut
// into several segments, whose results meet in a second launch by the rule of the softmax: with M the largest of their maxima m_i,
// out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i.
//
// Few rows are bound by the bytes of K and V (8 sequences of up to 2900 rows H32/8 D128 bf16 with 5 tokens each: 58 MB, 21.9 us, of which 8 before the first
// load, between the last and the output and in the second launch; 8 of 1000 rows H32 fp32 with one: 262 MB, 49 us, 5.3 TB/s), many rows by the matrix pipes (2048
// tokens behind 65000 rows H40/8: 2.47 to 2.68 ms from card to card, 1.03 to 1.12 PFLOP/s; fp32, 1024 first tokens of 32 heads: 134 us, 64 TFLOP/s).
#include <algorithm>
#include <type_traits>

#include "paged_tile.h"

namespace ec {

// Waves of a workgroup: four, of which a compute unit holds two workgroups, or eight where a batch has no more tiles than the chip has compute units. A wave
// alone on its SIMD issues half as much as two do.
constexpr int kFewWaves = 4, kManyWaves = 8;
// Workgroups that the chip holds at once
template <int DT, int D, int WAVES> constexpr int kChunkPlaces = WAVES == kFewWaves ? PagedTile<DT, D>::kResident * kComputeUnits : kComputeUnits;
constexpr int kMostPlaces = 2 * kComputeUnits, kChunkParts = 4 * kMostPlaces;  // kChunkParts: segments whose results the workspace holds, at most
constexpr int kMostGroups = 1 << 22;                      // of a launch, whose threads have to fit into 32 bits
constexpr int kShortUnits = 4;                            // units, of four waves, up to which tiles are never cut
constexpr int kChunkTiles = 128;                          // tiles from which on segments may take several rounds
constexpr int kJoinWaves = 4, kJoinGroups = 8;            // waves of a joining workgroup, and workgroups that share a tile's rows

// A tile whose segments' results are joined: rows r0 .. r1-1, `count` segments, those of the first from row `place` of the workspace on, `between` rows from
// one to the next.
struct CutTile {
    int place, between, count, r0, r1, t0, hk, unused;
};

struct ChunkStep {
    const void *q, *k_pages, *v_pages;
    void* out;
    float* lse;
    const int32_t *start_b, *token_start;
    Pages pages;
    int B, T, H, Hkv, group;
    uint32_t group_mul, group_shift;  // x / group = (4 x * group_mul >> 32) >> group_shift for x < 2^30
    uint32_t heads_mul, heads_shift;  // x / Hkv, as above
    int rounds, rounds_64;  // that segments may take, and if tiles of many rows have 64
    bool small;       // the units of all tiles have 29 bits, whatever token_start holds
    bool cut;         // whether tiles may be cut and the second launch follows
    float scale, scale_log2e;
    int* cut_tiles;   // tiles that are cut, which paged_chunk_join_kernel goes over
    CutTile* records;
    int part_rows;    // rows of a segment's place in the workspace
    float* partials;  // [segment][part_rows][D] of sequences that are cut
    float2* stats;    // [segment][part_rows] largest score, before its scale, and sum
};

// The lane, found out anew: as with the arguments, nothing is kept for it.
__device__ __forceinline__ int lane_anew() { return anew((int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0))) & (kWave - 1); }

// The launch's arguments, read anew: what a workgroup needs only at its start or its end takes no registers in between.
__device__ __forceinline__ ChunkStep chunk_args()
{
    typedef __attribute__((address_space(4))) const uint32_t const_u32;
    struct Words {
        uint32_t of[sizeof(ChunkStep) / 4];
    } words;
    const const_u32* from = (const const_u32*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(from));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(ChunkStep) / 4); ++i) words.of[i] = from[i];
    return __builtin_bit_cast(ChunkStep, words);
}

// x / by, not more and for x < 2^20 not less: a smaller reciprocal, and half a step further from where it changes. In fewer instructions than divided().
__device__ __forceinline__ float low_rcp(int by) { return __builtin_amdgcn_rcpf((float)by) * (1.f - 0x1p-21f); }
__device__ __forceinline__ int about(int x, float low) { return (int)(((float)x + 0.5f) * low); }

__device__ __forceinline__ int token_of(const ChunkStep& a, int row) { return (int)(__umulhi((uint32_t)row << 2, a.group_mul) >> a.group_shift); }

// What a sequence brings: `tiles` tiles of `tile_rows` rows, `units` units of UNIT slots that its last token sees.
struct ChunkSeq {
    int L, t0, n, rows, tile_rows, tiles, units, first_units;  // first_units: that the first tile sees
    bool live;
    // many: binary logarithm of the rows of a tile of a sequence with more than 32
    template <int UNIT> __device__ __forceinline__ void read(const ChunkStep& a, int b, int many)
    {
        L = -1, t0 = n = 0;
        if (b < a.B) {
            L = a.start_b[b];
            t0 = min(max(a.token_start[b], 0), a.T);
            n = max(min(a.token_start[b + 1], a.T) - t0, 0);
        }
        const int slots = a.pages.slots();
        live = L >= 0 && L < slots;
        rows = n * a.group;
        units = !n ? 0 : live ? (min(L + n, slots) + UNIT - 1) / UNIT : 1;
        tile<UNIT>(a, many);
    }
    // Tiles of as few rows as hold a sequence's where the bytes of K and V are the bound, so that few matrix instructions are spent on rows that are not there;
    // many share what comes in where they are many, in bf16 (32 rows of fp32 take four times as long in the matrix pipe as K and V take to come in
    // from the L2).
    template <int UNIT> __device__ __forceinline__ void tile(const ChunkStep& a, int many)
    {
        const int shift = rows <= 16 ? 4 : rows <= 32 ? 5 : many;
        tile_rows = 1 << shift;
        tiles = (rows + tile_rows - 1) >> shift;
        first_units = !n ? 0 : live ? min(L + token_of(a, min(tile_rows, rows) - 1), a.pages.slots() - 1) / UNIT + 1 : 1;
    }
};
// Sum over the wave, of numbers below 2^54.
__device__ __forceinline__ long long wave_sum(long long x)
{
    const int low = last_lane(wave_scan((int)(x & 0x3ffff))), middle = last_lane(wave_scan((int)(x >> 18 & 0x3ffff))), high = last_lane(wave_scan((int)(x >> 36)));
    return ((long long)high << 36) + ((long long)middle << 18) + low;
}
// How a sequence's tiles are cut: from the last tile on `whole` of them not at all, the others into `segments` of `each` units (those that see less into fewer).
struct ChunkCut {
    int whole, segments, each;
};
// What all of them are cut by: the units that are a place's share of the whole batch, and the rounds that segments may take.
// ONE: whether a launch can have one round only, which four waves of bf16 never have. SHORT: units up to which a sequence's tiles are never cut, as the host
// leaves the second launch away in tables of no more slots.
template <int UNIT, int SHORT, bool ONE> struct ChunkShare {
    int units, rounds;  // rounds 0: one, in which segments of at most `units` find places
    int many;           // see ChunkSeq
    // Units of a segment, at least: as many as its results, written and read again, take the time of (with 4 instead of 8 slots a row 2048 first tokens of 32
    // heads 110 us instead of 64), or half as many where workgroups would have nothing to do (8 drafts of 32 tokens over 2900 rows 33.4 us instead of 41.3,
    // with 6 36.3)
    __device__ __forceinline__ int least(const ChunkSeq& s) const { return max(min(s.rows, s.tile_rows) * (rounds > 1 ? 8 : 4), 256) / UNIT; }
    // Segments of a tile of U units of at most `units` each, but no less than `floor`.
    __device__ __forceinline__ int segments(int U, int floor) const
    {
        return U <= SHORT ? 1 : max(min(about(U + units - 1, low_rcp(units)), about(U, low_rcp(floor))), 1);
    }
    // A tile of U units, against a share of A:
    //   U > A       S = r U / A segments, which take r rounds: the r for which r (U / S) is least
    //   U <= A < 4U as many tiles whole as fit into rounds that are full, the rest cut into what is left of the share
    //   else        whole: the last tiles to start are short beside the rest
    // These are r tiles U / A segments of a sequence, or 2 tiles U / A: within what the workspace holds, as chunk_share sees to it.
    __device__ __forceinline__ ChunkCut of(const ChunkSeq& s) const
    {
        const int U = s.units, floor = least(s), A = max(units, floor);
        const float low = low_rcp(A);
        int n = 1, whole = 0;
        if (ONE && !rounds) {
            n = segments(U, floor);
        } else if (U <= SHORT) {
        } else if (U > A) {
            n = about(U, low);
            if (rounds > 1 && U < 4 * A) {
                int time = about(U + n - 1, low_rcp(n));
#pragma unroll
                for (int r = 2; r <= 4; ++r) {
                    const int m = about(r * U, low), t = r * about(U + m - 1, low_rcp(m)) + (r - 1) * floor;
                    if (r <= rounds && t < time) time = t, n = m;
                }
            }
        } else if (rounds > 1 && A < 4 * U) {
            const int k = divided(A, U), rest = A - k * U;
            if (rest >= floor && rest * 8 >= A && (long long)s.tiles * rest >= A && (long long)s.tiles * k * U < 1 << 24) {
                n = divided(U, rest);
                whole = divided(s.tiles * k * U, A);
            }
        }
        if (n <= 1) return {s.tiles, 1, U};
        return {whole, n, divided(U + n - 1, n)};
    }
};
// Sums over the batch, in 32 bits where the units of all tiles fit.
struct SmallSum {
    typedef uint32_t type;
    static __device__ __forceinline__ type of(long long x) { return last_lane(wave_scan((int)x)); }
};
struct LargeSum {
    typedef unsigned long long type;
    static __device__ __forceinline__ type of(long long x) { return wave_sum(x); }
};
// Rows of a tile of a sequence of bf16 with more than 32: 128, or 64 where neither tiles of 128 nor their segments (of ChunkShare::least units each) give all
// compute units something to do. 512 tokens behind 768 rows of 32 heads 25.1 us instead of 28.8, 100 behind 3000 rows H32/8 24.8 instead of 26.7, 32 behind
// 2900 18.8 instead of 22.4; where they do, 128 rows read K and V half as often: 8 sequences of 32 tokens behind 2900 rows 31.2 us instead of 43.3, 32
// tokens behind 65000 rows H40/8 79 instead of 87, 1024 first tokens of 32 heads 27.1 instead of 33.9.
// s: of this lane's sequence, read for tiles of 128 rows, if there are no more than lanes
template <int UNIT, class Sum> __device__ __forceinline__ int many_rows(const ChunkStep& a, ChunkSeq& s)
{
    typename Sum::type tiles = 0, items = 0;
    bool many = false;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        if (a.B > kWave) s.read<UNIT>(a, b0 + threadIdx.x % kWave, 7);
        many |= __any(s.rows > 32);
        if (!many && a.B <= kWave) return 7;
        tiles += Sum::of(s.tiles), items += Sum::of((long long)s.tiles * max(s.units * UNIT / (a.rounds > 1 ? 1024 : 512), 1));
    }
    return many && tiles * a.Hkv <= kComputeUnits / 2 && items * a.Hkv < kComputeUnits ? 6 : 7;
}
template <int UNIT, int SHORT, bool ONE, int PLACES, class Sum>
__device__ __forceinline__ ChunkShare<UNIT, SHORT, ONE> chunk_share_of(const ChunkStep& a, ChunkSeq& s, int many, int rounds)
{
    using N = typename Sum::type;
    N all = 0, most = 0;  // twice the units of all tiles, about; the units if every tile of a sequence saw as much as the last one: at most `all`
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        if (a.B > kWave) s.read<UNIT>(a, b0 + threadIdx.x % kWave, many);
        most += Sum::of((long long)s.tiles * s.units), all += Sum::of((long long)s.tiles * (s.units + s.first_units));
    }
    all *= a.Hkv, most *= a.Hkv;
    // one round: most / share <= PLACES parts; several: rounds * most / share and 2 most / share <= 4 PLACES, as most <= all
    const N share = rounds > 1 ? (all + (2 * PLACES - 1)) / (2 * PLACES) : (most + (PLACES - 1)) / PLACES;
    const int units = (int)min(max(share, (N)1), (N)((1 << 24) - 1));  // (from four times the units of the longest table on nothing is cut)
    if (ONE && rounds == 1 && a.B <= kWave) {  // the least units by which all segments find places at once, if a few more than the share do
        for (int more = 0; more < 4; ++more) {
            const ChunkShare<UNIT, SHORT, ONE> finer = {units + more, 0, many};
            if (Sum::of((long long)s.tiles * finer.segments(s.units, finer.least(s))) * a.Hkv <= PLACES) return finer;
        }
    }
    const N held = (N)4 * PLACES * units;
    return {units, rounds == 1 ? 1 : 4 * most <= held ? 4 : 3 * most <= held ? 3 : 2, many};
}
// s: of this lane's sequence afterwards, if there are no more than lanes
// MANY: binary logarithm of the rows of a tile of a sequence with more than 32, 0 for 6 or 7
template <int MANY, int UNIT, int SHORT, bool ONE, int PLACES>
__device__ __forceinline__ ChunkShare<UNIT, SHORT, ONE> chunk_share(const ChunkStep& a, ChunkSeq& s)
{
    int many = MANY ? MANY : 7, rounds = a.rounds;
    if (a.B <= kWave) s.read<UNIT>(a, threadIdx.x % kWave, many);
    if (MANY == 0) {
        many = a.small ? many_rows<UNIT, SmallSum>(a, s) : many_rows<UNIT, LargeSum>(a, s);
        if (many == 6) {
            rounds = a.rounds_64;
            if (a.B <= kWave) s.tile<UNIT>(a, many);
        }
    }
    if (!a.cut) return {1 << 22, 1, many};  // a share that no tile exceeds
    return a.small ? chunk_share_of<UNIT, SHORT, ONE, PLACES, SmallSum>(a, s, many, rounds) : chunk_share_of<UNIT, SHORT, ONE, PLACES, LargeSum>(a, s, many, rounds);
}

// Units that a tile's last row sees.
template <int UNIT> __device__ __forceinline__ int chunk_units(const ChunkStep& a, const ChunkSeq& s, int tile)
{
    if (!s.live) return 1;
    const int last = token_of(a, min((tile + 1) * s.tile_rows, s.rows) - 1);
    return min(s.L + last, a.pages.slots() - 1) / UNIT + 1;
}


struct ChunkItem {
    ChunkSeq s;
    int hk, segment, each;  // units of a segment
    int r0, r1, seen;       // rows of the tile, units that its last row sees
    size_t place;           // row of the segment's results in the workspace, of sequences that are cut
    int b;                  // < 0: none
};
// The item of a workgroup: heads change fastest, so that the eight XCDs, which get workgroups in turn, keep to their heads, then tiles from the last one,
// which sees most, then segments. s: as chunk_share leaves it.
template <int UNIT, int SHORT, bool ONE>
__device__ __forceinline__ ChunkItem chunk_item(const ChunkStep& a, const ChunkShare<UNIT, SHORT, ONE>& share, ChunkSeq& s, int id, int wave)
{
    const int lane = lane_anew(), j = (int)(__umulhi((uint32_t)id << 2, a.heads_mul) >> a.heads_shift), hk = id - j * a.Hkv;
    int before = 0, parts_before = 0;  // parts: and cut tiles in the high half, both at most kChunkParts
    ChunkItem it;
    it.b = -1;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        if (a.B > kWave) s.read<UNIT>(a, b0 + lane, share.many);
        const ChunkCut cut = share.of(s);
        const int cut_tiles = s.tiles - cut.whole, items = s.tiles + cut_tiles * (cut.segments - 1), parts = cut_tiles * cut.segments + (cut_tiles << 16);
        const int upto = wave_scan(items), parts_upto = wave_scan(parts);
        const unsigned long long beyond = __ballot(j < before + upto);
        if (beyond) {
            const int at = __ffsll(beyond) - 1;
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
            it.s = {of(s.L), of(s.t0), of(s.n), of(s.rows), of(s.tile_rows), of(s.tiles), of(s.units), of(s.first_units), of(s.live) != 0};
            const int in = j - before - (of(upto) - of(items)), whole = of(cut.whole), part = in - whole;
            if (in < 0 || in >= of(items)) return it;
            int tile = in;  // from the last one on
            it.segment = 0, it.each = it.s.units;
            const int tiles = it.s.tiles - whole;
            if (part >= 0) {
                it.segment = scalar(divided(part, tiles)), it.each = of(cut.each);
                tile = whole + part - it.segment * tiles;
            }
            const int nth = tile - whole;
            tile = it.s.tiles - 1 - tile;
            it.r0 = tile * it.s.tile_rows, it.r1 = min(it.r0 + it.s.tile_rows, it.s.rows);
            it.seen = scalar(chunk_units<UNIT>(a, it.s, tile));
            it.hk = hk;
            const int parts_of = parts_before + of(parts_upto) - of(parts);
            it.place = ((size_t)((parts_of & 0xffff) + max(part, 0)) * a.Hkv + hk) * a.part_rows;
            it.b = b0 + at;
            if (part >= 0 && it.segment == 0 && wave == 0 && lane == 0)
                a.records[((parts_of >> 16) + nth) * a.Hkv + hk] = {(int)it.place, tiles * a.Hkv * a.part_rows,
                                                                                            scalar(divided(it.seen + it.each - 1, it.each)), it.r0, it.r1, it.s.t0, hk, 0};
            return it;
        }
        before += last_lane(upto), parts_before += last_lane(parts_upto);
    }
    return it;
}
template <int UNIT, int SHORT, bool ONE> __device__ __forceinline__ void count_cut_tiles(const ChunkStep& a, const ChunkShare<UNIT, SHORT, ONE>& share, ChunkSeq& s)
{
    int n = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        if (a.B > kWave) s.read<UNIT>(a, b0 + threadIdx.x % kWave, share.many);
        n += last_lane(wave_scan(s.tiles - share.of(s).whole));
    }
    if (threadIdx.x == 0) *a.cut_tiles = n * a.Hkv;
}

template <int DT, int D> __device__ __forceinline__ void chunk_write(const ChunkStep& a, size_t at, float x, float y)
{
    if constexpr (DT == EC_BF16) static_cast<uint32_t*>(a.out)[at / 2] = (uint32_t)f32_to_bf16(x) | (uint32_t)f32_to_bf16(y) << 16;
    else *reinterpret_cast<float2*>(static_cast<float*>(a.out) + at) = make_float2(x, y);
}
// Number of the (token, query head) that a row is, in out and lse.
__device__ __forceinline__ size_t chunk_row(const ChunkStep& a, int t0, int hk, int row)
{
    const int token = token_of(a, row);
    return (size_t)(t0 + token) * a.H + hk * a.group + (row - token * a.group);
}

template <int DT, int D, int WAVES> __device__ __forceinline__ void chunk_nothing(const ChunkStep& a, const ChunkItem& at, int wave)
{
    const int r0 = at.r0, rows = at.r1 - r0;
    for (int i = wave * kWave + lane_anew(); i < rows * (D / 2); i += WAVES * kWave) {
        const size_t row = chunk_row(a, at.s.t0, at.hk, r0 + i / (D / 2));
        chunk_write<DT, D>(a, row * D + i % (D / 2) * 2, 0.f, 0.f);
        if (a.lse && i % (D / 2) == 0) a.lse[row] = -INFINITY;
    }
}

// Values that are no numbers, summed over up to 32 rows of V by kind: +inf counts 1, -inf 64 and NaN 4096 where the row has a weight, and 2^18 times that, which
// is NaN whichever it is, where it is seen with a weight of 0.
__device__ __forceinline__ float kind_of(float v) { return v == INFINITY ? 1.f : v == -INFINITY ? 64.f : v != v ? 4096.f : 0.f; }
__device__ __forceinline__ bf16x4 kind_of(bf16x4 v_)
{
    const s16x4 v = __builtin_bit_cast(s16x4, v_), inf = (short)0x7f80 - (s16x4){0, 0, 0, 0};
    return __builtin_bit_cast(bf16x4, ((v == inf) & (short)0x3f80) | ((v == (inf | (short)0x8000)) & (short)0x4280) | (((v & (short)0x7fff) > inf) & (short)0x4580));
}
__device__ __forceinline__ float kind_weight(float p, bool seen) { return p > 0.f ? 1.f : seen ? 0x1p18f : 0.f; }
__device__ __forceinline__ float with_kinds(float x, float n)
{
    const int kinds = (int)fminf(n, 4096.f);
    x += kinds & 0x3f ? INFINITY : 0.f;
    x += kinds & 0xfc0 ? -INFINITY : 0.f;
    return x + (kinds & 0x1000 ? NAN : 0.f);
}

// Up to 16 RB rows: the workgroup's waves share the slots, a wave takes every WAVES-th tile of TR of them and keeps a running (maximum, sum,
// weighted V) for the rows.
//   S^T = K . Q^T      matrix instructions, so that a lane owns one row in 16 and 4 consecutive slots of a block of 16
//   O^T += V^T . P^T   the probabilities are the second operand as they stand; V is transposed on its way out of LDS (bf16)
// A bf16 probability enters as the sum of three bf16 numbers, all its 24 bits: few rows are bound by the bytes of K and V, and the matrix pipes have the room.
// False: something has come out that is no number, with two blocks of fp32 rows, which leave the care for infinite V to single ones.
template <int DT, int D, int WAVES, int RB>
__device__ __forceinline__ bool chunk_few_rows(const ChunkStep& a, const ChunkItem& at, int wave, unsigned char* tiles, float* sh_m, float* sh_l, int* flags)
{
    using T = PagedTile<DT, D>;
    constexpr int TR = T::TR, ROW = T::kRowBytes, CH = T::CH, RPI = T::RPI, NI = T::NI, ROUND = WAVES * TR;
    constexpr int KB = ROW / 64;   // 64-byte blocks of a row: what the four quarters of a wave contract together
    constexpr int OB = D / 16;     // 16-feature blocks of the output
    constexpr int BLOCKS = TR / 16;
    const int lane = lane_anew(), tid = wave * kWave + lane;
    const int c16 = lane % 16, quarter = lane / 16;
    const int slots = a.pages.slots(), r0 = at.r0;
    const int first = at.segment * at.each, last = min(first + at.each, at.seen);
    if (first >= last) return true;  // a tile that sees fewer segments than its sequence has
    const bool whole = at.each >= at.seen;  // the tile's only segment

    // ------------------------------------------------------------------ rows into LDS
    const uint32_t mine = __builtin_amdgcn_readfirstlane(lds_address(tiles + wave * 4 * T::BYTES));
    const int lowest = min(at.s.L + token_of(a, r0), slots - 1);  // what the tile's first row sees last
    const int highest = min(at.s.L + token_of(a, min(r0 + 16 * RB, at.r1) - 1), slots - 1);
    const int shift = a.pages.shift, mask = (1 << shift) - 1, end = min(highest + 1, last * ROUND);
    const const_i32* table = (const const_i32*)(uintptr_t)(a.pages.table + (size_t)at.b * a.pages.max_pages);
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
                pl.from[u] = (size_t)(uint32_t)(page ? ids.id[u] : 0) * page_bytes + (at.hk * head_bytes + (uint32_t)(r & mask) * ROW);
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
            load_run_lds<T::IPG, T::kHalf>(tile_rsrc(static_cast<const char*>(a.k_pages) + pl.from[u], pl.bytes[u]), lds + u * 8 * ROW, k_part[u & 1]);
    };
    auto issue_v = [&](uint32_t lds, const Places& pl) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < T::GROUPS; ++u)
            load_run_lds<T::IPG, T::kHalf>(tile_rsrc(static_cast<const char*>(a.v_pages) + pl.from[u], pl.bytes[u]), lds + u * 8 * ROW, v_part);
    };

    int row = (first * WAVES + wave) * TR, left = last - first;  // rounds
    const Ids at_once = pages_of(row), ahead = pages_of(row + ROUND);
    const Places here = places_of(row, at_once);
    issue_k(mine, here);
    issue_v(mine + 2 * T::BYTES, here);

    // ------------------------------------------------------------------ one tile after the other
    f32x4 o[RB][OB];
    float m[RB], l[RB];  // l: of this lane's slots
    int limit[RB];       // last slot that the lane's row sees
    u32x4 qf[RB][KB];    // the lane's row, chunks 4 kb + quarter of its query
    const float of_diff = a.scale_log2e;  // differences of scores are scaled, so that no score leaves the range
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = r0 + rb * 16 + c16;
        limit[rb] = r < at.r1 ? min(at.s.L + token_of(a, r), slots - 1) : -1;
        const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.q) + chunk_row(a, at.s.t0, at.hk, min(r, at.r1 - 1)) * ROW);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) qf[rb][kb] = q[kb * 4 + quarter];
        m[rb] = kLowest, l[rb] = 0.f;
#pragma unroll
        for (int i = 0; i < OB; ++i) o[rb][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
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
    // off: which of the two places; left: tiles with this one; later: the tile after the next, whose loads are issued once this one is in registers
    auto tile = [&](uint32_t off, int row, int bad, int left, const Places& later) __attribute__((always_inline)) {
        if (left > 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");  // all loads but the next tile's have landed
        else wait_loads();
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
        f32x4 s[RB][BLOCKS];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            if constexpr (T::kHalf) {
                f32x4 part[BLOCKS][2];  // two chains
#pragma unroll
                for (int t = 0; t < BLOCKS; ++t) part[t][0] = part[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int t = 0; t < BLOCKS; ++t)
                        part[t][kb % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[kb][t]), __builtin_bit_cast(bf16x8, qf[rb][kb]),
                                                                                 part[t][kb % 2], 0, 0, 0);
#pragma unroll
                for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[rb][t][r] = part[t][0][r] + part[t][1][r];
            } else {
                f32x4 part[4];  // four chains, so that every partial sum is short
#pragma unroll
                for (int e = 0; e < 4; ++e) part[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        part[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[kb][0][e], __uint_as_float(qf[rb][kb][e]), part[e], 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[rb][0][r] = (part[0][r] + part[1][r]) + (part[2][r] + part[3][r]);
            }
        }
        wait_lds();
        if (left > 2) {
            issue_k(mine + off, later);
            issue_v(mine + 2 * T::BYTES + off, later);
        }

        const bool masked = bad || row + TR - 1 > lowest;  // some row does not see some slot of the tile
        auto sees = [&](int upto, int t, int r) __attribute__((always_inline)) { return row + t * 16 + quarter * 4 + r <= upto && !(bad >> (t * 2 + quarter / 2) & 1); };
        float p[RB][BLOCKS][4], least = 0.f;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            if (masked) {
#pragma unroll
                for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!sees(limit[rb], t, r)) s[rb][t][r] = -INFINITY;
            }
            float top = s[rb][0][0];
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, s[rb][t][r]);
            const float m_new = fmaxf(m[rb], head_max(top));
            if (__any(m_new > m[rb])) {
                const float c = exp2f((m[rb] - m_new) * of_diff);
                l[rb] *= c;
#pragma unroll
                for (int i = 0; i < OB; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[rb][i][r] *= c;
            }
            m[rb] = m_new;
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = (s[rb][t][r] - m[rb]) * of_diff;
                    if constexpr (T::kHalf) least = fminf(least, x);
                    p[rb][t][r] = __builtin_amdgcn_exp2f(x);
                    sum += p[rb][t][r];
                }
            l[rb] += sum;
        }

        if constexpr (T::kHalf) {
            using Parts = WeightParts<BLOCKS>;
            constexpr int PV = Parts::N;
            // Weights whose parts would leave bf16's range, which count where V is large enough, enter apart, times 2^64.
            bool small = __any(least < kSmallExponent);
            if (__builtin_expect(small, 0)) {
                bool some = false;  // what is not seen, and scores of -inf, whose weight is 0 either way, are none of them
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int e = 0; e < PV; ++e) some |= p[rb][e / 4][e % 4] > 0.f && p[rb][e / 4][e % 4] < kSmall;
                small = __any(some);
            }
            if (masked || small) {
                // An infinite V must not reach the rows that do not see it, as 0 times infinity would, nor those whose weight for it is in the other product: it
                // leaves the products, and every row adds the kinds that it sees, NaN where it sees any kind with a weight of 0.
                bool some = false;
#pragma unroll
                for (int i = 0; i < OB; ++i)
#pragma unroll
                    for (int t = 0; t < BLOCKS; ++t) {
                        const s16x4 is = (__builtin_bit_cast(s16x4, vh[i][t]) & (short)0x7f80) == (short)0x7f80;
                        some |= (is[0] | is[1] | is[2] | is[3]) != 0;
                    }
                if (__builtin_expect(__any(some), 0)) {
                    typename Parts::bf16xn weights[RB];
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        const int upto = anew(limit[rb]);  // (found out again, and not kept from above)
#pragma unroll
                        for (int e = 0; e < PV; ++e) weights[rb][e] = (__bf16)kind_weight(p[rb][e / 4][e % 4], sees(upto, e / 4, e % 4));
                    }
#pragma unroll
                    for (int i = 0; i < OB; ++i) {
                        bf16x4 kinds[BLOCKS];
#pragma unroll
                        for (int t = 0; t < BLOCKS; ++t) kinds[t] = kind_of(vh[i][t]);
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) {
                            const f32x4 n = Parts::multiply(kinds, weights[rb], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                            for (int r = 0; r < 4; ++r) o[rb][i][r] = with_kinds(o[rb][i][r], n[r]);
                        }
                        __builtin_amdgcn_sched_barrier(0);  // (one after the other: few registers)
                    }
#pragma unroll
                    for (int i = 0; i < OB; ++i)
#pragma unroll
                        for (int t = 0; t < BLOCKS; ++t) {
                            const s16x4 v = __builtin_bit_cast(s16x4, vh[i][t]), is = (v & (short)0x7f80) == (short)0x7f80;
                            vh[i][t] = __builtin_bit_cast(bf16x4, v & ~is);
                        }
                }
            }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                Parts parts;
                if (__builtin_expect(small, 0)) {
#pragma unroll
                    for (int e = 0; e < PV; ++e) {
                        float& x = p[rb][e / 4][e % 4];
                        parts.set(e, x < kSmall ? x * 0x1p64f : 0.f);
                        x = x < kSmall ? 0.f : x;
                    }
#pragma unroll
                    for (int i = 0; i < OB; ++i) {
                        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int part = 0; part < 3; ++part) x = Parts::multiply(vh[i], parts.of[part], x);
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[rb][i][r] = fmaf(x[r], 0x1p-64f, o[rb][i][r]);
                    }
                }
#pragma unroll
                for (int e = 0; e < PV; ++e) parts.set(e, p[rb][e / 4][e % 4]);
#pragma unroll
                for (int part = 0; part < 3; ++part)
#pragma unroll
                    for (int i = 0; i < OB; ++i) o[rb][i] = Parts::multiply(vh[i], parts.of[part], o[rb][i]);
            }
        } else {
            if (masked) {
                bool some = false;
#pragma unroll
                for (int i = 0; i < OB; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) some |= !(fabsf(vw[i][e]) < INFINITY);
                if (__builtin_expect(__any(some), 0)) {
                    // (what follows from V and the limits is found out again here, and not kept from above)
#pragma unroll
                    for (int i = 0; i < OB; ++i) asm volatile("" : "+v"(vw[i]));
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        const int upto = anew(limit[rb]);
                        f32x4 n[OB];
#pragma unroll
                        for (int i = 0; i < OB; ++i) n[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int i = 0; i < OB; ++i) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                n[i / 4 * 4 + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kind_of(vw[i][e]), kind_weight(p[rb][0][i % 4], sees(upto, 0, i % 4)),
                                                                                       n[i / 4 * 4 + e], 0, 0, 0);
                            __builtin_amdgcn_sched_barrier(0);  // (one after the other: few registers)
                        }
#pragma unroll
                        for (int i = 0; i < OB; ++i) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) o[rb][i][r] = with_kinds(o[rb][i][r], n[i][r]);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < OB; ++i) asm volatile("" : "+v"(vw[i]));
#pragma unroll
                    for (int i = 0; i < OB; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) vw[i][e] = fabsf(vw[i][e]) < INFINITY ? vw[i][e] : 0.f;
                }
            }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int i = 0; i < OB; ++i) {  // block i / 4 of 64 features, rows 4 quarter + i % 4
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[rb][i / 4 * 4 + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vw[i][e], p[rb][0][i % 4], o[rb][i / 4 * 4 + e], 0, 0, 0);
                }
        }
    };
    {
        // (what the compiler waits for by counting, the queries, comes between loads that it does not count: it waits for those before, too)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) asm volatile("" : "+v"(qf[rb][kb]));
        Places next = places_of(row + ROUND, ahead);
        uint32_t off = 0;
        int bad = here.bad, next_bad = next.bad;
        if constexpr (!T::kHalf && RB == 2) {
            // Two blocks of rows, fp32: the matrix pipe is the bound, and a wave is alone on its SIMD, of which it issues an instruction every eighth cycle, four
            // while a matrix instruction lasts. What a block's softmax takes is issued between the matrix instructions of the other block, the scores' or
            // the weighted sum's, loads between those of the first scores:
            //   S of block 0, loads of the tile after the next | S of block 1, softmax of block 0 | O of block 0, softmax of block 1 | O of block 1
            // with K of the next tile on its way out of LDS beside O, V beside S of block 0. 6900 cycles a tile of 16 slots, of which the matrix pipe works
            // 4096, where one block after the other took 7500 (1024 first tokens of 32 heads 143 -> 133 us); what is left is mostly instructions that
            // do not fit beside matrix instructions. (Raising the maximum in steps of 2^8, places in eight parts: no faster.)
            constexpr int N = KB * 4, STAGES = 9;  // matrix instructions of a block's scores; of its sums there are as many
            static_assert(N == OB * 4 && T::GROUPS == 2);
            f32x4 kf[KB], vw[OB], part[2][4], s[2], x[2];
            float correction[2];
            int beyond[2];  // the first of the lane's four slots that its row does not see
            auto read_k = [&](uint32_t off) __attribute__((always_inline)) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) kf[kb] = *(lds_f32x4*)(uintptr_t)(k_at[kb] + off);
            };
            auto score = [&](int rb, int n) __attribute__((always_inline)) {
                part[rb][n % 4] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[n / 4][n % 4], __uint_as_float(qf[rb][n / 4][n % 4]),
                                                                      n < 4 ? f32x4{0.f, 0.f, 0.f, 0.f} : part[rb][n % 4], 0, 0, 0);
            };
            auto weighted = [&](int rb, int n) __attribute__((always_inline)) {
                const int i = n / 4, e = n % 4;
                o[rb][i / 4 * 4 + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vw[i][e], x[rb][i % 4], o[rb][i / 4 * 4 + e], 0, 0, 0);
            };
            auto softmax = [&](int rb, int stage) __attribute__((always_inline)) {
                if (stage == 0) s[rb] = (part[rb][0] + part[rb][1]) + (part[rb][2] + part[rb][3]);
                if (stage == 1) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[rb][r] = r < beyond[rb] ? s[rb][r] : -INFINITY;
                }
                if (stage == 2) x[rb][0] = fmaxf(fmaxf(s[rb][0], s[rb][1]), fmaxf(s[rb][2], s[rb][3]));
                if (stage == 3) x[rb][0] = head_max(x[rb][0]);
                if (stage == 4) {
                    const float top = fmaxf(m[rb], x[rb][0]);
                    correction[rb] = m[rb] == top ? 0.f : m[rb] - top;
                    m[rb] = top;
                }
                if (stage == 5) correction[rb] = __builtin_amdgcn_exp2f(correction[rb] * of_diff);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (stage == 6) x[rb][r] = (s[rb][r] - m[rb]) * of_diff;
                    if (stage == 7) x[rb][r] = __builtin_amdgcn_exp2f(x[rb][r]);
                }
                if (stage == 8) {
                    l[rb] = fmaf(l[rb], correction[rb], (x[rb][0] + x[rb][1]) + (x[rb][2] + x[rb][3]));
                    asm volatile("" : "+v"(x[rb]), "+v"(l[rb]), "+v"(correction[rb]));  // (here, not where they are used)
                }
            };
            // the stages of a block's softmax that belong to matrix instruction n of N, from the third on
            auto beside = [&](int rb, int n) __attribute__((always_inline)) {
                constexpr int ROOM = N - 3;
#pragma unroll
                for (int i = 0; i < STAGES; ++i)
                    if (n >= 2 && i >= (n - 2) * STAGES / ROOM && i < (n - 1) * STAGES / ROOM) softmax(rb, i);
                __builtin_amdgcn_sched_barrier(0);
            };
            // with 512 registers a wave the sums stay in those that only matrix instructions reach, but for the times when they are rescaled
            auto keep = [&](int rb) __attribute__((always_inline)) {
                if constexpr (T::kResident == 1) {
#pragma unroll
                    for (int i = 0; i < OB; ++i) asm volatile("" : "+a"(o[rb][i]));
                }
            };
            auto rescale = [&](int rb) __attribute__((always_inline)) {
                if (__any(correction[rb] != 1.f)) {
                    keep(rb);
#pragma unroll
                    for (int i = 0; i < OB; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[rb][i][r] *= correction[rb];
                    keep(rb);
                }
                keep(rb);
            };
            // (behind the segment nothing is fetched: loads of no bytes, not a branch around them)
            issue_k(mine + T::BYTES, next);
            issue_v(mine + 3 * T::BYTES, next);
            next_bad = next.bad;
            next = places_of(row + 2 * ROUND, pages_of(row + 2 * ROUND));
            read_k(0);
            keep(0), keep(1);
            for (;; --left) {
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");  // all loads but the next tile's have landed
#pragma unroll
                for (int i = 0; i < OB; ++i) vw[i] = *(lds_f32x4*)(uintptr_t)(v_at[i] + off);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    score(0, n);
                    if (n == N / 2) wait_lds();  // V is in registers
                    if (n % (N / 8) == N / 8 - 1 && n >= N / 2) {
                        const int u = (n - N / 2) / (N / 8);
                        const u32x4 rsrc = tile_rsrc(static_cast<const char*>(u < 2 ? a.k_pages : a.v_pages) + next.from[u % 2], next.bytes[u % 2]);
                        load_run_lds<T::IPG, T::kHalf>(rsrc, mine + (u < 2 ? 0 : 2 * T::BYTES) + off + u % 2 * 8 * ROW, u < 2 ? k_part[u % 2] : v_part);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) beyond[rb] = (bad >> (quarter / 2) & 1 ? -1 : limit[rb]) + 1 - row - quarter * 4;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    score(1, n);
                    beside(0, n);
                }
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * NI) : "memory");  // all up to the next tile's K
                read_k(off ^ T::BYTES);
                const Ids ids = pages_of(row + 3 * ROUND);
                rescale(0);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    weighted(0, n);
                    beside(1, n);
                }
                rescale(1);
                bad = next_bad, next_bad = next.bad;
#pragma unroll
                for (int n = 0; n < N; ++n) weighted(1, n);
                next = places_of(row + 3 * ROUND, ids);
                keep(0), keep(1);
                if (left == 1) break;
                row += ROUND, off ^= T::BYTES;
            }
        } else {
            if (left > 1) {
                issue_k(mine + T::BYTES, next);
                issue_v(mine + 3 * T::BYTES, next);
            }
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
    }

    // ------------------------------------------------------------------ the waves' results together
    // Row r of a wave's sums lies in its tiles at r * D, the 16-byte chunk c of it at place c ^ r, so that the lanes of a row block meet all banks alike.
    wait_loads();  // nothing more arrives in the tiles, whose place the sums take
    const ChunkStep e = chunk_args();
    constexpr int ROWS = 16 * RB, CHUNKS = D / 4;
    static_assert(ROWS * D * 4 <= 4 * T::BYTES && CHUNKS >= 16);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const float all = head_sum(l[rb]);
        if (quarter == 0) sh_m[wave * ROWS + rb * 16 + c16] = m[rb], sh_l[wave * ROWS + rb * 16 + c16] = all;
#pragma unroll
        for (int i = 0; i < OB; ++i) {
            if constexpr (T::kHalf) {
                *(lds_f32x4*)(uintptr_t)(mine + (rb * 16 + c16) * (D * 4) + ((i * 4 + quarter) ^ c16) * 16) = o[rb][i];
            } else {  // features 64 (i / 4) + 4 (4 quarter + r) + i % 4
                typedef __attribute__((address_space(3))) float lds_float;
#pragma unroll
                for (int r = 0; r < 4; ++r) *(lds_float*)(uintptr_t)(mine + (rb * 16 + c16) * (D * 4) + ((i / 4 * 16 + quarter * 4 + r) ^ c16) * 16 + i % 4 * 4) = o[rb][i][r];
            }
        }
    }
    __syncthreads();
    const int rows = min(ROWS, at.r1 - r0);
    float zero = 0.f;
    for (int i = tid; i < rows * CHUNKS; i += WAVES * kWave) {
        const int r = i / CHUNKS, chunk = i % CHUNKS;
        float mw[WAVES], top = kLowest, sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) mw[w] = sh_m[w * ROWS + r];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, mw[w]);
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float c = __builtin_amdgcn_exp2f((mw[w] - top) * of_diff);
            const f32x4 v = *reinterpret_cast<const f32x4*>(tiles + w * 4 * T::BYTES + r * (D * 4) + (chunk ^ (r & 15)) * 16);
            sum = fmaf(sh_l[w * ROWS + r], c, sum);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = fmaf(v[k], c, x[k]);
        }
        if constexpr (!T::kHalf && RB == 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) zero = fmaf(x[k], 0.f, zero);
        }
        if (whole) {
            const size_t row = chunk_row(e, at.s.t0, at.hk, r0 + r), to = row * D + chunk * 4;
            const bool none = sum == 0.f;
            chunk_write<DT, D>(e, to, none ? 0.f : x[0] / sum, none ? 0.f : x[1] / sum);
            chunk_write<DT, D>(e, to + 2, none ? 0.f : x[2] / sum, none ? 0.f : x[3] / sum);
            if (e.lse && chunk == 0) e.lse[row] = none ? -INFINITY : fmaf(top, e.scale, logf(sum));
        } else {
            *reinterpret_cast<f32x4*>(e.partials + (at.place + r) * D + chunk * 4) = x;
            if (chunk == 0) e.stats[at.place + r] = make_float2(top, sum);
        }
    }
    if constexpr (!T::kHalf && RB == 2) {
        const bool mine = __any(!(zero == 0.f));
        if (lane_anew() == 0) flags[wave] = mine;
        __syncthreads();
        int any = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) any |= flags[w];
        return !any;
    }
    return true;
}

}  // namespace ec
#include "paged_chunk_many.h"
namespace ec {

// MANY: see chunk_share
template <int DT, int D, int WAVES, int MANY>
__global__ __launch_bounds__(WAVES* kWave, (PagedTile<DT, D>::kResident)) void paged_chunk_kernel(ChunkStep first)
{
    using T = PagedTile<DT, D>;
    constexpr int UNIT = WAVES * T::TR, SHORT = kShortUnits * kFewWaves / WAVES;
    __shared__ __align__(256) unsigned char tiles[WAVES * 4 * T::BYTES];  // of every wave: two tiles of K, two of V
    constexpr int SUMS = MANY == 0 ? 6 * kWave : WAVES * 32;  // (64 rows: three parts of two waves)
    __shared__ float sh_m[SUMS], sh_l[SUMS];
    __shared__ int flags[WAVES];
    const int first_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    ChunkSeq s;
    const auto share = chunk_share<MANY, UNIT, SHORT, (DT == EC_F32 || WAVES == kManyWaves), kChunkPlaces<DT, D, WAVES>>(first, s);
    if (blockIdx.x == 0 && first.cut && threadIdx.x < kWave) count_cut_tiles(first, share, s);
    auto take = [&](const ChunkStep& a, const ChunkItem& at, int wave) __attribute__((always_inline)) {
        if (!at.s.live) {
            chunk_nothing<DT, D, WAVES>(a, at, wave);
            return;
        }
        auto by_16 = [&] {
            ChunkItem part = at;
            for (; part.r0 < at.r1; part.r0 += 16, part.place += 16) {
                part.r1 = min(part.r0 + 16, at.r1);
                chunk_few_rows<DT, D, WAVES, 1>(a, part, wave, tiles, sh_m, sh_l, flags);
                __syncthreads();
            }
        };
        if constexpr (DT == EC_BF16) {
            static_assert(sizeof(tiles) >= WAVES * kManySlots * D * 2 && UNIT % kManySlots == 0);
            if (at.s.tile_rows > 32) {
                bool done;
                if (MANY == 0 && at.s.tile_rows == 64) {
                    asm volatile("; tiles of 64 rows" ::: "memory");  // (nothing of one is shared with the other, which would take registers)
                    done = chunk_many_rows<D, WAVES, MANY == 0 ? 2 : 4>(a, at, wave, tiles, sh_m, sh_l, flags, UNIT);
                    asm volatile("; end of tiles of 64 rows" ::: "memory");
                } else {
                    asm volatile("; tiles of 128 rows" ::: "memory");
                    done = chunk_many_rows<D, WAVES, 4>(a, at, wave, tiles, sh_m, sh_l, flags, UNIT);
                    asm volatile("; end of tiles of 128 rows" ::: "memory");
                }
                if (done) return;
                by_16();
                return;
            }
        }
        if constexpr (DT == EC_BF16) {
            if (at.s.tile_rows == 16) chunk_few_rows<DT, D, WAVES, 1>(a, at, wave, tiles, sh_m, sh_l, flags);
            else chunk_few_rows<DT, D, WAVES, 2>(a, at, wave, tiles, sh_m, sh_l, flags);
        } else {
            if (at.s.tile_rows == 16 || !chunk_few_rows<DT, D, WAVES, 2>(a, at, wave, tiles, sh_m, sh_l, flags)) by_16();
        }
    };
    for (int id = blockIdx.x;; id += gridDim.x) {
        const ChunkStep a = chunk_args();
        int wave = first_wave;  // (what follows from it is not kept from item to item)
        asm volatile("" : "+s"(wave));
        if (id != blockIdx.x && a.B <= kWave) s.read<UNIT>(a, lane_anew(), share.many);
        const ChunkItem at = chunk_item(a, share, s, id, wave);
        if (at.b < 0) return;
        take(a, at, wave);
        __syncthreads();  // the tiles have been read
    }
}

// Results of N segments at most, D / 4 lanes a row, all of them on their way at once (4 segments each of 64 tiles of 128 rows 6.2 us, a wave a row 10.1).
template <int DT, int D, int N> __device__ __forceinline__ void join_few(const ChunkStep& a, const CutTile& tile, int row, int step)
{
    constexpr int LANES = D / 4, ROWS = kWave / LANES;
    const int lane = threadIdx.x % kWave, chunk = lane % LANES;
    for (int r = tile.r0 + row * ROWS + lane / LANES; r < tile.r1; r += step * ROWS) {
        const int first = tile.place + (r - tile.r0);
        float2 x[N];
        f32x4 v[N], o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < N; ++g) {
            const size_t at = first + min(g, tile.count - 1) * tile.between;
            x[g] = a.stats[at], v[g] = *reinterpret_cast<const f32x4*>(a.partials + at * D + chunk * 4);
        }
        float top = kLowest, sum = 0.f;
#pragma unroll
        for (int g = 0; g < N; ++g)
            if (!(x[g].y == 0.f)) top = fmaxf(top, x[g].x);  // (NaN counts)
#pragma unroll
        for (int g = 0; g < N; ++g) {
            const float weight = x[g].y == 0.f ? 0.f : exp2f((x[g].x - top) * a.scale_log2e);
            if (g < tile.count) {  // (a segment of which the row sees nothing has sums of 0, one in which it sees scores of -inf only zeros or NaN)
                sum = fmaf(x[g].y, weight, sum);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(v[g][e], weight, o[e]);
            }
        }
        const size_t at = chunk_row(a, tile.t0, tile.hk, r);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = sum == 0.f ? 0.f : o[e] / sum;
        if constexpr (DT == EC_BF16) {
            const uint32_t w0 = (uint32_t)f32_to_bf16(y[0]) | (uint32_t)f32_to_bf16(y[1]) << 16, w1 = (uint32_t)f32_to_bf16(y[2]) | (uint32_t)f32_to_bf16(y[3]) << 16;
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at * D + chunk * 4) = make_uint2(w0, w1);
        } else {
            *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at * D + chunk * 4) = make_float4(y[0], y[1], y[2], y[3]);
        }
        if (a.lse && chunk == 0) a.lse[at] = sum == 0.f ? -INFINITY : fmaf(top, a.scale, logf(sum));
    }
}

// Results of any number of segments, a wave a row: a lane a segment for the statistics, then the sums, eight segments' in flight.
template <int DT, int D> __device__ __forceinline__ void join_many(const ChunkStep& a, const CutTile& tile, int row, int step)
{
    constexpr int E = D / kWave, AHEAD = 8;
    typedef __attribute__((ext_vector_type(E))) float of_row;
    const int lane = threadIdx.x % kWave;
    for (int r = tile.r0 + row; r < tile.r1; r += step) {
        const int first = tile.place + (r - tile.r0);
        float top = kLowest;
        for (int g = lane; g < tile.count; g += kWave) {
            const float2 x = a.stats[first + g * tile.between];
            if (!(x.y == 0.f)) top = fmaxf(top, x.x);  // (NaN counts)
        }
        top = wave_max(top);
        float sum = 0.f;
        of_row o = {};
        for (int g0 = 0; g0 < tile.count; g0 += kWave) {
            float2 x = make_float2(0.f, 0.f);
            if (g0 + lane < tile.count) x = a.stats[first + (g0 + lane) * tile.between];
            const float weight = x.y == 0.f ? 0.f : exp2f((x.x - top) * a.scale_log2e);
            const float share = x.y == 0.f ? 0.f : x.y * weight;
            for (int g = g0; g < min(g0 + kWave, tile.count); g += AHEAD) {
                of_row v[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
                    v[u] = *reinterpret_cast<const of_row*>(a.partials + (size_t)(first + min(g + u, tile.count - 1) * tile.between) * D + lane * E);
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (g + u >= tile.count) continue;
                    const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), g + u - g0));
                    sum += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(share), g + u - g0));
                    // a segment of which the row sees nothing has sums of 0
#pragma unroll
                    for (int e = 0; e < E; ++e) o[e] = fmaf(v[u][e], w, o[e]);
                }
            }
        }
        const size_t at = chunk_row(a, tile.t0, tile.hk, r);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = sum == 0.f ? 0.f : o[e] / sum;
            if constexpr (DT == EC_BF16) static_cast<uint16_t*>(a.out)[at * D + lane * E + e] = f32_to_bf16(x);
            else static_cast<float*>(a.out)[at * D + lane * E + e] = x;
        }
        if (a.lse && lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : fmaf(top, a.scale, logf(sum));
    }
}

// The segments' results of every row of tiles that are cut. Bound by latency: the tile, the statistics and the sums.
template <int DT, int D> __global__ __launch_bounds__(kJoinWaves* kWave) void paged_chunk_join_kernel(ChunkStep a)
{
    constexpr int step = kJoinGroups * kJoinWaves;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    int i = blockIdx.x;
    CutTile tile = a.records[i / kJoinGroups];  // (of nothing where there are fewer tiles)
    for (const int all = *a.cut_tiles * kJoinGroups; i < all;) {
        const int row = i % kJoinGroups * kJoinWaves + wave;
        if (tile.count > 8) join_many<DT, D>(a, tile, row, step);
        else if (tile.count > 4) join_few<DT, D, 8>(a, tile, row, step);
        else if (tile.count > 1) join_few<DT, D, 4>(a, tile, row, step);  // (one: written already)
        i += gridDim.x;
        if (i < all) tile = a.records[i / kJoinGroups];
    }
}

// Workspace: the results of the segments of tiles that are cut (see ChunkShare).
static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
static int part_rows(int T, int H) { return (int)std::min<long long>(((long long)T * H + 15) / 16 * 16, 128); }
// Tiles of all key/value heads that a call can have, and segments whose results its workspace holds: of any number of sequences and of key/value heads.
static long long most_tiles(long long T, long long group, long long Hkv, long long B, int rows) { return (T * group + std::min(B, T) * (rows - 1)) / rows * Hkv; }
static int most_parts(int T, int H) { return most_tiles(T, 1, H, T, 32) >= kChunkTiles ? kChunkParts : kMostPlaces; }
struct ChunkPlaces {  // where things lie in a workspace
    size_t records, stats, partials, end;
    ChunkPlaces(int T, int H, int D)
    {
        const size_t parts = most_parts(T, H), rows = parts * part_rows(T, H);
        records = 256, stats = records + up256(parts * sizeof(CutTile)), partials = stats + up256(rows * sizeof(float2));
        end = partials + rows * D * sizeof(float);
    }
};
size_t paged_chunk_ws(int T, int H, int D) { return ChunkPlaces(T, H, D).end; }

template <int DT, int D> static int launch(ChunkStep a, hipStream_t stream)
{
    constexpr int UNIT = kFewWaves * PagedTile<DT, D>::TR;
    const long long tiles = most_tiles(a.T, a.group, a.Hkv, a.B, DT == EC_F32 ? 32 : 128);
    const bool few = DT == EC_F32 || tiles > kComputeUnits;  // waves
    const int least_rows = DT == EC_F32 ? 32 : few ? 128 : 64;
    const long long least_tiles = most_tiles(a.T, a.group, a.Hkv, a.B, least_rows);
    a.rounds = tiles >= kChunkTiles ? 4 : 1, a.rounds_64 = least_tiles >= kChunkTiles ? 4 : 1;
    const long long seq_tiles = most_tiles(a.T, a.group, a.Hkv, 1, least_rows), units = (a.pages.slots() + UNIT - 1) / UNIT;
    a.small = a.B < 1 << 20 && seq_tiles < 1 << 20 && seq_tiles * a.B * 2 * units < 1 << 29;
    a.cut = units > kShortUnits;  // (the second launch takes longer than shorter sequences)
    // as many workgroups as there can be tiles, and as the chip holds if some may be cut: they go on to further segments where there are more
    auto go = [&](auto waves, auto many) {
        constexpr int W = decltype(waves)::value;
        const long long groups = std::min<long long>(a.cut ? std::max<long long>(tiles, kChunkPlaces<DT, D, W>) : least_tiles, kMostGroups);
        hipLaunchKernelGGL((paged_chunk_kernel<DT, D, W, decltype(many)::value>), dim3((unsigned)groups), dim3(W * kWave), 0, stream, a);
    };
    using Few = std::integral_constant<int, kFewWaves>;
    if constexpr (DT == EC_F32) go(Few{}, std::integral_constant<int, 5>{});
    else if (few) go(Few{}, std::integral_constant<int, 7>{});
    else go(std::integral_constant<int, kManyWaves>{}, std::integral_constant<int, 0>{});
    if (const int rc = status_from_hip(hipGetLastError())) return rc;
    if (!a.cut) return EC_OK;
    const long long joins = std::min<long long>(least_tiles, most_parts(a.T, a.H)) * kJoinGroups;
    hipLaunchKernelGGL((paged_chunk_join_kernel<DT, D>), dim3((unsigned)std::min<long long>(joins, 2048)), dim3(kJoinWaves * kWave), 0, stream, a);
    return status_from_hip(hipGetLastError());
}

int paged_chunk_dispatch(const void* q, const void* k_pages, const void* v_pages, const Pages& pages, const int32_t* start_b, const int32_t* token_start,
                         int B, int T, int H, int Hkv, int D, float scale, int dt, void* out, float* lse, void* ws, hipStream_t stream)
{
    const uint32_t group = H / Hkv;
    auto shift_of = [](uint32_t by) {
        uint32_t shift = 0;
        while (1u << shift < by) ++shift;
        return shift;
    };
    auto mul_of = [&](uint32_t by) { return (uint32_t)(((1ULL << (30 + shift_of(by))) + by - 1) / by); };
    const ChunkPlaces at(T, H, D);
    char* const w = static_cast<char*>(ws);
    const ChunkStep a{q, k_pages, v_pages, out, lse, start_b, token_start, pages, B, T, H, Hkv, (int)group, mul_of(group), shift_of(group),
                      mul_of(Hkv), shift_of(Hkv), 1, 1, false, false, scale, std::min(scale * kLog2e, -kLowest),
                      reinterpret_cast<int*>(w), reinterpret_cast<CutTile*>(w + at.records), part_rows(T, H), reinterpret_cast<float*>(w + at.partials),
                      reinterpret_cast<float2*>(w + at.stats)};
    if (dt == EC_BF16) return D == 128 ? launch<EC_BF16, 128>(a, stream) : launch<EC_BF16, 64>(a, stream);
    return D == 128 ? launch<EC_F32, 128>(a, stream) : launch<EC_F32, 64>(a, stream);
}

}  // namespace ec
