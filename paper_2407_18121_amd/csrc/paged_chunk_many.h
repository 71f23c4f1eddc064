// Attention of up to 128 or 64 rows (tokens times query heads of a key/value head) of a sequence over its pages, bf16: included by paged_chunk.hip.
//
// Four waves, 32 rows each (of 64 rows: two pairs, which take half of a tile's slots each); tiles of 64 slots, K and V in two places each, straight from their pages into LDS. The score tile is computed transposed,
// S^T = K . Q^T, with 32x32x16 instructions, so that a lane owns one row and 16 slots of a block of 32; rounded to bf16 the probabilities are
// the second operand of O^T += V^T . P^T as they stand, V transposed on its way out of LDS. Two phases a tile, each with vector work beside matrix work:
//   A  probabilities of tile i beside the scores of tile i + 1       B  O^T += V^T . P^T of tile i beside the row maximum of tile i + 1
// The probabilities' sum is that of the fp32 numbers; rounding them to bf16, half a step off each, is what keeps the product at one matrix instruction where
// few rows, which are bound by memory, take three: with many rows the matrix pipes are the bound. (In two parts, 16 bits: 2048 tokens behind 65000 rows H40/8 2680
// -> 4076 us, 1024 first tokens of 32 heads 27.0 -> 37.0, 512 behind 768 rows 25.5 -> 29.7; the outputs, rounded to bf16 themselves, are off by 1.66e-3 rms
// instead of 1.67e-3 to 1.70e-3.)
//
// A tile takes two workgroups of a compute unit 3300 cycles of 2048 in the matrix pipe (D128; the pipes of a busy unit work 61 % of the time over
// 65000 rows, H40/8, 2048 tokens: 2.47 to 2.68 ms from card to card, 1.03 to 1.12 PFLOP/s), what remains being the exponentials and the instructions between; a lone workgroup takes 3100. Where a
// batch has fewer tiles than the chip has compute units, a workgroup has eight waves, two groups of four that take turns at the tiles, each with tiles of
// its own in LDS: 4100 cycles a pair (512 tokens behind 768 rows, H32: 41.2 -> 30.9 us); where it has at most half as many, and segments do not make up for
// it, tiles of 64 rows (see many_rows; 30.9 -> 25.1). The sums of a row's parts meet in LDS at the end.
//
// Operands (lane l, half h = l / 32):  A (32 x 16): lane holds A[l % 32][8h .. 8h+7]    B (16 x 32): B[8h .. 8h+7][l % 32]
//                                      C (32 x 32): C[8g + 4h + t][l % 32] in register 4g + t, g,t in 0..3
#pragma once

namespace ec {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kManySlots = 64;   // of a tile
constexpr int kManyAhead = 4;    // LDS fragments requested ahead of the matrix pipe

// Chunk permutations of the LDS tiles: chunk c of row r lies at place c ^ at(r).
template <int D> struct ManySwizzleK {  // operand reads of 16 consecutive rows at one chunk number touch every bank once
    static __device__ __forceinline__ int at(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
};
template <int D> struct ManySwizzleV {  // four rows at the same 64 bytes (a transposed read's half) land in different banks
    static __device__ __forceinline__ int at(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
};

// False, and nothing written: something has come out that is no number.
// sh_m, sh_l: a float a thread of four waves.
template <int D, int WAVES, int QW>
__device__ __forceinline__ bool chunk_many_rows(const ChunkStep& a, const ChunkItem& at, int wave_wg, unsigned char* tiles, float* sh_m, float* sh_l, int* flags, int unit)
{
    constexpr int KS = WAVES / 4;  // groups of four waves that take turns at the tiles
    constexpr int SH = 4 / QW;     // of a group QW waves share the rows, 32 each, and SH the slots of a tile
    constexpr int NB = 2 / SH;     // 32-slot blocks of a wave's share
    constexpr int PARTS = KS * SH;  // sums of every row in a workgroup
    constexpr int ROW = D * 2, CH = ROW / 16, RPI = kWave / CH;  // bytes and chunks of a row, rows of a load instruction
    constexpr int KB = D / 16;    // contraction blocks of Q.K
    constexpr int DB = D / 32;    // 32-row blocks of O^T
    constexpr int NA = NB * KB;      // matrix instructions of phase A: (kb, 32-slot block)
    constexpr int NP = 2 * NB * DB;  // of phase B: (16-slot block, db)
    constexpr int EV = 16 * NB / NA;  // elements turned into probabilities per matrix instruction of phase A
    constexpr int TILE = kManySlots * ROW;
    constexpr int RUNS = 2, IPR = 8 / RPI;  // a wave moves 16 rows of a tile: two runs of 8, each in one page
    constexpr int K0 = 0, K1 = TILE, V0 = 2 * TILE, V1 = 3 * TILE;
    const int lane = lane_anew();
    const int grp = wave_wg / 4, wave = wave_wg % 4, part = grp * SH + wave / QW, rwave = wave % QW;
    const int in_tile = wave / QW * (32 * NB);  // slot of the tile where the wave's share starts
    const int c32 = lane % 32, h = lane / 32;
    const int slots = a.pages.slots(), rw = at.r0 + rwave * 32;  // first row of the workgroup, of this wave
    const int group = a.group, L = at.s.L;

    // tiles of the workgroup, and up to what this wave's rows see
    auto sees = [&](int row) { return min(L + token_of(a, min(row, at.s.rows - 1)), slots - 1); };  // last slot
    const int highest = scalar(sees(at.r0 + QW * 32 - 1));
    const int first = at.segment * at.each, last = min(first + at.each, at.seen);
    if (first >= last) return true;  // a tile that sees fewer segments than its sequence has
    const bool whole = at.each >= at.seen;
    const int t0 = first * (unit / kManySlots), t1 = min(last * (unit / kManySlots), highest / kManySlots + 1), n_iter = (t1 - t0 + KS - 1) / KS;
    auto nth = [&](int i) { return t0 + i * KS + grp; };  // the group's i-th tile
    const int end = min(highest + 1, t1 * kManySlots);  // rows behind it arrive as zeros
    const int lowest = scalar(sees(rw));
    const int count = rw < at.s.rows ? max(min(scalar(sees(rw + 31)) / kManySlots + 1, t1) - t0 - grp + KS - 1, 0) / KS : 0;

    // ------------------------------------------------------------------ rows into LDS
    const uint32_t base = lds_address(tiles) + grp * 4 * TILE;
    const int shift = a.pages.shift, mask = (1 << shift) - 1;
    const uint32_t head_bytes = (uint32_t)ROW << shift, page_bytes = head_bytes * (uint32_t)a.Hkv;
    const int32_t* table = a.pages.table + (size_t)at.b * a.pages.max_pages;
    // A lane's place in the first run that its wave moves; a load instruction further is RPI rows further. K's swizzle turns over with the row number, whose
    // bits that change from instruction to instruction are others than those that change from lane to lane.
    const uint32_t k_part = lane / CH * ROW + (lane % CH ^ ManySwizzleK<D>::at(lane / CH)) * 16;
    const uint32_t v_part = lane / CH * ROW + (lane % CH ^ ManySwizzleV<D>::at(lane / CH)) * 16;
    constexpr int KTURN = (D == 128 ? RPI : RPI / 2) * 16;  // bytes that a chunk's place turns over by
    // entries of a tile's eight runs, one in each of the first eight lanes; what lies behind the table is no slot of anybody
    auto ids_of = [&](int t) __attribute__((always_inline)) { return table[min((t * kManySlots + lane % 8 * 8) >> shift, a.pages.max_pages - 1)]; };
    struct Places {
        uint64_t from[RUNS];
        uint32_t bytes[RUNS], bad;  // bit u: run u of the tile has rows, but no page
    };
    auto places_of = [&](int t, int ids) __attribute__((always_inline)) {
        Places pl;
        const int row = t * kManySlots;
        const bool page = (unsigned)ids < (unsigned)a.pages.n_pages;
        pl.bad = (uint32_t)__ballot(!page && row + lane % 8 * 8 < end) & 0xff;
#pragma unroll
        for (int u = 0; u < RUNS; ++u) {
            const int run = wave * RUNS + u, id = __builtin_amdgcn_readlane(ids, run), r = row + run * 8;
            const bool there = (unsigned)id < (unsigned)a.pages.n_pages;
            pl.bytes[u] = there ? max(min(end - r, 8), 0) * ROW : 0;
            pl.from[u] = (uint64_t)(uint32_t)(there ? id : 0) * page_bytes + (at.hk * head_bytes + (uint32_t)(r & mask) * ROW);
        }
        return pl;
    };
    // run u of the wave's share
    auto move_k = [&](int to, const Places& pl, int u) __attribute__((always_inline)) {
        uint32_t from[IPR];
#pragma unroll
        for (int j = 0; j < IPR; ++j) from[j] = k_part ^ (u * IPR + j) * KTURN;
        load_run_lds<IPR, false>(tile_rsrc(static_cast<const char*>(a.k_pages) + pl.from[u], pl.bytes[u]), base + to + (wave * 16 + u * 8) * ROW, from);
    };
    auto move_v = [&](int to, const Places& pl, int u) __attribute__((always_inline)) {
        uint32_t from[IPR];
#pragma unroll
        for (int j = 0; j < IPR; ++j) from[j] = v_part;
        load_run_lds<IPR, false>(tile_rsrc(static_cast<const char*>(a.v_pages) + pl.from[u], pl.bytes[u]), base + to + (wave * 16 + u * 8) * ROW, from);
    };

    // A wave's 32 rows of queries travel through the place of its own share of the V tiles, 16 rows each
    const uint32_t q_at = base + V0 + wave * (16 * ROW);
    {
        int ids = ids_of(nth(0));
        asm volatile("" : "+v"(ids));
        const int token0 = scalar(token_of(a, min(rw, at.s.rows - 1)));
        const u32x4 q_rsrc = tile_rsrc(static_cast<const char*>(a.q) + (size_t)(at.s.t0 + token0) * a.H * ROW, 0xfffffff0u);
#pragma unroll
        for (int j = 0; j < 32 / RPI; ++j) {
            const int i = j * RPI + lane / CH, row = min(rw + i, at.s.rows - 1), token = token_of(a, row);
            const uint32_t from = ((uint32_t)(token - token0) * a.H + at.hk * group + (row - token * group)) * ROW + (lane % CH ^ ManySwizzleK<D>::at(i)) * 16;
            load_lds_16(q_rsrc, q_at + (j * RPI < 16 ? 0 : TILE - 16 * ROW) + j * RPI * ROW, from);
        }
        const Places pl = places_of(nth(0), ids);
#pragma unroll
        for (int u = 0; u < RUNS; ++u) move_k(K0, pl, u);
    }
    int ids1 = ids_of(nth(0)), ids2 = ids_of(nth(1)), ids3 = ids_of(nth(2));
    // A operand of S^T: row i of a 32-slot block is slot swap23(i) (bits 2 and 3 of i exchanged), so that registers 8G .. 8G+7 of a lane hold the 8
    // consecutive slots 16G + 8h .. +7: the P fragment of a P.V instruction is a run of registers.
    const int krow = (c32 & ~12) | ((c32 & 4) << 1) | ((c32 & 8) >> 1);
    uint32_t k_at[KB / 4];  // byte address of this lane's 16 bytes of contraction blocks 4 i and, turned over, 4 i + 1 .. 3 in tile K0
#pragma unroll
    for (int i = 0; i < KB / 4; ++i) k_at[i] = one_register(base + (in_tile + krow) * ROW + ((8 * i + h) ^ ManySwizzleK<D>::at(krow)) * 16);
    auto k_frag = [&](int kt, int f) __attribute__((always_inline)) {  // f = NB kb + 32-slot block
        const uint32_t from = k_at[f / NB / 4] ^ f / NB % 4 * 32;
        return *(lds_bf16x8*)(uintptr_t)(from + kt + f % NB * 32 * ROW);
    };
    uint32_t v_at[DB];  // of the transposing read: 4 features of one slot
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        const int row = h * 8 + (lane % 16) / 4, chunk = db * 4 + (lane / 16) % 2 * 2 + lane % 4 / 2;
        v_at[db] = one_register(base + (in_tile + row) * ROW + (chunk ^ ManySwizzleV<D>::at(row)) * 16 + lane % 2 * 8);
    }
    auto v_frag = [&](int vt, int g) __attribute__((always_inline)) {  // g = DB * (16-slot block) + db
        const uint32_t src = v_at[g % DB] + vt + g / DB * 16 * ROW;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(uintptr_t)src);
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(uintptr_t)(src + 4 * ROW));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    bf16x8 qf[KB];  // B operand: this lane's row
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
    // m: running maximum of the scores, before their scale, of every tile whose scores have been computed (one tile ahead of o and l, which are already
    // scaled to it); l: this half-wave's share of the row sum
    const float c = a.scale_log2e;
    float m = kLowest, l = 0.f;
    f32x16 sA[NB], sB[NB];
    bf16x8 pf[2 * NB];

    // scores of slots that the row does not see
    auto hide = [&](f32x16 (&s)[NB], int t, uint32_t bad) __attribute__((always_inline)) {
        const int n0 = t * kManySlots + in_tile;
        bad >>= in_tile / 8;
        if (bad || n0 + 32 * NB - 1 > lowest) {
            const int l = anew(lane);  // (a branch, not 64 instructions in every tile, and no register between tiles)
            const int upto = sees(rw + l % 32) - n0 - l / 32 * 8;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (nb * 32 + (r / 8) * 16 + (r % 8) > upto || (bad >> (nb * 4 + r / 8 * 2 + l / 32) & 1)) s[nb][r] = -INFINITY;
        }
    };
    auto raise_max = [&](float mx) __attribute__((always_inline)) {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        const float m_new = fmaxf(m, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
        const float corr = __builtin_amdgcn_exp2f((m - m_new) * c);  // 0 from kLowest to a score
        const bool grew = m_new > m;
        m = m_new;
        l *= corr;
        if (__any(grew)) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[db][r] *= corr;
        }
    };
    auto pin = [&](bf16x8 (&p)[2 * NB]) __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < 2 * NB; ++kk) {
            u32x4 w = __builtin_bit_cast(u32x4, p[kk]);
            asm volatile("" : "+v"(w));
            p[kk] = __builtin_bit_cast(bf16x8, w);
        }
    };
    // Phase A: probabilities of the tile in s (into pf and the row sum) beside sn = K.Q^T of the next one; extra(f) is issued behind the f-th matrix
    // instruction.
    auto phase_a = [&](auto next, f32x16 (&s)[NB], f32x16 (&sn)[NB], int kt, auto&& extra) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);  // of the SIMD's two waves the one with the vector work issues first
        bf16x8 ka[NA];
        if constexpr (next.value) {
#pragma unroll
            for (int f = 0; f < kManyAhead; ++f) ka[f] = k_frag(kt, f);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int r = 0; r < 16; ++r) sn[nb][r] = 0.f;
            __builtin_amdgcn_sched_barrier(0);
        }
        // s c - m c in one step is off by the rounding of m c, 2^-24 |m c|: where that counts (from 2^32 on it would take all weights out of the range),
        // differences first, as everywhere else
        float minus = -m * c;
        if (__builtin_expect(__any(!(fabsf(minus) < 0x1p13f)), 0)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[nb][r] -= m;
            minus = 0.f;
        }
        float x[EV], y[EV], ps[2] = {0.f, 0.f};
#pragma unroll
        for (int f = 0; f < NA + 2; ++f) {
            if constexpr (next.value)
                if (f < NA) {
                    sn[f % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[f], qf[f / NB], sn[f % NB], 0, 0, 0);
                    if (f + kManyAhead < NA) ka[f + kManyAhead] = k_frag(kt, f + kManyAhead);
                }
            extra(f);
            if (f >= 2) {  // third stage of the elements of two instructions ago: sum and round
#pragma unroll
                for (int e = 0; e < EV; ++e) {
                    const int el = (f - 2) * EV + e;
                    ps[e % 2] += y[e];
                    pf[el / 8][el % 8] = (__bf16)y[e];
                }
            }
            if (f >= 1 && f <= NA) {
#pragma unroll
                for (int e = 0; e < EV; ++e) y[e] = __builtin_amdgcn_exp2f(x[e]);
            }
            if (f < NA) {
#pragma unroll
                for (int e = 0; e < EV; ++e) {
                    const int el = f * EV + e;
                    x[e] = fmaf(s[el / 16][el % 16], c, minus);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        l += ps[0] + ps[1];
        asm volatile("" : "+v"(l));
        pin(pf);  // sum and probabilities are formed here, beside the matrix instructions, not where they are used
    };
    // Phase B: O^T += V^T.P^T of the tile in pf beside the row maximum of the scores in sn.
    auto phase_b = [&](auto next, f32x16 (&sn)[NB], int vt) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(0);
        float mx[2] = {-INFINITY, -INFINITY};
        bf16x8 va[NP];
#pragma unroll
        for (int g = 0; g < kManyAhead; ++g) va[g] = v_frag(vt, g);
        __builtin_amdgcn_sched_barrier(0);
        constexpr int MV = 16 * NB / NP;
#pragma unroll
        for (int g = 0; g < NP; ++g) {
            o[g % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[g], pf[g / DB], o[g % DB], 0, 0, 0);
            if (g + kManyAhead < NP) va[g + kManyAhead] = v_frag(vt, g + kManyAhead);
            if constexpr (next.value) {
#pragma unroll
                for (int e = 0; e < MV; e += 2) {
                    const int el = g * MV + e;
                    mx[(e / 2 + g) % 2] = fmaxf(fmaxf(mx[(e / 2 + g) % 2], sn[el / 16][el % 16]), sn[el / 16][el % 16 + 1]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (next.value) raise_max(fmaxf(mx[0], mx[1]));
    };
    wait_loads();  // this wave's queries and its share of the first K tile
    asm volatile("" : "+v"(ids1), "+v"(ids2), "+v"(ids3));
    Places pl1 = places_of(nth(0), ids1), pl2 = places_of(nth(1), ids2);  // of the next V tile and the next K tile but one
    const uint32_t bad = pl1.bad;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
        qf[kb] = *(lds_bf16x8*)(uintptr_t)(q_at + c32 / 16 * TILE + c32 % 16 * ROW + ((2 * kb + h) ^ ManySwizzleK<D>::at(c32)) * 16);
    wait_lds();  // their place is free
#pragma unroll
    for (int u = 0; u < RUNS; ++u) move_v(V0, pl1, u);
#pragma unroll
    for (int u = 0; u < RUNS; ++u) move_k(K1, pl2, u);
    pl1 = pl2;
    pl2 = places_of(nth(2), ids3);
    meet();
    if (count > 0) {  // scores of the first tile
        bf16x8 ka[NA];
#pragma unroll
        for (int f = 0; f < NA; ++f) ka[f] = k_frag(K0, f);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int r = 0; r < 16; ++r) sA[nb][r] = 0.f;
#pragma unroll
        for (int f = 0; f < NA; ++f) sA[f % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[f], qf[f / NB], sA[f % NB], 0, 0, 0);
        hide(sA, nth(0), bad);
        float mx = -INFINITY;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sA[nb][r]);
        raise_max(mx);
    }
    // One tile with a successor: K of tile i + 1 and V of tile i have landed; K of tile i + 2 goes where K of tile i was, V of tile i + 1 where V of tile
    // i - 1 was, both read for the last time before the barrier.
    // With scalar loads on their way (what the arguments are read by) the compiler could not tell LDS reads apart by their number: there are none from here on.
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    int ids = 0;
    auto body = [&](int i, f32x16 (&s)[NB], f32x16 (&sn)[NB], int k_old, int k_next, int v_cur, int v_next) __attribute__((always_inline)) {
        tile_barrier();
        if (i > 0) {
            asm volatile("" : "+v"(ids));
            pl1 = pl2, pl2 = places_of(nth(i + 2), ids);
        }
        ids = ids_of(nth(i + 3));
        phase_a(std::true_type{}, s, sn, k_next, [&](int f) __attribute__((always_inline)) {
            constexpr int EVERY = NA / (2 * RUNS);
            static_assert(EVERY >= 1, "a phase has room for its loads");
            if (f < NA && f % EVERY == 0) {
                if (f / EVERY < RUNS) move_k(k_old, pl2, f / EVERY);  // (behind the last tile nothing is fetched)
                else move_v(v_next, pl1, f / EVERY - RUNS);
            }
        });
        hide(sn, nth(i + 1), pl1.bad);
        phase_b(std::true_type{}, sn, v_cur);
    };
    int i = 0;
    for (; i + 2 < count; i += 2) {
        body(i, sA, sB, K0, K1, V0, V1);
        body(i + 1, sB, sA, K1, K0, V1, V0);
    }
    const bool odd = i + 1 < count;
    if (odd) {
        body(i, sA, sB, K0, K1, V0, V1);
        ++i;
    }
    // the wave's last tile, then nothing but its share of the loads that other waves still need
    for (bool work = i < count; i < n_iter; ++i, work = false) {
        tile_barrier();
        if (i > 0) {
            asm volatile("" : "+v"(ids));
            pl1 = pl2, pl2 = places_of(nth(i + 2), ids);
        }
        ids = ids_of(nth(i + 3));
        const bool even = i % 2 == 0;
        if (i + 2 < n_iter) {
#pragma unroll
            for (int u = 0; u < RUNS; ++u) move_k(even ? K0 : K1, pl2, u);
        }
        if (i + 1 < n_iter) {
#pragma unroll
            for (int u = 0; u < RUNS; ++u) move_v(even ? V1 : V0, pl1, u);
        }
        if (work) {
            if (odd) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) sA[nb] = sB[nb];
            }
            phase_a(std::false_type{}, sA, sB, K0, [](int) {});
            phase_b(std::false_type{}, sB, even ? V0 : V1);
        }
    }
    // An infinite V has reached the rows that do not see it too, as 0 times infinity. Where anything has come out that is no number the rows are left to
    // chunk_few_rows, which takes care of it.
    float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) zero[r % 4] = fmaf(o[db][r], 0.f, zero[r % 4]);
    const bool mine = __any(!((zero[0] + zero[1]) + (zero[2] + zero[3]) == 0.f));
    if (lane == 0) flags[wave_wg] = mine;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) any |= flags[w];
    if (any) return false;
    if constexpr (PARTS > 1) {
        // All parts of a row but the first hand their sums over through the tiles, at their end: the start is where the results leave through. Four words j of
        // lane t lie at 16 (j * 64 + t): consecutive lanes, consecutive addresses.
        constexpr int WORDS = DB * 4 * kWave;  // of 16 bytes
        static_assert((PARTS - 1) * QW * WORDS * 16 + QW * TILE <= KS * 4 * TILE);
        f32x4* sums = reinterpret_cast<f32x4*>(tiles + KS * 4 * TILE) - (PARTS - 1) * QW * WORDS;
        auto of_part = [&](int p) { return ((p - 1) * QW + rwave); };
        if (part) {
            const int at = of_part(part);
            sh_m[at * kWave + lane] = m, sh_l[at * kWave + lane] = l;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g) sums[at * WORDS + (db * 4 + g) * kWave + lane] = f32x4{o[db][g * 4], o[db][g * 4 + 1], o[db][g * 4 + 2], o[db][g * 4 + 3]};
        }
        __syncthreads();
        if (part) return true;
        float top = m;
#pragma unroll
        for (int p = 1; p < PARTS; ++p) top = fmaxf(top, sh_m[of_part(p) * kWave + lane]);
        const float f0 = __builtin_amdgcn_exp2f((m - top) * c);
        l *= f0;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[db][r] *= f0;
#pragma unroll
        for (int p = 1; p < PARTS; ++p) {
            const int at = of_part(p);
            const float f = __builtin_amdgcn_exp2f((sh_m[at * kWave + lane] - top) * c);
            l = fmaf(sh_l[at * kWave + lane], f, l);
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 y = sums[at * WORDS + (db * 4 + g) * kWave + lane];
#pragma unroll
                    for (int t = 0; t < 4; ++t) o[db][g * 4 + t] = fmaf(y[t], f, o[db][g * 4 + t]);
                }
        }
        m = top;
    }
    if (rw >= at.s.rows) return true;

    const ChunkStep e = chunk_args();
    const int el = anew(lane), ec = el % 32, eh = el / 32;  // lane, row and half of the way out
    const float sum = l + __shfl_xor(l, 32, kWave);
    const int row = rw + ec;
    if (!whole) {
        // The accumulators hold 16-byte pieces of 32 rows: turned through this wave's quarter of the tiles, which nobody reads any more, so that a store
        // instruction writes a stretch of 1 KB (two segments each of 128 tiles of 128 rows 38.5 -> 30.2 us with the join).
        constexpr int CHUNKS = D / 4, RPS = kWave / CHUNKS;  // 16-byte chunks of a row, rows per store instruction
        static_assert(32 * D * 4 <= TILE);
        const uint32_t stage = base + wave * TILE;
        const size_t place = at.place + wave * 32;
        if (eh == 0 && row < at.s.rows) e.stats[place + ec] = make_float2(m, sum);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 y;
#pragma unroll
                for (int t = 0; t < 4; ++t) y[t] = o[db][g * 4 + t];
                *(lds_f32x4*)(uintptr_t)(stage + ec * (D * 4) + ((db * 8 + g * 2 + eh) ^ (ec & 7)) * 16) = y;
            }
#pragma unroll
        for (int j = 0; j < 32 / RPS; ++j) {
            const int r = j * RPS + el / CHUNKS;
            const f32x4 y = *(lds_f32x4*)(uintptr_t)(stage + r * (D * 4) + ((el % CHUNKS) ^ (r & 7)) * 16);
            if (rw + r < at.s.rows) *reinterpret_cast<f32x4*>(e.partials + (place + r) * D + el % CHUNKS * 4) = y;
        }
        return true;
    }
    if (e.lse && eh == 0 && row < at.s.rows) e.lse[chunk_row(e, at.s.t0, at.hk, row)] = sum == 0.f ? -INFINITY : fmaf(m, e.scale, logf(sum));
    // The accumulators hold 8-byte pieces of 32 rows per register pair. Half a row at a time they are turned through this wave's share of tile K1 (every
    // wave has read K for the last time), so that a store instruction writes whole stretches of a row.
    constexpr int HC = D / 16;        // 16-byte chunks in half a row
    constexpr int RPS = kWave / HC;   // rows per store instruction
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const uint32_t stage = base + K1 + wave * (16 * ROW);
    auto place = [&](int r, int chunk) { return r * (HC * 16) + (chunk ^ (D == 128 ? r & 7 : (r >> 2) & 3)) * 16; };
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int d2 = 0; d2 < DB / 2; ++d2)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                bf16x4 y;
#pragma unroll
                for (int t = 0; t < 4; ++t) y[t] = (__bf16)(o[half * (DB / 2) + d2][g * 4 + t] * inv);
                *(lds_bf16x4*)(uintptr_t)(stage + place(ec, d2 * 4 + g) + eh * 8) = y;
            }
#pragma unroll
        for (int j = 0; j < 32 / RPS; ++j) {
            const int r = j * RPS + el / HC;
            const u32x4 y = __builtin_bit_cast(u32x4, *(lds_bf16x8*)(uintptr_t)(stage + place(r, el % HC)));
            if (rw + r < at.s.rows)
                *reinterpret_cast<u32x4*>(static_cast<char*>(e.out) + chunk_row(e, at.s.t0, at.hk, rw + r) * ROW + half * (ROW / 2) + el % HC * 16) = y;
        }
    }
    return true;
}

}  // namespace ec
