// Tiles of a few rows of K and V that a wave moves from their pages into its own part of the LDS, and what the kernels that multiply them by up to 16
// queries at a time share.
#pragma once

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

// N load instructions of consecutive rows into consecutive LDS (see load_lds_16): the instruction's offset moves both by 1 KB. The non-temporal hint
// keeps data that is read once from displacing cache lines (B16 H32 870 rows 39.0 us a step, 44.1 without; one cache of 131071 rows 89.3, 100.5).
#define EC_LOAD_RUN(HINT)                                                                                                                              \
    if constexpr (N == 1)                                                                                                                              \
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen" HINT " lds" ::"s"(lds), "v"(offset[0]), "s"(rsrc) : "memory"); \
    else if constexpr (N == 2)                                                                                                                         \
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %3, 0 offen" HINT " lds\n\t"                                             \
                     "buffer_load_dwordx4 %2, %3, 0 offen offset:1024" HINT " lds" ::"s"(lds), "v"(offset[0]), "v"(offset[1]), "s"(rsrc) : "memory");  \
    else                                                                                                                                               \
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %5, 0 offen" HINT " lds\n\t"                                             \
                     "buffer_load_dwordx4 %2, %5, 0 offen offset:1024" HINT " lds\n\tbuffer_load_dwordx4 %3, %5, 0 offen offset:2048" HINT " lds\n\t"    \
                     "buffer_load_dwordx4 %4, %5, 0 offen offset:%6" HINT " lds"                                                                       \
                     ::"s"(lds), "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "s"(rsrc), "n"(3 * 1024) : "memory")
template <int N, bool ONCE = true> __device__ __forceinline__ void load_run_lds(u32x4 rsrc, uint32_t lds, const uint32_t* offset)
{
    if constexpr (ONCE) {
        EC_LOAD_RUN(" nt");
    } else {
        EC_LOAD_RUN("");
    }
}
#undef EC_LOAD_RUN

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

constexpr float kSmallExponent = -100.f, kSmall = 0x1p-100f;  // probabilities below it are looked at apart

// Probabilities of a lane, 4 of every block of 16 rows, as sums of three bf16 numbers each, their 24 bits cut into eights (what is left is not negative); none
// of those of one of kSmall and more is 0, so that an infinite V stays infinite: 2^-24 and 2^-25 of it at least, less than its last bit.
template <int BLOCKS> struct WeightParts {
    static constexpr int N = BLOCKS * 4;
    typedef __attribute__((ext_vector_type(N))) __bf16 bf16xn;
    bf16xn of[3];
    __device__ __forceinline__ void set(int e, float x)
    {
        auto cut = [](float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); };
        const float high = cut(x), rest = x - high, middle = cut(rest);
        of[0][e] = (__bf16)high;
        of[1][e] = (__bf16)fmaxf(middle, x * 0x1p-24f);
        of[2][e] = (__bf16)fmaxf(rest - middle, x * 0x1p-25f);
    }
    // x + V^T . P^T of 16 features, P one of the parts
    static __device__ __forceinline__ f32x4 multiply(const bf16x4 (&v)[BLOCKS], const bf16xn& part, f32x4 x)
    {
        if constexpr (BLOCKS == 2)
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7), part, x, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, v[0]), __builtin_bit_cast(s16x4, part), x, 0, 0, 0);
    }
};

__device__ __forceinline__ int divided(int x, int by)  // 0 <= x < 2^24, by > 0
{
    const int q = (int)((float)x * __builtin_amdgcn_rcpf((float)by)), r = x - q * by;
    return q + (r >= by) - (r < 0);
}
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

}  // namespace ec
