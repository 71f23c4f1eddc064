// ec_paged_rotary_store: queries and keys of new tokens turned by their positions, keys and values into the pages.
//
// Pair i of a head, elements (x, y), becomes m (x cos a - y sin a, y cos a + x sin a) with a = position * freq_i: the position is an integer and the
// frequency an fp32 number, so that their product and its part beyond whole turns are formed in 64 bits and are right for every position;
// what is left, an eighth of a turn at most, goes through the sine and cosine of fp32. A token's angles are computed once for all its heads.
// Bound by its bytes, every one of which is read once and written once (8192 tokens H32/8 D128 bf16, 200 MB: 31 us, 6.4 TB/s); few tokens by the latency of a
// row number, a position, 64-bit products and a sine behind one another (16 tokens 4.5 us).
#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace ec {

constexpr int kRotaryThreads = 256, kRotaryTokens = 8;  // kRotaryTokens: of a workgroup, at most

struct Rotary {
    const void *q, *k, *v;
    int64_t q_step, k_step, v_step;  // bytes from token to token
    const int32_t* pos;
    const int64_t* rows;
    const float* freq;
    float mscale;
    int rot, T, H, Hkv, G, shift;
    int64_t n_rows;  // of the pools
    void *q_out, *k_pages, *v_pages;
    int32_t* pos_pages;
    float* mass_pages;
};

// m * (cos, sin) of pos * freq
__device__ __forceinline__ float2 turn_of(int pos, float freq, float m)
{
    const double turns = (double)pos * (double)freq * 0.15915494309189533577;  // / 2 pi
    const double quarters = rint(4.0 * turns), rest = fma(-0.25, quarters, turns);
    float s, c;
    sincospif(2.f * (float)rest, &s, &c);
    const int quarter = (int)fma(-4.0, floor(0.25 * quarters), quarters);  // 0 .. 3
    const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
    return make_float2(quarter == 1 || quarter == 2 ? -m * x : m * x, quarter & 2 ? -m * y : m * y);
}

// A workgroup takes a token (ONE) or `each` of them, a thread two 16-byte chunks of a head at a time: where halves are paired, the two that belong together.
// WHOLE: pairs lie in whole chunks (always, where neighbours are paired); else the other half of a pair is fetched from LDS, element by element (bf16 T8192
// H32/8 D128, 94 elements turned, read from memory that way: 63.6 us).
template <int DT, int D, bool NEIGHBOURS, bool WHOLE, bool ONE>
__global__ __launch_bounds__(kRotaryThreads) void paged_rotary_kernel(Rotary a, int each)
{
    constexpr int V = Elem<DT>::kPerChunk, E = Elem<DT>::kBytes, CH = D / V, ITEMS = CH / 2;
    using Word = typename Elem<DT>::type;
    constexpr int TOKENS = ONE ? 1 : kRotaryTokens;
    __shared__ float2 turns[TOKENS][D / 2];
    __shared__ int64_t row_of[TOKENS];
    __shared__ __align__(16) Word rows[WHOLE ? 1 : kRotaryThreads * 2 * V];
    const int t0 = ONE ? blockIdx.x : blockIdx.x * each, tid = threadIdx.x, half = a.rot / 2, count = ONE ? 1 : min(each, a.T - t0);
    auto is_row = [&](int64_t row) { return row >= 0 && row < a.n_rows; };
    const int64_t only = ONE ? a.rows[t0] : 0;
    if (ONE && !is_row(only)) return;  // no token
    for (int i = tid; i < count * half; i += kRotaryThreads) {
        const int t = ONE ? 0 : i / half;
        turns[t][i - t * half] = turn_of(a.pos[t0 + t], a.freq[i - t * half], a.mscale);
    }
    for (int i = tid; i < count * a.G; i += kRotaryThreads) {
        const int t = ONE ? 0 : i / a.G, g = i - t * a.G;
        const int64_t row = ONE ? only : a.rows[t0 + t];
        if (!ONE && g == 0) row_of[t] = is_row(row) ? row : -1;
        if (!is_row(row)) continue;  // no token
        const size_t at = ((size_t)((row >> a.shift) * a.G + g) << a.shift) + (row & ((1 << a.shift) - 1));
        if (a.pos_pages) a.pos_pages[at] = a.pos[t0 + t];
        if (a.mass_pages) a.mass_pages[at] = 0.f;
    }
    __syncthreads();
    const int pairs = NEIGHBOURS || !WHOLE ? 0 : half / V;  // of chunks that are turned together
    const int heads = a.H + 2 * a.Hkv, all = count * heads * ITEMS;
    for (int i0 = 0; i0 < all; i0 += kRotaryThreads) {
        const int i = min(i0 + tid, all - 1), t = ONE ? 0 : i / (heads * ITEMS), in = i - t * (heads * ITEMS), head = in / ITEMS, item = in % ITEMS;
        const int64_t row = ONE ? only : row_of[t];
        const bool live = i0 + tid < all && row >= 0;
        const bool is_q = head < a.H, is_k = !is_q && head < a.H + a.Hkv;
        const int h = is_q ? head : is_k ? head - a.H : head - a.H - a.Hkv;
        const char* from = static_cast<const char*>(is_q ? a.q : is_k ? a.k : a.v) + (int64_t)(t0 + t) * (is_q ? a.q_step : is_k ? a.k_step : a.v_step) +
                           (int64_t)h * (D * E);
        const int64_t page = row >> a.shift;
        char* to = static_cast<char*>(is_q ? a.q_out : is_k ? a.k_pages : a.v_pages) +
                   (is_q ? (size_t)(t0 + t) * a.H + h : ((size_t)(page * a.Hkv + h) << a.shift) + (row & ((1 << a.shift) - 1))) * (D * E);
        const int turned = is_q || is_k ? pairs : 0;
        const int lo = item < turned ? item : 2 * item, hi = item < turned ? item + turned : lo + 1;
        uint4 x = make_uint4(0, 0, 0, 0), y = x;
        if (live) x = reinterpret_cast<const uint4*>(from)[lo], y = reinterpret_cast<const uint4*>(from)[hi];
        if constexpr (!WHOLE) {
            uint4* mine = reinterpret_cast<uint4*>(rows) + tid * 2;  // the heads of a pass lie one behind the other
            mine[0] = x, mine[1] = y;
            __syncthreads();
        }
        if ((is_q || is_k) && (!WHOLE || NEIGHBOURS ? lo * V < a.rot : item < turned)) {
            float u[V], w[V];
            unpack<DT>(x, u);
            unpack<DT>(y, w);
            if constexpr (NEIGHBOURS) {
                auto turn = [&](float* f, int d) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 0; e < V; e += 2)
                        if (d + e < a.rot) {
                            const float2 r = turns[t][(d + e) / 2];
                            const float p = f[e], q = f[e + 1];
                            f[e] = p * r.x - q * r.y, f[e + 1] = q * r.x + p * r.y;
                        }
                };
                turn(u, lo * V);
                turn(w, hi * V);
            } else if constexpr (WHOLE) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 r = turns[t][lo * V + e];
                    const float p = u[e], q = w[e];
                    u[e] = p * r.x - q * r.y, w[e] = q * r.x + p * r.y;
                }
            } else {
                auto value = [](Word w) {
                    if constexpr (DT == EC_BF16) return bf16_to_f32(w);
                    else return w;
                };
                const Word* others = rows + tid / ITEMS * D;  // the head that this thread's chunks are of
                auto turn = [&](float* f, int d) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (d + e < a.rot) {
                            const bool second = d + e >= half;
                            const int other = second ? d + e - half : d + e + half;
                            const float2 r = turns[t][second ? other : d + e];
                            const float v = value(others[other]);
                            f[e] = f[e] * r.x + (second ? v : -v) * r.y;
                        }
                };
                turn(u, lo * V);
                turn(w, hi * V);
            }
            x = pack<DT>(u), y = pack<DT>(w);
        }
        if (live) {
            reinterpret_cast<uint4*>(to)[lo] = x;
            reinterpret_cast<uint4*>(to)[hi] = y;
        }
        if constexpr (!WHOLE) __syncthreads();
    }
}

template <int DT, int D> static void launch(const Rotary& a, bool neighbours, hipStream_t stream)
{
    // a token a workgroup, unless that leaves most of its threads without work, and the chip's compute units have four workgroups each all the same, or makes 2^32
    // threads, more than a launch can have
    const int items = (a.H + 2 * a.Hkv) * (D / Elem<DT>::kPerChunk / 2);
    const int each = std::max(1 + (a.T >> 24), std::min({kRotaryTokens, 2 * kRotaryThreads / items, a.T / (4 * kComputeUnits)}));
    const dim3 grid((a.T + each - 1) / each), block(kRotaryThreads);
    auto go = [&](auto pairs, auto whole) {
        if (each == 1) hipLaunchKernelGGL((paged_rotary_kernel<DT, D, pairs.value, whole.value, true>), grid, block, 0, stream, a, 1);
        else hipLaunchKernelGGL((paged_rotary_kernel<DT, D, pairs.value, whole.value, false>), grid, block, 0, stream, a, each);
    };
    if (neighbours) go(std::true_type{}, std::true_type{});
    else if (a.rot / 2 % Elem<DT>::kPerChunk == 0) go(std::false_type{}, std::true_type{});
    else go(std::false_type{}, std::false_type{});
}

int paged_rotary_dispatch(const void* q, const void* k, const void* v, int64_t q_step, int64_t k_step, int64_t v_step, const int32_t* pos,
                          const int64_t* rows, const float* freq, float mscale, int rot, bool neighbours, int T, int H, int Hkv, int G, int D, int page_shift,
                          int n_pages, int dt, void* q_out, void* k_pages, void* v_pages, int32_t* pos_pages, float* mass_pages, hipStream_t stream)
{
    const Rotary a{q, k, v, q_step, k_step, v_step, pos, rows, freq, mscale, rot, T, H, Hkv, G, page_shift, (int64_t)n_pages << page_shift,
                   q_out, k_pages, v_pages, pos_pages, mass_pages};
    if (dt == EC_BF16) D == 128 ? launch<EC_BF16, 128>(a, neighbours, stream) : launch<EC_BF16, 64>(a, neighbours, stream);
    else D == 128 ? launch<EC_F32, 128>(a, neighbours, stream) : launch<EC_F32, 64>(a, neighbours, stream);
    return status_from_hip(hipGetLastError());
}

}  // namespace ec
