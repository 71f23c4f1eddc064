// ec_paged_rotary_store: queries and keys of new tokens turned by their positions, keys and values into the pages.
//
// Pair i of a head, elements (x, y), becomes m (x cos a - y sin a, y cos a + x sin a) with a = position * freq_i: the position is an integer and the
// frequency an fp32 number, so that their product and its part beyond whole turns are formed in 64 bits and are right for every position;
// what is left, an eighth of a turn at most, goes through the sine and cosine of fp32. A token's angles are computed once for all its heads.
// Bound by its bytes, every one of which is read once and written once.
#include "paged.h"

namespace ec {

constexpr int kRotaryThreads = 256;

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

// A workgroup takes a token, a thread two 16-byte chunks of a head at a time: where halves are paired, the two that belong together.
// WHOLE: pairs lie in whole chunks (always, where neighbours are paired); else the other half of a pair is read element by element.
template <int DT, int D, bool NEIGHBOURS, bool WHOLE>
__global__ __launch_bounds__(kRotaryThreads) void paged_rotary_kernel(Rotary a)
{
    constexpr int V = Elem<DT>::kPerChunk, E = Elem<DT>::kBytes, CH = D / V, ITEMS = CH / 2;
    using Word = typename Elem<DT>::type;
    __shared__ float2 turns[D / 2];
    const int t = blockIdx.x, tid = threadIdx.x;
    const int64_t row = a.rows[t];
    if (row < 0 || row >= a.n_rows) return;  // no token
    const int pos = a.pos[t], half = a.rot / 2;
    if (tid < half) turns[tid] = turn_of(pos, a.freq[tid], a.mscale);
    const int64_t page = row >> a.shift;
    const int in_page = (int)(row & ((1 << a.shift) - 1));
    for (int g = tid; g < a.G; g += kRotaryThreads) {
        const size_t at = ((size_t)(page * a.G + g) << a.shift) + in_page;
        if (a.pos_pages) a.pos_pages[at] = pos;
        if (a.mass_pages) a.mass_pages[at] = 0.f;
    }
    __syncthreads();
    const int pairs = NEIGHBOURS || !WHOLE ? 0 : half / V;  // of chunks that are turned together
    auto value = [](Word w) {
        if constexpr (DT == EC_BF16) return bf16_to_f32(w);
        else return w;
    };
    for (int i = tid; i < (a.H + 2 * a.Hkv) * ITEMS; i += kRotaryThreads) {
        const int head = i / ITEMS, item = i % ITEMS;
        const bool is_q = head < a.H, is_k = !is_q && head < a.H + a.Hkv;
        const int h = is_q ? head : is_k ? head - a.H : head - a.H - a.Hkv;
        const char* from = static_cast<const char*>(is_q ? a.q : is_k ? a.k : a.v) + (int64_t)t * (is_q ? a.q_step : is_k ? a.k_step : a.v_step) + (int64_t)h * (D * E);
        char* to = static_cast<char*>(is_q ? a.q_out : is_k ? a.k_pages : a.v_pages) +
                   (is_q ? (size_t)t * a.H + h : ((size_t)(page * a.Hkv + h) << a.shift) + in_page) * (D * E);
        const int turned = is_q || is_k ? pairs : 0;
        const int lo = item < turned ? item : 2 * item, hi = item < turned ? item + turned : lo + 1;
        uint4 x = reinterpret_cast<const uint4*>(from)[lo], y = reinterpret_cast<const uint4*>(from)[hi];
        if ((is_q || is_k) && (!WHOLE || NEIGHBOURS ? lo * V < a.rot : item < turned)) {
            float u[V], w[V];
            unpack<DT>(x, u);
            unpack<DT>(y, w);
            if constexpr (NEIGHBOURS) {
                auto turn = [&](float* f, int d) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 0; e < V; e += 2)
                        if (d + e < a.rot) {
                            const float2 r = turns[(d + e) / 2];
                            const float p = f[e], q = f[e + 1];
                            f[e] = p * r.x - q * r.y, f[e + 1] = q * r.x + p * r.y;
                        }
                };
                turn(u, lo * V);
                turn(w, hi * V);
            } else if constexpr (WHOLE) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 r = turns[lo * V + e];
                    const float p = u[e], q = w[e];
                    u[e] = p * r.x - q * r.y, w[e] = q * r.x + p * r.y;
                }
            } else {
                auto turn = [&](float* f, int d) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (d + e < a.rot) {
                            const bool second = d + e >= half;
                            const float other = value(reinterpret_cast<const Word*>(from)[second ? d + e - half : d + e + half]);
                            const float2 r = turns[second ? d + e - half : d + e];
                            f[e] = f[e] * r.x + (second ? other : -other) * r.y;
                        }
                };
                turn(u, lo * V);
                turn(w, hi * V);
            }
            x = pack<DT>(u), y = pack<DT>(w);
        }
        reinterpret_cast<uint4*>(to)[lo] = x;
        reinterpret_cast<uint4*>(to)[hi] = y;
    }
}

template <int DT, int D> static void launch(const Rotary& a, bool neighbours, hipStream_t stream)
{
    const dim3 grid(a.T), block(kRotaryThreads);
    if (neighbours)
        hipLaunchKernelGGL((paged_rotary_kernel<DT, D, true, true>), grid, block, 0, stream, a);
    else if (a.rot / 2 % Elem<DT>::kPerChunk == 0)
        hipLaunchKernelGGL((paged_rotary_kernel<DT, D, false, true>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((paged_rotary_kernel<DT, D, false, false>), grid, block, 0, stream, a);
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
