// ec_paged_decode_step, ec_paged_decode_score_step: attention of one new token per sequence over a cache in pages.
#include "paged.h"

namespace ec {

struct PagedStep {
    const void *q, *k_new, *v_new;
    void *k_pages, *v_pages, *out;
    int32_t* pos_pages;
    const int32_t *len_b, *new_pos_b;
    Pages pages;
    int B, H, Hkv, G;
    float scale;
    float *raw, *lse;  // EMIT: [B,H,slots] scaled scores, [B,H] log of the softmax denominators
};

template <int DT> __device__ __forceinline__ float load_elem(const void* p, size_t i)
{
    if constexpr (DT == EC_F32) return static_cast<const float*>(p)[i];
    else return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}
template <int DT> __device__ __forceinline__ void store_elem(void* p, size_t i, float x)
{
    if constexpr (DT == EC_F32) static_cast<float*>(p)[i] = x;
    else static_cast<uint16_t*>(p)[i] = f32_to_bf16(x);
}

// One workgroup per (sequence, query head); a wave takes every fourth row, a lane D / 64 features of it.
template <int DT, int D, bool EMIT> __global__ __launch_bounds__(256) void paged_step_kernel(PagedStep a)
{
    constexpr int E = D / kWave, WAVES = 4;
    __shared__ float sh_m[WAVES], sh_l[WAVES], sh_o[WAVES][D];
    const int b = blockIdx.x / a.H, h = blockIdx.x % a.H, g = a.H / a.Hkv, hk = h / g;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const size_t out_at = ((size_t)b * a.H + h) * D;
    const int n = a.len_b[b];
    if (n < 0 || n >= a.pages.slots()) {  // no sequence in this place
        if (threadIdx.x < D) store_elem<DT>(a.out, out_at + threadIdx.x, 0.f);
        return;
    }
    const size_t new_at = ((size_t)b * a.Hkv + hk) * D;
    float q[E], o[E] = {}, m = kLowest, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = load_elem<DT>(a.q, out_at + lane + e * kWave);
    for (int j = wave; j <= n; j += WAVES) {
        const void *k = a.k_new, *v = a.v_new;
        size_t at = new_at;
        if (j < n) {
            const int id = a.pages.page_of(b, j);
            if (id < 0) {
                if (EMIT && lane == 0) a.raw[((size_t)b * a.H + h) * a.pages.slots() + j] = -INFINITY;
                continue;
            }
            k = a.k_pages, v = a.v_pages, at = a.pages.row(id, a.Hkv, hk, j) * D;
        }
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s = fmaf(q[e], load_elem<DT>(k, at + lane + e * kWave), s);
        s = group_sum<kWave>(s) * a.scale;
        if (EMIT && lane == 0) a.raw[((size_t)b * a.H + h) * a.pages.slots() + j] = s;
        const float m_new = fmaxf(m, s), c = expf(m - m_new), p = expf(s - m_new);
        m = m_new, l = l * c + p;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * c + p * load_elem<DT>(v, at + lane + e * kWave);
    }
    if (lane == 0) sh_m[wave] = m, sh_l[wave] = l;
#pragma unroll
    for (int e = 0; e < E; ++e) sh_o[wave][lane + e * kWave] = o[e];
    __syncthreads();
    if (threadIdx.x < D) {
        float top = sh_m[0], sum = 0.f, x = 0.f;
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, sh_m[w]);
        for (int w = 0; w < WAVES; ++w) {
            const float c = expf(sh_m[w] - top);
            sum += sh_l[w] * c, x += sh_o[w][threadIdx.x] * c;
        }
        store_elem<DT>(a.out, out_at + threadIdx.x, x / sum);
        if (EMIT && threadIdx.x == 0) a.lse[(size_t)b * a.H + h] = top + logf(sum);
    }
    if (h % g == 0) {  // the new row; nobody reads it in this launch
        const int id = a.pages.page_of(b, n);
        if (id >= 0 && threadIdx.x < D) {
            const size_t at = a.pages.row(id, a.Hkv, hk, n) * D + threadIdx.x;
            store_elem<DT>(a.k_pages, at, load_elem<DT>(a.k_new, new_at + threadIdx.x));
            store_elem<DT>(a.v_pages, at, load_elem<DT>(a.v_new, new_at + threadIdx.x));
        }
        if (id >= 0 && threadIdx.x == 0 && a.pos_pages && (a.G > 1 || hk == 0)) a.pos_pages[a.pages.row(id, a.G, a.G > 1 ? hk : 0, n)] = a.new_pos_b[b];
    }
}

// mass of every row += the mean of its group's probabilities; a thread a row, heads in ascending order.
__global__ __launch_bounds__(256) void paged_mass_kernel(const float* __restrict__ raw, const float* __restrict__ lse, float* mass_pages,
                                                         const int32_t* __restrict__ len_b, Pages pages, int H, int G)
{
    const int b = blockIdx.y / G, g = blockIdx.y % G, n = len_b[b];
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (n < 0 || n >= pages.slots() || j > n) return;
    const int id = pages.page_of(b, j);
    if (id < 0) return;
    const int heads = H / G;
    float sum = 0.f;
    for (int h = g * heads; h < (g + 1) * heads; ++h) sum += expf(raw[((size_t)b * H + h) * pages.slots() + j] - lse[(size_t)b * H + h]);
    float* m = mass_pages + pages.row(id, G, g, j);
    *m = (j == n ? 0.f : *m) + sum / (float)heads;
}

size_t paged_step_ws(int B, int H, int slots, bool emit)
{
    if (!emit) return 256;
    return (((size_t)B * H * slots * 4 + 255) & ~(size_t)255) + (((size_t)B * H * 4 + 255) & ~(size_t)255);
}

template <int DT, int D> static int launch(const PagedStep& a, float* mass_pages, hipStream_t stream)
{
    if (!mass_pages) {
        hipLaunchKernelGGL((paged_step_kernel<DT, D, false>), dim3(a.B * a.H), dim3(256), 0, stream, a);
        return status_from_hip(hipGetLastError());
    }
    hipLaunchKernelGGL((paged_step_kernel<DT, D, true>), dim3(a.B * a.H), dim3(256), 0, stream, a);
    if (const int rc = status_from_hip(hipGetLastError())) return rc;
    hipLaunchKernelGGL(paged_mass_kernel, dim3((a.pages.slots() + 255) / 256, a.B * a.G), dim3(256), 0, stream, a.raw, a.lse, mass_pages, a.len_b,
                       a.pages, a.H, a.G);
    return status_from_hip(hipGetLastError());
}

int paged_step_dispatch(const void* q, const void* k_new, const void* v_new, void* k_pages, void* v_pages, int32_t* pos_pages, float* mass_pages,
                        const Pages& pages, const int32_t* len_b, const int32_t* new_pos_b, int B, int H, int Hkv, int G, int D, float scale, int dt,
                        void* out, void* ws, hipStream_t stream)
{
    float* raw = static_cast<float*>(ws);
    float* lse = reinterpret_cast<float*>(static_cast<char*>(ws) + (((size_t)B * H * pages.slots() * 4 + 255) & ~(size_t)255));
    const PagedStep a{q, k_new, v_new, k_pages, v_pages, out, pos_pages, len_b, new_pos_b, pages, B, H, Hkv, G, scale, raw, lse};
    if (dt == EC_BF16) return D == 128 ? launch<EC_BF16, 128>(a, mass_pages, stream) : launch<EC_BF16, 64>(a, mass_pages, stream);
    return D == 128 ? launch<EC_F32, 128>(a, mass_pages, stream) : launch<EC_F32, 64>(a, mass_pages, stream);
}

}  // namespace ec
