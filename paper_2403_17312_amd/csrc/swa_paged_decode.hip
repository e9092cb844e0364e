// Attention of one new token per sequence over a paged cache.
//
// One wave per sequence and query head: 64 keys at a time, a lane each for the logits, then all lanes together for the values, with the running
// maximum and sum of the softmax.
#include <math.h>

#include <type_traits>

#include "swa_paged.hpp"

namespace swa {

struct PagedArgs {
    const char* q;
    int64_t q_stride;                              // bytes
    const int32_t *row_start, *block_table, *cache_len;
    const char *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    char* out;
    float* lse;
    int32_t* status;
    int32_t n_rows, h_q, h_kv, page_size, n_pages, max_pages, window, len_max;
    float scale;
};

size_t paged_partial_bytes(const swa_paged_params&) { return 0; }

template <typename T>
__device__ __forceinline__ float element(const char* row, int i)
{
    if constexpr (std::is_same_v<T, F32>) return reinterpret_cast<const float*>(row)[i];
    else if constexpr (std::is_same_v<T, F16>) return (float)reinterpret_cast<const _Float16*>(row)[i];
    else if constexpr (std::is_same_v<T, BF16>) return bf16_lo(reinterpret_cast<const uint16_t*>(row)[i]);
    else return (float)reinterpret_cast<const int8_t*>(row)[i];
}

template <typename T, typename C, int D>
__global__ void __launch_bounds__(64) swa_paged_decode_kernel(PagedArgs a)
{
    constexpr int kPer = D / 64;
    const int s = blockIdx.x, hq = blockIdx.y, lane = threadIdx.x, kv = hq / (a.h_q / a.h_kv);
    __shared__ float q[D];
    const int32_t n = a.cache_len[s];
    int row = s;
    if (a.row_start) {
        row = a.row_start[s + 1] - 1;
        if (row < a.row_start[s]) return;
    }
    if (n < 0 || row < 0 || row >= a.n_rows) return;
    if (n > a.len_max) {
        if (lane == 0) atomicOr(a.status, kStatusCapacityBit);
        return;
    }
    for (int i = 0; i < kPer; ++i)
        q[lane * kPer + i] = element<T>(a.q + row * a.q_stride + (int64_t)hq * D * Elem<T>::kBytes, lane * kPer + i) * a.scale;
    __syncthreads();
    float top = -INFINITY, sum = 0.f, acc[kPer] = {};
    const int lo = a.window && n > a.window ? n - a.window : 0;
    for (int t0 = lo; t0 < n; t0 += 64) {
        const int t = t0 + lane;
        float x = -INFINITY;
        int32_t r = -1;
        if (t < n) {
            const int32_t j = t / a.page_size, page = a.block_table[(int64_t)s * a.max_pages + j];
            if ((uint32_t)page < (uint32_t)a.n_pages) r = (page * a.h_kv + kv) * a.page_size + (t - j * a.page_size);
            else atomicOr(a.status, kStatusBadRequestBit);
        }
        if (r >= 0) {
            const char* const k = a.k_pages + (int64_t)r * (D * Elem<C>::kBytes);
            x = 0.f;
            for (int i = 0; i < D; ++i) x = __builtin_fmaf(q[i], element<C>(k, i), x);
            if (a.k_scale) x *= a.k_scale[r];
        }
        const float m = fmaxf(top, wave_max(x)), base = m == -INFINITY ? 0.f : m;
        const float p = r >= 0 ? __expf(x - base) : 0.f, old = __expf(top - base);
        sum = sum * old + wave_sum(p);
        for (int i = 0; i < kPer; ++i) acc[i] *= old;
        for (int u = 0; u < 64; ++u) {
            const int32_t ru = __shfl(r, u, 64);
            const float w = __shfl(p, u, 64) * (a.v_scale && ru >= 0 ? a.v_scale[ru] : 1.f);
            if (ru >= 0)
                for (int i = 0; i < kPer; ++i) acc[i] = __builtin_fmaf(w, element<C>(a.v_pages + (int64_t)ru * (D * Elem<C>::kBytes), lane * kPer + i), acc[i]);
        }
        top = m;
    }
    const int64_t at = (int64_t)row * a.h_q + hq;
    for (int i = 0; i < kPer; ++i)
        store_elem<T>(a.out + at * (D * Elem<T>::kBytes), lane * kPer + i, sum == 0.f ? 0.f : acc[i] / sum);
    if (a.lse && lane == 0) a.lse[at] = top + logf(sum);
}

int launch_paged_decode(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const void* k_pages,
                        const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table, const int32_t* cache_len,
                        void* out, float* lse, void* workspace, hipStream_t stream)
{
    PagedArgs a{};
    a.q = static_cast<const char*>(q.data);
    a.q_stride = q.stride * (p.dtype == SWA_F32 ? 4 : 2);
    a.row_start = row_start;
    a.block_table = block_table;
    a.cache_len = cache_len;
    a.k_pages = static_cast<const char*>(k_pages);
    a.v_pages = static_cast<const char*>(v_pages);
    a.k_scale = paged_int8(p) ? k_scale : nullptr;
    a.v_scale = paged_int8(p) ? v_scale : nullptr;
    a.out = static_cast<char*>(out);
    a.lse = lse;
    a.status = paged_status(workspace);
    a.n_rows = n_rows;
    a.h_q = p.h_q;
    a.h_kv = p.h_kv;
    a.page_size = p.page_size;
    a.n_pages = p.n_pages;
    a.max_pages = p.max_pages;
    a.window = p.window;
    a.len_max = p.max_pages * p.page_size;
    if (p.len_bound > 0 && p.len_bound < a.len_max) a.len_max = p.len_bound;
    a.scale = p.scale > 0.f ? p.scale : 1.f / sqrtf((float)p.d);
    const dim3 grid(p.b, p.h_q);
#define SWA_PAGED(T, C) \
    (p.d == 64 ? launch_kernel(swa_paged_decode_kernel<T, C, 64>, grid, dim3(64), 0, stream, a) \
               : launch_kernel(swa_paged_decode_kernel<T, C, 128>, grid, dim3(64), 0, stream, a))
    if (p.dtype == SWA_F32) SWA_PAGED(F32, F32);
    else if (p.dtype == SWA_F16) paged_int8(p) ? SWA_PAGED(F16, Q8) : SWA_PAGED(F16, F16);
    else paged_int8(p) ? SWA_PAGED(BF16, Q8) : SWA_PAGED(BF16, BF16);
#undef SWA_PAGED
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
