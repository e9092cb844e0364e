// C-ABI entry points of the paged cache: argument validation on the host, then launches on the caller's stream.
#include <math.h>

#include "swa_paged.hpp"

namespace swa {

static bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static int validate_paged(const swa_paged_params* p)
{
    if (!p) return SWA_ERR_NULL;
    if (p->dtype != SWA_F32 && p->dtype != SWA_F16 && p->dtype != SWA_BF16) return SWA_ERR_UNSUPPORTED_DTYPE;
    if (p->d != 64 && p->d != 128) return SWA_ERR_UNSUPPORTED_D;
    if (p->b < 1 || p->b > SWA_MAX_PAGED_SEQS || p->h_q < 1 || p->h_q > 65535 || p->h_kv < 1 || p->h_q % p->h_kv != 0) return SWA_ERR_BAD_SHAPE;
    if (p->page_size < 1 || p->n_pages < 1 || p->max_pages < 1) return SWA_ERR_BAD_SHAPE;
    if (p->page_size > SWA_MAX_CAP) return SWA_ERR_CAPACITY;
    // rows of the pool, and tokens of a sequence with what a launch adds to them, are 32-bit numbers in the kernels (their bytes are not)
    if ((int64_t)p->n_pages * p->page_size > 0x7fffffffLL / p->h_kv || (int64_t)p->max_pages * p->page_size > (1LL << 30)) return SWA_ERR_CAPACITY;
    if (!(p->scale >= 0.f) || isinf(p->scale) || !(p->eps >= 0.f) || isinf(p->eps)) return SWA_ERR_BAD_SHAPE;
    if (p->window < 0 || p->len_bound < 0) return SWA_ERR_BAD_SHAPE;
    if (p->flags & ~(SWA_KV_INT8 | SWA_ROPE_INTERLEAVED)) return SWA_ERR_BAD_SHAPE;
    if (paged_int8(*p) && p->dtype == SWA_F32) return SWA_ERR_UNSUPPORTED_DTYPE;
    if (p->rot_dim < 0 || p->rot_dim > p->d || p->rot_dim % 16 != 0 || p->axes < 1 || p->axes > SWA_MAX_ROPE_AXES) return SWA_ERR_BAD_SHAPE;
    int64_t pairs = 0;
    for (int i = 0; i < p->axes; ++i) {
        if (p->section[i] < 0) return SWA_ERR_BAD_SHAPE;
        pairs += p->section[i];
    }
    return pairs == p->rot_dim / 2 ? SWA_OK : SWA_ERR_BAD_SHAPE;
}

static int check_rows(const swa_paged_params& p, const swa_rows& r, int heads)
{
    if (!r.data) return SWA_ERR_NULL;
    const int bytes = p.dtype == SWA_F32 ? 4 : 2;
    if (r.stride < (int64_t)heads * p.d || r.stride > (INT64_C(1) << 40)) return SWA_ERR_BAD_SHAPE;
    return on16(r.data) && (r.stride * bytes) % 16 == 0 ? SWA_OK : SWA_ERR_ALIGNMENT;
}

static int check_pool(const swa_paged_params& p, const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale)
{
    if (!k_pages || !v_pages || (paged_int8(p) && (!k_scale || !v_scale))) return SWA_ERR_NULL;
    return on16(k_pages) && on16(v_pages) && (!paged_int8(p) || (on16(k_scale) && on16(v_scale))) ? SWA_OK : SWA_ERR_ALIGNMENT;
}

static int decode_call(const swa_paged_params* params, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                       const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                       const int32_t* cache_len, void* out, float* lse, void* workspace, void* stream)
{
    int rc = validate_paged(params);
    if (rc != SWA_OK) return rc;
    if (!block_table || !cache_len || !out || !workspace) return SWA_ERR_NULL;
    if ((rc = check_pool(*params, k_pages, v_pages, k_scale, v_scale)) != SWA_OK) return rc;
    if ((rc = check_rows(*params, q, params->h_q)) != SWA_OK) return rc;
    if (n_rows < 1 || n_rows > kMaxPlanRows || (!row_start && n_rows < params->b)) return SWA_ERR_BAD_SHAPE;
    if (!on16(out) || !on16(workspace)) return SWA_ERR_ALIGNMENT;
    return launch_paged_decode(*params, q, n_rows, row_start, slot, k_pages, v_pages, k_scale, v_scale, block_table, cache_len, out, lse,
                               workspace, static_cast<hipStream_t>(stream));
}

__global__ void swa_paged_zero_kernel(int32_t* p)
{
    if (threadIdx.x < 16) p[threadIdx.x] = 0;
}

}  // namespace swa

extern "C" {

size_t swa_paged_workspace_bytes(const swa_paged_params* params)
{
    if (swa::validate_paged(params) != SWA_OK) return 0;
    return (swa::kPagedPartialOffset + swa::paged_partial_bytes(*params) + 255) & ~(size_t)255;
}

int swa_paged_workspace_init(const swa_paged_params* params, void* workspace, void* stream)
{
    const int rc = swa::validate_paged(params);
    if (rc != SWA_OK) return rc;
    if (!workspace) return SWA_ERR_NULL;
    swa::launch_kernel(swa::swa_paged_zero_kernel, dim3(1), dim3(64), 0, static_cast<hipStream_t>(stream), swa::paged_status(workspace));
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

int swa_paged_check_status(const swa_paged_params* params, void* workspace, void* stream, int32_t* status_out)
{
    const int rc = swa::validate_paged(params);
    if (rc != SWA_OK) return rc;
    if (!workspace || !status_out) return SWA_ERR_NULL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    int32_t bits = 0;
    if (hipMemcpyAsync(&bits, swa::paged_status(workspace), sizeof(bits), hipMemcpyDeviceToHost, st) != hipSuccess) return SWA_ERR_HIP;
    if (hipStreamSynchronize(st) != hipSuccess) return SWA_ERR_HIP;
    if (bits != 0) {
        swa::launch_kernel(swa::swa_paged_zero_kernel, dim3(1), dim3(64), 0, st, swa::paged_status(workspace));
        if (hipGetLastError() != hipSuccess) return SWA_ERR_HIP;
    }
    *status_out = (bits & swa::kStatusCapacityBit) ? SWA_ERR_CAPACITY : (bits & swa::kStatusBadRequestBit) ? SWA_ERR_BAD_REQUEST : SWA_OK;
    return SWA_OK;
}

int swa_paged_plan(const swa_paged_params* params, const int32_t* new_cnt, const int32_t* cache_len, int32_t* new_len,
                   int32_t* block_table, int32_t* free_ring, const int32_t* free_state, int32_t* free_state_out, int32_t max_rows,
                   int32_t* row_start, int32_t* slot, int32_t* pos, void* workspace, void* stream)
{
    const int rc = swa::validate_paged(params);
    if (rc != SWA_OK) return rc;
    if (!new_cnt || !cache_len || !new_len || !block_table || !free_ring || !free_state || !free_state_out || !row_start || !slot || !pos ||
        !workspace)
        return SWA_ERR_NULL;
    if (max_rows < 1 || max_rows > swa::kMaxPlanRows) return SWA_ERR_BAD_SHAPE;
    // (workgroups read the old lists while others write the new ones)
    if (cache_len == new_len || new_cnt == new_len || free_state == free_state_out) return SWA_ERR_BAD_SHAPE;
    return swa::launch_paged_plan(*params, new_cnt, cache_len, new_len, block_table, free_ring, free_state, free_state_out, max_rows,
                                  row_start, slot, pos, workspace, static_cast<hipStream_t>(stream));
}

int swa_paged_append(const swa_paged_params* params, swa_rows q, swa_rows k, swa_rows v, int32_t n_rows, const int32_t* pos,
                     const int32_t* slot, const float* inv_freq, const void* q_weight, const void* k_weight, void* q_out, void* k_pages,
                     void* v_pages, float* k_scale, float* v_scale, void* workspace, void* stream)
{
    int rc = swa::validate_paged(params);
    if (rc != SWA_OK) return rc;
    if (!slot || !q_out || !workspace || (params->rot_dim > 0 && (!pos || !inv_freq))) return SWA_ERR_NULL;
    if ((rc = swa::check_pool(*params, k_pages, v_pages, k_scale, v_scale)) != SWA_OK) return rc;
    if ((rc = swa::check_rows(*params, q, params->h_q)) != SWA_OK) return rc;
    if ((rc = swa::check_rows(*params, k, params->h_kv)) != SWA_OK) return rc;
    if ((rc = swa::check_rows(*params, v, params->h_kv)) != SWA_OK) return rc;
    if (n_rows < 1 || n_rows > swa::kMaxPlanRows) return SWA_ERR_BAD_SHAPE;
    // q_out may be q itself, where a row's place is the same in both
    if (q.data == q_out && q.stride != (int64_t)params->h_q * params->d) return SWA_ERR_BAD_SHAPE;
    if (!swa::on16(q_out) || !swa::on16(q_weight) || !swa::on16(k_weight) || !swa::on16(workspace)) return SWA_ERR_ALIGNMENT;
    return swa::launch_paged_append(*params, q, k, v, n_rows, pos, slot, inv_freq, q_weight, k_weight, q_out, k_pages, v_pages, k_scale,
                                    v_scale, workspace, static_cast<hipStream_t>(stream));
}

int swa_paged_decode(const swa_paged_params* params, swa_rows q, int32_t n_rows, const int32_t* row_start, const void* k_pages,
                     const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                     const int32_t* cache_len, void* out, float* lse, void* workspace, void* stream)
{
    return swa::decode_call(params, q, n_rows, row_start, nullptr, k_pages, v_pages, k_scale, v_scale, block_table, cache_len, out, lse,
                            workspace, stream);
}

int swa_paged_decode_planned(const swa_paged_params* params, swa_rows q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                             const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale,
                             const int32_t* block_table, const int32_t* cache_len, void* out, float* lse, void* workspace, void* stream)
{
    if (!row_start || !slot) return SWA_ERR_NULL;
    return swa::decode_call(params, q, n_rows, row_start, slot, k_pages, v_pages, k_scale, v_scale, block_table, cache_len, out, lse,
                            workspace, stream);
}

}  // extern "C"
