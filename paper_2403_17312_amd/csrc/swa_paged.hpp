// The paged cache: launch interface between its entry points and its kernels.
#pragma once

#include "swa_kernels.hpp"

namespace swa {

constexpr int32_t kMaxPlanRows = 1 << 24;      // rows of one plan
constexpr int32_t kRowsSaturate = 1 << 30;     // what a sum of new tokens stops at

inline bool paged_int8(const swa_paged_params& p) { return (p.flags & SWA_KV_INT8) != 0; }

// Bytes of one key or value row in the pool.
inline int paged_row_bytes(const swa_paged_params& p) { return paged_int8(p) ? p.d : p.d * (p.dtype == SWA_F32 ? 4 : 2); }

inline int32_t* paged_status(void* workspace) { return reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + kWsStatusOffset); }

// t / page_size as (t * mul) >> shift, exact for 0 <= t < 2^31: with 2^(l-1) < page_size <= 2^l, mul = ceil(2^(31 + l) / page_size) is below 2^32, and it is
// too large by less than one, which t times over stays below 2^31 <= 2^(31 + l) / page_size, the step to the next quotient.
inline void page_divisor(int32_t page_size, uint32_t& mul, int32_t& shift)
{
    int l = 0;
    while ((1 << l) < page_size) ++l;
    shift = 31 + l;
    mul = (uint32_t)(((UINT64_C(1) << shift) + page_size - 1) / page_size);
}

// Longest sequence that a call takes, and its pages.
inline int32_t paged_len_max(const swa_paged_params& p)
{
    const int32_t table = p.max_pages * p.page_size;
    return p.len_bound > 0 && p.len_bound < table ? p.len_bound : table;
}
inline int32_t paged_pages_max(const swa_paged_params& p) { return (int32_t)(((int64_t)paged_len_max(p) + p.page_size - 1) / p.page_size); }

constexpr size_t kPagedPartialOffset = 256;    // the status word lies before the attention's partial results,
constexpr size_t kPagedLengthOffset = 128;     // and the length that a single sequence of swa_paged_decode_shared has for the call

// Query heads of a workgroup: the matrix cores' 16 columns, or twice as many, so that keys and values shared by more heads are read half as often.
inline int tile_heads_of(const swa_paged_params& p) { return p.h_q / p.h_kv > 16 ? 32 : 16; }

inline int row_tiles_of(const swa_paged_params& p) { return (p.h_q / p.h_kv + tile_heads_of(p) - 1) / tile_heads_of(p); }

constexpr int kPagedStep = 128;                // tokens

// Bytes of the partial results of swa_paged_decode, for any len_bound and window, and where they lie: [pieces, row tiles, heads, d] and [.., 2] (maximum, sum).
size_t paged_partial_bytes(const swa_paged_params& p);
void paged_partials(const swa_paged_params& p, void* workspace, float*& out, float*& sum);

int64_t paged_chunk_steps(const swa_paged_params& p, int64_t of_one);

// LDS of swa_paged_plan's workgroups, four lists of the same size.
size_t paged_plan_lds(int32_t b);

int launch_paged_plan(const swa_paged_params& p, const int32_t* new_cnt, const int32_t* cache_len, int32_t* new_len, int32_t* block_table,
                      int32_t* free_ring, const int32_t* free_state, int32_t* free_state_out, int32_t max_rows, int32_t* row_start,
                      int32_t* slot, int32_t* pos, void* workspace, hipStream_t stream);

// Waves that share a row of swa_paged_append, as a power of two; wide: in fp32.
int paged_append_log_parts(bool wide, bool codes, int passes, int64_t n_rows);

int launch_paged_append(const swa_paged_params& p, const swa_rows& q, const swa_rows& k, const swa_rows& v, int32_t n_rows, const int32_t* pos,
                        const int32_t* slot, const float* inv_freq, const void* q_weight, const void* k_weight, void* q_out, void* k_pages,
                        void* v_pages, float* k_scale, float* v_scale, void* workspace, hipStream_t stream);

// (slot may be null)
int launch_paged_decode(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                        const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                        const int32_t* cache_len, void* out, float* lse, void* workspace, hipStream_t stream);

int launch_paged_bounds(const swa_paged_params& p, int32_t n_rows, const int32_t* slot, const void* k_pages, const float* k_scale, void* bounds,
                        void* workspace, hipStream_t stream);

int launch_paged_score(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                       const void* bounds, const int32_t* block_table, const int32_t* cache_len, float* score, void* workspace, hipStream_t stream);

int launch_paged_select(const swa_paged_params& p, const float* score, const int32_t* cache_len, int32_t n_sel, int32_t first, int32_t last,
                        int32_t* sel, int32_t* sel_cnt, void* workspace, hipStream_t stream);

int launch_paged_selected(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                          const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                          const int32_t* cache_len, const int32_t* sel, const int32_t* sel_cnt, int32_t n_sel, void* out, float* lse,
                          void* workspace, hipStream_t stream);

// Bytes of the partial results of swa_paged_decode_shared, which lie where those of swa_paged_decode do.
size_t paged_shared_bytes(const swa_paged_params& p);

// Raises the LDS limit of its kernels on the current device.
int prepare_paged_shared();

int launch_paged_shared(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                        const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                        const int32_t* cache_len, const int32_t* prefix_of, void* out, float* lse, void* workspace, hipStream_t stream);

}  // namespace swa
