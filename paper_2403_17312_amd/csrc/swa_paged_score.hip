// An upper bound of the logits of each page's keys, from the smallest and largest values of its channels alone:
//   q . k = sum_c q_c k_c <= sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c,
// a product of a row of 2 D bounds with the query's negative and positive parts, so it goes to the matrix cores like the attention's logits: sixteen
// pages by sixteen query heads.  Bound: HBM, one read of the bounds; a page of n tokens costs a n-th of what its keys and values do.
#include "swa_paged_tile.hpp"

namespace swa {

struct ScoreArgs {
    const char* q;
    int64_t q_stride;                              // bytes
    PagedRows rows;
    const int32_t* block_table;
    const char* bounds;
    float* score;
    int32_t* status;
    int32_t b, h_kv, page_size, n_pages, max_pages;
    int32_t group, ranges;                         // query heads of a key head; workgroups that share a sequence's pages
    float scale;
};

// The negative or the positive values of a row, zeros for the others (what is no number is in one of the two).
template <typename T>
__device__ __forceinline__ Vec16 part_of(const Vec16& v, bool negative)
{
    auto word = [&](uint32_t w) {
        if constexpr (std::is_same_v<T, F32>) {
            const uint32_t sign = (uint32_t)((int32_t)w >> 31);
            return w & (negative ? sign : ~sign);
        } else {
            const uint32_t sign = ((w >> 15) & 0x00010001u) * 0xffffu;
            return w & (negative ? sign : ~sign);
        }
    };
    return Vec16{word(v.x), word(v.y), word(v.z), word(v.w)};
}

template <typename T, int D>
__global__ void __launch_bounds__(256) swa_paged_score_kernel(ScoreArgs a)
{
    constexpr int kRow = 2 * D * Elem<T>::kBytes, kSteps = kRow / 64, kHalf = kSteps / 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, j = lane >> 4;
    const int units = a.b * a.h_kv, range = blockIdx.x / units, unit = blockIdx.x - range * units, s = unit / a.h_kv, kv = unit - s * a.h_kv;
    int row, n;
    bool too_long = false;
    if (!paged_row(a.rows, s, row, n, too_long)) {
        if (too_long && range == 0 && kv == 0 && threadIdx.x == 0) atomicOr(a.status, kStatusCapacityBit);
        return;
    }
    const int pages = (int)(((int64_t)n + a.page_size - 1) / a.page_size);
    const int32_t* const table = a.block_table + (int64_t)s * a.max_pages;
    float* const to = a.score + ((int64_t)s * a.h_kv + kv) * a.max_pages;
    const char* const from = a.q + row * a.q_stride + (int64_t)kv * a.group * (D * Elem<T>::kBytes);
    bool bad = false;
    Vec16 q[kHalf];
    for (int base = (range * 4 + wave) * 16; base < pages; base += a.ranges * 64) {
        const int page = base + col < pages ? table[base + col] : 0;
        const bool there = (uint32_t)page < (uint32_t)a.n_pages;
        bad |= !there;
        const char* const row_of = a.bounds + ((int64_t)(there ? page : 0) * a.h_kv + kv) * kRow + j * 16;
        Vec16 box[kSteps];
#pragma unroll
        for (int c = 0; c < kSteps; ++c) box[c] = load16_stream(row_of + c * 64);
        float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        for (int head0 = 0; head0 < a.group; head0 += 16) {
            const bool head = head0 + col < a.group;
#pragma unroll
            for (int c = 0; c < kHalf; ++c)
                q[c] = head ? load16(from + (int64_t)(head0 + col) * (D * Elem<T>::kBytes) + c * 64 + j * 16) : Vec16{0u, 0u, 0u, 0u};
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < kHalf; ++c) {
                sum = mfma16<T>(box[c], part_of<T>(q[c], true), sum);
                sum = mfma16<T>(box[c + kHalf], part_of<T>(q[c], false), sum);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = sum[i] != sum[i] ? INFINITY : sum[i];
                best[i] = head ? fmaxf(best[i], x) : best[i];
            }
        }
        // the sixteen heads to one, within rows of 16 lanes
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            best[i] = fmaxf(best[i], dpp_move<0xB1>(best[i]));
            best[i] = fmaxf(best[i], dpp_move<0x4E>(best[i]));
            best[i] = fmaxf(best[i], dpp_move<0x141>(best[i]));
            best[i] = fmaxf(best[i], dpp_move<0x140>(best[i]));
        }
        const float mine = (col & 2) ? ((col & 1) ? best[3] : best[2]) : ((col & 1) ? best[1] : best[0]);
        const bool in_pool = __shfl((int)there, 4 * j + (col & 3), 64) != 0;
        const int p = base + 4 * j + col;
        if (col < 4 && p < pages) to[p] = in_pool ? mine * a.scale : -INFINITY;
    }
    if (bad) atomicOr(a.status, kStatusBadRequestBit);
}

int launch_paged_score(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                       const void* bounds, const int32_t* block_table, const int32_t* cache_len, float* score, void* workspace, hipStream_t stream)
{
    ScoreArgs a{};
    a.q = static_cast<const char*>(q.data);
    a.q_stride = q.stride * (p.dtype == SWA_F32 ? 4 : 2);
    a.rows = PagedRows{row_start, slot, cache_len, n_rows, paged_len_max(p)};
    a.block_table = block_table;
    a.bounds = static_cast<const char*>(bounds);
    a.score = score;
    a.status = paged_status(workspace);
    a.b = p.b;
    a.h_kv = p.h_kv;
    a.page_size = p.page_size;
    a.n_pages = p.n_pages;
    a.max_pages = p.max_pages;
    a.group = p.h_q / p.h_kv;
    a.scale = p.scale > 0.f ? p.scale : 1.f / sqrtf((float)p.d);
    const int64_t units = (int64_t)p.b * p.h_kv, blocks = ((int64_t)paged_pages_max(p) + 63) / 64;
    // Workgroups for every CU eight times, as far as there are pages.
    int64_t ranges = (2048 + units - 1) / units;
    if (ranges > blocks) ranges = blocks;
    a.ranges = (int32_t)ranges;
    if (units * ranges * 256 > 0xffffffffLL) return SWA_ERR_CAPACITY;
    const dim3 grid((unsigned)(units * ranges));
#define SWA_SCORE(T) (p.d == 64 ? launch_kernel(swa_paged_score_kernel<T, 64>, grid, dim3(256), 0, stream, a) \
                                : launch_kernel(swa_paged_score_kernel<T, 128>, grid, dim3(256), 0, stream, a))
    if (p.dtype == SWA_F32) SWA_SCORE(F32);
    else if (p.dtype == SWA_F16) SWA_SCORE(F16);
    else SWA_SCORE(BF16);
#undef SWA_SCORE
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
