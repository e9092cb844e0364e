// The pages that a sequence's attention reads: its first ones, its last ones, and of those between the ones of highest score, ties to the lowest page; in
// ascending order.  Bound: latency, a chain of counts and barriers of one workgroup for each sequence and key head: 500 pages 4.5 us, of which a launch is 3.5; 8192 in
// 1024 threads 10.3 (in 512 10.6, in 256 15.1).
//
// A thread holds pages that follow each other, so that its place in the list is one running sum over the threads.  The threshold comes from a histogram select
// over the keys' own range (swa_select.hpp).
#include "swa_paged.hpp"
#include "swa_select.hpp"

namespace swa {

struct PageSelectArgs {
    const float* score;
    const int32_t* cache_len;
    int32_t *sel, *sel_cnt, *status;
    int32_t b, h_kv, page_size, max_pages, len_max, n_sel, first, last;
};

// Order of scores: what is no number counts as infinite, and -0 as 0.
__device__ __forceinline__ uint32_t score_key(float f) { return order_key(f != f ? INFINITY : f + 0.f); }

// HELD: scores that a thread keeps in registers; 0: read again wherever they are needed.
template <int NT, int HELD>
__global__ void __launch_bounds__(NT) swa_paged_select_kernel(PageSelectArgs a)
{
    __shared__ SelectScratch<NT> scratch;
    __shared__ int32_t sums[NT / 64], equal[NT / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, s = blockIdx.x / a.h_kv, kv = blockIdx.x - s * a.h_kv;
    const int64_t pair = (int64_t)s * a.h_kv + kv;
    int32_t* const to = a.sel + pair * a.n_sel;
    int n = a.cache_len[s];
    if (n > a.len_max) {
        if (kv == 0 && tid == 0) atomicOr(a.status, kStatusCapacityBit);
        n = 0;
    }
    const int pages = n > 0 ? (int)(((int64_t)n + a.page_size - 1) / a.page_size) : 0;
    const int count = pages < a.n_sel ? pages : a.n_sel;
    if (tid == 0) a.sel_cnt[pair] = count;
    for (int i = count + tid; i < a.n_sel; i += NT) to[i] = -1;
    if (pages <= a.n_sel) {
        for (int i = tid; i < pages; i += NT) to[i] = i;
        return;
    }
    // candidates: first .. end - 1, of which `want` are taken
    const int end = pages - a.last, want = a.n_sel - a.first - a.last;
    for (int i = tid; i < a.first; i += NT) to[i] = i;
    for (int i = tid; i < a.last; i += NT) to[a.n_sel - a.last + i] = end + i;
    if (want == 0) return;
    const float* const score = a.score + pair * a.max_pages;
    const int per = (end - a.first + NT - 1) / NT, p0 = a.first + tid * per, p1 = p0 + per < end ? p0 + per : end;
    uint32_t held[HELD ? HELD : 1];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) held[i] = i < per && p0 + i < p1 ? score_key(score[p0 + i]) : 0u;
    }
    auto each = [&](auto f) __attribute__((always_inline)) {
        if constexpr (HELD > 0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i < per && p0 + i < p1) f(held[i]);
        } else {
            for (int p = p0; p < p1; ++p) f(score_key(score[p]));
        }
    };
    scratch.hist[2 * tid] = scratch.hist[2 * tid + 1] = 0;
    if (tid < 64) scratch.rank[tid] = 0;
    if (tid == 0) scratch.listed = 0;
    uint32_t lowest, highest, thr;
    int rem, n_eq;
    key_range<NT>(scratch, each, lowest, highest);
    select_threshold<NT>(scratch, want, lowest, highest, each, thr, rem, n_eq);
    // pages above the threshold, and equal ones, before this thread's
    int above = 0, same = 0;
    each([&](uint32_t key) {
        above += key > thr;
        same += key == thr;
    });
    const int above_to = wave_scan(above), same_to = wave_scan(same);
    if (lane == 63) {
        sums[wave] = above_to;
        equal[wave] = same_to;
    }
    __syncthreads();
    int above_before = above_to - above, same_before = same_to - same;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w)
        if (w < wave) {
            above_before += sums[w];
            same_before += equal[w];
        }
    int p = p0;
    each([&](uint32_t key) {
        const int before = above_before + (same_before < rem ? same_before : rem);
        if (key > thr || (key == thr && same_before < rem)) to[a.first + before] = p;
        above_before += key > thr;
        same_before += key == thr;
        ++p;
    });
}

int launch_paged_select(const swa_paged_params& p, const float* score, const int32_t* cache_len, int32_t n_sel, int32_t first, int32_t last,
                        int32_t* sel, int32_t* sel_cnt, void* workspace, hipStream_t stream)
{
    PageSelectArgs a{score, cache_len, sel, sel_cnt, paged_status(workspace), p.b, p.h_kv, p.page_size, p.max_pages, paged_len_max(p),
                     n_sel, first, last};
    const int64_t pages = paged_pages_max(p);
    const dim3 grid((unsigned)((int64_t)p.b * p.h_kv));
    if ((int64_t)p.b * p.h_kv >= 1 << 22) return SWA_ERR_CAPACITY;                     // (threads of a launch)
    if (pages <= 2048) launch_kernel(swa_paged_select_kernel<256, 8>, grid, dim3(256), 0, stream, a);
    else if (pages <= 8192) launch_kernel(swa_paged_select_kernel<1024, 8>, grid, dim3(1024), 0, stream, a);
    else launch_kernel(swa_paged_select_kernel<1024, 0>, grid, dim3(1024), 0, stream, a);
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
