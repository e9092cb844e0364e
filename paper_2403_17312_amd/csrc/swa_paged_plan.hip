// Block tables, slots and positions of a paged cache's new tokens.
//
// Three running sums over the sequences decide everything: rows (sum of new_cnt), pages asked for, and pages given back.  Every
// workgroup forms them anew in its LDS (b <= 4096: a few KB from L2) instead of waiting for one that does, and then deals itself
// rows, fresh pages and returned pages by their number, whose sequence a binary search in the sums finds.  No workgroup reads
// what another one writes: lengths and the ring's state have a second copy, fresh table entries are taken from the ring
// wherever they are needed, and returned pages go behind the ring's last free one.  Bound by latency: one launch, a chain of
// two block scans and one search.
#include "swa_paged.hpp"

namespace swa {

struct PlanArgs {
    const int32_t *new_cnt, *cache_len;
    int32_t *new_len, *block_table, *free_ring;
    const int32_t* free_state;
    int32_t *free_state_out, *row_start, *slot, *pos, *status;
    int32_t b, page_size, n_pages, max_pages, max_rows;
};

constexpr int kPlanThreads = 256;

__device__ __forceinline__ int32_t add_saturating(int32_t a, int32_t b)
{
    const uint32_t s = (uint32_t)a + (uint32_t)b;  // both at most 2^30
    return s < (uint32_t)kRowsSaturate ? (int32_t)s : kRowsSaturate;
}

// Sum over the threads before this one (saturating: of numbers in 0..2^30 that is associative).
__device__ __forceinline__ int32_t sum_before(int32_t v, int32_t* wave_sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int32_t u = __shfl_up(v, o, 64);
        if (lane >= o) v = add_saturating(v, u);
    }
    __syncthreads();                               // (the sums of the scan before this one have been read)
    if (lane == 63) wave_sums[wave] = v;
    __syncthreads();
    const int32_t up = __shfl_up(v, 1, 64);
    int32_t before = lane ? up : 0;
    for (int w = 0; w < wave; ++w) before = add_saturating(before, wave_sums[w]);
    return before;
}

// First of n ascending sums that is above x.
__device__ __forceinline__ int above(const int32_t* sums, int n, int32_t x)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

__global__ void __launch_bounds__(kPlanThreads) swa_paged_plan_kernel(PlanArgs a)
{
    extern __shared__ int32_t sums[];
    __shared__ int32_t wave_sums[kPlanThreads / 64];
    int32_t* const rows_to = sums;                 // rows up to and with sequence s
    int32_t* const asked_to = sums + a.b;          // pages that sequences up to s ask for
    int32_t* const back_to = sums + 2 * a.b;       // pages that sequences up to s give back
    const int tid = threadIdx.x, b = a.b, ps = a.page_size;
    const int32_t cap = a.max_pages * ps;
    const bool first = blockIdx.x == 0;
    int32_t head = a.free_state[0], free = a.free_state[1];
    free = free < 0 ? 0 : (free > a.n_pages ? a.n_pages : free);
    head = (head < 0 || head >= a.n_pages) ? 0 : head;
    int32_t bits = 0;

    const int per = (b + kPlanThreads - 1) / kPlanThreads, s0 = tid * per, s1 = s0 + per < b ? s0 + per : b;
    int32_t sum = 0;
    for (int s = s0; s < s1; ++s) {
        const int32_t c = a.new_cnt[s];
        sum = add_saturating(sum, c < 0 ? 0 : (c > kRowsSaturate ? kRowsSaturate : c));
        rows_to[s] = sum;
    }
    const int32_t rows_before = sum_before(sum, wave_sums);
    int32_t asked = 0, back = 0;                   // (asked: of sequences that have rows, so at most max_rows + b)
    for (int s = s0; s < s1; ++s) {
        const int32_t c = a.new_cnt[s], m = a.cache_len[s];
        rows_to[s] = add_saturating(rows_to[s], rows_before);
        if (m >= 0 && m <= cap) {
            const int32_t held = (int32_t)(((int64_t)m + ps - 1) / ps);
            if (c < 0)
                back = add_saturating(back, held < kRowsSaturate ? held : kRowsSaturate);
            else if (rows_to[s] <= a.max_rows && c <= cap - m)
                asked += (int32_t)(((int64_t)m + c + ps - 1) / ps) - held;
        } else if (m > cap) {
            bits |= kStatusBadRequestBit;
        }
        asked_to[s] = asked;
        back_to[s] = back;
    }
    const int32_t asked_before = sum_before(asked, wave_sums), back_before = sum_before(back, wave_sums);
    for (int s = s0; s < s1; ++s) {
        asked_to[s] += asked_before;
        back_to[s] = add_saturating(back_to[s], back_before);
    }
    __syncthreads();

    const int32_t total_rows = rows_to[b - 1];
    int32_t returned = back_to[b - 1];
    if (returned > a.n_pages - free) {             // more than the pool has: a table that names pages twice
        returned = a.n_pages - free;
        bits |= kStatusBadRequestBit;
    }
    const int stride = gridDim.x * kPlanThreads, at = blockIdx.x * kPlanThreads + tid;
    // pages that are given out: of the sequences that ask, those up to the first one whose pages are not all there
    int32_t given = asked_to[b - 1];
    if (given > free) {
        const int s = above(asked_to, b, free);    // the first one refused
        given = s ? asked_to[s - 1] : 0;
    }

    // 1. each sequence's length and first row
    for (int s = at; s < b; s += stride) {
        const int32_t c = a.new_cnt[s], m = a.cache_len[s], begin = s ? rows_to[s - 1] : 0;
        int32_t n = m;
        if (m >= 0 && m <= cap) {
            if (c < 0) {
                n = 0;
            } else if (c > 0) {
                const bool fits = rows_to[s] <= a.max_rows && c <= cap - m;
                const bool paged = asked_to[s] == (s ? asked_to[s - 1] : 0) || asked_to[s] <= given;
                if (fits && paged) n = m + c; else bits |= kStatusCapacityBit;
            }
        }
        a.new_len[s] = n;
        a.row_start[s] = begin;
    }
    if (first && tid == 0) {
        a.row_start[b] = total_rows;
        a.free_state_out[0] = (int32_t)(((int64_t)head + given) % a.n_pages);
        a.free_state_out[1] = free - given + returned;
    }

    // 2. fresh pages
    for (int32_t k = at; k < given; k += stride) {
        const int s = above(asked_to, b, k);
        const int32_t held = (int32_t)(((int64_t)a.cache_len[s] + ps - 1) / ps);
        const int32_t page = a.free_ring[(int32_t)(((int64_t)head + k) % a.n_pages)];
        if ((uint32_t)page >= (uint32_t)a.n_pages) bits |= kStatusBadRequestBit;
        a.block_table[(int64_t)s * a.max_pages + held + (k - (s ? asked_to[s - 1] : 0))] = page;
    }

    // 3. returned pages
    for (int32_t k = at; k < returned; k += stride) {
        const int s = above(back_to, b, k);
        const int32_t page = a.block_table[(int64_t)s * a.max_pages + (k - (s ? back_to[s - 1] : 0))];
        if ((uint32_t)page >= (uint32_t)a.n_pages) bits |= kStatusBadRequestBit;
        a.free_ring[(int32_t)(((int64_t)head + free + k) % a.n_pages)] = page;
    }

    // 4. rows
    for (int32_t r = at; r < a.max_rows; r += stride) {
        int32_t slot = -1, pos = 0;
        if (r < total_rows) {
            const int s = above(rows_to, b, r);
            const int32_t begin = s ? rows_to[s - 1] : 0, c = rows_to[s] - begin, m = a.cache_len[s];
            const int32_t asked0 = s ? asked_to[s - 1] : 0;
            if (m >= 0 && m <= cap && rows_to[s] <= a.max_rows && c <= cap - m && (asked_to[s] == asked0 || asked_to[s] <= given)) {
                const int32_t t = m + (r - begin), j = t / ps, held = (int32_t)(((int64_t)m + ps - 1) / ps);
                const int32_t page = j < held ? a.block_table[(int64_t)s * a.max_pages + j]
                                              : a.free_ring[(int32_t)(((int64_t)head + asked0 + (j - held)) % a.n_pages)];
                if ((uint32_t)page < (uint32_t)a.n_pages) {
                    slot = page * ps + (t - j * ps);
                    pos = t;
                } else {
                    bits |= kStatusBadRequestBit;
                }
            }
        }
        a.slot[r] = slot;
        a.pos[r] = pos;
    }
    if (bits) atomicOr(a.status, bits);
}

int launch_paged_plan(const swa_paged_params& p, const int32_t* new_cnt, const int32_t* cache_len, int32_t* new_len, int32_t* block_table,
                      int32_t* free_ring, const int32_t* free_state, int32_t* free_state_out, int32_t max_rows, int32_t* row_start,
                      int32_t* slot, int32_t* pos, void* workspace, hipStream_t stream)
{
    const PlanArgs a{new_cnt, cache_len, new_len, block_table, free_ring, free_state, free_state_out, row_start, slot, pos,
                     paged_status(workspace), p.b, p.page_size, p.n_pages, p.max_pages, max_rows};
    const int64_t items = max_rows > p.b ? max_rows : p.b;
    int64_t grid = (items + kPlanThreads - 1) / kPlanThreads;
    if (grid > 256) grid = 256;
    launch_kernel(swa_paged_plan_kernel, dim3((unsigned)grid), dim3(kPlanThreads), 3 * sizeof(int32_t) * (size_t)p.b, stream, a);
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
