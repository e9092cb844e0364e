// Block tables, slots and positions of a paged cache's new tokens.
//
// Three running sums over the sequences decide everything: rows (sum of new_cnt), pages asked for, and pages given back.  Every
// workgroup forms them anew in its LDS (b <= 4096: a few KB from L2) instead of waiting for one that does, and then deals itself
// rows, fresh pages and returned pages by their number, whose sequence a binary search in the sums finds.  No workgroup reads
// what another one writes: lengths and the ring's state have a second copy, fresh table entries are taken from the ring
// wherever they are needed, and returned pages go behind the ring's last free one.  Bound by latency: one launch, a chain of
// two block scans and one search.  Numbers of pages by multiplication: a division of 64 bits costs a microsecond in this chain.
#include "swa_paged.hpp"

namespace swa {

struct PlanArgs {
    const int32_t *new_cnt, *cache_len;
    int32_t *new_len, *block_table, *free_ring;
    const int32_t* free_state;
    int32_t *free_state_out, *row_start, *slot, *pos, *status;
    int32_t b, page_size, n_pages, max_pages, max_rows;
    uint32_t page_mul;                             // t / page_size = t * page_mul >> page_shift for 0 <= t < 2^31
    int32_t page_shift;
};

__device__ __forceinline__ int32_t add_saturating(int32_t a, int32_t b)
{
    const uint32_t s = (uint32_t)a + (uint32_t)b;  // both at most 2^30
    return s < (uint32_t)kRowsSaturate ? (int32_t)s : kRowsSaturate;
}

// Sums of two numbers over the threads before this one (saturating: of numbers in 0..2^30 that is associative).
__device__ __forceinline__ int2 sums_before(int32_t u, int32_t v, int2* wave_sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int32_t u2 = __shfl_up(u, o, 64), v2 = __shfl_up(v, o, 64);
        if (lane >= o) {
            u = add_saturating(u, u2);
            v = add_saturating(v, v2);
        }
    }
    __syncthreads();                               // (the sums of the scan before this one have been read)
    if (lane == 63) wave_sums[wave] = int2{u, v};
    __syncthreads();
    int2 before = {__shfl_up(u, 1, 64), __shfl_up(v, 1, 64)};
    if (lane == 0) before = int2{0, 0};
    for (int w = 0; w < wave; ++w) {
        before.x = add_saturating(before.x, wave_sums[w].x);
        before.y = add_saturating(before.y, wave_sums[w].y);
    }
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

// Sequences that each of the four lists in LDS has room for: even, so that the sums of the waves, pairs of numbers at the fourth one's beginning, lie on
// 8 bytes; and enough for those of sixteen waves.
__host__ __device__ constexpr int plan_room(int b) { return ((b < 32 ? 32 : b) + 1) & ~1; }

size_t paged_plan_lds(int32_t b) { return 4 * sizeof(int32_t) * (size_t)plan_room(b); }

// PER: sequences of a thread while the sums are formed.
template <int THREADS, int PER>
__global__ void __launch_bounds__(THREADS) swa_paged_plan_kernel(PlanArgs a)
{
    extern __shared__ __align__(16) int32_t lds[];
    const int tid = threadIdx.x, b = a.b, ps = a.page_size, room = plan_room(b);
    int32_t* const rows_to = lds;                  // rows up to and with sequence s
    int32_t* const asked_to = lds + room;          // pages that sequences up to s ask for
    int32_t* const back_to = lds + 2 * room;       // pages that sequences up to s give back
    int32_t* const held_len = lds + 3 * room;      // cache_len, -1 where a sequence gets nothing
    int2* const wave_sums = reinterpret_cast<int2*>(held_len);   // (until the lengths are written there)
    const int32_t cap = a.max_pages * ps;
    const bool first = blockIdx.x == 0;
    int32_t head = a.free_state[0], free = a.free_state[1];
    int32_t bits = 0;
    auto pages_of = [&](int32_t t) { return t > 0 ? (int32_t)(((uint64_t)(uint32_t)(t - 1) * a.page_mul) >> a.page_shift) + 1 : 0; };
    auto in_ring = [&](int32_t i) {                // place i behind the head, 0 <= i <= n_pages
        const uint32_t at = (uint32_t)head + (uint32_t)i;
        return (int32_t)(at < (uint32_t)a.n_pages ? at : at - (uint32_t)a.n_pages);
    };

    const int s0 = tid * PER;
    int32_t count[PER], len[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        count[i] = s0 + i < b ? a.new_cnt[s0 + i] : 0;
        len[i] = s0 + i < b ? a.cache_len[s0 + i] : -1;
    }
    if ((uint32_t)free > (uint32_t)a.n_pages || (uint32_t)head >= (uint32_t)a.n_pages) {   // no ring's: whatever lay there may be in use
        head = free = 0;
        bits |= kStatusBadRequestBit;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) sum = add_saturating(sum, count[i] < 0 ? 0 : (count[i] > kRowsSaturate ? kRowsSaturate : count[i]));
    int32_t rows = sums_before(sum, 0, wave_sums).x;
    int32_t asked = 0, back = 0;                   // (asked: of sequences that have rows, so at most max_rows + b)
    int32_t rows_of[PER], asked_of[PER], back_of[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int32_t c = count[i], m = len[i];
        rows = add_saturating(rows, c < 0 ? 0 : (c > kRowsSaturate ? kRowsSaturate : c));
        if (m > cap) {
            bits |= kStatusBadRequestBit;
            len[i] = -1;
        } else if (m >= 0) {
            const int32_t held = pages_of(m);
            if (c < 0) {
                back = add_saturating(back, held < kRowsSaturate ? held : kRowsSaturate);
            } else if (rows <= a.max_rows && c <= cap - m) {
                asked += pages_of(m + c) - held;
            } else {
                len[i] = -1;
                if (c > 0) bits |= kStatusCapacityBit;
            }
        }
        rows_of[i] = rows;
        asked_of[i] = asked;
        back_of[i] = back;
    }
    const int2 before = sums_before(asked, back, wave_sums);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (s0 + i < b) {
            rows_to[s0 + i] = rows_of[i];
            asked_to[s0 + i] = asked_of[i] + before.x;
            back_to[s0 + i] = add_saturating(back_of[i], before.y);
            held_len[s0 + i] = len[i];
        }
    __syncthreads();

    const int32_t total_rows = rows_to[b - 1];
    int32_t returned = back_to[b - 1];
    if (returned > a.n_pages - free) {             // more than the pool has: a table that names pages twice
        returned = a.n_pages - free;
        bits |= kStatusBadRequestBit;
    }
    const int stride = gridDim.x * THREADS, at = blockIdx.x * THREADS + tid;
    // pages that are given out: of the sequences that ask, those up to the first one whose pages are not all there
    int32_t given = asked_to[b - 1];
    if (given > free) {
        const int s = above(asked_to, b, free);    // the first one refused
        given = s ? asked_to[s - 1] : 0;
    }

    // 1. each sequence's length and first row
    for (int s = at; s < b; s += stride) {
        const int32_t c = a.new_cnt[s], m = held_len[s], asked0 = s ? asked_to[s - 1] : 0;
        int32_t n = m;
        if (m < 0) {
            n = a.cache_len[s];
        } else if (c < 0) {
            n = 0;
        } else if (c > 0) {
            if (asked_to[s] == asked0 || asked_to[s] <= given) n = m + c; else bits |= kStatusCapacityBit;
        }
        a.new_len[s] = n;
        a.row_start[s] = s ? rows_to[s - 1] : 0;
    }
    if (first && tid == 0) {
        a.row_start[b] = total_rows;
        a.free_state_out[0] = in_ring(given);
        a.free_state_out[1] = free - given + returned;
    }

    // 2. fresh pages
    for (int32_t k = at; k < given; k += stride) {
        const int s = above(asked_to, b, k);
        const int32_t page = a.free_ring[in_ring(k)];
        if ((uint32_t)page >= (uint32_t)a.n_pages) bits |= kStatusBadRequestBit;
        a.block_table[(int64_t)s * a.max_pages + pages_of(held_len[s]) + (k - (s ? asked_to[s - 1] : 0))] = page;
    }

    // 3. returned pages
    for (int32_t k = at; k < returned; k += stride) {
        const int s = above(back_to, b, k);
        const int32_t page = a.block_table[(int64_t)s * a.max_pages + (k - (s ? back_to[s - 1] : 0))];
        if ((uint32_t)page >= (uint32_t)a.n_pages) bits |= kStatusBadRequestBit;
        a.free_ring[in_ring(free + k)] = page;
    }

    // 4. rows
    for (int32_t r = at; r < a.max_rows; r += stride) {
        int32_t slot = -1, pos = 0;
        if (r < total_rows) {
            const int s = above(rows_to, b, r);
            const int32_t m = held_len[s], asked0 = s ? asked_to[s - 1] : 0;
            if (m >= 0 && (asked_to[s] == asked0 || asked_to[s] <= given)) {
                const int32_t t = m + (r - (s ? rows_to[s - 1] : 0)), j = pages_of(t + 1) - 1, held = pages_of(m);
                const int32_t page = j < held ? a.block_table[(int64_t)s * a.max_pages + j] : a.free_ring[in_ring(asked0 + (j - held))];
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
    PlanArgs a{new_cnt, cache_len, new_len, block_table, free_ring, free_state, free_state_out, row_start, slot, pos,
               paged_status(workspace), p.b, p.page_size, p.n_pages, p.max_pages, max_rows, 0, 0};
    page_divisor(p.page_size, a.page_mul, a.page_shift);
    const int64_t items = max_rows > p.b ? max_rows : p.b;
    const size_t lds = paged_plan_lds(p.b);
    static_assert(4 * sizeof(int32_t) * plan_room(SWA_MAX_PAGED_SEQS) <= 64 * 1024 && SWA_MAX_PAGED_SEQS <= 4 * 1024, "a workgroup holds all sums");
    // 1024 sequences with 256 / 512 / 1024 threads in a workgroup 8.5 / 7.3 / 8.1 us; 4096 with 256 / 1024 15.9 / 10.4; 1 and 256 sequences 3.7 and 4.9,
    // a launch that does nothing 3.5
    auto launch = [&](auto kernel, int threads) {
        int64_t grid = (items + threads - 1) / threads;
        if (grid > 256) grid = 256;
        launch_kernel(kernel, dim3((unsigned)grid), dim3(threads), lds, stream, a);
    };
    if (p.b <= 256) launch(swa_paged_plan_kernel<256, 1>, 256);
    else if (p.b <= 1024) launch(swa_paged_plan_kernel<512, 2>, 512);
    else launch(swa_paged_plan_kernel<1024, 4>, 1024);
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
