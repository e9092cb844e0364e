// Smallest and largest key values of pages, channel by channel: what swa_paged_score reads instead of the keys.
//
// The minimum of a page that grows is the minimum of what it was and of the new keys, so a call reads its new rows, and the old values of the pages that
// had tokens before.  Bound: the launch for a step (64 sequences, 8 key heads of 128 bf16 channels, 3.5 us) and its chain of loads for prompts: slots, rows, the page's old
// values.  A wave takes one key head of a page: the call's rows of that page follow each other in `slot`, the first of them finds the others, a load fetches as many whole rows
// as the wave holds, and four loads are under way at once (9.5 MB of 8-bit codes, pages of 64: 7.3 us; one load at a time, and teams of lanes joined by way of LDS, 9.7).
// Pages of thousands of tokens leave a prompt few waves; a score of so many tokens says little, and the kernel is not made for them.
#include <type_traits>

#include "swa_paged.hpp"

namespace swa {

struct BoundsArgs {
    const char* k_pages;
    const float* k_scale;
    char* bounds;
    const int32_t* slot;
    int32_t* status;
    int32_t n_rows, h_kv, page_size, n_pages;
    int32_t rows, head_groups;                     // rows of a wave, and waves that share its heads
    uint32_t page_mul;
    int32_t page_shift;
};

// (both keep what is no number)
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float most(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ int8_t code_at(const Vec16& v, int i)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    return (int8_t)(w[i >> 2] >> (8 * (i & 3)));
}

// T: type of the bounds, C: of the pages (Q8: codes).
template <typename T, typename C, int D>
__global__ void __launch_bounds__(256) swa_paged_bounds_kernel(BoundsArgs a)
{
    constexpr bool kCodes = std::is_same_v<C, Q8>;
    constexpr int kRow = D * Elem<C>::kBytes, kLanes = kRow / 16, kTeams = 64 / kLanes, kVec = Elem<C>::kPerVec;
    const int lane = threadIdx.x & 63, team = lane / kLanes, at = lane % kLanes;
    const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), block = wave / a.head_groups,
              head0 = wave - block * a.head_groups;
    const int r0 = block * a.rows;
    if (r0 >= a.n_rows) return;
    const int32_t slots = a.n_pages * a.page_size;
    auto page_of = [&](int32_t slot) { return (int32_t)(((uint64_t)(uint32_t)slot * a.page_mul) >> a.page_shift); };
    // (a slot outside the pool is no row's, like a negative one)
    auto page_at = [&](int r) {
        const int32_t slot = r >= 0 && r < a.n_rows ? a.slot[r] : -1;
        return slot >= 0 && slot < slots ? page_of(slot) : -1;
    };
    const int r = r0 + lane;
    const int32_t own = lane < a.rows ? page_at(r) : -1, before = lane < a.rows ? page_at(r - 1) : -1;
    if (lane < a.rows && r < a.n_rows && a.slot[r] >= slots && head0 == 0) atomicOr(a.status, kStatusBadRequestBit);
    uint64_t firsts = __ballot(own >= 0 && own != before);
    while (firsts) {
        const int first = __builtin_ctzll(firsts);
        firsts &= firsts - 1;
        const int32_t page = __builtin_amdgcn_readlane(own, first);
        // the rows behind the first, 64 at a time
        for (int head = head0; head < a.h_kv; head += a.head_groups) {
            const int64_t row0 = ((int64_t)page * a.h_kv + head) * a.page_size;
            float lo[kVec], hi[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                lo[i] = INFINITY;
                hi[i] = -INFINITY;
            }
            bool fresh = false;
            for (int from = r0 + first;; from += 64) {
                const int mine = from + lane;
                const uint64_t others = ~__ballot(page_at(mine) == page);
                const int count = others ? (int)__builtin_ctzll(others) : 64;
                const int32_t off = lane < count ? a.slot[mine] - page * a.page_size : 0;
                fresh |= __ballot(lane < count && off == 0) != 0;
                constexpr int kAhead = 4;                // loads under way at once
                for (int i = 0; i < count; i += kAhead * kTeams) {
                    Vec16 v[kAhead];
                    float scale[kAhead];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) {
                        const int row = i + k * kTeams + team;           // (the last one again where there are no more)
                        const int64_t at_row = row0 + __shfl(off, row < count ? row : count - 1, 64);
                        v[k] = load16(a.k_pages + at_row * kRow + at * 16);
                        if constexpr (kCodes) scale[k] = a.k_scale[at_row];
                    }
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) {
                        float f[kVec];
                        if constexpr (kCodes) {
#pragma unroll
                            for (int x = 0; x < kVec; ++x) f[x] = (float)code_at(v[k], x) * scale[k];
                        } else {
                            unpack<C>(v[k], f);
                        }
#pragma unroll
                        for (int x = 0; x < kVec; ++x) {
                            lo[x] = least(lo[x], f[x]);
                            hi[x] = most(hi[x], f[x]);
                        }
                    }
                }
                if (count < 64) break;
            }
            // the teams to one: lanes 8, 16 and 32 apart, as far as these are teams
#pragma unroll
            for (int x = 0; x < kVec; ++x) {
                if constexpr (kLanes <= 4) {
                    lo[x] = least(lo[x], __shfl_xor(lo[x], 4, 64));
                    hi[x] = most(hi[x], __shfl_xor(hi[x], 4, 64));
                }
                if constexpr (kLanes <= 8) {
                    lo[x] = least(lo[x], dpp_move<0x128>(lo[x]));        // row_ror 8
                    hi[x] = most(hi[x], dpp_move<0x128>(hi[x]));
                }
                if constexpr (kLanes <= 16) {
                    lo[x] = least(lo[x], __shfl_xor(lo[x], 16, 64));
                    hi[x] = most(hi[x], __shfl_xor(hi[x], 16, 64));
                }
                float a0, a1;
                both_halves(lo[x], a0, a1);
                lo[x] = least(a0, a1);
                both_halves(hi[x], a0, a1);
                hi[x] = most(a0, a1);
            }
            if (team) continue;
            constexpr int kT = Elem<T>::kBytes, kPer = Elem<T>::kPerVec;
            char* const to = a.bounds + ((int64_t)page * a.h_kv + head) * (2 * D * kT) + at * kVec * kT;
#pragma unroll
            for (int x = 0; x < kVec; x += kPer) {
                if (!fresh) {
                    float f[kPer];
                    unpack<T>(load16(to + x * kT), f);
#pragma unroll
                    for (int i = 0; i < kPer; ++i) lo[x + i] = least(lo[x + i], f[i]);
                    unpack<T>(load16(to + D * kT + x * kT), f);
#pragma unroll
                    for (int i = 0; i < kPer; ++i) hi[x + i] = most(hi[x + i], f[i]);
                }
                store16(to + x * kT, pack<T>(lo + x));
                store16(to + D * kT + x * kT, pack<T>(hi + x));
            }
        }
    }
}

int launch_paged_bounds(const swa_paged_params& p, int32_t n_rows, const int32_t* slot, const void* k_pages, const float* k_scale, void* bounds,
                        void* workspace, hipStream_t stream)
{
    BoundsArgs a{};
    a.k_pages = static_cast<const char*>(k_pages);
    a.k_scale = k_scale;
    a.bounds = static_cast<char*>(bounds);
    a.slot = slot;
    a.status = paged_status(workspace);
    a.n_rows = n_rows;
    a.h_kv = p.h_kv;
    a.page_size = p.page_size;
    a.n_pages = p.n_pages;
    page_divisor(p.page_size, a.page_mul, a.page_shift);
    // Two thousand waves where there is work for them: one row each, and as many heads apart, before rows are taken together.
    a.rows = 1;
    a.head_groups = p.h_kv < 64 ? p.h_kv : 64;
    while (a.rows < 16 && (int64_t)n_rows * a.head_groups > 4096 * (int64_t)a.rows) a.rows *= 2;
    const int64_t blocks = ((int64_t)n_rows + a.rows - 1) / a.rows;
    while (a.head_groups > 1 && blocks * a.head_groups > (1 << 22)) a.head_groups = (a.head_groups + 1) / 2;
    const dim3 grid((unsigned)((blocks * a.head_groups + 3) / 4));
#define SWA_BOUNDS(T, C) (p.d == 64 ? launch_kernel(swa_paged_bounds_kernel<T, C, 64>, grid, dim3(256), 0, stream, a) \
                                    : launch_kernel(swa_paged_bounds_kernel<T, C, 128>, grid, dim3(256), 0, stream, a))
    if (p.dtype == SWA_F32) SWA_BOUNDS(F32, F32);
    else if (p.dtype == SWA_F16) paged_int8(p) ? SWA_BOUNDS(F16, Q8) : SWA_BOUNDS(F16, F16);
    else paged_int8(p) ? SWA_BOUNDS(BF16, Q8) : SWA_BOUNDS(BF16, BF16);
#undef SWA_BOUNDS
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
