// Attention of one new token per sequence over a prefix that several sequences share, and over each one's own pages.
//
// A prefix's keys and values are read for all of its sequences at once: their query heads are the columns of its products, 16 ROWS of them to a workgroup.  The call's
// work is prefixes, then sequences, each by key head and tile of columns, in steps of 128 tokens; laid end to end it is cut into as many equal shares as there are
// workgroups, whatever the lengths and the numbers of sequences are.  Every workgroup sums it up by itself.  A share's part of a unit (one prefix or sequence, key head
// and tile) is a partial result of each of its columns; a second launch joins the prefix's and the sequence's own ones in their order.
//   Partial results: unit u's column i from share g lies at R_u + 16 ROWS g + i, with R_u the columns of the units before it: units and shares follow each
//   other in the same order, and a share that ends one unit begins the next behind that one's columns, so no two of them meet.
#include "swa_paged_tile.hpp"

namespace swa {

// Where the join finds a sequence's partial results (row < 0: the call leaves the sequence out).
struct alignas(16) SharedPlace {
    int32_t row, rank;                             // its row, and its number among the prefix's sequences
    int32_t members, prefix_at, prefix_steps;      // those, the prefix's first step (of one key head, like `at`), the steps of a unit
    int32_t first;                                 // sequences of the prefixes before
    int32_t at, steps;                             // of the sequence itself
};

struct SharedArgs {
    const char* q;
    int64_t q_stride;                              // bytes
    PagedRows rows;
    PagedPool pool;
    const int32_t *block_table, *prefix_of;
    char* out;
    float* lse;
    float *part_out, *part_sum;                    // [columns, D] and [.., 2] (maximum, sum)
    SharedPlace* place;                            // [b], and behind them the steps of the call
    int32_t* status;
    int32_t b, h_q, h_kv, page_size, n_pages, max_pages;
    int32_t group, shares;
    uint32_t page_mul;                             // t / page_size = t * page_mul >> page_shift for 0 <= t < 2^31
    int32_t page_shift;
    int32_t sixteens;                              // pages are whole sixteens of tokens
};

constexpr int kNoPrefix = 0, kLeftOut = 0xffff;    // of a sequence, where it has no prefix or the call leaves it out; else the prefix's number and 1

__device__ __forceinline__ int steps_of(int tokens) { return (tokens + kPagedStep - 1) / kPagedStep; }

// Tokens begin .. end - 1 of the pages in `table`, for query columns whose rows begin at from(g).
template <typename T, typename C, int D, int ROWS, typename Q, typename F>
__device__ __forceinline__ void shared_part(const SharedArgs& a, const int32_t* table, int kv, int begin, int end, int columns, float (&part)[4][16][D + 4],
                                            float (&tops)[4][16], float (&sums)[4][16], Q from, F emit)
{
    typedef PagedTile<T, C, D, ROWS> S;
    constexpr int kKeys = S::kKeys, kSteps = S::kSteps, kChannels = S::kChannels, kStride = 4 * kKeys;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, j = lane >> 4;
    Vec16 q[ROWS][kSteps];
#pragma unroll
    for (int g = 0; g < ROWS; ++g) {
        const bool there = 16 * g + col < columns;
        const char* const at = from(there ? 16 * g + col : 0);
#pragma unroll
        for (int c = 0; c < kSteps; ++c) q[g][c] = there ? load16(at + S::query_at(c, j)) : Vec16{0u, 0u, 0u, 0u};
    }
    float top[ROWS], sum[ROWS];
    f32x4_t acc[ROWS][kChannels];
#pragma unroll
    for (int g = 0; g < ROWS; ++g) {
        top[g] = -INFINITY;
        sum[g] = 0.f;
#pragma unroll
        for (int e = 0; e < kChannels; ++e) acc[g][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    bool bad = false;
    auto page_of = [&](int base) {
        const int t = base + (lane & (kKeys - 1));
        return (int)(((uint64_t)(uint32_t)(t < end ? t : end - 1) * a.page_mul) >> a.page_shift);
    };
    auto row_of = [&](int base, int page) {
        const int t = base + (lane & (kKeys - 1));
        const bool live = t < end, in_pool = (uint32_t)page < (uint32_t)a.n_pages;
        bad |= live && !in_pool;
        return live && in_pool ? (page * a.h_kv + kv) * a.page_size + t - page_of(base) * a.page_size : -1;
    };
    int next = begin + wave * kKeys, page = 0;
    if (next < end) page = table[page_of(next)];
    int left = next, left_end = end, r = 0;
    if (a.sixteens) {
        left = end;
        left_end = begin;
        while (next < end) {
            const int base = next, this_page = page;
            next += kStride;
            if (next < end) page = table[page_of(next)];
            const int rows = row_of(base, this_page);
            if (!__any(rows < 0)) {
                paged_take<T, C, D, ROWS, true>(a.pool, rows, q, top, sum, acc);
            } else {
                if (left == end) {
                    left = base;
                    r = rows;
                }
                left_end = base + 1;
            }
        }
    } else if (next < end) {
        r = row_of(next, page);
    }
    while (left < left_end) {
        paged_take<T, C, D, ROWS, false>(a.pool, r, q, top, sum, acc);
        do {
            left += kStride;
            if (left >= left_end) break;
            r = row_of(left, table[page_of(left)]);
        } while (a.sixteens && !__any(r < 0));
    }
    if (bad) atomicOr(a.status, kStatusBadRequestBit);
    int who = threadIdx.x;
    asm volatile("" : "+v"(who));                        // (addresses made from it are not kept in registers around the loop)
    paged_join_waves<T, C, D, ROWS, 4>(part, tops, sums, top, sum, acc, columns, who, emit);
}

// OWN: sixteens of columns in a unit of a sequence's own tokens, ROWS: of a prefix's.
template <typename T, typename C, int D, int ROWS, int OWN>
__global__ void __launch_bounds__(256, Elem<C>::kBytes * D == 512 && ROWS == 2 ? 1 : 2) swa_paged_shared_kernel(SharedArgs a)
{
    constexpr int kColumns = 16 * (ROWS > OWN ? ROWS : OWN), kOwn = 16 * OWN, kTile = 16 * ROWS;
    __shared__ float part[4][16][D + 4];
    __shared__ float tops[4][16], sums[4][16];
    __shared__ int scratch[4], member_row[kTile + 1];
    extern __shared__ int before[];                      // steps of a key head before prefix e, and before sequence e - b, for e <= 2 b
    uint16_t* const members = reinterpret_cast<uint16_t*>(before + 2 * a.b + 1);     // sequences of the prefixes before, b + 1 of them
    uint16_t* const prefix = members + a.b + 1;          // of a sequence
    const int tid = threadIdx.x, lane = tid & 63, b = a.b;
    // (shares that follow each other run on the same XCD, so that tiles of one prefix meet in its L2)
    const int share = (blockIdx.x & 7) * (a.shares >> 3) + (blockIdx.x >> 3), own_tiles = (a.group + kOwn - 1) / kOwn;

    for (int i = tid; i <= b; i += 256) before[i] = 0;
    __syncthreads();
    int bits = 0;
    for (int s = tid; s < b; s += 256) {
        int row, n, of = a.prefix_of[s], is = kLeftOut, steps = 0;
        bool too_long = false;
        if (paged_row(a.rows, s, row, n, too_long)) {
            is = kNoPrefix;
            if (of != -1) {
                const bool known = of >= 0 && of < b && of != s;
                const int m = known ? a.rows.cache_len[of] : -1;
                if (m < 0) bits |= kStatusBadRequestBit;
                else if (m > a.rows.len_max) bits |= kStatusCapacityBit;
                is = m < 0 || m > a.rows.len_max ? kLeftOut : of + 1;
            }
            if (is != kLeftOut) steps = steps_of(n) * own_tiles;
            if (is != kLeftOut && is != kNoPrefix) atomicAdd(&before[1 + of], 1);
        }
        if (too_long) bits |= kStatusCapacityBit;
        prefix[s] = (uint16_t)is;
        before[1 + b + s] = steps;
    }
    if (bits && blockIdx.x == 0) atomicOr(a.status, bits);
    __syncthreads();
    const int per = (b + 255) / 256, s0 = tid * per, s1 = s0 + per < b ? s0 + per : b;
    {
        int own = 0;
        for (int p = s0; p < s1; ++p) own += before[1 + p];
        int at = sum_to(own, scratch) - own;
        for (int p = s0; p < s1; ++p) {
            const int m = before[1 + p];
            members[p] = (uint16_t)at;
            at += m;
            before[1 + p] = m ? steps_of(a.rows.cache_len[p]) * ((m * a.group + kTile - 1) / kTile) : 0;
            if (p == b - 1) members[b] = (uint16_t)at;
        }
    }
    __syncthreads();
    {
        const int each = (2 * b + 255) / 256, e0 = tid * each, e1 = e0 + each < 2 * b ? e0 + each : 2 * b;
        int own = 0;
        for (int e = e0; e < e1; ++e) own += before[1 + e];
        int at = sum_to(own, scratch) - own;
        for (int e = e0; e < e1; ++e) {
            at += before[1 + e];
            before[1 + e] = at;
        }
    }
    __syncthreads();
    const int total = __builtin_amdgcn_readfirstlane(before[2 * b]) * a.h_kv;
    const PagedShares shares(total, a.shares);
    // what the join asks of this call: a wave has a sequence
    for (int s = blockIdx.x * 4 + (tid >> 6); s < b; s += gridDim.x * 4) {
        const int is = prefix[s];
        int rank = 0;
        if (is != kNoPrefix && is != kLeftOut)
            for (int i = lane; i < s; i += 64) rank += prefix[i] == is;
#pragma unroll
        for (int o = 32; o; o >>= 1) rank += __shfl_xor(rank, o, 64);
        if (lane == 0) {
            SharedPlace to{-1, rank, 0, 0, 0, 0, before[b + s], (before[1 + b + s] - before[b + s]) / own_tiles};
            if (is != kLeftOut) to.row = a.rows.row_start ? a.rows.row_start[s + 1] - 1 : s;
            if (is != kNoPrefix && is != kLeftOut) {
                to.members = members[is] - members[is - 1];
                to.first = members[is - 1];
                to.prefix_at = before[is - 1];
                to.prefix_steps = (before[is] - before[is - 1]) / ((to.members * a.group + kTile - 1) / kTile);
            }
            a.place[s] = to;
        }
    }
    if (blockIdx.x == 0 && tid == 0) *reinterpret_cast<int32_t*>(a.place + b) = total;

    int x = shares.begin(share), e = 0;
    const int x1 = shares.begin(share + 1);
    for (int above = 2 * b; e + 1 < above;) {
        const int mid = (e + above) >> 1;
        if (before[mid] * a.h_kv <= x) e = mid; else above = mid;
    }
    e = __builtin_amdgcn_readfirstlane(e);
    while (x < x1) {
        const int e_before = __builtin_amdgcn_readfirstlane(before[e]), of_head = __builtin_amdgcn_readfirstlane(before[e + 1]) - e_before;
        if (of_head == 0) {
            ++e;
            continue;
        }
        const bool is_prefix = e < b;
        const int s = is_prefix ? e : e - b, at_member = __builtin_amdgcn_readfirstlane((int)members[is_prefix ? e : 0]),
                  count = is_prefix ? __builtin_amdgcn_readfirstlane((int)members[e + 1]) - at_member : 1;
        const int columns = count * a.group, width = is_prefix ? kTile : kOwn, tiles = (columns + width - 1) / width, steps = of_head / tiles;
        const int in_e = x - e_before * a.h_kv, unit = in_e / steps, kv = unit / tiles, tile = unit - kv * tiles, first = in_e - unit * steps;
        const int last = steps - first < x1 - x ? steps : first + (x1 - x), n = a.rows.cache_len[s];
        const int begin = first * kPagedStep, end = last == steps ? n : last * kPagedStep, here = columns - tile * width < width ? columns - tile * width : width;
        const int64_t to = (int64_t)a.group * a.h_kv * (is_prefix ? at_member : b + s) + (int64_t)kv * columns + tile * width + (int64_t)share * kColumns;
        const int32_t* const table = a.block_table + (int64_t)s * a.max_pages;
        auto emit = [&](int i, float all, float sum, const float (&y)[D / 16]) __attribute__((always_inline)) {
            const int64_t at = to + i;
            const int c = (tid & 15) * (D / 16);
#pragma unroll
            for (int z = 0; z < D / 16; z += 4) *reinterpret_cast<f32x4_t*>(a.part_out + at * D + c + z) = f32x4_t{y[z], y[z + 1], y[z + 2], y[z + 3]};
            if (c == 0) *reinterpret_cast<float2*>(a.part_sum + at * 2) = float2{all, sum};
        };
        if (is_prefix) {
            // rows of the sequences whose heads are columns of this tile
            const int rank0 = tile * kTile / a.group, rank1 = (tile * kTile + here + a.group - 1) / a.group;
            int own = 0;
            for (int i = s0; i < s1; ++i) own += prefix[i] == e + 1;
            int rank = sum_to(own, scratch) - own;
            for (int i = s0; i < s1; ++i)
                if (prefix[i] == e + 1) {
                    if (rank >= rank0 && rank < rank1) member_row[rank - rank0] = a.rows.row_start ? a.rows.row_start[i + 1] - 1 : i;
                    ++rank;
                }
            __syncthreads();
            shared_part<T, C, D, ROWS>(a, table, kv, begin, end, here, part, tops, sums,
                                       [&](int i) __attribute__((always_inline)) {
                                           const int at = tile * kTile + i, rank = at / a.group;
                                           return a.q + member_row[rank - rank0] * a.q_stride + ((int64_t)kv * a.group + at - rank * a.group) * (D * Elem<T>::kBytes);
                                       },
                                       emit);
        } else {
            const int row = a.rows.row_start ? a.rows.row_start[s + 1] - 1 : s;
            const char* const heads = a.q + row * a.q_stride + ((int64_t)kv * a.group + tile * kOwn) * (D * Elem<T>::kBytes);
            shared_part<T, C, D, OWN>(a, table, kv, begin, end, here, part, tops, sums,
                                      [&](int i) __attribute__((always_inline)) { return heads + (int64_t)i * (D * Elem<T>::kBytes); }, emit);
        }
        x += last - first;
        if (x == (e_before + of_head) * a.h_kv) ++e;
    }
}

// A query head's partial results, the prefix's and its own, to its output.
template <typename T, int D>
__global__ void __launch_bounds__(256) swa_paged_join_shared_kernel(SharedArgs a, int tile, int own_tile)
{
    const int s = blockIdx.x / a.h_q, hq = blockIdx.x - s * a.h_q, kv = hq / a.group, head = hq - kv * a.group;
    const SharedPlace at = a.place[s];
    if (at.row < 0) return;
    const PagedShares shares(*reinterpret_cast<const int32_t*>(a.place + a.b), a.shares);
    const int width = tile > own_tile ? tile : own_tile;
    int64_t first[2];
    int count[2] = {0, 0};
    auto unit = [&](int which, int x, int steps, int64_t columns) __attribute__((always_inline)) {
        const int f = shares.of(x);
        count[which] = shares.of(x + steps - 1) - f + 1;
        first[which] = columns + (int64_t)f * width;
    };
    first[0] = first[1] = 0;
    if (at.prefix_steps > 0) {
        const int columns = at.members * a.group, i = at.rank * a.group + head, tiles = (columns + tile - 1) / tile;
        unit(0, at.prefix_at * a.h_kv + (kv * tiles + i / tile) * at.prefix_steps, at.prefix_steps,
             (int64_t)a.group * a.h_kv * at.first + (int64_t)kv * columns + i);
    }
    if (at.steps > 0) {
        const int tiles = (a.group + own_tile - 1) / own_tile;
        unit(1, at.at * a.h_kv + (kv * tiles + head / own_tile) * at.steps, at.steps, (int64_t)a.group * a.h_kv * (a.b + s) + (int64_t)kv * a.group + head);
    }
    paged_join_pieces<T, D>(a.part_out, a.part_sum, [&](int i) __attribute__((always_inline)) { return i < count[0] ? first[0] + (int64_t)i * width : first[1] + (int64_t)(i - count[0]) * width; },
                            count[0] + count[1], a.out, a.lse, (int64_t)at.row * a.h_q + hq);
}

constexpr int kSharedShares = 512;                 // two workgroups to a CU
constexpr size_t kSharedOwnLds = 36 * 1024;        // of the kernel, at most, beside the lists

// Sixteens of columns of a prefix's unit.
static int shared_rows(const swa_paged_params& p) { return (int64_t)(p.b - 1) * (p.h_q / p.h_kv) <= 16 ? 1 : 2; }

static int64_t shared_columns(const swa_paged_params& p) { return 2 * (int64_t)p.b * p.h_q + (int64_t)kSharedShares * 32; }

size_t paged_shared_bytes(const swa_paged_params& p)
{
    return (size_t)shared_columns(p) * (p.d + 2) * sizeof(float) + ((size_t)p.b + 1) * sizeof(SharedPlace);
}

template <typename T, typename C, int D>
static int launch_shared_form(const SharedArgs& a, int rows, int own, hipStream_t stream)
{
    auto kernel = rows == 1 ? (own == 1 ? swa_paged_shared_kernel<T, C, D, 1, 1> : swa_paged_shared_kernel<T, C, D, 1, 2>)
                            : (own == 1 ? swa_paged_shared_kernel<T, C, D, 2, 1> : swa_paged_shared_kernel<T, C, D, 2, 2>);
    const size_t lds = sizeof(int) * (2 * (size_t)a.b + 1) + sizeof(uint16_t) * (2 * (size_t)a.b + 1) + 2;
    if (lds + kSharedOwnLds > 64 * 1024) {
        const int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), lds > 49 * 1024 ? lds : 49 * 1024);
        if (rc != SWA_OK) return rc;
    }
    launch_kernel(kernel, dim3((unsigned)a.shares), dim3(256), lds, stream, a);
    launch_kernel(swa_paged_join_shared_kernel<T, D>, dim3((unsigned)(a.b * a.h_q)), dim3(256), 0, stream, a, 16 * rows, 16 * own);
    return SWA_OK;
}

int launch_paged_shared(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                        const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                        const int32_t* cache_len, const int32_t* prefix_of, void* out, float* lse, void* workspace, hipStream_t stream)
{
    SharedArgs a{};
    a.q = static_cast<const char*>(q.data);
    a.q_stride = q.stride * (p.dtype == SWA_F32 ? 4 : 2);
    a.rows = PagedRows{row_start, slot, cache_len, n_rows, paged_len_max(p)};
    a.pool = PagedPool{static_cast<const char*>(k_pages), static_cast<const char*>(v_pages), k_scale, v_scale,
                       (p.scale > 0.f ? p.scale : 1.f / sqrtf((float)p.d)) * 1.44269504088896340736f};
    a.block_table = block_table;
    a.prefix_of = prefix_of;
    a.out = static_cast<char*>(out);
    a.lse = lse;
    a.part_out = reinterpret_cast<float*>(static_cast<char*>(workspace) + kPagedPartialOffset);
    a.part_sum = a.part_out + shared_columns(p) * p.d;
    a.place = reinterpret_cast<SharedPlace*>(a.part_sum + shared_columns(p) * 2);
    a.status = paged_status(workspace);
    a.b = p.b;
    a.h_q = p.h_q;
    a.h_kv = p.h_kv;
    a.page_size = p.page_size;
    a.n_pages = p.n_pages;
    a.max_pages = p.max_pages;
    a.group = p.h_q / p.h_kv;
    a.shares = kSharedShares;
    page_divisor(p.page_size, a.page_mul, a.page_shift);
    a.sixteens = p.page_size % 16 == 0;
    const int rows = shared_rows(p), own = a.group > 16 ? 2 : 1;
    // (steps are 32-bit numbers: of every sequence's own tokens, and of as many prefixes as may be)
    const int64_t tiles = (int64_t)p.b * ((a.group + 16 * own - 1) / (16 * own)) + ((int64_t)p.b * a.group + 16 * rows - 1) / (16 * rows) + p.b;
    if (tiles * p.h_kv > 0x7fffffffLL / ((a.rows.len_max + kPagedStep - 1) / kPagedStep) || (uint64_t)p.b * p.h_q * 256 > 0xffffffffULL) return SWA_ERR_CAPACITY;
#define SWA_SHARED(T, C) (p.d == 64 ? launch_shared_form<T, C, 64>(a, rows, own, stream) : launch_shared_form<T, C, 128>(a, rows, own, stream))
    const int rc = p.dtype == SWA_F32   ? SWA_SHARED(F32, F32)
                   : p.dtype == SWA_F16 ? (paged_int8(p) ? SWA_SHARED(F16, Q8) : SWA_SHARED(F16, F16))
                                        : (paged_int8(p) ? SWA_SHARED(BF16, Q8) : SWA_SHARED(BF16, BF16));
#undef SWA_SHARED
    if (rc != SWA_OK) return rc;
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
