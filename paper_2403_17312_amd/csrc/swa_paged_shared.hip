// Attention of one new token per sequence over a prefix that several sequences share, and over each one's own pages.
//
// A prefix's keys and values are read for all of its sequences at once: their query heads are the columns of its products.  Units of work are a prefix, key head and tile of
// columns, and a sequence, key head and up to 16 of its query heads.  The prefixes' units, in steps of 128 tokens, are laid end to end and cut into as many equal shares as there
// are workgroups, and the sequences', in steps of 32, into as many as there are waves, whatever the lengths and the numbers of sequences are; every workgroup sums both up by
// itself.  So each has as much of either as the others, and a wave has a short sequence to itself, with no other wave to wait for (as units of eight waves they took 5 us each: 64
// sequences of 1 to 300 tokens behind 32768, 64 query and 8 key heads, 177 us on the last workgroups, 89 on the others).
//   A share's part of a unit is a partial result of each of its columns; a second launch joins the prefix's and the sequence's own ones in their order.  Unit u's column i
// from share g lies at R_u + W g + i, with R_u the columns of the units before it and W the columns of a unit at most: units and shares follow each other in the same order, and a
// share that ends one unit begins the next behind that one's columns, so no two of them meet.
#include "swa_paged_tile.hpp"

namespace swa {

// Where the join finds a sequence's partial results (row < 0: the call leaves the sequence out).
struct alignas(16) SharedPlace {
    int32_t row, rank;                             // its row, and its number among the prefix's sequences
    int32_t members, prefix_at, prefix_steps;      // those, the prefix's first step (of one key head, like `at`), the steps of a unit
    int32_t first;                                 // sequences of the prefixes before
    int32_t at, steps;                             // of the sequence itself, likewise
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
    SharedPlace* place;                            // [b], and behind them the steps of all prefixes, and of all sequences
    int32_t* status;
    int32_t b, h_q, h_kv, page_size, n_pages, max_pages;
    int32_t group, shares;                         // workgroups
    int64_t own_columns;                           // partial results of the prefixes, before those of the sequences
    uint32_t page_mul;                             // t / page_size = t * page_mul >> page_shift for 0 <= t < 2^31
    int32_t page_shift;
    int32_t sixteens;                              // pages are whole sixteens of tokens
    int32_t own_log;                               // tokens of a sequence's own step, as a power of two
};

constexpr int kNoPrefix = 0, kLeftOut = 0xffff;    // of a sequence, where it has no prefix or the call leaves it out; else the prefix's number and 1

__device__ __forceinline__ int steps_of(int tokens) { return (tokens + kPagedStep - 1) / kPagedStep; }

// A sequence's own tokens: steps of 32 (of more where a call could have 2^31 of them), and one that stands for what a unit costs before its first key.
constexpr int kOwnLog = 5, kOwnColumns = 16;
__host__ __device__ __forceinline__ int own_steps_of(int tokens, int log) { return tokens > 0 ? 1 + ((tokens - 1) >> log) + 1 : 0; }

// A partial result, by sixteen threads.
template <int D>
struct SharedEmit {
    float *part_out, *part_sum;
    int64_t to;                                          // of column 0
    __device__ __forceinline__ void operator()(int i, float all, float sum, const float (&y)[D / 16]) const
    {
        const int64_t at = to + i;
        const int c = (threadIdx.x & 15) * (D / 16);
#pragma unroll
        for (int z = 0; z < D / 16; z += 4) *reinterpret_cast<f32x4_t*>(part_out + at * D + c + z) = f32x4_t{y[z], y[z + 1], y[z + 2], y[z + 3]};
        if (c == 0) *reinterpret_cast<float2*>(part_sum + at * 2) = float2{all, sum};
    }
};

// Results of waves on their way to one.
template <int D, int WAVES>
struct SharedLds {
    float part[WAVES][16][D + 4];
    float tops[WAVES][16], sums[WAVES][16];
};

// Tokens begin .. end - 1 of the pages in `table`, for query columns whose rows begin at from(column).
template <typename T, typename C, int D, int ROWS, int WAVES, bool STREAM, typename Q, typename F>
__device__ __forceinline__ void shared_part(const SharedArgs& a, const int32_t* table, int kv, int begin, int end, int columns, SharedLds<D, WAVES>& lds, Q from, F emit)
{
    typedef PagedTile<T, C, D, ROWS> S;
    constexpr int kKeys = S::kKeys, kSteps = S::kSteps, kChannels = S::kChannels, kStride = WAVES * kKeys;
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
                paged_take<T, C, D, ROWS, true, STREAM>(a.pool, rows, q, top, sum, acc);
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
        paged_take<T, C, D, ROWS, false, STREAM>(a.pool, r, q, top, sum, acc);
        do {
            left += kStride;
            if (left >= left_end) break;
            r = row_of(left, table[page_of(left)]);
        } while (a.sixteens && !__any(r < 0));
    }
    if (bad) atomicOr(a.status, kStatusBadRequestBit);
    int who = threadIdx.x;
    asm volatile("" : "+v"(who));                        // (addresses made from it are not kept in registers around the loop)
    paged_join_waves<T, C, D, ROWS, WAVES>(lds.part, lds.tops, lds.sums, top, sum, acc, columns, who, emit);
}

// Tokens begin .. end - 1 of a sequence by one wave, for up to 16 query heads, which begin at `from`.
template <typename T, typename C, int D>
__device__ __forceinline__ void own_part(const SharedArgs& a, const int32_t* table, int kv, int begin, int end, int columns, const char* from, int64_t to)
{
    typedef PagedTile<T, C, D, 1> S;
    constexpr int kKeys = S::kKeys, kSteps = S::kSteps, kChannels = S::kChannels;
    const int lane = threadIdx.x & 63, col = lane & 15, j = lane >> 4;
    Vec16 q[1][kSteps];
    const char* const at = from + (col < columns ? col : 0) * (D * Elem<T>::kBytes);
#pragma unroll
    for (int c = 0; c < kSteps; ++c) q[0][c] = load16(at + S::query_at(c, j));
    float top[1] = {-INFINITY}, sum[1] = {0.f};
    f32x4_t acc[1][kChannels];
#pragma unroll
    for (int e = 0; e < kChannels; ++e) acc[0][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
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
    int next = begin, page = table[page_of(next)];
    while (next < end) {
        const int rows = row_of(next, page);
        next += kKeys;
        if (next < end) page = table[page_of(next)];
        if (a.sixteens && !__any(rows < 0)) paged_take<T, C, D, 1, true>(a.pool, rows, q, top, sum, acc);
        else paged_take<T, C, D, 1, false>(a.pool, rows, q, top, sum, acc);
    }
    if (bad) atomicOr(a.status, kStatusBadRequestBit);
    sum[0] += __shfl_xor(sum[0], 16, 64);
    sum[0] += __shfl_xor(sum[0], 32, 64);
    if (col < columns) {
        float* const out = a.part_out + (to + col) * D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < kChannels; e += 4)
                *reinterpret_cast<f32x4_t*>(out + (S::kWide ? (e / 4) * 64 + (4 * j + i) * 4 : (4 * j + i) * kChannels + e)) = f32x4_t{acc[0][e][i], acc[0][e + 1][i], acc[0][e + 2][i], acc[0][e + 3][i]};
        if (j == 0) *reinterpret_cast<float2*>(a.part_sum + (to + col) * 2) = float2{top[0] - S::kRaise, sum[0]};
    }
}

// What every workgroup sums up by itself, in LDS.
struct SharedLists {
    int *before, *own;                                   // [b + 1]: steps of a key head before prefix p, and before sequence s
    uint16_t *members, *prefix;                          // [b + 1]: sequences of the prefixes before; [b]: a sequence's own prefix
    int* scratch;                                        // three for each wave
    __device__ __forceinline__ SharedLists(int* lds, int b, int* scratch_) : before(lds), own(lds + b + 1), members(reinterpret_cast<uint16_t*>(own + b + 1)), prefix(members + b + 1), scratch(scratch_) {}
};
constexpr size_t shared_lists_bytes(int64_t b) { return (sizeof(int) * (2 * b + 2) + sizeof(uint16_t) * (2 * b + 1) + 15) / 16 * 16; }

// The unit of step x: its entry in a list of steps before entries (0 .. b), of which each has h_kv times as many.
__device__ __forceinline__ int entry_of(const int* before, int b, int h_kv, int x)
{
    int e = 0;
    for (int above = b; e + 1 < above;) {
        const int mid = (e + above) >> 1;
        if (before[mid] * h_kv <= x) e = mid; else above = mid;
    }
    return __builtin_amdgcn_readfirstlane(e);
}

// The lists, what the join asks of this call, and then this workgroup's shares: prefixes' units of TILE columns by prefix_part, and sequences.
template <typename T, typename C, int D, int TILE, int WAVES, typename P>
__device__ __forceinline__ void shared_share(const SharedArgs& a, const SharedLists& lists, int (&member_row)[TILE + 1], P prefix_part)
{
    constexpr int NT = 64 * WAVES;
    int *const before = lists.before, *const own = lists.own;
    uint16_t *const members = lists.members, *const prefix = lists.prefix;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = a.b;
    const int own_tiles = (a.group + kOwnColumns - 1) / kOwnColumns;

    for (int i = tid; i <= b; i += NT) before[i] = 0;
    if (tid == 0) own[0] = 0;
    __syncthreads();
    int bits = 0;
    for (int s = tid; s < b; s += NT) {
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
            if (is != kLeftOut) steps = own_steps_of(n, a.own_log) * own_tiles;
            if (is != kLeftOut && is != kNoPrefix) atomicAdd(&before[1 + of], 1);
        }
        if (too_long) bits |= kStatusCapacityBit;
        prefix[s] = (uint16_t)is;
        own[1 + s] = steps;
    }
    if (bits && blockIdx.x == 0) atomicOr(a.status, bits);
    __syncthreads();
    // running sums, over `per` entries that follow each other a thread
    const int per = (b + NT - 1) / NT, s0 = tid * per, s1 = s0 + per < b ? s0 + per : b;
    int sums[3] = {0, 0, 0};                             // sequences behind prefixes, those's steps, own steps
    for (int p = s0; p < s1; ++p) {
        const int m = before[1 + p];
        sums[0] += m;
        sums[1] += m ? steps_of(a.rows.cache_len[p]) * ((m * a.group + TILE - 1) / TILE) : 0;
        sums[2] += own[1 + p];
        members[p + 1] = (uint16_t)sums[0];
        before[1 + p] = sums[1];
        own[1 + p] = sums[2];
    }
    const int here[3] = {sums[0], sums[1], sums[2]};
    sums_to(sums, lists.scratch);
    for (int p = s0; p < s1; ++p) {
        members[p + 1] = (uint16_t)(members[p + 1] + sums[0] - here[0]);
        before[1 + p] += sums[1] - here[1];
        own[1 + p] += sums[2] - here[2];
    }
    if (tid == 0) members[0] = 0;
    __syncthreads();
    const int total = __builtin_amdgcn_readfirstlane(before[b]) * a.h_kv, own_total = __builtin_amdgcn_readfirstlane(own[b]) * a.h_kv;
    const PagedShares shares(total, a.shares), own_shares(own_total, a.shares * WAVES);
    // what the join asks of this call: a wave has a sequence
    for (int s = blockIdx.x * WAVES + wave; s < b; s += gridDim.x * WAVES) {
        const int is = prefix[s];
        int rank = 0;
        if (is != kNoPrefix && is != kLeftOut)
            for (int i = lane; i < s; i += 64) rank += prefix[i] == is;
#pragma unroll
        for (int o = 32; o; o >>= 1) rank += __shfl_xor(rank, o, 64);
        if (lane == 0) {
            SharedPlace to{-1, rank, 0, 0, 0, 0, own[s], (own[s + 1] - own[s]) / own_tiles};
            if (is != kLeftOut) to.row = a.rows.row_start ? a.rows.row_start[s + 1] - 1 : s;
            if (is != kNoPrefix && is != kLeftOut) {
                to.members = members[is] - members[is - 1];
                to.first = members[is - 1];
                to.prefix_at = before[is - 1];
                to.prefix_steps = (before[is] - before[is - 1]) / ((to.members * a.group + TILE - 1) / TILE);
            }
            a.place[s] = to;
        }
    }
    if (blockIdx.x == 0 && tid == 0) *reinterpret_cast<int2*>(a.place + b) = int2{total, own_total};

    auto row_of = [&](int s) { return a.rows.row_start ? a.rows.row_start[s + 1] - 1 : s; };
    auto prefixes = [&]() __attribute__((always_inline)) {
        // (Shares that follow each other run on the same XCD, so that tiles of one prefix meet in its L2; where there is less than a step for each, all XCDs get some.)
        const int share = total < a.shares ? blockIdx.x : (blockIdx.x & 7) * (a.shares >> 3) + (blockIdx.x >> 3), x1 = shares.begin(share + 1);
        int x = shares.begin(share), e = x < x1 ? entry_of(before, b, a.h_kv, x) : 0;
        while (x < x1) {
            const int e_before = __builtin_amdgcn_readfirstlane(before[e]), of_head = __builtin_amdgcn_readfirstlane(before[e + 1]) - e_before;
            if (of_head == 0) {
                ++e;
                continue;
            }
            const int at_member = __builtin_amdgcn_readfirstlane((int)members[e]), columns = (__builtin_amdgcn_readfirstlane((int)members[e + 1]) - at_member) * a.group,
                      tiles = (columns + TILE - 1) / TILE, steps = of_head / tiles;
            const int in_e = x - e_before * a.h_kv, unit = in_e / steps, kv = unit / tiles, tile = unit - kv * tiles, first = in_e - unit * steps;
            const int last = steps - first < x1 - x ? steps : first + (x1 - x), n = __builtin_amdgcn_readfirstlane(a.rows.cache_len[e]);
            const int begin = first * kPagedStep, end = last == steps ? n : last * kPagedStep, here = columns - tile * TILE < TILE ? columns - tile * TILE : TILE;
            const int64_t to = (int64_t)a.group * a.h_kv * at_member + (int64_t)kv * columns + tile * TILE + (int64_t)share * TILE;
            // rows of the sequences whose heads are columns of this tile
            const int rank0 = tile * TILE / a.group, rank1 = (tile * TILE + here + a.group - 1) / a.group;
            int mine = 0, row = 0;
            for (int i = s0; i < s1; ++i)
                if (prefix[i] == e + 1) {
                    if (mine++ == 0) row = row_of(i);
                }
            int rank = sum_to(mine, lists.scratch) - mine;
            for (int i = s0, k = 0; i < s1; ++i)
                if (prefix[i] == e + 1) {
                    if (rank >= rank0 && rank < rank1) member_row[rank - rank0] = k == 0 ? row : row_of(i);
                    ++rank;
                    ++k;
                }
            __syncthreads();
            prefix_part(a.block_table + (int64_t)e * a.max_pages, kv, begin, end, here, [&](int i) __attribute__((always_inline)) {
                const int at = tile * TILE + i, rank = at / a.group;
                return a.q + member_row[rank - rank0] * a.q_stride + ((int64_t)kv * a.group + at - rank * a.group) * (D * Elem<T>::kBytes);
            }, to);
            x += last - first;
            if (x == (e_before + of_head) * a.h_kv) ++e;
        }
    };
    auto sequences = [&]() __attribute__((always_inline)) {
        // (the first shares of either kind are the ones with a step more: they are not the same workgroup's)
        const int share = __builtin_amdgcn_readfirstlane((a.shares - 1 - (int)blockIdx.x) * WAVES + wave), x1 = own_shares.begin(share + 1);
        int x = own_shares.begin(share), s = x < x1 ? entry_of(own, b, a.h_kv, x) : 0;
        while (x < x1) {
            const int s_before = __builtin_amdgcn_readfirstlane(own[s]), of_head = __builtin_amdgcn_readfirstlane(own[s + 1]) - s_before;
            if (of_head == 0) {
                ++s;
                continue;
            }
            const int steps = of_head / own_tiles, in_s = x - s_before * a.h_kv, unit = in_s / steps, kv = unit / own_tiles, tile = unit - kv * own_tiles, first = in_s - unit * steps;
            const int last = steps - first < x1 - x ? steps : first + (x1 - x);
            if (last > 1) {                              // (a unit's first step has no tokens)
                const int row = row_of(s), n = __builtin_amdgcn_readfirstlane(a.rows.cache_len[s]);
                const int begin = first ? (first - 1) << a.own_log : 0, end = last == steps ? n : (last - 1) << a.own_log,
                          here = a.group - tile * kOwnColumns < kOwnColumns ? a.group - tile * kOwnColumns : kOwnColumns;
                own_part<T, C, D>(a, a.block_table + (int64_t)s * a.max_pages, kv, begin, end, here,
                                  a.q + row * a.q_stride + ((int64_t)kv * a.group + tile * kOwnColumns) * (D * Elem<T>::kBytes),
                                  a.own_columns + (int64_t)a.group * a.h_kv * s + (int64_t)kv * a.group + tile * kOwnColumns + (int64_t)share * kOwnColumns);
            }
            x += last - first;
            if (x == (s_before + of_head) * a.h_kv) ++s;
        }
    };
    sequences();
    prefixes();
}

// 16 ROWS columns to a prefix's unit: all types, pages of any size.  STREAM: prefixes have one unit a key head; else their tiles' loads stay in the caches for the next one (us, 128
// sequences of 16 to 300 tokens behind 8192, 32 query and 8 key heads of 128 channels: 8-bit codes 76.1 / 65.9, bf16 in pages of 20 104 / 79; 64 in fp32 121 / 111).
template <typename T, typename C, int D, int ROWS, bool STREAM>
__global__ void __launch_bounds__(256, Elem<C>::kBytes * D == 512 && ROWS == 2 ? 1 : 2) swa_paged_shared_kernel(SharedArgs a)
{
    __shared__ SharedLds<D, 4> lds;
    __shared__ int scratch[12], member_row[16 * ROWS + 1];
    extern __shared__ int lists[];
    shared_share<T, C, D, 16 * ROWS, 4>(a, SharedLists(lists, a.b, scratch), member_row,
                                        [&](const int32_t* table, int kv, int begin, int end, int columns, auto from, int64_t to) __attribute__((always_inline)) {
                                            shared_part<T, C, D, ROWS, 4, STREAM>(a, table, kv, begin, end, columns, lds, from, SharedEmit<D>{a.part_out, a.part_sum, to});
                                        });
}

// ---- prefixes of many columns, 16 bit -------------------------------------------------------------------------------------------------------
//
// Bound by the matrix cores and the softmax's exponentials next to them.  Eight waves: four groups of 32 columns, and two halves of a unit's tokens, every other 32 of
// them, whose results meet in LDS at its end (two workgroups of four waves would leave twice as many partial results).  As in swa_flash.hip a lane owns one column throughout: S^T = K Q^T
// leaves lane l the logits of 16 keys for column l % 32, O^T = V^T P^T takes its weights as they lie; key and value tiles go from L2 straight to LDS, three buffers of them,
// two tiles ahead, rows permuted by chunks instead of padded.  A wave stages eight tokens that follow each other, which lie in one page where page_size is a
// multiple of eight: their place is a scalar.
//
// 64 sequences behind 32768 fp16 tokens, 64 query and 8 key heads: 137 us in all, without own tokens 127 (0.9 PFLOP/s with the products of the weights' second numbers; the matrix
// cores are busy for a third of the clocks, the vector units for more than that).  Measured with weights of one number (101 us) and no faster: the halves in turns, one forming
// products while the other forms weights (102); more tiles' fragments ahead; three parts of the tokens.
//
// Weights go to the second product as two numbers, as in the other forms, so that what a sequence gets does not hang on how many others its cache has room for: rounded once
// they left outputs 1.3 to 1.4 times as far from 64 bits.  That is half as many products again.  Both are rounded to the nearest (split8), so an infinite value's product is
// none; a unit with such a result is done again by the other form of the work.  (us, one number / two: the above 103 / 137, 64 sequences behind 8192 bf16 tokens, 32 query heads
// 38 / 41, 128 behind three of 2049 to 8191 with up to 1500 of their own 103 / 107.)

// The 16 weights of one lane's column, exp2(c scale - m), their sum, and the rescaling that goes with them: formed with the reference m as it is, and again where that turns out
// too low: in bf16 by a sum above 2^15 (or not finite, as on the first tile); in fp16, where the loudest weight is 2^15, by one that is no fp16 number.
template <typename T, int CT>
__device__ __forceinline__ float column_weights(const float16_t& c, float scale, float& m, float& l, float16_t (&o)[CT], float (&p)[16])
{
    constexpr bool kHalf = std::is_same_v<T, F16>;
    constexpr float kRaise = kHalf ? 15.f : 0.f;
    float sum;
    auto weights = [&]() __attribute__((always_inline)) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(c[i], scale, -m));
            sum += p[i];
        }
    };
    weights();
    float loudest = sum;
    if constexpr (kHalf) {
        loudest = p[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) loudest = fmaxf(loudest, p[i]);
    }
    if (__any(loudest > (kHalf ? 65504.f : 32768.f))) {
        float most = c[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, c[i]);
        float lo, hi;
        both_halves(most, lo, hi);
        most = fmaxf(lo, hi) * scale - kRaise;
        const float to = most > m ? most : m, down = __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= down;
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] *= down;
        weights();
    }
    return sum;
}

constexpr int kWideColumns = 128;

template <int D>
constexpr int wide_tile_bytes() { return 32 * D * 2; }
template <int D>
constexpr int wide_lds_bytes() { return 12 * wide_tile_bytes<D>() > kWideColumns * (D + 6) * 4 ? 12 * wide_tile_bytes<D>() : kWideColumns * (D + 6) * 4; }

// Tokens begin .. end - 1 (begin a multiple of 32) for up to 128 columns.  False, and nothing is written: a page lies outside the pool (the first one stood in for it), or a result
// is not finite.
template <typename T, int D, typename Q>
__device__ __forceinline__ bool wide_part(const SharedArgs& a, const int32_t* table, int kv, int begin, int end, int columns, char* lds, Q from, int64_t to)
{
    constexpr int kRow = D * 2, kTile = wide_tile_bytes<D>(), NV = kRow / 32, CT = D / 32, kChunks = kRow / 16, kRowsPerLoad = 64 / kChunks, LD = 8 / kRowsPerLoad, PF = 2;
    static_assert(2 * LD == NV / 2, "one load behind every second product of the first contraction");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), group = wave & 3, half = wave >> 2, l32 = lane & 31, hb = lane >> 5;
    char* const buf = lds + half * (6 * kTile);
    char *const k0 = buf, *const v0 = buf + kTile, *const k1 = buf + 2 * kTile, *const v1 = buf + 3 * kTile, *const k2 = buf + 4 * kTile, *const v2 = buf + 5 * kTile;
    const int rounds = (end - begin + 63) >> 6;
    auto base_of = [&](int round) { return begin + round * 64 + half * 32; };

    // The eight tokens that this wave stages of a round's tile (the last eight where there are none), and their page: lane i has that of round 64 k + i.
    const int last8 = (end - 1) & ~7;
    auto token_of = [&](int round) {
        const int t = base_of(round) + group * 8;
        return t < last8 ? t : last8;
    };
    auto page_of = [&](int t) { return (int)(((uint64_t)(uint32_t)t * a.page_mul) >> a.page_shift); };
    auto swzK = [](int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); };
    auto swzV = [](int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); };
    uint32_t offK[LD], offV[LD];
    auto offsets = [&](int last) {                       // rows past `last` of the eight read that one
        int ln = lane;
        asm volatile("" : "+v"(ln));                     // (computed where it is needed, not kept in registers around the loop)
#pragma unroll
        for (int x = 0; x < LD; ++x) {
            const int j = x * kRowsPerLoad + ln / kChunks, r = j < last ? j : last, at = group * 8 + j;
            offK[x] = (uint32_t)(r * kRow + (((ln % kChunks) ^ swzK(at)) << 4));
            offV[x] = (uint32_t)(r * kRow + (((ln % kChunks) ^ swzV(at)) << 4));
        }
    };
    int pages = 0;
    bool bad = false;
    int64_t at_row = 0;                                  // bytes before the eight rows in the pool
    auto aim = [&](int round) __attribute__((always_inline)) {
        if ((round & 63) == 0) {
            pages = table[page_of(token_of(round + lane))];
            const bool in_pool = (uint32_t)pages < (uint32_t)a.n_pages;
            bad |= !in_pool;
            pages = in_pool ? pages : 0;
        }
        const int t = token_of(round), page = __builtin_amdgcn_readlane(pages, round & 63);
        at_row = ((int64_t)(page * a.h_kv + kv) * a.page_size + (t - page_of(t) * a.page_size)) * kRow;
        if (base_of(round) + 32 > end) offsets(end - 1 - t);
    };
    auto load = [&](int x, char* dk, char* dv) {
        if (x < LD) load_to_lds(a.pool.k_pages + at_row, offK[x], lds_address(dk) + (group * LD + x) * 1024);
        else load_to_lds(a.pool.v_pages + at_row, offV[x - LD], lds_address(dv) + (group * LD + x - LD) * 1024);
    };
    offsets(8);
    __syncthreads();                                     // (what was in LDS before has been read)
    aim(0);
#pragma unroll
    for (int x = 0; x < 2 * LD; ++x) load(x, k0, v0);
    Vec16 q[NV];
    const int column = group * 32 + l32;
    const char* const row = from(column < columns ? column : 0);
#pragma unroll
    for (int v = 0; v < NV; ++v) q[v] = load16(row + v * 32 + hb * 16);
    // Fragment addresses, as in swa_flash.hip: key fragment v is row l32, chunk 2 v + hb; value fragment (ct, v) keys 16 v + 4 hb + 0..3 and 16 v + 8 + 4 hb + 0..3 of channel
    // 32 ct + l32.
    const uint32_t ka = (uint32_t)(l32 * kRow + ((hb ^ swzK(l32)) << 4));
    const int j16 = lane & 15;
    const uint32_t va = (uint32_t)((4 * hb + (j16 >> 2)) * kRow + (((2 * ((lane >> 4) & 1) + ((j16 & 3) >> 1)) ^ swzV(j16 >> 2)) << 4) + (j16 & 1) * 8);
    // (the queries are waited for here, where the compiler sees it, and not with the tiles requested since in every round)
    __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0)
    if (rounds > 1) {
        aim(1);
#pragma unroll
        for (int x = 0; x < 2 * LD; ++x) load(x, k1, v1);
    }

    float16_t o[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -3.0e38f, l = 0.f;                         // (finite, so that logits of -inf weigh nothing before the first finite one too)
    const bool mine = group * 32 < columns;

    // tail: the round's tile may end inside; more: the tile two rounds on is requested
    auto compute = [&](bool tail, bool more, int round, const char* sk, const char* sv, char* nk, char* nv) __attribute__((always_inline)) {
        if (more) aim(round + 2);
        if (!mine) {
            if (more)
#pragma unroll
                for (int x = 0; x < 2 * LD; ++x) load(x, nk, nv);
            return;
        }
        float16_t c;
#pragma unroll
        for (int i = 0; i < 16; ++i) c[i] = 0.f;
        auto kfrag = [&](int v) { return load16(sk + (ka ^ (v << 5))); };
        Vec16 kf[NV];
#pragma unroll
        for (int v = 0; v < PF && v < NV; ++v) kf[v] = kfrag(v);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (v + PF < NV) kf[v + PF] = kfrag(v + PF);
            __builtin_amdgcn_sched_barrier(0);
            c = Mfma<T>::run(kf[v], q[v], c);
            __builtin_amdgcn_sched_barrier(0);
            if ((v & 1) && more) load(v >> 1, nk, nv);
        }
        if (tail) {
            const int left = end - base_of(round);
#pragma unroll
            for (int i = 0; i < 16; ++i) c[i] = 8 * (i / 4) + 4 * hb + (i % 4) < left ? c[i] : -INFINITY;
        }
        float p[16];
        const float sum = column_weights<T>(c, a.pool.scale, m, l, o, p);
        l += sum;
        Vec16 pv[2], rest[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) split8<T, true>(p + 8 * i, pv[i], rest[i]);
        auto vfrag = [&](int f) {
            const char* const at = sv + ((va ^ (f % CT << 6)) + f / CT * 16 * kRow);
            return lds_read_tr(at, at + 8 * kRow);
        };
        Vec16 vf[2 * CT];
#pragma unroll
        for (int f = 0; f < PF && f < 2 * CT; ++f) vf[f] = vfrag(f);
#pragma unroll
        for (int f = 0; f < 2 * CT; ++f) {
            if (f + PF < 2 * CT) vf[f + PF] = vfrag(f + PF);
            __builtin_amdgcn_sched_barrier(0);
            o[f % CT] = Mfma<T>::run(vf[f], pv[f / CT], o[f % CT]);
            o[f % CT] = Mfma<T>::run(vf[f], rest[f / CT], o[f % CT]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // A round's tiles are read while the next two are on their way; loads return in order, so "all but the newest tile's" is a count.
    auto ready = [&](bool newer) {
        if (newer) __builtin_amdgcn_s_waitcnt(0x0070 | (2 * LD));      // vmcnt(2 LD) lgkmcnt(0)
        else __builtin_amdgcn_s_waitcnt(0x0070);                       // vmcnt(0) lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    int round = 0;
    for (; round + 4 < rounds; round += 3) {
        ready(true);
        compute(false, true, round, k0, v0, k2, v2);
        ready(true);
        compute(false, true, round + 1, k1, v1, k0, v0);
        ready(true);
        compute(false, true, round + 2, k2, v2, k1, v1);
    }
    // one to four are left, of which the very last may end inside its tiles: the values behind its tokens are zeros then (a weight of 0 times what is no number is none)
    for (int i = 0; round < rounds; ++round, i = i == 2 ? 0 : i + 1) {
        char *const sk = i == 0 ? k0 : i == 1 ? k1 : k2, *const sv = i == 0 ? v0 : i == 1 ? v1 : v2, *const nk = i == 0 ? k2 : i == 1 ? k0 : k1,
                    *const nv = i == 0 ? v2 : i == 1 ? v0 : v1;
        ready(round + 1 < rounds);
        if (round + 1 == rounds && begin + rounds * 64 > end) {
            const int left = end - base_of(round) < 0 ? 0 : end - base_of(round);
            for (int x = (tid & 255) * 16 + left * kRow; x < kTile; x += 4096) store16(sv + x, Vec16{0u, 0u, 0u, 0u});
            __syncthreads();
        }
        compute(true, round + 2 < rounds, round, sk, sv, nk, nv);
    }
    float lo, hi;
    both_halves(l, lo, hi);
    l = lo + hi;
    float none = 0.f;
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) none = __builtin_fmaf(o[t][i], 0.f, none);
    if (__syncthreads_or(bad || none != none)) return false;

    // The second half's results to the first's, and from there to memory, whole rows at a time.
    constexpr int kPitch = D + 4;
    float* const result = reinterpret_cast<float*>(lds);
    float* const stats = result + kWideColumns * kPitch;
    if (half == 1 && mine) {
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4_t*>(result + column * kPitch + 32 * t + 8 * g + 4 * hb) = f32x4_t{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]};
        if (hb == 0) *reinterpret_cast<float2*>(stats + 2 * column) = float2{m, l};
    }
    __syncthreads();
    if (half == 0 && mine) {
        const float2 other = *reinterpret_cast<const float2*>(stats + 2 * column);
        const float top = fmaxf(m, other.x), here = __builtin_amdgcn_exp2f(m - top), there = __builtin_amdgcn_exp2f(other.x - top);
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4_t* const at = reinterpret_cast<f32x4_t*>(result + column * kPitch + 32 * t + 8 * g + 4 * hb);
                *at = f32x4_t{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]} * here + *at * there;
            }
        if (hb == 0 && column < columns) *reinterpret_cast<float2*>(a.part_sum + (to + column) * 2) = float2{top, l * here + other.y * there};
    }
    __syncthreads();
    for (int i = tid; i < columns * (D / 4); i += 512) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        *reinterpret_cast<f32x4_t*>(a.part_out + (to + r) * D + c) = *reinterpret_cast<const f32x4_t*>(result + r * kPitch + c);
    }
    return true;
}

template <typename T, int D>
__global__ void __launch_bounds__(512, 2) swa_paged_shared_wide_kernel(SharedArgs a)
{
    extern __shared__ __align__(16) char lds[];          // tiles, then the lists
    __shared__ int scratch[24], member_row[kWideColumns + 1];
    SharedLds<D, 8>& sums = *reinterpret_cast<SharedLds<D, 8>*>(lds);
    static_assert(sizeof(SharedLds<D, 8>) <= wide_lds_bytes<D>(), "in the tiles' place");
    shared_share<T, T, D, kWideColumns, 8>(
        a, SharedLists(reinterpret_cast<int*>(lds + wide_lds_bytes<D>()), a.b, scratch), member_row,
        [&](const int32_t* table, int kv, int begin, int end, int columns, auto from, int64_t to) __attribute__((always_inline)) {
            if (wide_part<T, D>(a, table, kv, begin, end, columns, lds, from, to)) return;
            // (the other form of the work leaves what a page outside the pool would hold out of the sums, and keeps infinite values)
            for (int c = 0; c < columns; c += 16)
                shared_part<T, T, D, 1, 8, false>(a, table, kv, begin, end, columns - c < 16 ? columns - c : 16, sums, [&](int i) __attribute__((always_inline)) { return from(c + i); },
                                           SharedEmit<D>{a.part_out, a.part_sum, to + c});
        });
}

// A query head's partial results, the prefix's and its own, to its output.
template <typename T, int D, int WAVES>
__global__ void __launch_bounds__(256) swa_paged_join_shared_kernel(SharedArgs a, int tile, int waves)
{
    const int of = __builtin_amdgcn_readfirstlane(blockIdx.x * (4 / WAVES) + (WAVES == 1 ? threadIdx.x >> 6 : 0));
    if (of >= a.b * a.h_q) return;
    const int s = of / a.h_q, hq = of - s * a.h_q, kv = hq / a.group, head = hq - kv * a.group;
    const SharedPlace at = a.place[s];
    if (at.row < 0) return;
    const int2 total = *reinterpret_cast<const int2*>(a.place + a.b);
    int64_t first = 0, own_first = 0;
    int count = 0, own_count = 0;
    if (at.prefix_steps > 0) {
        const int columns = at.members * a.group, i = at.rank * a.group + head, tiles = (columns + tile - 1) / tile;
        const int x = at.prefix_at * a.h_kv + (kv * tiles + i / tile) * at.prefix_steps;
        const PagedShares shares(total.x, a.shares);
        const int f = shares.of(x);
        count = shares.of(x + at.prefix_steps - 1) - f + 1;
        first = (int64_t)a.group * a.h_kv * at.first + (int64_t)kv * columns + i + (int64_t)f * tile;
    }
    if (at.steps > 0) {
        const int tiles = (a.group + kOwnColumns - 1) / kOwnColumns, x = at.at * a.h_kv + (kv * tiles + head / kOwnColumns) * at.steps;
        const PagedShares shares(total.y, a.shares * waves);
        const int f = shares.of(x + 1);                  // (of the first step with tokens)
        own_count = shares.of(x + at.steps - 1) - f + 1;
        own_first = a.own_columns + (int64_t)a.group * a.h_kv * s + (int64_t)kv * a.group + head + (int64_t)f * kOwnColumns;
    }
    paged_join_pieces<T, D, WAVES>(a.part_out, a.part_sum, [&](int i) __attribute__((always_inline)) { return i < count ? first + (int64_t)i * tile : own_first + (int64_t)(i - count) * kOwnColumns; },
                            count + own_count, a.out, a.lse, (int64_t)at.row * a.h_q + hq);
}

// A single sequence has no other one for a prefix: its length, where it has none, or that of an unused row.
__global__ void swa_paged_shared_alone_kernel(PagedRows rows, const int32_t* prefix_of, int32_t* len, int32_t* status)
{
    if (threadIdx.x) return;
    int row, n;
    bool too_long = false;
    const bool refused = paged_row(rows, 0, row, n, too_long) && prefix_of[0] != -1;
    if (refused) atomicOr(status, kStatusBadRequestBit);
    *len = refused ? -1 : n;
}

// Columns that a prefix can have.
static int64_t most_columns(const swa_paged_params& p) { return (int64_t)(p.b - 1) * (p.h_q / p.h_kv); }

// Columns of a prefix's unit, in sixteens.  More than 32 go to the wide form where it serves them: us, units of 32 / wide, 32 query and 8 key heads of 128 channels, sequences with 16
// to 300 tokens of their own: 10 behind 4096 23.0 / 24.8, 16 24.6 / 26.0, behind 32768 57.1 / 51.1, 24 behind 16000 44.5 / 42.2, 32 51.3 / 46.0, 64 behind 8192 45.8 / 41.0; 100 behind ten
// of 500 to 2000 43.3 / 46.5; 64 channels, 32 behind 16000 35.6 / 35.6.
static int shared_rows(const swa_paged_params& p)
{
    const int64_t most = most_columns(p);
    return most <= 16 ? 1 : most <= 32 || p.dtype == SWA_F32 || paged_int8(p) || p.page_size % 8 != 0 ? 2 : kWideColumns / 16;
}

static int shared_shares(int rows) { return rows > 2 ? 256 : 512; }    // a workgroup to a CU, or two
constexpr int kSharedWaves = 2048;                                     // of either

// Partial results of the prefixes, whatever page_size a call states, and of all.
static int64_t prefix_columns(const swa_paged_params& p) { return (int64_t)p.b * p.h_q + (most_columns(p) > 32 ? 256 * kWideColumns : 512 * 32); }
static int64_t shared_columns(const swa_paged_params& p) { return prefix_columns(p) + (int64_t)p.b * p.h_q + kSharedWaves * kOwnColumns; }

size_t paged_shared_bytes(const swa_paged_params& p)
{
    if (p.b == 1) return 0;
    return (size_t)shared_columns(p) * (p.d + 2) * sizeof(float) + ((size_t)p.b + 1) * sizeof(SharedPlace);
}

template <typename T, typename C, int D>
static int launch_shared_form(const SharedArgs& a, int rows, bool again, hipStream_t stream)
{
    void (*kernel)(SharedArgs) = rows == 1 ? swa_paged_shared_kernel<T, C, D, 1, true> : again ? swa_paged_shared_kernel<T, C, D, 2, false> : swa_paged_shared_kernel<T, C, D, 2, true>;
    size_t lds = shared_lists_bytes(a.b), of_its_own = 36 * 1024;
    int threads = 256;
    if constexpr (std::is_same_v<T, C> && !std::is_same_v<T, F32>) {
        if (rows > 2) {
            kernel = swa_paged_shared_wide_kernel<T, D>;
            lds += wide_lds_bytes<D>();
            of_its_own = 1024;
            threads = 512;
        }
    }
    if (lds + of_its_own > 64 * 1024) {
        const int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), lds > 49 * 1024 ? lds : 49 * 1024);
        if (rc != SWA_OK) return rc;
    }
    launch_kernel(kernel, dim3((unsigned)a.shares), dim3(threads), lds, stream, a);
    const unsigned heads = (unsigned)(a.b * a.h_q);
    if (heads >= 1024) launch_kernel(swa_paged_join_shared_kernel<T, D, 1>, dim3((heads + 3) / 4), dim3(256), 0, stream, a, 16 * rows, threads / 64);
    else launch_kernel(swa_paged_join_shared_kernel<T, D, 4>, dim3(heads), dim3(256), 0, stream, a, 16 * rows, threads / 64);
    return SWA_OK;
}

template <typename T, typename C, int D>
static int prepare_shared_form()
{
    for (void (*kernel)(SharedArgs) : {swa_paged_shared_kernel<T, C, D, 1, true>, swa_paged_shared_kernel<T, C, D, 2, true>, swa_paged_shared_kernel<T, C, D, 2, false>}) {
        const int rc = raise_dynamic_lds(reinterpret_cast<const void*>(kernel));
        if (rc != SWA_OK) return rc;
    }
    if constexpr (std::is_same_v<T, C> && !std::is_same_v<T, F32>) return raise_dynamic_lds(reinterpret_cast<const void*>(swa_paged_shared_wide_kernel<T, D>));
    return SWA_OK;
}

int prepare_paged_shared()
{
    for (int (*form)() : {prepare_shared_form<F32, F32, 64>, prepare_shared_form<F32, F32, 128>, prepare_shared_form<F16, F16, 64>, prepare_shared_form<F16, F16, 128>,
                          prepare_shared_form<F16, Q8, 64>, prepare_shared_form<F16, Q8, 128>, prepare_shared_form<BF16, BF16, 64>, prepare_shared_form<BF16, BF16, 128>,
                          prepare_shared_form<BF16, Q8, 64>, prepare_shared_form<BF16, Q8, 128>}) {
        const int rc = form();
        if (rc != SWA_OK) return rc;
    }
    return SWA_OK;
}

int launch_paged_shared(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                        const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                        const int32_t* cache_len, const int32_t* prefix_of, void* out, float* lse, void* workspace, hipStream_t stream)
{
    if (p.b == 1) {                                      // the decode's, with its limit and its workspace
        if (p.h_kv * (((int64_t)paged_len_max(p) + kPagedStep - 1) / kPagedStep) > 0x7fffffffLL) return SWA_ERR_CAPACITY;
        int32_t* const len = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + kPagedLengthOffset);
        launch_kernel(swa_paged_shared_alone_kernel, dim3(1), dim3(64), 0, stream, PagedRows{row_start, slot, cache_len, n_rows, paged_len_max(p)}, prefix_of, len,
                      paged_status(workspace));
        return launch_paged_decode(p, q, n_rows, row_start, slot, k_pages, v_pages, k_scale, v_scale, block_table, len, out, lse, workspace, stream);
    }
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
    page_divisor(p.page_size, a.page_mul, a.page_shift);
    a.sixteens = p.page_size % 16 == 0;
    const int rows = shared_rows(p);
    const bool again = most_columns(p) > 32;             // a prefix may have several units a key head
    a.shares = shared_shares(rows);
    a.own_columns = prefix_columns(p);
    // (steps are 32-bit numbers: of as many prefixes as may be, and of every sequence's own tokens, whose steps grow until they are)
    const int64_t own_units = (int64_t)p.b * ((a.group + kOwnColumns - 1) / kOwnColumns) * p.h_kv,
                  units = (((int64_t)p.b * a.group + 16 * rows - 1) / (16 * rows) + p.b) * p.h_kv, steps = ((int64_t)a.rows.len_max + kPagedStep - 1) / kPagedStep;
    if (units > 0x7fffffffLL / steps || (uint64_t)p.b * p.h_q * 256 > 0xffffffffULL) return SWA_ERR_CAPACITY;
    for (a.own_log = kOwnLog; own_units > 0x7fffffffLL / own_steps_of(a.rows.len_max, a.own_log); ++a.own_log) {}
#define SWA_SHARED(T, C) (p.d == 64 ? launch_shared_form<T, C, 64>(a, rows, again, stream) : launch_shared_form<T, C, 128>(a, rows, again, stream))
    const int rc = p.dtype == SWA_F32   ? SWA_SHARED(F32, F32)
                   : p.dtype == SWA_F16 ? (paged_int8(p) ? SWA_SHARED(F16, Q8) : SWA_SHARED(F16, F16))
                                        : (paged_int8(p) ? SWA_SHARED(BF16, Q8) : SWA_SHARED(BF16, BF16));
#undef SWA_SHARED
    if (rc != SWA_OK) return rc;
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
