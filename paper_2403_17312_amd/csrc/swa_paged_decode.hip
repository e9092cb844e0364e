// Attention of one new token per sequence over a paged cache.  Bound by HBM: every key and value of the window is read once, 4 flops for
// two elements and query head.
//
// A workgroup serves up to 16 (or 32) of the query heads that share a key head, over a range of one sequence's tokens; its four waves (one where
// sequences are short) take tiles of the range in turn, each with a running maximum and sum of the softmax.  Ranges come in two ways:
//   chunks   few sequences: each one's tokens in equal chunks, as many as fill the CUs evenly, a workgroup for each.
//   shares   many, and long ones: the call's work, in steps of 128 tokens of one sequence and key head, laid end to end and cut into as
//            many equal shares as there are workgroups, whatever the lengths are; each workgroup sums the lengths up by itself.  A share
//            holds whole sequences and at most two pieces.  128 sequences of 512 to 8192 tokens, 8 key heads of 128 bf16 channels: chunks
//            425 us, shares 353 (6.5 TB/s).
// Pieces leave partial results, which a second, small launch joins in their order.
// All products go to the matrix cores, whose 16 columns are the query heads (swa_paged_tile.hpp): also a single head's, since at their peak they are done in a
// fifteenth of the time that HBM takes for 16 bits, a seventh for codes, and in fp32 something more than a third (with 32 columns: twice those parts).
#include "swa_paged_tile.hpp"

namespace swa {

struct PagedArgs {
    const char* q;
    int64_t q_stride;                              // bytes
    const int32_t *row_start, *slot, *block_table, *cache_len;
    const char *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    char* out;
    float* lse;
    float *part_out, *part_sum;                    // [pieces, row_tiles, heads, D] and [.., 2] (maximum, sum); a share's first and last piece,
                                                   // or chunk `split` of sequence and key head
    int4* begun;                                   // [shares]: key head, row, pieces of the sequence that a share begins and does not end (x = 0: none)
    int32_t* status;
    int32_t b, n_rows, h_q, h_kv, page_size, n_pages, max_pages, window, len_max;
    int32_t group, row_tiles, heads, tile_heads;   // query heads of a key head, tiles of them, heads of a tile that there are at most, and that fit
    int32_t ranges;                                // shares, or chunks of a sequence at most
    int32_t span;                                  // tokens of a sequence that the call may see
    int32_t chunk;                                 // tokens of one; 0: the longest sequence says
    uint32_t page_mul;                             // t / page_size = t * page_mul >> page_shift for 0 <= t < 2^31
    int32_t page_shift;
    int32_t sixteens;                              // pages are whole sixteens of tokens
    float scale;                                   // of logits to the base 2
};

constexpr int kPagedWaves = 4;
constexpr int kPagedChunks = 256;                  // chunks of a sequence at most, which bounds what the join of one has to read

// Tokens of a sequence that a call may see, from a multiple of 32 on.
static int64_t paged_span(const swa_paged_params& p)
{
    int64_t n = (int64_t)p.max_pages * p.page_size;
    if (p.len_bound > 0 && p.len_bound < n) n = p.len_bound;
    return p.window > 0 && p.window < n ? (int64_t)p.window + 31 : n;
}

// Shares take about two microseconds longer (the sums, and pieces to join), and level the lengths out.  us, chunks / shares, 128 bf16 channels, lengths even
// over 100..8001 and all 4000, 32 query and 8 key heads: 8 sequences 33.3 / 32.0, 28.6 / 31.4; 16: 58.8 / 53.7, 47.9 / 50.5; 32: 113 / 95, 87 / 90; 64: 217 / 178,
// 174 / 176; 128: 398 / 345, 331 / 338.  Fewer pairs want more tokens; lengths 1..n and all n: 2 of 16000 24.9 / 22.9, 28.5 / 31.6, of 64000 73.9 / 50, 88 / 89;
// 6 of 4000 21.0 / 20.3, 24.1 / 27.3, of 16000 56.6 / 41, 68 / 71; one key head, 32 of 16000 41.5 / 37.5, 49.9 / 57, 16 of 16000 25.5 / 27.4.  One sequence has
// nothing to level.  16 sequences of 32 fp32 heads, 64 channels, a window of 512: 27.2 / 30.5.
static bool paged_in_shares(const swa_paged_params& p)
{
    if (paged_span(p) < 1024) return false;
    const int64_t pairs = (int64_t)p.b * p.h_kv;
    return pairs * row_tiles_of(p) >= 64 || (p.b > 1 && pairs * paged_span(p) * 2 * paged_row_bytes(p) >= (240 << 20));
}

static int64_t paged_units(const swa_paged_params& p) { return (int64_t)p.b * p.h_kv * row_tiles_of(p); }

constexpr bool paged_two(int row_bytes, int rows, int d) { return row_bytes == 512 || (rows == 2 && d == 128); }

// Shares of a call at most: the workgroups that the chip holds at once.  A CU has four of 64 channels in 16 bits, three of 64 in fp32 and of 128 (168
// registers a lane), two of 128 in fp32 and of 128 with 32 heads, which do not fit those (64 sequences of 4352 tokens, 8 key heads, fp32: three with
// spills 381 us, two 356).  768 / 1024 shares of 128 channels: the ragged 128 sequences above 345 / 387 us; 64 of 100..8001 tokens in 8 bits 107 / 123.
static int paged_max_shares(const swa_paged_params& p)
{
    const bool two = paged_two(paged_row_bytes(p), tile_heads_of(p) / 16, p.d);
    const int n = (two ? 512 : p.d == 64 && tile_heads_of(p) == 16 && p.dtype != SWA_F32 ? 1024 : 768) / row_tiles_of(p);
    return n < 1 ? 1 : n;
}

// Chunks of a sequence at most, for k workgroups on every CU.
static int paged_chunks(const swa_paged_params& p, int k)
{
    const int64_t n = 256 * k / paged_units(p);
    return n < 1 ? 1 : n > kPagedChunks ? kPagedChunks : (int)n;
}

// (for either form, whatever length and window a call states)
static int64_t paged_piece_rows(const swa_paged_params& p)
{
    const int group = p.h_q / p.h_kv;
    const int64_t shares = 2 * (int64_t)paged_max_shares(p) * row_tiles_of(p);
    const int64_t chunks = paged_chunks(p, 3) > 1 ? paged_chunks(p, 3) * paged_units(p) : 0;
    const int64_t pieces = (paged_units(p) >= 64 || p.b > 1) && shares > chunks ? shares : chunks;
    return 2 * ((pieces * (group < tile_heads_of(p) ? group : tile_heads_of(p)) + 1) / 2);
}

size_t paged_partial_bytes(const swa_paged_params& p)
{
    return (size_t)paged_piece_rows(p) * (p.d + 2) * sizeof(float) + (size_t)paged_max_shares(p) * sizeof(int4);
}

void paged_partials(const swa_paged_params& p, void* workspace, float*& out, float*& sum)
{
    out = reinterpret_cast<float*>(static_cast<char*>(workspace) + kPagedPartialOffset);
    sum = out + paged_piece_rows(p) * p.d;
}

// What a sequence asks of this call: its row, its tokens lo .. n-1, and steps (0: nothing).
__device__ __forceinline__ int paged_sequence(const PagedArgs& a, int s, int& row, int& lo, int& n, bool& too_long)
{
    n = a.cache_len[s];
    row = s;
    if (a.row_start) {
        row = a.row_start[s + 1] - 1;
        if (row < a.row_start[s]) return 0;
    }
    if (n < 0 || row < 0 || row >= a.n_rows) return 0;
    if (a.slot && a.slot[row] < 0) return 0;             // a row that the plan has not placed, whose query nobody wrote
    if (n > a.len_max) {
        too_long = true;
        return 0;
    }
    lo = a.window && n > a.window ? n - a.window : 0;
    const int tokens = n - (lo & ~31);                   // (tiles begin at multiples of 32)
    return tokens > kPagedStep ? (tokens + kPagedStep - 1) / kPagedStep : 1;
}

// Tokens of a chunk: a sequence has a.ranges chunks at most.  A bound or a table may be far above the lengths, so where its chunks were over 1024 tokens, or
// no bound is stated, the longest sequence says (of 64 at most, a wave's lanes), which takes 0.7 to 1.6 us.  `tokens`: of the sequence that is asked for.
__device__ __forceinline__ int paged_chunk(const PagedArgs& a, int tokens)
{
    if (a.chunk) return a.chunk;
    if (a.b > 1) {
        const int lane = threadIdx.x & 63;
        int row, lo = 0, n = 0;
        bool too_long = false;
        if (lane < a.b && paged_sequence(a, lane, row, lo, n, too_long)) tokens = n - (lo & ~31);
        auto larger = [](int x, int y) { return x > y ? x : y; };
        tokens = larger(tokens, __builtin_amdgcn_update_dpp(0, tokens, 0xB1, 0xf, 0xf, true));    // within rows of 16 lanes
        tokens = larger(tokens, __builtin_amdgcn_update_dpp(0, tokens, 0x4E, 0xf, 0xf, true));
        tokens = larger(tokens, __builtin_amdgcn_update_dpp(0, tokens, 0x141, 0xf, 0xf, true));
        tokens = larger(tokens, __builtin_amdgcn_update_dpp(0, tokens, 0x140, 0xf, 0xf, true));
        tokens = larger(tokens, __shfl_xor(tokens, 16, 64));
        tokens = larger(tokens, __shfl_xor(tokens, 32, 64));
    }
    const int per_step = a.ranges * kPagedStep;
    return __builtin_amdgcn_readfirstlane(tokens > per_step ? (tokens + per_step - 1) / per_step : 1) * kPagedStep;
}

// The shares: the first `more` of them have one step more than the others.
struct Shares {
    int steps, more;
    __device__ __forceinline__ int begin(int g) const { return g * steps + (g < more ? g : more); }
    __device__ __forceinline__ int of(int x) const
    {
        const int longer = more * (steps + 1);
        return x < longer ? x / (steps + 1) : more + (x - longer) / steps;
    }
};

// T: type of queries and outputs, C: of the pages (Q8: codes).
template <typename T, typename C, int D, bool SHARES, int ROWS, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, paged_two(Elem<C>::kBytes * D, ROWS, D) ? 2 : 3) swa_paged_decode_kernel(PagedArgs a)
{
    typedef PagedTile<T, C, D, ROWS> S;
    constexpr int kKeys = S::kKeys, kSteps = S::kSteps, kChannels = S::kChannels;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, j = lane >> 4;

    // Row tiles of one range read the same pages: eight ranges, then the same ones' next row tile, so that they meet in one XCD's L2.  Reads of HBM per
    // launch against the pages: 71 heads on one key head (three tiles), 16 sequences of 1000 to 8000 tokens, 64 channels, 1.02 times; 128 heads (four), 64 of 8000, 128
    // channels, 2.3 times.
    const int eighth = blockIdx.x >> 3, work = (eighth / a.row_tiles) * 8 + (blockIdx.x & 7), tile = eighth % a.row_tiles;
    const int heads = a.group - 16 * ROWS * tile < 16 * ROWS ? a.group - 16 * ROWS * tile : 16 * ROWS;

    constexpr int kPitch = D + 4;
    __shared__ float part[WAVES][16][kPitch];
    __shared__ float tops[WAVES][16], sums[WAVES][16];
    extern __shared__ int before[];                      // shares: steps of a key head before sequence s, for s <= b

    int s = 0, kv = 0, row, lo, n, split = 0, x = 0, x1 = 0;
    bool too_long = false;
    Shares shares{0, 0};
    int4 begun = {0, 0, 0, 0};
    const bool early = !SHARES && a.chunk && !a.window;
    int early_page = 0;
    if constexpr (SHARES) {
        if (work >= a.ranges) return;
        __shared__ int wave_steps[WAVES];
        const int per = (a.b + 64 * WAVES - 1) / (64 * WAVES), s0 = tid * per, s1 = s0 + per < a.b ? s0 + per : a.b;
        int own = 0;
        for (int i = s0; i < s1; ++i) {
            own += paged_sequence(a, i, row, lo, n, too_long);
            before[i + 1] = own;
        }
        if (too_long && blockIdx.x == 0) atomicOr(a.status, kStatusCapacityBit);
        int to = own;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(to, o, 64);
            if (lane >= o) to += up;
        }
        if (lane == 63) wave_steps[wave] = to;
        __syncthreads();
        int add = to - own;
        for (int w = 0; w < wave; ++w) add += wave_steps[w];
        for (int i = s0; i < s1; ++i) before[i + 1] += add;
        if (tid == 0) before[0] = 0;
        __syncthreads();
        const int total = __builtin_amdgcn_readfirstlane(before[a.b]) * a.h_kv;
        shares = Shares{total / a.ranges, total % a.ranges};
        x = shares.begin(work);
        x1 = shares.begin(work + 1);
        for (int above = a.b; s + 1 < above;) {          // the sequence that x lies in
            const int mid = (s + above) >> 1;
            if (before[mid] * a.h_kv <= x) s = mid; else above = mid;
        }
        s = __builtin_amdgcn_readfirstlane(s);
    } else {
        const int units = a.b * a.h_kv;
        split = work / units;
        if (split >= a.ranges) return;
        s = (work - split * units) / a.h_kv;
        kv = work - split * units - s * a.h_kv;
    }

    do {
        int begin, end;
        bool whole;                                          // all of the sequence
        int64_t piece = 0;
        if constexpr (SHARES) {
            if (x >= x1) break;
            const int s_before = __builtin_amdgcn_readfirstlane(before[s]), steps = __builtin_amdgcn_readfirstlane(before[s + 1]) - s_before;
            if (steps == 0) {
                ++s;
                continue;
            }
            const int in_s = x - s_before * a.h_kv;
            kv = in_s / steps;
            const int first = in_s - kv * steps, last = steps - first < x1 - x ? steps : first + (x1 - x);
            whole = first == 0 && last == steps;
            piece = 2 * work + (first == 0);
            paged_sequence(a, s, row, lo, n, too_long);
            begin = (lo & ~31) + first * kPagedStep;
            end = last == steps ? n : (lo & ~31) + last * kPagedStep;
            if (first == 0 && last < steps) begun = int4{1 + kv, row, shares.of(x + steps - 1) - work + 1, 0};
            x += last - first;
        } else {
            // Few sequences: a call is a chain of loads, so those whose place is known are under way before the length is (the page may be any
            // of the sequence's row then, and counts for nothing where the tokens end earlier).
            if (early) {
                const int t = split * a.chunk + wave * kKeys + (lane & (kKeys - 1)), page = (int)(((uint64_t)(uint32_t)t * a.page_mul) >> a.page_shift);
                early_page = a.block_table[(int64_t)s * a.max_pages + (page < a.max_pages ? page : a.max_pages - 1)];
            }
            row = s;
            if (a.row_start) {
                row = a.row_start[s + 1] - 1;
                if (row < 0 || row < a.row_start[s] || row >= a.n_rows) return;
            }
        }

        // Query operands: column col is query head 16 (ROWS tile + g) + col of the group.
        const int64_t head0 = (int64_t)kv * a.group + 16 * ROWS * tile;
        Vec16 q[ROWS][kSteps];
        {
            const char* const from = a.q + row * a.q_stride + (head0 + col) * (D * Elem<T>::kBytes);
#pragma unroll
            for (int g = 0; g < ROWS; ++g)
#pragma unroll
                for (int c = 0; c < kSteps; ++c) {
                    q[g][c] = 16 * g + col < heads ? load16(from + 16 * g * D * Elem<T>::kBytes + S::query_at(c, j)) : Vec16{0u, 0u, 0u, 0u};
                }
        }

        if constexpr (!SHARES) {
            if (!paged_sequence(a, s, row, lo, n, too_long)) {
                if (too_long && split == 0 && tid == 0) atomicOr(a.status, kStatusCapacityBit);
                return;
            }
            const int from = lo & ~31, chunk = paged_chunk(a, n - from);
            begin = from + split * chunk;
            if (split > 0 && begin >= n) return;
            end = n - begin < chunk ? n : begin + chunk;
            whole = n - from <= chunk;
            piece = ((int64_t)s * a.h_kv + kv) * a.ranges + split;
        }

        float top[ROWS], sum[ROWS];                          // of column col, the sum of this lane's keys alone
        f32x4_t acc[ROWS][kChannels];
#pragma unroll
        for (int g = 0; g < ROWS; ++g) {
            top[g] = -INFINITY;
            sum[g] = 0.f;
#pragma unroll
            for (int e = 0; e < kChannels; ++e) acc[g][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        const int32_t* const table = a.block_table + (int64_t)s * a.max_pages;
        bool bad = false;

        // Page that holds this lane's token of the tile at `base`, and the token's place there.
        auto page_of = [&](int base) {
            const int t = base + (lane & (kKeys - 1)), there = t < lo ? lo : (t < n ? t : n - 1);
            return (int)(((uint64_t)(uint32_t)there * a.page_mul) >> a.page_shift);
        };
        auto token_page = [&](int base) { return table[page_of(base)]; };
        auto token_off = [&](int base) { return base + (lane & (kKeys - 1)) - page_of(base) * a.page_size; };
        const PagedPool pool{a.k_pages, a.v_pages, a.k_scale, a.v_scale, a.scale};
        // Whole tiles first; the others, at the ends of the window and where a page is not in the pool, in a loop of their own, whose addresses then
        // take no registers from this one.
        constexpr int kStride = WAVES * kKeys;
        // The pool's rows of a tile's tokens, -1 where there is none.
        auto row_of = [&](int base, int page) {
            const int t = base + (lane & (kKeys - 1));
            const bool live = t >= lo && t < n, in_pool = (uint32_t)page < (uint32_t)a.n_pages;
            bad |= live && !in_pool;
            return live && in_pool ? (page * a.h_kv + kv) * a.page_size + token_off(base) : -1;
        };
        int next = begin + wave * kKeys, page = 0;
        if (next < end) page = early ? early_page : token_page(next);
        int left = next, left_end = end, r = 0;              // tiles that are left: from, up to, and the first one's rows
        if (a.sixteens) {
            left = end;
            left_end = begin;
            while (next < end) {
                const int base = next, this_page = page;
                next += kStride;
                if (next < end) page = token_page(next);
                const int rows = row_of(base, this_page);
                if (!__any(rows < 0)) {
                    paged_take<T, C, D, ROWS, true>(pool, rows, q, top, sum, acc);
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
            paged_take<T, C, D, ROWS, false>(pool, r, q, top, sum, acc);
            do {
                left += kStride;
                if (left >= left_end) break;
                r = row_of(left, token_page(left));
            } while (a.sixteens && !__any(r < 0));
        }
        if (bad) atomicOr(a.status, kStatusBadRequestBit);

        // The waves' results to one, in LDS: rows are query heads.
        int who = tid;
        if (SHARES) asm volatile("" : "+v"(who));            // (addresses made from it are not kept in registers around the loop)
        paged_join_waves<T, C, D, ROWS, WAVES>(part, tops, sums, top, sum, acc, heads, who, [&](int head, float all, float total, const float (&y)[kChannels]) __attribute__((always_inline)) {
            if (whole) {
                const int64_t at = (int64_t)row * a.h_q + head0 + head;
                paged_store<T, D>(a.out, a.lse, at, (who & 15) * kChannels, (who & 15) == 0, all, total, y);
            } else {
                const int64_t at = (piece * a.row_tiles + tile) * a.heads + head;
#pragma unroll
                for (int e = 0; e < kChannels; e += 4)
                    *reinterpret_cast<f32x4_t*>(a.part_out + at * D + (who & 15) * kChannels + e) = f32x4_t{y[e], y[e + 1], y[e + 2], y[e + 3]};
                if ((who & 15) == 0) *reinterpret_cast<float2*>(a.part_sum + at * 2) = float2{all, total};
            }
        });
        if (SHARES && kv == a.h_kv - 1 && x == before[s + 1] * a.h_kv) ++s;
    } while (SHARES);
    if (SHARES && tile == 0 && tid == 0) a.begun[work] = begun;
}

// The chunks of a sequence and query head to its output, in their order.
template <typename T, int D>
__global__ void __launch_bounds__(256) swa_paged_join_chunks_kernel(PagedArgs a)
{
    constexpr int kLanes = D / 4, kTeams = 256 / kLanes;
    const int s = blockIdx.x / a.h_q, hq = blockIdx.x - s * a.h_q, tid = threadIdx.x, team = tid / kLanes, lane = tid % kLanes;
    const int kv = hq / a.group, of = hq - kv * a.group;
    const int64_t stride = a.row_tiles * a.heads, first = ((int64_t)s * a.h_kv + kv) * a.ranges * stride + (of / a.tile_heads) * a.heads + of % a.tile_heads;
    __shared__ float weight[kPagedChunks], waves[4], waves2[4];
    __shared__ f32x4_t part[kTeams][kLanes];
    // (what may turn out not to be a chunk's is loaded all the same, while the length is on its way)
    float2 mine = tid < a.ranges ? *reinterpret_cast<const float2*>(a.part_sum + (first + tid * stride) * 2) : float2{-INFINITY, 0.f};
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    const bool ahead = a.ranges <= 32;                   // (8.4 / 8.6 us with 9 chunks, 51.5 / 49.9 with 128)
    if (ahead && team < a.ranges) y = *reinterpret_cast<const f32x4_t*>(a.part_out + (first + team * stride) * D + lane * 4);
    int row, lo, n;
    bool too_long;
    if (!paged_sequence(a, s, row, lo, n, too_long)) return;
    const int chunk = paged_chunk(a, n - (lo & ~31));
    if (n - (lo & ~31) <= chunk) return;
    const int count = (n - (lo & ~31) + chunk - 1) / chunk;
    mine = tid < count ? mine : float2{-INFINITY, 0.f};
    float top = wave_max(mine.x);
    if ((tid & 63) == 0) waves[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(waves[0], waves[1]), fmaxf(waves[2], waves[3]));
    const float w = __builtin_amdgcn_exp2f(mine.x - (top == -INFINITY ? 0.f : top));
    weight[tid] = w;
    const float sum = wave_sum(w * mine.y);
    if ((tid & 63) == 0) waves2[tid >> 6] = sum;
    __syncthreads();
    const float total = (waves2[0] + waves2[1]) + (waves2[2] + waves2[3]);
    y = ahead && team < count ? y * weight[team] : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = ahead ? team + kTeams : team; i < count; i += kTeams)
        y += *reinterpret_cast<const f32x4_t*>(a.part_out + (first + i * stride) * D + lane * 4) * weight[i];
    part[team][lane] = y;
    __syncthreads();
    if (team) return;
#pragma unroll
    for (int i = 1; i < kTeams; ++i) y += part[i][lane];
    const int64_t to = (int64_t)row * a.h_q + hq;
    const float inverse = 1.f / total;
#pragma unroll
    for (int i = 0; i < 4; ++i) store_elem<T>(a.out + to * (D * Elem<T>::kBytes), lane * 4 + i, total == 0.f ? 0.f : y[i] * inverse);
    if (a.lse && lane == 0) a.lse[to] = (top + __builtin_log2f(total)) * 0.69314718055994530942f;
}

// The pieces of the sequence that a share begins and does not end, likewise; a workgroup has `per` of its query heads, a power of two.
template <typename T, int D>
__global__ void __launch_bounds__(256) swa_paged_join_shares_kernel(PagedArgs a, int per)
{
    constexpr int kLanes = D / 4, kTeams = 256 / kLanes;
    const int blocks = (a.heads + per - 1) / per, share = blockIdx.x / (a.row_tiles * blocks), rest = blockIdx.x - share * a.row_tiles * blocks;
    const int4 unit = a.begun[share];
    if (unit.x == 0) return;
    const int kv = unit.x - 1, row = unit.y, count = unit.z, tile = rest / blocks, tid = threadIdx.x, team = tid / kLanes, lane = tid % kLanes,
              mates = kTeams / per, mate = team % mates, head = (rest - tile * blocks) * per + team / mates;
    const bool there = head < a.heads && a.tile_heads * tile + head < a.group;
    // the share's second piece, and then the first ones of the shares behind it
    auto at = [&](int i) { return ((int64_t)(2 * (share + i) + (i == 0)) * a.row_tiles + tile) * a.heads + head; };
    float top = -INFINITY, total = 0.f;
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    auto join = [&](float most, float part_total, const f32x4_t& part_y) {
        const float to = fmaxf(top, most), from = to == -INFINITY ? 0.f : to;
        const float old = __builtin_amdgcn_exp2f(top - from), w = __builtin_amdgcn_exp2f(most - from);
        y = y * old + part_y * w;
        total = total * old + part_total * w;
        top = to;
    };
    if (there) {
#pragma unroll 4
        for (int i = mate; i < count; i += mates) {
            const float2 m = *reinterpret_cast<const float2*>(a.part_sum + at(i) * 2);
            join(m.x, m.y, *reinterpret_cast<const f32x4_t*>(a.part_out + at(i) * D + lane * 4));
        }
    }
    __shared__ float tops[kTeams], sums[kTeams];
    __shared__ f32x4_t part[kTeams][kLanes];
    part[team][lane] = y;
    if (lane == 0) {
        tops[team] = top;
        sums[team] = total;
    }
    __syncthreads();
    if (mate || !there) return;
    for (int i = 1; i < mates; ++i) join(tops[team + i], sums[team + i], part[team + i][lane]);
    const int64_t to = (int64_t)row * a.h_q + (int64_t)kv * a.group + a.tile_heads * tile + head;
    const float inverse = 1.f / total;
#pragma unroll
    for (int i = 0; i < 4; ++i) store_elem<T>(a.out + to * (D * Elem<T>::kBytes), lane * 4 + i, total == 0.f ? 0.f : y[i] * inverse);
    if (a.lse && lane == 0) a.lse[to] = (top + __builtin_log2f(total)) * 0.69314718055994530942f;
}

template <typename T, typename C, int D>
static int launch_paged_form(const PagedArgs& a, bool in_shares, hipStream_t stream)
{
    const int64_t units = (int64_t)a.b * a.h_kv, works = (in_shares ? a.ranges : units * a.ranges);
    const dim3 grid((unsigned)((works + 7) / 8 * 8 * a.row_tiles));
    // Short sequences have work for one wave, and many of them more workgroups than four waves leave places for: us with four / one, lengths 1..n and all n,
    // bf16, d = 128, 32 key heads: 256 sequences n = 16 39.5 / 17.3, 41 / 20, n = 128 60.5 / 49.2, 91 / 86; 64 n = 32 12.2 / 7.8, 12.8 / 9.4, n = 256 28.1 / 26.8,
    // 45.5 / 44.3, n = 512 48.5 / 49.9, 84 / 84; 32 n = 128 11.9 / 10.7, 14.9 / 14.9, n = 256 17.1 / 18.1, 24.8 / 26.1.
    const int64_t all = units * a.row_tiles;
    const bool one = a.tile_heads == 16,
               single = !in_shares && a.ranges == 1 && (a.span <= 32 || (all >= 1024 && a.span <= 128) || (all >= 2048 && a.span <= 256));
    auto kernel = in_shares ? (one ? swa_paged_decode_kernel<T, C, D, true, 1, 4> : swa_paged_decode_kernel<T, C, D, true, 2, 4>)
                  : single  ? (one ? swa_paged_decode_kernel<T, C, D, false, 1, 1> : swa_paged_decode_kernel<T, C, D, false, 2, 1>)
                            : (one ? swa_paged_decode_kernel<T, C, D, false, 1, 4> : swa_paged_decode_kernel<T, C, D, false, 2, 4>);
    if (grid.x * UINT64_C(64) * (single ? 1 : kPagedWaves) > 0xffffffffULL) return SWA_ERR_CAPACITY;    // (threads of a launch; the join's are fewer)
    launch_kernel(kernel, grid, dim3(single ? 64 : 64 * kPagedWaves), in_shares ? sizeof(int) * ((size_t)a.b + 1) : 0, stream, a);
    if (a.ranges == 1) return SWA_OK;
    if (!in_shares) {
        launch_kernel(swa_paged_join_chunks_kernel<T, D>, dim3((unsigned)((int64_t)a.b * a.h_q)), dim3(256), 0, stream, a);
        return SWA_OK;
    }
    int per = 1;                                         // (where a sequence has few pieces, a workgroup joins several heads)
    while (per < 1024 / D && per < a.heads && a.ranges < 4 * units * per) per *= 2;
    launch_kernel(swa_paged_join_shares_kernel<T, D>, dim3((unsigned)((int64_t)a.ranges * a.row_tiles * ((a.heads + per - 1) / per))), dim3(256), 0,
                  stream, a, per);
    return SWA_OK;
}

// Steps of a chunk, where a sequence has so many.
// Work is even, so a call takes as long as the CU that has most of it.  us, as many chunks as make 1024 workgroups, 512, and by this rule (two
// on a CU before three before one): 131071 tokens, 4 key heads, 16 query heads each 54.5 / 50.4 / 50.4; 6 sequences of 32000, 8 key heads 126.8 /
// 155 (some CUs three) / 126.4; 2 of 10000, fp32 37.9 / 36.3 / 32.3.
// And the join, whose launch is worth about a step (2 us), and another one with a thousand query heads to join: us, by these chunks without that / one
// chunk, fp16, d = 128: 1 sequence, 8 key heads, 256 tokens 7.4 / 6.2, 384 7.5 / 7.8, 1000 8.3 / 20.2; 183 sequences of 16 query heads on one, 256 13.7 /
// 8.2, 1000 23.1 / 20.1; 48 of 64 on 8, 512 21.8 / 17.9, 1000 32.5 / 30.9.
int64_t paged_chunk_steps(const swa_paged_params& p, int64_t of_one)
{
    int64_t each = of_one, least = (paged_units(p) + 255) / 256 * of_one * 1024;     // steps of a chunk; of the CU that has most, in 1024ths
    for (int k : {2, 3, 1}) {
        const int64_t e = (of_one + paged_chunks(p, k) - 1) / paged_chunks(p, k), groups = paged_units(p) * ((of_one + e - 1) / e);
        const int64_t most = (groups + 255) / 256 * e * 1024 + 1024 + (int64_t)p.b * p.h_q;
        if (e < of_one && most < least) {
            least = most;
            each = e;
        }
    }
    return each;
}

int launch_paged_decode(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                        const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                        const int32_t* cache_len, void* out, float* lse, void* workspace, hipStream_t stream)
{
    PagedArgs a{};
    a.q = static_cast<const char*>(q.data);
    a.q_stride = q.stride * (p.dtype == SWA_F32 ? 4 : 2);
    a.row_start = row_start;
    a.slot = slot;
    a.block_table = block_table;
    a.cache_len = cache_len;
    a.k_pages = static_cast<const char*>(k_pages);
    a.v_pages = static_cast<const char*>(v_pages);
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.out = static_cast<char*>(out);
    a.lse = lse;
    a.status = paged_status(workspace);
    a.b = p.b;
    a.n_rows = n_rows;
    a.h_q = p.h_q;
    a.h_kv = p.h_kv;
    a.page_size = p.page_size;
    a.n_pages = p.n_pages;
    a.max_pages = p.max_pages;
    a.window = p.window;
    a.len_max = paged_len_max(p);
    a.group = p.h_q / p.h_kv;
    a.tile_heads = tile_heads_of(p);
    a.row_tiles = row_tiles_of(p);
    page_divisor(p.page_size, a.page_mul, a.page_shift);
    a.sixteens = p.page_size % 16 == 0;
    a.scale = (p.scale > 0.f ? p.scale : 1.f / sqrtf((float)p.d)) * 1.44269504088896340736f;

    const int64_t units = (int64_t)p.b * p.h_kv;
    const int64_t span = paged_span(p);
    a.span = (int32_t)span;
    const int64_t steps = units * ((span + kPagedStep - 1) / kPagedStep);
    if (steps > 0x7fffffffLL) return SWA_ERR_CAPACITY;
    a.heads = a.group < a.tile_heads ? a.group : a.tile_heads;
    const bool in_shares = paged_in_shares(p);
    if (in_shares) {
        a.ranges = paged_max_shares(p);
    } else {
        const int64_t of_one = steps / units, each = paged_chunk_steps(p, of_one);
        a.chunk = (p.len_bound > 0 && each <= 8) || p.b > 64 ? (int32_t)(each * kPagedStep) : 0;
        a.ranges = (int32_t)((of_one + each - 1) / each);
    }
    paged_partials(p, workspace, a.part_out, a.part_sum);
    a.begun = reinterpret_cast<int4*>(a.part_sum + paged_piece_rows(p) * 2);

#define SWA_PAGED(T, C) (p.d == 64 ? launch_paged_form<T, C, 64>(a, in_shares, stream) : launch_paged_form<T, C, 128>(a, in_shares, stream))
    const int rc = p.dtype == SWA_F32   ? SWA_PAGED(F32, F32)
                   : p.dtype == SWA_F16 ? (paged_int8(p) ? SWA_PAGED(F16, Q8) : SWA_PAGED(F16, F16))
                                        : (paged_int8(p) ? SWA_PAGED(BF16, Q8) : SWA_PAGED(BF16, BF16));
#undef SWA_PAGED
    if (rc != SWA_OK) return rc;
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
