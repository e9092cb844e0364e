// Attention of one new token per sequence over pages that a list names, for each key head its own (as swa_paged_select writes them).  Bound by HBM: the listed
// tokens' keys and values are read once: 64 sequences of 8 key heads, 2048 tokens each of 128 bf16 channels, 89 us, 6.0 TB/s (of 7.2 that a read stream reaches); with six
// waves to a workgroup 92, in chunks of half the tokens 92.5.  8-bit codes are bound by their conversion besides, as in the decode.
//
// The lists' tokens, page behind page, are a sequence like any other, and the workgroup's work is the decode's (swa_paged_tile.hpp): up to 16 (or 32) query heads of a
// key head over a chunk of it.  Lists are about equally long whatever the sequences are, so chunks are, too, and no workgroup needs to know the other ones'
// lengths.  A tile's rows come by way of two loads, list and table: the list's is under way two tiles ahead, the table's one.
#include "swa_paged_tile.hpp"

namespace swa {

struct SelectedArgs {
    const char* q;
    int64_t q_stride;                              // bytes
    PagedRows rows;
    PagedPool pool;
    const int32_t *block_table, *sel, *sel_cnt;
    char* out;
    float* lse;
    float *part_out, *part_sum;                    // [pieces, row_tiles, heads, D] and [.., 2] (maximum, sum): chunk `split` of sequence and key head
    int32_t* status;
    int32_t b, h_q, h_kv, page_size, n_pages, max_pages, n_sel;
    int32_t group, row_tiles, heads, tile_heads;   // query heads of a key head, tiles of them, heads of a tile that there are at most, and that fit
    int32_t ranges, chunk;                         // chunks of a list at most, and their tokens
    uint32_t page_mul;                             // t / page_size = t * page_mul >> page_shift for 0 <= t < 2^31
    int32_t page_shift;
    int32_t sixteens;                              // pages are whole sixteens of tokens
};

// Entries of a list that count.
__device__ __forceinline__ int selected_count(const SelectedArgs& a, int pair, bool& bad)
{
    const int count = a.sel_cnt[pair];
    bad = count < 0 || count > a.n_sel;
    return count < 0 ? 0 : count > a.n_sel ? a.n_sel : count;
}

template <typename T, typename C, int D, int ROWS, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, Elem<C>::kBytes * D == 512 || (ROWS == 2 && D == 128) ? 2 : 3) swa_paged_selected_kernel(SelectedArgs a)
{
    typedef PagedTile<T, C, D, ROWS> S;
    constexpr int kKeys = S::kKeys, kSteps = S::kSteps, kChannels = S::kChannels;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, j = lane >> 4;

    // (row tiles of one range read the same pages, and meet in one XCD's L2)
    const int eighth = blockIdx.x >> 3, work = (eighth / a.row_tiles) * 8 + (blockIdx.x & 7), tile = eighth % a.row_tiles;
    const int heads = a.group - 16 * ROWS * tile < 16 * ROWS ? a.group - 16 * ROWS * tile : 16 * ROWS;
    __shared__ float part[WAVES][16][D + 4];
    __shared__ float tops[WAVES][16], sums[WAVES][16];

    const int units = a.b * a.h_kv, split = work / units;
    if (split >= a.ranges) return;
    const int pair = work - split * units, s = pair / a.h_kv, kv = pair - s * a.h_kv;
    bool too_long = false, bad = false;
    int row, n;
    if (!paged_row(a.rows, s, row, n, too_long)) {
        if (too_long && split == 0 && tid == 0) atomicOr(a.status, kStatusCapacityBit);
        return;
    }
    const int64_t head0 = (int64_t)kv * a.group + 16 * ROWS * tile;
    Vec16 q[ROWS][kSteps];
    const char* const from = a.q + row * a.q_stride + (head0 + col) * (D * Elem<T>::kBytes);
#pragma unroll
    for (int g = 0; g < ROWS; ++g)
#pragma unroll
        for (int c = 0; c < kSteps; ++c)
            q[g][c] = 16 * g + col < heads ? load16(from + 16 * g * D * Elem<T>::kBytes + S::query_at(c, j)) : Vec16{0u, 0u, 0u, 0u};

    const int tokens = selected_count(a, pair, bad) * a.page_size, begin = split * a.chunk;
    if (split > 0 && begin >= tokens) return;
    const int end = tokens - begin < a.chunk ? tokens : begin + a.chunk;
    const bool whole = tokens <= a.chunk;

    float top[ROWS], sum[ROWS];
    f32x4_t acc[ROWS][kChannels];
#pragma unroll
    for (int g = 0; g < ROWS; ++g) {
        top[g] = -INFINITY;
        sum[g] = 0.f;
#pragma unroll
        for (int e = 0; e < kChannels; ++e) acc[g][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const int32_t* const list = a.sel + (int64_t)pair * a.n_sel;
    const int32_t* const table = a.block_table + (int64_t)s * a.max_pages;

    // Place in the list of this lane's token of the tile at `base`, the page of the sequence there, that page's in the pool, and the token's row there.
    auto place = [&](int base) {
        const int t = base + (lane & (kKeys - 1));
        return (int)(((uint64_t)(uint32_t)(t < tokens ? t : tokens - 1) * a.page_mul) >> a.page_shift);
    };
    auto listed = [&](int base) { return list[place(base)]; };
    auto pool_page = [&](int entry) { return table[(uint32_t)entry < (uint32_t)a.max_pages ? entry : 0]; };
    auto row_of = [&](int base, int entry, int page) {
        const int t = base + (lane & (kKeys - 1)), off = t - place(base) * a.page_size;
        const bool known = (uint32_t)entry < (uint32_t)a.max_pages, live = t < tokens && known && entry * a.page_size + off < n,
                   in_pool = (uint32_t)page < (uint32_t)a.n_pages;
        bad |= t < tokens && ((entry >= 0 && !known) || (live && !in_pool));
        return live && in_pool ? (page * a.h_kv + kv) * a.page_size + off : -1;
    };
    constexpr int kStride = WAVES * kKeys;
    int next = begin + wave * kKeys, entry = 0, page = 0, entry2 = 0;
    if (next < end) {
        entry = listed(next);
        if (next + kStride < end) entry2 = listed(next + kStride);
        page = pool_page(entry);
    }
    // Whole tiles first, the others in a loop of their own, whose addresses then take no registers from this one.
    int left = next, left_end = end, r = 0;
    if (a.sixteens) {
        left = end;
        left_end = begin;
        while (next < end) {
            const int base = next, this_entry = entry, this_page = page;
            next += kStride;
            if (next < end) {
                entry = entry2;
                page = pool_page(entry);
                if (next + kStride < end) entry2 = listed(next + kStride);
            }
            const int rows = row_of(base, this_entry, this_page);
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
        r = row_of(next, entry, page);
    }
    while (left < left_end) {
        paged_take<T, C, D, ROWS, false>(a.pool, r, q, top, sum, acc);
        do {
            left += kStride;
            if (left >= left_end) break;
            const int at = listed(left);
            r = row_of(left, at, pool_page(at));
        } while (a.sixteens && !__any(r < 0));
    }
    if (bad) atomicOr(a.status, kStatusBadRequestBit);

    const int64_t piece = (int64_t)pair * a.ranges + split;
    paged_join_waves<T, C, D, ROWS, WAVES>(part, tops, sums, top, sum, acc, heads, tid, [&](int head, float all, float total, const float (&y)[kChannels]) __attribute__((always_inline)) {
        const int c = (tid & 15) * kChannels;
        if (whole) {
            paged_store<T, D>(a.out, a.lse, (int64_t)row * a.h_q + head0 + head, c, c == 0, all, total, y);
        } else {
            const int64_t at = (piece * a.row_tiles + tile) * a.heads + head;
#pragma unroll
            for (int e = 0; e < kChannels; e += 4)
                *reinterpret_cast<f32x4_t*>(a.part_out + at * D + c + e) = f32x4_t{y[e], y[e + 1], y[e + 2], y[e + 3]};
            if (c == 0) *reinterpret_cast<float2*>(a.part_sum + at * 2) = float2{all, total};
        }
    });
}

// The chunks of a list and query head to its output.
template <typename T, int D, int WAVES>
__global__ void __launch_bounds__(256) swa_paged_join_selected_kernel(SelectedArgs a)
{
    const int at = blockIdx.x * (4 / WAVES) + (WAVES == 1 ? threadIdx.x >> 6 : 0);
    if (at >= a.b * a.h_q) return;
    const int s = at / a.h_q, hq = at - s * a.h_q, kv = hq / a.group, of = hq - kv * a.group, pair = s * a.h_kv + kv;
    int row, n;
    bool too_long = false, bad = false;
    if (!paged_row(a.rows, s, row, n, too_long)) return;
    const int tokens = selected_count(a, pair, bad) * a.page_size;
    if (tokens <= a.chunk) return;
    const int64_t stride = a.row_tiles * a.heads, first = pair * a.ranges * stride + of / a.tile_heads * a.heads + of % a.tile_heads;
    paged_join_pieces<T, D, WAVES>(a.part_out, a.part_sum, [&](int i) __attribute__((always_inline)) { return first + i * stride; }, (tokens + a.chunk - 1) / a.chunk, a.out, a.lse,
                            (int64_t)row * a.h_q + hq);
}

template <typename T, typename C, int D>
static int launch_selected_form(const SelectedArgs& a, int span, hipStream_t stream)
{
    const int64_t units = (int64_t)a.b * a.h_kv, all = units * a.row_tiles;
    const uint64_t groups = (uint64_t)((units * a.ranges + 7) / 8 * 8) * a.row_tiles;
    // (as in swa_paged_decode: one wave for short lists)
    const bool one = a.tile_heads == 16, single = a.ranges == 1 && (span <= 32 || (all >= 1024 && span <= 128) || (all >= 2048 && span <= 256));
    if (groups * 64 * (single ? 1 : 4) > 0xffffffffULL || (uint64_t)a.b * a.h_q * 256 > 0xffffffffULL) return SWA_ERR_CAPACITY;
    auto kernel = single ? (one ? swa_paged_selected_kernel<T, C, D, 1, 1> : swa_paged_selected_kernel<T, C, D, 2, 1>)
                         : (one ? swa_paged_selected_kernel<T, C, D, 1, 4> : swa_paged_selected_kernel<T, C, D, 2, 4>);
    launch_kernel(kernel, dim3((unsigned)groups), dim3(single ? 64 : 256), 0, stream, a);
    if (a.ranges > 1) {
        const unsigned rows = (unsigned)(a.b * a.h_q);
        if (rows >= 1024) launch_kernel(swa_paged_join_selected_kernel<T, D, 1>, dim3((rows + 3) / 4), dim3(256), 0, stream, a);
        else launch_kernel(swa_paged_join_selected_kernel<T, D, 4>, dim3(rows), dim3(256), 0, stream, a);
    }
    return SWA_OK;
}

int launch_paged_selected(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const int32_t* slot,
                          const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table,
                          const int32_t* cache_len, const int32_t* sel, const int32_t* sel_cnt, int32_t n_sel, void* out, float* lse,
                          void* workspace, hipStream_t stream)
{
    SelectedArgs a{};
    a.q = static_cast<const char*>(q.data);
    a.q_stride = q.stride * (p.dtype == SWA_F32 ? 4 : 2);
    a.rows = PagedRows{row_start, slot, cache_len, n_rows, paged_len_max(p)};
    a.pool = PagedPool{static_cast<const char*>(k_pages), static_cast<const char*>(v_pages), k_scale, v_scale,
                       (p.scale > 0.f ? p.scale : 1.f / sqrtf((float)p.d)) * 1.44269504088896340736f};
    a.block_table = block_table;
    a.sel = sel;
    a.sel_cnt = sel_cnt;
    a.out = static_cast<char*>(out);
    a.lse = lse;
    paged_partials(p, workspace, a.part_out, a.part_sum);
    a.status = paged_status(workspace);
    a.b = p.b;
    a.h_q = p.h_q;
    a.h_kv = p.h_kv;
    a.page_size = p.page_size;
    a.n_pages = p.n_pages;
    a.max_pages = p.max_pages;
    a.n_sel = n_sel;
    a.group = p.h_q / p.h_kv;
    a.tile_heads = tile_heads_of(p);
    a.row_tiles = row_tiles_of(p);
    a.heads = a.group < a.tile_heads ? a.group : a.tile_heads;
    page_divisor(p.page_size, a.page_mul, a.page_shift);
    a.sixteens = p.page_size % 16 == 0;
    const int64_t span = (int64_t)n_sel * p.page_size, of_one = (span + kPagedStep - 1) / kPagedStep, each = paged_chunk_steps(p, of_one);
    a.chunk = (int32_t)(each * kPagedStep);
    a.ranges = (int32_t)((of_one + each - 1) / each);
#define SWA_SELECTED(T, C) (p.d == 64 ? launch_selected_form<T, C, 64>(a, (int)span, stream) : launch_selected_form<T, C, 128>(a, (int)span, stream))
    const int rc = p.dtype == SWA_F32   ? SWA_SELECTED(F32, F32)
                   : p.dtype == SWA_F16 ? (paged_int8(p) ? SWA_SELECTED(F16, Q8) : SWA_SELECTED(F16, F16))
                                        : (paged_int8(p) ? SWA_SELECTED(BF16, Q8) : SWA_SELECTED(BF16, BF16));
#undef SWA_SELECTED
    if (rc != SWA_OK) return rc;
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
