// An upper bound of the logits of each page's keys, from the smallest and largest values of its channels alone:
//   q . k = sum_c q_c k_c <= sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c,
// a product of a row of 2 D bounds with the query's negative and positive parts, so it goes to the matrix cores like the attention's logits: sixteen
// rows of bounds by sixteen query heads.  Bound: HBM, one read of the bounds, where calls are large: 32 sequences of 1000 to 65536 tokens in pages of 16, 8 key heads of 128 bf16
// channels 51 us, 5.4 TB/s.  (With a load's lanes where the products want them, sixteen pieces of 64 bytes each, 96 us; more waves, or whole pages to a load, gain
// nothing.)
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
    int32_t group, ranges, log_heads;              // query heads of a key head; shares, or workgroups of a sequence; key heads of an item
    uint32_t group_mul;                            // t / group = t * group_mul >> group_shift
    int32_t group_shift;
    float scale, half_step;                        // of logits; what rounding may have moved a bound by, relative to it (codes)
};

// Waves of a workgroup, of which each has sixteen rows in LDS.
constexpr int score_waves(int row_bytes) { return row_bytes > 512 ? 2 : 4; }

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

// Sizes of 16-bit bounds, at least the smallest normal number, below which steps get no smaller.
template <typename T>
__device__ __forceinline__ Vec16 sizes_of(const Vec16& v)
{
    typedef uint16_t halves_t __attribute__((ext_vector_type(2)));
    constexpr uint16_t kLeast = std::is_same_v<T, F16> ? 0x0400 : 0x0080;
    auto word = [&](uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(halves_t, w & 0x7fff7fffu), halves_t{kLeast, kLeast}));
    };
    return Vec16{word(v.x), word(v.y), word(v.z), word(v.w)};
}
__device__ __forceinline__ Vec16 positive(const Vec16& v) { return Vec16{v.x & 0x7fff7fffu, v.y & 0x7fff7fffu, v.z & 0x7fff7fffu, v.w & 0x7fff7fffu}; }

// CODES: bounds of codes are the rounded ones, and half a step of each goes on top: sum_c |q_c| |bound_c| by the matrix cores, too (the 51 us
// above are 52.4, and 8 short sequences 5.47 instead of 5.28).  WHOLE: a load takes rows of one page.  SHARES: the items of all sequences are laid end to end and cut evenly, which every workgroup does by itself; else `ranges` workgroups serve one sequence.
template <typename T, int D, bool CODES, bool WHOLE, bool SHARES>
__global__ void __launch_bounds__(64 * score_waves(2 * D * Elem<T>::kBytes)) swa_paged_score_kernel(ScoreArgs a)
{
    constexpr int kHalf = D * Elem<T>::kBytes, kRow = 2 * kHalf, kSteps = kHalf / 64, kLoads = 2 * kSteps, kChunks = kRow / 16, kRows = 64 / kChunks,
                  kWaves = score_waves(kRow);
    __shared__ __align__(16) char tiles[kWaves][16 * kRow];
    __shared__ int scratch[kWaves];
    extern __shared__ int before[];                      // shares: items before sequence s, for s <= b
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, j = lane >> 4;
    char* const tile = tiles[wave];
    // An item is sixteen rows of bounds: `heads` key heads of 16 / heads pages.
    const int log_pages = 4 - a.log_heads, parts = a.h_kv >> a.log_heads;
    auto items_of = [&](int s, int& row, int& n, bool& too_long) {
        if (!paged_row(a.rows, s, row, n, too_long)) return 0;
        const int pages = (int)(((int64_t)n + a.page_size - 1) / a.page_size);
        return (pages + (1 << log_pages) - 1) / (1 << log_pages) * parts;
    };
    int row, n, s = 0, item, end, stride = kWaves, s_before = 0, s_end;
    bool too_long = false;
    if constexpr (SHARES) {
        const int per = (a.b + 64 * kWaves - 1) / (64 * kWaves), s0 = tid * per, s1 = s0 + per < a.b ? s0 + per : a.b;
        int own = 0;
        for (int i = s0; i < s1; ++i) {
            own += items_of(i, row, n, too_long);
            before[i + 1] = own;
        }
        if (too_long && blockIdx.x == 0) atomicOr(a.status, kStatusCapacityBit);
        const int add = sum_to(own, scratch) - own;
        for (int i = s0; i < s1; ++i) before[i + 1] += add;
        if (tid == 0) before[0] = 0;
        __syncthreads();
        const PagedShares shares(before[a.b], a.ranges);
        item = __builtin_amdgcn_readfirstlane(shares.begin(blockIdx.x) + wave);
        end = __builtin_amdgcn_readfirstlane(shares.begin(blockIdx.x + 1));
        for (int above = a.b; s + 1 < above;) {
            const int mid = (s + above) >> 1;
            if (before[mid] <= item) s = mid; else above = mid;
        }
        s = __builtin_amdgcn_readfirstlane(s);
        s_before = __builtin_amdgcn_readfirstlane(before[s]);
        s_end = __builtin_amdgcn_readfirstlane(before[s + 1]);
    } else {
        const int range = blockIdx.x / a.b;
        s = blockIdx.x - range * a.b;
        s_end = end = items_of(s, row, n, too_long);
        if (too_long && range == 0 && tid == 0) atomicOr(a.status, kStatusCapacityBit);
        item = range * kWaves + wave;
        stride = a.ranges * kWaves;
    }
    // The pool's pages of an item in its sequence, one a lane.
    auto page_at = [&](int item, int s, int s_before) {
        const int at = ((item - s_before) / parts << log_pages) + (lane & ((1 << log_pages) - 1));
        return at < a.max_pages ? a.block_table[(int64_t)s * a.max_pages + at] : 0;
    };
    // Of the sequence that `item` is in: query row and pages, which are loaded once for all of its items.
    int pages = 0;
    auto enter = [&]() {
        if constexpr (SHARES) {
            row = __builtin_amdgcn_readfirstlane(a.rows.row_start ? a.rows.row_start[s + 1] - 1 : s);
            n = __builtin_amdgcn_readfirstlane(a.rows.cache_len[s]);
        }
        pages = (int)(((int64_t)n + a.page_size - 1) / a.page_size);
    };
    bool bad = false;
    int next = 0;
    if (item < end) {
        next = page_at(item, s, s_before);
        enter();
    }
    while (item < end) {
        const int here = s, in_s = item - s_before, block = in_s / parts, kv0 = (in_s - block * parts) << a.log_heads, base = block << log_pages, pages_here = pages;
        const char* const from = a.q + row * a.q_stride + (int64_t)kv0 * a.group * kHalf;
        const bool used = base + (lane & ((1 << log_pages) - 1)) < pages, there = used && (uint32_t)next < (uint32_t)a.n_pages;
        const int page = there ? next : -1;
        bad |= used && !there;
        item += stride;
        if (item < end) {
            if (SHARES && item >= s_end) {
                do {
                    ++s;
                    s_before = s_end;
                    s_end = __builtin_amdgcn_readfirstlane(before[s + 1]);
                } while (item >= s_end);
                enter();
            }
            next = page_at(item, s, s_before);
        }
        // Column c of the products is query head c of the item's key heads.  (The first sixteen are on their way before the bounds.)
        const int columns = a.group << a.log_heads;
        Vec16 q[kSteps];
        auto load_queries = [&](int c0) __attribute__((always_inline)) {
            const char* const at = from + (int64_t)(c0 + col < columns ? c0 + col : 0) * kHalf + j * 16;
#pragma unroll
            for (int c = 0; c < kSteps; ++c) q[c] = load16(at + c * 64);
        };
        load_queries(0);
        // A page's rows of all heads lie behind each other, and a load takes 1 KiB: of one page, whose place is a scalar, or of several.  (Pages that there are none of
        // read the first one.)
        Vec16 box[kLoads];
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
            const int r = c * kRows + lane / kChunks, in_row = ((lane % kChunks) ^ r) * 16;
            if constexpr (WHOLE) {
                const int of = __builtin_amdgcn_readlane(page, c * kRows >> a.log_heads);
                const char* const at = a.bounds + ((int64_t)(of < 0 ? 0 : of) * a.h_kv + kv0 + (c * kRows & ((1 << a.log_heads) - 1))) * kRow;
                box[c] = load16_stream(at + (uint32_t)(lane / kChunks * kRow + in_row));
            } else {
                const int of = __shfl(page, r >> a.log_heads, 64);
                box[c] = load16_stream(a.bounds + ((int64_t)(of < 0 ? 0 : of) * a.h_kv + kv0 + (r & ((1 << a.log_heads) - 1))) * kRow + in_row);
            }
        }
        // To the lanes whose operands they are by way of LDS: chunk x of row r lies where x ^ r is, so that the sixteen rows of an operand lie on different banks.
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int c = 0; c < kLoads; ++c) store16(tile + c * 1024 + lane * 16, box[c]);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int c = 0; c < kLoads; ++c) box[c] = load16(tile + col * kRow + ((c * 4 + j) ^ col) * 16);
        // All rows by the query heads of all of the item's key heads, of which each row has its own ones.
        float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        for (int c0 = 0;;) {
            const int of = (int)(((uint64_t)(uint32_t)(c0 + col) * a.group_mul) >> a.group_shift);     // the key head of this lane's column
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
            if constexpr (CODES) {
#pragma unroll
                for (int c = 0; c < kSteps; ++c) {
                    sum = mfma16<T>(sizes_of<T>(box[c]), positive(part_of<T>(q[c], true)), sum);
                    sum = mfma16<T>(sizes_of<T>(box[kSteps + c]), part_of<T>(q[c], false), sum);
                }
                sum *= a.half_step;
            }
#pragma unroll
            for (int c = 0; c < kSteps; ++c) {
                sum = mfma16<T>(box[c], part_of<T>(q[c], true), sum);
                sum = mfma16<T>(box[kSteps + c], part_of<T>(q[c], false), sum);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = sum[i] != sum[i] ? INFINITY : sum[i];
                best[i] = c0 + col < columns && of == ((4 * j + i) & ((1 << a.log_heads) - 1)) ? fmaxf(best[i], x) : best[i];
            }
            c0 += 16;
            if (c0 >= columns) break;
            load_queries(c0);
        }
        // the sixteen columns to one, within rows of 16 lanes
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            best[i] = fmaxf(best[i], dpp_move<0xB1>(best[i]));
            best[i] = fmaxf(best[i], dpp_move<0x4E>(best[i]));
            best[i] = fmaxf(best[i], dpp_move<0x141>(best[i]));
            best[i] = fmaxf(best[i], dpp_move<0x140>(best[i]));
        }
        const float mine = (col & 2) ? ((col & 1) ? best[3] : best[2]) : ((col & 1) ? best[1] : best[0]);
        const int r = 4 * j + (col & 3), head = kv0 + (r & ((1 << a.log_heads) - 1)), p = base + (r >> a.log_heads), of = __shfl(page, r >> a.log_heads, 64);
        if (col < 4 && p < pages_here)
            a.score[((int64_t)here * a.h_kv + head) * a.max_pages + p] = of >= 0 ? mine * a.scale : -INFINITY;
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
    a.half_step = (p.dtype == SWA_F16 ? 0x1p-11f : 0x1p-8f) * (1.f + 0x1p-12f);       // (the second factor for code times scale in fp32)
    page_divisor(a.group, a.group_mul, a.group_shift);
    // As many key heads to an item as there are columns for: a page's rows of them lie behind each other.
    a.log_heads = 3;
    while (a.log_heads > 0 && (p.h_kv % (1 << a.log_heads) != 0 || (a.group << a.log_heads) > 16)) --a.log_heads;
    const int of_pages = 16 >> a.log_heads, row_bytes = 2 * p.d * (p.dtype == SWA_F32 ? 4 : 2);
    const int waves = score_waves(row_bytes);
    const int64_t items = ((int64_t)paged_pages_max(p) + of_pages - 1) / of_pages * (p.h_kv >> a.log_heads);     // of a sequence, at most
    if ((int64_t)paged_pages_max(p) * p.h_kv > 0x7fff0000LL / p.b) return SWA_ERR_CAPACITY;      // (items are no more, and a stride behind the last one is a number still)
    // Shares level lengths out, as far as the host may not know them, and cost their sums: us, a workgroup's own sequence / shares, 32 query and 8 key heads, bf16, 128
    // channels, pages of 16: 8 sequences of 1000 to 8003 tokens (2016 items) 5.3 / 5.85, to 16000 (4000) 7.9 / 7.2, all 16000 8.7 / 10.2, to 32000 (8000) 12.5 / 10.3; 32
    // of 1000 to 8000 (8064) 12.6 / 10.6; 64 of 100 to 4000 11.3 / 10.7, all 4000 14.5 / 16.2; 32 of 1000 to 65536 71 / 51.6; 16 query heads on one key head, 16 of 1000 to 65536
    // (4096) 8.7 / 9.8; 12 heads of their own, fp32, 64 channels, 4 of 1000 to 65536 (12288) 19.0 / 13.7; 256 of 1 to 2000 (16128) 17.3 / 18.1.
    const bool in_shares = p.b > 1 && items * p.b > 6000;
    int64_t ranges = in_shares ? 4096 / waves : (8192 / waves + p.b - 1) / p.b;
    if (!in_shares && ranges > (items + waves - 1) / waves) ranges = (items + waves - 1) / waves;
    a.ranges = (int32_t)ranges;
    const dim3 grid((unsigned)(in_shares ? ranges : p.b * ranges)), block(64 * waves);
    const size_t lds = in_shares ? sizeof(int) * ((size_t)p.b + 1) : 0;
    const bool whole = (row_bytes << a.log_heads) >= 1024;
#define SWA_SCORE_FORM(T, D, C, W) (in_shares ? launch_kernel(swa_paged_score_kernel<T, D, C, W, true>, grid, block, lds, stream, a) \
                                              : launch_kernel(swa_paged_score_kernel<T, D, C, W, false>, grid, block, lds, stream, a))
#define SWA_SCORE(T, C) (p.d == 64 ? (whole ? SWA_SCORE_FORM(T, 64, C, true) : SWA_SCORE_FORM(T, 64, C, false)) \
                                   : (whole ? SWA_SCORE_FORM(T, 128, C, true) : SWA_SCORE_FORM(T, 128, C, false)))
    if (p.dtype == SWA_F32) SWA_SCORE(F32, false);
    else if (p.dtype == SWA_F16) paged_int8(p) ? SWA_SCORE(F16, true) : SWA_SCORE(F16, false);
    else paged_int8(p) ? SWA_SCORE(BF16, true) : SWA_SCORE(BF16, false);
#undef SWA_SCORE
#undef SWA_SCORE_FORM
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
