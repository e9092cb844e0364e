// Attention of one new token per sequence over a paged cache.  Bound by HBM: every key and value of the window is read once, 4 flops for
// two elements and query head.
//
// A workgroup takes a chunk of one sequence's tokens and one key/value head, with up to 16 of the query heads that share it; its
// waves take tiles of the chunk in turn, each with a running maximum and sum of the softmax.  All products go to the matrix cores, whose
// 16 columns are the query heads: also a single head's, since the matrix cores have fifteen times the time that HBM leaves them.
//   logits   S^T = K Q^T: a lane's operand is 16 bytes of one key, as it lies in memory; a 64-byte piece of 16 keys a load.
//   values   O^T = V^T P^T: S^T leaves lane (j, c) with keys 4j..4j+3 of column c, which is what the product with V takes from that lane
//            if its contraction runs over the keys in that order; nothing moves between lanes.  For V^T a lane loads the same D / 16
//            channels of those keys (whole rows a load) and swaps halves of words, a byte permutation for two elements.
// Tiles go from memory to registers and need no LDS.  Partial results of a sequence's chunks are joined by a second, small launch.
#include <math.h>

#include <type_traits>

#include "swa_paged.hpp"

namespace swa {

struct PagedArgs {
    const char* q;
    int64_t q_stride;                              // bytes
    const int32_t *row_start, *block_table, *cache_len;
    const char *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    char* out;
    float* lse;
    float *part_out, *part_sum;                    // [b, h_q, splits, D] and [b, h_q, splits, 2] (maximum, sum) of chunks
    int32_t* status;
    int32_t b, n_rows, h_q, h_kv, page_size, n_pages, max_pages, window, len_max;
    int32_t group, row_tiles, splits, chunk;       // query heads of a key head, tiles of 16 of them, chunks at most, tokens of one
    uint32_t page_mul;                             // t / page_size = t * page_mul >> page_shift for 0 <= t < 2^31
    int32_t page_shift;
    float scale;                                   // of logits to the base 2
};

constexpr int kPagedWaves = 4;
constexpr int kPagedTargetGroups = 1024;           // workgroups that fill the chip: four on every CU
constexpr int kPagedMaxSplits = 256;

static int64_t paged_units(const swa_paged_params& p)
{
    const int group = p.h_q / p.h_kv;
    return (int64_t)p.b * p.h_kv * ((group + 15) / 16);
}

static int paged_max_splits(const swa_paged_params& p)
{
    const int64_t s = (kPagedTargetGroups + paged_units(p) - 1) / paged_units(p);
    return s < kPagedMaxSplits ? (int)s : kPagedMaxSplits;
}

size_t paged_partial_bytes(const swa_paged_params& p)
{
    const int s = paged_max_splits(p);
    return s == 1 ? 0 : (size_t)p.b * p.h_q * s * (p.d + 2) * sizeof(float);
}

typedef float f32x4_t __attribute__((ext_vector_type(4)));

template <typename C>
__device__ __forceinline__ f32x4_t mfma16(const Vec16& a, const Vec16& b, f32x4_t c)
{
    if constexpr (std::is_same_v<C, F16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    else if constexpr (std::is_same_v<C, BF16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else {
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(u2f(a.x), u2f(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(u2f(a.y), u2f(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(u2f(a.z), u2f(b.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x4f32(u2f(a.w), u2f(b.w), c, 0, 0, 0);
    }
}

template <typename M>
__device__ __forceinline__ uint32_t round2(float lo, float hi)
{
    if constexpr (std::is_same_v<M, F16>) return f32x2_to_f16x2_bits(lo, hi);
    else return f32x2_to_bf16x2_bits(lo, hi);
}

__device__ __forceinline__ float code(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

// What a sequence asks of this call: its row, and its tokens lo .. n-1.  False: nothing.
__device__ __forceinline__ bool paged_sequence(const PagedArgs& a, int s, int& row, int& lo, int& n, bool& too_long)
{
    n = a.cache_len[s];
    row = s;
    too_long = false;
    if (a.row_start) {
        row = a.row_start[s + 1] - 1;
        if (row < a.row_start[s]) return false;
    }
    if (n < 0 || row < 0 || row >= a.n_rows) return false;
    if (n > a.len_max) {
        too_long = true;
        return false;
    }
    lo = a.window && n > a.window ? n - a.window : 0;
    return true;
}

// T: type of queries and outputs, C: of the pages (Q8: codes), M: of the operands in the matrix cores.
template <typename T, typename C, int D>
__global__ void __launch_bounds__(64 * kPagedWaves) swa_paged_decode_kernel(PagedArgs a)
{
    constexpr bool kCodes = std::is_same_v<C, Q8>, kWide = std::is_same_v<C, F32>;
    // Codes are exact in bf16.  fp16 queries have three bits more than that and the weights are products with a scale: both go as two bf16
    // numbers, which hold 16 bits.
    typedef std::conditional_t<kCodes, BF16, T> M;
    constexpr bool kSplitQ = kCodes && std::is_same_v<T, F16>;
    constexpr int kKeys = kWide ? 16 : 32, kTiles = kKeys / 16, kRow = D * Elem<C>::kBytes;
    constexpr int kSteps = kWide ? D / 16 : D / 32;      // operands of a logit
    constexpr int kChannels = D / 16;                    // of V in a lane
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, j = lane >> 4;

    // Row tiles of one chunk read the same pages: eight chunks, then the same ones' next row tile, so that they meet in one XCD's L2.
    const int eighth = blockIdx.x >> 3, units = a.b * a.h_kv;
    const int work = (eighth / a.row_tiles) * 8 + (blockIdx.x & 7), tile = eighth % a.row_tiles;
    const int split = work / units, unit = work - split * units;
    if (split >= a.splits) return;
    const int s = unit / a.h_kv, kv = unit - s * a.h_kv;
    int row, lo, n;
    bool too_long;
    if (!paged_sequence(a, s, row, lo, n, too_long)) {
        if (too_long && split == 0 && tid == 0) atomicOr(a.status, kStatusCapacityBit);
        return;
    }
    const int base0 = lo & ~31, chunks = n > base0 ? (n - base0 + a.chunk - 1) / a.chunk : 1;
    if (split >= chunks) return;
    const int begin = base0 + split * a.chunk, end = n - begin < a.chunk ? n : begin + a.chunk;

    // Query operands: column col is query head 16 tile + col of the group.
    const int heads = a.group - 16 * tile < 16 ? a.group - 16 * tile : 16;
    const int64_t head0 = (int64_t)kv * a.group + 16 * tile;
    Vec16 q[kSteps], q_rest[kSplitQ ? kSteps : 1];
    {
        const char* const from = a.q + row * a.q_stride + (head0 + col) * (D * Elem<T>::kBytes);
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
            // (16 bytes of codes are two operands' channels)
            const int at = kCodes ? (c / 2) * 64 + j * 16 + (c & 1) * 8 : kWide ? c * 16 + j * 4 : c * 32 + j * 8;
            q[c] = col < heads ? load16(from + at * Elem<T>::kBytes) : Vec16{0u, 0u, 0u, 0u};
            if constexpr (kSplitQ) {
                float f[8], rest[8];
                unpack<F16>(q[c], f);
                q[c] = pack<BF16>(f);
                unpack<BF16>(q[c], rest);
#pragma unroll
                for (int i = 0; i < 8; ++i) rest[i] = f[i] - rest[i];
                q_rest[c] = pack<BF16>(rest);
            }
        }
    }

    float top = -INFINITY, sum = 0.f;                    // of column col, the sum of this lane's keys alone
    f32x4_t acc[kChannels];
#pragma unroll
    for (int e = 0; e < kChannels; ++e) acc[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int32_t* const table = a.block_table + (int64_t)s * a.max_pages;
    bool bad = false;

    // Row of the pool that holds this lane's token of the tile at `base` (-1: none).
    auto token_page = [&](int base, int& off) {
        const int t = base + (lane & (kKeys - 1));
        const int clamped = t < lo ? lo : (t < n ? t : n - 1);
        const int page = (int)(((uint64_t)(uint32_t)clamped * a.page_mul) >> a.page_shift);
        off = clamped - page * a.page_size;
        return table[page];
    };
    int next_off = 0, next_page = begin + wave * kKeys < end ? token_page(begin + wave * kKeys, next_off) : 0;
    for (int base = begin + wave * kKeys; base < end; base += kPagedWaves * kKeys) {
        const int page = next_page, off = next_off;
        if (base + kPagedWaves * kKeys < end) next_page = token_page(base + kPagedWaves * kKeys, next_off);
        const int t = base + (lane & (kKeys - 1));
        const bool in_pool = (uint32_t)page < (uint32_t)a.n_pages, live = t >= lo && t < n;
        bad |= live && !in_pool;
        const int r = in_pool && live ? (page * a.h_kv + kv) * a.page_size + off : -1;
        const bool edge = __any(r < 0);

        int rk[kTiles], rv[kTiles][4];
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            rk[u] = __shfl(r, u * 16 + col, 64);
#pragma unroll
            for (int i = 0; i < 4; ++i) rv[u][i] = __shfl(r, u * 16 + j * 4 + i, 64);
        }
        // keys, then values: all of a tile's loads before its first product
        constexpr int kLoads = kCodes ? D / 64 : kSteps, kVLoad = kWide ? D / 64 : 1, kVBytes = kWide ? 16 : kChannels * Elem<C>::kBytes;
        Vec16 k[kTiles][kLoads];
        struct alignas(kVBytes < 16 ? kVBytes : 16) Values { uint32_t w[kVBytes / 4]; } v[kTiles][4][kVLoad];
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            const char* const from = a.k_pages + (int64_t)(rk[u] < 0 ? 0 : rk[u]) * kRow + j * 16;
#pragma unroll
            for (int c = 0; c < kLoads; ++c) k[u][c] = load16_stream(from + c * 64);
        }
#pragma unroll
        for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const char* const from = a.v_pages + (int64_t)(rv[u][i] < 0 ? 0 : rv[u][i]) * kRow + col * kVBytes;
#pragma unroll
                for (int x = 0; x < kVLoad; ++x) v[u][i][x] = *reinterpret_cast<const Values*>(from + x * 256);
            }
        float k_scale = 0.f, v_scale = 0.f;
        if constexpr (kCodes) {
            k_scale = r < 0 ? 0.f : a.k_scale[r];
            v_scale = r < 0 ? 0.f : a.v_scale[r];
        }

        float x[kTiles][4];
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            f32x4_t logit = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < kSteps; ++c) {
                if constexpr (kCodes) {
                    const Vec16& b = k[u][c / 2];
                    const uint32_t w[2] = {c & 1 ? b.z : b.x, c & 1 ? b.w : b.y};
                    const Vec16 op = {round2<BF16>(code(w[0], 0), code(w[0], 1)), round2<BF16>(code(w[0], 2), code(w[0], 3)),
                                      round2<BF16>(code(w[1], 0), code(w[1], 1)), round2<BF16>(code(w[1], 2), code(w[1], 3))};
                    logit = mfma16<BF16>(op, q[c], logit);
                    if constexpr (kSplitQ) logit = mfma16<BF16>(op, q_rest[c], logit);
                } else {
                    logit = mfma16<M>(k[u][c], q[c], logit);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[u][i] = logit[i] * (kCodes ? a.scale * __shfl(k_scale, u * 16 + j * 4 + i, 64) : a.scale);
                if (edge && rv[u][i] < 0) x[u][i] = -INFINITY;
            }
        }
        float most = x[0][0];
#pragma unroll
        for (int i = 1; i < 4 * kTiles; ++i) most = fmaxf(most, x[i / 4][i % 4]);
        most = fmaxf(most, __shfl_xor(most, 16, 64));
        most = fmaxf(most, __shfl_xor(most, 32, 64));
        if (__any(most > top)) {
            const float to = fmaxf(top, most), down = __builtin_amdgcn_exp2f(top - (to == -INFINITY ? 0.f : to));
            top = to;
            sum *= down;
#pragma unroll
            for (int e = 0; e < kChannels; ++e) acc[e] *= down;
        }
        const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[u][i] = __builtin_amdgcn_exp2f(x[u][i] - from);
                sum += x[u][i];
                if constexpr (kCodes) x[u][i] *= __shfl(v_scale, u * 16 + j * 4 + i, 64);
                if (edge && rv[u][i] < 0) {
                    x[u][i] = 0.f;
#pragma unroll
                    for (int y = 0; y < kVLoad; ++y) v[u][i][y] = Values{};
                }
            }

        if constexpr (kWide) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < kChannels; ++e)
                    acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(u2f(v[0][i][e / 4].w[e % 4]), x[0][i], acc[e], 0, 0, 0);
        } else if constexpr (kCodes) {
            Vec16 p = {round2<BF16>(x[0][0], x[0][1]), round2<BF16>(x[0][2], x[0][3]), round2<BF16>(x[1][0], x[1][1]), round2<BF16>(x[1][2], x[1][3])};
            float f[8];
            unpack<BF16>(p, f);
            const Vec16 p_rest = {round2<BF16>(x[0][0] - f[0], x[0][1] - f[1]), round2<BF16>(x[0][2] - f[2], x[0][3] - f[3]),
                                  round2<BF16>(x[1][0] - f[4], x[1][1] - f[5]), round2<BF16>(x[1][2] - f[6], x[1][3] - f[7])};
#pragma unroll
            for (int e = 0; e < kChannels; ++e) {
                auto c = [&](int u, int i) { return code(v[u][i][0].w[e / 4], e % 4); };
                const Vec16 op = {round2<BF16>(c(0, 0), c(0, 1)), round2<BF16>(c(0, 2), c(0, 3)), round2<BF16>(c(1, 0), c(1, 1)),
                                  round2<BF16>(c(1, 2), c(1, 3))};
                acc[e] = mfma16<BF16>(op, p, acc[e]);
                acc[e] = mfma16<BF16>(op, p_rest, acc[e]);
            }
        } else {
            const Vec16 p = {round2<M>(x[0][0], x[0][1]), round2<M>(x[0][2], x[0][3]), round2<M>(x[1][0], x[1][1]), round2<M>(x[1][2], x[1][3])};
#pragma unroll
            for (int e = 0; e < kChannels; ++e) {
                constexpr uint32_t kLow = 0x05040100u, kHigh = 0x07060302u;
                auto two = [&](int u, int i) { return __builtin_amdgcn_perm(v[u][i + 1][0].w[e / 2], v[u][i][0].w[e / 2], e & 1 ? kHigh : kLow); };
                acc[e] = mfma16<M>(Vec16{two(0, 0), two(0, 2), two(1, 0), two(1, 2)}, p, acc[e]);
            }
        }
    }
    if (bad) atomicOr(a.status, kStatusBadRequestBit);

    // The waves' results to one, in LDS: rows are query heads.
    constexpr int kPitch = D + 4;
    __shared__ float part[kPagedWaves][16][kPitch];
    __shared__ float tops[kPagedWaves][16], sums[kPagedWaves][16];
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (j == 0) {
        tops[wave][col] = top;
        sums[wave][col] = sum;
    }
#pragma unroll
    for (int e = 0; e < kChannels; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][col][kWide ? (e / 4) * 64 + (4 * j + i) * 4 + e % 4 : (4 * j + i) * kChannels + e] = acc[e][i];
    __syncthreads();
    const int head = tid >> 4;
    if (head >= heads) return;
    float all = tops[0][head];
#pragma unroll
    for (int w = 1; w < kPagedWaves; ++w) all = fmaxf(all, tops[w][head]);
    float total = 0.f, y[kChannels] = {};
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(tops[w][head] - (all == -INFINITY ? 0.f : all));
        total = __builtin_fmaf(sums[w][head], f, total);
#pragma unroll
        for (int e = 0; e < kChannels; ++e) y[e] = __builtin_fmaf(part[w][head][(tid & 15) * kChannels + e], f, y[e]);
    }
    const int64_t hq = head0 + head;
    if (chunks == 1) {
        const float inverse = total == 0.f ? 0.f : 1.f / total;
        char* const to = a.out + ((int64_t)row * a.h_q + hq) * (D * Elem<T>::kBytes);
#pragma unroll
        for (int e = 0; e < kChannels; ++e) store_elem<T>(to, (tid & 15) * kChannels + e, total == 0.f ? 0.f : y[e] * inverse);
        if (a.lse && (tid & 15) == 0) a.lse[(int64_t)row * a.h_q + hq] = (all + __builtin_log2f(total)) * 0.69314718055994530942f;
        return;
    }
    const int64_t at = ((int64_t)s * a.h_q + hq) * a.splits + split;
#pragma unroll
    for (int e = 0; e < kChannels; e += 4)
        *reinterpret_cast<f32x4_t*>(a.part_out + at * D + (tid & 15) * kChannels + e) = f32x4_t{y[e], y[e + 1], y[e + 2], y[e + 3]};
    if ((tid & 15) == 0) *reinterpret_cast<float2*>(a.part_sum + at * 2) = float2{all, total};
}

// Chunks of a sequence and query head to its output, in their order.
template <typename T, int D>
__global__ void __launch_bounds__(256) swa_paged_join_kernel(PagedArgs a)
{
    constexpr int kLanes = D / 4, kShares = 256 / kLanes;
    const int s = blockIdx.x / a.h_q, hq = blockIdx.x - s * a.h_q, tid = threadIdx.x, share = tid / kLanes, c = (tid % kLanes) * 4;
    int row, lo, n;
    bool too_long;
    if (!paged_sequence(a, s, row, lo, n, too_long)) return;
    const int base0 = lo & ~31, chunks = n > base0 ? (n - base0 + a.chunk - 1) / a.chunk : 1;
    if (chunks == 1) return;
    const int64_t at = ((int64_t)s * a.h_q + hq) * a.splits;
    __shared__ float weight[kPagedMaxSplits], waves[4], waves2[4];
    __shared__ f32x4_t part[kShares][kLanes];
    const float2 mine = tid < chunks ? *reinterpret_cast<const float2*>(a.part_sum + (at + tid) * 2) : float2{-INFINITY, 0.f};
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
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = share; i < chunks; i += kShares) y += *reinterpret_cast<const f32x4_t*>(a.part_out + (at + i) * D + c) * weight[i];
    part[share][tid % kLanes] = y;
    __syncthreads();
    if (share) return;
#pragma unroll
    for (int i = 1; i < kShares; ++i) y += part[i][tid];
    char* const to = a.out + ((int64_t)row * a.h_q + hq) * (D * Elem<T>::kBytes);
    const float inverse = 1.f / total;
#pragma unroll
    for (int i = 0; i < 4; ++i) store_elem<T>(to, c + i, total == 0.f ? 0.f : y[i] * inverse);
    if (a.lse && tid == 0) a.lse[(int64_t)row * a.h_q + hq] = (top + __builtin_log2f(total)) * 0.69314718055994530942f;
}

int launch_paged_decode(const swa_paged_params& p, const swa_rows& q, int32_t n_rows, const int32_t* row_start, const void* k_pages,
                        const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* block_table, const int32_t* cache_len,
                        void* out, float* lse, void* workspace, hipStream_t stream)
{
    PagedArgs a{};
    a.q = static_cast<const char*>(q.data);
    a.q_stride = q.stride * (p.dtype == SWA_F32 ? 4 : 2);
    a.row_start = row_start;
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
    a.len_max = p.max_pages * p.page_size;
    if (p.len_bound > 0 && p.len_bound < a.len_max) a.len_max = p.len_bound;
    a.group = p.h_q / p.h_kv;
    a.row_tiles = (a.group + 15) / 16;
    // exact for numerators below 2^31: the error of page_mul, below page_size <= 2^l, times the numerator stays below 2^(31 + l)
    int l = 0;
    while ((1 << l) < p.page_size) ++l;
    a.page_shift = 31 + l;
    a.page_mul = (uint32_t)(((UINT64_C(1) << a.page_shift) + p.page_size - 1) / p.page_size);
    a.scale = (p.scale > 0.f ? p.scale : 1.f / sqrtf((float)p.d)) * 1.44269504088896340736f;

    const int64_t units = (int64_t)p.b * p.h_kv;
    const int step = kPagedWaves * 32;
    const int64_t span = p.window > 0 && p.window < a.len_max ? (int64_t)p.window + 31 : a.len_max;
    int64_t splits = paged_max_splits(p);
    if (splits > (span + step - 1) / step) splits = (span + step - 1) / step;
    a.chunk = (int32_t)(((span + splits - 1) / splits + step - 1) / step * step);
    a.splits = (int32_t)((span + a.chunk - 1) / a.chunk);
    a.part_out = reinterpret_cast<float*>(static_cast<char*>(workspace) + kPagedPartialOffset);
    a.part_sum = a.part_out + (int64_t)p.b * p.h_q * a.splits * p.d;

    const int64_t works = (units * a.splits + 7) / 8 * 8;
    if (works * a.row_tiles > 0x7fffffffLL) return SWA_ERR_BAD_SHAPE;
    const dim3 grid((unsigned)(works * a.row_tiles)), block(64 * kPagedWaves);
#define SWA_PAGED(T, C) \
    (p.d == 64 ? launch_kernel(swa_paged_decode_kernel<T, C, 64>, grid, block, 0, stream, a) \
               : launch_kernel(swa_paged_decode_kernel<T, C, 128>, grid, block, 0, stream, a))
    if (p.dtype == SWA_F32) SWA_PAGED(F32, F32);
    else if (p.dtype == SWA_F16) paged_int8(p) ? SWA_PAGED(F16, Q8) : SWA_PAGED(F16, F16);
    else paged_int8(p) ? SWA_PAGED(BF16, Q8) : SWA_PAGED(BF16, BF16);
#undef SWA_PAGED
    if (a.splits > 1) {
        const dim3 join((unsigned)((int64_t)p.b * p.h_q));
#define SWA_JOIN(T) (p.d == 64 ? launch_kernel(swa_paged_join_kernel<T, 64>, join, dim3(256), 0, stream, a) \
                               : launch_kernel(swa_paged_join_kernel<T, 128>, join, dim3(256), 0, stream, a))
        if (p.dtype == SWA_F32) SWA_JOIN(F32);
        else if (p.dtype == SWA_F16) SWA_JOIN(F16);
        else SWA_JOIN(BF16);
#undef SWA_JOIN
    }
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
