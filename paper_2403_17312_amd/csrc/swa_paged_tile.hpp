// What a wave of the paged attentions does with one tile of keys and values: logits, running softmax, weighted values, all on the matrix cores, whose 16
// columns are query rows.
//   logits   S^T = K Q^T: a lane's operand is 16 bytes of one key, as it lies in memory; a 64-byte piece of 16 keys a load.
//   values   O^T = V^T P^T: S^T leaves lane (j, c) with keys 4j..4j+3 of column c, which is what the product with V takes from that lane
//            if its contraction runs over the keys in that order; nothing moves between lanes.  For V^T a lane loads the same D / 16
//            channels of those keys (whole rows a load) and swaps halves of words, a byte permutation for two elements.
// Tiles go from memory to registers and need no LDS.
#pragma once

#include <math.h>

#include <type_traits>

#include "swa_paged.hpp"
#include "swa_select.hpp"

namespace swa {

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

// Eight weights (0 or more) as two numbers of the matrix cores' type each, big and rest.
//   FINITE (codes, or infinite results are looked after): rounded to the nearest both times.
//   else: the values may be infinite, and both of a weight's numbers have to be of its sign for an infinity to stay one.  So big is cut off, from what lies just below the
//   weight (bf16), or both are raised to fp16's smallest number, 2^-40 of the largest weight, however small the weight is (but for 0).
template <typename P, bool FINITE>
__device__ __forceinline__ void split8(const float* w, Vec16& big, Vec16& rest)
{
    constexpr uint32_t kHighHalves = 0x07060302u;
    float f[8], r[8];
    if constexpr (FINITE) {
        big = Vec16{round2<P>(w[0], w[1]), round2<P>(w[2], w[3]), round2<P>(w[4], w[5]), round2<P>(w[6], w[7])};
    } else if constexpr (std::is_same_v<P, F16>) {
        auto cut = [&](int i) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(w[i], w[i + 1])); };
        big = Vec16{cut(0), cut(2), cut(4), cut(6)};
    } else {
        auto below = [&](int i) { return __builtin_elementwise_sub_sat(f2u(w[i]), 1u); };
        auto cut = [&](int i) { return __builtin_amdgcn_perm(below(i + 1), below(i), kHighHalves); };
        big = Vec16{cut(0), cut(2), cut(4), cut(6)};
    }
    unpack<P>(big, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = w[i] - f[i];
    rest = Vec16{round2<P>(r[0], r[1]), round2<P>(r[2], r[3]), round2<P>(r[4], r[5]), round2<P>(r[6], r[7])};
    if constexpr (!FINITE && std::is_same_v<P, F16>) {
        typedef uint16_t halves_t __attribute__((ext_vector_type(2)));
        auto raise = [&](int i, uint32_t& a, uint32_t& b) {         // (as whole numbers, of which 1 is the smallest fp16 one)
            const halves_t least = __builtin_elementwise_min(__builtin_bit_cast(halves_t, __builtin_amdgcn_perm(f2u(w[i + 1]), f2u(w[i]), kHighHalves)), halves_t{1, 1});
            a = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(halves_t, a), least));
            b = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(halves_t, b), least));
        };
        raise(0, big.x, rest.x);
        raise(2, big.y, rest.y);
        raise(4, big.z, rest.z);
        raise(6, big.w, rest.w);
    }
}

template <typename V>
__device__ __forceinline__ V load_values(const char* p)
{
    typedef uint32_t words_t __attribute__((ext_vector_type(sizeof(V) / 4)));
    if constexpr (sizeof(V) == 4) return V{{__builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p))}};
    else return __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const words_t*>(p)));
}

__device__ __forceinline__ float code(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

// T: type of queries and outputs, C: of the pages (Q8: codes), ROWS: sixteens of query rows.
template <typename T, typename C, int D, int ROWS>
struct PagedTile {
    static constexpr bool kCodes = std::is_same_v<C, Q8>, kWide = std::is_same_v<C, F32>;
    // Codes are exact in either 16-bit type.  Keys get the queries' type; values get bf16, whose range the weights need, which are products with a
    // scale there.  In 16 bits weights go as two numbers, which hold 15 or 16 bits in bf16 and 21 in fp16: one alone left the output a tenth to a quarter farther from
    // the exact one than its own rounding does, and the second product is free (decode of 128 ragged sequences, bf16, 353.7 / 353.0 us, of one of 131071 tokens, fp16, 51.6 / 51.8).
    static constexpr int kTiles = kWide && (D == 128 || ROWS == 2) ? 1 : 2, kKeys = 16 * kTiles, kRow = D * Elem<C>::kBytes;
    static constexpr int kSteps = kWide ? D / 16 : D / 32;       // operands of a logit
    static constexpr int kChannels = D / 16;                     // of V in a lane
    // A weight is exp2(x - top + kRaise).  fp16 has 2^-14 to 2^16 for normal numbers: raised so far the largest weight is 2^16 (65504, and a rest of 32) and a step of
    // the smallest numbers 2^-40 of it.  Without, a wave lost what lies 17.4 nats below its loudest token, which for 131072 such tokens beside one
    // of small value was 6.7 % of the output.  The sum carries the same factor, so nothing takes it back but the maximum, as it is handed on.
    static constexpr float kRaise = std::is_same_v<C, F16> ? 16.f : 0.f;
    static constexpr int kLoads = kCodes ? D / 64 : kSteps, kVLoad = kWide ? D / 64 : 1, kVBytes = kWide ? 16 : kChannels * Elem<C>::kBytes;
    struct alignas(kVBytes < 16 ? kVBytes : 16) Values { uint32_t w[kVBytes / 4]; };
    // Where in a query row operand c of lanes `j` begins, in bytes (16 bytes of codes are two operands' channels).
    static __device__ __forceinline__ int query_at(int c, int j)
    {
        return (kCodes ? (c / 2) * 64 + j * 16 + (c & 1) * 8 : kWide ? c * 16 + j * 4 : c * 32 + j * 8) * Elem<T>::kBytes;
    }
};

// Whose rows a call serves.
struct PagedRows {
    const int32_t *row_start, *slot, *cache_len;
    int32_t n_rows, len_max;
};

// Row and length of a sequence; false: the call leaves it out (too_long: for its length).
__device__ __forceinline__ bool paged_row(const PagedRows& a, int s, int& row, int& n, bool& too_long)
{
    n = a.cache_len[s];
    row = s;
    if (a.row_start) {
        row = a.row_start[s + 1] - 1;
        if (row < a.row_start[s]) return false;
    }
    if (n < 0 || row < 0 || row >= a.n_rows) return false;
    if (a.slot && a.slot[row] < 0) return false;
    if (n > a.len_max) {
        too_long = true;
        return false;
    }
    return true;
}

// The shares: the first `more` of them have one step more than the others.
struct PagedShares {
    int steps, more;
    __device__ __forceinline__ PagedShares(int total, int shares) : steps(total / shares), more(total % shares) {}
    __device__ __forceinline__ int begin(int g) const { return g * steps + (g < more ? g : more); }
    __device__ __forceinline__ int of(int x) const
    {
        const int longer = more * (steps + 1);
        return x < longer ? x / (steps + 1) : more + (x - longer) / steps;
    }
};

// Sums of N values up to and including this thread of a workgroup (scratch: N of LDS for each wave; all threads arrive).
template <int N>
__device__ __forceinline__ void sums_to(int (&v)[N], int* scratch)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_scan(v[i]);
    __syncthreads();
    if (lane == 63)
#pragma unroll
        for (int i = 0; i < N; ++i) scratch[wave * N + i] = v[i];
    __syncthreads();
    for (int w = 0; w < wave; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += scratch[w * N + i];
}
__device__ __forceinline__ int sum_to(int v, int* scratch)
{
    int one[1] = {v};
    sums_to(one, scratch);
    return one[0];
}

// The pool, and the scale of logits to the base 2.
struct PagedPool {
    const char *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    float scale;
};

// One tile, whose tokens lie in rows r (of lane t % kKeys) of the pool.  In `whole` tiles all of them do, and sixteen at a time behind each
// other, so that addresses are a scalar and a lane's constant; in others each lane fetches its rows' numbers, and rows of -1 are left out.
// top and sum: of column lane % 16, the sum of this lane's keys alone.  STREAM: nobody reads the tile again.
template <typename T, typename C, int D, int ROWS, bool kWhole, bool STREAM = true>
__device__ __forceinline__ void paged_take(const PagedPool& a, const int r, const Vec16 (&q)[ROWS][PagedTile<T, C, D, ROWS>::kSteps], float (&top)[ROWS],
                                           float (&sum)[ROWS], f32x4_t (&acc)[ROWS][PagedTile<T, C, D, ROWS>::kChannels])
{
    typedef PagedTile<T, C, D, ROWS> S;
    typedef typename S::Values Values;
    constexpr bool kCodes = S::kCodes, kWide = S::kWide;
    constexpr int kTiles = S::kTiles, kRow = S::kRow, kSteps = S::kSteps, kChannels = S::kChannels, kLoads = S::kLoads, kVLoad = S::kVLoad, kVBytes = S::kVBytes;
    constexpr float kRaise = S::kRaise;
    const int lane = threadIdx.x & 63, col = lane & 15, j = lane >> 4;
    int rv[kTiles][4];
    Vec16 k[kTiles][kLoads];
    Values v[kTiles][4][kVLoad];
    f32x4_t k_scale[kTiles], v_scale[kTiles];
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
        const char* k_from;
        if constexpr (kWhole) {
            const int64_t first = __builtin_amdgcn_readlane(r, u * 16);
            k_from = a.k_pages + first * kRow + (uint32_t)(col * kRow + j * 16);
        } else {
            const int rk = __shfl(r, u * 16 + col, 64);
            k_from = a.k_pages + (int64_t)(rk < 0 ? 0 : rk) * kRow + j * 16;
        }
#pragma unroll
        for (int c = 0; c < kLoads; ++c) k[u][c] = STREAM ? load16_stream(k_from + c * 64) : load16(k_from + c * 64);
    }
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
        const int64_t first = kWhole ? __builtin_amdgcn_readlane(r, u * 16) : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const char* v_from;
            if constexpr (kWhole) {
                v_from = a.v_pages + first * kRow + (uint32_t)(j * 4 * kRow + col * kVBytes) + i * kRow;
            } else {
                rv[u][i] = __shfl(r, u * 16 + j * 4 + i, 64);
                v_from = a.v_pages + (int64_t)(rv[u][i] < 0 ? 0 : rv[u][i]) * kRow + col * kVBytes;
            }
#pragma unroll
            for (int x = 0; x < kVLoad; ++x) v[u][i][x] = STREAM ? load_values<Values>(v_from + x * 256) : *reinterpret_cast<const Values*>(v_from + x * 256);
        }
        if constexpr (kCodes) {
            if constexpr (kWhole) {
                k_scale[u] = *reinterpret_cast<const f32x4_t*>(a.k_scale + first + 4 * j);
                v_scale[u] = *reinterpret_cast<const f32x4_t*>(a.v_scale + first + 4 * j);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    k_scale[u][i] = rv[u][i] < 0 ? 0.f : a.k_scale[rv[u][i]];
                    v_scale[u][i] = rv[u][i] < 0 ? 0.f : a.v_scale[rv[u][i]];
                }
            }
        }
    }

    __builtin_amdgcn_sched_barrier(0);
    float x[ROWS][kTiles][4];
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
        f32x4_t logit[ROWS];
#pragma unroll
        for (int g = 0; g < ROWS; ++g) logit[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
            Vec16 op;
            if constexpr (kCodes) {
                const Vec16& b = k[u][c / 2];
                const uint32_t w[2] = {c & 1 ? b.z : b.x, c & 1 ? b.w : b.y};
                op = Vec16{round2<T>(code(w[0], 0), code(w[0], 1)), round2<T>(code(w[0], 2), code(w[0], 3)),
                           round2<T>(code(w[1], 0), code(w[1], 1)), round2<T>(code(w[1], 2), code(w[1], 3))};
            } else {
                op = k[u][c];
            }
#pragma unroll
            for (int g = 0; g < ROWS; ++g) logit[g] = mfma16<T>(op, q[g][c], logit[g]);
        }
#pragma unroll
        for (int g = 0; g < ROWS; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[g][u][i] = logit[g][i] * a.scale;
                if constexpr (kCodes) x[g][u][i] *= k_scale[u][i];
                if constexpr (!kWhole) x[g][u][i] = rv[u][i] < 0 ? -INFINITY : x[g][u][i];
            }
    }
    if constexpr (!kWhole) {                         // (a weight of 0 times what is no number is none either)
#pragma unroll
        for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t keep = rv[u][i] < 0 ? 0u : ~0u;
#pragma unroll
                for (int y = 0; y < kVLoad; ++y)
#pragma unroll
                    for (int z = 0; z < kVBytes / 4; ++z) v[u][i][y].w[z] &= keep;
            }
    }
#pragma unroll
    for (int g = 0; g < ROWS; ++g) {
        float most = x[g][0][0];
#pragma unroll
        for (int i = 1; i < 4 * kTiles; ++i) most = fmaxf(most, x[g][i / 4][i % 4]);
        most = fmaxf(most, __shfl_xor(most, 16, 64));
        most = fmaxf(most, __shfl_xor(most, 32, 64));
        if (__any(most > top[g])) {
            const float to = fmaxf(top[g], most), down = __builtin_amdgcn_exp2f(top[g] - (to == -INFINITY ? 0.f : to));
            top[g] = to;
            sum[g] *= down;
#pragma unroll
            for (int e = 0; e < kChannels; ++e) acc[g][e] *= down;
        }
        const float from = (top[g] == -INFINITY ? 0.f : top[g]) - kRaise;
#pragma unroll
        for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[g][u][i] = __builtin_amdgcn_exp2f(x[g][u][i] - from);
                sum[g] += x[g][u][i];
                if constexpr (kCodes) x[g][u][i] *= v_scale[u][i];
            }
    }

    if constexpr (kWide) {
#pragma unroll
        for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < kChannels; ++e)
#pragma unroll
                    for (int g = 0; g < ROWS; ++g)
                        acc[g][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(u2f(v[u][i][e / 4].w[e % 4]), x[g][u][i], acc[g][e], 0, 0, 0);
    } else {
#pragma unroll
        for (int u = 0; u < kTiles; u += 2) {        // 32 keys a product
            typedef std::conditional_t<kCodes, BF16, T> P;
            Vec16 p[ROWS], p_rest[ROWS];
#pragma unroll
            for (int g = 0; g < ROWS; ++g) split8<P, kCodes>(x[g][u], p[g], p_rest[g]);
#pragma unroll
            for (int e = 0; e < kChannels; ++e) {
                Vec16 op;
                if constexpr (kCodes) {
                    auto c = [&](int w, int i) { return code(v[u + w][i][0].w[e / 4], e % 4); };
                    op = Vec16{round2<BF16>(c(0, 0), c(0, 1)), round2<BF16>(c(0, 2), c(0, 3)), round2<BF16>(c(1, 0), c(1, 1)),
                               round2<BF16>(c(1, 2), c(1, 3))};
                } else {
                    constexpr uint32_t kLow = 0x05040100u, kHigh = 0x07060302u;
                    auto two = [&](int w, int i) {
                        return __builtin_amdgcn_perm(v[u + w][i + 1][0].w[e / 2], v[u + w][i][0].w[e / 2], e & 1 ? kHigh : kLow);
                    };
                    op = Vec16{two(0, 0), two(0, 2), two(1, 0), two(1, 2)};
                }
#pragma unroll
                for (int g = 0; g < ROWS; ++g) {
                    acc[g][e] = mfma16<P>(op, p[g], acc[g][e]);
                    acc[g][e] = mfma16<P>(op, p_rest[g], acc[g][e]);
                }
            }
        }
    }
}

// Channels c .. c + N - 1 of query row `at`, divided by the weights' sum, and the logarithm of that (all: the base that the weights go by).
template <typename T, int D, int N>
__device__ __forceinline__ void paged_store(char* out, float* lse, int64_t at, int c, bool first, float all, float total, const float (&y)[N])
{
    const float inverse = 1.f / total;
    char* const to = out + at * (D * Elem<T>::kBytes);
#pragma unroll
    for (int e = 0; e < N; ++e) store_elem<T>(to, c + e, total == 0.f ? 0.f : y[e] * inverse);
    if (lse && first) lse[at] = (all + __builtin_log2f(total)) * 0.69314718055994530942f;
}

// The waves' results to one, in LDS, where rows are query rows: emit(query row, maximum, sum, its channels (who & 15) * D / 16 ...) for rows < heads, sixteen threads
// to a row.  who: threadIdx.x.
template <typename T, typename C, int D, int ROWS, int WAVES, typename F>
__device__ __forceinline__ void paged_join_waves(float (&part)[WAVES][16][D + 4], float (&tops)[WAVES][16], float (&sums)[WAVES][16], const float (&top)[ROWS],
                                                 float (&sum)[ROWS], const f32x4_t (&acc)[ROWS][D / 16], int heads, int who, F emit)
{
    typedef PagedTile<T, C, D, ROWS> S;
    constexpr int kChannels = D / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), to_col = who & 15, to_j = (who >> 4) & 3;
#pragma unroll
    for (int g = 0; g < ROWS; ++g) {
        sum[g] += __shfl_xor(sum[g], 16, 64);
        sum[g] += __shfl_xor(sum[g], 32, 64);
        __syncthreads();                                     // (what was there before has been read)
        if (to_j == 0) {
            tops[wave][to_col] = top[g] - S::kRaise;
            sums[wave][to_col] = sum[g];
        }
#pragma unroll
        for (int e = 0; e < kChannels; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave][to_col][S::kWide ? (e / 4) * 64 + (4 * to_j + i) * 4 + e % 4 : (4 * to_j + i) * kChannels + e] = acc[g][e][i];
        __syncthreads();
        for (int head = who >> 4; head < 16 && 16 * g + head < heads; head += 4 * WAVES) {
            float all = tops[0][head];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) all = fmaxf(all, tops[w][head]);
            float total = 0.f, y[kChannels] = {};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(tops[w][head] - (all == -INFINITY ? 0.f : all));
                total = __builtin_fmaf(sums[w][head], f, total);
#pragma unroll
                for (int e = 0; e < kChannels; ++e) y[e] = __builtin_fmaf(part[w][head][(who & 15) * kChannels + e], f, y[e]);
            }
            emit(16 * g + head, all, total, y);
        }
    }
}

// Pieces of a query row, piece i at partial result piece_at(i), to its output, in an order that their number fixes.  By WAVES waves of a workgroup of 256 threads, of which
// each has a row of its own where WAVES is 1.
template <typename T, int D, int WAVES, typename F>
__device__ __forceinline__ void paged_join_pieces(const float* part_out, const float* part_sum, F piece_at, int count, char* out, float* lse, int64_t to)
{
    constexpr int kLanes = D / 4, kTeams = 64 / kLanes, kAll = WAVES * kTeams;
    const int tid = threadIdx.x & (64 * WAVES - 1), team = tid / kLanes, lane = tid % kLanes;
    float top = -INFINITY, total = 0.f;
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    auto join = [&](float most, float part_total, const f32x4_t& part_y) __attribute__((always_inline)) {
        const float now = fmaxf(top, most), from = now == -INFINITY ? 0.f : now;
        const float old = __builtin_amdgcn_exp2f(top - from), w = __builtin_amdgcn_exp2f(most - from);
        y = y * old + part_y * w;
        total = total * old + part_total * w;
        top = now;
    };
    constexpr int kAhead = 4;
    for (int i = team; i < count; i += kAhead * kAll) {
        float2 m[kAhead];
        f32x4_t x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t at = piece_at(i + k * kAll < count ? i + k * kAll : i);
            m[k] = *reinterpret_cast<const float2*>(part_sum + at * 2);
            x[k] = *reinterpret_cast<const f32x4_t*>(part_out + at * D + lane * 4);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k * kAll < count) join(m[k].x, m[k].y, x[k]);
    }
    // the teams of a wave
#pragma unroll
    for (int o = kLanes; o < 64; o <<= 1) {
        const f32x4_t other = {__shfl_xor(y[0], o, 64), __shfl_xor(y[1], o, 64), __shfl_xor(y[2], o, 64), __shfl_xor(y[3], o, 64)};
        const float other_top = __shfl_xor(top, o, 64), other_total = __shfl_xor(total, o, 64);
        join(other_top, other_total, other);
    }
    if constexpr (WAVES > 1) {
        __shared__ float tops[WAVES], sums[WAVES];
        __shared__ f32x4_t part[WAVES][kLanes];
        const int wave = tid >> 6;
        if (team % kTeams == 0) part[wave][lane] = y;
        if ((tid & 63) == 0) {
            tops[wave] = top;
            sums[wave] = total;
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int i = 1; i < WAVES; ++i) join(tops[i], sums[i], part[i][lane]);
    }
    if (team % kTeams) return;
    const float out4[4] = {y[0], y[1], y[2], y[3]};
    paged_store<T, D>(out, lse, to, lane * 4, lane == 0, top, total, out4);
}

}  // namespace swa
