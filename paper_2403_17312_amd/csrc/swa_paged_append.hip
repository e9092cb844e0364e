// New rows on their way into a paged cache: norm of queries and keys over each head, rotation by position, and the write into
// the row's slot, in one pass.  Bound by HBM where rows are many (each is read once and written once), by latency at a step.
//
// D / 8 lanes hold one head's row, 8 channels each, so a wave has 64 / (D / 8) heads in hand: the norm's sum is a DPP reduction over those
// lanes, and the other channel of a rotated pair, rot_dim / 2 channels on, is at the same place of another lane (or, for
// neighbouring pairs, in the same lane).  A wave takes one row's queries, keys and values in turn, a wave's heads of one kind at a time, with the
// next ones' loads under way.  The angles depend on row and channel alone: a lane forms its own sines and cosines once for all
// heads of the row, and with the norm's weights makes two factors of them, y = (x_i a_i + x_j b_i) / rms.  An angle of a far position has no
// digits left in fp32 (position 10^6: 0.06), so position * inv_freq / 2 pi is an fp64 product, whose whole turns go before it is rounded.  In 16 bits
// the hardware's sine and cosine of that serve, within 2^-22.9 (all of [-1/2, 1/2], in steps of 2^-24); fp32 rows get better ones.
#include <type_traits>

#include "swa_paged.hpp"

namespace swa {

struct AppendArgs {
    const char *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;          // bytes
    const int32_t *pos, *slot;
    const float* inv_freq;
    const char *q_weight, *k_weight;
    char *q_out, *k_pages, *v_pages;
    float *k_scale, *v_scale;
    int32_t* status;
    int32_t n_rows, h_q, h_kv, page_size, total_slots, rot_dim;
    int32_t axis_end[SWA_MAX_ROPE_AXES];           // first pair behind each axis
    float eps;
    int32_t log_parts;                             // waves that share a row
};

constexpr int kAppendThreads = 256;

// 8 elements of a lane, as loaded.
template <typename T>
struct Raw8 {
    Vec16 v[Elem<T>::kBytes / 2];
    static constexpr int kWords = Elem<T>::kBytes * 2;
    __device__ __forceinline__ void load(const char* p)
    {
#pragma unroll
        for (int i = 0; i < Elem<T>::kBytes / 2; ++i) v[i] = load16(p + 16 * i);
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(char* p) const
    {
#pragma unroll
        for (int i = 0; i < Elem<T>::kBytes / 2; ++i) {
            if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v[i]), reinterpret_cast<u32x4_t*>(p + 16 * i));
            else store16(p + 16 * i, v[i]);
        }
    }
    __device__ __forceinline__ void widen(float* f) const
    {
#pragma unroll
        for (int i = 0; i < Elem<T>::kBytes / 2; ++i) unpack<T>(v[i], f + Elem<T>::kPerVec * i);
    }
    __device__ __forceinline__ void round(const float* f)
    {
#pragma unroll
        for (int i = 0; i < Elem<T>::kBytes / 2; ++i) v[i] = pack<T>(f + Elem<T>::kPerVec * i);
    }
    __device__ __forceinline__ Raw8 from_lane(int lane) const
    {
        Raw8 r;
#pragma unroll
        for (int i = 0; i < Elem<T>::kBytes / 2; ++i) {
            r.v[i].x = (uint32_t)__shfl((int)v[i].x, lane, 64);
            r.v[i].y = (uint32_t)__shfl((int)v[i].y, lane, 64);
            r.v[i].z = (uint32_t)__shfl((int)v[i].z, lane, 64);
            r.v[i].w = (uint32_t)__shfl((int)v[i].w, lane, 64);
        }
        return r;
    }
};

// Largest magnitude over aligned groups of LANES lanes; as bits, so that a value that is not finite stays the largest.
template <int LANES>
__device__ __forceinline__ uint32_t group_max_bits(uint32_t v)
{
    auto other = [](uint32_t x, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true); };
    uint32_t u = other(v, std::integral_constant<int, 0xB1>{});
    v = v > u ? v : u;
    u = other(v, std::integral_constant<int, 0x4E>{});
    v = v > u ? v : u;
    u = other(v, std::integral_constant<int, 0x141>{});
    v = v > u ? v : u;
    if (LANES >= 16) {
        u = other(v, std::integral_constant<int, 0x140>{});
        v = v > u ? v : u;
    }
    return v;
}

// Sine and cosine of an angle in turns.  WIDE: of x quarter turns from the nearest whole one, |x| <= 1/2, by their Taylor series (the first terms left out are below 2^-29 and
// 2^-33).  The hardware's left rotated fp32 rows 1.66 times as far (rms) from the exact ones as sines rounded once do, these 1.11 times: 11.03 -> 11.19 us for 1001 rows of 96 heads.
template <bool WIDE>
__device__ __forceinline__ void sine_cosine(double turn, float& sine, float& cosine)
{
    if constexpr (WIDE) {
        const double quarters = 4.0 * (turn - __builtin_rint(turn)), whole = __builtin_rint(quarters);
        const float x = (float)(quarters - whole), y = x * x;
        const int at = (int)whole;                   // -2 .. 2
        const float s = x * __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, 1.6044118e-4f, -4.6817541e-3f), 7.9692626e-2f), -0.64596410f), 1.5707963f);
        const float c = __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, -2.5202042e-5f, 9.1926027e-4f), -2.0863481e-2f), 0.25366951f), -1.2337006f), 1.f);
        sine = at & 1 ? c : s;
        cosine = at & 1 ? s : c;
        sine = at & 2 ? -sine : sine;
        cosine = (at + 1) & 2 ? -cosine : cosine;
    } else {
        const float rest = (float)(turn - __builtin_rint(turn));
        sine = __builtin_amdgcn_sinf(rest);
        cosine = __builtin_amdgcn_cosf(rest);
    }
}

// x / by rounded correctly, from by's reciprocal: a product, and two steps that take the remainder, exact in an FMA, into account (the first makes the quotient one of the two
// neighbours, the second the nearer one).  A product alone gave another code where a quotient lies half way between two.
__device__ __forceinline__ float quotient(float x, float by, float inverse)
{
    float q = x * inverse;
    q = __builtin_fmaf(__builtin_fmaf(-q, by, x), inverse, q);
    return __builtin_fmaf(__builtin_fmaf(-q, by, x), inverse, q);
}

// A lane's channels of the heads of one pass.
template <typename T, int D>
__device__ __forceinline__ void fetch_heads(Raw8<T>& raw, const AppendArgs& a, int row, int pass, int q_passes, int kv_passes, int mine, int sub)
{
    constexpr int kHeads = 512 / D;
    const char* from = a.q + row * a.q_stride;
    int first = 0, heads = a.h_q;
    if (pass >= q_passes) {
        from = a.k + row * a.k_stride;
        first = q_passes;
        heads = a.h_kv;
    }
    if (pass >= q_passes + kv_passes) {
        from = a.v + row * a.v_stride;
        first = q_passes + kv_passes;
    }
    const int head = (pass - first) * kHeads + mine;
    raw = Raw8<T>{};
    if (head < heads) raw.load(from + (uint32_t)((head * D + 8 * sub) * Elem<T>::kBytes));
}

// STREAM: rows are stored past the caches.
template <typename T, int D, bool INT8, bool NEIGHBOURS, bool STREAM>
__global__ void __launch_bounds__(kAppendThreads) swa_paged_append_kernel(AppendArgs a)
{
    constexpr int kLanes = D / 8, kHeads = 64 / kLanes, kRow = D * Elem<T>::kBytes, kLane = 8 * Elem<T>::kBytes;
    const int lane = threadIdx.x & 63, sub = lane % kLanes, mine = lane / kLanes;
    const int64_t wave = (int64_t)blockIdx.x * (kAppendThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row64 = wave >> a.log_parts;
    if (row64 >= a.n_rows) return;
    const int row = (int)row64, part = (int)(wave & ((1 << a.log_parts) - 1));

    // Passes: kHeads queries each, then kHeads keys, then values.
    const int q_passes = (a.h_q + kHeads - 1) / kHeads, kv_passes = (a.h_kv + kHeads - 1) / kHeads, passes = q_passes + 2 * kv_passes;
    if (part >= passes) return;
    Raw8<T> next;
    fetch_heads<T, D>(next, a, row, part, q_passes, kv_passes, mine, sub);
    const int32_t slot = a.slot[row];
    if (slot < 0) return;
    if (slot >= a.total_slots) {
        if (part == 0 && lane == 0) atomicOr(a.status, kStatusBadRequestBit);
        return;
    }
    const int32_t page = slot / a.page_size, off = slot - page * a.page_size;
    const int64_t kv_row = (int64_t)page * a.h_kv * a.page_size + off;      // of key head 0

    // this lane's channels 8 sub .. 8 sub + 7: x <- x c + other s
    const int half = a.rot_dim / 16;               // lanes of half the rotated channels
    const bool turns = sub < 2 * half;
    const int other = NEIGHBOURS || !turns ? sub : (sub < half ? sub + half : sub - half);
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (NEIGHBOURS && (i & 1)) {
            c[i] = c[i - 1];
            s[i] = -s[i - 1];
            continue;
        }
        c[i] = 1.f;
        s[i] = 0.f;
        if (turns && part < q_passes + kv_passes) {
            const int pair = NEIGHBOURS ? 4 * sub + i / 2 : 8 * (sub < half ? sub : sub - half) + i;
            int axis = 0;
#pragma unroll
            for (int x = 0; x + 1 < SWA_MAX_ROPE_AXES; ++x) axis += pair >= a.axis_end[x];
            sine_cosine<std::is_same_v<T, F32>>((double)a.pos[(int64_t)axis * a.n_rows + row] * (double)a.inv_freq[pair] * 0.15915494309189533577, s[i], c[i]);
            if (NEIGHBOURS || sub < half) s[i] = -s[i];
        }
    }

    float own[8], cross[8];                        // what a channel and the other one of its pair are multiplied by, weights included
    int weighed = -1;                              // for queries (0) or keys (1)
    for (int pass = part; pass < passes; pass += 1 << a.log_parts) {
        Raw8<T> raw = next;
        if (pass + (1 << a.log_parts) < passes) fetch_heads<T, D>(next, a, row, pass + (1 << a.log_parts), q_passes, kv_passes, mine, sub);
        const bool is_q = pass < q_passes, is_v = pass >= q_passes + kv_passes;
        const int head = (pass - (is_v ? q_passes + kv_passes : is_q ? 0 : q_passes)) * kHeads + mine;
        const bool there = head < (is_q ? a.h_q : a.h_kv);
        const int64_t to_row = is_q ? (int64_t)row * a.h_q + head : kv_row + (int64_t)head * a.page_size;
        if (is_v && !INT8) {
            if (there) raw.template store<STREAM>(a.v_pages + to_row * kRow + sub * kLane);
            continue;
        }
        float x[8];
        raw.widen(x);
        if (!is_v) {
            const char* const weight = is_q ? a.q_weight : a.k_weight;
            if (weighed != (is_q ? 0 : 1)) {
                weighed = is_q ? 0 : 1;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    own[i] = c[i];
                    cross[i] = s[i];
                }
                if (weight) {
                    Raw8<T> w, w_other;
                    w.load(weight + sub * kLane);
                    w_other.load(weight + other * kLane);
                    float f[8], g[8];
                    w.widen(f);
                    w_other.widen(g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        own[i] *= f[i];
                        cross[i] *= g[NEIGHBOURS ? i ^ 1 : i];
                    }
                }
            }
            float norm = 1.f;
            if (weight) {
                float square = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) square = __builtin_fmaf(x[i], x[i], square);
                const float mean = group_sum<kLanes>(square) * (1.f / D) + a.eps;
                // (the root's instruction takes what lies below fp32's normal numbers for 0, and without an eps such a row would be infinite)
                const int up = mean < 0x1p-100f ? 32 : 0;
                norm = __builtin_amdgcn_ldexpf(__builtin_amdgcn_rsqf(__builtin_amdgcn_ldexpf(mean, 2 * up)), up);
            }
            float y[8], z[8];
            if (!NEIGHBOURS) raw.from_lane(mine * kLanes + other).widen(y);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = x[i] * own[i];
                z[i] = (turns ? __builtin_fmaf(NEIGHBOURS ? x[i ^ 1] : y[i], cross[i], t) : t) * norm;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = z[i];
        }
        if (!INT8 || is_q) {
            raw.round(x);
            if (there) raw.template store<STREAM>((is_q ? a.q_out : a.k_pages) + to_row * kRow + sub * kLane);
            continue;
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t m = f2u(x[i]) & 0x7fffffffu;
            top = m > top ? m : top;
        }
        // (rows below 2^-119 have no scale with a reciprocal in fp32: their codes are 0)
        top = group_max_bits<kLanes>(top);
        const float scale = quotient(u2f(top < 0x7f800000u ? top : 0x7fc00000u), 127.f, 1.f / 127.f);
        const bool tiny = scale < 1.17549435e-38f;
        float inverse = __builtin_amdgcn_rcpf(scale);
        inverse = tiny ? 0.f : __builtin_fmaf(__builtin_fmaf(-scale, inverse, 1.f), inverse, inverse);
        uint32_t codes[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = fminf(fmaxf(rintf(quotient(x[i], scale, inverse)), -127.f), 127.f);
            codes[i / 4] |= ((uint32_t)(int32_t)t & 0xffu) << (8 * (i % 4));
        }
        if (there) {
            *reinterpret_cast<uint2*>((is_v ? a.v_pages : a.k_pages) + to_row * D + 8 * sub) = uint2{codes[0], codes[1]};
            if (sub == 0) (is_v ? a.v_scale : a.k_scale)[to_row] = tiny ? 0.f : scale;
        }
    }
}

template <typename T, int D, bool INT8>
static void launch_append_form(const AppendArgs& a, bool neighbours, bool past, dim3 grid, hipStream_t stream)
{
    auto kernel = neighbours ? (past ? swa_paged_append_kernel<T, D, INT8, true, true> : swa_paged_append_kernel<T, D, INT8, true, false>)
                             : (past ? swa_paged_append_kernel<T, D, INT8, false, true> : swa_paged_append_kernel<T, D, INT8, false, false>);
    launch_kernel(kernel, grid, dim3(kAppendThreads), 0, stream, a);
}

// Waves that share a row's passes, as a power of two.  A wave has one pass's loads under way, so that few waves do not fill the chip; but each begins with the
// angles of the row, which its passes have to outweigh.  So they are halved below a number of waves that grows with the passes left to each.
// us with 1 / 2 / 4 / 8 waves a row: 32 query and 8 key heads of 128 bf16 channels (12 passes), 400 rows 10.0 / 7.1 / 5.9 / 7.1, 512 10.4 / 7.5 / 6.5 / 7.5, 1024 11.2 / 8.9 / 8.9, 2048 12.9 /
// 12.2, 3000 15.4 / 16.4; 28 and 4 heads (9 passes), 400 8.6 / 6.5 / 5.5 / 5.9, 2048 11.1 / 10.3, 3000 12.8 / 13.6; 64 and 8 heads (20 passes), 1024 15.7 / 11.6 / 11.1,
// 1800 17.9 / 15.8, 5000 45.0 / 50.0.  fp32 has twice the bytes under way: 12 passes, 900 12.9 / 11.1 / 12.0, 1800 19.6 / 19.4.
// Beyond that the chip is full, and what counts is how full the last waves leave it, whose time is that of a row.  Where rows are long and those waves are a third of
// it or less, two waves a row end sooner (of four rounds a few per cent at most: then no more): codes (7168 waves at once) of 20 passes, 7000 rows 61.7 / 62.5, 7300 73.7 / 69.5, 8100 80.2 / 73.9, 9000 84.7 / 79.4, 12000
// 102.7 / 102.4, 14500 127.1 / 122.0; 16 bits (8192), 16 passes, 8100 59.3 / 59.0, 8400 69.1 / 64.9, 9000 73.3 / 68.3, 12000 84.6 / 84.4; of 12 passes 10000 rows 58.9 / 56.9,
// but 16000 83.4 / 85.3 as codes.  Long rows in fp32 gain at any count: 20 passes, 3000 rows 58.2 / 57.5, 6000 115 / 109, 8000 155 / 142.
int paged_append_log_parts(bool wide, bool codes, int passes, int64_t n_rows)
{
    const int64_t at_once = wide || codes ? 7168 : 8192;     // by the kernels' registers
    auto more = [&](int64_t waves, int each) {
        const int64_t few = 1024 + (wide ? 64 : 128) * (int64_t)each, last = waves % at_once;
        if (waves < (few < at_once / 2 ? few : at_once / 2)) return true;
        return each >= 16 && waves <= 4 * at_once && (wide || (waves > at_once && last > 0 && last <= at_once / 3));
    };
    int log_parts = 0;
    while ((1 << log_parts) < passes && more(n_rows << log_parts, passes >> log_parts)) ++log_parts;
    return log_parts;
}

int launch_paged_append(const swa_paged_params& p, const swa_rows& q, const swa_rows& k, const swa_rows& v, int32_t n_rows, const int32_t* pos,
                        const int32_t* slot, const float* inv_freq, const void* q_weight, const void* k_weight, void* q_out, void* k_pages,
                        void* v_pages, float* k_scale, float* v_scale, void* workspace, hipStream_t stream)
{
    const int bytes = p.dtype == SWA_F32 ? 4 : 2;
    AppendArgs a{};
    a.q = static_cast<const char*>(q.data);
    a.k = static_cast<const char*>(k.data);
    a.v = static_cast<const char*>(v.data);
    a.q_stride = q.stride * bytes;
    a.k_stride = k.stride * bytes;
    a.v_stride = v.stride * bytes;
    a.pos = pos;
    a.slot = slot;
    a.inv_freq = inv_freq;
    a.q_weight = static_cast<const char*>(q_weight);
    a.k_weight = static_cast<const char*>(k_weight);
    a.q_out = static_cast<char*>(q_out);
    a.k_pages = static_cast<char*>(k_pages);
    a.v_pages = static_cast<char*>(v_pages);
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.status = paged_status(workspace);
    a.n_rows = n_rows;
    a.h_q = p.h_q;
    a.h_kv = p.h_kv;
    a.page_size = p.page_size;
    a.total_slots = p.n_pages * p.page_size;
    a.rot_dim = p.rot_dim;
    int32_t end = 0;
    for (int i = 0; i < SWA_MAX_ROPE_AXES; ++i) {
        if (i < p.axes) end += p.section[i];
        a.axis_end[i] = i + 1 < p.axes ? end : INT32_MAX;
    }
    a.eps = p.eps;
    const int of_wave = 64 / (p.d / 8), passes = (p.h_q + of_wave - 1) / of_wave + 2 * ((p.h_kv + of_wave - 1) / of_wave);
    a.log_parts = paged_append_log_parts(p.dtype == SWA_F32, paged_int8(p), passes, n_rows);
    // Many rows fill the caches with what nothing reads soon: 4096 rows as above 26.6 us stored through them, 19.3 past them; 8192 rows 49.5, 44.5 (4.5
    // TB/s); 256 rows and the attention behind them 47.1, 45.7.  Of few, the attention finds queries and keys there: 1 row and 100 tokens 8.7, 9.0.
    const bool past = (int64_t)n_rows * (p.h_q + 2 * p.h_kv) * p.d * bytes >= (2 << 20);
    const int64_t waves = (int64_t)n_rows << a.log_parts;
    const dim3 grid((unsigned)((waves + kAppendThreads / 64 - 1) / (kAppendThreads / 64)));
    const bool neighbours = (p.flags & SWA_ROPE_INTERLEAVED) != 0;
#define SWA_APPEND(T, INT8) \
    (p.d == 64 ? launch_append_form<T, 64, INT8>(a, neighbours, past, grid, stream) : launch_append_form<T, 128, INT8>(a, neighbours, past, grid, stream))
    if (p.dtype == SWA_F32) SWA_APPEND(F32, false);
    else if (p.dtype == SWA_F16) paged_int8(p) ? SWA_APPEND(F16, true) : SWA_APPEND(F16, false);
    else paged_int8(p) ? SWA_APPEND(BF16, true) : SWA_APPEND(BF16, false);
#undef SWA_APPEND
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
