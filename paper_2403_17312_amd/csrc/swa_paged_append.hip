// New rows on their way into a paged cache: norm of queries and keys over each head, rotation by position, and the write into
// the row's slot, in one pass.  Bound by HBM where rows are many (each is read once and written once), by latency at a step.
//
// D / 8 lanes hold one head's row, 8 channels each, so a wave has 64 / (D / 8) heads in hand: the norm's sum is a DPP reduction over those
// lanes, and the other channel of a rotated pair, rot_dim / 2 channels on, is at the same place of another lane (or, for
// neighbouring pairs, in the same lane).  The angles depend on row and channel alone: a lane forms its own sines and cosines once and
// keeps them for all heads of the row.  An angle of a far position has no digits left in fp32 (position 10^6: 0.06), so
// position * inv_freq / 2 pi is an fp64 product, whose whole turns go before it is rounded.
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
    __device__ __forceinline__ void store(char* p) const
    {
#pragma unroll
        for (int i = 0; i < Elem<T>::kBytes / 2; ++i) store16(p + 16 * i, v[i]);
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

template <typename T, int D, bool INT8, bool NEIGHBOURS>
__global__ void __launch_bounds__(kAppendThreads) swa_paged_append_kernel(AppendArgs a)
{
    constexpr int kLanes = D / 8, kHeads = 64 / kLanes;
    const int lane = threadIdx.x & 63, sub = lane % kLanes, mine = lane / kLanes;
    const int64_t wave = (int64_t)blockIdx.x * (kAppendThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row64 = wave >> a.log_parts;
    if (row64 >= a.n_rows) return;
    const int row = (int)row64, part = (int)(wave & ((1 << a.log_parts) - 1));
    const int32_t slot = a.slot[row];
    if (slot < 0) return;
    if (slot >= a.total_slots) {
        if (part == 0 && lane == 0) atomicOr(a.status, kStatusBadRequestBit);
        return;
    }
    const int32_t page = slot / a.page_size, off = slot - page * a.page_size;

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
        if (turns) {
            const int pair = NEIGHBOURS ? 4 * sub + i / 2 : 8 * (sub < half ? sub : sub - half) + i;
            int axis = 0;
#pragma unroll
            for (int x = 0; x + 1 < SWA_MAX_ROPE_AXES; ++x) axis += pair >= a.axis_end[x];
            const double turn = (double)a.pos[(int64_t)axis * a.n_rows + row] * (double)a.inv_freq[pair] * 0.15915494309189533577;
            sincospif(2.f * (float)(turn - __builtin_rint(turn)), &s[i], &c[i]);
            if (NEIGHBOURS || sub < half) s[i] = -s[i];
        }
    }

    const int heads = a.h_q + 2 * a.h_kv;
    for (int h0 = part * kHeads; h0 < heads; h0 += kHeads << a.log_parts) {
        const int head = h0 + mine;
        const bool there = head < heads, is_q = head < a.h_q, is_v = head >= a.h_q + a.h_kv;
        const int kv_head = is_v ? head - a.h_q - a.h_kv : head - a.h_q;
        const char* const src = is_q ? a.q + row * a.q_stride + (int64_t)head * (D * Elem<T>::kBytes)
                                : (is_v ? a.v + row * a.v_stride : a.k + row * a.k_stride) + (int64_t)kv_head * (D * Elem<T>::kBytes);
        Raw8<T> raw{};
        if (there) raw.load(src + 8 * Elem<T>::kBytes * sub);
        float x[8], y[8];
        raw.widen(x);
        const char* const weight = is_v ? nullptr : is_q ? a.q_weight : a.k_weight;
        float square = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) square = __builtin_fmaf(x[i], x[i], square);
        square = group_sum<kLanes>(square);
        const float norm = weight ? 1.f / sqrtf(square * (1.f / D) + a.eps) : 1.f;
        const Raw8<T> raw2 = NEIGHBOURS ? raw : raw.from_lane(mine * kLanes + other);
        raw2.widen(y);
        if (weight) {
            float w[8];
            Raw8<T> rw;
            rw.load(weight + 8 * Elem<T>::kBytes * sub);
            rw.widen(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * norm * w[i];
            if (!NEIGHBOURS) {
                rw.load(weight + 8 * Elem<T>::kBytes * other);
                rw.widen(w);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = y[i] * norm * w[i];
            }
        }
        if (NEIGHBOURS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
        }
        if (turns && !is_v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * c[i] + y[i] * s[i];
        }
        if (!INT8 || is_q) {
            raw.round(x);
            char* const dst = is_q ? a.q_out + ((int64_t)row * a.h_q + head) * (D * Elem<T>::kBytes)
                                   : (is_v ? a.v_pages : a.k_pages) +
                                         (((int64_t)page * a.h_kv + kv_head) * a.page_size + off) * (D * Elem<T>::kBytes);
            if (there) raw.store(dst + 8 * Elem<T>::kBytes * sub);
        }
        if (INT8) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t m = f2u(x[i]) & 0x7fffffffu;
                top = m > top ? m : top;
            }
            // rows below 2^-119 have no scale with a reciprocal in fp32: their codes are 0
            const float scale = u2f(group_max_bits<kLanes>(top)) * (1.f / 127.f);
            const bool tiny = scale < 1.17549435e-38f;
            const float inverse = tiny ? 0.f : 1.f / scale;
            uint32_t codes[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float t = rintf(x[i] * inverse);
                t = t < -127.f ? -127.f : (t > 127.f ? 127.f : t);
                codes[i / 4] |= ((uint32_t)(int32_t)t & 0xffu) << (8 * (i % 4));
            }
            if (there && !is_q) {
                const int64_t r = ((int64_t)page * a.h_kv + kv_head) * a.page_size + off;
                *reinterpret_cast<uint2*>((is_v ? a.v_pages : a.k_pages) + r * D + 8 * sub) = uint2{codes[0], codes[1]};
                if (sub == 0) (is_v ? a.v_scale : a.k_scale)[r] = tiny ? 0.f : scale;
            }
        }
    }
}

template <typename T, int D, bool INT8>
static void launch_append_form(const AppendArgs& a, bool neighbours, dim3 grid, hipStream_t stream)
{
    launch_kernel(neighbours ? swa_paged_append_kernel<T, D, INT8, true> : swa_paged_append_kernel<T, D, INT8, false>, grid, dim3(kAppendThreads), 0,
                  stream, a);
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
    // a row's heads are shared out while that leaves waves to fill the chip with
    const int passes = (p.h_q + 2 * p.h_kv + 64 / (p.d / 8) - 1) / (64 / (p.d / 8));
    while ((2 << a.log_parts) <= passes && ((int64_t)n_rows << a.log_parts) < 4096) ++a.log_parts;
    const int64_t waves = (int64_t)n_rows << a.log_parts;
    const dim3 grid((unsigned)((waves + kAppendThreads / 64 - 1) / (kAppendThreads / 64)));
    const bool neighbours = (p.flags & SWA_ROPE_INTERLEAVED) != 0;
#define SWA_APPEND(T, INT8) \
    (p.d == 64 ? launch_append_form<T, 64, INT8>(a, neighbours, grid, stream) : launch_append_form<T, 128, INT8>(a, neighbours, grid, stream))
    if (p.dtype == SWA_F32) SWA_APPEND(F32, false);
    else if (p.dtype == SWA_F16) paged_int8(p) ? SWA_APPEND(F16, true) : SWA_APPEND(F16, false);
    else paged_int8(p) ? SWA_APPEND(BF16, true) : SWA_APPEND(BF16, false);
#undef SWA_APPEND
    return hipGetLastError() == hipSuccess ? SWA_OK : SWA_ERR_HIP;
}

}  // namespace swa
