// Rotary position encoding by positions on several axes, and the write of K and V into the cache, in one pass over the rows:
//   (x, y) -> scale * (x cos a - y sin a, y cos a + x sin a), a = positions[axis_of[i]] * inv_freq[i] for channel pair i
// Floor: q, k and v once in and once out; two images of 8192 tokens in bf16 are 373.6 MB, 72.3 us at a copy's rate, and take 71.7 us.
#include "etv_common.h"
#include <type_traits>

namespace etv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct RotaryPtrs {
    const void *q, *k, *v;
    void *q_out, *k_out, *v_out, *k_cache, *v_cache;
};

// Sine and cosine of pos * f.  The product has up to 55 bits, in two parts; so is 2 / pi.  The quarter turns are split off within a fused multiply-add, the
// low parts added, and what is left, at most half a quarter, goes to the fp32 functions: its rounding is 2^-26 of a quarter turn.  (Without the low parts an
// angle near 2^31 is off by up to 7 * 2^-24.)
__device__ __forceinline__ float2 turn_of(int pos, float f, float scale, bool inverse) {
    constexpr double kQuarter = 0.6366197723675814, kQuarterLow = -3.935735335036497e-17;  // 2 / pi
    const double angle = (double)pos * (double)f, rest = fma((double)pos, (double)f, -angle);
    const double whole = rint(angle * kQuarter);
    const double part = fma(angle, kQuarter, -whole) + fma(angle, kQuarterLow, rest * kQuarter);
    float s, c;
    sincospif(0.5f * (float)part, &s, &c);
    const int n = (int)(long)(whole - 4.0 * floor(0.25 * whole));
    float cs = (n & 1) ? -s : c, sn = (n & 1) ? c : s;
    if (n & 2) cs = -cs, sn = -sn;
    if (inverse) sn = -sn;
    return make_float2(cs * scale, sn * scale);
}

template <class T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int N = 4;
    static __device__ void load(const u32x4 &u, float *x) {
        for (int i = 0; i < 4; i++) x[i] = __uint_as_float(u[i]);
    }
    static __device__ u32x4 store(const float *x) {
        u32x4 u;
        for (int i = 0; i < 4; i++) u[i] = __float_as_uint(x[i]);
        return u;
    }
};
template <>
struct Vec<uint16_t> {
    static constexpr int N = 8;
    static __device__ void load(const u32x4 &u, float *x) {
        for (int i = 0; i < 4; i++) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    static __device__ u32x4 store(const float *x) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        u32x4 u;
        for (int i = 0; i < 4; i++) u[i] = __builtin_bit_cast(unsigned int, __builtin_convertvector((f2){x[2 * i], x[2 * i + 1]}, b2));
        return u;
    }
};

// One token a workgroup, or as many as its 256 threads take at once: a token of 24 heads of 64 channels occupies 96 of them.  A thread has the same
// place in every head it comes to -- two 16-byte vectors, both members of a channel pair among them -- so
// that its sines and cosines, worked out once for the token and passed around by LDS, stay in its registers.  What bounds it is memory,
// and for few tokens the chain of loads: what the arguments alone say the place of is asked for before the angles are worked out, the first
// head's vectors among it, and every further head's before the one before it is finished.  8 tokens take 4.4 us; 32 trees of 60
// nodes, 41.3 MB, 9.2 us where the bytes take 8.0.
template <class T, bool INTER, bool MANY, bool ROWS_FIRST>
__global__ void __launch_bounds__(256) rotary_kernel(etv_rotary_desc dsc, RotaryPtrs p, const int32_t *positions, const float *inv_freq,
                                                     const int32_t *n_rows, const int32_t *slot_map, int tokens_a_wg, int lanes, uint32_t inv_T, uint32_t inv_upr,
                                                     uint32_t inv_lanes, uint32_t inv_half, uint32_t inv_bs) {
    constexpr int N = Vec<T>::N;
    extern __shared__ float2 s_turn[];  // [tokens][half]
    const int half = dsc.rot_dim / 2, upr = dsc.d / (2 * N), turning = half / N;
    uint32_t row, u32, lane;
    // `lanes` threads a token
    const int tokens = MANY ? tokens_a_wg : 1;
    const uint32_t mine = MANY ? fast_div(threadIdx.x, lanes, inv_lanes, lane) : 0;
    const int t = MANY ? lane : threadIdx.x;
    const uint32_t first_token = blockIdx.x * tokens, all = (uint32_t)dsc.B * dsc.T, token = MANY ? min(first_token + mine, all - 1) : first_token;
    const uint32_t b = fast_div(token, dsc.T, inv_T, row);
    const int first = (int)fast_div(t, upr, inv_upr, u32), u = (int)u32, step = (int)fast_div(MANY ? lanes : 256, upr, inv_upr, u32);
    const bool turns = u < turning;
    const int at = !turns ? dsc.rot_dim + (u - turning) * 2 * N : (INTER ? 2 : 1) * u * N, gap = turns && !INTER ? half : N;
    // heads of q, then of k, then of v; the remainder of the 256 threads has none
    const int heads = first < step && (!MANY || ((int)mine < tokens && first_token + mine < all)) ? dsc.Hq + dsc.Hkv + (p.v ? dsc.Hkv : 0) : 0;
    const auto rows_of = [&](const void *base, int i) { return static_cast<const T *>(base) + b * dsc.strides[2 * i] + row * dsc.strides[2 * i + 1]; };
    const T *src[3] = {rows_of(p.q, 0), rows_of(p.k, 1), rows_of(p.v, 2)};
    const auto pick = [&](int head, const auto &q, const auto &k, const auto &v, int &h) {
        const bool not_q = head >= dsc.Hq, is_v = head >= dsc.Hq + dsc.Hkv;
        h = head - (not_q ? dsc.Hq : 0) - (is_v ? dsc.Hkv : 0);
        return is_v ? v : not_q ? k : q;
    };
    const auto load = [&](int head, u32x4 &ra, u32x4 &rb) {
        int h;
        const T *from = pick(head, +src[0], +src[1], +src[2], h) + h * dsc.d + at;
        ra = *reinterpret_cast<const u32x4 *>(from);
        rb = *reinterpret_cast<const u32x4 *>(from + gap);
    };
    u32x4 ra = {}, rb = {};
    int rows = dsc.T;
    if (ROWS_FIRST) {
        rows = n_rows[b];
        if (!MANY && (int)row >= rows) return;
    }
    if (first < heads && (!ROWS_FIRST || (int)row < rows)) load(first, ra, rb);
    if (!ROWS_FIRST && n_rows) rows = n_rows[b];
    long slot = slot_map ? slot_map[token] : -1;
    const auto turn_at = [&](int i, uint32_t pair, uint32_t of) {
        s_turn[i] = turn_of(positions[(size_t)dsc.axis_of[pair] * all + of], inv_freq[pair], dsc.scale, dsc.flags & ETV_ROTARY_INVERSE);
    };
    if (MANY) {
        for (int i = threadIdx.x; i < tokens * half; i += 256) {
            uint32_t pair;
            const uint32_t of = fast_div(i, half, inv_half, pair);
            turn_at(i, pair, min(first_token + of, all - 1));
        }
    } else if (t < half) {
        turn_at(t, t, token);
    }
    __syncthreads();
    if ((int)row >= rows) return;
    if (slot >= dsc.cache_rows) slot = -1;
    uint32_t off = 0;
    const uint32_t block = slot >= 0 && dsc.block_size > 0 ? fast_div((uint32_t)slot, dsc.block_size, inv_bs, off) : 0;
    // where head 0 of the slot lies, and how far apart heads are
    const long cache_at = (dsc.block_size ? (long)block * dsc.Hkv * dsc.block_size + off : slot * dsc.Hkv) * dsc.d + at;
    const long cache_head = (long)(dsc.block_size ? dsc.block_size : 1) * dsc.d;
    T *out[3] = {const_cast<T *>(rows_of(p.q_out, 3)), const_cast<T *>(rows_of(p.k_out, 4)), const_cast<T *>(rows_of(p.v_out, 5))};
    float2 turn[N];
#pragma unroll
    for (int j = 0; j < N; j++) turn[j] = turns ? s_turn[(heads ? mine * half : 0) + u * N + j] : make_float2(1, 0);
    for (int head = first; head < heads; head += step) {
        u32x4 na = {}, nb = {};
        if (head + step < heads) load(head + step, na, nb);
        int h;
        const int which = pick(head, 0, 1, 2, h);
        if (turns && which < 2) {
            float xa[N], xb[N];
            Vec<T>::load(ra, xa);
            Vec<T>::load(rb, xb);
            const auto rotate = [](float &x, float &y, const float2 &c) {
                const float was = x;
                x = was * c.x - y * c.y;
                y = y * c.x + was * c.y;
            };
#pragma unroll
            for (int j = 0; j < N; j++) {
                if (!INTER) rotate(xa[j], xb[j], turn[j]);
                else if (j < N / 2) rotate(xa[2 * j], xa[2 * j + 1], turn[j]);
                else rotate(xb[2 * j - N], xb[2 * j - N + 1], turn[j]);
            }
            ra = Vec<T>::store(xa);
            rb = Vec<T>::store(xb);
        }
        if (pick(head, p.q_out, p.k_out, p.v_out, h)) {
            T *to = pick(head, +out[0], +out[1], +out[2], h) + h * dsc.d + at;
            *reinterpret_cast<u32x4 *>(to) = ra;
            *reinterpret_cast<u32x4 *>(to + gap) = rb;
        }
        if (slot >= 0 && which > 0) {
            T *to = static_cast<T *>(which == 1 ? p.k_cache : p.v_cache) + cache_at + h * cache_head;
            *reinterpret_cast<u32x4 *>(to) = ra;
            *reinterpret_cast<u32x4 *>(to + gap) = rb;
        }
        ra = na, rb = nb;
    }
}

}  // namespace etv

extern "C" int32_t etv_rotary_write_kv(const etv_rotary_desc *h, const void *q, const void *k, const void *v, const int32_t *positions,
                                       const float *inv_freq, const int32_t *n_rows, void *q_out, void *k_out, void *v_out, const int32_t *slot_map,
                                       void *k_cache, void *v_cache, void *stream) {
    if (!h || h->B < 0 || h->T < 1 || h->Hq < 0 || h->Hkv < 0 || h->Hq + h->Hkv < 1 || h->n_axes < 1 || h->block_size < 0) return ETV_ERR_INVALID_ARG;
    if (h->flags & ~(ETV_ROTARY_INTERLEAVED | ETV_ROTARY_INVERSE) || !(h->scale - h->scale == 0)) return ETV_ERR_INVALID_ARG;
    if (h->dtype != ETV_F32 && h->dtype != ETV_BF16) return ETV_ERR_UNSUPPORTED;
    if (h->d < 16 || h->d > 256 || h->d % 16 || h->rot_dim < 16 || h->rot_dim > h->d || h->rot_dim % 16) return ETV_ERR_UNSUPPORTED;
    if ((int64_t)h->B * h->T >= (1 << 24) || h->Hq > (1 << 16) || h->Hkv > (1 << 16)) return ETV_ERR_UNSUPPORTED;  // a launch has less than 2^32 threads
    for (int i = 0; i < h->rot_dim / 2; i++)
        if (h->axis_of[i] >= h->n_axes) return ETV_ERR_INVALID_ARG;
    if (h->B == 0) return ETV_OK;
    if ((h->Hq > 0) != (q != nullptr) || (h->Hq > 0) != (q_out != nullptr) || (h->Hkv > 0) != (k != nullptr) || (v && !k)) return ETV_ERR_INVALID_ARG;
    if ((k_out && !k) || (v_out && !v)) return ETV_ERR_INVALID_ARG;
    if ((slot_map != nullptr) != (k_cache != nullptr) || (slot_map != nullptr) != (v_cache != nullptr) || (slot_map && (!k || !v || h->cache_rows < 0)))
        return ETV_ERR_INVALID_ARG;
    if (k && !k_out && !k_cache) return ETV_ERR_INVALID_ARG;  // k would go nowhere
    etv_rotary_desc d = *h;
    if (d.scale == 0) d.scale = 1;
    const void *ends[8] = {q, k, v, q_out, k_out, v_out, k_cache, v_cache};
    for (int i = 0; i < 8; i++) {
        if ((uintptr_t)ends[i] & 15) return ETV_ERR_INVALID_ARG;
        if (i >= 6 || !ends[i]) continue;
        int64_t &seq = d.strides[2 * i], &tok = d.strides[2 * i + 1];
        if (d.B == 1) seq = 0;  // of one sequence, of one token: not used
        if (d.T == 1) tok = 0;
        const int64_t unit = d.dtype == ETV_BF16 ? 8 : 4, row = (int64_t)(i % 3 ? d.Hkv : d.Hq) * d.d;
        if (seq % unit || tok % unit || seq < 0 || tok < 0) return ETV_ERR_INVALID_ARG;
        if (i < 3) continue;
        // an output that is its input moves nothing; no two rows of an output lie on one another
        if (ends[i] == ends[i - 3] && (seq != d.strides[2 * i - 6] || tok != d.strides[2 * i - 5])) return ETV_ERR_INVALID_ARG;
        if ((d.B > 1 && seq < row) || (d.T > 1 && tok < row)) return ETV_ERR_INVALID_ARG;
        if (d.B > 1 && d.T > 1 && seq < (d.T - 1) * tok + row && tok < (d.B - 1) * seq + row) return ETV_ERR_INVALID_ARG;
    }
    if (!positions || !inv_freq) return ETV_ERR_INVALID_ARG;
    const etv::RotaryPtrs p{q, k, v, q_out, k_out, v_out, k_cache, v_cache};
    const bool inter = d.flags & ETV_ROTARY_INTERLEAVED;
    // threads of one token that have a head at once, and tokens a workgroup takes with that
    const int upr = d.d * (d.dtype == ETV_BF16 ? 2 : 4) / 32, units = upr * (d.Hq + d.Hkv + (v ? d.Hkv : 0)), half = d.rot_dim / 2;
    const int tokens = units < 256 ? 256 / units : 1, lanes = tokens > 1 ? units : 256 / upr * upr;
    const int wgs = (d.B * d.T + tokens - 1) / tokens;
    // padding is left unread where other workgroups hide the wait for n_rows: 25 trees of up to 943 rows 55.5 -> 52.9 us
    const bool rows_first = n_rows && wgs >= 2048;
    const auto choose = [&](auto type, auto inter, auto many) {
        using T = decltype(type);
        return rows_first ? etv::rotary_kernel<T, inter, many, true> : etv::rotary_kernel<T, inter, many, false>;
    };
    const auto variant = [&](auto type, auto inter) { return tokens > 1 ? choose(type, inter, std::true_type{}) : choose(type, inter, std::false_type{}); };
    const auto of_type = [&](auto type) { return inter ? variant(type, std::true_type{}) : variant(type, std::false_type{}); };
    const auto kernel = d.dtype == ETV_BF16 ? of_type(uint16_t{}) : of_type(float{});
    hipLaunchKernelGGL(kernel, dim3(wgs), dim3(256), (size_t)tokens * half * sizeof(float2), etv::as_stream(stream),
                       d, p, positions, inv_freq, n_rows, slot_map, tokens, lanes, etv::fast_div_inv(d.T), etv::fast_div_inv(upr), etv::fast_div_inv(lanes),
                       etv::fast_div_inv(half), d.block_size ? etv::fast_div_inv(d.block_size) : 0);
    return etv::check_launch();
}
