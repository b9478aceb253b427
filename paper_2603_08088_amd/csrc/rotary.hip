// Rotary position encoding by positions on several axes, and the write of K and V into the cache, in one pass over the rows.
#include "etv_common.h"

namespace etv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct RotaryPtrs {
    const void *q, *k, *v;
    void *q_out, *k_out, *v_out, *k_cache, *v_cache;
};

// Sine and cosine of pos * f.  The product has 55 bits of which 53 are kept, the quarter turns are split off in 64 bits, and what is left, at most
// half a quarter, goes to the fp32 functions: its rounding is 2^-26 of a quarter turn.
__device__ __forceinline__ float2 turn_of(int pos, float f, float scale, bool inverse) {
    const double quarters = (double)pos * (double)f * 0.63661977236758134308;  // 2 / pi
    const double whole = rint(quarters);
    float s, c;
    sincospif(0.5f * (float)(quarters - whole), &s, &c);
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
        u32x4 u;
        for (int i = 0; i < 4; i++) u[i] = float_to_bf16_bits(x[2 * i]) | (uint32_t)float_to_bf16_bits(x[2 * i + 1]) << 16;
        return u;
    }
};

// One token a workgroup: its sines and cosines once, in LDS, for all heads; then 16-byte vectors in pairs, both members of a channel pair with one lane.
template <class T>
__global__ void __launch_bounds__(256) rotary_kernel(etv_rotary_desc dsc, RotaryPtrs p, const int32_t *positions, const float *inv_freq,
                                                     const int32_t *n_rows, const int32_t *slot_map, uint32_t inv_T) {
    constexpr int N = Vec<T>::N;
    __shared__ float2 s_turn[128];
    const int t = threadIdx.x, half = dsc.rot_dim / 2;
    uint32_t row;
    const uint32_t b = fast_div(blockIdx.x, dsc.T, inv_T, row);
    if (n_rows && (int)row >= n_rows[b]) return;
    for (int i = t; i < half; i += 256)
        s_turn[i] = turn_of(positions[((size_t)dsc.axis_of[i] * dsc.B + b) * dsc.T + row], inv_freq[i], dsc.scale, dsc.flags & ETV_ROTARY_INVERSE);
    __syncthreads();
    long slot = slot_map ? slot_map[blockIdx.x] : -1;
    if (slot >= dsc.cache_rows) slot = -1;
    const int upr = dsc.d / (2 * N), turning = half / N, units = (dsc.Hq + 2 * dsc.Hkv) * upr;
    for (int x = t; x < units; x += 256) {
        const int head = x / upr, u = x - head * upr;
        const int which = head < dsc.Hq ? 0 : head < dsc.Hq + dsc.Hkv ? 1 : 2;
        const int h = head - (which == 0 ? 0 : which == 1 ? dsc.Hq : dsc.Hq + dsc.Hkv);
        const T *src = static_cast<const T *>(which == 0 ? p.q : which == 1 ? p.k : p.v);
        T *out = static_cast<T *>(which == 0 ? p.q_out : which == 1 ? p.k_out : p.v_out);
        T *cache = static_cast<T *>(which == 0 ? nullptr : which == 1 ? p.k_cache : p.v_cache);
        if (!src) continue;
        const int at = dsc.flags & ETV_ROTARY_INTERLEAVED || u >= turning ? (u < turning ? 2 * u * N : dsc.rot_dim + (u - turning) * 2 * N) : u * N;
        const int gap = dsc.flags & ETV_ROTARY_INTERLEAVED || u >= turning ? N : half;
        src += b * dsc.strides[2 * which] + row * dsc.strides[2 * which + 1] + h * dsc.d + at;
        u32x4 ra = *reinterpret_cast<const u32x4 *>(src), rb = *reinterpret_cast<const u32x4 *>(src + gap);
        if (which < 2 && u < turning) {
            float xa[N], xb[N];
            Vec<T>::load(ra, xa);
            Vec<T>::load(rb, xb);
            if (dsc.flags & ETV_ROTARY_INTERLEAVED) {
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    const float2 ca = s_turn[u * N + j / 2], cb = s_turn[u * N + N / 2 + j / 2];
                    const float a0 = xa[j], b0 = xb[j];
                    xa[j] = a0 * ca.x - xa[j + 1] * ca.y;
                    xa[j + 1] = xa[j + 1] * ca.x + a0 * ca.y;
                    xb[j] = b0 * cb.x - xb[j + 1] * cb.y;
                    xb[j + 1] = xb[j + 1] * cb.x + b0 * cb.y;
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const float2 c = s_turn[u * N + j];
                    const float a0 = xa[j];
                    xa[j] = a0 * c.x - xb[j] * c.y;
                    xb[j] = xb[j] * c.x + a0 * c.y;
                }
            }
            ra = Vec<T>::store(xa);
            rb = Vec<T>::store(xb);
        }
        if (out) {
            out += b * dsc.strides[6 + 2 * which] + row * dsc.strides[7 + 2 * which] + h * dsc.d + at;
            *reinterpret_cast<u32x4 *>(out) = ra;
            *reinterpret_cast<u32x4 *>(out + gap) = rb;
        }
        if (cache && slot >= 0) {
            const long bs = dsc.block_size;
            cache += (bs ? ((slot / bs * dsc.Hkv + h) * bs + slot % bs) : slot * dsc.Hkv + h) * dsc.d + at;
            *reinterpret_cast<u32x4 *>(cache) = ra;
            *reinterpret_cast<u32x4 *>(cache + gap) = rb;
        }
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
    if ((int64_t)h->B * h->T > INT32_MAX || h->Hq > (1 << 16) || h->Hkv > (1 << 16)) return ETV_ERR_UNSUPPORTED;
    for (int i = 0; i < h->rot_dim / 2; i++)
        if (h->axis_of[i] >= h->n_axes) return ETV_ERR_INVALID_ARG;
    if (h->B == 0) return ETV_OK;
    if ((h->Hq > 0) != (q != nullptr) || (h->Hq > 0) != (q_out != nullptr) || (h->Hkv > 0) != (k != nullptr) || (v && !k)) return ETV_ERR_INVALID_ARG;
    if ((k_out && !k) || (v_out && !v)) return ETV_ERR_INVALID_ARG;
    if ((slot_map != nullptr) != (k_cache != nullptr) || (slot_map != nullptr) != (v_cache != nullptr) || (slot_map && (!k || !v || h->cache_rows < 0)))
        return ETV_ERR_INVALID_ARG;
    if (k && !k_out && !k_cache) return ETV_ERR_INVALID_ARG;  // k would go nowhere
    const void *ends[8] = {q, k, v, q_out, k_out, v_out, k_cache, v_cache};
    for (int i = 0; i < 8; i++) {
        if ((uintptr_t)ends[i] & 15) return ETV_ERR_INVALID_ARG;
        if (i >= 6 || !ends[i]) continue;
        const int64_t unit = h->dtype == ETV_BF16 ? 8 : 4;
        if (h->strides[2 * i] % unit || h->strides[2 * i + 1] % unit) return ETV_ERR_INVALID_ARG;
    }
    if (!positions || !inv_freq) return ETV_ERR_INVALID_ARG;
    etv_rotary_desc d = *h;
    if (d.scale == 0) d.scale = 1;
    const etv::RotaryPtrs p{q, k, v, q_out, k_out, v_out, k_cache, v_cache};
    const auto kernel = d.dtype == ETV_BF16 ? etv::rotary_kernel<uint16_t> : etv::rotary_kernel<float>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(d.B * d.T)), dim3(256), 0, etv::as_stream(stream), d, p, positions, inv_freq, n_rows, slot_map,
                       etv::fast_div_inv(d.T));
    return etv::check_launch();
}
