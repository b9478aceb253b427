// tree_verify_attention_q4: tree attention against a prefix whose K and V are held in 4 bits (format: eagletv.h).
#include "etv_common.h"

namespace etv {

typedef __bf16 q4_bf16x2 __attribute__((ext_vector_type(2)));
typedef float q4_f32x2 __attribute__((ext_vector_type(2)));

struct Q4Attn {
    const void *q, *kt, *vt;
    const uint8_t *codes[2], *scales[2];  // K, V
    const int32_t *block_table, *prefix_len, *n_nodes;
    const uint64_t *bitmask;
    void *out;
    float *lse;
    int B, T_max, Hq, Hkv, G, block_size, max_blocks, num_blocks, P_cap, P_max, words;
    float scale_log2;  // of the scores, times log2(e)
    uint32_t inv_bs;
};

constexpr float kQ4Ln2 = 0.6931471805599453f;

__device__ __forceinline__ float q4_elem(const float *p, size_t i) { return p[i]; }
__device__ __forceinline__ float q4_elem(const uint16_t *p, size_t i) { return bf16_bits_to_float(p[i]); }
__device__ __forceinline__ void q4_store(float *p, size_t i, float v) { p[i] = v; }
__device__ __forceinline__ void q4_store(uint16_t *p, size_t i, float v) { p[i] = float_to_bf16_bits(v); }
__device__ __forceinline__ float q4_scale(uint32_t s) { return __uint_as_float(s == 255u ? 0x7fc00000u : s << 23); }

// Row of position `pos` of sequence b in the layer's codes and scales; a block outside the pool: `known` false, row 0.
__device__ __forceinline__ uint64_t q4_prefix_row(const Q4Attn &p, int b, int kvh, int pos, bool &known) {
    known = true;
    if (p.block_size == 0) return ((uint64_t)b * p.Hkv + kvh) * (uint64_t)p.P_cap + pos;
    uint32_t at;
    const uint32_t lb = fast_div((uint32_t)pos, (uint32_t)p.block_size, p.inv_bs, at);
    const int id = p.block_table[(size_t)b * p.max_blocks + lb];
    known = id >= 0 && id < p.num_blocks;
    return known ? ((uint64_t)id * p.Hkv + kvh) * (uint64_t)p.block_size + at : 0;
}

__device__ __forceinline__ float q4_wave_max(float v) {
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ float q4_wave_sum(float v) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// One wavefront per query row, 64 keys at a time: a lane per key for the scores, a lane per channel (pair) for the values.
// Vector arithmetic throughout; keys that the row does not see are never touched.  grid (T_max, Hq, B).
template <typename T, int D>
__global__ void __launch_bounds__(64) attn_q4_generic_kernel(Q4Attn p) {
    constexpr int NG = D / 32, C = D / 64;  // groups of a row; channels of a lane
    __shared__ float sq[D], sp[64];
    const int k = blockIdx.x, h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x, kvh = h / p.G;
    const int n = clampi(p.n_nodes[b], 0, p.T_max), P = clampi(p.prefix_len[b], 0, p.P_max);
    const size_t orow = (((size_t)b * p.T_max + k) * p.Hq + h) * D;
    float m = -INFINITY, l = 0.f, acc[C];
    for (int c = 0; c < C; c++) acc[c] = 0.f;
    if (k < n) {
        for (int c = 0; c < C; c++) sq[lane + 64 * c] = q4_elem(static_cast<const T *>(p.q), orow + lane + 64 * c);
        __syncthreads();
        for (int base = 0; base < P + n; base += base < P ? min(64, P - base) : 64) {
            const bool tree = base >= P;
            const int j = base + lane - (tree ? P : 0), count = tree ? min(64, n - (base - P)) : min(64, P - base);
            bool see = lane < count, known = true;
            if (see && tree) see = p.bitmask[((size_t)b * p.T_max + k) * p.words + (j >> 6)] >> (j & 63) & 1;
            float s = -INFINITY;
            if (see && tree) {
                const T *row = static_cast<const T *>(p.kt) + (((size_t)b * p.T_max + j) * p.Hkv + kvh) * D;
                s = 0.f;
                for (int c = 0; c < D; c++) s = fmaf(sq[c], q4_elem(row, c), s);
            } else if (see) {
                const uint64_t row = q4_prefix_row(p, b, kvh, j, known);
                const uint32_t *codes = reinterpret_cast<const uint32_t *>(p.codes[0] + row * (D / 2));
                s = 0.f;
                for (int w = 0; w < D / 8; w++) {
                    const uint32_t c8 = codes[w];
                    const float f = q4_scale(p.scales[0][row * NG + w / 4]);
                    const q4_f32x2 x0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c8, f, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c8, f, 1);
                    const q4_f32x2 x2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c8, f, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c8, f, 3);
                    const float *qq = sq + 8 * w;
                    s = fmaf(qq[0], x0[0], fmaf(qq[1], x0[1], fmaf(qq[2], x1[0], fmaf(qq[3], x1[1], s))));
                    s = fmaf(qq[4], x2[0], fmaf(qq[5], x2[1], fmaf(qq[6], x3[0], fmaf(qq[7], x3[1], s))));
                }
                if (!known) s = NAN;
            }
            s *= p.scale_log2;
            if (!see) s = -INFINITY;
            const float tile = q4_wave_max(s);
            // NaN scores do not show in a maximum; they reach the row through their own exponential
            const float m_new = fmaxf(m, tile), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = exp2f(m - ref), e = see ? exp2f(s - ref) : 0.f;
            l = l * alpha + q4_wave_sum(e);
            for (int c = 0; c < C; c++) acc[c] *= alpha;
            m = m_new;
            __syncthreads();
            sp[lane] = e;
            __syncthreads();
            const uint64_t seen = __ballot(see);
            for (int x = 0; x < count; x++) {
                if (!(seen >> x & 1)) continue;
                const int jj = base + x - (tree ? P : 0);
                if (tree) {
                    const T *row = static_cast<const T *>(p.vt) + (((size_t)b * p.T_max + jj) * p.Hkv + kvh) * D;
                    for (int c = 0; c < C; c++) acc[c] = fmaf(sp[x], q4_elem(row, C * lane + c), acc[c]);
                } else {
                    const uint64_t row = q4_prefix_row(p, b, kvh, jj, known);
                    const uint32_t byte = p.codes[1][row * (D / 2) + (C * lane) / 2];
                    const float f = q4_scale(p.scales[1][row * NG + (C * lane) / 32]);
                    const q4_f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(byte, f, 0);
                    if (C == 2) {
                        acc[0] = fmaf(sp[x], v[0], acc[0]);
                        acc[C - 1] = fmaf(sp[x], v[1], acc[C - 1]);
                    } else {
                        acc[0] = fmaf(sp[x], lane & 1 ? v[1] : v[0], acc[0]);
                    }
                }
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int c = 0; c < C; c++) q4_store(static_cast<T *>(p.out), orow + C * lane + c, acc[c] * inv);
    if (p.lse && lane == 0) p.lse[((size_t)b * p.Hq + h) * p.T_max + k] = l == 0.f ? -INFINITY : (m + log2f(l)) * kQ4Ln2;
}

// What is wrong with a descriptor by itself.
static int32_t q4_check_desc(const etv_attn_desc *h) {
    if (!h) return ETV_ERR_INVALID_ARG;
    if (h->B < 0 || h->T_max < 1 || h->Hq < 1 || h->Hkv < 1 || h->Hq % h->Hkv != 0) return ETV_ERR_INVALID_ARG;
    if (h->dtype != ETV_F32 && h->dtype != ETV_BF16) return ETV_ERR_UNSUPPORTED;
    if (h->d != 64 && h->d != 128) return ETV_ERR_UNSUPPORTED;
    if (h->T_max > ETV_ATTN_MAX_TREE || h->B > 65535 || h->Hq > 65535) return ETV_ERR_UNSUPPORTED;
    if (h->P_max < 0 || h->kv_split < 0 || h->block_size < 0) return ETV_ERR_INVALID_ARG;
    if (h->block_size % 16 != 0) return ETV_ERR_UNSUPPORTED;
    if (h->block_size > 0 && (h->max_blocks < 1 || h->num_blocks < 1)) return ETV_ERR_INVALID_ARG;
    if (h->P_max > (h->block_size > 0 ? (int64_t)h->max_blocks * h->block_size : (int64_t)h->P_cap)) return ETV_ERR_INVALID_ARG;
    if (h->scale != h->scale || (h->flags & ~ETV_ATTN_FLAG_GENERIC) != 0) return ETV_ERR_INVALID_ARG;
    return ETV_OK;
}

}  // namespace etv

extern "C" size_t etv_tree_verify_attention_q4_workspace_bytes(const etv_attn_desc *h) { return etv::q4_check_desc(h) == ETV_OK ? 256 : 0; }

extern "C" int32_t etv_tree_verify_attention_q4(const etv_attn_desc *h, const void *q, const uint8_t *k_codes, const uint8_t *k_scales,
                                                const uint8_t *v_codes, const uint8_t *v_scales, const int32_t *block_table,
                                                const int32_t *prefix_len, const void *kt, const void *vt, const uint64_t *bitmask,
                                                const int32_t *n_nodes, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                                void *stream) {
    if (!h || !q || !prefix_len || !kt || !vt || !bitmask || !n_nodes || !out) return ETV_ERR_INVALID_ARG;
    const int32_t rc = etv::q4_check_desc(h);
    if (rc != ETV_OK) return rc;
    if (h->block_size > 0 && !block_table) return ETV_ERR_INVALID_ARG;
    if (h->P_max > 0 && (!k_codes || !k_scales || !v_codes || !v_scales)) return ETV_ERR_INVALID_ARG;
    const uintptr_t align = (uintptr_t)q | (uintptr_t)kt | (uintptr_t)vt | (uintptr_t)out | (uintptr_t)k_codes | (uintptr_t)v_codes |
                            (uintptr_t)workspace;
    if (align & 15 || ((uintptr_t)k_scales | (uintptr_t)v_scales) & 3) return ETV_ERR_INVALID_ARG;
    if (h->B == 0) return ETV_OK;
    (void)workspace_bytes;
    etv::Q4Attn p{};
    p.q = q; p.kt = kt; p.vt = vt;
    p.codes[0] = k_codes; p.codes[1] = v_codes; p.scales[0] = k_scales; p.scales[1] = v_scales;
    p.block_table = block_table; p.prefix_len = prefix_len; p.n_nodes = n_nodes; p.bitmask = bitmask;
    p.out = out; p.lse = lse;
    p.B = h->B; p.T_max = h->T_max; p.Hq = h->Hq; p.Hkv = h->Hkv; p.G = h->Hq / h->Hkv;
    p.block_size = h->block_size; p.max_blocks = h->max_blocks; p.num_blocks = h->num_blocks; p.P_cap = h->P_cap; p.P_max = h->P_max;
    p.words = (h->T_max + 63) / 64;
    p.inv_bs = h->block_size ? etv::fast_div_inv(h->block_size) : 0;
    p.scale_log2 = (h->scale == 0.f ? 1.0f / sqrtf((float)h->d) : h->scale) * 1.4426950408889634f;
    const dim3 grid(h->T_max, h->Hq, h->B);
    hipStream_t st = etv::as_stream(stream);
    if (h->dtype == ETV_F32 && h->d == 64) hipLaunchKernelGGL((etv::attn_q4_generic_kernel<float, 64>), grid, dim3(64), 0, st, p);
    else if (h->dtype == ETV_F32) hipLaunchKernelGGL((etv::attn_q4_generic_kernel<float, 128>), grid, dim3(64), 0, st, p);
    else if (h->d == 64) hipLaunchKernelGGL((etv::attn_q4_generic_kernel<uint16_t, 64>), grid, dim3(64), 0, st, p);
    else hipLaunchKernelGGL((etv::attn_q4_generic_kernel<uint16_t, 128>), grid, dim3(64), 0, st, p);
    return etv::check_launch();
}
