// The 4-bit prefix cache: quantising rows as they are written (a prompt, a token, the accepted path of a tree) and reading
// them back.  Format and layouts: eagletv.h.
//
// Both directions only move bytes, so the split follows the cache, which is written in rows of one head: a thread that
// quantises has one group of 32 channels of K and the same one of V (its maximum needs no other lane, its codes are one
// 16-byte store, and the lanes of a wavefront store 16 or 32 consecutive rows of a head: 1 KiB of codes, 64 bytes of scales).
// The conversions are single instructions (two values each), exact in the scale, rounding to nearest even.
// Measured: 2 prompts of 4096 and 3001 rows, 8 layers, 8 heads of 128, bf16, other buffers every time: written in 63 us (4.7 TB/s), read
// back in 52 us (5.7 TB/s); a token of 8 sequences, 32 layers, or the path of one tree: 3 to 5 us a launch, which is the launch.
#include "etv_common.h"

namespace etv {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

struct Q4Cache {
    uint8_t *codes[2], *scales[2];  // K, V
};

// Row of (sequence, head, position) within a layer; the block id has been checked.
__device__ __forceinline__ uint64_t q4_row(const etv_q4_desc &dsc, const int32_t *table_row, uint32_t inv_bs, int b, int h, int pos) {
    if (dsc.block_size == 0) return ((uint64_t)b * dsc.Hkv + h) * (uint64_t)dsc.P_cap + pos;
    uint32_t at;
    const uint32_t lb = fast_div((uint32_t)pos, (uint32_t)dsc.block_size, inv_bs, at);
    return ((uint64_t)table_row[lb] * dsc.Hkv + h) * (uint64_t)dsc.block_size + at;
}

// What every workgroup of a sequence finds out by itself: may positions P .. P + n - 1 be used?  All threads; the result is
// the same in each.  first_bits: what the caller has against the sequence already (then nothing else is looked at).
__device__ __forceinline__ int32_t q4_check(const etv_q4_desc &dsc, const int32_t *table_row, uint32_t inv_bs, int P, int n, int64_t cap,
                                            int32_t first_bits, int32_t *s_status) {
    if (threadIdx.x == 0) *s_status = first_bits;
    __syncthreads();
    if (!first_bits && n > 0) {
        int32_t mine = 0;
        if (P < 0 || (int64_t)P + n > cap) {
            mine = ETV_COMMIT_CAPACITY;
        } else if (dsc.block_size == 0) {
            if ((int64_t)P + n > dsc.P_cap) mine = ETV_COMMIT_CAPACITY;
        } else {
            uint32_t rem;
            const int lo = (int)fast_div((uint32_t)P, (uint32_t)dsc.block_size, inv_bs, rem);
            const int hi = (int)fast_div((uint32_t)P + (uint32_t)n - 1, (uint32_t)dsc.block_size, inv_bs, rem);
            if (hi >= dsc.max_blocks) mine = ETV_COMMIT_CAPACITY;
            for (int j = lo + (int)threadIdx.x; j <= min(hi, dsc.max_blocks - 1); j += 256) {
                const int id = table_row[j];
                if (id < 0 || id >= dsc.num_blocks) mine |= ETV_COMMIT_BAD_BLOCK;
            }
        }
        if (mine) atomicOr(s_status, mine);
    }
    __syncthreads();
    return *s_status;
}

// 32 values of one group, as the source holds them.
template <typename T>
struct Group;
template <>
struct Group<uint16_t> {
    uint4 w[4];
    __device__ __forceinline__ void load(const uint16_t *p) {
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ uint32_t word(int i) const { return i & 1 ? (i & 2 ? w[i >> 2].w : w[i >> 2].y) : (i & 2 ? w[i >> 2].z : w[i >> 2].x); }
    // biased exponent of the largest magnitude rounded to two significant bits; 255 and above: something is not finite
    __device__ __forceinline__ uint32_t exponent(bool &finite) const {
        u16x2 m = __builtin_bit_cast(u16x2, word(0) & 0x7fff7fffu);
#pragma unroll
        for (int i = 1; i < 16; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, word(i) & 0x7fff7fffu));
        const uint32_t top = max((uint32_t)m[0], (uint32_t)m[1]);
        finite = top < 0x7f80u;
        return (top + 0x20u) >> 7;
    }
    template <int SEL>
    __device__ __forceinline__ uint32_t convert(uint32_t old, int i, float scale) const {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, word(i)), scale, SEL);
    }
};
template <>
struct Group<float> {
    float4 w[8];
    __device__ __forceinline__ void load(const float *p) {
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = reinterpret_cast<const float4 *>(p)[i];
    }
    __device__ __forceinline__ uint32_t exponent(bool &finite) const {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t a = max(__float_as_uint(w[i].x) & 0x7fffffffu, __float_as_uint(w[i].y) & 0x7fffffffu);
            const uint32_t c = max(__float_as_uint(w[i].z) & 0x7fffffffu, __float_as_uint(w[i].w) & 0x7fffffffu);
            top = max(top, max(a, c));
        }
        finite = top < 0x7f800000u;
        return (top + 0x200000u) >> 23;
    }
    template <int SEL>
    __device__ __forceinline__ uint32_t convert(uint32_t old, int i, float scale) const {
        const float a = i & 1 ? w[i >> 1].z : w[i >> 1].x, c = i & 1 ? w[i >> 1].w : w[i >> 1].y;
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, c, scale, SEL);
    }
};

template <typename T>
__device__ __forceinline__ void quantise_group(const Group<T> &x, uint8_t *codes, uint8_t *scale_at) {
    bool finite;
    const uint32_t e = x.exponent(finite);
    const uint32_t s = min(max(e, 4u) - 2u, 252u);
    const float scale = __uint_as_float(s << 23);
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        uint32_t r = x.template convert<0>(0, 4 * i, scale);
        r = x.template convert<1>(r, 4 * i + 1, scale);
        r = x.template convert<2>(r, 4 * i + 2, scale);
        c[i] = x.template convert<3>(r, 4 * i + 3, scale);
    }
    *reinterpret_cast<uint4 *>(codes) = finite ? uint4{c[0], c[1], c[2], c[3]} : uint4{0, 0, 0, 0};
    *scale_at = (uint8_t)(finite ? s : 255u);
}

// grid (ceil(Hkv * R * NG / 256), B, n_layers), NG groups a row, R rows at most (W for the commit).  Items in the order
// (head, row, group).  COMMIT: row i is node acc_nodes[i] of the tree buffer, count = accept_len.
template <typename T, int NG, bool COMMIT>
__global__ void __launch_bounds__(256) write_rows_kernel(etv_q4_desc dsc, Q4Cache cache, const T *__restrict__ src_k, const T *__restrict__ src_v,
                                                         const int32_t *__restrict__ block_table, const int32_t *__restrict__ prefix_len,
                                                         const int32_t *__restrict__ count, const int32_t *__restrict__ capacity,
                                                         const int32_t *__restrict__ n_nodes, const int32_t *__restrict__ acc_nodes,
                                                         int32_t *__restrict__ prefix_len_out, int32_t *__restrict__ slot_map,
                                                         int32_t *__restrict__ status, uint32_t inv_bs, uint32_t inv_rows) {
    __shared__ int32_t s_status;
    const int b = blockIdx.y, l = blockIdx.z, R = COMMIT ? dsc.W : dsc.rows;
    const uint32_t item = blockIdx.x * 256 + threadIdx.x, g = item % NG;
    uint32_t i;
    const uint32_t h = fast_div(item / NG, (uint32_t)R, inv_rows, i);
    const bool mine = h < (uint32_t)dsc.Hkv;
    const int32_t *const table_row = block_table + (size_t)b * dsc.max_blocks;  // not followed in a contiguous cache
    const int32_t *const acc_row = COMMIT ? acc_nodes + (size_t)b * dsc.W : nullptr;
    // the source rows are asked for before it is known whether they are wanted: they exist
    const int node = COMMIT ? (mine ? acc_row[i] : 0) : (int)i;
    Group<T> k, v;
    if (mine) {
        const size_t at = ((((size_t)l * dsc.B + b) * dsc.rows + clampi(node, 0, dsc.rows - 1)) * dsc.Hkv + h) * (NG * 32) + g * 32;
        k.load(src_k + at);
        v.load(src_v + at);
    }
    const int P = prefix_len[b], c = count[b], n = COMMIT ? c + 1 : c;
    int32_t bits = 0;
    if (COMMIT ? (c < 0 || c > dsc.W - 1) : (c < 0 || c > R)) bits = ETV_COMMIT_BAD_LEN;
    int32_t st = q4_check(dsc, table_row, inv_bs, P, n, capacity[b], bits, &s_status);
    if constexpr (COMMIT) {
        if (!bits) {
            __syncthreads();
            const int nodes = clampi(n_nodes[b], 0, dsc.rows);
            bool bad = false;
            for (int j = threadIdx.x; j < n; j += 256) bad = bad || acc_row[j] < 0 || acc_row[j] >= nodes;
            if (bad) atomicOr(&s_status, ETV_COMMIT_BAD_NODE);
            __syncthreads();
            st = s_status;
        }
    }
    if (blockIdx.x == 0 && l == 0) {
        if (threadIdx.x == 0) {
            status[b] = st;
            prefix_len_out[b] = st ? P : P + n;
        }
        if (COMMIT)
            for (int j = threadIdx.x; j < dsc.W; j += 256)
                slot_map[(size_t)b * dsc.W + j] = st || j >= n ? -1
                    : dsc.block_size ? table_row[(P + j) / dsc.block_size] * dsc.block_size + (P + j) % dsc.block_size : P + j;
    }
    if (st || !mine || (int)i >= n) return;
    const uint64_t row = (uint64_t)l * dsc.layer_rows + q4_row(dsc, table_row, inv_bs, b, (int)h, P + (int)i);
    quantise_group(k, cache.codes[0] + row * (NG * 16) + g * 16, cache.scales[0] + row * NG + g);
    quantise_group(v, cache.codes[1] + row * (NG * 16) + g * 16, cache.scales[1] + row * NG + g);
}

// Streams that this launch touches once pass the caches by.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void stream_out(void *p, u32x4 v) { __builtin_nontemporal_store(v, static_cast<u32x4 *>(p)); }

// 16 bytes of a row: eight bf16 channels from four bytes of codes, or four fp32 channels from two
template <typename T>
struct Piece;
template <>
struct Piece<uint16_t> {
    typedef uint32_t Codes;
    static __device__ __forceinline__ void put(uint16_t *out, uint32_t codes, float scale) {
        u32x4 r;
        r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
        r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
        r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
        r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
        stream_out(out, r);
    }
};
template <>
struct Piece<float> {
    typedef uint16_t Codes;
    static __device__ __forceinline__ void put(float *out, uint32_t codes, float scale) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
        const float4 r = {a[0], a[1], b[0], b[1]};
        stream_out(out, __builtin_bit_cast(u32x4, r));
    }
};

// The scale of a byte; the conversions pass a NaN on.
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s == 255u ? 0x7fc00000u : s << 23); }

// grid (ceil(Hkv * rows * pieces / (256 * U)), B, n_layers).  A thread has 16 bytes of K and of V of U items: its stores and its
// lane neighbours' are consecutive, which the wider of the two sides needs.  The rows written are not read here: past the caches,
// 8 x 4096 rows of 4 layers, bf16, take 136 us instead of 138 (the 640 MB come from and go to memory either way), and 7097 rows of 8 layers
// just written 116, the writing with them, instead of 147.
constexpr int kReadItems = 4;
template <typename T, int NG>
__global__ void __launch_bounds__(256) read_rows_kernel(etv_q4_desc dsc, Q4Cache cache, const int32_t *__restrict__ block_table,
                                                        const int32_t *__restrict__ first, const int32_t *__restrict__ n_rows, T *__restrict__ k,
                                                        T *__restrict__ v, int32_t *__restrict__ status, uint32_t inv_bs, uint32_t inv_rows) {
    __shared__ int32_t s_status;
    using P16 = Piece<T>;
    constexpr int U = kReadItems, PER = 16 / (int)sizeof(T), CH = NG * 32 / PER;  // channels of a piece, pieces of a row
    const int b = blockIdx.y, l = blockIdx.z;
    const int32_t *const table_row = block_table + (size_t)b * dsc.max_blocks;
    const int P = first[b], n = n_rows[b];
    const int32_t bits = n < 0 || n > dsc.rows || P < 0 ? ETV_COMMIT_BAD_LEN : 0;
    const int32_t st = q4_check(dsc, table_row, inv_bs, P, n, INT64_MAX, bits, &s_status);
    if (blockIdx.x == 0 && l == 0 && threadIdx.x == 0) status[b] = st;
    uint32_t codes[2][U], scale[2][U];
    size_t at[U];
    bool mine[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const uint32_t item = (blockIdx.x * U + u) * 256 + threadIdx.x, c = item % CH;
        uint32_t i;
        const uint32_t h = fast_div(item / CH, (uint32_t)dsc.rows, inv_rows, i);
        mine[u] = h < (uint32_t)dsc.Hkv;
        at[u] = ((((size_t)l * dsc.B + b) * dsc.rows + i) * dsc.Hkv + h) * (NG * 32) + c * PER;
        codes[0][u] = codes[1][u] = scale[0][u] = scale[1][u] = 0;
        if (mine[u] && !st && (int)i < n) {
            const uint64_t row = (uint64_t)l * dsc.layer_rows + q4_row(dsc, table_row, inv_bs, b, (int)h, P + (int)i);
#pragma unroll
            for (int x = 0; x < 2; x++) {
                codes[x][u] = *reinterpret_cast<const typename P16::Codes *>(cache.codes[x] + row * (NG * 16) + c * (PER / 2));
                scale[x][u] = cache.scales[x][row * NG + c * PER / 32];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; u++)
        if (mine[u]) {
            P16::put(k + at[u], codes[0][u], scale_of(scale[0][u]));
            P16::put(v + at[u], codes[1][u], scale_of(scale[1][u]));
        }
}

static int32_t check_q4(const etv_q4_desc *h, const void *k, const void *v, const Q4Cache &c, const int32_t *block_table, bool commit) {
    if (!h || !k || !v || !c.codes[0] || !c.codes[1] || !c.scales[0] || !c.scales[1]) return ETV_ERR_INVALID_ARG;
    if (h->B < 0 || h->rows < 1 || h->Hkv < 1 || h->n_layers < 1 || (commit && h->W < 1)) return ETV_ERR_INVALID_ARG;
    if (h->dtype != ETV_F32 && h->dtype != ETV_BF16) return ETV_ERR_UNSUPPORTED;
    if (h->d != 64 && h->d != 128) return ETV_ERR_UNSUPPORTED;
    if (h->block_size < 0 || h->layer_rows < 0) return ETV_ERR_INVALID_ARG;
    if (h->block_size % 16 != 0) return ETV_ERR_UNSUPPORTED;
    if (h->block_size > 0 && (!block_table || h->max_blocks < 1 || h->num_blocks < 1)) return ETV_ERR_INVALID_ARG;
    if (h->block_size == 0 && h->P_cap < 1) return ETV_ERR_INVALID_ARG;
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)c.codes[0] | (uintptr_t)c.codes[1]) & 15) return ETV_ERR_INVALID_ARG;
    if (((uintptr_t)c.scales[0] | (uintptr_t)c.scales[1]) & 3) return ETV_ERR_INVALID_ARG;
    // positions and items of a sequence are counted in 31 bits
    if (h->block_size > 0 && (int64_t)h->max_blocks * h->block_size > INT32_MAX) return ETV_ERR_UNSUPPORTED;
    if ((int64_t)h->Hkv * (commit ? h->W : h->rows) * (h->d / 4) > INT32_MAX - 1024) return ETV_ERR_UNSUPPORTED;
    if (h->B > 65535 || h->n_layers > 65535) return ETV_ERR_UNSUPPORTED;
    return ETV_OK;
}

template <bool COMMIT>
static int32_t write_rows(const etv_q4_desc *h, const Q4Cache &cache, const void *k, const void *v, const int32_t *block_table,
                          const int32_t *prefix_len, const int32_t *count, const int32_t *capacity, const int32_t *n_nodes,
                          const int32_t *acc_nodes, int32_t *prefix_len_out, int32_t *slot_map, int32_t *status, void *stream) {
    if (!prefix_len || !count || !capacity || !prefix_len_out || !status || prefix_len_out == prefix_len) return ETV_ERR_INVALID_ARG;
    const int32_t rc = check_q4(h, k, v, cache, block_table, COMMIT);
    if (rc != ETV_OK) return rc;
    if (h->B == 0) return ETV_OK;
    const int R = COMMIT ? h->W : h->rows, ng = h->d / 32;
    const dim3 grid((unsigned)(((int64_t)h->Hkv * R * ng + 255) / 256), h->B, h->n_layers);
    const uint32_t inv_bs = h->block_size ? fast_div_inv(h->block_size) : 0, inv_rows = fast_div_inv(R);
    const auto launch = [&](auto kernel, auto *ks, auto *vs) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, as_stream(stream), *h, cache, ks, vs, block_table, prefix_len, count, capacity, n_nodes,
                           acc_nodes, prefix_len_out, slot_map, status, inv_bs, inv_rows);
    };
    if (h->dtype == ETV_BF16) {
        const auto *ks = static_cast<const uint16_t *>(k), *vs = static_cast<const uint16_t *>(v);
        if (ng == 4) launch(write_rows_kernel<uint16_t, 4, COMMIT>, ks, vs);
        else launch(write_rows_kernel<uint16_t, 2, COMMIT>, ks, vs);
    } else {
        const auto *ks = static_cast<const float *>(k), *vs = static_cast<const float *>(v);
        if (ng == 4) launch(write_rows_kernel<float, 4, COMMIT>, ks, vs);
        else launch(write_rows_kernel<float, 2, COMMIT>, ks, vs);
    }
    return check_launch();
}

}  // namespace etv

extern "C" int32_t etv_quantize_kv_q4(const etv_q4_desc *h, const void *k, const void *v, uint8_t *k_codes, uint8_t *k_scales,
                                      uint8_t *v_codes, uint8_t *v_scales, const int32_t *block_table, const int32_t *prefix_len,
                                      const int32_t *n_rows, const int32_t *capacity, int32_t *prefix_len_out, int32_t *status,
                                      void *stream) {
    return etv::write_rows<false>(h, {{k_codes, v_codes}, {k_scales, v_scales}}, k, v, block_table, prefix_len, n_rows, capacity, nullptr,
                                  nullptr, prefix_len_out, nullptr, status, stream);
}

extern "C" int32_t etv_commit_accepted_kv_q4(const etv_q4_desc *h, const void *kt, const void *vt, uint8_t *k_codes, uint8_t *k_scales,
                                             uint8_t *v_codes, uint8_t *v_scales, const int32_t *block_table, const int32_t *prefix_len,
                                             const int32_t *capacity, const int32_t *n_nodes, const int32_t *acc_nodes,
                                             const int32_t *accept_len, int32_t *prefix_len_out, int32_t *slot_map, int32_t *status,
                                             void *stream) {
    if (!n_nodes || !acc_nodes || !slot_map) return ETV_ERR_INVALID_ARG;
    return etv::write_rows<true>(h, {{k_codes, v_codes}, {k_scales, v_scales}}, kt, vt, block_table, prefix_len, accept_len, capacity, n_nodes,
                                 acc_nodes, prefix_len_out, slot_map, status, stream);
}

extern "C" int32_t etv_dequantize_kv_q4(const etv_q4_desc *h, const uint8_t *k_codes, const uint8_t *k_scales, const uint8_t *v_codes,
                                        const uint8_t *v_scales, const int32_t *block_table, const int32_t *first, const int32_t *n_rows,
                                        void *k, void *v, int32_t *status, void *stream) {
    if (!first || !n_rows || !status) return ETV_ERR_INVALID_ARG;
    const etv::Q4Cache cache = {{const_cast<uint8_t *>(k_codes), const_cast<uint8_t *>(v_codes)},
                                {const_cast<uint8_t *>(k_scales), const_cast<uint8_t *>(v_scales)}};  // only read
    const int32_t rc = etv::check_q4(h, k, v, cache, block_table, false);
    if (rc != ETV_OK) return rc;
    if (h->B == 0) return ETV_OK;
    const int per_block = 256 * etv::kReadItems;
    const dim3 grid((unsigned)(((int64_t)h->Hkv * h->rows * (h->d * (h->dtype == ETV_BF16 ? 2 : 4) / 16) + per_block - 1) / per_block), h->B, h->n_layers);
    const uint32_t inv_bs = h->block_size ? etv::fast_div_inv(h->block_size) : 0, inv_rows = etv::fast_div_inv(h->rows);
    const auto launch = [&](auto kernel, auto *ko, auto *vo) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, etv::as_stream(stream), *h, cache, block_table, first, n_rows, ko, vo, status, inv_bs,
                           inv_rows);
    };
    if (h->dtype == ETV_BF16) {
        auto *ko = static_cast<uint16_t *>(k), *vo = static_cast<uint16_t *>(v);
        if (h->d == 128) launch(etv::read_rows_kernel<uint16_t, 4>, ko, vo);
        else launch(etv::read_rows_kernel<uint16_t, 2>, ko, vo);
    } else {
        auto *ko = static_cast<float *>(k), *vo = static_cast<float *>(v);
        if (h->d == 128) launch(etv::read_rows_kernel<float, 4>, ko, vo);
        else launch(etv::read_rows_kernel<float, 2>, ko, vo);
    }
    return etv::check_launch();
}
