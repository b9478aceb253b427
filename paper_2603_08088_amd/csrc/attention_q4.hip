// tree_verify_attention_q4: tree attention against a prefix whose K and V are held in 4 bits (format: eagletv.h).
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

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
    // matrix kernel: prefixes in splits, B * nsplit slots for them and, where there is more than one each (slots > B), B more for
    // the trees.  chunk: keys of a split, or 0: worked out on the device, where the lengths are (B <= 64).
    // Partials, if slots > B: part_o [Hkv][slots][rows_padded][D], part_ml (reference, sum) alike; split_tab [B] first slot, slots.
    int chunk, nsplit, slots, row_groups, rows_padded, units, span;
    uint32_t inv_g, inv_hkv, inv_groups, inv_nsplit;
    float *part_o;
    float2 *part_ml;
    int2 *split_tab;
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
    bool sees = false;
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
            sees = sees || seen != 0;
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
    const float inv = !sees ? 0.f : l == 0.f ? NAN : 1.f / l;  // nothing but scores of -inf: NaN
    for (int c = 0; c < C; c++) q4_store(static_cast<T *>(p.out), orow + C * lane + c, acc[c] * inv);
    if (p.lse && lane == 0) p.lse[((size_t)b * p.Hq + h) * p.T_max + k] = !sees ? -INFINITY : l == 0.f ? NAN : (m + log2f(l)) * kQ4Ln2;
}

// ------------------------------------------------------------------------------------------------
// The matrix kernel.  With the G * T_max query rows of a KV head packed into rows r = t * G + g, a wavefront has 32 of them and
// takes 32 or 64 keys at a time:
//   S^T[key, r]  = K Q^T     v_mfma_scale_f32_32x32x64_f8f6f4: K as the cache holds it (fp4, its scale bytes the instruction's),
//                            by way of LDS, q in NQ parts of 6 bits (e2m3)
//   P^T          = exp2(S^T * scale - reference)   a lane has 32 keys of one row; the reference follows the maximum lazily
//   O^T[d, r]   += V^T P^T   bf16: V is converted (exactly) into an LDS tile and comes back through the transpose read; P stays
//                            in registers as the product's B operand
// The parts of q: part x is q less the parts before it, rounded to e2m3 at scale 2^(e - 2 - 4x), e being the exponent of its group's
// maximum, one up where that comes within 1/32 of the next power of two: so the first part is never held at 7.5, the largest value
// there is (a value just under 8 would leave the next part one just under 8 again, and so on: 2^-16 of it after four), and of the
// maximum, at least 3.875 at that scale, no more than 2^-16 / 3.875 is left.  That is 2^-17.95 after four parts; fp32 takes six
// (2^-25.95).  (Three, 2^-13.95, are enough for outputs rounded to bf16, but show in lse.)  Six-bit and four-bit operands run at four
// times the bf16 rate: four parts cost what one bf16 product would, and K needs no conversion.
// fp32: P in three bf16 parts, exactly, and the tree's K, V and q likewise (products with parts below 2^-24 left out).
// RW wavefronts of a workgroup share their keys and have rows of their own; the groups of RW share the rows: few rows
// (a token, a small tree) leave reading the cache as the work, and every wavefront reads keys of its own.
typedef int q4_i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t q4_u32x6 __attribute__((ext_vector_type(6)));
typedef float q4_f32x16 __attribute__((ext_vector_type(16)));
typedef float q4_f32x32 __attribute__((ext_vector_type(32)));
typedef __bf16 q4_bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 q4_bf16x8 __attribute__((ext_vector_type(8)));
typedef short q4_s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) q4_s16x4 q4_lds_s16x4;

// memory that no kernel writes while it is read: uniform addresses go through scalar loads
typedef __attribute__((address_space(4))) const int32_t *const_ids;
constexpr float kQ4Lazy = 1024.f;  // the largest sum of a lane's weights in a tile without a new reference

// Dynamic LDS, by key group: V tiles [2][keys][D] bf16, K tiles [1 or 2][keys][D/2] and their scales [keys][4]; afterwards 64
// channels at a time of the outputs [wavefronts][32][64 + 4] fp32.
constexpr int q4_wavefronts(bool f32, int rw) { return rw == 4 || f32 ? 4 : 8; }  // of a workgroup
template <int D, bool F32, int RW>
struct Q4Geo {
    static constexpr int NW = q4_wavefronts(F32, RW);
    static constexpr int KB = RW == 4 ? 2 : 1, KEYS = 32 * KB;  // key blocks and keys of a tile
    static constexpr int ROW = 2 * D, TILE = KEYS * ROW, KW = NW / RW, BUFS = 2;
    static constexpr int K_BUFS = RW > 1 ? 2 : 1, K_TILE = KEYS * D / 2, K_SCALES = KEYS * 4;
    static constexpr int K_AT = KW * BUFS * TILE, K_SCALES_AT = K_AT + KW * K_BUFS * K_TILE, TILES = K_SCALES_AT + KW * K_BUFS * K_SCALES;
    // Do the scores' products start from less the reference (16 registers, all alike), or is it taken off each score?  The former
    // saves 16 instructions a key block; where registers are short it costs more in spills, whose reloads wait for every load on its
    // way (32 x 8 heads of 4096 keys, 8 nodes: 51.6 us, 39.4 the other way; 128 nodes: 468 and 275).
    static constexpr bool RELATIVE = !(RW != 2 && D == 128 && !F32);
    static constexpr int OUT_ROW = 64 + 4, OUT = NW * 32 * (OUT_ROW * 4 + 8);  // floats; four on from a multiple of the banks
    static constexpr int LDS = TILES > OUT ? TILES : OUT;
};

// 32 values to six bits (e2m3) and back.  These conversions work in several passes and read their scale in each, so
// the result must not lie on an operand.  The builtins let it lie on the scale (q then lost its lower parts, in a build with
// fewer registers): hence the early-clobbered results, and the wait states a following matrix instruction may need.
__device__ __forceinline__ q4_u32x6 q4_to_six_bits(q4_f32x16 even, q4_f32x16 odd, float scale) {
    q4_u32x6 r;
    asm volatile("v_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3\n\ts_nop 7" : "=&v"(r) : "v"(even), "v"(odd), "v"(scale));
    return r;
}
__device__ __forceinline__ q4_f32x32 q4_from_six_bits(q4_u32x6 x, float scale) {
    q4_f32x32 r;
    asm volatile("v_cvt_scalef32_pk32_f32_fp6 %0, %1, %2\n\ts_nop 7" : "=&v"(r) : "v"(x), "v"(scale));
    return r;
}
template <int OPA, int OPB>
__device__ __forceinline__ q4_f32x16 q4_scores(uint4 k, q4_u32x6 q, q4_f32x16 c, uint32_t k_scale, uint32_t q_scale) {
    const q4_i32x8 a = {(int)k.x, (int)k.y, (int)k.z, (int)k.w, 0, 0, 0, 0}, b = {(int)q[0], (int)q[1], (int)q[2], (int)q[3], (int)q[4], (int)q[5], 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 2, OPA, (int)k_scale, OPB, (int)q_scale);
}
__device__ __forceinline__ uint32_t q4_pair(float a, float b) {
    const q4_f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, q4_bf16x2));
}
// a, b = hi + mid + lo exactly (24 bits in three bf16); what is not finite stays in hi
__device__ __forceinline__ void q4_split(float a, float b, uint32_t &hi, uint32_t &mid, uint32_t &lo) {
    const auto upper = [](float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); };
    const auto halves = [](float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u); };
    hi = halves(a, b);
    a -= upper(a); b -= upper(b);
    mid = halves(a, b);
    lo = halves(a - upper(a), b - upper(b));
}
__device__ __forceinline__ float q4_half_max(float v) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float q4_half_sum(float v) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float q4_max3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}
// Positions of 16-byte pieces within a row of the V tile: the lanes of a transpose read reach all banks.  (16 lanes of a store, four to
// a row, reach half of them.  Of the cycles that LDS is busy, 43 % are conflicts of any kind: 32 x 8 heads of 4096 keys, 128 nodes.)
template <int D>
__device__ __forceinline__ int q4_swizzle(int row) { return D == 128 ? (((row & 3) << 1) | ((row >> 2) & 1)) : ((row & 2) << 1); }

template <class F, int... I>
__device__ __forceinline__ void q4_each(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void q4_for(F f) { q4_each(f, std::make_integer_sequence<int, N>{}); }

template <int D, bool F32, int RW>
struct Q4Wave {
    static constexpr int KM = D / 64, DB = D / 32, NP = F32 ? 3 : 1, NQ = F32 ? 6 : 4, QW = (NQ + 3) / 4;
    using G = Q4Geo<D, F32, RW>;
    static constexpr int KB = G::KB;
    const Q4Attn &p;
    uint8_t *smem;
    int lane, r, hh, kg, wr, stage;
    q4_f32x16 o[DB];
    q4_f32x16 off;    // less the reference in every element: what the scores' products start from
    float ref, sum[2];  // reference (log2); the row's sum in two chains: zero while nothing has been weighed, and no reference holds

    __device__ __forceinline__ uint8_t *buffer(int x) const { return smem + kg * G::BUFS * G::TILE + x * G::TILE; }
    __device__ __forceinline__ uint8_t *tile() const { return smem + (kg * G::BUFS + (stage & 1)) * G::TILE; }
    // Between the stores of a V tile and its reads.  Rows shared out: every wavefront has stored its part; the next tile goes to the
    // other buffer, which all have read before this barrier.  Else the tile is the wavefront's own, and LDS keeps its order.
    __device__ __forceinline__ void staged() const {
        if constexpr (RW > 1) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0xc07f);
            __builtin_amdgcn_s_barrier();
        }
        asm volatile("" ::: "memory");
    }

    // Keys whose bit of vis is clear are not seen.
    __device__ __forceinline__ void mask(q4_f32x16 (&s)[KB], uint64_t vis) const {
        const uint32_t v[2] = {(uint32_t)vis >> (4 * hh), (uint32_t)(vis >> 32) >> (4 * hh)};
#pragma unroll
        for (int kb = 0; kb < KB; kb++)
#pragma unroll
            for (int i = 0; i < 16; i++) s[kb][i] = v[kb] >> (8 * (i >> 2) + (i & 3)) & 1u ? s[kb][i] : -INFINITY;
    }

    // The largest score of a row.
    __device__ __forceinline__ static float largest(const q4_f32x16 (&s)[KB]) {
        float top[2] = {s[0][0], s[KB - 1][15]};
#pragma unroll
        for (int i = 0; i < 16 * KB; i += 2) top[i >> 1 & 1] = q4_max3(top[i >> 1 & 1], s[i / 16][i % 16], s[i / 16][i % 16 + 1]);
        return q4_half_max(__builtin_elementwise_maximum(top[0], top[1]));
    }
    __device__ __forceinline__ void refer_to(float reference) {
        ref = reference;
#pragma unroll
        for (int i = 0; i < 16; i++) off[i] = G::RELATIVE ? -reference : 0.f;
    }
    __device__ __forceinline__ void scale_outputs(float f) {
        sum[0] *= f;
        sum[1] *= f;
#pragma unroll
        for (int db = 0; db < DB; db++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[db][i] *= f;
    }
    __device__ __forceinline__ static void shift(q4_f32x16 (&s)[KB], float by) {
#pragma unroll
        for (int kb = 0; kb < KB; kb++)
#pragma unroll
            for (int i = 0; i < 16; i++) s[kb][i] -= by;
    }
    // Has the row a weight so far?  A reference's own key weighs 1, so a sum never falls back to zero.
    __device__ __forceinline__ float row_sum() const { return q4_half_sum(sum[0] + sum[1]); }
    // Scores become relative.  A row without a reference (`none`) takes the tile's largest score, if it sees any.  Returns the latter.
    __device__ __forceinline__ float enter(q4_f32x16 (&s)[KB], bool none) {
        const float top = largest(s);
        refer_to(!none ? ref : fabsf(top) < INFINITY ? top : 0.f);
        if (G::RELATIVE) shift(s, ref);
        return top;
    }

    // P^T: pair x of a tile's 8 KB pairs of relative scores to weights, and their part of the row's sum.
    template <int X>
    __device__ __forceinline__ void weigh(const q4_f32x16 (&s)[KB], uint32_t (&pk)[NP][KB][8], float (&part)[2]) const {
        constexpr int kb = X / 8, i = X % 8;
        const float by = G::RELATIVE ? 0.f : ref;
        const float a = __builtin_amdgcn_exp2f(G::RELATIVE ? s[kb][2 * i] : s[kb][2 * i] - by), b = __builtin_amdgcn_exp2f(G::RELATIVE ? s[kb][2 * i + 1] : s[kb][2 * i + 1] - by);
        if constexpr (F32) q4_split(a, b, pk[0][kb][i], pk[1][kb][i], pk[NP - 1][kb][i]);
        else pk[0][kb][i] = q4_pair(a, b);  // the value product takes them rounded to bf16, as on an unquantised cache, the sum (and lse) does not
        part[X & 1] = X < 2 ? a + b : part[X & 1] + (a + b);
    }
    __device__ __forceinline__ void weigh_all(const q4_f32x16 (&s)[KB], uint32_t (&pk)[NP][KB][8], float (&part)[2]) const {
        q4_for<8 * KB>([&](auto x) { weigh<decltype(x)::value>(s, pk, part); });
    }
    // A tile whose sum shows that its scores have left the reference behind gives the rows a new one; only then is the maximum
    // looked for.  s_next: scores of the next tile, relative to the old one.  (A NaN keeps its row coming here.)
    template <bool NEXT>
    __device__ __forceinline__ void settle(q4_f32x16 (&s)[KB], q4_f32x16 (&s_next)[KB], uint32_t (&pk)[NP][KB][8], float (&part)[2]) {
        if (__builtin_expect(__any(!(part[0] + part[1] <= kQ4Lazy)), 0)) {
            const float top = G::RELATIVE ? largest(s) : largest(s) - ref, lift = top > 0.f && top < INFINITY ? top : 0.f;
            scale_outputs(__builtin_amdgcn_exp2f(-lift));
            if (G::RELATIVE) shift(s, lift);
            if (G::RELATIVE && NEXT) shift(s_next, lift);
            refer_to(ref + lift);
            weigh_all(s, pk, part);
        }
        sum[0] += part[0];
        sum[1] += part[1];
    }

    // V^T of 16 keys (16 x of the tile) and 32 channels (32 db ..)
    __device__ __forceinline__ q4_bf16x8 v_fragment(const uint8_t *v, int x, int db) const {
        const int i16 = lane & 15, vrow = 4 * hh + (i16 >> 2), piece = 2 * (lane >> 4 & 1) + ((i16 & 3) >> 1), sub = 8 * (i16 & 1);
        const uint8_t *const at = v + (16 * x + vrow) * G::ROW + sub + (((4 * db + piece) ^ q4_swizzle<D>(vrow)) << 4);
        const q4_s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((q4_lds_s16x4 *)at);
        const q4_s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((q4_lds_s16x4 *)(at + 8 * G::ROW));
        return __builtin_shufflevector(__builtin_bit_cast(q4_bf16x4, v0), __builtin_bit_cast(q4_bf16x4, v1), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // O^T of 32 channels += V^T P^T over 16 keys, with the first PARTS of P
    template <int PARTS>
    __device__ __forceinline__ void multiply(q4_bf16x8 v, int x, int db, const uint32_t (&pk)[NP][KB][8]) {
#pragma unroll
        for (int y = 0; y < PARTS; y++) {
            const uint32_t(&w)[8] = pk[y][x / 2];
            const uint4 f = {w[4 * (x & 1)], w[4 * (x & 1) + 1], w[4 * (x & 1) + 2], w[4 * (x & 1) + 3]};
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(q4_bf16x8, f), o[db], 0, 0, 0);
        }
    }
    // The same one after the other, where there is nothing to do meanwhile.
    template <int PARTS>
    __device__ __forceinline__ void accumulate(const uint8_t *v, const uint32_t (&pk)[NP][KB][8]) {
#pragma unroll
        for (int x = 0; x < 2 * KB; x++)
#pragma unroll
            for (int db = 0; db < DB; db++) multiply<PARTS>(v_fragment(v, x, db), x, db, pk);
    }
};

// Eight consecutive channels of an unquantised row: as they lie in memory, and as NP bf16 parts.
template <typename T>
struct Q4Eight {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (size_t i = 0; i < sizeof(T) / 2; i++) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void parts(uint4 (&part)[1]) const { part[0] = w[0]; }
    __device__ __forceinline__ void parts(uint4 (&part)[3]) const {
        const uint4 &a = w[0], &b = w[sizeof(T) / 2 - 1];
        const auto f = [](uint32_t x) { return __uint_as_float(x); };
        q4_split(f(a.x), f(a.y), part[0].x, part[1].x, part[2].x);
        q4_split(f(a.z), f(a.w), part[0].y, part[1].y, part[2].y);
        q4_split(f(b.x), f(b.y), part[0].z, part[1].z, part[2].z);
        q4_split(f(b.z), f(b.w), part[0].w, part[1].w, part[2].w);
    }
};
// the values that are not finite out of eight bf16 (first parts); true if there were any
__device__ __forceinline__ bool q4_take_out(uint4 &w) {
    const auto ill = [](uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };
    const auto keep = [&](uint32_t x) { return x & ~((ill(x) >> 15) * 0xffffu); };
    const bool any = (ill(w.x) | ill(w.y) | ill(w.z) | ill(w.w)) != 0;
    w = uint4{keep(w.x), keep(w.y), keep(w.z), keep(w.w)};
    return any;
}

// Does a node see a key?  Asked only where its weights add up to nothing.
__device__ __forceinline__ bool q4_sees(const int32_t *prefix_len, const uint64_t *mask, int P_max, int n) {
    bool any = min(*prefix_len, P_max) > 0;
    for (int w = 0; 64 * w < n; w++) any = any || (n - 64 * w < 64 ? mask[w] & ((1ull << (n - 64 * w)) - 1) : mask[w]) != 0;
    return any;
}

// One row's eight channels from its sums, and its lse by the first of the threads.
template <typename T>
__device__ __forceinline__ void q4_finish(const Q4Attn &p, int b, int t, int head, int piece, int D, bool node, float ref, float sum, const float (&acc)[8]) {
    // no key: zeros; keys, but no weight (scores of -inf alone), an infinite score or a NaN among them: NaN
    if (node && sum == 0.f) {
        node = q4_sees(p.prefix_len + b, p.bitmask + ((size_t)b * p.T_max + t) * p.words, p.P_max, clampi(p.n_nodes[b], 0, p.T_max));
        sum = NAN;
    }
    const float inv = !node ? 0.f : sum < INFINITY ? 1.f / sum : NAN;
    T *const dst = static_cast<T *>(p.out) + (((size_t)b * p.T_max + t) * p.Hq + head) * D + 8 * piece;
    if constexpr (sizeof(T) == 4) {
        const float4 a = inv == 0.f ? float4{0, 0, 0, 0} : float4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
        const float4 c = inv == 0.f ? float4{0, 0, 0, 0} : float4{acc[4] * inv, acc[5] * inv, acc[6] * inv, acc[7] * inv};
        reinterpret_cast<float4 *>(dst)[0] = a;
        reinterpret_cast<float4 *>(dst)[1] = c;
    } else {
        uint4 v = {q4_pair(acc[0] * inv, acc[1] * inv), q4_pair(acc[2] * inv, acc[3] * inv), q4_pair(acc[4] * inv, acc[5] * inv), q4_pair(acc[6] * inv, acc[7] * inv)};
        *reinterpret_cast<uint4 *>(dst) = inv == 0.f ? uint4{0, 0, 0, 0} : v;
    }
    if (p.lse && piece == 0) p.lse[((size_t)b * p.Hq + head) * p.T_max + t] = inv == 0.f ? -INFINITY : inv != inv ? NAN : (ref + __builtin_amdgcn_logf(sum)) * kQ4Ln2;
}

// The largest finite score (log2) that a row has among the keys of the wavefront's first tile to have one, from position `from` on;
// -inf: none.  Asked only by rows whose first tile scores -inf throughout (products beyond the fp32 range): their reference.
// Vector arithmetic, a lane per row and every other key.
template <typename T, int D>
__device__ __forceinline__ float q4_some_score(const Q4Attn &p, const T *q, bool wanted, int b, int kvh, int from, int keys, int step, int to, int hh) {
    float best = -INFINITY;
    for (int base = from; base < to && __any(wanted && best == -INFINITY); base += step) {  // uniform
        float top = -INFINITY;
        for (int j = base + hh; j < min(base + keys, to); j += 2) {
            bool known;
            const uint64_t row = q4_prefix_row(p, b, kvh, j, known);
            float s = known ? 0.f : NAN;
#pragma unroll 1
            for (int c = 0; c < D; c += 2) {
                const q4_f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)p.codes[0][row * (D / 2) + c / 2], q4_scale(p.scales[0][row * (D / 32) + c / 32]), 0);
                s = fmaf(q4_elem(q, c) * p.scale_log2, x[0], fmaf(q4_elem(q, c + 1) * p.scale_log2, x[1], s));
            }
            if (fabsf(s) < INFINITY) top = fmaxf(top, s);
        }
        top = q4_half_max(top);
        if (wanted && best == -INFINITY) best = top;
    }
    return best;
}

// Which keys of which sequence a prefix slot stands for.  All splits of a call are of one size c (in rounds of `span` keys), about the
// smallest for which the slots suffice: not before c = ceil(rounds / slots), and with c = ceil(rounds / (slots - B)) always, a
// sequence's last split being the only one that is not full.  So a short sequence has few splits and the long ones of a ragged
// batch share the rest.  Every wavefront works it out for itself, a lane per sequence.
struct Q4Share {
    int b, k0, k1, first, count;  // count 0: nobody's slot.  first, count: the sequence's slots
};
__device__ __forceinline__ Q4Share q4_share(const Q4Attn &p, int slot, int lane) {
    const bool in = lane < p.B;
    const int P = in ? clampi(p.prefix_len[in ? lane : 0], 0, p.P_max) : 0;
    const int rounds = P > 0 && p.n_nodes[in ? lane : 0] > 0 ? (P + p.span - 1) / p.span : 0, slots = p.B * p.nsplit;
    // 64 prefixes of almost 2^31 positions are almost 2^31 rounds: the sums of rounds are unsigned
    const uint32_t total = (uint32_t)__builtin_amdgcn_readlane(wave_scan_sum(rounds), 63);
    int c = p.chunk > 0 ? p.chunk / p.span : max(1, (int)((total + slots - 1) / (uint32_t)slots));
    int count = (rounds + c - 1) / c, upto = wave_scan_sum(count);
    const int enough = p.chunk > 0 ? c : (int)((total + (uint32_t)(slots - p.B) - 1) / (uint32_t)max(1, slots - p.B));
    while (c < enough && __builtin_amdgcn_readlane(upto, 63) > slots) {
        c = min(c + 1 + c / 16, enough);
        count = (rounds + c - 1) / c;
        upto = wave_scan_sum(count);
    }
    const int b = __popcll(__ballot(upto <= slot));  // sequences that end before the slot; lanes behind the last repeat its end
    Q4Share r{};
    if (b >= p.B) return r;
    r.b = b;
    r.count = __builtin_amdgcn_readlane(count, b);
    r.first = __builtin_amdgcn_readlane(upto, b) - r.count;
    r.k0 = (slot - r.first) * c * p.span;
    r.k1 = r.k0 + min(c * p.span, __builtin_amdgcn_readlane(P, b) - r.k0);  // k0 + c * span may pass 2^31
    return r;
}

template <int D, bool F32, int RW, bool PAGED>
__global__ void __launch_bounds__(q4_wavefronts(F32, RW) * 64, F32 && D == 128 ? 1 : 2) attn_q4_kernel(Q4Attn p) {
    using T = std::conditional_t<F32, float, uint16_t>;
    using Wave = Q4Wave<D, F32, RW>;
    using G = Q4Geo<D, F32, RW>;
    constexpr int KM = Wave::KM, DB = Wave::DB, NP = Wave::NP, NQ = Wave::NQ, QW = Wave::QW, KW = G::KW, KB = G::KB, KEYS = G::KEYS;
    extern __shared__ __attribute__((aligned(1024))) uint8_t q4_smem[];
    const int tid = threadIdx.x;
    Wave w{p, q4_smem};
    w.lane = tid & 63;
    w.r = w.lane & 31;
    w.hh = w.lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    w.kg = wave / RW;
    w.wr = wave % RW;
    w.stage = 0;
    w.sum[0] = w.sum[1] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; db++)
#pragma unroll
        for (int i = 0; i < 16; i++) w.o[db][i] = 0.f;
    const int r = w.r, hh = w.hh;

    // The row groups of a unit read the same keys: their workgroups are eight apart, on one of the eight XCDs.  The trees' units,
    // which are short, come last.
    uint32_t group, kvh, rem;
    const uint32_t unit = fast_div(blockIdx.x >> 3, (uint32_t)p.row_groups, p.inv_groups, group) * 8 + (blockIdx.x & 7);
    if (unit >= (uint32_t)p.units) return;
    const int slot = (int)fast_div(unit, (uint32_t)p.Hkv, p.inv_hkv, kvh);
    const bool whole = p.slots == p.B, tree_here = whole || slot >= p.B * p.nsplit;
    int b = 0, k0 = 0, k1 = 0;
    if (tree_here) {
        b = whole ? slot : slot - p.B * p.nsplit;
        k1 = whole ? clampi(p.prefix_len[b], 0, p.P_max) : 0;
    } else if (p.B <= 64) {
        const Q4Share share = q4_share(p, slot, w.lane);
        if (share.count == 0) return;
        b = share.b;
        k0 = share.k0;
        k1 = share.k1;
        if (slot == share.first && kvh == 0 && group == 0 && tid == 0) p.split_tab[b] = int2{share.first, share.count};
    } else {
        b = (int)fast_div((uint32_t)slot, (uint32_t)p.nsplit, p.inv_nsplit, rem);
        const int P = clampi(p.prefix_len[b], 0, p.P_max);
        k0 = (int)min((int64_t)P, (int64_t)rem * p.chunk);
        k1 = (int)min((int64_t)P, (int64_t)k0 + p.chunk);
        if (rem == 0 && kvh == 0 && group == 0 && tid == 0) p.split_tab[b] = int2{slot, (int)(((uint32_t)P + (uint32_t)p.chunk - 1) / (uint32_t)p.chunk)};
        if (k0 >= k1) return;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    k0 = __builtin_amdgcn_readfirstlane(k0);
    k1 = __builtin_amdgcn_readfirstlane(k1);
    const int n = clampi(p.n_nodes[b], 0, p.T_max);
    uint32_t g;
    const int t = (int)fast_div(group * 32 * RW + 32 * w.wr + r, (uint32_t)p.G, p.inv_g, g);
    const size_t q_row = (((size_t)b * p.T_max + min(t, p.T_max - 1)) * p.Hq + kvh * p.G + g) * D;
    const bool live = (int)fast_div(group * 32 * RW, (uint32_t)p.G, p.inv_g, rem) < n;  // has the workgroup a row?
    if (!live && !whole) return;
    bool ill = false;  // the tree's V holds values that are not finite

    if (live && k0 < k1) {
        // q as six-bit parts; a group with something that is not finite is NaN
        q4_u32x6 qp[NQ][KM];
        uint32_t qs[QW][KM];
#pragma unroll
        for (int i = 0; i < KM; i++) {
            const T *const src = static_cast<const T *>(p.q) + q_row + 32 * (2 * i + hh);
            float x[32];
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
                if constexpr (F32) {
                    const float4 a = *reinterpret_cast<const float4 *>(src + c), d = *reinterpret_cast<const float4 *>(src + c + 4);
                    x[c] = a.x; x[c + 1] = a.y; x[c + 2] = a.z; x[c + 3] = a.w; x[c + 4] = d.x; x[c + 5] = d.y; x[c + 6] = d.z; x[c + 7] = d.w;
                } else {
                    const uint4 a = *reinterpret_cast<const uint4 *>(src + c);
                    const uint32_t ws[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                    for (int j = 0; j < 4; j++) { x[c + 2 * j] = __uint_as_float(ws[j] << 16); x[c + 2 * j + 1] = __uint_as_float(ws[j] & 0xffff0000u); }
                }
            }
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < 32; c++) {
                x[c] *= p.scale_log2;
                top = max(top, __float_as_uint(x[c]) & 0x7fffffffu);
            }
            const uint32_t e = max((top + 0x80000u) >> 23, 4 * NQ + 2u) - 2;  // every part's scale byte is at least 1
            qs[0][i] = e | (e - 4) << 8 | (e - 8) << 16 | (NQ > 3 ? (e - 12) << 24 : 0u);
            if constexpr (NQ > 4) qs[QW - 1][i] = (e - 16) | (e - 20) << 8;
            if (top >= 0x7f800000u)
                for (int j = 0; j < QW; j++) qs[j][i] = 0xffffffffu;
#pragma unroll
            for (int y = 0; y < NQ; y++) {
                const float scale = __uint_as_float((e - 4 * y) << 23);
                q4_f32x16 even, odd;  // the instruction takes two of 16 and interleaves them
#pragma unroll
                for (int c = 0; c < 16; c++) { even[c] = x[2 * c]; odd[c] = x[2 * c + 1]; }
                qp[y][i] = q4_to_six_bits(even, odd, scale);
                if (y + 1 < NQ) {
                    const q4_f32x32 done = q4_from_six_bits(qp[y][i], scale);
#pragma unroll
                    for (int c = 0; c < 32; c++) x[c] -= done[c];
                }
            }
        }

        // A wavefront's pieces of a tile are 16 whole rows each, a lane having a quarter of a row of K and of V: loads of consecutive
        // memory beside a scalar base.  (A lane that loads the rows and groups its products want takes the address unit four times as
        // long, and K would be loaded by every wavefront: 268 us for 32 x 8 heads of 4096 keys and 128 nodes, 250 this way, with q in
        // three parts.)
        constexpr int PC = KEYS / 16 / RW, VW = D / 32;  // pieces of a wavefront, words of a lane
        struct Codes {
            uint32_t k[PC][VW], v[PC][VW], ks[PC], vs[PC];  // K of a tile, V of the one before it; scales: the quarter's
        };
        struct Rows {
            uint32_t row[PC], bad[PC];  // scalar: first row in the layer's cache; all ones: in a block outside the pool
            int pos[PC];                // position of that row
        };
        const int key16 = w.lane >> 2, quarter = w.lane & 3;
        const int span = KEYS * KW, mine = k0 + KEYS * w.kg, rounds = (k1 - k0 + span - 1) / span;
        // The walk through the table: block and offset of the wavefront's next 16 positions, in scalar registers (blocks are multiples of
        // 16 positions, pieces begin at multiples of 16).  Behind the split it stays in the last block, whose rows exist.
        const const_ids table = (const_ids)(uintptr_t)(PAGED ? p.block_table + (size_t)b * p.max_blocks : nullptr);
        const uint32_t head_rows = kvh * (uint32_t)(PAGED ? p.block_size : p.P_cap), block_rows = (uint32_t)(p.Hkv * p.block_size);
        uint32_t walk = 0, walk_off = 0, jump = 0, jump_off = 0, last_block = 0;
        if constexpr (PAGED) {
            walk = fast_div((uint32_t)(mine + 16 * w.wr), (uint32_t)p.block_size, p.inv_bs, walk_off);
            jump = fast_div((uint32_t)(span - (PC - 1) * 16), (uint32_t)p.block_size, p.inv_bs, jump_off);
            last_block = fast_div((uint32_t)(k1 - 1), (uint32_t)p.block_size, p.inv_bs, rem);
        }
        const auto advance = [&](uint32_t blocks, uint32_t positions) {
            walk += blocks;
            walk_off += positions;
            if (walk_off >= (uint32_t)p.block_size) walk_off -= (uint32_t)p.block_size, walk++;
        };
        int ids[PC] = {};
        uint32_t offs[PC] = {};
        const auto fetch_ids = [&] {  // of the tile that is placed next
            if constexpr (PAGED)
#pragma unroll
                for (int j = 0; j < PC; j++) {
                    ids[j] = table[min(walk, last_block)];
                    offs[j] = walk_off;
                    advance(j + 1 < PC ? 0 : jump, j + 1 < PC ? 16 : jump_off);
                }
        };
        const auto place = [&](Rows &to, int base) {
#pragma unroll
            for (int j = 0; j < PC; j++) {
                to.pos[j] = base + 16 * (j * RW + w.wr);
                if constexpr (PAGED) {
                    to.bad[j] = (uint32_t)((ids[j] | (p.num_blocks - 1 - ids[j])) >> 31);  // negative or too large
                    to.row[j] = ((uint32_t)ids[j] & ~to.bad[j]) * block_rows + head_rows + offs[j];
                } else {
                    to.bad[j] = 0;
                    to.pos[j] = min(to.pos[j], (k1 - 1) & ~15);
                    to.row[j] = (uint32_t)b * p.Hkv * (uint32_t)p.P_cap + head_rows + (uint32_t)to.pos[j];
                }
            }
        };
        // Rows 16 on from a piece's first exist where they are a block's; in a contiguous cache they are held within the split.
        const auto load = [&](const uint8_t *codes, const uint8_t *scales, const Rows &rows, int j, uint32_t (&c)[PC][VW], uint32_t (&sc)[PC]) {
            const uint32_t key = PAGED ? (uint32_t)key16 : (uint32_t)min(key16, k1 - 1 - rows.pos[j]);
            const uint8_t *const from = codes + (uint64_t)rows.row[j] * (D / 2) + (key * (D / 2) + quarter * (D / 8));
            if constexpr (VW == 4) {
                const uint4 x = *reinterpret_cast<const uint4 *>(from);
                c[j][0] = x.x; c[j][1] = x.y; c[j][VW - 2] = x.z; c[j][VW - 1] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2 *>(from);
                c[j][0] = x.x; c[j][1] = x.y;
            }
            sc[j] = (scales + (uint64_t)rows.row[j] * (D / 32))[key * (D / 32) + (D == 128 ? quarter : quarter >> 1)];
        };
        const auto load_k = [&](Codes &to, const Rows &rows, int j) {
            load(p.codes[0], p.scales[0], rows, j, to.k, to.ks);
        };
        const auto load_v = [&](Codes &to, const Rows &rows, int j) {
            load(p.codes[1], p.scales[1], rows, j, to.v, to.vs);
        };
        uint8_t *const k_tiles = q4_smem + G::K_AT + w.kg * G::K_BUFS * G::K_TILE, *const k_scales = q4_smem + G::K_SCALES_AT + w.kg * G::K_BUFS * G::K_SCALES;
        // K as it came, its 16-byte pieces of a row (D 128) moved about so that eight rows' reads reach all banks; bad: NaN scales
        const auto put_k = [&](const Codes &from, uint32_t bad, int buffer, int j) {
            const int row = 16 * (j * RW + w.wr) + key16, x = G::K_BUFS > 1 ? buffer : 0;
            uint8_t *const to = k_tiles + x * G::K_TILE + row * (D / 2);
            if constexpr (VW == 4) *reinterpret_cast<uint4 *>(to + ((quarter ^ (key16 >> 2)) << 4)) = uint4{from.k[j][0], from.k[j][1], from.k[j][VW - 2], from.k[j][VW - 1]};
            else *reinterpret_cast<uint2 *>(to + 8 * quarter) = uint2{from.k[j][0], from.k[j][1]};
            (k_scales + x * G::K_SCALES)[row * (D / 32) + (D == 128 ? quarter : quarter >> 1)] = (uint8_t)(from.ks[j] | bad);
        };
        // V of a piece as bf16, eight channels of word x; keys behind the split weigh nothing and have to be numbers
        const auto put_v = [&](const Codes &from, int pos, uint8_t *tile, int u) {
            const int j = u / VW, x = u % VW, row = 16 * (j * RW + w.wr) + key16;
            const float f = q4_scale(key16 < k1 - pos - 16 * (j * RW) ? from.vs[j] : 127u);
            const uint32_t in = from.v[j][x];
            uint4 v;
            v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(in, f, 0));
            v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(in, f, 1));
            v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(in, f, 2));
            v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(in, f, 3));
            *reinterpret_cast<uint4 *>(tile + row * G::ROW + (((VW * quarter + x) ^ q4_swizzle<D>(row)) << 4)) = v;
        };
        // K of a tile as the products want it: of key row r of each key block the groups 2i + hh, the scales' bytes 0 and 2
        const auto get_k = [&](int buffer, int i, uint4 (&kf)[KB][KM], uint32_t (&ks)[KB]) {
            const int x = G::K_BUFS > 1 ? buffer : 0;
#pragma unroll
            for (int kb = 0; kb < KB; kb++) {
                const int row = 32 * kb + r;
                const uint8_t *const from = k_tiles + x * G::K_TILE + row * (D / 2), *const sc = k_scales + x * G::K_SCALES + row * (D / 32);
                kf[kb][i] = *reinterpret_cast<const uint4 *>(from + (D == 128 ? ((2 * i + hh) ^ (r >> 2 & 3)) << 4 : 16 * hh));
                if (i == 0) ks[kb] = (D == 128 ? *reinterpret_cast<const uint32_t *>(sc) : (uint32_t) * reinterpret_cast<const uint16_t *>(sc)) >> (8 * hh);
            }
        };
        // Scores: product X of a tile's QK, y the part of q.
        constexpr int QK = NQ * KM * KB, PV = 2 * KB * DB, UNITS = PC * VW;
        const auto score = [&](auto x, const uint4 (&kf)[KB][KM], const uint32_t (&ks)[KB], q4_f32x16 (&s)[KB]) {
            constexpr int X = decltype(x)::value, kb = X % KB, y = X / KB % NQ, i = X / (KB * NQ);
            s[kb] = q4_scores<2 * i, y & 3>(kf[kb][i], qp[y][i], X < KB ? w.off : s[kb], ks[kb], qs[y >> 2][i]);
        };

        // Software pipeline: a step has the scores of its tile already and works out the next tile's between its exponentials (or, where
        // they are not relative, before its value products); between those it stores the next tile's V and the K of the one after into LDS: the matrix and the vector unit are both busy
        // within one wavefront.  What is stored was asked for a step before (two steps ahead took 8 % longer where 32 x 8
        // heads of 4096 keys and 8 nodes leave the reading: more registers and a longer start).
        Codes start, second, codes;
        Rows first, rows, newer;  // rows, newer: of the tile whose K was asked for last, and of the next one
        uint32_t bad[PC];         // of the K in `codes`
        q4_f32x16 sa[KB], sb[KB];
        fetch_ids();
        place(first, mine);
#pragma unroll
        for (int j = 0; j < PC; j++) {
            load_k(start, first, j);
            load_v(start, first, j);
        }
        fetch_ids();
        place(rows, mine + span);
#pragma unroll
        for (int j = 0; j < PC; j++) load_k(second, rows, j);
        fetch_ids();
        place(newer, mine + 2 * span);
#pragma unroll
        for (int j = 0; j < PC; j++) {
            load_v(codes, rows, j);
            load_k(codes, newer, j);
            bad[j] = newer.bad[j];
        }
        uint4 kf[KB][KM];
        uint32_t ks[KB], pk[NP][KB][8];
        float part[2];
        w.refer_to(0.f);  // what the first scores start from; that tile brings the reference
#pragma unroll
        for (int j = 0; j < PC; j++) put_k(start, first.bad[j], 0, j);
#pragma unroll
        for (int u = 0; u < UNITS; u++) put_v(start, mine + 16 * w.wr, w.buffer(0), u);
        if constexpr (G::K_BUFS == 1) {
            asm volatile("" ::: "memory");
            q4_for<KM>([&](auto i) { get_k(0, decltype(i)::value, kf, ks); });
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int j = 0; j < PC; j++) put_k(second, rows.bad[j], 1, j);
        rows = newer;
        w.staged();
        if constexpr (G::K_BUFS > 1) q4_for<KM>([&](auto i) { get_k(0, decltype(i)::value, kf, ks); });
        q4_for<QK>([&](auto x) { score(x, kf, ks, sa); });
        // the last round alone may have tiles that are not whole
        const int last = mine + (rounds - 1) * span;
        const auto cut = [&] {
            if (last + KEYS > k1) w.mask(sa, last < k1 ? (1ull << (k1 - last)) - 1 : 0);
        };
        if (rounds == 1) cut();
        const float top = w.enter(sa, true);
        if (rounds > 1 && __builtin_expect(__any(top == -INFINITY), 0)) {
            const float some = q4_some_score<T, D>(p, static_cast<const T *>(p.q) + q_row, top == -INFINITY, b, kvh, mine + span, KEYS, span, k1, hh);
            if (some != -INFINITY) w.refer_to(some);
        }
        w.staged();
        const auto step = [&](auto buffer, int t, q4_f32x16 (&s)[KB], q4_f32x16 (&s_next)[KB]) {
            constexpr int NOW = decltype(buffer)::value, FLY = 3;  // fragments of V on their way from LDS
            const int base = mine + t * span;
            uint8_t *const tile = w.buffer(NOW), *const tile_next = w.buffer(1 - NOW);
            q4_bf16x8 v[FLY + 1];
            fetch_ids();
            get_k(1 - NOW, 0, kf, ks);
            q4_for<QK>([&](auto x) {
                constexpr int X = decltype(x)::value;
                if constexpr (KM == 2 && X == KB * NQ - 3) get_k(1 - NOW, KM - 1, kf, ks);  // no earlier: registers
                score(x, kf, ks, s_next);
                constexpr int LO = X * 8 * KB / QK, HI = (X + 1) * 8 * KB / QK;
                q4_for<HI - LO>([&](auto y) { w.template weigh<LO + decltype(y)::value>(s, pk, part); });
                __builtin_amdgcn_sched_barrier(0);
            });
            w.template settle<true>(s, s_next, pk, part);
            q4_for<FLY>([&](auto x) { v[decltype(x)::value] = w.v_fragment(tile, decltype(x)::value / DB, decltype(x)::value % DB); });
            q4_for<PV>([&](auto x) {
                constexpr int X = decltype(x)::value, Y = X + FLY;
                if constexpr (Y < PV) v[Y % (FLY + 1)] = w.v_fragment(tile, Y / DB, Y % DB);
                w.template multiply<NP>(v[X % (FLY + 1)], X / DB, X % DB, pk);
                if constexpr (X == 0) place(newer, base + 3 * span);
                if constexpr (X < UNITS) put_v(codes, base + span + 16 * w.wr, tile_next, X);
                if constexpr (X < UNITS && X % VW == VW - 1) {
                    constexpr int J = X / VW;
                    put_k(codes, bad[J], NOW, J);
                    bad[J] = newer.bad[J];
                    load_v(codes, rows, J);
                    load_k(codes, newer, J);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            rows = newer;
            w.staged();
        };
        int t = 0;
        for (; t + 2 < rounds; t += 2) {
            step(std::integral_constant<int, 0>{}, t, sa, sb);
            step(std::integral_constant<int, 1>{}, t + 1, sb, sa);
        }
        if (t + 1 < rounds) {
            step(std::integral_constant<int, 0>{}, t, sa, sb);
#pragma unroll
            for (int kb = 0; kb < KB; kb++) sa[kb] = sb[kb];
        }
        w.stage = rounds - 1;
        if (rounds > 1) cut();
        w.weigh_all(sa, pk, part);
        w.template settle<false>(sa, sb, pk, part);
        w.template accumulate<NP>(w.tile(), pk);
        w.stage++;
    }

    if (live && tree_here) {
        // The tree: bf16 parts throughout.  n >= 1 here.
        const T *const kt = static_cast<const T *>(p.kt), *const vt = static_cast<const T *>(p.vt);
        constexpr int KK = D / 16, PIECES = KEYS * D / 8 / (64 * RW);
        uint4 qf[KK][NP];
        {
            Q4Eight<T> raw[KK];
#pragma unroll
            for (int kk = 0; kk < KK; kk++) raw[kk].load(static_cast<const T *>(p.q) + q_row + 16 * kk + 8 * hh);
#pragma unroll
            for (int kk = 0; kk < KK; kk++) raw[kk].parts(qf[kk]);
        }
        for (int first = 0; first < n; first += KEYS * KW) {  // the same number of rounds for every wavefront
            const int base = first + KEYS * w.kg;
            // everything from memory at once: the mask, V (a wavefront's share of the tile) and K
            uint64_t vis = p.bitmask[((size_t)b * p.T_max + min(t, p.T_max - 1)) * p.words + (min(base, n - 1) >> 6)] >> (base & 63);
            Q4Eight<T> vraw[PIECES];
#pragma unroll
            for (int j = 0; j < PIECES; j++) {
                const int c = w.lane + 64 * w.wr + 64 * RW * j, key = min(base + c / (D / 8), n - 1);
                vraw[j].load(vt + (((size_t)b * p.T_max + key) * p.Hkv + kvh) * D + 8 * (c % (D / 8)));
            }
            Q4Eight<T> kraw[F32 ? 1 : KB][KK];
            const auto load_keys = [&](int kb) {
                const T *const row = kt + (((size_t)b * p.T_max + min(base + 32 * kb + r, n - 1)) * p.Hkv + kvh) * D + 8 * hh;
#pragma unroll
                for (int kk = 0; kk < KK; kk++) kraw[F32 ? 0 : kb][kk].load(row + 16 * kk);
            };
            if constexpr (!F32)
#pragma unroll
                for (int kb = 0; kb < KB; kb++) load_keys(kb);
            q4_f32x16 s[KB];
#pragma unroll
            for (int kb = 0; kb < KB; kb++) {
                if constexpr (F32) load_keys(kb);
#pragma unroll
                for (int i = 0; i < 16; i++) s[kb][i] = 0.f;
                bool bad = false;
#pragma unroll
                for (int kk = 0; kk < KK; kk++) {
                    uint4 kf[NP];
                    kraw[F32 ? 0 : kb][kk].parts(kf);
                    if constexpr (F32) bad |= q4_take_out(kf[0]);  // the products of its parts would be NaN
#pragma unroll
                    for (int x = 0; x < NP; x++)
#pragma unroll
                        for (int y = 0; x + y < NP; y++)
                            s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(q4_bf16x8, kf[x]), __builtin_bit_cast(q4_bf16x8, qf[kk][y]),
                                                                            s[kb], 0, 0, 0);
                }
                if constexpr (F32)
                    if (__any(bad)) {  // rare: these scores from the rows themselves
                        for (int i = 0; i < 16; i++) {
                            const int j = min(base + 32 * kb + 8 * (i >> 2) + 4 * hh + (i & 3), n - 1);
                            const T *const kr = kt + (((size_t)b * p.T_max + j) * p.Hkv + kvh) * D, *const qr = static_cast<const T *>(p.q) + q_row;
                            float sum = 0.f;
                            for (int c = 0; c < D; c++) sum = fmaf(q4_elem(kr, c), q4_elem(qr, c), sum);
                            s[kb][i] = sum;
                        }
                    }
            }
            if (base >= n || t >= n) vis = 0;
            else if (n - base < KEYS) vis &= (1ull << (n - base)) - 1;
#pragma unroll
            for (int kb = 0; kb < KB; kb++)
#pragma unroll
                for (int i = 0; i < 16; i++) s[kb][i] *= p.scale_log2;
            w.mask(s, vis);
            w.enter(s, w.row_sum() == 0.f);
            uint32_t pk[NP][KB][8];
            float part[2];
            w.weigh_all(s, pk, part);
            w.template settle<false>(s, s, pk, part);
            // V, one bf16 part of it at a time
            const auto stage_part = [&](int part) {
                uint8_t *const tile = w.tile();
#pragma unroll
                for (int j = 0; j < PIECES; j++) {
                    const int c = w.lane + 64 * w.wr + 64 * RW * j, key = c / (D / 8), piece = c % (D / 8);
                    uint4 vf[NP];
                    vraw[j].parts(vf);
                    if constexpr (F32) {
                        uint4 first_part = vf[0];
                        const bool bad = q4_take_out(first_part);
                        ill |= bad && base + key < n;
                        if (bad) {  // the other parts of such a value are NaN
                            uint4 &x = vf[1], &y = vf[2];
                            const auto only = [](uint32_t hi, uint32_t v) { return v & ~(((((hi & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu); };
                            x = uint4{only(vf[0].x, x.x), only(vf[0].y, x.y), only(vf[0].z, x.z), only(vf[0].w, x.w)};
                            y = uint4{only(vf[0].x, y.x), only(vf[0].y, y.y), only(vf[0].z, y.z), only(vf[0].w, y.w)};
                        }
                        vf[0] = first_part;
                    } else {
                        ill |= q4_take_out(vf[0]) && base + key < n;
                    }
                    uint4 v = vf[0];
                    if constexpr (F32) v = part == 0 ? vf[0] : part == 1 ? vf[1] : vf[2];
                    if (base + key >= n) v = uint4{0, 0, 0, 0};
                    *reinterpret_cast<uint4 *>(tile + key * G::ROW + ((piece ^ q4_swizzle<D>(key)) << 4)) = v;
                }
                w.staged();
            };
            stage_part(0);
            w.template accumulate<NP>(w.tile(), pk);
            w.stage++;
            if constexpr (F32) {
                stage_part(1);
                w.template accumulate<2>(w.tile(), pk);
                w.stage++;
                stage_part(2);
                w.template accumulate<1>(w.tile(), pk);
                w.stage++;
            }
        }
    }

    const float row_sum = w.row_sum();
    // Values of the tree's V that are not finite were left out: added here to the rows that see them, whose outputs are then
    // not finite whatever the weight.  (The barriers also end the last reads of the V tiles.)
    __shared__ int s_ill;
    if (tid == 0) s_ill = 0;
    __syncthreads();
    if (ill) s_ill = 1;
    __syncthreads();
    if (s_ill) {
        for (int j = 0; j < n; j++) {
            if ((j / KEYS) % KW != w.kg) continue;  // uniform: each key once
            const bool see = t < n && (p.bitmask[((size_t)b * p.T_max + min(t, p.T_max - 1)) * p.words + (j >> 6)] >> (j & 63) & 1);
            const T *const row = static_cast<const T *>(p.vt) + (((size_t)b * p.T_max + j) * p.Hkv + kvh) * D + 4 * hh;
#pragma unroll
            for (int db = 0; db < DB; db++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const float v = q4_elem(row, 32 * db + 8 * (i >> 2) + (i & 3));
                    if (see && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) w.o[db][i] += v;
                }
        }
    }

    // Outputs through LDS, 64 channels at a time: the key groups of a row are joined, and rows are stored in one piece.
    float *const mine = reinterpret_cast<float *>(q4_smem) + (wave * 32 + r) * G::OUT_ROW + 4 * hh;
    float2 *const ml = reinterpret_cast<float2 *>(q4_smem + G::NW * 32 * G::OUT_ROW * 4);
    if (hh == 0) ml[wave * 32 + r] = float2{row_sum == 0.f ? -INFINITY : w.ref, row_sum};
#pragma unroll
    for (int half = 0; half < D / 64; half++) {
        if (half) __syncthreads();
#pragma unroll
        for (int db = 0; db < 2; db++)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const q4_f32x16 &o = w.o[2 * half + db];
                *reinterpret_cast<float4 *>(mine + 32 * db + 2 * i) = float4{o[i], o[i + 1], o[i + 2], o[i + 3]};
            }
        __syncthreads();
        for (int c = tid; c < 32 * RW * 8; c += 64 * G::NW) {
            const int row = c >> 3, piece = c & 7, chunk = row / 32;  // chunk: the wavefront among the RW
            const uint32_t packed = group * 32 * RW + row;
            uint32_t gg;
            const int tt = (int)fast_div(packed, (uint32_t)p.G, p.inv_g, gg);
            float ref = -INFINITY, sum = 0.f, acc[8] = {};
#pragma unroll
            for (int x = 0; x < KW; x++) ref = fmaxf(ref, ml[(x * RW + chunk) * 32 + (row & 31)].x);
            const float zero = ref == -INFINITY ? 0.f : ref;
#pragma unroll
            for (int x = 0; x < KW; x++) {
                const float2 part = ml[(x * RW + chunk) * 32 + (row & 31)];
                const float f = KW == 1 ? 1.f : __builtin_amdgcn_exp2f(part.x - zero);
                const float *const src = reinterpret_cast<const float *>(q4_smem) + ((x * RW + chunk) * 32 + (row & 31)) * G::OUT_ROW + 8 * piece;
                sum += f * part.y;
#pragma unroll
                for (int j = 0; j < 8; j++) acc[j] += f * src[j];
            }
            if (!whole) {
                if (tt >= n) continue;
                const size_t at = ((size_t)kvh * p.slots + slot) * (size_t)p.rows_padded + packed;
                float4 *const dst = reinterpret_cast<float4 *>(p.part_o + at * D + 64 * half + 8 * piece);
                dst[0] = float4{acc[0], acc[1], acc[2], acc[3]};
                dst[1] = float4{acc[4], acc[5], acc[6], acc[7]};
                if (piece == 0 && half == 0) p.part_ml[at] = float2{ref, sum};
                continue;
            }
            if (tt >= p.T_max) continue;
            q4_finish<T>(p, b, tt, (int)kvh * p.G + (int)gg, 8 * half + piece, D, tt < n, ref, sum, acc);
        }
    }
}

// The partials of a row joined by WIDTH lanes: they have eight channels each, and where those are fewer than the lanes (WIDTH 64)
// the others share out the splits.  Few rows want the latter, many rows the narrow form (15360 rows of 5 partials: 12.4 and 7.5 us;
// 32 rows of 17: 4.6 and 11.8).  grid (ceil(T_max * Hq / (256 / WIDTH)), B).
template <int D, bool F32, int WIDTH>
__global__ void __launch_bounds__(256) join_q4_kernel(Q4Attn p) {
    using T = std::conditional_t<F32, float, uint16_t>;
    constexpr int PIECES = D / 8, WORKERS = WIDTH / PIECES, BATCH = 4;
    const int b = blockIdx.y, lane = threadIdx.x % WIDTH, piece = lane % PIECES, worker = lane / PIECES;
    const int x = blockIdx.x * (256 / WIDTH) + threadIdx.x / WIDTH;
    if (x >= p.T_max * p.Hq) return;
    const int t = x / p.Hq, head = x % p.Hq, kvh = head / p.G;
    const int n = clampi(p.n_nodes[b], 0, p.T_max);
    float ref = -INFINITY, sum = 0.f, acc[8] = {};
    if (t < n) {
        const int P = clampi(p.prefix_len[b], 0, p.P_max);
        const int2 tab = P > 0 ? p.split_tab[b] : int2{0, 0};
        const size_t row0 = (size_t)kvh * p.slots * p.rows_padded + (size_t)t * p.G + head % p.G;
        // entry 0 is the tree's, the others the splits'
        const int entries = tab.y + 1, tree = p.B * p.nsplit + b;
        const auto at = [&](int e) { return row0 + (size_t)(e == 0 ? tree : tab.x + e - 1) * p.rows_padded; };
        for (int first = 0; first < entries; first += WIDTH) {
            const int e = first + lane;
            const float2 ml = e < entries ? p.part_ml[at(e)] : float2{-INFINITY, 0.f};
            float top = ml.x;
            for (int o = WIDTH / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
            const float next = fmaxf(ref, top), zero = next == -INFINITY ? 0.f : next;
            const float f = e < entries ? __builtin_amdgcn_exp2f(ml.x - zero) : 0.f, old = __builtin_amdgcn_exp2f(ref - zero);
            ref = next;
            float part = f * ml.y;
            for (int o = WIDTH / 2; o; o >>= 1) part += __shfl_xor(part, o);
            sum = sum * old + part;
            for (int j = 0; j < 8; j++) acc[j] *= old;
            const int here = min(WIDTH, entries - first);
            for (int j0 = 0; j0 < here; j0 += WORKERS * BATCH) {  // all lanes stay: the shuffles need them
                const int j = j0 + worker;
                float4 v[BATCH][2];
                float g[BATCH];
#pragma unroll
                for (int u = 0; u < BATCH; u++) {
                    const int k = min(j + u * WORKERS, here - 1);
                    const float4 *const src = reinterpret_cast<const float4 *>(p.part_o + at(first + k) * D + 8 * piece);
                    v[u][0] = src[0];
                    v[u][1] = src[1];
                }
#pragma unroll
                for (int u = 0; u < BATCH; u++) {
                    const int k = j + u * WORKERS;
                    g[u] = __shfl(f, min(k, here - 1), WIDTH);
                    if (k < here) {
                        acc[0] += g[u] * v[u][0].x; acc[1] += g[u] * v[u][0].y; acc[2] += g[u] * v[u][0].z; acc[3] += g[u] * v[u][0].w;
                        acc[4] += g[u] * v[u][1].x; acc[5] += g[u] * v[u][1].y; acc[6] += g[u] * v[u][1].z; acc[7] += g[u] * v[u][1].w;
                    }
                }
            }
        }
        for (int j = 0; j < 8; j++)
            for (int o = PIECES; o < WIDTH; o <<= 1) acc[j] += __shfl_xor(acc[j], o);
    }
    if (worker == 0) q4_finish<T>(p, b, t, head, piece, D, t < n, ref, sum, acc);
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
    if ((int64_t)h->Hkv * h->block_size > INT32_MAX || h->P_max > INT32_MAX - 4096) return ETV_ERR_UNSUPPORTED;
    if ((h->block_size > 0 ? (int64_t)h->num_blocks * h->Hkv * h->block_size : (int64_t)h->B * h->Hkv * h->P_cap) > UINT32_MAX) return ETV_ERR_UNSUPPORTED;
    if (h->P_max > (h->block_size > 0 ? (int64_t)h->max_blocks * h->block_size : (int64_t)h->P_cap)) return ETV_ERR_INVALID_ARG;
    if (h->scale != 0.f && !(fabsf(h->scale) >= 1e-30f && fabsf(h->scale) <= 1e30f)) return ETV_ERR_INVALID_ARG;  // also NaN
    if ((h->flags & ~ETV_ATTN_FLAG_GENERIC) != 0) return ETV_ERR_INVALID_ARG;
    return ETV_OK;
}

struct Q4Plan {
    int rw, row_groups, chunk, nsplit, span;
    int64_t slots, units;
    bool fits() const { return units * row_groups <= INT32_MAX - 65536; }  // in a grid, and every count of the kernel in 31 bits
    int rows_padded() const { return row_groups * 32 * rw; }
    size_t rows() const { return (size_t)units * rows_padded(); }
    size_t workspace(const etv_attn_desc *h) const { return nsplit == 1 ? 256 : rows() * ((size_t)h->d * 4 + 8) + (size_t)h->B * 8 + 256; }
};

static Q4Plan q4_plan(const etv_attn_desc *h) {
    Q4Plan pl{};
    const int rows = h->T_max * (h->Hq / h->Hkv), B = std::max(1, h->B);
    pl.rw = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    pl.row_groups = (rows + 32 * pl.rw - 1) / (32 * pl.rw);
    const int waves = q4_wavefronts(h->dtype == ETV_F32, pl.rw);
    pl.span = (pl.rw == 4 ? 64 : 32) * (waves / pl.rw);
    const int64_t seqs = (int64_t)B * h->Hkv;
    const int rounds = std::max(1, (h->P_max + pl.span - 1) / pl.span);  // of a workgroup over the longest prefix
    pl.nsplit = 1;
    if (h->kv_split > 0) {
        pl.chunk = (int)std::min<int64_t>((h->kv_split + (int64_t)pl.span - 1) / pl.span, rounds) * pl.span;
        pl.nsplit = std::max(1, (int)(((int64_t)h->P_max + pl.chunk - 1) / pl.chunk));
    } else {
        // Eight wavefronts a compute unit.  In units of a round: starting and ending a workgroup 3, the second launch 3 and a little more
        // for every split whose rows it reads.
        double least = 1e30;
        int per = rounds;
        for (int ns = 1; ns <= std::min(rounds, 128); ns++) {
            const int each = (rounds + ns - 1) / ns;
            if (ns > 1 && each == per) continue;
            const double full = (double)seqs * pl.row_groups * ns / (2048 / waves), turns = full < 4 ? std::ceil(full) : full + 0.5;
            const double cost = turns * (3 + each) + (ns > 1 ? 3 + 0.05 * ns + 1e-5 * (double)seqs * rows * ns : (h->T_max + pl.span - 1) / pl.span);
            if (cost < least) least = cost, pl.nsplit = ns, per = each;
        }
        pl.chunk = B <= 64 ? 0 : per * pl.span;
    }
    pl.slots = (int64_t)B * (pl.nsplit == 1 ? 1 : pl.nsplit + 1);
    pl.units = pl.slots * h->Hkv;
    return pl;
}

template <int D, bool F32, int RW, bool PAGED>
static int32_t launch_q4(const Q4Attn &p, unsigned grid, hipStream_t st) {
    constexpr int lds = Q4Geo<D, F32, RW>::LDS;
    static_assert(lds <= (Q4Geo<D, F32, RW>::NW == 8 ? 150 : 78) * 1024, "eight wavefronts a compute unit, and static LDS beside it");
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(attn_q4_kernel<D, F32, RW, PAGED>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) {
        g_last_hip_error = (int32_t)e;
        return ETV_ERR_HIP;
    }
    hipLaunchKernelGGL((attn_q4_kernel<D, F32, RW, PAGED>), dim3(grid), dim3(Q4Geo<D, F32, RW>::NW * 64), lds, st, p);
    return check_launch();
}

template <int D, bool F32, int RW>
static int32_t launch_q4_form(const Q4Attn &p, unsigned grid, hipStream_t st) {
    return p.block_size ? launch_q4<D, F32, RW, true>(p, grid, st) : launch_q4<D, F32, RW, false>(p, grid, st);
}

template <int D, bool F32>
static int32_t run_q4(const Q4Plan &pl, const Q4Attn &p, hipStream_t st) {
    const unsigned grid = (unsigned)((pl.units + 7) / 8 * 8 * pl.row_groups);
    const int32_t rc = pl.rw == 1 ? launch_q4_form<D, F32, 1>(p, grid, st) : pl.rw == 2 ? launch_q4_form<D, F32, 2>(p, grid, st) : launch_q4_form<D, F32, 4>(p, grid, st);
    if (rc != ETV_OK || pl.nsplit == 1) return rc;
    const int rows = p.T_max * p.Hq;
    if ((int64_t)rows * p.B <= 2048) hipLaunchKernelGGL((join_q4_kernel<D, F32, 64>), dim3((rows + 3) / 4, p.B), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((join_q4_kernel<D, F32, D / 8>), dim3((rows + 2048 / D - 1) / (2048 / D), p.B), dim3(256), 0, st, p);
    return check_launch();
}

}  // namespace etv

extern "C" size_t etv_tree_verify_attention_q4_workspace_bytes(const etv_attn_desc *h) {
    if (etv::q4_check_desc(h) != ETV_OK) return 0;
    const etv::Q4Plan pl = etv::q4_plan(h);
    return pl.fits() ? pl.workspace(h) : (h->flags & ETV_ATTN_FLAG_GENERIC) != 0 ? 256 : 0;
}

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
    // scales: whole rows.  (A layer of a contiguous cache, heads of 64, starts at a multiple of two bytes; they are read byte by byte.)
    if (align & 15 || ((uintptr_t)k_scales | (uintptr_t)v_scales) & (uintptr_t)(h->d / 32 - 1)) return ETV_ERR_INVALID_ARG;
    if (h->B == 0) return ETV_OK;
    const etv::Q4Plan pl = etv::q4_plan(h);
    const bool generic = (h->flags & ETV_ATTN_FLAG_GENERIC) != 0;
    if (!generic && !pl.fits()) return ETV_ERR_UNSUPPORTED;
    if (!generic && pl.nsplit > 1 && (!workspace || workspace_bytes < pl.workspace(h))) return ETV_ERR_WORKSPACE_TOO_SMALL;
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
    hipStream_t st = etv::as_stream(stream);
    if (generic) {
        const dim3 grid(h->T_max, h->Hq, h->B);
        if (h->dtype == ETV_F32 && h->d == 64) hipLaunchKernelGGL((etv::attn_q4_generic_kernel<float, 64>), grid, dim3(64), 0, st, p);
        else if (h->dtype == ETV_F32) hipLaunchKernelGGL((etv::attn_q4_generic_kernel<float, 128>), grid, dim3(64), 0, st, p);
        else if (h->d == 64) hipLaunchKernelGGL((etv::attn_q4_generic_kernel<uint16_t, 64>), grid, dim3(64), 0, st, p);
        else hipLaunchKernelGGL((etv::attn_q4_generic_kernel<uint16_t, 128>), grid, dim3(64), 0, st, p);
        return etv::check_launch();
    }
    p.chunk = pl.chunk; p.nsplit = pl.nsplit; p.slots = (int)pl.slots; p.row_groups = pl.row_groups; p.rows_padded = pl.rows_padded();
    p.units = (int)pl.units; p.span = pl.span;
    p.inv_g = etv::fast_div_inv(p.G); p.inv_hkv = etv::fast_div_inv(p.Hkv); p.inv_groups = etv::fast_div_inv(p.row_groups);
    p.inv_nsplit = etv::fast_div_inv(p.nsplit);
    if (pl.nsplit > 1) {
        p.part_o = static_cast<float *>(workspace);
        p.part_ml = reinterpret_cast<float2 *>(p.part_o + pl.rows() * h->d);
        p.split_tab = reinterpret_cast<int2 *>(p.part_ml + pl.rows());
    }
    if (h->dtype == ETV_F32) return h->d == 64 ? etv::run_q4<64, true>(pl, p, st) : etv::run_q4<128, true>(pl, p, st);
    return h->d == 64 ? etv::run_q4<64, false>(pl, p, st) : etv::run_q4<128, false>(pl, p, st);
}
