// The best continuations over beams and vocabulary: one pass over the logits, then a merge per request.
#include "etv_common.h"
#include <cfloat>
#include <type_traits>

namespace etv {

// --------------------------------------------------------------------------------------------------------------
// beam_select
// --------------------------------------------------------------------------------------------------------------
// What a wavefront leaves of its segment of one row, relative to the segment's largest logit, and the list of its best logits in order.
struct ScanHead {
    float m;    // largest logit, -inf: none
    int32_t n;  // candidates in the list
    double s;   // sum of exp(x - m); NaN where a logit is NaN or +inf
};
struct Candidate {
    float x;
    int32_t v;
};
constexpr int kScanCap = 384;    // candidates a segment collects before it falls back on one round per candidate
constexpr int kMaxSteps = 8;     // steps of a segment
constexpr int kMergeCap = 1024;  // candidates a request collects, as in a segment

// What a beam offers: nothing, its end token, or its row of logits.
enum { kBeamNone, kBeamDone, kBeamLive, kBeamBad };
__device__ __forceinline__ int beam_state(const etv_beam_desc &dsc, const float *scores, const int32_t *n_beams, const uint8_t *finished, int b, int k) {
    if (n_beams && k >= n_beams[b]) return kBeamNone;
    const float s = scores[(size_t)b * dsc.K + k];
    if (!(s < INFINITY)) return kBeamBad;
    if (s == -INFINITY) return kBeamNone;
    return finished && finished[(size_t)b * dsc.K + k] ? kBeamDone : kBeamLive;
}

// Sixteen bytes of a row of logits, which begins at any element; `get` makes them fp32 where they are used, which keeps bf16 in half the registers.
template <class T>
struct Logits;
template <>
struct Logits<float> {
    static constexpr int N = 4;
    typedef float vec __attribute__((ext_vector_type(4)));
    typedef float vec_at __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ float get(const vec &u, int i) { return u[i]; }
    static __device__ void set(vec &u, int i, float x) { u[i] = x; }
    static __device__ float none() { return -INFINITY; }
    static __device__ float one(float x) { return x; }
};
template <>
struct Logits<uint16_t> {
    static constexpr int N = 8;
    typedef unsigned int vec __attribute__((ext_vector_type(4)));
    typedef unsigned int vec_at __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ float get(const vec &u, int i) { return __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16); }
    static __device__ void set(vec &u, int i, uint16_t x) { u[i / 2] = i & 1 ? (u[i / 2] & 0xffffu) | (uint32_t)x << 16 : (u[i / 2] & 0xffff0000u) | x; }
    static __device__ uint16_t none() { return 0xff80; }
    static __device__ float one(uint16_t x) { return bf16_bits_to_float(x); }
};

// The largest of three.  (fmaxf costs an instruction more for each operand that might be a signalling NaN; one here makes the sum NaN.)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Order of fp32 numbers as unsigned integers, and back.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// A number that at least R of the wavefront's 64 values of x reach, none below -FLT_MAX: the R-th largest with the low 16 of its 32 bits cut off,
// found bit by bit.
__device__ __forceinline__ float reached_by(float x, int R) {
    const uint32_t key = order_of(x) >> 16;
    uint32_t cut = 0;
#pragma unroll
    for (int bit = 15; bit >= 0; bit--) {
        const uint32_t trial = cut | 1u << bit;
        if (__popcll(__ballot(key >= trial)) >= R) cut = trial;
    }
    if (cut <= 0x007fu) return -FLT_MAX;  // the order of -inf
    const uint32_t full = cut << 16;
    return __uint_as_float(full & 0x80000000u ? full ^ 0x80000000u : ~full);
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double s_part[4];
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (s_part[0] + s_part[1]) + (s_part[2] + s_part[3]);
}

// The largest key, of equal ones that with the lowest place, over the workgroup.
template <class K, class P>
__device__ __forceinline__ void block_best(K &key, P &place) {
    __shared__ K s_key[4];
    __shared__ P s_place[4];
    const auto take = [&](K k, P p) {
        if (k > key || (k == key && p < place)) key = k, place = p;
    };
    for (int off = 32; off >= 1; off >>= 1) {
        const K k = __shfl_xor(key, off);
        const P p = __shfl_xor(place, off);
        take(k, p);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_key[threadIdx.x >> 6] = key, s_place[threadIdx.x >> 6] = place;
    __syncthreads();
    for (int w = 0; w < 4; w++) take(s_key[w], s_place[w]);
}

constexpr double kLog2e = 1.4426950408889634;

// 2^z for -1000 <= z <= 0, to 1.9e-9 of itself: a whole number n, taken off by a sum whose last bit is a one, and a polynomial in what is left (the
// smallest relative error on [-1/2, 1/2] at its degree, by Remez's exchange); n goes into the exponent.
__device__ __forceinline__ double exp2_fast(double z) {
    const double shifted = z + 6755399441055744.0;  // 1.5 * 2^52
    const double f = z - (shifted - 6755399441055744.0);
    double p = 0.0001534581201908092;
    p = fma(p, f, 0.0013399931219370265);
    p = fma(p, f, 0.0096184889570621);
    p = fma(p, f, 0.05550328776964647);
    p = fma(p, f, 0.24022646890634475);
    p = fma(p, f, 0.6931472057372681);
    p = fma(p, f, 1.0000000005541663);
    return __hiloint2double(__double2hiint(p) + (__double2loint(shifted) << 20), __double2loint(p));
}

// exp(t) for t <= 0 in fp32: within 2^-23 (1 + |t|) of itself, and without an error that many terms have in common: log2(e) is in two parts, and
// what the hardware's 2^y is off by in the mean (-3.4e-9, measured) is taken out of the sums.
__device__ __forceinline__ float term(float t) { return __builtin_amdgcn_exp2f(fmaf(t, 1.44269502f, t * 1.92596299e-8f)); }
constexpr double kTermMean = 1 + 3.4e-9;

// A segment of one row of logits by one wavefront: `steps` times 64 lanes' four vectors, the next step's on their way while one is worked on.  Every
// logit takes part in the running sum; of the order only the largest of each lane's sixteen or thirty-two is kept.  Those bound the M-th best of
// the segment from below (a number that M lanes reach), and the few vectors that reach the bound are read again, from the caches, for
// the candidates, which are ranked by counting.
template <class T>
__global__ void __launch_bounds__(64) beam_scan_kernel(etv_beam_desc dsc, const T *logits, const float *scores, const int32_t *n_beams,
                                                       const uint8_t *finished, int splits, int steps, int list, ScanHead *heads, Candidate *cands) {
    constexpr int N = Logits<T>::N, G = 4, E = G * N;
    __shared__ float s_most[kMaxSteps * 64];
    __shared__ Candidate s_cand[kScanCap];
    __shared__ int s_n;
    const int row = blockIdx.x / splits, split = blockIdx.x - row * splits, b = row / dsc.K, k = row - b * dsc.K, t = threadIdx.x;
    if (beam_state(dsc, scores, n_beams, finished, b, k) != kBeamLive) return;
    const T *x = logits + b * dsc.batch_stride + k * dsc.row_stride;
    const int V = dsc.V, v_begin = split * (64 * E * steps), v_end = min(V, v_begin + 64 * E * steps);
    // Vector g of a step begins at place(): the row's last N logits stand in for a vector that would leave the row, without those of
    // them that belong to the vectors before.
    const auto place = [&](int step, int g) { return v_begin + (step * G + g) * 64 * N + t * N; };
    typedef typename Logits<T>::vec vec;
    const auto load = [&](vec *raw, int step) {
#pragma unroll
        for (int g = 0; g < G; g++) {
            const int v = place(step, g), at = min(v, V - N);
            raw[g] = vec{};
            if (V >= N) raw[g] = *reinterpret_cast<const typename Logits<T>::vec_at *>(x + at);
            else
                for (int j = 0; j < V; j++) Logits<T>::set(raw[g], j + N - V, x[j]);
        }
    };
    const auto mask = [&](vec *raw, int step) {  // only where a step reaches behind the row
#pragma unroll
        for (int g = 0; g < G; g++) {
            const int v = place(step, g), at = min(v, V - N);
#pragma unroll
            for (int j = 0; j < N; j++)
                if (at + j < v) Logits<T>::set(raw[g], j, Logits<T>::none());
        }
    };
    if (t == 0) s_n = 0;
    vec raw[G];
    load(raw, 0);
    float ref = -INFINITY, best = -INFINITY;
    double s = 0;
    int step = 0;
    for (; step < steps && place(step, 0) - t * N < v_end; step++) {
        vec next[G];
        if (step + 1 < steps) load(next, step + 1);
        if (place(step + 1, 0) - t * N > V) mask(raw, step);
        float r[E], most = -INFINITY;
#pragma unroll
        for (int i = 0; i < E; i++) r[i] = Logits<T>::get(raw[i / N], i % N);
#pragma unroll
        for (int i = 0; i < E; i += 2) most = max3(r[i], r[i + 1], most);
        s_most[step * 64 + t] = most;
        best = fmaxf(best, most);
        const float top = wave_best(most, [](float p, float q) { return fmaxf(p, q); });
        if (top > ref) {
            s *= exp2_fast(fmax(((double)ref - (double)top) * kLog2e, -1000.0));
            ref = top;
        }
        // NaN and +inf make the sum NaN; before the first logit that is neither masked nor NaN there is nothing but zeros and NaN to add
        const float from = ref > -INFINITY ? ref : 0;
        float part[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < E; i++) part[i % 4] += term(r[i] - from);
        s += (double)(part[0] + part[1]) + (double)(part[2] + part[3]);
#pragma unroll
        for (int g = 0; g < G; g++) raw[g] = next[g];
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
    s *= kTermMean;
    const float cut = reached_by(best, dsc.M);
    uint32_t todo = 0;
    for (int i = 0; i < step; i++) todo |= (s_most[i * 64 + t] >= cut) << i;
    while (todo) {
        const int i = __builtin_ctz(todo);
        todo &= todo - 1;
        load(raw, i);
        mask(raw, i);
#pragma unroll
        for (int j = 0; j < E; j++) {
            const float y = Logits<T>::get(raw[j / N], j % N);
            if (y >= cut) {
                const int at = atomicAdd(&s_n, 1);
                if (at < kScanCap) s_cand[at] = {y, min(place(i, j / N), V - N) + j % N};
            }
        }
    }
    __syncthreads();
    Candidate *out = cands + (size_t)blockIdx.x * list;
    int n = s_n;
    if (n <= kScanCap) {
        for (int i = t; i < n; i += 64) {
            const Candidate own = s_cand[i];
            int rank = 0;
            for (int j = 0; j < n; j++) {
                const Candidate o = s_cand[j];
                rank += o.x > own.x || (o.x == own.x && o.v < own.v);
            }
            if (rank < dsc.M) out[rank] = own;
        }
    } else {  // many equal ones: the next best after the last, a round each
        Candidate last = {INFINITY, -1};
        for (n = 0; n < dsc.M; n++) {
            Candidate own = {-INFINITY, INT32_MAX};
            for (int v = v_begin + t; v < v_end; v += 64) {
                const float y = Logits<T>::one(x[v]);
                if ((y < last.x || (y == last.x && v > last.v)) && y > own.x) own = {y, v};
            }
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) {
                const Candidate o = {__shfl_xor(own.x, off), __shfl_xor(own.v, off)};
                if (o.x > own.x || (o.x == own.x && o.v < own.v)) own = o;
            }
            if (own.x == -INFINITY) break;
            if (t == 0) out[n] = own;
            last = own;
        }
    }
    if (t == 0) heads[blockIdx.x] = {ref, min(n, dsc.M), s};
}

// A request: the logarithms of its beams' sums, then the M best of all candidates.
//   total = (x - largest logit) + (score - log of the sum relative to it): nothing is lost where logits are large
// As in the scan: a bound on the M-th best from below, here from the heads of the lists, then only those above it.  Where two beams' totals next to each
// other are closer than their sums are good for, these are taken again in 64 bits from the logits, and the order with them.
template <class T>
__global__ void __launch_bounds__(256) beam_merge_kernel(etv_beam_desc dsc, const T *logits, const float *scores, const int32_t *n_beams,
                                                         const uint8_t *finished, int splits, int list, const ScanHead *heads, const Candidate *cands,
                                                         float *out_scores, int32_t *parent, int32_t *token, uint8_t *finished_out, int32_t *status) {
    constexpr double kClose = 0x1p-22;
    __shared__ double s_base[ETV_MAX_BEAMS], s_max[ETV_MAX_BEAMS];
    __shared__ int s_state[ETV_MAX_BEAMS], s_status, s_n;
    __shared__ float s_cut[4];
    __shared__ double s_total[kMergeCap], s_best[ETV_MAX_BEAMS];
    __shared__ long s_place[kMergeCap], s_best_place[ETV_MAX_BEAMS];
    __shared__ unsigned int s_again[2];
    const int b = blockIdx.x, t = threadIdx.x;
    const long V = dsc.V;
    const int lists = dsc.K * splits, M = dsc.M;
    heads += (size_t)b * lists;
    cands += (size_t)b * lists * list;
    if (t == 0) s_status = 0;
    if (t < 2) s_again[t] = 0;
    __syncthreads();
    // as many lanes a beam as it has segments, up to a wavefront
    const int width = splits > 32 ? 64 : splits > 16 ? 32 : splits > 8 ? 16 : splits > 4 ? 8 : splits > 2 ? 4 : splits;
    for (int k0 = 0; k0 < dsc.K; k0 += 256 / width) {
        const int k = k0 + t / width, lane = t % width;
        int state = k < dsc.K ? beam_state(dsc, scores, n_beams, finished, b, k) : kBeamNone;
        double base = 0, most = 0;
        float m = -INFINITY;
        double s = 0;
        const auto scale = [](float from, float to) { return from > -INFINITY && from != to ? exp2_fast(fmax(((double)from - (double)to) * kLog2e, -1000.0)) : 1.0; };
        if (state == kBeamLive)
            for (int i = lane; i < splits; i += width) {  // running: the sum is relative to the largest so far
                const ScanHead h = heads[k * splits + i];
                const float top = fmaxf(m, h.m);
                s = s * scale(m, top) + h.s * scale(h.m, top);  // without a logit: 0, or NaN
                m = top;
            }
        for (int off = 1; off < width; off <<= 1) {
            const float om = __shfl_xor(m, off), top = fmaxf(m, om);
            const double os = __shfl_xor(s, off) * scale(om, top), is = s * scale(m, top);
            s = t & off ? os + is : is + os;
            m = top;
        }
        if (k < dsc.K && lane == 0) {
            base = scores[(size_t)b * dsc.K + k];
            if (state == kBeamLive) {
                if (!(s < INFINITY)) {
                    atomicOr(&s_status, ETV_BEAM_BAD_LOGITS);
                    state = kBeamNone;
                }
                base -= log(s);
                most = m;
            } else if (state == kBeamBad) {
                atomicOr(&s_status, ETV_BEAM_BAD_SCORE);
                state = kBeamNone;
            }
            s_base[k] = base, s_max[k] = most, s_state[k] = state;
        }
    }
    __syncthreads();
    // entry i of list l
    const auto entries = [&](int l) {
        const int state = s_state[l / splits];
        return state == kBeamLive ? heads[l].n : state == kBeamDone && l % splits == 0 ? 1 : 0;
    };
    const auto entry = [&](int l, int i, double &x, long &place) {
        const int k = l / splits;
        if (s_state[k] == kBeamLive) {
            const Candidate c = cands[(size_t)l * list + i];
            x = ((double)c.x - s_max[k]) + s_base[k];
            place = k * V + c.v;
        } else {
            x = s_base[k];
            place = k * V + dsc.end_token;
        }
    };
    int n;
    for (int round = 0;; round++) {
        float top = -INFINITY;
        for (int l = t; l < lists; l += 256)
            if (entries(l) > 0) {
                double x;
                long place;
                entry(l, 0, x, place);
                top = fmaxf(top, (float)x);
            }
        const float mine = reached_by(top, M);
        if (t == 0) s_n = 0;
        if ((t & 63) == 0) s_cut[t >> 6] = mine;
        __syncthreads();
        float cut = fmaxf(fmaxf(s_cut[0], s_cut[1]), fmaxf(s_cut[2], s_cut[3]));
        cut = fmaxf(cut - fmaxf(fabsf(cut) * 0x1p-21f, 0x1p-20f), -FLT_MAX);  // and those too close to it
        for (int l = t; l < lists; l += 256) {
            const int have = entries(l);
            for (int i = 0; i < have; i++) {
                double x;
                long place;
                entry(l, i, x, place);
                if (!((float)x >= cut)) break;
                const int at = atomicAdd(&s_n, 1);
                if (at < kMergeCap) s_total[at] = x, s_place[at] = place;
            }
        }
        __syncthreads();
        const int found = s_n;
        if (found <= kMergeCap) {
            for (int i = t; i < found; i += 256) {
                const double x = s_total[i];
                const long place = s_place[i];
                int rank = 0;
                for (int j = 0; j < found; j++) rank += s_total[j] > x || (s_total[j] == x && s_place[j] < place);
                if (rank < M) s_best[rank] = x, s_best_place[rank] = place;
            }
            n = min(found, M);
        } else {
            double last = INFINITY;
            long last_place = -1;
            for (n = 0; n < M; n++) {
                double best = -INFINITY;
                long at = INT64_MAX;
                for (int l = t; l < lists; l += 256) {
                    const int have = entries(l);
                    for (int i = 0; i < have; i++) {
                        double x;
                        long place;
                        entry(l, i, x, place);
                        if ((x < last || (x == last && place > last_place)) && (x > best || (x == best && place < at))) {
                            best = x, at = place;
                            break;  // a list is in order
                        }
                    }
                }
                block_best(best, at);
                if (best == -INFINITY) break;
                if (t == 0) s_best[n] = best, s_best_place[n] = at;
                last = best, last_place = at;
            }
        }
        __syncthreads();
        if (round) break;
        // Two totals of different beams too close to call: neighbours of the M best, or the last of them and one left out.  (Equal ones are those of
        // equal rows.)
        const auto call = [&](double x, long place, double y, long other) {
            const int k = (int)(place / V), k1 = (int)(other / V);
            if (k != k1 && x > y && x - y < kClose) {
                atomicOr(&s_again[k >> 5], 1u << (k & 31));
                atomicOr(&s_again[k1 >> 5], 1u << (k1 & 31));
            }
        };
        if (t + 1 < n) call(s_best[t], s_best_place[t], s_best[t + 1], s_best_place[t + 1]);
        if (n == M && found <= kMergeCap) {
            for (int i = t; i < found; i += 256) call(s_best[M - 1], s_best_place[M - 1], s_total[i], s_place[i]);
        } else if (n == M) {
            for (int l = t; l < lists; l += 256) {
                const int have = entries(l);
                for (int i = 0; i < have; i++) {
                    double x;
                    long place;
                    entry(l, i, x, place);
                    call(s_best[M - 1], s_best_place[M - 1], x, place);
                }
            }
        }
        __syncthreads();
        uint64_t again = s_again[0] | (uint64_t)s_again[1] << 32;
        if (!again) break;
        for (; again; again &= again - 1) {
            const int k = __builtin_ctzll(again);
            if (s_state[k] != kBeamLive) continue;
            const T *x = logits + b * dsc.batch_stride + k * dsc.row_stride;
            double s = 0;
            for (int v = t; v < dsc.V; v += 256) s += exp2_fast(fmax(((double)Logits<T>::one(x[v]) - s_max[k]) * kLog2e, -1000.0));
            s = block_sum(s);
            // to multiples of 2^-40: rows with the same logits in another order tie, whatever order they were added in
            if (t == 0) s_base[k] = rint(((double)scores[(size_t)b * dsc.K + k] - log(s)) * 0x1p40) * 0x1p-40;
        }
        __syncthreads();
    }
    if (t < M) {
        const bool found = t < n;
        const long place = found ? s_best_place[t] : 0;
        const int k = (int)(place / V), v = (int)(place - k * V);
        const size_t o = (size_t)b * M + t;
        out_scores[o] = found ? (float)s_best[t] : -INFINITY;
        parent[o] = found ? k : -1;
        token[o] = found ? v : -1;
        if (finished_out) finished_out[o] = found && (s_state[k] == kBeamDone || v == dsc.end_token);
    }
    if (t == 0) status[b] = s_status | (n < M ? ETV_BEAM_SHORT : 0);
}

// Steps of a wavefront's segment: more of them mean fewer lists to merge, fewer more wavefronts.
static int beam_step(const etv_beam_desc *h) { return 64 * (h->dtype == ETV_BF16 ? 32 : 16); }
static int beam_steps(const etv_beam_desc *h) {
    const int64_t rows = (int64_t)h->B * h->K, all = (h->V + beam_step(h) - 1) / beam_step(h);
    int n = 1;
    while (n < kMaxSteps && rows * ((all + 2 * n - 1) / (2 * n)) >= 4096) n *= 2;
    return n;
}
static int beam_splits(const etv_beam_desc *h) {
    const int64_t segment = (int64_t)beam_step(h) * beam_steps(h);
    return (int)((h->V + segment - 1) / segment);
}

static int beam_list(const etv_beam_desc *h) { return (h->M + 3) & ~3; }

static int32_t check_beam(const etv_beam_desc *h) {
    if (!h || h->B < 0 || h->K < 1 || h->M < 1 || h->V < 1 || h->end_token < -1 || h->end_token >= h->V) return ETV_ERR_INVALID_ARG;
    if (h->K > 1 && h->row_stride < h->V) return ETV_ERR_INVALID_ARG;
    if (h->B > 1 && h->batch_stride < 0) return ETV_ERR_INVALID_ARG;
    if (h->dtype != ETV_F32 && h->dtype != ETV_BF16) return ETV_ERR_UNSUPPORTED;
    if (h->K > ETV_MAX_BEAMS || h->M > ETV_MAX_BEAMS || h->V > INT32_MAX - 65536) return ETV_ERR_UNSUPPORTED;
    if ((int64_t)h->B * h->K * beam_splits(h) > INT32_MAX) return ETV_ERR_UNSUPPORTED;
    return ETV_OK;
}

}  // namespace etv

extern "C" size_t etv_beam_select_workspace_bytes(const etv_beam_desc *h) {
    if (etv::check_beam(h) != ETV_OK) return 0;
    const size_t lists = (size_t)h->B * h->K * etv::beam_splits(h);
    return lists * (sizeof(etv::ScanHead) + etv::beam_list(h) * sizeof(etv::Candidate));
}

extern "C" int32_t etv_beam_select(const etv_beam_desc *h, const void *logits, const float *scores, const int32_t *n_beams, const uint8_t *finished,
                                   float *out_scores, int32_t *parent, int32_t *token, uint8_t *finished_out, int32_t *status, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    const int32_t rc = etv::check_beam(h);
    if (rc != ETV_OK) return rc;
    if (h->B == 0) return ETV_OK;
    if (!logits || !scores || !out_scores || !parent || !token || !status || (finished && h->end_token < 0)) return ETV_ERR_INVALID_ARG;
    if ((uintptr_t)logits % (h->dtype == ETV_BF16 ? 2 : 4) || (uintptr_t)workspace & 15) return ETV_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < etv_beam_select_workspace_bytes(h)) return ETV_ERR_WORKSPACE_TOO_SMALL;
    const int splits = etv::beam_splits(h), list = etv::beam_list(h), steps = etv::beam_steps(h);
    const unsigned lists = (unsigned)h->B * h->K * splits;
    auto *heads = static_cast<etv::ScanHead *>(workspace);
    auto *cands = reinterpret_cast<etv::Candidate *>(heads + lists);
    hipStream_t s = etv::as_stream(stream);
    const auto run = [&](auto *x) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(x)>>;
        hipLaunchKernelGGL(etv::beam_scan_kernel<T>, dim3(lists), dim3(64), 0, s, *h, x, scores, n_beams, finished, splits, steps, list, heads, cands);
        const int32_t rc = etv::check_launch();
        if (rc != ETV_OK) return rc;
        hipLaunchKernelGGL(etv::beam_merge_kernel<T>, dim3(h->B), dim3(256), 0, s, *h, x, scores, n_beams, finished, splits, list, heads, cands, out_scores,
                           parent, token, finished_out, status);
        return etv::check_launch();
    };
    return h->dtype == ETV_BF16 ? run(static_cast<const uint16_t *>(logits)) : run(static_cast<const float *>(logits));
}
