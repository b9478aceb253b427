// The best continuations over beams and vocabulary, total[k, v] = score[k] + x[k, v] - log sum_v' exp(x[k, v']): one pass over the logits, which
// leaves of every segment of a row its sum relative to a reference and its M best logits in order, then a merge per request.  Floor: the
// logits of the live beams once; 32 requests of 8 beams, 7 of them live, with 128000 bf16 logits are 57.3 MB, 8.0 us at the rate of a
// large read (7.15 TB/s).  The call takes 20.8 us there: the scan 16.6, the merge 6.6.
#include "etv_common.h"
#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace etv {

// What a wavefront leaves of its segment of one row: a sum, and the list of its best logits in order.
struct ScanHead {
    float m;    // the segment's reference, its largest logit or up to kSlack less; -inf: it has none
    int32_t n;  // candidates in the list
    double s;   // sum of exp(x - m); NaN where a logit is NaN or +inf
};
struct Candidate {
    float x;
    int32_t v;
};
constexpr int kMaxSteps = 16;    // steps of a segment
constexpr int kMergeThreads = 512;
constexpr int kThin = 320;       // candidates that are ranked as they are
constexpr int kMergeCap = 2048;  // candidates that a request collects; where more are close to its M-th best it looks for one after the other

// What a beam offers: nothing, its end token, or its row of logits.
enum { kBeamNone, kBeamDone, kBeamLive, kBeamBad };
__device__ __forceinline__ int beam_state(const etv_beam_desc &dsc, const float *scores, const int32_t *n_beams, const uint8_t *finished, int b, int k) {
    // asked for together
    const int beams = n_beams ? n_beams[b] : dsc.K;
    const float s = scores[(size_t)b * dsc.K + k];
    const int done = finished ? finished[(size_t)b * dsc.K + k] : 0;
    return k >= beams || s == -INFINITY ? kBeamNone : !(s < INFINITY) ? kBeamBad : done ? kBeamDone : kBeamLive;
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
    // the first n are not there
    static __device__ void drop(vec &u, int n) {
        for (int i = 0; i < 4; i++) u[i] = i < n ? -INFINITY : u[i];
    }
    static __device__ float one(float x) { return x; }
};
template <>
struct Logits<uint16_t> {
    static constexpr int N = 8;
    typedef unsigned int vec __attribute__((ext_vector_type(4)));
    typedef unsigned int vec_at __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ float get(const vec &u, int i) { return __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16); }
    static __device__ void set(vec &u, int i, uint16_t x) { u[i / 2] = i & 1 ? (u[i / 2] & 0xffffu) | (uint32_t)x << 16 : (u[i / 2] & 0xffff0000u) | x; }
    static __device__ void drop(vec &u, int n) {
        for (int i = 0; i < 4; i++) u[i] = 2 * i + 1 < n ? 0xff80ff80u : 2 * i < n ? (u[i] & 0xffff0000u) | 0xff80u : u[i];
    }
    static __device__ float one(uint16_t x) { return bf16_bits_to_float(x); }
};

// The largest of nine.  (fmaxf costs an instruction more for each operand that might be a signalling NaN; one here makes the sum NaN.)
__device__ __forceinline__ float max9(float m, const float *x) {
    asm("v_max3_f32 %0, %1, %2, %0\n\tv_max3_f32 %0, %3, %4, %0\n\tv_max3_f32 %0, %5, %6, %0\n\tv_max3_f32 %0, %7, %8, %0"
        : "+v"(m)
        : "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "v"(x[4]), "v"(x[5]), "v"(x[6]), "v"(x[7]));
    return m;
}

// Order of fp32 numbers as unsigned integers, and back.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order); }

// The least number whose order has these upper 16 bits, -FLT_MAX for that of -inf.
__device__ __forceinline__ float least_of(uint32_t key) {
    if (key <= 0x007fu) return -FLT_MAX;
    return number_of(key << 16);
}

// A number that at least R values reach, none below -FLT_MAX: the R-th largest with the low 16 of its 32 bits cut off, found bit by bit.  `count` tells how
// many have a key of at least its argument.
template <int UNROLL = 16, class F>
__device__ __forceinline__ float reached_by(F count, int R) {
    uint32_t cut = 0;
#pragma unroll UNROLL
    for (int bit = 15; bit >= 0; bit--) {
        const uint32_t trial = cut | 1u << bit;
        if (count(trial) >= R) cut = trial;
    }
    return least_of(cut);
}

// The largest, and the sum, over 2^width neighbouring lanes, in each of them: within a row of sixteen by lane moves of the vector unit.
template <int CTRL>
__device__ __forceinline__ float moved(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false)); }
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, false), __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, false));
}
template <class V, class F>
__device__ __forceinline__ V lanes_join(V v, int width, F f) {
    if (width > 0) v = f(v, moved<0xb1>(v));   // the neighbour: quads (1, 0, 3, 2)
    if (width > 1) v = f(v, moved<0x4e>(v));   // the other pair: quads (2, 3, 0, 1)
    if (width > 2) v = f(v, moved<0x141>(v));  // the other quad, whose lanes are alike: halves of a row mirrored
    if (width > 3) v = f(v, moved<0x140>(v));  // the other half: rows mirrored
    if (width > 4) v = f(v, __shfl_xor(v, 16));
    if (width > 5) v = f(v, __shfl_xor(v, 32));
    return v;
}
__device__ __forceinline__ float lanes_sum(float v, int width) { return lanes_join(v, width, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float lanes_best(float v, int width) { return lanes_join(v, width, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ double lanes_sum(double v, int width) { return lanes_join(v, width, [](double a, double b) { return a + b; }); }

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double s_part[kMergeThreads / 64];
    v = lanes_sum(v, 6);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < kMergeThreads / 64; w++) v += s_part[w];
    return v;
}

// The largest key, of equal ones that with the lowest place, over the workgroup.
template <class K, class P>
__device__ __forceinline__ void block_best(K &key, P &place) {
    __shared__ K s_key[kMergeThreads / 64];
    __shared__ P s_place[kMergeThreads / 64];
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
    for (int w = 0; w < kMergeThreads / 64; w++) take(s_key[w], s_place[w]);
}

constexpr double kLog2e = 1.4426950408889634;

// 2^z for |z| <= 1000, to 1.9e-9 of itself: a whole number n, taken off by a sum whose last bit is a one, and a polynomial in what is left (the
// smallest relative error on [-1/2, 1/2] at its degree, by Remez's exchange); n goes into the exponent.  For the few exponentials that join sums, and
// for sums that are taken again.
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

// exp(x) / 2^r in fp32, for a t = x - r ln(2) up to kSlack and |x| where it is not 0 up to kFarthest: within 2^-23 (1 + |t|) of itself.  log2(e) is in two
// parts, and the first product is rounded behind the subtraction.  The second one is less than half a unit of an exponent of 1 or more and mostly rounds
// away there, so that terms have an error in common: with it sums over logits of normal distribution are off by 1e-8 to 1e-7, within that bound.  What the
// hardware's 2^y is off by in the mean (-3.4e-9, measured) is taken out of the sums.  (In 64 bits all exponentials take the scan 35 us where these take 17.)
__device__ __forceinline__ float term(float x, float r) { return __builtin_amdgcn_exp2f(fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269502f, -r))); }
constexpr double kTermMean = 1 + 3.4e-9;
constexpr float kSlack = 1, kFarthest = 1 << 20;

// A segment of one row of logits by one wavefront: `steps` times 64 lanes' four vectors, the next step's on their way while one is worked on.  Every
// logit takes part in the running sum; of the order only the largest of every two vectors is kept, the best two of them for each lane.  Those bound the
// M-th best of the segment from below (a number that M of them reach), and the few vectors that reach the bound are read again, from the
// caches, for the candidates, which are ranked by counting.  TINY: fewer logits than a vector holds.
// One wavefront a workgroup, so that no barrier stops the stream.  Bounds: memory and the vector unit where rows are many -- of the 16.6 us above the
// loads alone take 11.5 and the vector instructions, 9.4 a logit, some 7.6; the rest are bound, candidates and ranking --, and the chain load, work, bound,
// candidates where they are few: 4 rows of 32000 fp32 logits 4.6 us, of which an empty launch is some 2.  Measured and left: wavefronts that go from
// segment to segment with the next one's first loads under way (half a us to two longer: 135 registers leave 12 of them a CU, 86 leave 20).
template <class T, bool TINY>
__global__ void __launch_bounds__(64) beam_scan_kernel(etv_beam_desc dsc, const T *logits, const float *scores, const int32_t *n_beams,
                                                       const uint8_t *finished, int splits, uint32_t inv_splits, uint32_t inv_K, int steps, int list, int room,
                                                       ScanHead *heads, Candidate *cands) {
    constexpr int N = Logits<T>::N, G = 4, E = G * N;
    extern __shared__ __attribute__((aligned(16))) Candidate s_cand[];  // [room + 16]
    float *s_most = reinterpret_cast<float *>(s_cand + room + 16);       // [steps][64]
    __shared__ int s_n;
    uint32_t split, k;
    const int t = threadIdx.x;
    const uint32_t row = fast_div(blockIdx.x, splits, inv_splits, split), b = fast_div(row, dsc.K, inv_K, k);
    const T *x = logits + b * dsc.batch_stride + k * dsc.row_stride;
    const int V = dsc.V, v_begin = (int)split * (64 * E * steps), v_end = min(V, v_begin + 64 * E * steps);
    // Vector g of a step begins at place(): the row's last N logits stand in for a vector that would leave the row, without those of
    // them that belong to the vectors before.
    const auto place = [&](int step, int g) { return v_begin + (step * G + g) * 64 * N + t * N; };
    typedef typename Logits<T>::vec vec;
    const auto load = [&](vec *raw, int step) {
#pragma unroll
        for (int g = 0; g < G; g++) {
            const int v = place(step, g), at = min(v, V - N);
            if (!TINY) raw[g] = *reinterpret_cast<const typename Logits<T>::vec_at *>(x + at);
            else {
                raw[g] = vec{};
#pragma unroll
                for (int j = 0; j < N; j++) Logits<T>::set(raw[g], j, x[max(at + j, 0)]);
            }
        }
    };
    const auto mask = [&](vec *raw, int step) {  // only where a step reaches behind the row
#pragma unroll
        for (int g = 0; g < G; g++) Logits<T>::drop(raw[g], place(step, g) - min(place(step, g), V - N));
    };
    if (t == 0) s_n = 0;
    vec raw[G];
    load(raw, 0);
    if (beam_state(dsc, scores, n_beams, finished, b, k) != kBeamLive) return;
    float ref = -INFINITY, ref2 = 0, best = -INFINITY, second = -INFINITY;
    double s = 0;
    const auto work = [&](const vec *raw, int step) {
        float r[E], half[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < E; i++) r[i] = Logits<T>::get(raw[i / N], i % N);
#pragma unroll
        for (int i = 0; i < E / 2; i += 8) {
            half[0] = max9(half[0], r + i);
            half[1] = max9(half[1], r + E / 2 + i);
        }
        const float most = fmaxf(half[0], half[1]);
        s_most[step * 64 + t] = most;
        second = fmaxf(fmaxf(second, fminf(half[0], half[1])), fminf(best, most));
        best = fmaxf(best, most);
        // the reference is the largest logit, or up to 1 less: a wavefront's maximum is taken where it may have to move, at first above all
        if (__ballot(most > ref + kSlack)) {
            const float top = wave_best(most, [](float p, float q) { return fmaxf(p, q); });
            // Finite where -inf may still be added: exp2(-inf - -inf) would be NaN.
            const float top2 = fmaxf((float)(top * kLog2e), -FLT_MAX);
            // The sum up to here weighs nothing against 2^-1000 of what comes, and behind a reference of a mask's value it may be infinite, since ref2 is
            // then off by more than exponents of fp32: only whether it is a number goes on.  (A reference that moves less is exact enough: within a
            // segment such moves come from -kFarthest - 16 * 694 at most.)
            if (ref > -INFINITY) {
                if (((double)ref - (double)top) * kLog2e < -1000) s = s == s ? 0 : s;
                else s *= exp2_fast(fmax((double)ref2 - (double)top2, -1000.0));
            }
            ref = top, ref2 = top2;
        }
        // a NaN makes the sum NaN; before the first logit that is neither masked nor NaN there is nothing but zeros and NaN to add
        float part[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < E; i++) part[i % 4] += term(r[i], ref2);
        s += (double)(part[0] + part[1]) + (double)(part[2] + part[3]);
    };
    const int count = (v_end - v_begin + 64 * E - 1) / (64 * E);
    // a step ahead: the loop's loads are counted, so that it waits for the older ones alone
    for (int step = 0; step + 1 < count; step++) {
        vec next[G];
        load(next, step + 1);
        work(raw, step);
#pragma unroll
        for (int g = 0; g < G; g++) raw[g] = next[g];
    }
    const bool reaches_behind = v_begin + count * (64 * E) > V;
    if (reaches_behind) mask(raw, count - 1);
    work(raw, count - 1);
    const auto all = [&](auto f) {
        for (int v = v_begin + t; v < v_end; v += 64) f(v, Logits<T>::one(x[v]));
    };
    if (fabsf(ref) < kFarthest) s *= exp2_fast((double)ref2 - ref * kLog2e);  // relative to ref instead of what 32 bits hold of its logarithm
    else if (ref != -INFINITY) {  // the differences themselves; with +inf they make the sum NaN
        s = 0;
        all([&](int, float y) { s += term(y - ref, 0); });
    }
    s = lanes_sum(s, 6) * kTermMean;
    const uint32_t key = order_of(best) >> 16, key2 = order_of(second) >> 16;
    const float cut = reached_by([&](uint32_t c) { return __popcll(__ballot(key >= c)) + __popcll(__ballot(key2 >= c)); }, dsc.M);
    uint32_t todo = 0;
    for (int i = 0; i < count; i++) todo |= (s_most[i * 64 + t] >= cut) << i;
    while (todo) {
        const int i = __builtin_ctz(todo);
        todo &= todo - 1;
        if (count > 1) load(raw, i);  // a single step's are still here
        if (reaches_behind) mask(raw, i);
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < E; j++) hits |= (uint32_t)(Logits<T>::get(raw[j / N], j % N) >= cut) << j;
        while (hits) {
            const int j = __builtin_ctz(hits);
            hits &= hits - 1;
            const int v = min(place(i, j / N), V - N) + j % N, at = atomicAdd(&s_n, 1);
            if (at < room) s_cand[at].v = v;
        }
    }
    __syncthreads();
    Candidate *out = cands + (size_t)blockIdx.x * list;
    int n = s_n;
    if (n <= room) {  // their logits, all at once
        for (int i = t; i < n; i += 64) s_cand[i].x = Logits<T>::one(x[s_cand[i].v]);
        __syncthreads();
    } else {  // large ones side by side in a few lanes: a bound from all logits
        const float closer = reached_by<1>(
            [&](uint32_t c) {
                int mine = 0;
                all([&](int, float y) { mine += order_of(y) >> 16 >= c; });
                return (int)lanes_sum((float)mine, 6);
            },
            dsc.M);
        __syncthreads();
        if (t == 0) s_n = 0;
        __syncthreads();
        all([&](int v, float y) {
            if (!(y >= closer)) return;
            const int at = atomicAdd(&s_n, 1);
            if (at < room) s_cand[at] = {y, v};
        });
        __syncthreads();
        n = s_n;
    }
    if (n <= room && n > dsc.M + 32) {  // ranking takes n^2 steps: first those below a closer bound go
        const auto closer_by = [&](auto at_most) {
            constexpr int A = decltype(at_most)::value;
            uint32_t keys[A];
#pragma unroll
            for (int i = 0; i < A; i++) keys[i] = i * 64 + t < n ? order_of(s_cand[i * 64 + t].x) >> 16 : 0;
            return reached_by<1>(
                [&](uint32_t c) {
                    int all = 0;
#pragma unroll
                    for (int i = 0; i < A; i++) all += __popcll(__ballot(keys[i] >= c));
                    return all;
                },
                dsc.M);
        };
        const float closer = n <= 256 ? closer_by(std::integral_constant<int, 4>{}) : closer_by(std::integral_constant<int, 16>{});  // of `room` at its largest
        int kept = 0;
        for (int i0 = 0; i0 < n; i0 += 64) {  // closing up behind the reads
            const Candidate own = s_cand[min(i0 + t, n - 1)];
            const bool keep = i0 + t < n && own.x >= closer;
            const uint64_t lanes = __ballot(keep);
            __syncthreads();
            if (keep) s_cand[kept + __popcll(lanes & ((1ull << t) - 1))] = own;
            kept += __popcll(lanes);
        }
        n = kept;
        __syncthreads();
    }
    if (n <= room) {
        // as one number each, larger for a larger logit (of which -0 is 0) and a lower place
        static_assert(sizeof(Candidate) == sizeof(uint64_t), "one number each");
        for (int i = t; i < n; i += 64) {
            const Candidate own = s_cand[i];
            s_cand[i] = __builtin_bit_cast(Candidate, (uint64_t)order_of(own.x + 0.0f) << 32 | ~(uint32_t)own.v);
        }
        if (t < 16) s_cand[n + t] = {0, 0};  // to a multiple of sixteen
        __syncthreads();
        const auto order = [&](int i) { return __builtin_bit_cast(uint64_t, s_cand[i]); };
        for (int i = t >> 2; i < n; i += 16) {  // four lanes a candidate, with a quarter of the others each
            const uint64_t own = order(i);
            int above = 0;
#pragma unroll 1
            for (int j0 = t & 3; j0 < n; j0 += 16)
#pragma unroll
                for (int j = j0; j < j0 + 16; j += 4) above += order(j) > own;
            const float rank = lanes_sum((float)above, 2);
            if (rank < dsc.M && (t & 3) == 0) out[(int)rank] = {number_of((uint32_t)(own >> 32)), (int32_t)~(uint32_t)own};
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
//   total = (x - reference) + (score - log of the sum relative to it): nothing is lost where logits are large
// As in the scan: a bound on the M-th best from below, here from the heads of the lists, then only those above it.  Where two beams' totals next to each
// other are closer than their sums are good for, these are taken again from the logits, with exp2_fast and, if that does not tell either, with exponentials
// of full precision: so the order is that of 64-bit sums.  A sum is good to 2^-23 times 1 + kSlack + 5 (ten additions in 32 bits) + the mean of max - x over its weights, which is at most ln V.
// Bound by the chain of its loads and barriers: 5.2 us for one request of 4 beams, 6.6 for 32 of 8 beams with 8 lists each.  A scan whose
// last workgroup merges would save this launch's 4 us on the host, but needs a counter that somebody clears, and a release to the whole device by every wavefront.
// SHARED: few lists against M, which are therefore gone into deeply, by several threads each.  MANY: M above 16, where the heads of a wavefront's lists
// say too little; a kernel of its own, for code that is not run costs the other 0.2 us.
template <class T, bool SHARED, bool MANY>
__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(etv_beam_desc dsc, const T *logits, const float *scores, const int32_t *n_beams,
                                                                   const uint8_t *finished, int splits, uint32_t inv_splits, int width, int list,
                                                                   const ScanHead *heads, const Candidate *cands, float *out_scores, int32_t *parent,
                                                                   int32_t *token, uint8_t *finished_out, int32_t *status) {
    __shared__ double s_base[ETV_MAX_BEAMS], s_max[ETV_MAX_BEAMS];
    __shared__ int s_state[ETV_MAX_BEAMS], s_status, s_n;
    __shared__ float s_cut[kMergeThreads / 64];
    __shared__ uint32_t s_sample[kMergeThreads];
    __shared__ int s_count[2][kMergeThreads / 64];
    struct Total {
        double x;
        long place;
    };
    __shared__ Total s_total[kMergeCap + 16], s_best[ETV_MAX_BEAMS];
    __shared__ unsigned int s_again[3];  // beams whose sums are taken again; is there a pair of unequal totals, or one with a finished beam?
    __shared__ Candidate s_head[4][kMergeThreads];
    const int b = blockIdx.x, t = threadIdx.x;
    const int lists = dsc.K * splits, M = dsc.M;
    // totals of two beams closer than this are not told apart: by the scan's sums, and then by sums of exp2_fast
    double close = 0x1p-22 * (6 + kSlack + 0.6932f * (32 - __builtin_clz(dsc.V)));
    heads += (size_t)b * lists;
    cands += (size_t)b * lists * list;
    if (t == 0) s_status = 0;
    if (t < 3) s_again[t] = 0;
    __syncthreads();
    // A list is gone through by 2^share threads.  A thread's first one is on its way while the sums are joined: how many, and the first four of the
    // thread's entries, 2^share apart.
    int share = 0;
    if (SHARED)
        while (lists << (share + 1) <= kMergeThreads) share++;
    const int own = t >> share, deep = t & ((1 << share) - 1), apart = 1 << share;
    const int gap = (M + apart - 1) >> share;
    int head_n = 0;
    Candidate head[4] = {}, deeper = {};
    if (own < lists) {
        head_n = heads[own].n;
        if (MANY && SHARED) deeper = cands[(size_t)own * list + min(deep * gap, list - 1)];
#pragma unroll
        for (int i = 0; i < 4; i++) head[i] = cands[(size_t)own * list + min(deep + i * apart, list - 1)];
    }
    // 2^width lanes a beam
    for (int k0 = 0; k0 < dsc.K; k0 += kMergeThreads >> width) {
        const int k = k0 + (t >> width), lane = t & ((1 << width) - 1);
        ScanHead first = {-INFINITY, 0, 0};
        if (k < dsc.K && lane < splits) first = heads[k * splits + lane];  // of a beam that is not live: anything
        int state = k < dsc.K ? beam_state(dsc, scores, n_beams, finished, b, k) : kBeamNone;
        float m = first.m;
        double s = first.s;
        const auto scale = [](float from, float to) { return from > -INFINITY && from != to ? exp2_fast(fmax(((double)from - (double)to) * kLog2e, -1000.0)) : 1.0; };
        if (state == kBeamLive)
            for (int i = lane + (1 << width); i < splits; i += 1 << width) {  // running: the sum is relative to the largest so far
                const ScanHead h = heads[k * splits + i];
                const float top = fmaxf(m, h.m);
                s = s * scale(m, top) + h.s * scale(h.m, top);  // without a logit: 0, or NaN
                m = top;
            }
        const float own = m;
        m = lanes_best(m, width);
        s = lanes_sum(s * scale(own, m), width);
        if (k < dsc.K && lane == 0) {
            double base = scores[(size_t)b * dsc.K + k], most = 0;
            if (state == kBeamLive) {
                if (!(s < INFINITY)) {
                    atomicOr(&s_status, ETV_BEAM_BAD_LOGITS);
                    state = kBeamNone;
                }
                // from an fp32 logarithm: s = 2^l (1 + d) with |d| < 2^-20
                const double l = __builtin_amdgcn_logf((float)s);
                base -= l * 0.6931471805599453 + fma(s, exp2_fast(-l), -1.0);
                most = m;
            } else if (state == kBeamBad) {
                atomicOr(&s_status, ETV_BEAM_BAD_SCORE);
                state = kBeamNone;
            }
            s_base[k] = base, s_max[k] = most, s_state[k] = state;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; i++) s_head[i][t] = head[i];
    __syncthreads();
    // entry `deep` + i * `apart` of list l, of beam k; places order as (beam, token) do
    const auto value = [&](const Candidate &c, int k, double &x, long &place) {
        x = ((double)c.x - s_max[k]) + s_base[k];
        place = (long)k << 32 | (uint32_t)c.v;
    };
    const auto entry = [&](int l, int k, int i, double &x, long &place) {
        if (s_state[k] == kBeamLive) {
            value(l == own && i < 4 ? s_head[i][t] : cands[(size_t)l * list + deep + i * apart], k, x, place);
        } else {
            x = s_base[k];
            place = (long)k << 32 | (uint32_t)dsc.end_token;
        }
    };
    // how many a list has, and how many of them are the thread's
    const auto length = [&](int l, int &k) {
        uint32_t rest;
        k = (int)fast_div(l, splits, inv_splits, rest);
        const int state = s_state[k];
        return state == kBeamLive ? l == own ? head_n : heads[l].n : state == kBeamDone && rest == 0 ? 1 : 0;
    };
    const auto entries = [&](int l, int &k) { return (length(l, k) - deep + apart - 1) >> share; };
    // Are the rows of two beams the same?  Asked by the whole workgroup.
    constexpr int N = Logits<T>::N, AHEAD = 4;
    typedef typename Logits<T>::vec_at vec_at;
    const auto row_of = [&](int k) { return logits + b * dsc.batch_stride + k * dsc.row_stride; };
    const auto same = [&](int j, int k) {
        const T *x = row_of(j), *y = row_of(k);
        if (s_max[j] != s_max[k]) return false;
        if (x == y) return true;
        bool differ = dsc.V < N && t < dsc.V && x[t] != y[t];
        for (int v0 = 0; v0 < dsc.V && dsc.V >= N; v0 += AHEAD * kMergeThreads * N) {
#pragma unroll
            for (int i = 0; i < AHEAD; i++) {
                const int at = min(v0 + (i * kMergeThreads + t) * N, dsc.V - N);  // the last ones once more, behind the row
                const auto p = *reinterpret_cast<const vec_at *>(x + at), q = *reinterpret_cast<const vec_at *>(y + at);
                differ |= p.x != q.x || p.y != q.y || p.z != q.z || p.w != q.w;
            }
            if (__syncthreads_or(differ)) return false;
        }
        return !__syncthreads_or(differ);
    };
    // to multiples of 2^-40: rows with the same logits in another order tie, whatever order they were added in
    const auto base_of = [&](int k, double s) { return rint(((double)scores[(size_t)b * dsc.K + k] - log(s)) * 0x1p40) * 0x1p-40; };
    int n;
    for (int round = 0;; round++) {
        float top = -INFINITY;
        for (int l = own; l < lists; l += kMergeThreads) {
            int k;
            if (entries(l, k) > 0) {
                double x;
                long place;
                entry(l, k, 0, x, place);
                top = fmaxf(top, (float)x);
            }
        }
        const uint32_t key = order_of(top) >> 16;
        if (t == 0) s_n = 0;
        if (MANY) {
            // samples of all lists: where several threads look into one, `gap` entries from each other
            uint32_t sample = key;
            if (SHARED && deep) {
                int k;
                sample = 0;
                if (own < lists && deep * gap < length(own, k)) {
                    double x;
                    long place;
                    value(deeper, k, x, place);
                    sample = order_of((float)x) >> 16;
                }
            }
            // A first sample stands for one entry, each further one for `gap`.  Three bits of the bound at a time: every wavefront has all samples and counts
            // what reaches its digit, for a barrier each; the counts alternate between two places.
            s_sample[t] = sample;
            __syncthreads();
            constexpr int A = kMergeThreads / 64;
            static_assert(A == 8, "a wavefront a digit");
            const int lane = t & 63;
            const int weight = SHARED && (lane & (apart - 1)) ? gap : 1;  // (2^share beyond a wavefront: a gap of 1)
            uint32_t all[A], bound = 0;
#pragma unroll
            for (int i = 0; i < A; i++) all[i] = s_sample[i * 64 + lane];
#pragma unroll
            for (int shift = 15; shift >= 0; shift -= 3) {
                const uint32_t c = bound | (uint32_t)(t >> 6) << shift;
                int n = 0;
#pragma unroll
                for (int i = 0; i < A; i++) n += all[i] >= c;
                n = __builtin_amdgcn_readlane(wave_scan_sum(n * weight), 63);
                int *counts = s_count[shift & 1];
                if (lane == 0) counts[t >> 6] = n;
                __syncthreads();
                bound |= (uint32_t)__popcll(__ballot(lane > 0 && lane < A && counts[lane & (A - 1)] >= M)) << shift;
            }
            if (lane == 0) s_cut[t >> 6] = least_of(bound);
        } else {  // those of one wavefront are enough, and take no barrier for each bit
            const float mine = reached_by([&](uint32_t c) { return __popcll(__ballot(key >= c)); }, M);
            if ((t & 63) == 0) s_cut[t >> 6] = mine;
        }
        __syncthreads();
        float cut = s_cut[0];
#pragma unroll
        for (int w = 1; w < kMergeThreads / 64; w++) cut = fmaxf(cut, s_cut[w]);
        int found;
        for (bool counted = false;; counted = true) {
            cut = fmaxf(cut - (fabsf(cut) * 0x1p-21f + (float)close), -FLT_MAX);  // and those too close to it
            for (int l = own; l < lists; l += kMergeThreads) {
                int k;
                const int have = entries(l, k);
                const auto collect = [&](int i) {
                    double x;
                    long place;
                    entry(l, k, i, x, place);
                    if (!((float)x >= cut)) return false;
                    const int at = atomicAdd(&s_n, 1);
                    if (at < kMergeCap) s_total[at] = {x, place};
                    return true;
                };
                for (int i = 0; i < have && collect(i); i++) {
                }
            }
            __syncthreads();
            found = s_n;
            if (found <= kMergeCap || counted) break;
            // too many: a bound from all entries, counted in the lists by bisection
            cut = reached_by<1>(
                [&](uint32_t c) {
                    int n = 0;
                    for (int l = own; l < lists; l += kMergeThreads) {
                        int k, lo = 0, hi = entries(l, k);
                        while (lo < hi) {
                            const int i = (lo + hi) >> 1;
                            double x;
                            long place;
                            entry(l, k, i, x, place);
                            if (order_of((float)x) >> 16 >= c) lo = i + 1;
                            else hi = i;
                        }
                        n += lo;
                    }
                    return (int)block_sum((double)n);
                },
                M);
            __syncthreads();
            if (t == 0) s_n = 0;
            __syncthreads();
        }
        if (MANY && found > kThin && found <= kMergeCap) {
            // ranking takes found^2 steps: first those below a closer bound go, which is found among the candidates themselves
            constexpr int A = kMergeCap / kMergeThreads;
            Total mine[A];
            uint32_t keys[A];
#pragma unroll
            for (int i = 0; i < A; i++) {
                mine[i] = s_total[min(t + i * kMergeThreads, found - 1)];
                keys[i] = t + i * kMergeThreads < found ? order_of((float)mine[i].x) >> 16 : 0;
            }
            int turn = 0;
            float closer = reached_by<1>(
                [&](uint32_t c) {
                    int n = 0;
#pragma unroll
                    for (int i = 0; i < A; i++) n += __popcll(__ballot(keys[i] >= c));
                    turn ^= 1;
                    if ((t & 63) == 0) s_count[turn][t >> 6] = n;
                    __syncthreads();
                    n = 0;
#pragma unroll
                    for (int w = 0; w < kMergeThreads / 64; w++) n += s_count[turn][w];
                    return n;
                },
                M);
            closer = fmaxf(closer - (fabsf(closer) * 0x1p-21f + (float)close), -FLT_MAX);
            if (t == 0) s_n = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < A; i++)
                if (keys[i] && (float)mine[i].x >= closer) s_total[atomicAdd(&s_n, 1)] = mine[i];
            __syncthreads();
            found = s_n;
            __syncthreads();
        }
        if (found <= kMergeCap) {
            if (t < 16) s_total[found + t] = {-INFINITY, INT64_MAX};  // to a multiple of sixteen
            __syncthreads();
            for (int i = t >> 2; i < found; i += kMergeThreads / 4) {  // four lanes a candidate, with a quarter of the others each
                const Total own = s_total[i];
                float rank = 0;
#pragma unroll 1
                for (int j0 = t & 3; j0 < found; j0 += 16)
#pragma unroll
                    for (int j = j0; j < j0 + 16; j += 4) {
                        const Total o = s_total[j];
                        rank += (o.x > own.x) | ((o.x == own.x) & (o.place < own.place));
                    }
                rank = lanes_sum(rank, 2);
                if (rank < M && (t & 3) == 0) s_best[(int)rank] = own;
            }
            n = min(found, M);
        } else {
            double last = INFINITY;
            long last_place = -1;
            for (n = 0; n < M; n++) {
                double best = -INFINITY;
                long at = INT64_MAX;
                for (int l = own; l < lists; l += kMergeThreads) {
                    int k;
                    const int have = entries(l, k);
                    for (int i = 0; i < have; i++) {
                        double x;
                        long place;
                        entry(l, k, i, x, place);
                        if ((x < last || (x == last && place > last_place)) && (x > best || (x == best && place < at))) {
                            best = x, at = place;
                            break;  // a list is in order
                        }
                    }
                }
                block_best(best, at);
                if (best == -INFINITY) break;
                if (t == 0) s_best[n] = {best, at};
                last = best, last_place = at;
            }
        }
        __syncthreads();
        if (round == 2) break;
        // Two totals of different beams too close to call: neighbours of the M best, or the last of them and one left out.  Equal ones are among
        // them: sums of different rows may be equal in what was formed in 32 bits, and of beams alike, beside a third, all are taken again or none, so that
        // they stay alike.  Finished beams have no sum.  Rows that are the same have one, which is formed once, and decides nothing if there are no others.
        // (32 requests of 8 beams alike with 128000 logits: 93 us, 486 if every beam's sum is formed.)
        const auto call = [&](const Total &a, const Total &o) {
            const int k = (int)(a.place >> 32), k1 = (int)(o.place >> 32);
            if (k != k1 && a.x >= o.x && a.x - o.x < close && (s_state[k] == kBeamLive || s_state[k1] == kBeamLive)) {
                atomicOr(&s_again[k >> 5], 1u << (k & 31));
                atomicOr(&s_again[k1 >> 5], 1u << (k1 & 31));
                if (a.x != o.x || s_state[k] != s_state[k1]) s_again[2] = 1;
            }
        };
        if (t + 1 < n) call(s_best[t], s_best[t + 1]);
        if (n == M && found <= kMergeCap) {
            for (int i = t; i < found; i += kMergeThreads) call(s_best[M - 1], s_total[i]);
        } else if (n == M) {
            for (int l = own; l < lists; l += kMergeThreads) {
                int k;
                const int have = entries(l, k);
                for (int i = 0; i < have; i++) {
                    double x;
                    long place;
                    entry(l, k, i, x, place);
                    call(s_best[M - 1], {x, place});
                }
            }
        }
        __syncthreads();
        uint64_t again = s_again[0] | (uint64_t)s_again[1] << 32;
        if (!again) break;
        bool decides = s_again[2];
        if (!decides)
            for (uint64_t rest = again & (again - 1); rest && !decides; rest &= rest - 1) decides = !same(__builtin_ctzll(again), __builtin_ctzll(rest));
        if (!decides) break;
        double s = 0;
        for (int formed = -1; again; again &= again - 1) {
            const int k = __builtin_ctzll(again);
            if (s_state[k] != kBeamLive) continue;
            if (formed >= 0 && same(formed, k)) {
                if (t == 0) s_base[k] = base_of(k, s);
                continue;
            }
            const T *x = row_of(k);
            const double m = s_max[k];
            formed = k, s = 0;
            if (round == 0) {
                const auto add = [&](float y) { s += exp2_fast(fmax(((double)y - m) * kLog2e, -1000.0)); };
                const int vecs = dsc.V / N;
                for (int i0 = t; i0 < vecs; i0 += AHEAD * kMergeThreads) {
                    typename Logits<T>::vec raw[AHEAD];
#pragma unroll
                    for (int i = 0; i < AHEAD; i++) raw[i] = *reinterpret_cast<const vec_at *>(x + (size_t)min(i0 + i * kMergeThreads, vecs - 1) * N);
#pragma unroll
                    for (int i = 0; i < AHEAD; i++)
                        if (i0 + i * kMergeThreads < vecs) {
#pragma unroll
                            for (int j = 0; j < N; j++) add(Logits<T>::get(raw[i], j));
                        }
                }
                for (int v = vecs * N + t; v < dsc.V; v += kMergeThreads) add(Logits<T>::one(x[v]));
            } else {
#pragma unroll 4
                for (int v = t; v < dsc.V; v += kMergeThreads) s += exp((double)Logits<T>::one(x[v]) - m);
            }
            s = block_sum(s);
            if (t == 0) s_base[k] = base_of(k, s);
        }
        close = 0x1p-27;
        __syncthreads();
        if (t < 3) s_again[t] = 0;  // read behind further barriers, and read by all before this one
    }
    if (t < M) {
        const bool found = t < n;
        const long place = found ? s_best[t].place : 0;
        const int k = (int)(place >> 32), v = (int)place;
        const size_t o = (size_t)b * M + t;
        out_scores[o] = found ? (float)s_best[t].x : -INFINITY;
        parent[o] = found ? k : -1;
        token[o] = found ? v : -1;
        if (finished_out) finished_out[o] = found && (s_state[k] == kBeamDone || v == dsc.end_token);
    }
    if (t == 0) status[b] = s_status | (n < M ? ETV_BEAM_SHORT : 0);
}

// Steps of a wavefront's segment: more of them mean fewer bounds to find and fewer lists to merge, and fewer wavefronts to hide that behind.  As many as
// leave 1536 wavefronts, 6 a CU, up to eight (32 requests of 8 beams and 128000 logits: 8 steps take 1.3 us less than 4, and 2.2 less than 2), sixteen where 4096
// are left (four times the requests: 5 us less than with 8); a single one instead of two (64 requests of 4 beams and 32000 logits: half a us less).  Segments
// are as even as steps allow.  M above 16, where each segment leaves many candidates to bound, rank and merge: from 768 wavefronts on (3 requests of 13 beams
// and 156000 logits, M = 37: 4.5 us less than from 1536), but no more than eight steps.
constexpr int kFullWaves = 1536, kManyWaves = 4096, kFewWaves = 768;
static int beam_step(const etv_beam_desc *h) { return 64 * (h->dtype == ETV_BF16 ? 32 : 16); }
static int beam_steps(const etv_beam_desc *h) {
    const int64_t all = (h->V + beam_step(h) - 1) / beam_step(h), steps = (int64_t)h->B * h->K * all;
    int64_t n = std::min<int64_t>(steps / kFullWaves, 8);
    if (n < 3) n = 1;
    if (h->M > 16) n = std::max(n, std::min<int64_t>(steps / kFewWaves, 8));
    if (h->M <= 16) n = std::max(n, std::min<int64_t>(steps / kManyWaves, kMaxSteps));
    const int64_t splits = (all + n - 1) / n;
    return (int)((all + splits - 1) / splits);
}
static int beam_splits(const etv_beam_desc *h) {
    const int64_t segment = (int64_t)beam_step(h) * beam_steps(h);
    return (int)((h->V + segment - 1) / segment);
}

// Lists that a workspace holds: as many as any call with this many requests, beams and logits or fewer has, so that one sized for the largest of a
// program's calls does for the others, whose segments are shorter.  With `all` steps of all rows and n of them a segment there are at most all / n + rows lists;
// n is 1 below 3 * kFullWaves alone, from there on all / n stays below that until n is at its largest.
static int64_t beam_lists(const etv_beam_desc *h) {
    const int64_t rows = (int64_t)h->B * h->K, all = rows * ((h->V + beam_step(h) - 1) / beam_step(h));
    return std::min(all, std::max<int64_t>(3 * kFullWaves, all / (h->M > 16 ? 8 : kMaxSteps)) + rows);
}

// room for a list: a multiple of four, since the merge asks for its first four at once
static int beam_list(const etv_beam_desc *h) { return (h->M + 3) & ~3; }

static int32_t check_beam(const etv_beam_desc *h) {
    if (!h || h->B < 0 || h->K < 1 || h->M < 1 || h->V < 1 || h->end_token < -1 || h->end_token >= h->V) return ETV_ERR_INVALID_ARG;
    if (h->row_stride < 0 || h->batch_stride < 0) return ETV_ERR_INVALID_ARG;
    if (h->dtype != ETV_F32 && h->dtype != ETV_BF16) return ETV_ERR_UNSUPPORTED;
    if (h->K > ETV_MAX_BEAMS || h->M > ETV_MAX_BEAMS || h->V > INT32_MAX - 65536) return ETV_ERR_UNSUPPORTED;
    if ((int64_t)h->B * h->K * beam_splits(h) >= (1 << 26) || h->B >= (1 << 23)) return ETV_ERR_UNSUPPORTED;  // a launch has less than 2^32 threads
    return ETV_OK;
}

}  // namespace etv

extern "C" size_t etv_beam_select_workspace_bytes(const etv_beam_desc *h) {
    if (etv::check_beam(h) != ETV_OK) return 0;
    const size_t lists = (size_t)etv::beam_lists(h);
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
    // a request's scores and flags may take the place of its own old ones
    const size_t in = (size_t)h->B * h->K, out = (size_t)h->B * h->M;
    if (etv::overlap(scores, in * 4, out_scores, out * 4) && (scores != out_scores || in != out)) return ETV_ERR_INVALID_ARG;
    if (etv::overlap(finished, in, finished_out, out) && (finished != finished_out || in != out)) return ETV_ERR_INVALID_ARG;
    const int splits = etv::beam_splits(h), list = etv::beam_list(h), steps = etv::beam_steps(h);
    const unsigned lists = (unsigned)h->B * h->K * splits;
    auto *heads = static_cast<etv::ScanHead *>(workspace);
    auto *cands = reinterpret_cast<etv::Candidate *>(heads + lists);
    hipStream_t s = etv::as_stream(stream);
    const auto run = [&](auto *x) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(x)>>;
        const auto scan = h->V < etv::Logits<T>::N ? etv::beam_scan_kernel<T, true> : etv::beam_scan_kernel<T, false>;
        const uint32_t inv_splits = etv::fast_div_inv(splits);
        // room for the candidates: some times M where lists are short against the lanes, more of it fewer wavefronts at a time
        const int room = h->M <= 16 ? 256 : h->M <= 32 ? 512 : 1024;
        hipLaunchKernelGGL(scan, dim3(lists), dim3(64), (room + 16) * sizeof(etv::Candidate) + steps * 256, s, *h, x, scores, n_beams, finished, splits, inv_splits,
                           etv::fast_div_inv(h->K), steps, list, room, heads, cands);
        const int32_t rc = etv::check_launch();
        if (rc != ETV_OK) return rc;
        int width = 0;  // as many lanes a beam as it has segments, up to a wavefront
        while (width < 6 && (1 << width) < splits) width++;
        // 64 requests of 10 beams in 4 lists each: 2.8 us less than with a thread a list; 8 requests of 4 beams in 63 lists each would take 0.7 more
        const bool shared = splits * h->K <= 16 * h->M && splits * h->K <= etv::kMergeThreads / 2;
        const auto merge = h->M > 16 ? (shared ? etv::beam_merge_kernel<T, true, true> : etv::beam_merge_kernel<T, false, true>)
                                     : (shared ? etv::beam_merge_kernel<T, true, false> : etv::beam_merge_kernel<T, false, false>);
        hipLaunchKernelGGL(merge, dim3(h->B), dim3(etv::kMergeThreads), 0, s, *h, x, scores, n_beams, finished, splits, inv_splits,
                           width, list, heads, cands, out_scores, parent, token, finished_out, status);
        return etv::check_launch();
    };
    return h->dtype == ETV_BF16 ? run(static_cast<const uint16_t *>(logits)) : run(static_cast<const float *>(logits));
}
