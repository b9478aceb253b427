// The step of a beam search (or of a draft tree's next level): the best continuations over beams and vocabulary, and the beams' block
// tables and half-filled blocks after it.
#include "etv_common.h"
#include "free_ring.h"

namespace etv {

// --------------------------------------------------------------------------------------------------------------
// beam_select
// --------------------------------------------------------------------------------------------------------------
constexpr int kBeamChunk = 4096;  // logits of a row that a workgroup takes

struct ScanHead {
    float m;   // largest logit of the chunk, -inf: none
    int32_t n; // candidates that follow
    double s;  // sum of exp(x - m); NaN where a logit is NaN or +inf
};
struct Candidate {
    float x;
    int32_t v;
};

__device__ __forceinline__ float logit(const float *p) { return *p; }
__device__ __forceinline__ float logit(const uint16_t *p) { return bf16_bits_to_float(*p); }

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double s_part[4];
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

// What a beam offers: nothing, its end token, or its row of logits.
enum { kBeamNone, kBeamDone, kBeamLive, kBeamBad };
__device__ __forceinline__ int beam_state(const etv_beam_desc &dsc, const float *scores, const int32_t *n_beams, const uint8_t *finished, int b, int k) {
    if (n_beams && k >= n_beams[b]) return kBeamNone;
    const float s = scores[(size_t)b * dsc.K + k];
    if (!(s < INFINITY)) return kBeamBad;
    if (s == -INFINITY) return kBeamNone;
    return finished && finished[(size_t)b * dsc.K + k] ? kBeamDone : kBeamLive;
}

// A chunk of one row of logits: its largest, its sum of exponentials, its M best in order.
template <class T>
__global__ void __launch_bounds__(256) beam_scan_kernel(etv_beam_desc dsc, const T *logits, const float *scores, const int32_t *n_beams,
                                                        const uint8_t *finished, int splits, ScanHead *heads, Candidate *cands) {
    const int row = blockIdx.x / splits, split = blockIdx.x - row * splits, b = row / dsc.K, k = row - b * dsc.K, t = threadIdx.x;
    if (beam_state(dsc, scores, n_beams, finished, b, k) != kBeamLive) return;
    const T *x = logits + b * dsc.batch_stride + k * dsc.row_stride;
    const int v0 = split * kBeamChunk, v1 = min(dsc.V, v0 + kBeamChunk);
    constexpr int E = kBeamChunk / 256;
    float r[E];
    float m = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < E; i++) {
        const int v = v0 + i * 256 + t;
        r[i] = v < v1 ? logit(x + v) : -INFINITY;
        m = fmaxf(m, r[i]);
        bad |= !(r[i] < INFINITY);
    }
    int none = 0;
    block_best(m, none);
    double s = 0;
    const float ref = m > -INFINITY ? m : 0;
#pragma unroll
    for (int i = 0; i < E; i++) s += exp((double)r[i] - (double)ref);
    if (bad) s = NAN;
    s = block_sum(s);
    float last = INFINITY;
    int last_v = -1, n = 0;
    Candidate *out = cands + (size_t)blockIdx.x * dsc.M;
    for (; n < dsc.M; n++) {
        float best = -INFINITY;
        int at = INT32_MAX;
#pragma unroll
        for (int i = 0; i < E; i++) {
            const int v = v0 + i * 256 + t;
            if ((r[i] < last || (r[i] == last && v > last_v)) && r[i] > best) best = r[i], at = v;
        }
        block_best(best, at);
        if (best == -INFINITY) break;
        if (t == 0) out[n] = {best, at};
        last = best, last_v = at;
    }
    if (t == 0) heads[blockIdx.x] = {m, n, s};
}

// A request: the logarithms of its beams' sums, then the M best of all candidates.
__global__ void __launch_bounds__(256) beam_merge_kernel(etv_beam_desc dsc, const float *scores, const int32_t *n_beams, const uint8_t *finished, int splits,
                                                         const ScanHead *heads, const Candidate *cands, float *out_scores, int32_t *parent, int32_t *token,
                                                         uint8_t *finished_out, int32_t *status) {
    // total = (x - largest logit) + (score - log of the sum relative to it): nothing is lost where logits are large
    __shared__ double s_base[ETV_MAX_BEAMS], s_max[ETV_MAX_BEAMS];
    __shared__ int s_state[ETV_MAX_BEAMS], s_status;
    const int b = blockIdx.x, t = threadIdx.x, lane = t & 63;
    if (t == 0) s_status = 0;
    __syncthreads();
    for (int k = t >> 6; k < dsc.K; k += 4) {
        int state = beam_state(dsc, scores, n_beams, finished, b, k);
        double base = scores[(size_t)b * dsc.K + k], most = 0;
        if (state == kBeamLive) {
            const ScanHead *h = heads + ((size_t)b * dsc.K + k) * splits;
            float m = -INFINITY;
            for (int i = lane; i < splits; i += 64) m = fmaxf(m, h[i].m);
            for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
            double s = 0;
            for (int i = lane; i < splits; i += 64) s += h[i].m > -INFINITY || h[i].s != h[i].s ? h[i].s * exp((double)h[i].m - (double)m) : 0;
            for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
            if (s != s) {
                if (lane == 0) atomicOr(&s_status, ETV_BEAM_BAD_LOGITS);
                state = kBeamNone;
            }
            base -= log(s);
            most = m;
        } else if (state == kBeamBad) {
            if (lane == 0) atomicOr(&s_status, ETV_BEAM_BAD_SCORE);
            state = kBeamNone;
        }
        if (lane == 0) s_base[k] = base, s_max[k] = most, s_state[k] = state;
    }
    __syncthreads();
    double last = INFINITY;
    long last_place = -1;
    const long V = dsc.V;
    const int lists = dsc.K * splits;
    int n = 0;
    for (; n < dsc.M; n++) {
        double best = -INFINITY;
        long at = INT64_MAX;
        const auto offer = [&](double x, long place) {
            if ((x < last || (x == last && place > last_place)) && (x > best || (x == best && place < at))) best = x, at = place;
        };
        for (int l = t; l < lists; l += 256) {
            const int k = l / splits;
            if (s_state[k] == kBeamDone && l == k * splits) offer(s_base[k], k * V + dsc.end_token);
            if (s_state[k] != kBeamLive) continue;
            const size_t list = (size_t)b * lists + l;
            const int have = heads[list].n;
            for (int i = 0; i < have; i++) offer((cands[list * dsc.M + i].x - s_max[k]) + s_base[k], k * V + cands[list * dsc.M + i].v);
        }
        block_best(best, at);
        if (best == -INFINITY) break;
        if (t == 0) {
            const int k = (int)(at / V), v = (int)(at - k * V);
            const size_t o = (size_t)b * dsc.M + n;
            out_scores[o] = (float)best;
            parent[o] = k;
            token[o] = v;
            if (finished_out) finished_out[o] = s_state[k] == kBeamDone || v == dsc.end_token;
        }
        last = best, last_place = at;
    }
    for (int i = n + t; i < dsc.M; i += 256) {
        const size_t o = (size_t)b * dsc.M + i;
        out_scores[o] = -INFINITY;
        parent[o] = token[o] = -1;
        if (finished_out) finished_out[o] = 0;
    }
    if (t == 0) status[b] = s_status | (n < dsc.M ? ETV_BEAM_SHORT : 0);
}

static int beam_splits(const etv_beam_desc *h) { return (h->V + kBeamChunk - 1) / kBeamChunk; }

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
    return lists * (sizeof(etv::ScanHead) + h->M * sizeof(etv::Candidate));
}

extern "C" int32_t etv_beam_select(const etv_beam_desc *h, const void *logits, const float *scores, const int32_t *n_beams, const uint8_t *finished,
                                   float *out_scores, int32_t *parent, int32_t *token, uint8_t *finished_out, int32_t *status, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    int32_t rc = etv::check_beam(h);
    if (rc != ETV_OK) return rc;
    if (h->B == 0) return ETV_OK;
    if (!logits || !scores || !out_scores || !parent || !token || !status || (finished && h->end_token < 0)) return ETV_ERR_INVALID_ARG;
    if ((uintptr_t)logits % (h->dtype == ETV_BF16 ? 2 : 4) || (uintptr_t)workspace & 15) return ETV_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < etv_beam_select_workspace_bytes(h)) return ETV_ERR_WORKSPACE_TOO_SMALL;
    const int splits = etv::beam_splits(h);
    const unsigned lists = (unsigned)h->B * h->K * splits;
    auto *heads = static_cast<etv::ScanHead *>(workspace);
    auto *cands = reinterpret_cast<etv::Candidate *>(heads + lists);
    hipStream_t s = etv::as_stream(stream);
    if (h->dtype == ETV_BF16)
        hipLaunchKernelGGL(etv::beam_scan_kernel<uint16_t>, dim3(lists), dim3(256), 0, s, *h, static_cast<const uint16_t *>(logits), scores, n_beams,
                           finished, splits, heads, cands);
    else
        hipLaunchKernelGGL(etv::beam_scan_kernel<float>, dim3(lists), dim3(256), 0, s, *h, static_cast<const float *>(logits), scores, n_beams, finished,
                           splits, heads, cands);
    rc = etv::check_launch();
    if (rc != ETV_OK) return rc;
    hipLaunchKernelGGL(etv::beam_merge_kernel, dim3(h->B), dim3(256), 0, s, *h, scores, n_beams, finished, splits, heads, cands, out_scores, parent, token,
                       finished_out, status);
    return etv::check_launch();
}
