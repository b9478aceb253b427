// The beams' block tables after a step: gathered from the parents', with blocks shared, the half-filled block copied where several beams go on
// from it, and the blocks that nobody refers to any more put back into the ring.  Two launches: the tables and what they need and
// give back, then -- every workgroup adding up what the requests before its own need -- the copies.  Nothing is counted by atomics, so that
// blocks go to the same beams in every run, and no call needs cleared memory.
// Floor: the tables twice and the copied rows twice.  32 requests of 8 beams, 6 layers of bf16 are 35.4 MB, 6.9 us at a copy's rate: the
// call takes 13.9 us.
#include "etv_common.h"
#include "free_ring.h"

namespace etv {

constexpr int kCols = 64;  // columns of the tables of one request that a workgroup -- one wavefront -- takes

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct ReorderShape {
    int B, K, M, max_blocks, num_blocks, block_size, chunks, stride;
};
// What the first launch finds.  Every workgroup of the second adds up what the requests before its own need and give, so that this is kept small
// and apart, for loads of 16 bytes: 256 requests of 4096 columns are 16 KB of status and took 69 us as records of 16 bytes a chunk.
struct ReorderWorkspace {
    uint8_t *st;    // [B][stride]: status bits of a chunk of columns; 0 behind the chunks
    int32_t *give;  // [B][stride]: blocks that the chunk gives back
    int32_t *need;  // [B]: blocks to copy into, if the request is not refused
    int32_t *from;  // [B][M]: the block to copy from, -1: none
    int32_t *list;  // [B][chunks][kCols * K]: the ids of the blocks given back
};

__device__ __forceinline__ int32_t length_status(const ReorderShape &sh, int len) {
    if (len < 0) return ETV_COMMIT_BAD_LEN;
    return ((long)len + sh.block_size - 1) / sh.block_size > sh.max_blocks ? ETV_COMMIT_CAPACITY : 0;
}

// grid (chunks, B): a lane per column of the table, and per new beam, whose parents are then a ballot or a lane read away.  The old beams' entries of its
// column are asked for eight at a time.  FEW: they are eight at most, stay in its registers, and one wavefront does it all; otherwise four share the
// beams, and the columns in which beams differ -- the last ones, as a rule --, where a lane is a beam and one round finds all that have a
// block.  Bound by the chain of its loads (3.5 us for one request) until the tables are large: 256 requests of 4 beams and 4096
// columns, 33.6 MB, 16 us.
constexpr int kPitch = kCols + 1;  // of a beam's columns in LDS: a column over the beams has no two in one bank
template <bool FEW>
__global__ void __launch_bounds__(FEW ? kCols : 4 * kCols) reorder_tables_kernel(ReorderShape sh, const int32_t *block_table, const int32_t *len, const int32_t *parent,
                                                                                int32_t *table_out, ReorderWorkspace ws) {
    extern __shared__ int32_t s_table[];  // [K][kPitch]
    constexpr int W = FEW ? 1 : 4;
    const int c = blockIdx.x, b = blockIdx.y, t = threadIdx.x & 63, w = FEW ? 0 : threadIdx.x >> 6, col = c * kCols + t;
    const int32_t *src = block_table + (size_t)b * sh.K * sh.max_blocks + min(col, sh.max_blocks - 1);
    int p = t < sh.M ? parent[(size_t)b * sh.M + t] : -1;
    int32_t id[8];
    for (int k0 = 8 * w; k0 < sh.K; k0 += 8 * W) {
#pragma unroll
        for (int i = 0; i < 8; i++) id[i] = src[(size_t)min(k0 + i, sh.K - 1) * sh.max_blocks];
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (k0 + i < sh.K) s_table[(k0 + i) * kPitch + t] = id[i];
        if (FEW) break;
    }
    int32_t st = length_status(sh, len[b]);
    const int L = st ? 0 : len[b], full = (int)((uint32_t)L / (uint32_t)sh.block_size), rows = L - full * sh.block_size, cols = full + (rows > 0);
    if (__ballot(p < -1 || p >= sh.K)) st |= ETV_COMMIT_BAD_NODE;
    if (p >= sh.K) p = -1;
    const auto either = [](uint32_t x, uint32_t y) { return x | y; };
    const uint64_t alive = wave_best(p >= 0 && p < 32 ? 1u << p : 0u, either) | (uint64_t)wave_best(p >= 32 ? 1u << (p - 32) : 0u, either) << 32;
    const auto outside = [&](int32_t x) { return (uint32_t)x >= (uint32_t)sh.num_blocks; };
    int bad = 0;
    __shared__ uint64_t s_differ[4], s_gone[kCols];
    const int32_t first = FEW ? 0 : (__syncthreads(), s_table[(alive ? __builtin_ctzll(alive) : 0) * kPitch + t]);  // the entry of a beam that goes on, if any does
    if (FEW) {
        if (col < cols) {
#pragma unroll
            for (int k = 0; k < 8; k++) bad |= (alive >> k & 1) && outside(id[k]);
        }
        bad = __ballot(bad) != 0;
    } else {
        int differ = 0;
        if (col < cols) {
#pragma unroll 4
            for (int k = w; k < sh.K; k += W) {
                const int32_t x = s_table[k * kPitch + t];
                bad |= (alive >> k & 1) && outside(x);
                differ |= x != first;
            }
        }
        const uint64_t columns = __ballot(differ);
        if (t == 0) s_differ[w] = columns;
        bad = __syncthreads_or(bad);
    }
    if (bad) st |= ETV_COMMIT_BAD_BLOCK;
    if (col < sh.max_blocks)
        for (int i = w; i < sh.M; i += W) {
            const int from = __builtin_amdgcn_readlane(p, i);
            table_out[((size_t)b * sh.M + i) * sh.max_blocks + col] = !st && from >= 0 && col < cols ? s_table[from * kPitch + t] : -1;
        }
    // blocks of beams without a child that neither a parent nor an earlier such beam has
    uint64_t gone = 0;
    if (FEW) {
        if (col < cols && !st) {
#pragma unroll
            for (int k = 0; k < 8; k++) {
                bool mine = k < sh.K && !(alive >> k & 1) && !outside(id[k]);
#pragma unroll
                for (int j = 0; j < 8; j++)
                    if (j != k) mine &= !((j < k || (alive >> j & 1)) && id[j] == id[k]);
                gone |= (uint64_t)mine << k;
            }
        }
    } else {
        const uint64_t differ = s_differ[0] | s_differ[1] | s_differ[2] | s_differ[3];
        int turn = 0;
        for (uint64_t todo = st ? 0 : differ; todo; todo &= todo - 1) {
            if ((turn++ & (W - 1)) != w) continue;
            const int at = __builtin_ctzll(todo);
            const int32_t x = t < sh.K ? s_table[t * kPitch + at] : -1;
            uint64_t mine = 0;
            for (uint64_t left = __ballot(!outside(x)) & ~alive; left;) {
                const int k = __builtin_ctzll(left);
                const uint64_t same = __ballot(x == __builtin_amdgcn_readlane(x, k)) & (~0ull >> (64 - sh.K));
                if (!(same & alive)) mine |= 1ull << k;
                left &= ~same;
            }
            if (t == 0) s_gone[at] = mine;
        }
        __syncthreads();
        if (w) return;
        // one block for all, if no beam goes on
        if (col < cols && !st) gone = differ >> t & 1 ? s_gone[t] : alive || outside(first) ? 0 : 1;
    }
    const int count = __popcll(gone), upto = wave_scan_sum(count), all = __builtin_amdgcn_readlane(upto, 63);
    int32_t *list = ws.list + ((size_t)b * sh.chunks + c) * kCols * sh.K;
    for (int at = upto - count; gone; gone &= gone - 1) list[at++] = s_table[__builtin_ctzll(gone) * kPitch + t];
    // the half-filled block: its first child keeps it
    const bool here = !st && rows > 0 && full / kCols == c;
    int need = 0;
    if (here) {
        if (FEW) __syncthreads();  // another lane's column
        const int32_t own = p >= 0 ? s_table[p * kPitch + full % kCols] : -1;
        bool later = false;
        for (int j = 0; j < sh.M; j++) later |= j < t && __builtin_amdgcn_readlane(own, j) == own;
        later = later && own >= 0;
        need = __popcll(__ballot(later));
        if (t < sh.M) ws.from[(size_t)b * sh.M + t] = later ? own : -1;
    }
    // one chunk says what the request needs: the half-filled block's, or the first (what a length is refused for, every chunk finds)
    if (t == 0 && c == (rows > 0 ? full / kCols : 0)) ws.need[b] = need;
    if (t < (c == sh.chunks - 1 ? sh.stride - c : 1)) {
        ws.st[(size_t)b * sh.stride + c + t] = t == 0 ? st : 0;
        ws.give[(size_t)b * sh.stride + c + t] = t == 0 ? all : 0;
    }
}

// What all chunks of a request say.
struct Request {
    int32_t st, need, give;
};
__device__ __forceinline__ Request request(const ReorderShape &sh, const ReorderWorkspace &ws, int b) {
    Request r{0, ws.need[b], 0};
    for (int c = 0; c < sh.chunks; c++) {
        r.st |= ws.st[(size_t)b * sh.stride + c];
        r.give += ws.give[(size_t)b * sh.stride + c];
    }
    if (r.st) r.need = r.give = 0;
    return r;
}

// Element i of n, 0 behind them; and f of the elements from one on, `threads` of them at a time and eight a thread on their way.  Few requests have as
// few elements as threads: those are asked for together, and the loop is for the rest.
template <class V>
__device__ __forceinline__ V element(const V *x, int i, int n) {
    return i < n ? x[i] : V{};
}
template <class V, class F>
__device__ __forceinline__ void elements(const V *x, int from, int n, int threads, F f) {
    for (int i0 = from; i0 < n; i0 += 8 * threads) {
        V v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = x[min(i0 + i * threads, n - 1)];
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i0 + i * threads < n) f(i0 + i * threads, v[i]);
    }
}
__device__ __forceinline__ uint32_t any_of(const u32x4 &v) { return v.x | v.y | v.z | v.w; }

struct CacheParts {
    uint8_t *base[4];
    size_t layer_bytes[4];
    int row_bytes[4];
    int parts, Hkv, n_layers;
};


// The rows of half-filled blocks, copies first, first + step, .. below n: one head's are consecutive.  Units of 16 bytes, or of 2 where a row is
// shorter, those of all copies in a row (not where 64 of them might pass 32 bits), AHEAD a thread on their way.  (A block of one layer has
// less than 2^32 bytes.)
template <class U, int AHEAD>
__device__ __forceinline__ void copy_rows(uint8_t *layer, const int2 *copies, int first, int step, int n, int num_blocks, int Hkv, int block_size,
                                          int row_bytes, int rows) {
    const uint32_t per_head = (uint32_t)((uint32_t)rows * (uint32_t)row_bytes / sizeof(U)), all = per_head * Hkv;
    const uint32_t inv = per_head == 1 ? 0xffffffffu : 0xffffffffu / per_head, inv_all = all == 1 ? 0xffffffffu : 0xffffffffu / all;
    const uint32_t head = (uint32_t)block_size * (uint32_t)row_bytes;
    const size_t block = (size_t)Hkv * head;
    if (first + step >= n || all >= (1u << 24)) {  // a copy at a time
        for (int copy = first; copy < n; copy += step) {
            if ((uint32_t)copies[copy].y >= (uint32_t)num_blocks) continue;
            const uint8_t *from = layer + copies[copy].x * block;
            uint8_t *to = layer + copies[copy].y * block;
            for (uint32_t u0 = threadIdx.x; u0 < all; u0 += AHEAD * 256) {
                U x[AHEAD];
                uint32_t at[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; i++) {
                    uint32_t unit;
                    const uint32_t h = fast_div(min(u0 + i * 256, all - 1), per_head, inv, unit);
                    at[i] = h * head + unit * (uint32_t)sizeof(U);
                    x[i] = *reinterpret_cast<const U *>(from + at[i]);
                }
#pragma unroll
                for (int i = 0; i < AHEAD; i++)
                    if (u0 + i * 256 < all) *reinterpret_cast<U *>(to + at[i]) = x[i];
            }
        }
        return;
    }
    const uint32_t units = ((n - 1 - first) / step + 1) * all;
    for (uint32_t u0 = threadIdx.x; u0 < units; u0 += AHEAD * 256) {
        U x[AHEAD];
        size_t to[AHEAD];
        uint32_t there = 0;
#pragma unroll
        for (int i = 0; i < AHEAD; i++) {
            uint32_t unit, in_head;
            const uint32_t copy = fast_div(min(u0 + i * 256, units - 1), all, inv_all, unit);
            const int2 c = copies[first + copy * step];
            const uint32_t at = fast_div(unit, per_head, inv, in_head) * head + in_head * (uint32_t)sizeof(U);
            x[i] = *reinterpret_cast<const U *>(layer + c.x * block + at);
            to[i] = c.y * block + at;
            there |= (u0 + i * 256 < units && (uint32_t)c.y < (uint32_t)num_blocks) << i;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; i++)
            if (there >> i & 1) *reinterpret_cast<U *>(layer + to[i]) = x[i];
    }
}

// Workgroups 0 .. B-1: status, the table entries of the copies and the ring.  Then B * n_layers * parts * G workgroups that copy.  16 requests that
// become 8 beams of 4 layers in fp32 copy 51.4 MB in 12.6 us: 4.1 TB/s, with the sums before it.
__global__ void __launch_bounds__(256) reorder_copy_kernel(ReorderShape sh, CacheParts cache, int G, const int32_t *len, int32_t *free_blocks,
                                                           const int32_t *free_state, int32_t *table_out, int32_t *free_state_out, int32_t *status,
                                                           ReorderWorkspace ws) {
    const Ring ring(free_state, sh.num_blocks);
    const int t = threadIdx.x, lane = t & 63;
    if ((int)blockIdx.x >= sh.B) {
        int x = blockIdx.x - sh.B;
        const int g = x % G;
        x /= G;
        const int part = x % cache.parts;
        x /= cache.parts;
        const int l = x % cache.n_layers, b = x / cache.n_layers;
        const int32_t from = lane < sh.M ? ws.from[(size_t)b * sh.M + lane] : -1;
        const int rows = (int)((uint32_t)len[b] % (uint32_t)sh.block_size);
        const u32x4 *status = reinterpret_cast<const u32x4 *>(ws.st);
        const int vectors = (b + 1) * (sh.stride / 16), need = ws.need[b];
        int before = element(ws.need, lane, b);
        uint32_t any = any_of(element(status, lane, vectors));
        if (g >= need) return;
        elements(ws.need, lane + 64, b, 64, [&](int, int n) { before += n; });
        elements(status, lane + 64, vectors, 64, [&](int, const u32x4 &v) { any |= any_of(v); });
        if (__ballot(any)) {  // a refused request needs none
            if (request(sh, ws, b).st) return;
            before = 0;
            for (int o = lane; o < b; o += 64) before += request(sh, ws, o).need;
        }
        before = __builtin_amdgcn_readlane(wave_scan_sum(before), 63);
        if ((long)before + need > ring.count) return;
        uint8_t *layer = cache.base[part] + (size_t)l * cache.layer_bytes[part];
        __shared__ int2 s_copy[ETV_MAX_BEAMS];
        const uint64_t copies = __ballot(from >= 0);
        if (t < 64 && from >= 0) {
            const int i = __popcll(copies & ((1ull << lane) - 1));
            s_copy[i] = make_int2(from, free_blocks[ring.place(before + i)]);
        }
        __syncthreads();
        if (cache.row_bytes[part] % 16 == 0) copy_rows<u32x4, 8>(layer, s_copy, g, G, need, sh.num_blocks, cache.Hkv, sh.block_size, cache.row_bytes[part], rows);
        else copy_rows<uint16_t, 2>(layer, s_copy, g, G, need, sh.num_blocks, cache.Hkv, sh.block_size, cache.row_bytes[part], rows);
        return;
    }
    __shared__ long s_need, s_give;
    __shared__ unsigned long long s_taken, s_given;
    __shared__ int s_part[4][4];
    const int b = blockIdx.x;
    // what the requests before need and give, this one, and whether one of them is refused.  (What all give is below 2^31: so are all entries.)
    const u32x4 *gives = reinterpret_cast<const u32x4 *>(ws.give), *refused = reinterpret_cast<const u32x4 *>(ws.st);
    const int own_at = b * (sh.stride / 4), gives_n = own_at + sh.stride / 4, refused_n = (b + 1) * (sh.stride / 16);
    int v[4] = {0, 0, 0, 0}, own_need = ws.need[b];
    const auto add_need = [&](int, int n) { v[0] += n; };
    const auto add_give = [&](int i, const u32x4 &x) {
        const int sum = (int)(x.x + x.y + x.z + x.w);
        v[1] += i < own_at ? sum : 0;
        v[2] += i < own_at ? 0 : sum;
    };
    const auto add_refused = [&](int, const u32x4 &x) { v[3] |= any_of(x) != 0; };
    const int need0 = element(ws.need, t, b);
    const u32x4 give0 = element(gives, t, gives_n), refused0 = element(refused, t, refused_n);
    add_need(t, need0);
    add_give(t, give0);
    add_refused(t, refused0);
    elements(ws.need, t + 256, b, 256, add_need);
    elements(gives, t + 256, gives_n, 256, add_give);
    elements(refused, t + 256, refused_n, 256, add_refused);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int sum = __builtin_amdgcn_readlane(wave_scan_sum(v[i]), 63);
        if (lane == 0) s_part[i][t >> 6] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = s_part[i][0] + s_part[i][1] + s_part[i][2] + s_part[i][3];
    long need_at = v[0], give_at = v[1], taken = need_at + own_need, given = give_at + v[2];
    int32_t st = 0;
    if (v[3] || taken > ring.count || given > ring.room()) {  // some are refused: one after the other
        if (t == 0) s_taken = s_given = 0;
        long needs = 0, gives = 0;
        for (int b0 = 0; b0 <= b; b0 += 256) {
            const int o = b0 + t;
            Request r{0, 0, 0};
            if (o <= b) r = request(sh, ws, o);
            const long need_end = block_scan_sum<4>(r.need, needs);
            int32_t os = r.st;
            if (!os && r.need > 0 && need_end > ring.count) os = ETV_BRANCH_NO_BLOCKS, r.give = 0;
            else if (r.need > 0) atomicMax(&s_taken, (unsigned long long)need_end);
            const long give_end = block_scan_sum<4>(r.give, gives);
            if (r.give > 0) {
                if (give_end > ring.room()) os |= ETV_BRANCH_BAD_FREE;
                else atomicMax(&s_given, (unsigned long long)give_end);
            }
            if (o == b) s_part[0][0] = os, s_part[1][0] = r.need, s_need = need_end - r.need, s_give = give_end - r.give;
        }
        __syncthreads();
        st = s_part[0][0], own_need = s_part[1][0], need_at = s_need, give_at = s_give, taken = (long)s_taken, given = (long)s_given;
    }
    if (b == sh.B - 1 && t == 0) ring.leave(free_state_out, taken, given);
    const int L = len[b];
    if (st) {
        for (size_t i = t; i < (size_t)sh.M * sh.max_blocks; i += 256) table_out[(size_t)b * sh.M * sh.max_blocks + i] = -1;
    } else {
        if (own_need) {
            const int32_t from = lane < sh.M ? ws.from[(size_t)b * sh.M + lane] : -1;
            const uint64_t copies = __ballot(from >= 0);
            const int32_t dst = from >= 0 ? free_blocks[ring.place(need_at + __popcll(copies & ((1ull << lane) - 1)))] : 0;
            const bool good = (uint32_t)dst < (uint32_t)sh.num_blocks;
            if (t < 64 && from >= 0 && good) table_out[((size_t)b * sh.M + lane) * sh.max_blocks + L / sh.block_size] = dst;
            for (uint64_t bad = __ballot(!good); bad; bad &= bad - 1) {
                st |= ETV_BRANCH_BAD_FREE;
                int32_t *row = table_out + ((size_t)b * sh.M + __builtin_ctzll(bad)) * sh.max_blocks;
                for (int j = t; j < sh.max_blocks; j += 256) row[j] = -1;
            }
        }
        long at = ring.count + give_at;
        for (int c0 = 0; v[2] && c0 < sh.chunks; c0 += 256) {  // 256 chunks at a time
            const int n = c0 + t < sh.chunks ? ws.give[(size_t)b * sh.stride + c0 + t] : 0;
            const long first = block_scan_sum<4>(n, at) - n;
            for (uint64_t todo = __ballot(n > 0); todo; todo &= todo - 1) {  // those of a wavefront's lanes, one after the other
                const int c = __builtin_ctzll(todo);
                const int32_t *list = ws.list + ((size_t)b * sh.chunks + c0 + (t & ~63) + c) * kCols * sh.K;
                const int count = __shfl(n, c);
                const long to = __shfl(first, c);
                for (int i = lane; i < count; i += 64) free_blocks[ring.place(to + i)] = list[i];
            }
        }
    }
    if (t == 0) status[b] = st;
}

// An empty batch takes and gives nothing.
__global__ void ring_copy_kernel(const int32_t *free_state, int32_t *free_state_out) { free_state_out[threadIdx.x] = free_state[threadIdx.x]; }

static int reorder_chunks(int max_blocks) { return (max_blocks - 1) / kCols + 1; }
static int reorder_stride(int chunks) { return (chunks + 15) & ~15; }

// The shapes whose sums and launches stay in their types: less than 2^31 entries in all tables, less than 2^32 threads.
static int32_t check_reorder(int64_t B, int64_t K, int64_t M, int64_t max_blocks) {
    if (B < 0 || K < 1 || M < 1 || max_blocks < 1) return ETV_ERR_INVALID_ARG;
    if (K > ETV_MAX_BEAMS || M > ETV_MAX_BEAMS || B > 65535 || max_blocks > (1 << 22) || B * K * max_blocks > INT32_MAX) return ETV_ERR_UNSUPPORTED;
    return B * reorder_chunks((int)max_blocks) >= (1 << 26) ? ETV_ERR_UNSUPPORTED : ETV_OK;
}

static ReorderShape reorder_shape(int B, int K, int M, int max_blocks, int num_blocks, int block_size) {
    const int chunks = max_blocks > 0 ? reorder_chunks(max_blocks) : 0;
    return {B, K, M, max_blocks, num_blocks, block_size, chunks, reorder_stride(chunks)};
}

static size_t reorder_bytes(int64_t B, int64_t K, int64_t M, int max_blocks) {
    const size_t chunks = reorder_chunks(max_blocks);
    return (size_t)B * (reorder_stride((int)chunks) * 5 + 4 + M * 4 + chunks * kCols * K * 4);
}

static int32_t reorder(const ReorderShape &shape, const CacheParts &cache, const int32_t *block_table, const int32_t *len, const int32_t *parent,
                       int32_t *free_blocks, const int32_t *free_state, int32_t *table_out, int32_t *free_state_out, int32_t *status, void *workspace,
                       size_t workspace_bytes, void *stream) {
    const ReorderShape sh = shape;
    const int32_t shape_rc = check_reorder(sh.B, sh.K, sh.M, sh.max_blocks);
    if (shape_rc == ETV_ERR_INVALID_ARG || sh.num_blocks < 1 || cache.n_layers < 1 || cache.Hkv < 1) return ETV_ERR_INVALID_ARG;
    if (shape_rc != ETV_OK || (int64_t)sh.num_blocks * sh.block_size > INT32_MAX) return ETV_ERR_UNSUPPORTED;
    if (!free_blocks || !free_state || !free_state_out || overlap(free_state, 8, free_state_out, 8)) return ETV_ERR_INVALID_ARG;
    hipStream_t s = as_stream(stream);
    if (sh.B == 0) {
        hipLaunchKernelGGL(ring_copy_kernel, dim3(1), dim3(2), 0, s, free_state, free_state_out);
        return check_launch();
    }
    if (!block_table || !len || !parent || !table_out || !status) return ETV_ERR_INVALID_ARG;
    const size_t columns = (size_t)sh.B * sh.max_blocks * 4, lens = (size_t)sh.B * 4;
    if (overlap(table_out, columns * sh.M, block_table, columns * sh.K) || overlap(status, lens, len, lens)) return ETV_ERR_INVALID_ARG;
    for (int i = 0; i < cache.parts; i++)
        if ((double)cache.Hkv * sh.block_size * cache.row_bytes[i] >= 0x1p32) return ETV_ERR_UNSUPPORTED;
    for (int i = 0; i < cache.parts; i++)
        if (!cache.base[i] || (uintptr_t)cache.base[i] % (cache.row_bytes[i] % 16 ? 2 : 16)) return ETV_ERR_INVALID_ARG;
    if ((uintptr_t)workspace & 15) return ETV_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < reorder_bytes(sh.B, sh.K, sh.M, sh.max_blocks)) return ETV_ERR_WORKSPACE_TOO_SMALL;
    ReorderWorkspace ws;
    ws.st = static_cast<uint8_t *>(workspace);
    ws.give = reinterpret_cast<int32_t *>(ws.st + (size_t)sh.B * sh.stride);
    ws.need = ws.give + (size_t)sh.B * sh.stride;
    ws.from = ws.need + sh.B;
    ws.list = ws.from + (size_t)sh.B * sh.M;
    // a workgroup per copy while they are few, a loop over a request's copies beyond
    const int64_t one = (int64_t)sh.B * cache.n_layers * cache.parts;
    int64_t G = 2048 / one;
    G = G < 1 ? 1 : G > sh.M ? sh.M : G;
    if (sh.B + one * G >= (1 << 24)) return ETV_ERR_UNSUPPORTED;  // a launch has less than 2^32 threads
    const bool few = sh.K <= 8;
    hipLaunchKernelGGL(few ? reorder_tables_kernel<true> : reorder_tables_kernel<false>, dim3(sh.chunks, sh.B), dim3(few ? kCols : 4 * kCols),
                       sizeof(int32_t) * sh.K * kPitch, s, sh, block_table, len, parent, table_out, ws);
    const int32_t rc = check_launch();
    if (rc != ETV_OK) return rc;
    hipLaunchKernelGGL(reorder_copy_kernel, dim3((unsigned)(sh.B + one * G)), dim3(256), 0, s, sh, cache, (int)G, len, free_blocks, free_state, table_out,
                       free_state_out, status, ws);
    return check_launch();
}

}  // namespace etv

extern "C" size_t etv_reorder_beams_workspace_bytes(int32_t B, int32_t K, int32_t M, int32_t max_blocks) {
    if (etv::check_reorder(B, K, M, max_blocks) != ETV_OK) return 0;
    return etv::reorder_bytes(B, K, M, max_blocks);
}

extern "C" int32_t etv_reorder_beams(const etv_cache_desc *h, void *k_cache, void *v_cache, const int32_t *block_table, const int32_t *len, int32_t K,
                                     const int32_t *parent, int32_t M, int32_t *free_blocks, const int32_t *free_state, int32_t *table_out,
                                     int32_t *free_state_out, int32_t *status, void *workspace, size_t workspace_bytes, void *stream) {
    if (!h || h->block_size < 0 || h->d < 1 || h->cache_layer_stride < 0) return ETV_ERR_INVALID_ARG;
    if (h->block_size == 0) return ETV_ERR_UNIMPLEMENTED;
    if ((h->elem_bytes != 2 && h->elem_bytes != 4) || (int64_t)h->d * h->elem_bytes % 16 || h->d > (1 << 16)) return ETV_ERR_UNSUPPORTED;
    const etv::ReorderShape sh = etv::reorder_shape(h->B, K, M, h->max_blocks, h->num_blocks, h->block_size);
    etv::CacheParts cache{};
    cache.parts = 2, cache.Hkv = h->Hkv, cache.n_layers = h->n_layers;
    for (int i = 0; i < 2; i++) {
        cache.base[i] = static_cast<uint8_t *>(i ? v_cache : k_cache);
        cache.layer_bytes[i] = (size_t)h->cache_layer_stride * h->elem_bytes;
        cache.row_bytes[i] = h->d * h->elem_bytes;
    }
    if (h->n_layers > 1 && cache.layer_bytes[0] % 16) return ETV_ERR_UNSUPPORTED;
    return etv::reorder(sh, cache, block_table, len, parent, free_blocks, free_state, table_out, free_state_out, status, workspace, workspace_bytes, stream);
}

extern "C" int32_t etv_reorder_beams_q4(const etv_q4_desc *h, uint8_t *k_codes, uint8_t *k_scales, uint8_t *v_codes, uint8_t *v_scales,
                                        const int32_t *block_table, const int32_t *len, int32_t K, const int32_t *parent, int32_t M, int32_t *free_blocks,
                                        const int32_t *free_state, int32_t *table_out, int32_t *free_state_out, int32_t *status, void *workspace,
                                        size_t workspace_bytes, void *stream) {
    if (!h || h->block_size < 0 || h->layer_rows < 0) return ETV_ERR_INVALID_ARG;
    if (h->block_size == 0) return ETV_ERR_UNIMPLEMENTED;
    if (h->block_size % 16 || (h->d != 64 && h->d != 128)) return ETV_ERR_UNSUPPORTED;
    const etv::ReorderShape sh = etv::reorder_shape(h->B, K, M, h->max_blocks, h->num_blocks, h->block_size);
    etv::CacheParts cache{};
    cache.parts = 4, cache.Hkv = h->Hkv, cache.n_layers = h->n_layers;
    uint8_t *base[4] = {k_codes, v_codes, k_scales, v_scales};
    for (int i = 0; i < 4; i++) {
        cache.base[i] = base[i];
        cache.row_bytes[i] = h->d / (i < 2 ? 2 : 32);
        cache.layer_bytes[i] = (size_t)h->layer_rows * cache.row_bytes[i];
    }
    return etv::reorder(sh, cache, block_table, len, parent, free_blocks, free_state, table_out, free_state_out, status, workspace, workspace_bytes, stream);
}
