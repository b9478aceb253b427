// Block tables and slot maps from the sequences' lengths: blocks taken from and given back to a ring of free ones, in one launch.
//   old = ceil(len / size), want = ceil(new_len / size); sequence b takes the ring's entries [sum_{b' < b} take, + take) with take = max(0, want - old)
// Every workgroup forms that sum for itself from the lengths (two words a sequence), which no workgroup writes, so that none waits for another.
// Floor: 4 bytes a slot and a block; 32 prompts of up to 8192 rows are 1.1 MB, 0.2 us: the launch and the chain lengths -> sum -> ring -> slots bound the
// call, 5.7 us there and 2.9 us for 64 sequences that grow by a token.
#include "etv_common.h"
#include "free_ring.h"
#include <initializer_list>

namespace etv {

constexpr int kPageWaves = 8, kPageThreads = 64 * kPageWaves;
constexpr int kSlotsPerWg = 1024;  // elements of slot_map that a workgroup writes
constexpr int kFewBlocks = 8;      // so many blocks of a sequence are taken or given back by a thread, all asked for at once, more by a wavefront
constexpr int kMaxRow = (1 << 22) - 1;  // longest table row: kPageThreads of them are counted in 31 bits

// What the lengths alone say of a sequence.
struct PagePlan {
    int32_t st;  // ETV_COMMIT_BAD_LEN / ETV_COMMIT_CAPACITY or 0
    int old, want;
    __device__ int take() const { return st == 0 && want > old ? want - old : 0; }
    __device__ int give() const { return st == 0 && want < old ? old - want : 0; }
};
__device__ __forceinline__ PagePlan page_plan(const etv_pages_desc &dsc, uint32_t inv_bs, int len, int new_len) {
    PagePlan p{0, 0, 0};
    if (len < 0 || new_len < 0 || (long)new_len - len > dsc.S) {
        p.st = ETV_COMMIT_BAD_LEN;
        return p;
    }
    uint32_t rem;
    p.old = (int)fast_div((uint32_t)len + (uint32_t)(dsc.block_size - 1), dsc.block_size, inv_bs, rem);
    p.want = (int)fast_div((uint32_t)new_len + (uint32_t)(dsc.block_size - 1), dsc.block_size, inv_bs, rem);
    if (p.old > dsc.max_blocks || p.want > dsc.max_blocks) p.st = ETV_COMMIT_CAPACITY;
    return p;
}

// Workgroup 0: what is given back, and the ring's new state.  kPageThreads sequences at a time, a thread each; those that give more than a thread holds
// are put in a list, whose sequences the wavefronts share out among themselves.
__device__ void give_back(const etv_pages_desc &dsc, uint32_t inv_bs, const int32_t *len, const int32_t *new_len, const int32_t *block_table,
                          int32_t *free_blocks, const Ring &ring, int32_t *free_state_out, int32_t *len_out, int32_t *status) {
    struct Giver {
        int b, first, n, bad;
        long at;
    };
    __shared__ Giver s_giver[kPageThreads];
    __shared__ unsigned long long s_most[2];
    const int t = threadIdx.x;
    // a wavefront's way along a row, eight entries a lane on their way at a time
    const auto walk = [&](const int32_t *row, int n, auto f) {
        for (int j0 = t & 63; j0 < n; j0 += 8 * 64) {
            int32_t block[8];
#pragma unroll
            for (int i = 0; i < 8; i++) block[i] = row[min(j0 + i * 64, n - 1)];
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (j0 + i * 64 < n) f(j0 + i * 64, block[i]);
        }
    };
    if (t < 2) s_most[t] = 0;
    long taken = 0, given = 0;
    for (int b0 = 0; b0 < dsc.B; b0 += kPageThreads) {
        const int b = b0 + t;
        int L = 0, N = 0;
        PagePlan p{0, 0, 0};
        if (b < dsc.B) {
            L = len[b], N = new_len[b];
            p = page_plan(dsc, inv_bs, L, N);
        }
        const int take = p.take(), give = p.give();
        const long t_end = block_scan_sum<kPageWaves>(take, taken);  // a barrier, too: s_most is set
        if (take > 0 && t_end <= ring.count) atomicMax(&s_most[0], (unsigned long long)t_end);
        if (!__syncthreads_or(give)) continue;
        const bool few = give <= kFewBlocks;
        int32_t own[kFewBlocks] = {};
        int bad = 0;
        if (give > 0 && few) {
            const int32_t *row = block_table + (size_t)b * dsc.max_blocks + p.want;
#pragma unroll
            for (int i = 0; i < kFewBlocks; i++) own[i] = row[min(i, give - 1)];
#pragma unroll
            for (int i = 0; i < kFewBlocks; i++) bad |= (uint32_t)own[i] >= (uint32_t)dsc.num_blocks;
        }
        long before = 0;
        const int place = (int)block_scan_sum<kPageWaves>(!few, before) - 1, n = (int)before;
        if (!few) s_giver[place] = {b, p.want, give, 0, 0};
        __syncthreads();
        for (int s = t >> 6; s < n; s += kPageWaves) {
            const int32_t *row = block_table + (size_t)s_giver[s].b * dsc.max_blocks + s_giver[s].first;
            int bad = 0;
            walk(row, s_giver[s].n, [&](int, int32_t block) { bad |= (uint32_t)block >= (uint32_t)dsc.num_blocks; });
            if (bad) s_giver[s].bad = 1;
        }
        __syncthreads();
        // in the order of the sequences
        if (!few) bad = s_giver[place].bad;
        const int good = bad ? 0 : give;
        const long g_end = block_scan_sum<kPageWaves>(good, given);
        if (give > 0) {
            const int32_t st = !good ? ETV_COMMIT_BAD_BLOCK : g_end > ring.room() ? ETV_BRANCH_BAD_FREE : 0;
            if (!st) atomicMax(&s_most[1], (unsigned long long)g_end);
            const long at = ring.count + g_end - good;
            if (few) {
#pragma unroll
                for (int i = 0; i < kFewBlocks; i++)
                    if (!st && i < give) free_blocks[ring.place(at + i)] = own[i];
            } else {
                s_giver[place].at = at;
                if (st) s_giver[place].n = 0;
            }
            status[b] = st;
            len_out[b] = st ? L : N;
        }
        __syncthreads();
        for (int s = t >> 6; s < n; s += kPageWaves) {
            const Giver g = s_giver[s];
            const int32_t *row = block_table + (size_t)g.b * dsc.max_blocks + g.first;
            walk(row, g.n, [&](int j, int32_t block) { free_blocks[ring.place(g.at + j)] = block; });
        }
        __syncthreads();
    }
    __syncthreads();
    if (t == 0) ring.leave(free_state_out, (long)s_most[0], (long)s_most[1]);
}

// Workgroups 1 ..: kSlotsPerWg elements of the slot map each, and the new table entries, lengths and status of the sequences that start in
// them.  Every workgroup adds up the blocks of the sequences before its own; the sequences' table rows and the ring's entries that
// are read here are written by nobody.
__device__ void grow(const etv_pages_desc &dsc, uint32_t inv_bs, uint32_t inv_S, const int32_t *len, const int32_t *new_len, int32_t *block_table,
                     const int32_t *free_blocks, const Ring &ring, int32_t *len_out, int32_t *slot_map, int32_t *status) {
    __shared__ int s_len[kSlotsPerWg], s_rows[kSlotsPerWg], s_old[kSlotsPerWg], s_tail[kSlotsPerWg], s_many;
    __shared__ long s_base[kSlotsPerWg];
    const int t = threadIdx.x;
    const uint32_t e0 = (blockIdx.x - 1) * kSlotsPerWg, last = (uint32_t)(dsc.B * dsc.S - 1);
    uint32_t rem;
    const int b_lo = (int)fast_div(e0, dsc.S, inv_S, rem), b_hi = (int)fast_div(min(e0 + kSlotsPerWg - 1, last), dsc.S, inv_S, rem);
    const int nb = b_hi - b_lo + 1;
    const int first_len = len[b_lo], first_new = new_len[b_lo];
    long mine = 0;
    for (int b = t; b < b_lo; b += kPageThreads) mine += page_plan(dsc, inv_bs, len[b], new_len[b]).take();
    long base = b_lo > 0 ? block_sum<kPageWaves>(mine) : 0;
    if (nb == 1) {
        // all of one sequence, the usual place of a workgroup where rows are many: tail, share of the ring and slots' blocks are asked for at once
        const PagePlan p = page_plan(dsc, inv_bs, first_len, first_new);
        const int take = p.take(), rows = p.st ? 0 : first_new - first_len;
        int32_t st = p.st;
        if (!st && take > 0 && base + take > ring.count) st = ETV_BRANCH_NO_BLOCKS;
        int32_t *row = block_table + (size_t)b_lo * dsc.max_blocks;
        const bool inside = rows > 0 && (long)p.old * dsc.block_size != first_len;
        const int32_t tail = inside ? row[p.old - 1] : 0;
        int bad = 0, block[kSlotsPerWg / kPageThreads], slot_of[kSlotsPerWg / kPageThreads];
#pragma unroll
        for (int i = 0; i < kSlotsPerWg / kPageThreads; i++) {
            const uint32_t e = e0 + t + i * kPageThreads, r = e - (uint32_t)b_lo * dsc.S;
            uint32_t off = 0;
            const int j = e <= last && (int)r < rows ? (int)fast_div((uint32_t)first_len + r, dsc.block_size, inv_bs, off) : -1;
            slot_of[i] = (int)off;
            block[i] = j < 0 ? -1 : j < p.old || st ? tail : free_blocks[ring.place(base + j - p.old)];
        }
        if (!st)
#pragma unroll 4
            for (int j = t; j < take; j += kPageThreads) bad |= (uint32_t)free_blocks[ring.place(base + j)] >= (uint32_t)dsc.num_blocks;
        bad = __syncthreads_or(bad);
        if (!st && inside && (uint32_t)tail >= (uint32_t)dsc.num_blocks) st = ETV_COMMIT_BAD_BLOCK;
        if (!st && bad) st = ETV_BRANCH_BAD_FREE;
        if (t == 0 && p.give() == 0 && (uint32_t)b_lo * dsc.S >= e0) {
            status[b_lo] = st;
            len_out[b_lo] = st ? first_len : first_new;
        }
#pragma unroll
        for (int i = 0; i < kSlotsPerWg / kPageThreads; i++) {
            const uint32_t e = e0 + t + i * kPageThreads, r = e - (uint32_t)b_lo * dsc.S;
            if (e > last) continue;
            const bool there = !st && (int)r < rows;
            if (slot_map) slot_map[e] = there ? block[i] * dsc.block_size + slot_of[i] : -1;
            if (there && slot_of[i] == 0) row[(first_len + r) / (uint32_t)dsc.block_size] = block[i];
        }
        return;
    }
    if (t == 0) s_many = 0;
    for (int s0 = 0; s0 < nb; s0 += kPageThreads) {
        const int s = s0 + t, b = b_lo + s;
        PagePlan p{0, 0, 0};
        int L = 0, N = 0;
        if (s < nb) {
            L = len[b], N = new_len[b];
            p = page_plan(dsc, inv_bs, L, N);
        }
        const int take = p.take();
        const long end = block_scan_sum<kPageWaves>(take, base);
        if (s >= nb) continue;
        int32_t st = p.st, tail = 0;
        const int rows = st ? 0 : N - L;
        if (!st && take > 0 && end > ring.count) st = ETV_BRANCH_NO_BLOCKS;
        if (rows > 0 && (long)p.old * dsc.block_size != L) {  // the new rows begin in a block that is there
            tail = block_table[(size_t)b * dsc.max_blocks + p.old - 1];
            if (!st && (uint32_t)tail >= (uint32_t)dsc.num_blocks) st = ETV_COMMIT_BAD_BLOCK;
        }
        const bool many = !st && take > kFewBlocks;
        if (many) s_many = 1;  // behind the scan's barriers
        if (!st && take > 0 && !many) {
            int32_t block[kFewBlocks] = {free_blocks[ring.place(end - take)]};
            if (take > 1) {
#pragma unroll
                for (int i = 1; i < kFewBlocks; i++) block[i] = free_blocks[ring.place(end - take + min(i, take - 1))];
#pragma unroll
                for (int i = 1; i < kFewBlocks; i++)
                    if ((uint32_t)block[i] >= (uint32_t)dsc.num_blocks) st = ETV_BRANCH_BAD_FREE;
            }
            if ((uint32_t)block[0] >= (uint32_t)dsc.num_blocks) st = ETV_BRANCH_BAD_FREE;
        }
        s_len[s] = L;
        s_rows[s] = st ? 0 : max(rows, 0);
        s_old[s] = p.old;
        s_tail[s] = tail;
        s_base[s] = end - take;
        const bool starts = (uint32_t)b * dsc.S >= e0;
        if (starts && p.give() == 0 && !many) {
            status[b] = st;
            len_out[b] = st ? L : N;
        }
    }
    __syncthreads();
    if (s_many) {  // every workgroup of a sequence checks all of its share of the ring
        for (int s = t >> 6; s < nb; s += kPageWaves) {
            const int rows = s_rows[s], b = b_lo + s;
            if (rows <= 0) continue;
            uint32_t off;
            const int take = (int)fast_div((uint32_t)s_len[s] + rows + dsc.block_size - 1, dsc.block_size, inv_bs, off) - s_old[s];
            if (take <= kFewBlocks) continue;
            int bad = 0;
#pragma unroll 4
            for (int j = t & 63; j < take; j += 64) bad |= (uint32_t)free_blocks[ring.place(s_base[s] + j)] >= (uint32_t)dsc.num_blocks;
            bad = __ballot(bad) != 0;
            if ((t & 63) == 0) {
                if (bad) s_rows[s] = 0;
                if ((uint32_t)b * dsc.S >= e0) {
                    status[b] = bad ? ETV_BRANCH_BAD_FREE : 0;
                    len_out[b] = s_len[s] + (bad ? 0 : rows);
                }
            }
        }
        __syncthreads();
    }
#pragma unroll 4
    for (int r = t; r < kSlotsPerWg; r += kPageThreads) {
        const uint32_t e = e0 + r;
        if (e > last) continue;
        uint32_t i;
        const int b = (int)fast_div(e, dsc.S, inv_S, i), s = b - b_lo;
        int32_t slot = -1;
        if ((int)i < s_rows[s]) {
            uint32_t off;
            const int j = (int)fast_div((uint32_t)s_len[s] + i, dsc.block_size, inv_bs, off);
            const int block = j < s_old[s] ? s_tail[s] : free_blocks[ring.place(s_base[s] + j - s_old[s])];
            slot = block * dsc.block_size + (int)off;
            if (j >= s_old[s] && off == 0) block_table[(size_t)b * dsc.max_blocks + j] = block;
        }
        if (slot_map) slot_map[e] = slot;
    }
}

__global__ void __launch_bounds__(kPageThreads) resize_tables_kernel(etv_pages_desc dsc, uint32_t inv_bs, uint32_t inv_S, const int32_t *len, const int32_t *new_len,
                                                            int32_t *block_table, int32_t *free_blocks, const int32_t *free_state, int32_t *free_state_out,
                                                            int32_t *len_out, int32_t *slot_map, int32_t *status) {
    const Ring ring(free_state, dsc.num_blocks);
    if (blockIdx.x == 0) give_back(dsc, inv_bs, len, new_len, block_table, free_blocks, ring, free_state_out, len_out, status);
    else grow(dsc, inv_bs, inv_S, len, new_len, block_table, free_blocks, ring, len_out, slot_map, status);
}

}  // namespace etv

extern "C" int32_t etv_resize_block_tables(const etv_pages_desc *h, const int32_t *len, const int32_t *new_len, int32_t *block_table,
                                           int32_t *free_blocks, const int32_t *free_state, int32_t *free_state_out, int32_t *len_out,
                                           int32_t *slot_map, int32_t *status, void *stream) {
    if (!h || h->B < 0 || h->S < 1 || h->block_size < 1 || h->max_blocks < 1 || h->num_blocks < 1) return ETV_ERR_INVALID_ARG;
    if (!free_blocks || !free_state || !free_state_out || etv::overlap(free_state, 8, free_state_out, 8)) return ETV_ERR_INVALID_ARG;
    if (h->B > 0 && (!len || !new_len || !block_table || !len_out || !status)) return ETV_ERR_INVALID_ARG;
    if ((int64_t)h->B * h->S > INT32_MAX - etv::kSlotsPerWg || (int64_t)h->num_blocks * h->block_size > INT32_MAX || h->max_blocks > etv::kMaxRow)
        return ETV_ERR_UNSUPPORTED;
    const size_t lens = 4 * (size_t)h->B;  // all workgroups read them
    for (const int32_t *in : {len, new_len})
        if (etv::overlap(in, lens, len_out, lens) || etv::overlap(in, lens, status, lens) || etv::overlap(in, lens, slot_map, lens * h->S)) return ETV_ERR_INVALID_ARG;
    const unsigned wgs = 1 + (unsigned)(((int64_t)h->B * h->S + etv::kSlotsPerWg - 1) / etv::kSlotsPerWg);
    hipLaunchKernelGGL(etv::resize_tables_kernel, dim3(wgs), dim3(etv::kPageThreads), 0, etv::as_stream(stream), *h, etv::fast_div_inv(h->block_size),
                       etv::fast_div_inv(h->S), len, new_len, block_table, free_blocks, free_state, free_state_out, len_out, slot_map, status);
    return etv::check_launch();
}
