// cg_paged_pages.cuh -- pages back on the free stack: the part of the page release that the commit of a
// tree shares.
#pragma once

#include <cooperative_groups.h>

#include "cg_paged.h"

namespace cg {
namespace {

// Request k < n with prefix[k] <= v < prefix[k + 1].
template <class T>
__device__ __forceinline__ int find_request(const T* prefix, int n, T v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Entries of the block table go on the stack in the order of one line, request by request. Those that are no
// pages are passed over, so that an entry's place is the number of pages before it, which only the entries
// tell. One cluster: each of its warps takes an equal piece of the line and counts its pages; after a
// prefix over the CTA's warps and, through distributed shared memory, the cluster's CTAs it puts the
// pages in their places (a piece of more than 128 entries is read once more). Four requests a thread and round,
// each CTA with the prefix of them all.
constexpr int kPushCtas = 8;
constexpr int kPushPer = 4;                        // requests of a thread and round

struct PushArgs {
    const int32_t *table, *count_in;
    int32_t *free_pages, *count_out;
    int n_pages, n_req, max_pages;
};

template <int THREADS, bool FROM_START>
struct PushSmem {
    static constexpr int kRound = THREADS * kPushPer, kWarps = THREADS / 32;
    int64_t first[kRound + 1];      // place in the line of each request's first entry
    int64_t entries[kWarps];        // of each warp's requests
    int64_t pages[kWarps];          // in each warp's piece
    int64_t total[2];               // pages in the CTA's pieces: this round's and the last one's
    int32_t col[FROM_START ? 1 : kRound];   // that entry's column
};

// Sum of the values of the lanes below `warp`, and of all (a value per warp of the CTA, 0 from `warps` on).
__device__ __forceinline__ int64_t over_warps(const int64_t* values, int warps, int warp, int64_t* all) {
    const int lane = threadIdx.x & 31;
    const int64_t v = lane < warps ? values[lane] : 0;
    int64_t incl = v;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const int64_t u = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += u;
    }
    *all = __shfl_sync(0xffffffffu, incl, 31);
    return __shfl_sync(0xffffffffu, incl - v, warp);
}

// lines.prepare(base, n): all threads, before a round's requests [base, base + n).
// lines.entries(i, k, col, flag): entries of request i, the round's k-th, from column *col on (kFromStart: 0).
// All CTAs of the cluster call; none returns before its count has been read.
template <int THREADS, class Lines>
__device__ __forceinline__ void push_pages(const PushArgs& a, PushSmem<THREADS, Lines::kFromStart>& S, const Lines& lines, int32_t* flag) {
    constexpr int kRound = THREADS * kPushPer, kWarps = THREADS / 32;
    auto cluster = cooperative_groups::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster.block_rank();
    int64_t count = *a.count_in;   // pages on the stack
    if (count < 0 || count > a.n_pages) {
        *flag |= CG_FLAG_PAGED_RANGE;
        count = count < 0 ? 0 : a.n_pages;
    }
    int round = 0;
    for (int base = 0; base < a.n_req; base += kRound, round++) {
        const int n = a.n_req - base < kRound ? a.n_req - base : kRound;
        lines.prepare(base, n);
        int64_t np[kPushPer], sum = 0;
#pragma unroll
        for (int k = 0; k < kPushPer; k++) {
            const int i = tid * kPushPer + k;
            np[k] = 0;
            if (i < n) {
                int col = 0;
                np[k] = lines.entries(base + i, i, &col, flag);
                if (!Lines::kFromStart) S.col[i] = col;
            }
            sum += np[k];
        }
        int64_t incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            const int64_t v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        if (lane == 31) S.entries[warp] = incl;
        __syncthreads();
        int64_t all, at = over_warps(S.entries, kWarps, warp, &all) + incl - sum;
#pragma unroll
        for (int k = 0; k < kPushPer; k++) {
            const int i = tid * kPushPer + k;
            if (i < n) S.first[i] = at;
            at += np[k];
        }
        if (tid == 0) S.first[n] = all;
        __syncthreads();

        // the warp's piece [lo, hi) of the line, whole groups of 32 entries
        const int64_t groups = (all + 31) / 32, piece = (groups + kPushCtas * kWarps - 1) / (kPushCtas * kWarps) * 32;
        const int64_t begin = (rank * kWarps + warp) * piece;
        const int64_t lo = begin < all ? begin : all, hi = lo + piece < all ? lo + piece : all;
        // lane's entries of four groups from f0 on; -1: none, or no page
        auto fetch = [&](int64_t f0, int32_t (&id)[4]) {
            int r = -1;
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const int64_t f = f0 + 32 * k + lane;
                id[k] = -1;
                if (f >= hi) continue;
                if (r < 0 || S.first[r + 1] <= f) r = find_request(S.first, n, f);
                const int col = Lines::kFromStart ? 0 : S.col[r];
                id[k] = a.table[(int64_t)(base + r) * a.max_pages + col + (f - S.first[r])];
            }
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (id[k] < -1 || id[k] >= a.n_pages) {
                    *flag |= CG_FLAG_PAGED_RANGE;
                    id[k] = -1;
                }
        };
        int32_t id[4];
        int64_t mine = 0;
        for (int64_t f0 = lo; f0 < hi; f0 += 128) {
            fetch(f0, id);
#pragma unroll
            for (int k = 0; k < 4; k++) mine += __popc(__ballot_sync(0xffffffffu, id[k] >= 0));
        }
        if (lane == 0) S.pages[warp] = mine;
        __syncthreads();
        int64_t here, to = count + over_warps(S.pages, kWarps, warp, &here);
        if (tid == 0) S.total[round & 1] = here;
        cluster.sync();
#pragma unroll
        for (int c = 0; c < kPushCtas; c++) {
            const int64_t v = *cluster.map_shared_rank(&S.total[round & 1], c);
            if (c < rank) to += v;
            count += v;
        }
        for (int64_t f0 = lo; f0 < hi; f0 += 128) {
            if (hi - lo > 128) fetch(f0, id);   // (else they are still there)
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const uint32_t mask = __ballot_sync(0xffffffffu, id[k] >= 0);
                const int64_t place = to + __popc(mask & ((1u << lane) - 1u));
                if (id[k] >= 0) {
                    if (place < a.n_pages) a.free_pages[place] = id[k];
                    else *flag |= CG_FLAG_PAGED_RANGE;
                }
                to += __popc(mask);
            }
        }
        __syncthreads();   // the round's prefix is free again
    }
    if (rank == 0 && tid == 0) *a.count_out = (int32_t)(count < a.n_pages ? count : a.n_pages);
    cluster.sync();        // no CTA ends while its count may be read
}

}  // namespace
}  // namespace cg
