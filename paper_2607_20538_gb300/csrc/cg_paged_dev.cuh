// cg_paged_dev.cuh -- device pieces shared by the paged attention kernels: what a request's rows
// see, 16-bit element helpers, warp-level MMA, TMA boxes of pages.
#pragma once

#include "cg_paged.h"
#include "cg_sm100.cuh"

namespace cg {
namespace paged {

using namespace sm100;

constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLog2e = 1.442695040888963407f;

// Weights are p = 2^(s - ref) with ref = (maximum when it was set) - kBias. The running reference of a
// row is raised only when a score exceeds that maximum by more than kLazy powers of two; below that the
// accumulators need no rescaling.
template <int BIAS, int LAZY>
struct Weights {
    static constexpr float kBias = BIAS, kLazy = LAZY;
    // log-sum-exp from the reference and the sum of the weights: the bias is taken out of both first, so that
    // what is added is small where the result is
    static __device__ __forceinline__ float lse(float ref, float sum) {
        constexpr float unbias = BIAS < 0 ? (float)(1 << (BIAS < 0 ? -BIAS : 0)) : 1.0f / (1 << (BIAS > 0 ? BIAS : 0));
        return ((ref + kBias) + log2f(sum * unbias)) * kLn2;
    }
};
// Tiles of the tensor cores: bf16 has the exponents of fp32, so the reference may lag far (8192 tokens'
// prompt: 378 us with 2^8, 364 with 2^16), and lies that far above the maximum when it is set: weights
// grow from 2^-16 to 1 and take no range from the values. fp16 has few small numbers, so there the bias
// moves the weights up: with 2^8 above it the largest is 2^15 < 65504, and weights down to 2^-21
// of the row's largest stay normal numbers. A row's largest weight is rounded like the others (relative
// error against 64 bits 0.0022 in bf16, 0.00027 in fp16).
template <bool FP16>
using TileWeights = Weights<FP16 ? 7 : -16, FP16 ? 8 : 16>;
// Decode rows: the reference is the maximum, so that a row's largest weight is a power of two and is not
// rounded (relative error against 64 bits 0.0017 in bf16 and 0.00021 in fp16, that of unrounded weights; 0.0022
// and 0.00025 where it may lag by 2^16 and 2^8). Copies bound that kernel: 64 histories of 16384 tokens take 635 us
// with either, 41 ragged ones under a window 191. fp16: largest weight 2^15, normal numbers down to 2^-29 of it.
template <bool FP16>
using RowWeights = Weights<FP16 ? 15 : 0, 0>;

// mbar_wait, whole in its place, for kernels that exchange registers between warps (setmaxnreg): with the
// wait as a call inside their loops the compiler finds no allocation within the split (it does for a call
// at the end of a tile).
__device__ __forceinline__ bool wait_here(uint64_t* bar, uint32_t parity, const volatile int* abort, uint64_t limit_ns) {
    const bool poll = limit_ns < 1000000ull;   // the diagnostic setting of mbar_wait
    if (!poll && mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    for (uint32_t it = 0;; it++) {
        if (poll ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)) return true;
        if (poll || (it & 63u) == 63u) {
            if (*abort) return false;
            if (globaltimer_ns() - t0 > limit_ns) return false;
        }
    }
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <bool FP16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {   // x in the low half
    if (FP16) {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&b);
}

// Row x of a request belongs to its token x / n_rep. rep_mul = ceil(2^shift / n_rep) with shift =
// 31 + ceil(log2 n_rep): the product is off by less than n_rep x / 2^shift < 1 / n_rep.
__device__ __forceinline__ int token_of(const PagedArgs& a, int x) {
    return (int)(((uint64_t)(uint32_t)x * a.rep_mul) >> a.rep_shift);
}

// A request as the attention sees it.
struct Request {
    int len, n, tok0;     // tokens in the pool, new ones, first query row
};

// What a kernel before this one may have written: a tree's kernels come while that one ends (cg_follow.cuh), and
// their loads stay behind the wait for it.
template <bool TREE, class T>
__device__ __forceinline__ T load_input(const T* p) {
    return TREE ? *p : __ldg(p);
}

// Loads and checks a request: lengths that are not covered by the arrays raise the flag (and, in a
// tree's call, more new tokens than tokens).
template <bool TREE>
__device__ __forceinline__ Request load_request(const PagedArgs& a, int i, int32_t* flag) {
    Request r;
    const int c0 = load_input<TREE>(a.cu_new + i), c1 = load_input<TREE>(a.cu_new + i + 1);
    r.len = load_input<TREE>(a.seq_lens + i);
    r.tok0 = c0;
    r.n = c1 - c0;
    const bool ok = c0 >= 0 && c1 >= c0 && c1 <= a.n_tok && r.n <= a.max_new && r.len >= (TREE ? r.n : 0) &&
           (int64_t)r.len <= (int64_t)a.max_pages << a.page_log2;
    if (!ok) {
        *flag |= CG_FLAG_PAGED_RANGE;
        r.n = 0;
    }
    return r;
}

// A tree's rows. Tokens below ctx = len - n are history, which every row sees (with a window: from its position
// on); token ctx + j is node j, seen where bit j of the row's mask says so. A position outside
// [ctx, ctx + node] raises the flag and counts as the nearest of them, so that the tiles of a request follow
// from its lengths alone. 0 where no window asks for it.
__device__ __forceinline__ int tree_position(const PagedArgs& a, const Request& r, int node, int32_t* flag) {
    if (!a.window) return 0;
    const int ctx = r.len - r.n, p = a.positions[r.tok0 + node];
    if (p < ctx || p > ctx + node) *flag |= CG_FLAG_PAGED_RANGE;
    return min(max(p, ctx), ctx + node);
}
// A node's row of masks.
__device__ __forceinline__ const uint32_t* tree_row(const PagedArgs& a, const Request& r, int node) {
    return a.masks + (int64_t)(r.tok0 + node) * a.words;
}
// Nodes [j, j + 32) of a request of n that the row sees, as a word; any j.
__device__ __forceinline__ uint32_t tree_word(const uint32_t* row, int words, int n, int j) {
    if (j <= -32 || j >= n) return 0u;
    const int w = j >> 5;                                  // -1 for j < 0
    const uint32_t lo = w >= 0 ? row[w] : 0u, hi = w + 1 < words ? row[w + 1] : 0u;
    const int left = n - j;                                // bits past the last node are no tokens
    return __funnelshift_r(lo, hi, j & 31) & (left >= 32 ? ~0u : (1u << left) - 1u);
}
// Whether the row of `node` at position p sees token t < len.
__device__ __forceinline__ bool tree_sees(const PagedArgs& a, const Request& r, int node, int p, int t) {
    const int j = t - (r.len - r.n);
    return j < 0 ? !a.window || t > p - a.window || t < a.sinks : (tree_word(tree_row(a, r, node), a.words, r.n, j) & 1u) != 0;
}

// Key tiles of TK tokens that rows at positions [p_first, p_last] of a request of length len see:
// tiles [0, n_sink) and [lo, hi), n_sink <= lo. At least one tile, so that a row that sees nothing
// is still written.
struct Tiles {
    int n_sink, lo, hi;
    __device__ __forceinline__ int count() const { return n_sink + hi - lo; }
    __device__ __forceinline__ int id(int k) const { return k < n_sink ? k : lo + (k - n_sink); }
};

template <int TK>
__device__ __forceinline__ Tiles visible_tiles(int window, int sinks, int p_first, int p_last) {
    Tiles t;
    t.hi = p_last < 0 ? 1 : p_last / TK + 1;
    t.lo = 0;
    t.n_sink = 0;
    if (window) {
        const int64_t from = (int64_t)p_first - window + 1;
        if (from > 0) {
            t.lo = (int)(from / TK);
            if (t.lo >= t.hi) t.lo = t.hi - 1;
            const int s = (int)(((int64_t)sinks + TK - 1) / TK);
            t.n_sink = s < t.lo ? s : t.lo;
        }
    }
    return t;
}

__device__ __forceinline__ void tma_load_3d(void* dst, const void* tmap, uint64_t* bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
        : "memory");
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}

template <bool FP16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (FP16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};\n"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};\n"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

}  // namespace paged
}  // namespace cg
