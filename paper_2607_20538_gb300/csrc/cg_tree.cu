// cg_tree.cu -- trees of drafted tokens over the paged cache: positions and masks from parents, the attention's
// entry point (its kernels are those of the paged attention), and the commit of an accepted path.
// Contract: include/codecgauge_tree.h.
#include "../../include/codecgauge_tree.h"
#include "cg_follow.cuh"
#include "cg_overlap.h"
#include "cg_paged.h"
#include "cg_paged_pages.cuh"
#include "cg_tc_common.cuh"

#define CG_EXPORT __attribute__((visibility("default")))

namespace cg {

int paged_check(const cg_pages* p);
int paged_check_sizes(const cg_pages* p);
int paged_check_output(int64_t n_tok, int64_t tok, int64_t heads, int64_t head);

namespace {

// The nodes' order (a parent before its children) makes a path a set of bits in ascending order, and the 32 nodes
// of a word a tree of their own: each lane's ancestors within its word by doubling, 5 rounds, `up` the first one
// before the word. From then on a path is climbed a word a step, whatever its depth.
constexpr int kBadParent = -2;   // ends a path like -1, and raises the flag

// Node 32 w + lane of `n`: its bit and those of its ancestors in the word, and the ancestor that follows.
__device__ __forceinline__ void climb_word(const int32_t* parents, int w, int n, uint32_t* mask, int* up) {
    const int lane = threadIdx.x & 31, k = 32 * w + lane;
    int u = k < n ? *(parents + k) : -1;
    if (u < -1 || u >= k) u = k < n ? kBadParent : -1;
    uint32_t m = 1u << lane;
#pragma unroll
    for (int r = 0; r < 5; r++) {
        const uint32_t om = __shfl_sync(0xffffffffu, m, u & 31);
        const int ou = __shfl_sync(0xffffffffu, u, u & 31);
        if (u >= 32 * w) {
            m |= om;
            u = ou;
        }
    }
    *mask = m;
    *up = u;
}

__device__ __forceinline__ uint32_t drop_lowest(uint32_t bits, int n) {
    for (; n > 0 && bits; n--) bits &= bits - 1;
    return bits;
}

// A request's nodes.
struct Tree {
    int ctx, n, tok0;
};
// most: tokens that a request may have. What does not fit counts as without nodes, behind all its tokens.
__device__ __forceinline__ Tree load_tree(const int32_t* lens, const int32_t* cu, int i, int n_tok, int max_new, int64_t most, int32_t* flag) {
    const int len = *(lens + i), c0 = *(cu + i), c1 = *(cu + i + 1);
    if (c0 >= 0 && c1 >= c0 && c1 <= n_tok && c1 - c0 <= max_new && len >= c1 - c0 && len <= most) return Tree{len - (c1 - c0), c1 - c0, c0};
    *flag |= CG_FLAG_PAGED_RANGE;
    return Tree{len < 0 ? 0 : len, 0, 0};
}

// ------------------------------------------------------------------------------------
// Tree plan. A CTA per request: words climbed by a warp each, into shared memory; then a thread per node
// climbs from word to word, once for its depth and once more, from the last word of its row to the first, for the
// bits. The nodes of a path within a word stand in order of depth, so that a window keeps a word's highest bits and
// sinks its lowest. Bound: launch latency and two dependent loads (lengths, parents). In a graph: one tree of 8 nodes 1.5 us,
// 256 of up to 64 1.9, one of 256 2.4, 64 of 512 6.2. Made for trees like these: a thread writes whole rows, of its share of the nodes, a
// word a step, so that time grows with the square of the nodes: one tree or 8 of 1024 nodes 21 and 23 us, of 8192 1.15 ms (floor of
// the 8: 10 us).
// ------------------------------------------------------------------------------------
constexpr int kPlanThreads = 128;

struct TreePlanArgs {
    const int32_t *parents, *lens, *cu;
    int32_t* positions;
    uint32_t* masks;
    int32_t* status;
    int n_req, n_tok, max_new, window, sinks, words;
};

__global__ void __launch_bounds__(kPlanThreads) tree_plan_kernel(TreePlanArgs a) {
    extern __shared__ uint32_t plan_sm[];
    uint32_t* mask = plan_sm;
    int* up = reinterpret_cast<int*>(plan_sm + a.max_new);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int32_t flag = 0;
    follow();
    const int end = *(a.cu + a.n_req);
    const Tree t = load_tree(a.lens, a.cu, blockIdx.x, a.n_tok, a.max_new, 0x7fffffff, &flag);
    for (int w = warp; 32 * w < t.n; w += kPlanThreads / 32) {
        uint32_t m;
        int u;
        climb_word(a.parents + t.tok0, w, t.n, &m, &u);
        if (32 * w + lane < t.n) {
            mask[32 * w + lane] = m;
            up[32 * w + lane] = u;
        }
    }
    __syncthreads();
    for (int k = tid; k < t.n; k += kPlanThreads) {
        int depth = -1, e = k;
        for (; e >= 0; e = up[e]) depth += __popc(mask[e]);
        if (e == kBadParent) flag |= CG_FLAG_PAGED_RANGE;
        const int64_t row = t.tok0 + k;
        a.positions[row] = t.ctx + depth;
        uint32_t* out = a.masks + row * a.words;
        int nearer = 0;   // nodes of the path behind the word
        e = k;
        for (int w = a.words - 1; w >= 0; w--) {
            uint32_t bits = 0u;
            if (e >= 0 && (e >> 5) == w) {
                bits = mask[e];
                const int c = __popc(bits);
                if (a.window) {
                    const int near = max(0, min(c, a.window - nearer));                    // the highest so many
                    const int far = max(0, min(c, a.sinks - (t.ctx + depth - nearer - c + 1)));   // and the lowest
                    bits = drop_lowest(bits, c - near) | (bits & ~drop_lowest(bits, far));
                }
                nearer += c;
                e = up[e];
            }
            out[w] = bits;
        }
    }
    // rows behind the last request, spread over the grid
    if (end < 0 || end > a.n_tok) flag |= CG_FLAG_PAGED_RANGE;
    else {
        for (int64_t r = end + (int64_t)blockIdx.x * kPlanThreads + tid; r < a.n_tok; r += (int64_t)gridDim.x * kPlanThreads) a.positions[r] = 0;
        const int64_t last = (int64_t)a.n_tok * a.words;
        for (int64_t x = (int64_t)end * a.words + (int64_t)blockIdx.x * kPlanThreads + tid; x < last; x += (int64_t)gridDim.x * kPlanThreads)
            a.masks[x] = 0u;
    }
    raise_flag(a.status, flag);
}

// ------------------------------------------------------------------------------------
// Commit. The first cluster gives pages back: each CTA finds the path lengths of an eighth of a round's requests, a
// warp each, and the others read them through distributed shared memory; then push_pages. The other CTAs move rows,
// a request each (or a part of its columns): the path as bits in shared memory, its rows' places from the block
// table, then each thread moves the same 16 bytes of row after row, in ascending order and a batch at a time.
// Row k receives row r_k >= k, and no later row of the path is read from a place already written, so a thread that
// goes upwards needs nobody else's leave. Bound: chains of dependent loads (lengths, parents, table, rows) for few
// rows; HBM, 4 H d layers bytes read and written a moved row, for many. In a graph: one path in one layer 4.1 us, 64 paths of
// trees of up to 48 nodes in 16 layers (25 MB) 9.9.
// ------------------------------------------------------------------------------------
constexpr int kCommitThreads = 256, kMoveBatch = 8;

struct CommitArgs {
    const int32_t *parents, *leaves, *lens, *cu, *table;
    uint16_t* pool;
    int32_t *lens_left, *status;
    int n_tok, max_new, layers, page, page_log2, n_pages, n_req, max_pages, H, d, parts;
    PushArgs push;
    __device__ __forceinline__ Tree tree(int i, int32_t* flag) const {
        return load_tree(lens, cu, i, n_tok, max_new, (int64_t)max_pages << page_log2, flag);
    }
    // The accepted node, or -1.
    __device__ __forceinline__ int leaf(int i, const Tree& t, int32_t* flag) const {
        const int e = *(leaves + i);
        if (e >= -1 && e < t.n) return e;
        *flag |= CG_FLAG_PAGED_RANGE;
        return -1;
    }
};

constexpr int kCommitRound = kCommitThreads * kPushPer;

struct CommitSmem {
    PushSmem<kCommitThreads, false> push;
    int32_t mine[kCommitRound / kPushCtas];   // path lengths of this CTA's requests
    int32_t path[kCommitRound];               // of all
};

struct Committed {
    static constexpr bool kFromStart = false;
    const CommitArgs& a;
    CommitSmem& S;
    int rank;
    int32_t* flag;

    __device__ __forceinline__ void prepare(int base, int n) const {
        auto cluster = cooperative_groups::this_cluster();
        const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, share = (n + kPushCtas - 1) / kPushCtas;
        for (int k = warp; k < share && rank * share + k < n; k += kCommitThreads / 32) {
            const int i = base + rank * share + k;
            const Tree t = a.tree(i, flag);
            int e = a.leaf(i, t, flag), m = 0;
            while (e >= 0) {
                uint32_t bits;
                int up;
                climb_word(a.parents + t.tok0, e >> 5, e + 1, &bits, &up);
                m += __popc(__shfl_sync(0xffffffffu, bits, e & 31));
                e = __shfl_sync(0xffffffffu, up, e & 31);
            }
            if (e == kBadParent) *flag |= CG_FLAG_PAGED_RANGE;
            if (lane == 0) S.mine[k] = m;
        }
        cluster.sync();
        for (int k = tid; k < n; k += kCommitThreads) S.path[k] = *cluster.map_shared_rank(&S.mine[k % share], k / share);
        __syncthreads();
    }
    __device__ __forceinline__ int64_t entries(int i, int k, int* col, int32_t* f) const {
        const Tree t = a.tree(i, f);
        const int keep = t.ctx + S.path[k];
        if (rank == 0) a.lens_left[i] = keep;
        if (t.n == 0) return 0;
        *col = (int)(((int64_t)keep + a.page - 1) >> a.page_log2);
        return (((int64_t)t.ctx + t.n + a.page - 1) >> a.page_log2) - *col;
    }
};

__device__ __forceinline__ void move_rows(const CommitArgs& a, unsigned char* smem, int i, int part, int32_t* flag) {
    uint32_t* mask = reinterpret_cast<uint32_t*>(smem);
    int* up = reinterpret_cast<int*>(smem) + a.max_new;
    int* words = up + a.max_new;                       // the path's bits
    int* before = words + (CG_TREE_NODES / 32);        // its nodes below each word, and in all
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Tree t = a.tree(i, flag);
    const int leaf = a.leaf(i, t, flag), n_words = (leaf >> 5) + 1;
    if (leaf < 0) return;
    for (int w = warp; w < n_words; w += kCommitThreads / 32) {
        uint32_t m;
        int u;
        climb_word(a.parents + t.tok0, w, leaf + 1, &m, &u);
        if (32 * w + lane <= leaf) {
            mask[32 * w + lane] = m;
            up[32 * w + lane] = u;
        }
    }
    for (int w = tid; w < n_words; w += kCommitThreads) words[w] = 0;
    __syncthreads();
    if (warp == 0) {
        if (lane == 0) {
            int e = leaf;
            for (; e >= 0; e = up[e]) words[e >> 5] = (int)mask[e];
            if (e == kBadParent) *flag |= CG_FLAG_PAGED_RANGE;
        }
        __syncwarp();
        int sum = 0;
        for (int w0 = 0; w0 < n_words; w0 += 32) {
            const int c = w0 + lane < n_words ? __popc((uint32_t)words[w0 + lane]) : 0;
            int incl = c;
#pragma unroll
            for (int off = 1; off < 32; off *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, incl, off);
                if (lane >= off) incl += v;
            }
            if (w0 + lane < n_words) before[w0 + lane] = sum + incl - c;
            sum += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) before[n_words] = sum;
    }
    __syncthreads();
    // the places of the rows, over the words that led there; -1: stays, or in no page
    int *from = reinterpret_cast<int*>(mask), *to = up;
    const int m = before[n_words];
    const int32_t* row = a.table + (int64_t)i * a.max_pages;
    int moved = 0;
    for (int k = tid; k <= leaf; k += kCommitThreads) {
        if (!((uint32_t)words[k >> 5] >> (k & 31) & 1u)) continue;
        const int at = before[k >> 5] + __popc((uint32_t)words[k >> 5] & ((1u << (k & 31)) - 1u));
        int src = -1, dst = -1;
        if (at != k) {
            const int s = t.ctx + k, d = t.ctx + at;
            const int sp = *(row + (s >> a.page_log2)), dp = *(row + (d >> a.page_log2));
            if (sp >= 0 && sp < a.n_pages && dp >= 0 && dp < a.n_pages) {
                src = (sp << a.page_log2) + (s & (a.page - 1));
                dst = (dp << a.page_log2) + (d & (a.page - 1));
                moved = 1;
            } else {
                *flag |= CG_FLAG_PAGED_RANGE;
            }
        }
        from[at] = src;
        to[at] = dst;
    }
    if (!__syncthreads_or(moved)) return;
    const int C = a.d >> 3;                                                  // 16-byte pieces of a row
    const int64_t head = (int64_t)a.page * a.d, half = head * a.H * a.n_pages;   // elements
    auto place = [&](int slot) { return (int64_t)(slot >> a.page_log2) * a.H * head + (int64_t)(slot & (a.page - 1)) * a.d; };
    const int64_t cols = (int64_t)a.layers * 2 * a.H * C;
    for (int64_t x = (int64_t)part * kCommitThreads + tid; x < cols; x += (int64_t)a.parts * kCommitThreads) {
        const int64_t unit = x / C, pool = unit / a.H;
        uint16_t* base = a.pool + pool * half + (unit - pool * a.H) * head + (x - unit * C) * 8;
        for (int k0 = 0; k0 < m; k0 += kMoveBatch) {
            uint4 v[kMoveBatch];
#pragma unroll
            for (int k = 0; k < kMoveBatch; k++)
                if (k0 + k < m && from[k0 + k] >= 0) v[k] = *reinterpret_cast<const uint4*>(base + place(from[k0 + k]));
#pragma unroll
            for (int k = 0; k < kMoveBatch; k++)
                if (k0 + k < m && from[k0 + k] >= 0) *reinterpret_cast<uint4*>(base + place(to[k0 + k])) = v[k];
        }
    }
}

__global__ void __cluster_dims__(kPushCtas, 1, 1) __launch_bounds__(kCommitThreads) tree_commit_kernel(CommitArgs a) {
    extern __shared__ __align__(16) unsigned char commit_sm[];
    int32_t flag = 0;
    follow();
    const int pages_ctas = a.lens_left ? kPushCtas : 0, b = (int)blockIdx.x - pages_ctas;
    if (b < 0) {
        CommitSmem& S = *reinterpret_cast<CommitSmem*>(commit_sm);
        push_pages<kCommitThreads>(a.push, S.push, Committed{a, S, (int)cooperative_groups::this_cluster().block_rank(), &flag}, &flag);
    } else if (b < (int64_t)a.n_req * a.parts && a.pool) {
        move_rows(a, commit_sm, b / a.parts, b % a.parts, &flag);
    }
    raise_flag(a.status, flag);
}

size_t commit_smem(int max_new, bool pages) {
    const size_t rows = (size_t)max_new * 8 + (CG_TREE_NODES / 32) * 8 + 16;
    return pages && rows < sizeof(CommitSmem) ? sizeof(CommitSmem) : rows;
}

bool al4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int log2_of(int v) {
    int k = 0;
    while ((1 << k) < v) k++;
    return k;
}

int check_nodes(int n_tok, int max_new) {
    if (n_tok < 0) return set_error(CG_EINVAL, "n_tok=%d: must be >= 0", n_tok);
    if (max_new < 0 || max_new > CG_TREE_NODES) return set_error(CG_EINVAL, "max_new=%d: nodes of a tree must be 0 .. %d", max_new, CG_TREE_NODES);
    return CG_OK;
}

int check_words(int words, int max_new) {
    if (words < 1 || words > 1 << 20 || (int64_t)words * 32 < max_new)
        return set_error(CG_EINVAL, "mask_words=%d: must hold max_new=%d bits", words, max_new);
    return CG_OK;
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" {

CG_EXPORT int cg_tree_plan(int32_t n_req, int32_t n_tok, int32_t max_new, int32_t window, int32_t sinks, const int32_t* parents,
                           const int32_t* seq_lens, const int32_t* cu_new, int32_t* positions, uint32_t* masks,
                           int32_t mask_words, void* stream) {
    set_error(CG_OK, "%s", "");
    if (n_req < 1 || n_req > 65536) return set_error(CG_EINVAL, "n_req=%d: must be 1 .. 65536", n_req);
    int rc = check_nodes(n_tok, max_new);
    if (!rc) rc = check_words(mask_words, max_new);
    if (rc) return rc;
    if (window < 0 || sinks < 0) return set_error(CG_EINVAL, "window and sinks must be >= 0");
    if (sinks > 0 && window == 0) return set_error(CG_EINVAL, "sinks need a window");
    if (!seq_lens || !cu_new || (n_tok && (!parents || !positions || !masks))) return set_error(CG_EINVAL, "null pointer");
    for (const void* p : {(const void*)parents, (const void*)seq_lens, (const void*)cu_new, (const void*)positions, (const void*)masks})
        if (!al4(p)) return set_error(CG_EINVAL, "pointers must be aligned to their type");
    const Rows pos = span(positions, 4 * (int64_t)n_tok), bits = span(masks, (__int128)n_tok * mask_words * 4);
    bool alias = overlap(pos, bits);
    for (const Rows& in : {span(parents, 4 * (int64_t)n_tok), span(seq_lens, 4 * (int64_t)n_req), span(cu_new, 4 * ((int64_t)n_req + 1))})
        alias = alias || overlap(pos, in) || overlap(bits, in);
    if (alias) return set_error(CG_EINVAL, "positions and masks must not alias the inputs or one another");
    TreePlanArgs a{};
    if ((rc = device_status(&a.status))) return rc;
    a.parents = parents;
    a.lens = seq_lens;
    a.cu = cu_new;
    a.positions = positions;
    a.masks = masks;
    a.n_req = n_req;
    a.n_tok = n_tok;
    a.max_new = max_new;
    a.window = window;
    a.sinks = sinks;
    a.words = mask_words;
    const size_t smem = (size_t)max_new * 8;
    cudaError_t e = cudaSuccess;
    if (smem > 48 * 1024) {
        static SmemOptIn opt_in;
        e = opt_in.set(reinterpret_cast<const void*>(tree_plan_kernel), CG_TREE_NODES * 8);
    }
    if (e == cudaSuccess) e = launch_following(tree_plan_kernel, (unsigned)n_req, kPlanThreads, smem, static_cast<cudaStream_t>(stream), 0, a);
    if (e != cudaSuccess) return set_error(CG_ECUDA, "tree plan launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

CG_EXPORT int cg_tree_attention(const cg_pages* pages, const cg_paged_attn* how, int32_t mask_words, const void* q, const void* pool,
                                const int32_t* block_table, const int32_t* seq_lens, const int32_t* cu_new,
                                const int32_t* positions, const uint32_t* masks, void* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
    set_error(CG_OK, "%s", "");
    PagedArgs a{};
    int rc = paged_attn_check(pages, how, &a);
    if (!rc) rc = check_words(mask_words, how->max_new);
    if (!rc) rc = paged_check_output(a.n_tok, a.o_tok, (int64_t)a.H * a.n_rep, a.o_head);
    if (rc) return rc;
    if (a.n_tok == 0 || a.max_new == 0) return CG_OK;
    if (!masks || (how->window && !positions)) return set_error(CG_EINVAL, "null masks, or positions with a window");
    if (!al4(masks) || !al4(positions)) return set_error(CG_EINVAL, "pointers must be aligned to their type");
    a.masks = masks;
    a.positions = positions;
    a.words = mask_words;
    return paged_attn_run(a, q, pool, block_table, seq_lens, cu_new, out, lse, workspace, workspace_bytes, stream);
}

CG_EXPORT int cg_tree_commit(const cg_pages* pages, int32_t n_tok, int32_t max_new, int32_t layers, const int32_t* parents,
                             const int32_t* leaves, const int32_t* seq_lens, const int32_t* cu_new, const int32_t* block_table,
                             void* pool, int32_t* lens_left, int32_t* free_pages, const int32_t* free_count,
                             int32_t* free_left, void* stream) {
    set_error(CG_OK, "%s", "");
    int rc = pool ? paged_check(pages) : paged_check_sizes(pages);
    if (!rc) rc = check_nodes(n_tok, max_new);
    if (rc) return rc;
    if (layers < 0 || layers > 65536 || (layers == 0) != !pool)
        return set_error(CG_EINVAL, "layers=%d: must be 1 .. 65536 with a pool, 0 without", layers);
    if (!leaves || !seq_lens || !cu_new || !block_table || (n_tok && !parents)) return set_error(CG_EINVAL, "null pointer");
    const bool give = lens_left != nullptr;
    if ((free_pages != nullptr) != give || (free_count != nullptr) != give || (free_left != nullptr) != give)
        return set_error(CG_EINVAL, "lens_left, free_pages, free_count and free_left go together");
    for (const void* p : {(const void*)parents, (const void*)leaves, (const void*)seq_lens, (const void*)cu_new, (const void*)block_table,
                          (const void*)lens_left, (const void*)free_pages, (const void*)free_count, (const void*)free_left})
        if (!al4(p)) return set_error(CG_EINVAL, "pointers must be aligned to their type");
    if (!al16(pool)) return set_error(CG_EINVAL, "pool must be 16-byte aligned");
    if (give) {
        const int64_t req = 4 * (int64_t)pages->n_req;
        const Rows in[] = {span(parents, 4 * (int64_t)n_tok), span(leaves, req), span(seq_lens, req), span(cu_new, req + 4),
                           span(block_table, (__int128)req * pages->max_pages), span(free_count, 4),
                           span(pool, (__int128)layers * 4 * pages->n_pages * pages->page * ((int64_t)pages->H * pages->d))};
        const Rows out[] = {span(lens_left, req), span(free_pages, 4 * (int64_t)pages->n_pages), span(free_left, 4)};
        for (const Rows& o : out)
            for (const Rows& i : in)
                if (overlap(o, i)) return set_error(CG_EINVAL, "lens_left, free_left and free_pages must not alias the inputs");
        if (overlap(out[0], out[1]) || overlap(out[0], out[2]) || overlap(out[1], out[2]))
            return set_error(CG_EINVAL, "lens_left, free_left and free_pages must not alias one another");
    }
    if (!give && !pool) return CG_OK;
    CommitArgs a{};
    if ((rc = device_status(&a.status))) return rc;
    a.parents = parents;
    a.leaves = leaves;
    a.lens = seq_lens;
    a.cu = cu_new;
    a.table = block_table;
    a.pool = static_cast<uint16_t*>(pool);
    a.lens_left = lens_left;
    a.n_tok = n_tok;
    a.max_new = max_new;
    a.layers = layers;
    a.page = pages->page;
    a.page_log2 = log2_of(pages->page);
    a.n_pages = pages->n_pages;
    a.n_req = pages->n_req;
    a.max_pages = pages->max_pages;
    a.H = pages->H;
    a.d = pages->d;
    a.push = PushArgs{block_table, free_count, free_pages, free_left, pages->n_pages, pages->n_req, pages->max_pages};
    // CTAs of one request: enough for a thread a column, as long as all of them fit the GPU at once
    const int64_t cols = (int64_t)layers * 2 * pages->H * (pages->d >> 3);
    const int64_t want = (cols + kCommitThreads - 1) / kCommitThreads, room = 8 * (int64_t)tc::num_sms() / pages->n_req;
    a.parts = pool ? (int)(want < room ? want : room < 1 ? 1 : room) : 0;
    const int64_t ctas = (give ? kPushCtas : 0) + (int64_t)a.n_req * a.parts, grid = (ctas + kPushCtas - 1) / kPushCtas * kPushCtas;
    static SmemOptIn opt_in;
    cudaError_t e = opt_in.set(reinterpret_cast<const void*>(tree_commit_kernel), (int)commit_smem(CG_TREE_NODES, true));
    if (e == cudaSuccess)
        e = launch_following(tree_commit_kernel, (unsigned)grid, kCommitThreads, commit_smem(max_new, give), static_cast<cudaStream_t>(stream), 0, a);
    if (e != cudaSuccess) return set_error(CG_ECUDA, "tree commit launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

}  // extern "C"
