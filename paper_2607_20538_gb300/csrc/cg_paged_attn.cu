// cg_paged_attn.cu -- attention of new tokens over a paged cache (contract and formulas:
// include/codecgauge_paged.h): the kernel for requests with few query rows, the merge of split
// work, and the entry point.
//
// paged_rows_kernel. A tile of work is 16 query rows of one request and KV head (rows are
// (token, query head of the group), so one read of a key serves all heads that share it) against
// the request's keys and values. It is bound by HBM: 4 d bytes per token and KV head for 4 d n_rep
// flops per query. So every byte is moved once, and everything else is sized to keep copies in
// flight: one warp issues TMA boxes of pages into a ring of 64-token stages; four warps take 16
// tokens each of a stage (mma.sync m16n8k16: the 16 rows fill the instruction, and a tcgen05 tile
// of 128 rows would be 7/8 padding), with their own running maximum, sum and accumulators, joined
// once per tile of work.
// Split: the chunks of all tiles form one line that is cut into equal shares, one per CTA (two CTAs
// per SM), so a batch of ragged lengths and a single long request both load every SM alike. A tile
// that a cut goes through is written in parts; the CTA that writes its last part joins them, in
// their order whoever is last (a merge kernel of its own took 3 us of GPU and 4 us of host time more a
// call). A tile is cut into at most kMaxParts.
// Measured, 8 KV heads of 128 with 4 query heads each: 64 histories of 16384 tokens 632 us, 6.8 TB/s;
// of 4096 174 us, 6.2 TB/s; 256 of 1001 177 us; one of 32768 44 us; one of 1000 14 us (start, four
// copies' latency and the join). Up to 16 rows a request: above, the tiles of cg_paged_chunk.cu are
// faster (4 query heads, 5 tokens = 20 rows: two tiles here read the keys twice).
#include <chrono>

#include "cg_paged_dev.cuh"
#include "cg_tc_common.cuh"
#include "cg_tmap.h"

#define CG_EXPORT __attribute__((visibility("default")))

namespace cg {

int paged_check(const cg_pages* p);
int paged_check_output(int64_t n_tok, int64_t tok, int64_t heads, int64_t head);

namespace {

using namespace paged;

constexpr int kRows = 16;        // query rows of a tile
constexpr int kTK = 64;          // tokens of a stage
constexpr int kWarps = 4;        // consumer warps, 16 tokens of a stage each
constexpr int kThreads = 256;    // the consumers' four warps, and four of which one issues the copies

// One part's place in the workspace: O [16][d], then the reference and sum of each row.
constexpr int part_floats(int d) { return kRows * d + 2 * kRows; }

constexpr int kMaxParts = 64;   // two a lane of the joining warp

template <int D>
struct RowsSmem {
    static constexpr int kStages = D == 64 ? 6 : 3;
    static constexpr uint32_t kHalf = kTK * 128;               // 64 tokens x 64 channels
    static constexpr uint32_t kK = kTK * D * 2;                // keys of a stage; values follow
    static constexpr uint32_t kStage = 2 * kK;
    static constexpr uint32_t merge = kStages * kStage;        // 2 x [16][D] fp32
    static constexpr uint32_t misc = merge + 2 * kRows * D * 4;
    static constexpr uint32_t total = misc + 512;
    static constexpr int kCtas = D == 256 ? 1 : 2;             // per SM
    static_assert(kCtas * (total + 1024) <= 233472, "shared memory budget");
};

struct RowsMisc {
    uint64_t full[6], empty[6];
    int64_t warp_sum[kThreads / 32];
    int64_t share, begin, before;
    int units;           // of the share: end - begin
    int warp_longest[kThreads / 32];
    int start_req, abort_flag, last_part;
    Request start_r;
    float ml[2][2 * kRows];
};
static_assert(sizeof(RowsMisc) <= 512, "misc block");

struct RowsParams {
    PagedArgs a;
    float* parts;
    unsigned long long* written;   // a word per part
    uint64_t epoch;                // of the call
    int max_rows;     // requests with more query rows are left to the other kernel
    int box_rows;
};

// A tile costs its chunks and kLead more, for its queries, joining and output: the copies in flight meanwhile
// fill the ring and no more, so that a CTA of many short tiles falls behind (by 2 to 3 us a tile, where
// a chunk takes 1.5 us). A cut of the line inside the lead falls before the tile. 41 ragged requests of up to
// 7000 tokens, 16 KV heads: 173 us with a lead of 2, 192 with 1, 229 without (172 with 3, which costs
// 64 histories of 16k tokens 637 us against 632). 1640 equal requests of 101 tokens have nothing to
// balance and take 508 us against 491.
constexpr int kLead = 2;

// Cost of a request in line units: (row tiles) x H x (chunks that its rows see, and their lead).
__device__ __forceinline__ int64_t request_cost(const RowsParams& P, int i, int32_t* flag, int* longest) {
    const Request r = load_request(P.a, i, flag);
    const int64_t rows = (int64_t)r.n * P.a.n_rep;
    if (r.n <= 0 || rows > P.max_rows) return 0;
    const Tiles t = visible_tiles<kTK>(P.a.window, P.a.sinks, r.len - r.n, r.len - 1);
    if (t.count() > *longest) *longest = t.count();
    return (rows + kRows - 1) / kRows * P.a.H * (t.count() + kLead);
}

// Walk over a share: request, tile of 16 rows within it (KV head outermost).
struct Walk {
    int i, u;             // request, tile
    int left, x;          // of the share, in line units; offset of the share in the tile
    int n_tiles, n_chunks;
    Request r;
    Tiles t;

    // the tile's first chunk in the share, and the one past its last; the tile goes on past the share
    __device__ __forceinline__ int c() const { return x > kLead ? x - kLead : 0; }
    __device__ __forceinline__ bool goes_on() const { return kLead + n_chunks - x > left; }
    __device__ __forceinline__ int end() const { return goes_on() ? x + left - kLead : n_chunks; }
    __device__ __forceinline__ void set(const RowsParams& P, const Request& req) {
        r = req;
        n_tiles = 0;
        n_chunks = 1;
        const int64_t rows = (int64_t)r.n * P.a.n_rep;
        if (r.n <= 0 || rows > P.max_rows) return;
        t = visible_tiles<kTK>(P.a.window, P.a.sinks, r.len - r.n, r.len - 1);
        n_chunks = t.count();
        n_tiles = (int)((rows + kRows - 1) / kRows) * P.a.H;
    }
    __device__ __forceinline__ void start(const RowsParams& P, int req, const Request& q, int64_t off, int share) {
        i = req;
        left = share;
        set(P, q);
        u = (int)(off / (kLead + n_chunks));
        x = (int)(off - (int64_t)u * (kLead + n_chunks));
        if (end() <= c()) left = 0;                           // the tile begins in the next share
    }
    __device__ __forceinline__ void next_tile(const RowsParams& P) {
        left -= kLead + n_chunks - x;
        x = 0;
        u++;
        while (u >= n_tiles && left > 0) {
            int32_t flag = 0;
            u = 0;
            if (++i >= P.a.n_req) left = 0;
            else set(P, load_request(P.a, i, &flag));
        }
        if (left <= kLead) left = 0;
    }
    // rows of the current tile
    __device__ __forceinline__ int per_head(const RowsParams& P) const { return n_tiles / P.a.H; }
    __device__ __forceinline__ int head(const RowsParams& P) const { return u / per_head(P); }
    __device__ __forceinline__ int row0(const RowsParams& P) const { return (u - head(P) * per_head(P)) * kRows; }
};

// Positions of a tile's first and last row, and whether chunk `id` shows any of them a token.
struct TileSpan {
    int p0, p1, h, row0, n_rows;
    __device__ __forceinline__ TileSpan(const RowsParams& P, const Walk& w) {
        h = w.head(P);
        row0 = w.row0(P);
        const int rows = w.r.n * P.a.n_rep;
        n_rows = rows - row0 < kRows ? rows - row0 : kRows;
        p0 = w.r.len - w.r.n + token_of(P.a, row0);
        p1 = w.r.len - w.r.n + token_of(P.a, row0 + n_rows - 1);
    }
    __device__ __forceinline__ bool sees(const PagedArgs& a, int id) const {
        const int t0 = id * kTK;
        return t0 <= p1 && (!a.window || t0 + kTK > p0 - a.window + 1 || t0 < a.sinks);
    }
    __device__ __forceinline__ bool sees_all(const PagedArgs& a, int id) const {
        const int t0 = id * kTK;
        return t0 + kTK <= p0 + 1 && (!a.window || t0 > p1 - a.window || t0 + kTK <= a.sinks);
    }
};

// With registers exchanged (two CTAs per SM) a wait in the loops must not be a call (wait_here); with one
// CTA it is, which leaves the loop more registers.
template <int D>
__device__ __forceinline__ bool bounded_wait(uint64_t* bar, uint32_t parity, const volatile int* abort, uint64_t limit_ns) {
    return RowsSmem<D>::kCtas == 2 ? wait_here(bar, parity, abort, limit_ns) : mbar_wait(bar, parity, abort, limit_ns);
}

// Special values (infinities, NaN) of a 16-bit pair, as a mask of its halves.
template <bool FP16>
__device__ __forceinline__ uint32_t special_mask(uint32_t v) {
    constexpr uint32_t e = FP16 ? 0x7c00u : 0x7f80u;
    return ((v & e) == e ? 0xffffu : 0u) | ((v & (e << 16)) == (e << 16) ? 0xffff0000u : 0u);
}

// A part's word, beside the part: the call's epoch once the part is written. Words of unused memory
// and of earlier calls hold something else, and the joining CTA leaves 0, so that a replay of a
// captured call starts without. Writes the word of this CTA's part and says whether those of all parts
// are written: of the CTAs that finish at the same time at least one sees so (each writes its own word
// before it reads the others', with a fence between); if two do, both join, to the same values. (A
// counter instead cost up to 16 us: a compare-and-swap per arrival and retry.) The warp that wrote the
// part calls. Its lanes wrote pieces of it on different ways: each fences its own, and the word follows
// when all have; the last fence stands between the words seen and the parts read (by this CTA, behind a
// barrier).
__device__ __forceinline__ bool all_written(unsigned long long* words, int mine, int b0, int parts, uint64_t epoch) {
    const int lane = threadIdx.x & 31;
    auto word = [&](int p) { return reinterpret_cast<volatile unsigned long long*>(words) + ((int64_t)(b0 + p) * 2 + (p == 0 ? 1 : 0)); };
    __threadfence();
    __syncwarp();
    if (lane == 0) reinterpret_cast<volatile unsigned long long*>(words)[mine] = epoch;
    __syncwarp();
    __threadfence();
    bool all = true;
    for (int p = lane; p < parts; p += 32) all &= *word(p) == epoch;
    __threadfence();
    all = __all_sync(0xffffffffu, all);
    if (all)
        for (int p = lane; p < parts; p += 32) *word(p) = 0ull;
    return all;
}

// Joins the parts of a tile: row r = sum_p 2^(ref_p - R) O_p / sum_p 2^(ref_p - R) l_p in the order of
// the parts: CTA b0's second slot, then each next CTA's first. A row per warp and turn.
template <bool FP16, int D>
__device__ __noinline__ void join_parts(const RowsParams& P, int b0, int parts, int tok0, int row0, int n_rows, int h) {
    const PagedArgs& a = P.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int V = D / 32;   // channels of a lane: V lane .. V lane + V - 1
    auto part = [&](int p) { return P.parts + ((int64_t)(b0 + p) * 2 + (p == 0 ? 1 : 0)) * part_floats(D); };
    for (int row = warp; row < n_rows; row += kWarps) {
        // references and sums of parts lane, lane + 32, and the first parts' rows, in one round of loads
        constexpr int kBatch = 32 / V;
        float x[kBatch][V], ref[kMaxParts / 32], ls[kMaxParts / 32], l = 0.0f, R = -INFINITY;
        auto fetch = [&](int p0) {
#pragma unroll
            for (int k = 0; k < kBatch; k++) {
                if (p0 + k >= parts) break;
                const float* src = part(p0 + k) + row * D + V * lane;
#pragma unroll
                for (int e = 0; e < V; e += 2) *reinterpret_cast<float2*>(&x[k][e]) = __ldcg(reinterpret_cast<const float2*>(src + e));
            }
        };
#pragma unroll
        for (int k = 0; k < kMaxParts / 32; k++) {
            const int p = lane + 32 * k;
            ref[k] = p < parts ? __ldcg(part(p) + kRows * D + row) : -INFINITY;
            ls[k] = p < parts ? __ldcg(part(p) + kRows * D + kRows + row) : 0.0f;
        }
        fetch(0);
#pragma unroll
        for (int k = 0; k < kMaxParts / 32; k++) R = fmaxf(R, ref[k]);
#pragma unroll
        for (int off = 16; off; off >>= 1) R = fmaxf(R, __shfl_xor_sync(0xffffffffu, R, off));
        const float Rs = R == -INFINITY ? 0.0f : R;
#pragma unroll
        for (int k = 0; k < kMaxParts / 32; k++) {
            ref[k] = ex2(ref[k] - Rs);
            l = fmaf(ref[k], ls[k], l);
        }
#pragma unroll
        for (int off = 16; off; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
        float o[V];
#pragma unroll
        for (int e = 0; e < V; e++) o[e] = 0.0f;
        for (int p0 = 0; p0 < parts; p0 += kBatch) {
#pragma unroll
            for (int k = 0; k < kBatch; k++) {
                const float f = __shfl_sync(0xffffffffu, p0 < 32 ? ref[0] : ref[1], (p0 + k) & 31);
                if (p0 + k < parts) {   // a part with nothing in it: weight 0, zeros
#pragma unroll
                    for (int e = 0; e < V; e++) o[e] = fmaf(f, x[k][e], o[e]);
                }
            }
            fetch(p0 + kBatch);
        }
        const int r = row0 + row, tk = token_of(a, r), hd = h * a.n_rep + (r - tk * a.n_rep);
        const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
        uint16_t* dst = a.out + (int64_t)(tok0 + tk) * a.o_tok + hd * a.o_head + V * lane;
#pragma unroll
        for (int e = 0; e < V; e += 2) *reinterpret_cast<uint32_t*>(dst + e) = pack2<FP16>(o[e] * inv, o[e + 1] * inv);
        if (a.lse && lane == 0)
            a.lse[(int64_t)(tok0 + tk) * a.H * a.n_rep + hd] = inv == 0.0f ? -INFINITY : RowWeights<FP16>::lse(R, l);
    }
}

template <bool FP16, int D>
__global__ void __launch_bounds__(kThreads, RowsSmem<D>::kCtas)
paged_rows_kernel(const __grid_constant__ RowsParams P, const __grid_constant__ CUtensorMap map) {
    using L = RowsSmem<D>;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the tiles kernel of the call may come beside
    extern __shared__ __align__(1024) unsigned char smem[];
    RowsMisc* M = reinterpret_cast<RowsMisc*>(smem + L::misc);
    float* merge = reinterpret_cast<float*>(smem + L::merge);
    const PagedArgs& a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int32_t flag = 0;

    // ---- this CTA's share of the line of chunks
    const int per = (a.n_req + kThreads - 1) / kThreads;
    const int i_lo = tid * per < a.n_req ? tid * per : a.n_req;
    const int i_hi = i_lo + per < a.n_req ? i_lo + per : a.n_req;
    int64_t mine = 0;
    int longest = 1;
    for (int i = i_lo; i < i_hi; i++) mine += request_cost(P, i, &flag, &longest);
    longest = __reduce_max_sync(0xffffffffu, longest);
    int64_t incl = mine;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const int64_t v = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += v;
    }
    if (lane == 31) {
        M->warp_sum[warp] = incl;
        M->warp_longest[warp] = longest;
    }
    if (tid == 0) {
        for (int s = 0; s < L::kStages; s++) {
            mbar_init(&M->full[s], 1);
            mbar_init(&M->empty[s], kWarps);
        }
        M->abort_flag = (smem_u32(smem) & 1023u) != 0;   // the swizzle needs the alignment asked for
        M->start_req = a.n_req;
        fence_barrier_init();
        prefetch_tmap(&map);
    }
    __syncthreads();
    int64_t before = incl - mine, total = 0;
    for (int w = 0; w < kThreads / 32; w++) {
        if (w < warp) before += M->warp_sum[w];
        total += M->warp_sum[w];
        longest = max(longest, M->warp_longest[w]);
    }
    int64_t share = (total + gridDim.x - 1) / gridDim.x;
    const int least = (longest + kMaxParts - 3) / (kMaxParts - 2);   // cut ends make two parts more
    if (share < least) share = least;
    const int64_t begin = share * blockIdx.x;
    const int64_t end = begin + share < total ? begin + share : total;
    if (begin >= before && begin < before + mine) {
        int64_t at = before;
        for (int i = i_lo; i < i_hi; i++) {
            const int64_t c = per == 1 ? mine : request_cost(P, i, &flag, &longest);
            if (begin < at + c) {
                M->start_req = i;
                M->start_r = load_request(a, i, &flag);
                M->before = begin - at;
                break;
            }
            at += c;
        }
    }
    if (tid == 0) {
        M->share = share;
        M->begin = begin;
        M->units = (int)(end - begin);
    }
    __syncthreads();
    if (blockIdx.x == 0) raise_flag(a.status, flag);
    if (begin >= end) return;
    volatile int* abort_flag = &M->abort_flag;
    Walk w;
    w.start(P, M->start_req, M->start_r, M->before, (int)(end - begin));

    // Registers: 128 a thread at launch; the consumers take what the others give up (128 x 200 + 128 x 56
    // of 256 x 128). With 168 each (five warps, no exchange) their loop spilled.
    if (warp >= kWarps) {
        if (L::kCtas == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp > kWarps) return;
        // ------------------------------------------------------------ producer
        // lane k < n_box carries the boxes of token rows [k box_rows, ...) of a stage
        const int n_box = kTK / P.box_rows;
        int st = 0, ph = 1, issued = 0;
        int32_t pflag = 0;
        bool dead = *abort_flag != 0;
        while (w.left > 0) {
            const TileSpan sp(P, w);
            const int wlo = a.window ? w.r.len - w.r.n - a.window + 1 : 0;   // first token the request still needs
            const int32_t* row = a.table + (int64_t)w.i * a.max_pages;
            const int first = w.c(), take = w.end() - first;
            // the places of a group of chunks are looked up at once, lane = chunk * n_box + box, one
            // group ahead of its use
            const int group = 32 / n_box, mine = lane / n_box, mybox = lane - mine * n_box;
            auto look = [&](int k0) {                // page of the lane's box, or -1: zeros
                const int k = k0 + mine;
                if (k >= take) return -1;
                const int t = w.t.id(first + k) * kTK + mybox * P.box_rows;
                if (!(t < w.r.len && (t + P.box_rows > wlo || t < a.sinks))) return -1;
                const int pg = __ldg(row + (t >> a.page_log2));
                if (pg < 0 || pg >= a.n_pages) {
                    pflag |= CG_FLAG_PAGED_RANGE;
                    return -1;
                }
                return pg;
            };
            int now = look(0), ahead = look(group), in = 0;
            for (int k = 0; k < take; k++, in++) {
                if (in == group) {
                    in = 0;
                    now = ahead;
                    ahead = look(k + group);
                }
                const int pg = __shfl_sync(0xffffffffu, now, (in * n_box + lane) & 31);
                const int id = w.t.id(first + k);
                if (!sp.sees(a, id)) continue;
                // past the pool (page 2 n_pages) the copy fills with zeros
                const int z = pg < 0 ? 2 * a.n_pages : pg, y = pg < 0 ? 0 : sp.h * a.page + ((id * kTK + lane * P.box_rows) & (a.page - 1));
                if (!dead && !__all_sync(0xffffffffu, bounded_wait<D>(&M->empty[st], ph, abort_flag, a.wait_ns))) {
                    dead = true;
                    *abort_flag = 1;
                }
                if (!dead) {
                    if (lane == 0) mbar_arrive_expect_tx(&M->full[st], L::kStage);
                    __syncwarp();
                    if (lane < n_box) {
                        unsigned char* dst = smem + st * L::kStage + lane * P.box_rows * 128;
                        const int zv = z < a.n_pages ? z + a.n_pages : z;
#pragma unroll
                        for (int hf = 0; hf < D / 64; hf++) {
                            tma_load_3d(dst + hf * L::kHalf, &map, &M->full[st], hf * 64, y, z);
                            tma_load_3d(dst + L::kK + hf * L::kHalf, &map, &M->full[st], hf * 64, y, zv);
                        }
                    }
                    issued++;
                }
                if (++st == L::kStages) {
                    st = 0;
                    ph ^= 1;
                }
            }
            w.next_tile(P);
        }
        raise_flag(a.status, pflag);
        // copies in flight land before the CTA ends, also where the consumers gave up on them
        const int zero = 0;
        for (int k = issued > L::kStages ? issued - L::kStages : 0; k < issued; k++)
            bounded_wait<D>(&M->full[k % L::kStages], (k / L::kStages) & 1, &zero, tc::kWaitLimitNs);
    } else {
        // ------------------------------------------------------------ consumers
        if (L::kCtas == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const int g = lane >> 2, j = lane & 3;   // rows g and g + 8; columns 2j, 2j + 1
        const float sl2 = a.scale * kLog2e;
        int st = 0, ph = 0;
        bool dead = *abort_flag != 0;
        while (w.left > 0) {
            const TileSpan sp(P, w);
            const int first = w.c(), take = w.end() - first;
            // queries of rows g, g + 8 as MMA operands
            uint32_t q[D / 16][4];
            int pos[2];
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                const int r = sp.row0 + g + 8 * hf;
                const bool have = g + 8 * hf < sp.n_rows;
                const int tk = token_of(a, r), hd = sp.h * a.n_rep + (r - tk * a.n_rep);
                pos[hf] = have ? w.r.len - w.r.n + tk : -1;
                const uint16_t* src = a.q + (int64_t)(w.r.tok0 + tk) * a.q_tok + hd * a.q_head + 2 * j;
#pragma unroll
                for (int k = 0; k < D / 16; k++) {
                    q[k][hf] = have ? __ldg(reinterpret_cast<const uint32_t*>(src + 16 * k)) : 0u;
                    q[k][2 + hf] = have ? __ldg(reinterpret_cast<const uint32_t*>(src + 16 * k + 8)) : 0u;
                }
            }
            float o[D / 8][4];
#pragma unroll
            for (int k = 0; k < D / 8; k++)
#pragma unroll
                for (int e = 0; e < 4; e++) o[k][e] = 0.0f;
            float ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};

            for (int kc = 0; kc < take; kc++) {
                const int id = w.t.id(first + kc);
                if (!sp.sees(a, id)) continue;
                if (!dead && !__all_sync(0xffffffffu, bounded_wait<D>(&M->full[st], ph, abort_flag, a.wait_ns))) {
                    dead = true;
                    *abort_flag = 1;
                }
                if (!dead) {
                    const uint32_t kbase = smem_u32(smem + st * L::kStage) + (warp * 16) * 128;
                    const uint32_t vbase = kbase + L::kK;
                    const uint32_t x = lane & 7;
                    float s[2][4];
#pragma unroll
                    for (int n = 0; n < 2; n++)
#pragma unroll
                        for (int e = 0; e < 4; e++) s[n][e] = 0.0f;
                    {
                        // matrices: (tokens 0-7, 8-15) x (channel octets 2k, 2k + 1)
                        const uint32_t rowoff = ((lane >> 4) * 8 + x) * 128, oct = (lane >> 3) & 1;
#pragma unroll
                        for (int k = 0; k < D / 16; k++) {
                            uint32_t b[4];
                            const uint32_t ch = 2 * k + oct;
                            ldsm4(b, kbase + (ch >> 3) * L::kHalf + rowoff + (((ch & 7) ^ x) << 4));
                            mma16816<FP16>(s[0], q[k], b[0], b[1]);
                            mma16816<FP16>(s[1], q[k], b[2], b[3]);
                        }
                    }
                    const int t0 = id * kTK + warp * 16 + 2 * j;   // token of s[n][e]: t0 + 8 n + (e & 1)
                    const bool edge = !sp.sees_all(a, id);
#pragma unroll
                    for (int n = 0; n < 2; n++)
#pragma unroll
                        for (int e = 0; e < 4; e++) s[n][e] *= sl2;
                    if (edge) {
#pragma unroll
                        for (int n = 0; n < 2; n++)
#pragma unroll
                            for (int e = 0; e < 4; e++) {
                                const int t = t0 + 8 * n + (e & 1), p = pos[e >> 1];
                                const bool see = t <= p && (!a.window || t > p - a.window || t < a.sinks);
                                s[n][e] = see ? s[n][e] : -INFINITY;
                            }
                    }
                    float mx[2];
#pragma unroll
                    for (int hf = 0; hf < 2; hf++) {
                        mx[hf] = fmaxf(fmaxf(s[0][2 * hf], s[0][2 * hf + 1]), fmaxf(s[1][2 * hf], s[1][2 * hf + 1]));
                        mx[hf] = fmaxf(mx[hf], __shfl_xor_sync(0xffffffffu, mx[hf], 1));
                        mx[hf] = fmaxf(mx[hf], __shfl_xor_sync(0xffffffffu, mx[hf], 2));
                    }
                    constexpr float kBias = RowWeights<FP16>::kBias, kLazy = RowWeights<FP16>::kLazy;
                    if (__any_sync(0xffffffffu, mx[0] > ref[0] + (kBias + kLazy) || mx[1] > ref[1] + (kBias + kLazy))) {
                        float f[2];
#pragma unroll
                        for (int hf = 0; hf < 2; hf++) {
                            const float nr = mx[hf] > ref[hf] + (kBias + kLazy) ? mx[hf] - kBias : ref[hf];
                            f[hf] = ref[hf] == nr ? 1.0f : ex2(ref[hf] - nr);   // 0 at a row's first token
                            ref[hf] = nr;
                            sum[hf] *= f[hf];
                        }
#pragma unroll
                        for (int k = 0; k < D / 8; k++) {
                            o[k][0] *= f[0];
                            o[k][1] *= f[0];
                            o[k][2] *= f[1];
                            o[k][3] *= f[1];
                        }
                    }
                    uint32_t pa[4];
                    {
                        const float r0 = ref[0] == -INFINITY ? 0.0f : ref[0], r1 = ref[1] == -INFINITY ? 0.0f : ref[1];
                        float p[2][4];
#pragma unroll
                        for (int n = 0; n < 2; n++)
#pragma unroll
                            for (int e = 0; e < 4; e++) p[n][e] = ex2(s[n][e] - (e < 2 ? r0 : r1));
                        sum[0] += (p[0][0] + p[0][1]) + (p[1][0] + p[1][1]);
                        sum[1] += (p[0][2] + p[0][3]) + (p[1][2] + p[1][3]);
                        pa[0] = pack2<FP16>(p[0][0], p[0][1]);
                        pa[1] = pack2<FP16>(p[0][2], p[0][3]);
                        pa[2] = pack2<FP16>(p[1][0], p[1][1]);
                        pa[3] = pack2<FP16>(p[1][2], p[1][3]);
                    }
                    {
                        // matrices: (channel octets c, c + 1) x (tokens 0-7, 8-15), transposed
                        const uint32_t rowoff = (((lane >> 3) & 1) * 8 + x) * 128, oct = lane >> 4;
                        if (!edge) {
#pragma unroll
                            for (int k = 0; k < D / 16; k++) {
                                uint32_t b[4];
                                const uint32_t ch = 2 * k + oct;
                                ldsm4t(b, vbase + (ch >> 3) * L::kHalf + rowoff + (((ch & 7) ^ x) << 4));
                                mma16816<FP16>(o[2 * k], pa, b[0], b[1]);
                                mma16816<FP16>(o[2 * k + 1], pa, b[2], b[3]);
                            }
                        } else {
                            // rows past the request hold anything: not used. A special value in a
                            // token that some rows see and others do not must not reach the others
                            // as 0 x inf: it is taken out of the product and added where its
                            // weight counts (the indicator products below).
                            const uint32_t k0 = (t0 < w.r.len ? 0xffffu : 0u) | (t0 + 1 < w.r.len ? 0xffff0000u : 0u);
                            const uint32_t k1 = (t0 + 8 < w.r.len ? 0xffffu : 0u) | (t0 + 9 < w.r.len ? 0xffff0000u : 0u);
                            uint32_t seen[4];   // 1 where the row sees the token
                            constexpr uint32_t kOne = FP16 ? 0x3c00u : 0x3f80u;
#pragma unroll
                            for (int e = 0; e < 4; e++)
                                seen[e] = (s[e >> 1][2 * (e & 1)] != -INFINITY ? kOne : 0u) |
                                          (s[e >> 1][2 * (e & 1) + 1] != -INFINITY ? kOne << 16 : 0u);
#pragma unroll
                            for (int k = 0; k < D / 16; k++) {
                                uint32_t b[4], sp4[4], any = 0;
                                const uint32_t ch = 2 * k + oct;
                                ldsm4t(b, vbase + (ch >> 3) * L::kHalf + rowoff + (((ch & 7) ^ x) << 4));
#pragma unroll
                                for (int e = 0; e < 4; e++) {
                                    b[e] &= e & 1 ? k1 : k0;
                                    sp4[e] = special_mask<FP16>(b[e]);
                                    any |= sp4[e];
                                }
                                if (__any_sync(0xffffffffu, any != 0)) {
                                    constexpr uint32_t kSign = 0x80008000u, kFrac = FP16 ? 0x03ff03ffu : 0x007f007fu;
#pragma unroll
                                    for (int n = 0; n < 2; n++) {
                                        uint32_t nan[2], pinf[2], ninf[2];
#pragma unroll
                                        for (int e = 0; e < 2; e++) {
                                            const uint32_t v = b[2 * n + e], m = sp4[2 * n + e];
                                            const uint32_t fr = ((v & kFrac & 0xffffu) ? 0xffffu : 0u) | ((v & kFrac & 0xffff0000u) ? 0xffff0000u : 0u);
                                            const uint32_t sg = ((v & kSign & 0xffffu) ? 0xffffu : 0u) | ((v & kSign & 0xffff0000u) ? 0xffff0000u : 0u);
                                            nan[e] = m & fr & (kOne * 0x10001u);
                                            pinf[e] = m & ~fr & ~sg & (kOne * 0x10001u);
                                            ninf[e] = m & ~fr & sg & (kOne * 0x10001u);
                                        }
                                        float cn[4] = {0, 0, 0, 0}, cp[4] = {0, 0, 0, 0}, cm[4] = {0, 0, 0, 0};
                                        mma16816<FP16>(cn, seen, nan[0], nan[1]);
                                        mma16816<FP16>(cp, seen, pinf[0], pinf[1]);
                                        mma16816<FP16>(cm, seen, ninf[0], ninf[1]);
#pragma unroll
                                        for (int e = 0; e < 4; e++) {
                                            if (cp[e] > 0.0f) o[2 * k + n][e] += INFINITY;
                                            if (cm[e] > 0.0f) o[2 * k + n][e] -= INFINITY;
                                            if (cn[e] > 0.0f) o[2 * k + n][e] = __uint_as_float(0x7fffffffu);
                                        }
                                    }
#pragma unroll
                                    for (int e = 0; e < 4; e++) b[e] &= ~sp4[e];
                                }
                                mma16816<FP16>(o[2 * k], pa, b[0], b[1]);
                                mma16816<FP16>(o[2 * k + 1], pa, b[2], b[3]);
                            }
                        }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&M->empty[st]);
                }
                if (++st == L::kStages) {
                    st = 0;
                    ph ^= 1;
                }
            }

            // ---- join the four warps: 2, 3 give to 0, 1, then 1 gives to 0
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                sum[hf] += __shfl_xor_sync(0xffffffffu, sum[hf], 1);
                sum[hf] += __shfl_xor_sync(0xffffffffu, sum[hf], 2);
            }
#pragma unroll
            for (int step = 2; step >= 1; step >>= 1) {
                float* buf = merge + (warp & (step - 1)) * kRows * D;
                float* ml = M->ml[warp & (step - 1)];
                if (warp >= step && warp < 2 * step) {
#pragma unroll
                    for (int k = 0; k < D / 8; k++) {
                        *reinterpret_cast<float2*>(buf + g * D + 8 * k + 2 * j) = make_float2(o[k][0], o[k][1]);
                        *reinterpret_cast<float2*>(buf + (g + 8) * D + 8 * k + 2 * j) = make_float2(o[k][2], o[k][3]);
                    }
                    if (j == 0) {
                        ml[g] = ref[0];
                        ml[g + 8] = ref[1];
                        ml[kRows + g] = sum[0];
                        ml[kRows + g + 8] = sum[1];
                    }
                }
                asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
                if (warp < step) {
                    float fa[2], fb[2];
#pragma unroll
                    for (int hf = 0; hf < 2; hf++) {
                        const float ro = ml[g + 8 * hf], so = ml[kRows + g + 8 * hf];
                        const float nr = fmaxf(ref[hf], ro);
                        fa[hf] = ref[hf] == nr ? 1.0f : ex2(ref[hf] - nr);
                        fb[hf] = ro == nr ? 1.0f : ex2(ro - nr);
                        sum[hf] = sum[hf] * fa[hf] + so * fb[hf];
                        ref[hf] = nr;
                    }
#pragma unroll
                    for (int k = 0; k < D / 8; k++) {
                        const float2 x0 = *reinterpret_cast<const float2*>(buf + g * D + 8 * k + 2 * j);
                        const float2 x1 = *reinterpret_cast<const float2*>(buf + (g + 8) * D + 8 * k + 2 * j);
                        o[k][0] = o[k][0] * fa[0] + x0.x * fb[0];
                        o[k][1] = o[k][1] * fa[0] + x0.y * fb[0];
                        o[k][2] = o[k][2] * fa[1] + x1.x * fb[1];
                        o[k][3] = o[k][3] * fa[1] + x1.y * fb[1];
                    }
                }
                asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
            }
            const bool whole = first == 0 && !w.goes_on();
            if (warp == 0) {
                if (whole) {
#pragma unroll
                    for (int hf = 0; hf < 2; hf++) {
                        if (g + 8 * hf >= sp.n_rows) continue;
                        const int r = sp.row0 + g + 8 * hf, tk = token_of(a, r), hd = sp.h * a.n_rep + (r - tk * a.n_rep);
                        const float inv = sum[hf] > 0.0f || sum[hf] != sum[hf] ? 1.0f / sum[hf] : 0.0f;
                        uint16_t* dst = a.out + (int64_t)(w.r.tok0 + tk) * a.o_tok + hd * a.o_head + 2 * j;
#pragma unroll
                        for (int k = 0; k < D / 8; k++)
                            *reinterpret_cast<uint32_t*>(dst + 8 * k) = pack2<FP16>(o[k][2 * hf] * inv, o[k][2 * hf + 1] * inv);
                        if (a.lse && j == 0)
                            a.lse[(int64_t)(w.r.tok0 + tk) * a.H * a.n_rep + hd] =
                                inv == 0.0f ? -INFINITY : RowWeights<FP16>::lse(ref[hf], sum[hf]);
                    }
                } else {
                    float* part = P.parts + ((int64_t)blockIdx.x * 2 + (first ? 0 : 1)) * part_floats(D);
#pragma unroll
                    for (int hf = 0; hf < 2; hf++) {
                        if (g + 8 * hf >= sp.n_rows) continue;
#pragma unroll
                        for (int k = 0; k < D / 8; k++)
                            *reinterpret_cast<float2*>(part + (g + 8 * hf) * D + 8 * k + 2 * j) = make_float2(o[k][2 * hf], o[k][2 * hf + 1]);
                        if (j == 0) {
                            part[kRows * D + g + 8 * hf] = ref[hf];
                            part[kRows * D + kRows + g + 8 * hf] = sum[hf];
                        }
                    }
                }
            }
            if (!whole) {
                const int64_t at = M->begin + (M->units - w.left) - w.x + kLead;   // of the tile's first chunk in the line
                const int b0 = (int)(at / M->share), parts = (int)((at + w.n_chunks - 1) / M->share) - b0 + 1;
                if (warp == 0) {
                    const bool all = all_written(P.written, blockIdx.x * 2 + (first ? 0 : 1), b0, parts, P.epoch);
                    if (lane == 0) M->last_part = all;
                }
                asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
                if (*(volatile int*)&M->last_part) join_parts<FP16, D>(P, b0, parts, w.r.tok0, sp.row0, sp.n_rows, sp.h);
            }
            w.next_tile(P);
        }
        if (dead && tid == 0) raise_flag(a.status, CG_FLAG_PIPE_TIMEOUT);
    }
}

// A number for each call, unlike those of other calls and unlike what unused memory holds: 64 bits that
// start at a hash of the clock, never 0.
uint64_t next_epoch() {
    static std::atomic<uint64_t> n{(uint64_t)std::chrono::high_resolution_clock::now().time_since_epoch().count() * 0x9e3779b97f4a7c15ull};
    const uint64_t e = n.fetch_add(1, std::memory_order_relaxed);
    return e ? e : next_epoch();
}

int rows_ctas(int d) { return tc::num_sms() * (d == 256 ? 1 : 2); }

template <bool FP16, int D>
cudaError_t launch_rows(const RowsParams& P, cudaStream_t st) {
    CUtensorMap map;
    if (!paged_pool_map(&map, P.a, P.box_rows)) return cudaErrorInvalidValue;
    constexpr size_t smem = RowsSmem<D>::total;
    static SmemOptIn opt_in;
    cudaError_t e = opt_in.set(reinterpret_cast<const void*>(paged_rows_kernel<FP16, D>), (int)smem);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)rows_ctas(D);
    paged_rows_kernel<FP16, D><<<grid, kThreads, smem, st>>>(P, map);
    return cudaGetLastError();
}

size_t rows_workspace(int d) {
    const size_t n = (size_t)rows_ctas(d);
    return n * 2 * part_floats(d) * sizeof(float) + n * 2 * sizeof(unsigned long long);
}

}  // namespace

// Tensor map of the pool as [2 n_pages][H page][d], boxes of box_rows x 64 channels, 128-byte swizzle.
bool paged_pool_map(CUtensorMap* map, const PagedArgs& a, uint32_t box_rows) {
    auto fn = tmap_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)a.d, (cuuint64_t)a.H * a.page, 2ull * a.n_pages};
    cuuint64_t strides[2] = {(cuuint64_t)a.d * 2, (cuuint64_t)a.H * a.page * a.d * 2};
    cuuint32_t box[3] = {64, box_rows, 1}, estr[3] = {1, 1, 1};
    return fn(map, a.dtype == CG_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
              const_cast<uint16_t*>(a.pool), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Requests of more query rows run on the 128-row tiles of cg_paged_chunk.cu. Among others up to 16, a
// tile here: 64 histories of 2000 tokens with 16 rows take 101 us here and 113 there, with 20 rows 175 and
// 114 (two tiles read the keys twice). One request alone is cut into many parts, whose rows four warps
// join here and many CTAs there: after 3000 tokens 8 rows take 21.0 us here and 19.5 there (300: 14.7, 16.3),
// 16 rows 28.7 and 19.7; for d = 256 8 rows 26.9 and 22.6.
static int rows_limit(int d, bool alone) { return !alone ? kRows : d == 256 ? 4 : 8; }

// The two kernels of a call may run beside each other: each has its own part of the workspace. The same
// for any number of requests, so that a program can size it once.
size_t paged_attn_workspace(const PagedArgs& a) {
    const size_t r = (rows_workspace(a.d) + 255) / 256 * 256;
    return (int64_t)a.max_new * a.n_rep > rows_limit(a.d, true) ? r + paged_chunk_workspace(a.d) : r;
}

cudaError_t launch_paged_attn(const PagedArgs& a, void* workspace, cudaStream_t st) {
    const int limit = rows_limit(a.d, a.n_req == 1);
    const bool long_ones = (int64_t)a.max_new * a.n_rep > limit;
    cudaError_t e = cudaSuccess;
    // short requests beside long ones; one request alone goes to the tiles whatever its rows
    const bool short_ones = !long_ones || (a.n_req > 1 && a.n_rep <= limit);
    if (short_ones) {
        RowsParams P{};
        P.a = a;
        P.parts = static_cast<float*>(workspace);
        P.written = reinterpret_cast<unsigned long long*>(P.parts + (size_t)rows_ctas(a.d) * 2 * part_floats(a.d));
        P.epoch = next_epoch();
        P.max_rows = limit;
        P.box_rows = a.page < kTK ? a.page : kTK;
        const bool h = a.dtype == CG_FP16;
        switch (a.d) {
            case 64: e = h ? launch_rows<true, 64>(P, st) : launch_rows<false, 64>(P, st); break;
            case 128: e = h ? launch_rows<true, 128>(P, st) : launch_rows<false, 128>(P, st); break;
            default: e = h ? launch_rows<true, 256>(P, st) : launch_rows<false, 256>(P, st); break;
        }
        if (e != cudaSuccess) return e;
    }
    if (long_ones)
        e = launch_paged_chunk(a, short_ones ? limit + 1 : 1, short_ones,
                               static_cast<unsigned char*>(workspace) + (rows_workspace(a.d) + 255) / 256 * 256, st);
    return e;
}

namespace {

int check_attn(const cg_pages* p, const cg_paged_attn* h, PagedArgs* a) {
    int rc = paged_check(p);
    if (rc) return rc;
    if (!h) return set_error(CG_EINVAL, "null attention parameters");
    if (h->n_tok < 0 || h->max_new < 0) return set_error(CG_EINVAL, "n_tok and max_new must be >= 0");
    if (h->n_rep < 1 || h->n_rep > 64) return set_error(CG_EINVAL, "n_rep=%d: query heads per KV head must be 1 .. 64", h->n_rep);
    if ((int64_t)h->n_tok * h->n_rep > 0x7fffffff) return set_error(CG_ERANGE, "n_tok * n_rep must be below 2^31");
    if (h->window < 0 || h->sinks < 0) return set_error(CG_EINVAL, "window and sinks must be >= 0");
    if (h->sinks > 0 && h->window == 0) return set_error(CG_EINVAL, "sinks need a window");
    if (!(h->scale == h->scale) || h->scale == INFINITY || h->scale == -INFINITY)
        return set_error(CG_EINVAL, "softmax scale must be finite");
    for (int64_t s : {h->q_tok, h->q_head, h->o_tok, h->o_head})
        if (s < 0 || s % 8) return set_error(CG_EINVAL, "strides must be non-negative multiples of 8 elements");
    a->dtype = p->dtype;
    a->n_pages = p->n_pages;
    a->page = p->page;
    a->page_log2 = 0;
    while ((1 << a->page_log2) < p->page) a->page_log2++;
    a->H = p->H;
    a->d = p->d;
    a->n_req = p->n_req;
    a->max_pages = p->max_pages;
    a->n_tok = h->n_tok;
    a->n_rep = h->n_rep;
    int up = 0;
    while ((1 << up) < h->n_rep) up++;
    a->rep_shift = 31 + up;
    a->rep_mul = (uint32_t)((((uint64_t)1 << a->rep_shift) + h->n_rep - 1) / h->n_rep);
    a->max_new = h->max_new;
    // a window as long as the longest request cuts nothing
    const bool cuts = h->window > 0 && h->window < (int64_t)p->max_pages * p->page;
    a->window = cuts ? h->window : 0;
    a->sinks = cuts ? h->sinks : 0;
    a->scale = h->scale;
    a->q_tok = h->q_tok;
    a->q_head = h->q_head;
    a->o_tok = h->o_tok;
    a->o_head = h->o_head;
    return CG_OK;
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" {

CG_EXPORT int cg_paged_attention_workspace_bytes(const cg_pages* pages, const cg_paged_attn* how, size_t* bytes) {
    set_error(CG_OK, "%s", "");
    PagedArgs a{};
    const int rc = check_attn(pages, how, &a);
    if (rc) return rc;
    if (bytes) *bytes = paged_attn_workspace(a);
    return CG_OK;
}

CG_EXPORT int cg_paged_attention(const cg_pages* pages, const cg_paged_attn* how, const void* q, const void* pool,
                                 const int32_t* block_table, const int32_t* seq_lens, const int32_t* cu_new, void* out,
                                 float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    set_error(CG_OK, "%s", "");
    PagedArgs a{};
    int rc = check_attn(pages, how, &a);
    if (rc) return rc;
    if ((rc = paged_check_output(a.n_tok, a.o_tok, (int64_t)a.H * a.n_rep, a.o_head))) return rc;
    if (a.n_tok == 0 || a.max_new == 0) return CG_OK;
    if (!q || !pool || !block_table || !seq_lens || !cu_new || !out || !workspace)
        return set_error(CG_EINVAL, "null q, pool, block_table, seq_lens, cu_new, out or workspace pointer");
    for (const void* p : {q, pool, (const void*)out, (const void*)workspace})
        if (reinterpret_cast<uintptr_t>(p) & 15u)
            return set_error(CG_EINVAL, "q, pool, out and workspace must be 16-byte aligned");
    for (const void* p : {(const void*)block_table, (const void*)seq_lens, (const void*)cu_new, (const void*)lse})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return set_error(CG_EINVAL, "pointers must be aligned to their type");
    const size_t need = paged_attn_workspace(a);
    if (workspace_bytes < need) return set_error(CG_EINVAL, "workspace needs %zu bytes (got %zu)", need, workspace_bytes);
    a.q = static_cast<const uint16_t*>(q);
    a.pool = static_cast<const uint16_t*>(pool);
    a.table = block_table;
    a.seq_lens = seq_lens;
    a.cu_new = cu_new;
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    if ((rc = device_status(&a.status))) return rc;
    a.wait_ns = wait_limit_ns();
    const cudaError_t e = launch_paged_attn(a, workspace, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return set_error(CG_ECUDA, "paged attention launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

}  // extern "C"
