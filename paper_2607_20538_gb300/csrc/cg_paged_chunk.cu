// cg_paged_chunk.cu -- paged attention of requests with many query rows (a chunk or a whole prompt):
// o = softmax(scale q K^T) V on the tensor cores (contract: include/codecgauge_paged.h).
//
// A tile of work is up to 256 query rows of one request and KV head, as two halves A and B of 128 rows
// (rows are (token, query head of the group), a half the whole tokens that fit); for d = 256 one half. One
// CTA per SM walks its share of the key tiles:
//   warps 0-3, 4-7  softmax of half A, half B: a thread owns a row: 128 scores from tensor memory,
//                   running reference and sum in registers, weights back to tensor memory;
//   warp 8          TMA: 128-token tiles of keys and values in rings of their own, boxes of pages;
//   warps 9, 10     one thread each issues half A's, half B's tcgen05.mma: S = Q K^T (both operands in
//                   shared memory) and O += P V (P in tensor memory over S, V token-major as it
//                   lies in the page);
//   warp 11         loads the queries of a tile (TMA boxes, or gathered: any strides, any n_rep) and
//                   inspects the values of tiles that not every row sees whole (below).
// A half's order is PV(j-1) S(j): while its softmax runs, the tensor cores work for the other half.
// (Both halves from one warp were slower, 0.89 ms against 0.79 ms on 2048 tokens after 32k: its own
// instructions between the products of the two halves, about 900 cycles a step, kept the tensor cores
// idle.) S(j) follows PV(j-1) in issue order, so S may overwrite P, and its completion tells the
// softmax that O is quiescent: the thread rescales its row of O itself on the rare steps that raise
// the reference (by more than TileWeights::kLazy powers of two).
// Bound: the tensor cores (4 x 128 x 128 x d multiply-adds per key tile against 128 x 256 exponentials
// and about four times as many other operations), as far as a half's chain lets them: for d = 128 a
// step takes 2500 cycles, its softmax 1400 of them, and both halves' products 2048. For d = 128 tensor
// memory is full (two halves of scores and accumulators), so that no scores are computed ahead; d = 64 leaves
// 128 columns of it unused. Measured, 32 query heads on 8 KV heads, in long runs (under the power cap):
// 2048 tokens after 32k 0.77 ms, 1.47 PFLOP/s; a prompt of 8192 0.39 ms, 1.41 PFLOP/s (0.68 and 0.365 ms in
// short ones); d = 64 0.29 ms, 0.96 PFLOP/s (half the products for the
// same softmax); d = 256 1.9 ms after 32k, 1.2 PFLOP/s: its tiles of 128 rows need 64 bytes a cycle
// and SM from L2. Sixteen softmax warps (two threads a row, 96 registers) took 1.09 ms: their loop spilled. A
// quarter of the exponentials as polynomials on the FMA units: 0.75 ms against 0.72 the same day.
//
// What a row does not see must not reach it, and 0 x inf would: in tiles that some rows see and
// others do not, warp 11 takes special values (and whatever lies past the request's end) out of the
// value tile before the product; rows that see them add them to O from the pool (a slow path that
// only such inputs take).
//
// Split: the key tiles of all work tiles form one line cut into equal shares, one per CTA; a tile
// that a cut goes through is written in parts and joined by paged_chunk_merge_kernel.
#include "cg_follow.cuh"
#include "cg_paged_dev.cuh"
#include "cg_tc_common.cuh"
#include "cg_tmap.h"

namespace cg {
namespace {

using namespace paged;

constexpr int kHalfRows = 128;    // rows of a half: as many whole tokens (of n_rep rows) as fit
// Tensor memory (512 columns of 128 rows) holds scores and accumulators: two halves of 128 + d columns
// for d <= 128; for d = 256 one half with two score buffers.
constexpr int halves(int d) { return d == 256 ? 1 : 2; }
constexpr int tile_rows(int d) { return halves(d) * kHalfRows; }
constexpr int kKT = 128;          // tokens of a key tile
constexpr int kChunkThreads = 384;

// One part: O as [d / 4][rows of a tile][4], then reference and sum of each row.
constexpr int chunk_part_floats(int d) { return tile_rows(d) * (d + 2); }

struct ChunkMeta {
    int last;            // last CTA with a part of the tile that starts here, or -1: none
    int tok0, n_tok, h;  // its first query row of the call, tokens and KV head
};

template <int D>
struct ChunkSmem {
    // Keys and values have rings of their own: every stage is then waited for, use by use, by each
    // warp that reads it and refilled only after all of them (a wait tells only even from odd uses).
    static constexpr int kKeyStages = D == 64 ? 4 : 2, kValStages = D == 64 ? 4 : 3;
    static constexpr int kStages = kKeyStages + kValStages;
    static constexpr uint32_t kPiece = kKT * 128;                 // 128 rows x 64 channels
    static constexpr int kCh = D < 128 ? D : 128;                 // channels of a stage
    static constexpr int kParts = D / kCh;                        // stages of a key or value tile
    static constexpr uint32_t kStage = kKT * kCh * 2;
    static constexpr uint32_t kQ = kHalfRows * D * 2;             // one half's queries
    static constexpr uint32_t q = 0;
    static constexpr uint32_t stages = halves(D) * kQ;
    static constexpr uint32_t misc = stages + kStages * kStage;
    static constexpr uint32_t total = misc + 512;
    static_assert(total <= 232448, "shared memory budget");
};

// A position in a ring of N stages and the parity of its use.
template <int N>
struct Ring {
    int st = 0, ph = 0;
    __device__ __forceinline__ void next() {
        if (++st == N) {
            st = 0;
            ph ^= 1;
        }
    }
};

struct ChunkMisc {
    uint64_t kfull[4], kempty[4], vfull[4], vempty[4];
    uint64_t sfull[2], pfull[2][2], ofull[2], qfull[2], qempty[2], vok[4], drain[2], pvdone;
    int64_t warp_sum[kChunkThreads / 32];
    uint32_t warp_tiles[kChunkThreads / 32];   // number of work tiles << 16 | units of the largest, both up to 65535
    int units;               // of the share
    int start[4];            // request, head, tile, key tile of the share's beginning
    int special[4];          // the inspected tile held special values
    int accum0[2];           // the half's O was prepared by its softmax before the first product
    int abort_flag;
    int turn;                // 1 while a half's second products and next scores are being issued
    uint32_t tmem;
};
static_assert(sizeof(ChunkMisc) <= 512, "misc block");

struct ChunkParams {
    PagedArgs a;
    float* parts;
    ChunkMeta* meta;
    int min_rows;      // requests with fewer query rows are left to the other kernel
    int min_share;     // key tiles
    int half_tok;      // tokens of a half: 128 / n_rep
    int tile_tok;      // tokens of a work tile
    int box_rows;
    int q_boxes;       // the queries of a half are whole boxes of qmap
};

// Rows of a request at positions p0 .. p1, and the key tiles (by number) that they see: some token
// of tiles [s0, s1) and those below ss, every token for every row of [f0, f1) and those below fs.
struct Span {
    int p0, p1, n, tok;   // (tok: tokens)
    int s0, s1, ss, f0, f1, fs;
    __device__ __forceinline__ bool sees(int id) const { return id < s1 && (id >= s0 || id < ss); }
    __device__ __forceinline__ bool sees_all(int id) const { return id < f1 && (id >= f0 || id < fs); }
    // token t is seen by some rows and not by others, or by none
    __device__ __forceinline__ bool partial(const PagedArgs& a, int t) const {
        return t > p0 || (a.window && t >= a.sinks && p1 - a.window >= t);
    }
};

// Tokens [tok, tok + most) of a request's new ones. Of a tree's nodes each may see every other, and each stands
// somewhere from the end of the history, behind which nothing is seen by all, to the last token: p0 is the
// last token of the history.
template <bool TREE>
__device__ __forceinline__ Span span_of(const PagedArgs& a, const Request& r, int tok, int most) {
    Span s;
    const int left = r.n - tok, n = left < 0 ? 0 : left < most ? left : most;
    s.n = n * a.n_rep;
    s.tok = n;
    s.p0 = TREE ? r.len - r.n - 1 : r.len - r.n + tok;
    s.p1 = TREE ? r.len - 1 : s.p0 + n - 1;
    s.s0 = s.ss = s.f0 = s.fs = 0;
    s.s1 = s.n && s.p1 >= 0 ? s.p1 / kKT + 1 : 0;
    s.f1 = s.p0 < 0 ? 0 : (s.p0 + 1) / kKT;
    if (a.window) {
        const int from = s.p0 + (TREE ? 1 : 0) - a.window + 1, last = s.p1 - a.window;   // first token row p0 sees; last one p1 does not
        s.s0 = from > 0 ? from / kKT : 0;
        s.f0 = last >= 0 ? last / kKT + 1 : 0;
        s.ss = (int)(((int64_t)a.sinks + kKT - 1) / kKT);
        s.fs = a.sinks / kKT;
    }
    return s;
}

template <bool TREE>
__device__ __forceinline__ Tiles tile_tiles(const ChunkParams& P, const Request& r, int m) {
    if (TREE) return visible_tiles<kKT>(P.a.window, P.a.sinks, r.len - r.n, r.len - 1);
    const int tok = m * P.tile_tok, left = r.n - tok, n = left < P.tile_tok ? left : P.tile_tok;
    return visible_tiles<kKT>(P.a.window, P.a.sinks, r.len - r.n + tok, r.len - r.n + tok + n - 1);
}

// A work tile costs its key tiles plus kTileCost (queries in, first scores, output out), in units of
// a key tile. A cut of the line inside those kTileCost units falls before the tile.
constexpr int kTileCost = 3;

// A tile cut in two costs about as much as kSplitCost key tiles: a second start and end, and the joining
// kernel; with few CTAs at work kSplitLeast, as their parts join faster. Where there are no more tiles than
// CTAs and the largest takes no longer than an equal share and that, each CTA takes a whole tile: a
// prompt of 1024 tokens (128 tiles of 4 to 11 units) 26.9 us against 30.4, of 300 18.8 against 20.7. With 12
// instead of 7, 512 tokens after 1000 took 32.4 us against 29.2; with 7 for few CTAs too, 4 tokens after 1000
// took 22.3 us against 18.7. (The look at it costs calls of many tiles 0.7 us.)
constexpr int kSplitCost = 7, kSplitLeast = 4;

__device__ __forceinline__ int row_tiles(const ChunkParams& P, const Request& r) {
    const int64_t rows = (int64_t)r.n * P.a.n_rep;
    return r.n <= 0 || rows < P.min_rows ? 0 : (r.n + P.tile_tok - 1) / P.tile_tok;
}

// Cost of one KV head of each lane's request, and its largest tile's. All lanes call: requests of many
// tiles are summed by the whole warp.
template <bool TREE>
__device__ __forceinline__ int64_t head_cost(const ChunkParams& P, const Request& r, int* largest) {
    const int lane = threadIdx.x & 31, n_m = row_tiles(P, r);
    int64_t sum = 0;
    if (n_m <= 2)
        for (int m = 0; m < n_m; m++) {
            const int c = tile_tiles<TREE>(P, r, m).count() + kTileCost;
            sum += c;
            *largest = max(*largest, c);
        }
    for (uint32_t big = __ballot_sync(0xffffffffu, n_m > 2); big; big &= big - 1) {
        const int src = __ffs(big) - 1;
        Request q;
        q.len = __shfl_sync(0xffffffffu, r.len, src);
        q.n = __shfl_sync(0xffffffffu, r.n, src);
        const int n = __shfl_sync(0xffffffffu, n_m, src);
        int64_t part = 0;
        for (int m = lane; m < n; m += 32) {
            const int c = tile_tiles<TREE>(P, q, m).count() + kTileCost;
            part += c;
            *largest = max(*largest, c);
        }
#pragma unroll
        for (int off = 16; off; off >>= 1) part += __shfl_xor_sync(0xffffffffu, part, off);
        if (lane == src) sum = part;
    }
    return sum;
}

// Row tile of one KV head at offset *off of its line; *off becomes the offset within the tile.
template <bool TREE>
__device__ __forceinline__ int tile_at(const ChunkParams& P, const Request& r, int64_t* off) {
    const int lane = threadIdx.x & 31, n_m = row_tiles(P, r);
    for (int m0 = 0;; m0 += 32) {
        const int m = m0 + lane;
        const int64_t mine = m < n_m ? tile_tiles<TREE>(P, r, m).count() + kTileCost : 0;
        int64_t incl = mine;
#pragma unroll
        for (int k = 1; k < 32; k *= 2) {
            const int64_t v = __shfl_up_sync(0xffffffffu, incl, k);
            if (lane >= k) incl += v;
        }
        const int64_t total = __shfl_sync(0xffffffffu, incl, 31);
        if (*off < total || m0 + 32 >= n_m) {
            const uint32_t here = __ballot_sync(0xffffffffu, *off >= incl - mine && *off < incl);
            const int src = here ? __ffs(here) - 1 : 0;
            *off -= __shfl_sync(0xffffffffu, incl - mine, src);
            return m0 + src;
        }
        *off -= total;
    }
}

// Walk over a share: request, KV head, row tile, key tile.
template <bool TREE>
struct ChunkWalk {
    int i, h, m, n_m;
    int c, take, n;       // first key tile of the current work tile, how many of it, of how many
    int left, x;          // of the share, in line units; offset of the share in the work tile
    bool goes_on;         // the work tile goes on past the share
    int64_t rest;         // by so many line units
    Request r;
    Tiles t;

    __device__ __forceinline__ void load(const ChunkParams& P) {
        int32_t flag = 0;
        n_m = 0;
        if (i >= P.a.n_req) return;
        r = load_request<TREE>(P.a, i, &flag);
        n_m = row_tiles(P, r);
    }
    __device__ __forceinline__ void tile(const ChunkParams& P) {
        t = tile_tiles<TREE>(P, r, m);
        n = t.count();
        c = x > kTileCost ? x - kTileCost : 0;
        goes_on = n + kTileCost - x > left;
        const int e = goes_on ? x + left - kTileCost : n;   // the share's end in the tile
        take = e > c ? e - c : 0;
        rest = n + kTileCost - x - left;
        if (take == 0) left = 0;                            // the tile begins in the next share
    }
    __device__ __forceinline__ void start(const ChunkParams& P, const int (&s)[4], int units) {
        left = units;
        i = s[0];
        h = s[1];
        m = s[2];
        x = s[3];
        if (left <= 0) return;
        load(P);
        tile(P);
    }
    __device__ __forceinline__ void next(const ChunkParams& P) {
        left -= n + kTileCost - x;
        x = 0;
        if (left <= 0) return;
        if (++m >= n_m) {
            m = 0;
            if (++h >= P.a.H) {
                h = 0;
                do {
                    i++;
                    load(P);
                } while (i < P.a.n_req && n_m == 0);
                if (i >= P.a.n_req) {
                    left = 0;
                    return;
                }
            }
        }
        tile(P);
    }
};

__device__ __forceinline__ void tma_load_4d(void* dst, const void* tmap, uint64_t* bar, int x, int y, int z, int w) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}

// ---------------------------------------------------------------- tcgen05 pieces
// Descriptors as halves: a step of the product only adds to the low one.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(d),
        "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}" ::"r"(d),
        "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_ld32p(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// 16 columns times f, in place
__device__ __forceinline__ void tmem_scale16(uint32_t taddr, float f) {
    uint32_t r[16];
    tmem_ld16(taddr, r);
    tmem_wait_ld();
#pragma unroll
    for (int k = 0; k < 16; k++) r[k] = __float_as_uint(__uint_as_float(r[k]) * f);
    tmem_st16(taddr, r);
}

__device__ __forceinline__ void tmem_ld32f(uint32_t taddr, float (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
          "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]),
          "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]),
          "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
        : "r"(taddr));
}
// Uses of r stay behind the wait that precedes this.
__device__ __forceinline__ void settle(float (&r)[32]) {
    asm volatile("" : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]),
                 "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]),
                 "+f"(r[16]), "+f"(r[17]), "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]),
                 "+f"(r[24]), "+f"(r[25]), "+f"(r[26]), "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31]));
}

__device__ __forceinline__ float max32(const float (&s)[32], float m) {
    float m0 = fmaxf(m, fmaxf(s[0], s[1])), m1 = fmaxf(s[2], s[3]);
#pragma unroll
    for (int k = 4; k < 32; k += 4) {
        m0 = fmaxf(m0, fmaxf(s[k], s[k + 1]));
        m1 = fmaxf(m1, fmaxf(s[k + 2], s[k + 3]));
    }
    return fmaxf(m0, m1);
}

// The row's largest score of a tile (128 columns); the first 64 scores stay in u and v.
__device__ __forceinline__ float row_max(uint32_t s_tm, float (&u)[32], float (&v)[32]) {
    tmem_ld32f(s_tm + 64, u);
    tmem_ld32f(s_tm + 96, v);
    tmem_wait_ld();
    settle(u);
    settle(v);
    float m = max32(u, -INFINITY);
    tmem_ld32f(s_tm, u);
    m = max32(v, m);
    tmem_ld32f(s_tm + 32, v);
    tmem_wait_ld();
    settle(u);
    settle(v);
    m = max32(u, m);
    return max32(v, m);
}

// Bits [lo, hi] of a word, for any lo, hi.
__device__ __forceinline__ uint32_t bits_between(int lo, int hi) {
    const uint32_t up = hi < 0 ? 0u : hi >= 31 ? ~0u : (2u << hi) - 1u;
    return lo <= 0 ? up : lo > 31 ? 0u : up & (~0u << lo);
}

// A tile that not every row sees whole: the row sees the columns [lo, hi] and those below sk; the
// others are set to -inf. 64 columns a turn.
template <class More>
__device__ __forceinline__ void mask_row_but(uint32_t s_tm, int lo, int hi, int sk, More more) {
#pragma unroll 1
    for (int c0 = 0; c0 < kKT; c0 += 64) {
        const uint32_t see0 = bits_between(lo - c0, hi - c0) | bits_between(0, (sk - 1 < hi ? sk - 1 : hi) - c0) | more(c0);
        const uint32_t see1 = bits_between(lo - c0 - 32, hi - c0 - 32) | bits_between(0, (sk - 1 < hi ? sk - 1 : hi) - c0 - 32) | more(c0 + 32);
        if (__all_sync(0xffffffffu, (see0 & see1) == ~0u)) continue;
        float u[32], v[32];
        tmem_ld32f(s_tm + c0, u);
        tmem_ld32f(s_tm + c0 + 32, v);
        tmem_wait_ld();
        settle(u);
        settle(v);
        uint32_t r[32];
#pragma unroll
        for (int k = 0; k < 32; k++) r[k] = see0 & (1u << k) ? __float_as_uint(u[k]) : 0xff800000u;
        tmem_st32(s_tm + c0, r);
#pragma unroll
        for (int k = 0; k < 32; k++) r[k] = see1 & (1u << k) ? __float_as_uint(v[k]) : 0xff800000u;
        tmem_st32(s_tm + c0 + 32, r);
    }
    tmem_wait_st();
}
__device__ __noinline__ void mask_row(uint32_t s_tm, int lo, int hi, int sk) {
    mask_row_but(s_tm, lo, hi, sk, [](int) { return 0u; });
}
// The same for a node's row: history, which ends before column -j0, and the nodes of its mask (column 0 is node j0; row
// null: no row, which sees nothing).
__device__ __noinline__ void mask_node(const uint32_t* row, int words, int n, uint32_t s_tm, int j0, int lo, int sk) {
    mask_row_but(s_tm, lo, row ? -1 - j0 : -1, sk, [&](int c) { return row ? tree_word(row, words, n, j0 + c) : 0u; });
}

// Each lane holds 8 pieces of 16 bytes of its row (128 bytes). The 8 lanes of a group transpose them
// (piece k of lane l to lane k, place l), so that a store instruction covers 4 whole lines instead of
// a piece of 32. dst: the row's address, or 0 (not written); off: bytes into the row.
__device__ __forceinline__ void store_rows(uint32_t (&b)[32], uint64_t dst, int off) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int step = 1; step < 8; step *= 2) {
        const bool up = lane & step;
#pragma unroll
        for (int k = 0; k < 8; k++) {
            if (k & step) continue;
#pragma unroll
            for (int e = 0; e < 4; e++) {   // pieces k of the upper lane and k + step of the lower one change places
                uint32_t &x = b[4 * k + e], &y = b[4 * (k + step) + e];
                const uint32_t other = __shfl_xor_sync(0xffffffffu, up ? x : y, step);
                if (up) x = other;
                else y = other;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 8; k++) {
        const uint64_t row = __shfl_sync(0xffffffffu, dst, (lane & 24) + k);
        if (row)
            *reinterpret_cast<uint4*>(row + off + 16 * (lane & 7)) = make_uint4(b[4 * k], b[4 * k + 1], b[4 * k + 2], b[4 * k + 3]);
    }
}

// Weights 2^(s sl2 + neg_ref) of 32 scores in 16 bits, and their sum.
template <bool FP16>
__device__ __forceinline__ void weights32(const float (&s)[32], uint32_t p_tm, float sl2, float neg_ref, float2& acc0, float2& acc1) {
    uint32_t p[16];
#pragma unroll
    for (int k = 0; k < 16; k++) {
        const float2 e = __ffma2_rn(make_float2(s[2 * k], s[2 * k + 1]), make_float2(sl2, sl2), make_float2(neg_ref, neg_ref));
        const float2 w = make_float2(ex2(e.x), ex2(e.y));
        if (k & 1) acc1 = __fadd2_rn(acc1, w);
        else acc0 = __fadd2_rn(acc0, w);
        p[k] = pack2<FP16>(w.x, w.y);
    }
    tmem_st16(p_tm, p);
}

template <bool FP16>
__host__ __device__ constexpr uint32_t idesc16(int M, int N) {
    return (1u << 4) | ((FP16 ? 0u : 1u) << 7) | ((FP16 ? 0u : 1u) << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
constexpr uint32_t kIdescBMnMajor = 1u << 16, kIdescNegateA = 1u << 13;

// Not 0 if a 16-bit value of v is an infinity or NaN (all exponent bits set: adding the lowest of
// them carries into the sign's place).
template <bool FP16>
__device__ __forceinline__ uint32_t special_bits(uint4 v) {
    constexpr uint32_t e = FP16 ? 0x7c007c00u : 0x7f807f80u, c = FP16 ? 0x04000400u : 0x00800080u;
    return (((v.x & e) + c) | ((v.y & e) + c) | ((v.z & e) + c) | ((v.w & e) + c)) & 0x80008000u;
}
template <bool FP16>
__device__ __forceinline__ uint32_t drop_special(uint32_t w) {
    constexpr uint32_t e = FP16 ? 0x7c00u : 0x7f80u;
    return w & (((w & e) == e ? 0u : 0xffffu) | ((w & (e << 16)) == (e << 16) ? 0u : 0xffff0000u));
}
template <bool FP16>
__device__ __forceinline__ float elem(uint32_t bits16) {
    if (FP16) return __half2float(__ushort_as_half((unsigned short)bits16));
    return __uint_as_float(bits16 << 16);
}

// Adds the special values of the partial tokens that this row sees to its row of O (columns of the
// half at o_tm, quiescent); `first`: O holds nothing yet and is set to zero first. All lanes call.
template <bool FP16, int D, bool TREE>
__device__ __noinline__ void add_special(const PagedArgs& a, const Request& r, int req, int h, Span item, int t0, int pos,
                                         int node, uint32_t o_tm, bool first) {
    for (int c0 = 0; c0 < D; c0 += 32) {
        uint32_t o[32];
        if (first) {
#pragma unroll
            for (int k = 0; k < 32; k++) o[k] = 0u;
        } else {
            tmem_ld32p(o_tm + c0, o);
            tmem_wait_ld();
        }
        for (int t = t0; t < t0 + kKT && t < r.len; t++) {
            if (!item.partial(a, t)) continue;
            const bool see = TREE ? node >= 0 && tree_sees(a, r, node, pos, t)
                                  : t <= pos && (!a.window || t > pos - a.window || t < a.sinks);
            if (!__any_sync(0xffffffffu, see)) continue;
            const int pg = load_input<TREE>(a.table + (int64_t)req * a.max_pages + (t >> a.page_log2));
            if (pg < 0 || pg >= a.n_pages) continue;
            const uint16_t* v = a.pool + ((((int64_t)a.n_pages + pg) * a.H + h) * a.page + (t & (a.page - 1))) * D + c0;
#pragma unroll
            for (int k = 0; k < 32; k++) {
                const uint32_t e = FP16 ? 0x7c00u : 0x7f80u, x = v[k];
                if (see && (x & e) == e) o[k] = __float_as_uint(__uint_as_float(o[k]) + elem<FP16>(x));
            }
        }
        tmem_st32(o_tm + c0, o);
    }
    tmem_wait_st();
}

// Takes the CTA's turn to issue (a bounded wait). Without it the two halves' products interleave
// when both are ready, both softmaxes then run at the same time, and the halves stay in step: 2900 to
// 3300 cycles per key tile instead of 2600.
__device__ __forceinline__ bool take_turn(int* turn, bool issue, const volatile int* abort, uint64_t limit_ns) {
    bool ok = true;
    if (issue && atomicCAS(turn, 0, 1) != 0) {
        const uint64_t t0 = globaltimer_ns();
        while (atomicCAS(turn, 0, 1) != 0) {
            if (*abort || globaltimer_ns() - t0 > limit_ns) {
                ok = false;
                break;
            }
        }
    }
    return __all_sync(0xffffffffu, ok);
}

template <bool FP16, int D, bool TREE>
__global__ void __launch_bounds__(kChunkThreads, 1)
paged_chunk_kernel(const __grid_constant__ ChunkParams P, const __grid_constant__ CUtensorMap map,
                   const __grid_constant__ CUtensorMap qmap) {
    using L = ChunkSmem<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    ChunkMisc* M = reinterpret_cast<ChunkMisc*>(smem + L::misc);
    const PagedArgs& a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int32_t flag = 0;
    if (TREE) follow();   // (barriers and tensor memory set up before it: 216 us where this order takes 213, 41 requests under a window)

    // ---- this CTA's share of the line of key tiles
    const int per = (a.n_req + kChunkThreads - 1) / kChunkThreads;
    const int i_lo = tid * per < a.n_req ? tid * per : a.n_req;
    const int i_hi = i_lo + per < a.n_req ? i_lo + per : a.n_req;
    int64_t mine = 0;
    int64_t first_cost = 0;
    int largest = 0;
    uint32_t tiles = 0;          // of this thread's requests, up to 65535
    for (int k = 0; k < per; k++) {
        Request r{};
        if (i_lo + k < i_hi) r = load_request<TREE>(a, i_lo + k, &flag);
        const int64_t c = head_cost<TREE>(P, r, &largest);
        if (k == 0) first_cost = c;
        mine += c * a.H;
        tiles = (uint32_t)min((int64_t)tiles + (int64_t)row_tiles(P, r) * a.H, (int64_t)65535);
    }
    int64_t incl = mine;
    uint32_t tiles_incl = tiles;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const int64_t v = __shfl_up_sync(0xffffffffu, incl, off);
        const uint32_t t = __shfl_up_sync(0xffffffffu, tiles_incl, off);
        if (lane >= off) {
            incl += v;
            tiles_incl += t;
        }
    }
    largest = __reduce_max_sync(0xffffffffu, largest);
    if (lane == 31) {
        M->warp_sum[warp] = incl;
        M->warp_tiles[warp] = min(tiles_incl, 65535u) << 16 | (uint32_t)min(largest, 65535);
    }
    if (tid == 0) {
        M->units = 0;
        for (int s = 0; s < 4; s++) {
            mbar_init(&M->kfull[s], 1);
            mbar_init(&M->kempty[s], halves(D));
            mbar_init(&M->vfull[s], 1);
            mbar_init(&M->vempty[s], halves(D));
        }
        for (int x = 0; x < 2; x++) {
            mbar_init(&M->sfull[x], 1);
            mbar_init(&M->pfull[x][0], 4);
            mbar_init(&M->pfull[x][1], 4);
            mbar_init(&M->ofull[x], 1);
            mbar_init(&M->qfull[x], 1);
            mbar_init(&M->qempty[x], 1);
            mbar_init(&M->drain[x], 1);
            M->accum0[x] = 0;
        }
        for (int s = 0; s < 4; s++) mbar_init(&M->vok[s], 1);
        mbar_init(&M->pvdone, 1);
        M->turn = 0;
        M->abort_flag = (smem_u32(smem) & 1023u) != 0;   // the swizzle needs the alignment asked for
        fence_barrier_init();
        prefetch_tmap(&map);
    }
    if (warp == 9) {
        tmem_alloc(&M->tmem, 512);
        tmem_relinquish();
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = M->tmem;
    int64_t before = incl - mine, total = 0;
    uint32_t tiles_before = tiles_incl - tiles, n_tiles = 0;
#pragma unroll
    for (int w = 0; w < kChunkThreads / 32; w++) {
        const uint32_t t = M->warp_tiles[w];
        if (w < warp) {
            before += M->warp_sum[w];
            tiles_before += t >> 16;
        }
        total += M->warp_sum[w];
        n_tiles += t >> 16;
        largest = max(largest, (int)(t & 0xffffu));
    }
    int64_t share = (total + gridDim.x - 1) / gridDim.x;
    if (share < P.min_share) share = P.min_share;
    const int64_t begin = share * blockIdx.x;
    const int64_t end = begin + share < total ? begin + share : total;
    // a tile for each CTA, or an equal share of the line
    const bool whole_tiles = n_tiles <= gridDim.x && largest <= share + kSplitLeast + (int)((kSplitCost - kSplitLeast) * total / (share * gridDim.x));
    if (whole_tiles) {
        const uint32_t b = blockIdx.x;
        if (b >= tiles_before && b < tiles_before + tiles) {
            uint32_t off = b - tiles_before;
            for (int i = i_lo; i < i_hi; i++) {
                const Request r = load_request<TREE>(a, i, &flag);
                const uint32_t n_m = row_tiles(P, r), n = n_m * a.H;
                if (off < n) {
                    const int m = off % n_m;
                    M->start[0] = i;
                    M->start[1] = off / n_m;
                    M->start[2] = m;
                    M->start[3] = 0;
                    M->units = tile_tiles<TREE>(P, r, m).count() + kTileCost;
                    break;
                }
                off -= n;
            }
        }
    } else if (__any_sync(0xffffffffu, begin >= before && begin < before + mine)) {   // one warp: its lanes look together
        Request r{};
        int req = -1;
        int64_t at = before, hc = 0, off = 0;
        for (int k = 0; k < per; k++) {
            Request q{};
            if (i_lo + k < i_hi) q = load_request<TREE>(a, i_lo + k, &flag);
            const int64_t c = per == 1 ? first_cost : head_cost<TREE>(P, q, &largest);
            if (begin >= at && begin < at + c * a.H) {
                req = i_lo + k;
                r = q;
                hc = c;
                off = begin - at;
            }
            at += c * a.H;
        }
        const int src = __ffs(__ballot_sync(0xffffffffu, req >= 0)) - 1;
        req = __shfl_sync(0xffffffffu, req, src);
        r.len = __shfl_sync(0xffffffffu, r.len, src);
        r.n = __shfl_sync(0xffffffffu, r.n, src);
        hc = __shfl_sync(0xffffffffu, hc, src);
        off = __shfl_sync(0xffffffffu, off, src);
        const int h = (int)(off / hc);
        off -= h * hc;
        const int m = tile_at<TREE>(P, r, &off);
        if (lane == 0) {
            M->start[0] = req;
            M->start[1] = h;
            M->start[2] = m;
            M->start[3] = (int)off;
        }
    }
    __syncthreads();
    if (blockIdx.x == 0) raise_flag(a.status, flag);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    volatile int* abort_flag = &M->abort_flag;
    ChunkWalk<TREE> w;
    w.start(P, M->start, whole_tiles ? M->units : begin < end ? (int)(end - begin) : 0);
    const uint32_t kS = tmem, kO = tmem + 256;

    constexpr bool kOne = halves(D) == 1;
    if (warp < 4 * halves(D)) {
        // ------------------------------------------------------------ softmax
        const int x = warp >> 2;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t o_tm = kO + x * D + lanes;
        // a scale of 0 becomes the least number, so that a masked -inf stays one
        const float sl2 = fmaxf(fabsf(a.scale) * kLog2e, 1.17549435e-38f);
        constexpr float kBias = TileWeights<FP16>::kBias, kLazy = TileWeights<FP16>::kLazy;
        int ns = 0, no = 0, nv = 0;   // active steps, tiles and value tiles so far
        bool head_part = w.left > 0 && w.c > 0, dead = *abort_flag != 0;
        int meta_last = -1;
        while (w.left > 0 && !dead) {
            const int tok = w.m * P.tile_tok + x * P.half_tok;   // the half's first new token
            const Span sp = span_of<TREE>(a, w.r, tok, P.half_tok), item = span_of<TREE>(a, w.r, w.m * P.tile_tok, P.tile_tok);
            const int take = w.take;
            if (!head_part && w.goes_on) {   // it starts here and goes on
                meta_last = (int)(blockIdx.x + (w.rest + share - 1) / share);
                if (tid == 0) {
                    ChunkMeta* m = P.meta + blockIdx.x;
                    m->last = meta_last;
                    m->tok0 = w.r.tok0 + w.m * P.tile_tok;
                    m->n_tok = item.tok;
                    m->h = w.h;
                }
            }
            if (sp.n > 0) {
                const int row = (warp & 3) * 32 + lane;
                const bool have = row < sp.n;
                const int rt = token_of(a, row), tk = tok + rt, hd = w.h * a.n_rep + (row - rt * a.n_rep);
                const int pos = !have ? -1 : TREE ? tree_position(a, w.r, tk, &flag) : sp.p0 + rt;
                float ref = -INFINITY, sum = 0.0f;
                bool started = false;
                for (int kc = 0; kc < take; kc++) {
                    const int id = w.t.id(w.c + kc);
                    if (!sp.sees(id)) continue;
                    // scores and weights: one buffer a half, or (one half) two in turn
                    const int buf = kOne ? ns & 1 : x, turn = kOne ? ns >> 1 : ns;
                    const uint32_t s_tm = kS + buf * 128 + lanes;
                    if (!__all_sync(0xffffffffu, mbar_wait(&M->sfull[buf], turn & 1, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    ns++;
                    // O is quiescent once the last step's product is done. With one buffer the scores
                    // came after it; with two it is waited for where O is touched.
                    auto quiet = [&]() {
                        if (kOne && started && !__all_sync(0xffffffffu, mbar_wait(&M->pvdone, ns & 1, abort_flag, a.wait_ns))) dead = true;
                        return !dead;
                    };
                    tc_fence_after();
                    const int t0 = id * kKT;
                    if (TREE && !sp.sees_all(id))
                        mask_node(have ? tree_row(a, w.r, tk) : nullptr, a.words, w.r.n, s_tm, t0 - (w.r.len - w.r.n), a.window ? pos - a.window + 1 - t0 : 0,
                                  a.sinks - t0);
                    else if (!sp.sees_all(id)) mask_row(s_tm, a.window ? pos - a.window + 1 - t0 : 0, pos - t0, a.sinks - t0);
                    float u[32], v[32];
                    const float mx = sl2 * row_max(s_tm, u, v);
                    // each row by its own scores alone: rows past the tile's end hold anything
                    const bool raise = have && mx > ref + (kBias + kLazy);
                    if (__any_sync(0xffffffffu, raise)) {
                        const float nr = raise ? mx - kBias : ref;
                        // never 0 x inf in O: a factor below all numbers becomes the least one
                        const float f = ref == nr ? 1.0f : fmaxf(ex2(ref - nr), 1.17549435e-38f);
                        if (started && __any_sync(0xffffffffu, raise && ref != -INFINITY)) {   // (a row that has seen nothing holds 0)
                            if (!quiet()) break;
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 16) tmem_scale16(o_tm + c0, f);
                        }
                        sum *= ref == -INFINITY ? 0.0f : f;
                        ref = nr;
                    }
                    if (!item.sees_all(id)) {
                        // the inspected value tile held special values: add those the row sees
                        int special = 0;
                        for (int c = 0; c < L::kParts && !dead; c++) {
                            const int nth = (nv + kc) * L::kParts + c;
                            if (!__all_sync(0xffffffffu, mbar_wait(&M->vok[nth & 3], (nth >> 2) & 1, abort_flag, a.wait_ns))) dead = true;
                            special |= *(volatile int*)&M->special[nth & 3];
                        }
                        if (dead) break;
                        if (special) {
                            if (!quiet()) break;
                            add_special<FP16, D, TREE>(a, w.r, w.i, w.h, item, t0, pos, have ? tk : -1, o_tm, !started);
                            if (!started && lane == 0) *(volatile int*)&M->accum0[x] = 1;
                        }
                    }
                    started = true;
                    // The last 64 scores are read again: 128 of them kept in registers would not leave
                    // room for the rest, and each group of weights lies over scores already read.
                    // The product starts on the first half of the weights.
                    const float nr = ref == -INFINITY ? 0.0f : -ref;
                    float2 acc0 = make_float2(0.0f, 0.0f), acc1 = acc0;
                    weights32<FP16>(u, s_tm, sl2, nr, acc0, acc1);
                    tmem_ld32f(s_tm + 64, u);
                    weights32<FP16>(v, s_tm + 16, sl2, nr, acc0, acc1);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&M->pfull[buf][0]);
                    tmem_ld32f(s_tm + 96, v);
                    tmem_wait_ld();
                    settle(u);
                    settle(v);
                    weights32<FP16>(u, s_tm + 32, sl2, nr, acc0, acc1);
                    weights32<FP16>(v, s_tm + 48, sl2, nr, acc0, acc1);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&M->pfull[buf][1]);
                    sum += (acc0.x + acc0.y) + (acc1.x + acc1.y);
                }
                if (dead) break;
                // on to the next tile while the last products run
                const bool whole = !head_part && !w.goes_on;
                const int tok0 = w.r.tok0;
                w.next(P);
                if (started) {
                    if (!__all_sync(0xffffffffu, mbar_wait(&M->ofull[x], no & 1, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    no++;
                }
                tc_fence_after();
                if (whole) {
                    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
                    uint16_t* dst = a.out + (int64_t)(tok0 + tk) * a.o_tok + hd * a.o_head;
                    const uint64_t my_dst = have ? reinterpret_cast<uint64_t>(dst) : 0;
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 64) {
                        uint32_t b[32];
#pragma unroll
                        for (int q = 0; q < 2; q++) {
                            float o[32];
                            tmem_ld32f(o_tm + c0 + 32 * q, o);
                            tmem_wait_ld();
                            settle(o);
#pragma unroll
                            for (int k = 0; k < 16; k++)
                                b[16 * q + k] = started && inv != 0.0f ? pack2<FP16>(o[2 * k] * inv, o[2 * k + 1] * inv) : 0u;
                        }
                        store_rows(b, my_dst, 2 * c0);
                    }
                    if (a.lse && have)
                        a.lse[(int64_t)(tok0 + tk) * a.H * a.n_rep + hd] = inv == 0.0f ? -INFINITY : TileWeights<FP16>::lse(ref, sum);
                } else {
                    float* part = P.parts + ((int64_t)blockIdx.x * 2 + (head_part ? 0 : 1)) * chunk_part_floats(D);
                    const int r = x * kHalfRows + row;
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 32) {
                        uint32_t o[32];
                        tmem_ld32p(o_tm + c0, o);
                        tmem_wait_ld();
                        if (have) {
#pragma unroll
                            for (int k = 0; k < 8; k++)
                                reinterpret_cast<uint4*>(part)[(c0 / 4 + k) * tile_rows(D) + r] =
                                    started ? make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]) : make_uint4(0, 0, 0, 0);
                        }
                    }
                    if (have) {
                        part[tile_rows(D) * D + r] = ref;
                        part[tile_rows(D) * (D + 1) + r] = sum;
                    }
                }
            }
            head_part = false;
            nv += take;
            if (sp.n <= 0) w.next(P);
        }
        if (tid == 0 && meta_last < 0) P.meta[blockIdx.x].last = -1;
        if (TREE) raise_flag(a.status, flag);   // (positions)
        if (dead) {
            *abort_flag = 1;
            if (lane == 0) raise_flag(a.status, CG_FLAG_PIPE_TIMEOUT);
        }
    } else {
        if (warp == 8) {
            // -------------------------------------------------------- keys and values
            // lane k < n_box carries the boxes of token rows [k box_rows, ...) of a tile
            const int n_box = kKT / P.box_rows;
            int32_t pflag = 0;
            Ring<L::kKeyStages> kr;
            Ring<L::kValStages> vr;
            int ki = 0, vi = 0;      // stages issued
            bool dead = *abort_flag != 0;
            while (w.left > 0 && !dead) {
                const int wlo = a.window ? w.r.len - w.r.n - a.window + 1 : 0;
                const int32_t* row = a.table + (int64_t)w.i * a.max_pages;
                const int take = w.take;
                // the places of a group of tiles are looked up at once, lane = tile * n_box + box,
                // one group ahead of its use
                const int group = 32 / n_box, mine = lane / n_box, mybox = lane - mine * n_box;
                auto look = [&](int kc0) {               // page of the lane's box, or -1: zeros
                    const int kc = kc0 + mine;
                    if (mine >= group || kc >= take) return -1;
                    const int t = w.t.id(w.c + kc) * kKT + mybox * P.box_rows;
                    if (!(t < w.r.len && (t + P.box_rows > wlo || t < a.sinks))) return -1;
                    const int pg = load_input<TREE>(row + (t >> a.page_log2));
                    if (pg < 0 || pg >= a.n_pages) {
                        pflag |= CG_FLAG_PAGED_RANGE;
                        return -1;
                    }
                    return pg;
                };
                int now = look(0), ahead = look(group), base = 0;   // base: first tile of `now`
                // the stages of the keys (kv = 0) or values of tile kc
                auto load = [&](int kc, int kv) {
                    const int in = kc - base;
                    const int pg = __shfl_sync(0xffffffffu, in < group ? now : ahead, ((in % group) * n_box + lane) & 31);
                    const int t = w.t.id(w.c + kc) * kKT + lane * P.box_rows;
                    const int z = pg < 0 ? 2 * a.n_pages : kv ? pg + a.n_pages : pg, y = pg < 0 ? 0 : w.h * a.page + (t & (a.page - 1));
#pragma unroll
                    for (int c = 0; c < L::kParts; c++) {
                        uint64_t *full = kv ? &M->vfull[vr.st] : &M->kfull[kr.st], *empty = kv ? &M->vempty[vr.st] : &M->kempty[kr.st];
                        if (dead || !__all_sync(0xffffffffu, mbar_wait(empty, (kv ? vr.ph : kr.ph) ^ 1, abort_flag, a.wait_ns))) {
                            dead = true;
                            return;
                        }
                        if (lane == 0) mbar_arrive_expect_tx(full, L::kStage);
                        __syncwarp();
                        if (lane < n_box) {
                            unsigned char* dst = smem + L::stages + (kv ? L::kKeyStages + vr.st : kr.st) * L::kStage + lane * P.box_rows * 128;
#pragma unroll
                            for (int hf = 0; hf < L::kCh / 64; hf++)
                                tma_load_3d(dst + hf * L::kPiece, &map, full, c * L::kCh + hf * 64, y, z);
                        }
                        if (kv) {
                            vi++;
                            vr.next();
                        } else {
                            ki++;
                            kr.next();
                        }
                    }
                };
                if (kOne) load(0, 0);   // with two score buffers the keys are one tile ahead
                for (int kc = 0; kc < take && !dead; kc++) {
                    if (!kOne) load(kc, 0);
                    else if (kc + 1 < take) load(kc + 1, 0);
                    load(kc, 1);
                    if (kc + 1 - base == group) {
                        base += group;
                        now = ahead;
                        ahead = look(base + group);
                    }
                }
                w.next(P);
            }
            raise_flag(a.status, pflag);
            if (dead) *abort_flag = 1;
            // copies in flight land before the CTA ends, also where the other warps gave up on them
            const int zero = 0;
            for (int k = ki > L::kKeyStages ? ki - L::kKeyStages : 0; k < ki; k++)
                mbar_wait(&M->kfull[k % L::kKeyStages], (k / L::kKeyStages) & 1, &zero, tc::kWaitLimitNs);
            for (int k = vi > L::kValStages ? vi - L::kValStages : 0; k < vi; k++)
                mbar_wait(&M->vfull[k % L::kValStages], (k / L::kValStages) & 1, &zero, tc::kWaitLimitNs);
        } else if (warp == 9 || (warp == 10 && !kOne)) {
            // -------------------------------------------------------- MMA issuer of one half
            // One half alone (d = 256): S(0) S(1) PV(0) S(2) PV(1) ..., the next scores in the other
            // buffer while a step's softmax runs; its step takes as long as the products.
            // The whole warp walks and waits, so that descriptors stay in uniform registers; one
            // thread issues. Everything a step needs is waited for ahead of the weights.
            const int x = warp - 9;
            const bool issue = elect_one();
            const uint32_t idesc_s = idesc16<FP16>(128, kKT) | (a.scale < 0.0f ? kIdescNegateA : 0u);
            constexpr uint32_t idesc_o = idesc16<FP16>(128, L::kCh) | kIdescBMnMajor;
            const uint64_t qd = sdesc_sw128(smem_u32(smem + L::q)), kd = sdesc_sw128(smem_u32(smem + L::stages));
            const uint64_t vd = sdesc_sw128_mn(smem_u32(smem + L::stages + L::kKeyStages * L::kStage), L::kPiece, 1024u);
            const uint32_t al = (uint32_t)qd + ((x * L::kQ) >> 4), k_lo = (uint32_t)kd, hi = (uint32_t)(kd >> 32);
            const uint32_t v_lo = (uint32_t)vd, v_hi = (uint32_t)(vd >> 32);
            const uint32_t ox = kO + x * D;
            Ring<L::kKeyStages> kr;
            Ring<L::kValStages> vr;
            int np = 0, nq = 0, nv = 0;
            bool dead = *abort_flag != 0;
            auto wait = [&](uint64_t* bar, int parity) {
                if (!__all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, a.wait_ns))) dead = true;
                return !dead;
            };
            int ns = 0;                        // scores issued (np: products)
            bool first = true;                 // of the tile's products
            // Scores of the keys at the ring's position into their buffer; the stages are released.
            // Where the half sees nothing of the tile the stages are only waited for.
            auto scores = [&](bool go, bool last) {
                const int buf = kOne ? ns & 1 : x;
#pragma unroll
                for (int c = 0; c < L::kParts; c++) {
                    if (!wait(&M->kfull[kr.st], kr.ph)) return;
                    tc_fence_after();
                    const uint32_t bk = k_lo + ((kr.st * L::kStage) >> 4);
                    if (issue) {
                        if (go) {
#pragma unroll
                            for (int k = 0; k < L::kCh / 16; k++) {
                                const uint32_t o = ((k >> 2) * L::kPiece + (k & 3) * 32) >> 4;
                                mma_ss(kS + buf * 128, al + ((c * L::kCh / 64 * L::kPiece) >> 4) + o, bk + o, hi, idesc_s, c + k ? 1u : 0u);
                            }
                            if (c == L::kParts - 1) mma_commit(&M->sfull[buf]);
                        }
                        if (last && c == L::kParts - 1) mma_commit(&M->qempty[x]);   // the queries were read
                        mma_commit(&M->kempty[kr.st]);
                    }
                    __syncwarp();
                    kr.next();
                }
                if (go) ns++;
            };
            // O += P V with the values at stages vst ...; in two steps, as the weights come.
            auto products = [&](int vst, uint32_t half, int buf) {
#pragma unroll
                for (int c = 0; c < L::kParts; c++) {
                    const int vs = kOne ? (vst + c) % L::kValStages : vst;
                    const uint32_t bv = v_lo + ((vs * L::kStage) >> 4);
                    const bool clear = first && half == 0;
#pragma unroll
                    for (int k = 0; k < kKT / 32; k++)
                        mma_ts(ox + c * L::kCh, kS + buf * 128 + 8 * (k + half * (kKT / 32)), bv + (((k + half * (kKT / 32)) * 2048) >> 4), v_hi,
                               idesc_o, clear && k == 0 ? 0u : 1u);
                }
            };
            // Waits for the values at the ring's position: landed, and inspected.
            auto values = [&]() {
#pragma unroll
                for (int c = 0; c < L::kParts; c++) {
                    const int vs = kOne ? (vr.st + c) % L::kValStages : vr.st, vp = kOne && vr.st + c >= L::kValStages ? vr.ph ^ 1 : vr.ph;
                    if (!wait(&M->vfull[vs], vp) || !wait(&M->vok[nv & 3], (nv >> 2) & 1)) return;
                    nv++;
                }
            };
            // First half of the weights of the next product.
            auto product0 = [&](int vst) {
                const int buf = kOne ? np & 1 : x, turn = kOne ? np >> 1 : np;
                if (!wait(&M->pfull[buf][0], turn & 1)) return;
                tc_fence_after();
                if (first && *(volatile int*)&M->accum0[x]) {   // the softmax has put something into O
                    __syncwarp();
                    *(volatile int*)&M->accum0[x] = 0;
                    first = false;
                }
                if (issue) products(vst, 0, buf);
                first = false;
            };
            while (w.left > 0 && !dead) {
                const Span sp = span_of<TREE>(a, w.r, w.m * P.tile_tok + x * P.half_tok, P.half_tok);
                const int take = w.take;
                bool prev = false, any = false;
                first = true;
                if (sp.n > 0 && !wait(&M->qfull[x], nq & 1)) break;
                if (kOne) {
                    const bool go = sp.s1 > 0;   // rows that see any tile see all of the tile's list
                    scores(go, sp.n > 0 && take == 1);
                    for (int j = 0; j < take && !dead; j++) {
                        // keys of step j + 1 are ahead of the values of step j in the ring
                        if (j + 1 < take) scores(go, sp.n > 0 && j + 2 == take);
                        if (dead) break;
                        const int vst = vr.st;
                        values();
                        if (dead) break;
                        if (go) {
                            product0(vst);
                            if (dead || !wait(&M->pfull[np & 1][1], (np >> 1) & 1)) break;
                            tc_fence_after();
                            if (issue) {
                                products(vst, 1, np & 1);
                                mma_commit(&M->pvdone);
                            }
                            np++;
                            any = true;
                        }
                        if (issue) {
#pragma unroll
                            for (int c = 0; c < L::kParts; c++) mma_commit(&M->vempty[(vst + c) % L::kValStages]);
                        }
                        __syncwarp();
#pragma unroll
                        for (int c = 0; c < L::kParts; c++) vr.next();
                    }
                } else {
                    for (int j = 0; j <= take; j++) {
                        // the values of step j - 1 at vst, then the keys of step j at kst
                        const bool next = j < take && sp.sees(w.t.id(w.c + j));
                        const int vst = vr.st;
                        if (j > 0) {
                            values();
                            vr.next();
                        }
                        const int kst = kr.st;
                        if (dead || (j < take && !wait(&M->kfull[kst], kr.ph))) break;
                        const uint32_t bv = v_lo + ((vst * L::kStage) >> 4), bk = k_lo + ((kst * L::kStage) >> 4);
                        const uint32_t sx = kS + x * 128;
                        if (prev) {
                            product0(vst);
                            // taken before the rest of the weights are there, which hides the atomic
                            if (dead || !take_turn(&M->turn, issue, abort_flag, a.wait_ns)) {
                                dead = true;
                                break;
                            }
                            if (!wait(&M->pfull[x][1], np & 1)) break;
                            np++;
                            any = true;
                        }
                        tc_fence_after();
                        if (issue) {   // the products' second half and the next scores without a pause
                            if (prev) {
#pragma unroll
                                for (int k = kKT / 32; k < kKT / 16; k++)
                                    mma_ts(ox, sx + 8 * k, bv + ((k * 2048) >> 4), v_hi, idesc_o, 1u);
                            }
                            if (next) {
#pragma unroll
                                for (int k = 0; k < D / 16; k++) {
                                    const uint32_t o = ((k >> 2) * L::kPiece + (k & 3) * 32) >> 4;
                                    mma_ss(sx, al + o, bk + o, hi, idesc_s, k ? 1u : 0u);
                                }
                                mma_commit(&M->sfull[x]);
                            }
                            if (prev) *(volatile int*)&M->turn = 0;
                            if (j == take - 1 && sp.n > 0) mma_commit(&M->qempty[x]);   // the queries were read
                            if (j > 0) mma_commit(&M->vempty[vst]);
                            if (j < take) mma_commit(&M->kempty[kst]);
                        }
                        __syncwarp();
                        if (j < take) kr.next();
                        prev = next;
                    }
                }
                if (dead) break;
                // only where the softmax had its turn: it could otherwise miss one of two
                if (any && issue) mma_commit(&M->ofull[x]);
                if (sp.n > 0) nq++;
                w.next(P);
            }
            if (dead) *abort_flag = 1;
            if (issue) mma_commit(&M->drain[x]);   // products in flight end before tensor memory is given back
            const int zero = 0;
            mbar_wait(&M->drain[x], 0, &zero, tc::kWaitLimitNs);
            __syncwarp();
        } else if (warp == 11) {
            // -------------------------------------------------------- queries, and inspector of values
            // (one warp: a tile's queries are loaded once the last tile's values are inspected)
            Ring<L::kValStages> vr;
            int nv = 0, nq[2] = {0, 0};
            bool dead = *abort_flag != 0, q_bytes = false;
            while (w.left > 0 && !dead) {
                const Span item = span_of<TREE>(a, w.r, w.m * P.tile_tok, P.tile_tok);
                const int take = w.take;
                for (int x = 0; x < halves(D) && !dead; x++) {
                    const int tok = w.m * P.tile_tok + x * P.half_tok;
                    const Span sp = span_of<TREE>(a, w.r, tok, P.half_tok);
                    if (sp.n <= 0) continue;
                    if (!__all_sync(0xffffffffu, mbar_wait(&M->qempty[x], (nq[x] & 1) ^ 1, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    nq[x]++;
                    unsigned char* dst0 = smem + L::q + x * L::kQ;
                    if (P.q_boxes) {   // the half's tokens x n_rep heads
                        if (lane == 0) {
                            mbar_arrive_expect_tx(&M->qfull[x], (uint32_t)(P.half_tok * a.n_rep * D * 2));
#pragma unroll
                            for (int hf = 0; hf < D / 64; hf++)
                                tma_load_4d(dst0 + hf * L::kPiece, &qmap, &M->qfull[x], hf * 64, 0, w.h, w.r.tok0 + tok);
                        }
                        q_bytes = true;
                        continue;
                    }
                    constexpr int kPer = D / 8, kStep = 32 / kPer;   // 16-byte pieces of a row, rows at a time
                    const uint32_t base = smem_u32(dst0);
                    const int ch = lane % kPer;
                    int r = lane / kPer, rt = token_of(a, r), rep = r - rt * a.n_rep;
                    const uint16_t* src = a.q + (int64_t)(w.r.tok0 + tok + rt) * a.q_tok + (int64_t)w.h * a.n_rep * a.q_head + ch * 8;
                    const uint32_t col = base + (ch >> 3) * L::kPiece;
                    for (; r < sp.n; r += kStep) {
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(col + r * 128 + (((ch & 7) ^ (r & 7)) << 4)),
                                     "l"(src + rep * a.q_head)
                                     : "memory");
                        rep += kStep;
                        while (rep >= a.n_rep) {
                            rep -= a.n_rep;
                            src += a.q_tok;
                        }
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&M->qfull[x]);
                }
                if (dead) break;
                for (int kv = 0; kv < take * L::kParts; kv++, nv++) {
                    const int kc = kv / L::kParts;
                    if (!__all_sync(0xffffffffu, mbar_wait(&M->vfull[vr.st], vr.ph, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    const int id = w.t.id(w.c + kc), t0 = id * kKT;
                    int found = 0;
                    if (!item.sees_all(id)) {
                        unsigned char* tile = smem + L::stages + (L::kKeyStages + vr.st) * L::kStage;
                        constexpr int kPer = L::kCh / 8, kStep = 32 / kPer;
                        const int ch = lane % kPer, r0 = lane / kPer;
                        auto at = [&](int r) {
                            return reinterpret_cast<uint4*>(tile + (ch >> 3) * L::kPiece + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
                        };
                        const int held = w.r.len - t0 < kKT ? w.r.len - t0 : kKT;
                        for (int r = (held > 0 ? held : 0) + r0; r < kKT; r += kStep) *at(r) = make_uint4(0, 0, 0, 0);
                        // rows [lo, hi) in batches of independent loads
                        auto scan = [&](int lo, int hi) {
                            constexpr int kBatch = 8;
                            for (int rb = lo + r0; __any_sync(0xffffffffu, rb < hi); rb += kBatch * kStep) {
                                uint4 v[kBatch];
                                uint32_t seen = 0;
#pragma unroll
                                for (int k = 0; k < kBatch; k++) v[k] = rb + k * kStep < hi ? *at(rb + k * kStep) : make_uint4(0, 0, 0, 0);
#pragma unroll
                                for (int k = 0; k < kBatch; k++) seen |= special_bits<FP16>(v[k]);
                                if (seen) {
                                    found = 1;
#pragma unroll
                                    for (int k = 0; k < kBatch; k++)
                                        if (rb + k * kStep < hi)
                                            *at(rb + k * kStep) = make_uint4(drop_special<FP16>(v[k].x), drop_special<FP16>(v[k].y),
                                                                             drop_special<FP16>(v[k].z), drop_special<FP16>(v[k].w));
                                }
                            }
                        };
                        // the partial tokens: those past the first row's position, and those that the
                        // last row's window has left
                        const int after = item.p0 + 1 - t0 > 0 ? item.p0 + 1 - t0 : 0;
                        scan(after, held);
                        if (a.window) {
                            const int lo = a.sinks - t0 > 0 ? a.sinks - t0 : 0, gone = item.p1 - a.window + 1 - t0;
                            const int hi = gone < after ? gone : after;
                            scan(lo, hi < held ? hi : held);
                        }
                        found = __any_sync(0xffffffffu, found);
                        fence_proxy_async_smem();
                    }
                    __syncwarp();
                    if (lane == 0) {
                        *(volatile int*)&M->special[nv & 3] = found;
                        mbar_arrive(&M->vok[nv & 3]);
                    }
                    vr.next();
                }
                if (dead) break;
                w.next(P);
            }
            if (dead) *abort_flag = 1;
            if (q_bytes) {   // boxes in flight land before the CTA ends
                const int zero = 0;
                for (int x = 0; x < halves(D); x++)
                    if (nq[x]) mbar_wait(&M->qfull[x], (nq[x] - 1) & 1, &zero, tc::kWaitLimitNs);
            }
        }
    }
    __syncthreads();
    if (tid == 0 && *abort_flag) raise_flag(a.status, CG_FLAG_PIPE_TIMEOUT);
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");   // not done before the rows kernel of the call
}

// Joins the parts of the tile that starts in CTA b's share. A thread owns a row and 16 channels
// (blockIdx.y). The first parts' values are asked for together with the references, so that the usual
// two or three parts take one round of loads.
template <bool FP16, int D>
__global__ void __launch_bounds__(tile_rows(D)) paged_chunk_merge_kernel(const __grid_constant__ ChunkParams P) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const PagedArgs& a = P.a;
    const ChunkMeta m = P.meta[blockIdx.x];
    // thread = row of the tile: half row >> 7, token rt of the half
    const int row = threadIdx.x, rr = row & (kHalfRows - 1), rt = token_of(a, rr);
    const int tk = (row >> 7) * P.half_tok + rt;
    if (m.last < 0 || rt >= P.half_tok || tk >= m.n_tok) return;
    const int parts = m.last - (int)blockIdx.x + 1;
    auto part = [&](int p) { return P.parts + ((int64_t)(blockIdx.x + p) * 2 + (p == 0 ? 1 : 0)) * chunk_part_floats(D); };
    constexpr int kFirst = 3;
    float ref[kFirst], sum[kFirst];
    float4 x[kFirst][4];
#pragma unroll
    for (int p = 0; p < kFirst; p++) {
        ref[p] = -INFINITY;
        sum[p] = 0.0f;
        if (p < parts) {
            const float* src = part(p);
            ref[p] = src[tile_rows(D) * D + row];
            sum[p] = src[tile_rows(D) * (D + 1) + row];
#pragma unroll
            for (int k = 0; k < 4; k++) x[p][k] = reinterpret_cast<const float4*>(src)[(4 * blockIdx.y + k) * tile_rows(D) + row];
        }
    }
    float R = fmaxf(fmaxf(ref[0], ref[1]), ref[2]);
    for (int p = kFirst; p < parts; p++) R = fmaxf(R, part(p)[tile_rows(D) * D + row]);
    const float Rs = R == -INFINITY ? 0.0f : R;
    float l = 0.0f, o[16];
#pragma unroll
    for (int k = 0; k < 16; k++) o[k] = 0.0f;
    auto add = [&](float r, float s, const float4 (&v)[4]) {
        const float f = r == -INFINITY ? 0.0f : fmaxf(ex2(r - Rs), 1.17549435e-38f);
        l = fmaf(f, s, l);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            o[4 * k] = fmaf(f, v[k].x, o[4 * k]);
            o[4 * k + 1] = fmaf(f, v[k].y, o[4 * k + 1]);
            o[4 * k + 2] = fmaf(f, v[k].z, o[4 * k + 2]);
            o[4 * k + 3] = fmaf(f, v[k].w, o[4 * k + 3]);
        }
    };
#pragma unroll
    for (int p = 0; p < kFirst; p++)
        if (p < parts) add(ref[p], sum[p], x[p]);
#pragma unroll 2
    for (int p = kFirst; p < parts; p++) {
        const float* src = part(p);
        float4 v[4];
#pragma unroll
        for (int k = 0; k < 4; k++) v[k] = reinterpret_cast<const float4*>(src)[(4 * blockIdx.y + k) * tile_rows(D) + row];
        add(src[tile_rows(D) * D + row], src[tile_rows(D) * (D + 1) + row], v);
    }
    const int hd = m.h * a.n_rep + (rr - rt * a.n_rep);
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    uint4* dst = reinterpret_cast<uint4*>(a.out + (int64_t)(m.tok0 + tk) * a.o_tok + hd * a.o_head + 16 * blockIdx.y);
#pragma unroll
    for (int q = 0; q < 2; q++) {
        uint32_t b[4];
#pragma unroll
        for (int k = 0; k < 4; k++) b[k] = inv == 0.0f ? 0u : pack2<FP16>(o[8 * q + 2 * k] * inv, o[8 * q + 2 * k + 1] * inv);
        dst[q] = make_uint4(b[0], b[1], b[2], b[3]);
    }
    if (a.lse && blockIdx.y == 0)
        a.lse[(int64_t)(m.tok0 + tk) * a.H * a.n_rep + hd] = inv == 0.0f ? -INFINITY : TileWeights<FP16>::lse(R, l);
}

// Queries as [n_tok][H][n_rep][d] (their strides), boxes of a half's tokens x n_rep heads x 64
// channels: its rows in their order. Queries with strides that a tensor map cannot hold (a broadcast
// dimension) are gathered by a warp instead.
bool query_map(CUtensorMap* map, const PagedArgs& a) {
    auto fn = tmap_encode_fn();
    const int64_t most = (int64_t)1 << 39;
    // the stride of a dimension of one element is free
    const int64_t q_head = a.H * a.n_rep == 1 ? a.d : a.q_head, q_tok = a.n_tok == 1 ? a.d : a.q_tok;
    if (!fn || q_head <= 0 || q_tok <= 0 || q_head * a.n_rep * 2 >= most || q_tok * 2 >= most) return false;
    cuuint64_t dims[4] = {(cuuint64_t)a.d, (cuuint64_t)a.n_rep, (cuuint64_t)a.H, (cuuint64_t)a.n_tok};
    cuuint64_t strides[3] = {(cuuint64_t)q_head * 2, (cuuint64_t)q_head * a.n_rep * 2, (cuuint64_t)q_tok * 2};
    cuuint32_t box[4] = {64, (cuuint32_t)a.n_rep, 1, (cuuint32_t)(kHalfRows / a.n_rep)}, estr[4] = {1, 1, 1, 1};
    return fn(map, a.dtype == CG_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
              const_cast<uint16_t*>(a.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool FP16, int D, bool TREE>
cudaError_t launch_chunk(ChunkParams P, bool after_rows, cudaStream_t st) {
    CUtensorMap map, qmap{};
    if (!paged_pool_map(&map, P.a, P.box_rows)) return cudaErrorInvalidValue;
    P.q_boxes = query_map(&qmap, P.a);
    constexpr size_t smem = ChunkSmem<D>::total;
    static SmemOptIn opt_in;
    cudaError_t e = opt_in.set(reinterpret_cast<const void*>(paged_chunk_kernel<FP16, D, TREE>), (int)smem);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)tc::num_sms();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kChunkThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    // Beside the rows kernel of the same call this one starts as soon as that one's CTAs leave room: it
    // reads none of its results (and ends after it, see its end). A tree's call has no such one, and waits for what was before it.
    cfg.numAttrs = after_rows || TREE ? 1 : 0;
    if ((e = cudaLaunchKernelEx(&cfg, paged_chunk_kernel<FP16, D, TREE>, P, map, qmap)) != cudaSuccess) return e;
    // the merge is scheduled while the last shares run; it waits for them on the device
    cfg.gridDim = dim3(grid, D / 16);
    cfg.blockDim = dim3(tile_rows(D));
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, paged_chunk_merge_kernel<FP16, D>, P);
}

template <int D>
cudaError_t launch_chunk(const ChunkParams& P, bool after_rows, cudaStream_t st) {
    const bool tree = P.a.masks != nullptr;
    if (P.a.dtype == CG_FP16) return tree ? launch_chunk<true, D, true>(P, after_rows, st) : launch_chunk<true, D, false>(P, after_rows, st);
    return tree ? launch_chunk<false, D, true>(P, after_rows, st) : launch_chunk<false, D, false>(P, after_rows, st);
}

}  // namespace

size_t paged_chunk_workspace(int d) {
    const size_t n = (size_t)tc::num_sms();
    return n * 2 * chunk_part_floats(d) * sizeof(float) + n * sizeof(ChunkMeta);
}

cudaError_t launch_paged_chunk(const PagedArgs& a, int min_rows, bool after_rows, void* workspace, cudaStream_t st) {
    ChunkParams P{};
    P.a = a;
    P.parts = static_cast<float*>(workspace);
    P.meta = reinterpret_cast<ChunkMeta*>(P.parts + (size_t)tc::num_sms() * 2 * chunk_part_floats(a.d));
    P.min_rows = min_rows;
    // Matters where few trees leave SMs idle. With 2, 3 and 4: a tree of 8 nodes alone after 1000 tokens 15.2, 16.0 and 16.4 us, after 4000
    // 18.6, 18.0 and 18.4, of 32 nodes after 1000 17.4, 17.3 and 18.5, two of 16 16.1, 16.5 and 17.2; one after 8000 tokens and more,
    // three after 3000 and batches of four and more take the same with each, to 0.3 us.
    P.min_share = a.masks ? 2 : 4;
    P.half_tok = kHalfRows / a.n_rep;
    P.tile_tok = halves(a.d) * P.half_tok;
    P.box_rows = a.page < kKT ? a.page : kKT;
    if (a.d == 64) return launch_chunk<64>(P, after_rows, st);
    if (a.d == 256) return launch_chunk<256>(P, after_rows, st);
    return launch_chunk<128>(P, after_rows, st);
}

}  // namespace cg
