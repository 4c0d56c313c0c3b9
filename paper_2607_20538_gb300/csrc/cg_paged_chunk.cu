// cg_paged_chunk.cu -- paged attention of requests with many query rows (a chunk or a whole prompt):
// o = softmax(scale q K^T) V on the tensor cores (contract: include/codecgauge_paged.h).
//
// A tile of work is 256 query rows of one request and KV head, as two halves A and B of 128 rows
// (rows are (token, query head of the group)). One CTA per SM walks its share of the key tiles:
//   warps 0-3, 4-7  softmax of half A, half B: a thread owns a row: 128 scores from tensor memory,
//                   running reference and sum in registers, weights back to tensor memory;
//   warp 8          TMA: 128-token tiles of keys and values, K0 V0 K1 V1 ..., boxes of pages;
//   warp 9          one thread issues tcgen05.mma: S = Q K^T (both operands in shared memory) and
//                   O += P V (P in tensor memory over S, V token-major as it lies in the page);
//   warp 10         loads the queries of a tile (any strides, any n_rep);
//   warp 11         inspects the values of tiles that not every row sees whole (below).
// The MMA order is PV_A(j-1) S_A(j) PV_B(j-1) S_B(j): while one half's softmax runs, the tensor
// cores work for the other. S_x(j) follows PV_x(j-1) in issue order, so S may overwrite P, and its
// completion tells the softmax that O_x is quiescent: the thread rescales its row of O itself on the
// rare steps that raise the reference by more than 2^8.
// Bound: the tensor cores (4 x 128 x 128 x d multiply-adds per key tile against 128 x 256
// exponentials and about four times as many other operations).
//
// What a row does not see must not reach it, and 0 x inf would: in tiles that some rows see and
// others do not, warp 11 takes special values (and whatever lies past the request's end) out of the
// value tile before the product; rows that see them add them to O from the pool (a slow path that
// only such inputs take).
//
// Split: the key tiles of all work tiles form one line cut into equal shares, one per CTA; a tile
// that a cut goes through is written in parts and joined by paged_chunk_merge_kernel.
#include "cg_paged_dev.cuh"
#include "cg_tc_common.cuh"
#include "cg_tmap.h"

namespace cg {
namespace {

using namespace paged;

constexpr int kHalfRows = 128;
constexpr int kTileRows = 256;
constexpr int kKT = 128;          // tokens of a key tile
constexpr int kChunkThreads = 384;
constexpr int kMaxStages = 8;

// One part: O as [d / 4][256 rows][4], then reference and sum of each row.
constexpr int chunk_part_floats(int d) { return kTileRows * d + 2 * kTileRows; }

struct ChunkMeta {
    int last, tok0, row0, n_rows, h, pad[3];
};

template <int D>
struct ChunkSmem {
    static constexpr int kStages = D == 64 ? 8 : 5;
    static constexpr uint32_t kPiece = kKT * 128;                 // 128 rows x 64 channels
    static constexpr uint32_t kStage = kKT * D * 2;               // one key or value tile
    static constexpr uint32_t kQ = kHalfRows * D * 2;             // one half's queries
    static constexpr uint32_t q = 0;
    static constexpr uint32_t stages = 2 * kQ;
    static constexpr uint32_t misc = stages + kStages * kStage;
    static constexpr uint32_t total = misc + 512;
    static_assert(total <= 232448, "shared memory budget");
};

struct ChunkMisc {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t sfull[2], pfull[2], ofull[2], qfull[2], qempty[2], vok[4], drain;
    int64_t warp_sum[kChunkThreads / 32];
    int start[4];            // request, head, tile, key tile of the share's beginning
    int special[4];          // the inspected tile held special values
    int accum0[2];           // the half's O was prepared by its softmax before the first product
    int abort_flag;
    uint32_t tmem;
};
static_assert(sizeof(ChunkMisc) <= 512, "misc block");

struct ChunkParams {
    PagedArgs a;
    float* parts;
    ChunkMeta* meta;
    int min_rows;      // requests with fewer query rows are left to the other kernel
    int min_share;     // key tiles
    int box_rows;
};

// Rows [row0, row0 + n_rows) of a request: their positions.
struct Span {
    int p0, p1, n;
    __device__ __forceinline__ bool sees(const PagedArgs& a, int t0) const {
        return n > 0 && t0 <= p1 && (!a.window || t0 + kKT > p0 - a.window + 1 || t0 < a.sinks);
    }
    __device__ __forceinline__ bool sees_all(const PagedArgs& a, int t0) const {
        return t0 + kKT <= p0 + 1 && (!a.window || t0 > p1 - a.window || t0 + kKT <= a.sinks);
    }
    // token t is seen by some rows and not by others, or by none
    __device__ __forceinline__ bool partial(const PagedArgs& a, int t) const {
        return t > p0 || (a.window && t >= a.sinks && p1 - a.window >= t);
    }
};

__device__ __forceinline__ Span span_of(const PagedArgs& a, const Request& r, int row0, int rows_max) {
    Span s;
    const int rows = r.n * a.n_rep - row0;
    s.n = rows < 0 ? 0 : rows < rows_max ? rows : rows_max;
    s.p0 = r.len - r.n + row0 / a.n_rep;
    s.p1 = s.n ? r.len - r.n + (row0 + s.n - 1) / a.n_rep : s.p0 - 1;
    return s;
}

__device__ __forceinline__ Tiles tile_tiles(const PagedArgs& a, const Request& r, int m) {
    const Span s = span_of(a, r, m * kTileRows, kTileRows);
    return visible_tiles<kKT>(a.window, a.sinks, s.p0, s.p1);
}

// Key tiles of one KV head of a request (all its row tiles).
__device__ __forceinline__ int64_t head_cost(const ChunkParams& P, const Request& r) {
    const int64_t rows = (int64_t)r.n * P.a.n_rep;
    if (rows < P.min_rows || r.n <= 0) return 0;
    int64_t sum = 0;
    for (int m = 0; m < (int)((rows + kTileRows - 1) / kTileRows); m++) sum += tile_tiles(P.a, r, m).count();
    return sum;
}

// Walk over a share: request, KV head, row tile, key tile.
struct ChunkWalk {
    int i, h, m, c, n_m, n_chunks;
    Request r;
    Tiles t;

    __device__ __forceinline__ void load(const ChunkParams& P) {
        int32_t flag = 0;
        n_m = 0;
        if (i >= P.a.n_req) return;
        r = load_request(P.a, i, &flag);
        const int64_t rows = (int64_t)r.n * P.a.n_rep;
        n_m = r.n <= 0 || rows < P.min_rows ? 0 : (int)((rows + kTileRows - 1) / kTileRows);
    }
    __device__ __forceinline__ void tile(const ChunkParams& P) {
        t = tile_tiles(P.a, r, m);
        n_chunks = t.count();
    }
    __device__ __forceinline__ void start(const ChunkParams& P, const int (&s)[4]) {
        i = s[0];
        h = s[1];
        m = s[2];
        c = s[3];
        load(P);
        tile(P);
    }
    __device__ __forceinline__ void next(const ChunkParams& P) {
        c = 0;
        if (++m >= n_m) {
            m = 0;
            if (++h >= P.a.H) {
                h = 0;
                do {
                    i++;
                    load(P);
                } while (i < P.a.n_req && n_m == 0);
                if (i >= P.a.n_req) return;
            }
        }
        tile(P);
    }
};

// ---------------------------------------------------------------- tcgen05 pieces
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc)
        : "memory");
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

// 16 columns times f, in place
__device__ __forceinline__ void tmem_scale16(uint32_t taddr, float f) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
    tmem_wait_ld();
#pragma unroll
    for (int k = 0; k < 16; k++) r[k] = __float_as_uint(__uint_as_float(r[k]) * f);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
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
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

// Scores of 32 columns from c0: sign (a negative scale), and where EDGE the columns that the row does
// not see set to -inf: it sees [lo, hi] and those below sk.
template <bool EDGE>
__device__ __forceinline__ void prepare32(float (&s)[32], int c0, bool flip, int lo, int hi, int sk) {
    if (flip) {
#pragma unroll
        for (int k = 0; k < 32; k++) s[k] = -s[k];
    }
    if (EDGE) {
#pragma unroll
        for (int k = 0; k < 32; k++) {
            const int c = c0 + k;
            s[k] = c <= hi && (c >= lo || c < sk) ? s[k] : -INFINITY;
        }
    }
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

// The row's largest score of a tile (128 columns).
template <bool EDGE>
__device__ __forceinline__ float row_max(uint32_t s_tm, bool flip, int lo, int hi, int sk) {
    float u[32], v[32];
    tmem_ld32f(s_tm, u);
    tmem_ld32f(s_tm + 32, v);
    tmem_wait_ld();
    settle(u);
    settle(v);
    prepare32<EDGE>(u, 0, flip, lo, hi, sk);
    float m = max32(u, -INFINITY);
    tmem_ld32f(s_tm + 64, u);
    prepare32<EDGE>(v, 32, flip, lo, hi, sk);
    m = max32(v, m);
    tmem_ld32f(s_tm + 96, v);
    tmem_wait_ld();
    settle(u);
    settle(v);
    prepare32<EDGE>(u, 64, flip, lo, hi, sk);
    m = max32(u, m);
    prepare32<EDGE>(v, 96, flip, lo, hi, sk);
    return max32(v, m);
}

template <bool FP16>
__device__ __forceinline__ void weights32(const float (&s)[32], uint32_t p_tm, float sl2, float neg_ref, float2& acc) {
    uint32_t p[16];
#pragma unroll
    for (int k = 0; k < 16; k++) {
        const float2 e = __ffma2_rn(make_float2(s[2 * k], s[2 * k + 1]), make_float2(sl2, sl2), make_float2(neg_ref, neg_ref));
        const float2 w = make_float2(ex2(e.x), ex2(e.y));
        acc = __fadd2_rn(acc, w);
        p[k] = pack2<FP16>(w.x, w.y);
    }
    tmem_st16(p_tm, p);
}

// Weights 2^(s sl2 + neg_ref) of the tile in 16 bits over the scores (columns [0, 64)), and their
// sum. The scores are read again: 128 of them kept in registers would not leave room for the rest,
// and each group of weights lies over scores already read.
template <bool FP16, bool EDGE>
__device__ __forceinline__ float row_weights(uint32_t s_tm, bool flip, int lo, int hi, int sk, float sl2, float neg_ref) {
    float u[32], v[32];
    float2 acc = make_float2(0.0f, 0.0f);
    tmem_ld32f(s_tm, u);
    tmem_ld32f(s_tm + 32, v);
    tmem_wait_ld();
    settle(u);
    settle(v);
    prepare32<EDGE>(u, 0, flip, lo, hi, sk);
    weights32<FP16>(u, s_tm, sl2, neg_ref, acc);
    tmem_ld32f(s_tm + 64, u);
    prepare32<EDGE>(v, 32, flip, lo, hi, sk);
    weights32<FP16>(v, s_tm + 16, sl2, neg_ref, acc);
    tmem_ld32f(s_tm + 96, v);
    tmem_wait_ld();
    settle(u);
    settle(v);
    prepare32<EDGE>(u, 64, flip, lo, hi, sk);
    weights32<FP16>(u, s_tm + 32, sl2, neg_ref, acc);
    prepare32<EDGE>(v, 96, flip, lo, hi, sk);
    weights32<FP16>(v, s_tm + 48, sl2, neg_ref, acc);
    return acc.x + acc.y;
}

template <bool FP16>
__host__ __device__ constexpr uint32_t idesc16(int M, int N) {
    return (1u << 4) | ((FP16 ? 0u : 1u) << 7) | ((FP16 ? 0u : 1u) << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
constexpr uint32_t kIdescBMnMajor = 1u << 16;

template <bool FP16>
__device__ __forceinline__ bool any_special(uint4 v) {
    constexpr uint32_t e = FP16 ? 0x7c00u : 0x7f80u;
    bool s = false;
    for (uint32_t w : {v.x, v.y, v.z, v.w}) s |= (w & e) == e || (w & (e << 16)) == (e << 16);
    return s;
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
template <bool FP16, int D>
__device__ __noinline__ void add_special(const PagedArgs& a, const Request& r, int req, int h, Span item, int t0, int pos,
                                         uint32_t o_tm, bool first) {
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
            const bool see = t <= pos && (!a.window || t > pos - a.window || t < a.sinks);
            if (!__any_sync(0xffffffffu, see)) continue;
            const int pg = __ldg(a.table + (int64_t)req * a.max_pages + (t >> a.page_log2));
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

template <bool FP16, int D>
__global__ void __launch_bounds__(kChunkThreads, 1)
paged_chunk_kernel(const __grid_constant__ ChunkParams P, const __grid_constant__ CUtensorMap map) {
    using L = ChunkSmem<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    ChunkMisc* M = reinterpret_cast<ChunkMisc*>(smem + L::misc);
    const PagedArgs& a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int32_t flag = 0;

    // ---- this CTA's share of the line of key tiles
    const int per = (a.n_req + kChunkThreads - 1) / kChunkThreads;
    const int i_lo = tid * per < a.n_req ? tid * per : a.n_req;
    const int i_hi = i_lo + per < a.n_req ? i_lo + per : a.n_req;
    int64_t mine = 0;
    for (int i = i_lo; i < i_hi; i++) mine += head_cost(P, load_request(a, i, &flag)) * a.H;
    int64_t incl = mine;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const int64_t v = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += v;
    }
    if (lane == 31) M->warp_sum[warp] = incl;
    if (tid == 0) {
        for (int s = 0; s < L::kStages; s++) {
            mbar_init(&M->full[s], 1);
            mbar_init(&M->empty[s], 1);
        }
        for (int x = 0; x < 2; x++) {
            mbar_init(&M->sfull[x], 1);
            mbar_init(&M->pfull[x], 4);
            mbar_init(&M->ofull[x], 1);
            mbar_init(&M->qfull[x], 1);
            mbar_init(&M->qempty[x], 1);
            M->accum0[x] = 0;
        }
        for (int s = 0; s < 4; s++) mbar_init(&M->vok[s], 1);
        mbar_init(&M->drain, 1);
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
    for (int w = 0; w < kChunkThreads / 32; w++) {
        if (w < warp) before += M->warp_sum[w];
        total += M->warp_sum[w];
    }
    int64_t share = (total + gridDim.x - 1) / gridDim.x;
    if (share < P.min_share) share = P.min_share;
    const int64_t begin = share * blockIdx.x;
    const int64_t end = begin + share < total ? begin + share : total;
    if (begin >= before && begin < before + mine) {
        int64_t at = before;
        for (int i = i_lo; i < i_hi; i++) {
            const Request r = load_request(a, i, &flag);
            const int64_t hc = head_cost(P, r);
            if (begin < at + hc * a.H) {
                int64_t off = begin - at;
                const int h = (int)(off / hc);
                off -= h * hc;
                int m = 0;
                for (;; m++) {
                    const int n = tile_tiles(a, r, m).count();
                    if (off < n) break;
                    off -= n;
                }
                M->start[0] = i;
                M->start[1] = h;
                M->start[2] = m;
                M->start[3] = (int)off;
                break;
            }
            at += hc * a.H;
        }
    }
    __syncthreads();
    if (blockIdx.x == 0) raise_flag(a.status, flag);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    volatile int* abort_flag = &M->abort_flag;
    int left = begin < end ? (int)(end - begin) : 0;
    ChunkWalk w;
    if (left) w.start(P, M->start);
    const uint32_t kS = tmem, kO = tmem + 256;

    if (warp < 8) {
        // ------------------------------------------------------------ softmax
        const int x = warp >> 2;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t s_tm = kS + x * 128 + lanes, o_tm = kO + x * D + lanes;
        // a scale of 0 becomes the least number, so that a masked -inf stays one
        const float sl2 = fmaxf(fabsf(a.scale) * kLog2e, 1.17549435e-38f);
        const bool flip = a.scale < 0.0f;
        constexpr float kBias = Weights<FP16>::kBias;
        int ns = 0, no = 0, nv = 0;   // active steps, tiles and value tiles so far
        bool head_part = left && w.c > 0, dead = *abort_flag != 0;
        int meta_last = -1;
        while (left > 0 && !dead) {
            const int row0 = w.m * kTileRows + x * kHalfRows;
            const Span sp = span_of(a, w.r, row0, kHalfRows), item = span_of(a, w.r, w.m * kTileRows, kTileRows);
            const int take = w.n_chunks - w.c < left ? w.n_chunks - w.c : left;
            const bool goes_on = w.c + take < w.n_chunks;
            if (sp.n > 0) {
                const int row = (warp & 3) * 32 + lane;
                const bool have = row < sp.n;
                const int tk = (row0 + row) / a.n_rep, hd = w.h * a.n_rep + (row0 + row - tk * a.n_rep);
                const int pos = have ? w.r.len - w.r.n + tk : -1;
                float ref = -INFINITY, sum = 0.0f;
                bool started = false;
                for (int kc = 0; kc < take; kc++) {
                    const int t0 = w.t.id(w.c + kc) * kKT;
                    if (!sp.sees(a, t0)) continue;
                    if (!__all_sync(0xffffffffu, mbar_wait(&M->sfull[x], ns & 1, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    ns++;
                    tc_fence_after();
                    const bool edge = !sp.sees_all(a, t0);
                    const int hi = pos - t0, lo = a.window ? pos - a.window + 1 - t0 : 0, sk = a.sinks - t0;
                    const float mx = sl2 * (edge ? row_max<true>(s_tm, flip, lo, hi, sk) : row_max<false>(s_tm, flip, 0, 0, 0));
                    if (__any_sync(0xffffffffu, mx > ref + (kBias + kLazy))) {
                        const float nr = fmaxf(ref, mx - kBias);
                        // never 0 x inf in O: a factor below all numbers becomes the least one
                        const float f = ref == nr ? 1.0f : fmaxf(ex2(ref - nr), 1.17549435e-38f);
                        if (started) {
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 16) tmem_scale16(o_tm + c0, f);
                        }
                        sum *= ref == -INFINITY ? 0.0f : f;
                        ref = nr;
                    }
                    const float nr = ref == -INFINITY ? 0.0f : -ref;
                    sum += edge ? row_weights<FP16, true>(s_tm, flip, lo, hi, sk, sl2, nr)
                                : row_weights<FP16, false>(s_tm, flip, 0, 0, 0, sl2, nr);
                    if (!item.sees_all(a, t0)) {
                        // the inspected value tile held special values: add those the row sees
                        const int v = nv + kc;
                        if (!__all_sync(0xffffffffu, mbar_wait(&M->vok[v & 3], (v >> 2) & 1, abort_flag, a.wait_ns))) {
                            dead = true;
                            break;
                        }
                        if (*(volatile int*)&M->special[v & 3]) {
                            add_special<FP16, D>(a, w.r, w.i, w.h, item, t0, pos, o_tm, !started);
                            if (!started && lane == 0) *(volatile int*)&M->accum0[x] = 1;
                        }
                    }
                    started = true;
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&M->pfull[x]);
                }
                if (dead || !__all_sync(0xffffffffu, mbar_wait(&M->ofull[x], no & 1, abort_flag, a.wait_ns))) {
                    dead = true;
                    break;
                }
                no++;
                tc_fence_after();
                if (!head_part && !goes_on) {
                    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
                    uint16_t* dst = a.out + (int64_t)(w.r.tok0 + tk) * a.o_tok + hd * a.o_head;
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 32) {
                        uint32_t o[32], b[16];
                        tmem_ld32p(o_tm + c0, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int k = 0; k < 16; k++)
                            b[k] = started && inv != 0.0f ? pack2<FP16>(__uint_as_float(o[2 * k]) * inv, __uint_as_float(o[2 * k + 1]) * inv) : 0u;
                        if (have) {
#pragma unroll
                            for (int k = 0; k < 4; k++)
                                *reinterpret_cast<uint4*>(dst + c0 + 8 * k) = make_uint4(b[4 * k], b[4 * k + 1], b[4 * k + 2], b[4 * k + 3]);
                        }
                    }
                    if (a.lse && have)
                        a.lse[(int64_t)(w.r.tok0 + tk) * a.H * a.n_rep + hd] = inv == 0.0f ? -INFINITY : (ref + log2f(sum)) * kLn2;
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
                                reinterpret_cast<uint4*>(part)[(c0 / 4 + k) * kTileRows + r] =
                                    started ? make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]) : make_uint4(0, 0, 0, 0);
                        }
                    }
                    if (have) {
                        part[kTileRows * D + r] = ref;
                        part[kTileRows * D + kTileRows + r] = sum;
                    }
                }
            }
            if (!head_part && goes_on) {   // it starts here and goes on
                const int64_t rest = (int64_t)w.n_chunks - w.c - take;
                meta_last = (int)(blockIdx.x + (rest + share - 1) / share);
                if (tid == 0) {
                    ChunkMeta* m = P.meta + blockIdx.x;
                    m->last = meta_last;
                    m->tok0 = w.r.tok0;
                    m->row0 = w.m * kTileRows;
                    m->n_rows = item.n;
                    m->h = w.h;
                }
            }
            head_part = false;
            nv += take;
            left -= take;
            if (left > 0) w.next(P);
        }
        if (tid == 0 && meta_last < 0) P.meta[blockIdx.x].last = -1;
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
            int st = 0, ph = 1, issued = 0;
            bool dead = *abort_flag != 0;
            while (left > 0 && !dead) {
                const int wlo = a.window ? w.r.len - w.r.n - a.window + 1 : 0;
                const int32_t* row = a.table + (int64_t)w.i * a.max_pages;
                const int take = w.n_chunks - w.c < left ? w.n_chunks - w.c : left;
                auto place = [&](int kc, int* z, int* y) {
                    *z = 2 * a.n_pages;                  // past the pool: the copy fills with zeros
                    *y = 0;
                    const int t = w.t.id(w.c + kc) * kKT + lane * P.box_rows;
                    if (lane < n_box && t < w.r.len && (t + P.box_rows > wlo || t < a.sinks)) {
                        const int pg = __ldg(row + (t >> a.page_log2));
                        if (pg >= 0 && pg < a.n_pages) {
                            *z = pg;
                            *y = w.h * a.page + (t & (a.page - 1));
                        } else {
                            pflag |= CG_FLAG_PAGED_RANGE;
                        }
                    }
                };
                int z, y;
                place(0, &z, &y);
                for (int kc = 0; kc < take && !dead; kc++) {
                    int zn = 0, yn = 0;
                    if (kc + 1 < take) place(kc + 1, &zn, &yn);   // the next tile's pages, ahead of the waits
#pragma unroll
                    for (int kv = 0; kv < 2; kv++) {
                        if (!__all_sync(0xffffffffu, mbar_wait(&M->empty[st], ph, abort_flag, a.wait_ns))) {
                            dead = true;
                            break;
                        }
                        if (lane == 0) mbar_arrive_expect_tx(&M->full[st], L::kStage);
                        __syncwarp();
                        if (lane < n_box) {
                            unsigned char* dst = smem + L::stages + st * L::kStage + lane * P.box_rows * 128;
                            const int zz = kv && z < a.n_pages ? z + a.n_pages : z;
#pragma unroll
                            for (int hf = 0; hf < D / 64; hf++) tma_load_3d(dst + hf * L::kPiece, &map, &M->full[st], hf * 64, y, zz);
                        }
                        issued++;
                        if (++st == L::kStages) {
                            st = 0;
                            ph ^= 1;
                        }
                    }
                    z = zn;
                    y = yn;
                }
                left -= take;
                if (left > 0) w.next(P);
            }
            raise_flag(a.status, pflag);
            if (dead) {   // copies in flight land before the CTA ends
                *abort_flag = 1;
                const int zero = 0;
                for (int k = issued > L::kStages ? issued - L::kStages : 0; k < issued; k++)
                    mbar_wait(&M->full[k % L::kStages], (k / L::kStages) & 1, &zero, tc::kWaitLimitNs);
            }
        } else if (warp == 9) {
            // -------------------------------------------------------- MMA issuer
            if (lane == 0) {
                constexpr uint32_t idesc_s = idesc16<FP16>(128, kKT);
                constexpr uint32_t idesc_o = idesc16<FP16>(128, D) | kIdescBMnMajor;
                const uint64_t qd[2] = {sdesc_sw128(smem_u32(smem + L::q)), sdesc_sw128(smem_u32(smem + L::q + L::kQ))};
                const uint64_t kd = sdesc_sw128(smem_u32(smem + L::stages));
                const uint64_t vd = sdesc_sw128_mn(smem_u32(smem + L::stages), L::kPiece, 1024u);
                int st = 0, ph = 0;                // ring position of the next tile to wait for
                int np[2] = {0, 0}, nq[2] = {0, 0}, nv = 0;
                bool dead = *abort_flag != 0;
                while (left > 0 && !dead) {
                    const Span sp[2] = {span_of(a, w.r, w.m * kTileRows, kHalfRows),
                                        span_of(a, w.r, w.m * kTileRows + kHalfRows, kHalfRows)};
                    const int take = w.n_chunks - w.c < left ? w.n_chunks - w.c : left;
                    bool first[2] = {true, true}, have_q[2] = {false, false};
                    int vst = 0, vph = 0, t_prev = 0;
                    for (int j = 0; j <= take && !dead; j++) {
                        // keys of step j at ring slot kst; values of step j - 1 at vst
                        const int t0 = j < take ? w.t.id(w.c + j) * kKT : 0;
                        const int kst = st, kph = ph;
                        bool k_ok = false;
                        if (j > 0) {   // landed, and inspected
                            const int v = nv + j - 1;
                            if (!mbar_wait(&M->full[vst], vph, abort_flag, a.wait_ns) ||
                                !mbar_wait(&M->vok[v & 3], (v >> 2) & 1, abort_flag, a.wait_ns)) {
                                dead = true;
                                break;
                            }
                        }
#pragma unroll
                        for (int x = 0; x < 2; x++) {
                            if (j > 0 && sp[x].sees(a, t_prev)) {
                                if (!mbar_wait(&M->pfull[x], np[x] & 1, abort_flag, a.wait_ns)) {
                                    dead = true;
                                    break;
                                }
                                np[x]++;
                                tc_fence_after();
                                uint32_t acc = first[x] ? 0u : 1u;
                                if (first[x] && *(volatile int*)&M->accum0[x]) {
                                    acc = 1u;
                                    *(volatile int*)&M->accum0[x] = 0;
                                }
                                first[x] = false;
                                const uint64_t bd = vd + (uint64_t)((vst * L::kStage) >> 4);
#pragma unroll
                                for (int k = 0; k < kKT / 16; k++) {
                                    mma_ts(kO + x * D, kS + x * 128 + 8 * k, bd + (uint64_t)(k * 2048 >> 4), idesc_o, acc);
                                    acc = 1u;
                                }
                            }
                            if (j < take && sp[x].sees(a, t0)) {
                                if (!have_q[x]) {
                                    if (!mbar_wait(&M->qfull[x], nq[x] & 1, abort_flag, a.wait_ns)) {
                                        dead = true;
                                        break;
                                    }
                                    have_q[x] = true;
                                }
                                if (!k_ok) {
                                    if (!mbar_wait(&M->full[kst], kph, abort_flag, a.wait_ns)) {
                                        dead = true;
                                        break;
                                    }
                                    k_ok = true;
                                    tc_fence_after();
                                }
                                const uint64_t bd = kd + (uint64_t)((kst * L::kStage) >> 4);
#pragma unroll
                                for (int k = 0; k < D / 16; k++) {
                                    const uint64_t o = (uint64_t)(((k >> 2) * L::kPiece + (k & 3) * 32) >> 4);
                                    mma_bf16(kS + x * 128, qd[x] + o, bd + o, idesc_s, k > 0);
                                }
                                mma_commit(&M->sfull[x]);
                            }
                        }
                        if (dead) break;
                        if (j > 0) mma_commit(&M->empty[vst]);
                        if (j < take) {
                            if (!k_ok && !mbar_wait(&M->full[kst], kph, abort_flag, a.wait_ns)) {
                                dead = true;
                                break;
                            }
                            mma_commit(&M->empty[kst]);
                            if (++st == L::kStages) {
                                st = 0;
                                ph ^= 1;
                            }
                            vst = st;   // the values follow the keys
                            vph = ph;
                            if (++st == L::kStages) {
                                st = 0;
                                ph ^= 1;
                            }
                        }
                        t_prev = t0;
                    }
                    if (dead) break;
#pragma unroll
                    for (int x = 0; x < 2; x++)
                        if (sp[x].n > 0) {
                            // a half whose rows see nothing of this share still takes its queries' turn
                            if (!have_q[x] && !mbar_wait(&M->qfull[x], nq[x] & 1, abort_flag, a.wait_ns)) dead = true;
                            nq[x]++;
                            mma_commit(&M->qempty[x]);
                            mma_commit(&M->ofull[x]);
                        }
                    nv += take;
                    left -= take;
                    if (left > 0) w.next(P);
                }
                if (dead) *abort_flag = 1;
                mma_commit(&M->drain);   // products in flight end before tensor memory is given back
                const int zero = 0;
                mbar_wait(&M->drain, 0, &zero, tc::kWaitLimitNs);
            }
            __syncwarp();
        } else if (warp == 10) {
            // -------------------------------------------------------- queries
            int nq[2] = {0, 0};
            bool dead = *abort_flag != 0;
            while (left > 0 && !dead) {
                const int take = w.n_chunks - w.c < left ? w.n_chunks - w.c : left;
                for (int x = 0; x < 2 && !dead; x++) {
                    const int row0 = w.m * kTileRows + x * kHalfRows;
                    const Span sp = span_of(a, w.r, row0, kHalfRows);
                    if (sp.n <= 0) continue;
                    if (!__all_sync(0xffffffffu, mbar_wait(&M->qempty[x], (nq[x] & 1) ^ 1, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    constexpr int kPer = D / 8;            // 16-byte pieces of a row
                    const uint32_t base = smem_u32(smem + L::q + x * L::kQ);
                    const int ch = lane % kPer;
                    for (int r = lane / kPer; r < sp.n; r += 32 / kPer) {
                        const int tk = (row0 + r) / a.n_rep, hd = w.h * a.n_rep + (row0 + r - tk * a.n_rep);
                        const uint16_t* src = a.q + (int64_t)(w.r.tok0 + tk) * a.q_tok + hd * a.q_head + ch * 8;
                        const uint32_t dst = base + (ch >> 3) * L::kPiece + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&M->qfull[x]);
                    nq[x]++;
                }
                left -= take;
                if (left > 0) w.next(P);
            }
            if (dead) *abort_flag = 1;
        } else {
            // -------------------------------------------------------- inspector of values
            int st = 0, ph = 0, nv = 0;
            bool dead = *abort_flag != 0;
            while (left > 0 && !dead) {
                const Span item = span_of(a, w.r, w.m * kTileRows, kTileRows);
                const int take = w.n_chunks - w.c < left ? w.n_chunks - w.c : left;
                for (int kc = 0; kc < take; kc++, nv++) {
                    if (++st == L::kStages) {   // past the keys
                        st = 0;
                        ph ^= 1;
                    }
                    if (!__all_sync(0xffffffffu, mbar_wait(&M->full[st], ph, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    const int t0 = w.t.id(w.c + kc) * kKT;
                    int found = 0;
                    if (!item.sees_all(a, t0)) {
                        unsigned char* tile = smem + L::stages + st * L::kStage;
                        constexpr int kPer = D / 8;
                        const int ch = lane % kPer;
                        for (int r = lane / kPer; r < kKT; r += 32 / kPer) {
                            const int t = t0 + r;
                            if (!item.partial(a, t)) continue;
                            uint4* p = reinterpret_cast<uint4*>(tile + (ch >> 3) * L::kPiece + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
                            if (t >= w.r.len) {
                                *p = make_uint4(0, 0, 0, 0);
                            } else {
                                const uint4 v = *p;
                                if (any_special<FP16>(v)) {
                                    *p = make_uint4(drop_special<FP16>(v.x), drop_special<FP16>(v.y), drop_special<FP16>(v.z), drop_special<FP16>(v.w));
                                    found = 1;
                                }
                            }
                        }
                        found = __any_sync(0xffffffffu, found);
                        fence_proxy_async_smem();
                    }
                    __syncwarp();
                    if (lane == 0) {
                        *(volatile int*)&M->special[nv & 3] = found;
                        mbar_arrive(&M->vok[nv & 3]);
                    }
                    if (++st == L::kStages) {
                        st = 0;
                        ph ^= 1;
                    }
                }
                left -= take;
                if (left > 0) w.next(P);
            }
            if (dead) *abort_flag = 1;
        }
    }
    __syncthreads();
    if (tid == 0 && *abort_flag) raise_flag(a.status, CG_FLAG_PIPE_TIMEOUT);
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Joins the parts of the tile that starts in CTA b's share. A thread owns a row and 8 channels
// (blockIdx.y): its parts' references, then one pass over the parts.
template <bool FP16, int D>
__global__ void __launch_bounds__(kTileRows) paged_chunk_merge_kernel(const __grid_constant__ ChunkParams P) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const PagedArgs& a = P.a;
    const ChunkMeta m = P.meta[blockIdx.x];
    const int row = threadIdx.x;
    if (m.last < 0 || row >= m.n_rows) return;
    const int parts = m.last - (int)blockIdx.x + 1;
    auto part = [&](int p) { return P.parts + ((int64_t)(blockIdx.x + p) * 2 + (p == 0 ? 1 : 0)) * chunk_part_floats(D); };
    float R = -INFINITY;
    for (int p = 0; p < parts; p++) R = fmaxf(R, part(p)[kTileRows * D + row]);
    const float Rs = R == -INFINITY ? 0.0f : R;
    float l = 0.0f, o[8];
#pragma unroll
    for (int k = 0; k < 8; k++) o[k] = 0.0f;
#pragma unroll 4
    for (int p = 0; p < parts; p++) {
        const float* src = part(p);
        const float ref = src[kTileRows * D + row];
        const float f = ref == -INFINITY ? 0.0f : fmaxf(ex2(ref - Rs), 1.17549435e-38f);
        l += f * src[kTileRows * D + kTileRows + row];
        const float4 u = reinterpret_cast<const float4*>(src)[(2 * blockIdx.y) * kTileRows + row];
        const float4 v = reinterpret_cast<const float4*>(src)[(2 * blockIdx.y + 1) * kTileRows + row];
        o[0] += f * u.x;
        o[1] += f * u.y;
        o[2] += f * u.z;
        o[3] += f * u.w;
        o[4] += f * v.x;
        o[5] += f * v.y;
        o[6] += f * v.z;
        o[7] += f * v.w;
    }
    const int r = m.row0 + row, tk = r / a.n_rep, hd = m.h * a.n_rep + (r - tk * a.n_rep);
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; k++) b[k] = inv == 0.0f ? 0u : pack2<FP16>(o[2 * k] * inv, o[2 * k + 1] * inv);
    *reinterpret_cast<uint4*>(a.out + (int64_t)(m.tok0 + tk) * a.o_tok + hd * a.o_head + 8 * blockIdx.y) =
        make_uint4(b[0], b[1], b[2], b[3]);
    if (a.lse && blockIdx.y == 0)
        a.lse[(int64_t)(m.tok0 + tk) * a.H * a.n_rep + hd] = inv == 0.0f ? -INFINITY : (R + log2f(l)) * kLn2;
}

template <bool FP16, int D>
cudaError_t launch_chunk(const ChunkParams& P, cudaStream_t st) {
    CUtensorMap map;
    if (!paged_pool_map(&map, P.a, P.box_rows)) return cudaErrorInvalidValue;
    constexpr size_t smem = ChunkSmem<D>::total;
    cudaError_t e = cudaFuncSetAttribute(paged_chunk_kernel<FP16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)tc::num_sms();
    paged_chunk_kernel<FP16, D><<<grid, kChunkThreads, smem, st>>>(P, map);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid, D / 8);
    cfg.blockDim = dim3(kTileRows);
    cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, paged_chunk_merge_kernel<FP16, D>, P);
}

}  // namespace

size_t paged_chunk_workspace(int d) {
    const size_t n = (size_t)tc::num_sms();
    return n * 2 * chunk_part_floats(d) * sizeof(float) + n * sizeof(ChunkMeta);
}

cudaError_t launch_paged_chunk(const PagedArgs& a, int min_rows, void* workspace, cudaStream_t st) {
    ChunkParams P{};
    P.a = a;
    P.parts = static_cast<float*>(workspace);
    P.meta = reinterpret_cast<ChunkMeta*>(P.parts + (size_t)tc::num_sms() * 2 * chunk_part_floats(a.d));
    P.min_rows = min_rows;
    P.min_share = 4;
    P.box_rows = a.page < kKT ? a.page : kKT;
    const bool h = a.dtype == CG_FP16;
    if (a.d == 64) return h ? launch_chunk<true, 64>(P, st) : launch_chunk<false, 64>(P, st);
    return h ? launch_chunk<true, 128>(P, st) : launch_chunk<false, 128>(P, st);
}

}  // namespace cg
