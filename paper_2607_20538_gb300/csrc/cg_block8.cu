// cg_block8.cu -- matrices in e4m3 with a scale for each block of 128 channels: encoding, and the product of two of
// them. Contract: include/codecgauge_block8.h.
#include <cooperative_groups.h>
#include <cuda_fp8.h>

#include "../../include/codecgauge_block8.h"
#include "cg_follow.cuh"
#include "cg_launch.h"
#include "cg_overlap.h"
#include "cg_paged.h"
#include "cg_sm100.cuh"
#include "cg_tc_common.cuh"
#include "cg_tmap.h"

#define CG_EXPORT __attribute__((visibility("default")))

namespace cg {
namespace {

using namespace sm100;

constexpr int kBlock = CG_BLOCK8;
constexpr float kTop = 448.0f;

// ------------------------------------------------------------------------------------
// Encoding. 8 lanes a row of a block, 16 channels each: 32 bytes in, 16 bytes out. The largest |x| is found on the
// bits (the order of non-negative numbers is that of their bits, infinities and NaN above all). A scale for one
// row needs the 8 lanes alone, one for 128 rows a CTA, whose threads keep their 4 rows in registers. Bound: HBM, 3
// bytes a value, and 3 us of start and end: 8192 x 4096 18.4 us, 5.5 TB/s; 16384 x 16384 128 us, 6.3 TB/s; 131072 x 4096 250 us, 6.5 TB/s;
// by 128 rows 16384 x 8192 65 us, 6.2 TB/s. (With unpacked arithmetic the first took 24.4, the second 164, the last 81 us.)
// ------------------------------------------------------------------------------------
constexpr int kEncThreads = 256, kGroup = 8, kEncRows = kEncThreads / kGroup;   // rows of blocks of a CTA and turn

struct EncArgs {
    const uint16_t* x;
    uint8_t* codes;
    float* scales;
    int32_t* status;
    int64_t R, K, x_stride, stride, nb;   // nb blocks a row
    int64_t step_row, step_b;             // of all CTAs' blocks of one turn
};

template <bool FP16>
__device__ __forceinline__ float2 floats(uint32_t w) {
    if (FP16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

struct Piece {
    uint32_t w[8];   // 16 values
    __device__ __forceinline__ void load(const uint16_t* p, bool have) {
        const uint4 zero = make_uint4(0, 0, 0, 0);
        const uint4 a = have ? *reinterpret_cast<const uint4*>(p) : zero, b = have ? *(reinterpret_cast<const uint4*>(p) + 1) : zero;
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
    // bits of the largest |x|
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; k++) m = __vmaxu2(m, w[k] & 0x7fff7fffu);
        return max(m & 0xffffu, m >> 16);
    }
};

// A block's scale from the bits of its largest |x|, and the codes of its values. The quotient x / s is rounded
// as a division rounds it: q = x r with the rounded reciprocal r, then q + r (x - q s), whose residual is exact
// (Markstein, 1990); where r or the residual could leave the normal numbers the division itself is used.
template <bool FP16>
struct Scale {
    float s, r;
    bool nonfinite, plain;
    __device__ __forceinline__ explicit Scale(uint32_t top) {
        nonfinite = top >= (FP16 ? 0x7c00u : 0x7f80u);
        s = nonfinite ? __uint_as_float(0x7fffffffu) : floats<FP16>(top).x / kTop;
        plain = !(s >= 0x1p-80f && s <= 0x1p100f);
        r = plain ? 0.0f : __frcp_rn(s);
    }
    __device__ __forceinline__ float2 quotients(float2 x) const {
        const float2 rr = make_float2(r, r), q = __fmul2_rn(x, rr);
        return __ffma2_rn(__ffma2_rn(q, make_float2(-s, -s), x), rr, q);
    }
    // the signs are put in behind: that of -0 is lost in the residual
    __device__ __forceinline__ uint32_t four(uint32_t w0, uint32_t w1) const {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(quotients(floats<FP16>(w0)), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(quotients(floats<FP16>(w1)), __NV_SATFINITE, __NV_E4M3);
        return (lo | hi << 16) | (__byte_perm(w0, w1, 0x7531) & 0x80808080u);
    }
    static __device__ __noinline__ uint32_t four_divided(uint32_t w0, uint32_t w1, float s) {
        const float2 x = floats<FP16>(w0), y = floats<FP16>(w1);
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x.x / s, x.y / s), __NV_SATFINITE, __NV_E4M3);
        return lo | (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y.x / s, y.y / s), __NV_SATFINITE, __NV_E4M3) << 16;
    }
    __device__ __forceinline__ uint4 codes(const Piece& p) const {
        uint32_t c[4];
        if (!plain) {
#pragma unroll
            for (int k = 0; k < 4; k++) c[k] = four(p.w[2 * k], p.w[2 * k + 1]);
        } else if (nonfinite || s == 0.0f) {
            c[0] = c[1] = c[2] = c[3] = nonfinite ? 0x7f7f7f7fu : 0u;
        } else {
#pragma unroll
            for (int k = 0; k < 4; k++) c[k] = four_divided(p.w[2 * k], p.w[2 * k + 1], s);
        }
        return make_uint4(c[0], c[1], c[2], c[3]);
    }
};

// rows = 1: a group of 8 lanes a block, U blocks at a time. A group walks from block to block in steps of (step_row, step_b).
template <bool FP16, int U>
__global__ void __launch_bounds__(kEncThreads) encode_rows_kernel(EncArgs a) {
    const int lane8 = threadIdx.x % kGroup;
    const int64_t first = (int64_t)blockIdx.x * kEncRows + threadIdx.x / kGroup;
    int64_t row = first / a.nb, b = first - row * a.nb;
    int32_t flag = 0;
    follow();
    while (__any_sync(0xffffffffu, row < a.R)) {
        Piece p[U];
        int64_t at_row[U], at_b[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            at_row[u] = row;
            at_b[u] = b;
            const int64_t ch = b * kBlock + lane8 * 16;
            p[u].load(a.x + row * a.x_stride + ch, row < a.R && ch < a.K);
            row += a.step_row;
            b += a.step_b;
            if (b >= a.nb) {
                b -= a.nb;
                row++;
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            uint32_t top = p[u].top();
#pragma unroll
            for (int off = 1; off < kGroup; off *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
            const Scale<FP16> s(top);
            if (s.nonfinite) flag = CG_FLAG_NONFINITE_INPUT;
            if (at_row[u] >= a.R) continue;
            const int64_t ch = at_b[u] * kBlock + lane8 * 16;
            if (ch < a.K) *reinterpret_cast<uint4*>(a.codes + at_row[u] * a.stride + ch) = s.codes(p[u]);
            if (lane8 == 0) a.scales[at_row[u] * a.nb + at_b[u]] = s.s;
        }
    }
    raise_flag(a.status, flag);
}

// rows = 128: a CTA a block.
template <bool FP16>
__global__ void __launch_bounds__(kEncThreads) encode_square_kernel(EncArgs a) {
    constexpr int kPer = kBlock / kEncRows;
    __shared__ uint32_t tops[kEncThreads / 32];
    const int lane8 = threadIdx.x % kGroup, r0 = threadIdx.x / kGroup, warp = threadIdx.x >> 5;
    const int64_t rb = (a.R + kBlock - 1) / kBlock, items = rb * a.nb;
    int32_t flag = 0;
    follow();
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int64_t r = it / a.nb, b = it - r * a.nb, ch = b * kBlock + lane8 * 16;
        Piece p[kPer];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < kPer; k++) {
            const int64_t row = r * kBlock + r0 + k * kEncRows;
            p[k].load(a.x + row * a.x_stride + ch, row < a.R && ch < a.K);
        }
#pragma unroll
        for (int k = 0; k < kPer; k++) top = max(top, p[k].top());
        top = __reduce_max_sync(0xffffffffu, top);
        if ((threadIdx.x & 31) == 0) tops[warp] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kEncThreads / 32; w++) top = max(top, tops[w]);
        __syncthreads();
        const Scale<FP16> s(top);
        if (s.nonfinite) flag = CG_FLAG_NONFINITE_INPUT;
#pragma unroll
        for (int k = 0; k < kPer; k++) {
            const int64_t row = r * kBlock + r0 + k * kEncRows;
            if (row < a.R && ch < a.K) *reinterpret_cast<uint4*>(a.codes + row * a.stride + ch) = s.codes(p[k]);
        }
        if (threadIdx.x == 0) a.scales[it] = s.s;
    }
    raise_flag(a.status, flag);
}

// ------------------------------------------------------------------------------------
// Product. A tile is 128 rows of x (the lanes of tensor memory) by 128 rows of w (its columns). Block by block of 128
// channels the tensor cores (tcgen05.mma, kind f8f6f4, four instructions of 32 channels) sum the products into one of
// four buffers of tensor memory; the accumulating warps read it, multiply by the block's two scales and add to sums in
// registers, while the other buffers fill.
//   warps 0 - 7   accumulate: warp w has lanes 32 (w % 4) .. + 31 and columns 64 (w / 4) .. + 63; lanes past the last row
//                 of x are left out
//   warp 8        TMA: both matrices' 128-byte pieces of rows into a ring of stages (128-byte swizzle)
//   warps 9, 10   one thread each issues tcgen05.mma, of the even and of the odd blocks (one warp's loop takes 650 cycles
//                 a block, its products 256)
// Few rows of x: a stage holds them in whole groups of 8, and more stages fit; the lanes that they do not fill multiply
// what lies behind, and nobody reads them.
// Few tiles: the blocks of channels are cut among the CTAs of a cluster; each writes its sums of a part of the rows into the
// shared memory of the CTA that adds those up, in the order of the ranks whatever their timing. (Left where they were and
// read from there they cost 333 x 1000 x 4112 4.1 us of 10.7, two rounds of loads' latency and a barrier more.) Bound: latency, of the
// start, the first block and a cluster's sums (5.6 of 8.4 us at 333 x 1000 x 4112), and, with few rows, that the warps of their lanes alone
// read, scale and send: 17 x 6144 x 4096 9.1 us, where the kernel for up to 8 rows takes in the same bytes in 6.4; 64 rows 9.8, 256 14.6.
// ------------------------------------------------------------------------------------
constexpr int kLanes = 128;

struct Tile {
    static constexpr int TC = 128, CW = 64;                     // columns, and those of a warp
    static constexpr int kWarps = 8, kThreads = (kWarps + 3) * 32;
    static constexpr uint32_t kB = TC * 128, ring = 196608;
    // a cluster's ring; the sums follow, [rank][columns / 4][rows of a part, an odd number][4]: a warp's store is 512 bytes in a
    // row (with the columns of a row together 64 KB took 2.5 us), and the columns of a row lie in different banks
    static constexpr uint32_t split_ring = 159744;
    static constexpr int kMost = 10;                            // stages
    static constexpr int kBufs = 4;                             // of tensor memory
    static constexpr uint32_t misc = 231936, total = misc + 512;
    static_assert(split_ring % 1024 == 0 && split_ring + (kLanes + 12) * TC * 4 <= misc && ring <= misc && ring + kWarps * 4096 <= misc && kMost * (kB + 1024) <= ring && total <= 232448, "tile");
};

struct MatArgs {
    const float *xs, *ws;
    void* out;
    int32_t* status;
    int64_t M, N, nb, out_stride;
    int64_t lane_tiles, col_tiles;
    uint64_t wait_ns;
    int fp16, vec;       // 16-byte stores are possible
    int vec_scales;      // 16-byte loads of scales are possible
    int split;           // CTAs of a cluster
    int group;           // lane tiles that are walked together
    int box_rows;        // of x in a stage
};

// The tiles of a CTA (or a pair, or a cluster), every step-th from the first: lane tiles in groups, so that those at work
// share both matrices' rows in L2.
struct TileWalk {
    int g, in, lt, ct;      // group, tile in it; lane tile, column tile
    __device__ __forceinline__ bool set(const MatArgs& a) {
        for (;;) {
            const int left = (int)a.lane_tiles - g * a.group, n = left < a.group ? left : a.group;
            if (n <= 0) return false;
            if (in < n * (int)a.col_tiles) {
                ct = in / n;
                lt = g * a.group + (in - ct * n);
                return true;
            }
            in -= n * (int)a.col_tiles;
            g++;
        }
    }
    __device__ __forceinline__ bool start(const MatArgs& a, int first) {
        g = 0;
        in = first;
        return set(a);
    }
    __device__ __forceinline__ bool next(const MatArgs& a, int step) {
        in += step;
        return set(a);
    }
};

struct MatMisc {
    uint64_t full[Tile::kMost], empty[Tile::kMost], tfull[Tile::kBufs], tempty[Tile::kBufs], drain;
    int abort_flag;
    uint32_t tmem;
};
static_assert(sizeof(MatMisc) <= 512, "misc block");

// One step of 32 channels. Descriptors as halves (a step only adds to the low ones) that the whole warp computes, so that
// they stay in uniform registers, and an elected thread: behind a branch on the lane number a block's issue took 500
// cycles, as long as its products.
template <bool PAIR>
__device__ __forceinline__ void mma_e4m3(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
    if (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
            "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
            "setp.ne.b32 p, %5, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], da, db, %4, p;\n\t}" ::"r"(d_tmem),
            "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
            "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
            "setp.ne.b32 p, %5, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n\t}" ::"r"(d_tmem),
            "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
            : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// Instruction descriptor (kind::f8f6f4): e4m3 A and B, both K-major, fp32 D, M x N.
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N) {
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Address of the same place in the shared memory of a CTA of the cluster.
__device__ __forceinline__ uint32_t at_rank(const void* p, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
// The cluster's barrier in halves; every thread calls both, in turn.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
          "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(taddr));
}
// Uses of r stay behind the wait that precedes this.
__device__ __forceinline__ void settle16(float (&r)[16]) {
    asm volatile("" : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]),
                 "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]));
}

__device__ __forceinline__ uint32_t pack(float x, float y, int fp16) {   // x in the low half
    if (fp16) {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&b);
}

// Up to 8 values (16 bytes) to dst.
__device__ __forceinline__ void store_piece(uint16_t* dst, uint4 v, int valid, bool vec) {
    if (vec && valid >= 8) {
        *reinterpret_cast<uint4*>(dst) = v;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e < valid) dst[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
}

// A warp's results in shared memory: boxes of 32 rows x 64 columns (4 KB) in the 128-byte swizzle. acc: the lane's row.
template <int COLS>
__device__ __forceinline__ void stage_results(unsigned char* box, const float2 (&acc)[COLS / 2], int fp16) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int q = 0; q < COLS / 8; q++) {
        const uint4 b = make_uint4(pack(acc[4 * q].x, acc[4 * q].y, fp16), pack(acc[4 * q + 1].x, acc[4 * q + 1].y, fp16),
                                   pack(acc[4 * q + 2].x, acc[4 * q + 2].y, fp16), pack(acc[4 * q + 3].x, acc[4 * q + 3].y, fp16));
        *reinterpret_cast<uint4*>(box + (q >> 3) * 4096 + lane * 128 + (((q & 7) ^ (lane & 7)) << 4)) = b;
    }
}
// Staged results to rows that begin anywhere, 8 rows at a time: a row's words of two values from its first even place on, side
// by side in the warp, the ends alone. (Value by value from registers 8192 x 6147 x 4096 took 356 us.) out: the first row's
// first column; rows <= 32, n <= COLS: rows and columns there are.
template <int COLS>
__device__ __forceinline__ void store_staged(const unsigned char* box, uint16_t* out, int64_t stride, int rows, int n) {
    const int lane = threadIdx.x & 31, end = n - 1;   // the last column, in word end / 2
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += 8) {
        uint32_t v[8][COLS / 64];                     // columns 2 lane, 2 lane + 1 of each box
#pragma unroll
        for (int k = 0; k < 8; k++)
#pragma unroll
            for (int i = 0; i < COLS / 64; i++)
                v[k][i] = *reinterpret_cast<const uint32_t*>(box + i * 4096 + (r0 + k) * 128 + ((((lane >> 2) ^ k) << 4) | ((lane & 3) << 2)));
#pragma unroll
        for (int k = 0; k < 8; k++) {
            if (r0 + k >= rows) break;
            uint16_t* row = out + (r0 + k) * stride;
            const int odd = (int)(reinterpret_cast<uintptr_t>(row) >> 1 & 1);
#pragma unroll
            for (int i = 0; i < COLS / 64; i++) {
                uint32_t w = v[k][i];
                const uint32_t down = __shfl_down_sync(0xffffffffu, w, 1), other = i + 1 < COLS / 64 ? __shfl_sync(0xffffffffu, v[k][(i + 1) % (COLS / 64)], 0) : 0u;
                if (odd) w = __funnelshift_r(w, lane < 31 ? down : other, 16);
                const int e = 64 * i + 2 * lane + odd;
                if (e + 1 < n) *reinterpret_cast<uint32_t*>(row + e) = w;
                if (((end - odd) & 1) == 0 && (end >> 1) == 32 * i + lane) row[end] = (uint16_t)(v[k][i] >> (16 * (end & 1)));
            }
            if (lane == 0 && odd) row[0] = (uint16_t)v[k][0];
        }
    }
}

// 32 columns of each lane's row. The lanes of a group of four transpose their pieces of 16 bytes, so that a store
// instruction covers 64 bytes of 8 rows instead of 16 of 32. row: of the output, or null; left: its columns from here on.
__device__ __forceinline__ void store_columns(uint32_t (&b)[16], uint16_t* row, int left) {
    const int lane = threadIdx.x & 31, j = lane & 3;
#pragma unroll
    for (int step = 1; step < 4; step *= 2) {
        const bool up = lane & step;
#pragma unroll
        for (int k = 0; k < 4; k++) {
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
    const int valid = left - 8 * j < 8 ? left - 8 * j : 8;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const uint64_t dst = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(row), (lane & 28) + k);
        if (dst && valid > 0)
            store_piece(reinterpret_cast<uint16_t*>(dst) + 8 * j, make_uint4(b[4 * k], b[4 * k + 1], b[4 * k + 2], b[4 * k + 3]), valid, true);
    }
}

__global__ void __launch_bounds__(Tile::kThreads, 1)
block8_tile_kernel(const __grid_constant__ MatArgs a, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map) {
    using T = Tile;
    extern __shared__ __align__(1024) unsigned char smem[];
    MatMisc* S = reinterpret_cast<MatMisc*>(smem + T::misc);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)(blockIdx.x % (unsigned)a.split);
    const int first = (int)(blockIdx.x / (unsigned)a.split), step = (int)(gridDim.x / (unsigned)a.split);
    const int kb0 = (int)(a.nb * rank / a.split), kb1 = (int)(a.nb * (rank + 1) / a.split);
    const uint32_t stage = a.box_rows * 128 + T::kB;
    const int stages = min(T::kMost, (int)((a.split > 1 ? T::split_ring : T::ring) / stage));
    if (a.split > 1) cluster_arrive();   // (waited for before anything is written into another CTA's shared memory: it has started then)
    if (tid == 0) {
        for (int s = 0; s < stages; s++) {
            mbar_init(&S->full[s], 1);
            mbar_init(&S->empty[s], 1);
        }
        for (int s = 0; s < T::kBufs; s++) {
            mbar_init(&S->tfull[s], 1);
            mbar_init(&S->tempty[s], T::kWarps);
        }
        mbar_init(&S->drain, 2);
        S->abort_flag = (smem_u32(smem) & 1023u) != 0;   // the swizzle needs the alignment asked for
        fence_barrier_init();
        prefetch_tmap(&x_map);
        prefetch_tmap(&w_map);
    }
    if (warp == T::kWarps + 1) {
        tmem_alloc(&S->tmem, T::kBufs * T::TC);
        tmem_relinquish();
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    follow();
    let_follow();
    const uint32_t tmem = S->tmem;
    volatile int* abort_flag = &S->abort_flag;
    TileWalk w;
    bool more = w.start(a, first);
    // of a cluster's tile: its place, its rows, and how many of them each CTA adds up
    const int64_t m0 = (int64_t)w.lt * kLanes, n0 = (int64_t)w.ct * T::TC;
    const int have = a.M - m0 < kLanes ? (int)(a.M - m0) : kLanes, part = (have + a.split - 1) / a.split;
    bool dead = *abort_flag != 0;

    if (warp < T::kWarps) {
        // ------------------------------------------------------------ accumulate
        const int col0 = (warp >> 2) * T::CW, row0 = 32 * (warp & 3), row = row0 + lane;
        const uint32_t t0 = tmem + ((uint32_t)row0 << 16) + col0;
        int buf = 0, ph = 0;
        for (; more && !dead; more = w.next(a, step)) {
            const int64_t r = (int64_t)w.lt * kLanes + row, c = (int64_t)w.ct * T::TC + col0;    // the thread's row, and first column
            const bool idle = (int64_t)w.lt * kLanes + row0 >= a.M;                   // no row of the warp's is one of x
            float2 acc[T::CW / 2];
#pragma unroll
            for (int k = 0; k < T::CW / 2; k++) acc[k] = make_float2(0.0f, 0.0f);
            // scales of four blocks, fetched four blocks ahead
            const float *px = a.xs + (r < a.M ? r : a.M - 1) * a.nb, *pw = a.ws + w.ct * a.nb;   // (128 columns: one block of w)
            float nx[4], nw[4], f[4];
            auto fetch = [&](int kb) {
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int k = kb + i < kb1 ? kb + i : kb1 - 1;
                    nx[i] = px[k];
                    nw[i] = pw[k];
                }
            };
            if (!idle && kb0 < kb1) fetch(kb0);
            for (int kb = kb0; kb < kb1; kb++) {
                const bool fresh = ((kb - kb0) & 3) == 0;
#pragma unroll
                for (int i = 0; i < 4; i++) f[i] = fresh ? nx[i] * nw[i] : f[i < 3 ? i + 1 : 3];
                if (fresh && !idle && kb + 4 < kb1) fetch(kb + 4);
                if (!__all_sync(0xffffffffu, mbar_wait(&S->tfull[buf], ph, abort_flag, a.wait_ns))) {
                    dead = true;
                    break;
                }
                tc_fence_after();
                if (!idle) {
                    float v[3][16];   // read in pairs, of which the next one's first half is asked for ahead
                    tmem_ld16(t0 + buf * T::TC, v[0]);
                    tmem_ld16(t0 + buf * T::TC + 16, v[1]);
#pragma unroll
                    for (int q = 0; q < T::CW / 16; q++) {
                        if ((q & 1) == 0) tmem_wait_ld();
                        settle16(v[q % 3]);
                        if ((q & 1) == 0) settle16(v[(q + 1) % 3]);
                        if (16 * (q + 2) < T::CW) tmem_ld16(t0 + buf * T::TC + 16 * (q + 2), v[(q + 2) % 3]);
                        const float2 ff = make_float2(f[0], f[0]);
#pragma unroll
                        for (int k = 0; k < 8; k++) acc[8 * q + k] = __ffma2_rn(make_float2(v[q % 3][2 * k], v[q % 3][2 * k + 1]), ff, acc[8 * q + k]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&S->tempty[buf]);
                if (++buf == T::kBufs) {
                    buf = 0;
                    ph ^= 1;
                }
            }
            if (dead) break;
            if (a.split > 1) {
                cluster_wait();
                if (row < have) {
                    const int pitch = part | 1, owner = row / part;
                    const float4* here = reinterpret_cast<const float4*>(smem + T::split_ring) + (rank * (T::TC / 4) + col0 / 4) * pitch + row - owner * part;
                    const uint32_t dst = at_rank(here, (uint32_t)owner);
#pragma unroll
                    for (int k = 0; k < T::CW / 4; k++)
                        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst + 16 * k * pitch), "f"(acc[2 * k].x), "f"(acc[2 * k].y),
                                     "f"(acc[2 * k + 1].x), "f"(acc[2 * k + 1].y)
                                     : "memory");
                }
                break;
            }
            const int rows = a.M - (r - lane) < 32 ? (int)(a.M - (r - lane)) : 32, n = a.N - c < T::CW ? (int)(a.N - c) : T::CW;
            if (rows <= 0 || n <= 0) continue;
            uint16_t* out = static_cast<uint16_t*>(a.out) + (r - lane) * a.out_stride + c;   // (the warp's first row)
            if (a.vec) {
#pragma unroll
                for (int q = 0; q < T::CW / 32; q++) {
                    uint32_t b[16];
#pragma unroll
                    for (int k = 0; k < 16; k++) b[k] = pack(acc[16 * q + k].x, acc[16 * q + k].y, a.fp16);
                    if (32 * q < n) store_columns(b, lane < rows ? out + lane * a.out_stride + 32 * q : nullptr, n - 32 * q);
                }
            } else {
                unsigned char* box = smem + T::ring + warp * 4096;
                stage_results<T::CW>(box, acc, a.fp16);
                __syncwarp();
                store_staged<T::CW>(box, out, a.out_stride, rows, n);
                __syncwarp();
            }
        }
    } else if (warp == T::kWarps) {
        // ------------------------------------------------------------ copies
        int st = 0, ph = 1;
        int64_t issued = 0;
        for (; more && !dead; more = w.next(a, step)) {
            for (int kb = kb0; kb < kb1; kb++) {
                if (!__all_sync(0xffffffffu, mbar_wait(&S->empty[st], ph, abort_flag, a.wait_ns))) {
                    dead = true;
                    break;
                }
                if (lane == 0) {
                    mbar_arrive_expect_tx(&S->full[st], stage);
                    tma_load_2d(smem + st * stage + a.box_rows * 128, &w_map, &S->full[st], kb * kBlock, w.ct * T::TC);
                    tma_load_2d(smem + st * stage, &x_map, &S->full[st], kb * kBlock, w.lt * kLanes);
                }
                __syncwarp();
                issued++;
                if (++st == stages) {
                    st = 0;
                    ph ^= 1;
                }
            }
        }
        if (dead) *abort_flag = 1;
        // copies in flight land before the CTA ends, also where the other warps gave up on them
        const int zero = 0;
        for (int64_t k = issued > stages ? issued - stages : 0; k < issued; k++)
            mbar_wait(&S->full[k % stages], (k / stages) & 1, &zero, tc::kWaitLimitNs);
    } else {
        // ------------------------------------------------------------ products of every other block
        constexpr uint32_t idesc = idesc_e4m3(kLanes, T::TC);
        const bool issue = elect_one();
        const uint64_t desc = sdesc_sw128(smem_u32(smem));
        const uint32_t a_lo = (uint32_t)desc, hi = (uint32_t)(desc >> 32);
        const int odd = warp - T::kWarps - 1, n = kb1 - kb0;
        int st = odd % stages, ph = odd / stages & 1, buf = odd, tph = 1, k0 = odd;
        for (; more && !dead; more = w.next(a, step)) {
            for (; k0 < n; k0 += 2) {
                if (!__all_sync(0xffffffffu, mbar_wait(&S->tempty[buf], tph, abort_flag, a.wait_ns)) ||
                    !__all_sync(0xffffffffu, mbar_wait(&S->full[st], ph, abort_flag, a.wait_ns))) {
                    dead = true;
                    break;
                }
                tc_fence_after();
                const uint32_t da = a_lo + ((st * stage) >> 4), db = da + ((a.box_rows * 128) >> 4), d = tmem + buf * T::TC;
                if (issue) {
#pragma unroll
                    for (int k = 0; k < kBlock / 32; k++) mma_e4m3<false>(d, da + 2 * k, db + 2 * k, hi, idesc, k ? 1u : 0u);
                    mma_commit(&S->tfull[buf]);
                    mma_commit(&S->empty[st]);
                }
                __syncwarp();
                buf += 2;
                if (buf >= T::kBufs) {
                    buf -= T::kBufs;
                    tph ^= 1;
                }
                st += 2;
                if (st >= stages) {
                    st -= stages;
                    ph ^= 1;
                }
            }
            k0 -= n;   // the warp's first block of the next tile
        }
        if (dead) *abort_flag = 1;
        if (issue) mma_commit(&S->drain);   // products in flight end before tensor memory is given back
        __syncwarp();
        const int zero = 0;
        mbar_wait(&S->drain, 0, &zero, tc::kWaitLimitNs);
    }
    __syncwarp();
    if (dead) {
        *abort_flag = 1;
        if (lane == 0) raise_flag(a.status, CG_FLAG_PIPE_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == T::kWarps + 1) {
        tc_fence_after();
        tmem_dealloc(tmem, T::kBufs * T::TC);
    }
    if (a.split > 1) {
        // ---- this CTA's part of the rows
        if (warp >= T::kWarps || dead) cluster_wait();   // (the others have)
        cooperative_groups::this_cluster().sync();
        const int r0 = rank * part, rows = have - r0 < part ? have - r0 : part;
        const float4* sums = reinterpret_cast<const float4*>(smem + T::split_ring);
        for (int x = tid; x < rows * (T::TC / 4); x += T::kThreads) {
            const int r = x / (T::TC / 4), c = x % (T::TC / 4), pitch = part | 1;
            const int64_t m = m0 + r0 + r, n = n0 + 4 * c;
            if (n >= a.N) continue;
            float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int k = 0; k < a.split; k++) {
                const float4 v = sums[(k * (T::TC / 4) + c) * pitch + r];
                s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
            }
            uint16_t* dst = static_cast<uint16_t*>(a.out) + m * a.out_stride + n;
            const uint2 w = make_uint2(pack(s.x, s.y, a.fp16), pack(s.z, s.w, a.fp16));
            if (a.vec && n + 4 <= a.N) *reinterpret_cast<uint2*>(dst) = w;
            else store_piece(dst, make_uint4(w.x, w.y, 0u, 0u), a.N - n < 4 ? (int)(a.N - n) : 4, false);
        }
    }
}

// ------------------------------------------------------------------------------------
// Product of many rows: pairs of CTAs (a cluster of two, tcgen05 cta_group::2). A tile is 256 rows of x by 256 rows of
// w; each CTA of the pair copies 128 rows of x and half the rows of w, and its tensor memory takes the sums of its
// own rows with all columns, so that a product reads 32 KB a block and SM where a CTA for itself would read 48.
// Bound: the tensor cores (512 cycles a block), and the sums' way through registers beside them: 8192 x 6144 x 4096 158 us, 2.6
// PFLOP/s, in long runs 173 (power cap); 8192 x 8192 x 8192 383 us, 2.9. The products alone 122 us, with the sums read 131.
// The two halves of the columns are products, buffers and barriers of their own (N = 128): while one half's sums are
// read, the other's products run.
//   warps 0 - 7   accumulate, as above: a thread a row and one half's columns, in 208 registers. Results go through
//                 shared memory and TMA stores, which run beside the next tile.
//   warp 8        TMA of the CTA's own halves
//   warps 9, 10   of the first CTA: one thread each issues the pair's tcgen05.mma of the even and of the odd blocks
//                 (a buffer of tensor memory each; one warp's loop took 850 cycles a block for 512 of products)
//   warp 11       waits for the CTA's own copies and arrives at the first one's `ready` (each CTA so waits for its own copies
//                 alone, and can at its end; the issuing warps have one barrier to look at for both)
// ------------------------------------------------------------------------------------
struct Pair {
    static constexpr int TC = 256, CW = TC / 2;
    static constexpr int kThreads = 384;
    static constexpr uint32_t kA = kLanes * 128, kB = CW / 2 * 128, kStage = kA + 2 * kB;
    static constexpr int kStages = 5;
    static constexpr uint32_t kOut = 32 * 128;                   // 32 rows x 64 columns of results, 128-byte swizzle
    static constexpr uint32_t out = kStages * kStage;            // [warp][2]
    static constexpr uint32_t misc = out + 16 * kOut, total = misc + 512;
    static_assert(CW == kBlock && kB % 1024 == 0 && total <= 232448, "tile");
};

struct PairMisc {
    uint64_t full[5], ready[5], empty[5], tfull[2][2], tempty[2][2], drain;   // (tensor memory: by buffer and half of the columns)
    int abort_flag;
    uint32_t tmem;
};
static_assert(sizeof(PairMisc) <= 512, "misc block");

// Arrival at a barrier of either CTA. What the other side may rely on goes through tensor memory (with its fences) and
// the copies' own barrier, not through this thread's loads and stores, so that the arrival need not wait for those:
// with .release.cluster here and .acquire.cluster in the waits a block took 2400 cycles.
__device__ __forceinline__ void arrive_at(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// mbar_wait, whole in its place: where warps exchange registers a wait in the loops must not be a call.
__device__ __forceinline__ bool pair_wait(uint64_t* bar, uint32_t parity, const volatile int* abort, uint64_t limit_ns) {
    const bool poll = limit_ns < 1000000ull;   // the diagnostic setting of mbar_wait
    if (!poll && mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    for (uint32_t it = 0;; it++) {
        if (poll ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)) return true;
        if (poll || (it & 63u) == 63u) {
            if (*abort || globaltimer_ns() - t0 > limit_ns) return false;
        }
    }
}

// Arrives at `bar` of both CTAs once the pair's products issued before are done.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Pair::kThreads, 1)
block8_pair_kernel(const __grid_constant__ MatArgs a, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map,
                   const __grid_constant__ CUtensorMap out_map) {
    using T = Pair;
    extern __shared__ __align__(1024) unsigned char smem[];
    PairMisc* S = reinterpret_cast<PairMisc*>(smem + T::misc);
    auto cluster = cooperative_groups::this_cluster();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster.block_rank();
    const int nb = (int)a.nb;
    if (tid == 0) {
        for (int s = 0; s < T::kStages; s++) {
            mbar_init(&S->full[s], 1);
            mbar_init(&S->ready[s], 2);
            mbar_init(&S->empty[s], 1);
        }
        for (int s = 0; s < 4; s++) {
            mbar_init(&S->tfull[s >> 1][s & 1], 1);
            mbar_init(&S->tempty[s >> 1][s & 1], 8);
        }
        mbar_init(&S->drain, 2);
        S->abort_flag = (smem_u32(smem) & 1023u) != 0;   // the swizzle needs the alignment asked for
        fence_barrier_init();
        prefetch_tmap(&x_map);
        prefetch_tmap(&w_map);
        if (a.vec) prefetch_tmap(&out_map);
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S->tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        tc_fence_before();
    }
    __syncthreads();
    cluster.sync();
    tc_fence_after();
    follow();
    const uint32_t tmem = S->tmem;
    volatile int* abort_flag = &S->abort_flag;
    bool dead = *abort_flag != 0;
    TileWalk w;

    // 168 registers a thread at launch: 256 x 208 + 128 x 88 of 384 x 168
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // ------------------------------------------------------------ accumulate
        const int half = warp >> 2, col0 = half * T::CW, row0 = 32 * (warp & 3);
        const uint32_t t0 = tmem + ((uint32_t)row0 << 16) + col0;
        const uint32_t released[2] = {at_rank(&S->tempty[0][half], 0), at_rank(&S->tempty[1][half], 0)};
        unsigned char* out_sm = smem + T::out + warp * 2 * T::kOut;
        int buf = 0, ph = 0;
        // scales of four blocks, fetched four blocks ahead, across tiles
        const float *px, *pw;
        float nx[4], nw[4], f[4];
        auto fetch = [&](int kb) {
            if (a.vec_scales) {   // (whole groups of four)
                *reinterpret_cast<float4*>(nx) = *reinterpret_cast<const float4*>(px + kb);
                *reinterpret_cast<float4*>(nw) = *reinterpret_cast<const float4*>(pw + kb);
            } else {
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int k = kb + i < nb ? kb + i : nb - 1;
                    nx[i] = px[k];
                    nw[i] = pw[k];
                }
            }
        };
        auto scales_of_tile = [&]() {
            const int64_t r = (int64_t)w.lt * (2 * kLanes) + rank * kLanes + row0 + lane, u = ((int64_t)w.ct * T::TC + col0) / kBlock, last = (a.N - 1) / kBlock;
            px = a.xs + (r < a.M ? r : a.M - 1) * a.nb;
            pw = a.ws + (u < last ? u : last) * a.nb;
            fetch(0);
        };
        bool more = w.start(a, (int)(blockIdx.x >> 1));
        if (more) scales_of_tile();
        while (more && !dead) {
            const int r0 = w.lt * (2 * kLanes) + (int)rank * kLanes + row0, c = w.ct * T::TC + col0;    // the warp's first row and column
            float2 acc[T::CW / 2];
#pragma unroll
            for (int k = 0; k < T::CW / 2; k++) acc[k] = make_float2(0.0f, 0.0f);
            for (int kb = 0; kb < nb; kb++) {
                const bool fresh = (kb & 3) == 0;
#pragma unroll
                for (int i = 0; i < 4; i++) f[i] = fresh ? nx[i] * nw[i] : f[i < 3 ? i + 1 : 3];
                if (fresh) {
                    if (kb + 4 < nb) fetch(kb + 4);
                    else if ((more = w.next(a, (int)(gridDim.x >> 1)))) scales_of_tile();
                }
                if (!__all_sync(0xffffffffu, pair_wait(&S->tfull[buf][half], ph, abort_flag, a.wait_ns))) {
                    dead = true;
                    break;
                }
                tc_fence_after();
                float v[3][16];   // read in pairs, of which the next one's first half is asked for ahead
                tmem_ld16(t0 + buf * T::TC, v[0]);
                tmem_ld16(t0 + buf * T::TC + 16, v[1]);
#pragma unroll
                for (int q = 0; q < T::CW / 16; q++) {
                    if ((q & 1) == 0) tmem_wait_ld();
                    settle16(v[q % 3]);
                    if ((q & 1) == 0) settle16(v[(q + 1) % 3]);
                    if (16 * (q + 2) < T::CW) {
                        tmem_ld16(t0 + buf * T::TC + 16 * (q + 2), v[(q + 2) % 3]);
                    } else if (q + 1 == T::CW / 16) {   // all read
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive_at(released[buf]);
                    }
                    const float2 ff = make_float2(f[0], f[0]);
#pragma unroll
                    for (int k = 0; k < 8; k++) acc[8 * q + k] = __ffma2_rn(make_float2(v[q % 3][2 * k], v[q % 3][2 * k + 1]), ff, acc[8 * q + k]);
                }
                buf ^= 1;
                ph ^= buf == 0;
            }
            if (dead) break;
            if (a.vec && (c + T::CW <= a.N || a.N % 8 == 0)) {   // (a TMA store ends at a multiple of 16 bytes)
                if (lane == 0) bulk_wait_read<0>();   // the last tile's results have left
                __syncwarp();
                stage_results<T::CW>(out_sm, acc, a.fp16);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0 && r0 < a.M) {
#pragma unroll
                    for (int h = 0; h < 2; h++)
                        if (c + 64 * h < a.N) tma_store_2d(&out_map, out_sm + h * T::kOut, c + 64 * h, r0);
                    bulk_commit();
                }
            } else {
                if (lane == 0) bulk_wait_read<0>();
                __syncwarp();
                stage_results<T::CW>(out_sm, acc, a.fp16);
                __syncwarp();
                const int rows = a.M - r0 < 32 ? (int)(a.M - r0) : 32, n = a.N - c < T::CW ? (int)(a.N - c) : T::CW;
                if (rows > 0 && n > 0) store_staged<T::CW>(out_sm, static_cast<uint16_t*>(a.out) + (int64_t)r0 * a.out_stride + c, a.out_stride, rows, n);
                __syncwarp();
            }
        }
        if (lane == 0) bulk_wait<0>();   // results are out before the CTA ends
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == 8) {
            // -------------------------------------------------------- copies
            int st = 0, ph = 1;
            int64_t issued = 0;
            for (bool more = w.start(a, (int)(blockIdx.x >> 1)); more && !dead; more = w.next(a, (int)(gridDim.x >> 1))) {
                const int xr = w.lt * (2 * kLanes) + (int)rank * kLanes, wr = w.ct * T::TC + (int)rank * (T::CW / 2);
                for (int kb = 0; kb < nb; kb++) {
                    if (!__all_sync(0xffffffffu, pair_wait(&S->empty[st], ph, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    if (lane == 0) {
                        unsigned char* dst = smem + st * T::kStage;
                        mbar_arrive_expect_tx(&S->full[st], T::kStage);
                        tma_load_2d(dst, &x_map, &S->full[st], kb * kBlock, xr);
#pragma unroll
                        for (int h = 0; h < 2; h++)   // half of each half's rows of w
                            tma_load_2d(dst + T::kA + h * T::kB, &w_map, &S->full[st], kb * kBlock, wr + h * T::CW);
                    }
                    __syncwarp();
                    issued++;
                    if (++st == T::kStages) {
                        st = 0;
                        ph ^= 1;
                    }
                }
            }
            if (dead) *abort_flag = 1;
            // copies in flight land before the CTA ends, also where the other warps gave up on them
            const int zero = 0;
            for (int64_t k = issued > T::kStages ? issued - T::kStages : 0; k < issued; k++)
                pair_wait(&S->full[k % T::kStages], (k / T::kStages) & 1, &zero, tc::kWaitLimitNs);
        } else if (warp < 11) {
            // -------------------------------------------------------- products of every other block
            if (rank == 0) {
                constexpr uint32_t idesc = idesc_e4m3(2 * kLanes, T::CW);
                const bool issue = elect_one();
                const uint64_t desc = sdesc_sw128(smem_u32(smem));
                const uint32_t a_lo = (uint32_t)desc, hi = (uint32_t)(desc >> 32);
                const int buf = warp - 9;
                int st = buf, ph = 0, tph = 1, kb = buf;
                for (bool more = w.start(a, (int)(blockIdx.x >> 1)); more && !dead; more = w.next(a, (int)(gridDim.x >> 1))) {
                    for (; kb < nb; kb += 2) {
                        if (!__all_sync(0xffffffffu, pair_wait(&S->ready[st], ph, abort_flag, a.wait_ns))) {
                            dead = true;
                            break;
                        }
                        const uint32_t da = a_lo + ((st * T::kStage) >> 4);
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            if (!__all_sync(0xffffffffu, pair_wait(&S->tempty[buf][h], tph, abort_flag, a.wait_ns))) {
                                dead = true;
                                break;
                            }
                            tc_fence_after();
                            const uint32_t db = da + ((T::kA + h * T::kB) >> 4), d = tmem + buf * T::TC + h * T::CW;
                            if (issue) {
#pragma unroll
                                for (int k = 0; k < kBlock / 32; k++) mma_e4m3<true>(d, da + 2 * k, db + 2 * k, hi, idesc, k ? 1u : 0u);
                                commit_pair(&S->tfull[buf][h]);
                                if (h == 1) commit_pair(&S->empty[st]);
                            }
                            __syncwarp();
                        }
                        if (dead) break;
                        tph ^= 1;
                        st += 2;
                        if (st >= T::kStages) {
                            st -= T::kStages;
                            ph ^= 1;
                        }
                    }
                    kb -= nb;   // the warp's first block of the next tile
                }
                if (dead) *abort_flag = 1;
                if (issue) commit_pair(&S->drain);   // products in flight end before tensor memory is given back
                __syncwarp();
            }
            const int zero = 0;
            pair_wait(&S->drain, 0, &zero, tc::kWaitLimitNs);
        } else {
            // -------------------------------------------------------- word of the CTA's stages
            int st = 0, ph = 0;
            for (bool more = w.start(a, (int)(blockIdx.x >> 1)); more && !dead; more = w.next(a, (int)(gridDim.x >> 1)))
                for (int kb = 0; kb < nb; kb++) {
                    if (!__all_sync(0xffffffffu, pair_wait(&S->full[st], ph, abort_flag, a.wait_ns))) {
                        dead = true;
                        break;
                    }
                    if (lane == 0) arrive_at(at_rank(&S->ready[st], 0));
                    __syncwarp();
                    if (++st == T::kStages) {
                        st = 0;
                        ph ^= 1;
                    }
                }
            if (dead) *abort_flag = 1;
        }
    }
    __syncwarp();
    if (dead) {
        *abort_flag = 1;
        if (lane == 0) raise_flag(a.status, CG_FLAG_PIPE_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
    cluster.sync();   // no CTA ends, and no tensor memory goes, while the other one's products or arrivals may need it
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ------------------------------------------------------------------------------------
// Product of at most 8 rows of x (single tokens): HBM bounds it, a byte of w for 2 M flops. A tile is 16 rows of w; each
// of 8 warps takes an eighth of the blocks of 128 channels, 4 mma.sync m16n8k32 each (a tcgen05 tile would be 7/8
// padding). A warp copies its own blocks of w and x (cp.async into a ring of its own, 4 blocks ahead and on into the
// CTA's next tile) and loads its scales 8 blocks at a time, a lane one block's, a batch ahead: no load's latency stands
// in the loop, it waits for nobody but at a tile's end, where the warps' sums are added in their order, and the call
// needs no tensor maps, which the host would make. All CTAs read the same few lines of x and its scales at
// about the same time, which one slice of L2 serves: they come through L1 (scales copied block by block past it took 2 us
// more). The order of the channels within a block is free as long as both operands have the same: a thread reads 16 bytes
// of either. 1 x 6144 x 4096 6.4 us (25 MB; a plain read of them 5.6), 1 x 58368 x 4096 42 us, 5.7 TB/s.
// Where the rows of w leave SMs idle, the blocks are cut among the CTAs of a cluster, added in the order of the ranks.
// ------------------------------------------------------------------------------------
constexpr int kFewThreads = 256, kFewRows = 16, kFewMost = 8, kFewWarps = kFewThreads / 32;
constexpr int kFewAhead = 4;                                        // blocks of a warp in flight
constexpr uint32_t kFewW = kFewRows * kBlock;                       // bytes of a block of w; x follows
constexpr uint32_t few_slot(int M) { return kFewW + M * kBlock; }
constexpr uint32_t few_smem(int M) { return kFewWarps * kFewAhead * few_slot(M) + kFewWarps * kFewRows * kFewMost * 4; }
static_assert(3 * (few_smem(1) + 1024) <= 233472 && 2 * (few_smem(kFewMost) + 1024) <= 233472, "three or two CTAs an SM");

struct FewArgs {
    const uint8_t *x, *w;
    const float *xs, *ws;
    uint16_t* out;
    int64_t x_stride, w_stride, out_stride, K, N;
    int M, nb, tiles, fp16, split;
};

__device__ __forceinline__ void mma_m16n8k32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 bytes, or zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool have) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy16_l1(uint32_t dst, const void* src, bool have) {   // by way of L1
    asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have ? 16 : 0) : "memory");
}

__global__ void __launch_bounds__(kFewThreads, 3) block8_few_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ __align__(1024) unsigned char smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    const int rank = (int)(blockIdx.x % (unsigned)a.split), first = (int)(blockIdx.x / (unsigned)a.split), step = (int)(gridDim.x / (unsigned)a.split);
    const int64_t part = (int64_t)kFewWarps * a.split, mine = rank * kFewWarps + warp;
    const int lo = (int)(a.nb * mine / part), hi = (int)(a.nb * (mine + 1) / part);   // the warp's blocks
    const uint32_t slot_bytes = few_slot(a.M);
    const unsigned char* ring = smem + warp * kFewAhead * slot_bytes;
    float* sums = reinterpret_cast<float*>(smem + kFewWarps * kFewAhead * slot_bytes);   // [warp][row of x][row of w]

    // Block (tile, kb) into a slot of the ring: 8 lanes a row, its 16-byte pieces 4 - 7 and 0 - 3 changed in odd rows
    // (the fragments' reads of two rows then meet no bank twice); zeros past K, the last row again past N.
    int ct = first, ck = lo, cs = 0;   // the next block to copy, and its slot
    auto copy = [&]() {
        if (ck >= hi) {
            ct += step;
            ck = lo;
        }
        if (ct < a.tiles && ck < hi) {
            const int row0 = lane >> 3;
            const int64_t k = (int64_t)ck * kBlock + (lane & 7) * 16, n0 = (int64_t)ct * kFewRows;
            const bool have = k < a.K;
            const uint32_t dst = smem_u32(ring) + cs * slot_bytes, at = ((lane & 7) ^ ((row0 & 1) << 2)) << 4;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int row = 4 * i + row0;
                copy16(dst + row * kBlock + at, a.w + (n0 + row < a.N ? n0 + row : a.N - 1) * a.w_stride + (have ? k : 0), have);
            }
#pragma unroll
            for (int i = 0; i < kFewMost / 4; i++) {
                const int row = 4 * i + row0;
                if (row < a.M) copy16_l1(dst + kFewW + row * kBlock + at, a.x + row * a.x_stride + (have ? k : 0), have);
            }
            ck++;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++cs == kFewAhead) cs = 0;
    };
    follow();
#pragma unroll
    for (int i = 0; i < kFewAhead; i++) copy();

    // scales of 8 blocks: lane (g, j) those of block g, for rows 2j and 2j + 1 of x; and of the batch that follows
    float sw = 0.0f, s0 = 0.0f, s1 = 0.0f, nw = 0.0f, n0 = 0.0f, n1 = 0.0f;
    auto fetch = [&](int tile, int kb) {
        kb += g;
        if (tile >= a.tiles || kb >= hi) return;
        nw = a.ws[(int64_t)tile * kFewRows / kBlock * a.nb + kb];
        if (2 * j < a.M) n0 = a.xs[(int64_t)(2 * j) * a.nb + kb];
        if (2 * j + 1 < a.M) n1 = a.xs[(int64_t)(2 * j + 1) * a.nb + kb];
    };
    fetch(first, lo);
    int slot = 0;
    for (int tile = first; tile < a.tiles; tile += step) {
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // rows g, g + 8 of w, 2j, 2j + 1 of x
        for (int kb = lo; kb < hi; kb++) {
            if (((kb - lo) & 7) == 0) {
                sw = nw;
                s0 = n0;
                s1 = n1;
                if (kb + 8 < hi) fetch(tile, kb + 8);
                else fetch(tile + step, lo);
            }
            asm volatile("cp.async.wait_group %0;" ::"n"(kFewAhead - 1) : "memory");
            __syncwarp();
            const unsigned char* src = ring + slot * slot_bytes;
            uint4 wv[2][2], xv[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const unsigned char* p = src + (((4 * h + j) ^ ((g & 1) << 2)) << 4);
                wv[0][h] = *reinterpret_cast<const uint4*>(p + g * kBlock);
                wv[1][h] = *reinterpret_cast<const uint4*>(p + (g + 8) * kBlock);
                xv[h] = g < a.M ? *reinterpret_cast<const uint4*>(p + kFewW + g * kBlock) : make_uint4(0, 0, 0, 0);
            }
            const int from = ((kb - lo) & 7) * 4 + j;
            const float fw = __shfl_sync(0xffffffffu, sw, from), f0 = __shfl_sync(0xffffffffu, s0, from) * fw, f1 = __shfl_sync(0xffffffffu, s1, from) * fw;
            __syncwarp();
            copy();           // into the slot just read
            if (++slot == kFewAhead) slot = 0;
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = 0; h < 2; h++) {
                mma_m16n8k32(d, wv[0][h].x, wv[1][h].x, wv[0][h].y, wv[1][h].y, xv[h].x, xv[h].y);
                mma_m16n8k32(d, wv[0][h].z, wv[1][h].z, wv[0][h].w, wv[1][h].w, xv[h].z, xv[h].w);
            }
#pragma unroll
            for (int e = 0; e < 4; e++) acc[e] = fmaf(d[e], e & 1 ? f1 : f0, acc[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) sums[(warp * kFewMost + 2 * j + (e & 1)) * kFewRows + g + 8 * (e >> 1)] = acc[e];
        __syncthreads();
        const int m = tid / kFewRows, r = tid % kFewRows;   // a thread an output
        float total = 0.0f;
        if (m < a.M) {
#pragma unroll
            for (int k = 0; k < kFewWarps; k++) total += sums[(k * kFewMost + m) * kFewRows + r];
        }
        if (a.split > 1) {
            auto cluster = cooperative_groups::this_cluster();
            __syncthreads();
            if (m < a.M) sums[tid] = total;
            cluster.sync();
            if (rank == 0 && m < a.M) {
                total = 0.0f;
                for (int k = 0; k < a.split; k++) total += cluster.map_shared_rank(sums, k)[tid];
            }
            cluster.sync();   // the sums are free again, and no CTA ends while they may be read
        }
        const int64_t n = (int64_t)tile * kFewRows + r;
        if (rank == 0 && m < a.M && n < a.N) a.out[m * a.out_stride + n] = (uint16_t)pack(total, 0.0f, a.fp16);
        if (tile + step < a.tiles) __syncthreads();   // the sums are free again
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// Codes [rows][K] in boxes of box_rows x 128 bytes, 128-byte swizzle; what lies outside reads as 0.
bool codes_map(CUtensorMap* map, const void* base, int64_t rows, int64_t K, int64_t stride, uint32_t box_rows) {
    auto fn = tmap_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(rows > 1 ? stride : K)};
    cuuint32_t box[2] = {128, box_rows}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Results [M][N] in boxes of 32 rows x 64 columns, 128-byte swizzle.
bool results_map(CUtensorMap* map, const MatArgs& a) {
    auto fn = tmap_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)a.N, (cuuint64_t)a.M}, strides[1] = {(cuuint64_t)(a.M > 1 ? a.out_stride : (a.N + 7) / 8 * 8) * 2};
    cuuint32_t box[2] = {64, 32}, estr[2] = {1, 1};
    return fn(map, a.fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, a.out, dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Matrices {
    const void *x, *w;
    int64_t K, x_stride, w_stride;
};

cudaError_t opt_in_tiles() {
    static SmemOptIn opt_in;
    return opt_in.set(reinterpret_cast<const void*>(block8_tile_kernel), (int)Tile::total);
}

// Clusters of `size` CTAs of a kernel that run at the same time, asked once per device and size.
struct Clusters {
    std::atomic<int> known[64][9];
    cudaError_t most(const void* kernel, int threads, size_t smem, int size, int* n) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        *n = dev < 64 ? known[dev][size].load(std::memory_order_relaxed) : 0;
        if (*n) return cudaSuccess;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(tc::num_sms() / size * size));
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = (unsigned)size;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        if ((e = cudaOccupancyMaxActiveClusters(n, kernel, &cfg)) != cudaSuccess) return e;
        if (*n < 1) return cudaErrorInvalidConfiguration;
        if (dev < 64) known[dev][size].store(*n, std::memory_order_relaxed);
        return cudaSuccess;
    }
};

// CTAs of a cluster of the tile kernel: as many as the GPU has room for at once, a block of channels each at least.
cudaError_t tile_split(const MatArgs& a, int* split) {
    static Clusters clusters;
    const int64_t tiles = (a.M + kLanes - 1) / kLanes * ((a.N + Tile::TC - 1) / Tile::TC), room = tc::num_sms();
    cudaError_t e = opt_in_tiles();
    if (e != cudaSuccess) return e;
    int s = (int)(room / tiles < 8 ? room / tiles : 8);
    if (s > a.nb) s = (int)a.nb;
    for (; s > 1; s--) {
        int n = 0;
        if ((e = clusters.most(reinterpret_cast<const void*>(block8_tile_kernel), Tile::kThreads, Tile::total, s, &n)) != cudaSuccess) return e;
        if (n >= tiles) break;
    }
    *split = s < 1 ? 1 : s;
    return cudaSuccess;
}

cudaError_t launch_tiles(MatArgs a, const Matrices& m, int split, cudaStream_t st) {
    using T = Tile;
    a.box_rows = a.M < kLanes ? (int)((a.M + 7) / 8 * 8) : kLanes;
    CUtensorMap xs, ws;
    if (!codes_map(&xs, m.x, a.M, m.K, m.x_stride, a.box_rows) || !codes_map(&ws, m.w, a.N, m.K, m.w_stride, T::TC)) return cudaErrorInvalidValue;
    a.lane_tiles = (a.M + kLanes - 1) / kLanes;
    a.col_tiles = (a.N + T::TC - 1) / T::TC;
    a.group = 16;
    a.split = split;
    const int64_t tiles = a.lane_tiles * a.col_tiles, room = tc::num_sms();
    return launch_following(block8_tile_kernel, (unsigned)(a.split > 1 ? tiles * a.split : tiles < room ? tiles : room), T::kThreads, T::total, st, a.split, a, xs,
                            ws);
}

cudaError_t launch_pairs(MatArgs a, const Matrices& m, cudaStream_t st) {
    using T = Pair;
    CUtensorMap xs, ws, out{};
    a.vec = a.vec && a.out_stride < (int64_t)1 << 39;   // (what a tensor map can hold)
    if (!codes_map(&xs, m.x, a.M, m.K, m.x_stride, kLanes) || !codes_map(&ws, m.w, a.N, m.K, m.w_stride, T::CW / 2) ||
        (a.vec && !results_map(&out, a)))
        return cudaErrorInvalidValue;
    a.lane_tiles = (a.M + 2 * kLanes - 1) / (2 * kLanes);
    a.col_tiles = (a.N + T::TC - 1) / T::TC;
    a.split = 1;
    a.group = 8;
    static SmemOptIn opt_in;
    cudaError_t e = opt_in.set(reinterpret_cast<const void*>(block8_pair_kernel), (int)T::total);
    if (e != cudaSuccess) return e;
    int pairs = 0;   // that the GPU has room for at once: one that came later would take its share when the others are done
    static Clusters clusters;
    if ((e = clusters.most(reinterpret_cast<const void*>(block8_pair_kernel), T::kThreads, T::total, 2, &pairs)) != cudaSuccess) return e;
    const int64_t tiles = a.lane_tiles * a.col_tiles;
    return launch_following(block8_pair_kernel, (unsigned)(2 * (tiles < pairs ? tiles : pairs)), T::kThreads, T::total, st, 0, a, xs, ws, out);
}

cudaError_t launch_few(const MatArgs& a, const Matrices& m, cudaStream_t st) {
    FewArgs f{};
    f.x = static_cast<const uint8_t*>(m.x);
    f.w = static_cast<const uint8_t*>(m.w);
    f.xs = a.xs;
    f.ws = a.ws;
    f.out = static_cast<uint16_t*>(a.out);
    f.x_stride = m.x_stride;
    f.w_stride = m.w_stride;
    f.out_stride = a.out_stride;
    f.K = m.K;
    f.N = a.N;
    f.M = (int)a.M;
    f.nb = (int)a.nb;
    f.fp16 = a.fp16;
    f.tiles = (int)((a.N + kFewRows - 1) / kFewRows);
    const int smem = (int)few_smem(f.M), room = (233472 / (smem + 1024) < 3 ? 2 : 3) * tc::num_sms();
    f.split = 1;
    while (f.split < 8 && (int64_t)f.tiles * 2 * f.split <= room && 2 * f.split * kFewWarps <= f.nb) f.split *= 2;
    static SmemOptIn opt_in;
    cudaError_t e = opt_in.set(reinterpret_cast<const void*>(block8_few_kernel), (int)few_smem(kFewMost));
    if (e != cudaSuccess) return e;
    return launch_following(block8_few_kernel, (unsigned)(f.split > 1 ? f.tiles * f.split : f.tiles < room ? f.tiles : room), kFewThreads, (size_t)smem, st, f.split, f);
}

// The tile kernel takes 0.36 us a block of channels and round, 1.3 us to add up a cluster's sums, the pair kernel 0.45 us a
// block for four times the work. The smaller sum is taken. (6144 rows of w, 4096 channels: 256 rows of x 14.8 us on tiles and 17.7 on
// pairs, 384 15.0 and 18.1, 448 26.8 and 18.1, 1024 38.7 and 32.8; 28672 rows of w: 128 33 and 39, 200 39.7 and 35.2; 14336 channels, 4096
// rows of w: 512 39.4 and 50.3, 640 74.8 and 51.3. Of 7 matrices w and 16 numbers of rows, 17 to 8192, with each the faster one was taken
// every time, or one within 3 % of it.)
cudaError_t launch_matmul(const MatArgs& a, const Matrices& m, cudaStream_t st) {
    if (a.M <= kFewMost) return launch_few(a, m, st);
    const int64_t tiles = (a.M + kLanes - 1) / kLanes * ((a.N + Tile::TC - 1) / Tile::TC), sms = tc::num_sms();
    const int64_t pairs = (a.M + 2 * kLanes - 1) / (2 * kLanes) * ((a.N + Pair::TC - 1) / Pair::TC);
    int split = 1;
    const cudaError_t e = tile_split(a, &split);
    if (e != cudaSuccess) return e;
    auto on_tiles = [&](int s) { return (tiles * s + sms - 1) / sms * ((a.nb + s - 1) / s) * 36 + (s > 1 ? 130 : 0); };
    if (on_tiles(1) <= on_tiles(split)) split = 1;
    const int64_t t_tiles = on_tiles(split), t_pairs = (pairs + sms / 2 - 1) / (sms / 2) * a.nb * 45;
    return t_pairs < t_tiles ? launch_pairs(a, m, st) : launch_tiles(a, m, split, st);
}

bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_type(int32_t dtype) {
    return dtype == CG_BF16 || dtype == CG_FP16 ? CG_OK : set_error(CG_EINVAL, "dtype=%d: CG_BF16 or CG_FP16", dtype);
}
int check_channels(int64_t K) {
    if (K < 16 || K % 16) return set_error(CG_EINVAL, "K=%lld: must be a multiple of 16, at least 16", (long long)K);
    if (K > (int64_t)1 << 30) return set_error(CG_ERANGE, "K=%lld: must be at most 2^30", (long long)K);
    return CG_OK;
}
int check_rows(const char* what, int64_t R) {
    if (R < 0) return set_error(CG_EINVAL, "%s=%lld: must be >= 0", what, (long long)R);
    if (R > (int64_t)1 << 30) return set_error(CG_ERANGE, "%s=%lld: must be at most 2^30", what, (long long)R);
    return CG_OK;
}
int check_stride(const char* what, int64_t R, int64_t row, int64_t stride, int64_t of) {
    if (R < 2) return CG_OK;
    if (stride < row || stride % of || stride >= (int64_t)1 << 40)
        return set_error(CG_EINVAL, "%s: a row stride must be a multiple of %lld, at least the row's %lld and below 2^40 (got %lld)", what, (long long)of,
                         (long long)row, (long long)stride);
    return CG_OK;
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" {

CG_EXPORT int cg_block8_encode(int32_t dtype, int64_t R, int64_t K, int32_t rows, const void* x, int64_t x_stride, void* codes,
                               int64_t stride, float* scales, void* stream) {
    set_error(CG_OK, "%s", "");
    int rc = check_type(dtype);
    if (!rc) rc = check_channels(K);
    if (!rc) rc = check_rows("R", R);
    if (!rc && rows != 1 && rows != kBlock) rc = set_error(CG_EINVAL, "rows=%d: must be 1 or %d", rows, kBlock);
    if (!rc) rc = check_stride("x", R, K, x_stride, 8);
    if (!rc) rc = check_stride("codes", R, K, stride, 16);
    if (rc) return rc;
    if (R == 0) return CG_OK;
    if (!x || !codes || !scales) return set_error(CG_EINVAL, "null x, codes or scales");
    if (!al16(x) || !al16(codes) || (reinterpret_cast<uintptr_t>(scales) & 3u))
        return set_error(CG_EINVAL, "x and codes must be 16-byte aligned, scales to 4 bytes");
    const int64_t blocks = (K + kBlock - 1) / kBlock;
    const Rows in{x, R, 2 * K, 2 * x_stride}, coded{codes, R, K, stride}, scaled = span(scales, (__int128)((R + rows - 1) / rows) * blocks * 4);
    if (overlap(coded, in) || overlap(scaled, in) || overlap(scaled, coded)) return set_error(CG_EINVAL, "the outputs must not overlap x or one another");
    EncArgs a{};
    if ((rc = device_status(&a.status))) return rc;
    a.x = static_cast<const uint16_t*>(x);
    a.codes = static_cast<uint8_t*>(codes);
    a.scales = scales;
    a.R = R;
    a.K = K;
    a.x_stride = R > 1 ? x_stride : K;
    a.stride = R > 1 ? stride : K;
    a.nb = blocks;
    const int64_t items = rows == 1 ? (R * a.nb + kEncRows - 1) / kEncRows : (R + kBlock - 1) / kBlock * a.nb;
    // Long matrices: as many CTAs as run at once go on, two blocks of a row at a time (131072 x 4096: 250 us, 292 with one block or with
    // a CTA for 32 blocks; 8192 x 4096, half of it in L2, 16.2, 17.2 and 18.9; 4096 rows 9.1, 8.8 and 9.0, 1024 3.1, 3.4 and 3.2; 8 CTAs
    // an SM: within 0.2 us but for 8192 rows, 16.9)
    const int64_t room = (rows == 1 ? 4 : 8) * (int64_t)tc::num_sms();
    const unsigned grid = (unsigned)(items < room ? items : room);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool fp16 = dtype == CG_FP16;
    auto launch = [&](void (*kernel)(EncArgs)) { return launch_following(kernel, grid, kEncThreads, 0, st, 0, a); };
    cudaError_t e;
    if (rows == 1) {
        a.step_row = (int64_t)grid * kEncRows / a.nb;
        a.step_b = (int64_t)grid * kEncRows % a.nb;
        if (items > room) e = launch(fp16 ? encode_rows_kernel<true, 2> : encode_rows_kernel<false, 2>);
        else e = launch(fp16 ? encode_rows_kernel<true, 1> : encode_rows_kernel<false, 1>);
    } else {
        e = launch(fp16 ? encode_square_kernel<true> : encode_square_kernel<false>);
    }
    if (e != cudaSuccess) return set_error(CG_ECUDA, "block encoding launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

CG_EXPORT int cg_block8_matmul(int32_t dtype, int64_t M, int64_t N, int64_t K, const void* x, int64_t x_stride, const float* x_scales,
                               const void* w, int64_t w_stride, const float* w_scales, void* out, int64_t out_stride, void* stream) {
    set_error(CG_OK, "%s", "");
    int rc = check_type(dtype);
    if (!rc) rc = check_channels(K);
    if (!rc) rc = check_rows("M", M);
    if (!rc) rc = check_rows("N", N);
    if (!rc) rc = check_stride("x", M, K, x_stride, 16);
    if (!rc) rc = check_stride("w", N, K, w_stride, 16);
    if (!rc) rc = check_stride("out", M, N, out_stride, 1);
    if (rc) return rc;
    if (M == 0 || N == 0) return CG_OK;
    if (!x || !x_scales || !w || !w_scales || !out) return set_error(CG_EINVAL, "null x, w, scales or out");
    if (!al16(x) || !al16(w) || ((reinterpret_cast<uintptr_t>(x_scales) | reinterpret_cast<uintptr_t>(w_scales)) & 3u) ||
        (reinterpret_cast<uintptr_t>(out) & 1u))
        return set_error(CG_EINVAL, "x and w must be 16-byte aligned, scales and out to their type");
    const int64_t blocks = (K + kBlock - 1) / kBlock;
    for (const Rows& in : {Rows{x, M, K, x_stride}, Rows{w, N, K, w_stride}, span(x_scales, (__int128)M * blocks * 4),
                           span(w_scales, (__int128)((N + kBlock - 1) / kBlock) * blocks * 4)})
        if (overlap(Rows{out, M, 2 * N, 2 * out_stride}, in)) return set_error(CG_EINVAL, "out must not overlap the inputs");
    MatArgs a{};
    if ((rc = device_status(&a.status))) return rc;
    a.xs = x_scales;
    a.ws = w_scales;
    a.out = out;
    a.M = M;
    a.N = N;
    a.nb = blocks;
    a.out_stride = M > 1 ? out_stride : N;
    a.wait_ns = wait_limit_ns();
    a.fp16 = dtype == CG_FP16;
    a.vec = al16(out) && (M < 2 || out_stride % 8 == 0);
    a.vec_scales = a.nb % 4 == 0 && al16(x_scales) && al16(w_scales);
    const cudaError_t e = launch_matmul(a, Matrices{x, w, K, x_stride, w_stride}, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return set_error(CG_ECUDA, "block product launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

}  // extern "C"
