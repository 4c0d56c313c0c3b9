// cg_paged.cu -- the paged cache's bookkeeping and what fills it: page plan and release (block
// tables, positions and slots from lengths), and rotary positions with the append into the pages.
// Contract: include/codecgauge_paged.h.
#include <cmath>

#include "cg_paged.h"
#include "cg_paged_pages.cuh"

#define CG_EXPORT __attribute__((visibility("default")))

namespace cg {
namespace {

// ------------------------------------------------------------------------------------
// Page plan. Two prefix sums over the requests (new tokens, fresh pages) and an expansion: every
// token and every fresh page finds its request by binary search in the prefix. All in one launch:
// each CTA takes a range of tokens and a range of fresh pages and runs the prefix itself, 2048
// requests at a time in shared memory, so nothing has to be exchanged between CTAs; it stops as
// soon as the prefix has passed its ranges. Bound: launch latency and one chain of dependent
// loads (lengths -> table entry) at decode sizes; the stores of 12 bytes per token at prompt sizes.
// ------------------------------------------------------------------------------------
constexpr int kPT = 256;         // threads
constexpr int kRound = 2048;     // requests per round
constexpr int kTokCta = 1024;    // tokens per CTA: 4 per thread (16- and 32-byte stores)

struct PlanArgs {
    const int32_t *ctx, *add, *free_in, *count_in;
    int32_t *table, *lens_out, *cu, *pos, *count_out;
    int64_t* slots;
    int32_t* status;
    int n_tok, n_pages, n_stack, page, page_log2, n_req, max_pages;
    int64_t pages_per_cta;
};

struct PlanSmem {
    int32_t tok[kRound + 1];   // first token of each request of the round (saturated)
    int32_t fresh[kRound + 1]; // first page item of each request of the round (saturated)
    int32_t ctx[kRound];       // tokens held
    int64_t warp_tok[kPT / 32], warp_page[kPT / 32];
};

__device__ __forceinline__ int32_t sat32(int64_t v) { return v > 0x7fffffff ? 0x7fffffff : (int32_t)v; }

// One request's tokens held, new tokens, and the pages that these need beyond those it has.
__device__ __forceinline__ void plan_request(const PlanArgs& a, int i, int64_t* ctx, int64_t* add, int64_t* items,
                                             int32_t* flag) {
    int64_t c = __ldg(a.ctx + i), n = __ldg(a.add + i);
    if (c < 0) {
        c = 0;
        *flag |= CG_FLAG_PAGED_RANGE;
    }
    if (n < 0 || n > a.n_tok) {
        n = 0;
        *flag |= CG_FLAG_PAGED_RANGE;
    }
    int64_t have = (c + a.page - 1) >> a.page_log2, want = (c + n + a.page - 1) >> a.page_log2;
    if (want > a.max_pages) {
        *flag |= CG_FLAG_PAGED_RANGE;
        want = a.max_pages;
        if (have > want) have = want;
    }
    *ctx = c;
    *add = n;
    *items = want - have;
}

// Entry k of the free stack counted from the top, or -1.
__device__ __forceinline__ int32_t take_page(const PlanArgs& a, int64_t count, int64_t k, int32_t* flag) {
    if (k >= count) {
        *flag |= CG_FLAG_PAGES_EXHAUSTED;
        return -1;
    }
    const int32_t id = __ldg(a.free_in + (count - 1 - k));
    if (id < 0 || id >= a.n_pages) {
        *flag |= CG_FLAG_PAGED_RANGE;
        return -1;
    }
    return id;
}

__global__ void __launch_bounds__(kPT) plan_kernel(PlanArgs a) {
    __shared__ PlanSmem S;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t flag = 0;
    const int64_t t_lo = (int64_t)blockIdx.x * kTokCta;
    const int64_t t_hi = t_lo + kTokCta < a.n_tok ? t_lo + kTokCta : a.n_tok;
    const bool last_cta = blockIdx.x == gridDim.x - 1;
    const int64_t f_lo = (int64_t)blockIdx.x * a.pages_per_cta;
    // A plan whose tokens fit n_tok needs no more pages than tokens. Wrong lengths can ask for any number:
    // those past this limit are not dealt out (the prefix in shared memory is right below 2^31 - 1 only).
    const int64_t most = (int64_t)a.n_tok + a.n_req < 0x7fffffff ? (int64_t)a.n_tok + a.n_req : 0x7fffffff;
    const int64_t f_hi = last_cta || f_lo + a.pages_per_cta > most ? most : f_lo + a.pages_per_cta;
    int64_t count = __ldg(a.count_in);
    if (count < 0 || count > a.n_stack) {
        flag |= CG_FLAG_PAGED_RANGE;
        count = count < 0 ? 0 : a.n_stack;
    }

    int64_t tok_base = 0, page_base = 0;   // prefix at the start of the round
    int round = 0;
    for (int base = 0; base < a.n_req; base += kRound, round++) {
        const int n = a.n_req - base < kRound ? a.n_req - base : kRound;
        const int per = (n + kPT - 1) / kPT;   // consecutive requests per thread
        int64_t nt[kRound / kPT], np[kRound / kPT], cx[kRound / kPT], st = 0, sp = 0;
#pragma unroll
        for (int k = 0; k < kRound / kPT; k++) {
            const int i = tid * per + k;
            nt[k] = np[k] = cx[k] = 0;
            if (k < per && i < n) plan_request(a, base + i, &cx[k], &nt[k], &np[k], &flag);
            st += nt[k];
            sp += np[k];
        }
        int64_t it = st, ip = sp;   // inclusive over the warp, then over the CTA
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            const int64_t u = __shfl_up_sync(0xffffffffu, it, off), v = __shfl_up_sync(0xffffffffu, ip, off);
            if (lane >= off) {
                it += u;
                ip += v;
            }
        }
        if (lane == 31) {
            S.warp_tok[warp] = it;
            S.warp_page[warp] = ip;
        }
        __syncthreads();
        int64_t et = tok_base + it - st, ep = page_base + ip - sp, total_t = tok_base, total_p = page_base;
#pragma unroll
        for (int w = 0; w < kPT / 32; w++) {
            if (w < warp) {
                et += S.warp_tok[w];
                ep += S.warp_page[w];
            }
            total_t += S.warp_tok[w];
            total_p += S.warp_page[w];
        }
        const bool writer = (int)(round % gridDim.x) == (int)blockIdx.x;   // of the per-request outputs
#pragma unroll
        for (int k = 0; k < kRound / kPT; k++) {
            const int i = tid * per + k;
            if (k < per && i < n) {
                S.tok[i] = sat32(et);
                S.fresh[i] = sat32(ep);
                S.ctx[i] = (int32_t)cx[k];
                if (writer) {
                    a.lens_out[base + i] = sat32(cx[k] + nt[k]);
                    a.cu[base + i] = sat32(et);
                    if (base + i == a.n_req - 1) a.cu[a.n_req] = sat32(et + nt[k]);
                }
                et += nt[k];
                ep += np[k];
            }
        }
        if (tid == 0) {
            S.tok[n] = sat32(total_t);
            S.fresh[n] = sat32(total_p);
        }
        __syncthreads();

        // page items of this pass in the CTA's range
        {
            const int64_t lo = f_lo > page_base ? f_lo : page_base, hi = f_hi < total_p ? f_hi : total_p;
            for (int64_t f = lo + tid; f < hi; f += kPT) {
                const int r = find_request(S.fresh, n, (int32_t)f);
                const int64_t row = (int64_t)(base + r) * a.max_pages, have = ((int64_t)S.ctx[r] + a.page - 1) >> a.page_log2;
                a.table[row + have + (f - S.fresh[r])] = take_page(a, count, f, &flag);
            }
        }
        // tokens of this pass in the CTA's range, four in a row per thread
        {
            const int64_t t0 = t_lo + tid * 4;
            if (t0 + 3 >= tok_base && t0 < total_t && t0 < t_hi) {
                int r = -1;
                int32_t pos[4];
                int64_t slot[4];
                bool have_t[4];
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const int64_t t = t0 + k;
                    pos[k] = 0;
                    slot[k] = -1;
                    have_t[k] = t >= tok_base && t < total_t && t < t_hi;
                    if (!have_t[k]) continue;
                    if (r < 0) r = find_request(S.tok, n, (int32_t)t);
                    while (S.tok[r + 1] <= t) r++;
                    const int64_t ctx = S.ctx[r], p = ctx + (t - S.tok[r]);
                    pos[k] = sat32(p);
                    const int64_t pg = p >> a.page_log2, have = (ctx + a.page - 1) >> a.page_log2;
                    int32_t id = -1;
                    if (pg < a.max_pages) {
                        if (pg >= have) {
                            id = take_page(a, count, S.fresh[r] + (pg - have), &flag);
                        } else {
                            id = a.table[(int64_t)(base + r) * a.max_pages + pg];
                            if (id < 0 || id >= a.n_pages) {
                                flag |= CG_FLAG_PAGED_RANGE;
                                id = -1;
                            }
                        }
                    }
                    if (id >= 0) slot[k] = (int64_t)id * a.page + (p & (a.page - 1));
                }
                if (have_t[0] && have_t[3]) {
                    *reinterpret_cast<int4*>(a.pos + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
                    longlong2* s2 = reinterpret_cast<longlong2*>(a.slots + t0);
                    s2[0] = make_longlong2(slot[0], slot[1]);
                    s2[1] = make_longlong2(slot[2], slot[3]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        if (have_t[k]) {
                            a.pos[t0 + k] = pos[k];
                            a.slots[t0 + k] = slot[k];
                        }
                }
            }
        }
        tok_base = total_t;
        page_base = total_p;
        __syncthreads();   // the round's prefixes are free again
        if (blockIdx.x != 0 && tok_base >= t_hi && page_base >= f_hi) {
            // nothing of the CTA's ranges is left; a later round that it writes the outputs of may be
            bool more = false;
            for (int rr = round + 1; rr * kRound < a.n_req; rr++) more |= (int)(rr % gridDim.x) == (int)blockIdx.x;
            if (!more) break;
        }
    }
    // padding past the last token (a CTA that left the loop early has none)
    for (int64_t t = (t_lo > tok_base ? t_lo : tok_base) + tid; t < t_hi; t += kPT) {
        a.pos[t] = 0;
        a.slots[t] = -1;
    }
    if (blockIdx.x == 0 && tid == 0) {
        const int64_t left = count - page_base;
        *a.count_out = (int32_t)(left < -0x7fffffff ? -0x7fffffff : left);
        if (tok_base > a.n_tok) flag |= CG_FLAG_PAGED_RANGE;
        if (left < 0) flag |= CG_FLAG_PAGES_EXHAUSTED;
    }
    raise_flag(a.status, flag);
}

// ------------------------------------------------------------------------------------
// Page release: the entries of the finished requests go on the stack (push_pages). Bound: launch latency and
// chains of dependent loads (length, entry). In a graph: 8 of 256 requests of 128 pages 5.8 us, all of them
// (32768 pages) 6.5, 102400 pages 18.4, 400 of 4096 requests 8.1.
// ------------------------------------------------------------------------------------
constexpr int kRelThreads = 1024;

struct ReleaseArgs {
    const int32_t *lens, *done;
    int32_t *lens_left, *status;
    int page, page_log2;
    PushArgs push;
};

// A finished request gives all its entries.
struct Finished {
    static constexpr bool kFromStart = true;
    const ReleaseArgs& a;
    int rank;
    __device__ __forceinline__ void prepare(int, int) const {}
    __device__ __forceinline__ int64_t entries(int i, int, int*, int32_t* flag) const {
        int64_t c = __ldg(a.lens + i);
        const bool done = __ldg(a.done + i) != 0;
        int64_t have = (c + a.page - 1) >> a.page_log2;
        if (c < 0) {
            c = have = 0;
            *flag |= CG_FLAG_PAGED_RANGE;
        }
        if (have > a.push.max_pages) {
            have = a.push.max_pages;
            *flag |= CG_FLAG_PAGED_RANGE;
        }
        if (rank == 0) a.lens_left[i] = done ? 0 : (int32_t)c;
        return done ? have : 0;
    }
};

__global__ void __cluster_dims__(kPushCtas, 1, 1) __launch_bounds__(kRelThreads) release_kernel(ReleaseArgs a) {
    __shared__ PushSmem<kRelThreads, true> S;
    int32_t flag = 0;
    push_pages<kRelThreads>(a.push, S, Finished{a, (int)cooperative_groups::this_cluster().block_rank()}, &flag);
    raise_flag(a.status, flag);
}

// ------------------------------------------------------------------------------------
// Rotary. A CTA takes a few tokens: first the cosine and sine of every pair of each token, once, into
// shared memory, then the heads. A unit of work is two 16-byte pieces (8 channels each) of two heads of
// a token, at channels 8c and rot / 2 + 8c: for the half layout these are the two sides of 8 pairs, for
// the interleaved layout 4 pairs each, so both layouts load and store whole 128-byte lines. The next
// unit's loads are issued ahead of a unit's stores, the first unit's ahead of the cosines. Past rot the
// pieces are copied; value heads are copied whole. Bound: HBM (every byte is read once and written
// once). A 16384-token prompt, 32 + 8 + 8 heads of 128, 403 MB: 66.6 us, 6.05 TB/s; with the cosines and
// sines computed by every thread for the heads that it turns, 68 us (two heads a thread), 70 (four) and
// 103 (one: the arithmetic then bounds it). 193 decode tokens: 12.5 us, most of it the call's latency.
// The angle is exact modulo a turn: position times the frequency in 2^-64 of a turn, in integers.
// ------------------------------------------------------------------------------------
struct RotArgs {
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *pool;      // pool null: no append, K and V absent
    const int32_t* pos;
    const int64_t* slots;
    const int64_t* table;
    int32_t* status;
    int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;
    int64_t n_slots, v_half;     // slots of the pool; elements from the key to the value half
    int n_tok, q_heads, H, d, rot, page, page_log2, transpose;
    int turn_groups, groups;     // pairs of heads that turn, and of all heads, per token
    int tokens;                  // of a CTA
    float mscale;
};

template <bool FP16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
    if (FP16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

template <bool FP16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
    if (FP16) {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&b);
}

constexpr int kRotThreads = 128, kRotTokens = 2;

template <bool FP16, bool INTER>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(RotArgs a) {
    extern __shared__ __align__(16) float2 turns_sm[];            // [tokens][rot / 2] (cosine, sine) x mscale
    const int C = a.d >> 4, tid = threadIdx.x;                    // C units along a pair of heads
    const int64_t tok0 = (int64_t)blockIdx.x * a.tokens;
    const int n_tok = a.n_tok - tok0 < a.tokens ? (int)(a.n_tok - tok0) : a.tokens;
    const int units = n_tok * a.groups * C, pairs = a.rot >> 1;
    const int64_t head_step = (int64_t)a.page * a.d;

    struct Unit {
        int t, c, o0, o1, head0;
        bool is_v, turns;
        uint4 x0[2], x1[2];
    };
    auto heads_of = [&](const Unit& u) { return u.is_v ? a.H : a.q_heads + a.H; };
    auto load = [&](int i, Unit& u) {
        if (i >= units) return;
        u.c = i & (C - 1);
        const int g = i / C;
        u.t = g / a.groups;
        const int grp = g - u.t * a.groups;
        u.is_v = grp >= a.turn_groups;
        u.turns = !u.is_v && u.c < (a.rot >> 4);
        u.o0 = u.turns || u.is_v ? 8 * u.c : a.rot + 16 * (u.c - (a.rot >> 4));
        u.o1 = u.turns ? (a.rot >> 1) + 8 * u.c : u.is_v ? (a.d >> 1) + 8 * u.c : u.o0 + 8;
        u.head0 = (u.is_v ? grp - a.turn_groups : grp) * 2;
        const int64_t tok = tok0 + u.t;
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int h = u.head0 + k;
            if (h < heads_of(u)) {
                const uint16_t* src = u.is_v ? a.v + tok * a.v_tok + h * a.v_head
                                      : h < a.q_heads ? a.q + tok * a.q_tok + h * a.q_head
                                                      : a.k + tok * a.k_tok + (h - a.q_heads) * a.k_head;
                u.x0[k] = *reinterpret_cast<const uint4*>(src + u.o0);
                u.x1[k] = *reinterpret_cast<const uint4*>(src + u.o1);
            }
        }
    };
    Unit now;
    load(tid, now);

    for (int i = tid; i < n_tok * pairs; i += kRotThreads) {
        const int t = i / pairs, pair = i - t * pairs;
        const int64_t p = __ldg(a.pos + tok0 + t);
        const uint64_t turn = (uint64_t)p * (uint64_t)__ldg(a.table + pair);
        const float f = (float)(int32_t)(turn >> 32) * 0x1p-31f;   // half turns, in [-1, 1]
        float sn, cs;
        sincospif(f, &sn, &cs);
        turns_sm[i] = make_float2(cs * a.mscale, a.transpose ? -sn * a.mscale : sn * a.mscale);
    }
    __syncthreads();

    for (int i = tid; i < units; i += kRotThreads) {
        Unit next;
        load(i + kRotThreads, next);
        int64_t dst0 = -1;   // element of the token's slot in the key half, head 0
        if (a.pool && now.head0 + 2 > (now.is_v ? 0 : a.q_heads)) {
            const int64_t slot = __ldg(a.slots + tok0 + now.t);
            if (slot >= 0 && slot < a.n_slots)
                dst0 = (((slot >> a.page_log2) * a.H << a.page_log2) + (slot & (a.page - 1))) * a.d;
            else if (slot != -1 && now.c == 0)
                raise_flag(a.status, CG_FLAG_PAGED_RANGE);
        }
        float cs[8], sn[8];
        if (now.turns) {
            // pairs of the pieces: 8 from 8c, or 4 each from o0 / 2 and o1 / 2
            const float2* row = turns_sm + now.t * pairs;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float4 v = *reinterpret_cast<const float4*>(row + (INTER ? ((e < 4 ? now.o0 : now.o1) >> 1) + (e & 3) : 8 * now.c + e));
                cs[e] = v.x;
                sn[e] = v.y;
                cs[e + 1] = v.z;
                sn[e + 1] = v.w;
            }
        }
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int h = now.head0 + k;
            if (h >= heads_of(now)) break;
            if (now.turns) {
                uint32_t u[4] = {now.x0[k].x, now.x0[k].y, now.x0[k].z, now.x0[k].w}, v[4] = {now.x1[k].x, now.x1[k].y, now.x1[k].z, now.x1[k].w};
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const float2 f = unpack2<FP16>(u[e]), g = unpack2<FP16>(v[e]);
                    if (INTER) {   // pairs (f.x, f.y) and (g.x, g.y)
                        u[e] = pack2<FP16>(f.x * cs[e] - f.y * sn[e], f.y * cs[e] + f.x * sn[e]);
                        v[e] = pack2<FP16>(g.x * cs[4 + e] - g.y * sn[4 + e], g.y * cs[4 + e] + g.x * sn[4 + e]);
                    } else {       // pairs (f.x, g.x) and (f.y, g.y)
                        const int i0 = 2 * e, i1 = 2 * e + 1;
                        u[e] = pack2<FP16>(f.x * cs[i0] - g.x * sn[i0], f.y * cs[i1] - g.y * sn[i1]);
                        v[e] = pack2<FP16>(g.x * cs[i0] + f.x * sn[i0], g.y * cs[i1] + f.y * sn[i1]);
                    }
                }
                now.x0[k] = make_uint4(u[0], u[1], u[2], u[3]);
                now.x1[k] = make_uint4(v[0], v[1], v[2], v[3]);
            }
            uint16_t* dst = nullptr;
            if (!now.is_v && h < a.q_heads) dst = a.q_out + (tok0 + now.t) * a.o_tok + h * a.o_head;
            else if (dst0 >= 0) dst = a.pool + dst0 + (now.is_v ? a.v_half + h * head_step : (h - a.q_heads) * head_step);
            if (dst) {
                *reinterpret_cast<uint4*>(dst + now.o0) = now.x0[k];
                *reinterpret_cast<uint4*>(dst + now.o1) = now.x1[k];
            }
        }
        now = next;
    }
}

cudaError_t launch_rotary(RotArgs a, bool fp16, bool inter, cudaStream_t st) {
    a.turn_groups = (a.q_heads + a.H + 1) / 2;
    a.groups = a.turn_groups + (a.pool ? (a.H + 1) / 2 : 0);
    // Two tokens a CTA where that leaves no SM idle: 16384 tokens take 66.6 us with two, 66.1 with four and
    // 68 with 256 threads and four; 4000 tokens 21.1, 22.8 and 22.8. One token a CTA below: 193 tokens take
    // 12.5 us, 13.1 with more a CTA.
    a.tokens = a.n_tok >= kRotTokens * 1024 ? kRotTokens : 1;
    const unsigned grid = (unsigned)(((int64_t)a.n_tok + a.tokens - 1) / a.tokens);
    const size_t smem = (size_t)a.tokens * (a.rot >> 1) * sizeof(float2);
    if (fp16) {
        if (inter) rotary_kernel<true, true><<<grid, kRotThreads, smem, st>>>(a);
        else rotary_kernel<true, false><<<grid, kRotThreads, smem, st>>>(a);
    } else {
        if (inter) rotary_kernel<false, true><<<grid, kRotThreads, smem, st>>>(a);
        else rotary_kernel<false, false><<<grid, kRotThreads, smem, st>>>(a);
    }
    return cudaGetLastError();
}

bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool al8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
bool al4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int log2_of(int v) {
    int k = 0;
    while ((1 << k) < v) k++;
    return k;
}

// Geometry shared by every paged entry point; `heads` also checks the fields of the vectors.
int check_pages(const cg_pages* p, bool heads) {
    if (!p) return set_error(CG_EINVAL, "null pages");
    if (!(p->page == 16 || p->page == 32 || p->page == 64 || p->page == 128 || p->page == 256))
        return set_error(CG_EINVAL, "page=%d: tokens per page must be 16, 32, 64, 128 or 256", p->page);
    if (p->n_pages < 1) return set_error(CG_EINVAL, "n_pages=%d: must be >= 1", p->n_pages);
    if ((int64_t)p->n_pages * p->page > 0x7fffffff)
        return set_error(CG_ERANGE, "n_pages * page = %lld: must be below 2^31", (long long)p->n_pages * p->page);
    if (!heads) return CG_OK;
    if (p->dtype != CG_BF16 && p->dtype != CG_FP16) return set_error(CG_EINVAL, "dtype=%d: CG_BF16 or CG_FP16", p->dtype);
    if (p->H < 1 || p->H > 1024) return set_error(CG_EINVAL, "H=%d: KV heads must be 1 .. 1024", p->H);
    if (!(p->d == 64 || p->d == 128 || p->d == 256))
        return set_error(CG_EUNSUPPORTED, "head dim d=%d: the paged operators support 64, 128 and 256", p->d);
    return CG_OK;
}

int check_table(const cg_pages* p) {
    if (p->n_req < 1 || p->n_req > 65536) return set_error(CG_EINVAL, "n_req=%d: must be 1 .. 65536", p->n_req);
    if (p->max_pages < 1) return set_error(CG_EINVAL, "max_pages=%d: must be >= 1", p->max_pages);
    if ((int64_t)p->max_pages * p->page > 0x7fffffff) return set_error(CG_ERANGE, "max_pages * page must be below 2^31");
    return CG_OK;
}

int check_rotary(const cg_rotary_params* r, int d, const void* table) {
    if (!r) return set_error(CG_EINVAL, "null rotary parameters");
    if (r->rot < 0 || r->rot > d || r->rot % 16)
        return set_error(CG_EINVAL, "rot=%d: must be a multiple of 16 from 0 to d=%d", r->rot, d);
    if (!std::isfinite(r->mscale)) return set_error(CG_EINVAL, "mscale must be finite");
    if (r->rot && (!table || !al8(table))) return set_error(CG_EINVAL, "null or misaligned rotary table");
    return CG_OK;
}

bool stride8(int64_t s) { return s >= 0 && s % 8 == 0; }

// Rows of an output on one another: a stride of 0 over more than one element.
int check_output(int64_t n_tok, int64_t tok, int64_t heads, int64_t head) {
    if ((n_tok > 1 && heads > 0 && tok == 0) || (heads > 1 && n_tok > 0 && head == 0))
        return set_error(CG_EINVAL, "an output stride is 0: rows of the output would lie on one another");
    return CG_OK;
}

int check_units(int64_t n_tok, int64_t heads, int d) {
    if (n_tok * heads * (d >> 4) > ((int64_t)1 << 31) * 8)
        return set_error(CG_ERANGE, "n_tok * heads is too large for one call");
    return CG_OK;
}

}  // namespace

int paged_check_output(int64_t n_tok, int64_t tok, int64_t heads, int64_t head) { return check_output(n_tok, tok, heads, head); }

int paged_check_sizes(const cg_pages* p) {
    int rc = check_pages(p, false);
    return rc ? rc : check_table(p);
}

int paged_check(const cg_pages* p) {
    int rc = check_pages(p, true);
    return rc ? rc : check_table(p);
}

}  // namespace cg

using namespace cg;

extern "C" {

CG_EXPORT int cg_page_plan(const cg_pages* pages, int32_t n_tok, const int32_t* ctx_lens, const int32_t* new_lens,
                           const int32_t* free_pages, const int32_t* free_count, int32_t* block_table,
                           int32_t* seq_lens, int32_t* cu_new, int32_t* positions, int64_t* slots,
                           int32_t* free_left, void* stream) {
    set_error(CG_OK, "%s", "");
    if (!free_pages) return set_error(CG_EINVAL, "null pointer");
    return cg_page_plan_stack(pages, n_tok, ctx_lens, new_lens, free_pages, pages ? pages->n_pages : 0, free_count, block_table,
                              seq_lens, cu_new, positions, slots, free_left, stream);
}

CG_EXPORT int cg_page_plan_stack(const cg_pages* pages, int32_t n_tok, const int32_t* ctx_lens, const int32_t* new_lens,
                                 const int32_t* free_pages, int32_t n_stack, const int32_t* free_count,
                                 int32_t* block_table, int32_t* seq_lens, int32_t* cu_new, int32_t* positions,
                                 int64_t* slots, int32_t* free_left, void* stream) {
    set_error(CG_OK, "%s", "");
    int rc = check_pages(pages, false);
    if (!rc) rc = check_table(pages);
    if (rc) return rc;
    if (n_tok < 0) return set_error(CG_EINVAL, "n_tok=%d: must be >= 0", n_tok);
    if (n_stack < 0) return set_error(CG_EINVAL, "n_stack=%d: must be >= 0", n_stack);
    if (!ctx_lens || !new_lens || (n_stack && !free_pages) || !free_count || !block_table || !seq_lens || !cu_new || !free_left)
        return set_error(CG_EINVAL, "null pointer");
    if (n_tok && (!positions || !slots)) return set_error(CG_EINVAL, "null positions or slots");
    if (!al16(positions) || !al16(slots)) return set_error(CG_EINVAL, "positions and slots must be 16-byte aligned");
    if (!al4(ctx_lens) || !al4(new_lens) || !al4(free_pages) || !al4(free_count) || !al4(block_table) ||
        !al4(seq_lens) || !al4(cu_new) || !al4(free_left))
        return set_error(CG_EINVAL, "pointers must be aligned to their type");
    if (seq_lens == ctx_lens || seq_lens == new_lens || free_left == free_count)
        return set_error(CG_EINVAL, "seq_lens and free_left must not alias the inputs");
    PlanArgs a{};
    if ((rc = device_status(&a.status))) return rc;
    a.ctx = ctx_lens;
    a.add = new_lens;
    a.free_in = free_pages;
    a.count_in = free_count;
    a.table = block_table;
    a.lens_out = seq_lens;
    a.cu = cu_new;
    a.pos = positions;
    a.slots = slots;
    a.count_out = free_left;
    a.n_tok = n_tok;
    a.n_pages = pages->n_pages;
    a.n_stack = n_stack < pages->n_pages ? n_stack : pages->n_pages;
    a.page = pages->page;
    a.page_log2 = log2_of(pages->page);
    a.n_req = pages->n_req;
    a.max_pages = pages->max_pages;
    const int64_t grid = n_tok ? (n_tok + (int64_t)kTokCta - 1) / kTokCta : 1;
    a.pages_per_cta = ((int64_t)n_tok / pages->page + pages->n_req) / grid + 1;
    plan_kernel<<<(unsigned)grid, kPT, 0, static_cast<cudaStream_t>(stream)>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return set_error(CG_ECUDA, "page plan launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

CG_EXPORT int cg_page_release(const cg_pages* pages, const int32_t* lens, const int32_t* done,
                              const int32_t* block_table, int32_t* free_pages, const int32_t* free_count,
                              int32_t* lens_left, int32_t* free_left, void* stream) {
    set_error(CG_OK, "%s", "");
    int rc = check_pages(pages, false);
    if (!rc) rc = check_table(pages);
    if (rc) return rc;
    if (!lens || !done || !block_table || !free_pages || !free_count || !lens_left || !free_left)
        return set_error(CG_EINVAL, "null pointer");
    if (!al4(lens) || !al4(done) || !al4(block_table) || !al4(free_pages) || !al4(free_count) || !al4(lens_left) ||
        !al4(free_left))
        return set_error(CG_EINVAL, "pointers must be aligned to their type");
    if (lens_left == lens || lens_left == done || free_left == free_count)
        return set_error(CG_EINVAL, "lens_left and free_left must not alias the inputs");
    ReleaseArgs a{};
    if ((rc = device_status(&a.status))) return rc;
    a.lens = lens;
    a.done = done;
    a.lens_left = lens_left;
    a.page = pages->page;
    a.page_log2 = log2_of(pages->page);
    a.push = PushArgs{block_table, free_count, free_pages, free_left, pages->n_pages, pages->n_req, pages->max_pages};
    release_kernel<<<kPushCtas, kRelThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return set_error(CG_ECUDA, "page release launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

CG_EXPORT int cg_rotary_table(int32_t rot, const cg_rope_scaling* s, int64_t* host_table, float* mscale) {
    set_error(CG_OK, "%s", "");
    if (!s || !host_table || !mscale) return set_error(CG_EINVAL, "null pointer");
    if (rot < 16 || rot % 16 || rot > 256) return set_error(CG_EINVAL, "rot=%d: must be a multiple of 16 from 16 to 256", rot);
    if (!(s->base > 1.0) || !std::isfinite(s->base)) return set_error(CG_EINVAL, "base must be finite and above 1");
    if (s->kind < CG_ROPE_NONE || s->kind > CG_ROPE_YARN) return set_error(CG_EINVAL, "unknown scaling kind %d", s->kind);
    if (s->kind != CG_ROPE_NONE && !(s->factor > 0.0 && std::isfinite(s->factor)))
        return set_error(CG_EINVAL, "factor must be finite and positive");
    const bool ramp = s->kind == CG_ROPE_BANDS || s->kind == CG_ROPE_YARN;
    if (ramp && !(s->original > 0.0 && std::isfinite(s->original) && s->low > 0.0 && s->high > s->low &&
                  std::isfinite(s->high)))
        return set_error(CG_EINVAL, "original must be positive and 0 < low < high");
    const double kTwoPi = 6.283185307179586476925286766559;
    auto at = [&](double turns) { return rot * std::log(s->original / (turns * kTwoPi)) / (2.0 * std::log(s->base)); };
    const double lo = s->kind == CG_ROPE_YARN ? std::fmax(std::floor(at(s->high)), 0.0) : 0.0;
    const double hi = s->kind == CG_ROPE_YARN ? std::fmin(std::ceil(at(s->low)), rot - 1.0) : 0.0;
    for (int c = 0; c < rot / 2; c++) {
        double f = std::pow(s->base, -2.0 * c / rot);
        if (s->kind == CG_ROPE_LINEAR) {
            f /= s->factor;
        } else if (ramp) {
            double t;
            if (s->kind == CG_ROPE_BANDS) t = (s->original * f / kTwoPi - s->low) / (s->high - s->low);
            else t = 1.0 - std::fmin(std::fmax((c - lo) / std::fmax(hi - lo, 1e-3), 0.0), 1.0);
            t = std::fmin(std::fmax(t, 0.0), 1.0);
            f = (1.0 - t) * f / s->factor + t * f;
        }
        double turns = f / kTwoPi;
        turns -= std::floor(turns);                       // whole turns do not count
        const double scaled = std::rint(std::ldexp(turns, 64));
        // a fraction that rounds up to a whole turn is none
        host_table[c] = scaled >= 18446744073709551616.0 ? 0 : (int64_t)(uint64_t)scaled;
    }
    *mscale = s->kind == CG_ROPE_YARN && s->factor > 1.0 ? (float)(0.1 * std::log(s->factor) + 1.0) : 1.0f;
    return CG_OK;
}

CG_EXPORT int cg_rotary(const cg_rotary_params* rotary, int32_t dtype, int32_t n_tok, int32_t heads, int32_t d,
                        const void* x, int64_t x_tok, int64_t x_head, const int32_t* positions, const int64_t* table,
                        void* out, int64_t out_tok, int64_t out_head, void* stream) {
    set_error(CG_OK, "%s", "");
    if (dtype != CG_BF16 && dtype != CG_FP16) return set_error(CG_EINVAL, "dtype=%d: CG_BF16 or CG_FP16", dtype);
    if (!(d == 64 || d == 128 || d == 256)) return set_error(CG_EUNSUPPORTED, "head dim d=%d: 64, 128 and 256 are supported", d);
    if (n_tok < 0 || heads < 0 || heads > 65536) return set_error(CG_EINVAL, "n_tok=%d, heads=%d out of range", n_tok, heads);
    int rc = check_rotary(rotary, d, table);
    if (!rc) rc = check_units(n_tok, heads, d);
    if (rc) return rc;
    if (!stride8(x_tok) || !stride8(x_head) || !stride8(out_tok) || !stride8(out_head))
        return set_error(CG_EINVAL, "strides must be non-negative multiples of 8 elements");
    if ((rc = check_output(n_tok, out_tok, heads, out_head))) return rc;
    if (n_tok == 0 || heads == 0) return CG_OK;
    if (!x || !out || !positions) return set_error(CG_EINVAL, "null x, out or positions");
    if (!al16(x) || !al16(out) || !al4(positions)) return set_error(CG_EINVAL, "x and out must be 16-byte aligned");
    RotArgs a{};
    if ((rc = device_status(&a.status))) return rc;
    a.q = static_cast<const uint16_t*>(x);
    a.q_out = static_cast<uint16_t*>(out);
    a.pos = positions;
    a.table = table;
    a.q_tok = x_tok;
    a.q_head = x_head;
    a.o_tok = out_tok;
    a.o_head = out_head;
    a.n_tok = n_tok;
    a.q_heads = heads;
    a.d = d;
    a.rot = rotary->rot;
    a.transpose = rotary->transpose != 0;
    a.mscale = rotary->mscale;
    const cudaError_t e = launch_rotary(a, dtype == CG_FP16, rotary->interleaved != 0, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return set_error(CG_ECUDA, "rotary launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

CG_EXPORT int cg_rotary_append(const cg_pages* pages, const cg_rotary_params* rotary, int32_t n_tok, int32_t q_heads,
                               const cg_append_strides* s, const void* q, const void* k, const void* v,
                               const int32_t* positions, const int64_t* slots, const int64_t* table, void* q_out,
                               void* pool, void* stream) {
    set_error(CG_OK, "%s", "");
    int rc = check_pages(pages, true);
    if (rc) return rc;
    if (n_tok < 0 || q_heads < 0 || q_heads > 65536)
        return set_error(CG_EINVAL, "n_tok=%d, q_heads=%d out of range", n_tok, q_heads);
    rc = check_rotary(rotary, pages->d, table);
    if (!rc) rc = check_units(n_tok, (int64_t)q_heads + 2 * pages->H, pages->d);
    if (rc) return rc;
    if (!s) return set_error(CG_EINVAL, "null strides");
    if (!stride8(s->q_tok) || !stride8(s->q_head) || !stride8(s->k_tok) || !stride8(s->k_head) || !stride8(s->v_tok) ||
        !stride8(s->v_head) || !stride8(s->o_tok) || !stride8(s->o_head))
        return set_error(CG_EINVAL, "strides must be non-negative multiples of 8 elements");
    if ((rc = check_output(n_tok, s->o_tok, q_heads, s->o_head))) return rc;
    if (n_tok == 0) return CG_OK;
    if (!k || !v || !positions || !slots || !pool || (q_heads && (!q || !q_out)))
        return set_error(CG_EINVAL, "null pointer");
    if (!al16(q) || !al16(k) || !al16(v) || !al16(q_out) || !al16(pool) || !al4(positions) || !al8(slots))
        return set_error(CG_EINVAL, "q, k, v, q_out and pool must be 16-byte aligned, the index arrays to their type");
    RotArgs a{};
    if ((rc = device_status(&a.status))) return rc;
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.pool = static_cast<uint16_t*>(pool);
    a.pos = positions;
    a.slots = slots;
    a.table = table;
    a.q_tok = s->q_tok;
    a.q_head = s->q_head;
    a.k_tok = s->k_tok;
    a.k_head = s->k_head;
    a.v_tok = s->v_tok;
    a.v_head = s->v_head;
    a.o_tok = s->o_tok;
    a.o_head = s->o_head;
    a.n_slots = (int64_t)pages->n_pages * pages->page;
    a.v_half = a.n_slots * pages->H * pages->d;
    a.n_tok = n_tok;
    a.q_heads = q_heads;
    a.H = pages->H;
    a.d = pages->d;
    a.rot = rotary->rot;
    a.page = pages->page;
    a.page_log2 = log2_of(pages->page);
    a.transpose = rotary->transpose != 0;
    a.mscale = rotary->mscale;
    const cudaError_t e = launch_rotary(a, pages->dtype == CG_FP16, rotary->interleaved != 0, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return set_error(CG_ECUDA, "rotary append launch: %s", cudaGetErrorString(e));
    return CG_OK;
}

}  // extern "C"
