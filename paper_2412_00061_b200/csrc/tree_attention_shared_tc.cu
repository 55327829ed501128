// Shared-prefix tree attention for bf16 on the 5th-generation tensor cores (tcgen05 + TMEM).
//
// Persistent CTAs, one per SM, each with a span of the line of key blocks (shared_attention.cuh).  A tile
// is 256 packed query rows in two halves of 128; every 128-key block of K and V is loaded once and serves
// both halves, in two steps of 64 keys.  Per half and step:
//   S[128 x 64] = Q K^T      tcgen05.mma, operands in shared memory (128-byte swizzle), S in tensor memory;
//   softmax                  one thread per query row reads its 64 scores at once, P = 2^(S - ref) goes back
//                            to tensor memory as bf16, over the scores it came from;
//   O[128 x D] += P V        tcgen05.mma with P from tensor memory and V as an MN-major operand.
// A half's two steps have a place of their own in tensor memory, so the scores of the next step are made while the
// current one is weighed, and the two halves fill each other's gaps besides.  (Measured: steps of 128 keys, one
// place per half, ran 1.6 times longer: scores, maximum, exponentials, P V and the next scores then
// form one chain of about 4600 cycles, against 2700 of tensor-core work for both halves.)
// What bounds it: a step takes about 1900 cycles - wait 130, reading the scores 250, maximum 150, exponentials 650-1000
// (two warps share a scheduler's unit), storing P 115, hand-over and loop 200-300 - and the tensor core 720 for each half
// (scores of 64 keys take it as long as scores of 128).  64 rows x 8 heads of 32 sequences on an 8192-row prefix: 517 us,
// 1.07 PFLOP/s.  Batches of single tokens are bound by HBM: 319 MB in 71 us, 13 us of that set-up and merge.
// P is rounded to bf16, by 2^-8 of a weight at most, because a tensor-core product takes both operands in one type and V is bf16:
// weights in 32 bits would take V widened to tf32 (half the rate, twice the space) or P in two bf16 parts (twice the
// products).  Scores, references, sums (of the unrounded weights), O and the parts are float32.  Against 64 bits the outputs are off
// by 0.0020-0.0022 relative, 1.1-1.3 times what rounding them to bf16 alone costs; tree_attention_tc.cu does the same.
// With at most 128 rows in a tile both halves work on the same rows, one on the even and one on the odd
// blocks, and their outputs are joined at the end: short batches keep both pipes busy too.
// ref, the exponent's reference, follows the row maximum lazily (only when it falls kSlack behind), so that O
// is hardly ever rescaled; sums and outputs are float32 throughout, P alone is rounded to bf16.
//
// Warp 0 loads K/V (TMA), warps 1 and 2 issue the MMAs of one half each, warp 3 looks after V rows that hold NaN
// or infinities, warps 4-7 and 8-11 are the softmax warps of the two halves.
//
// A weight of zero does not cancel a NaN.  In a block that some row of the tile sees only in part (ends of
// caches, trees, several sequences in one tile), warp 3 clears V rows that hold a NaN or an infinity
// before P V reads them, and leaves a note; a row that does see such a key becomes NaN at the end.
// One sequence's bad cache, or stale rows behind its end, cannot reach another sequence.
#include "shared_attention.cuh"
#include "tc_primitives.cuh"

#include <math.h>

namespace ctcsd {
namespace {

constexpr int kThreads = 384;
constexpr int kHalf = 128;             // rows per half
constexpr int kKeys = kTcKeys;
constexpr int kStep = 64;              // keys weighed at a time
constexpr float kSlack = 8.f;          // log2 units: P stays below 2^8
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kNoteBits = 2048;

template <int D> struct Shape;
template <> struct Shape<128> { static constexpr int kStages = 2; };
template <> struct Shape<64> { static constexpr int kStages = 4; };

struct __align__(8) SharedState {
    uint64_t q_full;
    uint64_t k_full[4], k_empty[4];
    uint64_t v_full[4], v_empty[4], v_ok[4];     // v_ok: the V block has been looked over
    uint64_t s_full[2][2], p_full[2][2];         // per half and step
    uint64_t pv_done[2], o_full[2];              // P V of a step; of the piece
    uint32_t tmem_base;
    int abort_flag, never_set;
    int any_note;
    unsigned note[kNoteBits / 32];               // blocks (fill number mod kNoteBits) in which a V row was cleared
    float join[2][kHalf];                        // reference and sum of the second half's rows when both serve the same
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two float32 in one 64-bit register pair: the packed instructions halve the issue slots.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void pair_split(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Maximum of three; a NaN among them comes out.
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ __nv_bfloat162 bf16_pair(uint32_t w) { return *reinterpret_cast<__nv_bfloat162*>(&w); }
// A wait has run out: record it once and let every other role stop waiting.
__device__ __forceinline__ void give_up(SharedState* sh, int* status, int site) {
    volatile int* f = &sh->abort_flag;
    if (*f == 0) report_error(status, CTCSD_ERR_TIMEOUT, site);
    *f = 1;
}
// All softmax threads (both halves) meet here.
__device__ __forceinline__ void halves_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <bool B> struct Flag { static constexpr bool value = B; };

// What every role has to know of a part of the span.
struct Piece {
    TileInfo ti;
    int g, blk0, blk1;
    bool split_keys;                   // both halves serve the same rows
    int seq_a, seq_b;                  // last sequence of the first half, first sequence of the second
    int pre_a, pre_b;                  // longest prefix share of each half
};

__device__ __forceinline__ Piece make_piece(const SharedPlan& pl, int B, const SpanWalk& at) {
    Piece c;
    c.g = at.g;
    c.blk0 = at.blk0;
    c.blk1 = at.blk1;
    c.ti = plan_tile(pl, B, kTcRows, at.t);
    c.split_keys = c.ti.nrows <= kHalf;
    c.seq_a = c.ti.b1;
    c.seq_b = c.ti.b0;
    c.pre_a = c.pre_b = c.ti.pmax;
    if (!c.split_keys && c.ti.b0 != c.ti.b1) {
        c.seq_a = plan_seq_of_row(pl, B, c.ti.row0 + kHalf - 1);
        c.seq_b = plan_seq_of_row(pl, B, c.ti.row0 + kHalf);
        if (c.ti.pmin != c.ti.pmax) {
            c.pre_a = plan_pre_max(pl, c.ti.b0, c.seq_a);
            c.pre_b = plan_pre_max(pl, c.seq_b, c.ti.b1);
        }
    }
    return c;
}

// Which halves work on a block, as a bit mask.
__device__ __forceinline__ unsigned takers(const Piece& c, const BlockIter& it, int blk) {
    if (c.split_keys) return 1u << ((blk - c.blk0) & 1);
    const bool a = it.seq < 0 ? it.key0 < c.pre_a : it.seq <= c.seq_a;
    const bool b = it.seq < 0 ? it.key0 < c.pre_b : it.seq >= c.seq_b;
    return (a ? 1u : 0u) | (b ? 2u : 0u);
}

// Whether some row of the tile sees the block only in part.
__device__ __forceinline__ bool mixed(const SharedPlan& pl, const Piece& c, const BlockIter& it) {
    if (it.seq < 0) return it.key0 + kKeys > c.ti.pmin;
    return c.ti.b0 != c.ti.b1 || it.key0 + kKeys > pl.kv[it.seq];
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
shared_attention_tc_kernel(const __grid_constant__ CUtensorMap tmKp, const __grid_constant__ CUtensorMap tmVp,
                           const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, SharedAttnParams p) {
    constexpr int DH = D / 64;
    constexpr int NS = Shape<D>::kStages;
    constexpr int kQHalf = kHalf * D * 2;
    constexpr int kTile = kKeys * D * 2;
    extern __shared__ __align__(1024) unsigned char dyn[];
    unsigned char* Qs = dyn;                                   // [half][DH][128 rows][128 B]
    unsigned char* Ks = Qs + 2 * kQHalf;                       // [NS][DH][128 keys][128 B]
    unsigned char* Vs = Ks + NS * kTile;
    SharedState* sh = reinterpret_cast<SharedState*>(Vs + NS * kTile);
    SharedPlan pl;
    plan_carve(pl, reinterpret_cast<int*>(sh + 1), p.B);
    if ((tc::smem_u32(dyn) & 1023u) != 0u) {                   // uniform over the CTA
        if (threadIdx.x == 0) report_error(p.status, CTCSD_ERR_INTERNAL, 34);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        tc::mbar_init(&sh->q_full, 8);
        for (int s = 0; s < NS; ++s) {
            tc::mbar_init(&sh->k_full[s], 1); tc::mbar_init(&sh->k_empty[s], 2);
            tc::mbar_init(&sh->v_full[s], 1); tc::mbar_init(&sh->v_empty[s], 2);
            tc::mbar_init(&sh->v_ok[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            for (int e = 0; e < 2; ++e) {
                tc::mbar_init(&sh->s_full[s][e], 1);
                tc::mbar_init(&sh->p_full[s][e], 4);
            }
            tc::mbar_init(&sh->pv_done[s], 1);
            tc::mbar_init(&sh->o_full[s], 1);
        }
        sh->abort_flag = 0;
        sh->never_set = 0;
        sh->any_note = 0;
        tc::fence_barrier_init();
    }
    for (int i = tid; i < kNoteBits / 32; i += kThreads) sh->note[i] = 0u;
    if (warp == 1) {
        tc::tmem_alloc(&sh->tmem_base, 512);
        tc::tmem_relinquish();
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    const uint32_t tmem = sh->tmem_base;                       // S: columns 0, 128; O: 256, 256 + D

    pdl_wait();
    pdl_trigger();
    plan_build(pl, p, kTcRows, kKeys, blockIdx.x == 0);
    const SpanMap sp = span_map(pl.tile_cum[pl.tiles], pl.tiles, p.Hkv, (int)gridDim.x, p.min_blocks, p.long_span);
    if (blockIdx.x == 0) plan_publish(pl, p, kTcRows, sp.spans);
    bool failed = false;
    SpanWalk at;
    bool more = at.init(pl, sp, blockIdx.x);

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (lane == 0) {
            const uint64_t pol = tc::policy_evict_last();
            int fill = 0;
            for (; more && !failed; more = at.next(pl)) {
                const Piece c = make_piece(pl, p.B, at);
                BlockIter it;
                it.init(pl, c.ti, kKeys, c.blk0);
                for (int blk = c.blk0; blk < c.blk1; ++blk, ++fill) {
                    const int s = fill % NS;
                    const uint32_t ph = (uint32_t)(fill / NS) & 1u;
                    const bool pre = it.seq < 0;
                    if (!tc::mbar_wait_suspended(&sh->k_empty[s], ph ^ 1u, abort_flag)) { failed = true; break; }
                    tc::mbar_arrive_expect_tx(&sh->k_full[s], (uint32_t)kTile);
                    tc::tma_load_5d(Ks + (size_t)s * kTile, pre ? &tmKp : &tmK, &sh->k_full[s], 0, it.key0, 0, c.g, pre ? 0 : it.seq, pol);
                    if (!tc::mbar_wait_suspended(&sh->v_empty[s], ph ^ 1u, abort_flag)) {
                        failed = true;
                        tc::mbar_wait_suspended(&sh->k_full[s], ph, &sh->never_set, 1ll << 24);      // the K copy lands first
                        break;
                    }
                    tc::mbar_arrive_expect_tx(&sh->v_full[s], (uint32_t)kTile);
                    tc::tma_load_5d(Vs + (size_t)s * kTile, pre ? &tmVp : &tmV, &sh->v_full[s], 0, it.key0, 0, c.g, pre ? 0 : it.seq, pol);
                    if (blk + 1 < c.blk1) it.next(pl, c.ti, kKeys);
                }
            }
            if (failed) {
                give_up(sh, p.status, 31);
                for (int back = 1; back <= NS && back <= fill; ++back) {                    // copies in flight land before the exit
                    const int j = fill - back;
                    tc::mbar_wait_suspended(&sh->k_full[j % NS], (uint32_t)(j / NS) & 1u, &sh->never_set, 1ll << 24);
                    tc::mbar_wait_suspended(&sh->v_full[j % NS], (uint32_t)(j / NS) & 1u, &sh->never_set, 1ll << 24);
                }
            }
        }
    } else if (warp < 3) {
        // ---------------- MMA issuer of one half ----------------
        // Both issuers visit every fill of the rings in order; for a block that is not its half's, an
        // issuer only hands the buffers back.
        if (lane == 0) {
            const int half = warp - 1;
            const uint32_t idesc_s = tc::idesc_bf16_f32(kHalf, kStep);
            const uint32_t idesc_o = tc::idesc_bf16_f32_b_mn(kHalf, D);
            const uint32_t tmem_s = tmem + (uint32_t)(half * 128), tmem_o = tmem + 256u + (uint32_t)(half * D);
            const uint64_t kdesc0 = tc::smem_desc_k_sw128(tc::smem_u32(Ks));
            const uint64_t vdesc0 = tc::smem_desc_mn_sw128(tc::smem_u32(Vs), kKeys * 128);
            int fill = 0, piece = 0;
            uint32_t count = 0u;                               // blocks whose P this issuer has waited for
            bool ok = true;
            for (; more && ok; more = at.next(pl), ++piece) {
                const Piece c = make_piece(pl, p.B, at);
                const uint64_t qdesc0 = tc::smem_desc_k_sw128(tc::smem_u32(Qs + (c.split_keys ? 0 : half * kQHalf)));
                BlockIter it;
                it.init(pl, c.ti, kKeys, c.blk0);
                int pend = -1;                                 // block (fill number) whose P V is still to be issued
                bool first = true;
                // O (+)= P V of one step of the pending block
                auto issue_pv = [&](int e) -> bool {
                    const int st = pend % NS;
                    const uint32_t ph = (uint32_t)(pend / NS) & 1u;
                    if (e == 0) {
                        if (!tc::mbar_wait_suspended(&sh->v_full[st], ph, abort_flag)) return false;
                        if (!tc::mbar_wait_suspended(&sh->v_ok[st], ph, abort_flag)) return false;
                    }
                    if (!tc::mbar_wait_suspended(&sh->p_full[half][e], count & 1u, abort_flag)) return false;
                    tc::tc_fence_after_sync();
                    const uint64_t vdesc = vdesc0 + (uint64_t)((st * kTile + e * kStep * 128) >> 4);
#pragma unroll
                    for (int kk = 0; kk < kStep / 16; ++kk)               // 16 keys: 8 columns of P, 16 rows of V
                        tc::mma_bf16_ts(tmem_o, tmem_s + (uint32_t)(e * kStep + kk * 8), vdesc + (uint64_t)((kk * 16 * 128) >> 4), idesc_o,
                                        !first || kk != 0 ? 1u : 0u);
                    tc::mma_commit(&sh->pv_done[half]);
                    first = false;
                    if (e == 1) {
                        tc::mma_commit(&sh->v_empty[st]);
                        ++count;
                    }
                    return true;
                };
                auto issue_s = [&](int e, int st) {
                    const uint64_t kdesc = kdesc0 + (uint64_t)((st * kTile + e * kStep * 128) >> 4);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint64_t along = (uint64_t)((kk / 4) * ((kHalf * 128) >> 4) + 2 * (kk % 4));
                        tc::mma_bf16_ss(tmem_s + (uint32_t)(e * kStep), qdesc0 + along, kdesc + along, idesc_s, kk != 0 ? 1u : 0u);
                    }
                    tc::mma_commit(&sh->s_full[half][e]);
                };
                // hands a V buffer of the other half's back
                auto pass_v = [&](int f) -> bool {
                    if (!tc::mbar_wait_suspended(&sh->v_full[f % NS], (uint32_t)(f / NS) & 1u, abort_flag)) return false;
                    tc::mbar_arrive(&sh->v_empty[f % NS]);
                    return true;
                };
                auto pass_k = [&](int f) -> bool {
                    if (!tc::mbar_wait_suspended(&sh->k_full[f % NS], (uint32_t)(f / NS) & 1u, abort_flag)) return false;
                    tc::mbar_arrive(&sh->k_empty[f % NS]);
                    return true;
                };
                ok = tc::mbar_wait_suspended(&sh->q_full, (uint32_t)piece & 1u, abort_flag);
                // (one more round than blocks: the last block's P V)
                for (int blk = c.blk0; blk <= c.blk1 && ok; ++blk) {
                    const int st = fill % NS;
                    const bool more_blocks = blk < c.blk1;
                    const bool mine = more_blocks && ((takers(c, it, blk) >> half) & 1u);
                    // a step's P is read by P V before the next S overwrites it: the tensor core works in issue order
#pragma unroll 1
                    for (int e = 0; e < 2 && ok; ++e) {
                        if (pend >= 0) ok = issue_pv(e);
                        if (ok && mine) {
                            if (e == 0) {
                                ok = tc::mbar_wait_suspended(&sh->k_full[st], (uint32_t)(fill / NS) & 1u, abort_flag);
                                tc::tc_fence_after_sync();
                            }
                            if (ok) issue_s(e, st);
                        }
                    }
                    if (!ok || !more_blocks) break;
                    pend = mine ? fill : -1;
                    if (mine) tc::mma_commit(&sh->k_empty[st]);
                    else ok = pass_k(fill) && pass_v(fill);
                    ++fill;
                    if (blk + 1 < c.blk1) it.next(pl, c.ti, kKeys);
                }
                if (ok) tc::mma_commit(&sh->o_full[half]);
            }
            if (!ok) give_up(sh, p.status, 32);
        }
    } else if (warp == 3) {
        // ---------------- V rows that hold NaN or infinities ----------------
        int fill = 0;
        for (; more && !failed; more = at.next(pl)) {
            const Piece c = make_piece(pl, p.B, at);
            BlockIter it;
            it.init(pl, c.ti, kKeys, c.blk0);
            for (int blk = c.blk0; blk < c.blk1; ++blk, ++fill) {
                const int st = fill % NS;
                if (!tc::mbar_wait_suspended(&sh->v_full[st], (uint32_t)(fill / NS) & 1u, abort_flag)) failed = true;
                failed = __any_sync(0xffffffffu, failed);
                if (failed) break;
                if (mixed(pl, c, it)) {
#pragma unroll 1
                    for (int rr = 0; rr < kKeys / 32; ++rr) {
                        unsigned char* row = Vs + (size_t)st * kTile + (rr * 32 + lane) * 128;
                        // 0 * w is NaN for a NaN or an infinity and 0 otherwise
                        __nv_bfloat162 z4[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) z4[i] = __float2bfloat162_rn(0.f);
                        const __nv_bfloat162 zero = __float2bfloat162_rn(0.f);
#pragma unroll
                        for (int i = 0; i < DH * 8; ++i) {
                            const uint4 w = *reinterpret_cast<const uint4*>(row + (i / 8) * (kKeys * 128) + (((i + lane) & 7) << 4));
                            z4[0] = __hfma2(bf16_pair(w.x), zero, z4[0]);
                            z4[1] = __hfma2(bf16_pair(w.y), zero, z4[1]);
                            z4[2] = __hfma2(bf16_pair(w.z), zero, z4[2]);
                            z4[3] = __hfma2(bf16_pair(w.w), zero, z4[3]);
                        }
                        const float2 sum = __bfloat1622float2(__hadd2(__hadd2(z4[0], z4[1]), __hadd2(z4[2], z4[3])));
                        if (sum.x + sum.y != 0.f) {
#pragma unroll 1
                            for (int i = 0; i < DH * 8; ++i)
                                *reinterpret_cast<uint4*>(row + (i / 8) * (kKeys * 128) + ((i & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                            atomicOr(&sh->note[(fill % kNoteBits) >> 5], 1u << (fill & 31));
                            sh->any_note = 1;
                        }
                    }
                    __threadfence_block();
                    tc::fence_proxy_async();
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sh->v_ok[st]);
                if (blk + 1 < c.blk1) it.next(pl, c.ti, kKeys);
            }
        }
        if (failed && lane == 0) give_up(sh, p.status, 33);
    } else {
        // ---------------- softmax: one thread per query row of a half ----------------
        // Every softmax thread executes every barrier of the halves, also after a wait has failed.
        const int half = (warp - 4) >> 2;
        const int q = warp & 3;                                // TMEM lane quarter this warp may read
        const int rl = q * 32 + lane;
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        const uint32_t tmem_s = tmem + (uint32_t)(half * 128) + lane_off;
        const uint32_t tmem_o = tmem + 256u + (uint32_t)(half * D) + lane_off;
        const int grp = p.grp;
        const int W = (p.max_nodes + 63) / 64;
        const float sl2 = p.scale * kLog2e;                    // scores are kept in log2 units
        const uint64_t sl22 = pair_of(sl2, sl2);
        uint32_t s_count = 0u, steps = 0u;                     // blocks and steps of this half so far
        int fill0 = 0, piece = 0;
        // After a wait that ran out, nothing is waited for any more: the loops run to their ends on meaningless scores,
        // and no output is written.
        auto wait = [&](uint64_t* bar, uint32_t parity, int site) {
            if (!failed && !tc::mbar_wait_suspended(bar, parity, abort_flag)) {
                failed = true;
                give_up(sh, p.status, site);
            }
        };
        for (; more; more = at.next(pl), ++piece) {
            const Piece c = make_piece(pl, p.B, at);
            // ---- this thread's row ----
            const int rt = (c.split_keys ? 0 : half * kHalf) + rl;      // row of the tile
            const bool live = rt < c.ti.nrows;
            int seq = -2, node = 0, head = 0, row_pre = 0, row_kv = 0, row_n = 0;
            if (live) {
                const int pr = c.ti.row0 + rt;
                seq = c.ti.b0 == c.ti.b1 ? c.ti.b0 : plan_seq_of_row(pl, p.B, pr);
                const int o = pr - pl.row_off[seq];
                node = o / grp;
                head = c.g * grp + (o - node * grp);
                row_pre = pl.pre[seq];
                row_kv = pl.kv[seq];
                row_n = pl.own_len[seq] - row_kv;
            }
            // (below 2^32: as many rows of 64 columns fill no GPU's memory)
            auto out_row = [&]() -> unsigned { return live ? ((unsigned)seq * p.max_nodes + node) * p.Hq + head : 0u; };
            auto visible32 = [&](int src, int key) -> uint32_t {
                return live ? visible32_of(src, key, seq, row_pre, row_kv, row_n, p.mask + ((size_t)seq * p.max_nodes + node) * W, W) : 0u;
            };
            const bool warp_live = __any_sync(0xffffffffu, live);
            halves_barrier();                                   // the previous piece is done with Q's memory
            if (!c.split_keys || half == 0) {
                // neighbouring lanes take neighbouring 16 bytes of a row
                constexpr int LR = D / 8, RI = 32 / LR;         // lanes per row, rows per instruction
                unsigned char* dst = Qs + half * kQHalf + (q * 32) * 128;
                const int cc = lane % LR;
                const unsigned orow = out_row(), there = __ballot_sync(0xffffffffu, live);
                const uint4* Qg = static_cast<const uint4*>(p.Q) + cc;
#pragma unroll 1
                for (int i0 = 0; i0 < LR; i0 += 8) {
                    uint4 w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)                 // (a row that is not there reads row 0)
                        w[i] = __ldg(Qg + (size_t)__shfl_sync(0xffffffffu, orow, (i0 + i) * RI + lane / LR) * LR);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int rr = (i0 + i) * RI + lane / LR;
                        if (!((there >> rr) & 1u)) w[i] = make_uint4(0u, 0u, 0u, 0u);
                        *reinterpret_cast<uint4*>(dst + rr * 128 + (cc / 8) * (kHalf * 128) + (((cc % 8) ^ (rr & 7)) << 4)) = w[i];
                    }
                }
                tc::fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sh->q_full);

            float ref = -INFINITY, sum = 0.f;
            bool first = true, poisoned = false;
            // One step of a block.  Open: every row of the warp sees all of its keys; else the rows' limits are looked at, and
            // their masks where a row sees some of the keys.  (Two copies of the code: with the masks inside the loop of
            // open blocks, which is most of them, its instructions take longer to fetch.)
            auto step = [&](auto open_tag, int e, int src, int key) {
                constexpr bool Open = decltype(open_tag)::value;
                const uint32_t tmem_se = tmem_s + (uint32_t)(e * kStep);
                bool none = false;                              // no row of the warp sees any of the step's keys
                bool plain = true, sees = true;                 // every row sees all of them or none; this one does
                if constexpr (!Open) {
                    const int all_to = src < 0 ? row_pre : (src == seq ? row_kv : 0);
                    const bool hidden = !live || all_to + (src == seq ? row_n : 0) <= key;
                    sees = live && all_to >= key + kStep;
                    none = __all_sync(0xffffffffu, hidden);
                    plain = __all_sync(0xffffffffu, hidden || sees);
                }
                wait(&sh->s_full[half][e], s_count & 1u, 35);
                __syncwarp();
                tc::tc_fence_after_sync();
                if (!Open && none) {
                    // nothing to see for this warp: P is zero (rows that are not there take no part at all)
                    if (warp_live) {
                        uint32_t z[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] = 0u;
                        tc::tmem_st32(tmem_se, z);
                    }
                } else {
                    uint32_t v[64];
                    tc::tmem_read64(tmem_se, v);
                    if (!Open && !plain) {
#pragma unroll
                        for (int cc = 0; cc < 2; ++cc) {
                            const uint32_t vis = visible32(src, key + cc * 32);
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[32 * cc + j] = ((vis >> j) & 1u) ? v[32 * cc + j] : 0xff800000u;
                        }
                    }
                    float b4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < 64; j += 2)
                        b4[(j >> 1) & 3] = max3_nan(b4[(j >> 1) & 3], __uint_as_float(v[j]), __uint_as_float(v[j + 1]));
                    float bm = max3_nan(max3_nan(b4[0], b4[1], b4[2]), b4[3], -INFINITY);
                    if (!Open && plain && !sees) bm = -INFINITY;
                    poisoned = poisoned || !(bm < INFINITY);       // a NaN or +inf score: the row is not meaningful
                    bm *= sl2;
                    const bool move = bm > ref + kSlack;           // also the first visible key (ref = -inf)
                    if (__builtin_expect(__any_sync(0xffffffffu, move), 0)) {
                        const float corr = move ? exp2_fast(ref - bm) : 1.f;
                        if (!first) {
                            // O must be at rest: P V of the step before (older ones precede this step's scores)
                            wait(&sh->pv_done[half], (steps - 1u) & 1u, 35);
                            __syncwarp();
                            tc::tc_fence_after_sync();
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 32) {
                                uint32_t o[32];
                                tc::tmem_read32(tmem_o + (uint32_t)c0, o);
#pragma unroll
                                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * corr);
                                tc::tmem_st32(tmem_o + (uint32_t)c0, o);
                            }
                        }
                        sum *= corr;
                        ref = move ? bm : ref;
                    }
                    const float off = ref == -INFINITY ? 0.f : -ref;
                    const uint64_t off2 = pair_of(off, off);
                    // Eight pairs at a time, stage by stage: the pairs' chains (scale, exponential, sum, round) run side
                    // by side.  (The exponential unit's 16 results a clock come to 2048 cycles a block, the tensor core's time at
                    // its best; with a share of them as polynomials on the FMA pipe an 8192-row prefix took 519-540 us
                    // against 517.)
                    uint64_t s2[4] = {0ull, 0ull, 0ull, 0ull};
                    uint32_t w[32];
#pragma unroll
                    for (int g0 = 0; g0 < 32; g0 += 8) {
                        uint64_t x[8];
                        float lo[8], hi[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int j = 2 * (g0 + i);
                            x[i] = fma2(pair_of(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), sl22, off2);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            pair_split(x[i], lo[i], hi[i]);
                            lo[i] = exp2_fast(lo[i]);
                            hi[i] = exp2_fast(hi[i]);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) s2[i % 4] = add2(s2[i % 4], pair_of(lo[i], hi[i]));
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[g0 + i] = pack_bf16(lo[i], hi[i]);
                    }
                    float sa, sb;
                    pair_split(add2(add2(s2[0], s2[1]), add2(s2[2], s2[3])), sa, sb);
                    float more_sum = sa + sb;
                    if (!Open && plain && !sees) {
                        more_sum = 0.f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) w[j] = 0u;
                    }
                    tc::tmem_st32(tmem_se, w);                     // over scores that have been read
                    sum += more_sum;
                }
                first = false;
                ++steps;
                tc::tmem_st_wait();
                tc::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sh->p_full[half][e]);
            };
            BlockIter it;
            it.init(pl, c.ti, kKeys, c.blk0);
            for (int blk = c.blk0; blk < c.blk1; ++blk) {
                // whole blocks from here on that every row of the warp sees
                int open = warp_live ? __reduce_min_sync(0xffffffffu, !live ? c.blk1 - blk : max((it.seq < 0 ? row_pre : (it.seq == seq ? row_kv : 0)) - it.key0, 0) / kKeys) : 0;
                open = min(open, c.blk1 - blk);
                if (open > 0) {
                    // (the half takes them all, unless the halves take turns)
                    const int by = c.split_keys ? 2 : 1;
#pragma unroll 1
                    for (int i = c.split_keys ? (blk - c.blk0 + half) & 1 : 0; i < open; i += by, ++s_count)
#pragma unroll 1
                        for (int e = 0; e < 2; ++e) step(Flag<true>(), e, 0, 0);
                    blk += open - 1;
                    it.key0 += (open - 1) * kKeys;
                } else if ((takers(c, it, blk) >> half) & 1u) {
#pragma unroll 1
                    for (int e = 0; e < 2; ++e) step(Flag<false>(), e, it.seq, it.key0 + e * kStep);
                    ++s_count;
                }
                if (blk + 1 < c.blk1) it.next(pl, c.ti, kKeys);
            }
            if (poisoned) sum = __uint_as_float(0x7fc00000u);
            // ---- the half's output is complete ----
            wait(&sh->o_full[half], (uint32_t)piece & 1u, 36);
            failed = __any_sync(0xffffffffu, failed);
            tc::tc_fence_after_sync();
            // a row that saw a V row that was cleared: NaN (rare: only if some block left a note)
            if (!failed && *(volatile int*)&sh->any_note != 0 && live) {
                BlockIter jt;
                jt.init(pl, c.ti, kKeys, c.blk0);
                for (int blk = c.blk0; blk < c.blk1; ++blk) {
                    const int f = fill0 + blk - c.blk0;
                    const bool noted = (*(volatile unsigned*)&sh->note[(f % kNoteBits) >> 5] >> (f & 31)) & 1u;
                    if (noted && ((takers(c, jt, blk) >> half) & 1u) && mixed(pl, c, jt)) {
                        const __nv_bfloat16* vb = jt.seq < 0 ? static_cast<const __nv_bfloat16*>(p.Vp) + (size_t)c.g * p.Pcap * D
                                                             : static_cast<const __nv_bfloat16*>(p.V) + ((size_t)jt.seq * p.Hkv + c.g) * (size_t)p.Lcap * D;
#pragma unroll 1
                        for (int k = 0; k < kKeys; ++k) {
                            if (!((visible32(jt.seq, jt.key0 + (k & ~31)) >> (k & 31)) & 1u)) continue;
                            const uint32_t* vr = reinterpret_cast<const uint32_t*>(vb + (size_t)(jt.key0 + k) * D);
                            uint32_t bad = 0u;
#pragma unroll 1
                            for (int d = 0; d < D / 2; ++d) bad |= (vr[d] & 0x7f807f80u) + 0x00800080u;
                            if (bad & 0x80008000u) sum = __uint_as_float(0x7fc00000u);
                        }
                    }
                    if (blk + 1 < c.blk1) jt.next(pl, c.ti, kKeys);
                }
            }
            fill0 += c.blk1 - c.blk0;
            float mine = 1.f, other = 0.f;                      // weights of the two halves' outputs
            float* join = reinterpret_cast<float*>(Qs);         // [128 rows][D], 16-byte chunks swizzled by the row
            if (c.split_keys) {
                halves_barrier();                               // both halves' products are done with Q
                if (half == 1) {
                    sh->join[0][rl] = ref;
                    sh->join[1][rl] = first ? 0.f : sum;
                    if (!first && !failed && warp_live) {
#pragma unroll 1
                        for (int c0 = 0; c0 < D; c0 += 32) {
                            uint32_t o[32];
                            tc::tmem_read32(tmem_o + (uint32_t)c0, o);
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                *reinterpret_cast<uint4*>(join + rl * D + ((((c0 / 4) + j) ^ (rl & 7)) << 2)) =
                                    make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                        }
                    }
                }
                halves_barrier();
                if (half == 0) {
                    const float r1 = sh->join[0][rl], s1 = sh->join[1][rl];
                    const float top = fmaxf(ref, r1), base = top == -INFINITY ? 0.f : top;
                    mine = exp2_fast(ref - base);
                    other = s1 != 0.f ? exp2_fast(r1 - base) : 0.f;     // (nothing seen: its output is not meaningful)
                    sum = sum * mine + (s1 != 0.f ? s1 * other : 0.f);
                    ref = top;
                }
            }
            // ---- output: this thread's row ----
            if (!failed && warp_live && (!c.split_keys || half == 0)) {
                const bool whole = at.whole();
                const float inv = whole ? (sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum)) : 1.f;
                const size_t part = (size_t)blockIdx.x * 2 + at.slot();
                // a finished row goes through shared memory (Q's place, or over its own part of the joined
                // rows, behind what has been read), so that it leaves in whole lines
                unsigned char* stage = c.split_keys ? Qs + rl * (D * 4) : Qs + half * kQHalf + rl * (D * 2);
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    float o[32];
                    if (!first) {
                        uint32_t u[32];
                        tc::tmem_read32(tmem_o + (uint32_t)c0, u);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = __uint_as_float(u[j]) * mine;
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = 0.f;
                    }
                    if (other != 0.f) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float4 w = *reinterpret_cast<const float4*>(join + rl * D + ((((c0 / 4) + j) ^ (rl & 7)) << 2));
                            o[4 * j] = fmaf(w.x, other, o[4 * j]); o[4 * j + 1] = fmaf(w.y, other, o[4 * j + 1]);
                            o[4 * j + 2] = fmaf(w.z, other, o[4 * j + 2]); o[4 * j + 3] = fmaf(w.w, other, o[4 * j + 3]);
                        }
                    }
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint4 w;
                            w.x = pack_bf16(o[8 * j + 0] * inv, o[8 * j + 1] * inv);
                            w.y = pack_bf16(o[8 * j + 2] * inv, o[8 * j + 3] * inv);
                            w.z = pack_bf16(o[8 * j + 4] * inv, o[8 * j + 5] * inv);
                            w.w = pack_bf16(o[8 * j + 6] * inv, o[8 * j + 7] * inv);
                            *reinterpret_cast<uint4*>(stage + (((c0 / 8 + j) ^ (rl & 7)) << 4)) = w;
                        }
                    } else if (live && CTCSD_IN_BOUNDS(p.status, 87, part * kTcRows + rt, 2ll * gridDim.x * kTcRows)) {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            p.part_o[(part * (D / 4) + c0 / 4 + j) * kTcRows + rt] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                    }
                }
                if (whole) {
                    __syncwarp();
                    constexpr int LR = D / 8, RI = 32 / LR;
                    const int cc = lane % LR;
                    const unsigned char* from = c.split_keys ? Qs + q * 32 * (D * 4) : Qs + half * kQHalf + q * 32 * (D * 2);
                    const int stride = c.split_keys ? D * 4 : D * 2;
                    const unsigned orow = out_row(), there = __ballot_sync(0xffffffffu, live);
#pragma unroll 2
                    for (int i = 0; i < LR; ++i) {
                        const int rr = i * RI + lane / LR;
                        const size_t dst = __shfl_sync(0xffffffffu, orow, rr);
                        const uint4 w = *reinterpret_cast<const uint4*>(from + rr * stride + ((cc ^ (rr & 7)) << 4));
                        if (((there >> rr) & 1u) && CTCSD_IN_BOUNDS(p.status, 88, dst, out_rows(p))) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.O) + dst * D + 8 * cc) = w;
                    }
                }
                if (live) {
                    if (!whole) {
                        if (CTCSD_IN_BOUNDS(p.status, 89, part * kTcRows + rt, 2ll * gridDim.x * kTcRows)) p.part_ml[part * kTcRows + rt] = make_float2(ref, sum);
                    } else if (p.lse && CTCSD_IN_BOUNDS(p.status, 90, out_row(), out_rows(p)))
                        p.lse[out_row()] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * kLn2;
                }
            }
            tc::tc_fence_before_sync();
        }
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc(tmem, 512);
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn get_encode_fn() {
    static EncodeTiledFn fn = nullptr;
    if (fn) return fn;
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qres) != cudaSuccess) return nullptr;
    if (qres != cudaDriverEntryPointSuccess) return nullptr;
    fn = reinterpret_cast<EncodeTiledFn>(sym);
    return fn;
}

// Rows [n][Hkv][len][D] seen as [n][Hkv][D/64][len][64]: a box is 128 keys of one head, all 64-column parts.
bool make_row_map(CUtensorMap* map, const void* base, int D, int len, int Hkv, int n) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[5] = {64, (cuuint64_t)len, (cuuint64_t)(D / 64), (cuuint64_t)Hkv, (cuuint64_t)n};
    cuuint64_t str[4] = {(cuuint64_t)D * 2, 128, (cuuint64_t)len * D * 2, (cuuint64_t)Hkv * len * D * 2};
    cuuint32_t box[5] = {64, (cuuint32_t)kKeys, (cuuint32_t)(D / 64), 1, 1};
    cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, str, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
int launch_tc(Handle* h, cudaStream_t s, const SharedAttnParams& p) {
    CUtensorMap tmKp, tmVp, tmK, tmV;
    if (!make_row_map(&tmK, p.K, D, p.Lcap, p.Hkv, p.B) || !make_row_map(&tmV, p.V, D, p.Lcap, p.Hkv, p.B)) return CTCSD_ERR_CUDA;
    tmKp = tmK;
    tmVp = tmV;
    if (p.Pcap > 0 && (!make_row_map(&tmKp, p.Kp, D, p.Pcap, p.Hkv, 1) || !make_row_map(&tmVp, p.Vp, D, p.Pcap, p.Hkv, 1)))
        return CTCSD_ERR_CUDA;
    const int max_tiles = (int)(((long long)p.B * p.max_nodes * (p.Hq / p.Hkv) + kTcRows - 1) / kTcRows);
    const size_t smem = (size_t)2 * kHalf * D * 2 + (size_t)Shape<D>::kStages * 2 * kKeys * D * 2 + sizeof(SharedState) +
                        sizeof(int) * plan_ints(p.B, max_tiles);
    auto kern = shared_attention_tc_kernel<D>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepSharedTc, kern));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(h->num_sms), dim3(kThreads), smem, s, 1, tmKp, tmVp, tmK, tmV, p));
    h->launches++;
    return CTCSD_OK;
}

}  // namespace

int launch_shared_attention_tc(Handle* h, cudaStream_t s, const SharedAttnParams& p) {
    return p.D == 64 ? launch_tc<64>(h, s, p) : launch_tc<128>(h, s, p);
}

}  // namespace ctcsd
