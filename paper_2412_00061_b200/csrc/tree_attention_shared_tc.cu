// Shared-prefix tree attention for bf16 on the 5th-generation tensor cores (tcgen05 + TMEM).
//
// Persistent CTAs, one per SM, each with a span of the line of key blocks (shared_attention.cuh).  A tile
// is 256 packed query rows in two halves of 128; every 128-key block of K and V is loaded once and serves
// both halves.  Per half and block:
//   S[128 x 128] = Q K^T     tcgen05.mma, operands in shared memory (128-byte swizzle), S in tensor memory;
//   softmax                  one thread per query row reads its 128 scores at once, P = 2^(S - ref) goes back
//                            to tensor memory as bf16, over the scores it came from;
//   O[128 x D] += P V        tcgen05.mma with P from tensor memory and V as an MN-major operand.
// The halves take turns: while one half's softmax runs, the tensor core works on the other's products.
// With at most 128 rows in a tile both halves work on the same rows, one on the even and one on the odd
// blocks, and their outputs are joined at the end: short batches keep both pipes busy too.
// ref, the exponent's reference, follows the row maximum lazily (only when it falls kSlack behind), so that O
// is hardly ever rescaled; sums and outputs are float32 throughout, P alone is rounded to bf16.
//
// Warp 0 loads K/V (TMA), warp 1 issues the MMAs, warps 2-3 look after V rows that hold NaN or infinities, warps
// 4-7 and 8-11 are the softmax warps of the two halves.
//
// A weight of zero does not cancel a NaN.  In a block that some row of the tile sees only in part (ends of
// caches, trees, several sequences in one tile), warps 2-3 clear V rows that hold a NaN or an infinity
// before P V reads them, and leave a note; a row that does see such a key becomes NaN at the end.
// One sequence's bad cache, or stale rows behind its end, cannot reach another sequence.
#include "shared_attention.cuh"
#include "tc_primitives.cuh"

#include <math.h>

namespace ctcsd {
namespace {

constexpr int kThreads = 384;
constexpr int kHalf = 128;             // rows per half
constexpr int kKeys = kTcKeys;
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
    uint64_t s_full[2], p_full[2], o_full[2];
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
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
// A wait has run out: record it once and let every other role stop waiting.
__device__ __forceinline__ void give_up(SharedState* sh, int* status, int site) {
    volatile int* f = &sh->abort_flag;
    if (*f == 0) report_error(status, CTCSD_ERR_TIMEOUT, site);
    *f = 1;
}
// All softmax threads (both halves) meet here.
__device__ __forceinline__ void halves_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// One part of the span: blocks [blk0, blk1) of a tile of a kv head, and what every role has to know of it.
struct Piece {
    TileInfo ti;
    int g, blk0, blk1;
    bool whole, split_keys;            // split_keys: both halves serve the same rows
    int slot;
    int sb0[2], sb1[2];                // sequences of each half
    int spre[2];                       // longest prefix share of each half
};

__device__ __forceinline__ Piece make_piece(const SharedPlan& pl, const SharedAttnParams& p, const SpanMap& sp, long long x, long long x1) {
    Piece c;
    c.g = (int)(x / sp.per_head);
    const int xh = (int)(x - (long long)c.g * sp.per_head);
    const int t = plan_tile_of_block(pl.tile_cum, pl.tiles, xh);
    c.ti = plan_tile(pl, p.B, kTcRows, t);
    const int nblk = pl.tile_cum[t + 1] - pl.tile_cum[t];
    c.blk0 = xh - pl.tile_cum[t];
    c.blk1 = (int)(x1 - x < nblk - c.blk0 ? c.blk0 + (x1 - x) : nblk);
    c.whole = c.blk0 == 0 && c.blk1 == nblk;
    c.slot = c.blk0 > 0 ? 0 : 1;
    c.split_keys = c.ti.nrows <= kHalf;
    c.sb0[0] = c.ti.b0;
    c.sb1[1] = c.ti.b1;
    c.sb1[0] = c.split_keys ? c.ti.b1 : plan_seq_of_row(pl, p.B, c.ti.row0 + kHalf - 1);
    c.sb0[1] = c.split_keys ? c.ti.b0 : plan_seq_of_row(pl, p.B, c.ti.row0 + kHalf);
    for (int s = 0; s < 2; ++s) {
        c.spre[s] = 0;
        for (int b = c.sb0[s]; b <= c.sb1[s]; ++b) c.spre[s] = max(c.spre[s], pl.pre[b]);
    }
    return c;
}

// Which halves work on a block, as a bit mask.
__device__ __forceinline__ unsigned takers(const Piece& c, const BlockIter& it, int blk) {
    if (c.split_keys) return 1u << ((blk - c.blk0) & 1);
    unsigned m = 0u;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const bool in = it.seq < 0 ? it.key0 < c.spre[s] : (it.seq >= c.sb0[s] && it.seq <= c.sb1[s]);
        m |= in ? 1u << s : 0u;
    }
    return m;
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
    pl.row_off = reinterpret_cast<int*>(sh + 1);
    pl.own_len = pl.row_off + p.B + 1;
    pl.kv = pl.own_len + p.B;
    pl.pre = pl.kv + p.B;
    pl.tile_cum = pl.pre + p.B;
    if ((tc::smem_u32(dyn) & 1023u) != 0u) {                   // uniform over the CTA
        if (threadIdx.x == 0) report_error(p.status, CTCSD_ERR_INTERNAL, 34);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        tc::mbar_init(&sh->q_full, 8);
        for (int s = 0; s < NS; ++s) {
            tc::mbar_init(&sh->k_full[s], 1); tc::mbar_init(&sh->k_empty[s], 1);
            tc::mbar_init(&sh->v_full[s], 1); tc::mbar_init(&sh->v_empty[s], 1);
            tc::mbar_init(&sh->v_ok[s], 2);
        }
        for (int s = 0; s < 2; ++s) {
            tc::mbar_init(&sh->s_full[s], 1);
            tc::mbar_init(&sh->p_full[s], 4);
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
    const SpanMap sp = span_map(pl.tile_cum[pl.tiles], p.Hkv, (int)gridDim.x, p.min_blocks);
    if (blockIdx.x == 0) plan_publish(pl, p, sp.spans);
    const bool idle = (int)blockIdx.x >= sp.spans || sp.total == 0;
    const long long xbeg = idle ? 0 : sp.start(blockIdx.x), xend = idle ? 0 : sp.start(blockIdx.x + 1);
    bool failed = false;

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (lane == 0) {
            const uint64_t pol = tc::policy_evict_last();
            int fill = 0;
            for (long long x = xbeg; x < xend && !failed;) {
                const Piece c = make_piece(pl, p, sp, x, xend);
                x += c.blk1 - c.blk0;
                BlockIter it;
                it.init(pl, c.ti, kKeys, c.blk0);
                for (int blk = c.blk0; blk < c.blk1; ++blk, ++fill) {
                    const int s = fill % NS;
                    const uint32_t ph = (uint32_t)(fill / NS) & 1u;
                    const bool pre = it.seq < 0;
                    if (!tc::mbar_wait(&sh->k_empty[s], ph ^ 1u, abort_flag)) { failed = true; break; }
                    tc::mbar_arrive_expect_tx(&sh->k_full[s], (uint32_t)kTile);
                    tc::tma_load_5d(Ks + (size_t)s * kTile, pre ? &tmKp : &tmK, &sh->k_full[s], 0, it.key0, 0, c.g, pre ? 0 : it.seq, pol);
                    if (!tc::mbar_wait(&sh->v_empty[s], ph ^ 1u, abort_flag)) {
                        failed = true;
                        tc::mbar_wait(&sh->k_full[s], ph, &sh->never_set, 1ll << 24);      // the K copy lands first
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
                    tc::mbar_wait(&sh->k_full[j % NS], (uint32_t)(j / NS) & 1u, &sh->never_set, 1ll << 24);
                    tc::mbar_wait(&sh->v_full[j % NS], (uint32_t)(j / NS) & 1u, &sh->never_set, 1ll << 24);
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0) {
            const uint32_t idesc_s = tc::idesc_bf16_f32(kHalf, kKeys);
            const uint32_t idesc_o = tc::idesc_bf16_f32_b_mn(kHalf, D);
            int fill = 0, piece = 0;
            uint32_t p_count[2] = {0u, 0u};
            // 4 bits per fill: halves that still have to read its V (twice the stages: S of a fill may be issued
            // while the stage's previous V is still waiting for a half)
            unsigned left = 0u;
            bool ok = true;
            for (long long x = xbeg; x < xend && ok; ++piece) {
                const Piece c = make_piece(pl, p, sp, x, xend);
                x += c.blk1 - c.blk0;
                BlockIter it;
                it.init(pl, c.ti, kKeys, c.blk0);
                int pend[2] = {-1, -1};                        // block (fill number) whose P V is still to be issued
                bool first[2] = {true, true};
                // O (+)= P V of half s for its pending block
                auto issue_pv = [&](int s) -> bool {
                    const int f = pend[s], st = f % NS;
                    const uint32_t ph = (uint32_t)(f / NS) & 1u;
                    pend[s] = -1;
                    if (!tc::mbar_wait(&sh->v_full[st], ph, abort_flag)) return false;
                    if (!tc::mbar_wait(&sh->v_ok[st], ph, abort_flag)) return false;
                    if (!tc::mbar_wait(&sh->p_full[s], p_count[s] & 1u, abort_flag)) return false;
                    ++p_count[s];
                    tc::tc_fence_after_sync();
                    const uint32_t v_addr = tc::smem_u32(Vs + (size_t)st * kTile);
#pragma unroll
                    for (int kk = 0; kk < kKeys / 16; ++kk) {
                        const uint64_t bdesc = tc::smem_desc_mn_sw128(v_addr + kk * (16 * 128), kKeys * 128);
                        tc::mma_bf16_ts(tmem + 256u + (uint32_t)(s * D), tmem + (uint32_t)(s * 128 + kk * 8), bdesc, idesc_o,
                                        !first[s] || kk != 0 ? 1u : 0u);
                    }
                    first[s] = false;
                    const int lb = 4 * (f % (2 * NS));
                    left -= 1u << lb;
                    if (((left >> lb) & 15u) == 0u) tc::mma_commit(&sh->v_empty[st]);
                    return true;
                };
                ok = tc::mbar_wait(&sh->q_full, (uint32_t)piece & 1u, abort_flag);
                for (int blk = c.blk0; blk < c.blk1 && ok; ++blk, ++fill) {
                    const int st = fill % NS;
                    const unsigned who = takers(c, it, blk);
                    left += (unsigned)__popc(who) << (4 * (fill % (2 * NS)));
                    bool here = false;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        if (!((who >> s) & 1u) || !ok) continue;
                        // the half's P is read by P V before S overwrites it: the tensor core works in issue order
                        if (pend[s] >= 0 && !issue_pv(s)) { ok = false; continue; }
                        if (!here) {
                            if (!tc::mbar_wait(&sh->k_full[st], (uint32_t)(fill / NS) & 1u, abort_flag)) { ok = false; continue; }
                            here = true;
                        }
                        tc::tc_fence_after_sync();
                        const uint32_t k_addr = tc::smem_u32(Ks + (size_t)st * kTile);
                        const uint32_t q_addr = tc::smem_u32(Qs + (c.split_keys ? 0 : s * kQHalf));
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint64_t adesc = tc::smem_desc_k_sw128(q_addr + (kk / 4) * (kHalf * 128)) + 2 * (kk % 4);
                            const uint64_t bdesc = tc::smem_desc_k_sw128(k_addr + (kk / 4) * (kKeys * 128)) + 2 * (kk % 4);
                            tc::mma_bf16_ss(tmem + (uint32_t)(s * 128), adesc, bdesc, idesc_s, kk != 0 ? 1u : 0u);
                        }
                        tc::mma_commit(&sh->s_full[s]);
                        pend[s] = fill;
                    }
                    if (ok) tc::mma_commit(&sh->k_empty[st]);
                    // a half that sits out the next blocks must not keep this V block from being refilled
#pragma unroll
                    for (int s = 0; s < 2; ++s)
                        if (ok && pend[s] >= 0 && pend[s] <= fill - NS && !issue_pv(s)) ok = false;
                    if (blk + 1 < c.blk1) it.next(pl, c.ti, kKeys);
                }
                const int early = pend[1] >= 0 && (pend[0] < 0 || pend[1] < pend[0]) ? 1 : 0;
                if (ok && pend[early] >= 0 && !issue_pv(early)) ok = false;
                if (ok && pend[early ^ 1] >= 0 && !issue_pv(early ^ 1)) ok = false;
                if (ok) { tc::mma_commit(&sh->o_full[0]); tc::mma_commit(&sh->o_full[1]); }
            }
            if (!ok) give_up(sh, p.status, 32);
        }
    } else if (warp < 4) {
        // ---------------- V rows that hold NaN or infinities ----------------
        int fill = 0;
        for (long long x = xbeg; x < xend && !failed;) {
            const Piece c = make_piece(pl, p, sp, x, xend);
            x += c.blk1 - c.blk0;
            BlockIter it;
            it.init(pl, c.ti, kKeys, c.blk0);
            for (int blk = c.blk0; blk < c.blk1; ++blk, ++fill) {
                const int st = fill % NS;
                if (!tc::mbar_wait(&sh->v_full[st], (uint32_t)(fill / NS) & 1u, abort_flag)) failed = true;
                failed = __any_sync(0xffffffffu, failed);
                if (failed) break;
                if (mixed(pl, c, it)) {
#pragma unroll 1
                    for (int rr = 0; rr < 2; ++rr) {
                        unsigned char* row = Vs + (size_t)st * kTile + ((warp - 2) * 64 + rr * 32 + lane) * 128;
                        uint32_t bad = 0u;
#pragma unroll
                        for (int i = 0; i < DH * 8; ++i) {
                            const uint4 w = *reinterpret_cast<const uint4*>(row + (i / 8) * (kKeys * 128) + (((i + lane) & 7) << 4));
                            // an exponent of all ones carries into the sign's place
                            bad |= ((w.x & 0x7f807f80u) + 0x00800080u) | ((w.y & 0x7f807f80u) + 0x00800080u) |
                                   ((w.z & 0x7f807f80u) + 0x00800080u) | ((w.w & 0x7f807f80u) + 0x00800080u);
                        }
                        if (bad & 0x80008000u) {
#pragma unroll
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
        const int grp = p.Hq / p.Hkv;
        const int W = (p.max_nodes + 63) / 64;
        const float sl2 = p.scale * kLog2e;                    // scores are kept in log2 units
        uint32_t s_count = 0u;
        int fill0 = 0, piece = 0;
        for (long long x = xbeg; x < xend; ++piece) {
            const Piece c = make_piece(pl, p, sp, x, xend);
            x += c.blk1 - c.blk0;
            // ---- this thread's row ----
            const int rt = (c.split_keys ? 0 : half * kHalf) + rl;      // row of the tile
            const bool live = rt < c.ti.nrows;
            int seq = -2, node = 0, row_pre = 0, row_kv = 0, row_n = 0;
            size_t orow = 0;
            unsigned long long m0 = 0ull, m1 = 0ull;
            const unsigned long long* mrow = p.mask;
            if (live) {
                const int pr = c.ti.row0 + rt;
                seq = plan_seq_of_row(pl, p.B, pr);
                const int o = pr - pl.row_off[seq];
                node = o / grp;
                orow = ((size_t)seq * p.max_nodes + node) * p.Hq + c.g * grp + (o - node * grp);
                row_pre = pl.pre[seq];
                row_kv = pl.kv[seq];
                row_n = pl.own_len[seq] - row_kv;
                mrow = p.mask + ((size_t)seq * p.max_nodes + node) * W;
                m0 = mrow[0];
                if (W > 1) m1 = mrow[1];
            }
            const bool warp_live = __any_sync(0xffffffffu, live);
            halves_barrier();                                   // the previous piece is done with Q's memory
            if (!c.split_keys || half == 0) {
                const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.Q) + orow * D);
                unsigned char* dst = Qs + half * kQHalf + rl * 128;
#pragma unroll
                for (int cc = 0; cc < D / 8; ++cc) {
                    const uint4 w = live ? __ldg(src + cc) : make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4*>(dst + (cc / 8) * (kHalf * 128) + (((cc % 8) ^ (rl & 7)) << 4)) = w;
                }
                tc::fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sh->q_full);

            float ref = -INFINITY, sum = 0.f;
            bool first = true;
            BlockIter it;
            it.init(pl, c.ti, kKeys, c.blk0);
            for (int blk = c.blk0; blk < c.blk1; ++blk) {
                if ((takers(c, it, blk) >> half) & 1u) {
                    if (!failed && !tc::mbar_wait(&sh->s_full[half], s_count & 1u, abort_flag)) failed = true;
                    ++s_count;
                    failed = __any_sync(0xffffffffu, failed);
                    if (failed) {
                        if (lane == 0) give_up(sh, p.status, 35);
                        break;
                    }
                    tc::tc_fence_after_sync();
                    if (warp_live) {
                        const bool all = !live || (it.seq < 0 ? it.key0 + kKeys <= row_pre : (it.seq == seq && it.key0 + kKeys <= row_kv));
                        const bool open = __all_sync(0xffffffffu, all);        // no row of the warp has anything masked
                        const bool none = !live || (it.seq < 0 ? it.key0 >= row_pre : it.seq != seq);
                        if (__all_sync(0xffffffffu, none)) {
                            // nothing to see for this warp: P is zero
                            uint32_t z[32];
#pragma unroll
                            for (int j = 0; j < 32; ++j) z[j] = 0u;
                            tc::tmem_st32(tmem_s, z);
                            tc::tmem_st32(tmem_s + 32u, z);
                        } else {
                            uint32_t v[4][32];
#pragma unroll
                            for (int cc = 0; cc < 4; ++cc) tc::tmem_ld32(tmem_s + (uint32_t)(cc * 32), v[cc]);
                            tc::tmem_ld_wait();
                            if (!open) {
#pragma unroll
                                for (int cc = 0; cc < 4; ++cc) {
                                    const uint32_t vis = live ? visible32_of(it.seq, it.key0 + cc * 32, seq, row_pre, row_kv, row_n, m0, m1, mrow, W) : 0u;
#pragma unroll
                                    for (int j = 0; j < 32; ++j) v[cc][j] = ((vis >> j) & 1u) ? v[cc][j] : 0xff800000u;
                                }
                            }
                            float b4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                            for (int cc = 0; cc < 4; ++cc)
#pragma unroll
                                for (int j = 0; j < 32; ++j) b4[j & 3] = fmaxf(b4[j & 3], __uint_as_float(v[cc][j]));
                            const float bm = fmaxf(fmaxf(b4[0], b4[1]), fmaxf(b4[2], b4[3])) * sl2;
                            const bool move = bm > ref + kSlack;               // also the first visible key (ref = -inf)
                            if (__any_sync(0xffffffffu, move)) {
                                const float corr = move ? exp2_fast(ref - bm) : 1.f;
                                // S of this block was issued after P V of the half's last one: O is at rest
                                if (!first) {
#pragma unroll 1
                                    for (int c0 = 0; c0 < D; c0 += 32) {
                                        uint32_t o[32];
                                        tc::tmem_ld32(tmem_o + (uint32_t)c0, o);
                                        tc::tmem_ld_wait();
#pragma unroll
                                        for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * corr);
                                        tc::tmem_st32(tmem_o + (uint32_t)c0, o);
                                    }
                                }
                                sum *= corr;
                                ref = move ? bm : ref;
                            }
                            const float off = ref == -INFINITY ? 0.f : -ref;
                            float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int hh = 0; hh < 2; ++hh) {
                                uint32_t w[32];
#pragma unroll
                                for (int j = 0; j < 32; ++j) {
                                    const int e = 2 * j;
                                    const float a = exp2_fast(fmaf(__uint_as_float(v[2 * hh + e / 32][e % 32]), sl2, off));
                                    const float b = exp2_fast(fmaf(__uint_as_float(v[2 * hh + e / 32][e % 32 + 1]), sl2, off));
                                    s4[(2 * j) & 3] += a;
                                    s4[(2 * j + 1) & 3] += b;
                                    w[j] = pack_bf16(a, b);
                                }
                                tc::tmem_st32(tmem_s + (uint32_t)(hh * 32), w);
                            }
                            sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
                        }
                        tc::tmem_st_wait();
                    }
                    first = false;
                    tc::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&sh->p_full[half]);
                }
                if (blk + 1 < c.blk1) it.next(pl, c.ti, kKeys);
            }
            // ---- the half's output is complete ----
            if (!failed && !tc::mbar_wait(&sh->o_full[half], (uint32_t)piece & 1u, abort_flag)) failed = true;
            failed = __any_sync(0xffffffffu, failed);
            if (failed && lane == 0) give_up(sh, p.status, 36);
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
                        for (int k = 0; k < kKeys; ++k) {
                            if (!((visible32_of(jt.seq, jt.key0 + (k & ~31), seq, row_pre, row_kv, row_n, m0, m1, mrow, W) >> (k & 31)) & 1u)) continue;
                            const uint32_t* vr = reinterpret_cast<const uint32_t*>(vb + (size_t)(jt.key0 + k) * D);
                            uint32_t bad = 0u;
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
                            tc::tmem_ld32(tmem_o + (uint32_t)c0, o);
                            tc::tmem_ld_wait();
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
                const float inv = c.whole ? (sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum)) : 1.f;
                const size_t part = (size_t)blockIdx.x * 2 + c.slot;
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.O) + orow * D;
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    float o[32];
                    if (!first) {
                        uint32_t u[32];
                        tc::tmem_ld32(tmem_o + (uint32_t)c0, u);
                        tc::tmem_ld_wait();
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
                    if (!live) continue;
                    if (c.whole) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint4 w;
                            w.x = pack_bf16(o[8 * j + 0] * inv, o[8 * j + 1] * inv);
                            w.y = pack_bf16(o[8 * j + 2] * inv, o[8 * j + 3] * inv);
                            w.z = pack_bf16(o[8 * j + 4] * inv, o[8 * j + 5] * inv);
                            w.w = pack_bf16(o[8 * j + 6] * inv, o[8 * j + 7] * inv);
                            *reinterpret_cast<uint4*>(out + c0 + 8 * j) = w;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            p.part_o[(part * (D / 4) + c0 / 4 + j) * kTcRows + rt] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                    }
                }
                if (live) {
                    if (!c.whole) p.part_ml[part * kTcRows + rt] = make_float2(ref, sum);
                    else if (p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * kLn2;
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
    CTCSD_CUDA_CHECK(h, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(h->num_sms), dim3(kThreads), smem, s, 1, tmKp, tmVp, tmK, tmV, p));
    h->launches++;
    return CTCSD_OK;
}

}  // namespace

int launch_shared_attention_tc(Handle* h, cudaStream_t s, const SharedAttnParams& p) {
    return p.D == 64 ? launch_tc<64>(h, s, p) : launch_tc<128>(h, s, p);
}

}  // namespace ctcsd
