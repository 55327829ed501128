// Tree attention over a 4-bit cache for bf16 on the 5th-generation tensor cores (tcgen05 + TMEM): more than 16 query rows of a kv head.
//
// Persistent CTAs, one per SM, each with a span of the line of key blocks (q4_attention.cuh).  A tile is TR query rows of a sequence, in halves of
// 128.  Per block of 128 keys four warps turn the levels of K and V into bfloat16 values, in the 128-byte-swizzled tiles that the
// products read (tree rows are copied); a block serves both halves, in two steps of 64 keys.  Per half and step:
//   S[128 x 64] = Q K^T      tcgen05.mma, operands in shared memory, S in tensor memory;
//   softmax                  one thread per query row: reads its 64 scores, P = 2^(S - ref) goes back as bf16, over the scores;
//   O[128 x D] += P V        tcgen05.mma with P from tensor memory, V as an MN-major operand.
// With at most 128 rows in a tile both halves work on the same rows, one on the even and one on the odd blocks, and each joins half of
// the columns of both outputs at the end (row r is lane r of both).
// ref, the exponent's reference, follows the row maximum lazily (only when it falls kSlack behind), so that O is hardly ever
// rescaled.  P is rounded to bf16, by 2^-8 of a weight at most, because a product takes both operands in one type and V is bf16; scores,
// references, sums (of the unrounded weights), O and the parts are float32.
//
// Warps 0 and 3 bring levels in by bulk copies, warps 1 and 2 issue the products of one half each, warps 4-7 and 8-11 are the softmax warps of the
// halves, 12-15 make the tiles.  All have 128 registers (168 for the softmax warps, taken from the others with setmaxnreg, made case B below
// 2 us slower).
//
// What bounds it: no unit, but what stands in line.  A step of 64 keys takes the softmax warps about 1300 cycles (the exponentials alone take their units 512
// for each of the two warps of a scheduler), and they wait another 450-1600 for its scores; where those go was not taken apart.  (With no waiting it would be
// 3100 cycles a block of 128 keys and 256 rows, 1570 TFLOP/s.)  A piece's beginning, last products and output take some 12,000 cycles, in which the next piece's Q
// cannot come, since its memory is also where outputs are turned; short sequences pay that often.
//   A: 32 sequences of 1024-4096 cached rows, 64 nodes, 64 query heads on 8 kv heads    228 us with the merge, 590 TFLOP/s (bfloat16 rows: 247 us)
//   B: 8 sequences of 512-2048 rows, 64 nodes, 32 heads of their own                     59 us with the merge (bfloat16 rows: 42 us)
//
// A weight of zero does not cancel a NaN.  Cached rows are seen by every row of the tile, and those behind the last are made zeros; a
// tree row whose value holds a NaN or an infinity is made zeros too and noted, and a row that does see it becomes NaN at the end.
#include "q4_ring.cuh"

#include <math.h>

namespace ctcsd {
namespace {

constexpr int kThreads = 512;
constexpr int kHalf = 128;             // rows per half
constexpr int kKeys = kAq4TcKeys;
constexpr int kStep = 64;              // keys weighed at a time
constexpr int kStages = 2;             // K and V tiles
constexpr int kMaxRaw = 16;
constexpr float kSlack = 8.f;          // log2 units: P stays below 2^8
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct __align__(8) TcShared {
    uint64_t q_full;
    uint64_t raw_full[kMaxRaw], raw_empty[kMaxRaw];
    uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
    uint64_t s_full[2][2], p_full[2][2];         // per half and step
    uint64_t pv_done[2], o_full[2];              // P V of a step; of the piece
    uint32_t tmem_base;
    int abort_flag, never_set;
    unsigned bad[4][8];                          // tree rows whose value is no number: of a piece (mod 4)
    float2 join[2][kHalf];                       // reference and sum of the halves' rows when both serve the same
};

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
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void give_up(TcShared* sh, int* status, int site) {
    volatile int* f = &sh->abort_flag;
    if (*f == 0) report_error(status, CTCSD_ERR_TIMEOUT, site);
    *f = 1;
}
// All softmax threads (both halves) meet here.
__device__ __forceinline__ void halves_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <bool B> struct Flag { static constexpr bool value = B; };

// Levels of a side come in whole blocks, or in halves where shared memory has room for three blocks' only.
template <int D, int TR> __host__ __device__ constexpr int raw_parts() { return D == 128 && TR == 256 ? 2 : 1; }

template <int D, int TR>
__global__ void __launch_bounds__(kThreads, 1) attention_q4_tc_kernel(AttnQ4Params p, int nraw) {
    constexpr int DH = D / 64;
    constexpr int kQHalf = kHalf * D * 2;
    constexpr int kTile = kKeys * D * 2;
    constexpr int kParts = raw_parts<D, TR>(), kPart = kKeys / kParts, kSlot = RawQ4<D>::bytes(kPart);
    extern __shared__ __align__(1024) unsigned char dyn[];
    unsigned char* Qs = dyn;                                   // [TR / 128][DH][128 rows][128 B]
    unsigned char* Ks = Qs + TR / kHalf * kQHalf;              // [kStages][DH][128 keys][128 B]
    unsigned char* Vs = Ks + kStages * kTile;
    unsigned char* raw = Vs + kStages * kTile;                 // [side][nraw][kPart rows]
    TcShared* sh = reinterpret_cast<TcShared*>(raw + 2 * nraw * kSlot);
    PlanQ4 pl;
    pl.carve(reinterpret_cast<int*>(sh + 1), p.B);
    if ((tc::smem_u32(dyn) & 1023u) != 0u) {                   // uniform over the CTA
        if (threadIdx.x == 0) report_error(p.status, CTCSD_ERR_INTERNAL, 61);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        tc::mbar_init(&sh->q_full, 8);
        for (int s = 0; s < 2 * nraw; ++s) { tc::mbar_init(&sh->raw_full[s], 2); tc::mbar_init(&sh->raw_empty[s], 2); }
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(&sh->k_full[s], 2); tc::mbar_init(&sh->k_empty[s], 2);
            tc::mbar_init(&sh->v_full[s], 2); tc::mbar_init(&sh->v_empty[s], 2);
        }
        for (int s = 0; s < 2; ++s) {
            for (int e = 0; e < 2; ++e) { tc::mbar_init(&sh->s_full[s][e], 1); tc::mbar_init(&sh->p_full[s][e], 4); }
            tc::mbar_init(&sh->pv_done[s], 1);
            tc::mbar_init(&sh->o_full[s], 1);
        }
        sh->abort_flag = 0;
        sh->never_set = 0;
        tc::fence_barrier_init();
    }
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
    const SpansQ4 sp = plan_q4_build(pl, p, TR, kKeys, (int)gridDim.x);
    bool failed = false;
    WalkQ4 at;
    bool more = at.init(pl, sp, p.B, kKeys, blockIdx.x);
    attn_q4_sides<__nv_bfloat16, D>(p, pl, sp, at, more);

    if (warp < 4) {
        if (warp == 0 || warp == 3) {
            // ---------------- levels: of K and of V ----------------
            if (lane == 0) {
                const int side = warp == 0 ? 0 : 1;
                const uint64_t pol = tc::policy_evict_last();
                const long long rows = (long long)p.B * p.Hkv * p.Lcap;
                unsigned char* ring = raw + side * nraw * kSlot;
                uint64_t *full = sh->raw_full + side * nraw, *empty = sh->raw_empty + side * nraw;
                int s = 0, fill = 0;
                uint32_t phase = 1u;
                for (; more && !failed; more = at.next(pl, p.B, kKeys)) {
                    const long long base = ((long long)at.b * p.Hkv + at.g) * p.Lcap;
                    const int kv = pl.kv[at.b];
                    for (int row = at.blk0 * kKeys; row < at.blk1 * kKeys && row < kv; row += kPart, ++fill) {
                        const int n = kv - row < kPart ? kv - row : kPart;
                        if (!tc::mbar_wait_ready(empty + s, phase, abort_flag)) { failed = true; break; }
                        RawQ4<D>::request_levels(ring + s * kSlot, side ? p.Vq : p.Kq, base + row, n, full + s, pol);
                        RawQ4<D>::request_pairs(ring + s * kSlot, side ? p.Vs : p.Ks, kPart, base + row, n, rows, full + s, pol);
                        if (++s == nraw) { s = 0; phase ^= 1u; }
                    }
                }
                if (failed) {
                    give_up(sh, p.status, 62);
                    for (int back = 1; back <= nraw && back <= fill; ++back) {              // copies in flight land before the exit
                        const int j = fill - back;
                        tc::mbar_wait_suspended(full + j % nraw, (uint32_t)(j / nraw) & 1u, &sh->never_set, 1ll << 24);
                    }
                }
            }
        } else if (warp < 3) {
            // ---------------- products of one half ----------------
            // Both issuers visit every tile in order; for a block that is not its half's, an issuer only hands the tiles back.  The whole warp goes
            // through the loops and one lane issues, so that descriptors stay in uniform registers.
            const int half = warp - 1;
            const uint32_t idesc_s = tc::idesc_bf16_f32(kHalf, kStep);
            const uint32_t idesc_o = tc::idesc_bf16_f32_b_mn(kHalf, D);
            const uint32_t tmem_s = tmem + (uint32_t)(half * 128), tmem_o = tmem + 256u + (uint32_t)(half * D);
            const uint64_t kdesc0 = tc::smem_desc_k_sw128(tc::smem_u32(Ks));
            const uint64_t vdesc0 = tc::smem_desc_mn_sw128(tc::smem_u32(Vs), kKeys * 128);
            int fill = 0, piece = 0;
            uint32_t count = 0u;                               // blocks whose P this issuer has waited for
            bool ok = true;
            auto wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, tc::mbar_wait_ready(bar, parity, abort_flag)) != 0; };
            for (; more && ok; more = at.next(pl, p.B, kKeys), ++piece) {
                const bool split = TR == kHalf || pl.n[at.b] * p.grp - at.t * TR <= kHalf;
                const uint64_t qdesc0 = tc::smem_desc_k_sw128(tc::smem_u32(Qs + (split ? 0 : half * kQHalf)));
                int pend = -1;                                 // block (fill number) whose P V is still to be issued
                bool first = true;
                auto issue_pv = [&](int e) -> bool {
                    const int st = pend % kStages;
                    if (e == 0 && !wait(&sh->v_full[st], (uint32_t)(pend / kStages) & 1u)) return false;
                    if (!wait(&sh->p_full[half][e], count & 1u)) return false;
                    tc::tc_fence_after_sync();
                    if (tc::elect_one()) {
                        const uint64_t vdesc = vdesc0 + (uint64_t)((st * kTile + e * kStep * 128) >> 4);
#pragma unroll
                        for (int kk = 0; kk < kStep / 16; ++kk)               // 16 keys: 8 columns of P, 16 rows of V
                            tc::mma_bf16_ts(tmem_o, tmem_s + (uint32_t)(e * kStep + kk * 8), vdesc + (uint64_t)((kk * 16 * 128) >> 4), idesc_o,
                                            !first || kk != 0 ? 1u : 0u);
                        tc::mma_commit(&sh->pv_done[half]);
                        if (e == 1) tc::mma_commit(&sh->v_empty[st]);
                    }
                    __syncwarp();
                    first = false;
                    if (e == 1) ++count;
                    return true;
                };
                auto issue_s = [&](int e, int st) {
                    if (tc::elect_one()) {
                        const uint64_t kdesc = kdesc0 + (uint64_t)((st * kTile + e * kStep * 128) >> 4);
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint64_t along = (uint64_t)((kk / 4) * ((kHalf * 128) >> 4) + 2 * (kk % 4));
                            tc::mma_bf16_ss(tmem_s + (uint32_t)(e * kStep), qdesc0 + along, kdesc + along, idesc_s, kk != 0 ? 1u : 0u);
                        }
                        tc::mma_commit(&sh->s_full[half][e]);
                        if (e == 1) tc::mma_commit(&sh->k_empty[st]);
                    }
                    __syncwarp();
                };
                ok = wait(&sh->q_full, (uint32_t)piece & 1u);
                // (one more round than blocks: the last block's P V)
                for (int blk = at.blk0; blk <= at.blk1 && ok; ++blk) {
                    const int st = fill % kStages;
                    const uint32_t ph = (uint32_t)(fill / kStages) & 1u;
                    const bool more_blocks = blk < at.blk1;
                    const bool mine = more_blocks && (!split || ((blk - at.blk0) & 1) == half);
                    // a step's P is read by P V before the next S overwrites it: the tensor core works in issue order
#pragma unroll 1
                    for (int e = 0; e < 2 && ok; ++e) {
                        if (pend >= 0) ok = issue_pv(e);
                        if (ok && mine) {
                            if (e == 0) {
                                ok = wait(&sh->k_full[st], ph);
                                tc::tc_fence_after_sync();
                            }
                            if (ok) issue_s(e, st);
                        }
                    }
                    if (!ok || !more_blocks) break;
                    pend = mine ? fill : -1;
                    if (!mine) {
                        ok = wait(&sh->k_full[st], ph);
                        if (ok && lane == 0) tc::mbar_arrive(&sh->k_empty[st]);
                        ok = ok && wait(&sh->v_full[st], ph);
                        if (ok && lane == 0) tc::mbar_arrive(&sh->v_empty[st]);
                        __syncwarp();
                    }
                    ++fill;
                }
                if (ok && tc::elect_one()) tc::mma_commit(&sh->o_full[half]);
                __syncwarp();
            }
            if (!ok && lane == 0) give_up(sh, p.status, 63);
        }
    } else if (warp >= 12) {
        // ---------------- tiles of values ----------------
        // Two warps make K's tiles, two V's.
        const int mw = (warp - 12) & 1, side = (warp - 12) >> 1;
        // levels: a lane takes chunk c (32 values) of a row, 8 rows (D = 64: 16) at a time.  Its four words go to four 16-byte places of the row; lanes of
        // the upper 64 columns begin with word 2, so that a store's lanes meet in no bank.
        constexpr int CH = D / 32, RI = 32 / CH;               // chunks of a row, rows an instruction
        const int c = lane % CH, r0 = mw * (kPart / 2) + lane / CH, turn = (c >> 1) << 1;
        unsigned put[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) put[i] = (c >> 1) * (kKeys * 128) + (((((c & 1) << 2) | (i ^ turn)) ^ (r0 & 7)) << 4);
        const unsigned char* ring = raw + side * nraw * kSlot;
        uint64_t *full = sh->raw_full + side * nraw, *empty = sh->raw_empty + side * nraw;
        int s = 0, fill = 0, piece = 0;
        uint32_t phase = 0u;
        for (; more && !failed; more = at.next(pl, p.B, kKeys), ++piece) {
            const size_t pair = (size_t)at.b * p.Hkv + at.g;
            const int kv = pl.kv[at.b], n = pl.n[at.b];
            for (int blk = at.blk0; blk < at.blk1 && !failed; ++blk, ++fill) {
                const int st = fill % kStages;
                const uint32_t ph = ((uint32_t)(fill / kStages) & 1u) ^ 1u;
                unsigned char* tile = (side ? Vs : Ks) + st * kTile;
                if (!tc::mbar_wait_ready(side ? &sh->v_empty[st] : &sh->k_empty[st], ph, abort_flag)) failed = true;
                if (blk < at.cached) {
#pragma unroll 1
                    for (int part = 0; part < kParts; ++part) {
                        const int row = blk * kKeys + part * kPart, left = kv - row;       // rows there are
                        if (!failed && left > 0 && !tc::mbar_wait_ready(full + s, phase, abort_flag)) failed = true;
                        failed = __any_sync(0xffffffffu, failed);
                        if (failed) break;
                        const unsigned char* from = ring + s * kSlot;
                        const uint32_t* so = RawQ4<D>::pairs(from, kPart, (long long)pair * p.Lcap + row);
                        unsigned char* to = tile + part * (kPart * 128);
#pragma unroll 2
                        for (int i0 = 0; i0 < kPart / 2; i0 += RI) {
                            const int r = r0 + i0;
                            uint4 u = make_uint4(0u, 0u, 0u, 0u);
                            uint32_t pr = 0u;                  // (behind the last row: zeros, whatever stands there)
                            if (r < left) {
                                u = *reinterpret_cast<const uint4*>(from + r * RawQ4<D>::kLevels + c * 16);
                                pr = so[r * CH + c];
                            }
                            const uint32_t w[4] = {turn ? u.z : u.x, turn ? u.w : u.y, turn ? u.x : u.z, turn ? u.y : u.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(to + r * 128 + put[i]) = q4_values_bf16(w[i], pr);
                        }
                        __syncwarp();
                        if (left > 0) {
                            if (lane == 0) tc::mbar_arrive(empty + s);
                            if (++s == nraw) { s = 0; phase ^= 1u; }
                        }
                    }
                    if (failed) break;
                } else {
                    failed = __any_sync(0xffffffffu, failed);
                    if (failed) break;
                    // the tree's own rows, one a lane
                    const int tb = blk - at.cached;
#pragma unroll 1
                    for (int i32 = mw * 2; i32 < mw * 2 + 2; ++i32) {
                        const int r = i32 * 32 + lane, row = tb * kKeys + r;
                        const uint4* src = static_cast<const uint4*>(side ? p.Vt : p.Kt) + (pair * p.max_nodes + (row < n ? row : 0)) * (D / 8);
                        bool is_bad = false;
#pragma unroll 1
                        for (int h = 0; h < DH; ++h) {
                            uint4 v[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = row < n ? __ldg(src + h * 8 + i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                // (an exponent of ones carries into the bit above it)
                                const uint32_t e = ((v[i].x & 0x7f807f80u) + 0x00800080u) | ((v[i].y & 0x7f807f80u) + 0x00800080u) |
                                                   ((v[i].z & 0x7f807f80u) + 0x00800080u) | ((v[i].w & 0x7f807f80u) + 0x00800080u);
                                is_bad = is_bad || (e & 0x80008000u) != 0u;
                                *reinterpret_cast<uint4*>(tile + h * (kKeys * 128) + r * 128 + ((i ^ (r & 7)) << 4)) = v[i];
                            }
                        }
                        if (side) {
                            if (is_bad)
#pragma unroll 1
                                for (int i = 0; i < DH * 8; ++i)
                                    *reinterpret_cast<uint4*>(tile + (i >> 3) * (kKeys * 128) + r * 128 + ((i & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                            const unsigned word = __ballot_sync(0xffffffffu, is_bad);
                            if (lane == 0) sh->bad[piece & 3][tb * 4 + i32] = word;
                        }
                    }
                }
                tc::fence_proxy_async();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(side ? &sh->v_full[st] : &sh->k_full[st]);
            }
        }
        if (failed && lane == 0) give_up(sh, p.status, 64);
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
        const int MW = (p.max_nodes + 63) / 64;
        const float sl2 = p.scale * kLog2e;                    // scores are kept in log2 units
        const uint64_t sl22 = pair_of(sl2, sl2);
        uint32_t s_count = 0u, steps = 0u;                     // blocks and steps of this half so far
        int piece = 0;
        // After a wait that ran out, nothing is waited for any more: the loops run to their ends on meaningless scores,
        // and no output is written.
        auto wait = [&](uint64_t* bar, uint32_t parity, int site) {
            if (!failed && !tc::mbar_wait_ready(bar, parity, abort_flag)) {
                failed = true;
                give_up(sh, p.status, site);
            }
        };
        for (; more; more = at.next(pl, p.B, kKeys), ++piece) {
            const int kv = pl.kv[at.b], n = pl.n[at.b], row0 = at.t * TR;
            const int nrows = n * grp - row0 < TR ? n * grp - row0 : TR;
            const bool split = TR == kHalf || nrows <= kHalf;
            // ---- this thread's row ----
            const int rt = (split ? 0 : half * kHalf) + rl;    // row of the tile
            const bool live = rt < nrows, warp_live = (split ? 0 : half * kHalf) + q * 32 < nrows;
            const int node = live ? (row0 + rt) / grp : 0;
            // (below 2^32: as many rows of 64 columns fill no GPU's memory)
            const unsigned orow = live ? ((unsigned)at.b * p.max_nodes + node) * p.Hq + at.g * grp + (row0 + rt - node * grp) : 0u;
            const unsigned long long* mrow = p.mask + ((size_t)at.b * p.max_nodes + node) * MW;
            halves_barrier();                                  // the previous piece is done with Q's memory
            if (!split || half == 0) {
                // neighbouring lanes take neighbouring 16 bytes of a row
                constexpr int LR = D / 8, RI = 32 / LR;        // lanes per row, rows per instruction
                unsigned char* dst = Qs + half * kQHalf + (q * 32) * 128;
                const int cc = lane % LR;
                const unsigned there = __ballot_sync(0xffffffffu, live);
                const uint4* Qg = static_cast<const uint4*>(p.Q) + cc;
                uint4 w[LR];                                   // (all loads at once: a piece waits for them once)
#pragma unroll
                for (int i = 0; i < LR; ++i)                   // (a row that is not there reads row 0)
                    w[i] = __ldg(Qg + (size_t)__shfl_sync(0xffffffffu, orow, i * RI + lane / LR) * LR);
#pragma unroll
                for (int i = 0; i < LR; ++i) {
                    const int rr = i * RI + lane / LR;
                    if (!((there >> rr) & 1u)) w[i] = make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4*>(dst + rr * 128 + (cc / 8) * (kHalf * 128) + (((cc % 8) ^ (rr & 7)) << 4)) = w[i];
                }
                tc::fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sh->q_full);

            float ref = -INFINITY, sum = 0.f;
            bool first = true, poisoned = false;
            // One step of a block.  Open: the row sees all keys; else those of vis (two words).  (Two copies of the code: with the masks inside the loop of
            // open blocks, which is most of them, its instructions take longer to fetch.)
            auto step = [&](auto open_tag, int e, uint32_t vis0, uint32_t vis1) {
                constexpr bool Open = decltype(open_tag)::value;
                const uint32_t tmem_se = tmem_s + (uint32_t)(e * kStep);
                const bool none = !Open && __all_sync(0xffffffffu, (vis0 | vis1) == 0u);
                wait(&sh->s_full[half][e], s_count & 1u, 65);
                __syncwarp();
                tc::tc_fence_after_sync();
                if (!warp_live) {
                    // rows that are not there: P is not looked at
                } else if (!Open && none) {
                    uint32_t z[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) z[j] = 0u;
                    tc::tmem_st32(tmem_se, z);
                } else {
                    uint32_t v[64];
                    tc::tmem_read64(tmem_se, v);
                    if (!Open) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            v[j] = ((vis0 >> j) & 1u) ? v[j] : 0xff800000u;
                            v[32 + j] = ((vis1 >> j) & 1u) ? v[32 + j] : 0xff800000u;
                        }
                    }
                    float b4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < 64; j += 2)
                        b4[(j >> 1) & 3] = max3_nan(b4[(j >> 1) & 3], __uint_as_float(v[j]), __uint_as_float(v[j + 1]));
                    float bm = max3_nan(max3_nan(b4[0], b4[1], b4[2]), b4[3], -INFINITY);
                    poisoned = poisoned || !(bm < INFINITY);       // a NaN or +inf score: the row is not meaningful
                    bm *= sl2;
                    const bool move = bm > ref + kSlack;           // also the first visible key (ref = -inf)
                    if (__builtin_expect(__any_sync(0xffffffffu, move), 0)) {
                        const float corr = move ? exp2_q4(ref - bm) : 1.f;
                        if (!first) {
                            // O must be at rest: P V of the step before (older ones precede this step's scores)
                            wait(&sh->pv_done[half], (steps - 1u) & 1u, 65);
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
                    // eight pairs at a time, stage by stage: the pairs' chains (scale, exponential, sum, round) run side by side
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
                            lo[i] = exp2_q4(lo[i]);
                            hi[i] = exp2_q4(hi[i]);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) s2[i % 4] = add2(s2[i % 4], pair_of(lo[i], hi[i]));
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[g0 + i] = pack_bf16(lo[i], hi[i]);
                    }
                    float sa, sb;
                    pair_split(add2(add2(s2[0], s2[1]), add2(s2[2], s2[3])), sa, sb);
                    tc::tmem_st32(tmem_se, w);                     // over scores that have been read
                    sum += sa + sb;
                }
                first = false;
                ++steps;
                tc::tmem_st_wait();
                tc::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sh->p_full[half][e]);
            };
            const int by = split ? 2 : 1;
            int blk = at.blk0 + (split ? half : 0);
            const int open_to = min(at.blk1, kv / kKeys);          // blocks that every row sees whole
#pragma unroll 1
            for (; blk < open_to; blk += by, ++s_count)
#pragma unroll 1
                for (int e = 0; e < 2; ++e) step(Flag<true>(), e, 0u, 0u);
#pragma unroll 1
            for (; blk < at.blk1; blk += by, ++s_count)
#pragma unroll 1
                for (int e = 0; e < 2; ++e) {
                    uint32_t vis[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int key = (blk < at.cached ? blk : blk - at.cached) * kKeys + e * kStep + 32 * i;
                        const int left = kv - key;
                        if (blk < at.cached) vis[i] = left >= 32 ? 0xffffffffu : (left > 0 ? (1u << left) - 1u : 0u);
                        else vis[i] = live ? tree_bits32(mrow, MW, key, n) : 0u;
                    }
                    step(Flag<false>(), e, vis[0], vis[1]);
                }
            // ---- the half's output is complete ----
            wait(&sh->o_full[half], (uint32_t)piece & 1u, 66);
            failed = __any_sync(0xffffffffu, failed);
            tc::tc_fence_after_sync();
            // a row that saw a tree row that was cleared: NaN
            if (live && at.blk1 > at.cached) {
                const int t0 = (at.blk0 > at.cached ? at.blk0 - at.cached : 0) * 4, t1 = min((at.blk1 - at.cached) * 4, (n + 31) / 32);
#pragma unroll 1
                for (int i = t0; i < t1; ++i) {
                    // (of the blocks that this half took: the others' notes may not be there yet, and their half looks at them)
                    if (split && ((at.cached + (i >> 2) - at.blk0) & 1) != half) continue;
                    const unsigned cleared = *(volatile unsigned*)&sh->bad[piece & 3][i];
                    if (cleared != 0u && (cleared & tree_bits32(mrow, MW, i * 32, n)) != 0u) poisoned = true;
                }
            }
            if (poisoned) sum = __uint_as_float(0x7fc00000u);
            float mine = 1.f, other = 0.f;                      // weights of this half's output and of the other's
            if (first) { ref = -INFINITY; sum = 0.f; }
            bool other_there = false;
            if (split) {
                sh->join[half][rl] = make_float2(ref, sum);
                halves_barrier();                               // both outputs are complete
                tc::tc_fence_after_sync();
                const float2 o = sh->join[half ^ 1][rl];
                const float top = fmaxf(ref, o.x), base = top == -INFINITY ? 0.f : top;
                mine = exp2_q4(ref - base);
                other = exp2_q4(o.x - base);
                sum = (half == 0 ? sum * mine + o.y * other : o.y * other + sum * mine);
                other_there = at.blk1 - at.blk0 > (half ^ 1);   // (the other half had a block; one without has no output)
                if (ref == -INFINITY) mine = 0.f;
                if (o.x == -INFINITY) other = 0.f;
                ref = top;
            }
            // ---- output: this thread's row (of the halves' common rows, half of the columns) ----
            if (!failed && *abort_flag == 0 && warp_live) {
                const bool whole = at.whole();
                const float inv = whole ? (sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum)) : 1.f;
                const size_t part = (size_t)blockIdx.x * 2 + at.slot();
                const int c_lo = split ? half * (D / 2) : 0, c_hi = split ? c_lo + D / 2 : D;
                const uint32_t tmem_other = tmem + 256u + (uint32_t)((half ^ 1) * D) + lane_off;
                // Whole rows go through Q's memory, which no product reads any more, so that neighbouring lanes write neighbouring 16 bytes (a row a lane took
                // 32 lines an instruction).
                unsigned char* stage = Qs + (split ? 0 : half * kQHalf) + (q * 32) * 128;
                // (16 columns at a time: code that runs once a piece is mostly fetched, so it is kept short)
                if (first) mine = 0.f;
                if (!other_there) other = 0.f;
                mine *= inv;
                other *= inv;
#pragma unroll 1
                for (int c0 = c_lo; c0 < c_hi; c0 += 16) {
                    float o[16];
                    uint32_t u[16];
                    tc::tmem_read16(tmem_o + (uint32_t)c0, u);
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = mine != 0.f ? __uint_as_float(u[j]) * mine : 0.f;
                    if (split) {
                        tc::tmem_read16(tmem_other + (uint32_t)c0, u);
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = other != 0.f ? fmaf(__uint_as_float(u[j]), other, o[j]) : o[j];
                    }
                    if (whole) {
                        unsigned char* to = stage + (c0 / 64) * (kHalf * 128) + lane * 128;
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            *reinterpret_cast<uint4*>(to + (((c0 % 64 / 8 + j) ^ (lane & 7)) << 4)) =
                                make_uint4(pack_bf16(o[8 * j], o[8 * j + 1]), pack_bf16(o[8 * j + 2], o[8 * j + 3]), pack_bf16(o[8 * j + 4], o[8 * j + 5]),
                                           pack_bf16(o[8 * j + 6], o[8 * j + 7]));
                    } else if (live && CTCSD_IN_BOUNDS(p.status, 152, part * TR + rt, 2ll * gridDim.x * TR)) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            p.part_o[(part * (D / 4) + c0 / 4 + j) * TR + rt] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                    }
                }
                if (whole) {
                    const unsigned there = __ballot_sync(0xffffffffu, live);
                    const int per = (c_hi - c_lo) / 8, c = c_lo / 8 + lane % per;          // 16-byte places of a row; this lane's
                    __syncwarp();
#pragma unroll 4
                    for (int r0 = 0; r0 < 32; r0 += 32 / per) {
                        const int rr = r0 + lane / per;
                        const unsigned row = __shfl_sync(0xffffffffu, orow, rr);
                        const uint4 w = *reinterpret_cast<const uint4*>(stage + (c / 8) * (kHalf * 128) + rr * 128 + (((c % 8) ^ (rr & 7)) << 4));
                        if (((there >> rr) & 1u) && CTCSD_IN_BOUNDS(p.status, 151, row, out_rows(p))) static_cast<uint4*>(p.O)[(size_t)row * (D / 8) + c] = w;
                    }
                    __syncwarp();
                }
                if (live && (!split || half == 0)) {
                    if (!whole) {
                        if (CTCSD_IN_BOUNDS(p.status, 153, part * TR + rt, 2ll * gridDim.x * TR)) p.part_ml[part * TR + rt] = make_float2(ref, sum);
                    } else if (p.lse && CTCSD_IN_BOUNDS(p.status, 154, orow, out_rows(p))) {
                        p.lse[orow] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * kLn2;
                    }
                }
            }
            tc::tc_fence_before_sync();
            // (the other half may read this one's output: the next piece's first P V waits for Q, and Q for both halves at the barrier above)
        }
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc(tmem, 512);
    }
}

template <int D, int TR>
int launch_tc(Handle* h, cudaStream_t s, const AttnQ4Params& p) {
    const size_t fixed = (size_t)TR * D * 2 + (size_t)kStages * 2 * kKeys * D * 2 + sizeof(TcShared) + sizeof(int) * PlanQ4::ints(p.B);
    const size_t slots = 2 * (size_t)RawQ4<D>::bytes(kKeys / raw_parts<D, TR>());      // one of each side
    size_t n = (kMaxDynamicSmem - 1024 - fixed) / slots;
    if (n > kMaxRaw / 2) n = kMaxRaw / 2;
    if (n < 1) return CTCSD_ERR_UNSUPPORTED;
    auto kern = attention_q4_tc_kernel<D, TR>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepAttnQ4Tc, kern));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(h->num_sms), dim3(kThreads), fixed + n * slots, s, 1, p, (int)n));
    h->launches++;
    return CTCSD_OK;
}

}  // namespace

int launch_attention_q4_tc(Handle* h, cudaStream_t s, const AttnQ4Params& p, int TR) {
    if (TR == 128) return p.D == 64 ? launch_tc<64, 128>(h, s, p) : launch_tc<128, 128>(h, s, p);
    return p.D == 64 ? launch_tc<64, 256>(h, s, p) : launch_tc<128, 256>(h, s, p);
}

}  // namespace ctcsd
