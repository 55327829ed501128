// Tree attention over a 4-bit cache for bf16 and few query rows (up to 16 of a kv head): plain decoding and small trees.
//
// Besides its bytes it has 256 levels a key to make values.  So levels go from shared memory
// to the registers that the matrix instruction (mma.m16n8k16, 16 query rows) reads, and nowhere else:
//   S = Q K^T   a lane holds the K operand of one key in a quarter of the head dimension: 16 bytes of levels of that row, in order, since the
//               order of the summed index is free as long as Q has it too;
//   O += P V    a lane's S fragment is its P fragment; the V operand pairs two keys of a column, and a lane takes the same bytes
//               of four rows and joins halves of words, D/8 columns of its own (the order of columns is free as well).
// One shift-and-or and half a multiply-add per value.  A warp takes 16 keys of every block and keeps maximum, sum and O of its own;
// the warps' are joined when a tile ends.  Four warps bring the blocks in by bulk copies, up to five of them (150 KB) ahead.
// P is rounded to bfloat16, by 2^-8 of a weight at most, because a product takes both operands in one type and V is bfloat16; scores, references,
// sums (of the unrounded weights), O and the parts are float32.
//
// One token of 40 heads over 16001-32767 rows, batch 4: 202 us, 3.2 TB/s (bfloat16 rows: 395 us).  Latency bounds it: three warps of a scheduler go
// through levels, S, two shuffles, exponentials, levels and P V in turn (0.51 instructions a cycle and scheduler, ALU pipe 47 %, mma.sync 27 %, DRAM 32 %).
#include "q4_ring.cuh"

#include <math.h>

namespace ctcsd {
namespace {

constexpr int kWarps = 12;
constexpr int kProducers = 4;            // of K's levels and pairs, V's levels and pairs
constexpr int kThreads = (kWarps + kProducers) * 32;
constexpr int kRows = kAq4MmaRows;
constexpr int kKeys = kAq4MmaKeys;
constexpr int kMaxStages = 16;
constexpr float kSlack = 8.f;            // log2 units: P stays below 2^8
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
static_assert(kKeys == kWarps * 16 && kWarps % 4 == 0, "a warp takes 16 keys of a block");

struct __align__(8) MmaShared {
    uint64_t full[kMaxStages], empty[kMaxStages];
    int abort_flag, never_set;
    float ref[kWarps][kRows], sum[kWarps][kRows];
};

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// The consumer warps meet here.
__device__ __forceinline__ void consumers_barrier() { asm volatile("bar.sync 1, 384;" ::: "memory"); }

// Place of 16-byte chunk c of row r in the buffer that joins the warps' outputs: the eight lanes of a phase write to eight banks.
template <int D> __device__ __forceinline__ int join_at(int r, int c) {
    constexpr int per = D / 16;                              // chunks of a lane
    const int t = c / per, i = c % per;
    const int f = per == 8 ? i ^ (t + 4 * (r & 1)) : i ^ ((t >> 1) + 2 * (r & 1));
    return r * (D / 4) + t * per + f;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) attention_q4_mma_kernel(AttnQ4Params p, int nstages) {
    constexpr int LW = D / 32;                               // words of a K row that a lane takes
    constexpr int VW = D / 64;                               // words of a V row that a lane takes
    constexpr int NT = D / 8;                                // column tiles of O
    constexpr int kSide = RawQ4<D>::bytes(kKeys);
    extern __shared__ __align__(128) unsigned char dyn[];
    unsigned char* ring = dyn;                               // [nstages][K side | V side]
    uint4* join = reinterpret_cast<uint4*>(ring + (size_t)nstages * 2 * kSide);      // [4][16][D/4] of four floats
    uint4* qs = join + 4 * kRows * (D / 4);                  // [2 LW][32 lanes]: Q as operand A
    MmaShared* sh = reinterpret_cast<MmaShared*>(qs + 2 * LW * 32);
    PlanQ4 pl;
    pl.carve(reinterpret_cast<int*>(sh + 1), p.B);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        for (int s = 0; s < nstages; ++s) { tc::mbar_init(&sh->full[s], kProducers); tc::mbar_init(&sh->empty[s], kWarps); }
        sh->abort_flag = 0;
        sh->never_set = 0;
        tc::fence_barrier_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    const SpansQ4 sp = plan_q4_build(pl, p, kRows, kKeys, (int)gridDim.x);
    WalkQ4 at;
    bool more = at.init(pl, sp, p.B, kKeys, blockIdx.x);
    attn_q4_sides<__nv_bfloat16, D>(p, pl, sp, at, more);
    if (warp >= kWarps) {
        // ---------------- producers ----------------
        // (a thread spends some 600 cycles on a request: one for all four arrays took as long as the block's copies, 281 us for 13B tokens
        // over 16001-32767 rows)
        const int what = warp - kWarps;
        if (lane == 0) {
            const uint64_t pol = tc::policy_evict_first();
            const long long rows = (long long)p.B * p.Hkv * p.Lcap;
            int fill = 0, s = 0;
            uint32_t phase = 1u;
            bool failed = false;
            for (; more && !failed; more = at.next(pl, p.B, kKeys)) {
                const long long base = ((long long)at.b * p.Hkv + at.g) * p.Lcap;
                const int kv = pl.kv[at.b];
                for (int blk = at.blk0; blk < at.blk1 && blk < at.cached; ++blk, ++fill) {
                    if (!tc::mbar_wait_ready(&sh->empty[s], phase, abort_flag)) { failed = true; break; }
                    const long long row0 = base + (long long)blk * kKeys;
                    const int n = kv - blk * kKeys < kKeys ? kv - blk * kKeys : kKeys;
                    unsigned char* dst = ring + (size_t)s * 2 * kSide;
                    if (what & 1) RawQ4<D>::request_pairs(dst + (what >> 1) * kSide, what >> 1 ? p.Vs : p.Ks, kKeys, row0, n, rows, &sh->full[s], pol);
                    else RawQ4<D>::request_levels(dst + (what >> 1) * kSide, what >> 1 ? p.Vq : p.Kq, row0, n, &sh->full[s], pol);
                    if (++s == nstages) { s = 0; phase ^= 1u; }
                }
            }
            if (failed) {
                if (*abort_flag == 0) report_error(p.status, CTCSD_ERR_TIMEOUT, 51);
                *abort_flag = 1;
                for (int back = 1; back <= nstages && back <= fill; ++back) {            // copies in flight land before the exit
                    const int j = fill - back;
                    tc::mbar_wait_suspended(&sh->full[j % nstages], (uint32_t)(j / nstages) & 1u, &sh->never_set, 1ll << 24);
                }
            }
        }
        return;
    }
    // ---------------- products and softmax ----------------
    // (after a wait that ran out nothing is waited for any more, and no output is written: every warp goes on to every barrier)
    const int g = lane >> 2, t = lane & 3;
    const int MW = (p.max_nodes + 63) / 64;
    const float sl2 = p.scale * kLog2e;
    int st = 0;                                              // stage of the ring, and its turn
    uint32_t phase = 0u;
    bool failed = false;
    for (; more; more = at.next(pl, p.B, kKeys)) {
        const int b = at.b, kv = pl.kv[b], n = pl.n[b], row0 = at.t * kRows;
        const int nrows = n * p.grp - row0 < kRows ? n * p.grp - row0 : kRows;
        const size_t pair = (size_t)b * p.Hkv + at.g;
        auto out_row = [&](int r) -> size_t {
            const int node = (row0 + r) / p.grp;
            return ((size_t)b * p.max_nodes + node) * p.Hq + at.g * p.grp + (row0 + r - node * p.grp);
        };
        // Q as operand A: rows g and g + 8, elements D/4 t .. of the head
        // (in shared memory, for the registers' sake: with eight warps that held it, two to a scheduler, instructions waited for one another and 13B
        // tokens took 265 us; twelve: 202 us)
        if (warp < LW) {
            const uint4 z = make_uint4(0u, 0u, 0u, 0u);
            const uint4* Qg = static_cast<const uint4*>(p.Q);
            const uint4 a = g < nrows ? __ldg(Qg + out_row(g) * (D / 8) + t * LW + warp) : z;
            const uint4 b8 = g + 8 < nrows ? __ldg(Qg + out_row(g + 8) * (D / 8) + t * LW + warp) : z;
            qs[(2 * warp) * 32 + lane] = make_uint4(a.x, b8.x, a.y, b8.y);
            qs[(2 * warp + 1) * 32 + lane] = make_uint4(a.z, b8.z, a.w, b8.w);
        }
        consumers_barrier();
        float o[NT][4], ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) o[i][q] = 0.f;
        bool poisoned[2] = {false, false};
        // scores of 16 keys (two tiles of 8) against the reference -> P as operand A; s: masked scores
        const bool upper = nrows > 8;                            // rows 8 .. are there
        auto weigh = [&](float (&s)[2][4], uint32_t (&pa)[4]) __attribute__((always_inline)) {
            float bm[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (r == 1 && !upper) continue;
                bm[r] = max_nan(max_nan(s[0][2 * r], s[0][2 * r + 1]), max_nan(s[1][2 * r], s[1][2 * r + 1]));
                bm[r] = max_nan(bm[r], __shfl_xor_sync(0xffffffffu, bm[r], 1));
                bm[r] = max_nan(bm[r], __shfl_xor_sync(0xffffffffu, bm[r], 2));
                poisoned[r] = poisoned[r] || !(bm[r] < INFINITY);
                bm[r] *= sl2;
            }
            const bool move = bm[0] > ref[0] + kSlack || bm[1] > ref[1] + kSlack;
            if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float top = bm[r] > ref[r] + kSlack ? bm[r] : ref[r];
                    const float corr = top == ref[r] ? 1.f : exp2_q4(ref[r] - top);
                    ref[r] = top;
                    sum[r] *= corr;
#pragma unroll
                    for (int i = 0; i < NT; ++i) { o[i][2 * r] *= corr; o[i][2 * r + 1] *= corr; }
                }
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (r == 1 && !upper) {
                    pa[1] = pa[3] = 0u;
                    continue;
                }
                const float off = ref[r] == -INFINITY ? 0.f : -ref[r];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float e0 = exp2_q4(fmaf(s[j][2 * r], sl2, off)), e1 = exp2_q4(fmaf(s[j][2 * r + 1], sl2, off));
                    sum[r] += e0 + e1;
                    pa[2 * j + r] = pack_bf16(e0, e1);
                }
            }
        };
        for (int blk = at.blk0; blk < at.blk1; ++blk) {
            if (blk >= at.cached) {
                // ---- the tree's own rows (16 at most), from global memory, by the first warp ----
                if (warp == 0) {
                    float s[2][4];
                    const uint4* Kt = static_cast<const uint4*>(p.Kt) + pair * p.max_nodes * (D / 8);
                    const uint32_t* Vt = static_cast<const uint32_t*>(p.Vt) + pair * p.max_nodes * (D / 2);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
                        const int key = j * 8 + g;
#pragma unroll
                        for (int i = 0; i < LW; ++i) {
                            const uint4 k = key < n ? __ldg(Kt + (size_t)key * (D / 8) + t * LW + i) : make_uint4(0u, 0u, 0u, 0u);
                            const uint4 q0 = qs[(2 * i) * 32 + lane], q1 = qs[(2 * i + 1) * 32 + lane];
                            mma_16816(s[j], q0.x, q0.y, q0.z, q0.w, k.x, k.y);
                            mma_16816(s[j], q1.x, q1.y, q1.z, q1.w, k.z, k.w);
                        }
                    }
                    uint32_t vis[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        vis[r] = g + 8 * r < nrows ? tree_bits32(p.mask + ((size_t)b * p.max_nodes + (row0 + g + 8 * r) / p.grp) * MW, MW, 0, n) : 0u;
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (!((vis[r] >> (j * 8 + 2 * t + e)) & 1u)) s[j][2 * r + e] = -INFINITY;
                    }
                    uint32_t pa[4];
                    weigh(s, pa);
                    // values: words of four keys; a row with a NaN or an infinity counts as zero, and as NaN for the rows that see it
                    uint32_t v[4][D / 16];
                    uint32_t bad = 0u;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int key = (k >> 1) * 8 + 2 * t + (k & 1);
                        bool is_bad = false;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            v[k][i] = key < n ? __ldg(Vt + (size_t)key * (D / 2) + g * (D / 16) + i) : 0u;
                            is_bad = is_bad || (v[k][i] & 0x7f80u) == 0x7f80u || (v[k][i] & 0x7f800000u) == 0x7f800000u;
                        }
                        if (is_bad) bad |= 1u << key;
                    }
                    bad = __reduce_or_sync(0xffffffffu, bad);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if ((bad >> ((k >> 1) * 8 + 2 * t + (k & 1))) & 1u)
#pragma unroll
                            for (int i = 0; i < D / 16; ++i) v[k][i] = 0u;
#pragma unroll
                    for (int r = 0; r < 2; ++r) poisoned[r] = poisoned[r] || (vis[r] & bad) != 0u;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        mma_16816(o[2 * i], pa[0], pa[1], pa[2], pa[3], __byte_perm(v[0][i], v[1][i], 0x5410), __byte_perm(v[2][i], v[3][i], 0x5410));
                        mma_16816(o[2 * i + 1], pa[0], pa[1], pa[2], pa[3], __byte_perm(v[0][i], v[1][i], 0x7632), __byte_perm(v[2][i], v[3][i], 0x7632));
                    }
                }
                continue;
            }
            if (!failed && !tc::mbar_wait_ready(&sh->full[st], phase, abort_flag)) failed = true;
            failed = __any_sync(0xffffffffu, failed);
            const int left = kv - blk * kKeys - warp * 16;                    // keys of this warp that there are
            if (!failed && left > 0) {
                const unsigned char* Kside = ring + (size_t)st * 2 * kSide;
                const unsigned char* Vside = Kside + kSide;
                const long long grow = (long long)pair * p.Lcap + (long long)blk * kKeys;
                const uint32_t* Kso = RawQ4<D>::pairs(Kside, kKeys, grow);
                const uint32_t* Vso = RawQ4<D>::pairs(Vside, kKeys, grow);
                // scores, in two sums that run side by side for each tile of 8 keys (an instruction waits for the one before it in its own)
                float s[2][4], s2[2][4];
                uint32_t kw[2][LW], kso[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int key = warp * 16 + j * 8 + g;
                    if constexpr (LW == 4) {
                        const uint4 u = *reinterpret_cast<const uint4*>(Kside + key * RawQ4<D>::kLevels + t * 16);
                        kw[j][0] = u.x; kw[j][1] = u.y; kw[j][2] = u.z; kw[j][3] = u.w;
                    } else {
                        const uint2 u = *reinterpret_cast<const uint2*>(Kside + key * RawQ4<D>::kLevels + t * 8);
                        kw[j][0] = u.x; kw[j][1] = u.y;
                    }
                    kso[j] = Kso[key * (D / 32) + t * (D / 32) / 4];
                    s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
                    s2[j][0] = s2[j][1] = s2[j][2] = s2[j][3] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < LW; ++i) {
                    const uint4 q0 = qs[(2 * i) * 32 + lane], q1 = qs[(2 * i + 1) * 32 + lane];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint4 k = q4_values_bf16(kw[j][i], kso[j]);
                        mma_16816(s[j], q0.x, q0.y, q0.z, q0.w, k.x, k.y);
                        mma_16816(s2[j], q1.x, q1.y, q1.z, q1.w, k.z, k.w);
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) s[j][q] += s2[j][q];
                if (left < 16) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (j * 8 + 2 * t + e >= left) s[j][e] = s[j][2 + e] = -INFINITY;
                }
                uint32_t pa[4];
                weigh(s, pa);
                uint32_t w[4][VW], sc[2], og[2];                             // levels of four keys; scales and origins of two pairs of keys
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t so[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int kk = h * 8 + 2 * t + e, key = warp * 16 + kk;
                        if constexpr (VW == 2) {
                            const uint2 u = *reinterpret_cast<const uint2*>(Vside + key * RawQ4<D>::kLevels + g * 8);
                            w[2 * h + e][0] = u.x; w[2 * h + e][1] = u.y;
                        } else {
                            w[2 * h + e][0] = *reinterpret_cast<const uint32_t*>(Vside + key * RawQ4<D>::kLevels + g * 4);
                        }
                        so[e] = Vso[key * (D / 32) + g * (D / 32) / 8];
                        if (kk >= left) so[e] = 0u;                          // (behind the last row: zero, whatever stands there)
                    }
                    sc[h] = __byte_perm(so[0], so[1], 0x5410);
                    og[h] = __byte_perm(so[0], so[1], 0x7632);
                }
#pragma unroll
                for (int i = 0; i < VW; ++i) {
                    // even and odd columns of the two keys of a pair, in the halves of a word
                    uint32_t ev[2][4], od[2][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) q4_pairs2(w[2 * h][i], w[2 * h + 1][i], ev[h], od[h]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        mma_16816(o[8 * i + 2 * c], pa[0], pa[1], pa[2], pa[3], q4_fma2(ev[0][c], sc[0], og[0]), q4_fma2(ev[1][c], sc[1], og[1]));
                        mma_16816(o[8 * i + 2 * c + 1], pa[0], pa[1], pa[2], pa[3], q4_fma2(od[0][c], sc[0], og[0]), q4_fma2(od[1][c], sc[1], og[1]));
                    }
                }
            }
            __syncwarp();
            if (lane == 0 && !failed) tc::mbar_arrive(&sh->empty[st]);
            if (++st == nstages) { st = 0; phase ^= 1u; }              // (counted: a division by a number not known to the compiler costs as much as a word's values)
        }
        if (failed && lane == 0) {
            if (*abort_flag == 0) report_error(p.status, CTCSD_ERR_TIMEOUT, 52);
            *abort_flag = 1;
        }
        // ---- join the warps ----
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 1);
            sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 2);
            if (poisoned[r]) sum[r] = __uint_as_float(0x7fc00000u);
            if (t == 0) { sh->ref[warp][g + 8 * r] = ref[r]; sh->sum[warp][g + 8 * r] = sum[r]; }
        }
        consumers_barrier();
        float top[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            top[r] = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top[r] = fmaxf(top[r], sh->ref[w][g + 8 * r]);
            const float wt = ref[r] == -INFINITY ? 0.f : exp2_q4(ref[r] - top[r]);
#pragma unroll
            for (int i = 0; i < NT; ++i) { o[i][2 * r] *= wt; o[i][2 * r + 1] *= wt; }
        }
        // a lane's columns of rows g and g + 8: D/4 t .. : first those of its even position, then of its odd one
        auto put = [&](bool add) {
            float4* buf = reinterpret_cast<float4*>(join) + (warp & 3) * kRows * (D / 4);
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const int e = c < D / 32 ? 0 : 1, i0 = 4 * (c - e * (D / 32));
                    float4 v = make_float4(o[i0][2 * r + e], o[i0 + 1][2 * r + e], o[i0 + 2][2 * r + e], o[i0 + 3][2 * r + e]);
                    float4* at4 = buf + join_at<D>(g + 8 * r, t * (D / 16) + c);
                    if (add) { const float4 u = *at4; v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w; }
                    *at4 = v;
                }
        };
#pragma unroll 1
        for (int w0 = kWarps - 4; w0 >= 0; w0 -= 4) {        // four warps at a time
            if (warp >= w0 && warp < w0 + 4) put(w0 + 4 < kWarps);
            consumers_barrier();
        }
        // ---- output: 16 threads a row ----
        if (warp < 8) {
            const int r = tid >> 4, c0 = (tid & 15) * (D / 64);               // this thread's chunks of four columns
            float rtop = -INFINITY, rsum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) rtop = fmaxf(rtop, sh->ref[w][r]);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float wr = sh->ref[w][r], ws = sh->sum[w][r];
                rsum += wr == -INFINITY ? (ws == ws ? 0.f : ws) : ws * exp2_q4(wr - rtop);
            }
            float4 v[D / 64];
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                v[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float4 u = reinterpret_cast<const float4*>(join)[w * kRows * (D / 4) + join_at<D>(r, c0 + c)];
                    v[c].x += u.x; v[c].y += u.y; v[c].z += u.z; v[c].w += u.w;
                }
            }
            if (r < nrows && !failed && *abort_flag == 0) {
                if (at.whole()) {
                    const size_t orow = out_row(r);
                    if (CTCSD_IN_BOUNDS(p.status, 141, orow, out_rows(p))) {
                        const float inv = rsum > 0.f ? 1.f / rsum : (rsum == 0.f ? 0.f : rsum);
                        uint2* out = reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.O) + orow * D) + c0;
#pragma unroll
                        for (int c = 0; c < D / 64; ++c)
                            out[c] = make_uint2(pack_bf16(v[c].x * inv, v[c].y * inv), pack_bf16(v[c].z * inv, v[c].w * inv));
                        if ((tid & 15) == 0 && p.lse) p.lse[orow] = rsum == 0.f ? -INFINITY : (rtop + log2f(rsum)) * kLn2;
                    }
                } else {
                    const size_t part = (size_t)blockIdx.x * 2 + at.slot();
                    if (CTCSD_IN_BOUNDS(p.status, 142, part * kRows + r, 2ll * gridDim.x * kRows)) {
#pragma unroll
                        for (int c = 0; c < D / 64; ++c) p.part_o[(part * (D / 4) + c0 + c) * kRows + r] = v[c];
                        if ((tid & 15) == 0) p.part_ml[part * kRows + r] = make_float2(rtop, rsum);
                    }
                }
            }
        }
        consumers_barrier();                                 // the buffers are free for the next tile
    }
}

template <int D>
int launch_mma(Handle* h, cudaStream_t s, const AttnQ4Params& p) {
    const size_t fixed = sizeof(float4) * 4 * kRows * (D / 4) + sizeof(uint4) * 2 * (D / 32) * 32 + sizeof(MmaShared) + sizeof(int) * PlanQ4::ints(p.B);
    const size_t stage = 2 * (size_t)RawQ4<D>::bytes(kKeys);
    size_t n = (kMaxDynamicSmem - 1024 - fixed) / stage;
    if (n > kMaxStages) n = kMaxStages;
    auto kern = attention_q4_mma_kernel<D>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepAttnQ4Mma, kern));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(h->num_sms), dim3(kThreads), fixed + n * stage, s, 1, p, (int)n));
    h->launches++;
    return CTCSD_OK;
}

}  // namespace

int launch_attention_q4_mma(Handle* h, cudaStream_t s, const AttnQ4Params& p) {
    return p.D == 64 ? launch_mma<64>(h, s, p) : launch_mma<128>(h, s, p);
}

}  // namespace ctcsd
