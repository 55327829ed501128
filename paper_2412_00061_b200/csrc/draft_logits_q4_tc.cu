// Draft head over 4-bit weights for bfloat16, on the 5th-generation tensor cores (tcgen05 + TMEM), for up to 128 activation rows in a pass.
//
// D[128 x N] = A[128 x H] B[N x H]^T per tile: A = eight panels of weights (draft_q4.cuh) as bfloat16 values, in tensor memory (lane = class); B =
// the activation rows, K-major with the 128-byte swizzle in shared memory, N the rows rounded up to 16; 128 hidden elements to a stage;
// D in tensor memory (lane = class, column = row).
// Sixteen warps turn levels into values, four to a stage, 32 classes each: a lane reads its class's levels of a block, 64 bytes, and writes 64 columns of
// tensor memory.  So the values never pass through shared memory, and a row costs its share of B and D only.  (Weights as the B operand, written to
// swizzled tiles in shared memory, with activations padded to 128 rows as A: 403 us for 32 rows of the 70B shape, 185 us for 16 rows of the 7B shape.
// mma.sync with the values in registers, for up to eight rows: 95-99 us for one row of the 7B shape, 108 for eight, 179 for four mapped rows of the
// 13B shape, which it read without the kernel that gathers them here: one form serves all numbers of rows.)
// The tensor core cuts a sum's last bits off at every addition, always towards zero, and long chains drift (log-probabilities off by
// 6e-6 at H = 8192, by 5e-7 so).  So sums begin again every kStretch blocks, and the four warps that read D back add them up in rounded arithmetic, in
// tensor memory.  They then turn 32 classes x R rows through shared memory, so that a lane has a row, and keep each row's maximum, sum of
// exponentials and best k.
// Roles: warps 0-3 read sums back (32 classes each), 4-19 make values, 20 loads activations, 21 loads levels, 22 and 23 issue
// products, of every other block each, into sums of their own (an issue takes some 700 cycles of waiting, describing and committing, more than its
// products: 32 rows of the 70B shape 346 us with one issuer, 255 with two, 280 with four).
//
// 7B shape (5 slots of 32001 classes, H = 4096, groups of 128): 1 row 101 us, 3.4 TB/s of weights; 16 rows 112 us.  13B shape (8 slots, H = 5120, groups of 64):
// 4 mapped rows 182 us.  70B shape (6 slots, H = 8192): 32 rows 258 us.  No unit is at its limit (7B shape, 1 row: DRAM 36 %, ALU pipe 58 %, 0.59
// instructions a cycle and scheduler).  24 instructions are issued for each word of eight weights where the makers' loop has eleven: the rest are waits,
// hand-overs, sums that are read back and looked through, and what is how much of that was not taken apart.  Left out one at a time, the stores to tensor memory
// are worth 32 us of the 7B shape, products and stores 38, reading sums back 14.
#include "draft_q4.cuh"
#include "tc_primitives.cuh"

#include <type_traits>

namespace ctcsd {
namespace {

constexpr int kEpi = kDraftQ4TcStates;
constexpr int kGroups = 4;               // groups of four warps that make values
constexpr int kMakers = 4 * kGroups;
constexpr int kStages = kGroups;         // a stage holds a block; each group has its own, so that it sees every fill of it and no turn of its barriers goes by unseen
constexpr int kMaxXStages = 8;           // of activations
constexpr int kMaxRing = 8;
constexpr int kMaxAccs = 4;              // sums in tensor memory that take turns
constexpr int kIssuers = 2;              // warps that issue products
constexpr int kThreads = (kEpi + kMakers + 2 + kIssuers) * 32;
constexpr int kTile = 128, kTilePanels = kTile / kQ4Panel;
constexpr int kStretch = 8;              // blocks whose products the tensor core adds up, per issuing warp
constexpr int kTurn = 32 * 33;           // floats of a warp's 32 x 32 turning buffer
constexpr int kSaved = 2 * kTopSlots + 2;    // words of a row's running state

struct __align__(8) TcState {
    uint64_t raw_full[kMaxRing], raw_empty[kMaxRing];    // levels of the tile's panels, two blocks of each
    uint64_t v_full[kStages], v_empty[kStages];          // values
    uint64_t x_full[kMaxXStages], x_empty[kMaxXStages];  // activations
    uint64_t acc_full[kMaxAccs], acc_empty[kMaxAccs];
    uint32_t tmem_base;
    int abort_flag, never_set, merge[2];
};

struct TcGeo {
    int tiles;                           // tiles of a draft slot
    int n;                               // rows of the product: those there are, rounded up to 16 (those behind the last are zeros)
    int chunks;                          // 32-row chunks
    int xstages;                         // stages of activations (a multiple of the issuers: each sees every fill of its own)
    int issuers;                         // issuing warps at work (a power of two), with every issuers-th block each, into sums of their own
    int accs;                            // sums that take turns, of each
    int cols;                            // columns of a sum: the rows, rounded up to 32 where they are more than 16 (512: 64 a stage, the sums, the total)
};

__device__ __forceinline__ void give_up(TcState* sh, int* status, int site) {
    volatile int* f = &sh->abort_flag;
    if (*f == 0) report_error(status, CTCSD_ERR_TIMEOUT, site);
    *f = 1;
}

__global__ void __launch_bounds__(kThreads, 1) draft_q4_tc_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, DraftQ4Params p,
                                                                  TcGeo geo) {
    extern __shared__ __align__(1024) unsigned char dyn[];
    const int x_plane = geo.n * 128, x_bytes = 2 * x_plane;                   // activations of a stage (a plane: 64 elements)
    unsigned char* ring = dyn + geo.xstages * x_bytes;
    const int bb = q4_block_bytes(p.group), slot_bytes = kTilePanels * 2 * bb;
    float* turn = reinterpret_cast<float*>(ring + (size_t)p.nring * slot_bytes);            // [kEpi][kTurn]
    uint32_t* saved = reinterpret_cast<uint32_t*>(turn + kEpi * kTurn);                     // [kEpi][chunks][kSaved][32]
    TcState* sh = reinterpret_cast<TcState*>(saved + kEpi * geo.chunks * kSaved * 32);
    if ((tc::smem_u32(dyn) & 1023u) != 0u) {                   // uniform over the CTA
        if (threadIdx.x == 0) report_error(p.status, CTCSD_ERR_INTERNAL, 45);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        for (int s = 0; s < p.nring; ++s) { tc::mbar_init(&sh->raw_full[s], 1); tc::mbar_init(&sh->raw_empty[s], kMakers / 2); }
        for (int s = 0; s < kStages; ++s) { tc::mbar_init(&sh->v_full[s], 4); tc::mbar_init(&sh->v_empty[s], 1); }
        for (int s = 0; s < geo.xstages; ++s) { tc::mbar_init(&sh->x_full[s], 1); tc::mbar_init(&sh->x_empty[s], 1); }
        for (int a = 0; a < geo.accs; ++a) { tc::mbar_init(&sh->acc_full[a], geo.issuers); tc::mbar_init(&sh->acc_empty[a], kEpi); }
        sh->abort_flag = 0;
        sh->never_set = 0;
        tc::fence_barrier_init();
    }
    if (warp == kEpi + kMakers + 1) {
        tc::tmem_alloc(&sh->tmem_base, 512);
        tc::tmem_relinquish();
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    // columns: values of the stages, the sums, the total
    const uint32_t tmem = sh->tmem_base, tmem_d = tmem + 64u * kStages, acc_cols = geo.cols, tmem_t = tmem_d + geo.accs * geo.issuers * acc_cols;
    // this CTA's tiles: u0 .. u1-1 of the line of all slots' tiles
    const long long total = (long long)geo.tiles * p.slots;
    const int u0 = (int)(total * blockIdx.x / gridDim.x), u1 = (int)(total * (blockIdx.x + 1) / gridDim.x);
    const int slot0 = u0 / geo.tiles;
    const int segs = u1 > (slot0 + 1) * geo.tiles ? 2 : 1;
    // Every CTA begins at a place of its own along the hidden axis (and wraps), so that at any moment the CTAs ask L2 for different parts of the
    // activations that they all share.
    const int pairs = (p.blocks + 1) / 2, start = (int)((long long)blockIdx.x * pairs / gridDim.x);       // pairs of blocks; the last may be one block
    // (with an odd number of blocks, an empty one behind the last goes the others' way, without products: its place in the CTA's order)
    const int blocks2 = 2 * pairs, empty_at = (p.blocks & 1) ? 2 * (pairs - 1 - start) + 1 : -1;
    const int stretch = kStretch * geo.issuers;
    bool failed = false;

    if (warp < kEpi) {
        // ---------------- logits ----------------
        pdl_wait();
        pdl_trigger();
        const uint32_t lane_off = (uint32_t)(warp * 32) << 16;                // the quarter of the tensor memory's lanes that the warp reads
        float* const my_turn = turn + warp * kTurn;
        uint32_t* const my_saved = saved + warp * geo.chunks * kSaved * 32 + lane;
        RunState st;
        float floor;                                           // a logit has to be above it to be among the k best,
        bool listed;                                           // unless the list holds fewer
        auto look = [&]() {
#pragma unroll
            for (int s = 0; s < kTopSlots; ++s) {
                float f = st.val[s];
                int i = st.id[s];
                asm("" : "+f"(f), "+r"(i));                    // (else the compiler makes it a look-up by k, and the list leaves the registers)
                if (s == p.k - 1) { floor = f; listed = i != INT_MAX; }
            }
        };
        auto save = [&](int c) {
            uint32_t* to = my_saved + c * kSaved * 32;
            to[0] = __float_as_uint(st.mx); to[32] = __float_as_uint(st.sum);
#pragma unroll
            for (int s = 0; s < kTopSlots; ++s) { to[(2 + 2 * s) * 32] = __float_as_uint(st.val[s]); to[(3 + 2 * s) * 32] = (uint32_t)st.id[s]; }
        };
        auto load = [&](int c) {
            const uint32_t* from = my_saved + c * kSaved * 32;
            st.mx = __uint_as_float(from[0]); st.sum = __uint_as_float(from[32]);
#pragma unroll
            for (int s = 0; s < kTopSlots; ++s) { st.val[s] = __uint_as_float(from[(2 + 2 * s) * 32]); st.id[s] = (int)from[(3 + 2 * s) * 32]; }
        };
        // the warp's states of a draft slot, one for every row (few rows stand in a warp two or four times, with other classes)
        auto publish = [&](int seg) {
            for (int c = 0; c < geo.chunks; ++c) {
                load(c);
                if (p.mcount <= 8) combine_best<24>(st, p.k);
                else if (p.mcount <= 16) combine_best<16>(st, p.k);
                const int m = c * 32 + lane;
                const size_t o = ((size_t)(warp * p.mcount + m) * gridDim.x + blockIdx.x) * 2 + seg;
                if (m < p.mcount && CTCSD_IN_BOUNDS(p.status, 171, o, p.part_room)) st.store(p.part + o);
            }
        };
        auto begin = [&]() {
            st.init();
            for (int c = 0; c < geo.chunks; ++c) save(c);
        };
        // A chunk of a tile's logits: R rows of 32 classes, turned so that a lane has a row and R classes of it.
        auto look_through = [&](auto rows, int c, int slot, int v0, int left) __attribute__((always_inline)) {
            constexpr int R = decltype(rows)::value, J = R;     // J classes a lane
            uint32_t r[32];
            if constexpr (R == 32) tc::tmem_read32(tmem_t + c * 32 + lane_off, r);
            else tc::tmem_read16(tmem_t + lane_off, reinterpret_cast<uint32_t(&)[16]>(r));
#pragma unroll
            for (int j = 0; j < R; ++j) my_turn[j * 33 + lane] = __uint_as_float(r[j]);
            __syncwarp();
            float z[J];
            const int row = lane % R, j0 = lane / R * J;
#pragma unroll
            for (int j = 0; j < J; ++j) z[j] = my_turn[row * 33 + j0 + j];      // class v0 + j0 + j, row c * 32 + row
            __syncwarp();
            const int m = c * 32 + row;
            const bool live = m < p.mcount;
            load(c);
            look();
            v0 += j0;
            left -= j0;                                        // classes that the lane has
            if (left <= J) {                                   // (the last one is the blank)
                float bias = 0.f;
                if (live && left > 0 && p.blank_bias != nullptr) bias = p.blank_bias[p.row_seq ? p.row_seq[p.m0 + m] : p.m0 + m];
#pragma unroll
                for (int j = 0; j < J; ++j) z[j] = j < left ? z[j] + (j == left - 1 ? bias : 0.f) : -INFINITY;
            }
            if (p.logits_dbg != nullptr && live) {
                const size_t o = ((size_t)(p.m0 + m) * p.slots + slot) * p.classes + v0;
#pragma unroll
                for (int j = 0; j < J; ++j)
                    if (j < left && CTCSD_IN_BOUNDS(p.status, 172, o + j, (long long)p.rows * p.slots * p.classes)) p.logits_dbg[o + j] = z[j];
            }
            float top = z[0];
#pragma unroll
            for (int j = 1; j < J; ++j) top = fmaxf(top, z[j]);
            if (top > st.mx) {
                st.sum *= __expf(st.mx - top);                 // exp(-inf) = 0 covers the first chunk
                st.mx = top;
            }
            const float base = st.mx == -INFINITY ? 0.f : st.mx;                   // (nothing but -inf so far: they add nothing)
            float add = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) add += __expf(z[j] - base);
            st.sum += add;
            if (__any_sync(0xffffffffu, live && left > 0 && (top > floor || !listed))) {
                uint32_t above = 0u;                           // logits that may be among the best
#pragma unroll
                for (int j = 0; j < J; ++j) above |= z[j] > floor || !listed ? 1u << j : 0u;
                if (left < J) above &= left > 0 ? (1u << left) - 1u : 0u;
                if (!live) above = 0u;
                // every lane takes its own, the largest first, so that few come to be tried (at most one more than stay)
                while (__any_sync(0xffffffffu, above != 0u)) {
                    float best = -INFINITY;
                    int at = -1;
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const bool better = ((above >> j) & 1u) && (at < 0 || z[j] > best);
                        best = better ? z[j] : best;
                        at = better ? j : at;
                    }
                    if (at >= 0) {
                        above &= ~(1u << at);
                        if (best > floor || !listed) {
                            topk_insert(st.val, st.id, best, v0 + at);
                            look();
                        } else {
                            above = 0u;
                        }
                    }
                }
            }
            save(c);
        };
        begin();
        int a = 0, seg = 0;
        uint32_t phase = 0u;
        for (int u = u0; u < u1 && !failed; ++u) {
            const int slot = u / geo.tiles, v0 = (u - slot * geo.tiles) * kTile + warp * 32;
            const int left = p.classes - v0;                   // classes that the warp has
            if (slot - slot0 != seg) {
                publish(0);
                begin();
                seg = 1;
            }
            for (int kb0 = 0; kb0 < blocks2; kb0 += stretch) {
                if (!tc::mbar_wait_ready(&sh->acc_full[a], phase, abort_flag)) failed = true;
                failed = __any_sync(0xffffffffu, failed);
                if (failed) break;
                tc::tc_fence_after_sync();
                if (left > 0) {
                    // (the second of two issuers has none where there is the empty block only)
                    const uint32_t from = tmem_d + a * geo.issuers * acc_cols + lane_off;
                    const int parts = kb0 + 2 == blocks2 && empty_at == kb0 + 1 ? 1 : geo.issuers;
                    for (int c = 0; c * 16 < geo.n; ++c) {                                           // 16 rows at a time
                        uint32_t r[16];
                        tc::tmem_read16(from + c * 16, r);
                        for (int i = 1; i < parts; ++i) {
                            uint32_t s[16];
                            tc::tmem_read16(from + i * acc_cols + c * 16, s);
#pragma unroll
                            for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) + __uint_as_float(s[j]));
                        }
                        if (kb0 > 0) {
                            uint32_t s[16];
                            tc::tmem_read16(tmem_t + c * 16 + lane_off, s);
#pragma unroll
                            for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) + __uint_as_float(s[j]));
                        }
                        tc::tmem_st16(tmem_t + c * 16 + lane_off, r);
                    }
                    tc::tmem_st_wait();
                }
                tc::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sh->acc_empty[a]);
                if (++a == geo.accs) { a = 0; phase ^= 1u; }
            }
            if (failed) break;
            if (left <= 0) continue;
            if (p.mcount <= 8) look_through(std::integral_constant<int, 8>(), 0, slot, v0, left);
            else if (p.mcount <= 16) look_through(std::integral_constant<int, 16>(), 0, slot, v0, left);
            else
                for (int c = 0; c < geo.chunks; ++c) look_through(std::integral_constant<int, 32>(), c, slot, v0, left);
        }
        if (failed && lane == 0) give_up(sh, p.status, 46);
        if (!failed) publish(seg);
    } else if (warp < kEpi + kMakers) {
        // ---------------- values ----------------
        pdl_wait();
        pdl_trigger();
        const int q = warp & 3, stage = (warp - kEpi) >> 2;    // (a warp writes the quarter of the tensor memory's lanes that its number names)
        const int panel = 2 * q + (lane >> 4), cls = lane & 15;
        const int gpb = kQ4Block / p.group;
        // Of four blocks, two ring slots, the group takes one: with an even number of ring slots it sees every fill of those that it takes from.
        const int kb = stage & 1;
        int n = 0, s = stage >> 1;                             // pairs so far, the group's next ring slot
        uint32_t phase = 0u, v_phase = 1u;
        for (int u = u0; u < u1 && !failed; ++u) {
            const bool there = (u % geo.tiles) * kTile + q * 32 < p.classes;  // (behind a slot's last class: nothing to make)
            for (int pc = 0, at = start; pc < pairs; ++pc, at = at + 1 == pairs ? 0 : at + 1, ++n) {
                if ((n & 1) == (stage >> 1)) {
                    // (lanes that wait for different barriers at once wake late: with one lane to a barrier the 7B shape took 152 us in place of 104)
                    const bool ok = tc::mbar_wait_ready(&sh->raw_full[s], phase, abort_flag) && tc::mbar_wait_ready(&sh->v_empty[stage], v_phase, abort_flag);
                    if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                    tc::tc_fence_after_sync();
                    if (there && 2 * at + kb < p.blocks) {
                        const unsigned char* blk = ring + s * slot_bytes + (panel * 2 + kb) * bb;
                        const uint32_t* so = reinterpret_cast<const uint32_t*>(blk + 1024) + cls * gpb;
                        const uint32_t to = tmem + 64u * stage + ((uint32_t)(q * 32) << 16);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t v[32];
#pragma unroll
                            for (int t = 0; t < 2; ++t) {
                                const uint4 w = *reinterpret_cast<const uint4*>(blk + ((2 * half + t) * kQ4Panel + cls) * 16);
                                const uint32_t pr = so[((2 * half + t) * gpb) >> 2];
                                const uint32_t w4[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const uint4 x = q4_values_bf16(w4[i], pr);
                                    v[(t * 4 + i) * 4] = x.x; v[(t * 4 + i) * 4 + 1] = x.y; v[(t * 4 + i) * 4 + 2] = x.z; v[(t * 4 + i) * 4 + 3] = x.w;
                                }
                            }
                            tc::tmem_st32(to + 32u * half, v);
                        }
                        tc::tmem_st_wait();
                    }
                    tc::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        tc::mbar_arrive(&sh->v_full[stage]);
                        tc::mbar_arrive(&sh->raw_empty[s]);
                    }
                    v_phase ^= 1u;
                    if ((s += 2) >= p.nring) { s -= p.nring; phase ^= 1u; }
                }
            }
        }
        if (failed && lane == 0) give_up(sh, p.status, 47);
    } else if (warp == kEpi + kMakers + 1) {
        // ---------------- levels ----------------
        if (lane == 0) {
            // (weights are not written while they are in use: the ring fills while the predecessor in the stream drains, and nothing else is
            // read before this kernel's other warps have waited for it)
            const uint64_t pol = tc::policy_evict_first();
            const uint32_t bytes = (uint32_t)slot_bytes;
            int s = 0, fill = 0;
            uint32_t phase = 1u;
            for (int u = u0; u < u1 && !failed; ++u) {
                const int slot = u / geo.tiles, pan = slot * p.panels + (u - slot * geo.tiles) * kTilePanels;
                for (int pc = 0, at = start; pc < pairs; ++pc, at = at + 1 == pairs ? 0 : at + 1, ++fill) {
                    if (fill == p.nring) {
                        pdl_wait();
                        pdl_trigger();
                    }
                    if (!tc::mbar_wait_ready(&sh->raw_empty[s], phase, abort_flag)) { failed = true; break; }
                    tc::mbar_arrive_expect_tx(&sh->raw_full[s], bytes);
                    // (64 bytes x the blocks' lines x eight panels; what lies behind a panel's end or the last panel arrives as zeros)
                    tc::tma_load_3d(ring + s * slot_bytes, &tmW, &sh->raw_full[s], 0, at * 2 * (bb / 64), pan, pol);
                    if (++s == p.nring) { s = 0; phase ^= 1u; }
                }
            }
            if (failed) {
                give_up(sh, p.status, 50);
                for (int back = 1; back <= p.nring && back <= fill; ++back) {            // copies in flight land before the exit
                    const int j = fill - back;
                    tc::mbar_wait_suspended(&sh->raw_full[j % p.nring], (uint32_t)(j / p.nring) & 1u, &sh->never_set, 1ll << 24);
                }
            }
        }
        pdl_wait();
        pdl_trigger();
    } else if (warp == kEpi + kMakers) {
        // ---------------- activations ----------------
        pdl_wait();
        pdl_trigger();
        if (lane == 0) {
            const uint64_t pol = tc::policy_evict_last();
            const int steps = (u1 - u0) * blocks2;
            int it = 0, kb = 2 * start, st = 0;
            uint32_t phase = 1u;
            for (; it < steps; ++it) {
                if (!tc::mbar_wait_ready(&sh->x_empty[st], phase, abort_flag)) { failed = true; break; }
                unsigned char* dst = dyn + st * x_bytes;
                if (kb < p.blocks) {
                    tc::mbar_arrive_expect_tx(&sh->x_full[st], (uint32_t)x_bytes);
                    // (elements behind H and rows behind the last are outside the tensor and arrive as zeros)
                    tc::tma_load_2d(dst, &tmX, &sh->x_full[st], kb * kQ4Block, 0, pol);
                    tc::tma_load_2d(dst + x_plane, &tmX, &sh->x_full[st], kb * kQ4Block + 64, 0, pol);
                } else {
                    tc::mbar_arrive(&sh->x_full[st]);
                }
                if (++kb == blocks2) kb = 0;
                if (++st == geo.xstages) { st = 0; phase ^= 1u; }
            }
            if (failed) {
                give_up(sh, p.status, 48);
                for (int back = 1; back <= geo.xstages && back <= it; ++back) {          // copies in flight land before the exit
                    const int j = it - back;
                    tc::mbar_wait_suspended(&sh->x_full[j % geo.xstages], (uint32_t)(j / geo.xstages) & 1u, &sh->never_set, 1ll << 24);
                }
            }
        }
    } else {
        // ---------------- products ----------------
        pdl_wait();
        pdl_trigger();
        // (the whole warp goes through the loop and one lane issues: descriptors stay in uniform registers.  Turns are counted, not divided for: a
        // division takes some 200 cycles.)
        const uint32_t idesc = tc::idesc_bf16_f32(kTile, geo.n);
        const uint64_t x_desc0 = tc::smem_desc_k_sw128(tc::smem_u32(dyn));
        const int mine = warp - (kEpi + kMakers + 2);
        int it = 0, a = 0, done = -1;                          // blocks so far, the last one that was issued here
        int xs = mine;
        uint32_t a_phase = 1u, x_phase = 0u;
        for (int u = u0; u < u1 && !failed && mine < geo.issuers; ++u) {
            for (int kb0 = 0; kb0 < blocks2 && !failed; kb0 += stretch) {
                const int nb = min(stretch, blocks2 - kb0);
                const uint32_t d = tmem_d + (a * geo.issuers + mine) * acc_cols;
                bool first = true, waited = false;
                for (int k0 = mine; k0 < nb; k0 += geo.issuers) {
                    const int st = (it + k0) % kStages;
                    bool ok = waited || tc::mbar_wait_ready(&sh->acc_empty[a], a_phase, abort_flag);
                    ok = ok && tc::mbar_wait_ready(&sh->x_full[xs], x_phase, abort_flag) &&
                         tc::mbar_wait_ready(&sh->v_full[st], (uint32_t)((it + k0) / kStages) & 1u, abort_flag);
                    if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                    tc::tc_fence_after_sync();
                    if (tc::elect_one()) {
                        const uint64_t xd = x_desc0 + (uint64_t)((uint32_t)(xs * x_bytes) >> 4);
                        if (kb0 + k0 != empty_at) {
#pragma unroll
                            for (int half = 0; half < 2; ++half)
#pragma unroll
                                for (int k = 0; k < 4; ++k)    // 16 elements along K: 8 columns of A, 32 bytes of B
                                    tc::mma_bf16_ts(d, tmem + 64u * st + 32u * half + 8u * k, xd + (uint64_t)((uint32_t)(half * x_plane) >> 4) + 2 * k, idesc,
                                                    first && (half | k) == 0 ? 0u : 1u);
                        }
                        tc::mma_commit(&sh->v_empty[st]);
                        tc::mma_commit(&sh->x_empty[xs]);
                    }
                    __syncwarp();
                    first = first && kb0 + k0 == empty_at;
                    waited = true;
                    done = it + k0;
                    if ((xs += geo.issuers) >= geo.xstages) { xs -= geo.xstages; x_phase ^= 1u; }
                }
                if (failed) break;
                if (tc::elect_one()) tc::mma_commit(&sh->acc_full[a]);
                __syncwarp();
                if (++a == geo.accs) { a = 0; a_phase ^= 1u; }
                it += nb;
            }
        }
        if (failed && lane == 0) {
            give_up(sh, p.status, 49);
            if (done >= 0) tc::mbar_wait_suspended(&sh->v_empty[done % kStages], (uint32_t)(done / kStages) & 1u, &sh->never_set, 1ll << 24);
        }
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    if (warp == kEpi + kMakers + 1) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc(tmem, 512);
    }
    if (*abort_flag != 0) return;                              // (uniform: set before the barrier or not at all)
    // a row's states in this CTA become one, in the place of the first
    for (int i = warp; i < segs * p.mcount; i += kThreads / 32) {
        const int seg = i / p.mcount, m = i - seg * p.mcount;
        const size_t o = ((size_t)m * gridDim.x + blockIdx.x) * 2 + seg;
        DraftPartial* at = p.part + o;
        RunState ms;
        ms.init();
        if (lane < kEpi) ms.absorb(load_partial_cg(at + (size_t)lane * p.mcount * gridDim.x * 2));
        combine_best<31>(ms, p.k);
        if (lane == 0 && CTCSD_IN_BOUNDS(p.status, 173, o, p.part_room)) ms.store(at);
    }
    draft_q4_finish(p, geo.tiles, slot0, segs, sh->merge);
}

// Activation rows picked by a row map, one behind the other; a map that leaves x gives a zero row.
__global__ void __launch_bounds__(256) draft_q4_gather_kernel(const uint4* x, int x_row_count, const int* x_rows, int m0, int chunks, uint4* out, long long room, int* status) {
    pdl_wait();
    pdl_trigger();
    const int m = blockIdx.x, r = x_rows[m0 + m];
    const bool there = r >= 0 && r < x_row_count;
    if (!there && threadIdx.x == 0) report_error(status, CTCSD_ERR_INVALID_ARG, m0 + m);
    for (int c = threadIdx.x; c < chunks; c += 256)
        if (CTCSD_IN_BOUNDS(status, 174, (size_t)m * chunks + c, room)) out[(size_t)m * chunks + c] = there ? x[(size_t)r * chunks + c] : make_uint4(0u, 0u, 0u, 0u);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    if (fn) return fn;
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess) return nullptr;
    fn = reinterpret_cast<EncodeTiledFn>(sym);
    return fn;
}

// [rows][H] bf16, box = [box_rows][64], 128-byte swizzle, zeros outside.
bool make_x_map(CUtensorMap* map, const void* x, int rows, int H, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)H, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)H * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(x), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Packed weights as [panels][lines][64 bytes], box = [eight panels][`lines` lines][64 bytes].
bool make_w_map(CUtensorMap* map, const void* w, long long panels, int panel_bytes, int lines) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {16, (cuuint64_t)(panel_bytes / 64), (cuuint64_t)panels};
    cuuint64_t strides[2] = {64, (cuuint64_t)panel_bytes};
    cuuint32_t box[3] = {16, (cuuint32_t)lines, (cuuint32_t)kTilePanels};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(w), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

// One pass: rows m0 .. m0 + mcount - 1.
int launch_draft_q4_tc(Handle* h, cudaStream_t s, DraftQ4Params p) {
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(p.x) + (size_t)p.m0 * p.H;
    if (p.x_rows) {
        uint4* rows = reinterpret_cast<uint4*>(h->ws + h->lay.q4_rows_off);
        CTCSD_CUDA_CHECK(h, launch_pdl(draft_q4_gather_kernel, dim3(p.mcount), dim3(256), 0, s, 1, static_cast<const uint4*>(p.x), p.x_row_count, p.x_rows, p.m0,
                                       p.H / 8, rows, (long long)((h->lay.q4_part_off - h->lay.q4_rows_off) / sizeof(uint4)), p.status));
        h->launches++;
        x = reinterpret_cast<const __nv_bfloat16*>(rows);
    }
    p.part = reinterpret_cast<DraftPartial*>(h->ws + h->lay.q4_part_off);
    p.part_room = (long long)((h->lay.total - h->lay.q4_part_off) / sizeof(DraftPartial));
    TcGeo geo;
    geo.tiles = (p.panels + kTilePanels - 1) / kTilePanels;
    geo.n = (p.mcount + 15) / 16 * 16;
    geo.chunks = (p.mcount + 31) / 32;
    // As many issuers as the columns hold sums for (more than 64 rows: one; the activations then take as long as its issues).  As many sums
    // as there is room for: products go on while a tile's logits are looked through.
    geo.cols = geo.n == 16 ? 16 : geo.chunks * 32;
    const int sums = (512 - 64 * kStages) / geo.cols - 1;
    geo.issuers = sums >= kIssuers ? kIssuers : 1;
    geo.accs = sums / geo.issuers < kMaxAccs ? sums / geo.issuers : kMaxAccs;
    // (activations come from L2, some 1000 cycles a request: eight blocks ahead, six or three where the rows take the room)
    geo.xstages = geo.chunks == 1 ? 8 : (geo.chunks == 2 ? 6 : 3);
    const size_t bb = q4_block_bytes(p.group);
    const size_t fixed = (size_t)geo.xstages * geo.n * 256 + sizeof(float) * kEpi * kTurn + sizeof(uint32_t) * kEpi * geo.chunks * kSaved * 32 + sizeof(TcState);
    const size_t room = kMaxDynamicSmem - 1024 - fixed, slot = kTilePanels * 2 * bb;
    p.nring = (int)(room / slot < kMaxRing ? room / slot : kMaxRing);         // (two at least: 128 rows and groups of 32 take 2 x 20 KB of 76 KB)
    p.nring &= ~1;
    if (p.nring < 2) return CTCSD_ERR_UNSUPPORTED;
    CUtensorMap tmX;
    CUtensorMap tmW;
    if (!make_x_map(&tmX, x, p.mcount, p.H, geo.n) ||
        !make_w_map(&tmW, p.W, (long long)p.panels * p.slots, (int)(p.blocks * bb), (int)(2 * bb / 64))) return CTCSD_ERR_CUDA;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepDraftQ4Tc, draft_q4_tc_kernel));
    const long long total = (long long)geo.tiles * p.slots;
    const unsigned grid = (unsigned)(total < h->num_sms ? total : h->num_sms);         // (total >= slots: a range touches two slots at most)
    CTCSD_CUDA_CHECK(h, launch_pdl(draft_q4_tc_kernel, dim3(grid), dim3(kThreads), fixed + p.nring * slot, s, 1, tmX, tmW, p, geo));
    h->launches++;
    return CTCSD_OK;
}

}  // namespace ctcsd
