// Draft head over 4-bit weights: ctcsd_quantize_weights_q4 (packs them once) and ctcsd_draft_logits_q4.
//   z[m,t,v] = sum_h x[m,h] w[t,v,h] (+ blank_bias on v == V),  w = round(origin + scale (16 + q)) per group along h;
//   log-sum-exp and the k best per (m, t), as ctcsd_draft_logits.
//
// Packed weights.  Sixteen neighbouring classes of a slot are a panel (the last one of a slot filled up with zero rows), 128
// hidden elements of a panel a block, blocks of a panel follow one another:
//   block = levels [2][32 lanes][16 bytes], lane 4g + t of half h: class 8h + g, elements 32t .. 32t + 31, four words (q4.cuh), for t >= 2 in
//           the order 2, 3, 0, 1 (the lanes of a warp that write values to a tensor-core tile then meet in no bank);
//           pairs  [16 classes][128 / group] (scale, origin).
// This is the order in which the lanes of a warp hold the operand A of mma.m16n8k16 (with the hidden index permuted alike for x),
// so a lane takes its share of a block by two 16-byte reads without bank conflicts, and a panel is one piece of memory.
#include "draft_q4.cuh"
#include "tc_primitives.cuh"

#include <limits.h>
#include <math.h>

namespace ctcsd {
namespace {

struct PackParams {
    const void* W;                       // [T,V+1,H]
    unsigned char* out;
    int H, classes, panels, blocks, group;
};

// One warp per two classes of a block: lane = (class parity, eight elements).
template <typename T>
__global__ void __launch_bounds__(256) quantize_weights_q4_kernel(PackParams p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kb = blockIdx.x, t = blockIdx.z;
    const int bytes = q4_block_bytes(p.group), per = p.group / 8;                // lanes of a group
    for (int panel = blockIdx.y; panel < p.panels; panel += gridDim.y) {
        unsigned char* blk = p.out + (((size_t)t * p.panels + panel) * p.blocks + kb) * bytes;
        const int r = warp * 2 + (lane >> 4), e = (lane & 15) * 8;            // class of the panel, first element of the block
        const int cls = panel * kQ4Panel + r, k = kb * kQ4Block + e;
        const bool in = cls < p.classes && k < p.H;                           // (H is a multiple of 8)
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        float lo = INFINITY, hi = -INFINITY;
        if (in) {
            load8(static_cast<const T*>(p.W) + ((size_t)t * p.classes + cls) * p.H + k, v);
            lo = hi = v[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) { lo = min_nan(lo, v[i]); hi = max_nan(hi, v[i]); }
        }
        for (int o = 1; o < per; o <<= 1) {
            lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        // (a group without elements: zeros)
        const bool some = cls < p.classes && kb * kQ4Block + e / p.group * p.group < p.H;
        const uint32_t so = some ? q4_scale_origin(lo, hi) : 0u;
        const uint32_t w = in ? q4_word(v, so) : 0u;
        reinterpret_cast<uint32_t*>(blk)[(r >> 3) * 128 + ((r & 7) * 4 + (e >> 5)) * 4 + (((e >> 3) & 3) ^ ((e >> 6) << 1))] = w;
        if ((lane & 15) % per == 0) reinterpret_cast<uint32_t*>(blk + 1024)[r * (kQ4Block / p.group) + e / p.group] = so;
    }
}

// Launched behind the packing without the attribute that lets kernels overlap: the draft head begins to read weights
// before its predecessor in the stream has ended, and that must not be the kernel that writes them.
__global__ void order_kernel() {}

// The running state of an activation row in a lane: the k best logits in order, in a list of kTopSlots.
struct BestQ4 {
    RunState st;
    float floor;                         // a logit has to be above it to be among the k best,
    int have;                            // unless the list holds fewer
    __device__ __forceinline__ void init() { st.init(); floor = -INFINITY; have = 0; }
    // (a lane's classes come in rising order: an equal logit ranks behind)
    __device__ __forceinline__ void push(float z, int v, int k) {
        if (z > st.mx) {
            st.sum = st.sum * __expf(st.mx - z) + 1.f;
            st.mx = z;
        } else {
            st.sum += __expf(z - st.mx);
        }
        if (z > floor || have < k) {
            topk_insert(st.val, st.id, z, v);
            have += z == z ? 1 : 0;
#pragma unroll
            for (int s = 0; s < kTopSlots; ++s) {
                float f = st.val[s];
                asm("" : "+f"(f));       // (else the compiler makes it a look-up by k, and the list leaves the registers)
                if (s == k - 1) floor = f;
            }
        }
    }
};

// D[16x8] += A[16x16] * B[16x8], bf16 operands, fp32 accumulators (warp-wide).
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int kF32Rows = 4;              // activation rows of a float32 pass
constexpr int kF32Chunk = 36;            // floats from one 32-element chunk of x to the next (four lanes read four chunks: no bank conflict)
constexpr int kMaxRing = 4;              // ring slots of a warp

// Bytes of the activation rows of a pass in shared memory.
//   bfloat16: the lanes' shares of operand B, [block][word][row][chunk t][16 bytes] (a column without a row reads the last row's: its sums are not used);
//   float32: [row][chunk][36 floats].
template <typename T> __host__ __device__ inline size_t x_bytes(int blocks, int rows) {
    return sizeof(T) == 2 ? (size_t)blocks * rows * 256 : (size_t)rows * blocks * 4 * kF32Chunk * 4;
}

// Warps of a CTA: as many as leave a thread the registers for its states (one of 19 registers per activation row it looks after).
template <typename T> struct Shape {
    static constexpr int warps = 16;
    static constexpr int states = sizeof(T) == 2 ? 2 : 1;
};

struct __align__(8) RingState {
    uint64_t full[16 * kMaxRing];
    int abort_flag, never_set, merge[2];
};

// A warp's way through the CTA's panels: whole panels in turn with the other warps, and at the end, when fewer panels than warps are left,
// a share of the blocks of one of those.
struct PanelWalk {
    int pan, blk, end;                   // panel, next block of it and the block behind the last
    bool shared;                         // this is a share
    int npan, whole, per, warps, warp, blocks;   // panels; panels that warps take whole; warps to a panel of the rest
    __device__ __forceinline__ void init(int npan_, int warps_, int warp_, int blocks_) {
        npan = npan_; warps = warps_; warp = warp_; blocks = blocks_;
        whole = npan / warps * warps;
        per = whole < npan ? warps / (npan - whole) : 1;
        pan = warp; blk = 0; end = blocks; shared = false;
        if (pan >= whole) share();
    }
    __device__ __forceinline__ void share() {
        shared = true;
        const int i = warp / per, j = warp - i * per;
        pan = whole + i;
        blk = blocks * j / per;
        end = blocks * (j + 1) / per;
        if (pan >= npan) end = blk;      // (nothing left for this warp)
    }
    __device__ __forceinline__ bool done() const { return shared && blk >= end; }
    __device__ __forceinline__ void next_panel() {           // after the last block of a whole panel
        pan += warps;
        blk = 0;
        if (pan >= whole) share();
    }
};

// One CTA per SM with a contiguous range of panels.  Every warp streams panels of its own through a small ring in shared memory with the
// bulk-copy engine (its first lane asks for the next piece when a slot has been read): levels to values (one multiply-add for
// two), values times activations on the tensor cores (bfloat16: 16 classes x 8 rows an instruction; float32: fused
// multiply-adds), and the lanes that hold a panel's logits keep the running maximum, sum of exponentials and best k.  Warps meet
// at the end only.  (Sets of 4 or 8 warps that shared a panel and handed partial sums to epilogue warps took 93-113 us
// at the 7B shape, half of it in hand-overs.)
template <typename T>
__global__ void __launch_bounds__(Shape<T>::warps * 32, 1) draft_q4_kernel(DraftQ4Params p) {
    constexpr bool kMma = sizeof(T) == 2;
    constexpr int kWarps = Shape<T>::warps, kThreads = kWarps * 32, kStates = Shape<T>::states;
    constexpr int kRows = kMma ? 8 : kF32Rows;
    extern __shared__ __align__(128) unsigned char dyn[];
    unsigned char* xs = dyn;
    unsigned char* ring = xs + x_bytes<T>(p.blocks, p.mcount);
    const int bb = q4_block_bytes(p.group), slot_bytes = p.piece * bb;
    RingState* sh = reinterpret_cast<RingState*>(ring + (size_t)kWarps * p.nring * slot_bytes);
    DraftPartial* s_state = reinterpret_cast<DraftPartial*>(sh + 1);         // [2][warps][kRows]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        for (int s = 0; s < kWarps * p.nring; ++s) tc::mbar_init(&sh->full[s], 1);
        sh->abort_flag = 0;
        sh->never_set = 0;
        tc::fence_barrier_init();
    }
    __syncthreads();

    const long long total = (long long)p.panels * p.slots;
    const long long p0 = total * blockIdx.x / gridDim.x, p1 = total * (blockIdx.x + 1) / gridDim.x;
    const int npan = (int)(p1 - p0);
    const int slot0 = (int)(p0 / p.panels);                                   // draft slot of the first panel
    const int n_seg0 = (int)(((long long)(slot0 + 1) * p.panels < p1 ? (long long)(slot0 + 1) * p.panels : p1) - p0);
    const unsigned char* const W0 = p.W + (size_t)p0 * p.blocks * bb;
    const uint64_t policy = tc::policy_evict_first();
    PanelWalk ahead;                                                          // of what is asked for
    ahead.init(npan, kWarps, warp, p.blocks);
    unsigned char* const my_ring = ring + (size_t)warp * p.nring * slot_bytes;
    uint64_t* const my_full = sh->full + warp * p.nring;
    // asks for the next piece (nothing where the warp's panels are done); all lanes follow the walk, the first asks
    auto ask = [&](int s) {
        if (ahead.done()) return;
        const int nb = min(p.piece, ahead.end - ahead.blk);
        if (lane == 0) {
            const uint32_t bytes = (uint32_t)(nb * bb);
            tc::mbar_arrive_expect_tx(my_full + s, bytes);
            tc::bulk_load_1d(my_ring + s * slot_bytes, W0 + ((size_t)ahead.pan * p.blocks + ahead.blk) * bb, bytes, my_full + s, policy);
        }
        ahead.blk += nb;
        if (!ahead.shared && ahead.blk == ahead.end) ahead.next_panel();
    };
    // (weights are not written while they are in use: the ring fills while the predecessor in the stream drains)
    for (int s = 0; s < p.nring; ++s) ask(s);
    pdl_wait();
    pdl_trigger();
    // ---- activations to shared memory, in the order in which the lanes take them ----
    auto source_row = [&](int m) -> long long {                              // -1: none
        long long r = p.m0 + m;
        if (p.x_rows != nullptr) {
            r = p.x_rows[p.m0 + m];
            if (r < 0 || r >= p.x_row_count) { report_error(p.status, CTCSD_ERR_INVALID_ARG, p.m0 + m); r = -1; }
        }
        return r;
    };
    if constexpr (kMma) {
        const int pieces16 = p.blocks * 16;                                  // 16-byte pieces of a row: [block][chunk t][word i]
        for (int m = 0; m < p.mcount; ++m) {
            const long long r = source_row(m);
#pragma unroll 2
            for (int c = tid; c < pieces16; c += kThreads) {
                uint4 w = make_uint4(0u, 0u, 0u, 0u);
                if (r >= 0 && c * 8 < p.H) w = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.x) + (size_t)r * p.H + c * 8);
                const int kb = c >> 4, t = (c >> 2) & 3, i = (c & 3) ^ ((t >> 1) << 1);   // (in the order of the weights' words)
                *reinterpret_cast<uint4*>(xs + (((size_t)(kb * 4 + i) * p.mcount + m) * 4 + t) * 16) = w;
            }
        }
    } else {
        const int chunks = p.blocks * 4;
        for (int m = 0; m < p.mcount; ++m) {
            const long long r = source_row(m);
            for (int c = tid; c < chunks * 8; c += kThreads) {               // four floats each
                float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
                if (r >= 0 && c * 4 < p.H) w = *reinterpret_cast<const float4*>(static_cast<const T*>(p.x) + (size_t)r * p.H + c * 4);
                *reinterpret_cast<float4*>(reinterpret_cast<float*>(xs) + ((size_t)m * chunks + (c >> 3)) * kF32Chunk + (c & 7) * 4) = w;
            }
        }
    }
    __syncthreads();

    const int g = lane >> 2, t = lane & 3;
    // the lane's activation rows (columns of the product), and their states
    auto col_of = [&](int c) -> int { return kMma ? 2 * t + c : t; };
    BestQ4 best[kStates];
    float bias[kStates];
#pragma unroll
    for (int c = 0; c < kStates; ++c) {
        best[c].init();
        bias[c] = 0.f;
        const int m = col_of(c);
        if (m < p.mcount && p.blank_bias != nullptr) bias[c] = p.blank_bias[p.row_seq ? p.row_seq[p.m0 + m] : p.m0 + m];
    }
    // the warp's states of a draft slot, one for every row, to shared memory
    auto put_states = [&](int seg) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < kStates; ++c) {
            combine_best<28>(best[c].st, p.k);
            if (g == 0 && col_of(c) < kRows) best[c].st.store(&s_state[(seg * kWarps + warp) * kRows + col_of(c)]);
            best[c].init();
        }
    };
    int cur_seg = 0;
    // the panel's logits: z[c][u] is class g + 8u, row col_of(c)
    auto push = [&](int pan, const float (&z)[kStates][2]) __attribute__((always_inline)) {
        const int seg = pan >= n_seg0 ? 1 : 0, slot = slot0 + seg;
        if (seg != cur_seg) { put_states(0); cur_seg = 1; }
        const int v0 = (int)(p0 + pan - (long long)slot * p.panels) * kQ4Panel + g;
#pragma unroll
        for (int c = 0; c < kStates; ++c) {
            const int m = col_of(c);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int v = v0 + 8 * u;
                if (m < p.mcount && v < p.classes) {
                    const float zz = z[c][u] + (v == p.classes - 1 ? bias[c] : 0.f);
                    if (p.logits_dbg) p.logits_dbg[((size_t)(p.m0 + m) * p.slots + slot) * p.classes + v] = zz;
                    best[c].push(zz, v, p.k);
                }
            }
        }
    };

    const int gpb = kQ4Block / p.group;                                        // groups of a block
    const unsigned so_a = 1024u + (g * gpb + t * 32 / p.group) * 4, so_b = so_a + 8 * gpb * 4;
    const unsigned xstep = (unsigned)p.mcount * 64u;                          // bytes from a word's activations to the next word's
    const unsigned xblock = kMma ? 4u * xstep : 4u * kF32Chunk * 4u;
    const unsigned xrow = (g < p.mcount ? g : p.mcount - 1) * 64u + t * 16u;
    constexpr int kChains = 2;                                               // sums that run side by side (an instruction waits for the one before it in its own)
    float acc[kChains][4];
    // The tensor core cuts a sum's last bits off at every addition, always towards zero, so long chains drift: a piece's sums are
    // added here in rounded arithmetic and begin again (7B shape: log-probabilities off by 1.1e-6 without, MEASURED with).
    float tot[kStates][2];
    float facc[2][kF32Rows];
    auto clear = [&]() {
#pragma unroll
        for (int u = 0; u < kChains; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[u][q] = 0.f;
#pragma unroll
        for (int m = 0; m < kF32Rows; ++m) facc[0][m] = facc[1][m] = 0.f;
#pragma unroll
        for (int c = 0; c < kStates; ++c) tot[c][0] = tot[c][1] = 0.f;
    };
    clear();
    auto gather = [&]() {
#pragma unroll
        for (int c = 0; c < kStates; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) tot[c][u] += acc[0][2 * u + c] + acc[1][2 * u + c];
#pragma unroll
        for (int u = 0; u < kChains; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[u][q] = 0.f;
    };
    auto finish = [&](float (&z)[kStates][2]) __attribute__((always_inline)) {   // the sums as logits, and zero again
        if constexpr (kMma) {
#pragma unroll
            for (int c = 0; c < kStates; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u) z[c][u] = tot[c][u];
        } else {
#pragma unroll
            for (int m = 0; m < kF32Rows; ++m)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    facc[u][m] += __shfl_xor_sync(0xffffffffu, facc[u][m], 1);
                    facc[u][m] += __shfl_xor_sync(0xffffffffu, facc[u][m], 2);
                    if (t == m) z[0][u] = facc[u][m];
                }
        }
        clear();
    };

    PanelWalk at;
    at.init(npan, kWarps, warp, p.blocks);
    bool failed = false;
    uint32_t phase = 0u;
    for (int s = 0; !at.done();) {
        if (!tc::mbar_wait(my_full + s, phase, abort_flag)) { failed = true; break; }
        const int nb = min(p.piece, at.end - at.blk);
        const unsigned char* blk = my_ring + s * slot_bytes;
        const unsigned char* xb = xs + (unsigned)at.blk * xblock;
        for (int kb = 0; kb < nb; ++kb, blk += bb, xb += xblock) {
            const uint4 wa = *reinterpret_cast<const uint4*>(blk + lane * 16);
            const uint4 wb = *reinterpret_cast<const uint4*>(blk + 512 + lane * 16);
            const uint32_t sa = *reinterpret_cast<const uint32_t*>(blk + so_a);
            const uint32_t sb = *reinterpret_cast<const uint32_t*>(blk + so_b);
            const uint32_t a4[4] = {wa.x, wa.y, wa.z, wa.w}, b4[4] = {wb.x, wb.y, wb.z, wb.w};
            if constexpr (kMma) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 va = q4_values_bf16(a4[i], sa), vb = q4_values_bf16(b4[i], sb);
                    const uint4 x = *reinterpret_cast<const uint4*>(xb + i * xstep + xrow);
                    mma_16816(acc[0], va.x, vb.x, va.y, vb.y, x.x, x.y);
                    mma_16816(acc[1], va.z, vb.z, va.w, vb.w, x.z, x.w);
                }
            } else {
                const float* xf = reinterpret_cast<const float*>(xb) + t * kF32Chunk;
                const unsigned row = (unsigned)p.blocks * 4 * kF32Chunk;
                const float s0 = bf16lo(sa), o0 = bf16hi(sa), s1 = bf16lo(sb), o1 = bf16hi(sb);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float va[8], vb[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) { va[e] = q4_value_f32(a4[i], e, s0, o0); vb[e] = q4_value_f32(b4[i], e, s1, o1); }
#pragma unroll
                    for (int m = 0; m < kF32Rows; ++m) {
                        if (m >= p.mcount) break;
                        float x[8];
                        load8(xf + m * row + (i ^ ((t >> 1) << 1)) * 8, x);
#pragma unroll
                        for (int e = 0; e < 8; ++e) { facc[0][m] = fmaf(va[e], x[e], facc[0][m]); facc[1][m] = fmaf(vb[e], x[e], facc[1][m]); }
                    }
                }
            }
        }
        at.blk += nb;
        if constexpr (kMma) gather();
        __syncwarp();                                                        // the slot has been read
        ask(s);
        if (++s == p.nring) { s = 0; phase ^= 1u; }
        if (at.shared || at.blk < at.end) continue;
        float z[kStates][2];
        finish(z);
        push(at.pan, z);
        at.next_panel();
    }
    if (failed && lane == 0) {
        if (*abort_flag == 0) report_error(p.status, CTCSD_ERR_TIMEOUT, 43);
        *abort_flag = 1;
        // copies in flight land before the CTA's memory is given back (both parities: the newest fill of a slot has one of them)
        for (int s = 0; s < p.nring; ++s)
            for (uint32_t q = 0; q < 2; ++q) tc::mbar_wait_suspended(my_full + s, q, &sh->never_set, 1ll << 20);
    }
    __syncthreads();                                                         // all rings have been read
    if (*abort_flag != 0) return;                                            // (uniform: set before the barrier or not at all)
    // ---- the panels that were shared: partial sums through the rings' memory, one warp adds a panel's up ----
    if (at.whole < npan) {
        float* sums = reinterpret_cast<float*>(ring);                        // [warps][kStates * 2][32 lanes]
        float z[kStates][2];
        finish(z);
#pragma unroll
        for (int c = 0; c < kStates; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) sums[(warp * kStates * 2 + 2 * c + u) * 32 + lane] = z[c][u];
        __syncthreads();
        const int rest = npan - at.whole;
        if (warp < rest) {
#pragma unroll
            for (int c = 0; c < kStates; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    z[c][u] = 0.f;
                    for (int w = 0; w < at.per; ++w) z[c][u] += sums[((warp * at.per + w) * kStates * 2 + 2 * c + u) * 32 + lane];
                }
            push(at.whole + warp, z);
        }
    }
    const int segs = npan > n_seg0 ? 2 : 1;
#pragma unroll 1
    for (int seg = cur_seg; seg < segs; ++seg) put_states(seg);
    __syncthreads();
    // fold the warps' states: a warp, a (segment, row) at a time
    for (int i = warp; i < segs * p.mcount; i += kWarps) {
        const int seg = i / p.mcount, m = i - seg * p.mcount;
        RunState ms;
        ms.init();
        if (lane < kWarps) ms.absorb(s_state[(seg * kWarps + lane) * kRows + m]);
        combine_best<31>(ms, p.k);
        if (lane == 0) ms.store(p.part + ((size_t)m * gridDim.x + blockIdx.x) * 2 + seg);
    }
    draft_q4_finish(p, p.panels, 0, 1, slot0, segs, sh->merge);
}

int panels_of(const ctcsd_config& c) { return (c.V + 1 + kQ4Panel - 1) / kQ4Panel; }
int blocks_of(const ctcsd_config& c) { return (c.H + kQ4Block - 1) / kQ4Block; }

constexpr size_t kSmemBudget = kMaxDynamicSmem - 1024;                       // (1 KB of every CTA is the system's)

template <typename T>
size_t fixed_smem(int blocks, int rows) {
    return x_bytes<T>(blocks, rows) + sizeof(RingState) + sizeof(DraftPartial) * 2 * Shape<T>::warps * (sizeof(T) == 2 ? 8 : kF32Rows);
}

// Ring geometry: blocks of a slot, slots of a warp.  False where there is no room for two blocks a warp.
template <typename T>
bool ring_shape(DraftQ4Params& p) {
    constexpr size_t warps = Shape<T>::warps;
    const size_t fixed = fixed_smem<T>(p.blocks, p.mcount);
    if (fixed > kSmemBudget) return false;
    const size_t bb = (size_t)q4_block_bytes(p.group), most = (kSmemBudget - fixed) / (warps * bb);        // blocks there is room for, a warp
    if (most < 2) return false;
    // two slots, of 8 blocks at most; three where they are small then
    p.piece = (int)(most / 2 < 8 ? most / 2 : 8);
    if (p.piece > p.blocks) p.piece = p.blocks;
    p.nring = (int)(most / p.piece < kMaxRing ? most / p.piece : kMaxRing);
    return true;
}

template <typename T>
int launch_pass(Handle* h, cudaStream_t s, DraftQ4Params& p) {
    if (!ring_shape<T>(p)) return CTCSD_ERR_UNSUPPORTED;
    const size_t smem = fixed_smem<T>(p.blocks, p.mcount) + (size_t)Shape<T>::warps * p.nring * p.piece * q4_block_bytes(p.group);
    auto kern = draft_q4_kernel<T>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, sizeof(T) == 4 ? kPrepDraftQ4F32 : kPrepDraftQ4, kern));
    const long long total = (long long)p.panels * p.slots;
    const unsigned grid = (unsigned)(total < h->num_sms ? total : h->num_sms);        // (total >= slots: a range touches two slots at most)
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(grid), dim3(Shape<T>::warps * 32), smem, s, 1, p));
    h->launches++;
    return CTCSD_OK;
}

bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }

}  // namespace
}  // namespace ctcsd

using namespace ctcsd;

extern "C" int ctcsd_weights_q4_bytes(const ctcsd_config* cfg, int group, size_t* out_bytes) {
    if (!cfg || !out_bytes || !group_ok(group)) return CTCSD_ERR_INVALID_ARG;
    const int rc = validate_config(*cfg);
    if (rc != CTCSD_OK) return rc;
    *out_bytes = (size_t)cfg->T * panels_of(*cfg) * blocks_of(*cfg) * q4_block_bytes(group);
    return CTCSD_OK;
}

extern "C" int ctcsd_quantize_weights_q4(ctcsd_handle* hh, void* stream, const void* Wd, int group, void* out_Wq) {
    if (!hh || !Wd || !out_Wq || !group_ok(group)) return CTCSD_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(Wd) | reinterpret_cast<uintptr_t>(out_Wq)) & 15) return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    PackParams p;
    p.W = Wd; p.out = static_cast<unsigned char*>(out_Wq);
    p.H = c.H; p.classes = c.V + 1; p.panels = panels_of(c); p.blocks = blocks_of(c); p.group = group;
    const DeviceGuard on(h->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid(p.blocks, p.panels < 65535 ? p.panels : 65535, c.T);
    if (c.dtype == CTCSD_DTYPE_BF16) quantize_weights_q4_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(p);
    else quantize_weights_q4_kernel<float><<<grid, 256, 0, s>>>(p);
    CTCSD_LAUNCH_CHECK(h);
    order_kernel<<<1, 32, 0, s>>>();
    CTCSD_LAUNCH_CHECK(h);
    return CTCSD_OK;
}

extern "C" int ctcsd_draft_logits_q4(ctcsd_handle* hh, void* stream, int M, const void* x, int x_row_count, const int* x_rows,
                                     const void* Wq, int group, const int* row_seq, const float* blank_bias,
                                     int* out_topk_id, float* out_topk_lp, float* out_lse, float* out_logits_dbg) {
    if (!hh || !x || !Wq || !out_topk_id || !out_topk_lp || !out_lse || !group_ok(group)) return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    if (M < 1 || M > c.max_draft_rows || (x_rows ? x_row_count < 1 : x_row_count < M)) return CTCSD_ERR_INVALID_ARG;
    if (!row_seq && blank_bias && M > c.B) return CTCSD_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(Wq)) & 15) return CTCSD_ERR_INVALID_ARG;
    DraftQ4Params p = {};
    p.x = x; p.x_rows = x_rows; p.x_row_count = x_row_count;
    p.W = static_cast<const unsigned char*>(Wq);
    p.row_seq = row_seq; p.blank_bias = blank_bias;
    p.H = c.H; p.classes = c.V + 1; p.panels = panels_of(c); p.blocks = blocks_of(c); p.group = group; p.slots = c.T;
    p.part = reinterpret_cast<DraftPartial*>(h->ws + h->lay.draft_part_off);
    p.counter = counter_ptr(h);
    p.k = c.k; p.out_topk_id = out_topk_id; p.out_topk_lp = out_topk_lp; p.out_lse = out_lse; p.logits_dbg = out_logits_dbg;
    p.status = status_ptr(h);
    const DeviceGuard on(h->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf16 = c.dtype == CTCSD_DTYPE_BF16;
    // more than 8 rows: the tensor memory's kernel, whose cost hardly depends on the rows (7B shape: 8 rows 108 us here, 16 rows 185 us there)
    if (bf16 && M > 8 && c.H >= 64) {
        for (int m0 = 0; m0 < M; m0 += kDraftQ4TcRows) {
            p.m0 = m0;
            p.mcount = M - m0 < kDraftQ4TcRows ? M - m0 : kDraftQ4TcRows;
            const int rc = launch_draft_q4_tc(h, s, p);
            if (rc != CTCSD_OK) return rc;
        }
        return CTCSD_OK;
    }
    // rows of a pass: 8 (float32: 4), or as many as leave the rings room
    auto fits = [&](int rows) {
        DraftQ4Params q = p;
        q.mcount = rows;
        return bf16 ? ring_shape<__nv_bfloat16>(q) : ring_shape<float>(q);
    };
    int per_pass = bf16 ? 8 : kF32Rows;
    if (per_pass > M) per_pass = M;
    while (per_pass > 1 && !fits(per_pass)) per_pass = (per_pass + 1) / 2;
    for (int m0 = 0; m0 < M; m0 += per_pass) {
        p.m0 = m0;
        p.mcount = M - m0 < per_pass ? M - m0 : per_pass;
        const int rc = bf16 ? launch_pass<__nv_bfloat16>(h, s, p) : launch_pass<float>(h, s, p);
        if (rc != CTCSD_OK) return rc;
    }
    return CTCSD_OK;
}
