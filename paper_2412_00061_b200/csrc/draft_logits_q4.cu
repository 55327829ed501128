// Draft head over 4-bit weights: ctcsd_quantize_weights_q4 (packs them once) and ctcsd_draft_logits_q4.
//   z[m,t,v] = sum_h x[m,h] w[t,v,h] (+ blank_bias on v == V),  w = round(origin + scale (16 + q)) per group along h;
//   log-sum-exp and the k best per (m, t), as ctcsd_draft_logits.
//
// Packed weights.  Sixteen neighbouring classes of a slot are a panel (the last one of a slot filled up with zero rows), 128
// hidden elements of a panel a block, blocks of a panel follow one another:
//   block = levels [2][32 lanes][16 bytes], lane 4g + t of half h: class 8h + g, elements 32t .. 32t + 31, four words (q4.cuh);
//           pairs  [16 classes][128 / group] (scale, origin).
// This is the order in which the lanes of a warp hold the operand A of mma.m16n8k16 (with the hidden index permuted alike for x),
// so a lane takes its share of a block by two 16-byte reads without bank conflicts, and a panel is one piece of memory.
#include "q4.cuh"
#include "run_state.cuh"
#include "tc_primitives.cuh"

#include <limits.h>
#include <math.h>

namespace ctcsd {
namespace {

constexpr int kWarps = 8;                // warps that multiply: they share a panel's blocks
constexpr int kPanel = 16;               // classes of a panel
constexpr int kBlock = 128;              // hidden elements of a block
constexpr int kMaxSlots = 16;            // ring slots
constexpr int kDepth = 4;                // panels whose partial sums are on their way to the epilogue

__host__ __device__ inline int block_bytes(int group) { return 1024 + kPanel * 4 * (kBlock / group); }

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
    const int bytes = block_bytes(p.group), per = p.group / 8;                // lanes of a group
    for (int panel = blockIdx.y; panel < p.panels; panel += gridDim.y) {
        unsigned char* blk = p.out + (((size_t)t * p.panels + panel) * p.blocks + kb) * bytes;
        const int r = warp * 2 + (lane >> 4), e = (lane & 15) * 8;            // class of the panel, first element of the block
        const int cls = panel * kPanel + r, k = kb * kBlock + e;
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
        const bool some = cls < p.classes && kb * kBlock + e / p.group * p.group < p.H;
        const uint32_t so = some ? q4_scale_origin(lo, hi) : 0u;
        const uint32_t w = in ? q4_word(v, so) : 0u;
        reinterpret_cast<uint32_t*>(blk)[(r >> 3) * 128 + ((r & 7) * 4 + (e >> 5)) * 4 + ((e >> 3) & 3)] = w;
        if ((lane & 15) % per == 0) reinterpret_cast<uint32_t*>(blk + 1024)[r * (kBlock / p.group) + e / p.group] = so;
    }
}

// Launched behind the packing without the attribute that lets kernels overlap: the draft head begins to read weights
// before its predecessor in the stream has ended, and that must not be the kernel that writes them.
__global__ void order_kernel() {}

struct DraftQ4Params {
    const void* x;                       // [x_row_count,H]
    const int* x_rows;                   // [M] or null
    int x_row_count;
    const unsigned char* W;              // packed
    const int* row_seq;
    const float* blank_bias;
    int m0, mcount;                      // rows of this pass
    int H, classes, panels, blocks, group;   // panels per draft slot, blocks per panel
    int slots;                           // draft slots (T)
    int piece_blocks, pieces;            // blocks of a piece, pieces of a panel
    int slot_pieces, nring;              // pieces of a ring slot (whole panels, or a piece of one), ring slots
    DraftPartial* part;                  // [rows of a pass][grid][2]
    int* part_slot;                      // [grid][2]
    unsigned* counter;
    int k;
    int* out_topk_id;
    float* out_topk_lp;
    float* out_lse;
    float* logits_dbg;
    int* status;
};

struct __align__(8) RingState {
    uint64_t full[kMaxSlots], empty[kMaxSlots];
    uint64_t cfull[kDepth], cempty[kDepth];
    int abort_flag, never_set, is_last;
};

// D[16x8] += A[16x16] * B[16x8], bf16 operands, fp32 accumulators (warp-wide).
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int kF32Rows = 4;              // activation rows of a float32 pass
constexpr int kF32Chunk = 36;            // floats from one 32-element chunk of x to the next (four lanes read four chunks: no bank conflict)

template <typename T, int NT> struct XShape;
// bfloat16: fragments of B, [block][tile][word][lane][16 bytes]; float32: [row][chunk][36 floats]
template <int NT> struct XShape<__nv_bfloat16, NT> {
    __host__ __device__ static size_t bytes(int blocks) { return (size_t)blocks * NT * 2048; }
};
template <int NT> struct XShape<float, NT> {
    __host__ __device__ static size_t bytes(int blocks) { return (size_t)kF32Rows * blocks * 4 * kF32Chunk * 4; }
};

template <int NT> struct Threads { static constexpr int value = (kWarps + 1 + 4 * NT) * 32; };

// One CTA per SM with a contiguous range of panels.  Warp 8 streams them through a ring in shared memory with the bulk-copy engine.  Warps
// 0..7 share the blocks of every panel: levels to values (one multiply-add for two), values times activations on the tensor
// cores (bfloat16: 16 classes x 8 rows an instruction; float32: fused multiply-adds); the eight partial sums of a panel
// go through a small ring to the epilogue warps, a thread per (class of the panel, row), which keep the running maximum, sum of
// exponentials and best eight.  The CTA that ends last merges all states.
template <typename T, int NT>
__global__ void __launch_bounds__(Threads<NT>::value, 1) draft_q4_kernel(DraftQ4Params p) {
    constexpr bool kMma = sizeof(T) == 2;
    constexpr int kThreads = Threads<NT>::value;
    constexpr int kRows = 8 * NT;
    extern __shared__ __align__(128) unsigned char dyn[];
    unsigned char* xs = dyn;
    unsigned char* ring = xs + XShape<T, NT>::bytes(p.blocks);
    const int bb = block_bytes(p.group);
    const int piece_bytes = p.piece_blocks * bb, slot_bytes = p.slot_pieces * piece_bytes;
    RingState* sh = reinterpret_cast<RingState*>(ring + (size_t)p.nring * slot_bytes);
    float* cpart = reinterpret_cast<float*>(sh + 1);                         // [kDepth][kWarps][16][kRows]
    DraftPartial* s_part = reinterpret_cast<DraftPartial*>(ring);            // [2][16][kRows], over the ring when it has been read
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        for (int s = 0; s < p.nring; ++s) { tc::mbar_init(&sh->full[s], 1); tc::mbar_init(&sh->empty[s], kWarps); }
        for (int d = 0; d < kDepth; ++d) { tc::mbar_init(&sh->cfull[d], kWarps); tc::mbar_init(&sh->cempty[d], 4 * NT); }
        sh->abort_flag = 0;
        sh->never_set = 0;
        sh->is_last = 0;
        tc::fence_barrier_init();
    }
    __syncthreads();

    const long long total = (long long)p.panels * p.slots;
    const long long p0 = total * blockIdx.x / gridDim.x, p1 = total * (blockIdx.x + 1) / gridDim.x;
    const int npan = (int)(p1 - p0);
    const int slot0 = (int)(p0 / p.panels);                                   // draft slot of the first panel
    const int n_seg0 = (int)(((long long)(slot0 + 1) * p.panels < p1 ? (long long)(slot0 + 1) * p.panels : p1) - p0);
    // the CTA's stream of pieces: blocks piece_blocks * i .. of a panel (its last piece may be shorter)
    const size_t panel_bytes = (size_t)p.blocks * bb;
    const int npieces = npan * p.pieces;
    const int nfill = (npieces + p.slot_pieces - 1) / p.slot_pieces;

    const uint64_t policy = tc::policy_evict_first();
    int prod_j = 0;
    bool prod_ok = true;
    // bytes of the CTA's stream before piece i
    auto offset_of = [&](int i) -> size_t {
        const int pan = i / p.pieces;
        return (size_t)pan * panel_bytes + (size_t)(i - pan * p.pieces) * piece_bytes;
    };
    auto issue_fill = [&](int j) -> bool {
        const int s = j % p.nring;
        if (!tc::mbar_wait(&sh->empty[s], ((uint32_t)(j / p.nring) & 1u) ^ 1u, abort_flag)) return false;
        const int i0 = j * p.slot_pieces, i1 = i0 + p.slot_pieces < npieces ? i0 + p.slot_pieces : npieces;
        const size_t from = offset_of(i0), bytes = offset_of(i1) - from;
        if (bytes == 0 || bytes > (size_t)slot_bytes || (bytes & 15) != 0) {  // never hand the copy engine a range outside the ring
            report_error(p.status, CTCSD_ERR_INTERNAL, 41);
            return false;
        }
        tc::mbar_arrive_expect_tx(&sh->full[s], (uint32_t)bytes);
        tc::bulk_load_1d(ring + (size_t)s * slot_bytes, p.W + (size_t)p0 * panel_bytes + from, (uint32_t)bytes, &sh->full[s], policy);
        return true;
    };
    // (weights are not written while they are in use: the ring fills while the predecessor in the stream drains)
    if (warp == kWarps && lane == 0)
        while (prod_ok && prod_j < nfill && prod_j < p.nring) {
            prod_ok = issue_fill(prod_j);
            if (prod_ok) ++prod_j;
        }
    pdl_wait();
    pdl_trigger();
    // ---- activations to shared memory, in the order in which the lanes take them ----
    auto source_row = [&](int m) -> long long {                              // -1: none
        if (m >= p.mcount) return -1;
        long long r = p.m0 + m;
        if (p.x_rows != nullptr) {
            r = p.x_rows[p.m0 + m];
            if (r < 0 || r >= p.x_row_count) { report_error(p.status, CTCSD_ERR_INVALID_ARG, p.m0 + m); r = -1; }
        }
        return r;
    };
    if constexpr (kMma) {
        const int pieces16 = p.blocks * 16;                                  // 16-byte pieces of a row: [block][chunk t][word i]
        for (int m = warp; m < kRows; m += kThreads / 32) {                  // (a warp, a row)
            const long long r = source_row(m);
            for (int c = lane; c < pieces16; c += 32) {
                uint4 w = make_uint4(0u, 0u, 0u, 0u);
                if (r >= 0 && c * 8 < p.H) w = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.x) + (size_t)r * p.H + c * 8);
                const int kb = c >> 4, t = (c >> 2) & 3, i = c & 3;
                *reinterpret_cast<uint4*>(xs + ((((size_t)kb * NT + (m >> 3)) * 4 + i) * 32 + (m & 7) * 4 + t) * 16) = w;
            }
        }
    } else {
        const int chunks = p.blocks * 4;
        for (int m = 0; m < kF32Rows; ++m) {
            const long long r = source_row(m);
            for (int c = tid; c < chunks * 8; c += kThreads) {               // four floats each
                float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
                if (r >= 0 && c * 4 < p.H) w = *reinterpret_cast<const float4*>(static_cast<const T*>(p.x) + (size_t)r * p.H + c * 4);
                *reinterpret_cast<float4*>(reinterpret_cast<float*>(xs) + ((size_t)m * chunks + (c >> 3)) * kF32Chunk + (c & 7) * 4) = w;
            }
        }
    }
    __syncthreads();

    bool failed = false;
    RunState st;
    st.init();
    int cur_seg = 0;
    const int ei = (warp - kWarps - 1) * 32 + lane;                          // epilogue: class of the panel, row of the pass
    const int own_r = ei / kRows, own_m = ei - own_r * kRows;
    const bool owner = warp > kWarps && own_m < p.mcount;
    RunState first_seg;                                                      // (filled when the CTA's range enters the next draft slot)
    first_seg.init();
    if (warp == kWarps) {
        // ---------------- producer ----------------
        if (lane == 0) {
            bool ok = prod_ok;
            int j = prod_j;
            while (ok && j < nfill) {
                ok = issue_fill(j);
                if (ok) ++j;
            }
            if (!ok) {
                if (*abort_flag == 0) report_error(p.status, CTCSD_ERR_TIMEOUT, 42);
                *abort_flag = 1;
            }
            if (*abort_flag != 0)                                            // copies in flight land before the CTA's memory is given back
                for (int back = 1; back <= p.nring && back <= j; ++back) {
                    const int q = j - back;
                    tc::mbar_wait(&sh->full[q % p.nring], (uint32_t)(q / p.nring) & 1u, &sh->never_set, 1ll << 24);
                }
        }
    } else if (warp < kWarps) {
        // ---------------- products ----------------
        const int g = lane >> 2, t = lane & 3;
        const int gpb = kBlock / p.group, gi = t * 32 / p.group;             // groups of a block, this lane's
        float acc[2][NT][4];
        float facc[2][kF32Rows];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[u][nt][q] = 0.f;
#pragma unroll
            for (int m = 0; m < kF32Rows; ++m) facc[u][m] = 0.f;
        }
        int pan = 0, part_of = 0;                                            // panel and piece of it
        for (int j = 0; j < nfill && !failed; ++j) {
            const int s = j % p.nring;
            if (!tc::mbar_wait(&sh->full[s], (uint32_t)(j / p.nring) & 1u, abort_flag)) { failed = true; break; }
            const int here = npieces - j * p.slot_pieces < p.slot_pieces ? npieces - j * p.slot_pieces : p.slot_pieces;
            size_t at = 0;
            for (int pc = 0; pc < here; ++pc) {
                const int b0 = part_of * p.piece_blocks;
                const int nb = p.blocks - b0 < p.piece_blocks ? p.blocks - b0 : p.piece_blocks;
                const unsigned char* base = ring + (size_t)s * slot_bytes + at;
                for (int kb = warp; kb < nb; kb += kWarps) {
                    const unsigned char* blk = base + (size_t)kb * bb;
                    const uint4 wa = *reinterpret_cast<const uint4*>(blk + lane * 16);
                    const uint4 wb = *reinterpret_cast<const uint4*>(blk + 512 + lane * 16);
                    const uint32_t sa = *reinterpret_cast<const uint32_t*>(blk + 1024 + (g * gpb + gi) * 4);
                    const uint32_t sb = *reinterpret_cast<const uint32_t*>(blk + 1024 + ((g + 8) * gpb + gi) * 4);
                    const uint32_t a4[4] = {wa.x, wa.y, wa.z, wa.w}, b4[4] = {wb.x, wb.y, wb.z, wb.w};
                    if constexpr (kMma) {
                        const uint4* xf = reinterpret_cast<const uint4*>(xs) + (size_t)(b0 + kb) * NT * 128 + lane;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint4 va = q4_values_bf16(a4[i], sa), vb = q4_values_bf16(b4[i], sb);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                const uint4 x = xf[(nt * 4 + i) * 32];
                                mma_16816(acc[0][nt], va.x, vb.x, va.y, vb.y, x.x, x.y);
                                mma_16816(acc[1][nt], va.z, vb.z, va.w, vb.w, x.z, x.w);
                            }
                        }
                    } else {
                        const float* xf = reinterpret_cast<const float*>(xs) + ((size_t)(b0 + kb) * 4 + t) * kF32Chunk;
                        const size_t row = (size_t)p.blocks * 4 * kF32Chunk;
                        const float s0 = bf16lo(sa), o0 = bf16hi(sa), s1 = bf16lo(sb), o1 = bf16hi(sb);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float va[8], vb[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) { va[e] = q4_value_f32(a4[i], e, s0, o0); vb[e] = q4_value_f32(b4[i], e, s1, o1); }
#pragma unroll
                            for (int m = 0; m < kF32Rows; ++m) {
                                float x[8];
                                load8(xf + m * row + i * 8, x);
#pragma unroll
                                for (int e = 0; e < 8; ++e) { facc[0][m] = fmaf(va[e], x[e], facc[0][m]); facc[1][m] = fmaf(vb[e], x[e], facc[1][m]); }
                            }
                        }
                    }
                }
                at += (size_t)nb * bb;
                if (++part_of < p.pieces) continue;
                // ---- the panel's partial sums ----
                part_of = 0;
                const int d = pan % kDepth;
                if (!tc::mbar_wait(&sh->cempty[d], ((uint32_t)(pan / kDepth) & 1u) ^ 1u, abort_flag)) { failed = true; break; }
                float* cp = cpart + (size_t)(d * kWarps + warp) * kPanel * kRows;
                if constexpr (kMma) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        *reinterpret_cast<float2*>(cp + g * kRows + nt * 8 + 2 * t) = make_float2(acc[0][nt][0] + acc[1][nt][0], acc[0][nt][1] + acc[1][nt][1]);
                        *reinterpret_cast<float2*>(cp + (g + 8) * kRows + nt * 8 + 2 * t) = make_float2(acc[0][nt][2] + acc[1][nt][2], acc[0][nt][3] + acc[1][nt][3]);
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[0][nt][q] = acc[1][nt][q] = 0.f;
                    }
                } else {
#pragma unroll
                    for (int m = 0; m < kF32Rows; ++m) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            facc[u][m] += __shfl_xor_sync(0xffffffffu, facc[u][m], 1);
                            facc[u][m] += __shfl_xor_sync(0xffffffffu, facc[u][m], 2);
                            if (t == 0) cp[(g + 8 * u) * kRows + m] = facc[u][m];
                            facc[u][m] = 0.f;
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sh->cfull[d]);
                ++pan;
            }
            __syncwarp();
            if (lane == 0 && !failed) tc::mbar_arrive(&sh->empty[s]);
        }
        if (failed && lane == 0) {
            if (*abort_flag == 0) report_error(p.status, CTCSD_ERR_TIMEOUT, 43);
            *abort_flag = 1;
        }
    } else {
        // ---------------- epilogue ----------------
        float bias = 0.f;
        if (owner && p.blank_bias != nullptr) bias = p.blank_bias[p.row_seq ? p.row_seq[p.m0 + own_m] : p.m0 + own_m];
        for (int pan = 0; pan < npan; ++pan) {
            const int d = pan % kDepth;
            if (!tc::mbar_wait(&sh->cfull[d], (uint32_t)(pan / kDepth) & 1u, abort_flag)) { failed = true; break; }
            float z = 0.f;
            if (owner) {
                const float* cp = cpart + (size_t)d * kWarps * kPanel * kRows + own_r * kRows + own_m;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) z += cp[w * kPanel * kRows];
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sh->cempty[d]);
            const int seg = pan >= n_seg0 ? 1 : 0, slot = slot0 + seg;
            const int v = (int)(p0 + pan - (long long)slot * p.panels) * kPanel + own_r;
            if (owner && v < p.classes) {
                if (seg != cur_seg) { first_seg = st; st.init(); cur_seg = 1; }
                if (v == p.classes - 1) z += bias;
                if (p.logits_dbg) p.logits_dbg[((size_t)(p.m0 + own_m) * p.slots + slot) * p.classes + v] = z;
                st.push(z, v);
            }
        }
        if (failed && lane == 0) {
            if (*abort_flag == 0) report_error(p.status, CTCSD_ERR_TIMEOUT, 44);
            *abort_flag = 1;
        }
    }
    __syncthreads();                                                         // the ring has been read (or, after a failure, has landed)
    if (*abort_flag != 0) return;                                            // (uniform: set before the barrier or not at all)
    if (owner) {
        RunState none;
        none.init();
        (cur_seg == 0 ? st : first_seg).store(&s_part[own_r * kRows + own_m]);
        (cur_seg == 0 ? none : st).store(&s_part[(kPanel + own_r) * kRows + own_m]);
    }
    __syncthreads();
    // fold the CTA's states: a warp, a (segment, row) at a time
    for (int i = warp; i < 2 * p.mcount; i += kThreads / 32) {
        const int seg = i / p.mcount, m = i - seg * p.mcount;
        RunState ms;
        ms.init();
        if (lane < kPanel) ms.absorb(s_part[(seg * kPanel + lane) * kRows + m]);
        warp_combine(ms);
        if (lane == 0) ms.store(p.part + ((size_t)m * gridDim.x + blockIdx.x) * 2 + seg);
    }
    if (tid < 2) p.part_slot[blockIdx.x * 2 + tid] = (tid == 0 ? n_seg0 : npan - n_seg0) > 0 ? slot0 + tid : -1;
    __threadfence();
    __syncthreads();
    if (tid == 0) sh->is_last = atomicAdd(p.counter, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!sh->is_last) return;
    __threadfence();
    for (int task = warp; task < p.mcount * p.slots; task += kThreads / 32) {
        const int m = task / p.slots, slot = task - m * p.slots;
        RunState fs;
        fs.init();
        // the CTAs whose panels touch this draft slot are neighbours
        const long long n = gridDim.x, lo = (long long)slot * p.panels, hi = lo + p.panels;
        long long c0 = lo * n / total, c1 = hi * n / total;
        while (c0 > 0 && total * c0 / n > lo) --c0;
        if (c1 > n - 1) c1 = n - 1;
        for (long long c = c0 + lane; c <= c1; c += 32) {
            const int seg = slot - (int)((total * c / n) / p.panels);
            if (seg < 0 || seg > 1) continue;
            const int e = (int)(2 * c + seg);
            if (__ldcg(p.part_slot + e) == slot) fs.absorb(load_partial_cg(p.part + (size_t)m * n * 2 + e));
        }
        warp_combine(fs);
        if (lane == 0) {
            const int row = p.m0 + m;
            const float lse = fs.mx + logf(fs.sum);
            p.out_lse[(size_t)row * p.slots + slot] = lse;
#pragma unroll
            for (int j = 0; j < kTopSlots; ++j)
                if (j < p.k) {
                    const size_t o = ((size_t)row * p.slots + slot) * p.k + j;
                    p.out_topk_id[o] = fs.id[j];
                    p.out_topk_lp[o] = fs.val[j] - lse;
                }
        }
    }
    if (tid == 0) *p.counter = 0u;
}

int panels_of(const ctcsd_config& c) { return (c.V + 1 + kPanel - 1) / kPanel; }
int blocks_of(const ctcsd_config& c) { return (c.H + kBlock - 1) / kBlock; }

constexpr size_t kSmemBudget = kMaxDynamicSmem - 1024;                       // (1 KB of every CTA is the system's)

template <typename T, int NT>
size_t fixed_smem(int blocks) {
    return XShape<T, NT>::bytes(blocks) + sizeof(RingState) + sizeof(float) * kDepth * kWarps * kPanel * 8 * NT;
}

// Ring geometry: pieces of a panel and pieces of a slot.  False where not even two slots fit.
template <typename T, int NT>
bool ring_shape(DraftQ4Params& p) {
    const size_t fixed = fixed_smem<T, NT>(p.blocks);
    const size_t state = sizeof(DraftPartial) * 2 * kPanel * 8 * NT;         // the states at the end lie over the ring
    if (fixed + state > kSmemBudget) return false;
    const size_t room = kSmemBudget - fixed;
    const size_t bb = (size_t)block_bytes(p.group), panel = bb * p.blocks;
    // slots of about a third of the room, at most 40 KB: whole panels where they are smaller, else equal parts of one
    size_t want = room / 3 < 40 * 1024 ? room / 3 : 40 * 1024;
    if (panel <= want) {
        p.pieces = 1;
        p.piece_blocks = p.blocks;
        p.slot_pieces = (int)(want / panel);
    } else {
        p.pieces = (int)((panel + want - 1) / want);
        p.piece_blocks = (p.blocks + p.pieces - 1) / p.pieces;
        p.pieces = (p.blocks + p.piece_blocks - 1) / p.piece_blocks;
        p.slot_pieces = 1;
    }
    const size_t slot = (size_t)p.slot_pieces * p.piece_blocks * bb;
    size_t n = room / slot;
    if (n > kMaxSlots) n = kMaxSlots;
    while (n * slot < state && n < kMaxSlots) ++n;                           // (tiny panels: the states need the room)
    if (n < 2 || n * slot < state || n * slot > room) return false;
    p.nring = (int)n;
    return true;
}

template <typename T, int NT>
int launch_pass(Handle* h, cudaStream_t s, DraftQ4Params& p) {
    if (!ring_shape<T, NT>(p)) return CTCSD_ERR_UNSUPPORTED;
    const size_t smem = fixed_smem<T, NT>(p.blocks) + (size_t)p.nring * p.slot_pieces * p.piece_blocks * block_bytes(p.group);
    auto kern = draft_q4_kernel<T, NT>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, sizeof(T) == 4 ? kPrepDraftQ4F32 : (NT == 1 ? kPrepDraftQ4 : kPrepDraftQ4x2), kern));
    const long long total = (long long)p.panels * p.slots;
    const unsigned grid = (unsigned)(total < h->num_sms ? total : h->num_sms);        // (total >= slots: a range touches two slots at most)
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(grid), dim3(Threads<NT>::value), smem, s, 1, p));
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
    *out_bytes = (size_t)cfg->T * panels_of(*cfg) * blocks_of(*cfg) * block_bytes(group);
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
    p.part_slot = reinterpret_cast<int*>(h->ws + h->lay.part_slot_off);
    p.counter = counter_ptr(h);
    p.k = c.k; p.out_topk_id = out_topk_id; p.out_topk_lp = out_topk_lp; p.out_lse = out_lse; p.logits_dbg = out_logits_dbg;
    p.status = status_ptr(h);
    const DeviceGuard on(h->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf16 = c.dtype == CTCSD_DTYPE_BF16;
    DraftQ4Params probe = p;
    const bool wide = bf16 && M > 8 && ring_shape<__nv_bfloat16, 2>(probe);
    const int per_pass = bf16 ? (wide ? 16 : 8) : kF32Rows;
    for (int m0 = 0; m0 < M; m0 += per_pass) {
        p.m0 = m0;
        p.mcount = M - m0 < per_pass ? M - m0 : per_pass;
        int rc;
        if (!bf16) rc = launch_pass<float, 1>(h, s, p);
        else rc = p.mcount > 8 ? launch_pass<__nv_bfloat16, 2>(h, s, p) : launch_pass<__nv_bfloat16, 1>(h, s, p);
        if (rc != CTCSD_OK) return rc;
    }
    return CTCSD_OK;
}
