// Draft head over 4-bit weights: ctcsd_quantize_weights_q4 (packs them once) and ctcsd_draft_logits_q4.
//   z[m,t,v] = sum_h x[m,h] w[t,v,h] (+ blank_bias on v == V),  w = round(origin + scale (16 + q)) per group along h;
//   log-sum-exp and the k best per (m, t), as ctcsd_draft_logits.
//
// Packed weights.  Sixteen neighbouring classes of a slot are a panel (the last one of a slot filled up with zero rows), 128
// hidden elements of a panel a block, blocks of a panel follow one another:
//   block = levels [4 chunks][16 classes][16 bytes], the 32 elements of a chunk as four words (q4.cuh);
//           pairs  [16 classes][128 / group] (scale, origin).
// Neighbouring lanes take neighbouring classes, so that reads of 16 bytes a lane meet in no bank, and a panel is one piece of memory.
//
// bfloat16: draft_logits_q4_tc.cu.  float32: the kernel below.
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
    int* status;
};

// One warp per two classes of a block: lane = (class parity, eight elements).
template <typename T>
__global__ void __launch_bounds__(256) quantize_weights_q4_kernel(PackParams p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kb = blockIdx.x, t = blockIdx.z;
    const int bytes = q4_block_bytes(p.group), per = p.group / 8;                // lanes of a group
    for (int panel = blockIdx.y; panel < p.panels; panel += gridDim.y) {
        const size_t base = (((size_t)t * p.panels + panel) * p.blocks + kb) * (bytes / 4);
        uint32_t* blk = reinterpret_cast<uint32_t*>(p.out) + base;
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
        const int at = ((e >> 5) * kQ4Panel + r) * 4 + ((e >> 3) & 3), at_so = 256 + r * (kQ4Block / p.group) + e / p.group;
        const long long room = (long long)gridDim.z * p.panels * p.blocks * (bytes / 4);
        if (CTCSD_IN_BOUNDS(p.status, 163, base + at, room)) blk[at] = w;
        if ((lane & 15) % per == 0 && CTCSD_IN_BOUNDS(p.status, 164, base + at_so, room)) blk[at_so] = so;
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

constexpr int kRows = 4;                 // activation rows of a pass
constexpr int kMaxRing = 4;              // ring slots of a warp
constexpr int kWarps = 16, kThreads = kWarps * 32;

__host__ __device__ inline size_t x_bytes(int blocks, int rows) { return (size_t)rows * blocks * kQ4Block * 4; }

struct __align__(8) RingState {
    uint64_t full[kWarps * kMaxRing];
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

// float32.  One CTA per SM with a contiguous range of panels.  Every warp streams panels of its own through a small ring in shared memory with the
// bulk-copy engine (its first lane asks for the next piece when a slot has been read); lane = (chunk t, class g and g + 8) makes values and multiplies
// them with the activations of its chunk, held in shared memory; the sums of the four chunks are joined by shuffles, and lane (t, g) keeps the
// running maximum, sum of exponentials and best k of row t.  Warps meet at the end only.  A weight takes four instructions (three to pick its level, a
// multiply-add for its value) and one a row, which is half of the time where there are many weights: 5 slots of 32001 classes, H = 4096: 170 us for 1 row, 259 for
// 4 (its bytes 53; the instructions alone 88 and 141).  Small shapes are latency: 1 row of 256 x 4004 15 us, 4 rows and 26 million weights 28.
__global__ void __launch_bounds__(kThreads, 1) draft_q4_f32_kernel(DraftQ4Params p) {
    extern __shared__ __align__(128) unsigned char dyn[];
    unsigned char* xs = dyn;
    unsigned char* ring = xs + x_bytes(p.blocks, p.mcount);
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
    const int quads = p.blocks * (kQ4Block / 4);
    for (int m = 0; m < p.mcount; ++m) {
        const long long r = source_row(m);
        for (int c = tid; c < quads; c += kThreads) {                        // four floats each
            float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r >= 0 && c * 4 < p.H) w = *reinterpret_cast<const float4*>(static_cast<const float*>(p.x) + (size_t)r * p.H + c * 4);
            reinterpret_cast<float4*>(xs)[(size_t)m * quads + c] = w;
        }
    }
    __syncthreads();

    const int g = lane & 7, t = lane >> 3;
    BestQ4 best;                                                              // of row t
    best.init();
    float bias = 0.f;
    if (t < p.mcount && p.blank_bias != nullptr) bias = p.blank_bias[p.row_seq ? p.row_seq[p.m0 + t] : p.m0 + t];
    // the warp's states of a draft slot, one for every row, to shared memory
    auto put_states = [&](int seg) __attribute__((always_inline)) {
        combine_best<7>(best.st, p.k);
        if (g == 0 && CTCSD_IN_BOUNDS(p.status, 166, (seg * kWarps + warp) * kRows + t, 2 * kWarps * kRows))
            best.st.store(&s_state[(seg * kWarps + warp) * kRows + t]);
        best.init();
    };
    int cur_seg = 0;
    // the panel's logits: z[u] is class g + 8u, row t
    auto push = [&](int pan, const float (&z)[2]) __attribute__((always_inline)) {
        const int seg = pan >= n_seg0 ? 1 : 0, slot = slot0 + seg;
        if (seg != cur_seg) { put_states(0); cur_seg = 1; }
        const int v0 = (int)(p0 + pan - (long long)slot * p.panels) * kQ4Panel + g;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int v = v0 + 8 * u;
            if (t < p.mcount && v < p.classes) {
                const float zz = z[u] + (v == p.classes - 1 ? bias : 0.f);
                const size_t o = ((size_t)(p.m0 + t) * p.slots + slot) * p.classes + v;
                if (p.logits_dbg && CTCSD_IN_BOUNDS(p.status, 165, o, (long long)p.rows * p.slots * p.classes)) p.logits_dbg[o] = zz;
                best.push(zz, v, p.k);
            }
        }
    };

    const int gpb = kQ4Block / p.group;                                        // groups of a block
    const unsigned so_a = 1024u + (g * gpb + t * 32 / p.group) * 4, so_b = so_a + 8 * gpb * 4;
    float acc[2][kRows];
    auto clear = [&]() {
#pragma unroll
        for (int m = 0; m < kRows; ++m) acc[0][m] = acc[1][m] = 0.f;
    };
    clear();
    auto finish = [&](float (&z)[2]) __attribute__((always_inline)) {         // the sums as logits, and zero again
#pragma unroll
        for (int m = 0; m < kRows; ++m)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                acc[u][m] += __shfl_xor_sync(0xffffffffu, acc[u][m], 8);
                acc[u][m] += __shfl_xor_sync(0xffffffffu, acc[u][m], 16);
                if (t == m) z[u] = acc[u][m];
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
        const float* xb = reinterpret_cast<const float*>(xs) + (size_t)at.blk * kQ4Block + t * 32;
        const unsigned row = (unsigned)p.blocks * kQ4Block;
        for (int kb = 0; kb < nb; ++kb, blk += bb, xb += kQ4Block) {
            const uint4 wa = *reinterpret_cast<const uint4*>(blk + (t * kQ4Panel + g) * 16);
            const uint4 wb = *reinterpret_cast<const uint4*>(blk + (t * kQ4Panel + g + 8) * 16);
            const uint32_t sa = *reinterpret_cast<const uint32_t*>(blk + so_a);
            const uint32_t sb = *reinterpret_cast<const uint32_t*>(blk + so_b);
            const uint32_t a4[4] = {wa.x, wa.y, wa.z, wa.w}, b4[4] = {wb.x, wb.y, wb.z, wb.w};
            const float s0 = bf16lo(sa), o0 = bf16hi(sa), s1 = bf16lo(sb), o1 = bf16hi(sb);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float va[8], vb[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) { va[e] = q4_value_f32(a4[i], e, s0, o0); vb[e] = q4_value_f32(b4[i], e, s1, o1); }
#pragma unroll
                for (int m = 0; m < kRows; ++m) {
                    if (m >= p.mcount) break;
                    float x[8];
                    load8(xb + m * row + i * 8, x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) { acc[0][m] = fmaf(va[e], x[e], acc[0][m]); acc[1][m] = fmaf(vb[e], x[e], acc[1][m]); }
                }
            }
        }
        at.blk += nb;
        __syncwarp();                                                        // the slot has been read
        ask(s);
        if (++s == p.nring) { s = 0; phase ^= 1u; }
        if (at.shared || at.blk < at.end) continue;
        float z[2];
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
        float* sums = reinterpret_cast<float*>(ring);                        // [warps][2][32 lanes]
        float z[2];
        finish(z);
#pragma unroll
        for (int u = 0; u < 2; ++u) sums[(warp * 2 + u) * 32 + lane] = z[u];
        __syncthreads();
        const int rest = npan - at.whole;
        if (warp < rest) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                z[u] = 0.f;
                for (int w = 0; w < at.per; ++w) z[u] += sums[((warp * at.per + w) * 2 + u) * 32 + lane];
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
        const size_t o = ((size_t)m * gridDim.x + blockIdx.x) * 2 + seg;
        if (lane == 0 && CTCSD_IN_BOUNDS(p.status, 167, o, p.part_room)) ms.store(p.part + o);
    }
    draft_q4_finish(p, p.panels, slot0, segs, sh->merge);
}

int panels_of(const ctcsd_config& c) { return (c.V + 1 + kQ4Panel - 1) / kQ4Panel; }
int blocks_of(const ctcsd_config& c) { return (c.H + kQ4Block - 1) / kQ4Block; }

constexpr size_t kSmemBudget = kMaxDynamicSmem - 1024;                       // (1 KB of every CTA is the system's)

size_t fixed_smem(int blocks, int rows) { return x_bytes(blocks, rows) + sizeof(RingState) + sizeof(DraftPartial) * 2 * kWarps * kRows; }

// Ring geometry: blocks of a slot, slots of a warp.  False where there is no room for two blocks a warp.
bool ring_shape(DraftQ4Params& p) {
    const size_t fixed = fixed_smem(p.blocks, p.mcount);
    if (fixed > kSmemBudget) return false;
    const size_t bb = (size_t)q4_block_bytes(p.group), most = (kSmemBudget - fixed) / (kWarps * bb);       // blocks there is room for, a warp
    if (most < 2) return false;
    // two slots, of 8 blocks at most; three where they are small then
    p.piece = (int)(most / 2 < 8 ? most / 2 : 8);
    if (p.piece > p.blocks) p.piece = p.blocks;
    p.nring = (int)(most / p.piece < kMaxRing ? most / p.piece : kMaxRing);
    return true;
}

int launch_pass(Handle* h, cudaStream_t s, DraftQ4Params& p) {
    if (!ring_shape(p)) return CTCSD_ERR_UNSUPPORTED;
    const size_t smem = fixed_smem(p.blocks, p.mcount) + (size_t)kWarps * p.nring * p.piece * q4_block_bytes(p.group);
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepDraftQ4F32, draft_q4_f32_kernel));
    const long long total = (long long)p.panels * p.slots;
    const unsigned grid = (unsigned)(total < h->num_sms ? total : h->num_sms);        // (total >= slots: a range touches two slots at most)
    CTCSD_CUDA_CHECK(h, launch_pdl(draft_q4_f32_kernel, dim3(grid), dim3(kThreads), smem, s, 1, p));
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
    p.status = status_ptr(h);
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
    p.rows = M;
    p.part = reinterpret_cast<DraftPartial*>(h->ws + h->lay.draft_part_off);
    p.part_room = (long long)((h->lay.part_slot_off - h->lay.draft_part_off) / sizeof(DraftPartial));
    p.counter = counter_ptr(h);
    p.k = c.k; p.out_topk_id = out_topk_id; p.out_topk_lp = out_topk_lp; p.out_lse = out_lse; p.logits_dbg = out_logits_dbg;
    p.status = status_ptr(h);
    const DeviceGuard on(h->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf16 = c.dtype == CTCSD_DTYPE_BF16;
    // rows of a pass (float32: or as many as leave the rings room)
    int per_pass = bf16 ? kDraftQ4TcRows : kRows;
    if (per_pass > M) per_pass = M;
    auto fits = [&](int rows) {
        DraftQ4Params q = p;
        q.mcount = rows;
        return ring_shape(q);
    };
    while (!bf16 && per_pass > 1 && !fits(per_pass)) per_pass = (per_pass + 1) / 2;
    for (int m0 = 0; m0 < M; m0 += per_pass) {
        p.m0 = m0;
        p.mcount = M - m0 < per_pass ? M - m0 : per_pass;
        const int rc = bf16 ? launch_draft_q4_tc(h, s, p) : launch_pass(h, s, p);
        if (rc != CTCSD_OK) return rc;
    }
    return CTCSD_OK;
}
