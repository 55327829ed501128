// Draft head over 4-bit weights for more than 8 activation rows, on the 5th-generation tensor cores (tcgen05 + TMEM).
//
// D[128 x 192] = A[128 x H] B[192 x H]^T per tile: A = up to 128 activation rows, B = twelve panels of weights (draft_q4.cuh) as bfloat16 values,
// both K-major with the 128-byte swizzle, 128 hidden elements to a stage, two stages; D in tensor memory (lane = activation row, column
// = class), twice, so that a tile is read back while the next one is multiplied.
// Twelve warps each take one panel of the tile from a ring that one TMA copy fills for all of them (a warp that asked for its own panel spent some 600
// cycles on every request), turn its levels into values and write them into the stage, a 128-element block of 16 classes by
// eight 16-byte stores a lane, which meet in no bank.  The cost hardly depends on the activation rows, so 9 to 128 of them take one pass.
// Roles: warps 0-3 read the accumulators back (a quarter of the activation rows each), 4-15 make values, 16 loads activations, 17
// issues the products, 18 loads levels.
#include "draft_q4.cuh"
#include "tc_primitives.cuh"

namespace ctcsd {
namespace {

constexpr int kEpi = 4;
constexpr int kStages = 2;
constexpr int kMaxRing = 8;
constexpr int kMakers = 12;              // warps that make values: one panel of the tile each
constexpr int kThreads = (kEpi + kMakers + 3) * 32;
constexpr int kTileN = kMakers * kQ4Panel, kBBytes = kTileN * kQ4Block * 2;
constexpr int kAccCols = 256;            // columns from one accumulator to the other

struct __align__(8) TcState {
    uint64_t raw_full[kMaxRing], raw_empty[kMaxRing];    // levels of the tile's panels, a few blocks of each
    uint64_t a_full[kStages], b_full[kStages], empty[kStages];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort_flag, never_set, merge[2];
};

struct TcGeo {
    int tiles;                           // tiles of a draft slot
    int a_rows;                          // activation rows of a stage: 64 or 128 (products read 128: with 64, the rows behind are whatever follows, and their
                                         // sums are not looked at)
    int rows, copies;                    // they are `copies` times `rows`
};

__device__ __forceinline__ void give_up(TcState* sh, int* status, int site) {
    volatile int* f = &sh->abort_flag;
    if (*f == 0) report_error(status, CTCSD_ERR_TIMEOUT, site);
    *f = 1;
}

__global__ void __launch_bounds__(kThreads, 1) draft_q4_tc_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, DraftQ4Params p,
                                                                              TcGeo geo) {
    extern __shared__ __align__(1024) unsigned char dyn[];
    const int a_plane = geo.a_rows * 128, a_bytes = 2 * a_plane, stage_bytes = a_bytes + kBBytes;   // (a plane: 64 elements)
    unsigned char* ring = dyn + kStages * stage_bytes;
    const int bb = q4_block_bytes(p.group), slot_bytes = (kMakers * p.piece * bb + 127) / 128 * 128;
    TcState* sh = reinterpret_cast<TcState*>(ring + (size_t)p.nring * slot_bytes);
    if ((tc::smem_u32(dyn) & 1023u) != 0u) {                   // uniform over the CTA
        if (threadIdx.x == 0) report_error(p.status, CTCSD_ERR_INTERNAL, 45);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        for (int s = 0; s < p.nring; ++s) { tc::mbar_init(&sh->raw_full[s], 1); tc::mbar_init(&sh->raw_empty[s], kMakers); }
        for (int s = 0; s < kStages; ++s) { tc::mbar_init(&sh->a_full[s], 1); tc::mbar_init(&sh->b_full[s], kMakers); tc::mbar_init(&sh->empty[s], 1); }
        for (int a = 0; a < 2; ++a) { tc::mbar_init(&sh->acc_full[a], 1); tc::mbar_init(&sh->acc_empty[a], kEpi); }
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
    const uint32_t tmem = sh->tmem_base;
    // this CTA's tiles: u0 .. u1-1 of the line of all slots' tiles
    const long long total = (long long)geo.tiles * p.slots;
    const int u0 = (int)(total * blockIdx.x / gridDim.x), u1 = (int)(total * (blockIdx.x + 1) / gridDim.x);
    const int slot0 = u0 / geo.tiles;
    const int segs = u1 > (slot0 + 1) * geo.tiles ? 2 : 1;
    // Every CTA begins at a place of its own along the hidden axis (and wraps), so that at any moment the CTAs ask L2 for different parts of the
    // activations that they all share.
    const int pieces = (p.blocks + p.piece - 1) / p.piece, start = (int)((long long)blockIdx.x * pieces / gridDim.x);
    bool failed = false;

    if (warp < kEpi) {
        // ---------------- logits ----------------
        pdl_wait();
        pdl_trigger();
        // A warp reads a quarter of the tensor memory's lanes.  Up to 32 rows stand there twice, and two warps take turns with chunks of 32
        // columns (four copies take room from the ring: 444 us against 400 for 32 rows of the 70B shape).
        const int copy = warp * 32 / geo.rows, row = warp * 32 + lane, m = row - copy * geo.rows;
        const uint32_t lane_addr = tmem + ((uint32_t)(warp * 32) << 16);
        const bool live = row < geo.a_rows && m < p.mcount, warp_live = warp * 32 < geo.a_rows && m - lane < p.mcount;
        float bias = 0.f;
        if (live && p.blank_bias != nullptr) bias = p.blank_bias[p.row_seq ? p.row_seq[p.m0 + m] : p.m0 + m];
        RunState st;
        st.init();
        float floor = -INFINITY;                               // a logit has to be above it to be among the k best,
        int have = 0;                                          // unless the list holds fewer
        int n = 0, seg = 0;
        for (int u = u0; u < u1; ++u, ++n) {
            const int slot = u / geo.tiles, v0 = (u - slot * geo.tiles) * kTileN;
            if (slot - slot0 != seg) {
                if (live) st.store(p.part + ((size_t)row * gridDim.x + blockIdx.x) * 2);
                st.init();
                floor = -INFINITY;
                have = 0;
                seg = 1;
            }
            if (!tc::mbar_wait_suspended(&sh->acc_full[n & 1], (uint32_t)(n >> 1) & 1u, abort_flag)) failed = true;
            failed = __any_sync(0xffffffffu, failed);
            if (failed) break;
            tc::tc_fence_after_sync();
            if (warp_live) {
#pragma unroll 1
                for (int c0 = copy * 32; c0 < kTileN && v0 + c0 < p.classes; c0 += 32 * geo.copies) {
                    uint32_t r[32];
                    const uint32_t addr = lane_addr + (uint32_t)((n & 1) * kAccCols + c0);
                    tc::tmem_read32(addr, r);
                    const int left = p.classes - v0 - c0;      // classes of the chunk
                    const bool blank = left <= 32;             // its last one is the blank
                    float top = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        float z = __uint_as_float(r[j]);
                        if (blank && j == left - 1) z += bias;
                        if (j < left) {
                            if (p.logits_dbg != nullptr && live)
                                p.logits_dbg[((size_t)(p.m0 + m) * p.slots + slot) * p.classes + v0 + c0 + j] = z;
                        } else {
                            z = -INFINITY;
                        }
                        r[j] = __float_as_uint(z);
                        top = fmaxf(top, z);
                    }
                    if (top > st.mx) {
                        st.sum *= __expf(st.mx - top);         // exp(-inf) = 0 covers the first chunk
                        st.mx = top;
                    }
                    uint32_t above = 0u;                       // logits that may be among the best
                    float add = 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const float z = __uint_as_float(r[j]);
                        add += j < left ? __expf(z - st.mx) : 0.f;
                        above |= z > floor ? 1u << j : 0u;
                    }
                    st.sum += add;
                    if (have < p.k) above = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
                    // every lane takes its own, the largest first, so that few come to be tried (at most one more than stay)
                    while (__any_sync(0xffffffffu, above != 0u)) {
                        float z = -INFINITY;
                        int at = -1;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const bool better = ((above >> j) & 1u) && (at < 0 || __uint_as_float(r[j]) > z);
                            z = better ? __uint_as_float(r[j]) : z;
                            at = better ? j : at;
                        }
                        if (at >= 0) {
                            above &= ~(1u << at);
                            if (z > floor || have < p.k) {
                                topk_insert(st.val, st.id, z, v0 + c0 + at);
                                have += z == z ? 1 : 0;
#pragma unroll
                                for (int s = 0; s < kTopSlots; ++s) {
                                    float f = st.val[s];
                                    asm("" : "+f"(f));         // (else the compiler makes it a look-up by k, and the list leaves the registers)
                                    if (s == p.k - 1) floor = f;
                                }
                            } else {
                                above = 0u;
                            }
                        }
                    }
                }
            }
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sh->acc_empty[n & 1]);
        }
        if (failed && lane == 0) give_up(sh, p.status, 46);
        if (!failed && live) st.store(p.part + ((size_t)row * gridDim.x + blockIdx.x) * 2 + seg);
    } else if (warp < kEpi + kMakers) {
        // ---------------- values ----------------
        pdl_wait();
        pdl_trigger();
        const int mk = warp - kEpi;
        const int g = lane >> 2, t = lane & 3;
        const int gpb = kQ4Block / p.group;
        const unsigned so_a = 1024u + (g * gpb + t * 32 / p.group) * 4, so_b = so_a + 8 * gpb * 4;
        // word i of row g: place in the stage (row g + 8 stands 1024 bytes behind)
        unsigned put[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            put[i] = a_bytes + (t >> 1) * (kTileN * 128) + (mk * kQ4Panel + g) * 128 + ((((t & 1) * 4 + (i ^ ((t >> 1) << 1))) ^ g) << 4);
        int it = 0, s = 0;
        uint32_t phase = 0u;
        for (int u = u0; u < u1 && !failed; ++u) {
            const bool there = (u % geo.tiles) * kMakers + mk < p.panels;     // (behind a slot's last panel: nothing to make)
            for (int pc = 0, at = start; pc < pieces && !failed; ++pc, at = at + 1 == pieces ? 0 : at + 1) {
                const int nb = min(p.piece, p.blocks - at * p.piece);
                if (!tc::mbar_wait_suspended(&sh->raw_full[s], phase, abort_flag)) failed = true;
                for (int kb = 0; kb < nb; ++kb, ++it) {
                    const int st = it % kStages;
                    if (!failed && !tc::mbar_wait_suspended(&sh->empty[st], ((uint32_t)(it / kStages) & 1u) ^ 1u, abort_flag)) failed = true;
                    failed = __any_sync(0xffffffffu, failed);
                    if (failed) break;
                    if (there) {
                        const unsigned char* blk = ring + s * slot_bytes + (mk * p.piece + kb) * bb;
                        unsigned char* dst = dyn + st * stage_bytes;
                        const uint4 wa = *reinterpret_cast<const uint4*>(blk + lane * 16);
                        const uint4 wb = *reinterpret_cast<const uint4*>(blk + 512 + lane * 16);
                        const uint32_t sa = *reinterpret_cast<const uint32_t*>(blk + so_a);
                        const uint32_t sb = *reinterpret_cast<const uint32_t*>(blk + so_b);
                        const uint32_t a4[4] = {wa.x, wa.y, wa.z, wa.w}, b4[4] = {wb.x, wb.y, wb.z, wb.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            *reinterpret_cast<uint4*>(dst + put[i]) = q4_values_bf16(a4[i], sa);
                            *reinterpret_cast<uint4*>(dst + put[i] + 1024) = q4_values_bf16(b4[i], sb);
                        }
                        tc::fence_proxy_async();
                    }
                    __syncwarp();
                    if (lane == 0) {
                        tc::mbar_arrive(&sh->b_full[st]);
                        if (kb == nb - 1) tc::mbar_arrive(&sh->raw_empty[s]);
                    }
                }
                if (++s == p.nring) { s = 0; phase ^= 1u; }
            }
        }
        if (failed && lane == 0) give_up(sh, p.status, 47);
    } else if (warp == kEpi + kMakers + 2) {
        // ---------------- levels ----------------
        if (lane == 0) {
            // (weights are not written while they are in use: the ring fills while the predecessor in the stream drains, and nothing else is
            // read before this kernel's other warps have waited for it)
            const uint64_t pol = tc::policy_evict_first();
            const uint32_t bytes = (uint32_t)(kMakers * p.piece * bb);
            int s = 0, fill = 0;
            uint32_t phase = 1u;
            for (int u = u0; u < u1 && !failed; ++u) {
                const int slot = u / geo.tiles, pan = slot * p.panels + (u - slot * geo.tiles) * kMakers;
                for (int pc = 0, at = start; pc < pieces; ++pc, at = at + 1 == pieces ? 0 : at + 1, ++fill) {
                    if (fill == p.nring) {
                        pdl_wait();
                        pdl_trigger();
                    }
                    if (!tc::mbar_wait_suspended(&sh->raw_empty[s], phase, abort_flag)) { failed = true; break; }
                    tc::mbar_arrive_expect_tx(&sh->raw_full[s], bytes);
                    // (64 bytes x the blocks' lines x twelve panels; what lies behind a panel's end or the last panel arrives as zeros)
                    tc::tma_load_3d(ring + s * slot_bytes, &tmW, &sh->raw_full[s], 0, at * p.piece * (bb / 64), pan, pol);
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
            const int steps = (u1 - u0) * p.blocks;
            int it = 0, kb = start * p.piece;
            for (; it < steps; ++it) {
                const int st = it % kStages;
                if (!tc::mbar_wait_suspended(&sh->empty[st], ((uint32_t)(it / kStages) & 1u) ^ 1u, abort_flag)) { failed = true; break; }
                unsigned char* dst = dyn + st * stage_bytes;
                tc::mbar_arrive_expect_tx(&sh->a_full[st], (uint32_t)a_bytes);
                // (elements behind H and rows behind the last are outside the tensor and arrive as zeros)
                for (int c = 0; c < geo.copies; ++c) {
                    tc::tma_load_2d(dst + c * geo.rows * 128, &tmX, &sh->a_full[st], kb * kQ4Block, 0, pol);
                    tc::tma_load_2d(dst + a_plane + c * geo.rows * 128, &tmX, &sh->a_full[st], kb * kQ4Block + 64, 0, pol);
                }
                if (++kb == p.blocks) kb = 0;
            }
            if (failed) {
                give_up(sh, p.status, 48);
                for (int back = 1; back <= kStages && back <= it; ++back) {              // copies in flight land before the exit
                    const int j = it - back;
                    tc::mbar_wait_suspended(&sh->a_full[j % kStages], (uint32_t)(j / kStages) & 1u, &sh->never_set, 1ll << 24);
                }
            }
        }
    } else {
        // ---------------- products ----------------
        pdl_wait();
        pdl_trigger();
        if (lane == 0) {
            const uint32_t idesc = tc::idesc_bf16_f32(128, kTileN);
            int it = 0, n = 0;
            for (int u = u0; u < u1 && !failed; ++u, ++n) {
                const uint32_t d = tmem + (uint32_t)((n & 1) * kAccCols);
                if (!tc::mbar_wait_suspended(&sh->acc_empty[n & 1], ((uint32_t)(n >> 1) & 1u) ^ 1u, abort_flag)) { failed = true; break; }
                tc::tc_fence_after_sync();
                for (int kb = 0; kb < p.blocks; ++kb, ++it) {
                    const int st = it % kStages;
                    const uint32_t ph = (uint32_t)(it / kStages) & 1u;
                    if (!tc::mbar_wait_suspended(&sh->a_full[st], ph, abort_flag) || !tc::mbar_wait_suspended(&sh->b_full[st], ph, abort_flag)) { failed = true; break; }
                    tc::tc_fence_after_sync();
                    const uint32_t base = tc::smem_u32(dyn + st * stage_bytes);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint64_t adesc = tc::smem_desc_k_sw128(base + (uint32_t)(half * a_plane));
                        const uint64_t bdesc = tc::smem_desc_k_sw128(base + (uint32_t)(a_bytes + half * (kTileN * 128)));
#pragma unroll
                        for (int k = 0; k < 4; ++k)            // 16 elements along K = 32 bytes
                            tc::mma_bf16_ss(d, adesc + 2 * k, bdesc + 2 * k, idesc, (kb | half | k) != 0 ? 1u : 0u);
                    }
                    tc::mma_commit(&sh->empty[st]);
                }
                if (!failed) tc::mma_commit(&sh->acc_full[n & 1]);
            }
            if (failed) give_up(sh, p.status, 49);
        }
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    if (warp == kEpi + kMakers + 1) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc(tmem, 512);
    }
    if (*abort_flag != 0) return;                              // (uniform: set before the barrier or not at all)
    draft_q4_finish(p, geo.tiles, geo.rows, geo.copies, slot0, segs, sh->merge);
}

// Activation rows picked by a row map, one behind the other; a map that leaves x gives a zero row.
__global__ void __launch_bounds__(256) draft_q4_gather_kernel(const uint4* x, int x_row_count, const int* x_rows, int m0, int chunks, uint4* out, int* status) {
    pdl_wait();
    pdl_trigger();
    const int m = blockIdx.x, r = x_rows[m0 + m];
    const bool there = r >= 0 && r < x_row_count;
    if (!there && threadIdx.x == 0) report_error(status, CTCSD_ERR_INVALID_ARG, m0 + m);
    for (int c = threadIdx.x; c < chunks; c += 256) out[(size_t)m * chunks + c] = there ? x[(size_t)r * chunks + c] : make_uint4(0u, 0u, 0u, 0u);
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

// Packed weights as [panels][lines][64 bytes], box = [twelve panels][`lines` lines][64 bytes].
bool make_w_map(CUtensorMap* map, const void* w, long long panels, int panel_bytes, int lines) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {16, (cuuint64_t)(panel_bytes / 64), (cuuint64_t)panels};
    cuuint64_t strides[2] = {64, (cuuint64_t)panel_bytes};
    cuuint32_t box[3] = {16, (cuuint32_t)lines, (cuuint32_t)kMakers};
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
                                       p.H / 8, rows, p.status));
        h->launches++;
        x = reinterpret_cast<const __nv_bfloat16*>(rows);
    }
    p.part = reinterpret_cast<DraftPartial*>(h->ws + h->lay.q4_part_off);
    TcGeo geo;
    geo.tiles = (p.panels + kMakers - 1) / kMakers;
    geo.rows = p.mcount <= 32 ? 32 : (p.mcount <= 64 ? 64 : 128);
    geo.a_rows = geo.rows <= 64 ? 64 : 128;
    geo.copies = geo.a_rows / geo.rows;
    const size_t bb = q4_block_bytes(p.group), fixed = (size_t)kStages * (geo.a_rows * 256 + kBBytes) + sizeof(TcState);
    // ring slots of two blocks a panel where three of them fit, else of one
    const size_t room = kMaxDynamicSmem - 1024 - fixed;
    p.piece = p.blocks > 1 && room >= 3 * (kMakers * 2 * bb + 128) ? 2 : 1;
    const size_t slot = (kMakers * p.piece * bb + 127) / 128 * 128;
    p.nring = (int)(room / slot < kMaxRing ? room / slot : kMaxRing);
    if (p.nring < 2) return CTCSD_ERR_UNSUPPORTED;
    CUtensorMap tmX;
    CUtensorMap tmW;
    if (!make_x_map(&tmX, x, p.mcount, p.H, geo.rows) ||
        !make_w_map(&tmW, p.W, (long long)p.panels * p.slots, (int)(p.blocks * bb), (int)(p.piece * bb / 64))) return CTCSD_ERR_CUDA;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepDraftQ4Tc, draft_q4_tc_kernel));
    const long long total = (long long)geo.tiles * p.slots;
    const unsigned grid = (unsigned)(total < h->num_sms ? total : h->num_sms);         // (total >= slots: a range touches two slots at most)
    CTCSD_CUDA_CHECK(h, launch_pdl(draft_q4_tc_kernel, dim3(grid), dim3(kThreads), fixed + p.nring * slot, s, 1, tmX, tmW, p, geo));
    h->launches++;
    return CTCSD_OK;
}

}  // namespace ctcsd
