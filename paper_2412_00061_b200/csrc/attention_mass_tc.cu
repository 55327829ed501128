// Attention mass for bf16 on the 5th-generation tensor cores (tcgen05 + TMEM): many query rows.
//
// A block of 128 keys is the M side of S[128 x R] = K Q^T (keys as TMA brings them, the path's rows as the N
// side), so a thread of the epilogue owns a key and adds up its R weights by itself: no exchange between
// lanes, no atomics, a fixed order.  Persistent CTAs, two per SM where the rows leave room (one's change of rows hides
// behind the other, and the next call's set-up behind this one's end), each with a span of the line of key blocks.
//   warp 0       K blocks into a ring (TMA, 128-byte swizzle);
//   warp 1       MMAs, S alternating between two places in tensor memory;
//   warps 4-11   epilogue, four warps per place; together they also bring the query rows of a (sequence, kv head)
//                into shared memory.
// HBM bounds it while the rows are few: a 128-key block costs 512 cycles of tensor core, 8 R of exponentials (128 R at 16 a
// clock) and 1400 of memory (700 at head dimension 64), so that from about 175 rows (90) on the exponentials do.
// Measured: 179 MB (32 sequences, 8 kv heads, up to 7 x 8 query rows) in 36.5 us, 4.9 TB/s; 112 MB (8 sequences, 8 kv heads, up to 9 x 24 rows) in
// 57.6 us, 1.9 TB/s.
#include "attention_mass.cuh"
#include "tc_primitives.cuh"

namespace ctcsd {
namespace {

constexpr int kThreads = 384;
constexpr int kKeys = 128;
constexpr int kMaxRows = 256;          // query rows per pass (the N side of an MMA); more rows take another pass over K
constexpr int kMaxStages = 8;

struct __align__(8) MassShared {
    uint64_t k_full[kMaxStages], k_empty[kMaxStages];
    uint64_t q_full, s_full[2], s_empty[2];
    uint32_t tmem_base;
    int abort_flag, never_set;
};

__device__ __forceinline__ void give_up(MassShared* sh, int* status, int site) {
    volatile int* f = &sh->abort_flag;
    if (*f == 0) report_error(status, CTCSD_ERR_TIMEOUT, site);
    *f = 1;
}
__device__ __forceinline__ void epilogue_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
attention_mass_tc_kernel(const __grid_constant__ CUtensorMap tmK, MassParams p, int rcap, int stages, int place) {
    constexpr int kTile = kKeys * D * 2;
    extern __shared__ __align__(1024) unsigned char dyn[];
    unsigned char* Ks = dyn;                                     // [stages][DH][128 keys][128 B]
    unsigned char* Qs = Ks + (size_t)stages * kTile;             // [DH][rcap rows][128 B]
    float* nlse = reinterpret_cast<float*>(Qs + (size_t)rcap * D * 2);      // [rcap] minus the row's log-sum-exp, log2 units
    MassShared* sh = reinterpret_cast<MassShared*>(nlse + rcap);
    int* cum = reinterpret_cast<int*>(sh + 1);                   // [B+1]
    if ((tc::smem_u32(dyn) & 1023u) != 0u) {                     // uniform over the CTA
        if (threadIdx.x == 0) report_error(p.status, CTCSD_ERR_INTERNAL, 44);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh->abort_flag;
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) { tc::mbar_init(&sh->k_full[s], 1); tc::mbar_init(&sh->k_empty[s], 1); }
        tc::mbar_init(&sh->q_full, 1);
        for (int s = 0; s < 2; ++s) { tc::mbar_init(&sh->s_full[s], 1); tc::mbar_init(&sh->s_empty[s], 4); }
        sh->abort_flag = 0;
        sh->never_set = 0;
        tc::fence_barrier_init();
    }
    if (warp == 1) {
        tc::tmem_alloc(&sh->tmem_base, (uint32_t)(2 * place));
        tc::tmem_relinquish();
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    const uint32_t tmem = sh->tmem_base;                         // S: columns 0 and `place`
    pdl_wait();
    pdl_trigger();
    mass_plan(p, kKeys, cum);
    const int grp = p.Hq / p.Hkv;
    const long long total = (long long)cum[p.B] * p.Hkv;
    const long long xbeg = total * blockIdx.x / gridDim.x, xend = total * (blockIdx.x + 1) / gridDim.x;
    bool failed = false;

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (lane == 0) {
            const uint64_t pol = tc::policy_evict_first();
            int fill = 0;
            for (long long x = xbeg; x < xend && !failed;) {
                const MassPiece m = mass_piece(p, cum, x, xend);
                x += m.blk1 - m.blk0;
                // (one pass whatever the path's length, where the longest fits)
                const int R = rcap < kMaxRows ? 1 : (p.acc_len[m.b] + 1) * grp;
                for (int r0 = 0; r0 < R && !failed; r0 += kMaxRows)
                    for (int blk = m.blk0; blk < m.blk1; ++blk, ++fill) {
                        const int s = fill % stages;
                        if (!tc::mbar_wait_suspended(&sh->k_empty[s], ((uint32_t)(fill / stages) & 1u) ^ 1u, abort_flag)) { failed = true; break; }
                        tc::mbar_arrive_expect_tx(&sh->k_full[s], (uint32_t)kTile);
                        tc::tma_load_5d(Ks + (size_t)s * kTile, &tmK, &sh->k_full[s], 0, blk * kKeys, 0, m.g, m.b, pol);
                    }
            }
            if (failed) {
                give_up(sh, p.status, 41);
                for (int back = 1; back <= stages && back <= fill; ++back) {       // copies in flight land before the exit
                    const int j = fill - back;
                    tc::mbar_wait(&sh->k_full[j % stages], (uint32_t)(j / stages) & 1u, &sh->never_set, 1ll << 24);
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0) {
            const uint64_t kdesc0 = tc::smem_desc_k_sw128(tc::smem_u32(Ks)), qdesc0 = tc::smem_desc_k_sw128(tc::smem_u32(Qs));
            int fill = 0, pass = 0;
            bool ok = true;
            for (long long x = xbeg; x < xend && ok;) {
                const MassPiece m = mass_piece(p, cum, x, xend);
                x += m.blk1 - m.blk0;
                const int R = (p.acc_len[m.b] + 1) * grp;
                for (int r0 = 0; r0 < R && ok; r0 += kMaxRows, ++pass) {
                    const int cols = (min(R - r0, kMaxRows) + 15) / 16 * 16;
                    const uint32_t idesc = tc::idesc_bf16_f32(kKeys, cols);
                    ok = tc::mbar_wait_suspended(&sh->q_full, (uint32_t)pass & 1u, abort_flag);
                    for (int blk = m.blk0; blk < m.blk1 && ok; ++blk, ++fill) {
                        const int s = fill % stages, buf = fill & 1;
                        ok = tc::mbar_wait_suspended(&sh->k_full[s], (uint32_t)(fill / stages) & 1u, abort_flag) &&
                             tc::mbar_wait_suspended(&sh->s_empty[buf], ((uint32_t)(fill >> 1) & 1u) ^ 1u, abort_flag);
                        if (!ok) break;
                        tc::tc_fence_after_sync();
                        const uint64_t kdesc = kdesc0 + (uint64_t)((s * kTile) >> 4);
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk)
                            tc::mma_bf16_ss(tmem + (uint32_t)(buf * place), kdesc + (uint64_t)((kk / 4) * ((kKeys * 128) >> 4) + 2 * (kk % 4)),
                                            qdesc0 + (uint64_t)((kk / 4) * ((rcap * 128) >> 4) + 2 * (kk % 4)), idesc, kk != 0 ? 1u : 0u);
                        tc::mma_commit(&sh->k_empty[s]);
                        tc::mma_commit(&sh->s_full[buf]);
                    }
                }
            }
            if (!ok) give_up(sh, p.status, 42);
        }
    } else if (warp >= 4) {
        // ---------------- epilogue: one thread per key ----------------
        // Every epilogue thread executes every barrier, also after a wait has failed.
        const int buf = (warp - 4) >> 2;                         // place in tensor memory: blocks of this parity
        const int kl = (warp & 3) * 32 + lane;                   // key of the block
        const uint32_t tmem_s = tmem + (uint32_t)(buf * place) + ((uint32_t)((warp & 3) * 32) << 16);
        const int et = tid - 128;                                // 0..255
        const float sl2 = p.scale * kMassLog2e;
        int fill = 0;
        for (long long x = xbeg; x < xend;) {
            const MassPiece m = mass_piece(p, cum, x, xend);
            x += m.blk1 - m.blk0;
            const int kv = p.kv_len[m.b], acc = p.acc_len[m.b], base = kv - 1 - acc;
            const int R = (acc + 1) * grp;
            const size_t krow0 = ((size_t)m.b * p.Hkv + m.g) * (size_t)p.Lcap;
            for (int r0 = 0; r0 < R; r0 += kMaxRows) {
                const int nr = min(R - r0, kMaxRows), cols = (nr + 15) / 16 * 16;
                __threadfence_block();                           // (a later pass reads the mass that this one wrote)
                epilogue_barrier();                              // every S of the previous rows has been read
                constexpr int LR = D / 8;                        // 16-byte chunks of a row
                for (int i = et; i < cols * LR; i += 256) {
                    const int r = i / LR, cc = i % LR;
                    uint4 w = make_uint4(0u, 0u, 0u, 0u);
                    if (r < nr) {
                        const size_t qr = mass_query_row(p, m.b, m.g, grp, r0 + r);
                        const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.Q) + qr * D) + cc);
                        if (mass_row_counts(p.lse[qr])) w = q;
                    }
                    *reinterpret_cast<uint4*>(Qs + (size_t)(cc / 8) * rcap * 128 + r * 128 + (((cc % 8) ^ (r & 7)) << 4)) = w;
                }
                // rows that fill up the last 16 weigh 2^(-inf) = 0
                if (et < cols) nlse[et] = et < nr ? -mass_row_lse2(p.lse[mass_query_row(p, m.b, m.g, grp, r0 + et)]) : -INFINITY;
                tc::fence_proxy_async();
                epilogue_barrier();
                if (et == 0) tc::mbar_arrive(&sh->q_full);
                for (int blk = m.blk0; blk < m.blk1; ++blk, ++fill) {
                    if ((fill & 1) != buf || failed) continue;
                    const int j = blk * kKeys + kl;
                    float old = 0.f;
                    if (j < kv && (j < base || r0 > 0)) old = p.mass[krow0 + j];
                    if (!tc::mbar_wait_suspended(&sh->s_full[buf], (uint32_t)(fill >> 1) & 1u, abort_flag)) failed = true;
                    failed = __any_sync(0xffffffffu, failed);
                    if (failed) {
                        if (lane == 0) give_up(sh, p.status, 43);
                        continue;
                    }
                    tc::tc_fence_after_sync();
                    // query l sees rows up to base + l: the first rows of the pass do not count for a new key
                    const int hidden = j <= base ? 0 : (j - base) * grp - r0;
                    float w4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                    for (int c0 = 0; c0 < cols; c0 += 16) {
                        uint32_t v[16];
                        tc::tmem_read16(tmem_s + (uint32_t)c0, v);
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float4 ls = *reinterpret_cast<const float4*>(nlse + c0 + i);
                            const float e0 = mass_exp2(fmaf(__uint_as_float(v[i]), sl2, ls.x)), e1 = mass_exp2(fmaf(__uint_as_float(v[i + 1]), sl2, ls.y));
                            const float e2 = mass_exp2(fmaf(__uint_as_float(v[i + 2]), sl2, ls.z)), e3 = mass_exp2(fmaf(__uint_as_float(v[i + 3]), sl2, ls.w));
                            w4[0] += c0 + i >= hidden ? e0 : 0.f;
                            w4[1] += c0 + i + 1 >= hidden ? e1 : 0.f;
                            w4[2] += c0 + i + 2 >= hidden ? e2 : 0.f;
                            w4[3] += c0 + i + 3 >= hidden ? e3 : 0.f;
                        }
                    }
                    tc::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&sh->s_empty[buf]);
                    mass_put(p, m.b, krow0, j, kv, base, p.decay, old, (w4[0] + w4[1]) + (w4[2] + w4[3]), r0 == 0);
                }
            }
        }
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc(tmem, (uint32_t)(2 * place));
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

template <int D>
int launch_tc(Handle* h, cudaStream_t s, const MassParams& p) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return CTCSD_ERR_CUDA;
    CUtensorMap tmK;
    {   // K [B][Hkv][Lcap][D] seen as [B][Hkv][D/64][Lcap][64]: a box is 128 keys of one head, all 64-column parts
        cuuint64_t dims[5] = {64, (cuuint64_t)p.Lcap, (cuuint64_t)(D / 64), (cuuint64_t)p.Hkv, (cuuint64_t)p.B};
        cuuint64_t str[4] = {(cuuint64_t)D * 2, 128, (cuuint64_t)p.Lcap * D * 2, (cuuint64_t)p.Hkv * p.Lcap * D * 2};
        cuuint32_t box[5] = {64, (cuuint32_t)kKeys, (cuuint32_t)(D / 64), 1, 1};
        cuuint32_t estr[5] = {1, 1, 1, 1, 1};
        if (fn(&tmK, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(p.K), dims, str, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return CTCSD_ERR_CUDA;
    }
    const int rows = (p.T + 1) * (p.Hq / p.Hkv);
    const int rcap = rows < kMaxRows ? (rows + 15) / 16 * 16 : kMaxRows;
    int place = 32;                                              // columns of one S
    while (place < rcap) place *= 2;
    const size_t rest = (size_t)rcap * (D * 2 + 4) + sizeof(MassShared) + sizeof(int) * (size_t)(p.B + 1), tile = (size_t)kKeys * D * 2;
    // two CTAs per SM (228 KB between them, 1 KB each taken by the system) if three K blocks fit beside the rows
    const size_t half = 113 * 1024;
    const bool two = place <= 128 && rest + 3 * tile <= half;
    int stages = (int)(((two ? half : (size_t)kMaxDynamicSmem) - rest) / tile);
    if (stages > kMaxStages) stages = kMaxStages;
    auto kern = attention_mass_tc_kernel<D>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepMassTc, kern));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(h->num_sms * (two ? 2 : 1)), dim3(kThreads), stages * tile + rest, s, 1, tmK, p, rcap, stages, place));
    h->launches++;
    return CTCSD_OK;
}

}  // namespace

int launch_attention_mass_tc(Handle* h, cudaStream_t s, const MassParams& p, int D) {
    return D == 64 ? launch_tc<64>(h, s, p) : launch_tc<128>(h, s, p);
}

}  // namespace ctcsd
