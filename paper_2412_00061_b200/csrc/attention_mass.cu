// ctcsd_attention_mass: the attention weight that every cached row has gathered.
//   w[b,g,j] = sum_l sum_h exp(scale q[b,node_l,h].k[b,g,j] - lse[b,node_l,h]),   j <= base + l,
// over the accepted path l = 0..acc_len[b] (node_0 the root) and the query heads h of group g, where
// base = kv_len - 1 - acc_len is the cache row of the root;  mass = decay * mass + w  (rows from base
// on are new: mass = w, row_pos = n_evicted + j).
//
// The attention's log-sum-exp makes this one pass over K: no maximum, no sum over keys, and every key's
// weight is formed by one warp in a fixed order (no atomics).  The key blocks of all (sequence, kv head)
// pairs form one line that is cut into equal spans, one per CTA.
#include "attention_mass.cuh"

namespace ctcsd {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ---------------------------------------------------------------------------------------
// bf16, at most 16 query rows (single heads, short paths).  HBM bounds it: 666 MB (two sequences, 40 heads, 32768 rows, nine
// query rows) in 113 us, 5.9 TB/s; 8.8 MB in 5.4 us, most of that the launch.  A warp takes 16 keys as the M
// side of mma.m16n8k16 and the path's rows as the N side.  Keys go from global memory straight into the
// fragments by 128-bit loads - the k index is permuted alike for both operands - and the next block's
// keys are requested before the current block is multiplied; the rows sit in shared memory in fragment
// order.  (An mma.sync takes some 26 cycles of its scheduler here: beyond two row tiles that time passes the
// loads', and the tcgen05 kernel takes over.  Measured with all rows on this kernel: 54 us for the 179 MB of a batch
// of 32 with 7 x 8 rows, 37 us on tcgen05.)
// ---------------------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(kThreads, 2) attention_mass_mma_kernel(MassParams p) {
    constexpr int KB = 128;              // keys per block: 16 per warp
    constexpr int NC = D / 32;           // 16-byte chunks of a key per thread
    constexpr int RC = kMassMmaRows;
    __shared__ uint4 Qf[RC / 8 * NC * 32];                                  // [row tile of 8][NC][32 lanes]
    __shared__ float2 lse2[RC / 2];
    __shared__ int2 lim[RC / 2];         // last cache row a query sees, relative to base
    extern __shared__ int cum[];         // [B+1]
    const int grp = p.Hq / p.Hkv;
    pdl_wait();
    pdl_trigger();
    mass_plan(p, KB, cum);
    const long long total = (long long)cum[p.B] * p.Hkv;
    const long long x1 = total * (blockIdx.x + 1) / gridDim.x;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
    const float sl2 = p.scale * kMassLog2e;
    for (long long x = total * blockIdx.x / gridDim.x; x < x1;) {
        const MassPiece m = mass_piece(p, cum, x, x1);
        x += m.blk1 - m.blk0;
        const int kv = p.kv_len[m.b], acc = p.acc_len[m.b], base = kv - 1 - acc;
        const int R = (acc + 1) * grp, tiles = (R + 7) / 8;
        const size_t krow0 = ((size_t)m.b * p.Hkv + m.g) * (size_t)p.Lcap;
        const __nv_bfloat16* Kb = static_cast<const __nv_bfloat16*>(p.K) + krow0 * D;
        auto load_keys = [&](uint4 (&a)[2][NC], int blk) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const int j = blk * KB + warp * 16 + hf * 8 + gid;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    a[hf][c] = make_uint4(0u, 0u, 0u, 0u);
                    if (j < kv) a[hf][c] = __ldg(reinterpret_cast<const uint4*>(Kb + (size_t)j * D) + c * 4 + tig);
                }
            }
        };
        uint4 cur[2][NC];
        load_keys(cur, m.blk0);
        __syncthreads();                 // the previous piece's rows have been read
        for (int i = tid; i < tiles * NC * 32; i += kThreads) {
            const int ln = i & 31, c = (i >> 5) % NC, r = (i >> 5) / NC * 8 + (ln >> 2);
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (r < R) {
                const size_t qr = mass_query_row(p, m.b, m.g, grp, r);
                const uint4 q = *(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.Q) + qr * D) + c * 4 + (ln & 3));
                if (mass_row_counts(p.lse[qr])) v = q;
            }
            Qf[i] = v;
        }
        if (tid < RC) {
            reinterpret_cast<float*>(lse2)[tid] = tid < R ? mass_row_lse2(p.lse[mass_query_row(p, m.b, m.g, grp, tid)]) : INFINITY;
            reinterpret_cast<int*>(lim)[tid] = tid < R ? tid / grp : -1;
        }
        __syncthreads();
        for (int blk = m.blk0; blk < m.blk1; ++blk) {
            uint4 nxt[2][NC];
            if (blk + 1 < m.blk1) load_keys(nxt, blk + 1);
            const int j0 = blk * KB + warp * 16 + gid, j1 = j0 + 8;
            const bool writes = tig == 0;
            float old0 = 0.f, old1 = 0.f;
            if (writes && j0 < base) old0 = p.mass[krow0 + j0];
            if (writes && j1 < base) old1 = p.mass[krow0 + j1];
            const bool tail = blk * KB + KB > base;                         // some key is not seen by every query
            float w0 = 0.f, w1 = 0.f;
#pragma unroll
            for (int rt = 0; rt < RC / 8; ++rt) {
                if (rt >= tiles) break;
                float ca[4] = {0.f, 0.f, 0.f, 0.f}, cb[4] = {0.f, 0.f, 0.f, 0.f};      // two chains of products
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const uint4 q = Qf[(rt * NC + c) * 32 + lane];
                    mma_bf16(ca, cur[0][c].x, cur[1][c].x, cur[0][c].y, cur[1][c].y, q.x, q.y);
                    mma_bf16(cb, cur[0][c].z, cur[1][c].z, cur[0][c].w, cur[1][c].w, q.z, q.w);
                }
                const float2 ls = lse2[rt * 4 + tig];
                float e0 = mass_exp2(fmaf(ca[0] + cb[0], sl2, -ls.x)), e1 = mass_exp2(fmaf(ca[1] + cb[1], sl2, -ls.y));
                float e2 = mass_exp2(fmaf(ca[2] + cb[2], sl2, -ls.x)), e3 = mass_exp2(fmaf(ca[3] + cb[3], sl2, -ls.y));
                if (tail) {
                    const int2 lm = lim[rt * 4 + tig];
                    e0 = lm.x >= 0 && j0 - base <= lm.x ? e0 : 0.f;
                    e1 = lm.y >= 0 && j0 - base <= lm.y ? e1 : 0.f;
                    e2 = lm.x >= 0 && j1 - base <= lm.x ? e2 : 0.f;
                    e3 = lm.y >= 0 && j1 - base <= lm.y ? e3 : 0.f;
                }
                w0 += e0 + e1;
                w1 += e2 + e3;
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                w0 += __shfl_xor_sync(0xffffffffu, w0, o);
                w1 += __shfl_xor_sync(0xffffffffu, w1, o);
            }
            if (writes) {
                mass_put(p, m.b, krow0, j0, kv, base, p.decay, old0, w0, true);
                mass_put(p, m.b, krow0, j1, kv, base, p.decay, old1, w1, true);
            }
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int c = 0; c < NC; ++c) cur[hf][c] = nxt[hf][c];
        }
    }
}

// ---------------------------------------------------------------------------------------
// float32.  64 keys per block in shared memory (row stride D + 4: 128-bit loads without bank conflicts); a thread owns one key and four rows
// at a time, the four threads of a key add up their rows.  Bound by shared-memory reads and by turns: loads and products do not
// overlap within a CTA, a key's 16 bytes serve four rows only, and up to 16 query rows cost what 16 do.  (546 MB, 8 sequences, 32 heads, 4096
// rows, up to six query rows: 444 us, 1.2 TB/s - shared-memory pipe 56 % busy, FMA 19 %, the longest stalls those on loads from memory; 95 MB,
// 8 kv heads, up to 56 query rows: 199 us.)
// ---------------------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(kThreads) attention_mass_f32_kernel(MassParams p) {
    constexpr int KB = 64, ST = D + 4, RC = 64;                             // RC rows at a time
    extern __shared__ __align__(16) unsigned char dyn[];
    float* Ks = reinterpret_cast<float*>(dyn);                              // [KB][ST]
    float* Qs = Ks + KB * ST;                                               // [RC][D]
    float* lse2 = Qs + RC * D;                                              // [RC]
    float* part = lse2 + RC;                                                // [4][KB]
    int* lim = reinterpret_cast<int*>(part + 4 * KB);                       // [RC]
    int* cum = lim + RC;                                                    // [B+1]
    pdl_wait();
    pdl_trigger();
    mass_plan(p, KB, cum);
    const int grp = p.Hq / p.Hkv;
    const long long total = (long long)cum[p.B] * p.Hkv;
    const long long x1 = total * (blockIdx.x + 1) / gridDim.x;
    const int tid = threadIdx.x, key = tid & 63, rg = tid >> 6;
    const float sl2 = p.scale * kMassLog2e;
    for (long long x = total * blockIdx.x / gridDim.x; x < x1;) {
        const MassPiece m = mass_piece(p, cum, x, x1);
        x += m.blk1 - m.blk0;
        const int kv = p.kv_len[m.b], acc = p.acc_len[m.b], base = kv - 1 - acc;
        const int R = (acc + 1) * grp;
        const size_t krow0 = ((size_t)m.b * p.Hkv + m.g) * (size_t)p.Lcap;
        const float* Kb = static_cast<const float*>(p.K) + krow0 * D;
        for (int blk = m.blk0; blk < m.blk1; ++blk) {
            const int j = blk * KB + key;
            __syncthreads();             // the previous block's keys and partial sums have been read
            for (int i = tid; i < KB * (D / 4); i += kThreads) {
                const int k = i / (D / 4), c = i - k * (D / 4);
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (blk * KB + k < kv) v = __ldg(reinterpret_cast<const float4*>(Kb + (size_t)(blk * KB + k) * D) + c);
                *reinterpret_cast<float4*>(Ks + k * ST + 4 * c) = v;
            }
            float w = 0.f;
            for (int r0 = 0; r0 < R; r0 += RC) {
                const int nr = min(R - r0, RC), nr4 = (nr + 15) / 16 * 16;
                // (one chunk of rows serves a whole piece)
                if (r0 > 0 || R > RC || blk == m.blk0) {
                    if (r0 > 0) __syncthreads();
                    for (int i = tid; i < nr4 * (D / 4); i += kThreads) {
                        const int r = i / (D / 4), c = i - r * (D / 4);
                        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (r < nr) {
                            const size_t qr = mass_query_row(p, m.b, m.g, grp, r0 + r);
                            const float4 q = reinterpret_cast<const float4*>(static_cast<const float*>(p.Q) + qr * D)[c];
                            if (mass_row_counts(p.lse[qr])) v = q;
                        }
                        *reinterpret_cast<float4*>(Qs + r * D + 4 * c) = v;
                    }
                    for (int r = tid; r < nr4; r += kThreads) {
                        lse2[r] = r < nr ? mass_row_lse2(p.lse[mass_query_row(p, m.b, m.g, grp, r0 + r)]) : INFINITY;
                        lim[r] = r < nr ? (r0 + r) / grp : -1;
                    }
                }
                __syncthreads();
                for (int r = rg * 4; r < nr4; r += 16) {
                    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
                    for (int d = 0; d < D; d += 4) {
                        const float4 k4 = *reinterpret_cast<const float4*>(Ks + key * ST + d);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 q4 = *reinterpret_cast<const float4*>(Qs + (r + i) * D + d);
                            s[i] = fmaf(q4.x, k4.x, s[i]);
                            s[i] = fmaf(q4.y, k4.y, s[i]);
                            s[i] = fmaf(q4.z, k4.z, s[i]);
                            s[i] = fmaf(q4.w, k4.w, s[i]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e = mass_exp2(fmaf(s[i], sl2, -lse2[r + i]));
                        w += lim[r + i] >= 0 && j - base <= lim[r + i] ? e : 0.f;
                    }
                }
            }
            part[rg * KB + key] = w;
            __syncthreads();
            if (rg == 0 && j < kv && CTCSD_IN_BOUNDS(p.status, 72, j, p.Lcap)) {
                const float ws = (part[key] + part[KB + key]) + (part[2 * KB + key] + part[3 * KB + key]);
                if (j >= base) {
                    p.mass[krow0 + j] = ws;
                    p.row_pos[krow0 + j] = (p.n_evicted ? p.n_evicted[m.b] : 0) + j;
                } else {
                    p.mass[krow0 + j] = fmaf(p.decay, p.mass[krow0 + j], ws);
                }
            }
        }
    }
}

template <int D>
int launch_mass(Handle* h, cudaStream_t s, const MassParams& p, bool bf16) {
    if (bf16) {
        if ((p.T + 1) * (p.Hq / p.Hkv) > kMassMmaRows) return launch_attention_mass_tc(h, s, p, D);
        CTCSD_CUDA_CHECK(h, launch_pdl(attention_mass_mma_kernel<D>, dim3(h->num_sms * 2), dim3(kThreads), sizeof(int) * (size_t)(p.B + 1), s, 1, p));
    } else {
        const size_t smem = sizeof(float) * (64 * (D + 4) + 64 * D + 64 + 4 * 64 + 64) + sizeof(int) * (size_t)(p.B + 1);
        CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepMassF32, attention_mass_f32_kernel<D>));
        CTCSD_CUDA_CHECK(h, launch_pdl(attention_mass_f32_kernel<D>, dim3(h->num_sms * 2), dim3(kThreads), smem, s, 1, p));
    }
    h->launches++;
    return CTCSD_OK;
}

}  // namespace
}  // namespace ctcsd

using namespace ctcsd;

extern "C" int ctcsd_attention_mass(ctcsd_handle* hh, void* stream, const void* Q, const void* K, int Lcap,
                                    const int* kv_len, const int* acc_len, const int* acc_nodes, const float* lse,
                                    float scale, float decay, const int* n_evicted, float* mass, int* row_pos) {
    if (!hh || !Q || !K || !kv_len || !acc_len || !acc_nodes || !lse || !mass || !row_pos) return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    if (Lcap < 1 || !(decay >= 0.f && decay <= 1.f) || !(scale > 0.f) || isinf(scale)) return CTCSD_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(K)) & 15) return CTCSD_ERR_INVALID_ARG;
    if (c.B > kMassMaxB) return CTCSD_ERR_UNSUPPORTED;
    MassParams p;
    p.Q = Q; p.K = K; p.kv_len = kv_len; p.acc_len = acc_len; p.acc_nodes = acc_nodes; p.lse = lse; p.n_evicted = n_evicted;
    p.mass = mass; p.row_pos = row_pos;
    p.B = c.B; p.Hq = c.Hq; p.Hkv = c.Hkv; p.Lcap = Lcap; p.T = c.T; p.max_nodes = c.max_nodes;
    p.scale = scale; p.decay = decay;
    p.status = status_ptr(h);
    const bool bf16 = c.dtype == CTCSD_DTYPE_BF16;
    const DeviceGuard on(h->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return c.D == 64 ? launch_mass<64>(h, s, p, bf16) : launch_mass<128>(h, s, p, bf16);
}
