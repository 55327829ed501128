// ctcsd_attention_mass: the attention weight that every cached row has gathered.
//   w[b,g,j] = sum_l sum_h exp(scale q[b,node_l,h].k[b,g,j] - lse[b,node_l,h]),   j <= base + l,
// over the accepted path l = 0..acc_len[b] (node_0 the root) and the query heads h of group g, where
// base = kv_len - 1 - acc_len is the cache row of the root;  mass = decay * mass + w  (rows from base
// on are new: mass = w, row_pos = n_evicted + j).
//
// The attention's log-sum-exp makes this one pass over K: no maximum, no sum over keys, and every key's
// weight is formed by one warp in a fixed order (no atomics).  The key blocks of all (sequence, kv head)
// pairs form one line that is cut into equal spans, one per CTA.
#include "common.cuh"

#include <math.h>

namespace ctcsd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;
constexpr int kMaxRows = 256;          // query rows held in shared memory at a time; more rows take another pass over K
constexpr int kMassMaxB = 1024;

template <int N> struct Count { static constexpr int value = N; };

struct MassParams {
    const void* Q; const void* K;      // [B,max_nodes,Hq,D], [B,Hkv,Lcap,D]
    const int* kv_len; const int* acc_len; const int* acc_nodes;
    const float* lse;                  // [B,max_nodes,Hq]
    const int* n_evicted;              // [B] or null
    float* mass; int* row_pos;         // [B,Hkv,Lcap]
    int B, Hq, Hkv, Lcap, T, max_nodes;
    float scale, decay;
    int* status;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Blocks of KB keys before each sequence (times Hkv: their place on the line); a sequence whose lengths
// would read outside its arrays has none.  Executed by the whole block, ends with a barrier.
__device__ inline void mass_plan(const MassParams& p, int KB, int* cum) {
    const int tid = threadIdx.x, lane = tid & 31;
    for (int b = tid; b < p.B; b += blockDim.x) {
        const int kv = p.kv_len[b], n = p.acc_len[b];
        bool bad = n < 0 || n > p.T || kv < n + 1 || kv > p.Lcap;
        for (int l = 0; l < n && !bad; ++l) {
            const int node = p.acc_nodes[b * p.T + l];
            bad = node < 0 || node >= p.max_nodes;
        }
        if (bad && blockIdx.x == 0) report_error(p.status, CTCSD_ERR_INVALID_ARG, b);
        cum[b + 1] = bad ? 0 : (kv + KB - 1) / KB;
    }
    if (tid == 0) cum[0] = 0;
    __syncthreads();
    if (tid < 32) {
        int run = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            int v = b0 + lane < p.B ? cum[b0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            if (b0 + lane < p.B) cum[b0 + lane + 1] = run + v;
            run += __shfl_sync(0xffffffffu, v, 31);
        }
    }
    __syncthreads();
}

// One run of blocks of one (sequence, kv head).
struct MassPiece { int b, g, blk0, blk1; };

__device__ __forceinline__ MassPiece mass_piece(const MassParams& p, const int* cum, long long x, long long x1) {
    int lo = 0, hi = p.B - 1;                              // sequence: smallest b with cum[b+1] * Hkv > x
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((long long)cum[mid + 1] * p.Hkv > x) hi = mid; else lo = mid + 1;
    }
    MassPiece m;
    m.b = lo;
    const int nb = cum[lo + 1] - cum[lo];
    const long long o = x - (long long)cum[lo] * p.Hkv;
    m.g = (int)(o / nb);
    m.blk0 = (int)(o - (long long)m.g * nb);
    m.blk1 = (int)(x1 - x < nb - m.blk0 ? m.blk0 + (x1 - x) : nb);
    return m;
}

// Row r of the accepted path's rows of a kv head: query l = r / grp, head g*grp + r % grp.
__device__ __forceinline__ size_t mass_query_row(const MassParams& p, int b, int g, int grp, int r) {
    const int l = r / grp, hh = r - l * grp;
    const int node = l == 0 ? 0 : p.acc_nodes[b * p.T + l - 1];
    return ((size_t)b * p.max_nodes + node) * p.Hq + g * grp + hh;
}

// Log-sum-exp in log2 units.  A query that saw nothing (-inf) adds nothing, and so do the rows that fill up
// a tile: an infinite value makes every weight 2^(-inf) = 0.
__device__ __forceinline__ float row_lse2(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ---------------------------------------------------------------------------------------
// bf16.  HBM bounds it (2 R flops per byte of K, R the path's rows).  A warp takes 16 keys as the M side
// of mma.m16n8k16 and the path's rows as the N side.  Keys go from global memory straight into the
// fragments by 128-bit loads - the k index is permuted alike for both operands - and the next block's
// keys are requested before the current block is multiplied; the rows sit in shared memory in fragment
// order.  Few rows against many keys is not tcgen05's shape (its M side would be 128 of them).
// ---------------------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(kThreads, 2) attention_mass_mma_kernel(MassParams p) {
    constexpr int KB = 128;              // keys per block: 16 per warp
    constexpr int NC = D / 32;           // 16-byte chunks of a key per thread
    extern __shared__ __align__(16) unsigned char dyn[];
    uint4* Qf = reinterpret_cast<uint4*>(dyn);                              // [row tile of 8][NC][32 lanes]
    const int grp = p.Hq / p.Hkv;
    const int rcap = min(kMaxRows, ((p.T + 1) * grp + 7) / 8 * 8);
    float* lse2 = reinterpret_cast<float*>(Qf + rcap / 8 * NC * 32);        // [rcap]
    int* lim = reinterpret_cast<int*>(lse2 + rcap);                         // [rcap] last cache row the query sees, relative to base
    int* cum = lim + rcap;                                                  // [B+1]
    pdl_wait();
    pdl_trigger();
    mass_plan(p, KB, cum);
    const long long total = (long long)cum[p.B] * p.Hkv;
    const long long x1 = total * (blockIdx.x + 1) / gridDim.x;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
    const float sl2 = p.scale * kLog2e;
    for (long long x = total * blockIdx.x / gridDim.x; x < x1;) {
        const MassPiece m = mass_piece(p, cum, x, x1);
        x += m.blk1 - m.blk0;
        const int kv = p.kv_len[m.b], acc = p.acc_len[m.b], base = kv - 1 - acc;
        const int R = (acc + 1) * grp;
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
        for (int r0 = 0; r0 < R; r0 += kMaxRows) {
            const int nr = min(R - r0, kMaxRows), tiles = (nr + 7) / 8;
            uint4 cur[2][NC];
            load_keys(cur, m.blk0);
            __syncthreads();             // the previous piece's rows have been read
            for (int i = tid; i < tiles * NC * 32; i += kThreads) {
                const int ln = i & 31, c = (i >> 5) % NC, rt = (i >> 5) / NC;
                const int r = rt * 8 + (ln >> 2);
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (r < nr)
                    v = *(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.Q) + mass_query_row(p, m.b, m.g, grp, r0 + r) * D) +
                          c * 4 + (ln & 3));
                Qf[i] = v;
            }
            for (int r = tid; r < tiles * 8; r += kThreads) {
                lse2[r] = r < nr ? row_lse2(p.lse[mass_query_row(p, m.b, m.g, grp, r0 + r)]) : INFINITY;
                lim[r] = r < nr ? (r0 + r) / grp : -1;
            }
            __syncthreads();
            for (int blk = m.blk0; blk < m.blk1; ++blk) {
                uint4 nxt[2][NC];
                if (blk + 1 < m.blk1) load_keys(nxt, blk + 1);
                const int j0 = blk * KB + warp * 16 + gid, j1 = j0 + 8;
                const bool writes = tig == 0;
                float old0 = 0.f, old1 = 0.f;
                if (writes && j0 < kv && (j0 < base || r0 > 0)) old0 = p.mass[krow0 + j0];
                if (writes && j1 < kv && (j1 < base || r0 > 0)) old1 = p.mass[krow0 + j1];
                const bool tail = blk * KB + KB > base;                     // some key is not seen by every query
                float w0 = 0.f, w1 = 0.f;
                // N row tiles at a time: an mma.sync that waits for the one before takes some 200 cycles here, so
                // several chains run side by side (a lone tile is cut into two chains)
                auto weigh = [&](auto count, int rt) {
                    constexpr int N = decltype(count)::value, CH = N >= 4 ? 1 : 2;
                    float c4[N][CH][4];
#pragma unroll
                    for (int i = 0; i < N * CH * 4; ++i) c4[i / (CH * 4)][(i / 4) % CH][i % 4] = 0.f;
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const uint4 q = Qf[((rt + i) * NC + c) * 32 + lane];
                            mma_bf16(c4[i][0], cur[0][c].x, cur[1][c].x, cur[0][c].y, cur[1][c].y, q.x, q.y);
                            mma_bf16(c4[i][CH - 1], cur[0][c].z, cur[1][c].z, cur[0][c].w, cur[1][c].w, q.z, q.w);
                        }
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        float s[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) s[x] = CH == 2 ? c4[i][0][x] + c4[i][CH - 1][x] : c4[i][0][x];
                        const float2 ls = *reinterpret_cast<const float2*>(lse2 + (rt + i) * 8 + tig * 2);
                        float e0 = exp2_fast(fmaf(s[0], sl2, -ls.x)), e1 = exp2_fast(fmaf(s[1], sl2, -ls.y));
                        float e2 = exp2_fast(fmaf(s[2], sl2, -ls.x)), e3 = exp2_fast(fmaf(s[3], sl2, -ls.y));
                        if (tail) {
                            const int2 lm = *reinterpret_cast<const int2*>(lim + (rt + i) * 8 + tig * 2);
                            e0 = lm.x >= 0 && j0 - base <= lm.x ? e0 : 0.f;
                            e1 = lm.y >= 0 && j0 - base <= lm.y ? e1 : 0.f;
                            e2 = lm.x >= 0 && j1 - base <= lm.x ? e2 : 0.f;
                            e3 = lm.y >= 0 && j1 - base <= lm.y ? e3 : 0.f;
                        }
                        w0 += e0 + e1;
                        w1 += e2 + e3;
                    }
                };
                int rt = 0;
                for (; rt + 4 <= tiles; rt += 4) weigh(Count<4>(), rt);
                if (rt + 2 <= tiles) { weigh(Count<2>(), rt); rt += 2; }
                if (rt < tiles) weigh(Count<1>(), rt);
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    w0 += __shfl_xor_sync(0xffffffffu, w0, o);
                    w1 += __shfl_xor_sync(0xffffffffu, w1, o);
                }
                if (writes) {
                    const float dk = r0 > 0 ? 1.f : p.decay;
                    auto put = [&](int j, float old, float w) {
                        if (j >= kv) return;
                        const bool fresh = j >= base && r0 == 0;
                        p.mass[krow0 + j] = fresh ? w : fmaf(dk, old, w);
                        if (fresh) p.row_pos[krow0 + j] = (p.n_evicted ? p.n_evicted[m.b] : 0) + j;
                    };
                    put(j0, old0, w0);
                    put(j1, old1, w1);
                }
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                    for (int c = 0; c < NC; ++c) cur[hf][c] = nxt[hf][c];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------
// float32.  64 keys per block in shared memory (row stride D + 4: 128-bit loads without bank
// conflicts); a thread owns one key and four rows at a time, the four threads of a key add up their rows.
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
    const float sl2 = p.scale * kLog2e;
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
                        if (r < nr)
                            v = reinterpret_cast<const float4*>(static_cast<const float*>(p.Q) + mass_query_row(p, m.b, m.g, grp, r0 + r) * D)[c];
                        *reinterpret_cast<float4*>(Qs + r * D + 4 * c) = v;
                    }
                    for (int r = tid; r < nr4; r += kThreads) {
                        lse2[r] = r < nr ? row_lse2(p.lse[mass_query_row(p, m.b, m.g, grp, r0 + r)]) : INFINITY;
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
                        const float e = exp2_fast(fmaf(s[i], sl2, -lse2[r + i]));
                        w += lim[r + i] >= 0 && j - base <= lim[r + i] ? e : 0.f;
                    }
                }
            }
            part[rg * KB + key] = w;
            __syncthreads();
            if (rg == 0 && j < kv) {
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
    const int grp = p.Hq / p.Hkv;
    const int rows = (p.T + 1) * grp;
    size_t smem;
    if (bf16) {
        const int rcap = rows < kMaxRows ? (rows + 7) / 8 * 8 : kMaxRows;
        smem = (size_t)rcap * D * 2 + (size_t)rcap * 8 + sizeof(int) * (p.B + 1);
    } else {
        smem = sizeof(float) * (64 * (D + 4) + 64 * D + 64 + 4 * 64 + 64) + sizeof(int) * (p.B + 1);
    }
    auto kern = bf16 ? attention_mass_mma_kernel<D> : attention_mass_f32_kernel<D>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, bf16 ? kPrepMassMma : kPrepMassF32, kern));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(h->num_sms * 2), dim3(kThreads), smem, s, 1, p));
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
