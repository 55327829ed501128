// Attention mass: parameters, and the division of its work that the kernels share (see attention_mass.cu).
#pragma once

#include "common.cuh"

#include <math.h>

namespace ctcsd {

constexpr float kMassLog2e = 1.4426950408889634f;
constexpr int kMassMmaRows = 16;       // query rows up to which the kernel on mma.sync serves
constexpr int kMassMaxB = 1024;

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

#ifdef __CUDACC__

__device__ __forceinline__ float mass_exp2(float x) {
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
        for (int l = 0; l < p.T; ++l) {                                    // (all T entries: loads that do not wait for one another)
            const int node = p.acc_nodes[b * p.T + l];
            bad = bad || (l < n && (node < 0 || node >= p.max_nodes));
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
// a tile: an infinite value makes every weight 2^(-inf) = 0.  Their scores must be finite for that: both are zero rows to
// the products, since the attention looked at no query that saw nothing, and such a row of Q may hold anything.
__device__ __forceinline__ float mass_row_lse2(float lse) { return lse == -INFINITY ? INFINITY : lse * kMassLog2e; }

__device__ __forceinline__ bool mass_row_counts(float lse) { return lse != -INFINITY; }

// Row j's weight of one pass: `first` pass applies the decay to the old mass and gives new rows (j >= base) their
// position; a later pass (more query rows than fit) adds.
__device__ __forceinline__ void mass_put(const MassParams& p, int b, size_t krow0, int j, int kv, int base, float decay, float old, float w, bool first) {
    if (j >= kv || !CTCSD_IN_BOUNDS(p.status, 71, j, p.Lcap)) return;
    const bool fresh = first && j >= base;
    p.mass[krow0 + j] = fresh ? w : (first ? fmaf(decay, old, w) : old + w);
    if (fresh) p.row_pos[krow0 + j] = (p.n_evicted ? p.n_evicted[b] : 0) + j;
}

#endif  // __CUDACC__

// bf16 on tcgen05, for many query rows.
int launch_attention_mass_tc(Handle* h, cudaStream_t s, const MassParams& p, int D);

}  // namespace ctcsd
