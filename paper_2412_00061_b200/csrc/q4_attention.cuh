// Tree attention over a 4-bit cache: parameters, and the division of its work that the kernels share.
//
// Query rows.  A sequence's live rows of a kv head - its tree nodes times the query heads of the group - are cut into tiles of
// TR rows; a tile holds rows of one sequence only, since nothing is shared between sequences.
// Keys.  A tile's blocks: the cached rows, KB at a time, then the tree's own rows, KB at a time (those in full precision, masked).
// Balance.  The blocks of all (kv head, sequence, tile) form one line, which is cut into equal spans, one per CTA (cut_spans).  A tile inside
// one span is finished there; a tile that crosses a cut leaves (O, reference, sum) of each part in the workspace, and the merge kernel
// joins the parts in span order.  A span has at most two such parts: slot 0 continues a tile, slot 1 begins one.
#pragma once

#include "q4.cuh"

namespace ctcsd {

struct AttnQ4Params {
    const void* Q;                       // [B,max_nodes,Hq,D]
    const uint32_t* Kq; const uint32_t* Ks;    // [B,Hkv,Lcap] rows of D/8 words, D/32 pairs
    const uint32_t* Vq; const uint32_t* Vs;
    const void* Kt; const void* Vt;      // [B,Hkv,max_nodes,D]
    void* O;                             // [B,max_nodes,Hq,D]
    float* lse;                          // [B,max_nodes,Hq] or null
    const int* kv_len; const int* n_nodes;     // [B]
    const unsigned long long* mask;      // [B,max_nodes,ceil(max_nodes/64)]
    int B, Hq, Hkv, D, max_nodes, Lcap, grp;      // grp = Hq / Hkv
    float scale;
    int* status;
    int spans;                           // that the workspace has room for
    int4* cuts;                          // workspace: [span] (written by its CTA, read by the merge): kv head, sequence, tile and last span of the tile
                                         // that the span continues from the one before it, -1 if there is none or a span further back began it
    float2* part_ml;                     // workspace: [span][2][TR] (reference in log2 units, sum)
    float4* part_o;                      // workspace: [span][2][D/4][TR]
};

constexpr int kAq4MaxB = 1024;
constexpr int kAq4SimpleRows = 64, kAq4SimpleKeys = 64, kAq4SimplePerSm = 2;
constexpr int kAq4MmaRows = 16, kAq4MmaKeys = 192;
constexpr int kAq4TcKeys = 128;

// The plan in shared memory.
struct PlanQ4 {
    int* blk_off;                        // [B+1] blocks (of a kv head) before each sequence
    int* kv;                             // [B] cached rows
    int* n;                              // [B] live nodes (0: the sequence takes no part)
    __host__ __device__ static int ints(int B) { return 3 * B + 1; }
    __host__ __device__ void carve(int* at, int B) { blk_off = at; kv = at + B + 1; n = kv + B; }
};

// The line of blocks and its spans (their lengths differ by one at most).
struct SpansQ4 {
    long long each;
    int extra, count, per_head;
    __host__ __device__ long long start(int c) const { return each * c + (c < extra ? c : extra); }
    __host__ __device__ int span_of(long long x) const {
        const long long big = (each + 1) * extra;
        return x < big ? (int)(x / (each + 1)) : extra + (int)((x - big) / each);
    }
};

__host__ __device__ inline SpansQ4 spans_of(int per_head, int Hkv, int count) {
    SpansQ4 m;
    const long long total = (long long)per_head * Hkv;
    m.per_head = per_head;
    m.count = total < count ? (total > 0 ? (int)total : 1) : count;
    m.each = total / m.count;
    m.extra = (int)(total - m.each * m.count);
    return m;
}

// A span's parts, one (kv head, sequence, tile, range of blocks) at a time.
struct WalkQ4 {
    int g, b, t, blk0, blk1, nblk, cached;     // cached: blocks of cached rows among the tile's nblk
    long long rest;
    __host__ __device__ bool init(const PlanQ4& p, const SpansQ4& m, int B, int KB, int span) {
        if (span >= m.count) { rest = 0; return false; }
        const long long x = m.start(span);
        rest = m.start(span + 1) - x;
        if (rest <= 0) return false;
        g = (int)(x / m.per_head);
        const int xh = (int)(x - (long long)g * m.per_head);
        int lo = 0, hi = B - 1;                // smallest b with blk_off[b+1] > xh
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (p.blk_off[mid + 1] > xh) hi = mid; else lo = mid + 1;
        }
        b = lo;
        sizes(p, KB);
        t = (xh - p.blk_off[b]) / nblk;
        blk0 = xh - p.blk_off[b] - t * nblk;
        clip();
        return true;
    }
    __host__ __device__ bool next(const PlanQ4& p, int B, int KB) {
        rest -= blk1 - blk0;
        if (rest <= 0) return false;
        blk0 = 0;
        ++t;
        if (p.blk_off[b] + t * nblk >= p.blk_off[b + 1]) {                   // the sequence's last tile is done
            t = 0;
            do {
                if (++b == B) { b = 0; ++g; }
            } while (p.blk_off[b + 1] == p.blk_off[b]);
            sizes(p, KB);
        }
        clip();
        return true;
    }
    __host__ __device__ void sizes(const PlanQ4& p, int KB) {
        cached = (p.kv[b] + KB - 1) / KB;
        nblk = cached + (p.n[b] + KB - 1) / KB;
    }
    __host__ __device__ void clip() { blk1 = rest < nblk - blk0 ? blk0 + (int)rest : nblk; }
    __host__ __device__ bool whole() const { return blk0 == 0 && blk1 == nblk; }
    __host__ __device__ int slot() const { return blk0 > 0 ? 0 : 1; }
};

// At most this many blocks a kv head has; the plan numbers them in 32 bits.
inline bool plan_q4_fits(int B, int max_nodes, int grp, int TR, int KB, int Lcap) {
    const long long tiles = ((long long)max_nodes * grp + TR - 1) / TR;
    const long long blocks = ((long long)Lcap + KB - 1) / KB + (max_nodes + KB - 1) / KB;
    return B * tiles * blocks < (1ll << 31);
}

#ifdef __CUDACC__

// Fills the plan; executed by the whole block, ends with a barrier.  A sequence whose lengths would read outside its arrays is
// reported (by block 0) and takes no part.
__device__ inline SpansQ4 plan_q4_build(PlanQ4& p, const AttnQ4Params& a, int TR, int KB, int spans) {
    const int lane = threadIdx.x & 31;
    if (threadIdx.x < 32) {
        int before = 0;
#pragma unroll 1
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int b = b0 + lane;
            int n = 0, L = 0;
            if (b < a.B) {
                n = a.n_nodes[b];
                L = a.kv_len[b];
                if (n < 0 || n > a.max_nodes || L < 0 || L > a.Lcap) {
                    if (blockIdx.x == 0) report_error(a.status, CTCSD_ERR_INVALID_ARG, b);
                    n = 0;
                }
                if (n == 0) L = 0;
                p.n[b] = n;
                p.kv[b] = L;
            }
            int v = (n * a.grp + TR - 1) / TR * ((L + KB - 1) / KB + (n + KB - 1) / KB);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            if (b < a.B) p.blk_off[b + 1] = before + v;
            before += __shfl_sync(0xffffffffu, v, 31);
        }
        if (lane == 0) p.blk_off[0] = 0;
    }
    __syncthreads();
    return spans_of(p.blk_off[a.B], a.Hkv, spans);
}

// What the block does besides its span: the rows of unused nodes become 0 and -inf (all heads of a node are neighbours), and the merge
// is told whether the span continues a tile.  `at`: the span's first part.
template <typename T, int D>
__device__ inline void attn_q4_sides(const AttnQ4Params& a, const PlanQ4& p, const SpansQ4& m, const WalkQ4& at, bool more) {
    constexpr int E = 16 / (int)sizeof(T);
    const int words = a.Hq * D / E;
#pragma unroll 1
    for (int i = blockIdx.x; i < a.B * a.max_nodes; i += gridDim.x) {
        const int b = i / a.max_nodes;
        if (i - b * a.max_nodes < p.n[b]) continue;
        uint4* out = reinterpret_cast<uint4*>(static_cast<T*>(a.O) + (size_t)i * a.Hq * D);
#pragma unroll 1
        for (int w = threadIdx.x; w < words; w += blockDim.x)
            if (CTCSD_IN_BOUNDS(a.status, 131, (long long)i * words + w, (long long)a.B * a.max_nodes * words)) out[w] = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse)
#pragma unroll 1
            for (int h = threadIdx.x; h < a.Hq; h += blockDim.x)
                if (CTCSD_IN_BOUNDS(a.status, 135, (long long)i * a.Hq + h, (long long)a.B * a.max_nodes * a.Hq)) a.lse[(size_t)i * a.Hq + h] = -INFINITY;
    }
    if (threadIdx.x == 0) {
        int4 cut = make_int4(-1, 0, 0, 0);
        if (more && at.blk0 > 0) {
            const long long x0 = (long long)at.g * m.per_head + p.blk_off[at.b] + at.t * at.nblk;
            if (m.span_of(x0) == (int)blockIdx.x - 1) cut = make_int4(at.g, at.b, at.t, m.span_of(x0 + at.nblk - 1));
        }
        if (CTCSD_IN_BOUNDS(a.status, 136, blockIdx.x, a.spans)) a.cuts[blockIdx.x] = cut;
    }
}

__device__ __forceinline__ float exp2_q4(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Bits of the 32 tree rows from t0 on that a row with ancestor mask mrow (W words) sees among n live ones.
__device__ __forceinline__ uint32_t tree_bits32(const unsigned long long* mrow, int W, int t0, int n) {
    if (t0 >= n) return 0u;
    uint32_t bits = (uint32_t)(mrow[t0 >> 6] >> (t0 & 63));                 // (t0 is a multiple of 32)
    const int left = n - t0;
    if (left < 32) bits &= (1u << left) - 1u;
    return bits;
}

__device__ __forceinline__ long long out_rows(const AttnQ4Params& a) { return (long long)a.B * a.max_nodes * a.Hq; }

#endif  // __CUDACC__

// bf16, up to 16 query rows of a kv head.
int launch_attention_q4_mma(Handle* h, cudaStream_t s, const AttnQ4Params& p);
// bf16, more: tiles of TR (128 or 256) rows.
int launch_attention_q4_tc(Handle* h, cudaStream_t s, const AttnQ4Params& p, int TR);

}  // namespace ctcsd
