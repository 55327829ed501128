// Shared-prefix tree attention: parameters, and the division of its work that the kernels share.
//
// Query rows.  All live rows of a kv head g - every live tree node of every sequence times the query
// heads of the group - are numbered densely ("packed rows"): sequence b owns rows
// row_off[b] .. row_off[b+1]-1, node by node, head by head.  A tile is TR consecutive packed rows and
// may hold rows of several sequences, so that a batch of single tokens fills a tile as well as trees do.
// Keys.  A tile's keys come in blocks of KB: first the shared prefix (as far as the longest share
// among the tile's sequences), then each of its sequences' own rows (cache, then tree).  A row takes no
// weight from keys that are not its own.
// Balance.  The blocks of all (kv head, tile) pairs form one line, which is cut into equal spans, one
// per CTA.  A tile inside one span is finished there; a tile that crosses a cut leaves (O, reference,
// sum) of each part in the workspace and the merge kernel joins the parts.  A span has at most two such
// parts: slot 0 continues a tile of the previous span, slot 1 begins a tile that the next one continues.
//
// Loops here stay rolled: they run a few times per call, and the kernels' code has to stay small, since the roles of a CTA
// fetch theirs side by side (the bf16 kernel's: 135 KB, 88 KB with these and its own rare loops rolled).
#pragma once

#include "common.cuh"

namespace ctcsd {

struct SharedAttnParams {
    const void* Q;          // [B,max_nodes,Hq,D]
    const void* Kp;         // [Hkv,Pcap,D], null without a prefix
    const void* Vp;
    const void* K;          // [B,Hkv,Lcap,D]
    const void* V;
    void* O;                // [B,max_nodes,Hq,D]
    float* lse;             // [B,max_nodes,Hq] or null
    const int* prefix_len;  // [B] or null
    const int* kv_len;      // [B]
    const int* n_nodes;     // [B]
    const unsigned long long* mask;   // [B,max_nodes,ceil(max_nodes/64)]
    int B, Hq, Hkv, D, max_nodes, Lcap, Pcap, grp;      // grp = Hq / Hkv
    float scale;
    int* status;
    int* plan;              // workspace: header, row_off, tile_cum (written by CTA 0, read by the merge)
    float4* part_o;         // workspace: [span][2][D/4][TR]
    float2* part_ml;        // workspace: [span][2][TR] (reference in log2 units, sum)
    int min_blocks, long_span;   // see span_map
};

constexpr int kSharedMaxB = 1024;              // sequences
constexpr int kSharedMaxRows = 1 << 19;        // packed rows per kv head
constexpr int kSharedSpansPerSm = 2;           // of the kernel without tensor cores
constexpr int kPlanHeader = 8;                 // ints: rows, tiles, blocks per kv head, spans

constexpr int kSimpleRows = 64;                // tile and block of the kernel without tensor cores
constexpr int kSimpleKeys = 64;
constexpr int kTcRows = 256;                   // of the tensor-core kernel (two 128-row halves)
constexpr int kTcKeys = 128;

// The plan's arrays in shared memory (kernels) or in host memory (tests/shared_plan_host.cu).
struct SharedPlan {
    int* row_off;    // [B+1] packed rows before each sequence
    int* own_cum;    // [B+1] blocks of own keys before each sequence
    int* own_len;    // [B] own keys: cached + tree rows (0: the sequence takes no part)
    int* kv;         // [B] cached rows
    int* pre;        // [B] share of the prefix
    int* edge;       // [2] shortest and longest share among the sequences that take part
    int* tile_cum;   // [tiles+1] key blocks before each tile
    int rows, tiles;
};

__host__ __device__ inline int plan_ints(int B, int max_tiles) { return 2 * (B + 1) + 3 * B + 2 + max_tiles + 1; }

__host__ __device__ inline void plan_carve(SharedPlan& p, int* at, int B) {
    p.row_off = at;
    p.own_cum = p.row_off + B + 1;
    p.own_len = p.own_cum + B + 1;
    p.kv = p.own_len + B;
    p.pre = p.kv + B;
    p.edge = p.pre + B;
    p.tile_cum = p.edge + 2;
}

// Sequence that owns packed row r (0 <= r < rows).
__host__ __device__ inline int plan_seq_of_row(const SharedPlan& p, int B, int r) {
    int lo = 0, hi = B - 1;                    // smallest b with row_off[b+1] > r
#pragma unroll 1
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p.row_off[mid + 1] > r) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// Longest share of the prefix among sequences b0..b1.
__host__ __device__ inline int plan_pre_max(const SharedPlan& p, int b0, int b1) {
    if (p.edge[0] == p.edge[1]) return p.edge[1];          // all alike
    int m = 0;
#pragma unroll 1
    for (int b = b0; b <= b1; ++b) m = p.pre[b] > m ? p.pre[b] : m;
    return m;
}

// What a tile looks at.
struct TileInfo {
    int row0, nrows;     // packed rows
    int b0, b1;          // its first and last sequence
    int pmax, pmin;      // longest and shortest share of the prefix among its sequences
};

__host__ __device__ inline TileInfo plan_tile(const SharedPlan& p, int B, int TR, int t) {
    TileInfo ti;
    ti.row0 = t * TR;
    ti.nrows = p.rows - ti.row0 < TR ? p.rows - ti.row0 : TR;
    ti.b0 = plan_seq_of_row(p, B, ti.row0);
    ti.b1 = plan_seq_of_row(p, B, ti.row0 + ti.nrows - 1);
    ti.pmax = ti.pmin = p.edge[1];
    if (p.edge[0] != p.edge[1]) {
        ti.pmax = 0;
#pragma unroll 1
        for (int b = ti.b0; b <= ti.b1; ++b) {
            if (p.own_len[b] == 0) continue;
            ti.pmax = p.pre[b] > ti.pmax ? p.pre[b] : ti.pmax;
            ti.pmin = p.pre[b] < ti.pmin ? p.pre[b] : ti.pmin;
        }
    }
    return ti;
}

__host__ __device__ inline int plan_tile_blocks(const SharedPlan& p, const TileInfo& ti, int KB) {
    return (ti.pmax + KB - 1) / KB + p.own_cum[ti.b1 + 1] - p.own_cum[ti.b0];
}

// At most this many key blocks a kv head's tiles have together: every tile the whole prefix, and a sequence's own blocks once for each
// tile that holds rows of it (tiles + B such pairs, since rows of a sequence are neighbours).
inline long long plan_most_blocks(int B, int max_nodes, int grp, int TR, int KB, int Pcap, int Lcap) {
    const long long tiles = ((long long)B * max_nodes * grp + TR - 1) / TR;
    return tiles * (((long long)Pcap + KB - 1) / KB) + (tiles + B) * (((long long)Lcap + KB - 1) / KB);
}
// The plan numbers a kv head's blocks in 32 bits.  (Capacities decide, since only the device knows the lengths; a million rows of prefix
// and of each cache fit with the most query rows.)
inline bool plan_fits(int B, int max_nodes, int grp, int TR, int KB, int Pcap, int Lcap) {
    return plan_most_blocks(B, max_nodes, grp, TR, KB, Pcap, Lcap) < (1ll << 31);
}

// The line of blocks and its spans (their lengths differ by one at most).
struct SpanMap {
    long long total, each;   // blocks of all kv heads; blocks of a span
    int extra, spans;        // the first `extra` spans hold one more
    int per_head;
    __host__ __device__ long long start(int c) const { return each * c + (c < extra ? c : extra); }
    __host__ __device__ int span_of(long long x) const {
        const long long big = (each + 1) * extra;
        if (total < (1ll << 31))                           // (the short division)
            return x < big ? (int)((unsigned)x / (unsigned)(each + 1)) : extra + (int)((unsigned)(x - big) / (unsigned)each);
        return x < big ? (int)(x / (each + 1)) : extra + (int)((x - big) / each);
    }
};

__host__ __device__ inline SpanMap span_map_n(int per_head, int Hkv, int spans) {
    SpanMap m;
    m.per_head = per_head;
    m.total = (long long)per_head * Hkv;
    m.spans = spans;
    if (m.total < (1ll << 31)) {                           // (the short division)
        m.each = (unsigned)m.total / (unsigned)spans;
        m.extra = (int)((unsigned)m.total - (unsigned)m.each * (unsigned)spans);
    } else {
        m.each = m.total / spans;
        m.extra = (int)(m.total - m.each * spans);
    }
    return m;
}

// How many spans to cut the line into.  A span that crosses from one tile into the next pays for a second set of
// queries and a second output, as much as several blocks.  So with few (kv head, tile) pairs every pair gets the same
// number of spans, none shorter than min_blocks on average, and the cuts fall on the tiles' ends when
// these have equal work; where spans are long (over `long_span` blocks) or the pairs outnumber them, balance counts more
// and all max_spans are used.
// Measured, in us.  min_blocks of bf16 at 1 / 2 / 3 / 4 / 6: 32 heads, one 64-node tree, prefix 200, own 300: 20.4 / 21.5 / 18.9 / 19.0 / 19.0; prefix and own
// 1024: 24.4 / 24.7 / 24.6 / 24.7 / 28.7; 12 heads on 3 of 64, four trees, prefix 3000: 27.4 / 27.6 / 27.5 / 28.6 / 31.3.  Of float32 at 1 / 2 / 3: 4 heads, prefix
// and own 128: 15.5 / 29.0 / 38.1; 32 heads, 512: 58 / 67 / 83.  long_span at 4 / 8 / 16 / 32 / never: four tokens, 32 heads, prefix 4096: 41.5 / 41.0 /
// 38.4 / 38.6 / 38.5; eight trees, 32 heads, prefix 2048: 85.6 / 85.5 / 85.4 / 93.6 / 93.5; eight tokens, prefix 8192: 70.5 / 70.3 / 70.2 / 70.7 / 76.4.
__host__ __device__ inline SpanMap span_map(int per_head, int tiles, int Hkv, int max_spans, int min_blocks, int long_span) {
    const long long total = (long long)per_head * Hkv;
    const int pairs = tiles * Hkv;                         // (below 2^31: 2^13 tiles at most, and Hkv of them fit no GPU's memory beyond)
    if (pairs <= 0) return span_map_n(per_head, Hkv, 1);
    if (pairs >= max_spans || total >= (long long)max_spans * long_span) return span_map_n(per_head, Hkv, max_spans);
    const unsigned room = (unsigned)max_spans / (unsigned)pairs, want = (unsigned)total / (unsigned)(pairs * min_blocks);
    const unsigned each = want < 1u ? 1u : (want < room ? want : room);
    return span_map_n(per_head, Hkv, pairs * (int)each);
}

// Tile that holds block x (0 <= x < tile_cum[tiles]) of a kv head.
__host__ __device__ inline int plan_tile_of_block(const int* tile_cum, int tiles, int x) {
    int lo = 0, hi = tiles - 1;                // smallest t with tile_cum[t+1] > x
#pragma unroll 1
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (tile_cum[mid + 1] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// Walks a span's parts: a (kv head, tile, range of blocks) at a time.
struct SpanWalk {
    int g, t, blk0, blk1, nblk;
    long long rest;      // blocks of the span from this part on
    __host__ __device__ bool init(const SharedPlan& p, const SpanMap& m, int span) {
        const long long x = m.start(span);
        rest = span < m.spans ? m.start(span + 1) - x : 0;
        if (rest <= 0) { rest = 0; return false; }
        g = x < (1ll << 31) ? (int)((unsigned)x / (unsigned)m.per_head) : (int)(x / m.per_head);
        const int xh = (int)(x - (long long)g * m.per_head);
        t = plan_tile_of_block(p.tile_cum, p.tiles, xh);
        blk0 = xh - p.tile_cum[t];
        clip(p);
        return true;
    }
    __host__ __device__ bool next(const SharedPlan& p) {
        rest -= blk1 - blk0;
        if (rest <= 0) return false;
        blk0 = 0;
        if (++t == p.tiles) { t = 0; ++g; }
        clip(p);
        return true;
    }
    __host__ __device__ void clip(const SharedPlan& p) {
        nblk = p.tile_cum[t + 1] - p.tile_cum[t];
        blk1 = rest < nblk - blk0 ? blk0 + (int)rest : nblk;
    }
    __host__ __device__ bool whole() const { return blk0 == 0 && blk1 == nblk; }
    __host__ __device__ int slot() const { return blk0 > 0 ? 0 : 1; }
};

// Walks the key blocks of a tile.
struct BlockIter {
    int seq;             // -1: the shared prefix, else the sequence whose own rows these are
    int key0;            // first key of the block within that source
    int len;             // keys of that source
    __host__ __device__ void init(const SharedPlan& p, const TileInfo& ti, int KB, int blk) {
        const int pb = (ti.pmax + KB - 1) / KB;
        if (blk < pb) { seq = -1; key0 = blk * KB; len = ti.pmax; return; }
        blk += p.own_cum[ti.b0] - pb;
        int lo = ti.b0, hi = ti.b1;            // smallest b with own_cum[b+1] > blk
#pragma unroll 1
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (p.own_cum[mid + 1] > blk) hi = mid; else lo = mid + 1;
        }
        seq = lo; key0 = (blk - p.own_cum[lo]) * KB; len = p.own_len[lo];
    }
    // (only called while another block of the tile follows)
    __host__ __device__ void next(const SharedPlan& p, const TileInfo& ti, int KB) {
        key0 += KB;
        if (key0 < len) return;
        int b = seq < 0 ? ti.b0 : seq + 1;
#pragma unroll 1
        while (b < ti.b1 && p.own_len[b] == 0) ++b;
        seq = b; key0 = 0; len = p.own_len[b];
    }
};

#ifdef __CUDACC__

// Tiles if every node were live: what the plan's arrays have room for.
__device__ __forceinline__ int plan_max_tiles(const SharedAttnParams& a, int TR) { return (a.B * a.max_nodes * a.grp + TR - 1) / TR; }
// Output rows, for the debug build's checks.
__device__ __forceinline__ long long out_rows(const SharedAttnParams& a) { return (long long)a.B * a.max_nodes * a.Hq; }

// Fills the plan's arrays; executed by the whole block, ends with a barrier.  A sequence whose lengths
// would read outside its cache is reported (by the block that publishes) and takes no part.
__device__ inline void plan_build(SharedPlan& p, const SharedAttnParams& a, int TR, int KB, bool publish) {
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31;
    const int grp = a.grp;
    if (tid < 32) {
        int rows = 0, blocks = 0, pmin = 0x7fffffff, pmax = 0;
#pragma unroll 1
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int b = b0 + lane;
            int n = 0, L = 0, P = 0;
            if (b < a.B) {
                n = a.n_nodes[b];
                L = a.kv_len[b];
                P = a.prefix_len ? a.prefix_len[b] : 0;
                if (n < 0 || n > a.max_nodes || L < 0 || L > a.Lcap - n || P < 0 || P > a.Pcap) {
                    if (publish) report_error(a.status, CTCSD_ERR_INVALID_ARG, b);
                    n = 0;
                }
                if (n == 0) { L = 0; P = 0; }
                p.own_len[b] = L + n;
                p.kv[b] = L;
                p.pre[b] = P;
            }
            if (n > 0) { pmin = min(pmin, P); pmax = max(pmax, P); }
            int v = n * grp, w = (L + n + KB - 1) / KB;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v1 = __shfl_up_sync(0xffffffffu, v, o), w1 = __shfl_up_sync(0xffffffffu, w, o);
                if (lane >= o) { v += v1; w += w1; }
            }
            if (b < a.B) { p.row_off[b + 1] = rows + v; p.own_cum[b + 1] = blocks + w; }
            rows += __shfl_sync(0xffffffffu, v, 31);
            blocks += __shfl_sync(0xffffffffu, w, 31);
        }
        pmin = __reduce_min_sync(0xffffffffu, pmin);
        pmax = __reduce_max_sync(0xffffffffu, pmax);
        if (lane == 0) { p.row_off[0] = 0; p.own_cum[0] = 0; p.edge[0] = min(pmin, pmax); p.edge[1] = pmax; }
    }
    __syncthreads();
    p.rows = p.row_off[a.B];
    p.tiles = (p.rows + TR - 1) / TR;
    if (p.tiles <= 32) {                       // (one warp does it all)
        if (tid < 32) {
            int v = lane < p.tiles ? plan_tile_blocks(p, plan_tile(p, a.B, TR, lane), KB) : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            if (lane < p.tiles && CTCSD_IN_BOUNDS(a.status, 81, lane, plan_max_tiles(a, TR))) p.tile_cum[lane + 1] = v;
            if (lane == 0) p.tile_cum[0] = 0;
        }
        __syncthreads();
        return;
    }
#pragma unroll 1
    for (int t = tid; t < p.tiles; t += nt)
        if (CTCSD_IN_BOUNDS(a.status, 81, t, plan_max_tiles(a, TR))) p.tile_cum[t + 1] = plan_tile_blocks(p, plan_tile(p, a.B, TR, t), KB);
    if (tid == 0) p.tile_cum[0] = 0;
    __syncthreads();
    if (tid < 32) {
        int run = 0;
#pragma unroll 1
        for (int t0 = 0; t0 < p.tiles; t0 += 32) {
            int v = t0 + lane < p.tiles ? p.tile_cum[t0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            if (t0 + lane < p.tiles) p.tile_cum[t0 + lane + 1] = run + v;
            run += __shfl_sync(0xffffffffu, v, 31);
        }
    }
    __syncthreads();
}

// CTA 0 leaves what the merge kernel needs.
__device__ inline void plan_publish(const SharedPlan& p, const SharedAttnParams& a, int TR, int spans) {
#pragma unroll 1
    for (int b = threadIdx.x; b <= a.B; b += blockDim.x) a.plan[kPlanHeader + b] = p.row_off[b];
#pragma unroll 1
    for (int t = threadIdx.x; t <= p.tiles; t += blockDim.x)
        if (CTCSD_IN_BOUNDS(a.status, 82, t, plan_max_tiles(a, TR) + 1)) a.plan[kPlanHeader + a.B + 1 + t] = p.tile_cum[t];
    if (threadIdx.x == 0) {
        a.plan[0] = p.rows;
        a.plan[1] = p.tiles;
        a.plan[2] = p.tile_cum[p.tiles];
        a.plan[3] = spans;
    }
}

// Visibility of the 32 keys from `first_key` on (of the shared prefix if seq < 0, else of that sequence's own
// keys) for a row of sequence `row_seq`, as a bit mask.  mrow: the row's ancestor mask (W words).
__device__ __forceinline__ uint32_t visible32_of(int seq, int first_key, int row_seq, int row_pre, int row_kv, int row_n,
                                                 const unsigned long long* mrow, int W) {
    if (seq >= 0 && seq != row_seq) return 0u;
    const int full = (seq < 0 ? row_pre : row_kv) - first_key;     // keys from here on that every row of the sequence sees
    if (full >= 32) return 0xffffffffu;
    uint32_t bits = full > 0 ? (1u << full) - 1u : 0u;
    if (seq >= 0) {
        const int t0 = first_key - row_kv;                         // tree index of the first key (may be negative)
        if (t0 >= row_n || t0 <= -32) return bits;
        unsigned long long w;
        if (t0 < 0) {
            w = mrow[0] << (-t0);
        } else {
            const int k = t0 >> 6, s = t0 & 63;
            w = mrow[k] >> s;                                      // (t0 < row_n <= 64 W)
            if (s > 32 && k + 1 < W) w |= mrow[k + 1] << (64 - s);
        }
        uint32_t tree = (uint32_t)w;
        const int left = row_n - t0;                               // bits of nodes past the tree do not count
        if (left < 32) tree &= (1u << left) - 1u;
        bits |= tree;
    }
    return bits;
}

#endif  // __CUDACC__

// bf16 on tcgen05 / tensor memory.
int launch_shared_attention_tc(Handle* h, cudaStream_t s, const SharedAttnParams& p);
// Joins the parts of tiles that cross a cut, zeroes the rows of unused nodes.
int launch_shared_attention_merge(Handle* h, cudaStream_t s, const SharedAttnParams& p, int TR);

}  // namespace ctcsd
