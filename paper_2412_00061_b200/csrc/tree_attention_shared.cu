// ctcsd_tree_attention_shared: tree attention for a batch whose sequences share a prefix, which is
// read once for all of them.
//   O[b,i,h] = sum_j p_j v_j,  p = softmax_j(scale q.k_j),  j over the first prefix_len[b] rows of the
//   shared cache, the kv_len[b] rows of the sequence's own cache and the tree rows of node i's mask;
//   lse[b,i,h] = log sum_j exp(scale q.k_j).
// The work is divided as shared_attention.cuh describes.  This file holds the entry points, the kernel
// without tensor cores (float32) and the merge of tiles that were cut.
#include "shared_attention.cuh"

#include <math.h>

namespace ctcsd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---------------------------------------------------------------------------------------
// float32: 64 packed rows x 64 keys per step, 256 threads.  A thread computes 4 x 4 scores and 4 x D/16 outputs from
// 128-bit shared loads; rows and keys are dealt 16 apart, which keeps the loads free of bank conflicts (row stride D + 4).
// K and V take turns in one buffer so that two CTAs fit on an SM and hide each other's loads.  Shared-memory reads bound it: eight
// 128-bit loads feed 64 multiply-adds, their pipe is 72 % busy, the FMA pipe 49 %.  (Measured: eight trees of 64
// nodes, 32 heads of 128, prefix 2048: 552 us, 31 TFLOP/s of the FP32 pipe's 74.)
// ---------------------------------------------------------------------------------------
constexpr int kSimpleThreads = 256;

template <bool B> struct Flag { static constexpr bool value = B; };

template <int D>
__global__ void __launch_bounds__(kSimpleThreads, 2) shared_attention_simple_kernel(SharedAttnParams p) {
    constexpr int TR = kSimpleRows, KB = kSimpleKeys, ST = D + 4, PS = KB + 4, DC = D / 64;
    extern __shared__ __align__(16) float sm[];
    float* Qs = sm;                      // [TR][ST]
    float* Ts = Qs + TR * ST;            // [KB][ST]: a K block, then its V block
    float* Ps = Ts + KB * ST;            // [TR][PS]
    SharedPlan pl;
    plan_carve(pl, reinterpret_cast<int*>(Ps + TR * PS), p.B);

    pdl_wait();
    pdl_trigger();
    plan_build(pl, p, TR, KB, blockIdx.x == 0);
    const SpanMap sp = span_map(pl.tile_cum[pl.tiles], pl.tiles, p.Hkv, (int)gridDim.x, p.min_blocks, p.long_span);
    if (blockIdx.x == 0) plan_publish(pl, p, TR, sp.spans);
    SpanWalk at;

    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int grp = p.grp;
    const int W = (p.max_nodes + 63) / 64;
    const float sl2 = p.scale * kLog2e;
    const float* Q = static_cast<const float*>(p.Q);
    for (bool more = at.init(pl, sp, blockIdx.x); more; more = at.next(pl)) {
        const int g = at.g, blk0 = at.blk0, blk1 = at.blk1, slot = at.slot();
        const bool whole = at.whole();
        const TileInfo ti = plan_tile(pl, p.B, TR, at.t);

        __syncthreads();                 // the previous tile's shared memory is free
        for (int i = tid; i < TR * (D / 4); i += kSimpleThreads) {
            const int r = i / (D / 4), c = i - r * (D / 4);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < ti.nrows) {
                const int pr = ti.row0 + r, b = plan_seq_of_row(pl, p.B, pr), o = pr - pl.row_off[b];
                const int node = o / grp, hh = o - node * grp;
                v = reinterpret_cast<const float4*>(Q + (((size_t)b * p.max_nodes + node) * p.Hq + g * grp + hh) * D)[c];
            }
            *reinterpret_cast<float4*>(Qs + r * ST + 4 * c) = v;
        }
        // what this thread's four rows are
        int rseq[4], rnode[4];
        size_t orow[4];                  // output row: ((b * max_nodes + node) * Hq + head)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = ty + 16 * i;
            rseq[i] = -2; rnode[i] = 0; orow[i] = 0;
            if (r < ti.nrows) {
                const int pr = ti.row0 + r, b = plan_seq_of_row(pl, p.B, pr), o = pr - pl.row_off[b];
                rseq[i] = b;
                rnode[i] = o / grp;
                orow[i] = ((size_t)b * p.max_nodes + rnode[i]) * p.Hq + g * grp + (o - rnode[i] * grp);
            }
        }
        float acc[4][4 * DC], ref[4], sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ref[i] = -INFINITY; sum[i] = 0.f;
#pragma unroll
            for (int d = 0; d < 4 * DC; ++d) acc[i][d] = 0.f;
        }
        BlockIter it;
        it.init(pl, ti, KB, blk0);
        for (int blk = blk0; blk < blk1; ++blk) {
            const float *Kb, *Vb;
            if (it.seq < 0) {
                Kb = static_cast<const float*>(p.Kp) + (size_t)g * p.Pcap * D;
                Vb = static_cast<const float*>(p.Vp) + (size_t)g * p.Pcap * D;
            } else {
                const size_t off = ((size_t)it.seq * p.Hkv + g) * (size_t)p.Lcap * D;
                Kb = static_cast<const float*>(p.K) + off;
                Vb = static_cast<const float*>(p.V) + off;
            }
            const int nkey = it.len - it.key0 < KB ? it.len - it.key0 : KB;
            __syncthreads();             // V of the previous block has been read
            for (int i = tid; i < KB * (D / 4); i += kSimpleThreads) {
                const int k = i / (D / 4), c = i - k * (D / 4);
                *reinterpret_cast<float4*>(Ts + k * ST + 4 * c) =
                    k < nkey ? reinterpret_cast<const float4*>(Kb + (size_t)(it.key0 + k) * D)[c] : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            __syncthreads();
            float s[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                float4 q4[4], k4[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) q4[i] = *reinterpret_cast<const float4*>(Qs + (ty + 16 * i) * ST + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) k4[j] = *reinterpret_cast<const float4*>(Ts + (tx + 16 * j) * ST + d);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[i][j] = fmaf(q4[i].x, k4[j].x, s[i][j]);
                        s[i][j] = fmaf(q4[i].y, k4[j].y, s[i][j]);
                        s[i][j] = fmaf(q4[i].z, k4[j].z, s[i][j]);
                        s[i][j] = fmaf(q4[i].w, k4[j].w, s[i][j]);
                    }
            }
            // masked scores become -inf by selection, so a NaN there does not count
            bool mine = true;            // every key of the block is visible to all of this thread's rows
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t lo = 0u, hi = 0u;
                if (rseq[i] >= 0) {
                    const unsigned long long* mrow = p.mask + ((size_t)rseq[i] * p.max_nodes + rnode[i]) * W;
                    const int n = pl.own_len[rseq[i]] - pl.kv[rseq[i]];
                    lo = visible32_of(it.seq, it.key0, rseq[i], pl.pre[rseq[i]], pl.kv[rseq[i]], n, mrow, W);
                    hi = visible32_of(it.seq, it.key0 + 32, rseq[i], pl.pre[rseq[i]], pl.kv[rseq[i]], n, mrow, W);
                }
                mine = mine && (rseq[i] < 0 || (lo & hi) == 0xffffffffu);
                float bm = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int k = tx + 16 * j;
                    const bool vis = ((k < 32 ? lo >> k : hi >> (k - 32)) & 1u) != 0u;
                    s[i][j] = vis ? s[i][j] * sl2 : -INFINITY;
                    bm = fmaxf(bm, s[i][j]);
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) bm = fmaxf(bm, __shfl_xor_sync(0xffffffffu, bm, o));
                const float nref = fmaxf(ref[i], bm);
                const float base = nref == -INFINITY ? 0.f : nref;
                const float corr = exp2_fast(ref[i] - base);             // 2^(-inf) = 0 before the first key
                ref[i] = nref;
                float ps = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = exp2_fast(s[i][j] - base);
                    ps += e;
                    Ps[(ty + 16 * i) * PS + tx + 16 * j] = e;
                }
                sum[i] = sum[i] * corr + ps;
#pragma unroll
                for (int d = 0; d < 4 * DC; ++d) acc[i][d] *= corr;
            }
            const bool open = __syncthreads_and(mine ? 1 : 0) != 0;      // K has been read, P is complete
            for (int i = tid; i < KB * (D / 4); i += kSimpleThreads) {
                const int k = i / (D / 4), c = i - k * (D / 4);
                *reinterpret_cast<float4*>(Ts + k * ST + 4 * c) =
                    k < nkey ? reinterpret_cast<const float4*>(Vb + (size_t)(it.key0 + k) * D)[c] : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            __syncthreads();
            // In a block that some row sees only in part, a weight of zero must not meet a NaN or an infinity
            // of a value that is not the row's: such products are left out.
            auto pv = [&](auto guarded) {
#pragma unroll 2
                for (int k = 0; k < KB; k += 4) {
                    float4 p4[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) p4[i] = *reinterpret_cast<const float4*>(Ps + (ty + 16 * i) * PS + k);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                        for (int c = 0; c < DC; ++c) {
                            const float4 v = *reinterpret_cast<const float4*>(Ts + (k + kk) * ST + 64 * c + 4 * tx);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float w = kk == 0 ? p4[i].x : (kk == 1 ? p4[i].y : (kk == 2 ? p4[i].z : p4[i].w));
                                if (!decltype(guarded)::value || w != 0.f) {
                                    acc[i][4 * c + 0] = fmaf(w, v.x, acc[i][4 * c + 0]);
                                    acc[i][4 * c + 1] = fmaf(w, v.y, acc[i][4 * c + 1]);
                                    acc[i][4 * c + 2] = fmaf(w, v.z, acc[i][4 * c + 2]);
                                    acc[i][4 * c + 3] = fmaf(w, v.w, acc[i][4 * c + 3]);
                                }
                            }
                        }
                }
            };
            if (open) pv(Flag<false>()); else pv(Flag<true>());
            if (blk + 1 < blk1) it.next(pl, ti, KB);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float s = sum[i];
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            const int r = ty + 16 * i;
            if (rseq[i] < 0) continue;
            if (whole) {
                if (!CTCSD_IN_BOUNDS(p.status, 83, orow[i], out_rows(p))) continue;
                const float inv = s > 0.f ? 1.f / s : (s == 0.f ? 0.f : s);      // a NaN sum stays a NaN
                float* out = static_cast<float*>(p.O) + orow[i] * D;
#pragma unroll
                for (int c = 0; c < DC; ++c)
                    *reinterpret_cast<float4*>(out + 64 * c + 4 * tx) =
                        make_float4(acc[i][4 * c] * inv, acc[i][4 * c + 1] * inv, acc[i][4 * c + 2] * inv, acc[i][4 * c + 3] * inv);
                if (tx == 0 && p.lse) p.lse[orow[i]] = s == 0.f ? -INFINITY : (ref[i] + log2f(s)) * kLn2;
            } else {
                const size_t part = (size_t)blockIdx.x * 2 + slot;
                if (!CTCSD_IN_BOUNDS(p.status, 84, part * TR + r, 2ll * gridDim.x * TR)) continue;
#pragma unroll
                for (int c = 0; c < DC; ++c)
                    p.part_o[(part * (D / 4) + 16 * c + tx) * TR + r] =
                        make_float4(acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]);
                if (tx == 0) p.part_ml[part * TR + r] = make_float2(ref[i], s);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------
// Merge.  A block looks after 32 packed rows of one kv head (lane = row, so that the transposed parts are
// read in whole lines; warps share the head dimension), and after as many output rows for the zero
// rows of unused nodes.  Parts are joined in span order: the result does not depend on timing.
// Bound by the latency of dependent rounds of loads (plan, parts), which come from L2 where the parts fit: 12.8 us
// cold for 128 parts of 256 rows of 128 columns.
// ---------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ void store8(T* out, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<float>(float* out, const float (&v)[8]) {
    reinterpret_cast<float4*>(out)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(out)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* out, const float (&v)[8]) {
    __nv_bfloat162 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(out) = *reinterpret_cast<uint4*>(w);
}

// A warp holds 8 columns of 32 rows: D / 8 warps.  The parts of a tile are taken four at a time, all their loads on the
// way at once, against a reference that follows the largest so far.
template <typename T, int D, int TR>
__global__ void __launch_bounds__(D * 4) shared_attention_merge_kernel(SharedAttnParams p, unsigned units) {
    constexpr int kWarps = D / 8, U = 4;
    extern __shared__ int row_off[];                         // [B+1]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int grp = p.grp;
    pdl_wait();
    pdl_trigger();
    const int* tile_cum = p.plan + kPlanHeader + p.B + 1;
    const int rows = p.plan[0], per_head = p.plan[2], spans = p.plan[3];
    for (int b = threadIdx.x; b <= p.B; b += kWarps * 32) row_off[b] = p.plan[kPlanHeader + b];
    const SpanMap sp = span_map_n(per_head, p.Hkv, spans);
    const int node_rows = p.max_nodes * grp;
    const int max_rows = p.B * node_rows;                    // packed rows if every node were live
    const int chunks = (max_rows + 31) / 32;
    __syncthreads();
    for (unsigned u = blockIdx.x; u < units; u += gridDim.x) {
        const int g = (int)(u / (unsigned)chunks), ch = (int)(u - (unsigned)g * (unsigned)chunks);
        {   // zero rows: output row (b, node, head of group g) for the nodes that are not used
            const int m = ch * 32 + lane;
            if (m < max_rows) {
                const int b = m / node_rows, o = m - b * node_rows;
                if (o >= row_off[b + 1] - row_off[b]) {
                    const int node = o / grp;
                    const size_t orow = ((size_t)b * p.max_nodes + node) * p.Hq + g * grp + (o - node * grp);
                    const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    if (CTCSD_IN_BOUNDS(p.status, 85, orow, out_rows(p))) {
                        store8<T>(static_cast<T*>(p.O) + orow * D + 8 * warp, z);
                        if (warp == 0 && p.lse) p.lse[orow] = -INFINITY;
                    }
                }
            }
        }
        const int pr0 = ch * 32;
        if (pr0 >= rows) continue;
        const int t = pr0 / TR;                              // 32 divides TR: one tile for all lanes
        const long long xs = (long long)g * per_head + tile_cum[t], xe = (long long)g * per_head + tile_cum[t + 1];
        const int c0 = sp.span_of(xs), c1 = sp.span_of(xe - 1);
        if (c0 == c1) continue;                              // finished by its span
        const int pr = pr0 + lane;
        if (pr >= rows) continue;
        const int r = pr - t * TR;
        // only the first part can be one that a span begins (slot 1); the others continue a tile (slot 0)
        float ref = -INFINITY, sum = 0.f, a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = 0.f;
        for (int c = c0; c <= c1; c += U) {
            float2 ml[U];
            float4 o[U][2];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                // (the last part again past the end, with no weight)
                const int cc = min(c + i, c1);
                const size_t part = (size_t)cc * 2 + (cc == c0 ? 1 : 0);
                ml[i] = p.part_ml[part * TR + r];
                o[i][0] = p.part_o[(part * (D / 4) + 2 * warp) * TR + r];
                o[i][1] = p.part_o[(part * (D / 4) + 2 * warp + 1) * TR + r];
                if (c + i > c1) ml[i] = make_float2(-INFINITY, 0.f);
            }
            float top = ref;
#pragma unroll
            for (int i = 0; i < U; ++i) top = fmaxf(top, ml[i].x);
            const float base = top == -INFINITY ? 0.f : top;
            const float keep = exp2_fast(ref - base);
            sum *= keep;
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] *= keep;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const float w = exp2_fast(ml[i].x - base);
                sum = fmaf(w, ml[i].y, sum);
                if (!(ml[i].y != 0.f)) continue;             // this part saw nothing: its output is not meaningful
                a[0] = fmaf(w, o[i][0].x, a[0]); a[1] = fmaf(w, o[i][0].y, a[1]);
                a[2] = fmaf(w, o[i][0].z, a[2]); a[3] = fmaf(w, o[i][0].w, a[3]);
                a[4] = fmaf(w, o[i][1].x, a[4]); a[5] = fmaf(w, o[i][1].y, a[5]);
                a[6] = fmaf(w, o[i][1].z, a[6]); a[7] = fmaf(w, o[i][1].w, a[7]);
            }
            ref = top;
        }
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (row_off[mid + 1] > pr) hi = mid; else lo = mid + 1;
        }
        const int o = pr - row_off[lo], node = o / grp;
        const size_t orow = ((size_t)lo * p.max_nodes + node) * p.Hq + g * grp + (o - node * grp);
        if (!CTCSD_IN_BOUNDS(p.status, 86, orow, out_rows(p))) continue;
        const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] *= inv;
        store8<T>(static_cast<T*>(p.O) + orow * D + 8 * warp, a);
        if (warp == 0 && p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * kLn2;
    }
}

template <typename T, int D, int TR>
int launch_merge(Handle* h, cudaStream_t s, const SharedAttnParams& p) {
    const long long max_rows = (long long)p.B * p.max_nodes * (p.Hq / p.Hkv);
    const unsigned units = (unsigned)((max_rows + 31) / 32) * (unsigned)p.Hkv;       // (at most 2^14 per kv head)
    const unsigned cap = (unsigned)h->num_sms * 16u;
    CTCSD_CUDA_CHECK(h, launch_pdl(shared_attention_merge_kernel<T, D, TR>, dim3(units < cap ? units : cap),
                                   dim3(D * 4), sizeof(int) * (size_t)(p.B + 1), s, 1, p, units));
    h->launches++;
    return CTCSD_OK;
}

template <int D>
int launch_simple(Handle* h, cudaStream_t s, const SharedAttnParams& p) {
    constexpr int TR = kSimpleRows, KB = kSimpleKeys;
    const int max_tiles = (int)(((long long)p.B * p.max_nodes * (p.Hq / p.Hkv) + TR - 1) / TR);
    const size_t smem = sizeof(float) * (TR * (D + 4) + KB * (D + 4) + TR * (KB + 4)) + sizeof(int) * plan_ints(p.B, max_tiles);
    auto kern = shared_attention_simple_kernel<D>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepSharedSimple, kern));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(h->num_sms * kSharedSpansPerSm), dim3(kSimpleThreads), smem, s, 1, p));
    h->launches++;
    return CTCSD_OK;
}

// Workspace: plan, part sums, part outputs; sized for the larger of the two kernels' needs.
struct SharedLayout { size_t plan, ml, o, total; };

SharedLayout shared_layout(const ctcsd_config& c) {
    const bool tc = c.dtype == CTCSD_DTYPE_BF16;
    const int TR = tc ? kTcRows : kSimpleRows;
    const size_t spans = (size_t)kLayoutSms * (tc ? 1 : kSharedSpansPerSm);
    const long long rows = (long long)c.B * c.max_nodes * (c.Hq / c.Hkv);
    SharedLayout l;
    l.plan = 0;
    l.ml = align_up(sizeof(int) * (size_t)(kPlanHeader + c.B + 1 + (rows + TR - 1) / TR + 1), 256);
    l.o = align_up(l.ml + sizeof(float2) * spans * 2 * TR, 256);
    l.total = align_up(l.o + sizeof(float) * spans * 2 * TR * (size_t)c.D, 256);
    return l;
}

bool shared_supported(const ctcsd_config& c) {
    return c.B <= kSharedMaxB && (long long)c.B * c.max_nodes * (c.Hq / c.Hkv) <= kSharedMaxRows;
}

}  // namespace

int launch_shared_attention_merge(Handle* h, cudaStream_t s, const SharedAttnParams& p, int TR) {
    if (TR == kTcRows) {
        if (p.D == 64) return launch_merge<__nv_bfloat16, 64, kTcRows>(h, s, p);
        return launch_merge<__nv_bfloat16, 128, kTcRows>(h, s, p);
    }
    if (p.D == 64) return launch_merge<float, 64, kSimpleRows>(h, s, p);
    return launch_merge<float, 128, kSimpleRows>(h, s, p);
}

}  // namespace ctcsd

using namespace ctcsd;

extern "C" int ctcsd_tree_attention_shared_workspace_bytes(const ctcsd_config* cfg, size_t* out_bytes) {
    if (!cfg || !out_bytes) return CTCSD_ERR_INVALID_ARG;
    const int rc = validate_config(*cfg);
    if (rc != CTCSD_OK) return rc;
    if (!shared_supported(*cfg)) return CTCSD_ERR_UNSUPPORTED;
    *out_bytes = shared_layout(*cfg).total;
    return CTCSD_OK;
}

extern "C" int ctcsd_tree_attention_shared(ctcsd_handle* hh, void* stream, void* workspace, size_t workspace_bytes,
                                           const void* Q, const void* Kp, const void* Vp, int Pcap, const int* prefix_len,
                                           const void* K, const void* V, int Lcap, const int* kv_len, const int* n_nodes,
                                           const unsigned long long* mask, float scale, void* out_O, float* out_lse) {
    if (!hh || !Q || !K || !V || !kv_len || !n_nodes || !mask || !out_O) return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    if (!shared_supported(c)) return CTCSD_ERR_UNSUPPORTED;
    if (Lcap < 1 || Pcap < 0) return CTCSD_ERR_INVALID_ARG;
    if (Pcap > 0 && (!Kp || !Vp || !prefix_len)) return CTCSD_ERR_INVALID_ARG;
    const bool tc = c.dtype == CTCSD_DTYPE_BF16;
    if (!plan_fits(c.B, c.max_nodes, c.Hq / c.Hkv, tc ? kTcRows : kSimpleRows, tc ? kTcKeys : kSimpleKeys, Pcap, Lcap)) return CTCSD_ERR_UNSUPPORTED;
    if (!(scale > 0.f) || isinf(scale)) return CTCSD_ERR_INVALID_ARG;      // the row maximum is taken before scaling
    const uintptr_t all = reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(Kp) | reinterpret_cast<uintptr_t>(Vp) |
                          reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) | reinterpret_cast<uintptr_t>(out_O);
    if (all & 15) return CTCSD_ERR_INVALID_ARG;
    const SharedLayout l = shared_layout(c);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < l.total) return CTCSD_ERR_WORKSPACE;
    SharedAttnParams p;
    p.Q = Q; p.Kp = Pcap > 0 ? Kp : nullptr; p.Vp = Pcap > 0 ? Vp : nullptr; p.K = K; p.V = V; p.O = out_O; p.lse = out_lse;
    p.prefix_len = Pcap > 0 ? prefix_len : nullptr; p.kv_len = kv_len; p.n_nodes = n_nodes; p.mask = mask;
    p.B = c.B; p.Hq = c.Hq; p.Hkv = c.Hkv; p.D = c.D; p.max_nodes = c.max_nodes; p.Lcap = Lcap; p.Pcap = Pcap; p.grp = c.Hq / c.Hkv;
    p.scale = scale;
    p.status = status_ptr(h);
    char* ws = static_cast<char*>(workspace);
    p.plan = reinterpret_cast<int*>(ws + l.plan);
    p.part_ml = reinterpret_cast<float2*>(ws + l.ml);
    p.part_o = reinterpret_cast<float4*>(ws + l.o);
    p.min_blocks = tc ? 3 : 1;
    p.long_span = 16;
    const DeviceGuard on(h->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int rc;
    if (tc) rc = launch_shared_attention_tc(h, s, p);
    else rc = c.D == 64 ? launch_simple<64>(h, s, p) : launch_simple<128>(h, s, p);
    if (rc != CTCSD_OK) return rc;
    return launch_shared_attention_merge(h, s, p, tc ? kTcRows : kSimpleRows);
}
