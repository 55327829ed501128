// ctcsd_tree_attention_q4: tree attention over a cache held in 4 bits.
//   O[b,i,h] = sum_j p_j v_j,  p = softmax_j(scale q.k_j),  j over the kv_len[b] cached rows (4 bits, q4.cuh) and the tree rows of
//   node i's mask (full precision);  lse[b,i,h] = log sum_j exp(scale q.k_j).
// The work is divided as q4_attention.cuh describes.  This file holds the entry points, the kernel without tensor cores (float32)
// and the merge of tiles that were cut.
#include "q4_attention.cuh"

#include <math.h>

namespace ctcsd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ---------------------------------------------------------------------------------------
// Without tensor cores: 64 rows x 64 keys per step, 256 threads; a thread computes 4 x 4 scores and 4 x D/16 outputs from 128-bit
// shared loads, rows and keys dealt 16 apart (row stride D + 4: no bank conflicts).  Levels become float32 values on the way
// into shared memory.
// ---------------------------------------------------------------------------------------
constexpr int kSimpleThreads = 256;

template <bool B> struct Flag { static constexpr bool value = B; };

template <typename T> __device__ __forceinline__ void store4(T* p, float4 v);
template <> __device__ __forceinline__ void store4<float>(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
template <> __device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16* p, float4 v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

template <int D>
__global__ void __launch_bounds__(kSimpleThreads, kAq4SimplePerSm) attention_q4_simple_kernel(AttnQ4Params p) {
    constexpr int TR = kAq4SimpleRows, KB = kAq4SimpleKeys, ST = D + 4, PS = KB + 4, DC = D / 64, W = D / 8;
    extern __shared__ __align__(16) float sm[];
    float* Qs = sm;                      // [TR][ST]
    float* Ts = Qs + TR * ST;            // [KB][ST]: a K block, then its V block
    float* Ps = Ts + KB * ST;            // [TR][PS]
    PlanQ4 pl;
    pl.carve(reinterpret_cast<int*>(Ps + TR * PS), p.B);
    pdl_wait();
    pdl_trigger();
    const SpansQ4 sp = plan_q4_build(pl, p, TR, KB, (int)gridDim.x);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int MW = (p.max_nodes + 63) / 64;
    const float sl2 = p.scale * kLog2e;
    WalkQ4 at;
    bool more = at.init(pl, sp, p.B, KB, blockIdx.x);
    attn_q4_sides<float, D>(p, pl, sp, at, more);
    for (; more; more = at.next(pl, p.B, KB)) {
        const int g = at.g, b = at.b, kv = pl.kv[b], n = pl.n[b], row0 = at.t * TR;
        const int nrows = n * p.grp - row0 < TR ? n * p.grp - row0 : TR;
        const size_t pair = (size_t)b * p.Hkv + g;
        auto out_row = [&](int r) -> size_t {                                // row of the tile -> row of Q, O, lse
            const int node = (row0 + r) / p.grp;
            return ((size_t)b * p.max_nodes + node) * p.Hq + g * p.grp + (row0 + r - node * p.grp);
        };
        __syncthreads();                 // the previous tile's shared memory is free
        for (int i = tid; i < TR * (D / 4); i += kSimpleThreads) {
            const int r = i / (D / 4), c = i - r * (D / 4);
            *reinterpret_cast<float4*>(Qs + r * ST + 4 * c) =
                r < nrows ? *reinterpret_cast<const float4*>(static_cast<const float*>(p.Q) + out_row(r) * D + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float acc[4][4 * DC], ref[4], sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ref[i] = -INFINITY; sum[i] = 0.f;
#pragma unroll
            for (int d = 0; d < 4 * DC; ++d) acc[i][d] = 0.f;
        }
        // keys key0 .. key0+nkey-1 of the cache (or of the tree) as values, zeros behind them
        auto load_tile = [&](const uint32_t* q, const uint32_t* so, const void* tree, bool cached, int key0, int nkey) {
            for (int i = tid; i < KB * W; i += kSimpleThreads) {
                const int k = i / W, c = i - k * W;
                float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (k < nkey) {
                    if (cached) {
                        const size_t a = (pair * p.Lcap + key0 + k) * W + c;
                        const uint32_t w = q[a], pr = so[a >> 2];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = q4_value_f32(w, e, bf16lo(pr), bf16hi(pr));
                    } else {
                        load8(static_cast<const float*>(tree) + ((pair * p.max_nodes + key0 + k) * W + c) * 8, v);
                    }
                }
                float* dst = Ts + k * ST + 8 * c;
                reinterpret_cast<float4*>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4*>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
        };
        for (int blk = at.blk0; blk < at.blk1; ++blk) {
            const bool cached = blk < at.cached;
            const int key0 = (cached ? blk : blk - at.cached) * KB, len = cached ? kv : n;
            const int nkey = len - key0 < KB ? len - key0 : KB;
            __syncthreads();             // V of the previous block has been read
            load_tile(p.Kq, p.Ks, p.Kt, cached, key0, nkey);
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
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = ty + 16 * i;
                uint32_t lo = 0u, hi = 0u;                                   // keys of the block that the row sees
                if (r < nrows) {
                    if (cached) {
                        lo = nkey >= 32 ? 0xffffffffu : (1u << nkey) - 1u;
                        hi = nkey >= 64 ? 0xffffffffu : (nkey > 32 ? (1u << (nkey - 32)) - 1u : 0u);
                    } else {
                        const unsigned long long* mrow = p.mask + ((size_t)b * p.max_nodes + (row0 + r) / p.grp) * MW;
                        lo = tree_bits32(mrow, MW, key0, n);
                        hi = tree_bits32(mrow, MW, key0 + 32, n);
                    }
                }
                // masked scores become -inf by selection, so a NaN there does not count
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
                const float corr = exp2_q4(ref[i] - base);                   // 2^(-inf) = 0 before the first key
                ref[i] = nref;
                float ps = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = exp2_q4(s[i][j] - base);
                    ps += e;
                    Ps[r * PS + tx + 16 * j] = e;
                }
                sum[i] = sum[i] * corr + ps;
#pragma unroll
                for (int d = 0; d < 4 * DC; ++d) acc[i][d] *= corr;
            }
            __syncthreads();             // K has been read, P is complete
            load_tile(p.Vq, p.Vs, p.Vt, cached, key0, nkey);
            __syncthreads();
            // Every row of the tile sees every cached row; of the tree's rows it sees some, and a weight of zero must not meet a NaN or an
            // infinity there: such products are left out.
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
            if (cached) pv(Flag<false>()); else pv(Flag<true>());
        }
        const bool whole = at.whole();
        const size_t part = (size_t)blockIdx.x * 2 + at.slot();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float s = sum[i];
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            const int r = ty + 16 * i;
            if (r >= nrows) continue;
            if (whole) {
                const size_t orow = out_row(r);
                if (!CTCSD_IN_BOUNDS(p.status, 132, orow, out_rows(p))) continue;
                const float inv = s > 0.f ? 1.f / s : (s == 0.f ? 0.f : s);  // a NaN sum stays a NaN
                float* out = static_cast<float*>(p.O) + orow * D;
#pragma unroll
                for (int c = 0; c < DC; ++c)
                    store4(out + 64 * c + 4 * tx, make_float4(acc[i][4 * c] * inv, acc[i][4 * c + 1] * inv, acc[i][4 * c + 2] * inv, acc[i][4 * c + 3] * inv));
                if (tx == 0 && p.lse) p.lse[orow] = s == 0.f ? -INFINITY : (ref[i] + log2f(s)) * kLn2;
            } else if (CTCSD_IN_BOUNDS(p.status, 133, part * TR + r, 2ll * gridDim.x * TR)) {
#pragma unroll
                for (int c = 0; c < DC; ++c)
                    p.part_o[(part * (D / 4) + 16 * c + tx) * TR + r] = make_float4(acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]);
                if (tx == 0) p.part_ml[part * TR + r] = make_float2(ref[i], s);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------
// Merge of tiles that were cut.  A block for a span and a share of the columns: if the span is the second of a tile's, the block joins the tile's parts
// in span order, four at a time (the result does not depend on timing), else it has nothing to do.  A thread holds eight columns
// of a row; neighbours take neighbouring rows, so that the transposed parts are read in whole lines.  Latency bounds it: one round of loads for the cut and
// one for every four parts.
// ---------------------------------------------------------------------------------------
constexpr int kMergeThreads = 512;
// Eights of columns of a block: as many as give every thread one.
__host__ __device__ constexpr int merge_eights(int D, int TR) { return kMergeThreads / TR < D / 8 ? kMergeThreads / TR : D / 8; }

template <typename T, int D>
__global__ void __launch_bounds__(kMergeThreads) attention_q4_merge_kernel(AttnQ4Params p, int TR) {
    constexpr int U = 4;
    pdl_wait();
    pdl_trigger();
    const int4 cut = p.cuts[blockIdx.x];
    if (cut.x < 0) return;
    const int g = cut.x, b = cut.y, row0 = cut.z * TR, c0 = (int)blockIdx.x - 1, c1 = cut.w;
    const int left = p.n_nodes[b] * p.grp - row0, nrows = left < TR ? left : TR;
    const int eights = merge_eights(D, TR), i = threadIdx.x;
    const int tr = i % TR, c8 = blockIdx.y * eights + i / TR;                // row of the tile, columns 8 c8 ..
    if (i < TR * eights && tr < nrows) {
        // only the first part can be one that a span begins (slot 1); the others continue a tile (slot 0)
        float ref = -INFINITY, sum = 0.f, a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = 0.f;
        for (int c = c0; c <= c1; c += U) {
            float2 ml[U];
            float4 o[U][2];
#pragma unroll
            for (int k = 0; k < U; ++k) {                                    // (the last part again past the end, with no weight)
                const int cc = min(c + k, c1);
                const size_t part = (size_t)cc * 2 + (cc == c0 ? 1 : 0);
                ml[k] = p.part_ml[part * TR + tr];
                o[k][0] = p.part_o[(part * (D / 4) + 2 * c8) * TR + tr];
                o[k][1] = p.part_o[(part * (D / 4) + 2 * c8 + 1) * TR + tr];
                if (c + k > c1) ml[k] = make_float2(-INFINITY, 0.f);
            }
            float top = ref;
#pragma unroll
            for (int k = 0; k < U; ++k) top = fmaxf(top, ml[k].x);
            const float base = top == -INFINITY ? 0.f : top;
            const float keep = exp2_q4(ref - base);
            sum *= keep;
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] *= keep;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const float w = exp2_q4(ml[k].x - base);
                sum = fmaf(w, ml[k].y, sum);
                if (!(ml[k].y != 0.f)) continue;                             // this part saw nothing
                a[0] = fmaf(w, o[k][0].x, a[0]); a[1] = fmaf(w, o[k][0].y, a[1]);
                a[2] = fmaf(w, o[k][0].z, a[2]); a[3] = fmaf(w, o[k][0].w, a[3]);
                a[4] = fmaf(w, o[k][1].x, a[4]); a[5] = fmaf(w, o[k][1].y, a[5]);
                a[6] = fmaf(w, o[k][1].z, a[6]); a[7] = fmaf(w, o[k][1].w, a[7]);
            }
            ref = top;
        }
        const int node = (row0 + tr) / p.grp;
        const size_t orow = ((size_t)b * p.max_nodes + node) * p.Hq + g * p.grp + (row0 + tr - node * p.grp);
        if (!CTCSD_IN_BOUNDS(p.status, 134, orow, out_rows(p))) return;
        const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
        T* out = static_cast<T*>(p.O) + orow * D + 8 * c8;
        store4(out, make_float4(a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv));
        store4(out + 4, make_float4(a[4] * inv, a[5] * inv, a[6] * inv, a[7] * inv));
        if (c8 == 0 && p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * kLn2;
    }
}

template <typename T, int D>
int launch_merge(Handle* h, cudaStream_t s, const AttnQ4Params& p, int TR, int spans) {
    CTCSD_CUDA_CHECK(h, launch_pdl(attention_q4_merge_kernel<T, D>, dim3(spans, D / 8 / merge_eights(D, TR)), dim3(kMergeThreads), 0, s, 1, p, TR));
    h->launches++;
    return CTCSD_OK;
}

template <int D>
int launch_simple(Handle* h, cudaStream_t s, const AttnQ4Params& p) {
    constexpr int TR = kAq4SimpleRows, KB = kAq4SimpleKeys;
    const size_t smem = sizeof(float) * (TR * (D + 4) + KB * (D + 4) + TR * (KB + 4)) + sizeof(int) * PlanQ4::ints(p.B);
    auto kern = attention_q4_simple_kernel<D>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, kPrepAttnQ4Simple, kern));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(h->num_sms * kAq4SimplePerSm), dim3(kSimpleThreads), smem, s, 1, p));
    h->launches++;
    return CTCSD_OK;
}

bool few_rows(const ctcsd_config& c) { return c.dtype == CTCSD_DTYPE_BF16 && c.max_nodes * (c.Hq / c.Hkv) <= kAq4MmaRows; }

// Which kernel serves a handle: its tile, block and largest grid.
struct Form { int TR, KB, spans; };
Form form_of(const ctcsd_config& c) {
    if (few_rows(c)) return {kAq4MmaRows, kAq4MmaKeys, kLayoutSms};
    if (c.dtype == CTCSD_DTYPE_BF16) return {c.max_nodes * (c.Hq / c.Hkv) <= 128 ? 128 : 256, kAq4TcKeys, kLayoutSms};
    return {kAq4SimpleRows, kAq4SimpleKeys, kLayoutSms * kAq4SimplePerSm};
}

// Workspace: cuts, part sums, part outputs.
struct AttnLayout { size_t cuts, ml, o, total; };
AttnLayout attn_layout(const ctcsd_config& c) {
    const Form f = form_of(c);
    AttnLayout l;
    l.cuts = 0;
    l.ml = align_up(sizeof(int4) * (size_t)f.spans, 256);
    l.o = align_up(l.ml + sizeof(float2) * f.spans * 2 * f.TR, 256);
    l.total = align_up(l.o + sizeof(float) * f.spans * 2 * f.TR * (size_t)c.D, 256);
    return l;
}

bool attn_supported(const ctcsd_config& c) {
    return c.B <= kAq4MaxB;
}

}  // namespace
}  // namespace ctcsd

using namespace ctcsd;

extern "C" int ctcsd_tree_attention_q4_workspace_bytes(const ctcsd_config* cfg, size_t* out_bytes) {
    if (!cfg || !out_bytes) return CTCSD_ERR_INVALID_ARG;
    const int rc = validate_config(*cfg);
    if (rc != CTCSD_OK) return rc;
    if (!attn_supported(*cfg)) return CTCSD_ERR_UNSUPPORTED;
    *out_bytes = attn_layout(*cfg).total;
    return CTCSD_OK;
}

extern "C" int ctcsd_tree_attention_q4(ctcsd_handle* hh, void* stream, void* workspace, size_t workspace_bytes, const void* Q,
                                       const void* Kq, const void* Ks, const void* Vq, const void* Vs, int Lcap,
                                       const void* Kt, const void* Vt, const int* kv_len, const int* n_nodes,
                                       const unsigned long long* mask, float scale, void* out_O, float* out_lse) {
    if (!hh || !Q || !Kq || !Ks || !Vq || !Vs || !Kt || !Vt || !kv_len || !n_nodes || !mask || !out_O) return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    if (!attn_supported(c)) return CTCSD_ERR_UNSUPPORTED;
    if (Lcap < 1 || !(scale > 0.f) || isinf(scale)) return CTCSD_ERR_INVALID_ARG;            // the row maximum is taken before scaling
    const uintptr_t all = reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(Kq) | reinterpret_cast<uintptr_t>(Ks) |
                          reinterpret_cast<uintptr_t>(Vq) | reinterpret_cast<uintptr_t>(Vs) | reinterpret_cast<uintptr_t>(Kt) |
                          reinterpret_cast<uintptr_t>(Vt) | reinterpret_cast<uintptr_t>(out_O);
    if (all & 15) return CTCSD_ERR_INVALID_ARG;
    const Form f = form_of(c);
    const int grp = c.Hq / c.Hkv;
    if (!plan_q4_fits(c.B, c.max_nodes, grp, f.TR, f.KB, Lcap)) return CTCSD_ERR_UNSUPPORTED;
    const AttnLayout l = attn_layout(c);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < l.total) return CTCSD_ERR_WORKSPACE;
    AttnQ4Params p;
    p.Q = Q; p.O = out_O; p.lse = out_lse; p.Kt = Kt; p.Vt = Vt;
    p.Kq = static_cast<const uint32_t*>(Kq); p.Ks = static_cast<const uint32_t*>(Ks);
    p.Vq = static_cast<const uint32_t*>(Vq); p.Vs = static_cast<const uint32_t*>(Vs);
    p.kv_len = kv_len; p.n_nodes = n_nodes; p.mask = mask;
    p.B = c.B; p.Hq = c.Hq; p.Hkv = c.Hkv; p.D = c.D; p.max_nodes = c.max_nodes; p.Lcap = Lcap; p.grp = grp;
    p.scale = scale;
    p.status = status_ptr(h);
    char* ws = static_cast<char*>(workspace);
    p.spans = f.spans;
    p.cuts = reinterpret_cast<int4*>(ws + l.cuts);
    p.part_ml = reinterpret_cast<float2*>(ws + l.ml);
    p.part_o = reinterpret_cast<float4*>(ws + l.o);
    const DeviceGuard on(h->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int rc;
    if (few_rows(c)) rc = launch_attention_q4_mma(h, s, p);
    else if (c.dtype == CTCSD_DTYPE_BF16) rc = launch_attention_q4_tc(h, s, p, f.TR);
    else rc = c.D == 64 ? launch_simple<64>(h, s, p) : launch_simple<128>(h, s, p);
    if (rc != CTCSD_OK) return rc;
    const int spans = c.dtype == CTCSD_DTYPE_BF16 ? h->num_sms : h->num_sms * kAq4SimplePerSm;
    if (c.dtype == CTCSD_DTYPE_BF16) return c.D == 64 ? launch_merge<__nv_bfloat16, 64>(h, s, p, f.TR, spans) : launch_merge<__nv_bfloat16, 128>(h, s, p, f.TR, spans);
    return c.D == 64 ? launch_merge<float, 64>(h, s, p, f.TR, spans) : launch_merge<float, 128>(h, s, p, f.TR, spans);
}
