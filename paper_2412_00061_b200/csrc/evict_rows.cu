// ctcsd_evict_rows: cuts every sequence's cache to a budget of rows, per kv head the ones with the most
// gathered attention weight (ctcsd_attention_mass), the first `sinks` and the newest `recent` positions.
//
// Attention does not care about the order of cache rows, so nothing is shifted: the k-th kept row behind
// the new length moves into the k-th dropped row before it.  Sources and destinations are then
// disjoint ranges - no ordering between the copies - and a step that drops three rows moves three.  row_pos
// holds every row's position, which is what "newest" is decided on.
//
// One thread-block cluster per (kv head, sequence): radix selection of the threshold (11 + 11 + 10 bits, the
// histograms added up through distributed shared memory), ranks by block scans, then the copies.  With few (kv head,
// sequence) pairs their clusters leave most SMs idle, so the copies then are a second kernel's, spread evenly over all.
//
// Measured: 256 pairs that lose 1-7 of 2055 rows 11.8 us (the passes of the selection; 9.5 MB, 1.5 us of HBM); 256 pairs cut from up to
// 8192 rows to 1024 50 us for 219 MB: all CTAs select at once, for 10 us at least (measured with nothing to move), while HBM idles, and then copy at
// about 5.4 TB/s (rows of 256 bytes, scattered both ways); 8 pairs cut from 65536 rows to 16384 52 us, 28 of
// them the selection on 64 CTAs and the rest the moves (108 us with both in one kernel and loads one at a time).
#include "common.cuh"
#include "tc_primitives.cuh"

#include <math.h>

namespace ctcsd {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048;
// Keys a CTA keeps in shared memory; a longer share is read again from L2 in every pass (8 pairs cut to 16384 rows: from 65536 rows,
// the most that eight CTAs keep, 52 us, from 81920 97, from 131072 125).
constexpr int kCacheKeys = 8192;
constexpr int kMaxCluster = 8;
constexpr int kMaxRun = 17;            // rows a thread looks after at a time (odd: its neighbours' rows lie in other banks)

struct EvictParams {
    void* K; void* V;                  // [B,Hkv,Lcap,D]
    const float* mass; const int* row_pos;         // [B,Hkv,Lcap]
    const int* kv_len; const int* n_evicted;       // [B]
    float* out_mass; int* out_row_pos; int* out_kv_len; int* out_n_evicted;
    int* lists;                        // workspace [B,Hkv,Lcap]: dropped rows from the front, moving rows from the back
    int* n_move;                       // workspace [B,Hkv]: rows that move, where another kernel copies them, else null
    int B, Hkv, Lcap, row_bytes, budget, sinks, recent;
    unsigned* seq_ticket;              // [B], zero between calls
    int* status;
};

__device__ __forceinline__ void cluster_sync(int cs) {
    if (cs == 1) __syncthreads();
    else asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int4 ld_peer4(const void* local, int rank) {
    uint32_t a;
    int4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

// Copies pieces [i, n) in steps of `step`: piece k * chunks + c is 16 bytes (column c) of the k-th moving row, of K and
// of V.  Four at a time, so that a thread has eight loads on their way.  The lists are the workspace's; Near: those
// given, in shared memory.
template <bool Near>
__device__ __forceinline__ void move_pieces(const EvictParams& p, size_t row0, long long i, long long n, long long step, const int* near_holes = nullptr,
                                            const int* near_movers = nullptr) {
    const int row_bytes = p.row_bytes;
    unsigned char* Kb = static_cast<unsigned char*>(p.K) + row0 * row_bytes;
    unsigned char* Vb = static_cast<unsigned char*>(p.V) + row0 * row_bytes;
    const int* hole_list = Near ? near_holes : p.lists + row0;
    const int* mover_list = Near ? near_movers : hole_list + p.Lcap / 2;
    const int chunks = row_bytes / 16;                                     // a power of two: 8, 16 or 32
    const int sh = 31 - __clz(chunks);
    constexpr int U = 4;
    for (; i < n; i += U * step) {
        size_t src[U], dst[U];
        uint4 kk[U], vv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long x = i + u * step;
            src[u] = dst[u] = 0;
            if (x < n) {
                const int k = (int)(x >> sh), c = (int)(x & (chunks - 1));
                const int from = Near ? mover_list[k] : __ldcg(mover_list + k), to = Near ? hole_list[k] : __ldcg(hole_list + k);
                src[u] = (size_t)from * row_bytes + c * 16;
                dst[u] = (size_t)to * row_bytes + c * 16;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * step < n) {
                kk[u] = *reinterpret_cast<const uint4*>(Kb + src[u]);
                vv[u] = *reinterpret_cast<const uint4*>(Vb + src[u]);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * step < n && CTCSD_IN_BOUNDS(p.status, 63, dst[u], (size_t)p.Lcap * row_bytes)) {
                *reinterpret_cast<uint4*>(Kb + dst[u]) = kk[u];
                *reinterpret_cast<uint4*>(Vb + dst[u]) = vv[u];
            }
    }
}

constexpr unsigned kTopKey = 0xffffffffu;        // protected rows

// Ranking key: larger is kept first.  Protected rows lead; then the weight, +0 and -0 alike, NaN last.
__device__ __forceinline__ unsigned rank_key(float m, int pos, int sinks, int newest_from) {
    if (pos < sinks || pos >= newest_from) return kTopKey;
    if (m != m) return 0u;
    const unsigned u = __float_as_uint(m + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct __align__(16) EvictShared {
    int hist[3][kBins];
    int scan[2][kWarps];               // warp totals of a block scan (two buffers: one barrier per scan)
    int4 cta_cnt[2];                   // [0] ties; [1] dropped rows, moving rows
    int pick[3][3];                    // per round: digit, rows above it, rows in it
};

// Alone: a CTA by itself for each pair, which also copies (else a cluster of cs, or another kernel for the copies).
template <bool Alone>
__global__ void __launch_bounds__(kThreads, 2) evict_rows_kernel(EvictParams p, int cs_) {
    extern __shared__ __align__(16) unsigned char dyn[];
    EvictShared* sh = reinterpret_cast<EvictShared*>(dyn);
    unsigned* cache = reinterpret_cast<unsigned*>(sh + 1);                 // [kCacheKeys]
    const int g = blockIdx.y, b = blockIdx.z, rank = blockIdx.x;           // a cluster is one row of the grid
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cs = Alone ? 1 : cs_;
    pdl_wait();
    pdl_trigger();
    const int L = p.kv_len[b], ev = p.n_evicted[b];
    const bool bad = L < 0 || L > p.Lcap;
    if (bad && tid == 0 && rank == 0 && g == 0) report_error(p.status, CTCSD_ERR_INVALID_ARG, b);
    const size_t row0 = ((size_t)b * p.Hkv + g) * (size_t)p.Lcap;
    const float* mass = p.mass + row0;
    const int* row_pos = p.row_pos + row0;
    float* out_mass = p.out_mass + row0;
    int* out_pos = p.out_row_pos + row0;
    const bool in_place = p.mass == p.out_mass && p.row_pos == p.out_row_pos;
    const int keep = L < p.budget ? L : p.budget;
    const int share = ((L + cs - 1) / cs + 31) / 32 * 32;                  // rows of this CTA: [lo, hi)
    const int lo = min(rank * share, L), hi = min(lo + share, L);

    if (!bad && L <= p.budget) {
        if (!in_place)
            for (int j = lo + tid; j < hi; j += kThreads)
                if (CTCSD_IN_BOUNDS(p.status, 64, j, p.Lcap)) { out_mass[j] = mass[j]; out_pos[j] = row_pos[j]; }
    } else if (!bad) {
        const int newest_from = ev + L - p.recent;
        const bool cached = hi - lo <= kCacheKeys;
        for (int i = tid; i < 3 * kBins; i += kThreads) sh->hist[i / kBins][i % kBins] = 0;
        auto key_of = [&](int j) -> unsigned { return rank_key(mass[j], row_pos[j], p.sinks, newest_from); };
        auto key_at = [&](int j) -> unsigned { return cached ? cache[j - lo] : key_of(j); };
        __syncthreads();
        int flip = 0;
        // exclusive prefix over the block's threads, and the total
        auto block_scan = [&](int v, int& total) -> int {
            int incl = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += u;
            }
            if (lane == 31) sh->scan[flip][warp] = incl;
            __syncthreads();
            int below = 0;
            total = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const int x = sh->scan[flip][w];
                below += w < warp ? x : 0;
                total += x;
            }
            flip ^= 1;
            return below + incl - v;
        };
        // ---- threshold: the keep-th largest key, 11 + 11 + 10 bits from the top ----
        unsigned prefix = 0u;
        int shift = 32, left = keep;                                       // rows still to be found among the keys with this prefix
        for (int rd = 0; rd < 3; ++rd) {
            const int bits = rd == 2 ? 10 : 11, up = shift;
            shift -= bits;
            if (rd == 0) {
                constexpr int U = 8;                                       // loads on their way per thread and array
                for (int j0 = lo + tid; j0 < hi; j0 += U * kThreads) {
                    float m[U];
                    int q[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int j = min(j0 + u * kThreads, hi - 1);
                        m[u] = mass[j];
                        q[u] = row_pos[j];
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int j = j0 + u * kThreads;
                        if (j >= hi) continue;
                        const unsigned key = rank_key(m[u], q[u], p.sinks, newest_from);
                        if (cached) cache[j - lo] = key;
                        // (rows that go are overwritten by the moves, behind a barrier)
                        if (!in_place && j < keep && CTCSD_IN_BOUNDS(p.status, 65, j, p.Lcap)) { out_mass[j] = m[u]; out_pos[j] = q[u]; }
                        atomicAdd(&sh->hist[0][key >> shift], 1);
                    }
                }
            } else {
                for (int j = lo + tid; j < hi; j += kThreads) {
                    const unsigned key = key_at(j);
                    if ((key >> up) == prefix) atomicAdd(&sh->hist[rd][(key >> shift) & ((1u << bits) - 1u)], 1);
                }
            }
            cluster_sync(cs);
            const int nb = 1 << bits;
            // descending order of bins: thread t looks after bins nb-1-4t .. nb-4-4t
            static_assert(kBins / kThreads == 4, "a thread reads its bins as one vector");
            int v[4] = {0, 0, 0, 0};
            const int bin0 = nb - 4 - 4 * tid;                             // lowest of this thread's four
            if (bin0 >= 0) {
                if (cs == 1) {
                    const int4 h = *reinterpret_cast<const int4*>(&sh->hist[rd][bin0]);
                    v[0] = h.w; v[1] = h.z; v[2] = h.y; v[3] = h.x;
                } else {
                    int4 h[kMaxCluster];                                   // all requested, then added
#pragma unroll
                    for (int c = 0; c < kMaxCluster; ++c) h[c] = c < cs ? ld_peer4(&sh->hist[rd][bin0], c) : make_int4(0, 0, 0, 0);
#pragma unroll
                    for (int c = 0; c < kMaxCluster; ++c) { v[0] += h[c].w; v[1] += h[c].z; v[2] += h[c].y; v[3] += h[c].x; }
                }
            }
            const int sum = v[0] + v[1] + v[2] + v[3];
            int in_block;
            int before = block_scan(sum, in_block);
#pragma unroll
            for (int i = 0; i < kBins / kThreads; ++i) {
                if (before < left && before + v[i] >= left) {              // exactly one bin of one thread
                    sh->pick[rd][0] = nb - 1 - (tid * (kBins / kThreads) + i);
                    sh->pick[rd][1] = before;
                    sh->pick[rd][2] = v[i];
                }
                before += v[i];
            }
            __syncthreads();
            prefix = (prefix << bits) | (unsigned)sh->pick[rd][0];
            left -= sh->pick[rd][1];
            if (sh->pick[rd][2] == left) break;                            // the whole bin stays: no need to look closer
        }
        // rows whose key's top bits are above the threshold stay; of those equal to it the first `left`
        const bool ties_split = shift == 0;
        // every thread owns a run of rows, so that ranks follow row order; a share that is not in shared memory is
        // looked at in several tiles, and again in every pass
        const int n = hi - lo;
        const int run = min((n + kThreads - 1) / kThreads | 1, kMaxRun), tile = run * kThreads;
        auto classify = [&](int t0, unsigned& above, unsigned& ties) {     // bit i: row lo + t0 + tid * run + i
            above = ties = 0u;
            const int r0 = lo + t0 + tid * run;
            for (int i = 0; i < run && r0 + i < hi; ++i) {
                const unsigned top = key_at(r0 + i) >> shift;
                above |= top > prefix ? 1u << i : 0u;
                ties |= top == prefix ? 1u << i : 0u;
            }
        };
        int tie_base = 0;                                                  // ties in the CTAs before this one
        if (ties_split && cs > 1) {
            int cnt = 0, total;
            for (int t0 = 0; t0 < n; t0 += tile) {
                unsigned above, ties;
                classify(t0, above, ties);
                cnt += __popc(ties);
            }
            block_scan(cnt, total);
            if (tid == 0) sh->cta_cnt[0] = make_int4(total, 0, 0, 0);
            cluster_sync(cs);
            int4 q[kMaxCluster];
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) q[c] = c < rank ? ld_peer4(&sh->cta_cnt[0], c) : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) tie_base += q[c].x;
        }
        // rows of the tile that are dropped before the new length, and that are kept behind it; `place`: how many of
        // each (low and high half) come before this thread's in the tile, `sum`: in the whole tile
        int tie_run = tie_base;
        auto sort_out = [&](int t0, unsigned& holes, unsigned& movers, int& place, int& sum) {
            unsigned above, ties;
            classify(t0, above, ties);
            if (ties_split) {
                int total;
                int allow = left - tie_run - block_scan(__popc(ties), total);
                tie_run += total;
                for (; ties != 0u && allow > 0; --allow) {
                    above |= ties & (0u - ties);
                    ties &= ties - 1u;
                }
            } else {
                above |= ties;
            }
            const int r0 = lo + t0 + tid * run;
            const int mine = max(0, min(run, hi - r0)), front = max(0, min(mine, keep - r0));
            const unsigned all = (1u << mine) - 1u, before = (1u << front) - 1u;       // (mine <= 17)
            holes = ~above & before;
            movers = above & all & ~before;
            place = block_scan(__popc(holes) | __popc(movers) << 16, sum);
        };
        unsigned holes = 0u, movers = 0u;
        int place = 0, n_holes = 0, n_movers = 0;
        for (int t0 = 0; t0 < n; t0 += tile) {
            int sum;
            sort_out(t0, holes, movers, place, sum);
            n_holes += sum & 0xffff;
            n_movers += sum >> 16;
        }
        int hole_at = 0, mover_at = 0, n_move = n_holes;
        if (cs > 1) {
            if (tid == 0) sh->cta_cnt[1] = make_int4(n_holes, n_movers, 0, 0);
            cluster_sync(cs);
            int4 q[kMaxCluster];
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) q[c] = c < cs ? ld_peer4(&sh->cta_cnt[1], c) : make_int4(0, 0, 0, 0);
            n_move = 0;
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) {
                hole_at += c < rank ? q[c].x : 0;
                mover_at += c < rank ? q[c].y : 0;
                n_move += q[c].x;
            }
        }
        // as many rows move as there are holes, at most half of L: the lists share one array of L entries; short ones of a CTA by
        // itself stay with it, in the place of the histograms (batch-32 cut 57 -> 53 us)
        const bool near = Alone && n_move <= kBins;
        int* hole_list = near ? sh->hist[1] : p.lists + row0;
        int* mover_list = near ? sh->hist[2] : p.lists + row0 + p.Lcap / 2;
        tie_run = tie_base;
        for (int t0 = 0; t0 < n; t0 += tile) {
            int sum = 0;
            if (n > tile) sort_out(t0, holes, movers, place, sum);         // (else they are still in registers)
            const int r0 = lo + t0 + tid * run;
            int h = hole_at + (place & 0xffff), m = mover_at + (place >> 16);
            for (; holes != 0u; holes &= holes - 1u, ++h)
                if (CTCSD_IN_BOUNDS(p.status, 61, h, p.Lcap / 2)) hole_list[h] = r0 + __ffs(holes) - 1;
            for (; movers != 0u; movers &= movers - 1u, ++m)
                if (CTCSD_IN_BOUNDS(p.status, 62, m, p.Lcap - p.Lcap / 2)) mover_list[m] = r0 + __ffs(movers) - 1;
            hole_at += sum & 0xffff;
            mover_at += sum >> 16;
        }
        cluster_sync(cs);                                                  // the lists are complete; every weight has been read
        // ---- the moves: 16 bytes per thread and tensor, neighbours on one row ----
        if (p.n_move) {
            if (rank == 0 && tid == 0) p.n_move[b * p.Hkv + g] = n_move;
        } else {
            const long long pieces = (long long)n_move * (p.row_bytes / 16);
            if (near) move_pieces<true>(p, row0, tid, pieces, kThreads, sh->hist[1], sh->hist[2]);
            else move_pieces<false>(p, row0, (long long)rank * kThreads + tid, pieces, (long long)cs * kThreads);
        }
        auto move_mass = [&](int src, int dst) {
            if (!CTCSD_IN_BOUNDS(p.status, 66, dst, keep)) return;
            out_mass[dst] = mass[src];
            out_pos[dst] = row_pos[src];
        };
        if (near)
            for (int k = tid; k < n_move; k += kThreads) move_mass(sh->hist[2][k], sh->hist[1][k]);
        else
            for (int k = rank * kThreads + tid; k < n_move; k += cs * kThreads) move_mass(__ldcg(mover_list + k), __ldcg(hole_list + k));
    }
    if (p.n_move && rank == 0 && tid == 0 && (bad || L <= p.budget)) p.n_move[b * p.Hkv + g] = 0;
    // out_kv_len / out_n_evicted may be the very input arrays: the last kv head's cluster writes them, when
    // every head has read the old values (all CTAs of this cluster have: barrier)
    cluster_sync(cs);
    if (rank == 0 && tid == 0) {
        __threadfence();
        if (atomicAdd(&p.seq_ticket[b], 1u) == (unsigned)p.Hkv - 1u) {
            p.seq_ticket[b] = 0u;
            p.out_kv_len[b] = bad ? L : keep;
            p.out_n_evicted[b] = bad ? ev : ev + (L - keep);
        }
    }
}

// The copies of all pairs, dealt evenly: the pairs' pieces form one line, a CTA takes an equal span of it.
__global__ void __launch_bounds__(kThreads) evict_move_kernel(EvictParams p) {
    extern __shared__ long long cum[];                                     // [B*Hkv+1] pieces before each pair
    pdl_wait();
    pdl_trigger();
    const int units = p.B * p.Hkv, chunks = p.row_bytes / 16, lane = threadIdx.x & 31;
    if (threadIdx.x < 32) {
        long long run = 0;
        for (int u0 = 0; u0 < units; u0 += 32) {
            long long v = u0 + lane < units ? (long long)p.n_move[u0 + lane] * chunks : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long w = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += w;
            }
            if (u0 + lane < units) cum[u0 + lane + 1] = run + v;
            run += __shfl_sync(0xffffffffu, v, 31);
        }
        if (lane == 0) cum[0] = 0;
    }
    __syncthreads();
    const long long total = cum[units], x0 = total * blockIdx.x / gridDim.x, x1 = total * (blockIdx.x + 1) / gridDim.x;
    for (int u = 0; u < units; ++u) {
        const long long from = x0 > cum[u] ? x0 : cum[u], to = x1 < cum[u + 1] ? x1 : cum[u + 1];
        if (from >= to) continue;
        move_pieces<false>(p, (size_t)u * p.Lcap, from - cum[u] + threadIdx.x, to - cum[u], kThreads);
    }
}

}  // namespace
}  // namespace ctcsd

using namespace ctcsd;

extern "C" int ctcsd_evict_rows_workspace_bytes(const ctcsd_config* cfg, int Lcap, size_t* out_bytes) {
    if (!cfg || !out_bytes || Lcap < 1) return CTCSD_ERR_INVALID_ARG;
    const int rc = validate_config(*cfg);
    if (rc != CTCSD_OK) return rc;
    *out_bytes = align_up(sizeof(int) * (size_t)cfg->B * cfg->Hkv * ((size_t)Lcap + 1), 256);
    return CTCSD_OK;
}

extern "C" int ctcsd_evict_rows(ctcsd_handle* hh, void* stream, void* workspace, size_t workspace_bytes,
                                void* K, void* V, int Lcap, const float* mass, const int* row_pos,
                                const int* kv_len, const int* n_evicted, int budget, int sinks, int recent,
                                float* out_mass, int* out_row_pos, int* out_kv_len, int* out_n_evicted) {
    if (!hh || !K || !V || !mass || !row_pos || !kv_len || !n_evicted || !out_mass || !out_row_pos || !out_kv_len || !out_n_evicted)
        return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    if (Lcap < 1 || budget < 1 || sinks < 0 || recent < 0 || sinks > budget || recent > budget - sinks) return CTCSD_ERR_INVALID_ARG;
    if ((out_mass == mass) != (out_row_pos == row_pos)) return CTCSD_ERR_INVALID_ARG;      // both in place or neither
    if ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 15) return CTCSD_ERR_INVALID_ARG;
    if (c.B > 65535 || c.Hkv > 65535) return CTCSD_ERR_UNSUPPORTED;
    size_t need = 0;
    const int rc = ctcsd_evict_rows_workspace_bytes(&c, Lcap, &need);
    if (rc != CTCSD_OK) return rc;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < need) return CTCSD_ERR_WORKSPACE;
    EvictParams p;
    p.K = K; p.V = V; p.mass = mass; p.row_pos = row_pos; p.kv_len = kv_len; p.n_evicted = n_evicted;
    p.out_mass = out_mass; p.out_row_pos = out_row_pos; p.out_kv_len = out_kv_len; p.out_n_evicted = out_n_evicted;
    p.lists = static_cast<int*>(workspace);
    p.B = c.B; p.Hkv = c.Hkv; p.Lcap = Lcap; p.budget = budget; p.sinks = sinks; p.recent = recent;
    p.row_bytes = c.D * (c.dtype == CTCSD_DTYPE_BF16 ? 2 : 4);
    p.seq_ticket = reinterpret_cast<unsigned*>(h->ws + h->lay.seq_ticket_off);
    p.status = status_ptr(h);
    // a cluster per (kv head, sequence): more CTAs while they all run at once (two fit on an SM) and each
    // still has rows to look at.  (Measured with 512 / 1024 / 2048 rows a CTA at least, in us: 32 heads of one sequence cut from 4096 rows to
    // 1024 27.3 / 18.2 / 19.1; 8 heads, 32768 to 8192 31.1 / 32.4 / 31.3; 8192 to 2048 19.3 / 18.0 / 16.3; three rows leave 2051, 32 heads, 15.3 / 12.8 / 8.4,
    // 8 heads, three leave 8195 16.8 / 17.0 / 14.6.)
    const long long pairs = (long long)c.B * c.Hkv;
    int cs = 1;
    while (cs < kMaxCluster && pairs * cs * 2 <= 2ll * h->num_sms && Lcap / (cs * 2) >= 1024) cs *= 2;
    // the clusters cover less than half of the SMs, and there may be enough to copy: a kernel of its own for that.  The capacity decides,
    // since only the device knows the lengths.  (Measured apart / in one kernel, in us, 8 heads: 65536 rows cut to 16384 52 / 66, 16384 to 4096 20.6 / 23.1, 8192
    // to 2048, at the limit, 18.0 / 18.3, 4096 to 1024, below it, 15.8 / 16.1; three rows leave 2051 in a buffer of that size, below it, 15.4 / 12.8, in a buffer
    // of 65048 rows 19.1 / 16.1.)
    const long long movable = budget < Lcap - budget ? budget : Lcap - budget;
    const bool apart = pairs * cs * 2 <= h->num_sms && movable > 0 && pairs * movable * p.row_bytes >= (4ll << 20);
    p.n_move = apart ? p.lists + (size_t)pairs * Lcap : nullptr;
    const size_t smem = sizeof(EvictShared) + sizeof(unsigned) * kCacheKeys;
    const DeviceGuard on(h->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool alone = cs == 1 && !apart;
    auto kern = alone ? evict_rows_kernel<true> : evict_rows_kernel<false>;
    CTCSD_CUDA_CHECK(h, prepare_kernel(h, alone ? kPrepEvictAlone : kPrepEvict, kern));
    CTCSD_CUDA_CHECK(h, launch_pdl(kern, dim3(cs, c.Hkv, c.B), dim3(kThreads), smem, s, cs, p, cs));
    h->launches++;
    if (apart) {
        CTCSD_CUDA_CHECK(h, launch_pdl(evict_move_kernel, dim3(2 * h->num_sms), dim3(kThreads), sizeof(long long) * (size_t)(pairs + 1), s, 1, p));
        h->launches++;
    }
    return CTCSD_OK;
}
