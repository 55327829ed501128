// Rows of a 4-bit cache: ctcsd_store_rows_q4 (a prompt's keys and values), ctcsd_commit_accepted_q4 (the accepted path of a
// step) and ctcsd_load_rows_q4 (rows back as values).
//
// A cached row is D/2 bytes of levels and D/32 (scale, origin) pairs (q4.cuh); K and V have an array of each, [B,Hkv,Lcap].  A thread
// deals with eight values: 16 bytes of bfloat16 on one side, one word of levels on the other, and four neighbouring
// threads with a group, whose limits they find by two shuffles.
#include "q4.cuh"

namespace ctcsd {
namespace {

struct RowsQ4 {
    uint32_t* Kq; uint32_t* Ks;          // levels [rows][D/8 words], scales and origins [rows][D/32 words]
    uint32_t* Vq; uint32_t* Vs;
};

constexpr int kThreads = 256;

template <typename T> __device__ __forceinline__ void store8(T* out, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<float>(float* out, const float (&v)[8]) {
    reinterpret_cast<float4*>(out)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(out)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Eight values as they stand in memory, and as their word (by four neighbouring lanes a group; all lanes of the warp take part).
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void zero() { w = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ uint32_t quantize(uint32_t& so) const {
        // (limits two at a time)
        uint32_t lo = min2_nan(min2_nan(w.x, w.y), min2_nan(w.z, w.w)), hi = max2_nan(max2_nan(w.x, w.y), max2_nan(w.z, w.w));
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            lo = min2_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = max2_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        so = q4_scale_origin(min_nan(bf16lo(lo), bf16hi(lo)), max_nan(bf16lo(hi), bf16hi(hi)));
        const float v[8] = {bf16lo(w.x), bf16hi(w.x), bf16lo(w.y), bf16hi(w.y), bf16lo(w.z), bf16hi(w.z), bf16lo(w.w), bf16hi(w.w)};
        return q4_word(v, so);
    }
};
template <> struct Eight<float> {
    float v[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    __device__ __forceinline__ void load(const float* p) { load8(p, v); }
    __device__ __forceinline__ uint32_t quantize(uint32_t& so) const {
        float lo = v[0], hi = v[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) { lo = min_nan(lo, v[i]); hi = max_nan(hi, v[i]); }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        so = q4_scale_origin(lo, hi);
        return q4_word(v, so);
    }
};

struct StoreParams {
    const void* K; const void* V;        // [B,Hkv,Lsrc,D]
    RowsQ4 c;
    const int* n_rows; const int* at;    // [B]
    int Hkv, Lsrc, Lcap;
    int* status;
};

// One CTA per (kv head, sequence) and share of the rows.  Threads of a warp take neighbouring words, so whole lines go both ways.
// (32 prompts of 1024-4096 rows of 8 heads of 128: 144 us, of which finding levels, with a test for ties and its branch for every value, is 60; the bytes 69.
// Reading them back takes 118, mostly writing.)
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) store_rows_q4_kernel(StoreParams p) {
    constexpr int W = D / 8;             // words of a row
    pdl_wait();
    pdl_trigger();
    const int g = blockIdx.y, b = blockIdx.z;
    const int n = p.n_rows[b], at = p.at ? p.at[b] : 0;
    if (n < 0 || n > p.Lsrc || at < 0 || at > p.Lcap - n) {
        if (threadIdx.x == 0 && blockIdx.x == 0 && g == 0) report_error(p.status, CTCSD_ERR_INVALID_ARG, b);
        return;
    }
    const size_t pair = (size_t)b * p.Hkv + g;
    const long long words = (long long)n * W, step = (long long)gridDim.x * kThreads;
    const size_t dst = (pair * p.Lcap + at) * W;
    const T* src[2] = {static_cast<const T*>(p.K) + pair * p.Lsrc * D, static_cast<const T*>(p.V) + pair * p.Lsrc * D};
    uint32_t* q[2] = {p.c.Kq + dst, p.c.Vq + dst};
    uint32_t* s[2] = {p.c.Ks + dst / 4, p.c.Vs + dst / 4};
    // (the same number of turns for all lanes of a warp: a group's lanes shuffle; the next turn's values are on their way meanwhile)
    auto fetch = [&](long long i, Eight<T> (&v)[2]) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (i < words) v[k].load(src[k] + i * 8);
            else v[k].zero();
        }
    };
    const int lane = threadIdx.x & 31;
    long long i0 = (long long)blockIdx.x * kThreads + (threadIdx.x & ~31);
    Eight<T> v[2], next[2];
    fetch(i0 + lane, v);
    for (; i0 < words; i0 += step) {
        const long long i = i0 + lane;
        fetch(i + step, next);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t so;
            const uint32_t w = v[k].quantize(so);
            if (i < words && CTCSD_IN_BOUNDS(p.status, 121, at * (long long)W + i, (long long)p.Lcap * W)) {
                q[k][i] = w;
                if ((i & 3) == 0) s[k][i >> 2] = so;
            }
            v[k] = next[k];
        }
    }
}

struct LoadParams {
    RowsQ4 c;
    const int* first; const int* n_rows; // [B]
    void* K; void* V;                    // [B,Hkv,Lout,D]
    int Hkv, Lcap, Lout;
    int* status;
};

template <typename T> __device__ __forceinline__ void store_values(T* out, uint32_t w, uint32_t so);
template <> __device__ __forceinline__ void store_values<__nv_bfloat16>(__nv_bfloat16* out, uint32_t w, uint32_t so) {
    *reinterpret_cast<uint4*>(out) = q4_values_bf16(w, so);
}
template <> __device__ __forceinline__ void store_values<float>(float* out, uint32_t w, uint32_t so) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = q4_value_f32(w, i, bf16lo(so), bf16hi(so));
    store8<float>(out, v);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) load_rows_q4_kernel(LoadParams p) {
    constexpr int W = D / 8;
    pdl_wait();
    pdl_trigger();
    const int g = blockIdx.y, b = blockIdx.z;
    int n = p.n_rows[b], first = p.first ? p.first[b] : 0;
    if (n < 0 || n > p.Lout || first < 0 || first > p.Lcap - n) {
        if (threadIdx.x == 0 && blockIdx.x == 0 && g == 0) report_error(p.status, CTCSD_ERR_INVALID_ARG, b);
        n = first = 0;
    }
    const size_t pair = (size_t)b * p.Hkv + g;
    const long long words = (long long)n * W, all = (long long)p.Lout * W, step = (long long)gridDim.x * kThreads;
    const size_t from = (pair * p.Lcap + first) * W;
    const uint32_t* q[2] = {p.c.Kq + from, p.c.Vq + from};
    const uint32_t* s[2] = {p.c.Ks + from / 4, p.c.Vs + from / 4};
    T* out[2] = {static_cast<T*>(p.K) + pair * p.Lout * D, static_cast<T*>(p.V) + pair * p.Lout * D};
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < all; i += step) {
        uint32_t w[2] = {0u, 0u}, so[2] = {0u, 0u};      // (a level of a group of zeros: rows past the last are zero)
        if (i < words) {
#pragma unroll
            for (int k = 0; k < 2; ++k) { w[k] = q[k][i]; so[k] = s[k][i >> 2]; }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (CTCSD_IN_BOUNDS(p.status, 122, i, all)) store_values<T>(out[k] + i * 8, w[k], so[k]);
    }
}

struct CommitQ4Params {
    const void* Kt; const void* Vt;      // [B,Hkv,max_nodes,D]
    RowsQ4 c;
    const int* kv_len; const int* acc_len; const int* acc_nodes;
    int Hkv, Lcap, T, max_nodes;
    int* out_kv_len; int* out_sel_row;
    unsigned* seq_ticket;                // [B], zero between calls
    int* status;
};

// One CTA per (kv head, sequence): the root and the accepted nodes, at most nine rows, to rows kv_len .. of the cache.  A launch and one
// round of loads bound it.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) commit_accepted_q4_kernel(CommitQ4Params p) {
    constexpr int W = D / 8;
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    pdl_wait();
    pdl_trigger();
    const int L = p.kv_len[b];
    int n = p.acc_len[b];
    bool bad = n < 0 || n > p.T || L < 0 || L > p.Lcap - 1 - n;
    for (int l = 0; l < n && !bad; ++l) {
        const int node = p.acc_nodes[b * p.T + l];
        bad = node < 1 || node >= p.max_nodes;
    }
    if (bad && tid == 0) report_error(p.status, CTCSD_ERR_INVALID_ARG, b);
    const size_t pair = (size_t)b * p.Hkv + g;
    const int words = bad ? 0 : 2 * (n + 1) * W;         // K's rows, then V's
    for (int i0 = tid & ~31; i0 < words; i0 += kThreads) {
        const int i = i0 + (tid & 31);
        const int which = i >= (n + 1) * W ? 1 : 0, r = i - which * (n + 1) * W;
        const int l = r / W, w = r - l * W;
        Eight<T> v;
        v.zero();
        if (i < words) {
            const int node = l > 0 ? p.acc_nodes[b * p.T + l - 1] : 0;
            v.load(static_cast<const T*>(which ? p.Vt : p.Kt) + ((pair * p.max_nodes + node) * W + w) * 8);
        }
        uint32_t so;
        const uint32_t word = v.quantize(so);
        if (i < words && CTCSD_IN_BOUNDS(p.status, 123, L + l, p.Lcap)) {
            const size_t at = (pair * p.Lcap + L + l) * W + w;
            (which ? p.c.Vq : p.c.Kq)[at] = word;
            if ((w & 3) == 0) (which ? p.c.Vs : p.c.Ks)[at >> 2] = so;
        }
    }
    // out_kv_len may be the array kv_len: the new length is written when every kv head's CTA has read the old one
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        if (atomicAdd(&p.seq_ticket[b], 1u) == (unsigned)p.Hkv - 1u) {
            p.seq_ticket[b] = 0u;
            p.out_kv_len[b] = bad ? L : L + 1 + n;
            if (p.out_sel_row) p.out_sel_row[b] = b * p.max_nodes + (!bad && n > 0 ? p.acc_nodes[b * p.T + n - 1] : 0);
        }
    }
}

bool aligned16(const void* a, const void* b) { return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 15) == 0; }

// Checks of the cache's arrays, common to the calls.
bool cache_ok(const void* Kq, const void* Ks, const void* Vq, const void* Vs, int Lcap) {
    return Kq && Ks && Vq && Vs && Lcap >= 1 && aligned16(Kq, Ks) && aligned16(Vq, Vs);
}

RowsQ4 rows_of(const void* Kq, const void* Ks, const void* Vq, const void* Vs) {
    RowsQ4 c;
    c.Kq = static_cast<uint32_t*>(const_cast<void*>(Kq)); c.Ks = static_cast<uint32_t*>(const_cast<void*>(Ks));
    c.Vq = static_cast<uint32_t*>(const_cast<void*>(Vq)); c.Vs = static_cast<uint32_t*>(const_cast<void*>(Vs));
    return c;
}

// CTAs for the rows of one (kv head, sequence): enough for every row at four words a thread, as many as fill the GPU a few
// times over at most.
unsigned row_ctas(const Handle* h, int rows) {
    const long long want = ((long long)rows * (h->cfg.D / 8) + kThreads * 4 - 1) / (kThreads * 4);
    const long long pairs = (long long)h->cfg.B * h->cfg.Hkv;
    const long long most = ((long long)h->num_sms * 32 + pairs - 1) / pairs;
    const long long n = want < most ? want : most;
    return (unsigned)(n < 1 ? 1 : n);
}

// kernel(T, D) for the handle's type and head dimension.
#define CTCSD_Q4_DISPATCH(c, KERNEL, ...)                                                                                  \
    ((c).dtype == CTCSD_DTYPE_BF16 ? ((c).D == 64 ? launch_pdl(KERNEL<__nv_bfloat16, 64>, __VA_ARGS__)                     \
                                                  : launch_pdl(KERNEL<__nv_bfloat16, 128>, __VA_ARGS__))                   \
                                   : ((c).D == 64 ? launch_pdl(KERNEL<float, 64>, __VA_ARGS__) : launch_pdl(KERNEL<float, 128>, __VA_ARGS__)))

}  // namespace
}  // namespace ctcsd

using namespace ctcsd;

extern "C" int ctcsd_store_rows_q4(ctcsd_handle* hh, void* stream, const void* K, const void* V, int Lsrc, const int* n_rows,
                                   const int* at, void* Kq, void* Ks, void* Vq, void* Vs, int Lcap) {
    if (!hh || !K || !V || !n_rows || Lsrc < 1 || !cache_ok(Kq, Ks, Vq, Vs, Lcap) || !aligned16(K, V)) return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    if (c.Hkv > 65535 || c.B > 65535) return CTCSD_ERR_UNSUPPORTED;
    StoreParams p;
    p.K = K; p.V = V; p.c = rows_of(Kq, Ks, Vq, Vs);
    p.n_rows = n_rows; p.at = at; p.Hkv = c.Hkv; p.Lsrc = Lsrc; p.Lcap = Lcap; p.status = status_ptr(h);
    const DeviceGuard on(h->device);
    CTCSD_CUDA_CHECK(h, CTCSD_Q4_DISPATCH(c, store_rows_q4_kernel, dim3(row_ctas(h, Lsrc), c.Hkv, c.B), dim3(kThreads), 0,
                                          static_cast<cudaStream_t>(stream), 1, p));
    h->launches++;
    return CTCSD_OK;
}

extern "C" int ctcsd_load_rows_q4(ctcsd_handle* hh, void* stream, const void* Kq, const void* Ks, const void* Vq, const void* Vs,
                                  int Lcap, const int* first, const int* n_rows, void* out_K, void* out_V, int Lout) {
    if (!hh || !out_K || !out_V || !n_rows || Lout < 1 || !cache_ok(Kq, Ks, Vq, Vs, Lcap) || !aligned16(out_K, out_V)) return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    if (c.Hkv > 65535 || c.B > 65535) return CTCSD_ERR_UNSUPPORTED;
    LoadParams p;
    p.c = rows_of(Kq, Ks, Vq, Vs); p.first = first; p.n_rows = n_rows; p.K = out_K; p.V = out_V;
    p.Hkv = c.Hkv; p.Lcap = Lcap; p.Lout = Lout; p.status = status_ptr(h);
    const DeviceGuard on(h->device);
    CTCSD_CUDA_CHECK(h, CTCSD_Q4_DISPATCH(c, load_rows_q4_kernel, dim3(row_ctas(h, Lout), c.Hkv, c.B), dim3(kThreads), 0,
                                          static_cast<cudaStream_t>(stream), 1, p));
    h->launches++;
    return CTCSD_OK;
}

extern "C" int ctcsd_commit_accepted_q4(ctcsd_handle* hh, void* stream, const void* Kt, const void* Vt, void* Kq, void* Ks, void* Vq,
                                        void* Vs, int Lcap, const int* kv_len, const int* acc_len, const int* acc_nodes,
                                        int* out_kv_len, int* out_sel_row) {
    if (!hh || !Kt || !Vt || !kv_len || !acc_len || !acc_nodes || !out_kv_len || !cache_ok(Kq, Ks, Vq, Vs, Lcap) || !aligned16(Kt, Vt))
        return CTCSD_ERR_INVALID_ARG;
    Handle* h = &hh->h;
    const ctcsd_config& c = h->cfg;
    if (c.B > 65535) return CTCSD_ERR_UNSUPPORTED;
    CommitQ4Params p;
    p.Kt = Kt; p.Vt = Vt; p.c = rows_of(Kq, Ks, Vq, Vs);
    p.kv_len = kv_len; p.acc_len = acc_len; p.acc_nodes = acc_nodes;
    p.Hkv = c.Hkv; p.Lcap = Lcap; p.T = c.T; p.max_nodes = c.max_nodes;
    p.out_kv_len = out_kv_len; p.out_sel_row = out_sel_row;
    p.seq_ticket = reinterpret_cast<unsigned*>(h->ws + h->lay.seq_ticket_off);
    p.status = status_ptr(h);
    const DeviceGuard on(h->device);
    CTCSD_CUDA_CHECK(h, CTCSD_Q4_DISPATCH(c, commit_accepted_q4_kernel, dim3(c.Hkv, c.B), dim3(kThreads), 0,
                                          static_cast<cudaStream_t>(stream), 1, p));
    h->launches++;
    return CTCSD_OK;
}
