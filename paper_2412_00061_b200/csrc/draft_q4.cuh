// What the two kernels of the draft head over 4-bit weights share: the packed layout, and the merge of running states.
#pragma once

#include "q4.cuh"
#include "run_state.cuh"

#include <limits.h>
#include <math.h>

namespace ctcsd {

constexpr int kQ4Panel = 16;             // classes of a panel
constexpr int kQ4Block = 128;            // hidden elements of a block

__host__ __device__ inline int q4_block_bytes(int group) { return 1024 + kQ4Panel * 4 * (kQ4Block / group); }

struct DraftQ4Params {
    const void* x;                       // [x_row_count,H]
    const int* x_rows;                   // [M] or null
    int x_row_count;
    const unsigned char* W;              // packed
    const int* row_seq;
    const float* blank_bias;
    int m0, mcount, rows;                // rows of this pass, rows of the call
    int H, classes, panels, blocks, group;   // panels per draft slot, blocks per panel
    int slots;                           // draft slots (T)
    int piece, nring;                    // blocks of a ring slot, ring slots
    DraftPartial* part;                  // [rows of a pass][grid][2]
    long long part_room;                 // states that the workspace has room for
    unsigned* counter;                   // [draft slots], zero between calls
    int k;
    int* out_topk_id;
    float* out_topk_lp;
    float* out_lse;
    float* logits_dbg;
    int* status;
};

#ifdef __CUDACC__

// Unsigned numbers in the order of the floats; 0 for an entry that is not there.
__device__ __forceinline__ uint32_t rank_of(float v, int id) {
    if (id == INT_MAX) return 0u;
    const uint32_t u = __float_as_uint(v);
    return (u >> 31) ? ~u : u | 0x80000000u;
}
// Combines the states of the lanes that differ in the bits of `over` (31: all of the warp; 7: the eight with the same lane / 8): maximum, sum, and
// the k best (ties to the lower id) in each of them.
template <int over> __device__ __forceinline__ void combine_best(RunState& st, int k) {
    float gmx = st.mx;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (over & o) gmx = fmaxf(gmx, __shfl_xor_sync(0xffffffffu, gmx, o));
    st.sum = st.mx == -INFINITY ? 0.f : st.sum * __expf(st.mx - gmx);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (over & o) st.sum += __shfl_xor_sync(0xffffffffu, st.sum, o);
    st.mx = gmx;
    float ov[kTopSlots];
    int oi[kTopSlots];
#pragma unroll
    for (int r = 0; r < kTopSlots; ++r) {
        ov[r] = -INFINITY;
        oi[r] = INT_MAX;
        if (r < k) {
            const uint32_t mine = rank_of(st.val[0], st.id[0]);
            uint32_t top = mine;
            unsigned id;
            if constexpr (over == 31) {
                top = __reduce_max_sync(0xffffffffu, mine);
                id = __reduce_min_sync(0xffffffffu, mine == top ? (unsigned)st.id[0] : 0x7fffffffu);
            } else {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
                    if (over & o) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                id = mine == top ? (unsigned)st.id[0] : 0x7fffffffu;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
                    if (over & o) id = min(id, __shfl_xor_sync(0xffffffffu, id, o));
            }
            oi[r] = (int)id;
            if (top != 0u) ov[r] = __uint_as_float((top >> 31) ? top & 0x7fffffffu : ~top);
            if ((unsigned)st.id[0] == id && id != 0x7fffffffu) {              // (an id stands in one lane's list only)
#pragma unroll
                for (int q = 0; q < kTopSlots - 1; ++q) { st.val[q] = st.val[q + 1]; st.id[q] = st.id[q + 1]; }
                st.val[kTopSlots - 1] = -INFINITY;
                st.id[kTopSlots - 1] = INT_MAX;
            }
        }
    }
#pragma unroll
    for (int q = 0; q < kTopSlots; ++q) { st.val[q] = ov[q]; st.id[q] = oi[q]; }
}


// The end of a pass.  The line of units (panels or tiles, `per_slot` of them in each draft slot) is divided evenly among the CTAs in order, so the CTAs whose
// units touch a draft slot are neighbours; a CTA touches two slots at most and leaves a state for each (p.part).  Called by the whole
// block when its states are written: for each of its slots, the CTA that ends last merges the states and writes the outputs.
// `merge`: two ints in shared memory.
__device__ inline void draft_q4_finish(const DraftQ4Params& p, int per_slot, int slot0, int segs, int* merge) {
    const long long n = gridDim.x, total = (long long)per_slot * p.slots;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    __threadfence();
    __syncthreads();
    auto first_cta = [&](int slot) -> int {                                  // the first whose units reach beyond the slot's first
        const long long lo = (long long)slot * per_slot;
        long long c = lo * n / total;
        while (c > 0 && total * c / n > lo) --c;
        while (total * (c + 1) / n <= lo) ++c;
        return (int)c;
    };
    auto last_cta = [&](int slot) -> int {                                   // the last whose units begin before the slot's end
        const long long hi = (long long)(slot + 1) * per_slot;
        long long c = hi * n / total;
        if (c > n - 1) c = n - 1;
        while (total * c / n >= hi) --c;
        while (c < n - 1 && total * (c + 1) / n < hi) ++c;
        return (int)c;
    };
    if (tid < segs) {
        const int slot = slot0 + tid, touch = last_cta(slot) - first_cta(slot) + 1;
        const bool mine = atomicAdd(p.counter + slot, 1u) == (unsigned)touch - 1u;
        if (mine) p.counter[slot] = 0u;
        merge[tid] = mine ? 1 : 0;
    }
    __syncthreads();
    __threadfence();
    for (int seg = 0; seg < segs; ++seg) {
        if (!merge[seg]) continue;
        const int slot = slot0 + seg, c0 = first_cta(slot), c1 = last_cta(slot);
        for (int m = warp; m < p.mcount; m += warps) {
            RunState fs;
            fs.init();
            for (int c = c0 + lane; c <= c1; c += 32) {
                const int which = slot - (int)(total * c / n / per_slot);                  // the slot is the CTA's first or second
                fs.absorb(load_partial_cg(p.part + ((size_t)m * n + c) * 2 + which));
            }
            combine_best<31>(fs, p.k);
            if (lane == 0) {
                const int row = p.m0 + m;
                const float lse = fs.mx + logf(fs.sum);
                if (CTCSD_IN_BOUNDS(p.status, 161, (long long)row * p.slots + slot, (long long)p.rows * p.slots)) p.out_lse[(size_t)row * p.slots + slot] = lse;
#pragma unroll
                for (int j = 0; j < kTopSlots; ++j)
                    if (j < p.k) {
                        const size_t o = ((size_t)row * p.slots + slot) * p.k + j;
                        if (!CTCSD_IN_BOUNDS(p.status, 162, o, (long long)p.rows * p.slots * p.k)) continue;
                        p.out_topk_id[o] = fs.id[j];
                        p.out_topk_lp[o] = fs.val[j] - lse;
                    }
            }
        }
    }
}

#endif  // __CUDACC__

// bf16, up to kDraftQ4TcRows activation rows in a pass, on tcgen05 / tensor memory.
constexpr int kDraftQ4TcRows = 128;
constexpr int kDraftQ4TcStates = 4;      // states of a row that a CTA keeps for a while (one of each warp that reads sums)
int launch_draft_q4_tc(Handle* h, cudaStream_t s, DraftQ4Params p);

}  // namespace ctcsd
