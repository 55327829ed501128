// Blocks of a 4-bit cache on their way into shared memory (the tensor-core attention kernels).
#pragma once

#include "q4_attention.cuh"
#include "tc_primitives.cuh"

namespace ctcsd {

// One side (K or V) of a block of cached rows: levels, then scales and origins.
template <int D> struct RawQ4 {
    static constexpr int kLevels = D / 2, kPairs = D / 8;                    // bytes of a row
    // (D = 64: a row's pairs are 8 bytes and may start 8 bytes behind a 16-byte boundary)
    __host__ __device__ static constexpr int bytes(int keys) { return keys * (kLevels + kPairs) + (D == 64 ? 16 : 0); }
    // Rows row0 .. row0+n-1 (counted over all sequences and heads, of `rows` in the array) whose pairs the engine copies: from a 16-byte
    // boundary to a 16-byte boundary, taking a neighbour's row along where needed; behind the array's last row there is none.
    __device__ static __forceinline__ long long first(long long row0) { return D == 64 ? row0 & ~1ll : row0; }
    __device__ static __forceinline__ long long end(long long row0, int n, long long rows) {
        const long long past = row0 + n;
        if (D == 128 || !(past & 1)) return past;
        return past == rows ? past - 1 : past + 1;
    }
    // The pairs of row 0 of the block, behind levels for `keys` rows.
    __device__ static __forceinline__ const uint32_t* pairs(const unsigned char* dst, int keys, long long row0) {
        return reinterpret_cast<const uint32_t*>(dst + keys * kLevels + (D == 64 && (row0 & 1) ? kPairs : 0));
    }
    // Asks for the block's levels, or its pairs.  One thread each; an arrival on the barrier is part of it.
    __device__ static __forceinline__ void request_levels(unsigned char* dst, const uint32_t* levels, long long row0, int n, uint64_t* bar, uint64_t policy) {
        tc::mbar_arrive_expect_tx(bar, (uint32_t)n * kLevels);
        tc::bulk_load_1d(dst, levels + row0 * (kLevels / 4), (uint32_t)n * kLevels, bar, policy);
    }
    __device__ static __forceinline__ void request_pairs(unsigned char* dst, const uint32_t* so, int keys, long long row0, int n, long long rows,
                                                         uint64_t* bar, uint64_t policy) {
        const long long f = first(row0), e = end(row0, n, rows);
        const uint32_t bytes = e > f ? (uint32_t)(e - f) * kPairs : 0u;
        tc::mbar_expect_tx(bar, bytes);
        if (bytes) tc::bulk_load_1d(dst + keys * kLevels, so + f * (kPairs / 4), bytes, bar, policy);
        if (D == 64 && e < row0 + n) {                                       // the array's last row, which stands alone
            const uint2 w = *reinterpret_cast<const uint2*>(so + e * (kPairs / 4));
            *reinterpret_cast<uint2*>(dst + keys * kLevels + (e - f) * kPairs) = w;
            tc::fence_proxy_async();                                         // (the engine writes there again)
        }
        tc::mbar_arrive(bar);
    }
};

}  // namespace ctcsd
