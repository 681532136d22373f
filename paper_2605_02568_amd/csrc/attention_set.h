// What the kernels that attend over TopK(t) U Window(t) have in common: the set as a list in LDS, the swizzle of a tile of
// gathered rows, and the launches' LDS limits.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

namespace si {

constexpr int kTileKeys = 32;        // keys per gathered tile
constexpr float kRescaleSlack = 8.0f;  // log2 units a tile may exceed the reference maximum

// LDS slot (16-byte unit inside the tile) of piece `piece` (8 elements) of tile row `row`.
// Rows are unpadded (2*D bytes); the pieces of a row are XOR-swizzled with a number made of the row's, so that lanes served
// together hit different bank groups.  D = 128: eight consecutive rows get eight different numbers modulo 8 for the row reads of the
// first product (16 bytes from each of 8 rows), and four consecutive rows four that differ above the lowest bit for the transposing
// reads of the second one (two neighbouring pieces from each of 4 rows).  With the row number itself, where rows 2 i and 2 i + 1 share
// two pieces' banks, 16384 queries, k = 512 + 128, 64 heads had 56.6 M conflict cycles instead of 18.9 M; decoding, whose chain
// the reads are part of, took 2 to 4 % longer.  D = 64, two rows to the 64 banks: half the row number (the other form: 289 -> 308 us).
template <int D>
__device__ __forceinline__ int row_swizzle(int row) {
    return D == 128 ? ((row & 3) << 1) | ((row >> 2) & 1) | (row & 8) : (row >> 1) % (D / 8);
}
template <int D>
__device__ __forceinline__ int tile_slot(int row, int piece) {
    return row * (D / 8) + (piece ^ row_swizzle<D>(row));
}

// The value lane (l ^ 32) holds, by v_permlane32_swap instead of an LDS round trip: of the swap's two
// results one carries the low half-wave's values in both halves, the other the high half-wave's;
// each lane picks the one that is not its own.
__device__ __forceinline__ float other_half(float v) {
    const unsigned bits = __builtin_bit_cast(unsigned, v);
    const auto both = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? both[0] : both[1]);
}

// U(t) into s_list: the list's entries in 0 .. rows - 1 that are outside the window (distinct by contract), in list order,
// then the window [w0, legal), padded to whole tiles with key 0; returns their number.  The workgroup's W waves take an
// equal share of the list, up to 512 entries each and round, all requested before the first is used: one trip to
// memory, where one wave taking 64 at a time made k / 64 (16384 queries, k = 512: 495 -> 484 us; without
// the exchange of counts, every wave going through the whole list: 497).  s_kept: W ints.
template <int W>
__device__ __forceinline__ int build_list(const int32_t* __restrict__ row, int k, int rows, int w0, int legal, int* s_list, int* s_kept) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    int n = 0;
    constexpr int kPer = 8;
    const int per = min(kPer, (k + 64 * W - 1) / (64 * W));  // runs of 64 entries a wave takes in a round
    const bool one_run = k <= 64;  // every wave counts it by itself, and wave 0 stores it
    for (int j0 = 0; j0 < k; j0 += W * per * 64) {
        const int first = j0 + (one_run ? 0 : wave * (per * 64)) + lane;
        int s[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < per) s[i] = row[min(first + 64 * i, k - 1)];
        unsigned long long kept[kPer];
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            kept[i] = 0ull;
            if (i < per) kept[i] = __ballot(first + 64 * i < k && static_cast<unsigned>(s[i]) < static_cast<unsigned>(rows) &&
                                           !(s[i] >= w0 && s[i] < legal));
            mine += static_cast<int>(__popcll(kept[i]));
        }
        int pos = n, total = mine;
        if (W > 1 && !one_run) {
            if (j0 > 0) __syncthreads();  // the previous round's counts have been read
            if (lane == 0) s_kept[wave] = mine;
            __syncthreads();
            total = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const int c = s_kept[i];
                pos += i < wave ? c : 0;
                total += c;
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int below = __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(kept[i] >> 32),
                              __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(kept[i]), 0u));
            if (((kept[i] >> lane) & 1) && (!one_run || wave == 0)) s_list[pos + below] = s[i];
            pos += static_cast<int>(__popcll(kept[i]));
        }
        n += total;
    }
    for (int s = w0 + static_cast<int>(threadIdx.x); s < legal; s += 64 * W) s_list[n + (s - w0)] = s;
    n += legal - w0;
    const int padded = (n + kTileKeys - 1) / kTileKeys * kTileKeys;
    for (int j = n + static_cast<int>(threadIdx.x); j < padded; j += 64 * W) s_list[j] = 0;
    return n;
}

inline size_t list_bytes(int k, int n_win) {
    return static_cast<size_t>((k + n_win + kTileKeys - 1) / kTileKeys * kTileKeys) * sizeof(int);
}

// Raises the dynamic LDS limit of a kernel once per device and size (as in the write-out kernel).
template <typename Kernel>
hipError_t allow_lds(Kernel kernel, size_t bytes, std::atomic<size_t>* allowed) {
    if (bytes <= 48 * 1024) return hipSuccess;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const bool tracked = dev >= 0 && dev < 64;
    if (tracked && allowed[dev].load(std::memory_order_acquire) >= bytes) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                            static_cast<int>(bytes));
    if (e == hipSuccess && tracked) {
        size_t seen = allowed[dev].load(std::memory_order_relaxed);
        while (seen < bytes && !allowed[dev].compare_exchange_weak(seen, bytes, std::memory_order_release)) {}
    }
    return e;
}

}  // namespace si
