// Rows into and out of the pages of a cache (si_store_pages, si_load_pages).
//
//   page, row = table[b, s / page_rows], s % page_rows          of row s of sequence b
//   e    = least exponent with max |x| <= 448 * 2^e over a row, in -64 .. 63
//   code = x / 2^e to the nearest 8-bit value (ties to the even code);  value = code * 2^e
//
// The power of two costs no precision, as the codes have exponents of their own, and makes all steps but the one rounding exact.
// Both kernels are bound by memory.  A wave takes neighbouring rows of one head, so that codes, values and scale bytes of a page go out by
// whole lines where the rows are neighbours.

#include <hip/hip_runtime.h>

#include "dense.h"

namespace si {

namespace {

constexpr int kThreads = 256;

struct Pages {
    void* data[2];            // keys, values
    unsigned char* scales[2];
    const int32_t* table;
    int32_t table_pages, n_pages, page_lg, H;
};

// Row of the pages' arrays that position `at` of sequence b has for head h, -1 where there is none.
__device__ __forceinline__ int64_t row_in_pages(const Pages& p, int b, int64_t at, int h) {
    const int64_t i = at >> p.page_lg;
    if (at < 0 || i >= p.table_pages) return -1;
    const int page = p.table[static_cast<int64_t>(b) * p.table_pages + i];
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.n_pages)) return -1;
    return ((static_cast<int64_t>(page) * p.H + h) << p.page_lg) + (at & ((1 << p.page_lg) - 1));
}

// Sequence and position of packed row n; false where it belongs to none.  Lanes of a wave have ascending n.
__device__ __forceinline__ bool place_of(const Packed& seq, const int32_t* start, int n, int& b, int64_t& at) {
    if (!seq.offsets) {
        const int per = seq.N / seq.B;
        b = n / per;
        at = n - static_cast<int64_t>(b) * per;
    } else {
        b = last_not_above(seq.B, __builtin_amdgcn_readfirstlane(n), [&](int i) { return static_cast<int64_t>(seq.offsets[i]); });
        while (b + 1 < seq.B && seq.offsets[b + 1] <= n) ++b;
        at = static_cast<int64_t>(n) - seq.offsets[b];
        if (at < 0 || n >= seq.offsets[b + 1]) return false;
    }
    at += start ? start[b] : 0;
    return true;
}

// Biased exponent of a row whose largest magnitude has the bf16 bits `top`: with |x| = 1.f * 2^E, the least e with |x| <= 448 * 2^e = 1.75 * 2^(8 + e) is
// E - 8 where the fraction f (7 bits) is at most 0.75, else E - 7; the sum carries into the exponent field exactly then.
__device__ __forceinline__ int row_exponent(int top) {
    return min(max(((top + 0x1F) >> 7) - 8, 127 + kLowestExponent), 127 + kHighestExponent);
}

// Thread: 8 values.  Workgroup: kThreads / (D / 8) rows of one head of the keys or of the values (blockIdx.y: tensor and head).
template <int D, int BITS>
__global__ __launch_bounds__(kThreads) void store_pages_kernel(const uintx4* __restrict__ k_rows, const uintx4* __restrict__ v_rows, Packed seq,
                                                               const int32_t* __restrict__ start, Pages pages) {
    constexpr int kUnits = D / 8;
    const int h = blockIdx.y % pages.H, which = blockIdx.y / pages.H;
    const int piece = threadIdx.x % kUnits;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / kUnits) + threadIdx.x / kUnits;
    const int n = static_cast<int>(min(row, static_cast<int64_t>(seq.N) - 1));
    const uintx4 x = (which ? v_rows : k_rows)[(static_cast<int64_t>(n) * pages.H + h) * kUnits + piece];
    int b;
    int64_t at;
    const bool there = place_of(seq, start, n, b, at) && row < seq.N;
    const int64_t to = there ? row_in_pages(pages, b, at, h) : -1;
    if constexpr (BITS == 16) {
        if (to >= 0) static_cast<uintx4*>(pages.data[which])[to * kUnits + piece] = x;
    } else {
        constexpr int kLargest = ((127 + 8 + kHighestExponent) << 7) | 0x60;  // 448 * 2^63
        int top = 0;
        uintx4 y = x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int lo = x[j] & 0x7FFF, hi = (x[j] >> 16) & 0x7FFF;
            top = max(top, lo > 0x7F80 ? 0 : lo);  // a NaN does not count
            top = max(top, hi > 0x7F80 ? 0 : hi);
            y[j] = (x[j] & 0x80008000u) | (lo > 0x7F80 ? lo : min(lo, kLargest)) | ((hi > 0x7F80 ? hi : min(hi, kLargest)) << 16);
        }
#pragma unroll
        for (int i = 1; i < kUnits; i *= 2) top = max(top, __shfl_xor(top, i));
        if (to < 0) return;
        const int e = row_exponent(top);
        const float power = scale_power(e);
        const bf16x8 v = __builtin_bit_cast(bf16x8, y);
        shortx2 lo = {0, 0}, hi = {0, 0};
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, bf16x2{v[0], v[1]}, power, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, bf16x2{v[2], v[3]}, power, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, bf16x2{v[4], v[5]}, power, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, bf16x2{v[6], v[7]}, power, true);
        static_cast<uintx2*>(pages.data[which])[to * kUnits + piece] = uintx2{__builtin_bit_cast(unsigned, lo), __builtin_bit_cast(unsigned, hi)};
        if (piece == 0) pages.scales[which][to] = static_cast<unsigned char>(e);
    }
}

template <int D, int BITS>
__global__ __launch_bounds__(kThreads) void load_pages_kernel(uintx4* __restrict__ k_rows, uintx4* __restrict__ v_rows, Packed seq,
                                                              const int32_t* __restrict__ start, Pages pages) {
    constexpr int kUnits = D / 8;
    const int h = blockIdx.y % pages.H, which = blockIdx.y / pages.H;
    const int piece = threadIdx.x % kUnits;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / kUnits) + threadIdx.x / kUnits;
    const int n = static_cast<int>(min(row, static_cast<int64_t>(seq.N) - 1));
    uintx4* const rows = which ? v_rows : k_rows;
    int b;
    int64_t at;
    if (!place_of(seq, start, n, b, at) || row >= seq.N || !rows) return;
    const int64_t from = row_in_pages(pages, b, at, h);
    uintx4 x = {0, 0, 0, 0};
    if (from >= 0) {
        if constexpr (BITS == 16) {
            x = static_cast<const uintx4*>(pages.data[which])[from * kUnits + piece];
        } else {
            const uintx2 codes = static_cast<const uintx2*>(pages.data[which])[from * kUnits + piece];
            uintx4 out[2];
            codes_to_bf16(uintx4{codes[0], codes[1], 0, 0}, scale_power(pages.scales[which][from]), out);
            x = out[0];
        }
    }
    rows[(static_cast<int64_t>(n) * pages.H + h) * kUnits + piece] = x;
}

si_status check_rows(const si_paged_cache* cache, int32_t N, const int32_t* offsets, const int32_t* start, const void* k_rows, const void* v_rows) {
    const si_status ok = check_cache(cache);
    if (ok == SI_ERR_INVALID_ARG) return ok;
    if (N < 1 || !aligned4(offsets) || !aligned4(start) || !aligned16(k_rows) || !aligned16(v_rows)) return SI_ERR_INVALID_ARG;
    if (!offsets && N % cache->B != 0) return SI_ERR_INVALID_ARG;
    if (ok != SI_OK) return ok;
    if (static_cast<int64_t>(N) * cache->H_kv * cache->D > (int64_t{1} << 36) || N > (1 << 27)) return SI_ERR_UNSUPPORTED_SHAPE;
    return SI_OK;
}

Pages pages_of(const si_paged_cache& c) {
    int lg = 0;
    while ((1 << lg) < c.page_rows) ++lg;
    return {{c.K, c.V}, {static_cast<unsigned char*>(c.K_scales), static_cast<unsigned char*>(c.V_scales)}, c.table, c.table_pages, c.n_pages, lg, c.H_kv};
}

dim3 grid_for(const si_paged_cache& c, int32_t N, bool values) {
    const int rows = kThreads / (c.D / 8);
    return dim3(static_cast<unsigned>((static_cast<int64_t>(N) + rows - 1) / rows), static_cast<unsigned>(c.H_kv * (values ? 2 : 1)));
}

}  // namespace

}  // namespace si

using namespace si;

extern "C" {

si_status si_store_pages(const void* k_rows, const void* v_rows, int32_t N, const int32_t* offsets, const int32_t* start,
                         const si_paged_cache* cache, void* stream) {
    const si_status ok = check_rows(cache, N, offsets, start, k_rows, v_rows);
    if (ok == SI_ERR_INVALID_ARG) return ok;
    if (!k_rows || (cache->V && !v_rows)) return SI_ERR_INVALID_ARG;
    if (ok != SI_OK) return ok;
    const dim3 grid = grid_for(*cache, N, cache->V != nullptr);
    const Packed seq = {offsets, cache->B, N};
#define SI_LAUNCH(DD, BITS)                                                                                                          \
    hipLaunchKernelGGL((store_pages_kernel<DD, BITS>), grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream),                    \
                       static_cast<const uintx4*>(k_rows), static_cast<const uintx4*>(v_rows), seq, start, pages_of(*cache))
    if (cache->bits == 16) {
        if (cache->D == 128) SI_LAUNCH(128, 16);
        else SI_LAUNCH(64, 16);
    } else {
        if (cache->D == 128) SI_LAUNCH(128, 8);
        else SI_LAUNCH(64, 8);
    }
#undef SI_LAUNCH
    return report(hipGetLastError());
}

si_status si_load_pages(const si_paged_cache* cache, int32_t N, const int32_t* offsets, const int32_t* start, void* k_rows, void* v_rows,
                        void* stream) {
    const si_status ok = check_rows(cache, N, offsets, start, k_rows, v_rows);
    if (ok == SI_ERR_INVALID_ARG) return ok;
    if ((!k_rows && !v_rows) || (v_rows && !cache->V)) return SI_ERR_INVALID_ARG;
    if (ok != SI_OK) return ok;
    const dim3 grid = grid_for(*cache, N, v_rows != nullptr);
    const Packed seq = {offsets, cache->B, N};
#define SI_LAUNCH(DD, BITS)                                                                                                          \
    hipLaunchKernelGGL((load_pages_kernel<DD, BITS>), grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream),                     \
                       static_cast<uintx4*>(k_rows), static_cast<uintx4*>(v_rows), seq, start, pages_of(*cache))
    if (cache->bits == 16) {
        if (cache->D == 128) SI_LAUNCH(128, 16);
        else SI_LAUNCH(64, 16);
    } else {
        if (cache->D == 128) SI_LAUNCH(128, 8);
        else SI_LAUNCH(64, 8);
    }
#undef SI_LAUNCH
    return report(hipGetLastError());
}

}  // extern "C"
