// What the operators over packed sequences and over pages have in common: which sequence a packed row belongs to, where its rows are, what a
// position sees, and 8-bit values.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_call.h"
#include "si_internal.h"
#include "streamindex_pages.h"

namespace si {

constexpr int kLowestExponent = -64, kHighestExponent = 63;  // of an 8-bit row's power of two

typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef short shortx2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The packed rows of sequences: offsets of sequence b's first row, or equal shares.
struct Packed {
    const int32_t* offsets;  // [B + 1] or NULL
    int32_t B, N;
    __device__ int64_t at(int b) const {  // 0 <= b <= B
        return offsets ? offsets[b] : static_cast<int64_t>(b) * (N / B);
    }
    // the same inside 0 .. N, whatever the offsets hold
    __device__ int in_range(int b) const { return static_cast<int>(min(max(at(b), static_cast<int64_t>(0)), static_cast<int64_t>(N))); }
    // [first, last) rows of sequence b
    __device__ void rows(int b, int& first, int& last) const {
        first = in_range(b);
        last = max(first, in_range(b + 1));
    }
};

// The largest b of 0 .. B - 1 with slot(b) <= u, 0 if there is none; slot does not decrease.  All 64 lanes call it, with the same u: each step
// looks at 64 places at once, so 64 sequences take one trip to memory and 4096 two.
template <typename Slot>
__device__ __forceinline__ int last_not_above(int B, int64_t u, Slot slot) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64;
        const int64_t probe = lo + static_cast<int64_t>(lane) * step;
        const bool below = probe < hi && slot(static_cast<int>(probe)) <= u;
        const int n = max(1, static_cast<int>(__popcll(__ballot(below))));
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Legal rows of position t = first + i among `rows` (Section 4.2), none where t < 0.  t + 1 is below 2^32, as first < 2^31 and i < 2^30.
__device__ __forceinline__ int legal_rows(int first, int i, int rows, int m, int mask_mode) {
    if (mask_mode == SI_MASK_NONE) return rows;
    if (static_cast<int64_t>(first) + i < 0) return 0;
    const uint32_t n = static_cast<uint32_t>(first) + static_cast<uint32_t>(i) + 1u;
    return static_cast<int>(min(m == 1 ? n : n / static_cast<uint32_t>(m), static_cast<uint32_t>(rows)));
}

// 2^e of a scale byte.
__device__ __forceinline__ float scale_power(int byte) { return __uint_as_float(static_cast<unsigned>(byte) << 23); }

// 16 codes of 8 bits as 2 x 8 bf16 values, times a power of two: exact.
__device__ __forceinline__ void codes_to_bf16(uintx4 codes, float power, uintx4 (&out)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const unsigned c = codes[2 * i + j];
            out[i][2 * j] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, power, false));
            out[i][2 * j + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, power, true));
        }
}

// Not 0 where one of 8 bf16 values is not finite: an exponent of ones carries into the bit of the sign.
__device__ __forceinline__ unsigned not_finite(bf16x8 x) {
    const uintx4 v = __builtin_bit_cast(uintx4, x);
    unsigned found = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) found |= (v[w] & 0x7F807F80u) + 0x00800080u;
    return found & 0x80008000u;
}
// The 8 with zeros in their place.
__device__ __forceinline__ bf16x8 finite_or_zero(bf16x8 x) {
    uintx4 v = __builtin_bit_cast(uintx4, x);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if ((v[w] & 0x7F80u) == 0x7F80u) v[w] &= 0xFFFF0000u;
        if ((v[w] & 0x7F800000u) == 0x7F800000u) v[w] &= 0x0000FFFFu;
    }
    return __builtin_bit_cast(bf16x8, v);
}
// Adds w * v[i] to acc for those of 4 neighbouring values that are not finite.
template <typename Acc>
__device__ __forceinline__ void add_not_finite(Acc& acc, int at, bf16x4 v, float w, bool sees) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = static_cast<float>(v[i]);
        acc[at + i] = sees && !(__builtin_fabsf(x) < __builtin_huge_valf()) ? acc[at + i] + w * x : acc[at + i];
    }
}

// ln of l * 2^m_ref, from the sum's mantissa and exponent apart: the logarithm instruction's last place is a part of the mantissa's logarithm only.
__device__ __forceinline__ float log_of(float m_ref, float l) {
    constexpr float kLn2 = 0.6931471805599453f;
    const float e = static_cast<float>(__builtin_amdgcn_frexp_expf(l));
    return __builtin_fmaf(m_ref + e, kLn2, __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l)) * kLn2);
}

inline bool is_power_of_two(int x) { return x > 0 && (x & (x - 1)) == 0; }

// What is wrong with a cache, on the host.
inline si_status check_cache(const si_paged_cache* c) {
    if (!c || !c->K || !c->table) return SI_ERR_INVALID_ARG;
    if (c->B < 1 || c->table_pages < 1 || c->n_pages < 1 || c->page_rows < 1 || c->H_kv < 1 || c->D < 1) return SI_ERR_INVALID_ARG;
    if (!aligned16(c->K) || !aligned16(c->V) || !aligned4(c->table)) return SI_ERR_INVALID_ARG;
    if (c->bits != 16 && c->bits != 8) return SI_ERR_INVALID_ARG;
    if (c->bits == 8 && (!c->K_scales || (c->V && !c->V_scales) || !aligned16(c->K_scales) || !aligned16(c->V_scales))) return SI_ERR_INVALID_ARG;
    if ((c->D != 64 && c->D != 128) || c->page_rows < 16 || c->page_rows > 1024 || !is_power_of_two(c->page_rows)) return SI_ERR_UNSUPPORTED_SHAPE;
    if (c->H_kv > 1024 || c->B > (1 << 20) || static_cast<int64_t>(c->table_pages) * c->page_rows > (1 << 30)) return SI_ERR_UNSUPPORTED_SHAPE;
    return SI_OK;
}

}  // namespace si
