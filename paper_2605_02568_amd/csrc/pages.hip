// Rows into and out of the pages of a cache (si_store_pages, si_load_pages).
//
//   page, row = table[b, s / page_rows], s % page_rows          of row s of sequence b
//   e    = least exponent with max |x| <= 448 * 2^e over a row, in -64 .. 63
//   code = x / 2^e to the nearest 8-bit value (ties to the even code);  value = code * 2^e
//
// The power of two costs no precision, as the codes have exponents of their own, and makes all steps but the one rounding exact.
// Both kernels are bound by memory: 33,047 rows of 8 heads of 128, keys and values, 204 MB, into 8 bits in 45 us and back in 32; 65,536 rows out of pages of 16 bits,
// 537 MB, in 103 (5.2 TB/s; a copy of 2 GiB runs at 4.9).  A wave takes neighbouring rows of one head, so that codes, values and scale bytes of a page go out by
// whole lines where the rows are neighbours.

#include <hip/hip_runtime.h>

#include "dense.h"

namespace si {

namespace {

constexpr int kThreads = 256;
constexpr int kMostBlocks = 1 << 15;  // of a grid's second axis

struct Pages {
    void* data[2];            // keys, values
    unsigned char* scales[2];
    const int32_t* table;
    int32_t table_pages, n_pages, page_lg, H;
};

template <bool ONCE, typename T>
__device__ __forceinline__ T read(const T* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}

// Row of the pages' arrays that position `at` of sequence b has for head h, -1 where there is none.
__device__ __forceinline__ int64_t row_in_pages(const Pages& p, int b, int64_t at, int h) {
    const int64_t i = at >> p.page_lg;
    if (at < 0 || i >= p.table_pages) return -1;
    const int page = p.table[static_cast<int64_t>(b) * p.table_pages + i];
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.n_pages)) return -1;
    return ((static_cast<int64_t>(page) * p.H + h) << p.page_lg) + (at & ((1 << p.page_lg) - 1));
}

// Sequences and positions of packed rows n[0], n[1], .. of each lane; b = -1 where a row belongs to none.  first and last are the wave's first and last row.
template <int PER>
__device__ __forceinline__ void places_of(const Packed& seq, const int32_t* start, int first, int last, const int (&n)[PER], int (&b)[PER], int64_t (&at)[PER]) {
    if (!seq.offsets) {
        const int per = seq.N / seq.B;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            b[j] = n[j] / per;
            at[j] = n[j] - static_cast<int64_t>(b[j]) * per + (start ? start[b[j]] : 0);
        }
        return;
    }
    const int b0 = last_not_above(seq.B, first, [&](int i) { return static_cast<int64_t>(seq.offsets[i]); });
    const int from = seq.offsets[b0], to = seq.offsets[b0 + 1];
    if (from <= first && last < to) {  // all of the same sequence, as nearly all waves are
        const int64_t shift = static_cast<int64_t>(start ? start[b0] : 0) - from;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            b[j] = b0;
            at[j] = n[j] + shift;
        }
        return;
    }
    // of several: the offsets behind b0's come 64 at a time, a lane each, and all rows are compared with one after the other
    const int lane = threadIdx.x & 63;
    int mine_from[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        b[j] = b0;
        mine_from[j] = from;
    }
    for (int i0 = b0 + 1, n_below = 64; n_below == 64; i0 += 64) {
        const int offset = i0 + lane < seq.B ? seq.offsets[i0 + lane] : 0x7FFFFFFF;
        n_below = static_cast<int>(__popcll(__ballot(offset <= last)));
        for (int i = 0; i < n_below; ++i) {
            const int o = __builtin_amdgcn_readlane(offset, i);
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                mine_from[j] = o <= n[j] ? o : mine_from[j];
                b[j] = o <= n[j] ? i0 + i : b[j];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int mine_to = seq.offsets[b[j] + 1], mine_start = start ? start[b[j]] : 0;
        at[j] = static_cast<int64_t>(n[j]) - mine_from[j] + mine_start;
        if (n[j] < mine_from[j] || n[j] >= mine_to) b[j] = -1;
    }
}

// Biased exponent of a row whose largest magnitude has the bf16 bits `top`: with |x| = 1.f * 2^E, the least e with |x| <= 448 * 2^e = 1.75 * 2^(8 + e) is
// E - 8 where the fraction f (7 bits) is at most 0.75, else E - 7; the sum carries into the exponent field exactly then.
__device__ __forceinline__ int row_exponent(int top) {
    return min(max(((top + 0x1F) >> 7) - 8, 127 + kLowestExponent), 127 + kHighestExponent);
}

// A thread takes 8 values of PER rows, a wave PER * 64 / (D / 8) rows in a row of one head of the keys or of the values.  Tensor and head are the grid's first
// axis, so that a packed row's heads are read and written at about the same time (the other way round 2 % slower).  Many rows
// take 4: enough on its way to make up for the trips to the offsets and the table before it (16 prompts of 33,000 rows of 8 heads, 8 bits: in 72 -> 58 us, out
// 47 -> 33).  Where that would be less than a wave a SIMD, 1: a wave's rows are then of fewer sequences (one row of each of 64: 6.5 -> 3.6 us).
template <int D, int PER>
struct Share {
    static constexpr int kUnits = D / 8;             // threads of a row
    static constexpr int kStep = 64 / kUnits;        // rows of a wave's load
    static constexpr int kWaveRows = PER * kStep;
    static constexpr int kRows = kThreads / 64 * kWaveRows;
    int piece, h, which, first, last;
    int n[PER], b[PER];
    int64_t at[PER];
    bool there[PER];  // such a row is in the call
    __device__ __forceinline__ Share(const Packed& seq, int H) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        which = blockIdx.x >= static_cast<unsigned>(H);
        h = static_cast<int>(blockIdx.x) - which * H;
        piece = lane % kUnits;
        const int64_t row = (static_cast<int64_t>(blockIdx.z) * kMostBlocks + blockIdx.y) * kRows + wave * kWaveRows;
        first = static_cast<int>(min(row, static_cast<int64_t>(seq.N) - 1));
        last = static_cast<int>(min(row + kWaveRows, static_cast<int64_t>(seq.N)) - 1);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            n[j] = min(first + j * kStep + lane / kUnits, seq.N - 1);
            there[j] = row + j * kStep + lane / kUnits < seq.N;
        }
    }
};

template <int D, int BITS, int kPer, bool kOnce>
__global__ __launch_bounds__(kThreads) void store_pages_kernel(const uintx4* __restrict__ k_rows, const uintx4* __restrict__ v_rows, Packed seq,
                                                               const int32_t* __restrict__ start, Pages pages) {
    constexpr int kUnits = D / 8;
    Share<D, kPer> s(seq, pages.H);
    const uintx4* const rows = (s.which ? v_rows : k_rows) + static_cast<int64_t>(s.h) * kUnits + s.piece;
    uintx4 x[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[j] = read<kOnce>(rows + static_cast<int64_t>(s.n[j]) * pages.H * kUnits);
    places_of(seq, start, s.first, s.last, s.n, s.b, s.at);
    int64_t to[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) to[j] = s.there[j] && s.b[j] >= 0 ? row_in_pages(pages, s.b[j], s.at[j], s.h) : -1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if constexpr (BITS == 16) {
            if (to[i] >= 0) static_cast<uintx4*>(pages.data[s.which])[to[i] * kUnits + s.piece] = x[i];
        } else {
            constexpr int kLargest = ((127 + 8 + kHighestExponent) << 7) | 0x60;  // 448 * 2^63
            int top = 0;
            uintx4 y = x[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int lo = y[j] & 0x7FFF, hi = (y[j] >> 16) & 0x7FFF;
                top = max(top, lo > 0x7F80 ? 0 : lo);  // a NaN does not count
                top = max(top, hi > 0x7F80 ? 0 : hi);
                y[j] = (y[j] & 0x80008000u) | (lo > 0x7F80 ? lo : min(lo, kLargest)) | ((hi > 0x7F80 ? hi : min(hi, kLargest)) << 16);
            }
#pragma unroll
            for (int j = 1; j < kUnits; j *= 2) top = max(top, __shfl_xor(top, j));
            if (to[i] < 0) continue;
            const int e = row_exponent(top);
            const float power = scale_power(e);
            const bf16x8 v = __builtin_bit_cast(bf16x8, y);
            shortx2 lo = {0, 0}, hi = {0, 0};
            lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, bf16x2{v[0], v[1]}, power, false);
            lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, bf16x2{v[2], v[3]}, power, true);
            hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, bf16x2{v[4], v[5]}, power, false);
            hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, bf16x2{v[6], v[7]}, power, true);
            static_cast<uintx2*>(pages.data[s.which])[to[i] * kUnits + s.piece] = uintx2{__builtin_bit_cast(unsigned, lo), __builtin_bit_cast(unsigned, hi)};
            if (s.piece == 0) pages.scales[s.which][to[i]] = static_cast<unsigned char>(e);
        }
    }
}

template <int D, int BITS, int kPer, bool kOnce>
__global__ __launch_bounds__(kThreads) void load_pages_kernel(uintx4* __restrict__ k_rows, uintx4* __restrict__ v_rows, Packed seq,
                                                              const int32_t* __restrict__ start, Pages pages) {
    constexpr int kUnits = D / 8;
    Share<D, kPer> s(seq, pages.H);
    uintx4* const rows = s.which ? v_rows : k_rows;
    if (!rows) return;
    places_of(seq, start, s.first, s.last, s.n, s.b, s.at);
    uintx4 x[kPer];
    unsigned power[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int64_t from = s.b[j] >= 0 ? row_in_pages(pages, s.b[j], s.at[j], s.h) : -1;
        x[j] = uintx4{0, 0, 0, 0};
        power[j] = 127;
        if (from >= 0) {
            if constexpr (BITS == 16) {
                x[j] = read<kOnce>(static_cast<const uintx4*>(pages.data[s.which]) + from * kUnits + s.piece);
            } else {
                const uintx2 codes = read<kOnce>(static_cast<const uintx2*>(pages.data[s.which]) + from * kUnits + s.piece);
                x[j] = uintx4{codes[0], codes[1], 0, 0};
                power[j] = pages.scales[s.which][from];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if constexpr (BITS == 8) {
            uintx4 out[2];
            codes_to_bf16(x[j], scale_power(power[j]), out);
            x[j] = out[0];
        }
        if (s.there[j] && s.b[j] >= 0) {
            uintx4* const to = rows + (static_cast<int64_t>(s.n[j]) * pages.H + s.h) * kUnits + s.piece;
            if constexpr (kOnce) __builtin_nontemporal_store(x[j], to);
            else *to = x[j];
        }
    }
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

// Rows a thread takes, and the grid of it.
int rows_a_thread(const si_paged_cache& c, int32_t N, bool values) {
    constexpr int kSimds = 1024;
    return static_cast<int64_t>(N) * c.H_kv * (values ? 2 : 1) * (c.D / 8) >= int64_t{4} * 64 * kSimds ? 4 : 1;
}
// Whether what a call reads once goes past the caches, as do the packed rows that it makes: out of the way of what it and the next call read again (16 prompts of
// 33,000 rows of 8 heads in 8 bits, 135 MB of packed rows, in and out: 89 -> 80 us; 65,536 rows of 16 bits out: 113 -> 106).  Packed rows of less than 64 MB may well
// be in the caches, or the next call finds them there (9,219 rows of 5 heads of 64 out of 8 bits, again and again: 7.9 us, past the caches 9.6).
bool past_the_caches(const si_paged_cache& c, int32_t N, bool values) {
    return static_cast<int64_t>(N) * c.H_kv * c.D * (values ? 4 : 2) >= int64_t{64} << 20;
}
dim3 grid_for(const si_paged_cache& c, int32_t N, bool values) {
    const int rows = kThreads / (c.D / 8) * rows_a_thread(c, N, values);
    const int64_t blocks = (static_cast<int64_t>(N) + rows - 1) / rows;
    return dim3(static_cast<unsigned>(c.H_kv * (values ? 2 : 1)), static_cast<unsigned>(std::min<int64_t>(blocks, kMostBlocks)),
                static_cast<unsigned>((blocks + kMostBlocks - 1) / kMostBlocks));
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
    const int per = rows_a_thread(*cache, N, cache->V != nullptr);
    const bool once = past_the_caches(*cache, N, cache->V != nullptr);
    const dim3 grid = grid_for(*cache, N, cache->V != nullptr);
    const Packed seq = {offsets, cache->B, N};
#define SI_LAUNCH(DD, BITS)                                                                                                          \
    if (once) SI_LAUNCH_PER(DD, BITS, 4, true);                                                                                      \
    else if (per == 4) SI_LAUNCH_PER(DD, BITS, 4, false);                                                                            \
    else SI_LAUNCH_PER(DD, BITS, 1, false)
#define SI_LAUNCH_PER(DD, BITS, PER, ONCE)                                                                                              \
    hipLaunchKernelGGL((store_pages_kernel<DD, BITS, PER, ONCE>), grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream),                    \
                       static_cast<const uintx4*>(k_rows), static_cast<const uintx4*>(v_rows), seq, start, pages_of(*cache))
    if (cache->bits == 16) {
        if (cache->D == 128) {
            SI_LAUNCH(128, 16);
        } else {
            SI_LAUNCH(64, 16);
        }
    } else {
        if (cache->D == 128) {
            SI_LAUNCH(128, 8);
        } else {
            SI_LAUNCH(64, 8);
        }
    }
#undef SI_LAUNCH
#undef SI_LAUNCH_PER
    return report(hipGetLastError());
}

si_status si_load_pages(const si_paged_cache* cache, int32_t N, const int32_t* offsets, const int32_t* start, void* k_rows, void* v_rows,
                        void* stream) {
    const si_status ok = check_rows(cache, N, offsets, start, k_rows, v_rows);
    if (ok == SI_ERR_INVALID_ARG) return ok;
    if ((!k_rows && !v_rows) || (v_rows && !cache->V)) return SI_ERR_INVALID_ARG;
    if (ok != SI_OK) return ok;
    const int per = rows_a_thread(*cache, N, v_rows != nullptr);
    const bool once = past_the_caches(*cache, N, v_rows != nullptr);
    const dim3 grid = grid_for(*cache, N, v_rows != nullptr);
    const Packed seq = {offsets, cache->B, N};
#define SI_LAUNCH(DD, BITS)                                                                                                          \
    if (once) SI_LAUNCH_PER(DD, BITS, 4, true);                                                                                      \
    else if (per == 4) SI_LAUNCH_PER(DD, BITS, 4, false);                                                                            \
    else SI_LAUNCH_PER(DD, BITS, 1, false)
#define SI_LAUNCH_PER(DD, BITS, PER, ONCE)                                                                                              \
    hipLaunchKernelGGL((load_pages_kernel<DD, BITS, PER, ONCE>), grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream),                     \
                       static_cast<uintx4*>(k_rows), static_cast<uintx4*>(v_rows), seq, start, pages_of(*cache))
    if (cache->bits == 16) {
        if (cache->D == 128) {
            SI_LAUNCH(128, 16);
        } else {
            SI_LAUNCH(64, 16);
        }
    } else {
        if (cache->D == 128) {
            SI_LAUNCH(128, 8);
        } else {
            SI_LAUNCH(64, 8);
        }
    }
#undef SI_LAUNCH
#undef SI_LAUNCH_PER
    return report(hipGetLastError());
}

}  // extern "C"
