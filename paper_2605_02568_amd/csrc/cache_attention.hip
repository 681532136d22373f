// Attention over TopK(t) U Window(t) where the cache is held in 4 bits (si_quantized_attention), and what the cache's rows
// receive of its softmax (si_accumulate_weights):
//
//   out[t,h,:]   = sum_{s in U(t)} p_s V[s,:],   p = softmax_{s in U(t)}( scale * <qa[t,h,:], V[s,:]> )
//   lse[t,h]     = ln sum_{s in U(t)} exp( scale * <qa[t,h,:], V[s,:]> )
//   weights[s]  += sum_{t,h} exp( scale * <qa[t,h,:], V[s,:]> - lse[t,h] )
//
// V[s, 32 j + i] = code * 2^e(s, j).  Codes times their power are exact in fp16 (exponents -13 .. 13), and so are the queries once a
// head is scaled by a power of two, which goes into the softmax scale; heads whose values lie too far apart for that are multiplied in bf16.  So the
// first product is that of the bf16 operands, and the second one takes the weights in two fp16 parts, up to 22 mantissa bits, at the cost that two
// bf16 parts with 16 bits would have.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "attention_set.h"
#include "cache_call.h"
#include "si_internal.h"
#include "streamindex_cache.h"
#include "wave_ops.h"

namespace si {

namespace {

typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef __fp16 fp16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned short shortx2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eRest = 1.925962989e-8f;  // log2(e) - kLog2e: left out of an lse of 7, 9e-8 too much for every row alike
constexpr float kLn2 = 0.6931471805599453f;
// The weights are 2^7 times exp2(x - reference): at most 2^15 with the slack of 2^8.  The first fp16 part is a normal number down to 2^-21 of the
// reference's weight; the second one, whose step is 2^-24 at least, adds 11 bits to it down to 2^-9, and below that leaves a weight off by up to 2^-25
// as it is held, 2^-32 of the reference's.
constexpr float kWeightShift = 7.0f;

// Between what some lanes of a wave write to LDS and others of it read there: the hardware does a wave's LDS accesses in order, and this keeps
// the compiler to that order.  No instruction comes of it.
__device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); }

__device__ __forceinline__ float power_of(unsigned scale_byte) { return __uint_as_float(scale_byte << 23); }

// Rows that batch b holds, and legal rows of query t.
__device__ __forceinline__ int held_rows(const int32_t* __restrict__ lengths, int b, int T) {
    return lengths ? min(max(lengths[b], 0), T) : T;
}

// ln(l * 2^(m_ref - 7)).  The logarithm instruction gets the mantissa alone: of l itself, whose logarithm is up to 20, its last place is 2e-6, and it
// was off by -0.2 of that on the average, which all weights that are then made of lse share.
__device__ __forceinline__ float log_sum(float m_ref, float l) {
    const float e = static_cast<float>(__builtin_amdgcn_frexp_expf(l)) - kWeightShift;
    return __builtin_fmaf(m_ref + e, kLn2, __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l)) * kLn2);
}

// The product of a query and a row where the query's bf16 values enter as they are, which may be anything bf16 holds: to_log2 * <q, 2^exponent V> is
// the logit in log2 units.  V is below 2^16 and D 2^7 at most, so exponent -27 keeps every sum below 2^124, and where |scale| is below 1 what fp32
// then loses at its lower end is nothing to the logit.  With larger scales a sum that fp32 cannot hold is of a logit it cannot hold either, and from 2^32
// on, where the lower end matters, the rows are 2^27 times as large.  A scale of 0 is one of 2^-126 on rows 2^-64 times as large, whose logits are
// below 2^-38: not 0, so that -inf times it is -inf.  It costs nothing: the exponent is added to a row's scale byte as that is shifted.
struct BareProduct {
    float to_log2;
    int exponent;
};

// A lane's part of a query's head, 8 bf16 values an element, as the products take it: fp16, times a power of two that brings the head's
// largest magnitude into [2^14, 2^15), with the sign of the softmax scale; values of exponents down to 31 below the largest one's stay exact.  The
// factor |scale| log2(e) over that power takes a product of these operands to the log2 domain.  A block of heads one of which holds smaller values
// too, or needs a factor that fp32 does not hold, takes the bare product instead, at twice the conversions (all heads of 16384 queries of 640 rows
// 471 -> 665 us, of 32 queries of 1152 9.6 -> 16.6): rows of zeros where the query's large values are would leave logits that consist of what fp16 lost.

// Magnitudes of a head's values, as bf16's bits: in the low half the largest, in the high half 2^16 less the smallest that is not 0 (or 0).  Of two
// parts: the larger of each half.
__device__ __forceinline__ unsigned joint(unsigned a, unsigned b) {
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(shortx2, a), __builtin_bit_cast(shortx2, b)));
}
template <int N>
__device__ __forceinline__ unsigned extent(const uintx4 (&raw)[N]) {
    shortx2 top = {0, 0}, low = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const shortx2 size = __builtin_bit_cast(shortx2, raw[i][j] & 0x7FFF7FFFu);
            top = __builtin_elementwise_max(top, size);
            low = __builtin_elementwise_max(low, static_cast<shortx2>(shortx2{0, 0} - size));
        }
    return static_cast<unsigned>(max(top[0], top[1])) | (static_cast<unsigned>(max(low[0], low[1])) << 16);
}
// The power, in to_log2 that factor, and in border the bits below which a value (but 0) is too small for fp16; denormal numbers have the least exponent's
// steps.  A head that is not finite has NaN whatever the power, and makes no demands: other heads' bits do not depend on it.
__device__ __forceinline__ float query_power(unsigned top, float scale_log2e, float& to_log2, unsigned& border) {
    const int e = top < 0x7F80u ? static_cast<int>(top >> 7) : 0;  // exponent field of the largest
    const int up = min(268 - e, 254);                              // field of the power: 2^(14 - (e - 127))
    // not 0, so that -inf times it is -inf: a logit that such a factor makes is 0 either way
    to_log2 = fmaxf(__builtin_ldexpf(__builtin_fabsf(scale_log2e), 127 - up), 1.1754944e-38f);
    border = static_cast<unsigned>(max(e - 31, 0)) << 7;
    border = max(border, 1u);
    return __uint_as_float(static_cast<unsigned>(up) << 23) * (scale_log2e < 0.0f ? -1.0f : 1.0f);
}
// Whether a block has a head that needs the bare product: `lost` where a lane has values below a head's border.
__device__ __forceinline__ bool needs_bare(bool lost, float to_log2) { return __ballot(lost | (to_log2 == __builtin_huge_valf())) != 0ull; }
template <int N>
__device__ __forceinline__ void scale_query(const uintx4 (&raw)[N], float power, halfx8 (&qf)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float lo = __uint_as_float(raw[i][j] << 16) * power;
            const float hi = __uint_as_float(raw[i][j] & 0xFFFF0000u) * power;
            const halfx2 pair = __builtin_convertvector(floatx2{lo, hi}, halfx2);
            qf[i][2 * j] = pair[0];
            qf[i][2 * j + 1] = pair[1];
        }
}

// Weights as two fp16 parts, p = hi + lo, each rounded to nearest.  The remainder is an fma that takes hi as it is and rounds to fp16 at once:
// three instructions a pair of weights (the factor 1 comes from a register, as the compiler would otherwise convert hi, subtract and convert).
__device__ __forceinline__ void split_weights(const float (&p)[16], halfx8 (&hi)[2], halfx8 (&lo)[2]) {
    float one = 1.0f;
    asm("" : "+s"(one));
#pragma unroll
    for (int jj = 0; jj < 8; ++jj) {
        const float p0 = p[2 * jj], p1 = p[2 * jj + 1];
        const halfx2 a = __builtin_convertvector(floatx2{p0, p1}, halfx2);
        hi[jj >> 2][2 * (jj & 3)] = a[0];
        hi[jj >> 2][2 * (jj & 3) + 1] = a[1];
        lo[jj >> 2][2 * (jj & 3)] = static_cast<_Float16>(__builtin_fmaf(-static_cast<float>(a[0]), one, p0));
        lo[jj >> 2][2 * (jj & 3) + 1] = static_cast<_Float16>(__builtin_fmaf(-static_cast<float>(a[1]), one, p1));
    }
}

// Weights of a tile's rows for one head, 2^7 exp2(x - m_ref) with x = to_log2 * s, and their sum over this half-wave's rows; `live`: bit r says whether
// row r of the tile counts.  m_ref is some earlier tile's maximum.  Whether it still does is read off the sum, which is needed anyway: only where a
// head's weights exceed 2^15 in sum (m_ref too low, or still -inf) the tile's maximum is taken, m_ref raised to it, and what was
// accumulated brought down: raise(alpha).  Every tile's maximum and its exchange between the half-waves would cost 13 instructions and
// the wait for them before the first exponential.
template <typename Raise>
__device__ __forceinline__ float weigh(floatx16& s, float to_log2, unsigned live, int half, float& m_ref, float (&p)[16], Raise raise) {
    if (live != 0xFFFFFFFFu) {  // the last tile, or one with pads: their weights become 0 (to_log2 is never 0)
        float low = -__builtin_huge_valf();
        asm volatile("" : "+v"(low));  // keeps this block a branch instead of 16 selects per tile
        const unsigned mine = live >> (4 * half);
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (!((mine >> (8 * (j >> 2) + (j & 3))) & 1)) s[j] = low;
    }
    float sum;
    auto exponentials = [&]() {
        const float shift = kWeightShift - m_ref;
#pragma unroll
        for (int j = 0; j < 16; ++j) p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j], to_log2, shift));
        sum = p[0] + p[1];
#pragma unroll
        for (int j = 2; j < 16; ++j) sum += p[j];
    };
    exponentials();
    const bool over = !(sum <= 32768.0f);  // also where the first tile's rows that do not count gave inf - inf
    if (__ballot(over) != 0ull) {
        float top = s[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) top = fmaxf(top, s[j]);
        top *= to_log2;
        top = fmaxf(top, other_half(top));  // of the head: both half-waves decide alike
        const float theirs = other_half(over ? 1.0f : 0.0f);  // outside of the condition below: every lane takes part in the exchange
        const bool up = over || theirs != 0.0f;
        const float m_new = up ? fmaxf(top, m_ref) : m_ref;
        raise(__builtin_amdgcn_exp2f(m_ref - m_new));  // 1 where nothing changes, 0 on the first tile
        m_ref = m_new;
        exponentials();
    }
    return sum;
}

// U(t) in tiles of 32 rows as they stand: the list's, then the window's; a lane knows its own row of a tile (row = lane % 32).
struct Tiles {
    const int32_t* list;
    int k, last, held, w0, legal, list_tiles;
    // What the list has at this lane's place of tile `tile` (of the window's tiles: of its last one).  On its own, and without a branch, so that a
    // loop can ask for a tile's entries well before it needs them: judged at once they would be waited for at once.
    __device__ __forceinline__ int entry(int tile, int col) const { return list[min(tile * kTileKeys + col, last)]; }
    // The row that this lane has of tile `tile`, with what entry() gave; -1 where U(t) has none there: a pad, an entry that the window has, the
    // end of either.
    __device__ __forceinline__ int row(int entry, int tile, int col) const {
        const bool listed = (tile * kTileKeys + col < k) & (static_cast<unsigned>(entry) < static_cast<unsigned>(held)) & !((entry >= w0) & (entry < legal));
        const int in_window = w0 + (tile - list_tiles) * kTileKeys + col;
        const int from_list = (tile - list_tiles) >> 31;  // all bits or none: a choice by a branch would cut the loop's body in pieces
        return ((listed ? entry : -1) & from_list) | ((in_window < legal ? in_window : -1) & ~from_list);
    }
    __device__ __forceinline__ int count() const { return list_tiles + (legal - w0 + kTileKeys - 1) / kTileKeys; }
};
__device__ __forceinline__ Tiles tiles_of(const int32_t* __restrict__ idx, const void* readable, int64_t row_q, int t, int k, int held, int n_win, int m, int mask_mode) {
    Tiles u;
    u.list = k > 0 ? idx + row_q * k : static_cast<const int32_t*>(readable);  // without lists: anything that may be read
    u.k = k;
    u.last = max(k - 1, 0);
    u.held = held;
    u.legal = legal_count(t, held, m, mask_mode);
    u.w0 = max(0, u.legal - n_win);
    u.list_tiles = (k + kTileKeys - 1) / kTileKeys;
    return u;
}

// Eight codes as the values they stand for, `power` the row's power of two.
__device__ __forceinline__ halfx8 f16_values(unsigned codes, float power) {
    const halfx2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, power, 0);
    const halfx2 v1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, power, 1);
    const halfx2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, power, 2);
    const halfx2 v3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, power, 3);
    return halfx8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
}
__device__ __forceinline__ bf16x8 bf16_values(unsigned codes, float power) {
    const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 0);
    const bf16x2 v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 1);
    const bf16x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 2);
    const bf16x2 v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 3);
    return bf16x8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
}

// A lane's part of the tiles of 32 rows that its wave takes: row lane % 32, values D/2 * (lane / 32) .. + D/2, read from memory as codes and
// scale bytes.  As fp16 they are the first product's operand as they are (the contraction order is permuted alike on the query); for the
// second one they go through LDS, into a tile of the wave's own, row-major and swizzled (attention_set.h).  A wave's LDS accesses are done in
// order (wave_order()), so no wave waits for another.
// The scale bytes stay as they were read until they are used: taken apart at once they would be waited for at once.
template <int D>
struct Rows {
    static constexpr int kLoads = D / 64;  // 16-byte pieces of codes, a scale byte each
    uintx4 run[kLoads];
    std::conditional_t<D == 128, uint16_t, uint8_t> bytes;
    __device__ __forceinline__ void read(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales, int64_t row) {
        bytes = *reinterpret_cast<const decltype(bytes)*>(scales + row * (D / 32));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) run[i] = *reinterpret_cast<const uintx4*>(codes + row * (D / 2) + i * 16);
    }
    __device__ __forceinline__ unsigned byte(int i) const { return (static_cast<unsigned>(bytes) >> (8 * i)) & 0xFFu; }
    // values 8 ks .. 8 ks + 8 of the lane's part
    __device__ __forceinline__ halfx8 values(int ks) const {
        return f16_values(run[ks / 4][ks % 4], power_of(byte(ks / 4)));
    }
    // the same in bf16, times 2^(exponent)
    __device__ __forceinline__ bf16x8 values_bf16(int ks, int exponent) const {
        return bf16_values(run[ks / 4][ks % 4], power_of(byte(ks / 4) + static_cast<unsigned>(exponent)));
    }
};

// LDS offsets of a wave's tile at `base` (a multiple of 2 D): where the lane's pieces of its row go, and the transposing reads (attention.hip
// says how these are laid out).  The swizzle takes numbers of pieces apart by exclusive or, so all offsets of a kind are one register's with bits
// turned over: a piece's is put ^ 16 i.
template <int D>
struct Places {
    static constexpr int kReads = 4;
    int put, va[kReads];
    __device__ __forceinline__ Places(int lane, int base) {
        const int col = lane & 31, half = lane >> 5;
        put = base + tile_slot<D>(col, half * (D / 16)) * 16;
        const int G = lane >> 4, s = lane & 15;
        const int r = 4 * (G >> 1) + (s >> 2), d = 16 * (G & 1) + 4 * (s & 3);
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            if (D == 128) va[i] = base + tile_slot<D>(r, (32 * i + d) / 8) * 16 + ((d % 8) / 4) * 8;
            else va[i] = base + tile_slot<D>(r + 8 * (i & 1), (32 * (i >> 1) + d) / 8) * 16 + ((d % 8) / 4) * 8;
        }
    }
    __device__ __forceinline__ int put_at(int i) const { return put ^ (16 * i); }
    // d block db, rows 8 w + ..: for D = 128 row + 8 turns over the piece's bit 3, which is the block's bit 1
    __device__ __forceinline__ int read_at(int db, int w) const { return D == 128 ? va[db ^ (2 * w)] + w * 8 * 2 * D : va[2 * db + w]; }
};

// O^T += tile^T . P^T : contraction index e of step u <-> tile row 16 u + 8 (e / 4) + 4 half + e % 4 on both operands.
template <int D>
__device__ __forceinline__ void add_values(const unsigned char* tb, const Places<D>& at, const halfx8 (&p_hi)[2], const halfx8 (&p_lo)[2],
                                           floatx16 (&acc)[D / 32]) {
    typedef __attribute__((address_space(3))) fp16x4 lds_fp16x4;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
            const halfx4 v0 = __builtin_bit_cast(halfx4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_fp16x4*)(tb + at.read_at(db, 0) + u * 32 * D)));
            const halfx4 v1 = __builtin_bit_cast(halfx4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_fp16x4*)(tb + at.read_at(db, 1) + u * 32 * D)));
            const halfx8 vf = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, p_hi[u], acc[db], 0, 0, 0);
            acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, p_lo[u], acc[db], 0, 0, 0);
        }
}

// What a wave has of a query's block of 32 heads: O^T (register j of block db = d row 32 db + 8 (j / 4) + 4 half + j % 4, head = lane % 32),
// reference maximum of the lane's head (log2 domain) and the sum of the weights over the half-wave's rows.
template <int D>
struct Heads {
    floatx16 acc[D / 32];
    float m_ref, l_sum;
    __device__ __forceinline__ Heads() : m_ref(-__builtin_huge_valf()), l_sum(0.0f) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[db][j] = 0.0f;
    }
    // The scores of a tile, whose rows go to LDS on the way: after this `rows` may be read anew, while the rest of the tile's steps run.
    __device__ __forceinline__ floatx16 scores(const Rows<D>& rows, const halfx8 (&qf)[D / 16], unsigned char* lds, const Places<D>& at) const {
        floatx16 s = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            const halfx8 v = rows.values(ks);
            *reinterpret_cast<halfx8*>(lds + at.put_at(ks)) = v;
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, qf[ks], s, 0, 0, 0);
        }
        return s;
    }
    // Weights and second product; `live`: bit r says whether row r of the tile counts (not 0).
    __device__ __forceinline__ void take(floatx16& s, unsigned live, float to_log2, int half, const unsigned char* lds, const Places<D>& at) {
        float p[16];
        l_sum += weigh(s, to_log2, live, half, m_ref, p, [&](float alpha) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[db][j] *= alpha;
            l_sum *= alpha;
        });
        halfx8 p_hi[2], p_lo[2];
        split_weights(p, p_hi, p_lo);
        wave_order();
        add_values<D>(lds, at, p_hi, p_lo, acc);
        wave_order();
    }
};

// The same for a block of 16 heads (narrow_..), with the matrix instructions of half the size (16 x 16 x 32): half the work of a tile and half the
// registers.  A lane's part of a tile: rows lane % 16 and lane % 16 + 16, values D/4 * (lane / 16) .. + D/4; of the scores: rows 4 (lane / 16) + 0 .. 3
// and those + 16, head lane % 16.  Of the second product the `part`-th of DS parts of d: register j of block db = d row 16 (DB part + db) + 4 (lane / 16) + j.
template <int D>
struct HalfRows {
    typedef std::conditional_t<D == 128, uintx4, uintx2> run_t;
    run_t run[2];
    uint8_t bytes[2];
    __device__ __forceinline__ void read(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales, int64_t row, int which) {
        bytes[which] = scales[row * (D / 32)];
        run[which] = *reinterpret_cast<const run_t*>(codes + row * (D / 2));
    }
    __device__ __forceinline__ halfx8 values(int which, int ks) const {
        return f16_values(run[which][ks], power_of(bytes[which]));
    }
    __device__ __forceinline__ bf16x8 values_bf16(int which, int ks, int exponent) const {
        return bf16_values(run[which][ks], power_of(bytes[which] + static_cast<unsigned>(exponent)));
    }
};

// LDS offsets for such a block, of a wave's tile at `base`: where the lane's pieces of its two rows go, where its transposing reads begin (source lane s
// of 16 points at 4 consecutive d of row 4 (lane / 16) + s / 4, and 16 rows on).
template <int D>
struct NarrowPlaces {
    int put[2], va;
    __device__ __forceinline__ NarrowPlaces(int lane, int base) {
        const int col = lane & 15, quarter = lane >> 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) put[i] = base + tile_slot<D>(col + 16 * i, quarter * (D / 32)) * 16;
        va = base + tile_slot<D>(4 * quarter + (col >> 2), (col & 3) >> 1) * 16 + (col & 1) * 8;
    }
};

// The scores of half i of a tile, whose rows go to LDS on the way.
template <int D, int DS>
__device__ __forceinline__ floatx4 narrow_scores(const HalfRows<D>& rows, int i, const halfx8 (&qf)[D / 32], unsigned char* lds, int put, int quarter,
                                                 int part) {
    floatx4 x = {0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
        const halfx8 v = rows.values(i, ks);
        if (DS == 1 || quarter / (4 / DS) == part) *reinterpret_cast<halfx8*>(lds + (put ^ (16 * ks))) = v;
        x = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, qf[ks], x, 0, 0, 0);
    }
    return x;
}

// The number as one that the compiler does not know: what is made of it in a loop is not kept in registers from before the loop.
__device__ __forceinline__ int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// A condition that the compiler does not join with the one before it, of which it is the other case: it would lay out the rare way first, and hold
// there what the other one needs.
__device__ __forceinline__ int known_late(int condition) {
    condition = __builtin_amdgcn_readfirstlane(condition);
    asm volatile("" : "+s"(condition));
    return condition;
}

// The same of both halves by the bare product, whose query is as it stands in qa: lane lane % 16 has head lane % 16.  A step after the other, nothing read
// ahead: what the second conversion takes comes from the registers of the form above, which nearly all calls run.
template <int D>
__device__ __forceinline__ void bare_query(const __bf16* __restrict__ head, int quarter, BareProduct product, bf16x8 (&qf)[D / 32]) {
    const unsigned sign = product.to_log2 < 0.0f ? 0x80008000u : 0u;  // the factor that follows is above 0
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uintx4*>(head + quarter * (D / 4) + ks * 8) ^ sign);
}
template <int D, int DS>
__device__ __forceinline__ void bare_scores(const unsigned char* __restrict__ codes_b, const unsigned char* __restrict__ scales_b, const int (&row)[2],
                                            const bf16x8 (&qf)[D / 32], int exponent, unsigned char* lds, const NarrowPlaces<D>& at, int quarter, int part,
                                            floatx4 (&x)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        HalfRows<D> rows;
        rows.read(codes_b, scales_b, row[i], i);
        x[i] = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) {
            if (DS == 1 || quarter / (4 / DS) == part) *reinterpret_cast<halfx8*>(lds + (at.put[i] ^ (16 * ks))) = rows.values(i, ks);
            x[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rows.values_bf16(i, ks, exponent), qf[ks], x[i], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Weights and second product of a tile; `live`: bit r says whether row r of it counts (not 0).
template <int D, int DS>
__device__ __forceinline__ void narrow_take(floatx4 (&acc)[D / 16 / DS], float& m_ref, float& l_sum, floatx4 (&x)[2], unsigned live, float to_log2, int col,
                                            int quarter, const unsigned char* lds, const NarrowPlaces<D>& at, int part) {
    constexpr int DB = D / 16 / DS;
    if (live != 0xFFFFFFFFu) {
        float low = -__builtin_huge_valf();
        asm volatile("" : "+v"(low));
        const unsigned mine = live >> (4 * quarter);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!((mine >> (16 * (j >> 2) + (j & 3))) & 1)) x[j >> 2][j & 3] = low;
    }
    float p[8], sum;
    auto exponentials = [&]() {  // weigh() above says why without a maximum first
        const float shift = kWeightShift - m_ref;
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j >> 2][j & 3], to_log2, shift));
            sum += p[j];
        }
    };
    unsigned long long over = __ballot(m_ref == -__builtin_huge_valf());  // all heads on the first tile, later none but those of NaN
    if (__builtin_expect(over != ~0ull, 1)) {
        exponentials();
        over |= __ballot(!(sum <= 32768.0f));
    }
    if (over != 0ull) {
        over |= over >> 32;
        over |= over >> 16;  // bit h: head h, in any quarter
        float highest = x[0][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) highest = fmaxf(highest, x[j >> 2][j & 3]);
        highest *= to_log2;
        highest = fmaxf(highest, __shfl_xor(highest, 16));
        highest = fmaxf(highest, __shfl_xor(highest, 32));
        const float m_new = (over >> col) & 1 ? fmaxf(highest, m_ref) : m_ref;
        const float alpha = __builtin_amdgcn_exp2f(m_ref - m_new);
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] *= alpha;
        l_sum *= alpha;
        m_ref = m_new;
        exponentials();
    }
    l_sum += sum;
    float one = 1.0f;
    asm("" : "+s"(one));
    halfx8 p_hi, p_lo;
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
        const halfx2 a = __builtin_convertvector(floatx2{p[2 * jj], p[2 * jj + 1]}, halfx2);
        p_hi[2 * jj] = a[0];
        p_hi[2 * jj + 1] = a[1];
        p_lo[2 * jj] = static_cast<_Float16>(__builtin_fmaf(-static_cast<float>(a[0]), one, p[2 * jj]));
        p_lo[2 * jj + 1] = static_cast<_Float16>(__builtin_fmaf(-static_cast<float>(a[1]), one, p[2 * jj + 1]));
    }
    wave_order();
    // contraction index e <-> tile row 16 (e / 4) + 4 quarter + e % 4 on both operands
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        typedef __attribute__((address_space(3))) fp16x4 lds_fp16x4;
        const unsigned char* from = lds + (at.va ^ (32 * (DB * part + db)));
        const halfx4 v0 = __builtin_bit_cast(halfx4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_fp16x4*)from));
        const halfx4 v1 = __builtin_bit_cast(halfx4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_fp16x4*)(from + 16 * D * 2)));
        const halfx8 vf = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p_hi, acc[db], 0, 0, 0);
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p_lo, acc[db], 0, 0, 0);
    }
    wave_order();
}

// The end of such a block's way: sums over the quarters, out through the wave's tile.
template <int D>
__device__ __forceinline__ void narrow_out(int lane, floatx4 (&acc)[D / 16], float m_ref, float l_sum, int64_t row_q, int h0, int H, unsigned char* lds,
                                           int base, float* __restrict__ out, float* __restrict__ lse) {
    const int col = lane & 15, quarter = lane >> 4;
    const int h = h0 + col;
    l_sum += __shfl_xor(l_sum, 16);
    l_sum += __shfl_xor(l_sum, 32);
    const float inv = 1.0f / l_sum;
    constexpr int kSlots = D / 4;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) *reinterpret_cast<floatx4*>(lds + base + (col * kSlots + ((4 * db + quarter) ^ col)) * 16) = acc[db] * inv;
    wave_order();
#pragma unroll
    for (int i = 0; i < kSlots / 4; ++i) {
        const int head = i * (64 / kSlots) + lane / kSlots, slot = lane % kSlots;
        const floatx4 v = *reinterpret_cast<const floatx4*>(lds + base + (head * kSlots + (slot ^ head)) * 16);
        if (h0 + head < H) __builtin_nontemporal_store(v, reinterpret_cast<floatx4*>(out + (row_q * H + h0 + head) * D + 4 * slot));
    }
    if (lse && quarter == 0 && h < H) lse[row_q * H + h] = log_sum(m_ref, l_sum);
    wave_order();
}

// A wave's way through a query's list with a block of up to 16 heads from h0 on, by the bare product; base: of its tile in `lds`.
template <int D, typename Live>
__device__ __forceinline__ void bare_heads(const __bf16* __restrict__ qa, const unsigned char* __restrict__ codes_b, const unsigned char* __restrict__ scales_b,
                                           const int* s_list, int n_tiles, Live live, int64_t row_q, int h0, int H, BareProduct product, unsigned char* lds,
                                           int base, float* __restrict__ out, float* __restrict__ lse) {
    const int lane = fresh(threadIdx.x & 63), col = lane & 15, quarter = lane >> 4;
    bf16x8 qf[D / 32];
    bare_query<D>(qa + (row_q * H + min(h0 + col, H - 1)) * D, quarter, product, qf);
    const float to_log2 = __builtin_fabsf(product.to_log2);
    floatx4 acc[D / 16];
    float m_ref = -__builtin_huge_valf(), l_sum = 0.0f;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) acc[db] = floatx4{0, 0, 0, 0};
    for (int tile = 0; tile < n_tiles; ++tile) {
        const NarrowPlaces<D> at(fresh(lane), base);
        const int row[2] = {s_list[tile * kTileKeys + col], s_list[tile * kTileKeys + col + 16]};
        floatx4 x[2];
        bare_scores<D, 1>(codes_b + quarter * (D / 8), scales_b + quarter * D / 128, row, qf, product.exponent, lds, at, quarter, 0, x);
        narrow_take<D, 1>(acc, m_ref, l_sum, x, live(tile), to_log2, col, quarter, lds, at, 0);
    }
    narrow_out<D>(fresh(lane), acc, m_ref, l_sum, row_q, h0, H, lds, base, out, lse);
}

// The same in fp16.
template <int D, typename Live>
__device__ __forceinline__ void narrow_query(const __bf16* __restrict__ qa, const unsigned char* __restrict__ codes_b, const unsigned char* __restrict__ scales_b,
                                             const int* s_list, int n_tiles, Live live, int64_t row_q, int h0, int H, float scale_log2e, BareProduct product,
                                             unsigned char* lds, int base, float* __restrict__ out, float* __restrict__ lse) {
    constexpr int KS = D / 32;
    const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
    const int h = h0 + col;
    codes_b += quarter * (D / 8);
    scales_b += quarter * D / 128;
    HalfRows<D> rows;
#pragma unroll
    for (int i = 0; i < 2; ++i) rows.read(codes_b, scales_b, s_list[col + 16 * i], i);
    uintx4 raw[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) raw[ks] = *reinterpret_cast<const uintx4*>(qa + (row_q * H + min(h, H - 1)) * D + quarter * (D / 4) + ks * 8);
    unsigned sizes = extent(raw);
    sizes = joint(sizes, static_cast<unsigned>(__shfl_xor(static_cast<int>(sizes), 16)));
    sizes = joint(sizes, static_cast<unsigned>(__shfl_xor(static_cast<int>(sizes), 32)));
    float to_log2;
    unsigned border;
    const float power = query_power(sizes & 0xFFFFu, scale_log2e, to_log2, border);
    const int bare_block = needs_bare(0x10000u - (sizes >> 16) < border, to_log2);
    if (!bare_block) {
        halfx8 qf[KS];
        scale_query(raw, power, qf);
        const NarrowPlaces<D> at(lane, base);
        floatx4 acc[D / 16];
        float m_ref = -__builtin_huge_valf(), l_sum = 0.0f;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) acc[db] = floatx4{0, 0, 0, 0};
        int next[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) next[i] = s_list[min(1, n_tiles - 1) * kTileKeys + col + 16 * i];
        for (int tile = 0; tile < n_tiles; ++tile) {
            floatx4 x[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[i] = narrow_scores<D, 1>(rows, i, qf, lds, at.put[i], quarter, 0);
                rows.read(codes_b, scales_b, next[i], i);
                next[i] = s_list[min(tile + 2, n_tiles - 1) * kTileKeys + col + 16 * i];
            }
            narrow_take<D, 1>(acc, m_ref, l_sum, x, live(tile), to_log2, col, quarter, lds, at, 0);
        }
        narrow_out<D>(lane, acc, m_ref, l_sum, row_q, h0, H, lds, base, out, lse);
    }
    if (__builtin_expect(known_late(bare_block), 0))
        bare_heads<D>(qa, codes_b - quarter * (D / 8), scales_b - quarter * D / 128, s_list, n_tiles, live, row_q, h0, H, product, lds, base, out, lse);
}

// One workgroup = one query; wave w owns heads [32 w, 32 w + 32) and goes through the query's list (attention_set.h) by itself: each wave turns the
// codes it needs into a tile of its own, which costs the conversions twice and no barrier (a tile shared by two waves: 560 us, a wave by itself 520).
// 16384 queries of 640 rows, 64 heads of 128, take 445 to 515 us (300 GFLOP, 450 with the second part of the weights; the first kernel after a pause
// is the fastest).  The units that return gathered codes are busiest, 79 %: every row is gathered by both waves of a query.  The vector units are busy
// 63 %, the matrix pipe 53 %, at 1.82 GHz, which is what the power drawn leaves.  The form si_sparse_attention has of this, on rows of 256 bytes in place of 68, takes 475 to 500.
// Dynamic LDS: a tile of 32 x D fp16 a wave, the list.
template <int D, int HW, bool NARROW>
__global__ __launch_bounds__(64 * HW) __attribute__((amdgpu_waves_per_eu(3)))
void quantized_attention_kernel(const __bf16* __restrict__ qa, const unsigned char* __restrict__ codes,
                                const unsigned char* __restrict__ scales, const int32_t* __restrict__ lengths,
                                const int32_t* __restrict__ idx, int S, int H, int T, int m, int mask_mode, int k, int n_win,
                                float scale_log2e, BareProduct product, float* __restrict__ out, float* __restrict__ lse) {
    constexpr int kTileBytes = kTileKeys * D * 2;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    int* const s_list = reinterpret_cast<int*>(lds + HW * kTileBytes);
    __shared__ int s_kept[HW];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int col = lane & 31;
    const int half = lane >> 5;
    const int64_t row_q = blockIdx.x;  // b * S + t
    const int b = static_cast<int>(row_q / S);
    const int t = static_cast<int>(row_q % S);
    const int held = held_rows(lengths, b, T);
    const int legal = legal_count(t, held, m, mask_mode);
    const int w0 = max(0, legal - n_win);
    const int n = build_list<HW>(idx + row_q * k, k, held, w0, legal, s_list, s_kept);
    __syncthreads();
    const int n_u = __builtin_amdgcn_readfirstlane(n);
    const int h = 32 * wave + col;
    if (n_u == 0) {
        for (int i = threadIdx.x; i < H * D; i += 64 * HW) out[row_q * H * D + i] = 0.0f;
        if (lse && h < H && half == 0) lse[row_q * H + h] = -__builtin_huge_valf();
        return;
    }
    const int n_tiles = (n_u + kTileKeys - 1) / kTileKeys;
    const unsigned char* codes_b = codes + static_cast<int64_t>(b) * T * (D / 2);
    const unsigned char* scales_b = scales + static_cast<int64_t>(b) * T * (D / 32);
    // rows of U(t) from tile on: a tile's worth, or the last ones
    auto live = [&](int tile) {
        const int left = n_u - tile * kTileKeys;
        return left >= kTileKeys ? 0xFFFFFFFFu : (1u << left) - 1;
    };
    if (NARROW && (HW == 1 || wave == HW - 1)) {
        narrow_query<D>(qa, codes_b, scales_b, s_list, n_tiles, live, row_q, 32 * wave, H, scale_log2e, product, lds, wave * kTileBytes, out, lse);
        return;
    }
    codes_b += half * (D / 4);
    scales_b += half * (D / 64);
    Rows<D> rows;
    rows.read(codes_b, scales_b, s_list[col]);
    halfx8 qf[D / 16];
    uintx4 raw[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) raw[ks] = *reinterpret_cast<const uintx4*>(qa + (row_q * H + min(h, H - 1)) * D + half * (D / 2) + ks * 8);
    const unsigned mine_extent = extent(raw);
    const auto both = __builtin_amdgcn_permlane32_swap(mine_extent, mine_extent, false, false);
    float to_log2;
    unsigned border;
    const unsigned sizes = joint(both[0], both[1]);
    const float power = query_power(sizes & 0xFFFFu, scale_log2e, to_log2, border);
    const Places<D> at(lane, wave * kTileBytes);
    Heads<D> o;
    const int bare_block = needs_bare(0x10000u - (sizes >> 16) < border, to_log2);
    if (!bare_block) {
        scale_query(raw, power, qf);
        int s_next = s_list[min(1, n_tiles - 1) * kTileKeys + col];
        for (int tile = 0; tile < n_tiles; ++tile) {
            floatx16 x = o.scores(rows, qf, lds, at);
            rows.read(codes_b, scales_b, s_next);
            s_next = s_list[min(tile + 2, n_tiles - 1) * kTileKeys + col];
            o.take(x, live(tile), to_log2, half, lds, at);
        }
        const float l_all = o.l_sum + other_half(o.l_sum);
        const float inv = 1.0f / l_all;
        // out through the wave's tile, 64 (D = 64: 32) d of 32 heads at a time, so that it is written by whole lines, and past the caches' other contents:
        // a lane's own pieces, 16 bytes of each of 32 heads a store, took 241 us in place of 204 where a query has 128 rows, 432 / 418 where 512.
        constexpr int kSlots = kTileBytes / (32 * 16);  // pieces of four d
        float* const to = out + (row_q * H + 32 * wave) * D;
        const unsigned mine = static_cast<unsigned>(lane / kSlots * D + 4 * (lane % kSlots));
#pragma unroll
        for (int part = 0; part < D / (4 * kSlots); ++part) {
            unsigned char* const stage = lds + wave * kTileBytes;
#pragma unroll
            for (int db = 0; db < kSlots / 8; ++db)
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const floatx16& acc = o.acc[part * (kSlots / 8) + db];
                    const floatx4 v = {acc[4 * a] * inv, acc[4 * a + 1] * inv, acc[4 * a + 2] * inv, acc[4 * a + 3] * inv};
                    *reinterpret_cast<floatx4*>(stage + (col * kSlots + ((8 * db + 2 * a + half) ^ (col % kSlots))) * 16) = v;
                }
            wave_order();
#pragma unroll
            for (int i = 0; i < kSlots / 2; ++i) {
                const int head = i * (64 / kSlots) + lane / kSlots, slot = lane % kSlots;
                const floatx4 v = *reinterpret_cast<const floatx4*>(stage + (head * kSlots + (slot ^ (head % kSlots))) * 16);
                // one address a lane; the rest is the same for all
                if (head < H - 32 * wave) __builtin_nontemporal_store(v, reinterpret_cast<floatx4*>(to + (i * (64 / kSlots) * D + part * 4 * kSlots) + mine));
            }
            wave_order();
        }
        if (lse && half == 0 && h < H) lse[row_q * H + h] = log_sum(o.m_ref, l_all);
    }
    if (__builtin_expect(known_late(bare_block), 0)) {
#pragma unroll 1
        for (int h0 = 32 * wave; h0 < min(32 * wave + 32, H); h0 += 16)
            bare_heads<D>(qa, codes_b - half * (D / 4), scales_b - half * (D / 64), s_list, n_tiles, live, row_q, h0, H, product, lds, wave * kTileBytes, out, lse);
    }
}

// Few queries, which would leave most of the chip idle and walk their tiles one after the other: a workgroup takes one query and one block of
// 16 heads, and each of its 8 or 16 waves every 8th or 16th tile, with a reference, sums and accumulators of its own; the waves' results are joined at
// the end.  With blocks of 16 heads twice the waves share out the tiles on twice the compute units.  With DS = 2 two workgroups share a block of
// heads: both score all rows, each has half of d in the second product, the rows in LDS and the join.
// All workgroups of a query are on one XCD (32 queries, 1152 rows: 12.9 -> 9.8 us; each XCD's L2 read the rows again).  Bound by a wave's chain
// of dependent steps: of 9.5 us at 32 queries and 1152 rows 4.3 are launch, first tile and join, 1 a tile of a wave.
// Dynamic LDS: a tile of 32 x D fp16 a wave; for the join 16 x D / DS floats a wave.
constexpr int kFewHeads = 16;
constexpr int kXcds = 8;
template <int D, int WAVES>
constexpr int few_lds_bytes() { return WAVES * kTileKeys * D * 2; }

template <int D, int DS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(4)))
void quantized_attention_few_kernel(const __bf16* __restrict__ qa, const unsigned char* __restrict__ codes,
                                    const unsigned char* __restrict__ scales, const int32_t* __restrict__ lengths,
                                    const int32_t* __restrict__ idx, int S, int H, int T, int m, int mask_mode, int k, int n_win,
                                    int64_t n_queries, int head_blocks, float scale_log2e, BareProduct product, float* __restrict__ out, float* __restrict__ lse) {
    constexpr int W = WAVES;
    constexpr int KS = D / 32;       // matrix instructions along d in the first product
    constexpr int DB = D / 16 / DS;  // blocks of 16 d in the second
    constexpr int kPieces = D / 4 / DS;  // of four d
    constexpr int kTileBytes = kTileKeys * D * 2;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    __shared__ float s_ref[W][kFewHeads], s_sum[W][kFewHeads];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int col = lane & 15;   // row of a half tile, head
    const int quarter = lane >> 4;
    // workgroups go round the chip's eight XCDs: all of a query are on one, whose L2 then has the rows for all of them
    const unsigned turn = blockIdx.x / kXcds;
    const int part = static_cast<int>(turn % DS);  // of d
    const int h0 = kFewHeads * static_cast<int>(turn / DS % head_blocks);
    const int64_t row_q = static_cast<int64_t>(turn / DS / head_blocks) * kXcds + blockIdx.x % kXcds;
    if (row_q >= n_queries) return;
    const int b = static_cast<int>(row_q / S);
    const int t = static_cast<int>(row_q - static_cast<int64_t>(b) * S);
    const Tiles u = tiles_of(idx, qa, row_q, t, k, held_rows(lengths, b, T), n_win, m, mask_mode);
    const int n_tiles = u.count();
    const int waves = min(W, n_tiles);  // that have a tile
    const unsigned char* const codes_b = codes + static_cast<int64_t>(b) * T * (D / 2) + quarter * (D / 8);
    const unsigned char* const scales_b = scales + static_cast<int64_t>(b) * T * (D / 32) + quarter * D / 128;

    float m_ref = -__builtin_huge_valf();
    float l_sum = 0.0f;
    floatx4 acc[DB];  // register j of block db = d row 16 (DB part + db) + 4 quarter + j, head = col
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = floatx4{0, 0, 0, 0};
    // the query, one or two heads a wave, to fp16 and to LDS: pieces of 8 values turned over by the head's number as those of a tile's rows
    __shared__ __attribute__((aligned(16))) _Float16 s_query[kFewHeads * D];
    __shared__ float s_scale[kFewHeads];
    __shared__ int s_lost[W];  // whether one of a wave's heads needs the bare product
    bool lost = false;
    constexpr int kHeadsPerWave = kFewHeads / W;
    constexpr int kPair = D / 64;  // values of a lane
    typedef std::conditional_t<D == 128, unsigned, uint16_t> pair_t;
    unsigned pair[kHeadsPerWave];
#pragma unroll
    for (int i = 0; i < kHeadsPerWave; ++i)
        pair[i] = reinterpret_cast<const pair_t*>(qa + (row_q * H + min(h0 + wave + i * W, H - 1)) * D)[lane];
    int s_now[2] = {-1, -1}, next[2] = {-1, -1};
    HalfRows<D> rows;
    if (wave < waves) {
#pragma unroll
        for (int i = 0; i < 2; ++i) s_now[i] = u.entry(wave, col + 16 * i);
#pragma unroll
        for (int i = 0; i < 2; ++i) next[i] = u.entry(wave + W, col + 16 * i);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s_now[i] = u.row(s_now[i], wave, col + 16 * i);
            rows.read(codes_b, scales_b, max(s_now[i], 0), i);
        }
    }
#pragma unroll
    for (int i = 0; i < kHeadsPerWave; ++i) {
        const int head = wave + i * W;
        const unsigned first = pair[i] & 0x7FFFu, second = (pair[i] >> 16) & 0x7FFFu;
        float to_log2;
        unsigned border;
        const float power = query_power(wave_max(max(first, second)), scale_log2e, to_log2, border);
        lost |= min(first - 1, second - 1) < border - 1;
        const int at = head * D + (((lane * kPair / 8) ^ (head % (D / 8))) * 8 + lane * kPair % 8);
        s_query[at] = static_cast<_Float16>(__uint_as_float(pair[i] << 16) * power);
        if (kPair == 2) s_query[at + 1] = static_cast<_Float16>(__uint_as_float(pair[i] & 0xFFFF0000u) * power);
        if (lane == 0) s_scale[head] = to_log2;
    }
    const bool wave_lost = __ballot(lost) != 0ull;
    if (lane == 0) s_lost[wave] = wave_lost;
    __syncthreads();
    if (wave < waves) {
        halfx8 qf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const halfx8*>(s_query + (col * (D / 8) + ((quarter * KS + ks) ^ (col % (D / 8)))) * 8);
        float to_log2 = s_scale[col];
        const int lost_of = s_lost[lane % W];
        const NarrowPlaces<D> at(lane, wave * kTileBytes);
        auto live_rows = [&]() {
            unsigned live = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) live |= (static_cast<unsigned>(__ballot(s_now[i] >= 0)) & 0xFFFFu) << (16 * i);
            return live;
        };
        for (int tile = wave; tile < n_tiles; tile += W) {
            const unsigned live = live_rows();
            floatx4 x[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[i] = narrow_scores<D, DS>(rows, i, qf, lds, at.put[i], quarter, part);
                s_now[i] = u.row(next[i], tile + W, col + 16 * i);
                rows.read(codes_b, scales_b, max(s_now[i], 0), i);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) next[i] = u.entry(tile + 2 * W, col + 16 * i);
            if (live == 0) continue;
            narrow_take<D, DS>(acc, m_ref, l_sum, x, live, to_log2, col, quarter, lds, at, part);
        }
        // Asked only now, and by every wave alike: asked before the loop, what leads to the loop was waiting for the answer, 0.2 us of 5.2 to 9.5.
        if (__builtin_expect(needs_bare(lost_of != 0, to_log2), 0)) {
            to_log2 = __builtin_fabsf(product.to_log2);
            m_ref = -__builtin_huge_valf();
            l_sum = 0.0f;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = floatx4{0, 0, 0, 0};
            bf16x8 qb[KS];
            bare_query<D>(qa + (row_q * H + min(h0 + col, H - 1)) * D, quarter, product, qb);
            for (int tile = wave; tile < n_tiles; tile += W) {
#pragma unroll
                for (int i = 0; i < 2; ++i) s_now[i] = u.row(u.entry(tile, col + 16 * i), tile, col + 16 * i);
                const unsigned live = live_rows();
                if (live == 0) continue;
                const int row[2] = {max(s_now[0], 0), max(s_now[1], 0)};
                const NarrowPlaces<D> here(fresh(lane), wave * kTileBytes);
                floatx4 x[2];
                bare_scores<D, DS>(codes_b, scales_b, row, qb, product.exponent, lds, here, quarter, part, x);
                narrow_take<D, DS>(acc, m_ref, l_sum, x, live, to_log2, col, quarter, lds, here, part);
            }
        }
        l_sum += __shfl_xor(l_sum, 16);
        l_sum += __shfl_xor(l_sum, 32);
        if (quarter == 0) s_ref[wave][col] = m_ref;
    }
    // ---- join: the largest reference of the waves, sums and accumulators brought to it
    __syncthreads();  // also: every wave is done with its tile
    float m_all = -__builtin_huge_valf();
#pragma unroll
    for (int w = 0; w < W; ++w) m_all = fmaxf(m_all, w < waves ? s_ref[w][col] : -__builtin_huge_valf());
    floatx4* const s_acc = reinterpret_cast<floatx4*>(lds);  // [wave][piece of four d][head]
    if (wave < waves) {
        const float alpha = m_ref == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f(m_ref - m_all);
#pragma unroll
        for (int db = 0; db < DB; ++db) s_acc[(wave * kPieces + 4 * db + quarter) * kFewHeads + col] = acc[db] * alpha;
        if (quarter == 0) s_sum[wave][col] = l_sum * alpha;
    }
    __syncthreads();
    const int h = h0 + col;
    if (h >= H) return;
    for (int piece = 4 * wave + quarter; piece < kPieces; piece += 4 * W) {
        float l_all = 0.0f;
        floatx4 v = {0, 0, 0, 0};
        if (waves == W) {  // unrolled, the reads wait for LDS once: 1 us of 12.7 at 16 waves
#pragma unroll
            for (int w = 0; w < W; ++w) {
                l_all += s_sum[w][col];
                v += s_acc[(w * kPieces + piece) * kFewHeads + col];
            }
        } else {
            for (int w = 0; w < waves; ++w) {
                l_all += s_sum[w][col];
                v += s_acc[(w * kPieces + piece) * kFewHeads + col];
            }
        }
        *reinterpret_cast<floatx4*>(out + (row_q * H + h) * D + part * (D / DS) + 4 * piece) = v * (l_all == 0.0f ? 0.0f : 1.0f / l_all);
        if (lse && piece == 0 && part == 0)
            lse[row_q * H + h] = l_all == 0.0f ? -__builtin_huge_valf() : log_sum(m_all, l_all);
    }
}

// A query's heads as the first product's operand, one wave: head 32 hb + lane % 32, values D/2 * (lane / 32) + 8 ks .. + 8; of H heads the last
// stands in for those there are not.  Whole lines are read and parted out through 4 KiB of LDS: read head by head into the registers a line
// would be asked for eight times.
template <int D, int HB>
__device__ __forceinline__ void load_heads(const __bf16* __restrict__ query, int H, unsigned char* buffer, bf16x8 (&qf)[HB][D / 16]) {
    constexpr int KS = D / 16;
    constexpr int kRounds = D / 64;  // four pieces of 8 values of each half of a head a round
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    uintx4 piece[HB][kRounds][4];
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int head = i * 8 + lane / 8, p = lane % 8;
                piece[hb][r][i] = *reinterpret_cast<const uintx4*>(query + static_cast<int64_t>(min(32 * hb + head, H - 1)) * D + ((p / 4) * KS + 4 * r + p % 4) * 8);
            }
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int head = i * 8 + lane / 8, p = lane % 8;
                *reinterpret_cast<uintx4*>(buffer + (head * 8 + (p ^ (head % 8))) * 16) = piece[hb][r][i];
            }
            wave_order();
#pragma unroll
            for (int k = 0; k < 4; ++k) qf[hb][4 * r + k] = *reinterpret_cast<const bf16x8*>(buffer + (col * 8 + ((half * 4 + k) ^ (col % 8))) * 16);
            wave_order();
        }
}

// What rows of U(t) receive of a query: S[32 heads x 32 rows] = q . tile^T with the heads on the M side, so that a lane holds 16 heads of
// one row and the sum over heads is in-lane (and one exchange).  A lane's codes go from memory to its registers as they are needed there
// (row = lane % 32, values D/2 * (lane / 32) .. + D/2: the contraction order is permuted alike on the query) and on to bf16, in which
// both operands are exact, the row's with the factor of BareProduct: neither list nor tile goes through LDS.  The vector units bound it: 64 heads of 128 take 16 matrix instructions a
// tile, 512 cycles, against 32 conversions, 32 fma, 32 additions and 32 exponentials, which take longer.
// One wave: tiles [first, last) of query row_q; add(row, sum) for every row of U(t) there, on the lanes below 32.  lds: kWeighBytes of the wave.
constexpr int kWeighBytes = 4096 + 256;
template <int D, int HB, typename Add>
__device__ __forceinline__ void weigh_tiles(const __bf16* __restrict__ qa, const unsigned char* __restrict__ codes,
                                            const unsigned char* __restrict__ scales, const float* __restrict__ lse, int64_t row_q, int H,
                                            int64_t first_row, const Tiles& u, int first, int last, BareProduct product, unsigned char* lds, Add add) {
    constexpr int KS = D / 16;
    if (first >= last) return;
    const int lane = threadIdx.x & 63;
    const int col = lane & 31;
    const int half = lane >> 5;
    const unsigned char* const codes_b = codes + first_row * (D / 2) + half * (D / 4);
    const unsigned char* const scales_b = scales + first_row * (D / 32) + half * (D / 64);
    float* const s_lse = reinterpret_cast<float*>(lds + 4096);
    int s_now = u.row(u.entry(first, col), first, col);
    int next = u.entry(first + 1, col);
    const float given = lse[row_q * H + min(lane, H - 1)];
    s_lse[lane] = lane < H ? __builtin_fmaf(-kLog2e, given, -kLog2eRest * given) : -__builtin_huge_valf();  // no head there: weight 0
    bf16x8 qf[HB][KS];
    load_heads<D, HB>(qa + row_q * H * D, H, lds, qf);
    Rows<D> rows;
    rows.read(codes_b, scales_b, max(s_now, 0));
    for (int tile = first; tile < last; ++tile) {
        floatx16 x[HB];
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) x[hb] = floatx16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const bf16x8 v = rows.values_bf16(ks, product.exponent);
#pragma unroll
            for (int hb = 0; hb < HB; ++hb) x[hb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[hb][ks], v, x[hb], 0, 0, 0);
        }
        const int s = s_now;
        // also behind the last tile, where nothing comes of them: without branches the loads on their way can be told apart when one is waited for
        s_now = u.row(next, tile + 1, col);
        rows.read(codes_b, scales_b, max(s_now, 0));
        next = u.entry(tile + 2, col);
        if (__ballot(s >= 0) == 0ull) continue;
        float sum = 0.0f;
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const floatx4 minus_lse = *reinterpret_cast<const floatx4*>(s_lse + 32 * hb + 8 * a + 4 * half);  // of these heads
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[hb][4 * a + j], product.to_log2, minus_lse[j]));
            }
        sum += other_half(sum);
        // A sum that is no number (some head's lse is none) is not added: it would stay in the weights for good, and has no fixed-point form.  A head
        // gives a row 1 at most, whatever the rounding of a large lse makes of it.
        if (half == 0 && s >= 0 && sum == sum) add(s, fminf(sum, static_cast<float>(H)));
    }
}

// A sum in units of 1 / per_unit (a power of two), to the nearest: both halves are exact in fp32 but where the sum is below 2^24 units.
__device__ __forceinline__ unsigned long long to_fixed(float sum, float per_unit) {
    const float units = sum * per_unit;
    const float high = __builtin_floorf(units * (1.0f / 4294967296.0f));
    const unsigned low = static_cast<unsigned>(__builtin_rintf(__builtin_fmaf(high, -4294967296.0f, units)));
    return (static_cast<unsigned long long>(static_cast<unsigned>(high)) << 32) | low;
}

constexpr int kWeightWaves = 4;
// A wave takes `per` tiles of a query (n_parts such parts a query).  S == 1: every row has one sum a call, added to
// weights;  S > 1: 64-bit sums in the workspace, in any order.
template <int D, int HB>
__global__ __launch_bounds__(64 * kWeightWaves) __attribute__((amdgpu_waves_per_eu(3)))
void accumulate_weights_kernel(const __bf16* __restrict__ qa, const unsigned char* __restrict__ codes,
                               const unsigned char* __restrict__ scales, const int32_t* __restrict__ lengths,
                               const int32_t* __restrict__ idx, int64_t n_queries, int n_parts, int per, int S, int H, int T, int m, int mask_mode,
                               int k, int n_win, BareProduct product, const float* __restrict__ lse, float* __restrict__ weights,
                               unsigned long long* __restrict__ sums, float per_unit) {
    __shared__ __attribute__((aligned(16))) unsigned char lds[kWeightWaves][kWeighBytes];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // all workgroups of a query are on one XCD, as in the kernel for few queries
    const int groups = (n_parts + kWeightWaves - 1) / kWeightWaves;
    const unsigned turn = blockIdx.x / kXcds;
    const int64_t row_q = static_cast<int64_t>(turn / groups) * kXcds + blockIdx.x % kXcds;
    const int part = static_cast<int>(turn % groups) * kWeightWaves + wave;
    if (row_q >= n_queries || part >= n_parts) return;
    const int b = static_cast<int>(row_q / S);
    const int t = static_cast<int>(row_q - static_cast<int64_t>(b) * S);
    const Tiles u = tiles_of(idx, qa, row_q, t, k, held_rows(lengths, b, T), n_win, m, mask_mode);
    const int64_t first_row = static_cast<int64_t>(b) * T;
    weigh_tiles<D, HB>(qa, codes, scales, lse, row_q, H, first_row, u, part * per, min(u.count(), (part + 1) * per), product, lds[wave],
                       [&](int s, float sum) {
                           if (sums) atomicAdd(sums + first_row + s, to_fixed(sum, per_unit));
                           else weights[first_row + s] += sum;
                       });
}

// Many queries of few rows: 8192 of 640 of 2048 rows, 64 heads of 128, take 95 us of 99 to 103 in this kernel.  The units that return gathered codes are
// busy 70 %, vector units 59 %, matrix pipe 37 % (without exponentials 12 us less, without products 27, without reads of rows 15).  A workgroup adds up in LDS what its queries (every n_groups-th wave's worth of a batch) give the batch's rows,
// and then adds that to the workspace, row after row.  Added up there at once, the sums wait for one another: 8192 queries of 640 of 2048 rows took
// 657 us, 12 adds a nanosecond.
template <int D, int HB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(3)))
void gather_weights_kernel(const __bf16* __restrict__ qa, const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                           const int32_t* __restrict__ lengths, const int32_t* __restrict__ idx, int n_groups, int S, int H, int T, int m,
                           int mask_mode, int k, int n_win, BareProduct product, const float* __restrict__ lse,
                           unsigned long long* __restrict__ sums, float per_unit) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    unsigned long long* const s_sums = reinterpret_cast<unsigned long long*>(lds + WAVES * kWeighBytes);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / n_groups;
    const int group = blockIdx.x % n_groups;
    for (int i = threadIdx.x; i < T; i += 64 * WAVES) s_sums[i] = 0;
    __syncthreads();
    const int held = held_rows(lengths, b, T);
    for (int t = group * WAVES + wave; t < S; t += n_groups * WAVES) {
        const int64_t row_q = static_cast<int64_t>(b) * S + t;
        const Tiles u = tiles_of(idx, qa, row_q, t, k, held, n_win, m, mask_mode);
        weigh_tiles<D, HB>(qa, codes, scales, lse, row_q, H, static_cast<int64_t>(b) * T, u, 0, u.count(), product, lds + wave * kWeighBytes,
                           [&](int s, float sum) { atomicAdd(s_sums + s, to_fixed(sum, per_unit)); });
    }
    __syncthreads();
    for (int i = threadIdx.x; i < T; i += 64 * WAVES)
        if (s_sums[i]) atomicAdd(sums + static_cast<int64_t>(b) * T + i, s_sums[i]);
}

__global__ void clear_sums_kernel(unsigned long long* sums, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * blockDim.x)
        sums[i] = 0;
}
__global__ void add_sums_kernel(const unsigned long long* __restrict__ sums, int64_t n, double unit, float* __restrict__ weights) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * blockDim.x)
        if (sums[i]) weights[i] = static_cast<float>(weights[i] + static_cast<double>(sums[i]) * unit);
}

constexpr int64_t kMostQueries = (int64_t{1} << 24) - 8;
constexpr int32_t kMostRows = 1 << 30;

struct Call {
    const __bf16* qa;
    const unsigned char *codes, *scales;
    const int32_t *lengths, *idx;
    si_dims d;
    int32_t m, mask_mode, k, n_win;
    float scale_log2e;
    hipStream_t stream;
};

BareProduct bare_product(float scale_log2e) {
    const float size = std::fabs(scale_log2e);
    if (size == 0.0f) return {1.1754944e-38f, -64};
    const int exponent = size < 1.0f ? -27 : size < 4294967296.0f ? 0 : 27;
    return {std::ldexp(scale_log2e, -exponent), exponent};
}

template <int D, int HW, bool NARROW>
hipError_t launch_attention(const Call& c, float* out, float* lse) {
    static std::atomic<size_t> allowed[64];
    const size_t lds = HW * static_cast<size_t>(kTileKeys) * D * 2 + list_bytes(c.k, c.n_win);
    hipError_t e = allow_lds(quantized_attention_kernel<D, HW, NARROW>, lds, allowed);
    if (e != hipSuccess) return e;
    const int64_t rows = static_cast<int64_t>(c.d.B) * c.d.S;
    hipLaunchKernelGGL((quantized_attention_kernel<D, HW, NARROW>), dim3(static_cast<unsigned>(rows)), dim3(64 * HW), lds, c.stream, c.qa,
                       c.codes, c.scales, c.lengths, c.idx, c.d.S, c.d.H_I, c.d.T, c.m, c.mask_mode, c.k, c.n_win, c.scale_log2e,
                       bare_product(c.scale_log2e), out, lse);
    return hipGetLastError();
}

template <int D, int DS, int WAVES>
hipError_t launch_few(const Call& c, float* out, float* lse) {
    static std::atomic<size_t> allowed[64];
    constexpr int kBytes = few_lds_bytes<D, WAVES>();
    hipError_t e = allow_lds(quantized_attention_few_kernel<D, DS, WAVES>, kBytes, allowed);
    if (e != hipSuccess) return e;
    const int head_blocks = (c.d.H_I + kFewHeads - 1) / kFewHeads;
    const int64_t n_queries = static_cast<int64_t>(c.d.B) * c.d.S;
    const int64_t grid = (n_queries + kXcds - 1) / kXcds * kXcds * head_blocks * DS;
    hipLaunchKernelGGL((quantized_attention_few_kernel<D, DS, WAVES>), dim3(static_cast<unsigned>(grid)), dim3(64 * WAVES), kBytes, c.stream, c.qa,
                       c.codes, c.scales, c.lengths, c.idx, c.d.S, c.d.H_I, c.d.T, c.m, c.mask_mode, c.k, c.n_win, n_queries, head_blocks,
                       c.scale_log2e, bare_product(c.scale_log2e), out, lse);
    return hipGetLastError();
}

// A wave a block of 32 heads; a last block of up to 16 takes the matrix instructions of half the size.  With those of the full size and without
// (us): 8192 queries of 640 rows, 16 heads of 128 110 -> 75, 40 heads 210 -> 182, 48 heads of 64 127 -> 110, 3000 of 264 rows, 9 heads of 128 24 -> 17.
template <int D>
hipError_t launch_attention(const Call& c, float* out, float* lse) {
    const int H = c.d.H_I;
    if (H <= 16) return launch_attention<D, 1, true>(c, out, lse);
    if (H <= 32) return launch_attention<D, 1, false>(c, out, lse);
    return H <= 48 ? launch_attention<D, 2, true>(c, out, lse) : launch_attention<D, 2, false>(c, out, lse);
}

// Blocks of 16 heads of all queries, and the rows a query may attend to by its list and window (the host does not know how many are held), decide.
// Measured at 64 heads of 128, and taken for other numbers and sizes of heads as it is (us; B queries of 64 heads of 128, 4 B blocks):
// the kernel for many queries against this one's, rows 1152: B = 32 33 -> 9.5, 128 34 -> 16, 192 34 -> 23, 256 35 -> 29, 384 47 -> 40, 512 47 -> 52;
// 384 rows: 128 15 -> 9, 192 15.2 -> 13.1, 256 15.8 -> 16.0; 64 rows: 32 5.5 -> 4.6, 160 6.9 -> 8.7.
bool few_queries(const si_dims& d, int k, int n_win) {
    const int64_t blocks = static_cast<int64_t>(d.B) * d.S * ((d.H_I + kFewHeads - 1) / kFewHeads);
    return blocks <= 512 || (blocks < 1024 && k + n_win >= 384) || (blocks <= 1536 && k + n_win >= 1024);
}
// Measured at 64 heads of 128, as above.  Halves of d where these fit the chip's compute units once (B = 32: 10.4 -> 9.5, B = 48: 10.6 -> 13.4); 16 waves where a workgroup has a unit to
// itself and more than five tiles a wave (B = 32, rows 1152 / 1536 / 2048 / 4096: 8 waves 9.5 / 11.7 / 14.3 / 23.8, 16 waves 9.8 / 11.2 / 13.2 / 20.1;
// B = 64: 11.0 / 13.5 / 17.0 / - and 11.6 / 13.5 / 16.0 / -).
template <int D>
hipError_t launch_few(const Call& c, float* out, float* lse) {
    const int64_t blocks = static_cast<int64_t>(c.d.B) * c.d.S * ((c.d.H_I + kFewHeads - 1) / kFewHeads);
    const bool wide = c.k + c.n_win > 1536;
    if (blocks <= 128) return wide ? launch_few<D, 2, 16>(c, out, lse) : launch_few<D, 2, 8>(c, out, lse);
    return wide && blocks <= 256 ? launch_few<D, 1, 16>(c, out, lse) : launch_few<D, 1, 8>(c, out, lse);
}

// Units of 1: as fine as 64 bits allow where all S queries and H heads give a row 1 each, S H = 2^30 at most.  With units of 2^-32 for every call, what
// a query gave below 2^-33 was nothing, and eviction ranked such rows by their numbers: all but one where one row's logits are 30 above the others'.
double sums_per_unit(const si_dims& d) {
    int bits = 0;
    while ((int64_t{1} << bits) < static_cast<int64_t>(d.S) * d.H_I) ++bits;
    return std::ldexp(1.0, 63 - bits);
}

template <int D, int HB, int WAVES>
hipError_t launch_gather(const Call& c, int most_groups, const float* lse, unsigned long long* sums) {
    static std::atomic<size_t> allowed[64];
    const int n_groups = std::min((c.d.S + WAVES - 1) / WAVES, std::max(1, most_groups / c.d.B));  // of a batch
    const size_t lds = WAVES * kWeighBytes + static_cast<size_t>(c.d.T) * sizeof(unsigned long long);
    hipError_t e = allow_lds(gather_weights_kernel<D, HB, WAVES>, lds, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((gather_weights_kernel<D, HB, WAVES>), dim3(static_cast<unsigned>(c.d.B) * n_groups), dim3(64 * WAVES), lds, c.stream, c.qa,
                       c.codes, c.scales, c.lengths, c.idx, n_groups, c.d.S, c.d.H_I, c.d.T, c.m, c.mask_mode, c.k, c.n_win, bare_product(c.scale_log2e),
                       lse, sums, static_cast<float>(sums_per_unit(c.d)));
    return hipGetLastError();
}

constexpr int kGatherRows = 15360;  // whose sums fit LDS beside the waves' parts: 120 KiB
static_assert(8 * kWeighBytes + kGatherRows * 8 <= 159 * 1024, "the longest cache fits");

// Many queries in one go over rows whose sums fit LDS; three workgroups of four waves a compute unit while LDS holds three, then one of eight.
// Measured (us): sums in the workspace at once / 8 waves, 256 workgroups / 4 waves, 768 workgroups, 64 heads of 128: 8192 queries of 640 of 2048 rows
// 657 / 116 / 106, 4000 of 1128 of 4000 381 / 104 / 95, 2 x 6000 of 428 of 6000 358 / 124 / 137, 10000 of 164 of 10000 114 / 63 / 90, 300 of 100 of 300
// 22 / 16 / 17; few queries, whose tiles are then not shared out: 64 of 640 of 4000 8.7 / 28 / 22, 64 x 4 of 640 of 8192 16 / 25 / 26.
// Longer caches take the sums in the workspace at once, at 17 to 22 rows a nanosecond (65536 queries of 640 of 16384 rows 2.4 ms, 262144 of 1152 of 65536
// 13.8 ms) in place of 38 to 46 (61440 of 640 of 15360 0.82 ms): their adds, scattered over all rows, bound them, for 16 heads as for 64.
bool gathers(const si_dims& d) {
    return d.T <= kGatherRows && (d.S >= 128 || (d.S >= 16 && static_cast<int64_t>(d.B) * d.S >= 1024));
}

template <int D, int HB>
hipError_t launch_weights(const Call& c, const float* lse, float* weights, unsigned long long* sums) {
    if (gathers(c.d)) return c.d.T <= 4096 ? launch_gather<D, HB, 4>(c, 768, lse, sums) : launch_gather<D, HB, 8>(c, 256, lse, sums);
    const int64_t rows = static_cast<int64_t>(c.d.B) * c.d.S;
    const int tiles = (c.k + kTileKeys - 1) / kTileKeys + (c.n_win + kTileKeys - 1) / kTileKeys;
    // parts of at least two tiles, as many as fill the chip's waves once
    const int64_t most = std::max<int64_t>(1, 2048 / rows);
    const int per = static_cast<int>(std::max<int64_t>(2, (tiles + most - 1) / most));
    const int n_parts = std::max(1, (tiles + per - 1) / per);
    const int64_t grid = (rows + kXcds - 1) / kXcds * kXcds * ((n_parts + kWeightWaves - 1) / kWeightWaves);
    hipLaunchKernelGGL((accumulate_weights_kernel<D, HB>), dim3(static_cast<unsigned>(grid)), dim3(64 * kWeightWaves), 0, c.stream, c.qa, c.codes,
                       c.scales, c.lengths, c.idx, rows, n_parts, per, c.d.S, c.d.H_I,
                       c.d.T, c.m, c.mask_mode, c.k, c.n_win, bare_product(c.scale_log2e), lse, weights, sums, static_cast<float>(sums_per_unit(c.d)));
    return hipGetLastError();
}

float in_log2(float scale) { return static_cast<float>(scale * 1.4426950408889634); }

si_status check(const void* qa, const void* codes, const void* scales, const int32_t* lengths, const int32_t* idx, const si_dims* dims,
                int32_t m, int32_t k, si_mask_mode mask_mode, int32_t n_win, float scale) {
    if (!dims || !qa || !codes || !scales || (!idx && k != 0)) return SI_ERR_INVALID_ARG;
    if (!aligned16(qa) || !aligned16(codes) || !aligned16(scales) || !aligned16(idx) || !aligned4(lengths)) return SI_ERR_INVALID_ARG;
    if (dims->B < 1 || dims->S < 1 || dims->H_I < 1 || dims->D < 1 || dims->T < 1 || m < 1 || k < 0 || n_win < 0) return SI_ERR_INVALID_ARG;
    if (mask_mode != SI_MASK_NONE && mask_mode != SI_MASK_CAUSAL_BLOCK) return SI_ERR_INVALID_ARG;
    const float scale_log2e = in_log2(scale);
    if (scale_log2e - scale_log2e != 0.0f) return SI_ERR_INVALID_ARG;  // NaN, infinite, or not to be had in log2 units
    if (dims->D != 64 && dims->D != 128) return SI_ERR_UNSUPPORTED_SHAPE;
    if (dims->H_I > kMaxHeads || k > kMaxK || n_win > kMaxK) return SI_ERR_UNSUPPORTED_SHAPE;
    // a launch has fewer than 2^32 threads in a dimension, up to 256 a query, queries in eights; row numbers beyond a window's end fit 32 bits
    if (static_cast<int64_t>(dims->B) * dims->S > kMostQueries || dims->T > kMostRows) return SI_ERR_UNSUPPORTED_SHAPE;
    return SI_OK;
}

}  // namespace

}  // namespace si

using namespace si;

extern "C" {

si_status si_quantized_attention(const void* qa, const void* codes, const void* scales, const int32_t* lengths,
                                 const int32_t* idx, const si_dims* dims, int32_t m, int32_t k, si_mask_mode mask_mode,
                                 int32_t n_win, float scale, float* out, float* lse, void* stream) {
    const si_status ok = check(qa, codes, scales, lengths, idx, dims, m, k, mask_mode, n_win, scale);
    if (ok != SI_OK) return ok;
    if (!out || !aligned16(out) || !aligned16(lse)) return SI_ERR_INVALID_ARG;
    const Call c = {static_cast<const __bf16*>(qa), static_cast<const unsigned char*>(codes), static_cast<const unsigned char*>(scales),
                    lengths, idx, *dims, m, mask_mode, k, n_win, in_log2(scale), static_cast<hipStream_t>(stream)};
    if (few_queries(*dims, k, n_win)) return report(dims->D == 128 ? launch_few<128>(c, out, lse) : launch_few<64>(c, out, lse));
    return report(dims->D == 128 ? launch_attention<128>(c, out, lse) : launch_attention<64>(c, out, lse));
}

size_t si_accumulate_workspace_bytes(const si_dims* dims) {
    if (!dims || dims->B < 1 || dims->S < 1 || dims->T < 1) return 0;
    return dims->S == 1 ? 0 : static_cast<size_t>(dims->B) * static_cast<size_t>(dims->T) * sizeof(unsigned long long);
}

si_status si_accumulate_weights(const void* qa, const void* codes, const void* scales, const int32_t* lengths,
                                const int32_t* idx, const si_dims* dims, int32_t m, int32_t k, si_mask_mode mask_mode,
                                int32_t n_win, float scale, const float* lse, float* weights, void* workspace,
                                size_t workspace_bytes, void* stream) {
    const si_status ok = check(qa, codes, scales, lengths, idx, dims, m, k, mask_mode, n_win, scale);
    if (ok != SI_OK) return ok;
    if (!lse || !weights || !aligned16(lse) || !aligned16(weights)) return SI_ERR_INVALID_ARG;
    const size_t need = si_accumulate_workspace_bytes(dims);
    if (need > 0 && (!workspace || !aligned16(workspace))) return SI_ERR_INVALID_ARG;
    if (workspace_bytes < need) return SI_ERR_WORKSPACE_TOO_SMALL;
    const Call c = {static_cast<const __bf16*>(qa), static_cast<const unsigned char*>(codes), static_cast<const unsigned char*>(scales),
                    lengths, idx, *dims, m, mask_mode, k, n_win, in_log2(scale), static_cast<hipStream_t>(stream)};
    unsigned long long* sums = need > 0 ? static_cast<unsigned long long*>(workspace) : nullptr;
    const int64_t n = static_cast<int64_t>(dims->B) * dims->T;
    const unsigned blocks = static_cast<unsigned>(n < (int64_t{1} << 20) ? (n + 255) / 256 : 4096);
    hipError_t e = hipSuccess;
    if (sums) {
        hipLaunchKernelGGL(clear_sums_kernel, dim3(blocks), dim3(256), 0, c.stream, sums, n);
        e = hipGetLastError();
    }
    if (e == hipSuccess) {
        const bool two = dims->H_I > 32;
        e = dims->D == 128 ? (two ? launch_weights<128, 2>(c, lse, weights, sums) : launch_weights<128, 1>(c, lse, weights, sums))
                           : (two ? launch_weights<64, 2>(c, lse, weights, sums) : launch_weights<64, 1>(c, lse, weights, sums));
    }
    if (e == hipSuccess && sums) {
        hipLaunchKernelGGL(add_sums_kernel, dim3(blocks), dim3(256), 0, c.stream, sums, n, 1.0 / sums_per_unit(*dims), weights);
        e = hipGetLastError();
    }
    return report(e);
}

}  // extern "C"
