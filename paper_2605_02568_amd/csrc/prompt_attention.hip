// Dense attention of packed prompts (si_prompt_attention).
//
//   out[i,g,:] = sum_{s in seen(t)} exp(x_s - lse) V[s,h,:],  x_s = scale <q[i,g,:], K[s,h,:]>,  lse = ln sum exp(x_s),  t = first[b] + i
//
// Bound by the matrix pipe: 4 D operations a pair of query and row, whose rows all workgroups of a head find in their XCD's L2; with heads of 64, where an
// exponential comes with half as many operations, by the vector units beside it.  8,192 queries, causal, 64 heads of 128 on 8: 0.995 ms, 1,105 TFLOP/s (a product
// of 8192^3 by the library runs at 1,214, both at the clock that their power leaves); heads of 64: 0.59 ms, 920.
// The queries and heads that share a head of keys and values are the columns of one product (column r of a sequence: query r / G, head r % G
// of the group of G), 32 a wave, 128 or 256 a workgroup; so short prompts and large groups fill a workgroup, and the masked part of a tile
// on the diagonal is as small as 256 / G queries.  The workgroup's waves share tiles of 32 or 64 rows, which go straight from memory to LDS, one on its
// way while the one before is used (two on their way: 1 % slower).  Per block of 32 rows and wave:
//   S^T[32 rows x 32 columns] = K q^T       v_mfma_f32_32x32x16_bf16: a lane has 16 rows of one column, so a column's statistics are in-lane
//   p = exp2(x - m_ref)                     reference of a column raised (and the sums rescaled) only when a lane's sum of weights
//                                           passes 2^10; fp32
//   O^T[D x 32] += V^T P^T                  P^T is an operand straight from the registers of S^T (the rows' order inside the
//                                           contraction is the same on both sides), V^T comes from LDS by transposing reads
// p is rounded to bf16 for that product only (off by 2^-8 of itself at most); the sum of weights is of p itself.

#include <hip/hip_runtime.h>

#include <cmath>

#include "attention_set.h"
#include "dense.h"
#include "streamindex_prompt.h"
#include "wave_ops.h"

namespace si {

namespace {

constexpr int kSlots = 3;               // tiles in LDS: two in use, one on its way
constexpr float kMostWeight = 1024.0f;  // sum of a lane's weights of a block beyond which the reference is raised,
constexpr float kMostShift = 8.0f;      // or where the maximum is known, its distance from the reference in log2 units

struct Call {
    const __bf16* q;
    const __bf16* K;
    const __bf16* V;
    Packed queries, rows;
    const int32_t* first;
    __bf16* out;
    float* lse;
    float scale_log2e;
    int H, H_kv, G, m, mask_mode, n_win;
    int slots;  // of a workgroup's columns, of all sequences
    uint32_t by_G;  // 2^(31 + by_shift) / G, rounded up
    int by_shift;   // least with G <= 2^by_shift
    // x / G for 0 <= x < 2^30: by_G is too large by less than 1, which makes less than x / 2^(31 + by_shift) <= 1 / (2 G) of a quotient whose fraction is 1 / G below the next one
    __device__ __forceinline__ int over_G(int x) const { return static_cast<int>(__umulhi(2u * static_cast<uint32_t>(x), by_G) >> by_shift); }
};

// Orders the lanes of a wave's LDS accesses for the compiler; the hardware keeps a wave's LDS instructions in order.
__device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

typedef __attribute__((address_space(3))) unsigned char lds_byte;

// Starts a wave's loads of a tile, from the `bytes` bytes at k and at v: LOADS times 1 KB into LDS at `to` the keys, `apart` behind them the values (none
// where v is NULL).  A lane's first 16 bytes are at `offset`, the next ones 64 / (D / 8) rows of `stride` bytes further, where the swizzle of the row's number differs.
// What lies at or past `bytes` is not read and lands as zeros.
template <int D, int LOADS>
__device__ __forceinline__ void request_pieces(const __bf16* k, const __bf16* v, int bytes, int offset, int stride, lds_byte* to, int apart) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) void lds_void;
    constexpr int kStep = 64 / (D / 8);
    const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<__bf16*>(k), 0, bytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<__bf16*>(v), 0, bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int at = (offset ^ (row_swizzle<D>(i * kStep) * 16)) + i * kStep * stride;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void*)(to + i * 1024), 16, at, 0, 0, 0);
        if (v) __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void*)(to + apart + i * 1024), 16, at, 0, 0, 0);
    }
#else
    (void)k; (void)v; (void)bytes; (void)offset; (void)stride; (void)to; (void)apart;
#endif
}

// Both halves' values: of the exchange's two results one carries the lower half-wave's in both halves, the other the higher one's.
__device__ __forceinline__ floatx2 both_halves(float x) {
    const unsigned bits = __builtin_bit_cast(unsigned, x);
    const auto both = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    const unsigned low = both[0], high = both[1];  // not cast as they are: a cast of either element takes the first
    return floatx2{__builtin_bit_cast(float, low), __builtin_bit_cast(float, high)};
}
// A value that all lanes have, in a scalar register.
__device__ __forceinline__ float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }
// The lane's number where it is not worth a register through the loop.
__device__ __forceinline__ int lane_again() {
    int lane;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
    return lane;
}

// Tiles of keys and values; then 32 rows of 64 d of the results a wave, with the weights of 8 rows in the same place.  With heads of 64 the results go to the tiles' place,
// behind a barrier more, as three workgroups have to fit a compute unit.
template <int D>
constexpr int wave_bytes() { return D == 64 ? 8 * 32 * 4 : 32 * 128; }
template <int D, int kWaves, int kRows>
constexpr int lds_bytes() { return kSlots * 2 * kRows * D * 2 + kWaves * wave_bytes<D>(); }

// Grid: (slots of columns, the last ones first) x heads of keys and values, heads next to each other so that with 8 of them each has an XCD.  A sequence's
// slots begin at (its first packed column) / (columns of a workgroup) + (its number): slots enough for any lengths, with no sum over the sequences before.
template <int D, int kWaves, int kRows>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2)))
void prompt_attention_kernel(Call c) {
    constexpr int kColumns = 32 * kWaves;  // of a workgroup
    constexpr int KS = D / 16;      // steps along d of the first product
    constexpr int DB = D / 32;      // blocks of 32 rows of O^T
    constexpr int kRowBytes = D * 2;
    constexpr int kPieces = D / 8;  // 16-byte pieces of a row
    constexpr int kTileBytes = kRows * kRowBytes;
    constexpr int kLoads = kTileBytes / 1024 / kWaves;  // of a wave, of a tile's keys or values
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    lds_byte* const tiles = (lds_byte*)lds;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int col = lane & 31, half = lane >> 5;
    const int hk = blockIdx.x % c.H_kv;
    const int u = c.slots - 1 - blockIdx.x / c.H_kv;

    auto slot_of = [&](int at, int b) { return at * c.G / kColumns + b; };  // of sequence b, whose first packed query is `at`
    int b, q_first, q_last, k_first, k_last, first;
    if (c.queries.B < 64) {  // all that there is to know of the sequences, a lane each, in one trip
        const int i = min(lane, c.queries.B);
        const int q_at = c.queries.in_range(i), k_at = c.rows.in_range(i), before = c.first ? c.first[min(lane, c.queries.B - 1)] : 0;
        b = max(0, static_cast<int>(__popcll(__ballot(lane < c.queries.B && slot_of(q_at, lane) <= u))) - 1);
        q_first = lane_value(q_at, b);
        q_last = max(q_first, lane_value(q_at, b + 1));
        k_first = lane_value(k_at, b);
        k_last = max(k_first, lane_value(k_at, b + 1));
        first = lane_value(before, b);
    } else {
        b = last_not_above(c.queries.B, u, [&](int i) { return static_cast<int64_t>(slot_of(c.queries.in_range(i), i)); });
        c.queries.rows(b, q_first, q_last);
        c.rows.rows(b, k_first, k_last);
        first = c.first ? c.first[b] : 0;
    }
    const int n_columns = (q_last - q_first) * c.G;
    const int r0 = (u - slot_of(q_first, b)) * kColumns;
    if (r0 < 0 || r0 >= n_columns) return;
    const int held = k_last - k_first;

    // what this lane's column sees
    const int column = min(r0 + wave * 32 + col, n_columns - 1);  // columns that there are not repeat the last one
    const int query = c.over_G(column);
    const int legal = c.n_win > 0 ? legal_rows(first, query, held, c.m, c.mask_mode) : 0;
    const int from = max(0, legal - c.n_win);
    // What all columns of the wave see, and any: neither end falls from a column to the next.  Then any of the workgroup.
    const int any_from = lane_value(from, 0), all_from = lane_value(from, 31);
    const int all_to = lane_value(legal, 0), any_to = lane_value(legal, 31);
    const int last_query = c.over_G(min(r0 + kColumns, n_columns) - 1);
    const int end = c.n_win > 0 ? legal_rows(first, last_query, held, c.m, c.mask_mode) : 0;
    const int begin = max(0, legal_rows(first, c.over_G(r0), held, c.m, c.mask_mode) - c.n_win) / kRows * kRows;
    const int64_t q_row = static_cast<int64_t>(q_first + query) * c.H + hk * c.G + (column - query * c.G);

    // queries: lane has column col, d = 16 ks + 8 half .. + 7
    bf16x8 qf[KS];
    {
        const uintx4* const src = reinterpret_cast<const uintx4*>(c.q + q_row * D);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, src[2 * ks + half]);
    }

    // ---- a tile's keys and values, by 1 KiB pieces of LDS; rows at or past the last one that anybody sees land as zeros
    const int stride = c.H_kv * kRowBytes;
    static_assert(kLoads > 0 && (kLoads & (kLoads - 1)) == 0, "a load's number and a wave's first row share no bits");
    auto request = [&](int s0, lds_byte* to) {
        const int n = min(kRows, end - s0);
        const int bytes = (n - 1) * stride + kRowBytes;
        const int64_t at = (static_cast<int64_t>(k_first + s0) * c.H_kv + hk) * D;
        const unsigned lane2 = lane_again(), first_row = wave * kLoads * (64 / kPieces) + lane2 / kPieces;
        const int lane_offset = first_row * stride + ((lane2 % kPieces) ^ row_swizzle<D>(first_row)) * 16;
        request_pieces<D, kLoads>(c.K + at, c.V ? c.V + at : nullptr, bytes, lane_offset, stride, to + wave * kLoads * 1024, kTileBytes);
    };
    if (begin < end) request(begin, tiles);

    const float to_log2 = uniform(c.scale_log2e == 0.0f ? 1.0f : __builtin_fabsf(c.scale_log2e));
    const int apart = c.V ? kTileBytes : 0;  // values behind the keys, or the keys' rows
    // Places in a block, of which there is one number each: the others follow by exclusive or, as the swizzle is one and blocks begin at multiples of 256 bytes.
    // First product: row col, piece 2 ks + half.
    int key_at = tile_slot<D>(col, half) * 16;
    auto read_keys = [&](const lds_byte* block, int ks) {
        typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
        return *(lds_bf16x8*)((reinterpret_cast<uintptr_t>(block) + key_at) ^ (32 * ks));  // blocks begin at multiples of 256 bytes
    };
    // Second product, by transposing reads: source lane s of a group of 16 points at 4 consecutive d of row 4 half + s / 4 (+ 8; + 16 for the second part), at
    // d = 32 db + 16 (group % 2) + 4 (s % 4).
    int value_at = apart + tile_slot<D>(4 * half + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + (lane & 3) / 2) * 16 + (lane & 1) * 8;
    auto read_values = [&](const lds_byte* block, int i) {  // 16 rows of 32 d, by the place of their block's keys; i = s * DB + db
        typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
        const int s = i / DB, db = i % DB;
        const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(block + (value_at ^ (64 * db)) + s * 16 * kRowBytes));
        const bf16x4 v1 =
            __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(block + (value_at ^ (64 * db) ^ (row_swizzle<D>(8) * 16)) + (16 * s + 8) * kRowBytes));
        return bf16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
    };

    const floatx16 zero16 = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    floatx16 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = zero16;
    float shift = __builtin_huge_valf(), l_sum = 0.0f;  // minus the reference; no reference yet makes every weight too large or NaN

    // scores of a block of 32 rows: register j has row 8 (j / 4) + 4 half + j % 4
    auto score = [&](const lds_byte* block, floatx16& x) {
        x = zero16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_keys(block, ks), qf[ks], x, 0, 0, 0);
    };
    auto two_weights = [&](bf16x8 (&pf)[2], int j, float p0, float p1) {
        const bf16x2 two = __builtin_convertvector(floatx2{p0, p1}, bf16x2);
        pf[j / 8][j % 8] = two[0];
        pf[j / 8][j % 8 + 1] = two[1];
    };
    // The reference of the columns in `over` (bit i: column i) becomes at least `highest`, in log2 units.
    auto raise = [&](unsigned over, float highest) {
        const floatx2 of_halves = both_halves(highest);
        highest = fmaxf(of_halves[0], of_halves[1]);
        const float raised = (over >> (lane_again() & 31)) & 1 ? fminf(-highest, shift) : shift;
        const float alpha = raised == shift ? 1.0f : __builtin_amdgcn_exp2f(raised - shift);
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] *= alpha;
        l_sum *= alpha;
        shift = raised;
    };

    // A block of which some column does not see some row.
    auto take_masked = [&](int s0, const lds_byte* block) {
        floatx16 x;
        score(block, x);
        float highest = -__builtin_huge_valf();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int s = s0 + 8 * (j >> 2) + 4 * half + (j & 3);
            if (s < from || s >= legal) x[j] = -__builtin_huge_valf();
            highest = fmaxf(highest, x[j]);
        }
        highest *= to_log2;
        unsigned long long over = __ballot(!(highest + shift <= kMostShift));
        if (over != 0ull) raise(static_cast<unsigned>(over | (over >> 32)), highest);
        const float by = shift == __builtin_huge_valf() ? 0.0f : shift;  // a column that has seen nothing yet
        bf16x8 pf[2];
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            x[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], to_log2, by));
            x[j + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j + 1], to_log2, by));
            l_sum += x[j] + x[j + 1];
            two_weights(pf, j, x[j], x[j + 1]);
        }
        bf16x8 vf[2 * DB];
        unsigned found = 0;
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) {
            vf[i] = read_values(block, i);
            found |= not_finite(vf[i]);
        }
        // values that are not finite go in by themselves, row by row: 0 times a NaN must not enter a column that does not see it
        const bool odd = __ballot(found != 0) != 0ull;
        if (odd) {
#pragma unroll
            for (int i = 0; i < 2 * DB; ++i) vf[i] = finite_or_zero(vf[i]);
            float* const weights = reinterpret_cast<float*>(lds + kSlots * 2 * kTileBytes + wave * wave_bytes<D>());
            typedef __attribute__((address_space(3))) const bf16x4 lds_bf16x4;
#pragma unroll
            for (int part = 0; part < 4; ++part) {  // 8 rows at a time
#pragma unroll
                for (int j = 0; j < 4; ++j) weights[(4 * half + j) * 32 + col] = x[4 * part + j];
                wave_order();
#pragma unroll 1
                for (int r = 8 * part; r < 8 * part + 8; ++r) {
                    const float w = weights[(r & 7) * 32 + col];
                    const bool sees = s0 + r >= from && s0 + r < legal;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int a = 0; a < 4; ++a)
                            add_not_finite(acc[db], 4 * a, *(lds_bf16x4*)(block + apart + tile_slot<D>(r, 4 * db + a) * 16 + half * 8), w, sees);
                }
                wave_order();
            }
        }
        // contraction index e of part i / DB <-> row 16 (i / DB) + 8 (e / 4) + 4 half + e % 4 of the block on both operands
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], pf[i / DB], acc[i % DB], 0, 0, 0);
    };

    // The tile at s0 is there for all waves, and none uses the slot of the one after it; that is asked for.
    auto after = [&](lds_byte* slot) { return slot == tiles + (kSlots - 1) * 2 * kTileBytes ? tiles : slot + 2 * kTileBytes; };
    auto arrive = [&](int s0, lds_byte* slot_after) {
        __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's part of the tile
        __syncthreads();
        if (s0 + kRows < end) request(s0 + kRows, slot_after);
    };

    // Tiles that all columns see whole: a pipeline over blocks of 32 rows.  A step has block g's weights from its scores, while the matrix pipe
    // adds block g - 1's values and makes block g + 1's scores, instruction by instruction: after each product a part of the weights and a read from LDS
    // for a product half a step later.
    bf16x8 vf[2 * DB], pf[2];  // values of the block before, and its weights
    auto step = [&](const lds_byte* block, const lds_byte* next, floatx16& x, floatx16& xn) {
        constexpr int kProducts = KS + 2 * DB, kEach = 16 / kProducts;
        static_assert(KS == 2 * DB && kProducts * kEach == 16, "products and weights go together");
        asm volatile("" : "+v"(key_at), "+v"(value_at));  // the other places are made here, not kept in registers through the loop
        xn = zero16;
        bf16x8 kf[KS], pn[2];
        float p[16], sum = 0.0f;
#pragma unroll
        for (int n = 0; n < kProducts; ++n) {
            if (n < KS) {
                acc[n % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[n], pf[n / DB], acc[n % DB], 0, 0, 0);
                kf[n] = read_keys(next, n);
            } else {
                xn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[n - KS], qf[n - KS], xn, 0, 0, 0);
                vf[n - KS] = read_values(block, n - KS);
            }
#pragma unroll
            for (int e = n * kEach; e < (n + 1) * kEach; ++e) {
                p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], to_log2, shift));
                if (e > 0) sum += p[e - 1];
                if (e > 1 && e % 2 == 0) two_weights(pn, e - 2, p[e - 2], p[e - 1]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        sum += p[15];
        two_weights(pn, 14, p[14], p[15]);
        unsigned long long over = __ballot(!(sum <= kMostWeight));
        if (__builtin_expect(over != 0ull, 0)) {
            score(block, x);  // again: that costs the few blocks that come here less than keeping the scores costs all others
            float highest = x[0];
#pragma unroll
            for (int j = 1; j < 16; ++j) highest = fmaxf(highest, x[j]);
            raise(static_cast<unsigned>(over | (over >> 32)), highest * to_log2);
            const float by = shift == __builtin_huge_valf() ? 0.0f : shift;  // all scores so far are minus infinity
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], to_log2, by)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j + 1], to_log2, by));
                sum += p0;  // in the order of the products above: a column whose reference stays keeps its bits, whatever its neighbours need
                sum += p1;
                two_weights(pn, j, p0, p1);
            }
        }
        l_sum += sum;
        pf[0] = pn[0];
        pf[1] = pn[1];
    };

    // A tile, with its first block's scores in x; then x or y has those of the next tile's first block.  That tile is at `next`, and the one after it is asked
    // for, to `to`, which nothing in here reads, as the compiler has to know (__restrict__): else the transposing reads wait for all that is on its way to LDS
    // (four prompts of 33 to 300: 17.2 -> 16.6 us, 8,192 queries 1,026 -> 997, 23 prompts of up to 1,500 with heads of 64 180 -> 166).
    auto take_whole = [&](const lds_byte* now, const lds_byte* next, lds_byte* __restrict__ to, int s0, bool last, floatx16& x, floatx16& y) {
        if constexpr (kRows == 64) step(now, now + 32 * kRowBytes, x, y);
        if (!last) arrive(s0 + kRows, to);
        const lds_byte* const then = last ? now : next;  // behind the last block the scores are not used
        if constexpr (kRows == 64) step(now + 32 * kRowBytes, then, y, x);
        else step(now, then, x, y);
    };

    // The queries have arrived with the first tile.  A negative scale goes into them (exact), a scale of 0 makes zeros of them.
    int s0 = begin;
    lds_byte* tile = tiles;
    if (s0 < end) arrive(s0, after(tile));
    if (c.scale_log2e <= 0.0f) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (c.scale_log2e < 0.0f) qf[ks] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(uintx4, qf[ks]) ^ 0x80008000u);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) qf[ks][j] = static_cast<__bf16>(static_cast<float>(qf[ks][j]) * 0.0f);
        }
    }

    // Every wave meets every tile's barrier.
    const int whole_from = (all_from + kRows - 1) / kRows * kRows, whole_to = all_to / kRows * kRows;
    while (s0 < end) {
        if (s0 < whole_from || s0 >= whole_to) {
#pragma unroll 1
            for (int i = 0; i < kRows; i += 32, s0 += 32)
                if (s0 < any_to && s0 + 32 > any_from) take_masked(s0, tile + i * kRowBytes);
        } else {
            floatx16 x, y;
            score(tile, x);
#pragma unroll
            for (int i = 0; i < 2 * DB; ++i) vf[i] = __builtin_bit_cast(bf16x8, uintx4{0, 0, 0, 0});
            pf[0] = pf[1] = vf[0];
            auto take = [&](floatx16& x, floatx16& y) {
                const bool last = s0 + kRows >= whole_to;
                lds_byte* const next = after(tile);
                take_whole(tile, next, after(next), s0, last, x, y);
                s0 += kRows;
                if (!last) tile = next;
                return last;
            };
            if constexpr (kRows == 64) {
#pragma unroll 1
                while (!take(x, y)) {}
            } else {
                bool last = false;
                if (((whole_to - s0) / kRows) & 1) {
                    last = take(x, y);
                    x = y;
                }
#pragma unroll 1
                while (!last) {
                    take(x, y);
                    last = take(y, x);
                }
            }
#pragma unroll
            for (int i = 0; i < 2 * DB; ++i) acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], pf[i / DB], acc[i % DB], 0, 0, 0);
        }
        if (s0 < end) {
            tile = after(tile);
            arrive(s0, after(tile));
        }
    }
    const float m_ref = -shift;

    // ---- register j of block db = d row 32 db + 8 (j / 4) + 4 half + j % 4.  64 d of the wave's columns go through LDS, so that the results are
    // written by whole lines (four prompts of 33 to 300: 15.5 us; 8 bytes a lane and 32 rows at once: 17.0).
    const floatx2 l_halves = both_halves(l_sum);
    float l = l_halves[0] + l_halves[1];
    bool none = m_ref == -__builtin_huge_valf() && l == 0.0f;
    int r_first = r0 + wave * 32;
    const int lane2 = lane_again(), col2 = lane2 & 31, half2 = lane2 >> 5;
    asm volatile("" : "+s"(r_first));  // places are made again here, not kept in registers through the loop
    const int left = n_columns - r_first;  // columns that there are
    auto row_of = [&](int r) {  // of the results, for column r
        const int i_query = c.over_G(r);
        return static_cast<int64_t>(q_first + i_query) * c.H + hk * c.G + (r - i_query * c.G);
    };
    if (__builtin_expect(__ballot(none) != 0ull, 0)) {  // where rows are seen, all logits are minus infinity: NaN if it is the query that makes them so
        const int r = min(r_first + col2, n_columns - 1);
        const int to = c.n_win > 0 ? legal_rows(first, c.over_G(r), held, c.m, c.mask_mode) : 0;
        const bf16x8* const q = reinterpret_cast<const bf16x8*>(c.q + row_of(r) * D);
        unsigned found = 0;
#pragma unroll 1
        for (int ks = 0; ks < KS; ++ks) found |= not_finite(q[2 * ks + half2]);
        const unsigned long long odd = __ballot(found != 0);
        if (none && to > 0 && (static_cast<unsigned>(odd | odd >> 32) >> col2) & 1) {
            l = __builtin_nanf("");
            none = false;
        }
    }
    const float inv = none ? 0.0f : 1.0f / l;
    if (c.lse && half2 == 0 && col2 < left) c.lse[row_of(r_first + col2)] = none ? -__builtin_huge_valf() : log_of(m_ref, l);
    static_assert(kWaves * 32 * 128 <= kSlots * 2 * kTileBytes, "the tiles' place");
    unsigned char* const mine = lds + (D == 64 ? 0 : kSlots * 2 * kTileBytes) + wave * (32 * 128);
    if constexpr (D == 64) __syncthreads();  // all tiles have been read
#pragma unroll
    for (int db0 = 0; db0 < DB; db0 += 2) {
        wave_order();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = static_cast<__bf16>(acc[db0 + i][4 * a + e] * inv);
                *reinterpret_cast<bf16x4*>(mine + col2 * 128 + (((4 * i + a) ^ (col2 & 7)) * 16) + half2 * 8) = v;
            }
        wave_order();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * i + lane2 / 8, piece = lane2 % 8;
            const uintx4 v = *reinterpret_cast<const uintx4*>(mine + row * 128 + ((piece ^ (row & 7)) * 16));
            if (row < left) *reinterpret_cast<uintx4*>(c.out + row_of(r_first + row) * D + 32 * db0 + 8 * piece) = v;
        }
    }
}

template <int D, int kWaves, int kRows>
hipError_t launch(Call c, int64_t n_columns, hipStream_t stream) {
    static std::atomic<size_t> allowed[64];
    constexpr int kBytes = lds_bytes<D, kWaves, kRows>();
    const hipError_t e = allow_lds(prompt_attention_kernel<D, kWaves, kRows>, kBytes, allowed);
    if (e != hipSuccess) return e;
    c.slots = static_cast<int>(n_columns / (32 * kWaves) + c.queries.B);
    hipLaunchKernelGGL((prompt_attention_kernel<D, kWaves, kRows>), dim3(static_cast<unsigned>(c.slots) * c.H_kv), dim3(64 * kWaves), kBytes, stream, c);
    return hipGetLastError();
}

// Heads of 64: 128 columns a workgroup, so that three share a compute unit and one's start and end go by beside the others' products, and tiles of 64 rows (23 prompts
// of up to 1,500, 33 heads on 3: 159 us, 8,192 queries, 64 heads on 8: 597; tiles of 32 rows 164 and 610; 256 columns 177 and 612).
// Heads of 128: 256 columns and 64 rows, which load a tile for twice as many products (8,192 queries, 64 heads on 8: 993 us; the smaller form 1,037; 4 prompts of 4,000,
// 32 heads on 32: 575 and 594).  The smaller form, two a unit, where start and end count for more, as a sequence has few rows to see (16 prompts of 1,000: 391 -> 372 us,
// 300 of 100: 424 -> 322, 16,384 queries with a window of 128: 268 -> 206; 8 of 2,000: 597 and 600) or few columns, which leave more of 256 than of 128 without work (100
// parts of 100 queries behind 2,000: 866 -> 789; 30 of 500 behind 2,000: 1,075 and 1,117).  And where 256 columns would be fewer workgroups than compute units (1,024
// queries: 33.3 -> 30.2 us); where they would be fewer than half as many, 128 columns and 64 rows, of which one fits a unit, so that they spread (512 queries behind 8,192:
// 163 us in the smaller form, 156 in this; 300 behind 4,000: 79 and 74).
template <int D>
hipError_t launch(const Call& c, hipStream_t stream) {
    constexpr int kUnits = 256;
    const int64_t n_columns = static_cast<int64_t>(c.queries.N) * c.G;
    if constexpr (D == 64) {
        return launch<D, 4, 64>(c, n_columns, stream);
    } else {
        const int64_t sequences = c.queries.B, workgroups = std::max(n_columns / 256, sequences) * c.H_kv;
        const int64_t seen = std::min<int64_t>(c.n_win, c.rows.N / sequences);  // rows, by a sequence of mean length
        if (workgroups <= kUnits / 2) return launch<D, 4, 64>(c, n_columns, stream);
        if (workgroups <= kUnits || seen < 2048 || n_columns < 1024 * sequences) return launch<D, 4, 32>(c, n_columns, stream);
        return launch<D, 8, 64>(c, n_columns, stream);
    }
}

}  // namespace

}  // namespace si

using namespace si;

extern "C" {

si_status si_prompt_attention(const void* q, const void* K, const void* V, const si_packed_dims* dims, const int32_t* q_offsets,
                              const int32_t* k_offsets, const int32_t* first, int32_t m, si_mask_mode mask_mode, int32_t n_win, float scale,
                              void* out, float* lse, void* stream) {
    if (!q || !K || !dims || !out) return SI_ERR_INVALID_ARG;
    const si_packed_dims& d = *dims;
    if (d.B < 1 || d.N_q < 1 || d.N_k < 1 || d.H < 1 || d.H_kv < 1 || d.D < 1 || d.H % d.H_kv != 0 || m < 1 || n_win < 0) return SI_ERR_INVALID_ARG;
    if (mask_mode != SI_MASK_NONE && mask_mode != SI_MASK_CAUSAL_BLOCK) return SI_ERR_INVALID_ARG;
    if ((!q_offsets && d.N_q % d.B != 0) || (!k_offsets && d.N_k % d.B != 0)) return SI_ERR_INVALID_ARG;
    const float scale_log2e = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
    if (!std::isfinite(scale) || !std::isfinite(scale_log2e)) return SI_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(K) || !aligned16(V) || !aligned16(out)) return SI_ERR_INVALID_ARG;
    if (!aligned4(q_offsets) || !aligned4(k_offsets) || !aligned4(first) || !aligned4(lse)) return SI_ERR_INVALID_ARG;
    if ((d.D != 64 && d.D != 128) || d.H > 1024 || d.N_q > (1 << 30) || d.N_k > (1 << 30) || d.B > (1 << 20) ||
        static_cast<int64_t>(d.N_q) * d.H + int64_t{128} * d.B * d.H_kv >= (1 << 30))  // a launch has fewer than 2^32 threads
        return SI_ERR_UNSUPPORTED_SHAPE;
    const int G = d.H / d.H_kv;
    int shift = 0;
    while ((1 << shift) < G) ++shift;
    const Call c = {static_cast<const __bf16*>(q), static_cast<const __bf16*>(K), static_cast<const __bf16*>(V),
                    {q_offsets, d.B, d.N_q}, {k_offsets, d.B, d.N_k}, first, static_cast<__bf16*>(out), lse, scale_log2e,
                    d.H, d.H_kv, G, m, mask_mode, n_win, 0, static_cast<uint32_t>(((int64_t{1} << (31 + shift)) + G - 1) / G), shift};
    return report(d.D == 128 ? launch<128>(c, static_cast<hipStream_t>(stream)) : launch<64>(c, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
