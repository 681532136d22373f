// Attention of the newest positions of each sequence over the pages of a cache (si_paged_attention).
//
//   out[b,i,g,:] = sum_{s in seen(t)} exp(x_s - lse) V[s,h,:],  x_s = scale <q[b,i,g,:], K[s,h,:]>,  lse = ln sum exp(x_s),  t = first[b] + i
//
// All rows of a sequence are read once, so a call is bound by memory.  The positions and heads that share a head of the cache are the
// columns of one product (column r: position r / G, head r % G of the group of G), 16 or 32 of them a workgroup.
//
// The rows are dealt out on the device, as the host does not know the lengths: every wave adds up the sequences' tiles of 32 rows, makes
// chunks of them so that all sequences together have about as many chunks as the chip takes, and finds the sequence that its workgroup's chunk is of.
// The waves of a workgroup take the chunk's tiles in turn, each by itself, and join once at the end; chunks of the same sequence are
// joined by a second kernel.  Per tile and wave:
//   S^T[32 rows x 16 columns] = Ktile q^T   v_mfma_f32_16x16x32_bf16 from registers: a lane has 8 rows of one column
//   p = exp2(x - m_ref)                     reference of a column raised (and the sums rescaled) only when a lane's sum of weights
//                                           passes 2^10; fp32
//   O^T[D x 16] += Vtile^T P^T              P^T is an operand straight from the registers of S^T (the rows' order inside the
//                                           contraction is the same on both sides), Vtile^T comes from the wave's own tile in LDS by transposing reads
// p is rounded to bf16 for that product only; the sum of weights is of p itself.

#include <hip/hip_runtime.h>

#include <cmath>

#include "attention_set.h"
#include "dense.h"
#include "wave_ops.h"

namespace si {

namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kMinTiles = kWaves;       // of a chunk: one a wave
constexpr int kWorkgroups = 1024;       // about as many in all
constexpr float kMostWeight = 1024.0f;  // sum of a lane's weights of a tile beyond which the reference is raised
constexpr int kMaxSequences = 1 << 14;

struct Call {
    const __bf16* q;
    const void* data[2];
    const unsigned char* scales[2];
    const int32_t* table;
    const int32_t* lengths;
    const int32_t* first;
    __bf16* out;
    float* lse;
    float* parts_out;   // [parts][S * H][D], not divided by their sums
    float* parts_sums;  // [parts][S * H][2]: reference, sum
    float scale_log2e;
    int B, S, H, H_kv, G, table_pages, n_pages, page_lg, m, mask_mode, n_win;
    int blocks;  // of columns
    int target;  // chunks of all sequences, beside one more of each
};

// Rows that the positions of sequence b see: [lo, hi) all of them together.
struct Rows {
    int lo, hi;
    __device__ int tiles() const { return hi > lo ? (hi + kTileKeys - 1) / kTileKeys - lo / kTileKeys : 0; }
};
__device__ __forceinline__ int held_rows(const Call& c, int b) {
    const int most = c.table_pages << c.page_lg;
    return c.lengths ? min(max(c.lengths[b], 0), most) : most;
}
__device__ __forceinline__ Rows rows_of(const Call& c, int b) {
    const int held = held_rows(c, b);
    const int first = c.first ? c.first[b] : 0;
    return {max(0, legal_rows(first, 0, held, c.m, c.mask_mode) - c.n_win), c.n_win > 0 ? legal_rows(first, c.S - 1, held, c.m, c.mask_mode) : 0};
}

// The chunk of a workgroup, or the chunks of a sequence.
struct Chunk {
    int b;         // sequence, -1: there is no such chunk
    int first;     // the sequence's first chunk
    int n;         // chunks of the sequence
    int n_tiles;   // tiles of a chunk
};
__device__ __forceinline__ int tiles_of_chunks(const Call& c) {
    const int lane = threadIdx.x & 63;
    int low = 0, high = 0;  // sums of the tiles' lower 16 bits and of the rest: 2^14 sequences of 2^25 tiles
    for (int b = lane; b < c.B; b += 64) {
        const int t = rows_of(c, b).tiles();
        low += t & 0xFFFF;
        high += t >> 16;
    }
    low = lane_value(wave_prefix_sum(low), 63);
    high = lane_value(wave_prefix_sum(high), 63);
    const int64_t total = (static_cast<int64_t>(high) << 16) + low;
    return static_cast<int>(max(static_cast<int64_t>(kMinTiles), (total + c.target - 1) / c.target));
}
__device__ __forceinline__ int chunks_of(const Call& c, int b, int n_tiles) { return max(1, (rows_of(c, b).tiles() + n_tiles - 1) / n_tiles); }

// by_chunk: the sequence that chunk `i` is of; otherwise sequence i's.
__device__ __forceinline__ Chunk find_chunk(const Call& c, int i, bool by_chunk) {
    const int lane = threadIdx.x & 63;
    const int n_tiles = tiles_of_chunks(c);
    int before = 0;
    for (int b0 = 0; b0 < c.B; b0 += 64) {
        const int mine = b0 + lane < c.B ? chunks_of(c, b0 + lane, n_tiles) : 0;
        const int upto = wave_prefix_sum(mine);
        const int all = lane_value(upto, 63);
        if (by_chunk ? i < before + all : i < b0 + 64) {
            const int l = by_chunk ? static_cast<int>(__popcll(__ballot(before + upto <= i))) : i - b0;
            const int n = lane_value(mine, l);
            return {b0 + l, before + lane_value(upto, l) - n, n, n_tiles};
        }
        before += all;
    }
    return {-1, 0, 0, n_tiles};
}

// Value that lanes l, l ^ 16, l ^ 32 and l ^ 48 hold the most, or the sum, of.
__device__ __forceinline__ float quarters_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quarters_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// Orders the lanes of a wave's LDS accesses for the compiler; the hardware keeps a wave's LDS instructions in order.
__device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

template <int D, int NB>
constexpr int lds_bytes() {
    constexpr int kTiles = kWaves * kTileKeys * D * 2;          // a tile of values a wave
    constexpr int kWeights = kWaves * kTileKeys * 16 * 4;       // weights of a column block, for rows of values that are not finite
    constexpr int kJoin = kWaves * NB * 16 * (D + 2) * 4;       // sums, reference and sum of weights of each wave
    return kTiles + kWeights > kJoin ? kTiles + kWeights : kJoin;
}

// Grid: (chunks x heads of the cache x column blocks), the blocks of a chunk and head on one XCD.
template <int D, int BITS, int NB>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void paged_attention_kernel(Call c) {
    constexpr int KS = D / 32;                  // steps along d of the first product
    constexpr int DB = D / 16;                  // blocks of 16 rows of O^T
    constexpr int kRowBytes = D * 2;            // in LDS
    constexpr int kLoads = BITS == 16 ? 2 * KS : KS;   // 16-byte loads a lane of a tile's keys, or of its values
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int col = lane & 15, quarter = lane >> 4;
    const int slot = blockIdx.x / 8;
    const int block = slot % c.blocks;
    const int item = (slot / c.blocks) * 8 + blockIdx.x % 8;
    const int hk = item % c.H_kv;
    const int which = item / c.H_kv;
    const Chunk chunk = find_chunk(c, which, true);
    if (chunk.b < 0) return;
    const int b = chunk.b;

    // what the columns see
    const int R = c.S * c.G;
    const int held = held_rows(c, b);
    const int first = c.first ? c.first[b] : 0;
    const Rows rows = rows_of(c, b);
    int legal[NB], from[NB], q_row[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = min((block * NB + nb) * 16 + col, R - 1);  // columns that there are not repeat the last one
        const int i = r / c.G;
        legal[nb] = legal_rows(first, i, held, c.m, c.mask_mode);
        from[nb] = max(0, legal[nb] - c.n_win);
        q_row[nb] = (b * c.S + i) * c.H + hk * c.G + r % c.G;
    }
    // rows that all positions see: from the last one's first to the first one's last
    const int all_from = max(0, legal_rows(first, c.S - 1, held, c.m, c.mask_mode) - c.n_win);
    const int all_to = legal_rows(first, 0, held, c.m, c.mask_mode);

    // queries: lane has column col; step ks of the contraction is d = 32 ks + 8 quarter .. + 7 in 16 bits, and in 8, where a lane loads 16 codes of a row,
    // d = 64 (ks / 2) + 16 quarter + 8 (ks % 2) .. + 7.  A negative scale goes into the query (exact), a scale of 0 makes zeros of it.
    float to_log2 = __builtin_fabsf(c.scale_log2e);
    bf16x8 qf[NB][KS];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const uintx4* const src = reinterpret_cast<const uintx4*>(c.q + static_cast<int64_t>(q_row[nb]) * D);
        const unsigned sign = c.scale_log2e < 0.0f ? 0x80008000u : 0u;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int piece = BITS == 16 ? 4 * ks + quarter : 8 * (ks / 2) + 2 * quarter + ks % 2;
            qf[nb][ks] = __builtin_bit_cast(bf16x8, src[piece] ^ sign);
        }
    }
    if (to_log2 == 0.0f) {
        to_log2 = 1.0f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int j = 0; j < 8; ++j) qf[nb][ks][j] = static_cast<__bf16>(static_cast<float>(qf[nb][ks][j]) * 0.0f);
    }

    const int first_tile = rows.lo / kTileKeys + (which - chunk.first) * chunk.n_tiles;
    const int last_tile = min(first_tile + chunk.n_tiles, rows.lo / kTileKeys + rows.tiles());

    unsigned char* const tile_lds = lds + wave * (kTileKeys * kRowBytes);
    float* const weights_lds = reinterpret_cast<float*>(lds + kWaves * kTileKeys * kRowBytes) + wave * (kTileKeys * 16);

    // A tile's rows are 16 + 16, each half in one page.
    struct Place {
        int64_t row[2];  // of the pages' arrays
        bool there[2];
    };
    auto place = [&](int tile) {
        Place p;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int s = tile * kTileKeys + 16 * u;
            const int page = c.table[static_cast<int64_t>(b) * c.table_pages + min(s >> c.page_lg, c.table_pages - 1)];
            p.there[u] = static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages);
            p.row[u] = ((static_cast<int64_t>(p.there[u] ? page : 0) * c.H_kv + hk) << c.page_lg) + (s & ((1 << c.page_lg) - 1));
        }
        return p;
    };
    // keys: lane has row col (+ 16 u), quarter's pieces of it
    uintx4 kraw[kLoads];
    int kpower[2];
    auto load_keys = [&](const Place& p) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uintx4* const src = static_cast<const uintx4*>(c.data[0]) + (p.row[u] + col) * (D * BITS / 128);
#pragma unroll
            for (int j = 0; j < kLoads / 2; ++j) kraw[u * (kLoads / 2) + j] = src[4 * j + quarter];
            if constexpr (BITS == 8) kpower[u] = c.scales[0][p.row[u] + col];
        }
    };
    // values: a wave's load j has the 64 consecutive 16-byte units of the tile from 64 j on
    uintx4 vraw[kLoads];
    int vpower[kLoads];
    constexpr int kUnits = D * BITS / 128;  // of a row
    auto load_values = [&](const Place& p) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int u = j / (kLoads / 2), unit = (j % (kLoads / 2)) * 64 + lane;
            vraw[j] = (static_cast<const uintx4*>(c.data[1]) + p.row[u] * kUnits)[unit];
            if constexpr (BITS == 8) vpower[j] = c.scales[1][p.row[u] + unit / kUnits];
        }
    };
    auto values_to_lds = [&](unsigned live) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int unit = (j % (kLoads / 2)) * 64 + lane, r = j / (kLoads / 2) * 16 + unit / kUnits, piece = unit % kUnits;
            uintx4 x[2] = {vraw[j], vraw[j]};
            if constexpr (BITS == 8) codes_to_bf16(vraw[j], scale_power(vpower[j]), x);
            if (live != 0xFFFFFFFFu && !((live >> r) & 1)) x[0] = x[1] = uintx4{0, 0, 0, 0};  // rows that no position sees may hold anything
            if constexpr (BITS == 16) {
                *reinterpret_cast<uintx4*>(tile_lds + tile_slot<D>(r, piece) * 16) = x[0];
            } else {
                *reinterpret_cast<uintx4*>(tile_lds + tile_slot<D>(r, 2 * piece) * 16) = x[0];
                *reinterpret_cast<uintx4*>(tile_lds + tile_slot<D>(r, 2 * piece + 1) * 16) = x[1];
            }
        }
    };
    // transposing read of 16 d of 4 rows by 16 lanes: lane s of the 16 points at 4 consecutive d of row 4 quarter + s / 4, and gets d = s of the four rows
    const int vat = tile_slot<D>(4 * quarter + (col >> 2), (col & 3) / 2) * 16 + (col & 1) * 8;

    floatx4 acc[NB][DB];
    float m_ref[NB], l_sum[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        m_ref[nb] = -__builtin_huge_valf();
        l_sum[nb] = 0.0f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[nb][db] = floatx4{0, 0, 0, 0};
    }

    Place here = {};
    if (first_tile + wave < last_tile) {
        here = place(first_tile + wave);
        load_keys(here);
        load_values(here);
    }
    for (int tile = first_tile + wave; tile < last_tile; tile += kWaves) {
        const int s0 = tile * kTileKeys;
        const bool more = tile + kWaves < last_tile;
        const Place then = more ? place(tile + kWaves) : here;
        // rows that some position sees
        unsigned live = (here.there[0] ? 0xFFFFu : 0u) | (here.there[1] ? 0xFFFF0000u : 0u);
        if (s0 < rows.lo) live &= ~0u << (rows.lo - s0);
        if (s0 + kTileKeys > rows.hi) live &= ~0u >> (s0 + kTileKeys - rows.hi);
        const bool masked = live != 0xFFFFFFFFu || s0 < all_from || s0 + kTileKeys > all_to;
        here = then;

        floatx4 x[NB][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uintx4 kf[KS];
            if constexpr (BITS == 16) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kf[ks] = kraw[u * KS + ks];
            } else {
#pragma unroll
                for (int j = 0; j < KS / 2; ++j) {
                    uintx4 two[2];
                    codes_to_bf16(kraw[u * (KS / 2) + j], scale_power(kpower[u]), two);
                    kf[2 * j] = two[0];
                    kf[2 * j + 1] = two[1];
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                x[nb][u] = floatx4{0, 0, 0, 0};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    x[nb][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[ks]), qf[nb][ks], x[nb][u], 0, 0, 0);
            }
        }
        if (more) load_keys(then);
        wave_order();  // the tile before has been read
        values_to_lds(live);
        if (more) load_values(then);
        wave_order();

        bool odd_values = false;
        if (masked) {
            // values that are not finite, of rows that some position sees and another may not
            bool odd = false;
#pragma unroll
            for (int j = 0; j < kTileKeys * kRowBytes / 1024; ++j) {
                const uintx4 v = *reinterpret_cast<const uintx4*>(tile_lds + (j * 64 + lane) * 16);
                odd |= not_finite(__builtin_bit_cast(bf16x8, v)) != 0;
            }
            odd_values = __ballot(odd) != 0ull;
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            unsigned mine = 0xFFFFFFFFu;  // rows that this column sees
            if (masked) {
                mine = live;
                const int lo = from[nb] - s0, hi = legal[nb] - s0;
                if (lo > 0) mine &= lo >= kTileKeys ? 0u : ~0u << lo;
                if (hi < kTileKeys) mine &= hi <= 0 ? 0u : ~0u >> (kTileKeys - hi);
                float low = -__builtin_huge_valf();
                asm volatile("" : "+v"(low));
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!((mine >> (16 * (j >> 2) + 4 * quarter + (j & 3))) & 1)) x[nb][j >> 2][j & 3] = low;
            }
            float p[8], sum;
            auto exponentials = [&]() {
                const float shift = m_ref[nb] == -__builtin_huge_valf() ? 0.0f : -m_ref[nb];
                sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[nb][j >> 2][j & 3], to_log2, shift));
                    sum += p[j];
                }
            };
            exponentials();
            unsigned long long over = __ballot(!(sum <= kMostWeight) || m_ref[nb] == -__builtin_huge_valf());
            if (over != 0ull) {
                over |= over >> 32;
                over |= over >> 16;  // bit i: column i, in any quarter
                float highest = x[nb][0][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) highest = fmaxf(highest, x[nb][j >> 2][j & 3]);
                highest = quarters_max(highest * to_log2);
                const float m_new = (over >> col) & 1 ? fmaxf(highest, m_ref[nb]) : m_ref[nb];
                const float alpha = m_new == m_ref[nb] ? 1.0f : __builtin_amdgcn_exp2f(m_ref[nb] - m_new);
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[nb][db] *= alpha;
                l_sum[nb] *= alpha;
                m_ref[nb] = m_new;
                exponentials();
            }
            l_sum[nb] += sum;
            bf16x8 pf;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x2 two = __builtin_convertvector(floatx2{p[2 * j], p[2 * j + 1]}, bf16x2);
                pf[2 * j] = two[0];
                pf[2 * j + 1] = two[1];
            }
            // contraction index e <-> tile row 16 (e / 4) + 4 quarter + e % 4 on both operands
            auto values = [&](int db) {
                typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
                const unsigned char* const at = tile_lds + (vat ^ (32 * db));
                const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)at);
                const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + 16 * kRowBytes));
                return bf16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            };
            if (!odd_values) {
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values(db), pf, acc[nb][db], 0, 0, 0);
            } else {
                // values that are not finite by themselves, row by row: 0 times a NaN must not enter a column that does not see it
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    acc[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(finite_or_zero(values(db)), pf, acc[nb][db], 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 8; ++j) weights_lds[(16 * (j >> 2) + 4 * quarter + (j & 3)) * 16 + col] = p[j];
                wave_order();
#pragma unroll 1
                for (int r = 0; r < kTileKeys; ++r) {
                    const float w = weights_lds[r * 16 + col];
                    const bool sees = (mine >> r) & 1;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
                        add_not_finite(acc[nb][db], 0, *reinterpret_cast<const bf16x4*>(tile_lds + tile_slot<D>(r, 2 * db + quarter / 2) * 16 + (quarter & 1) * 8),
                                       w, sees);
                }
                wave_order();
            }
        }
    }

    // ---- the workgroup's waves join: references, then sums
    __syncthreads();
    float* const join = reinterpret_cast<float*>(lds);                    // [wave][column][D]
    float* const join_sums = join + kWaves * NB * 16 * D;                 // [wave][column][2]
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int column = nb * 16 + col;
        const float l = quarters_sum(l_sum[nb]);
        if (quarter == 0) {
            join_sums[(wave * NB * 16 + column) * 2] = m_ref[nb];
            join_sums[(wave * NB * 16 + column) * 2 + 1] = l;
        }
#pragma unroll
        for (int db = 0; db < DB; ++db)
            *reinterpret_cast<floatx4*>(join + (wave * NB * 16 + column) * D + (((4 * db + quarter) ^ (col & 7)) * 4)) = acc[nb][db];
    }
    __syncthreads();
    const bool whole = chunk.n == 1;
    for (int i = threadIdx.x; i < NB * 16 * (D / 4); i += kThreads) {
        const int column = i / (D / 4), piece = i % (D / 4);
        const int r = block * NB * 16 + column;
        if (r >= R) continue;
        float top = -__builtin_huge_valf();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, join_sums[(w * NB * 16 + column) * 2]);
        const float shift = top == -__builtin_huge_valf() ? 0.0f : top;
        float l = 0.0f;
        floatx4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float part = join_sums[(w * NB * 16 + column) * 2];
            const float a = part == top ? 1.0f : __builtin_amdgcn_exp2f(part - shift);
            l += a * join_sums[(w * NB * 16 + column) * 2 + 1];
            o += a * *reinterpret_cast<const floatx4*>(join + (w * NB * 16 + column) * D + ((piece ^ (column & 7)) * 4));
        }
        const int position = r / c.G, head = hk * c.G + r % c.G;
        if (whole) {
            const int64_t row = (static_cast<int64_t>(b) * c.S + position) * c.H + head;
            const float inv = top == -__builtin_huge_valf() && l == 0.0f ? 0.0f : 1.0f / l;
            bf16x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = static_cast<__bf16>(o[j] * inv);
            *reinterpret_cast<bf16x4*>(c.out + row * D + 4 * piece) = v;
            if (c.lse && piece == 0) c.lse[row] = inv == 0.0f ? -__builtin_huge_valf() : log_of(top, l);
        } else {
            const int64_t row = static_cast<int64_t>(which) * c.S * c.H + position * c.H + head;
            *reinterpret_cast<floatx4*>(c.parts_out + row * D + 4 * piece) = o;
            if (piece == 0) {
                c.parts_sums[row * 2] = top;
                c.parts_sums[row * 2 + 1] = l;
            }
        }
    }
}

// Chunks of a sequence together: a wave a query's head.
template <int D>
__global__ __launch_bounds__(256) void join_chunks_kernel(Call c) {
    const int lane = threadIdx.x & 63;
    const int row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // (b * S + i) * H + head
    const int per = c.S * c.H;
    if (row >= c.B * per) return;
    const int b = row / per;
    const Chunk chunk = find_chunk(c, b, false);
    if (chunk.n <= 1) return;  // written by its workgroup
    const int64_t part0 = static_cast<int64_t>(chunk.first) * per + row % per;
    float top = -__builtin_huge_valf();
    for (int i = lane; i < chunk.n; i += 64) top = fmaxf(top, c.parts_sums[(part0 + static_cast<int64_t>(i) * per) * 2]);
    top = wave_max(top);
    const float shift = top == -__builtin_huge_valf() ? 0.0f : top;
    float l = 0.0f, o[D / 64] = {};
    for (int i = 0; i < chunk.n; ++i) {
        const int64_t part = part0 + static_cast<int64_t>(i) * per;
        const float m = c.parts_sums[part * 2];
        const float a = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - shift);
        l += a * c.parts_sums[part * 2 + 1];
#pragma unroll
        for (int j = 0; j < D / 64; ++j) o[j] += a * c.parts_out[part * D + lane * (D / 64) + j];
    }
    const float inv = top == -__builtin_huge_valf() && l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) c.out[static_cast<int64_t>(row) * D + lane * (D / 64) + j] = static_cast<__bf16>(o[j] * inv);
    if (c.lse && lane == 0) c.lse[row] = inv == 0.0f ? -__builtin_huge_valf() : log_of(top, l);
}

// Blocks of 16 columns a wave takes, blocks of a call and chunks of all sequences.
struct Shape {
    int nb, blocks, target;
};
Shape shape_of(int S, int H, int H_kv) {
    const int R = S * (H / H_kv);
    const int nb = R <= 16 ? 1 : 2;
    const int blocks = (R + 16 * nb - 1) / (16 * nb);
    return {nb, blocks, std::max(1, (kWorkgroups + H_kv * blocks - 1) / (H_kv * blocks))};
}

bool fits(int32_t B, int32_t S, int32_t H) { return H <= 1024 && static_cast<int64_t>(B) * S <= (1 << 22) && static_cast<int64_t>(B) * S * H <= (1 << 22); }

template <int D, int BITS, int NB>
hipError_t launch(const Call& c, hipStream_t stream) {
    static std::atomic<size_t> allowed[64];
    constexpr int kBytes = lds_bytes<D, NB>();
    hipError_t e = allow_lds(paged_attention_kernel<D, BITS, NB>, kBytes, allowed);
    if (e != hipSuccess) return e;
    const int64_t most_tiles = ((static_cast<int64_t>(c.table_pages) << c.page_lg) + kTileKeys - 1) / kTileKeys;
    const bool one_each = most_tiles <= kMinTiles;  // no sequence can have two chunks
    const int64_t items = static_cast<int64_t>(one_each ? c.B : c.target + c.B) * c.H_kv;
    const unsigned grid = static_cast<unsigned>((items + 7) / 8 * 8 * c.blocks);
    hipLaunchKernelGGL((paged_attention_kernel<D, BITS, NB>), dim3(grid), dim3(kThreads), kBytes, stream, c);
    e = hipGetLastError();
    if (e != hipSuccess || one_each) return e;
    hipLaunchKernelGGL((join_chunks_kernel<D>), dim3((c.B * c.S * c.H + 3) / 4), dim3(256), 0, stream, c);
    return hipGetLastError();
}

}  // namespace

}  // namespace si

using namespace si;

extern "C" {

size_t si_paged_workspace_bytes(int32_t B, int32_t S, int32_t H, int32_t H_kv, int32_t D) {
    if (B < 1 || S < 1 || H < 1 || H_kv < 1 || D < 1 || H % H_kv != 0 || B > kMaxSequences || !fits(B, S, H)) return 0;
    return static_cast<size_t>(shape_of(S, H, H_kv).target + B) * S * H * (D + 2) * sizeof(float);
}

si_status si_paged_attention(const void* q, const si_paged_cache* cache, int32_t S, int32_t H, const int32_t* lengths, const int32_t* first,
                             int32_t m, si_mask_mode mask_mode, int32_t n_win, float scale, void* out, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream) {
    const si_status ok = check_cache(cache);
    if (ok == SI_ERR_INVALID_ARG) return ok;
    if (!q || !out || !workspace || S < 1 || H < 1 || H % cache->H_kv != 0 || m < 1 || n_win < 0) return SI_ERR_INVALID_ARG;
    if (mask_mode != SI_MASK_NONE && mask_mode != SI_MASK_CAUSAL_BLOCK) return SI_ERR_INVALID_ARG;
    const float scale_log2e = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
    if (!std::isfinite(scale) || !std::isfinite(scale_log2e)) return SI_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) || !aligned4(lengths) || !aligned4(first) || !aligned4(lse)) return SI_ERR_INVALID_ARG;
    if (ok != SI_OK) return ok;
    if (cache->B > kMaxSequences || !fits(cache->B, S, H)) return SI_ERR_UNSUPPORTED_SHAPE;
    if (workspace_bytes < si_paged_workspace_bytes(cache->B, S, H, cache->H_kv, cache->D)) return SI_ERR_WORKSPACE_TOO_SMALL;
    const Shape shape = shape_of(S, H, cache->H_kv);
    int lg = 0;
    while ((1 << lg) < cache->page_rows) ++lg;
    float* const parts = static_cast<float*>(workspace);
    const Call c = {static_cast<const __bf16*>(q),
                    {cache->K, cache->V ? cache->V : cache->K},
                    {static_cast<const unsigned char*>(cache->K_scales), static_cast<const unsigned char*>(cache->V ? cache->V_scales : cache->K_scales)},
                    cache->table, lengths, first, static_cast<__bf16*>(out), lse,
                    parts, parts + static_cast<size_t>(shape.target + cache->B) * S * H * cache->D,
                    scale_log2e, cache->B, S, H, cache->H_kv, H / cache->H_kv, cache->table_pages, cache->n_pages, lg, m, mask_mode, n_win,
                    shape.blocks, shape.target};
    const hipStream_t st = static_cast<hipStream_t>(stream);
#define SI_LAUNCH(DD, BITS) report(shape.nb == 1 ? launch<DD, BITS, 1>(c, st) : launch<DD, BITS, 2>(c, st))
    if (cache->bits == 16) return cache->D == 128 ? SI_LAUNCH(128, 16) : SI_LAUNCH(64, 16);
    return cache->D == 128 ? SI_LAUNCH(128, 8) : SI_LAUNCH(64, 8);
#undef SI_LAUNCH
}

}  // extern "C"
