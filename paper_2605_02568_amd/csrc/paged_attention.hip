// Attention of the newest positions of each sequence over the pages of a cache (si_paged_attention).
//
//   out[b,i,g,:] = sum_{s in seen(t)} exp(x_s - lse) V[s,h,:],  x_s = scale <q[b,i,g,:], K[s,h,:]>,  lse = ln sum exp(x_s),  t = first[b] + i
//
// The rows of a sequence are read once for up to 64 columns that share a head; each 64 columns more read them again, from the caches where they find them there
// (128 positions of 64 heads on 8: 16 workgroups a chunk and head).  So a call of few positions is bound by memory: 64 requests of 1,025 to 8,191 rows, 64 heads of 128 on 8, 16 bits: 1.21 GB in 205 us, 5.9 TB/s
// (loads alone reach 7.1 here).  Where 64 heads share one row of 8 bits, the vector units (36 % of the time) and the matrix pipe (18 %) take as long together as
// memory does: 8 requests of 65,536 to 131,072 rows: 203 MB in 59 us, of which the chunks' start, end and join take 18.
// The positions and heads that share a head of the cache are the columns of one product (column r: position r / G, head r % G of the group of G), 16, 32 or 64 of
// them a workgroup.
//
// The rows are dealt out on the device, as the host does not know the lengths: every wave adds up the sequences' tiles of 32 rows, makes
// chunks of them so that all sequences together have about as many chunks as the chip takes, and finds the sequence that its workgroup's chunk is of; where there
// are many sequences a kernel before does that for all.
// The 4 or 8 waves of a workgroup take the chunk's tiles in turn, each by itself with tiles on their way to a ring of its own in LDS, and join once at the end;
// chunks of the same sequence are joined by a second kernel.  Per tile and wave:
//   S^T[32 rows x 16 columns] = Ktile q^T   v_mfma_f32_16x16x32_bf16: a lane has 8 rows of one column; 8-bit codes become bf16 on the way from LDS, exactly
//   p = exp2(x - m_ref)                     reference of a column 0 to begin with, changed (and the sums rescaled) only when a lane's sum of weights passes
//                                           2^10, or on the first tile is below 2^-10; fp32
//   O^T[D x 16] += Vtile^T P^T              P^T is an operand straight from the registers of S^T (the rows' order inside the
//                                           contraction is the same on both sides), Vtile^T comes from the wave's own tile in LDS by transposing reads
// p, in 8 bits times the value's power of two, is rounded to bf16 for that product only (off by 2^-8 of itself at most); the sum of weights is of p itself.

#include <hip/hip_runtime.h>

#include <cmath>

#include "attention_set.h"
#include "dense.h"
#include "wave_ops.h"

namespace si {

namespace {

constexpr int kMinTiles = 8;            // of a chunk (4 or 16: one request of 2,048 rows as fast, no other call faster)
constexpr int kUnits = 256;             // compute units
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
    int2* chunks;       // [B]: a sequence's first chunk, and how many it has
    float scale_log2e;
    int B, S, H, H_kv, G, table_pages, n_pages, page_lg, m, mask_mode, n_win;
    int blocks;  // of columns
    int target;  // chunks that fit the chip at once
    int most_tiles;  // of what the positions of a sequence see
    bool one_each;   // a sequence is a chunk
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

// The chunk of a workgroup.
struct Chunk {
    int b;        // sequence, -1: there is no such chunk
    int first;    // the sequence's first chunk
    int n;        // chunks of the sequence
    int n_tiles;  // tiles of a chunk
};

// In how many rounds of workgroups the chunks may go through the chip.  A sequence's last chunk costs half of one, so where there are more sequences than an eighth
// of the chunks that fit at once, these may leave much of the chip idle; where there are twice as many sequences as such chunks, four rounds and more are needed anyway.
__host__ __device__ inline int most_rounds(int B, int target) { return 8 * static_cast<int64_t>(B) <= target ? 1 : B <= 2 * static_cast<int64_t>(target) ? 2 : 4; }

// x / n rounded up, for 0 <= x <= 2^25 and n >= kMinTiles: the quotient is at most 2^22 and three roundings of 2^-24 to 2^-23 off, less than 1, so its whole
// part is off by 1 at most, which the remainder tells.
__device__ __forceinline__ int over(int x, int n) {
    int q = static_cast<int>(static_cast<float>(x) * __builtin_amdgcn_rcpf(static_cast<float>(n)));
    int left = x - q * n;
    if (left <= -n) {
        --q;
        left += n;
    }
    return q + (left > 0) + (left > n);
}

// Tiles of a chunk, where all sequences together have `total` and count(n) is how many chunks they make of n tiles.  Chunks have as many tiles as it takes for all
// of them to fit the chip at once; where sequences of different lengths would make that more than a quarter longer than an even share, half as many, twice (64
// requests of 1,025 to 8,191 rows on 64 chunks: 223 us at once, 207 in two rounds; 24 of 77 to 5,003, where the length is little more than the share: 28 and 36).
// It is an even share at least, and kMinTiles, so there are at most as many chunks as fit in the rounds, and one more of each sequence.
template <typename Count>
__device__ __forceinline__ int chunk_length(const Call& c, int64_t total, Count count) {
    auto even_for = [&](int target) {
        const int64_t even = (total >> 31) ? (total + target - 1) / target : (static_cast<uint32_t>(total) + target - 1) / target;
        return static_cast<int>(min(max(static_cast<int64_t>(kMinTiles), even), int64_t{1} << 25));  // no sequence has more
    };
    auto length_for = [&](int target) {
        const int even = even_for(target);
        int n_tiles = even;
        for (int i = 0; i < 4; ++i) {
            const int n = count(n_tiles);
            if (n <= target) break;
            const float more = static_cast<float>(n_tiles) * static_cast<float>(n - target) * __builtin_amdgcn_rcpf(static_cast<float>(target));  // a guess
            n_tiles = min(2 * even, n_tiles + __builtin_amdgcn_readfirstlane(max(1, static_cast<int>(fminf(more, 1 << 25)))));
        }
        return n_tiles;
    };
    const int rounds = most_rounds(c.B, c.target);
    if (rounds == 4) return even_for(4 * c.target);
    const int n_tiles = length_for(c.target);
    return rounds == 1 || static_cast<int64_t>(n_tiles) * c.target * 4 <= 5 * total + 4 * kMinTiles * c.target ? n_tiles : length_for(2 * c.target);
}

constexpr int kFewSequences = 64;  // every wave deals them out for itself, a lane each; more are dealt out by a workgroup that does nothing else

// The chunk with number `which`.  All 64 lanes call it.
__device__ __forceinline__ Chunk find_chunk(const Call& c, int which) {
    auto parts_of = [&](int t, int n) { return static_cast<int>((static_cast<uint32_t>(t) + n - 1) / static_cast<uint32_t>(n)); };
    if (c.one_each) return {which < c.B ? which : -1, which, 1, which < c.B ? rows_of(c, which).tiles() : 0};
    if (c.B > kFewSequences) {
        const int b = last_not_above(c.B, which, [&](int i) { return static_cast<int64_t>(c.chunks[i].x); });
        const int2 chunk = c.chunks[b];
        return {which < chunk.x + chunk.y ? b : -1, chunk.x, chunk.y, parts_of(rows_of(c, b).tiles(), chunk.y)};
    }
    const int lane = threadIdx.x & 63;
    const int t = lane < c.B ? rows_of(c, lane).tiles() : 0;
    const int low = lane_value(wave_prefix_sum(t & 0xFFFF), 63), high = lane_value(wave_prefix_sum(t >> 16), 63);
    const int n_tiles = chunk_length(c, (static_cast<int64_t>(high) << 16) + low,
                                     [&](int n) { return lane_value(wave_prefix_sum(lane < c.B ? max(1, over(t, n)) : 0), 63); });
    const int mine = lane < c.B ? max(1, over(t, n_tiles)) : 0;
    const int upto = wave_prefix_sum(mine);
    if (which >= lane_value(upto, 63)) return {-1, 0, 0, 0};
    const int b = static_cast<int>(__popcll(__ballot(upto <= which)));
    const int n = lane_value(mine, b);
    return {b, lane_value(upto, b) - n, n, parts_of(lane_value(t, b), n)};
}

// The chunks of more sequences than kFewSequences: one workgroup, a thread up to 16 neighbouring ones.  1,024 requests of 256 rows, 64
// heads of 128 on 8: 190 us, 4,096 of 64 rows 317; where every wave added them up for itself 710 us and 8.9 ms (128 of 2,048 rows: 177 and 175).
__global__ __launch_bounds__(1024) void deal_chunks_kernel(Call c) {
    constexpr int kMost = kMaxSequences / 1024;
    __shared__ int s_sums[16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    auto scan = [&](int x, int& all) {  // sum up to this thread, and of all
        const int upto = wave_prefix_sum(x);
        if (lane == 63) s_sums[wave] = upto;
        __syncthreads();
        const int sums = wave_prefix_sum(lane < 16 ? s_sums[lane] : 0);
        __syncthreads();
        all = lane_value(sums, 15);
        return upto + (wave > 0 ? lane_value(sums, max(wave - 1, 0)) : 0);
    };
    const int per = (c.B + 1023) / 1024, b0 = static_cast<int>(threadIdx.x) * per;
    int t[kMost], low = 0, high = 0;  // lower 16 bits and the rest: 2^14 sequences of 2^25 tiles
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        t[i] = i < per && b0 + i < c.B ? rows_of(c, b0 + i).tiles() : -1;
        low += t[i] < 0 ? 0 : t[i] & 0xFFFF;
        high += t[i] < 0 ? 0 : t[i] >> 16;
    }
    auto parts = [&](int i, int n) { return t[i] < 0 ? 0 : max(1, over(t[i], n)); };
    auto mine_of = [&](int n) {
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kMost; ++i) mine += parts(i, n);
        return mine;
    };
    int all_low, all_high, all;
    scan(low, all_low);
    scan(high, all_high);
    const int n_tiles = chunk_length(c, (static_cast<int64_t>(all_high) << 16) + all_low, [&](int n) {
        scan(mine_of(n), all);
        return all;
    });
    const int mine = mine_of(n_tiles);
    int first = scan(mine, all) - mine;
#pragma unroll
    for (int i = 0; i < kMost; ++i)
        if (t[i] >= 0) {
            const int n = parts(i, n_tiles);
            c.chunks[b0 + i] = make_int2(first, n);
            first += n;
        }
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

// A tile on its way in LDS: keys, then values, then in 8 bits the scale bytes of either.
template <int D, int BITS>
struct Tile {
    static constexpr int kRowBytes = D * BITS / 8;
    static constexpr int kBytes = kTileKeys * kRowBytes;          // keys, or values
    static constexpr int kAll = 2 * kBytes + (BITS == 8 ? 256 : 0);
    static constexpr int kRing = 16384 / (2 * kBytes);            // tiles on the way: 16 KB a wave, 128 KB a compute unit
    static constexpr int kPieces = kRowBytes / 16;                // of a row
    static constexpr int kHalfLoads = kBytes / 2048;              // 1 KB loads of 16 rows
    static constexpr int kLoads = 4 * kHalfLoads + (BITS == 8);   // of a tile
    // Pieces of a row are swizzled so that lanes served together meet different banks: by the row reads of the first product (a piece of rows 0 .. 3 and 8 .. 11,
    // or of 8 rows in a row) and by the transposing reads of the second (two pieces of 4 rows; in 8 bits a piece of 8).
    __device__ static constexpr int swizzle(int row) {
        if constexpr (BITS == 16) return row_swizzle<D>(row);
        if constexpr (D == 128) return ((row >> 1) & 1) | ((row >> 2) & 2) | (row & 4);
        return ((row >> 3) & 1) | ((row >> 1) & 2);
    }
    __device__ static int place(int row, int piece) { return (row * kPieces + (piece ^ swizzle(row))) * 16; }
};
// A workgroup of NB blocks of 16 columns.  With one or two, 4 waves have the queries in registers, and two workgroups share a compute unit.  With four,
// 64 columns, 8 waves share one copy of the queries in LDS, as a wave's sums take half its registers.
template <int D, int BITS, int NB>
struct Group {
    using T = Tile<D, BITS>;
    static constexpr bool kSharedQueries = NB == 4;
    static constexpr int kWaves = NB == 4 ? 8 : 4;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kWaveBytes = T::kRing * T::kAll + 16 * 16 * 4;  // tiles; weights of 16 rows of a block, for values that are not finite
    static constexpr int kQueries = kWaves * kWaveBytes;                 // where the shared queries begin
    static constexpr int kAtOnce = NB == 4 ? 2 : NB;                     // blocks that are joined at once
    static constexpr int kJoin = kWaves * (kAtOnce * 16 * D + NB * 16 * 2) * 4;  // sums of each wave; its reference and sum of weights
    static constexpr int kColumns = kQueries + (kSharedQueries ? NB * 16 * D * 2 : 0);  // where the columns' table begins
    static constexpr int kBytes = kColumns + NB * 16 * 16;
    static_assert(kJoin <= kQueries && kBytes <= 160 * 1024, "LDS");
};

// Starts the loads of 16 rows of keys, or of values: `bytes` bytes from src on, to LDS at `to`, 1 KB at a time.  A load's rows follow the one's before, so its
// offset in memory and in LDS is the instruction's, and a lane's place among them, `offset`, changes by the swizzle of the rows' number only.
// What lies at or past `bytes` is not read and lands as zeros.  ONCE: no other workgroup of the sequence reads the rows, so they need not stay in the caches: 64 requests
// of 4,352 rows, 64 heads of 128 on 8, 16 bits: 175 us, without the hint 197; 8 bits 92 and 106.  Of pages that are in several tables the hint is the wrong one, and the
// host does not know of them: the same requests with 4,096 rows in common 58 and 53 us (8 bits 52 and 52), 16 with 16,384 in common and 512 of their own 76 and 47.
template <typename T, bool ONCE, int I = 0>
__device__ __forceinline__ void request_half(const char* src, int bytes, int offset, unsigned char* to) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) void lds_void;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(src), 0, bytes, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)to, 16, offset ^ (T::swizzle(I * (64 / T::kPieces)) * 16), 0, I * 1024, ONCE ? 2 : 0);
    if constexpr (I + 1 < T::kHalfLoads) request_half<T, ONCE, I + 1>(src, bytes, offset, to);
#else
    (void)src; (void)bytes; (void)offset; (void)to;
#endif
}
// One dword a lane, to LDS at `to` + 4 lane.
__device__ __forceinline__ void request_dword(const unsigned char* src, unsigned char* to) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) void lds_void;
    typedef __attribute__((address_space(1))) const void gbl_void;
    __builtin_amdgcn_global_load_lds((gbl_void*)src, (lds_void*)to, 4, 0, 0);
#else
    (void)src; (void)to;
#endif
}
// All but the last N of the wave's loads have arrived.
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N < 64, "a counter of 6 bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ unsigned lds_address(const unsigned char* p) {
    typedef __attribute__((address_space(3))) const unsigned char lds_byte;
    return static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_byte*)p));
}
// Transposing reads of 4 times 16 d of values, and the wait for them.  (As builtins they would wait for all loads on their way to LDS.)
// 16 bits: of rows 4 quarter .. + 3, and of the rows APART bytes behind; 8 bits: of rows 8 quarter .. + 7.
template <int APART>
__device__ __forceinline__ void read_columns(const unsigned (&at)[4], uintx2 (&lo)[4], uintx2 (&hi)[4]) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %4, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %1, %9\n\tds_read_b64_tr_b16 %5, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %2, %10\n\tds_read_b64_tr_b16 %6, %10 offset:%12\n\t"
        "ds_read_b64_tr_b16 %3, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(lo[0]), "=&v"(lo[1]), "=&v"(lo[2]), "=&v"(lo[3]), "=&v"(hi[0]), "=&v"(hi[1]), "=&v"(hi[2]), "=&v"(hi[3])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(APART)
        : "memory");
}
__device__ __forceinline__ void read_columns(const unsigned (&at)[4], uintx2 (&codes)[4]) {
    asm volatile(
        "ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %5\n\tds_read_b64_tr_b8 %2, %6\n\tds_read_b64_tr_b8 %3, %7\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(codes[0]), "=&v"(codes[1]), "=&v"(codes[2]), "=&v"(codes[3])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3])
        : "memory");
}

// Grid: (chunks x heads of the cache x column blocks), the blocks of a chunk and head on one XCD.
template <int D, int BITS, int NB>
__global__ __launch_bounds__((Group<D, BITS, NB>::kThreads)) __attribute__((amdgpu_waves_per_eu(2)))
void paged_attention_kernel(Call c) {
    using T = Tile<D, BITS>;
    using W = Group<D, BITS, NB>;
    constexpr int kWaves = W::kWaves;
    constexpr int kThreads = W::kThreads;
    constexpr int KS = D / 32;  // steps along d of the first product
    constexpr int DB = D / 16;  // blocks of 16 rows of O^T
    constexpr int kRing = T::kRing;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int col = lane & 15, quarter = lane >> 4;
    const int slot = blockIdx.x / 8;
    const int block = slot % c.blocks;
    const int item = (slot / c.blocks) * 8 + blockIdx.x % 8;
    const int hk = item % c.H_kv;
    const int which = item / c.H_kv;
    const Chunk chunk = find_chunk(c, which);
    if (chunk.b < 0) return;
    const int b = chunk.b;
    if (which == chunk.first && hk == 0 && block == 0 && threadIdx.x == 0 && c.B <= kFewSequences) c.chunks[b] = make_int2(chunk.first, chunk.n);

    const int R = c.S * c.G;
    const int held = held_rows(c, b);
    const int first = c.first ? c.first[b] : 0;
    const Rows rows = rows_of(c, b);
    const int first_tile = rows.lo / kTileKeys + (which - chunk.first) * chunk.n_tiles;
    const int last_tile = min(first_tile + chunk.n_tiles, rows.lo / kTileKeys + rows.tiles());
    const int n_mine = max(0, (last_tile - first_tile - wave + kWaves - 1) / kWaves);  // this wave's tiles: first_tile + wave, then every kWaves-th
    unsigned char* const ring = lds + wave * W::kWaveBytes;
    float* const weights_lds = reinterpret_cast<float*>(ring + kRing * T::kAll);

    // ---- tiles: 16 + 16 rows, each half in one page.  Lane i has the page of half i of the next 32 tiles.
    const int offset = lane / T::kPieces * T::kRowBytes + ((lane % T::kPieces) ^ T::swizzle(lane / T::kPieces)) * 16;
    int pages = 0;
    const auto request = [&](int k) {  // the wave's tile k, into its place of the ring; returns which rows some position sees
        if (k % 32 == 0) {
            const int s = (first_tile + wave + (k + lane / 2) * kWaves) * kTileKeys + 16 * (lane & 1);
            pages = c.table[static_cast<int64_t>(b) * c.table_pages + min(s >> c.page_lg, c.table_pages - 1)];
            asm volatile("" : "+v"(pages));  // waited for here, not wherever a page is looked up, where tiles would be waited for too
        }
        const int s0 = (first_tile + wave + k * kWaves) * kTileKeys;
        unsigned char* const to = ring + k % kRing * T::kAll;
        int64_t row[2];
        unsigned live = 0;
        int at = offset;
        asm volatile("" : "+v"(at));  // the swizzled places are made here, not kept in registers through the loop
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int s = s0 + 16 * u, page = __builtin_amdgcn_readlane(pages, 2 * (k % 32) + u);
            const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages);
            const int n = __builtin_amdgcn_readfirstlane(there ? min(max(rows.hi - s, 0), 16) : 0);
            row[u] = ((static_cast<int64_t>(there ? page : 0) * c.H_kv + hk) << c.page_lg) + (s & ((1 << c.page_lg) - 1));
            live |= (0xFFFFu >> (16 - n)) << (16 * u);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const char* const src = static_cast<const char*>(c.data[w]) + row[u] * T::kRowBytes;
                unsigned char* const half = to + w * T::kBytes + u * (T::kBytes / 2);
                if (NB == 1 || c.blocks == 1) request_half<T, true>(src, n * T::kRowBytes, at, half);
                else request_half<T, false>(src, n * T::kRowBytes, at, half);
            }
        }
        if constexpr (BITS == 8) {  // lanes 0 .. 7 the keys' scale bytes, 8 .. 15 the values'
            const unsigned char* const scales = (lane & 8) ? c.scales[1] : c.scales[0];
            request_dword(scales + ((lane & 4) ? row[1] : row[0]) + 4 * (lane & 3), to + 2 * T::kBytes);
        }
        return s0 < rows.lo ? live & (~0u << (rows.lo - s0)) : live;
    };
    unsigned live[kRing];
#pragma unroll
    for (int k = 0; k < kRing; ++k) live[k] = k < n_mine ? request(k) : 0u;

    // ---- what the columns see, and what all of them do: from the last position's first row to the first one's last
    // a column's query, the rows [y, z) that it sees, and its place among the sequence's results: every wave makes the same table, a lane a column
    // (the compiler has this store to LDS wait for all tiles on their way there, so the queries are asked for once the first tiles have landed)
    int4* const columns = reinterpret_cast<int4*>(lds + W::kColumns);
    if (lane < NB * 16) {
        const int r = min(block * NB * 16 + lane, R - 1), i = r / c.G;  // columns that there are not repeat the last one
        const int legal = legal_rows(first, i, held, c.m, c.mask_mode);
        columns[lane] = make_int4(i * c.H + hk * c.G + (r - i * c.G), max(0, legal - c.n_win), legal, 0);
    }
    wave_order();
    const int all_from = max(0, legal_rows(first, c.S - 1, held, c.m, c.mask_mode) - c.n_win);
    const int all_to = legal_rows(first, 0, held, c.m, c.mask_mode);

    // queries: lane has column col; step ks of the contraction is d = 32 ks + 8 quarter .. + 7 in 16 bits, and in 8, where a lane reads 16 codes of a row,
    // d = 64 (ks / 2) + 16 quarter + 8 (ks % 2) .. + 7.  A negative scale goes into the query (exact), a scale of 0 makes zeros of it.
    const float to_log2 = c.scale_log2e == 0.0f ? 1.0f : __builtin_fabsf(c.scale_log2e);
    auto query = [&](int row, int ks) {
        const int piece = BITS == 16 ? 4 * ks + quarter : 8 * (ks / 2) + 2 * quarter + ks % 2;
        uintx4 raw = reinterpret_cast<const uintx4*>(c.q + (static_cast<int64_t>(b) * c.S * c.H + row) * D)[piece];
        if (c.scale_log2e < 0.0f) raw ^= 0x80008000u;
        bf16x8 q = __builtin_bit_cast(bf16x8, raw);
        if (c.scale_log2e == 0.0f)
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = static_cast<__bf16>(static_cast<float>(q[j]) * 0.0f);
        return q;
    };
    bf16x8 kept[W::kSharedQueries ? 1 : NB][KS];
    bf16x8* const shared = reinterpret_cast<bf16x8*>(lds + W::kQueries) + lane;  // [nb][ks][lane]
    if constexpr (W::kSharedQueries) {
        constexpr int kEach = NB * KS / kWaves;
        bf16x8 mine[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) mine[i] = query(columns[(i * kWaves + wave) / KS * 16 + col].x, (i * kWaves + wave) % KS);
#pragma unroll
        for (int i = 0; i < kEach; ++i) shared[(i * kWaves + wave) * 64] = mine[i];
        wait_lds();
        __builtin_amdgcn_s_barrier();
    } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int row = columns[nb * 16 + col].x;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kept[nb][ks] = query(row, ks);
        }
    }
    auto query_of = [&](int nb, int ks) {
        if constexpr (W::kSharedQueries) return shared[(nb * KS + ks) * 64];
        else return kept[nb][ks];
    };

    // Row of the tile that score j of a lane is of: half j / 4 of the matrix instruction's rows has, in 16 bits, the tile's rows in order, so that a
    // lane's rows are 4 quarter .. + 3 of either half; in 8 bits rows 8 (r / 4) + 4 (j / 4) + r % 4, so that they are 8 in a row, as the transposing
    // read of 8 bits wants them.
    auto row_of = [&](int j) { return BITS == 16 ? 16 * (j >> 2) + 4 * quarter + (j & 3) : 8 * quarter + j; };
    int key_at[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) key_at[u] = T::place(BITS == 16 ? 16 * u + col : 8 * (col >> 2) + 4 * u + (col & 3), quarter);
    // transposing reads: source lane s of 16 points, in 16 bits, at 4 consecutive d of row 4 quarter + s / 4, in 8 at 8 consecutive d of row 8 quarter + s / 2
    const int value_at = BITS == 16 ? T::place(4 * quarter + (col >> 2), (col & 3) / 2) + (col & 1) * 8 : T::place(8 * quarter + (col >> 1), 0) + (col & 1) * 8;

    floatx4 acc[NB][DB];
    // minus the reference.  It begins as 0, which stays wherever the first tile's weights are neither too large nor too small, as they mostly are; where a
    // column has seen nothing yet it is infinite, which makes every weight too large or NaN.
    float shift[NB], l_sum[NB], least = 1.0f / kMostWeight;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        shift[nb] = n_mine > 0 ? 0.0f : __builtin_huge_valf();
        l_sum[nb] = 0.0f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[nb][db] = floatx4{0, 0, 0, 0};
    }

#pragma unroll 1
    for (int k = 0; k < n_mine; ++k) {
        if (k + kRing <= n_mine) wait_loads<(kRing - 1) * T::kLoads>();
        else wait_loads<0>();
        const int s0 = (first_tile + wave + k * kWaves) * kTileKeys;
        int at_ring = k % kRing * T::kAll;
        asm volatile("" : "+s"(at_ring));  // addresses in the tile are made where they are needed, not kept in registers through the loop
        const unsigned char* const tile = ring + at_ring;
        const bool masked = live[0] != 0xFFFFFFFFu || s0 < all_from || s0 + kTileKeys > all_to;

        floatx4 x[NB][2];
        auto rows_seen = [&](int nb) {  // of the tile, by this column
            const int4 r = columns[nb * 16 + col];
            const int lo = r.y - s0, hi = r.z - s0;
            unsigned mine = live[0];
            if (lo > 0) mine &= lo >= kTileKeys ? 0u : ~0u << lo;
            if (hi < kTileKeys) mine &= hi <= 0 ? 0u : ~0u >> (kTileKeys - hi);
            return mine;
        };
        auto scores = [&]() {
            float power[2] = {1.0f, 1.0f};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if constexpr (BITS == 8) power[u] = scale_power(tile[2 * T::kBytes + 8 * (col >> 2) + 4 * u + (col & 3)]);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) x[nb][u] = floatx4{0, 0, 0, 0};
            }
#pragma unroll
            for (int j = 0; j < KS / 2; ++j) {  // two steps at a time, which is what 16 codes are
                bf16x8 kf[2][2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if constexpr (BITS == 16) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) kf[u][i] = *reinterpret_cast<const bf16x8*>(tile + (key_at[u] ^ (64 * (2 * j + i))));
                    } else {
                        uintx4 two[2];
                        codes_to_bf16(*reinterpret_cast<const uintx4*>(tile + (key_at[u] ^ (64 * j))), power[u], two);
                        kf[u][0] = __builtin_bit_cast(bf16x8, two[0]);
                        kf[u][1] = __builtin_bit_cast(bf16x8, two[1]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const bf16x8 q = query_of(nb, 2 * j + i);
#pragma unroll
                        for (int u = 0; u < 2; ++u) x[nb][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u][i], q, x[nb][u], 0, 0, 0);
                    }
                if (NB == 4) __builtin_amdgcn_sched_barrier(0);  // no operands further ahead: there are no registers for them
            }
            if (masked) {
                float low = -__builtin_huge_valf();
                asm volatile("" : "+v"(low));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const unsigned mine = rows_seen(nb) >> row_of(0);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!((mine >> (row_of(j) - row_of(0))) & 1)) x[nb][j >> 2][j & 3] = low;
                }
            }
        };
        // weights, in place of the scores
        float sum[NB];
        auto exponentials = [&](int nb, float by) {
            sum[nb] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[nb][j >> 2][j & 3] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[nb][j >> 2][j & 3], to_log2, by));
                sum[nb] += x[nb][j >> 2][j & 3];
            }
        };
        scores();
        bool over = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            exponentials(nb, shift[nb]);
            over |= !(sum[nb] <= kMostWeight && sum[nb] >= least);
        }
        if (__builtin_expect(__ballot(over) != 0ull, 0)) {
            // the scores again: that costs the few tiles that come here less than keeping them costs all others
            scores();
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                unsigned long long raise = __ballot(!(sum[nb] <= kMostWeight && sum[nb] >= least));
                raise |= raise >> 32;
                raise |= raise >> 16;  // bit i: column i, in any quarter
                float highest = x[nb][0][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) highest = fmaxf(highest, x[nb][j >> 2][j & 3]);
                highest = quarters_max(highest * to_log2);
                // on the first tile the reference may fall, too; there is nothing yet to rescale
                const float raised = (raise >> col) & 1 ? (k == 0 ? -highest : fminf(-highest, shift[nb])) : shift[nb];
                const float alpha = k == 0 || raised == shift[nb] ? 1.0f : __builtin_amdgcn_exp2f(raised - shift[nb]);
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[nb][db] *= alpha;
                l_sum[nb] *= alpha;
                shift[nb] = raised;
                float by = raised == __builtin_huge_valf() ? 0.0f : raised;  // a column that has seen nothing yet
                // or rows whose logits are all minus infinity: NaN if the query is what makes them so
                const bool sees = raised == __builtin_huge_valf() && rows_seen(nb) != 0;
                if (__ballot(sees) != 0ull) {
                    unsigned found = 0;
#pragma unroll 1
                    for (int ks = 0; ks < KS; ++ks) {
                        if constexpr (W::kSharedQueries) found |= not_finite(query_of(nb, ks));
                        else found |= not_finite(query(columns[nb * 16 + col].x, ks));
                    }
                    unsigned long long odd = __ballot(found != 0);
                    odd |= odd >> 32;
                    odd |= odd >> 16;
                    if (sees && (odd >> col) & 1) by = __builtin_nanf("");
                }
                exponentials(nb, by);
            }
        }
        float powers[8];  // of the values: they go into the weights, which is exact
        if constexpr (BITS == 8) {
            const unsigned alive = live[0] >> row_of(0);
            const uintx2 bytes = *reinterpret_cast<const uintx2*>(tile + 2 * T::kBytes + kTileKeys + 8 * quarter);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                powers[j] = scale_power((bytes[j >> 2] >> (8 * (j & 3))) & 0xFF);
                if (masked && !((alive >> j) & 1)) powers[j] = 0.0f;  // a row that nobody sees may have any scale byte
            }
        }
        bf16x8 pf[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            l_sum[nb] += sum[nb];
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                float p0 = x[nb][j >> 2][j & 3], p1 = x[nb][j >> 2][(j & 3) + 1];
                if constexpr (BITS == 8) {
                    p0 *= powers[j];
                    p1 *= powers[j + 1];
                }
                const bf16x2 two = __builtin_convertvector(floatx2{p0, p1}, bf16x2);
                pf[nb][j] = two[0];
                pf[nb][j + 1] = two[1];
            }
        }

        // contraction index j <-> row_of(j) on both operands
        const unsigned at = lds_address(tile + T::kBytes);
#pragma unroll
        for (int db0 = 0; db0 < DB; db0 += 4) {
            unsigned from_lds[4];
            bf16x8 vf[4];
            unsigned found = 0;
            if constexpr (BITS == 16) {
                uintx2 lo[4], hi[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) from_lds[i] = at + (value_at ^ (32 * (db0 + i)));
                read_columns<16 * T::kRowBytes>(from_lds, lo, hi);
#pragma unroll
                for (int i = 0; i < 4; ++i) vf[i] = __builtin_bit_cast(bf16x8, uintx4{lo[i][0], lo[i][1], hi[i][0], hi[i][1]});
                if (masked)
#pragma unroll
                    for (int i = 0; i < 4; ++i) found |= not_finite(vf[i]);
            } else {
                uintx2 codes[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) from_lds[i] = at + (value_at ^ (16 * (db0 + i)));
                read_columns(from_lds, codes);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uintx4 out[2];
                    codes_to_bf16(uintx4{codes[i][0], codes[i][1], 0, 0}, 1.0f, out);
                    vf[i] = __builtin_bit_cast(bf16x8, out[0]);
                    if (masked)
#pragma unroll
                        for (int w = 0; w < 2; ++w) found |= ((codes[i][w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
                }
            }
            // values that are not finite go in by themselves, row by row: 0 times a NaN must not enter a column that does not see it
            if (masked && __ballot(found != 0) != 0ull) {
#pragma unroll
                for (int i = 0; i < 4; ++i) vf[i] = finite_or_zero(vf[i]);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const unsigned mine = rows_seen(nb);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {  // 16 rows at a time: weights j of half u
#pragma unroll
                        for (int j = 0; j < 4; ++j) weights_lds[(4 * quarter + j) * 16 + col] = static_cast<float>(pf[nb][4 * u + j]);
                        wave_order();
#pragma unroll 1
                        for (int n = 0; n < 16; ++n) {
                            const int r = BITS == 16 ? 16 * u + n : 8 * (n >> 2) + 4 * u + (n & 3);
                            const float w = weights_lds[n * 16 + col];
                            const bool sees = (mine >> r) & 1;
                            const unsigned char* const values = tile + T::kBytes;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                bf16x4 v;
                                if constexpr (BITS == 16) {
                                    v = *reinterpret_cast<const bf16x4*>(values + T::place(r, 2 * (db0 + i) + quarter / 2) + (quarter & 1) * 8);
                                } else {
                                    uintx4 out[2];
                                    codes_to_bf16(uintx4{*reinterpret_cast<const unsigned*>(values + T::place(r, db0 + i) + 4 * quarter), 0, 0, 0}, 1.0f, out);
                                    const bf16x8 eight = __builtin_bit_cast(bf16x8, out[0]);
                                    v = bf16x4{eight[0], eight[1], eight[2], eight[3]};
                                }
                                add_not_finite(acc[nb][db0 + i], 0, v, w, sees);
                            }
                        }
                        wave_order();
                    }
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nb][db0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], pf[nb], acc[nb][db0 + i], 0, 0, 0);
        }
        least = 0.0f;
        wait_lds();  // the tile has been read: its place is free
#pragma unroll
        for (int i = 1; i < kRing; ++i) live[i - 1] = live[i];
        live[kRing - 1] = k + kRing < n_mine ? request(k + kRing) : 0u;
    }

    // ---- the workgroup's waves join.  The barriers wait for LDS only, not for what goes to memory.
    auto barrier = [&]() {
        wait_lds();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr int N = W::kAtOnce;                                                   // blocks of columns
    float* const join = reinterpret_cast<float*>(lds);                              // [wave][column][D]
    floatx2* const parts = reinterpret_cast<floatx2*>(join + kWaves * N * 16 * D);  // [column][wave]: minus the reference, sum of weights
    barrier();  // all tiles have been read
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const float l = quarters_sum(l_sum[nb]);
        if (quarter == 0) parts[(nb * 16 + col) * kWaves + wave] = floatx2{shift[nb], l};
    }
#pragma unroll
    for (int nb0 = 0; nb0 < NB; nb0 += N) {
        if (nb0 > 0) barrier();
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int db = 0; db < DB; ++db)
                *reinterpret_cast<floatx4*>(join + (wave * N * 16 + i * 16 + col) * D + (((4 * db + quarter) ^ (col & 7)) * 4)) = acc[nb0 + i][db];
        barrier();
#pragma unroll
        for (int i0 = 0; i0 < N * 16 * (D / 4); i0 += kThreads) {
            const int i = i0 + static_cast<int>(threadIdx.x);
            const int column = i / (D / 4), piece = i % (D / 4);
            if (i >= N * 16 * (D / 4) || (block * NB + nb0) * 16 + column >= R) continue;
            floatx2 part[kWaves], sums = {__builtin_huge_valf(), 0.0f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                part[w] = parts[(nb0 * 16 + column) * kWaves + w];
                sums[0] = fminf(sums[0], part[w][0]);
            }
            floatx4 o = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const floatx4 x = *reinterpret_cast<const floatx4*>(join + (w * N * 16 + column) * D + ((piece ^ (column & 7)) * 4));
                const float alpha = part[w][0] == sums[0] ? 1.0f : __builtin_amdgcn_exp2f(sums[0] - part[w][0]);  // 0 where the wave saw nothing
                sums[1] = __builtin_fmaf(alpha, part[w][1], sums[1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(alpha, x[e], o[e]);
            }
            const int place = columns[nb0 * 16 + column].x;
            if (chunk.n == 1) {
                const int64_t row = static_cast<int64_t>(b) * c.S * c.H + place;
                const bool none = sums[0] == __builtin_huge_valf() && sums[1] == 0.0f;
                const float inv = none ? 0.0f : 1.0f / sums[1];
                bf16x4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = static_cast<__bf16>(o[j] * inv);
                *reinterpret_cast<bf16x4*>(c.out + row * D + 4 * piece) = v;
                if (c.lse && piece == 0) c.lse[row] = none ? -__builtin_huge_valf() : log_of(-sums[0], sums[1]);
            } else {
                const int64_t row = static_cast<int64_t>(which) * c.S * c.H + place;
                *reinterpret_cast<floatx4*>(c.parts_out + row * D + 4 * piece) = o;
                if (piece == 0) *reinterpret_cast<floatx2*>(c.parts_sums + row * 2) = floatx2{-sums[0], sums[1]};
            }
        }
    }
}

// Chunks of a sequence together.  SPLIT waves take a query's head, each every SPLIT-th chunk.
template <int D, int SPLIT>
__global__ __launch_bounds__(256) void join_chunks_kernel(Call c) {
    constexpr int kPer = D / 64;  // values a lane
    __shared__ float s_top[4], s_sum[4], s_out[4][D];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int per = c.S * c.H;
    const int row = blockIdx.x * (4 / SPLIT) + wave / SPLIT;  // (b * S + i) * H + head
    const int part_of = wave % SPLIT;
    const int2 chunks = row < c.B * per ? c.chunks[row / per] : make_int2(0, 0);
    const int n = __builtin_amdgcn_readfirstlane(chunks.y);
    if (SPLIT == 1 ? n <= 1 : __syncthreads_or(n > 1) == 0) return;  // written by its workgroup
    const int64_t part0 = static_cast<int64_t>(chunks.x) * per + row % per;
    float top = -__builtin_huge_valf(), l = 0.0f, o[kPer] = {};
    constexpr int kAtOnce = 8;
    for (int i0 = part_of; i0 < n; i0 += SPLIT * kAtOnce) {
        float m[kAtOnce], sums[kAtOnce], x[kAtOnce][kPer];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int64_t part = part0 + static_cast<int64_t>(min(i0 + SPLIT * j, n - 1)) * per;
            const floatx2 two = *reinterpret_cast<const floatx2*>(c.parts_sums + part * 2);
            m[j] = two[0];
            sums[j] = two[1];
#pragma unroll
            for (int e = 0; e < kPer; ++e) x[j][e] = c.parts_out[part * D + lane * kPer + e];
        }
        float highest = top;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) highest = fmaxf(highest, m[j]);
        const float shift = highest == -__builtin_huge_valf() ? 0.0f : highest;
        const float before = top == highest ? 1.0f : __builtin_amdgcn_exp2f(top - shift);
        l *= before;
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] *= before;
        top = highest;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (i0 + SPLIT * j < n) {
                const float a = m[j] == top ? 1.0f : __builtin_amdgcn_exp2f(m[j] - shift);
                l += a * sums[j];
#pragma unroll
                for (int e = 0; e < kPer; ++e) o[e] += a * x[j][e];
            }
    }
    if constexpr (SPLIT > 1) {
        if (lane == 0) {
            s_top[wave] = top;
            s_sum[wave] = l;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) s_out[wave][lane * kPer + e] = o[e];
        __syncthreads();
        if (part_of != 0 || n <= 1) return;
#pragma unroll
        for (int w = 1; w < SPLIT; ++w) top = fmaxf(top, s_top[wave + w]);
        const float shift = top == -__builtin_huge_valf() ? 0.0f : top;
        const float own = s_top[wave] == top ? 1.0f : __builtin_amdgcn_exp2f(s_top[wave] - shift);
        l *= own;
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] *= own;
#pragma unroll
        for (int w = 1; w < SPLIT; ++w) {
            const float a = s_top[wave + w] == top ? 1.0f : __builtin_amdgcn_exp2f(s_top[wave + w] - shift);
            l += a * s_sum[wave + w];
#pragma unroll
            for (int e = 0; e < kPer; ++e) o[e] += a * s_out[wave + w][lane * kPer + e];
        }
    }
    const float inv = top == -__builtin_huge_valf() && l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < kPer; ++e) c.out[static_cast<int64_t>(row) * D + lane * kPer + e] = static_cast<__bf16>(o[e] * inv);
    if (c.lse && lane == 0) c.lse[row] = inv == 0.0f ? -__builtin_huge_valf() : log_of(top, l);
}

// Blocks of 16 columns a wave takes, workgroups side by side, and chunks of all sequences: as few blocks as have all columns, as every further workgroup reads
// the rows again (64 columns, 8 requests of 65,536 to 131,072 rows of 8 bits: 65 us at once, 75 in two workgroups of 32).
struct Shape {
    int nb, blocks, target;
};
Shape shape_of(int S, int H, int H_kv) {
    const int R = S * (H / H_kv);
    const int nb = R <= 16 ? 1 : R <= 32 ? 2 : 4;
    const int blocks = (R + 16 * nb - 1) / (16 * nb);
    const int at_once = nb == 4 ? kUnits : 2 * kUnits;  // workgroups that fit the chip
    return {nb, blocks, std::max(1, at_once / (H_kv * blocks))};
}

// Chunks that there may be.
int64_t parts_of(int B, int target) { return static_cast<int64_t>(most_rounds(B, target)) * target + B; }

bool fits(int32_t B, int32_t S, int32_t H) { return H <= 1024 && static_cast<int64_t>(B) * S <= (1 << 22) && static_cast<int64_t>(B) * S * H <= (1 << 22); }

template <int D, int BITS, int NB>
hipError_t launch(const Call& c, hipStream_t stream) {
    static std::atomic<size_t> allowed[64];
    using W = Group<D, BITS, NB>;
    hipError_t e = allow_lds(paged_attention_kernel<D, BITS, NB>, W::kBytes, allowed);
    if (e != hipSuccess) return e;
    const int64_t chunks = c.one_each ? c.B : std::min<int64_t>(parts_of(c.B, c.target), static_cast<int64_t>(c.B) * ((c.most_tiles + kMinTiles - 1) / kMinTiles));
    if (!c.one_each && c.B > kFewSequences) {
        hipLaunchKernelGGL(deal_chunks_kernel, dim3(1), dim3(1024), 0, stream, c);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int64_t items = chunks * c.H_kv;
    const unsigned grid = static_cast<unsigned>((items + 7) / 8 * 8 * c.blocks);
    hipLaunchKernelGGL((paged_attention_kernel<D, BITS, NB>), dim3(grid), dim3(W::kThreads), W::kBytes, stream, c);
    e = hipGetLastError();
    if (e != hipSuccess || c.one_each) return e;
    // Four waves a query's head where a sequence has more than 8 chunks, which is what one wave asks for at a time (8 requests of 32 chunks each: 59 us, with one
    // wave 63; where there are few chunks the other way round: 64 requests of one to four 207 us, with four waves 211; 24 of two or three 28 and 32).
    const int rows = c.B * c.S * c.H;
    if (c.target > 8 * c.B) hipLaunchKernelGGL((join_chunks_kernel<D, 4>), dim3(rows), dim3(256), 0, stream, c);
    else hipLaunchKernelGGL((join_chunks_kernel<D, 1>), dim3((rows + 3) / 4), dim3(256), 0, stream, c);
    return hipGetLastError();
}

}  // namespace

}  // namespace si

using namespace si;

extern "C" {

size_t si_paged_workspace_bytes(int32_t B, int32_t S, int32_t H, int32_t H_kv, int32_t D) {
    if (B < 1 || S < 1 || H < 1 || H_kv < 1 || D < 1 || H % H_kv != 0 || B > kMaxSequences || !fits(B, S, H)) return 0;
    return static_cast<size_t>(parts_of(B, shape_of(S, H, H_kv).target)) * S * H * (D + 2) * sizeof(float) + B * sizeof(int2);
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
    // S positions see n_win + S - 1 rows at most, all of them together: rows that begin and end inside a tile
    const int64_t held = static_cast<int64_t>(cache->table_pages) * cache->page_rows, seen = static_cast<int64_t>(n_win) + S - 1;
    const int64_t most_tiles = std::min((held + kTileKeys - 1) / kTileKeys, (seen + 2 * kTileKeys - 2) / kTileKeys);
    // Sequences of so few tiles stay whole, which takes one launch instead of two (64 heads of 128 on 8, 512 rows: 14.6 -> 10.1 us, 1,024 rows 13.6 -> 11.2, 64 requests of
    // them 45 -> 43; 2,048 rows 14.7 and 17.5).  With 64 columns a tile takes longer (512 rows 16.1 -> 13.7, 1,024 rows 16.9 and 18.2).
    const bool one_each = most_tiles <= (shape.nb == 4 ? 16 : 32);
    int lg = 0;
    while ((1 << lg) < cache->page_rows) ++lg;
    float* const parts = static_cast<float*>(workspace);
    const size_t n_parts = static_cast<size_t>(parts_of(cache->B, shape.target));
    // Where keys are the values, rows are asked for twice, the second time mostly from the caches: 64 requests of 1,025 to 8,191 rows, 64 heads of 128 on 8, take 123 us in 16
    // bits and 84 in 8, with values of their own 198 and 112; where 64 heads share a head of 8 bits the loads are not what bounds it (50 and 53 us).
    const Call c = {static_cast<const __bf16*>(q),
                    {cache->K, cache->V ? cache->V : cache->K},
                    {static_cast<const unsigned char*>(cache->K_scales), static_cast<const unsigned char*>(cache->V ? cache->V_scales : cache->K_scales)},
                    cache->table, lengths, first, static_cast<__bf16*>(out), lse,
                    parts, parts + n_parts * S * H * cache->D, reinterpret_cast<int2*>(parts + n_parts * S * H * (cache->D + 2)),
                    scale_log2e, cache->B, S, H, cache->H_kv, H / cache->H_kv, cache->table_pages, cache->n_pages, lg, m, mask_mode, n_win,
                    shape.blocks, shape.target, static_cast<int>(most_tiles), one_each};
    const hipStream_t st = static_cast<hipStream_t>(stream);
#define SI_LAUNCH(DD, BITS) report(shape.nb == 1 ? launch<DD, BITS, 1>(c, st) : shape.nb == 2 ? launch<DD, BITS, 2>(c, st) : launch<DD, BITS, 4>(c, st))
    if (cache->bits == 16) return cache->D == 128 ? SI_LAUNCH(128, 16) : SI_LAUNCH(64, 16);
    return cache->D == 128 ? SI_LAUNCH(128, 8) : SI_LAUNCH(64, 8);
#undef SI_LAUNCH
}

}  // extern "C"
