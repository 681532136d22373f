// Eviction (si_evict_rows): of the n rows that a batch holds, the first n_sink, the last n_recent and those with the largest
// weights stay, n_keep in all, and the arrays that belong to the rows are compacted in order.
//
// A weight is compared as a 32-bit word whose unsigned order is that of the weights: NaN 0, then -inf .. +inf, and rows that
// always stay above all.  The n_keep-th largest word of a batch is found by radix descent over 11, 11 and 10 bits; rows above it
// stay, and of those that equal it as many of the first as there is room for.  Then each workgroup takes a chunk of rows, lists those that stay
// (where its list begins is known from the counts of the chunks before it) and copies what belongs to them.
//
// The copies bound it: 2 * n_keep * (bytes of a row in all arrays).

#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_call.h"
#include "si_internal.h"
#include "streamindex_cache.h"
#include "wave_ops.h"

namespace si {

namespace {

constexpr int kSelectThreads = 1024;
constexpr int kCountThreads = 512;
constexpr int kMoveThreads = 256;
constexpr int kChunk = 256;                      // rows a workgroup of the copies takes
constexpr int kGroupChunks = 16;
constexpr int kGroup = kGroupChunks * kChunk;    // rows a workgroup of the histograms and counts takes
constexpr int kBins = 2048;
constexpr int kPasses = 3;                       // digits of 11, 11 and 10 bits
constexpr int kMostRegisterRows = 32 * kSelectThreads;

// Where a batch stands in the descent, and at its end what the copies have to know.
struct Border {
    uint32_t word;  // digits found so far; in the end: rows whose word is larger stay ..
    int32_t equal;  // rows still to be found among those with these digits; in the end: .. and the first so many of those with this word
    int32_t held;   // rows that the batch holds
    int32_t stay;   // rows that stay
};

struct Workspace {
    Border* borders;  // [kPasses + 1][B], the last one is the result
    int* bins;        // [B][kPasses][kBins], for batches that do not fit one workgroup's registers
    int2* chunks;     // [B][chunks]: rows above and at the border before a chunk, within its group
    int2* groups;     // [B][groups]: the same of a whole group
    size_t bytes;
};

struct Moves {
    const unsigned char* src[SI_MAX_ROW_MOVES];
    unsigned char* dst[SI_MAX_ROW_MOVES];
    int32_t row_bytes[SI_MAX_ROW_MOVES];
    int32_t n;
};

struct Rule {
    int T, n_keep, n_sink, n_recent;
};

__device__ __forceinline__ uint32_t word_of(float w, int row, int held, const Rule& r) {
    if (row < r.n_sink || row >= held - r.n_recent) return 0xFFFFFFFFu;
    const uint32_t bits = __float_as_uint(w + 0.0f);  // -0 and +0 are equal
    return w == w ? score_to_ordered(bits) : 0u;
}

__device__ __forceinline__ Border first_border(const int32_t* __restrict__ lengths, int b, const Rule& r) {
    const int held = lengths ? min(max(lengths[b], 0), r.T) : r.T;
    const int stay = min(held, r.n_keep);
    return {0u, stay, held, stay};  // where all rows stay: those above 0, and as many as there are that equal it
}

__device__ __forceinline__ int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t digit_mask(int pass) { return pass < 2 ? 0x7FFu : 0x3FFu; }
__device__ __forceinline__ uint32_t seen_mask(int pass) { return pass == 0 ? 0u : 0xFFFFFFFFu << digit_shift(pass - 1); }

// The highest digit down to which a histogram counts the rows still to be found; at.equal becomes how many of them have this digit.  The whole
// workgroup; s_waves: THREADS / 64 + 2 ints.
template <int THREADS>
__device__ __forceinline__ int find_digit(const int* bins, Border& at, int* s_waves) {
    constexpr int kPer = kBins / THREADS;  // a thread has so many bins, the highest first
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int top = kBins - 1 - kPer * static_cast<int>(threadIdx.x);
    int c[kPer], mine = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        c[i] = bins[top - i];
        mine += c[i];
    }
    const int upto = wave_prefix_sum(mine);
    __syncthreads();  // an earlier digit has been read
    if (lane == 63) s_waves[wave] = upto;
    __syncthreads();
    const int earlier = lane < wave ? s_waves[lane] : 0;  // all at once: a loop would wait for LDS wave after wave
    int above = upto - mine + lane_value(wave_prefix_sum(earlier), 63);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (above < at.equal && at.equal <= above + c[i]) {
            s_waves[THREADS / 64] = top - i;
            s_waves[THREADS / 64 + 1] = above;
        }
        above += c[i];
    }
    __syncthreads();
    at.equal -= s_waves[THREADS / 64 + 1];
    return s_waves[THREADS / 64];
}

// Batches of up to kMostRegisterRows rows: one workgroup a batch keeps the words in registers, KEYS a thread, finds the border and counts the
// chunks.  Row i * 1024 + thread is a thread's i-th.  The digits are those of a word's distance from the smallest one, from its highest bit on: weights
// spread over that range, where their upper 11 bits (sign, exponent) are a few dozen numbers; the smallest word itself, which rows that received
// nothing share, is counted by ballots.  A chain of dependent steps bounds it, not the counts' conflicts: 32 batches of 16411 rows, a third of
// them 0, take 20 us, as much as with digits of the words themselves (24 with a branch a row and prefix sums that waited for LDS once a wave).
template <int KEYS>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const float* __restrict__ weights, const int32_t* __restrict__ lengths,
                                                                     Rule r, int B, Workspace ws, int n_chunks, int n_groups,
                                                                     int32_t* __restrict__ kept) {
    constexpr int kWaves = kSelectThreads / 64;
    __shared__ int s_bins[kBins];
    __shared__ int s_waves[kWaves + 2];
    __shared__ uint32_t s_range[2][kWaves];
    const int b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Border at = first_border(lengths, b, r);
    const float* const w = weights + static_cast<int64_t>(b) * r.T;
    float raw[KEYS];
#pragma unroll
    for (int i = 0; i < KEYS; ++i)
        if (i * kSelectThreads < r.T) raw[i] = w[min(i * kSelectThreads + static_cast<int>(threadIdx.x), r.T - 1)];
    uint32_t x[KEYS];
#pragma unroll
    for (int i = 0; i < KEYS; ++i)
        if (i * kSelectThreads < r.T) x[i] = word_of(raw[i], i * kSelectThreads + static_cast<int>(threadIdx.x), at.held, r);
    if (at.held > at.stay) {
        // more rows are held than stay, so first and last ones do not overlap; they stay, and these are left to be found:
        at.equal -= r.n_sink + r.n_recent;
        if (at.equal == 0) {
            at.word = 0xFFFFFFFFu;  // nothing else
            at.equal = at.stay;
        } else {
            uint32_t low = 0xFFFFFFFFu, high = 0;
#pragma unroll
            for (int i = 0; i < KEYS; ++i)
                if (i * kSelectThreads < at.held && i * kSelectThreads + static_cast<int>(threadIdx.x) < at.held && x[i] != 0xFFFFFFFFu) {
                    low = min(low, x[i]);
                    high = max(high, x[i]);
                }
            low = wave_min(low);
            high = wave_max(high);
            if (lane == 0) {
                s_range[0][wave] = low;
                s_range[1][wave] = high;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                low = min(low, s_range[0][i]);
                high = max(high, s_range[1][i]);
            }
            // words of low .. low + 2^(shift + digits) - 1 are in question
            int shift = max(0, 32 - __clz(static_cast<int>(high - low)) - 11);
            uint32_t span = high - low;  // largest distance in question
            while (true) {
                for (int i = threadIdx.x; i < kBins; i += kSelectThreads) s_bins[i] = 0;
                __syncthreads();
                int lowest = 0;
#pragma unroll
                for (int i = 0; i < KEYS; ++i) {
                    if (i * kSelectThreads >= at.held) break;  // uniform
                    const bool here = i * kSelectThreads + static_cast<int>(threadIdx.x) < at.held && x[i] != 0xFFFFFFFFu && x[i] >= low && x[i] - low <= span;
                    lowest += static_cast<int>(__popcll(__ballot(here && x[i] == low)));
                    if (here && x[i] != low) atomicAdd(&s_bins[(x[i] - low) >> shift], 1);
                }
                if (lane == 0) atomicAdd(&s_bins[0], lowest);
                __syncthreads();
                const int digit = find_digit<kSelectThreads>(s_bins, at, s_waves);
                __syncthreads();
                low += static_cast<uint32_t>(digit) << shift;
                if (shift == 0) break;
                span = (1u << shift) - 1;
                shift = max(0, shift - 11);
            }
            at.word = low;
        }
    }
    // runs of 64 rows in order: run i * 16 + wave; above and equal in one word
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
        const bool here = i * kSelectThreads < at.held && i * kSelectThreads + static_cast<int>(threadIdx.x) < at.held;
        const unsigned long long above = __ballot(here && x[i] > at.word), equal = __ballot(here && x[i] == at.word);
        if (lane == 0) s_bins[i * kWaves + wave] = static_cast<int>(__popcll(above) | (__popcll(equal) << 16));
    }
    __syncthreads();
    if (wave < (KEYS * kWaves + 255) / 256) {  // a lane sums a chunk's four runs, a wave up to 64 chunks; waves behind the first sum those before
        constexpr int kRunsPerChunk = kChunk / 64;
        int2 before = {0, 0};
        for (int v = 0; v < wave; ++v)
            for (int q = 0; q < kRunsPerChunk; ++q) {
                const int c = s_bins[(v * 64 + lane) * kRunsPerChunk + q];
                before.x += c & 0xFFFF;
                before.y += c >> 16;
            }
        before.x = lane_value(wave_prefix_sum(before.x), 63);
        before.y = lane_value(wave_prefix_sum(before.y), 63);
        const int chunk = wave * 64 + lane;
        int2 mine = {0, 0};
        if (chunk * kRunsPerChunk < KEYS * kWaves)
            for (int q = 0; q < kRunsPerChunk; ++q) {
                const int c = s_bins[chunk * kRunsPerChunk + q];
                mine.x += c & 0xFFFF;
                mine.y += c >> 16;
            }
        before.x += wave_prefix_sum(mine.x) - mine.x;
        before.y += wave_prefix_sum(mine.y) - mine.y;
        if (chunk < n_chunks) ws.chunks[static_cast<int64_t>(b) * n_chunks + chunk] = before;
    }
    if (static_cast<int>(threadIdx.x) < n_groups) ws.groups[static_cast<int64_t>(b) * n_groups + threadIdx.x] = {0, 0};  // counted from the batch's first row
    for (int j = at.stay + static_cast<int>(threadIdx.x); j < r.n_keep; j += kSelectThreads) kept[static_cast<int64_t>(b) * r.n_keep + j] = -1;
    if (threadIdx.x == 0) ws.borders[static_cast<int64_t>(kPasses) * B + b] = at;
}

// Longer batches: a workgroup a group of rows.  A kernel a digit adds its rows' digits up in the workspace; the next kernel's workgroups
// each read the digit off the histogram.
__global__ __launch_bounds__(kCountThreads) void evict_clear_kernel(const int32_t* __restrict__ lengths, Rule r, Workspace ws, int parts,
                                                                   int32_t* __restrict__ kept) {
    const int b = blockIdx.x / parts, part = blockIdx.x % parts;
    int* const bins = ws.bins + static_cast<int64_t>(b) * kPasses * kBins;
    for (int i = part * kCountThreads + static_cast<int>(threadIdx.x); i < kPasses * kBins; i += parts * kCountThreads) bins[i] = 0;
    const int stay = first_border(lengths, b, r).stay;
    for (int64_t j = stay + static_cast<int64_t>(part) * kCountThreads + threadIdx.x; j < r.n_keep; j += parts * kCountThreads)
        kept[static_cast<int64_t>(b) * r.n_keep + j] = -1;
}

constexpr int kRowsPerThread = kGroup / kCountThreads;

__device__ __forceinline__ void load_words(const float* __restrict__ w, int first, int held, const Rule& r, uint32_t (&x)[kRowsPerThread]) {
    float raw[kRowsPerThread];
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i) raw[i] = w[min(first + i * kCountThreads, r.T - 1)];
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i) x[i] = word_of(raw[i], first + i * kCountThreads, held, r);
}

__global__ __launch_bounds__(kCountThreads) void evict_digits_kernel(const float* __restrict__ weights, const int32_t* __restrict__ lengths, Rule r,
                                                                    int B, int pass, Workspace ws, int n_groups) {
    __shared__ int s_bins[kBins];
    __shared__ int s_waves[kCountThreads / 64 + 2];
    const int b = blockIdx.x / n_groups, group = blockIdx.x % n_groups;
    Border at = first_border(lengths, b, r);
    if (at.held <= at.stay || group * kGroup >= at.held) return;
    if (pass == 2) at = ws.borders[static_cast<int64_t>(pass - 1) * B + b];
    const int first = group * kGroup + static_cast<int>(threadIdx.x);
    uint32_t x[kRowsPerThread];
    load_words(weights + static_cast<int64_t>(b) * r.T, first, at.held, r, x);
    for (int i = threadIdx.x; i < kBins; i += kCountThreads) s_bins[i] = 0;
    int* const bins = ws.bins + static_cast<int64_t>(b) * kPasses * kBins;
    if (pass > 0) {
        at.word |= static_cast<uint32_t>(find_digit<kCountThreads>(bins + (pass - 1) * kBins, at, s_waves)) << digit_shift(pass - 1);
        if (group == 0 && threadIdx.x == 0) ws.borders[static_cast<int64_t>(pass) * B + b] = at;
    }
    __syncthreads();
    const uint32_t seen = seen_mask(pass), mask = digit_mask(pass);
    const int shift = digit_shift(pass);
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i)
        if (first + i * kCountThreads < at.held && (x[i] & seen) == at.word) atomicAdd(&s_bins[(x[i] >> shift) & mask], 1);
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kCountThreads)
        if (s_bins[i]) atomicAdd(&bins[pass * kBins + i], s_bins[i]);
}

__global__ __launch_bounds__(kCountThreads) void evict_count_kernel(const float* __restrict__ weights, const int32_t* __restrict__ lengths, Rule r,
                                                                   int B, Workspace ws, int n_chunks, int n_groups) {
    constexpr int kWaves = kCountThreads / 64;
    static_assert(kRowsPerThread * kWaves == 64 && kGroupChunks == 16, "a run a lane, four a chunk");
    __shared__ int s_waves[kWaves + 2];
    __shared__ int s_runs[64];
    const int b = blockIdx.x / n_groups, group = blockIdx.x % n_groups;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Border at = first_border(lengths, b, r);
    if (at.held > at.stay) {
        at = ws.borders[static_cast<int64_t>(kPasses - 1) * B + b];
        at.word |= static_cast<uint32_t>(find_digit<kCountThreads>(ws.bins + (static_cast<int64_t>(b) * kPasses + kPasses - 1) * kBins, at, s_waves));
    }
    const int first = group * kGroup + static_cast<int>(threadIdx.x);
    uint32_t x[kRowsPerThread];
    load_words(weights + static_cast<int64_t>(b) * r.T, first, at.held, r, x);
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i) {
        const bool here = first + i * kCountThreads < at.held;
        const unsigned long long above = __ballot(here && x[i] > at.word), equal = __ballot(here && x[i] == at.word);
        if (lane == 0) s_runs[i * kWaves + wave] = static_cast<int>(__popcll(above) | (__popcll(equal) << 16));
    }
    __syncthreads();
    if (wave == 0) {
        const int2 mine = {s_runs[lane] & 0xFFFF, s_runs[lane] >> 16};
        const int2 upto = {wave_prefix_sum(mine.x), wave_prefix_sum(mine.y)};
        const int chunk = group * kGroupChunks + lane / 4;
        if (lane % 4 == 0 && chunk < n_chunks)
            ws.chunks[static_cast<int64_t>(b) * n_chunks + chunk] = {upto.x - mine.x, upto.y - mine.y};
        if (lane == 63) ws.groups[static_cast<int64_t>(b) * n_groups + group] = upto;
    }
    if (group == 0 && threadIdx.x == 0) ws.borders[static_cast<int64_t>(kPasses) * B + b] = at;
}

// Copies rows s_rows[0 .. n) of one array to n rows in a row, in units of type V, four of a thread on their way at once.
template <typename V>
__device__ __forceinline__ void copy_rows(const unsigned char* __restrict__ src, unsigned char* __restrict__ dst, int row_bytes,
                                          const int* s_rows, int n) {
    const unsigned units = static_cast<unsigned>(row_bytes) / static_cast<unsigned>(sizeof(V));
    constexpr int kAhead = 4;
    if (units <= 4096) {
        // i / units as a product: exact for i < 2^20 and units <= 2^12 (the excess of the factor adds less than 2^-12)
        const unsigned inverse = static_cast<unsigned>(((1ull << 32) + units - 1) / units);
        const unsigned total = static_cast<unsigned>(n) * units;
        for (unsigned i0 = threadIdx.x; i0 < total; i0 += kAhead * kMoveThreads) {
            V v[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const unsigned i = min(i0 + a * kMoveThreads, total - 1);
                const unsigned j = units == 1 ? i : __umulhi(i, inverse);
                v[a] = reinterpret_cast<const V*>(src + static_cast<int64_t>(s_rows[j]) * row_bytes)[i - j * units];
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
                if (i0 + a * kMoveThreads < total) reinterpret_cast<V*>(dst)[i0 + a * kMoveThreads] = v[a];
        }
        return;
    }
    for (int j = 0; j < n; ++j) {  // rows longer than a workgroup's trip
        const V* const from = reinterpret_cast<const V*>(src + static_cast<int64_t>(s_rows[j]) * row_bytes);
        V* const to = reinterpret_cast<V*>(dst + static_cast<int64_t>(j) * row_bytes);
        for (unsigned u = threadIdx.x; u < units; u += kMoveThreads) to[u] = from[u];
    }
}

__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(const float* __restrict__ weights, Rule r, int B, Workspace ws, int n_chunks,
                                                                 int n_groups, Moves moves, int32_t* __restrict__ kept,
                                                                 int32_t* __restrict__ new_lengths) {
    constexpr int kWaves = kMoveThreads / 64;
    __shared__ int s_rows[kChunk];
    __shared__ int s_waves[4][kWaves];
    static_assert(kChunk == kMoveThreads, "a thread a row");
    const int64_t b = blockIdx.x / n_chunks;
    const int c = static_cast<int>(blockIdx.x % n_chunks);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = c * kChunk + static_cast<int>(threadIdx.x);
    const float w = weights[b * r.T + min(row, r.T - 1)];  // these three at once
    const int2 before_chunk = ws.chunks[b * n_chunks + c];
    const Border border = ws.borders[static_cast<int64_t>(kPasses) * B + b];
    // lengths may be the same array: no kernel reads it any more
    if (c == 0 && threadIdx.x == 0 && new_lengths) new_lengths[b] = border.stay;
    if (c * kChunk >= border.held) return;
    const bool here = row < border.held;
    const uint32_t x = here ? word_of(w, row, border.held, r) : 0u;
    int2 before = {0, 0};  // of the groups before this one
    for (int g = threadIdx.x; g < c / kGroupChunks; g += kMoveThreads) {
        const int2 v = ws.groups[b * n_groups + g];
        before.x += v.x;
        before.y += v.y;
    }
    const unsigned long long equal = __ballot(here && x == border.word);
    before.x = wave_prefix_sum(before.x);
    before.y = wave_prefix_sum(before.y);
    if (lane == 63) {
        s_waves[0][wave] = static_cast<int>(__popcll(equal));
        s_waves[2][wave] = before.x;
        s_waves[3][wave] = before.y;
    }
    __syncthreads();
    before = before_chunk;
    for (int i = 0; i < kWaves; ++i) {
        before.x += s_waves[2][i];
        before.y += s_waves[3][i];
    }
    int rank = before.y + __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(equal >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(equal), 0u));
    for (int i = 0; i < wave; ++i) rank += s_waves[0][i];
    const bool stays = here && (x > border.word || (x == border.word && rank < border.equal));
    const unsigned long long mine = __ballot(stays);
    if (lane == 0) s_waves[1][wave] = static_cast<int>(__popcll(mine));
    __syncthreads();
    int place = __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(mine >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(mine), 0u));
    int n = 0;
    for (int i = 0; i < kWaves; ++i) {
        if (i < wave) place += s_waves[1][i];
        n += s_waves[1][i];
    }
    const int64_t to = b * r.n_keep + before.x + min(before.y, border.equal);  // the chunk's first place
    if (stays) {
        s_rows[place] = row;
        kept[to + place] = row;
    }
    __syncthreads();
    if (n == 0) return;
    for (int a = 0; a < moves.n; ++a) {
        const int row_bytes = moves.row_bytes[a];
        const unsigned char* const src = moves.src[a] + b * r.T * row_bytes;
        unsigned char* const dst = moves.dst[a] + to * row_bytes;
        if (row_bytes % 16 == 0) copy_rows<uint4>(src, dst, row_bytes, s_rows, n);
        else if (row_bytes % 4 == 0) copy_rows<uint32_t>(src, dst, row_bytes, s_rows, n);
        else if (row_bytes % 2 == 0) copy_rows<uint16_t>(src, dst, row_bytes, s_rows, n);
        else copy_rows<unsigned char>(src, dst, row_bytes, s_rows, n);
    }
}

int chunks_of(int32_t T) { return static_cast<int>((static_cast<int64_t>(T) + kChunk - 1) / kChunk); }
int groups_of(int32_t T) { return (chunks_of(T) + kGroupChunks - 1) / kGroupChunks; }

Workspace carve(void* base, int32_t B, int32_t T) {
    Workspace ws;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void* p = static_cast<unsigned char*>(base) + at;
        at += (bytes + 15) / 16 * 16;
        return p;
    };
    ws.borders = static_cast<Border*>(take(static_cast<size_t>(kPasses + 1) * B * sizeof(Border)));
    ws.bins = static_cast<int*>(take(T > kMostRegisterRows ? static_cast<size_t>(B) * kPasses * kBins * sizeof(int) : 0));
    ws.chunks = static_cast<int2*>(take(static_cast<size_t>(B) * chunks_of(T) * sizeof(int2)));
    ws.groups = static_cast<int2*>(take(static_cast<size_t>(B) * groups_of(T) * sizeof(int2)));
    ws.bytes = at;
    return ws;
}

struct Range {
    uintptr_t begin;
    size_t bytes;
};
bool overlap(const Range& x, const Range& y) { return x.begin < y.begin + y.bytes && y.begin < x.begin + x.bytes; }
Range range_of(const void* p, size_t bytes) { return {reinterpret_cast<uintptr_t>(p), bytes}; }

}  // namespace

}  // namespace si

using namespace si;

extern "C" {

size_t si_evict_workspace_bytes(int32_t B, int32_t T) {
    if (B < 1 || T < 1) return 0;
    return carve(nullptr, B, T).bytes;
}

si_status si_evict_rows(const float* weights, const int32_t* lengths, int32_t B, int32_t T, int32_t n_keep, int32_t n_sink,
                        int32_t n_recent, const si_row_move* moves, int32_t n_moves, int32_t* kept, int32_t* new_lengths,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!weights || !kept || !workspace || (!moves && n_moves != 0)) return SI_ERR_INVALID_ARG;
    if (B < 1 || T < 1 || n_keep < 1 || n_keep > T || n_sink < 0 || n_recent < 0 || n_sink > n_keep || n_recent > n_keep - n_sink)
        return SI_ERR_INVALID_ARG;
    if (n_moves < 0 || n_moves > SI_MAX_ROW_MOVES) return SI_ERR_INVALID_ARG;
    if (!aligned16(weights) || !aligned16(kept) || !aligned16(workspace) || !aligned4(lengths) || !aligned4(new_lengths)) return SI_ERR_INVALID_ARG;
    const int n_chunks = chunks_of(T);
    if (static_cast<int64_t>(B) * n_chunks >= (int64_t{1} << 32) / kMoveThreads || B >= (1 << 22) || T > (1 << 30)) return SI_ERR_UNSUPPORTED_SHAPE;
    if (workspace_bytes < si_evict_workspace_bytes(B, T)) return SI_ERR_WORKSPACE_TOO_SMALL;
    const size_t rows = static_cast<size_t>(B) * T, places = static_cast<size_t>(B) * n_keep;
    Moves mv = {};
    mv.n = n_moves;
    for (int a = 0; a < n_moves; ++a) {
        if (!moves[a].src || !moves[a].dst || moves[a].row_bytes < 1) return SI_ERR_INVALID_ARG;
        if (!aligned16(moves[a].src) || !aligned16(moves[a].dst)) return SI_ERR_INVALID_ARG;
        mv.src[a] = static_cast<const unsigned char*>(moves[a].src);
        mv.dst[a] = static_cast<unsigned char*>(moves[a].dst);
        mv.row_bytes[a] = moves[a].row_bytes;
    }
    // what is written must not be what is read, or written as something else; new_lengths may be lengths
    Range written[SI_MAX_ROW_MOVES + 3], read[SI_MAX_ROW_MOVES + 2];
    int n_written = 0, n_read = 0;
    for (int a = 0; a < n_moves; ++a) {
        written[n_written++] = range_of(mv.dst[a], places * mv.row_bytes[a]);
        read[n_read++] = range_of(mv.src[a], rows * mv.row_bytes[a]);
    }
    written[n_written++] = range_of(kept, places * sizeof(int32_t));
    written[n_written++] = range_of(workspace, si_evict_workspace_bytes(B, T));
    read[n_read++] = range_of(weights, rows * sizeof(float));
    if (lengths && lengths != new_lengths) read[n_read++] = range_of(lengths, B * sizeof(int32_t));
    if (new_lengths) written[n_written++] = range_of(new_lengths, B * sizeof(int32_t));
    for (int i = 0; i < n_written; ++i) {
        for (int j = 0; j < n_read; ++j)
            if (overlap(written[i], read[j])) return SI_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(written[i], written[j])) return SI_ERR_INVALID_ARG;
    }
    const Workspace ws = carve(workspace, B, T);
    const int n_groups = groups_of(T);
    const Rule r = {T, n_keep, n_sink, n_recent};
    hipStream_t hs = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (T <= kMostRegisterRows) {
#define SI_LAUNCH(KEYS)                                                                                                            \
    hipLaunchKernelGGL((evict_select_kernel<KEYS>), dim3(B), dim3(kSelectThreads), 0, hs, weights, lengths, r, B, ws, n_chunks, n_groups, \
                       kept)
        if (T <= 4 * kSelectThreads) SI_LAUNCH(4);
        else if (T <= 16 * kSelectThreads) SI_LAUNCH(16);
        else SI_LAUNCH(32);
#undef SI_LAUNCH
        e = hipGetLastError();
    } else {
        const unsigned grid = static_cast<unsigned>(B) * static_cast<unsigned>(n_groups);
        constexpr int kClearParts = 4;
        hipLaunchKernelGGL(evict_clear_kernel, dim3(static_cast<unsigned>(B) * kClearParts), dim3(kCountThreads), 0, hs, lengths, r, ws,
                           kClearParts, kept);
        e = hipGetLastError();
        for (int pass = 0; pass < kPasses && e == hipSuccess; ++pass) {
            hipLaunchKernelGGL(evict_digits_kernel, dim3(grid), dim3(kCountThreads), 0, hs, weights, lengths, r, B, pass, ws, n_groups);
            e = hipGetLastError();
        }
        if (e == hipSuccess) {
            hipLaunchKernelGGL(evict_count_kernel, dim3(grid), dim3(kCountThreads), 0, hs, weights, lengths, r, B, ws, n_chunks, n_groups);
            e = hipGetLastError();
        }
    }
    if (e == hipSuccess) {
        hipLaunchKernelGGL(evict_move_kernel, dim3(static_cast<unsigned>(B) * static_cast<unsigned>(n_chunks)), dim3(kMoveThreads), 0, hs,
                           weights, r, B, ws, n_chunks, n_groups, mv, kept, new_lengths);
        e = hipGetLastError();
    }
    return report(e);
}

}  // extern "C"
