// Eviction (si_evict_rows): of the n rows that a batch holds, the first n_sink, the last n_recent and those with the largest
// weights stay, n_keep in all, and the arrays that belong to the rows are compacted in order.
//
// A weight is compared as a 32-bit word whose unsigned order is that of the weights: NaN 0, then -inf .. +inf, and rows that
// always stay above all.  The n_keep-th largest word of a batch is found by radix descent over 11, 11 and 10 bits; rows above it
// stay, and of those that equal it as many of the first as there is room for.  Then each workgroup takes a chunk of rows, lists those that stay
// (where its list begins is known from the counts of the chunks before it) and copies what belongs to them.  Small calls do all of it in one launch.
//
// The copies bound long and many rows: 2 * (rows that stay) * (bytes of a row in all arrays), 191 MB of 32 batches of 8205 to 16411 rows in 48.5 us where
// nothing of it is in the caches (32 on the same arrays again), right behind 12.5 for the borders;
// 1 x 262144 rows, 104 MB, 19.5 after 24 of five launches that each hold little more than their chain of dependent steps (groups of half as many rows,
// half or twice the threads: within 3 %).  Few rows take 7.5 us, a launch and that chain.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "attention_set.h"
#include "cache_call.h"
#include "si_internal.h"
#include "streamindex_cache.h"
#include "wave_ops.h"

namespace si {

namespace {

constexpr int kSelectThreads = 1024;             // 512: 32 batches of 16411 rows 1.3 times as long, 2048 rows alike
constexpr int kCountThreads = 512;
constexpr int kMoveThreads = 256;
constexpr int kChunk = 256;                      // rows a workgroup of the copies takes
constexpr int kGroupChunks = 16;
constexpr int kGroup = kGroupChunks * kChunk;    // rows a workgroup of the histograms and counts takes
constexpr int kBins = 2048;
constexpr int kPasses = 3;                       // digits of 11, 11 and 10 bits
constexpr int kMostSelectRows = 32768;

// Where a batch stands in the descent, and at its end what the copies have to know.
struct Border {
    uint32_t word;  // digits found so far; in the end: rows whose word is larger stay ..
    int32_t equal;  // rows still to be found among those with these digits; in the end: .. and the first so many of those with this word (maybe 0)
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
// workgroup, once a kernel; s_waves: THREADS / 64 + 2 ints.
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

// Batches of up to kMostSelectRows rows: one workgroup has the words of a batch in LDS, finds the border and counts runs of 64 rows.  The digits, of 9
// bits, are those of a word's distance from the smallest one, from its highest bit on: weights spread over that range, where their upper bits (sign,
// exponent) are a few dozen numbers; the smallest word itself, which rows that received nothing share, is counted by ballots.  Every wave finds the
// digit by itself.  Once a digit is down to 64 rows, these are listed, and each counts those above it.
// What bounds it is a chain of short steps between barriers, which 16 waves on one compute unit do in turn: 2048 rows take 8,500 cycles, a digit
// about 2,700 of them.  With the words in registers (4, 16 or 32 a thread, every loop over them unrolled), digits of 11 bits, and no list of the last
// rows, 32 batches of 16411 rows took 19.9 us and 2048 rows 6.1; as it stands 11.5 and 4.4.
constexpr int kSelectDigit = 9;
constexpr int kSelectBins = 1 << kSelectDigit;
constexpr int kSelectRounds = 4;  // that 32 bits have
constexpr int kFewRows = 64;
struct SelectShared {
    int bins[kSelectRounds][kSelectBins];
    int lowest[kSelectRounds];
    int runs[kMostSelectRows / 64];  // rows of a run above the border and, in the upper half, those at it
    uint32_t range[2][kSelectThreads / 64];
    uint32_t few[kFewRows];
    int n_few;
};

// The whole workgroup; `words`: LDS for a batch's, whole runs.  It may read the runs' counts when this returns.
__device__ __forceinline__ Border select_rows(const float* __restrict__ w, const int32_t* __restrict__ lengths, int b, const Rule& r, SelectShared& sh,
                                              uint32_t* words) {
    constexpr int kWaves = kSelectThreads / 64;
    typedef const __attribute__((address_space(1))) void gbl_void;
    typedef __attribute__((address_space(3))) void lds_void;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Border at = first_border(lengths, b, r);
    const int n_runs = (at.held + 63) / 64;
    // a wave's own runs, here and below
    for (int run = wave; run < n_runs; run += kWaves)
        __builtin_amdgcn_global_load_lds((gbl_void*)(w + min(run * 64 + lane, r.T - 1)), (lds_void*)(words + run * 64), 4, 0, 0);
    for (int i = threadIdx.x; i < kSelectRounds * kSelectBins; i += kSelectThreads) sh.bins[0][i] = 0;
    if (threadIdx.x < kSelectRounds) sh.lowest[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.n_few = 0;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    uint32_t low = 0xFFFFFFFFu, high = 0;
    for (int row = threadIdx.x; row < n_runs * 64; row += kSelectThreads) {
        const uint32_t x = row < at.held ? word_of(__uint_as_float(words[row]), row, at.held, r) : 0xFFFFFFFFu;
        words[row] = x;
        low = min(low, x);
        high = max(high, x == 0xFFFFFFFFu ? 0u : x);  // rows that always stay, or are not there, do not count
    }
    if (at.held > at.stay) {
        // more rows are held than stay, so first and last ones do not overlap; they stay, and these are left to be found:
        at.equal -= r.n_sink + r.n_recent;
        if (at.equal == 0) {
            at.word = 0xFFFFFFFEu;  // nothing else
        } else {
            low = wave_min(low);
            high = wave_max(high);
            if (lane == 0) {
                sh.range[0][wave] = low;
                sh.range[1][wave] = high;
            }
            __syncthreads();
            low = wave_min(sh.range[0][lane % kWaves]);
            high = wave_max(sh.range[1][lane % kWaves]);
            int there;  // rows with the word in the end
            for (int round = 0;; ++round) {
                // the words low .. high are in question: low itself, and the distances from low + 1, whose digit counts
                const uint32_t span = high - low;
                const int shift = max(0, 32 - __clz(static_cast<int>(span)) - kSelectDigit);
                int lowest = 0;
                for (int row = threadIdx.x; row < n_runs * 64; row += kSelectThreads) {
                    const uint32_t far = words[row] - low;
                    lowest += static_cast<int>(__popcll(__ballot(far == 0)));
                    if (far - 1 < span) atomicAdd(&sh.bins[round][(far - 1) >> shift], 1);
                }
                if (lane == 0 && lowest > 0) atomicAdd(&sh.lowest[round], lowest);
                __syncthreads();
                // a lane has 8 bins, the highest first
                constexpr int kPer = kSelectBins / 64;
                const int top = kSelectBins - 1 - kPer * lane;
                int c[kPer], mine = 0;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    c[i] = sh.bins[round][top - i];
                    mine += c[i];
                }
                const int upto = wave_prefix_sum(mine);
                const unsigned long long in = __ballot(at.equal <= upto);
                if (in == 0ull) {  // as a rule rows that received nothing
                    at.equal -= lane_value(upto, 63);
                    there = sh.lowest[round];
                    break;
                }
                const int at_lane = __ffsll(in) - 1;
                int left = at.equal - lane_value(upto - mine, at_lane), digit = kSelectBins - 1 - kPer * at_lane;
                there = lane_value(c[0], at_lane);
#pragma unroll
                for (int i = 1; i < kPer; ++i)
                    if (left > there) {
                        left -= there;
                        there = lane_value(c[i], at_lane);
                        --digit;
                    }
                at.equal = left;
                low += 1 + (static_cast<uint32_t>(digit) << shift);
                if (shift == 0) break;
                high = min(low + ((1u << shift) - 1), high);
                if (there <= kFewRows) {
                    for (int row = threadIdx.x; row < n_runs * 64; row += kSelectThreads) {
                        const uint32_t x = words[row];
                        if (x - low <= high - low) sh.few[atomicAdd(&sh.n_few, 1)] = x - low;  // `there` of them
                    }
                    __syncthreads();
                    const uint32_t far = sh.few[min(lane, there - 1)];
                    unsigned long long alive = there == 64 ? ~0ull : (1ull << there) - 1;
                    for (int bit = shift - 1; bit >= 0; --bit) {
                        const unsigned long long ones = __ballot((far >> bit) & 1) & alive;
                        const int n = static_cast<int>(__popcll(ones));
                        if (at.equal <= n) {
                            alive = ones;
                            low += 1u << bit;
                        } else {
                            alive &= ~ones;
                            at.equal -= n;
                        }
                    }
                    there = static_cast<int>(__popcll(alive));
                    break;
                }
            }
            at.word = low;
            if (at.equal == there) {  // all of them: the rows above the word before it (there is one, as not all rows stay)
                at.word -= 1;
                at.equal = 0;
            }
        }
    }
    for (int run = wave; run * 64 < r.T; run += kWaves) {
        int n = 0;
        if (run < n_runs) {
            const uint32_t x = words[run * 64 + lane];
            const bool here = run * 64 + lane < at.held;
            n = static_cast<int>(__popcll(__ballot(here && x > at.word)) | (__popcll(__ballot(here && x == at.word)) << 16));
        }
        if (lane == 0) sh.runs[run] = n;
    }
    __syncthreads();
    return at;
}

constexpr int kRunsPerChunk = kChunk / 64;

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const float* __restrict__ weights, const int32_t* __restrict__ lengths,
                                                                     Rule r, int B, Workspace ws, int n_chunks, int n_groups,
                                                                     int32_t* __restrict__ kept) {
    extern __shared__ uint32_t words[];
    __shared__ SelectShared sh;
    const int b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Border at = select_rows(weights + static_cast<int64_t>(b) * r.T, lengths, b, r, sh, words);
    if (wave * 64 < n_chunks) {  // a lane sums a chunk's runs, a wave 64 chunks; waves behind the first sum those before
        const int n_runs = (r.T + 63) / 64;
        auto counts = [&](int chunk) {
            int2 n = {0, 0};
#pragma unroll
            for (int q = 0; q < kRunsPerChunk; ++q) {
                const int run = chunk * kRunsPerChunk + q;
                const int c = run < n_runs ? sh.runs[run] : 0;
                n.x += c & 0xFFFF;
                n.y += c >> 16;
            }
            return n;
        };
        int2 before = {0, 0};
        for (int v = 0; v < wave; ++v) {
            const int2 n = counts(v * 64 + lane);
            before.x += n.x;
            before.y += n.y;
        }
        const int2 mine = counts(wave * 64 + lane);
        before.x = lane_value(wave_prefix_sum(before.x), 63) + wave_prefix_sum(mine.x) - mine.x;
        before.y = lane_value(wave_prefix_sum(before.y), 63) + wave_prefix_sum(mine.y) - mine.y;
        const int chunk = wave * 64 + lane;
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

// Lanes of a ballot before this one.
__device__ __forceinline__ int lanes_below(unsigned long long lanes) {
    return static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(lanes >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(lanes), 0u)));
}

// Copies rows s_rows[0 .. n) of one array to n rows in a row, in units of type V, four of a thread on their way at once.
template <typename V, int THREADS>
__device__ __forceinline__ void copy_rows(const unsigned char* __restrict__ src, unsigned char* __restrict__ dst, int row_bytes,
                                          const int* s_rows, int n) {
    const unsigned units = static_cast<unsigned>(row_bytes) / static_cast<unsigned>(sizeof(V));
    constexpr int kAhead = 4;
    if (units <= 4096) {
        // i / units as a product: exact for i < 2^20 and units <= 2^12 (the excess of the factor adds less than 2^-12)
        const unsigned inverse = static_cast<unsigned>(((1ull << 32) + units - 1) / units);
        const unsigned total = static_cast<unsigned>(n) * units;
        for (unsigned i0 = threadIdx.x; i0 < total; i0 += kAhead * THREADS) {
            V v[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const unsigned i = min(i0 + a * THREADS, total - 1);
                const unsigned j = units == 1 ? i : __umulhi(i, inverse);
                v[a] = reinterpret_cast<const V*>(src + static_cast<int64_t>(s_rows[j]) * row_bytes)[i - j * units];
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
                if (i0 + a * THREADS < total) reinterpret_cast<V*>(dst)[i0 + a * THREADS] = v[a];
        }
        return;
    }
    for (int j = 0; j < n; ++j) {  // rows longer than a workgroup's trip
        const V* const from = reinterpret_cast<const V*>(src + static_cast<int64_t>(s_rows[j]) * row_bytes);
        V* const to = reinterpret_cast<V*>(dst + static_cast<int64_t>(j) * row_bytes);
        for (unsigned u = threadIdx.x; u < units; u += THREADS) to[u] = from[u];
    }
}

// Rows s_rows[0 .. n) of batch b in every parts-th array, to places from `to` on.
template <int THREADS>
__device__ __forceinline__ void copy_chunk(const Moves& moves, int part, int parts, int64_t b, const Rule& r, int64_t to, const int* s_rows, int n) {
    for (int a = part; a < moves.n; a += parts) {
        const int row_bytes = moves.row_bytes[a];
        const unsigned char* const src = moves.src[a] + b * r.T * row_bytes;
        unsigned char* const dst = moves.dst[a] + to * row_bytes;
        if (row_bytes % 16 == 0) copy_rows<uint4, THREADS>(src, dst, row_bytes, s_rows, n);
        else if (row_bytes % 4 == 0) copy_rows<uint32_t, THREADS>(src, dst, row_bytes, s_rows, n);
        else if (row_bytes % 2 == 0) copy_rows<uint16_t, THREADS>(src, dst, row_bytes, s_rows, n);
        else copy_rows<unsigned char, THREADS>(src, dst, row_bytes, s_rows, n);
    }
}

__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(const float* __restrict__ weights, Rule r, int B, Workspace ws, int n_chunks,
                                                                 int n_groups, Moves moves, int parts, int32_t* __restrict__ kept,
                                                                 int32_t* __restrict__ new_lengths) {
    constexpr int kWaves = kMoveThreads / 64;
    __shared__ int s_rows[kChunk];
    __shared__ int s_waves[4][kWaves];
    static_assert(kChunk == kMoveThreads, "a thread a row");
    // a workgroup copies every parts-th array of a chunk's rows
    const int part = static_cast<int>(blockIdx.x % parts);
    const int64_t b = blockIdx.x / parts / n_chunks;
    const int c = static_cast<int>(blockIdx.x / parts % n_chunks);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = c * kChunk + static_cast<int>(threadIdx.x);
    const float w = weights[b * r.T + min(row, r.T - 1)];  // these three at once
    const int2 before_chunk = ws.chunks[b * n_chunks + c];
    const Border border = ws.borders[static_cast<int64_t>(kPasses) * B + b];
    // lengths may be the same array: no kernel reads it any more
    if (c == 0 && part == 0 && threadIdx.x == 0 && new_lengths) new_lengths[b] = border.stay;
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
    int rank = before.y + lanes_below(equal);
    for (int i = 0; i < wave; ++i) rank += s_waves[0][i];
    const bool stays = here && (x > border.word || (x == border.word && rank < border.equal));
    const unsigned long long mine = __ballot(stays);
    if (lane == 0) s_waves[1][wave] = static_cast<int>(__popcll(mine));
    __syncthreads();
    int place = lanes_below(mine);
    int n = 0;
    for (int i = 0; i < kWaves; ++i) {
        if (i < wave) place += s_waves[1][i];
        n += s_waves[1][i];
    }
    const int64_t to = b * r.n_keep + before.x + min(before.y, border.equal);  // the chunk's first place
    if (stays) {
        s_rows[place] = row;
        if (part == 0) kept[to + place] = row;
    }
    __syncthreads();
    if (n == 0) return;
    copy_chunk<kMoveThreads>(moves, part, parts, b, r, to, s_rows, n);
}

// Few rows in all: a workgroup a chunk and array, each of which finds its batch's border by itself.  One launch and no way through the workspace.
// `lengths` is read by all of them, so new_lengths must be elsewhere.
__global__ __launch_bounds__(kSelectThreads) void evict_few_kernel(const float* __restrict__ weights, const int32_t* __restrict__ lengths, Rule r,
                                                                  int n_chunks, Moves moves, int parts, int32_t* __restrict__ kept,
                                                                  int32_t* __restrict__ new_lengths) {
    extern __shared__ uint32_t words[];
    __shared__ SelectShared sh;
    __shared__ int s_rows[kChunk];
    const int part = static_cast<int>(blockIdx.x % parts);
    const int b = static_cast<int>(blockIdx.x / parts / n_chunks);
    const int c = static_cast<int>(blockIdx.x / parts % n_chunks);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Border at = select_rows(weights + static_cast<int64_t>(b) * r.T, lengths, b, r, sh, words);
    const int64_t first_place = static_cast<int64_t>(b) * r.n_keep;
    if (c == 0 && part == 0) {
        if (threadIdx.x == 0 && new_lengths) new_lengths[b] = at.stay;
        for (int j = at.stay + static_cast<int>(threadIdx.x); j < r.n_keep; j += kSelectThreads) kept[first_place + j] = -1;
    }
    if (c * kChunk >= at.held) return;
    // rows above the border and at it before the chunk, and before its runs (both counts in one word)
    unsigned counted = 0;
    for (int run = lane; run < c * kRunsPerChunk; run += 64) counted += static_cast<unsigned>(sh.runs[run]);
    unsigned before[kRunsPerChunk + 1];
    before[0] = static_cast<unsigned>(lane_value(wave_prefix_sum(static_cast<int>(counted)), 63));
#pragma unroll
    for (int q = 0; q < kRunsPerChunk; ++q) {
        const int run = c * kRunsPerChunk + q;
        before[q + 1] = before[q] + (run * 64 < r.T ? static_cast<unsigned>(sh.runs[run]) : 0u);
    }
    auto stay_before = [&](unsigned n) { return static_cast<int>(n & 0xFFFFu) + min(static_cast<int>(n >> 16), at.equal); };
    const int first = stay_before(before[0]), n = stay_before(before[kRunsPerChunk]) - first;
#pragma unroll
    for (int q = 0; q < kRunsPerChunk; ++q)
        if (wave == q) {
            const int row = c * kChunk + static_cast<int>(threadIdx.x);
            const bool here = row < at.held;
            const uint32_t x = here ? words[row] : 0u;
            const unsigned long long equal = __ballot(here && x == at.word);
            const int rank = static_cast<int>(before[q] >> 16) + lanes_below(equal);
            const bool stays = here && (x > at.word || (x == at.word && rank < at.equal));
            const unsigned long long mine = __ballot(stays);
            const int place = stay_before(before[q]) + lanes_below(mine);
            if (stays) {
                s_rows[place - first] = row;
                if (part == 0) kept[first_place + place] = row;
            }
        }
    __syncthreads();
    if (n > 0) copy_chunk<kSelectThreads>(moves, part, parts, b, r, first_place + first, s_rows, n);
}

// Up to so many chunks in all one launch does (a compute unit has two of its workgroups at once), up to so many of them with a workgroup an array, so that
// no array waits for another one.  Measured (us, two launches / one / one with a workgroup an array; rows of 64 + 4 + 4 + 256 bytes, three quarters stay):
// 1 x 512 rows 11 / 8.1 / 6.3, 1 x 2048 12.8 / 9.6 / 7.5, 8 x 2048 13.6 / 10.2 / 8.8, 1 x 16384 20.6 / 17.2 / 15.9, 1 x 32768 29.9 / 25.9 / 26.0,
// 32 x 2048 17.5 / 12.5 / -, 64 x 2048 21.8 / 18.1 / -, 8 x 16384 28.6 / 28.7 / -, 32 x 16384 68 / 101 / -.
constexpr int64_t kFewChunks = 512;
constexpr int64_t kFewestChunks = 100;

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
    ws.bins = static_cast<int*>(take(T > kMostSelectRows ? static_cast<size_t>(B) * kPasses * kBins * sizeof(int) : 0));
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
    const int64_t grid = static_cast<int64_t>(B) * n_chunks;
    const int parts = grid <= kFewestChunks ? std::max(1, std::min(n_moves, static_cast<int32_t>(kFewChunks / grid))) : 1;  // of a chunk
    if (grid <= kFewChunks && T <= kMostSelectRows && (!lengths || lengths != new_lengths)) {
        static std::atomic<size_t> allowed[64];
        const size_t lds = static_cast<size_t>((T + 63) / 64 * 64) * sizeof(uint32_t);
        e = allow_lds(evict_few_kernel, lds, allowed);
        if (e != hipSuccess) return report(e);
        hipLaunchKernelGGL(evict_few_kernel, dim3(static_cast<unsigned>(grid * parts)), dim3(kSelectThreads), lds, hs, weights, lengths, r, n_chunks, mv,
                           parts, kept, new_lengths);
        return report(hipGetLastError());
    }
    if (T <= kMostSelectRows) {
        static std::atomic<size_t> allowed[64];
        const size_t lds = static_cast<size_t>((T + 63) / 64 * 64) * sizeof(uint32_t);
        e = allow_lds(evict_select_kernel, lds, allowed);
        if (e != hipSuccess) return report(e);
        hipLaunchKernelGGL(evict_select_kernel, dim3(B), dim3(kSelectThreads), lds, hs, weights, lengths, r, B, ws, n_chunks, n_groups, kept);
        e = hipGetLastError();
    } else {
        const unsigned groups = static_cast<unsigned>(B) * static_cast<unsigned>(n_groups);
        constexpr int kClearParts = 4;
        hipLaunchKernelGGL(evict_clear_kernel, dim3(static_cast<unsigned>(B) * kClearParts), dim3(kCountThreads), 0, hs, lengths, r, ws,
                           kClearParts, kept);
        e = hipGetLastError();
        for (int pass = 0; pass < kPasses && e == hipSuccess; ++pass) {
            hipLaunchKernelGGL(evict_digits_kernel, dim3(groups), dim3(kCountThreads), 0, hs, weights, lengths, r, B, pass, ws, n_groups);
            e = hipGetLastError();
        }
        if (e == hipSuccess) {
            hipLaunchKernelGGL(evict_count_kernel, dim3(groups), dim3(kCountThreads), 0, hs, weights, lengths, r, B, ws, n_chunks, n_groups);
            e = hipGetLastError();
        }
    }
    if (e == hipSuccess) {
        hipLaunchKernelGGL(evict_move_kernel, dim3(static_cast<unsigned>(grid * parts)), dim3(kMoveThreads), 0, hs, weights, r, B, ws, n_chunks,
                           n_groups, mv, parts, kept, new_lengths);
        e = hipGetLastError();
    }
    return report(e);
}

}  // extern "C"
