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

#include "si_internal.h"
#include "streamindex_cache.h"
#include "wave_ops.h"

namespace si {

namespace {

constexpr int kSelectThreads = 1024;
constexpr int kMoveThreads = 256;
constexpr int kChunk = 256;  // rows a workgroup of the copies takes
constexpr int kBins = 2048;

// Per batch: what the copies have to know.
struct Border {
    uint32_t word;  // rows whose word is larger stay ..
    int32_t equal;  // .. and the first so many of those with this word
    int32_t held;   // rows that the batch holds
    int32_t stay;   // rows that stay
};

struct Moves {
    const unsigned char* src[SI_MAX_ROW_MOVES];
    unsigned char* dst[SI_MAX_ROW_MOVES];
    int32_t row_bytes[SI_MAX_ROW_MOVES];
    int32_t n;
};

__device__ __forceinline__ uint32_t word_of(float w, int row, int held, int n_sink, int n_recent) {
    if (row < n_sink || row >= held - n_recent) return 0xFFFFFFFFu;
    const uint32_t bits = __float_as_uint(w + 0.0f);  // -0 and +0 are equal
    return w == w ? score_to_ordered(bits) : 0u;
}

// One workgroup a batch: the border, and for every chunk of rows how many rows stay and how many equal the border's word before it.
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const float* __restrict__ weights, const int32_t* __restrict__ lengths,
                                                                     int T, int n_keep, int n_sink, int n_recent, int n_chunks,
                                                                     Border* __restrict__ borders, int2* __restrict__ chunks,
                                                                     int32_t* __restrict__ kept, int32_t* __restrict__ new_lengths) {
    __shared__ int s_bins[kBins];
    __shared__ int s_waves[kSelectThreads / 64];
    __shared__ int s_digit, s_above;
    const int b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int held = lengths ? min(max(lengths[b], 0), T) : T;
    const int stay = min(held, n_keep);
    const float* const w = weights + static_cast<int64_t>(b) * T;
    uint32_t word = 0;  // the digits found so far
    int left = stay;    // rows still to be found among those with these digits
    if (held > n_keep) {
        int shift = 32;
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = pass < 2 ? 11 : 10;
            const uint32_t seen = pass == 0 ? 0u : 0xFFFFFFFFu << shift;
            shift -= bits;
            for (int i = threadIdx.x; i < kBins; i += kSelectThreads) s_bins[i] = 0;
            __syncthreads();
            for (int row = threadIdx.x; row < held; row += kSelectThreads) {
                const uint32_t x = word_of(w[row], row, held, n_sink, n_recent);
                if ((x & seen) == word) atomicAdd(&s_bins[(x >> shift) & ((1u << bits) - 1)], 1);
            }
            __syncthreads();
            // thread i has bins 2 i and 2 i + 1 from the top: how many rows are in the bins above them
            const int top = kBins - 1 - 2 * static_cast<int>(threadIdx.x);
            const int c0 = s_bins[top], c1 = s_bins[top - 1];
            const int upto = wave_prefix_sum(c0 + c1);
            if (lane == 63) s_waves[wave] = upto;
            __syncthreads();
            int above = upto - (c0 + c1);
            for (int i = 0; i < wave; ++i) above += s_waves[i];
            if (above < left && left <= above + c0) {
                s_digit = top;
                s_above = above;
            } else if (above + c0 < left && left <= above + c0 + c1) {
                s_digit = top - 1;
                s_above = above + c0;
            }
            __syncthreads();
            word |= static_cast<uint32_t>(s_digit) << shift;
            left -= s_above;
            __syncthreads();
        }
    } else {
        left = held;  // every row stays: those above 0, and all that equal it
    }
    // chunks in order: a wave counts one chunk, then the counts of the round are added up
    int stays = 0, equals = 0;  // before this round
    for (int c0 = 0; c0 < n_chunks; c0 += kSelectThreads / 64) {
        const int c = c0 + wave;
        int above = 0, equal = 0;
        if (c < n_chunks)
            for (int i = lane; i < kChunk; i += 64) {
                const int row = c * kChunk + i;
                if (row < held) {
                    const uint32_t x = word_of(w[row], row, held, n_sink, n_recent);
                    above += x > word;
                    equal += x == word;
                }
            }
        above = lane_value(wave_prefix_sum(above), 63);
        equal = lane_value(wave_prefix_sum(equal), 63);
        __syncthreads();  // the last round's counts have been read
        if (lane == 0) {
            s_bins[2 * wave] = above;
            s_bins[2 * wave + 1] = equal;
        }
        __syncthreads();
        int mine_above = stays, mine_equal = equals;
        for (int i = 0; i < kSelectThreads / 64; ++i) {
            if (i == wave) { mine_above = stays; mine_equal = equals; }
            stays += s_bins[2 * i];
            equals += s_bins[2 * i + 1];
        }
        if (lane == 0 && c < n_chunks) chunks[static_cast<int64_t>(b) * n_chunks + c] = make_int2(mine_above + min(mine_equal, left), mine_equal);
    }
    for (int j = stay + static_cast<int>(threadIdx.x); j < n_keep; j += kSelectThreads) kept[static_cast<int64_t>(b) * n_keep + j] = -1;
    if (threadIdx.x == 0) {
        borders[b] = {word, left, held, stay};
        if (new_lengths) new_lengths[b] = stay;
    }
}

// Copies rows s_rows[0 .. n) of one array to n rows in a row, in units of type V.
template <typename V>
__device__ __forceinline__ void copy_rows(const unsigned char* __restrict__ src, unsigned char* __restrict__ dst, int row_bytes,
                                          const int* s_rows, int n) {
    const int units = row_bytes / static_cast<int>(sizeof(V));
    const int64_t total = static_cast<int64_t>(n) * units;
    for (int64_t i = threadIdx.x; i < total; i += kMoveThreads) {
        const int j = static_cast<int>(i / units);
        const int u = static_cast<int>(i - static_cast<int64_t>(j) * units);
        reinterpret_cast<V*>(dst)[i] = reinterpret_cast<const V*>(src + static_cast<int64_t>(s_rows[j]) * row_bytes)[u];
    }
}

__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(const float* __restrict__ weights, int T, int n_keep, int n_sink,
                                                                 int n_recent, int n_chunks, const Border* __restrict__ borders,
                                                                 const int2* __restrict__ chunks, Moves moves, int32_t* __restrict__ kept) {
    __shared__ int s_rows[kChunk];
    __shared__ int s_waves[2][kMoveThreads / 64];
    static_assert(kChunk == kMoveThreads, "a thread a row");
    const int64_t b = blockIdx.x / n_chunks;
    const int c = static_cast<int>(blockIdx.x % n_chunks);
    const Border border = borders[b];
    if (c * kChunk >= border.held) return;
    const int2 before = chunks[b * n_chunks + c];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = c * kChunk + static_cast<int>(threadIdx.x);
    uint32_t x = 0;
    const bool here = row < border.held;
    if (here) x = word_of(weights[b * T + row], row, border.held, n_sink, n_recent);
    const unsigned long long equal = __ballot(here && x == border.word);
    if (lane == 0) s_waves[0][wave] = static_cast<int>(__popcll(equal));
    __syncthreads();
    int rank = before.y + __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(equal >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(equal), 0u));
    for (int i = 0; i < wave; ++i) rank += s_waves[0][i];
    const bool stays = here && (x > border.word || (x == border.word && rank < border.equal));
    const unsigned long long mine = __ballot(stays);
    if (lane == 0) s_waves[1][wave] = static_cast<int>(__popcll(mine));
    __syncthreads();
    int place = __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(mine >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(mine), 0u));
    int n = 0;
    for (int i = 0; i < kMoveThreads / 64; ++i) {
        if (i < wave) place += s_waves[1][i];
        n += s_waves[1][i];
    }
    if (stays) {
        s_rows[place] = row;
        kept[b * n_keep + before.x + place] = row;
    }
    __syncthreads();
    for (int a = 0; a < moves.n; ++a) {
        const int row_bytes = moves.row_bytes[a];
        const unsigned char* const src = moves.src[a] + b * T * row_bytes;
        unsigned char* const dst = moves.dst[a] + (b * n_keep + before.x) * row_bytes;
        if (row_bytes % 16 == 0) copy_rows<uint4>(src, dst, row_bytes, s_rows, n);
        else if (row_bytes % 4 == 0) copy_rows<uint32_t>(src, dst, row_bytes, s_rows, n);
        else if (row_bytes % 2 == 0) copy_rows<uint16_t>(src, dst, row_bytes, s_rows, n);
        else copy_rows<unsigned char>(src, dst, row_bytes, s_rows, n);
    }
}

struct Range {
    uintptr_t begin;
    size_t bytes;
};
bool overlap(const Range& x, const Range& y) { return x.begin < y.begin + y.bytes && y.begin < x.begin + x.bytes; }
Range range_of(const void* p, size_t bytes) { return {reinterpret_cast<uintptr_t>(p), bytes}; }

int chunks_of(int32_t T) { return static_cast<int>((static_cast<int64_t>(T) + kChunk - 1) / kChunk); }

}  // namespace

}  // namespace si

using namespace si;

extern "C" {

size_t si_evict_workspace_bytes(int32_t B, int32_t T) {
    if (B < 1 || T < 1) return 0;
    return static_cast<size_t>(B) * (sizeof(Border) + static_cast<size_t>(chunks_of(T)) * sizeof(int2));
}

si_status si_evict_rows(const float* weights, const int32_t* lengths, int32_t B, int32_t T, int32_t n_keep, int32_t n_sink,
                        int32_t n_recent, const si_row_move* moves, int32_t n_moves, int32_t* kept, int32_t* new_lengths,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!weights || !kept || !workspace || (!moves && n_moves != 0)) return SI_ERR_INVALID_ARG;
    if (B < 1 || T < 1 || n_keep < 1 || n_keep > T || n_sink < 0 || n_recent < 0 || n_sink > n_keep || n_recent > n_keep - n_sink)
        return SI_ERR_INVALID_ARG;
    if (n_moves < 0 || n_moves > SI_MAX_ROW_MOVES) return SI_ERR_INVALID_ARG;
    if (!aligned16(weights) || !aligned16(kept) || !aligned16(workspace)) return SI_ERR_INVALID_ARG;
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
    Border* const borders = static_cast<Border*>(workspace);
    int2* const chunks = reinterpret_cast<int2*>(borders + B);
    hipStream_t hs = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(evict_select_kernel, dim3(B), dim3(kSelectThreads), 0, hs, weights, lengths, T, n_keep, n_sink, n_recent, n_chunks,
                       borders, chunks, kept, new_lengths);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) {
        hipLaunchKernelGGL(evict_move_kernel, dim3(static_cast<unsigned>(B) * static_cast<unsigned>(n_chunks)), dim3(kMoveThreads), 0, hs,
                           weights, T, n_keep, n_sink, n_recent, n_chunks, borders, chunks, mv, kept);
        e = hipGetLastError();
    }
    return report(e);
}

}  // extern "C"
