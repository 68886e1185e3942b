// Tokens by expert and back: the (token, k) pairs sorted by expert, the tokens' rows copied into that order, the experts' rows
// added up by token, and the gradient of that sum.
#include <algorithm>
#include <type_traits>

#include "block_device.h"
#include "block_ops.h"

namespace fluxmoe {
namespace {

// ================================================================ sort
// A counting sort that keeps an expert's pairs in ascending order, with no atomics on what is ordered.  A wavefront takes 64
// neighbouring pairs at a time; ballots over the bits of the expert's number tell each lane which lanes have the same
// expert, so that a pair's rank among its wavefront's pairs of that expert is what the wavefront had before plus the number
// of equal lanes below.  The wavefronts' counts, added up over wavefronts (and chunks) and experts, give where each begins.
// A few bytes for each pair: bound by the launches and by the steps that follow each other inside them.  Measured (us, a launch's own
// 2.1 included): 10 pairs 2.8; 4096 pairs of 160 experts in one workgroup 5.9; 16384 of 8 5.9 (two launches); 81920 of 512 11.2 and
// 655360 of 512 19 (three).

// The experts of this wavefront's 64 * GROUPS pairs, -1: none of the layer's.
template <int GROUPS>
__device__ __forceinline__ void load_experts(const int32_t* ids, uint32_t first, uint32_t end, uint32_t E, int32_t (&expert)[GROUPS]) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const uint32_t p = first + g * 64 + (threadIdx.x & 63);
        const int32_t e = p < end ? ids[p] : -1;
        expert[g] = uint32_t(e) < E ? e : -1;
    }
}

// Pairs of the expert before the pair, within this wavefront's.  hist: this wavefront's counts, [E], zero at the start.
template <int GROUPS>
__device__ __forceinline__ void rank_pairs(uint32_t E, uint16_t* hist, const int32_t (&expert)[GROUPS], uint32_t (&rank)[GROUPS]) {
    const uint32_t bits = 32 - __builtin_clz(E);         // minus one has the bit above those of the numbers below E set, too
    uint32_t same[GROUPS][2];                            // the lanes with the lane's expert, low and high half
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) same[g][0] = same[g][1] = ~0u;
    for (uint32_t b = 0; b < bits; ++b) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const uint32_t mine = uint32_t(__builtin_amdgcn_sbfe(expert[g], b, 1));       // all bits the lane's bit b
            const uint64_t with = __ballot(mine != 0);
            same[g][0] &= ~(uint32_t(with) ^ mine);
            same[g][1] &= ~(uint32_t(with >> 32) ^ mine);
        }
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const uint32_t below = __builtin_amdgcn_mbcnt_hi(same[g][1], __builtin_amdgcn_mbcnt_lo(same[g][0], 0));
        uint32_t had = 0;
        if (expert[g] >= 0) had = hist[expert[g]];
        wave_fence();
        rank[g] = had + below;
        if (expert[g] >= 0 && below == 0) hist[expert[g]] = uint16_t(had + __builtin_popcount(same[g][0]) + __builtin_popcount(same[g][1]));
        wave_fence();
    }
}

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_0(uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, ROWS, 0xF, false));
}

// Exclusive prefix sum of one value per thread over the workgroup; `scratch` holds a value per wavefront.
template <int WAVES>
__device__ __forceinline__ uint32_t exclusive_scan(uint32_t v, uint32_t* scratch, uint32_t& total) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t incl = v;                                   // within 16 lanes, then across the four sixteens
    incl += dpp_or_0<0x111, 0xF>(incl);                  // the lane 1, 2, 4, 8 below
    incl += dpp_or_0<0x112, 0xF>(incl);
    incl += dpp_or_0<0x114, 0xF>(incl);
    incl += dpp_or_0<0x118, 0xF>(incl);
    incl += dpp_or_0<0x142, 0xA>(incl);                  // the last lane of the sixteen before, to the second and fourth
    incl += dpp_or_0<0x143, 0xC>(incl);                  // lane 31, to the upper half
    if (lane == 63) scratch[wave] = incl;
    __syncthreads();
    uint32_t part[WAVES], before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) part[w] = scratch[w];
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += uint32_t(w) < wave ? part[w] : 0;
        total += part[w];
    }
    return before + incl - v;
}

// Rows first .. cap - 1 without a pair, by neighbouring threads.  Where groups have gaps this goes over all rows before the pairs get
// theirs (each expert's thread marking its own gap took 37 us for 400 x 10 of 512 at 128, this 9); at align 1 only the rows past
// the last group are marked, when that is known (8192 x 2 of 8 and the rows' copy 36.5 us, 37.3 with all rows marked first).
__device__ __forceinline__ void clear_rows(const SortArgs& a, uint32_t first, uint32_t thread, uint32_t threads) {
    typedef int32_t four __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t n = a.cap - first;
    int32_t* rows = a.row_pair + first;
    for (uint32_t i = thread; i < n / 4; i += threads) *reinterpret_cast<four*>(rows + uint64_t(i) * 4) = four{-1, -1, -1, -1};
    if (thread < n % 4) rows[n - 1 - thread] = -1;
}

// From the experts' counts: where their rows begin (each at a multiple of align).  The whole workgroup calls it; start[e] holds
// expert e's count and receives its first row.  Only the workgroup that is asked to writes offsets and counts.
template <int WAVES>
__device__ __forceinline__ void place_experts(const SortArgs& a, uint32_t* start, uint32_t* scratch, bool write) {
    const uint32_t per = (a.E + WAVES * 64 - 1) / (WAVES * 64), e0 = threadIdx.x * per, e1 = min(e0 + per, a.E);
    auto pad = [&](uint32_t n) { return a.align == 1 ? n : (n + a.align - 1) / a.align * a.align; };
    uint32_t sum = 0, total;
    for (uint32_t e = e0; e < e1; ++e) sum += pad(start[e]);
    uint32_t at = exclusive_scan<WAVES>(sum, scratch, total);
    for (uint32_t e = e0; e < e1; ++e) {
        const uint32_t n = start[e], padded = per == 1 ? sum : pad(n);
        start[e] = at;
        if (write) {
            a.offsets[e] = int32_t(at);
            a.counts[e] = int32_t(n);
        }
        at += padded;
    }
    if (write && threadIdx.x == 0) a.offsets[a.E] = int32_t(total);
    if (a.align == 1) clear_rows(a, total, blockIdx.x * (WAVES * 64) + threadIdx.x, gridDim.x * (WAVES * 64));
}

template <int GROUPS>
__device__ __forceinline__ void write_pairs(const SortArgs& a, uint32_t first, uint32_t end, const uint32_t* start, const uint16_t* before,
                                            const int32_t (&expert)[GROUPS], const uint32_t (&rank)[GROUPS]) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const uint32_t p = first + g * 64 + (threadIdx.x & 63);
        if (p >= end) continue;
        const int32_t e = expert[g];
        const int32_t row = e >= 0 ? int32_t(start[e] + before[e] + rank[g]) : -1;
        a.pair_row[p] = row;
        if (row >= 0) a.row_pair[row] = int32_t(p);
    }
}

// The wavefronts' counts become the number of pairs in the wavefronts before; returns the expert's sum.
template <int WAVES>
__device__ __forceinline__ uint32_t over_waves(uint16_t* hist, uint32_t E, uint32_t e) {
    uint32_t c[WAVES], n = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) c[w] = hist[w * E + e];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        hist[w * E + e] = uint16_t(n);
        n += c[w];
    }
    return n;
}

// LDS of a sort workgroup: the wavefronts' counts, `words` for each expert, the scratch of the scan.  48 KiB at most (2048 experts,
// 8 wavefronts, 2 words).
uint32_t sort_lds_bytes(uint32_t waves, uint32_t E, uint32_t words) { return (waves * E * 2 + 3) / 4 * 4 + words * E * 4 + 64; }

// All pairs in one workgroup: one launch for decode batches.
template <int WAVES, int GROUPS>
__global__ __launch_bounds__(WAVES * 64) void sort_one_kernel(SortArgs a) {
    extern __shared__ __align__(16) uint32_t lds[];
    uint16_t* hist = reinterpret_cast<uint16_t*>(lds);
    uint32_t* start = lds + (WAVES * a.E * 2 + 3) / 4;
    uint32_t* scratch = start + a.E;
    const uint32_t wave = threadIdx.x >> 6;
    int32_t expert[GROUPS];
    if (a.align != 1) clear_rows(a, 0, threadIdx.x, WAVES * 64);
    load_experts<GROUPS>(a.ids, wave * 64 * GROUPS, a.P, a.E, expert);
    for (uint32_t i = threadIdx.x; i < (WAVES * a.E + 1) / 2; i += WAVES * 64) lds[i] = 0;
    __syncthreads();
    uint32_t rank[GROUPS];
    rank_pairs<GROUPS>(a.E, hist + wave * a.E, expert, rank);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.E; e += WAVES * 64) start[e] = over_waves<WAVES>(hist, a.E, e);
    __syncthreads();
    place_experts<WAVES>(a, start, scratch, true);
    __syncthreads();
    write_pairs<GROUPS>(a, wave * 64 * GROUPS, a.P, start, hist + wave * a.E, expert, rank);
}

// Large batches: chunks of kSortChunkPairs pairs.  First each chunk's counts (and where groups have gaps, all rows without a pair) ...
__global__ __launch_bounds__(256) void sort_count_kernel(SortArgs a) {
    extern __shared__ __align__(16) uint32_t lds[];
    for (uint32_t e = threadIdx.x; e < a.E; e += 256) lds[e] = 0;
    if (a.align != 1) clear_rows(a, 0, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
    __syncthreads();
    const uint32_t first = blockIdx.x * kSortChunkPairs, end = min(first + kSortChunkPairs, a.P);
    for (uint32_t p = first + threadIdx.x; p < end; p += 256) {
        const uint32_t e = uint32_t(a.ids[p]);
        if (e < a.E) atomicAdd(&lds[e], 1u);
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.E; e += 256) a.chunk_count[uint64_t(blockIdx.x) * a.E + e] = int32_t(lds[e]);
}

// ... then, for 16 experts to a workgroup, what each chunk has in the chunks before, and what the experts have in all: 64 threads
// share an expert's chunks.
__global__ __launch_bounds__(1024) void sort_scan_kernel(SortArgs a) {
    __shared__ uint32_t part[64][17];
    const uint32_t lane = threadIdx.x & 15, share = threadIdx.x >> 4, e = blockIdx.x * 16 + lane;
    const uint32_t per = (a.n_chunks + 63) / 64, c0 = min(share * per, a.n_chunks), c1 = min(c0 + per, a.n_chunks);
    uint32_t n = 0;
    if (e < a.E) {
#pragma unroll 4
        for (uint32_t c = c0; c < c1; ++c) n += uint32_t(a.chunk_count[uint64_t(c) * a.E + e]);
    }
    part[share][lane] = n;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (uint32_t s = 0; s < 64; ++s) {
        const uint32_t p = part[s][lane];
        before += s < share ? p : 0;
        all += p;
    }
    if (e >= a.E) return;
    if (share == 0) a.counts[e] = int32_t(all);
    for (uint32_t c = c0; c < c1; ++c) {
        int32_t& at = a.chunk_count[uint64_t(c) * a.E + e];
        const uint32_t v = uint32_t(at);
        at = int32_t(before);
        before += v;
    }
}

// Up to so many counts of chunks a launch less pays (16 chunks of 160 experts 8.0 us against 9.6, 32 of 160 9.6 / 10.1, 80 of 512
// 34 / 11).
constexpr uint32_t kAddCounts = 5120;

// ... and each chunk puts its pairs in place, after it has worked out where the experts begin (the first one also writes that).
// ADD: it adds up the counts of the chunks before it and of all itself, a launch less for reading all of them.
template <int WAVES, int GROUPS, bool ADD>
__global__ __launch_bounds__(WAVES * 64) void sort_place_kernel(SortArgs a) {
    static_assert(WAVES * GROUPS * 64 == kSortChunkPairs, "a workgroup ranks a chunk");
    extern __shared__ __align__(16) uint32_t lds[];
    uint16_t* hist = reinterpret_cast<uint16_t*>(lds);
    uint32_t* start = lds + (WAVES * a.E * 2 + 3) / 4;
    const uint32_t wave = threadIdx.x >> 6;
    const uint32_t chunk = blockIdx.x * kSortChunkPairs, end = min(chunk + kSortChunkPairs, a.P), first = chunk + wave * 64 * GROUPS;
    int32_t expert[GROUPS];
    load_experts<GROUPS>(a.ids, first, end, a.E, expert);
    for (uint32_t i = threadIdx.x; i < (WAVES * a.E + 1) / 2; i += WAVES * 64) lds[i] = 0;
    uint32_t* before = start + a.E;                      // ADD only
    uint32_t* scratch = ADD ? before + a.E : before;
    if constexpr (ADD) {
        for (uint32_t e = threadIdx.x; e < 2 * a.E; e += WAVES * 64) start[e] = 0;
        __syncthreads();
        const uint32_t total = a.n_chunks * a.E, own = blockIdx.x * a.E;
#pragma unroll 8
        for (uint32_t i = threadIdx.x; i < total; i += WAVES * 64) {
            const uint32_t n = uint32_t(a.chunk_count[i]), e = i % a.E;
            if (n) {
                atomicAdd(&start[e], n);
                if (i < own) atomicAdd(&before[e], n);
            }
        }
    } else {
        for (uint32_t e = threadIdx.x; e < a.E; e += WAVES * 64) start[e] = uint32_t(a.counts[e]);
    }
    __syncthreads();
    place_experts<WAVES>(a, start, scratch, blockIdx.x == 0);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.E; e += WAVES * 64)
        start[e] += ADD ? before[e] : uint32_t(a.chunk_count[uint64_t(blockIdx.x) * a.E + e]);
    __syncthreads();
    uint32_t rank[GROUPS];
    rank_pairs<GROUPS>(a.E, hist + wave * a.E, expert, rank);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.E; e += WAVES * 64) (void)over_waves<WAVES>(hist, a.E, e);
    __syncthreads();
    write_pairs<GROUPS>(a, first, end, start, hist + wave * a.E, expert, rank);
}

// ================================================================ rows
// Rows past the tokens: a workgroup behind the tokens' ones looks through kRowsPerPadGroup rows and clears those of no pair, and
// goes on to further ones where there are more than kMostPadGroups times that (a launch has fewer than 2^32 threads).
constexpr uint32_t kRowsPerPadGroup = 16, kMostPadGroups = 1u << 20;

template <typename E>      // E: what is cleared at once (16 bytes, or an element)
__device__ __forceinline__ void clear_pad_rows(const int32_t* row_pair, uint32_t cap, uint32_t token_wgs, char* rows, uint64_t row_bytes_apart,
                                               uint32_t row_bytes) {
    const uint32_t lane = threadIdx.x & 63, step = (gridDim.x - token_wgs) * kRowsPerPadGroup;
    for (uint32_t first = (blockIdx.x - token_wgs) * kRowsPerPadGroup; first < cap; first += step) {
        uint64_t pads = __ballot(lane < kRowsPerPadGroup && first + lane < cap && row_pair[min(first + lane, cap - 1)] < 0);
        for (; pads; pads &= pads - 1) {
            const uint64_t r = first + __builtin_ctzll(pads);
            E* dst = reinterpret_cast<E*>(rows + r * row_bytes_apart);
            for (uint32_t i = threadIdx.x; i < row_bytes / sizeof(E); i += blockDim.x) dst[i] = E{};
        }
    }
}

struct RowPlan {
    uint32_t threads, rows_per_wg, token_wgs, pad_wgs;
};
// `units`: what a thread takes at once, to a row
RowPlan row_plan(uint32_t T, uint32_t cap, uint32_t units) {
    RowPlan p;
    const uint32_t waves = std::min(std::max((units + 63) / 64, 1u), 16u);
    p.rows_per_wg = waves >= 3 ? 1 : 4 / waves;
    p.threads = 64 * waves * p.rows_per_wg;
    p.token_wgs = (T + p.rows_per_wg - 1) / p.rows_per_wg;
    p.pad_wgs = std::min((cap + kRowsPerPadGroup - 1) / kRowsPerPadGroup, kMostPadGroups);
    return p;
}

__device__ __forceinline__ void store_past(uint4* p, const uint4& v) { store_stream16(p, v); }
template <typename E>
__device__ __forceinline__ void store_past(E* p, E v) { *p = v; }

// A token's row is read once and written to its K places: the places past the caches (8192 x 4096 top-2 31 us, 6.6 TB/s; through
// them 38; past the caches for the row, too, 38).  512 x 5120 top-8 with groups at multiples of 16 rows, 40 % of them of no pair,
// 13.8 us (5.2 TB/s).
template <typename E>
__global__ __launch_bounds__(1024) void dispatch_kernel(RowsArgs a, uint32_t elem_bytes, uint32_t rows_per_wg, uint32_t token_wgs) {
    const uint32_t row_bytes = a.H * elem_bytes;
    char* rows = static_cast<char*>(a.rows_out);
    const uint64_t apart = a.out_stride * elem_bytes;
    if (blockIdx.x >= token_wgs) {
        clear_pad_rows<E>(a.row_pair, a.cap, token_wgs, rows, apart, row_bytes);
        return;
    }
    const uint32_t per_row = blockDim.x / rows_per_wg;
    const uint32_t t = __builtin_amdgcn_readfirstlane(blockIdx.x * rows_per_wg + threadIdx.x / per_row);
    if (t >= a.T) return;
    const E* src = reinterpret_cast<const E*>(static_cast<const char*>(a.x) + t * (a.x_stride * elem_bytes));
    const int32_t* at = a.pair_row + uint64_t(t) * a.K;
    for (uint32_t i = threadIdx.x % per_row; i < row_bytes / sizeof(E); i += per_row) {
        const E v = src[i];
        for (uint32_t k = 0; k < a.K; ++k) {
            const uint32_t r = uint32_t(scalar_at(at, k));
            if (r < a.cap) store_past(reinterpret_cast<E*>(rows + r * apart) + i, v);
        }
    }
}

constexpr uint32_t kRowColumns = 8192;       // eight columns to each lane of 16 wavefronts

// out_t = sum over k of gate * row, in the order of k and in FP32.  Bound by memory: 4001 tokens of ten rows of 2048, BF16 to FP32,
// 33 us (6.0 TB/s; four rows of 1024 to a token 6.2, one of 4096 4.9, and 5.7 in one type).  What a row's address needs comes through the scalar cache for
// four rows together, so that four rows' loads are under way; fetched row by row through the vector caches it was 44 us.
template <typename R, int N, int ROWS>
__device__ __forceinline__ void add_rows(const RowsArgs& a, const int32_t* at, const float* gate, uint32_t c, float (&acc)[N]) {
    uint32_t r[ROWS];
    float g[ROWS];
    Pack<R, N> v[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        r[i] = uint32_t(scalar_at(at, i));
        g[i] = gate ? scalar_at(gate, i) : 1.0f;
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const bool here = r[i] < a.cap;
        v[i].template load<kStream>(row_at(static_cast<const R*>(a.rows_in), here ? r[i] : 0, a.in_stride, here ? a.H : 0), c);
        g[i] = here ? g[i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] += g[i] * v[i][j];
}

template <typename R, typename O, int N>
__global__ __launch_bounds__(1024) void combine_kernel(RowsArgs a, uint32_t rows_per_wg) {
    const uint32_t per_row = blockDim.x / rows_per_wg;
    const uint32_t t = __builtin_amdgcn_readfirstlane(blockIdx.x * rows_per_wg + threadIdx.x / per_row);
    if (t >= a.T) return;
    const row_t out = row_at(static_cast<O*>(a.out), t, a.out_stride, a.H);
    const int32_t* at = a.pair_row + uint64_t(t) * a.K;
    const float* gate = a.gates ? a.gates + uint64_t(t) * a.K : nullptr;
    for (uint32_t c = threadIdx.x % per_row * N; c < a.H; c += per_row * N) {
        float acc[N] = {};
        uint32_t k = 0;
        for (; k + 4 <= a.K; k += 4) add_rows<R, N, 4>(a, at + k, gate ? gate + k : nullptr, c, acc);
        if (k + 2 <= a.K) {
            add_rows<R, N, 2>(a, at + k, gate ? gate + k : nullptr, c, acc);
            k += 2;
        }
        if (k < a.K) add_rows<R, N, 1>(a, at + k, gate ? gate + k : nullptr, c, acc);
        if (a.accumulate) {
            Pack<O, N> v;
            v.template load<kCached>(out, c);
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] += v[j];
        }
        store<O, N, kStream>(out, c, acc);
    }
}

// Any width and alignment: a column at a time.
template <typename R, typename O>
__global__ __launch_bounds__(1024) void combine_any_kernel(RowsArgs a) {
    const uint32_t t = blockIdx.x;
    const R* rows = static_cast<const R*>(a.rows_in);
    O* out = static_cast<O*>(a.out) + t * a.out_stride;
    for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
        float acc = 0.0f;
        for (uint32_t k = 0; k < a.K; ++k) {
            const uint32_t r = uint32_t(a.pair_row[uint64_t(t) * a.K + k]);
            if (r < a.cap) acc += (a.gates ? a.gates[uint64_t(t) * a.K + k] : 1.0f) * to_float(rows[r * a.in_stride + c]);
        }
        from_float(out + c, a.accumulate ? acc + to_float(out[c]) : acc);
    }
}

// d_rows = gate * d_out, d_gates = <d_out, row>: a lane's eight columns of d_out stay in registers for a token's K rows.  Bound by
// memory: 2048 tokens of eight rows of 5120, BF16, 69 us (5.2 TB/s: eight rows read and eight written at as many places).  Walking
// through the tokens with the next rows' loads under way took 68.7, taking the rows in their own order 70 to 72.
template <typename R, typename O>
__global__ __launch_bounds__(1024) void combine_grad_kernel(RowsArgs a, uint32_t rows_per_wg, uint32_t token_wgs) {
    constexpr int N = kPiece<R, O>, P = 8 / N;           // columns of a piece, pieces of a lane
    __shared__ float s_dot[16][kRouteMaxTopK];           // the wavefronts' parts of the K products
    R* d_rows = static_cast<R*>(a.rows_out);
    if (blockIdx.x >= token_wgs) {
        clear_pad_rows<uint4>(a.row_pair, a.cap, token_wgs, static_cast<char*>(a.rows_out), a.out_stride * sizeof(R), a.H * sizeof(R));
        return;
    }
    const uint32_t per_row = blockDim.x / rows_per_wg, waves = per_row / 64;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), in_row = threadIdx.x % per_row;
    const uint32_t t = __builtin_amdgcn_readfirstlane(blockIdx.x * rows_per_wg + threadIdx.x / per_row);
    const bool valid = t < a.T;
    const int32_t* at = a.pair_row + uint64_t(valid ? t : 0) * a.K;
    const float* gate = a.gates + uint64_t(valid ? t : 0) * a.K;
    uint32_t c[P];
    Pack<O, N> d[P];
    const row_t d_out = row_at(static_cast<const O*>(a.x), valid ? t : 0, a.x_stride, valid ? a.H : 0);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        c[p] = (p * per_row + in_row) * N;
        d[p].template load<kStream>(d_out, c[p]);
    }
    auto some = [&](uint32_t k0, auto rows_at_once) {
        constexpr int ROWS = decltype(rows_at_once)::value;
        uint32_t r[ROWS];
        float g[ROWS];
        Pack<R, N> v[ROWS][P];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            r[i] = uint32_t(scalar_at(at, k0 + i));
            g[i] = scalar_at(gate, k0 + i);
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const bool here = valid && r[i] < a.cap;
            const row_t row = row_at(static_cast<const R*>(a.rows_in), here ? r[i] : 0, a.in_stride, here ? a.H : 0);
#pragma unroll
            for (int p = 0; p < P; ++p) v[i][p].template load<kStream>(row, c[p]);
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const bool here = valid && r[i] < a.cap;
            const row_t row = row_at(d_rows, here ? r[i] : 0, a.out_stride, here ? a.H : 0);
            float dot = 0.0f;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float o[N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    dot += d[p][j] * v[i][p][j];
                    o[j] = g[i] * d[p][j];
                }
                store<R, N, kStream>(row, c[p], o);
            }
            dot = group_sum<64>(dot);
            if ((threadIdx.x & 63) == 0) s_dot[wave][k0 + i] = here ? dot : 0.0f;
        }
    };
    uint32_t k = 0;
    for (; k + 4 <= a.K; k += 4) some(k, std::integral_constant<int, 4>());
    if (k + 2 <= a.K) {
        some(k, std::integral_constant<int, 2>());
        k += 2;
    }
    if (k < a.K) some(k, std::integral_constant<int, 1>());
    __syncthreads();
    if (valid && in_row < a.K) {
        float sum = 0.0f;
        for (uint32_t w = 0; w < waves; ++w) sum += s_dot[wave + w][in_row];     // in_row < 64: the row's first wavefront
        a.d_gates[uint64_t(t) * a.K + in_row] = sum;
    }
}

// Any width and alignment: a column at a time, d_out read again for each row.
template <typename R, typename O>
__global__ __launch_bounds__(1024) void combine_grad_any_kernel(RowsArgs a, uint32_t token_wgs) {
    __shared__ float s_dot[16][kRouteMaxTopK];
    R* d_rows = static_cast<R*>(a.rows_out);
    if (blockIdx.x >= token_wgs) {
        clear_pad_rows<R>(a.row_pair, a.cap, token_wgs, static_cast<char*>(a.rows_out), a.out_stride * sizeof(R), a.H * sizeof(R));
        return;
    }
    const uint32_t t = blockIdx.x;
    const R* rows = static_cast<const R*>(a.rows_in);
    const O* d_out = static_cast<const O*>(a.x) + t * a.x_stride;
    for (uint32_t k = 0; k < a.K; ++k) {
        const uint32_t r = uint32_t(a.pair_row[uint64_t(t) * a.K + k]);
        float dot = 0.0f;
        if (r < a.cap) {
            const float g = a.gates[uint64_t(t) * a.K + k];
            for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
                const float d = to_float(d_out[c]);
                dot += d * to_float(rows[r * a.in_stride + c]);
                from_float(d_rows + r * a.out_stride + c, g * d);
            }
        }
        dot = group_sum<64>(dot);
        if ((threadIdx.x & 63) == 0) s_dot[threadIdx.x >> 6][k] = dot;
    }
    __syncthreads();
    if (threadIdx.x < a.K) {
        float sum = 0.0f;
        for (uint32_t w = 0; w < blockDim.x / 64; ++w) sum += s_dot[w][threadIdx.x];
        a.d_gates[uint64_t(t) * a.K + threadIdx.x] = sum;
    }
}

uint32_t any_threads(uint32_t H) { return H >= 1024 ? 1024 : (H + 63) / 64 * 64; }

template <typename R, typename O>
hipError_t go_combine(const RowsArgs& a, hipStream_t stream) {
    if (a.vec) {
        constexpr int N = kPiece<R, O>;
        const RowPlan p = row_plan(a.T, 0, a.H / N);
        hipLaunchKernelGGL((combine_kernel<R, O, N>), dim3(p.token_wgs), dim3(p.threads), 0, stream, a, p.rows_per_wg);
    } else {
        hipLaunchKernelGGL((combine_any_kernel<R, O>), dim3(a.T), dim3(any_threads(a.H)), 0, stream, a);
    }
    return hipGetLastError();
}

template <typename R, typename O>
hipError_t go_combine_grad(const RowsArgs& a, hipStream_t stream) {
    if (a.vec && a.H <= kRowColumns) {
        const RowPlan p = row_plan(a.T, a.cap, a.H / 8);
        hipLaunchKernelGGL((combine_grad_kernel<R, O>), dim3(p.token_wgs + p.pad_wgs), dim3(p.threads), 0, stream, a, p.rows_per_wg, p.token_wgs);
    } else {
        const RowPlan p = row_plan(a.T, a.cap, 1024);
        hipLaunchKernelGGL((combine_grad_any_kernel<R, O>), dim3(a.T + p.pad_wgs), dim3(any_threads(a.H)), 0, stream, a, a.T);
    }
    return hipGetLastError();
}

template <int WAVES, int GROUPS>
hipError_t go_sort_one(const SortArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((sort_one_kernel<WAVES, GROUPS>), dim3(1), dim3(WAVES * 64), sort_lds_bytes(WAVES, a.E, 1), stream, a);
    return hipGetLastError();
}

template <int WAVES, int GROUPS, bool ADD>
hipError_t go_sort_place(const SortArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((sort_place_kernel<WAVES, GROUPS, ADD>), dim3(a.n_chunks), dim3(WAVES * 64), sort_lds_bytes(WAVES, a.E, ADD ? 2 : 1), stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sort(const SortArgs& a, hipStream_t stream) {
    if (a.n_chunks == 0) {
        // up to 40 KiB of LDS: 2-byte counts of each wavefront and two words for every expert
        if (a.P <= 256) return go_sort_one<4, 1>(a, stream);
        if (a.E > 1024) return go_sort_one<4, 16>(a, stream);
        if (a.P <= 1024) return go_sort_one<16, 1>(a, stream);
        if (a.P <= 2048) return go_sort_one<16, 2>(a, stream);
        return go_sort_one<16, 4>(a, stream);
    }
    hipLaunchKernelGGL(sort_count_kernel, dim3(a.n_chunks), dim3(256), a.E * 4, stream, a);
    if (a.E <= 2048 && uint64_t(a.n_chunks) * a.E <= kAddCounts) return go_sort_place<8, 2, true>(a, stream);
    hipLaunchKernelGGL(sort_scan_kernel, dim3((a.E + 15) / 16), dim3(1024), 0, stream, a);
    return a.E <= 2048 ? go_sort_place<8, 2, false>(a, stream) : go_sort_place<4, 4, false>(a, stream);
}

hipError_t launch_dispatch(const RowsArgs& a, uint32_t elem_bytes, hipStream_t stream) {
    const uint32_t unit = a.vec ? 16 : elem_bytes;
    const RowPlan p = row_plan(a.T, a.cap, a.H * elem_bytes / unit);
    const dim3 grid(p.token_wgs + p.pad_wgs), wg(p.threads);
    if (unit == 16) hipLaunchKernelGGL(dispatch_kernel<uint4>, grid, wg, 0, stream, a, elem_bytes, p.rows_per_wg, p.token_wgs);
    else if (unit == 4) hipLaunchKernelGGL(dispatch_kernel<uint32_t>, grid, wg, 0, stream, a, elem_bytes, p.rows_per_wg, p.token_wgs);
    else hipLaunchKernelGGL(dispatch_kernel<uint16_t>, grid, wg, 0, stream, a, elem_bytes, p.rows_per_wg, p.token_wgs);
    return hipGetLastError();
}

hipError_t launch_combine(const RowsArgs& a, bool rows_f32, bool out_f32, hipStream_t stream) {
    if (rows_f32) return out_f32 ? go_combine<float, float>(a, stream) : go_combine<float, bf16_t>(a, stream);
    return out_f32 ? go_combine<bf16_t, float>(a, stream) : go_combine<bf16_t, bf16_t>(a, stream);
}

hipError_t launch_combine_grad(const RowsArgs& a, bool rows_f32, bool out_f32, hipStream_t stream) {
    if (rows_f32) return out_f32 ? go_combine_grad<float, float>(a, stream) : go_combine_grad<float, bf16_t>(a, stream);
    return out_f32 ? go_combine_grad<bf16_t, float>(a, stream) : go_combine_grad<bf16_t, bf16_t>(a, stream);
}

}  // namespace fluxmoe
