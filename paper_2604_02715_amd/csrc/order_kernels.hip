// Tokens by expert and back: the (token, k) pairs sorted by expert, the tokens' rows copied into that order, the experts' rows
// added up by token, and the gradient of that sum.
#include <algorithm>

#include "block_device.h"
#include "block_ops.h"

namespace fluxmoe {
namespace {

// ================================================================ sort
// A counting sort that keeps an expert's pairs in ascending order, with no atomics on what is ordered.  A wavefront takes 64
// neighbouring pairs at a time; ballots over the bits of the expert's number tell each lane which lanes have the same
// expert, so that a pair's rank among its wavefront's pairs of that expert is what the wavefront had before plus the number
// of equal lanes below.  The wavefronts' counts, added up over wavefronts (and chunks) and experts, give where each begins.

// Pairs of the expert before the pair, within this wavefront's 64 * GROUPS pairs.  hist: this wavefront's counts, [E], zero
// at the start.  e < 0: no expert of the layer.
template <int GROUPS>
__device__ __forceinline__ void rank_pairs(const int32_t* ids, uint32_t first, uint32_t end, uint32_t E, uint16_t* hist,
                                           int32_t (&expert)[GROUPS], uint32_t (&rank)[GROUPS]) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const uint32_t p = first + g * 64 + lane;
        int32_t e = p < end ? ids[p] : -1;
        if (uint32_t(e) >= E) e = -1;
        expert[g] = e;
    }
    const uint32_t bits = 32 - __builtin_clz(E);         // minus one has the bit above those of the numbers below E set, too
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        uint64_t same = ~0ull;
        for (uint32_t b = 0; b < bits; ++b) {
            const bool set = (expert[g] >> b) & 1;
            const uint64_t with = __ballot(set);
            same &= set ? with : ~with;
        }
        const uint32_t below = __builtin_popcountll(same & ((1ull << lane) - 1));
        uint32_t had = 0;
        if (expert[g] >= 0) had = hist[expert[g]];
        wave_fence();
        rank[g] = had + below;
        if (expert[g] >= 0 && below == 0) hist[expert[g]] = uint16_t(had + __builtin_popcountll(same));
        wave_fence();
    }
}

// Exclusive prefix sum of one value per thread over the workgroup; `scratch` holds a value per wavefront.
__device__ __forceinline__ uint32_t exclusive_scan(uint32_t v, uint32_t* scratch, uint32_t& total) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
    uint32_t incl = v;
#pragma unroll
    for (uint32_t d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(incl, d, 64);
        if (lane >= d) incl += o;
    }
    if (lane == 63) scratch[wave] = incl;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
    for (uint32_t w = 0; w < n_waves; ++w) {
        if (w == wave) before = total;
        total += scratch[w];
    }
    __syncthreads();
    return before + incl - v;
}

// From the experts' counts: where their rows begin (each at a multiple of align), the rows of no pair marked.  The whole
// workgroup calls it; start[e] receives the first row of expert e.
__device__ __forceinline__ void place_experts(const SortArgs& a, const uint32_t* count, uint32_t* start, uint32_t* scratch) {
    const uint32_t per = (a.E + blockDim.x - 1) / blockDim.x, e0 = threadIdx.x * per;
    uint32_t sum = 0, total;
    for (uint32_t e = e0; e < min(e0 + per, a.E); ++e) sum += (count[e] + a.align - 1) / a.align * a.align;
    uint32_t at = exclusive_scan(sum, scratch, total);
    for (uint32_t e = e0; e < min(e0 + per, a.E); ++e) {
        const uint32_t n = count[e], padded = (n + a.align - 1) / a.align * a.align;
        start[e] = at;
        a.offsets[e] = int32_t(at);
        a.counts[e] = int32_t(n);
        for (uint32_t r = at + n; r < at + padded; ++r) a.row_pair[r] = -1;
        at += padded;
    }
    if (threadIdx.x == 0) a.offsets[a.E] = int32_t(total);
    for (uint32_t r = total + threadIdx.x; r < a.cap; r += blockDim.x) a.row_pair[r] = -1;
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
    uint32_t n = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const uint32_t c = hist[w * E + e];
        hist[w * E + e] = uint16_t(n);
        n += c;
    }
    return n;
}

// LDS of a sort workgroup: the wavefronts' counts and the experts' first rows; with all pairs in one, the experts' counts and
// the scratch of the scan, too
uint32_t place_lds_bytes(uint32_t waves, uint32_t E) { return (waves * E * 2 + 3) / 4 * 4 + E * 4; }
uint32_t sort_one_lds_bytes(uint32_t waves, uint32_t E) { return place_lds_bytes(waves, E) + E * 4 + 64; }

// All pairs in one workgroup: one launch for decode batches.
template <int WAVES, int GROUPS>
__global__ __launch_bounds__(WAVES * 64) void sort_one_kernel(SortArgs a) {
    extern __shared__ __align__(16) uint32_t lds[];
    uint16_t* hist = reinterpret_cast<uint16_t*>(lds);
    uint32_t* start = lds + (WAVES * a.E * 2 + 3) / 4;
    uint32_t* count = start + a.E;
    uint32_t* scratch = count + a.E;
    const uint32_t wave = threadIdx.x >> 6;
    for (uint32_t i = threadIdx.x; i < (WAVES * a.E + 1) / 2; i += WAVES * 64) lds[i] = 0;
    __syncthreads();
    int32_t expert[GROUPS];
    uint32_t rank[GROUPS];
    rank_pairs<GROUPS>(a.ids, wave * 64 * GROUPS, a.P, a.E, hist + wave * a.E, expert, rank);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.E; e += WAVES * 64) count[e] = over_waves<WAVES>(hist, a.E, e);
    __syncthreads();
    place_experts(a, count, start, scratch);
    __syncthreads();
    write_pairs<GROUPS>(a, wave * 64 * GROUPS, a.P, start, hist + wave * a.E, expert, rank);
}

// Large batches: chunks of kSortChunkPairs pairs.  First each chunk's counts ...
__global__ __launch_bounds__(256) void sort_count_kernel(SortArgs a) {
    extern __shared__ __align__(16) uint32_t lds[];
    for (uint32_t e = threadIdx.x; e < a.E; e += 256) lds[e] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * kSortChunkPairs, end = min(first + kSortChunkPairs, a.P);
    for (uint32_t p = first + threadIdx.x; p < end; p += 256) {
        const uint32_t e = uint32_t(a.ids[p]);
        if (e < a.E) atomicAdd(&lds[e], 1u);
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.E; e += 256) a.chunk_count[uint64_t(blockIdx.x) * a.E + e] = int32_t(lds[e]);
}

// ... then, in one workgroup, for each chunk and expert the pairs in the chunks before, and where the experts begin.  With
// fewer experts than threads, several threads share an expert's chunks.
__global__ __launch_bounds__(1024) void sort_scan_kernel(SortArgs a) {
    extern __shared__ __align__(16) uint32_t lds[];
    uint32_t* start = lds;
    uint32_t* count = start + a.E;
    uint32_t* scratch = count + a.E;
    uint32_t* part = scratch + 16;                       // [parts][E], only where E <= 512
    const uint32_t parts = a.E <= 512 ? 1024 / a.E : 1;
    const uint32_t per = (a.n_chunks + parts - 1) / parts;
    for (uint32_t i = threadIdx.x; i < parts * a.E; i += 1024) {
        const uint32_t e = i % a.E, c0 = min(i / a.E * per, a.n_chunks), c1 = min(c0 + per, a.n_chunks);
        uint32_t n = 0;
#pragma unroll 8
        for (uint32_t c = c0; c < c1; ++c) n += uint32_t(a.chunk_count[uint64_t(c) * a.E + e]);
        if (parts > 1) part[i] = n;
        else count[e] = n;
    }
    __syncthreads();
    if (parts > 1) {
        if (threadIdx.x < a.E) {
            uint32_t n = 0;
            for (uint32_t s = 0; s < parts; ++s) {
                const uint32_t c = part[s * a.E + threadIdx.x];
                part[s * a.E + threadIdx.x] = n;
                n += c;
            }
            count[threadIdx.x] = n;
        }
        __syncthreads();
    }
    for (uint32_t i = threadIdx.x; i < parts * a.E; i += 1024) {
        const uint32_t e = i % a.E, c0 = min(i / a.E * per, a.n_chunks), c1 = min(c0 + per, a.n_chunks);
        uint32_t n = parts > 1 ? part[i] : 0;
#pragma unroll 8
        for (uint32_t c = c0; c < c1; ++c) {
            int32_t& at = a.chunk_count[uint64_t(c) * a.E + e];
            const uint32_t v = uint32_t(at);
            at = int32_t(n);
            n += v;
        }
    }
    place_experts(a, count, start, scratch);
}

// ... and each chunk puts its pairs in place.
template <int WAVES, int GROUPS>
__global__ __launch_bounds__(WAVES * 64) void sort_place_kernel(SortArgs a) {
    static_assert(WAVES * GROUPS * 64 == kSortChunkPairs, "a workgroup ranks a chunk");
    extern __shared__ __align__(16) uint32_t lds[];
    uint16_t* hist = reinterpret_cast<uint16_t*>(lds);
    uint32_t* start = lds + (WAVES * a.E * 2 + 3) / 4;
    const uint32_t wave = threadIdx.x >> 6;
    for (uint32_t i = threadIdx.x; i < (WAVES * a.E + 1) / 2; i += WAVES * 64) lds[i] = 0;
    for (uint32_t e = threadIdx.x; e < a.E; e += WAVES * 64)
        start[e] = uint32_t(a.offsets[e]) + uint32_t(a.chunk_count[uint64_t(blockIdx.x) * a.E + e]);
    __syncthreads();
    const uint32_t chunk = blockIdx.x * kSortChunkPairs, end = min(chunk + kSortChunkPairs, a.P), first = chunk + wave * 64 * GROUPS;
    int32_t expert[GROUPS];
    uint32_t rank[GROUPS];
    rank_pairs<GROUPS>(a.ids, first, end, a.E, hist + wave * a.E, expert, rank);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.E; e += WAVES * 64) (void)over_waves<WAVES>(hist, a.E, e);
    __syncthreads();
    write_pairs<GROUPS>(a, first, end, start, hist + wave * a.E, expert, rank);
}

// ================================================================ rows
// Rows past the tokens: a workgroup behind the tokens' ones looks through kRowsPerPadGroup rows and clears those of no pair.
constexpr uint32_t kRowsPerPadGroup = 16;

template <typename E>      // E: what is cleared at once (16 bytes, or an element)
__device__ __forceinline__ void clear_pad_rows(const int32_t* row_pair, uint32_t cap, uint32_t group, char* rows, uint64_t row_bytes_apart,
                                               uint32_t row_bytes) {
    for (uint32_t r = group * kRowsPerPadGroup; r < min((group + 1) * kRowsPerPadGroup, cap); ++r) {
        if (row_pair[r] >= 0) continue;
        E* dst = reinterpret_cast<E*>(rows + r * row_bytes_apart);
        for (uint32_t i = threadIdx.x; i < row_bytes / sizeof(E); i += blockDim.x) dst[i] = E{};
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
    p.pad_wgs = (cap + kRowsPerPadGroup - 1) / kRowsPerPadGroup;
    return p;
}

// A token's row is read once and written to its K places.
template <typename E>
__global__ __launch_bounds__(1024) void dispatch_kernel(RowsArgs a, uint32_t elem_bytes, uint32_t rows_per_wg, uint32_t token_wgs) {
    const uint32_t row_bytes = a.H * elem_bytes;
    char* rows = static_cast<char*>(a.rows_out);
    const uint64_t apart = a.out_stride * elem_bytes;
    if (blockIdx.x >= token_wgs) {
        clear_pad_rows<E>(a.row_pair, a.cap, blockIdx.x - token_wgs, rows, apart, row_bytes);
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
            const uint32_t r = uint32_t(at[k]);
            if (r < a.cap) reinterpret_cast<E*>(rows + r * apart)[i] = v;
        }
    }
}

constexpr uint32_t kRowsAtOnce = 4;          // of a token's K rows, loads that are on their way together
constexpr uint32_t kRowColumns = 8192;       // eight columns to each lane of 16 wavefronts

// out_t = sum over k of gate * row, in the order of k and in FP32
template <typename R, typename O>
__global__ __launch_bounds__(1024) void combine_kernel(RowsArgs a, uint32_t rows_per_wg) {
    const uint32_t per_row = blockDim.x / rows_per_wg;
    const uint32_t t = __builtin_amdgcn_readfirstlane(blockIdx.x * rows_per_wg + threadIdx.x / per_row);
    if (t >= a.T) return;
    const R* rows = static_cast<const R*>(a.rows_in);
    O* out = static_cast<O*>(a.out) + t * a.out_stride;
    const int32_t* at = a.pair_row + uint64_t(t) * a.K;
    const float* gate = a.gates ? a.gates + uint64_t(t) * a.K : nullptr;
    for (uint32_t c = threadIdx.x % per_row * 8; c < a.H; c += per_row * 8) {
        float acc[8] = {};
        for (uint32_t k0 = 0; k0 < a.K; k0 += kRowsAtOnce) {
            Pack8<R> v[kRowsAtOnce];
            float g[kRowsAtOnce];
#pragma unroll
            for (uint32_t i = 0; i < kRowsAtOnce; ++i) {
                const uint32_t k = min(k0 + i, a.K - 1), r = uint32_t(at[k]);
                if (k0 + i < a.K && r < a.cap) {
                    v[i].load(rows + r * a.in_stride + c);
                    g[i] = gate ? gate[k] : 1.0f;
                } else {
                    v[i].zero();
                    g[i] = 0.0f;
                }
            }
#pragma unroll
            for (uint32_t i = 0; i < kRowsAtOnce; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += g[i] * v[i][j];
        }
        if (a.accumulate) {
            Pack8<O> v;
            v.load(out + c);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += v[j];
        }
        store8(out + c, acc);
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

// d_rows = gate * d_out, d_gates = <d_out, row>: a lane's eight columns of d_out stay in registers for a token's K rows.
template <typename R, typename O>
__global__ __launch_bounds__(1024) void combine_grad_kernel(RowsArgs a, uint32_t rows_per_wg, uint32_t token_wgs) {
    __shared__ float s_dot[16][kRouteMaxTopK];           // the wavefronts' parts of the K products
    R* d_rows = static_cast<R*>(a.rows_out);
    if (blockIdx.x >= token_wgs) {
        clear_pad_rows<uint4>(a.row_pair, a.cap, blockIdx.x - token_wgs, static_cast<char*>(a.rows_out), a.out_stride * sizeof(R), a.H * sizeof(R));
        return;
    }
    const uint32_t per_row = blockDim.x / rows_per_wg, waves = per_row / 64;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), in_row = threadIdx.x % per_row;
    const uint32_t t = __builtin_amdgcn_readfirstlane(blockIdx.x * rows_per_wg + threadIdx.x / per_row);
    const bool valid = t < a.T;
    const uint32_t c = in_row * 8;
    const bool in = valid && c < a.H;
    const R* rows = static_cast<const R*>(a.rows_in);
    const int32_t* at = a.pair_row + uint64_t(valid ? t : 0) * a.K;
    const float* gate = a.gates + uint64_t(valid ? t : 0) * a.K;
    Pack8<O> d;
    if (in) d.load(static_cast<const O*>(a.x) + t * a.x_stride + c);
    else d.zero();
    for (uint32_t k0 = 0; k0 < a.K; k0 += kRowsAtOnce) {
        Pack8<R> v[kRowsAtOnce];
        uint32_t r[kRowsAtOnce];
#pragma unroll
        for (uint32_t i = 0; i < kRowsAtOnce; ++i) {
            r[i] = valid && k0 + i < a.K ? uint32_t(at[min(k0 + i, a.K - 1)]) : ~0u;
            if (in && r[i] < a.cap) v[i].load(rows + r[i] * a.in_stride + c);
            else v[i].zero();
        }
#pragma unroll
        for (uint32_t i = 0; i < kRowsAtOnce; ++i) {
            if (k0 + i >= a.K) break;
            float dot = 0.0f;
            if (r[i] < a.cap) {
                const float g = gate[k0 + i];
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    dot += d[j] * v[i][j];
                    o[j] = g * d[j];
                }
                if (in) store8(d_rows + r[i] * a.out_stride + c, o);
            }
            dot = group_sum<64>(dot);
            if ((threadIdx.x & 63) == 0) s_dot[wave][k0 + i] = dot;
        }
    }
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
        clear_pad_rows<R>(a.row_pair, a.cap, blockIdx.x - token_wgs, static_cast<char*>(a.rows_out), a.out_stride * sizeof(R), a.H * sizeof(R));
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
        const RowPlan p = row_plan(a.T, 0, a.H / 8);
        hipLaunchKernelGGL((combine_kernel<R, O>), dim3(p.token_wgs), dim3(p.threads), 0, stream, a, p.rows_per_wg);
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
    hipLaunchKernelGGL((sort_one_kernel<WAVES, GROUPS>), dim3(1), dim3(WAVES * 64), sort_one_lds_bytes(WAVES, a.E), stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sort(const SortArgs& a, hipStream_t stream) {
    if (a.n_chunks == 0) {
        // up to 40 KiB of LDS: 2-byte counts of each wavefront and two words for every expert
        if (a.P <= 256) return go_sort_one<4, 1>(a, stream);
        if (a.E > 1024) return go_sort_one<4, 16>(a, stream);
        if (a.P <= 1024) return go_sort_one<16, 1>(a, stream);
        return go_sort_one<16, 4>(a, stream);
    }
    hipLaunchKernelGGL(sort_count_kernel, dim3(a.n_chunks), dim3(256), a.E * 4, stream, a);
    hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), a.E * 8 + 64 + (a.E <= 512 ? 4096 : 0), stream, a);
    hipLaunchKernelGGL((sort_place_kernel<4, 4>), dim3(a.n_chunks), dim3(256), place_lds_bytes(4, a.E), stream, a);
    return hipGetLastError();
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
