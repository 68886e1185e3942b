// Arguments and launchers of the operators around the routed experts: router, tokens by expert, norms.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace fluxmoe {

// ---------------------------------------------------------------- router (route_kernels.hip)
constexpr uint32_t kRouteMaxExperts = 4096;
constexpr uint32_t kRouteMaxTopK = 64;       // a lane of the wavefront keeps a chosen expert

struct RouteArgs {
    const void* logits;          // [T][E], rows row_stride elements apart
    const float* bias;           // [E] or nullptr, sigmoid only
    int32_t* ids;                // [T][K]
    float* gates;                // [T][K]
    const float* d_gates;        // gradient only: [T][K]
    void* d_logits;              // gradient only: [T][E], rows d_stride elements apart
    uint64_t row_stride, d_stride;
    uint32_t T, E, K;
    uint32_t renormalize;
    uint32_t vec, d_vec;         // rows are 16-byte aligned
    float scale;
};
hipError_t launch_route(const RouteArgs& a, bool f32, bool sigmoid, hipStream_t stream);
hipError_t launch_route_grad(const RouteArgs& a, bool f32, bool sigmoid, hipStream_t stream);

// ---------------------------------------------------------------- tokens by expert (order_kernels.hip)
constexpr uint32_t kSortMaxAlign = 1024;
constexpr uint32_t kSortChunkPairs = 1024;   // pairs that one workgroup of the chunked sort ranks
constexpr uint32_t kSortOneMaxPairs = 4096;  // up to here one workgroup sorts them all

struct SortArgs {
    const int32_t* ids;          // [P]
    int32_t* offsets;            // [E + 1]
    int32_t* counts;             // [E]
    int32_t* pair_row;           // [P]
    int32_t* row_pair;           // [cap]
    int32_t* chunk_count;        // [n_chunks][E], chunked sort only
    uint32_t P, E, align, cap;
    uint32_t n_chunks;           // 0: one workgroup sorts all pairs
};
// chunks of the chunked sort, which also takes over where one workgroup's counts would not fit its LDS
inline uint32_t sort_chunks(uint64_t P, uint32_t E) {
    return P <= kSortOneMaxPairs && E <= 2048 ? 0 : uint32_t((P + kSortChunkPairs - 1) / kSortChunkPairs);
}
hipError_t launch_sort(const SortArgs& a, hipStream_t stream);

struct RowsArgs {
    const void* x;               // dispatch: [T][H]; combine_grad: d_out [T][H]
    const void* rows_in;         // combine, combine_grad: [cap][H]
    void* rows_out;              // dispatch, combine_grad: [cap][H]
    void* out;                   // combine: [T][H]
    const int32_t* pair_row;     // [T][K]
    const int32_t* row_pair;     // [cap]
    const float* gates;          // [T][K], combine: may be nullptr (1)
    float* d_gates;              // combine_grad: [T][K]
    uint64_t x_stride, in_stride, out_stride;   // in elements: x / d_out; rows_in; rows_out or out
    uint32_t T, K, H, cap;
    uint32_t accumulate;
    uint32_t vec;                // every row is 16-byte aligned and a multiple of 16 bytes long (dispatch) or of 8 elements
};
hipError_t launch_dispatch(const RowsArgs& a, uint32_t elem_bytes, hipStream_t stream);
hipError_t launch_combine(const RowsArgs& a, bool rows_f32, bool out_f32, hipStream_t stream);
hipError_t launch_combine_grad(const RowsArgs& a, bool rows_f32, bool out_f32, hipStream_t stream);

// ---------------------------------------------------------------- norms around a block (norm_kernels.hip)
struct NormArgs {
    const void* y;               // [T][H] or nullptr
    const void* residual;        // forward: the stream before the sum; gradient: after it
    const void* w_pre;           // [H]
    const void* w_post;          // [H] or nullptr
    const float* gate;           // [T] or [H] or nullptr
    void* residual_out;          // forward, nullptr: not written
    uint16_t* normed;            // forward, BF16
    uint64_t y_stride, residual_stride, residual_out_stride, normed_stride;
    uint32_t T, H;
    uint32_t gate_token, gate_channel, gate_sigmoid, zero_centred, weight_f32;
    float eps, scale;
    // gradient
    const void* d_residual_out;  // or nullptr (0)
    const uint16_t* d_normed;
    void* d_residual;
    void* d_y;
    float* d_gate;
    float* d_w_pre;
    float* d_w_post;
    float* partials;             // [sums][n_partials][H]: for w_pre, then for w_post and a channel's gate
    uint64_t d_residual_out_stride, d_normed_stride, d_residual_stride, d_y_stride;
    uint32_t n_partials;
};
hipError_t launch_block_norm(const NormArgs& a, bool y_f32, bool residual_f32, bool vec, hipStream_t stream);
hipError_t launch_block_norm_grad(const NormArgs& a, bool y_f32, bool residual_f32, bool vec, hipStream_t stream);
uint32_t norm_grad_partials(uint32_t T, uint32_t H);     // sums over the tokens that the gradient's workgroups leave, of each kind

}  // namespace fluxmoe
