// Arguments and launchers of the experts in 4-bit floating point (MXFP4): rows to 4 bits and back, products, SwiGLU.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "mx_plan.h"

namespace fluxmoe {

constexpr uint32_t kMxBlock = 32;            // columns that share a scale
constexpr uint32_t kMxMaxExperts = 4096;     // their counts are added up by one workgroup's threads

// ---------------------------------------------------------------- rows (mx_rows.hip)
struct MxRowsArgs {
    const void* x;               // quantize: [rows][cols]
    uint8_t* codes;              // [rows][cols / 2]; dequantize reads it
    uint8_t* scales;             // [rows][cols / 32]
    void* out;                   // dequantize: [rows][cols]
    uint64_t x_stride, codes_stride, scales_stride;  // x / out in elements, the others in bytes
    uint64_t rows, cols;
    uint32_t vec;                // x / out rows are 16-byte aligned, the codes' 4-byte
};
hipError_t launch_mx_quantize(const MxRowsArgs& a, bool f32, hipStream_t stream);
hipError_t launch_mx_dequantize(const MxRowsArgs& a, bool f32, hipStream_t stream);

struct SwigluArgs {
    const void* gate_up;         // [rows][2 F]: gates, then ups
    const void* d_h;             // gradient only: [rows][F]
    void* out;                   // [rows][F]; gradient: [rows][2 F]
    uint64_t in_stride, d_stride, out_stride;
    uint64_t rows;
    uint32_t F;
    uint32_t vec;                // every half row is 16-byte aligned
};
// in_f32: type of gate_up (and its gradient), h_f32: of h (and its gradient)
hipError_t launch_swiglu(const SwigluArgs& a, bool in_f32, bool h_f32, hipStream_t stream);
hipError_t launch_swiglu_grad(const SwigluArgs& a, bool in_f32, bool h_f32, hipStream_t stream);

// ---------------------------------------------------------------- products (mx_product.hip)
struct MxProductArgs {
    const void* rows;            // BF16 [cap][K] or codes [cap][K / 2]; gradient: d_out BF16 [cap][N]
    const uint8_t* row_scales;   // [cap][K / 32], codes only
    const int32_t* offsets;      // [E + 1]
    const int32_t* counts;       // [E]
    const uint8_t* w;            // codes [E][N][K / 2]
    const uint8_t* ws;           // scales [E][N][K / 32]
    void* out;                   // [cap][N]; gradient: d_rows [cap][K]
    uint64_t row_stride, row_scales_stride, out_stride;   // all in bytes
    uint32_t E, N, K, cap;
    uint32_t rows_vec;           // rows at 16-byte addresses
    uint32_t out_vec;            // out's rows at 16-byte addresses
};
hipError_t launch_mx_product(const MxProductArgs& a, bool mx_rows, bool out_f32, hipStream_t stream);
// Wide tiles, as chosen (mx_tiles.hip)
hipError_t launch_mx_wide(const MxProductArgs& a, const MxChoice& choice, bool mx_rows, bool out_f32, hipStream_t stream);
hipError_t launch_mx_wide_grad(const MxProductArgs& a, const MxChoice& choice, bool out_f32, hipStream_t stream);
hipError_t launch_mx_product_grad(const MxProductArgs& a, bool out_f32, hipStream_t stream);

}  // namespace fluxmoe
