// C entry points of the experts in 4-bit floating point (MXFP4): argument checks, then one launcher call.  No context: they take
// device pointers and sizes, keep nothing between calls and allocate nothing.
#include "api_checks.h"
#include "mx_ops.h"

using namespace fluxmoe;

namespace {

constexpr uint32_t kMaxColumns = 1u << 20;
constexpr uint64_t kMaxRows = 1ull << 32;    // of a matrix whose rows go to 4 bits and back: all experts' outputs
constexpr uint64_t kMaxCap = 1ull << 31;     // of a matrix of tokens' rows

int check_columns(const char* name, uint32_t columns, uint32_t multiple) {
    if (columns >= 1 && columns <= kMaxColumns && columns % multiple == 0) return FLUXMOE_OK;
    return set_error(FLUXMOE_EINVAL, "%s must be a multiple of %u in 1..%u (got %u)", name, multiple, kMaxColumns, columns);
}

int mx_rows_args(const void* x, uint32_t type, uint64_t rows, uint32_t columns, uint64_t x_stride, const uint8_t* codes, uint64_t codes_stride,
                 const uint8_t* scales, uint64_t scales_stride, MxRowsArgs& a) {
    if (!known(type)) return set_error(FLUXMOE_EINVAL, "unknown element type %u", type);
    if (rows > kMaxRows) return set_error(FLUXMOE_EINVAL, "rows must be at most 2^32");
    if (int rc = check_columns("columns", columns, kMxBlock)) return rc;
    if (int rc = check_stride("x_stride", x_stride, columns)) return rc;
    if (int rc = check_stride("codes_stride", codes_stride, columns / 2)) return rc;
    if (int rc = check_stride("scales_stride", scales_stride, columns / kMxBlock)) return rc;
    if (rows == 0) return FLUXMOE_OK;
    if (!x || !codes || !scales) return set_error(FLUXMOE_EINVAL, "NULL argument");
    const uint32_t bytes = elem_bytes(type);
    if (!aligned(x, bytes)) return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    a.codes = const_cast<uint8_t*>(codes);
    a.scales = const_cast<uint8_t*>(scales);
    a.x_stride = x_stride;
    a.codes_stride = codes_stride;
    a.scales_stride = scales_stride;
    a.rows = rows;
    a.cols = columns;
    a.vec = rows_aligned(x, x_stride, bytes) && aligned(codes, 4) && codes_stride % 4 == 0;
    return FLUXMOE_OK;
}

int swiglu_args(const void* gate_up, uint32_t type, uint64_t rows, uint32_t F, uint64_t stride, const void* h, uint32_t h_type, uint64_t h_stride) {
    if (!known(type) || !known(h_type)) return set_error(FLUXMOE_EINVAL, "unknown element type");
    if (rows >= kMaxCap) return set_error(FLUXMOE_EINVAL, "rows must be below 2^31");
    if (int rc = check_columns("ffn", F, 1)) return rc;
    if (int rc = check_stride("gate_up's stride", stride, 2 * F)) return rc;
    if (int rc = check_stride("h's stride", h_stride, F)) return rc;
    if (rows == 0) return FLUXMOE_OK;
    if (!gate_up || !h) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (!aligned(gate_up, elem_bytes(type)) || !aligned(h, elem_bytes(h_type)))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    return FLUXMOE_OK;
}
// both halves of every row at 16-byte addresses
bool halves_aligned(const void* p, uint64_t stride, uint32_t F, uint32_t type) {
    return rows_aligned(p, stride, elem_bytes(type)) && uint64_t(F) * elem_bytes(type) % 16 == 0;
}

// What the product and its gradient have in common; grad: `rows` is d_rows and `out` d_out.
int product_args(const fluxmoe_mx_product_desc* d, const void* rows, const uint8_t* row_scales, const int32_t* offsets, const int32_t* counts,
                 const uint8_t* w_codes, const uint8_t* w_scales, const void* out, bool grad, MxProductArgs& a) {
    if (!d) return set_error(FLUXMOE_EINVAL, "desc is NULL");
    if (d->E == 0 || d->E > kMxMaxExperts) return set_error(FLUXMOE_EINVAL, "E must be in 1..%u (got %u)", kMxMaxExperts, d->E);
    if (int rc = check_columns("K", d->K, kMxBlock)) return rc;
    if (int rc = check_columns("N", d->N, 1)) return rc;
    if (d->reserved) return set_error(FLUXMOE_EINVAL, "reserved must be 0");
    if (d->rows_cap >= kMaxCap) return set_error(FLUXMOE_EINVAL, "rows_cap must be below 2^31");
    const bool mx = d->rows_type == FLUXMOE_MXFP4;
    if (grad) {
        if (!known(d->rows_type)) return set_error(FLUXMOE_EINVAL, "d_rows is BF16 or FP32");
        if (d->out_type != FLUXMOE_BF16) return set_error(FLUXMOE_EINVAL, "d_out is BF16");
    } else {
        if (!mx && d->rows_type != FLUXMOE_BF16) return set_error(FLUXMOE_EINVAL, "rows are BF16 or MXFP4");
        if (!known(d->out_type)) return set_error(FLUXMOE_EINVAL, "out is BF16 or FP32");
    }
    const uint32_t rb = mx ? 1 : elem_bytes(d->rows_type), ob = elem_bytes(d->out_type);
    const uint32_t row_width = mx ? d->K / 2 : d->K;
    const uint64_t rs = d->rows_stride ? d->rows_stride : row_width, os = d->out_stride ? d->out_stride : d->N;
    const uint64_t ss = d->row_scales_stride ? d->row_scales_stride : d->K / kMxBlock;
    if (int rc = check_stride("rows_stride", rs, row_width)) return rc;
    if (int rc = check_stride("out_stride", os, d->N)) return rc;
    if (int rc = check_stride("row_scales_stride", ss, d->K / kMxBlock)) return rc;
    if (!mx && row_scales) return set_error(FLUXMOE_EINVAL, "row_scales go with rows of MXFP4");
    if (d->rows_cap == 0) return FLUXMOE_OK;
    if (!rows || !out || !offsets || !counts || !w_codes || !w_scales || (mx && !row_scales)) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (!aligned(rows, rb) || !aligned(out, ob) || !aligned(offsets, 4) || !aligned(counts, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    if (!aligned(w_codes, 16)) return set_error(FLUXMOE_EINVAL, "w_codes must be 16-byte aligned");
    a.rows = grad ? out : rows;
    a.row_scales = row_scales;
    a.offsets = offsets;
    a.counts = counts;
    a.w = w_codes;
    a.ws = w_scales;
    a.out = const_cast<void*>(grad ? rows : out);
    a.row_stride = grad ? os * ob : rs * rb;
    a.row_scales_stride = ss;
    a.out_stride = grad ? rs * rb : os * ob;
    a.E = d->E;
    a.N = d->N;
    a.K = d->K;
    a.cap = uint32_t(d->rows_cap);
    a.rows_vec = rows_aligned(a.rows, a.row_stride, 1);
    a.out_vec = rows_aligned(a.out, a.out_stride, 1);
    return FLUXMOE_OK;
}

}  // namespace

extern "C" {

int fluxmoe_mx_quantize(const void* x, uint32_t type, uint64_t rows, uint32_t columns, uint64_t x_stride, uint8_t* codes, uint64_t codes_stride,
                        uint8_t* scales, uint64_t scales_stride, void* stream) {
    MxRowsArgs a{};
    if (int rc = mx_rows_args(x, type, rows, columns, x_stride, codes, codes_stride, scales, scales_stride, a)) return rc;
    if (rows == 0) return FLUXMOE_OK;
    a.x = x;
    HIPCHECK(launch_mx_quantize(a, type == FLUXMOE_F32, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_mx_dequantize(const uint8_t* codes, uint64_t codes_stride, const uint8_t* scales, uint64_t scales_stride, uint64_t rows,
                          uint32_t columns, void* out, uint32_t type, uint64_t out_stride, void* stream) {
    MxRowsArgs a{};
    if (int rc = mx_rows_args(out, type, rows, columns, out_stride, codes, codes_stride, scales, scales_stride, a)) return rc;
    if (rows == 0) return FLUXMOE_OK;
    a.out = out;
    HIPCHECK(launch_mx_dequantize(a, type == FLUXMOE_F32, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_mx_product(const fluxmoe_mx_product_desc* desc, const void* rows, const uint8_t* row_scales, const int32_t* offsets,
                       const int32_t* counts, const uint8_t* w_codes, const uint8_t* w_scales, void* out, void* stream) {
    MxProductArgs a{};
    if (int rc = product_args(desc, rows, row_scales, offsets, counts, w_codes, w_scales, out, false, a)) return rc;
    if (a.cap == 0) return FLUXMOE_OK;
    HIPCHECK(launch_mx_product(a, desc->rows_type == FLUXMOE_MXFP4, desc->out_type == FLUXMOE_F32, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_mx_product_grad(const fluxmoe_mx_product_desc* desc, const uint16_t* d_out, const int32_t* offsets, const int32_t* counts,
                            const uint8_t* w_codes, const uint8_t* w_scales, void* d_rows, void* stream) {
    MxProductArgs a{};
    if (int rc = product_args(desc, d_rows, nullptr, offsets, counts, w_codes, w_scales, d_out, true, a)) return rc;
    if (a.cap == 0) return FLUXMOE_OK;
    HIPCHECK(launch_mx_product_grad(a, desc->rows_type == FLUXMOE_F32, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_swiglu(const void* gate_up, uint32_t type, uint64_t rows, uint32_t ffn, uint64_t gate_up_stride, void* h, uint32_t h_type,
                   uint64_t h_stride, void* stream) {
    if (int rc = swiglu_args(gate_up, type, rows, ffn, gate_up_stride, h, h_type, h_stride)) return rc;
    if (rows == 0) return FLUXMOE_OK;
    SwigluArgs a{};
    a.gate_up = gate_up;
    a.out = h;
    a.in_stride = gate_up_stride;
    a.out_stride = h_stride;
    a.rows = rows;
    a.F = ffn;
    a.vec = halves_aligned(gate_up, gate_up_stride, ffn, type) && halves_aligned(h, h_stride, ffn, h_type);
    HIPCHECK(launch_swiglu(a, type == FLUXMOE_F32, h_type == FLUXMOE_F32, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_swiglu_grad(const void* gate_up, uint32_t type, uint64_t rows, uint32_t ffn, uint64_t gate_up_stride, const void* d_h,
                        uint32_t h_type, uint64_t d_h_stride, void* d_gate_up, uint64_t d_gate_up_stride, void* stream) {
    if (int rc = swiglu_args(gate_up, type, rows, ffn, gate_up_stride, d_h, h_type, d_h_stride)) return rc;
    if (int rc = check_stride("d_gate_up's stride", d_gate_up_stride, 2 * ffn)) return rc;
    if (rows == 0) return FLUXMOE_OK;
    if (!d_gate_up) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (!aligned(d_gate_up, elem_bytes(type))) return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    SwigluArgs a{};
    a.gate_up = gate_up;
    a.d_h = d_h;
    a.out = d_gate_up;
    a.in_stride = gate_up_stride;
    a.d_stride = d_h_stride;
    a.out_stride = d_gate_up_stride;
    a.rows = rows;
    a.F = ffn;
    a.vec = halves_aligned(gate_up, gate_up_stride, ffn, type) && halves_aligned(d_h, d_h_stride, ffn, h_type) &&
            halves_aligned(d_gate_up, d_gate_up_stride, ffn, type);
    HIPCHECK(launch_swiglu_grad(a, type == FLUXMOE_F32, h_type == FLUXMOE_F32, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

}  // extern "C"
