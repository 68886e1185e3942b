// C entry points of the operators around the routed experts: argument checks, then one launcher call.  No context: they take
// device pointers and sizes, keep nothing between calls and allocate nothing.
#include "block_ops.h"
#include "fluxmoe_internal.h"

using namespace fluxmoe;

namespace {

constexpr uint32_t kMaxTokens = 1u << 20;    // keeps every launch below 2^32 threads
constexpr uint32_t kMaxHidden = 1u << 20;

uint32_t elem_bytes(uint32_t type) { return type == FLUXMOE_F32 ? 4 : 2; }
bool known(uint32_t type) { return type == FLUXMOE_BF16 || type == FLUXMOE_F32; }
bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
// Rows of `bytes` per element, `stride` elements apart, each at a 16-byte address; absent tensors do not stand in the way.
bool rows_aligned(const void* p, uint64_t stride, uint32_t bytes) { return !p || (aligned(p, 16) && stride * bytes % 16 == 0); }

int check_tokens(uint32_t T) {
    return T <= kMaxTokens ? FLUXMOE_OK : set_error(FLUXMOE_EINVAL, "T must be at most %u (got %u)", kMaxTokens, T);
}
int check_hidden(uint32_t H) {
    return H >= 1 && H <= kMaxHidden ? FLUXMOE_OK : set_error(FLUXMOE_EINVAL, "hidden must be in 1..%u (got %u)", kMaxHidden, H);
}
int check_stride(const char* name, uint64_t stride, uint32_t width) {
    if (stride >= width && stride < (1ull << 40)) return FLUXMOE_OK;
    return set_error(FLUXMOE_EINVAL, "%s (%llu) must be at least the row's %u elements", name, (unsigned long long)stride, width);
}
int check_experts(uint32_t E, uint32_t K) {
    if (E == 0 || E > kRouteMaxExperts) return set_error(FLUXMOE_EINVAL, "E must be in 1..%u (got %u)", kRouteMaxExperts, E);
    if (K == 0 || K > E || K > kRouteMaxTopK)
        return set_error(FLUXMOE_EINVAL, "K must be in 1..min(E, %u) (got %u of %u)", kRouteMaxTopK, K, E);
    return FLUXMOE_OK;
}

int check_route(uint32_t type, uint32_t T, uint32_t E, uint32_t K, uint32_t flags) {
    if (int rc = check_tokens(T)) return rc;
    if (int rc = check_experts(E, K)) return rc;
    if (!known(type)) return set_error(FLUXMOE_EINVAL, "unknown element type %u", type);
    if (flags & ~(FLUXMOE_ROUTE_SIGMOID | FLUXMOE_ROUTE_RENORMALIZE)) return set_error(FLUXMOE_EINVAL, "unknown flags 0x%x", flags);
    return FLUXMOE_OK;
}

// What dispatch, combine and its gradient have in common.
int check_rows(uint32_t T, uint32_t K, uint32_t H, uint64_t rows_cap) {
    if (int rc = check_tokens(T)) return rc;
    if (int rc = check_hidden(H)) return rc;
    if (K == 0 || K > kRouteMaxTopK) return set_error(FLUXMOE_EINVAL, "K must be in 1..%u (got %u)", kRouteMaxTopK, K);
    if (rows_cap >= (1ull << 31)) return set_error(FLUXMOE_EINVAL, "rows_cap too large");
    return FLUXMOE_OK;
}

// With T = 0 the addresses of what has a row for each token (y, a token's gate) say nothing: an empty tensor's is NULL.
int norm_args(const fluxmoe_norm_desc* d, uint32_t T, const void* y, const void* residual, const float* gate, const void* w_post,
              const void* w_pre, NormArgs& a) {
    if (!d) return set_error(FLUXMOE_EINVAL, "desc is NULL");
    if (int rc = check_tokens(T)) return rc;
    if (int rc = check_hidden(d->hidden)) return rc;
    if (!known(d->y_type) || !known(d->residual_type) || !known(d->weight_type)) return set_error(FLUXMOE_EINVAL, "unknown element type");
    const uint32_t all = FLUXMOE_NORM_GATE_TOKEN | FLUXMOE_NORM_GATE_CHANNEL | FLUXMOE_NORM_GATE_SIGMOID | FLUXMOE_NORM_ZERO_CENTRED;
    if (d->reserved) return set_error(FLUXMOE_EINVAL, "reserved must be 0");
    if (d->flags & ~all) return set_error(FLUXMOE_EINVAL, "unknown flags 0x%x", d->flags);
    const uint32_t kind = d->flags & (FLUXMOE_NORM_GATE_TOKEN | FLUXMOE_NORM_GATE_CHANNEL);
    if (kind == (FLUXMOE_NORM_GATE_TOKEN | FLUXMOE_NORM_GATE_CHANNEL)) return set_error(FLUXMOE_EINVAL, "a gate is either the token's or the channels'");
    const bool told = T || kind != FLUXMOE_NORM_GATE_TOKEN;
    if (told && (kind != 0) != (gate != nullptr)) return set_error(FLUXMOE_EINVAL, "the flags and the gate pointer disagree on whether there is a gate");
    if ((d->flags & FLUXMOE_NORM_GATE_SIGMOID) && !kind) return set_error(FLUXMOE_EINVAL, "FLUXMOE_NORM_GATE_SIGMOID without a gate");
    if (T && !y && (gate || w_post)) return set_error(FLUXMOE_EINVAL, "a gate or w_post without y");
    if (!(d->eps >= 0.0f)) return set_error(FLUXMOE_EINVAL, "eps must not be negative");
    a = NormArgs{};
    a.T = T;
    a.H = d->hidden;
    a.y = y;
    a.residual = residual;
    a.gate = gate;
    a.w_post = w_post;
    a.w_pre = w_pre;
    a.gate_token = kind == FLUXMOE_NORM_GATE_TOKEN;
    a.gate_channel = kind == FLUXMOE_NORM_GATE_CHANNEL;
    a.gate_sigmoid = (d->flags & FLUXMOE_NORM_GATE_SIGMOID) != 0;
    a.zero_centred = (d->flags & FLUXMOE_NORM_ZERO_CENTRED) != 0;
    a.weight_f32 = d->weight_type == FLUXMOE_F32;
    a.eps = d->eps;
    a.scale = d->scale;
    auto stride = [&](uint64_t s) { return s ? s : uint64_t(d->hidden); };
    a.y_stride = stride(d->y_stride);
    a.residual_stride = stride(d->residual_stride);
    a.residual_out_stride = stride(d->residual_out_stride);
    a.normed_stride = stride(d->normed_stride);
    a.d_y_stride = stride(d->d_y_stride);
    a.d_residual_stride = stride(d->d_residual_stride);
    a.d_residual_out_stride = stride(d->d_residual_out_stride);
    a.d_normed_stride = stride(d->d_normed_stride);
    for (uint64_t s : {a.y_stride, a.residual_stride, a.residual_out_stride, a.normed_stride, a.d_y_stride, a.d_residual_stride,
                       a.d_residual_out_stride, a.d_normed_stride})
        if (int rc = check_stride("a stride", s, d->hidden)) return rc;
    const uint32_t yb = elem_bytes(d->y_type), rb = elem_bytes(d->residual_type), wb = elem_bytes(d->weight_type);
    if (!aligned(y, yb) || !aligned(residual, rb) || !aligned(w_pre, wb) || !aligned(w_post, wb) || !aligned(gate, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    return FLUXMOE_OK;
}

}  // namespace

extern "C" {

int fluxmoe_route(const void* logits, uint32_t type, uint32_t T, uint32_t E, uint64_t row_stride, const float* bias, uint32_t K, float scale,
                  uint32_t flags, int32_t* topk_ids, float* topk_w, void* stream) {
    if (int rc = check_route(type, T, E, K, flags)) return rc;
    if (bias && !(flags & FLUXMOE_ROUTE_SIGMOID)) return set_error(FLUXMOE_EINVAL, "bias goes with FLUXMOE_ROUTE_SIGMOID");
    if (T == 0) return FLUXMOE_OK;
    if (!logits || !topk_ids || !topk_w) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (int rc = check_stride("row_stride", row_stride, E)) return rc;
    const uint32_t bytes = elem_bytes(type);
    if (!aligned(logits, bytes) || !aligned(bias, 4) || !aligned(topk_ids, 4) || !aligned(topk_w, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    RouteArgs a{};
    a.logits = logits;
    a.bias = bias;
    a.ids = topk_ids;
    a.gates = topk_w;
    a.row_stride = row_stride;
    a.T = T;
    a.E = E;
    a.K = K;
    a.scale = scale;
    a.renormalize = (flags & FLUXMOE_ROUTE_RENORMALIZE) != 0;
    a.vec = rows_aligned(logits, row_stride, bytes);
    HIPCHECK(launch_route(a, type == FLUXMOE_F32, (flags & FLUXMOE_ROUTE_SIGMOID) != 0, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_route_grad(const void* logits, uint32_t type, uint32_t T, uint32_t E, uint64_t row_stride, const int32_t* topk_ids, uint32_t K,
                       float scale, uint32_t flags, const float* d_topk_w, void* d_logits, uint64_t d_row_stride, void* stream) {
    if (int rc = check_route(type, T, E, K, flags)) return rc;
    if (T == 0) return FLUXMOE_OK;
    if (!logits || !topk_ids || !d_topk_w || !d_logits) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (int rc = check_stride("row_stride", row_stride, E)) return rc;
    if (int rc = check_stride("d_row_stride", d_row_stride, E)) return rc;
    const uint32_t bytes = elem_bytes(type);
    if (!aligned(logits, bytes) || !aligned(d_logits, bytes) || !aligned(topk_ids, 4) || !aligned(d_topk_w, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    RouteArgs a{};
    a.logits = logits;
    a.ids = const_cast<int32_t*>(topk_ids);
    a.d_gates = d_topk_w;
    a.d_logits = d_logits;
    a.row_stride = row_stride;
    a.d_stride = d_row_stride;
    a.T = T;
    a.E = E;
    a.K = K;
    a.scale = scale;
    a.renormalize = (flags & FLUXMOE_ROUTE_RENORMALIZE) != 0;
    a.vec = rows_aligned(logits, row_stride, bytes);
    a.d_vec = rows_aligned(d_logits, d_row_stride, bytes);
    HIPCHECK(launch_route_grad(a, type == FLUXMOE_F32, (flags & FLUXMOE_ROUTE_SIGMOID) != 0, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

uint64_t fluxmoe_sorted_rows(uint32_t T, uint32_t K, uint32_t E, uint32_t align) {
    const uint64_t pairs = uint64_t(T) * K;
    return pairs + (align > 1 ? (pairs < E ? pairs : E) * (align - 1) : 0);
}

uint64_t fluxmoe_sort_workspace_bytes(uint32_t T, uint32_t K, uint32_t E) {
    return uint64_t(sort_chunks(uint64_t(T) * K, E)) * E * sizeof(int32_t);
}

int fluxmoe_sort_tokens(const int32_t* topk_ids, uint32_t T, uint32_t K, uint32_t E, uint32_t align, int32_t* offsets, int32_t* counts,
                        int32_t* pair_row, int32_t* row_pair, uint64_t rows_cap, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (int rc = check_tokens(T)) return rc;
    if (int rc = check_experts(E, 1)) return rc;
    if (K == 0 || K > kRouteMaxTopK) return set_error(FLUXMOE_EINVAL, "K must be in 1..%u (got %u)", kRouteMaxTopK, K);
    if (align == 0 || align > kSortMaxAlign) return set_error(FLUXMOE_EINVAL, "align must be in 1..%u (got %u)", kSortMaxAlign, align);
    if (!offsets || !counts || (T && (!topk_ids || !pair_row)) || (rows_cap && !row_pair)) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (!aligned(topk_ids, 4) || !aligned(offsets, 4) || !aligned(counts, 4) || !aligned(pair_row, 4) || !aligned(row_pair, 4) || !aligned(workspace, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    if (rows_cap >= (1ull << 31)) return set_error(FLUXMOE_EINVAL, "rows_cap too large");
    if (const uint64_t need = fluxmoe_sorted_rows(T, K, E, align); rows_cap < need)
        return set_error(FLUXMOE_ENOMEM, "row_pair holds %llu rows, T=%u K=%u E=%u align=%u can need %llu", (unsigned long long)rows_cap, T, K, E,
                         align, (unsigned long long)need);
    if (const uint64_t need = fluxmoe_sort_workspace_bytes(T, K, E); need && (!workspace || workspace_bytes < need))
        return set_error(FLUXMOE_ENOMEM, "the workspace holds %llu bytes, T=%u K=%u E=%u needs %llu",
                         (unsigned long long)(workspace ? workspace_bytes : 0), T, K, E, (unsigned long long)need);
    SortArgs a{};
    a.ids = topk_ids;
    a.offsets = offsets;
    a.counts = counts;
    a.pair_row = pair_row;
    a.row_pair = row_pair;
    a.chunk_count = static_cast<int32_t*>(workspace);
    a.P = T * K;
    a.E = E;
    a.align = align;
    a.cap = uint32_t(rows_cap);
    a.n_chunks = sort_chunks(a.P, E);
    HIPCHECK(launch_sort(a, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_dispatch(const void* x, uint32_t type, uint32_t T, uint32_t H, uint64_t x_stride, const int32_t* pair_row, uint32_t K,
                     const int32_t* row_pair, uint64_t rows_cap, void* rows, uint64_t rows_stride, void* stream) {
    if (int rc = check_rows(T, K, H, rows_cap)) return rc;
    if (!known(type)) return set_error(FLUXMOE_EINVAL, "unknown element type %u", type);
    if (T == 0 && rows_cap == 0) return FLUXMOE_OK;
    if ((T && (!x || !pair_row)) || (rows_cap && (!row_pair || !rows))) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (int rc = check_stride("x_stride", x_stride, H)) return rc;
    if (int rc = check_stride("rows_stride", rows_stride, H)) return rc;
    const uint32_t bytes = elem_bytes(type);
    if (!aligned(x, bytes) || !aligned(rows, bytes) || !aligned(pair_row, 4) || !aligned(row_pair, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    RowsArgs a{};
    a.x = x;
    a.rows_out = rows;
    a.pair_row = pair_row;
    a.row_pair = row_pair;
    a.x_stride = x_stride;
    a.out_stride = rows_stride;
    a.T = T;
    a.K = K;
    a.H = H;
    a.cap = uint32_t(rows_cap);
    a.vec = uint64_t(H) * bytes % 16 == 0 && rows_aligned(x, x_stride, bytes) && rows_aligned(rows, rows_stride, bytes);
    HIPCHECK(launch_dispatch(a, bytes, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_combine(const void* rows, uint32_t rows_type, uint64_t rows_cap, uint32_t H, uint64_t rows_stride, const int32_t* pair_row,
                    const float* topk_w, uint32_t T, uint32_t K, void* out, uint32_t out_type, uint64_t out_stride, uint32_t flags,
                    void* stream) {
    if (int rc = check_rows(T, K, H, rows_cap)) return rc;
    if (!known(rows_type) || !known(out_type)) return set_error(FLUXMOE_EINVAL, "unknown element type");
    if (flags & ~FLUXMOE_FFN_ACCUMULATE) return set_error(FLUXMOE_EINVAL, "only FLUXMOE_FFN_ACCUMULATE is accepted");
    if (T == 0) return FLUXMOE_OK;
    if ((rows_cap && !rows) || !pair_row || !out) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (int rc = check_stride("rows_stride", rows_stride, H)) return rc;
    if (int rc = check_stride("out_stride", out_stride, H)) return rc;
    const uint32_t rb = elem_bytes(rows_type), ob = elem_bytes(out_type);
    if (!aligned(rows, rb) || !aligned(out, ob) || !aligned(pair_row, 4) || !aligned(topk_w, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    RowsArgs a{};
    a.rows_in = rows;
    a.out = out;
    a.pair_row = pair_row;
    a.gates = topk_w;
    a.in_stride = rows_stride;
    a.out_stride = out_stride;
    a.T = T;
    a.K = K;
    a.H = H;
    a.cap = uint32_t(rows_cap);
    a.accumulate = (flags & FLUXMOE_FFN_ACCUMULATE) != 0;
    a.vec = H % 8 == 0 && rows_aligned(rows, rows_stride, rb) && rows_aligned(out, out_stride, ob);
    HIPCHECK(launch_combine(a, rows_type == FLUXMOE_F32, out_type == FLUXMOE_F32, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_combine_grad(const void* d_out, uint32_t out_type, uint64_t d_out_stride, const void* rows, uint32_t rows_type, uint64_t rows_cap,
                         uint32_t H, uint64_t rows_stride, const int32_t* pair_row, const int32_t* row_pair, const float* topk_w, uint32_t T,
                         uint32_t K, void* d_rows, uint64_t d_rows_stride, float* d_topk_w, void* stream) {
    if (int rc = check_rows(T, K, H, rows_cap)) return rc;
    if (!known(rows_type) || !known(out_type)) return set_error(FLUXMOE_EINVAL, "unknown element type");
    if (T == 0 && rows_cap == 0) return FLUXMOE_OK;
    if ((T && (!d_out || !pair_row || !topk_w || !d_topk_w)) || (rows_cap && (!rows || !row_pair || !d_rows)))
        return set_error(FLUXMOE_EINVAL, "NULL argument");
    if (int rc = check_stride("d_out_stride", d_out_stride, H)) return rc;
    if (int rc = check_stride("rows_stride", rows_stride, H)) return rc;
    if (int rc = check_stride("d_rows_stride", d_rows_stride, H)) return rc;
    const uint32_t rb = elem_bytes(rows_type), ob = elem_bytes(out_type);
    if (!aligned(d_out, ob) || !aligned(rows, rb) || !aligned(d_rows, rb) || !aligned(pair_row, 4) || !aligned(row_pair, 4) || !aligned(topk_w, 4) ||
        !aligned(d_topk_w, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    RowsArgs a{};
    a.x = d_out;
    a.rows_in = rows;
    a.rows_out = d_rows;
    a.pair_row = pair_row;
    a.row_pair = row_pair;
    a.gates = topk_w;
    a.d_gates = d_topk_w;
    a.x_stride = d_out_stride;
    a.in_stride = rows_stride;
    a.out_stride = d_rows_stride;
    a.T = T;
    a.K = K;
    a.H = H;
    a.cap = uint32_t(rows_cap);
    a.vec = H % 8 == 0 && rows_aligned(d_out, d_out_stride, ob) && rows_aligned(rows, rows_stride, rb) && rows_aligned(d_rows, d_rows_stride, rb);
    HIPCHECK(launch_combine_grad(a, rows_type == FLUXMOE_F32, out_type == FLUXMOE_F32, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

int fluxmoe_block_norm(const fluxmoe_norm_desc* d, uint32_t T, const void* y, const void* residual, const float* gate, const void* w_post,
                       const void* w_pre, void* residual_out, uint16_t* normed, void* stream) {
    NormArgs a;
    if (int rc = norm_args(d, T, y, residual, gate, w_post, w_pre, a)) return rc;
    if (T == 0) return FLUXMOE_OK;
    if (!residual || !w_pre || !normed) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if ((residual_out != nullptr) != (y != nullptr)) return set_error(FLUXMOE_EINVAL, "residual_out is written where there is a y to add, and only there");
    if (residual_out == residual && a.residual_out_stride != a.residual_stride)
        return set_error(FLUXMOE_EINVAL, "residual_out in the residual's place must have its stride");
    if (!aligned(residual_out, elem_bytes(d->residual_type)) || !aligned(normed, 2)) return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    a.residual_out = residual_out;
    a.normed = normed;
    const uint32_t yb = elem_bytes(d->y_type), rb = elem_bytes(d->residual_type);
    const bool vec = a.H % 8 == 0 && rows_aligned(y, a.y_stride, yb) && rows_aligned(residual, a.residual_stride, rb) &&
                     rows_aligned(residual_out, a.residual_out_stride, rb) && rows_aligned(normed, a.normed_stride, 2) && aligned(w_pre, 16) &&
                     aligned(w_post, 16) && (!a.gate_channel || aligned(gate, 16));
    HIPCHECK(launch_block_norm(a, d->y_type == FLUXMOE_F32, d->residual_type == FLUXMOE_F32, vec, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

uint64_t fluxmoe_block_norm_grad_workspace_bytes(uint32_t T, uint32_t H) {
    return uint64_t(norm_grad_partials(T, H)) * H * 2 * sizeof(float);
}

int fluxmoe_block_norm_grad(const fluxmoe_norm_desc* d, uint32_t T, const void* y, const void* residual_out, const float* gate,
                            const void* w_post, const void* w_pre, const void* d_residual_out, const uint16_t* d_normed, void* d_residual,
                            void* d_y, float* d_gate, float* d_w_post, float* d_w_pre, void* workspace, uint64_t workspace_bytes,
                            void* stream) {
    NormArgs a;
    if (int rc = norm_args(d, T, y, residual_out, gate, w_post, w_pre, a)) return rc;
    if ((d_w_post != nullptr) != (w_post != nullptr) || ((T || a.gate_channel) && (d_gate != nullptr) != (gate != nullptr)) ||
        (T && (d_y != nullptr) != (y != nullptr)))
        return set_error(FLUXMOE_EINVAL, "d_y, d_gate and d_w_post go with y, gate and w_post");
    if (!d_w_pre || !w_pre || (T && (!residual_out || !d_normed || !d_residual))) return set_error(FLUXMOE_EINVAL, "NULL argument");
    if ((T && d_residual == d_residual_out && a.d_residual_stride != a.d_residual_out_stride) || (d_y && d_y == y && a.d_y_stride != a.y_stride))
        return set_error(FLUXMOE_EINVAL, "a gradient in its input's place must have its stride");
    const uint32_t yb = elem_bytes(d->y_type), rb = elem_bytes(d->residual_type);
    if (!aligned(d_residual_out, rb) || !aligned(d_normed, 2) || !aligned(d_residual, rb) || !aligned(d_y, yb) || !aligned(d_gate, 4) ||
        !aligned(d_w_post, 4) || !aligned(d_w_pre, 4))
        return set_error(FLUXMOE_EINVAL, "a pointer is not aligned to its elements");
    if (const uint64_t need = fluxmoe_block_norm_grad_workspace_bytes(T, d->hidden); need && (!workspace || workspace_bytes < need))
        return set_error(FLUXMOE_ENOMEM, "the workspace holds %llu bytes, T=%u hidden=%u needs %llu",
                         (unsigned long long)(workspace ? workspace_bytes : 0), T, d->hidden, (unsigned long long)need);
    if (!aligned(workspace, 16)) return set_error(FLUXMOE_EINVAL, "workspace must be 16-byte aligned");
    a.residual_stride = a.residual_out_stride;
    a.d_residual_out = d_residual_out;
    a.d_normed = d_normed;
    a.d_residual = d_residual;
    a.d_y = d_y;
    a.d_gate = d_gate;
    a.d_w_pre = d_w_pre;
    a.d_w_post = d_w_post;
    a.partials = static_cast<float*>(workspace);
    const bool vec = a.H % 8 == 0 && rows_aligned(y, a.y_stride, yb) && rows_aligned(residual_out, a.residual_stride, rb) &&
                     rows_aligned(d_residual_out, a.d_residual_out_stride, rb) && rows_aligned(d_normed, a.d_normed_stride, 2) &&
                     rows_aligned(d_residual, a.d_residual_stride, rb) && rows_aligned(d_y, a.d_y_stride, yb) && aligned(w_pre, 16) &&
                     aligned(w_post, 16) && (!a.gate_channel || aligned(gate, 16));
    HIPCHECK(launch_block_norm_grad(a, d->y_type == FLUXMOE_F32, d->residual_type == FLUXMOE_F32, vec, static_cast<hipStream_t>(stream)));
    return FLUXMOE_OK;
}

}  // extern "C"
