// C ABI of the operators beside the layer (see include/dsmoe.h): argument checks and launches.
#include "block_norm.h"
#include "clip_grads.h"
#include "gated.h"
#include "grouped.h"
#include "int4_matmul.h"
#include "int8_matmul.h"

using namespace dsmoe;

namespace dsmoe {
int& no_ctx_hip_error() {
  static thread_local int error = 0;
  return error;
}
}  // namespace dsmoe

namespace {

// At most a workgroup of 256 threads for a row or a tile, and a launch of 2^32 threads and more is silently cut short.  (The kernels for groups of few
// rows launch more for the same call: their own rule leaves such calls to the others.)
constexpr int64_t kMostWidth = 1 << 24, kMostRows = 1 << 23, kMostGroups = 1 << 16, kMostPieces = 1 << 23;

inline int status(hipError_t e) {
  if (e == hipSuccess) return DSMOE_OK;
  no_ctx_hip_error() = (int)e;
  return DSMOE_EHIP;
}
inline bool float_type(int32_t t) { return t == DSMOE_F32 || t == DSMOE_BF16 || t == DSMOE_F16; }
inline bool aligned_to(const void* p, int32_t type) { return ((uintptr_t)p & (elem_bytes(type) - 1)) == 0; }
inline bool width_ok(int64_t v) { return v >= 1 && v <= kMostWidth; }
// strides of inputs (their rows may overlap) and of outputs
inline bool in_stride(int64_t s) { return s >= 0 && s <= (int64_t)1 << 40; }
inline bool out_stride(int64_t s, int64_t width) { return s >= width && s <= (int64_t)1 << 40; }
inline int64_t tiles(int64_t v, int64_t t) { return (v + t - 1) / t; }
inline bool sizes_ok(int64_t rows, int64_t groups, int64_t k, int64_t n) {
  return rows >= 0 && rows <= kMostRows && groups >= 1 && groups <= kMostGroups && width_ok(k) && width_ok(n);
}

// as far as the workspaces' sizes go
GroupedArgs sizes_of(int rows, int groups, int K, int N) {
  static const int32_t some = 0;
  GroupedArgs g = {};
  g.off = &some;
  g.R = rows;
  g.G = groups;
  g.M = g.K = K;
  g.N = N;
  return g;
}

bool norm_args_ok(const dsmoe_block_norm_args* a) {
  return a && a->tokens >= 0 && a->tokens <= kMostRows && width_ok(a->d) && float_type(a->dtype) && a->gate_kind >= 0 && a->gate_kind <= 3 &&
         a->eps >= 0.f && in_stride(a->x_stride) && in_stride(a->branch_stride) && in_stride(a->gate_stride);
}
BlockNormArgs norm_args(const dsmoe_block_norm_args* a, const void* x, const void* branch, const void* branch_weight, const void* gate,
                        const void* weight) {
  BlockNormArgs n = {};
  n.x = x;
  n.branch = branch;
  n.gate = gate;
  n.branch_weight = branch_weight;
  n.weight = weight;
  n.x_row = a->x_stride;
  n.branch_row = a->branch_stride;
  n.gate_row = a->gate_stride;
  n.T = a->tokens;
  n.D = a->d;
  n.gate_kind = a->gate_kind;
  n.type = a->dtype;
  n.scale = a->scale;
  n.offset = a->weight_offset;
  n.eps = a->eps;
  return n;
}

bool grads_ok(const dsmoe_grad* grads, int32_t count, bool written, const float* norm, const void* workspace) {
  if (!grads || count < 1 || count > 1 << 20 || !norm || ((uintptr_t)norm & 3) != 0 || !workspace || ((uintptr_t)workspace & 255) != 0) return false;
  for (int32_t i = 0; i < count; ++i) {
    const dsmoe_grad& g = grads[i];
    if (!float_type(g.dtype) || g.rows < 0 || g.rows > INT32_MAX || g.width < 0 || g.width > (g.rows > 1 ? (int64_t)INT32_MAX : (int64_t)1 << 40)) return false;
    if (g.rows == 0 || g.width == 0) continue;
    if (g.rows > ((int64_t)1 << 44) / g.width || !g.grad || !aligned_to(g.grad, g.dtype) || (g.rows > 1 && !in_stride(g.grad_stride))) return false;
    if (written && (!g.out || !aligned_to(g.out, g.dtype) || (g.rows > 1 && !out_stride(g.out_stride, g.width)))) return false;
    if (written && g.out == g.grad && g.rows > 1 && g.out_stride != g.grad_stride) return false;
  }
  return true;
}

bool int4_args_ok(const dsmoe_int4_args* a) {
  return a && sizes_ok(a->rows, a->groups, a->k, a->n) && float_type(a->dtype) && (a->scale_dtype == a->dtype || a->scale_dtype == DSMOE_F32) &&
         a->block >= 32 && (a->block & (a->block - 1)) == 0 && row_tiles_bound(a->rows, a->groups, true, 128) * tiles(a->n, 128) <= kMostPieces;
}
Int4Args int4_args(const dsmoe_int4_args* a) {
  const int64_t e = elem_bytes(a->dtype);
  Int4Args g = {};
  g.x_row = a->x_stride * e;
  g.y_row = a->y_stride * e;
  g.w_row = a->w_row_stride;
  g.w_group = a->w_group_stride;
  g.s_row = a->scale_row_stride;
  g.s_group = a->scale_group_stride;
  g.z_row = a->zero_row_stride;
  g.z_group = a->zero_group_stride;
  g.R = a->rows;
  g.G = a->groups;
  g.N = a->n;
  g.K = a->k;
  g.type = a->dtype;
  g.scale_type = a->scale_dtype;
  g.shift = __builtin_ctz((unsigned)a->block);
  g.blocks = (int32_t)tiles(a->k, a->block);
  return g;
}

bool gated_args_ok(const dsmoe_gated_args* a) {
  return a && sizes_ok(a->rows, a->groups, a->k, a->n) && float_type(a->dtype) && (a->activation == DSMOE_SILU || a->activation == DSMOE_GELU_TANH) &&
         in_stride(a->x_stride) && in_stride(a->w_group_stride) && in_stride(a->w_row_stride) &&
         row_tiles_bound(a->rows, a->groups, true, 128) * tiles(a->n, 64) <= kMostPieces;
}
bool gated_backward_args_ok(const dsmoe_gated_args* a) {
  return gated_args_ok(a) && in_stride(a->h_stride) && row_tiles_bound(a->rows, a->groups, true, 128) * tiles(a->k, 128) <= kMostPieces &&
         tiles(a->k, 128) * tiles(a->n, 128) <= kMostPieces / a->groups;
}
GatedArgs gated_args(const dsmoe_gated_args* a, const void* x, const void* w1, const void* w3, const int32_t* offsets, void* workspace) {
  GatedArgs g = {};
  g.x = x;
  g.w1 = w1;
  g.w3 = w3;
  g.offsets = offsets;
  g.x_row = a->x_stride;
  g.w_row = a->w_row_stride;
  g.w_group = a->w_group_stride;
  g.h_row = a->h_stride;
  g.R = a->rows;
  g.G = a->groups;
  g.K = a->k;
  g.N = a->n;
  g.type = a->dtype;
  g.act = a->activation;
  g.workspace = (char*)workspace;
  return g;
}

}  // namespace

extern "C" {

int moe_grouped_matmul(const void* x, int64_t x_stride, const void* w, int64_t w_group_stride, int64_t w_row_stride,
                       const int32_t* offsets, int32_t rows, int32_t groups, int32_t k, int32_t n, int32_t transposed, int32_t dtype,
                       void* y, int64_t y_stride, void* workspace, void* stream) {
  if (!sizes_ok(rows, groups, k, n) || !float_type(dtype) || transposed < 0 || transposed > 1) return DSMOE_EINVAL;
  if (!in_stride(x_stride) || !in_stride(w_group_stride) || !in_stride(w_row_stride) || !out_stride(y_stride, transposed ? k : n)) return DSMOE_EINVAL;
  if (rows == 0) return DSMOE_OK;
  if (!x || !w || !offsets || !y || !aligned_to(x, dtype) || !aligned_to(w, dtype) || !aligned_to(y, dtype) || ((uintptr_t)workspace & 255) != 0) return DSMOE_EINVAL;
  if (row_tiles_bound(rows, groups, true, 128) * tiles(transposed ? k : n, 128) > kMostPieces) return DSMOE_EINVAL;
  const int64_t e = elem_bytes(dtype);
  GroupedArgs g = {};
  g.a = (const char*)x;
  g.b = (const char*)w;
  g.c = (char*)y;
  g.off = offsets;
  g.a_row = x_stride * e;
  g.b_row = w_row_stride * e;
  g.b_group = w_group_stride * e;
  g.c_row = y_stride * e;
  g.R = rows;
  g.G = groups;
  g.N = transposed ? k : n;
  g.K = transposed ? n : k;
  g.partial = (char*)workspace;
  return status(launch_grouped(g, dtype, transposed != 0, (hipStream_t)stream));
}

size_t dsmoe_grouped_workspace_bytes(int32_t rows, int32_t groups, int32_t k, int32_t n, int32_t transposed, int32_t dtype) {
  if (!sizes_ok(rows, groups, k, n) || !float_type(dtype) || transposed < 0 || transposed > 1) return 0;
  return grouped_workspace_bytes(sizes_of(rows, groups, transposed ? n : k, transposed ? k : n), dtype, transposed != 0);
}

size_t dsmoe_grouped_dw_workspace_bytes(int32_t rows, int32_t groups, int32_t k, int32_t n, int32_t dtype) {
  if (!sizes_ok(rows, groups, k, n) || !float_type(dtype) || tiles(k, 128) * tiles(n, 128) > kMostPieces / groups) return 0;
  return grouped_dw_workspace_bytes(sizes_of(rows, groups, k, n), dtype);
}

int moe_grouped_matmul_dw(const void* x, int64_t x_stride, const void* dy, int64_t dy_stride, const int32_t* offsets, int32_t rows,
                          int32_t groups, int32_t k, int32_t n, int32_t dtype, void* dw, int64_t dw_group_stride, int64_t dw_row_stride,
                          void* workspace, void* stream) {
  if (!sizes_ok(rows, groups, k, n) || !float_type(dtype) || ((uintptr_t)workspace & 255) != 0) return DSMOE_EINVAL;
  if (!in_stride(x_stride) || !in_stride(dy_stride) || !out_stride(dw_row_stride, n) || !out_stride(dw_group_stride, (k - 1) * dw_row_stride + n))
    return DSMOE_EINVAL;
  if (!offsets || !dw || !aligned_to(dw, dtype)) return DSMOE_EINVAL;
  if (rows > 0 && (!x || !dy || !aligned_to(x, dtype) || !aligned_to(dy, dtype))) return DSMOE_EINVAL;
  if (tiles(k, 128) * tiles(n, 128) > kMostPieces / groups) return DSMOE_EINVAL;
  const int64_t e = elem_bytes(dtype);
  GroupedArgs g = {};
  g.a = (const char*)x;
  g.b = (const char*)dy;
  g.c = (char*)dw;
  g.off = offsets;
  g.a_row = x_stride * e;
  g.b_row = dy_stride * e;
  g.c_row = dw_row_stride * e;
  g.c_group = dw_group_stride * e;
  g.R = rows;
  g.G = groups;
  g.M = k;
  g.N = n;
  g.partial = (char*)workspace;
  return status(launch_grouped_dw(g, dtype, (hipStream_t)stream));
}

size_t dsmoe_int8_workspace_bytes(int32_t rows, int32_t groups, int32_t k, int32_t n) {
  return !sizes_ok(rows, groups, k, n) || k > 1 << 17 ? 0 : int8_workspace_bytes(rows, groups, k, n);
}

int moe_int8_matmul(const void* x, int64_t x_stride, const int8_t* w, int64_t w_group_stride, int64_t w_row_stride, const float* w_scale,
                    int64_t w_scale_group_stride, const int32_t* offsets, int32_t rows, int32_t groups, int32_t k, int32_t n,
                    int32_t dtype, void* y, int64_t y_stride, void* workspace, void* stream) {
  if (!sizes_ok(rows, groups, k, n) || k > 1 << 17 || !float_type(dtype) || (!offsets && groups != 1)) return DSMOE_EINVAL;
  if (!in_stride(x_stride) || !in_stride(w_group_stride) || !in_stride(w_row_stride) || !in_stride(w_scale_group_stride) || !out_stride(y_stride, n))
    return DSMOE_EINVAL;
  if (rows == 0) return DSMOE_OK;
  if (!x || !w || !w_scale || !y || !workspace || ((uintptr_t)workspace & 255) != 0 || !aligned_to(x, dtype) || !aligned_to(y, dtype) ||
      ((uintptr_t)w_scale & 3) != 0)
    return DSMOE_EINVAL;
  if (row_tiles_bound(rows, groups, offsets != nullptr, 128) * tiles(n, 128) > kMostPieces) return DSMOE_EINVAL;
  Int8Args a = {};
  a.x = x;
  a.x_row = x_stride;
  a.w = w;
  a.w_row = w_row_stride;
  a.w_group = w_group_stride;
  a.w_scale = w_scale;
  a.ws_group = w_scale_group_stride;
  a.offsets = offsets;
  a.y = y;
  a.y_row = y_stride;
  a.R = rows;
  a.G = groups;
  a.N = n;
  a.K = k;
  a.type = dtype;
  a.workspace = (char*)workspace;
  return status(launch_int8_matmul(a, (hipStream_t)stream));
}

size_t dsmoe_int4_workspace_bytes(const dsmoe_int4_args* args) {
  static const int32_t some = 0;
  if (!int4_args_ok(args)) return 0;
  Int4Args g = int4_args(args);
  g.off = &some;
  return int4_workspace_bytes(g);
}

int moe_int4_matmul(const dsmoe_int4_args* args, const void* x, const uint8_t* w, const void* w_scale, const uint8_t* w_zero,
                    const int32_t* offsets, void* y, void* workspace, void* stream) {
  const dsmoe_int4_args* a = args;
  if (!int4_args_ok(a) || (!offsets && a->groups != 1) || ((uintptr_t)workspace & 255) != 0) return DSMOE_EINVAL;
  if (!in_stride(a->x_stride) || !out_stride(a->y_stride, a->n)) return DSMOE_EINVAL;
  for (const int64_t s : {a->w_group_stride, a->w_row_stride, a->scale_group_stride, a->scale_row_stride})
    if (!in_stride(s)) return DSMOE_EINVAL;
  if (w_zero && (!in_stride(a->zero_group_stride) || !in_stride(a->zero_row_stride))) return DSMOE_EINVAL;
  if (a->rows == 0) return DSMOE_OK;
  if (!x || !w || !w_scale || !y || !aligned_to(x, a->dtype) || !aligned_to(y, a->dtype) || !aligned_to(w_scale, a->scale_dtype)) return DSMOE_EINVAL;
  Int4Args g = int4_args(a);
  g.x = (const char*)x;
  g.w = w;
  g.scale = (const char*)w_scale;
  g.zero = w_zero;
  g.off = offsets;
  g.y = (char*)y;
  g.partial = (char*)workspace;
  return status(launch_int4_matmul(g, (hipStream_t)stream));
}

int moe_block_norm(const dsmoe_block_norm_args* args, const void* x, const void* branch, const void* branch_weight, const void* gate,
                   const void* weight, void* y, void* h, float* stats, void* stream) {
  if (!norm_args_ok(args)) return DSMOE_EINVAL;
  if (args->tokens == 0) return DSMOE_OK;
  if (!x || !branch || !branch_weight || !weight || !y || !h || (args->gate_kind != 0) != (gate != nullptr)) return DSMOE_EINVAL;
  for (const void* p : {x, branch, branch_weight, gate, weight, (const void*)y, (const void*)h})
    if (!aligned_to(p, args->dtype)) return DSMOE_EINVAL;
  BlockNormArgs n = norm_args(args, x, branch, branch_weight, gate, weight);
  n.y = y;
  n.h = h;
  n.stats = stats;
  return status(launch_block_norm(n, (hipStream_t)stream));
}

size_t dsmoe_block_norm_workspace_bytes(const dsmoe_block_norm_args* args) {
  return norm_args_ok(args) ? block_norm_backward_bytes(args->tokens, args->d, args->gate_kind) : 0;
}

int moe_block_norm_backward(const dsmoe_block_norm_args* args, const void* dy, const void* dh, const void* x, const void* branch,
                            const void* branch_weight, const void* gate, const void* weight, const float* stats, void* dx, void* dbranch,
                            void* dbranch_weight, void* dgate, void* dweight, void* workspace, void* stream) {
  if (!norm_args_ok(args) || !in_stride(args->dy_stride) || !in_stride(args->dh_stride)) return DSMOE_EINVAL;
  const bool has_gate = args->gate_kind != 0;
  if (!branch_weight || !weight || !dbranch_weight || !dweight) return DSMOE_EINVAL;
  if (args->tokens > 0 && (!dy || !dh || !x || !branch || !stats || !dx || !dbranch || !workspace || has_gate != (gate != nullptr))) return DSMOE_EINVAL;
  if (has_gate != (dgate != nullptr) && (args->tokens > 0 || args->gate_kind == 2)) return DSMOE_EINVAL;
  if (((uintptr_t)workspace & 255) != 0 || ((uintptr_t)stats & 3) != 0) return DSMOE_EINVAL;
  for (const void* p : {dy, dh, x, branch, branch_weight, gate, weight, (const void*)dx, (const void*)dbranch, (const void*)dbranch_weight,
                        (const void*)dgate, (const void*)dweight})
    if (!aligned_to(p, args->dtype)) return DSMOE_EINVAL;
  BlockNormArgs n = norm_args(args, x, branch, branch_weight, gate, weight);
  n.stats = const_cast<float*>(stats);
  n.dy = dy;
  n.dh = dh;
  n.dy_row = args->dy_stride;
  n.dh_row = args->dh_stride;
  n.dx = dx;
  n.dbranch = dbranch;
  n.dgate = dgate;
  n.dbranch_weight = dbranch_weight;
  n.dweight = dweight;
  n.partial = (float*)workspace;
  return status(launch_block_norm_backward(n, (hipStream_t)stream));
}

size_t dsmoe_gated_workspace_bytes(const dsmoe_gated_args* args) {
  return gated_args_ok(args) ? gated_workspace_bytes(gated_args(args, nullptr, nullptr, nullptr, nullptr, nullptr)) : 0;
}

int moe_gated_matmul(const dsmoe_gated_args* args, const void* x, const void* w1, const void* w3, const int32_t* offsets, void* h, float* saved,
                     void* workspace, void* stream) {
  if (!gated_args_ok(args) || !out_stride(args->h_stride, args->n) || (!offsets && args->groups != 1) || ((uintptr_t)workspace & 255) != 0) return DSMOE_EINVAL;
  if (args->rows == 0) return DSMOE_OK;
  if (!x || !w1 || !w3 || !h || ((uintptr_t)saved & 3) != 0) return DSMOE_EINVAL;
  for (const void* p : {x, w1, w3, (const void*)h})
    if (!aligned_to(p, args->dtype)) return DSMOE_EINVAL;
  GatedArgs g = gated_args(args, x, w1, w3, offsets, workspace);
  g.h = h;
  g.saved = saved;
  return status(launch_gated(g, (hipStream_t)stream));
}

size_t dsmoe_gated_backward_workspace_bytes(const dsmoe_gated_args* args) {
  return gated_backward_args_ok(args) ? gated_backward_workspace_bytes(gated_args(args, nullptr, nullptr, nullptr, nullptr, nullptr)) : 0;
}

int moe_gated_matmul_backward(const dsmoe_gated_args* args, const void* dh, const void* x, const void* w1, const void* w3, const float* saved,
                              const int32_t* offsets, void* dx, void* dw1, void* dw3, void* workspace, void* stream) {
  if (!gated_backward_args_ok(args) || (!offsets && args->groups != 1) || ((uintptr_t)workspace & 255) != 0 || ((uintptr_t)saved & 3) != 0) return DSMOE_EINVAL;
  if (!dw1 || !dw3 || (args->rows > 0 && (!dh || !x || !w1 || !w3 || !saved || !dx || !workspace))) return DSMOE_EINVAL;
  for (const void* p : {dh, x, w1, w3, (const void*)dx, (const void*)dw1, (const void*)dw3})
    if (!aligned_to(p, args->dtype)) return DSMOE_EINVAL;
  GatedArgs g = gated_args(args, x, w1, w3, offsets, workspace);
  g.dh = dh;
  g.saved = const_cast<float*>(saved);
  g.dx = dx;
  g.dw1 = dw1;
  g.dw3 = dw3;
  return status(launch_gated_backward(g, (hipStream_t)stream));
}

size_t dsmoe_clip_workspace_bytes(void) { return clip_grads_bytes(); }

int moe_grad_norm(const dsmoe_grad* grads, int32_t count, float* norm, void* workspace, void* stream) {
  if (!grads_ok(grads, count, false, norm, workspace)) return DSMOE_EINVAL;
  return status(launch_clip_grads(grads, count, false, 0.f, 0.f, norm, (double*)workspace, (hipStream_t)stream));
}

int moe_clip_grads(const dsmoe_grad* grads, int32_t count, float max_norm, float eps, float* norm, void* workspace, void* stream) {
  if (!grads_ok(grads, count, true, norm, workspace) || !(max_norm >= 0.f) || !(eps >= 0.f)) return DSMOE_EINVAL;
  return status(launch_clip_grads(grads, count, true, max_norm, eps, norm, (double*)workspace, (hipStream_t)stream));
}

}  // extern "C"
