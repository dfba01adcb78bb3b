// C ABI of the operators beside the layer (see include/dsmoe.h): argument checks and launches.
#include "block_norm.h"
#include "grouped.h"
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

}  // extern "C"
