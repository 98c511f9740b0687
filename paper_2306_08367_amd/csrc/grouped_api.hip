// C entry points of the grouped operators: validation, the choice between aligned and unaligned reads, workspaces.
#include "grouped.h"

namespace lq {
namespace {

constexpr int64_t MAX_POSITIONS = 1ll << 30;
constexpr int32_t MAX_WIDTH = 1 << 30;

int check_stack(const lq_stack* w, const char* what, int32_t count, int32_t rows, int32_t cols, bool output) {
  if (!w) return fail(LQ_ERR_NULL, "%s is NULL", what);
  if (!dtype_ok(w->dtype)) return fail(LQ_ERR_DTYPE, "%s: unknown dtype %d", what, w->dtype);
  if (w->count != count || w->rows != rows || w->cols != cols)
    return fail(LQ_ERR_SHAPE, "%s is %d x %d x %d, expected %d x %d x %d", what, w->count, w->rows, w->cols, count, rows, cols);
  if (w->ld < w->cols) return fail(LQ_ERR_SHAPE, "%s: ld %lld < cols %d", what, (long long)w->ld, w->cols);
  if (w->stride < 0) return fail(LQ_ERR_SHAPE, "%s: negative stride", what);
  if (output && count > 1 && w->stride < (rows - 1) * w->ld + cols) return fail(LQ_ERR_SHAPE, "%s: matrices overlap", what);
  if (!w->data) return fail(LQ_ERR_NULL, "%s: data is NULL", what);
  if (!aligned(w->data, dtype_size(w->dtype))) return fail(LQ_ERR_SHAPE, "%s: data is not aligned to its element size", what);
  return LQ_OK;
}

int check_groups(const lq_groups* g) {
  if (!g) return fail(LQ_ERR_NULL, "groups is NULL");
  if (g->n < 0 || g->n > MAX_POSITIONS) return fail(LQ_ERR_SHAPE, "n %lld outside 0..2^30", (long long)g->n);
  if (g->n_groups < 1 || g->n_groups > LQ_MAX_MODELS)
    return fail(LQ_ERR_SHAPE, "n_groups %d outside 1..%d", g->n_groups, LQ_MAX_MODELS);
  if (!g->offsets) return fail(LQ_ERR_NULL, "offsets is NULL");
  if (!aligned(g->offsets, 4) || !aligned(g->order, 4)) return fail(LQ_ERR_SHAPE, "offsets or order is not 4-byte aligned");
  return LQ_OK;
}

// A matrix of `rows` x `cols`; data may be missing only where there are no rows.
int check_shape(const lq_mat* m, const char* what, int64_t rows, int32_t cols) {
  if (!m) return fail(LQ_ERR_NULL, "%s is NULL", what);
  int rc = check_mat(*m, what, -1, true);
  if (rc) return rc;
  if (m->rows != rows || m->cols != cols)
    return fail(LQ_ERR_SHAPE, "%s is %lld x %d, expected %lld x %d", what, (long long)m->rows, m->cols, (long long)rows, cols);
  return LQ_OK;
}

int check_workspace(const void* ws, size_t ws_bytes, size_t need, const char* why) {
  if (need == 0) return LQ_OK;
  if (!ws || ws_bytes < need || !aligned(ws, 256))
    return fail(LQ_ERR_WORKSPACE, "%s needs a 256-byte aligned workspace of %zu bytes", why, need);
  return LQ_OK;
}

// Whether two columns of 4-byte entries share memory.
bool share(const int32_t* a, int64_t na, const int32_t* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + 4 * static_cast<uintptr_t>(nb) && y < x + 4 * static_cast<uintptr_t>(na);
}

int read_flag(const int32_t* flag, int32_t* value, hipStream_t s) {
  LQ_HIP_TRY(hipMemcpyAsync(value, flag, sizeof(*value), hipMemcpyDeviceToHost, s));
  LQ_HIP_TRY(hipStreamSynchronize(s));
  return LQ_OK;
}

// LQ_CHECK_FKS: verifies offsets and order on the device and waits for the answer.
int verify_groups(const lq_groups& g, uint32_t flags, void* ws, size_t ws_bytes, hipStream_t s) {
  if (!(flags & LQ_CHECK_FKS)) return LQ_OK;
  int rc = check_workspace(ws, ws_bytes, 256, "LQ_CHECK_FKS");
  if (rc) return rc;
  int32_t* flag = static_cast<int32_t*>(ws);
  if ((rc = launch_check_groups(g, flag, s))) return rc;
  int32_t bad = 0;
  if ((rc = read_flag(flag, &bad, s))) return rc;
  if (bad & 1) return fail(LQ_ERR_FK_RANGE, "offsets do not ascend from 0 to at most n");
  if (bad & 2) return fail(LQ_ERR_FK_RANGE, "an entry of order lies outside [0, n)");
  return LQ_OK;
}

// The pieces (16 or 4 bytes, 0: elements of two) in which rows may be read: they start and end on boundaries of those.
int piece_bytes(const void* data, int64_t ld, int32_t cols, int64_t stride, int32_t dtype) {
  const int64_t size = static_cast<int64_t>(dtype_size(dtype));
  for (const int bytes : {16, 4})
    if (aligned(data, bytes) && ld * size % bytes == 0 && cols * size % bytes == 0 && stride * size % bytes == 0) return bytes;
  return 0;
}
int piece_bytes(const lq_mat& m) { return piece_bytes(m.data, m.ld, m.cols, 0, m.dtype); }
int piece_bytes(const lq_stack& w) { return piece_bytes(w.data, w.ld, w.cols, w.count > 1 ? w.stride : 0, w.dtype); }
// Rows that start on 16-byte boundaries.
bool aligned_rows(const void* data, int64_t ld, int32_t dtype) { return aligned(data, 16) && ld % (16 / static_cast<int64_t>(dtype_size(dtype))) == 0; }

}  // namespace
}  // namespace lq

using namespace lq;

extern "C" {

size_t lq_group_rows_workspace_bytes(int64_t n, int32_t n_groups) {
  if (n < 0 || n > MAX_POSITIONS || n_groups < 1 || n_groups > LQ_MAX_MODELS) return 0;
  return group_rows_ws_bytes(n, n_groups);
}

int lq_group_rows(const int32_t* keys, int64_t n, int32_t n_groups, int32_t* offsets, int32_t* order, void* ws, size_t ws_bytes,
                  uint32_t flags, void* hip_stream) {
  clear_error();
  if (n < 0 || n > MAX_POSITIONS) return fail(LQ_ERR_SHAPE, "n %lld outside 0..2^30", (long long)n);
  if (n_groups < 1 || n_groups > LQ_MAX_MODELS) return fail(LQ_ERR_SHAPE, "n_groups %d outside 1..%d", n_groups, LQ_MAX_MODELS);
  if (!offsets || (n > 0 && (!keys || !order))) return fail(LQ_ERR_NULL, "keys, offsets or order is NULL");
  if (!aligned(keys, 4) || !aligned(offsets, 4) || !aligned(order, 4))
    return fail(LQ_ERR_SHAPE, "keys, offsets or order is not 4-byte aligned");
  if (flags & ~LQ_CHECK_FKS) return fail(LQ_ERR_UNSUPPORTED, "unknown flags 0x%x", flags);
  int rc = check_workspace(ws, ws_bytes, group_rows_ws_bytes(n, n_groups), "lq_group_rows");
  if (rc) return rc;
  if ((flags & LQ_CHECK_FKS) && n > 0 && (rc = check_workspace(ws, ws_bytes, 256, "LQ_CHECK_FKS"))) return rc;
  // (keys are read again while order is written: changed ones would give places outside of it)
  if (n > 0 && (share(order, n, keys, n) || share(offsets, n_groups + 1, keys, n) || share(offsets, n_groups + 1, order, n)))
    return fail(LQ_ERR_SHAPE, "keys, offsets and order overlap");
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if ((flags & LQ_CHECK_FKS) && n > 0) {
    int32_t bad = 0, *flag = static_cast<int32_t*>(ws);
    if ((rc = launch_check_keys(keys, n, n_groups, flag, s))) return rc;
    if ((rc = read_flag(flag, &bad, s))) return rc;
    if (bad) return fail(LQ_ERR_FK_RANGE, "a key is %d or more", n_groups);
  }
  return launch_group_rows(keys, n, n_groups, offsets, order, ws, s);
}

size_t lq_grouped_workspace_bytes(int64_t n, int32_t n_groups, int32_t k, int32_t l, int32_t dtype) {
  if (n < 0 || n > MAX_POSITIONS || n_groups < 1 || n_groups > LQ_MAX_MODELS || k < 1 || l < 1 || !dtype_ok(dtype)) return 0;
  return grouped_product_ws_bytes(n, n_groups, k, l, dtype);
}
size_t lq_grouped_gradient_workspace_bytes(int64_t n, int32_t n_groups, int32_t k, int32_t l, int32_t dtype) {
  if (n < 0 || n > MAX_POSITIONS || n_groups < 1 || n_groups > LQ_MAX_MODELS || k < 1 || l < 1 || !dtype_ok(dtype)) return 0;
  return grouped_gradient_ws_bytes(n, n_groups, k, l, dtype);
}

int lq_grouped_product(const lq_groups* groups, const lq_mat* X, int32_t x_slots, const lq_stack* W, const lq_mat* bias,
                       const lq_mat* gate, lq_mat* Y, void* ws, size_t ws_bytes, uint32_t flags, void* hip_stream) {
  clear_error();
  int rc = check_groups(groups);
  if (rc) return rc;
  if (flags & ~(LQ_CHECK_FKS | LQ_RELU | LQ_TRANSPOSED | LQ_X_GROUPED | LQ_Y_GROUPED))
    return fail(LQ_ERR_UNSUPPORTED, "unknown flags 0x%x", flags);
  const bool transposed = flags & LQ_TRANSPOSED;
  if (!X || !W || !Y) return fail(LQ_ERR_NULL, "X, W or Y is NULL");
  if ((rc = check_stack(W, "W", groups->n_groups, W->rows, W->cols, false))) return rc;
  const int32_t K = transposed ? W->cols : W->rows, N = transposed ? W->rows : W->cols;
  if (K < 1 || N < 1) return fail(LQ_ERR_SHAPE, "W has no rows or no columns");
  if (K > MAX_WIDTH || N > MAX_WIDTH) return fail(LQ_ERR_SHAPE, "W has more than 2^30 rows or columns");
  const int64_t n = groups->n;
  if (x_slots < 1 || (x_slots > 1 && (transposed || (flags & LQ_X_GROUPED))))
    return fail(LQ_ERR_SHAPE, "x_slots %d: must be 1, or more without LQ_TRANSPOSED and LQ_X_GROUPED", x_slots);
  if (n % x_slots) return fail(LQ_ERR_SHAPE, "%lld positions are not a multiple of x_slots %d", (long long)n, x_slots);
  if ((rc = check_shape(X, "X", n / x_slots, K))) return rc;
  if ((rc = check_shape(Y, "Y", n, N))) return rc;
  if (X->dtype != W->dtype) return fail(LQ_ERR_DTYPE, "X and W differ in dtype");
  if (Y->dtype != X->dtype && X->dtype != LQ_BF16) return fail(LQ_ERR_DTYPE, "bf16 output needs bf16 inputs");
  if (bias) {
    if ((rc = check_shape(bias, "bias", groups->n_groups, N))) return rc;
    if (bias->dtype != X->dtype) return fail(LQ_ERR_DTYPE, "bias and X differ in dtype");
  }
  if (gate) {
    if ((rc = check_shape(gate, "gate", n, N))) return rc;
    if (gate->dtype != X->dtype) return fail(LQ_ERR_DTYPE, "gate and X differ in dtype");
  }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if ((rc = verify_groups(*groups, flags, ws, ws_bytes, s))) return rc;
  if (n == 0) return LQ_OK;

  GroupedArgs a{};
  a.off = groups->offsets; a.order = groups->order; a.G = groups->n_groups; a.n = static_cast<int32_t>(n);
  a.X = X->data; a.ldx = X->ld;
  a.W = W->data; a.ldw = W->ld; a.sw = W->stride;
  if (bias) { a.bias = bias->data; a.ldb = bias->ld; }
  if (gate) { a.gate = gate->data; a.ldg = gate->ld; }
  a.Y = Y->data; a.ldy = Y->ld; a.y_bf16 = Y->dtype == LQ_BF16;
  a.K = K; a.N = N; a.n_store = N;
  a.slots = x_slots;
  a.x_grouped = (flags & LQ_X_GROUPED) != 0; a.y_grouped = (flags & LQ_Y_GROUPED) != 0;
  a.relu = (flags & LQ_RELU) != 0;
  a.y_vec = aligned_rows(Y->data, Y->ld, Y->dtype) && (!gate || aligned_rows(gate->data, gate->ld, gate->dtype)) &&
            (!bias || aligned_rows(bias->data, bias->ld, bias->dtype));
  if (ws && !aligned(ws, 256)) return fail(LQ_ERR_WORKSPACE, "lq_grouped_product: the workspace is not 256-byte aligned");
  return launch_grouped_product(a, X->dtype, transposed, std::min(piece_bytes(*X), piece_bytes(*W)), ws, ws_bytes, s);
}

int lq_grouped_gradient(const lq_groups* groups, const lq_mat* X, int32_t x_slots, const lq_mat* dY, lq_stack* dW, lq_mat* db,
                        void* ws, size_t ws_bytes, uint32_t flags, void* hip_stream) {
  clear_error();
  int rc = check_groups(groups);
  if (rc) return rc;
  if (flags & ~(LQ_CHECK_FKS | LQ_X_GROUPED | LQ_Y_GROUPED)) return fail(LQ_ERR_UNSUPPORTED, "unknown flags 0x%x", flags);
  if (!X || !dY || !dW) return fail(LQ_ERR_NULL, "X, dY or dW is NULL");
  const int64_t n = groups->n;
  if (x_slots < 1 || (x_slots > 1 && (flags & LQ_X_GROUPED)))
    return fail(LQ_ERR_SHAPE, "x_slots %d: must be 1, or more without LQ_X_GROUPED", x_slots);
  if (n % x_slots) return fail(LQ_ERR_SHAPE, "%lld positions are not a multiple of x_slots %d", (long long)n, x_slots);
  if (X->cols < 1 || dY->cols < 1) return fail(LQ_ERR_SHAPE, "X or dY has no columns");
  if (X->cols > MAX_WIDTH || dY->cols > MAX_WIDTH) return fail(LQ_ERR_SHAPE, "X or dY has more than 2^30 columns");
  if ((rc = check_shape(X, "X", n / x_slots, X->cols))) return rc;
  if ((rc = check_shape(dY, "dY", n, dY->cols))) return rc;
  if (X->dtype != dY->dtype) return fail(LQ_ERR_DTYPE, "X and dY differ in dtype");
  if ((rc = check_stack(dW, "dW", groups->n_groups, X->cols, dY->cols, true))) return rc;
  if (dW->dtype != X->dtype && X->dtype != LQ_BF16) return fail(LQ_ERR_DTYPE, "bf16 output needs bf16 inputs");
  if (db) {
    if ((rc = check_shape(db, "db", groups->n_groups, dY->cols))) return rc;
    if (db->dtype != dW->dtype) return fail(LQ_ERR_DTYPE, "db and dW differ in dtype");
  }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if ((rc = verify_groups(*groups, flags, ws, ws_bytes, s))) return rc;

  GradientArgs a{};
  a.off = groups->offsets; a.order = groups->order; a.G = groups->n_groups; a.n = static_cast<int32_t>(n);
  a.X = X->data; a.ldx = X->ld; a.slots = x_slots; a.x_grouped = (flags & LQ_X_GROUPED) != 0;
  a.dY = dY->data; a.ldy = dY->ld; a.y_grouped = (flags & LQ_Y_GROUPED) != 0;
  a.dW = dW->data; a.ldw = dW->ld; a.sw = dW->stride; a.w_bf16 = dW->dtype == LQ_BF16;
  if (db) { a.db = db->data; a.ldb = db->ld; }
  a.k = X->cols; a.l = dY->cols;
  if (ws && !aligned(ws, 256)) return fail(LQ_ERR_WORKSPACE, "lq_grouped_gradient: the workspace is not 256-byte aligned");
  return launch_grouped_gradient(a, X->dtype, std::min(piece_bytes(*X), piece_bytes(*dY)), ws, ws_bytes, s);
}

size_t lq_adapter_workspace_bytes(int64_t n, int32_t n_groups, int32_t k, int32_t l, int32_t rank, int32_t dtype) {
  if (n < 0 || n > MAX_POSITIONS || n_groups < 1 || n_groups > LQ_MAX_MODELS || k < 1 || l < 1 || rank < 1 || rank > LQ_MAX_RANK ||
      !dtype_ok(dtype))
    return 0;
  return adapter_ws_bytes(n, n_groups, k, l, rank, dtype);
}

int lq_adapter_product(const lq_groups* groups, const lq_mat* X, const lq_mat* W, const lq_mat* bias, const lq_stack* A,
                       const lq_stack* B, const float* scale, lq_mat* Y, void* ws, size_t ws_bytes, uint32_t flags, void* hip_stream) {
  clear_error();
  int rc = check_groups(groups);
  if (rc) return rc;
  if (flags & ~LQ_CHECK_FKS) return fail(LQ_ERR_UNSUPPORTED, "unknown flags 0x%x", flags);
  if (!X || !W || !A || !B || !Y) return fail(LQ_ERR_NULL, "X, W, A, B or Y is NULL");
  const int64_t n = groups->n;
  if (W->rows < 1 || W->cols < 1) return fail(LQ_ERR_SHAPE, "W has no rows or no columns");
  if (W->rows > MAX_WIDTH || W->cols > MAX_WIDTH) return fail(LQ_ERR_SHAPE, "W has more than 2^30 rows or columns");
  const int32_t k = static_cast<int32_t>(W->rows), l = W->cols, rank = A->cols;
  if (rank < 1 || rank > LQ_MAX_RANK) return fail(LQ_ERR_SHAPE, "rank %d outside 1..%d", rank, LQ_MAX_RANK);
  if ((rc = check_shape(W, "W", k, l))) return rc;
  if ((rc = check_shape(X, "X", n, k))) return rc;
  if ((rc = check_shape(Y, "Y", n, l))) return rc;
  if ((rc = check_stack(A, "A", groups->n_groups, k, rank, false))) return rc;
  if ((rc = check_stack(B, "B", groups->n_groups, rank, l, false))) return rc;
  if (X->dtype != W->dtype || A->dtype != W->dtype || B->dtype != W->dtype)
    return fail(LQ_ERR_DTYPE, "X, W, A and B differ in dtype");
  if (Y->dtype != X->dtype && X->dtype != LQ_BF16) return fail(LQ_ERR_DTYPE, "bf16 output needs bf16 inputs");
  if (bias) {
    if ((rc = check_shape(bias, "bias", 1, l))) return rc;
    if (bias->dtype != X->dtype) return fail(LQ_ERR_DTYPE, "bias and X differ in dtype");
  }
  if (!aligned(scale, 4)) return fail(LQ_ERR_SHAPE, "scale is not 4-byte aligned");
  const int32_t dt = X->dtype;
  if ((rc = check_workspace(ws, ws_bytes, lq_adapter_workspace_bytes(n, groups->n_groups, k, l, rank, dt), "lq_adapter_product"))) return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if ((rc = verify_groups(*groups, flags, ws, ws_bytes, s))) return rc;
  if (n == 0) return LQ_OK;

  GroupedArgs a{};
  a.off = groups->offsets; a.order = groups->order; a.G = groups->n_groups; a.n = static_cast<int32_t>(n);
  a.X = X->data; a.ldx = X->ld; a.K = k; a.slots = 1;
  a.W = W->data; a.ldw = W->ld;
  if (bias) { a.bias = bias->data; a.ldb = bias->ld; }
  a.Y = Y->data; a.ldy = Y->ld; a.y_bf16 = Y->dtype == LQ_BF16; a.N = l; a.n_store = l;
  a.y_vec = aligned_rows(Y->data, Y->ld, Y->dtype) && (!bias || aligned_rows(bias->data, bias->ld, bias->dtype));
  a.B = B->data; a.ldB = B->ld; a.sB = B->stride; a.rank = rank;
  const int of_x = piece_bytes(*X);
  return launch_adapter_product(a, *A, scale, ws, dt, std::min({of_x, piece_bytes(*W), piece_bytes(*B)}), std::min(of_x, piece_bytes(*A)), s);
}

}  // extern "C"
