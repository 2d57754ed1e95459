// extern "C" entry points of the 8-bit floating-point layers, the norms and log probabilities: argument checks and dispatch.
#include "bsp_f8.h"

#include <string.h>

namespace {

inline bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool value_type(int d) { return d == BSP_F32 || d == BSP_BF16; }
inline bool code_type(int d) { return d == BSP_E4M3 || d == BSP_E5M2; }
inline unsigned size_of(int d) { return d == BSP_F32 ? 4 : 2; }
constexpr int32_t kMost = INT32_MAX - 65536;  // rows and columns: sizes rounded up stay in 32 bits
constexpr int32_t kWide = 1 << 24;            // columns of codes: 256 rows' offsets stay in 32 bits
constexpr int32_t kSlots = 1024, kRank = 128;  // adapters of a set, ranks of one
constexpr int32_t kRequests = 1 << 26;        // rows of a batch with adapters: their tiles' threads are counted along one dimension of a launch
constexpr int32_t kVocabulary = 1 << 21;      // logits of a row: 64 chunks of what a workgroup's registers hold
constexpr float kSharpest = 0x1p100f;         // of a temperature's inverse: times log2 e it is a number
constexpr int32_t kTop = 64;                  // likeliest tokens: one of 64 groups' largest is below the last of them

// a matrix of values whose rows are `ld` elements apart; rows of an input may be the same one (ld = 0)
int check_values(const void* p, int dtype, int64_t ld, int T, int K, bool input) {
  if (!value_type(dtype)) return BSP_ERR_DTYPE;
  if (T < 0 || T > kMost || K < 1 || K > kMost) return BSP_ERR_SHAPE;
  if (!(ld >= K || (input && ld == 0) || T <= 1) || ld < 0 || ld > INT64_MAX / 64 / (T + 1)) return BSP_ERR_SHAPE;
  if (T > 0 && !p) return BSP_ERR_NULL;
  return aligned(p, size_of(dtype)) ? BSP_OK : BSP_ERR_ALIGN;
}

int check_codes(const bsp_codes* c) {
  if (!c) return BSP_ERR_NULL;
  if (!code_type(c->dtype)) return BSP_ERR_DTYPE;
  if (c->T < 0 || c->T > kMost || c->K < 1 || c->K > kWide) return BSP_ERR_SHAPE;
  if (c->T > 0 && (!c->codes || !c->scale)) return BSP_ERR_NULL;
  return aligned(c->codes, 16) && aligned(c->scale, 16) ? BSP_OK : BSP_ERR_ALIGN;
}

int check_weights(const bsp_weights_f8* w) {
  if (!w) return BSP_ERR_NULL;
  if (w->O < 1 || w->O > kWide || w->I < 1 || w->I > kWide) return BSP_ERR_SHAPE;
  if (w->nnzb < 0 || w->nnzb > INT32_MAX || w->nnzb > (int64_t)f8_blocks(w->O) * f8_blocks(w->I)) return BSP_ERR_SHAPE;
  if (!w->row_ptr || !w->col_ptr) return BSP_ERR_NULL;
  if (w->nnzb > 0 && (!w->col_idx || !w->row_idx || !w->payload || !w->scale || !w->payload_t || !w->scale_t)) return BSP_ERR_NULL;
  return aligned(w->payload, 16) && aligned(w->payload_t, 16) && aligned(w->row_ptr, 4) && aligned(w->col_idx, 4) &&
                 aligned(w->col_ptr, 4) && aligned(w->row_idx, 4)
             ? BSP_OK
             : BSP_ERR_ALIGN;
}

F8Rows rows_of(const bsp_weights_f8* w, bool transposed) {
  if (transposed) return F8Rows{w->col_ptr, w->row_idx, w->payload_t, w->scale_t, w->I, w->O, w->nnzb};
  return F8Rows{w->row_ptr, w->col_idx, w->payload, w->scale, w->O, w->I, w->nnzb};
}

// Whether values become codes inside the kernel that multiplies them: few rows, of whole aligned pieces of 16 bytes, that fit its LDS.
bool in_kernel(const void* X, int dtype, int64_t ld, int T, int K) {
  return T <= 16 && f8_few_staged(T, K) <= kFewStaged &&
         ((reinterpret_cast<uintptr_t>(X) | (uintptr_t)(ld * size_of(dtype)) | (uintptr_t)(K * (int64_t)size_of(dtype))) & 15u) == 0;
}
// up to here the kernel without LDS tiles (us, it and the smallest tile: 32 x 4096 -> 4096 8.8 and 10.7, 64 x 4096 -> 4096 12.5 and 11.0,
// 64 x 16384 -> 1024 38.8 and 34.8, 64 x 512 -> 16384 9.3 and 5.7)
constexpr int kFewRows = 32;

int check_product(const bsp_weights_f8* w, int32_t transposed, int32_t T, const float* bias, const void* residual, int32_t relu,
                  const bsp_codes* gate, void* Y, int32_t y_dtype, F8Epilogue* q) {
  int rc = check_weights(w);
  if (rc != BSP_OK) return rc;
  if (!value_type(y_dtype)) return BSP_ERR_DTYPE;
  const int out = transposed ? w->I : w->O;
  if (gate) {
    rc = check_codes(gate);
    if (rc != BSP_OK) return rc;
    if (gate->T != T || gate->K != out) return BSP_ERR_SHAPE;
  }
  if (T > 0 && !Y) return BSP_ERR_NULL;
  if (!aligned(Y, 16) || !aligned(residual, 16) || !aligned(bias, 4)) return BSP_ERR_ALIGN;
  *q = F8Epilogue{Y, bias, residual, gate ? gate->codes : nullptr, relu != 0, gate ? gate->dtype == BSP_E5M2 : 0};
  return BSP_OK;
}

int split_of(const F8Rows& rows, int T, bool f32) { return T <= kFewRows ? f8_few_split(rows, T) : f8_tile_split(rows, T, f32); }

int64_t sums_bytes(const F8Rows& rows, int T) {
  int64_t split = 1;
  for (int f32 = 0; f32 < 2 && T > 0; ++f32) {  // results of either type fit
    const int64_t s = split_of(rows, T, f32);
    if (s > split) split = s;
  }
  return split > 1 ? split * T * ((rows.out + 3) / 4) * 16 : 0;
}

int multiply(const F8Rows& rows, const F8Input& x, int T, const F8Low& low, const F8Epilogue& q, int32_t y_dtype, void* sums, hipStream_t st) {
  const bool f32 = y_dtype == BSP_F32;
  const int rc = T <= kFewRows ? f8_launch_few(rows, x, T, low, q, f32, (float*)sums, st) : f8_launch_tile(rows, x, T, low, q, f32, (float*)sums, st);
  if (rc != BSP_OK) return rc;
  const int split = split_of(rows, T, f32);
  return split > 1 ? f8_launch_join((const float*)sums, split, T, rows.out, q, f32, st) : BSP_OK;
}

// rows given as values: workspace holds `sums` bytes, behind them the codes of rows that do not become codes in the product's kernel
int multiply_values(const F8Rows& rows, const void* X, int x_dtype, int64_t ldx, int T, int K, bool e5, const F8Epilogue& q, int32_t y_dtype,
                    void* workspace, int64_t sums, hipStream_t st) {
  if (in_kernel(X, x_dtype, ldx, T, K)) return multiply(rows, F8Input{X, nullptr, x_dtype, e5, ldx}, T, F8Low{}, q, y_dtype, workspace, st);
  const int64_t ld = (int64_t)f8_blocks(K) * F8_BLOCK;
  uint8_t *codes = (uint8_t*)workspace + sums, *scale = codes + T * ld;
  const int rc = f8_launch_save(X, x_dtype == BSP_F32, ldx, T, K, e5, codes, scale, st);
  if (rc != BSP_OK) return rc;
  return multiply(rows, F8Input{codes, scale, e5 ? BSP_E5M2 : BSP_E4M3, e5, ld}, T, F8Low{}, q, y_dtype, workspace, st);
}

int check_workspace(const void* workspace, int64_t bytes, int64_t need) {
  if (bytes < need) return BSP_ERR_CAPACITY;
  if (need > 0 && !workspace) return BSP_ERR_NULL;
  return aligned(workspace, 16) ? BSP_OK : BSP_ERR_ALIGN;
}

int check_adapters(const bsp_f8_adapters* d) {
  if (!d) return BSP_ERR_NULL;
  if (d->N < 1 || d->N > kSlots || d->R < 1 || d->R > kRank || d->I < 1 || d->I > kWide || d->O < 1 || d->O > kWide) return BSP_ERR_SHAPE;
  if (!d->a || !d->a_t || !d->b || !d->b_t || !d->scale) return BSP_ERR_NULL;
  return aligned(d->a, 16) && aligned(d->a_t, 16) && aligned(d->b, 16) && aligned(d->b_t, 16) && aligned(d->scale, 4) ? BSP_OK : BSP_ERR_ALIGN;
}
int check_requests(const bsp_f8_requests* r) {
  if (!r) return BSP_ERR_NULL;
  if (r->T < 0 || r->T > kRequests || r->N < 1 || r->N > kSlots) return BSP_ERR_SHAPE;
  if (r->T > 0 && !r->plan) return BSP_ERR_NULL;
  return aligned(r->plan, 16) ? BSP_OK : BSP_ERR_ALIGN;
}
// whether rows of several adapters may be multiplied in another order than their own (see F8Low)
bool sorts(const F8Adapters& d, int T) { return d.N > 1 && T > kFewRows; }
int64_t in16(int64_t bytes) { return (bytes + 15) & ~(int64_t)15; }
int64_t low_bytes(const F8Adapters& d, int T, int K, bool grad) { return (int64_t)T * d.Rp * 4 * f8_down_slices(T, d.N, K, grad); }

int64_t codes_bytes(int T, int K) { return ((int64_t)T * f8_blocks(K) * F8_BLOCK) + f8_scale_rows(T) * f8_blocks(K); }

}  // namespace

extern "C" {

int bsp_f8_save(const void* X, int32_t x_dtype, int64_t ldx, const bsp_codes* c, void* stream) {
  int rc = check_codes(c);
  if (rc != BSP_OK) return rc;
  rc = check_values(X, x_dtype, ldx, c->T, c->K, true);
  if (rc != BSP_OK || c->T == 0) return rc;
  return f8_launch_save(X, x_dtype == BSP_F32, ldx, c->T, c->K, c->dtype == BSP_E5M2, c->codes, c->scale, (hipStream_t)stream);
}

int bsp_f8_load(const bsp_codes* c, void* Y, int32_t y_dtype, int64_t ldy, void* stream) {
  int rc = check_codes(c);
  if (rc != BSP_OK) return rc;
  rc = check_values(Y, y_dtype, ldy, c->T, c->K, false);
  if (rc != BSP_OK || c->T == 0) return rc;
  return f8_launch_load(c->codes, c->scale, c->T, c->K, c->dtype == BSP_E5M2, Y, y_dtype == BSP_F32, ldy, (hipStream_t)stream);
}

int bsp_f8_pack(const bsp_weights_f8* w, const void* W, int32_t w_dtype, int64_t ldw, void* stream) {
  int rc = check_weights(w);
  if (rc != BSP_OK) return rc;
  rc = check_values(W, w_dtype, ldw, w->O, w->I, true);
  if (rc != BSP_OK || w->nnzb == 0) return rc;
  return f8_launch_pack(w, W, w_dtype == BSP_F32, ldw, (hipStream_t)stream);
}

int bsp_f8_fc(const bsp_weights_f8* w, int32_t transposed, const bsp_codes* X, const float* bias, const void* residual,
              int32_t relu, const bsp_codes* gate, void* Y, int32_t y_dtype, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_codes(X);
  if (rc != BSP_OK) return rc;
  F8Epilogue q;
  rc = check_product(w, transposed, X->T, bias, residual, relu, gate, Y, y_dtype, &q);
  if (rc != BSP_OK) return rc;
  if (X->K != (transposed ? w->O : w->I)) return BSP_ERR_SHAPE;
  if (X->T == 0) return BSP_OK;
  const F8Input x{X->codes, X->scale, X->dtype, X->dtype == BSP_E5M2, (int64_t)f8_blocks(X->K) * F8_BLOCK};
  const F8Rows rows = rows_of(w, transposed != 0);
  rc = check_workspace(workspace, workspace_bytes, sums_bytes(rows, X->T));
  return rc != BSP_OK ? rc : multiply(rows, x, X->T, F8Low{}, q, y_dtype, workspace, (hipStream_t)stream);
}

int bsp_f8_fc_workspace(const bsp_weights_f8* w, int32_t transposed, int32_t T, int32_t coded, int64_t* bytes) {
  if (!bytes) return BSP_ERR_NULL;
  const int rc = check_weights(w);
  if (rc != BSP_OK) return rc;
  if (T < 0 || T > kMost) return BSP_ERR_SHAPE;
  *bytes = sums_bytes(rows_of(w, transposed != 0), T) + (coded ? 0 : codes_bytes(T, transposed ? w->O : w->I));
  return BSP_OK;
}

int bsp_f8_fc_values(const bsp_weights_f8* w, int32_t transposed, const void* X, int32_t x_dtype, int64_t ldx, int32_t T,
                     int32_t code, const float* bias, const void* residual, int32_t relu, const bsp_codes* gate,
                     void* Y, int32_t y_dtype, void* workspace, int64_t workspace_bytes, void* stream) {
  F8Epilogue q;
  int rc = check_product(w, transposed, T, bias, residual, relu, gate, Y, y_dtype, &q);
  if (rc != BSP_OK) return rc;
  if (!code_type(code)) return BSP_ERR_DTYPE;
  const int K = transposed ? w->O : w->I;
  rc = check_values(X, x_dtype, ldx, T, K, true);
  if (rc != BSP_OK || T == 0) return rc;
  const bool e5 = code == BSP_E5M2;
  hipStream_t st = (hipStream_t)stream;
  const F8Rows rows = rows_of(w, transposed != 0);
  const int64_t sums = sums_bytes(rows, T);
  rc = check_workspace(workspace, workspace_bytes, sums + (in_kernel(X, x_dtype, ldx, T, K) ? 0 : codes_bytes(T, K)));
  if (rc != BSP_OK) return rc;
  return multiply_values(rows, X, x_dtype, ldx, T, K, e5, q, y_dtype, workspace, sums, st);
}

int bsp_f8_fc_grad_workspace(const bsp_weights_f8* w, int32_t T, int64_t* bytes) {
  if (!bytes) return BSP_ERR_NULL;
  const int rc = check_weights(w);
  if (rc != BSP_OK) return rc;
  if (T < 0 || T > kMost) return BSP_ERR_SHAPE;
  const int64_t split = f8_grad_split(w->nnzb, T);
  *bytes = split > 1 ? split * (w->nnzb * F8_BLOCK_BYTES + w->O) * 4 : 0;
  return BSP_OK;
}

int bsp_f8_fc_grad(const bsp_weights_f8* w, const void* dY, int64_t ldy, const bsp_codes* X, float* dW, float* db,
                   void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_codes(X);
  if (rc != BSP_OK) return rc;
  int64_t need = 0;
  rc = bsp_f8_fc_grad_workspace(w, X->T, &need);
  if (rc != BSP_OK) return rc;
  rc = check_values(dY, BSP_BF16, ldy, X->T, w->O, true);
  if (rc != BSP_OK) return rc;
  if (X->K != w->I || ldy > (1 << 25) || f8_blocks(w->O) * (int64_t)f8_blocks(w->I) > INT32_MAX) return BSP_ERR_SHAPE;
  if (!aligned(dW, 16) || !aligned(db, 16) || !aligned(workspace, 16)) return BSP_ERR_ALIGN;
  if (workspace_bytes < need) return BSP_ERR_CAPACITY;
  if (need > 0 && !workspace) return BSP_ERR_NULL;
  if (!dW && !db) return BSP_OK;
  F8GradArgs a{};
  a.dY = (const uint16_t*)dY, a.ldy = ldy, a.codes = X->codes, a.scale = X->scale, a.row_ptr = w->row_ptr, a.col_idx = w->col_idx;
  a.dW = dW, a.db = db, a.T = X->T, a.O = w->O, a.I = w->I, a.nnzb = w->nnzb;
  a.nbo = f8_blocks(w->O), a.nbi = f8_blocks(w->I), a.e5 = X->dtype == BSP_E5M2, a.split = f8_grad_split(w->nnzb, X->T);
  a.part = (float*)workspace, a.part_db = a.part + (int64_t)a.split * w->nnzb * F8_BLOCK_BYTES;
  return f8_launch_grad(a, (hipStream_t)stream);
}

int bsp_layer_norm(const void* X, int32_t dtype, int64_t ldx, int32_t T, int32_t D, const float* weight, const float* bias,
                   float eps, void* Y, int64_t ldy, const bsp_codes* codes, float* mean, float* rstd, void* stream) {
  int rc = check_values(X, dtype, ldx, T, D, true);
  if (rc != BSP_OK) return rc;
  if (!(eps >= 0.f)) return BSP_ERR_SHAPE;
  if ((Y != nullptr) == (codes != nullptr) && T > 0) return BSP_ERR_NULL;  // one of the two
  if (codes) {
    rc = check_codes(codes);
    if (rc != BSP_OK) return rc;
    if (codes->T != T || codes->K != D) return BSP_ERR_SHAPE;
  } else {
    rc = check_values(Y, dtype, ldy, T, D, false);
    if (rc != BSP_OK) return rc;
  }
  if (T == 0) return BSP_OK;
  if (!mean || !rstd) return BSP_ERR_NULL;
  if (!aligned(mean, 4) || !aligned(rstd, 4) || !aligned(weight, 4) || !aligned(bias, 4)) return BSP_ERR_ALIGN;
  return norm_launch_forward(X, dtype == BSP_F32, ldx, T, D, weight, bias, eps, Y, ldy, codes ? codes->dtype : 0,
                             codes ? codes->codes : nullptr, codes ? codes->scale : nullptr, mean, rstd, (hipStream_t)stream);
}

int bsp_layer_norm_grad_workspace(int32_t T, int32_t D, int64_t* bytes) {
  if (!bytes) return BSP_ERR_NULL;
  if (T < 0 || T > kMost || D < 1 || D > kMost) return BSP_ERR_SHAPE;
  const int64_t parts = norm_parts(T, D);
  *bytes = parts > 1 ? parts * 2 * D * 4 : 0;
  return BSP_OK;
}

int bsp_layer_norm_grad(const void* dY, int64_t ld_dy, const void* X, int64_t ldx, int32_t dtype, int32_t T, int32_t D,
                        const float* mean, const float* rstd, const float* weight, void* dX, int64_t ld_dx,
                        float* dweight, float* dbias, void* workspace, int64_t workspace_bytes, void* stream) {
  int64_t need = 0;
  int rc = bsp_layer_norm_grad_workspace(T, D, &need);
  if (rc != BSP_OK) return rc;
  rc = check_values(dY, dtype, ld_dy, T, D, true);
  if (rc != BSP_OK) return rc;
  rc = check_values(X, dtype, ldx, T, D, true);
  if (rc != BSP_OK) return rc;
  rc = check_values(dX, dtype, ld_dx, T, D, false);
  if (rc != BSP_OK) return rc;
  if (T > 0 && (!mean || !rstd)) return BSP_ERR_NULL;
  if (!aligned(mean, 4) || !aligned(rstd, 4) || !aligned(weight, 4) || !aligned(dweight, 4) || !aligned(dbias, 4) || !aligned(workspace, 16)) return BSP_ERR_ALIGN;
  if (workspace_bytes < need) return BSP_ERR_CAPACITY;
  if (need > 0 && !workspace) return BSP_ERR_NULL;
  return norm_launch_backward(dY, ld_dy, X, ldx, dtype == BSP_F32, mean, rstd, weight, T, D, dX, ld_dx, dweight, dbias, (float*)workspace, (hipStream_t)stream);
}

int bsp_f8_adapters_size(int32_t R, int32_t I, int32_t O, int64_t* a_elements, int64_t* b_elements) {
  if (!a_elements || !b_elements) return BSP_ERR_NULL;
  if (R < 1 || R > kRank || I < 1 || I > kWide || O < 1 || O > kWide) return BSP_ERR_SHAPE;
  bsp_f8_adapters d{};
  d.R = R, d.I = I, d.O = O;
  const F8Adapters v = f8_adapters_of(&d);
  *a_elements = (int64_t)v.Rp * v.Ip, *b_elements = (int64_t)v.Rp * v.Op;
  return BSP_OK;
}

int bsp_f8_adapters_set(const bsp_f8_adapters* d, int32_t slot, int32_t rank, const void* A, int64_t lda, const void* B, int64_t ldb, int32_t dtype,
                        float scale, void* stream) {
  int rc = check_adapters(d);
  if (rc != BSP_OK) return rc;
  if (slot < 0 || slot >= d->N || rank < 0 || rank > d->R) return BSP_ERR_SHAPE;
  if (rank > 0) {
    rc = check_values(A, dtype, lda, rank, d->I, true);
    if (rc == BSP_OK) rc = check_values(B, dtype, ldb, d->O, rank, true);
    if (rc != BSP_OK) return rc;
  } else if (!value_type(dtype)) {
    return BSP_ERR_DTYPE;
  }
  return f8_launch_set(f8_adapters_of(d), slot, rank, A, lda, B, ldb, dtype == BSP_F32, scale, (hipStream_t)stream);
}

int bsp_f8_requests_size(int32_t T, int32_t N, int64_t* bytes) {
  if (!bytes) return BSP_ERR_NULL;
  if (T < 0 || T > kRequests || N < 1 || N > kSlots) return BSP_ERR_SHAPE;
  *bytes = f8_requests_bytes(T, N);
  return BSP_OK;
}

int bsp_f8_requests_plan(const bsp_f8_requests* r, const void* which, int32_t which_bytes, void* stream) {
  const int rc = check_requests(r);
  if (rc != BSP_OK) return rc;
  if (which_bytes != 4 && which_bytes != 8) return BSP_ERR_DTYPE;
  if (r->T == 0 && !r->plan) return BSP_OK;
  if (r->T > 0 && !which) return BSP_ERR_NULL;
  if (!aligned(which, which_bytes)) return BSP_ERR_ALIGN;
  return f8_launch_plan(r, which, which_bytes == 8, (hipStream_t)stream);
}

int bsp_f8_fc_adapted_workspace(const bsp_weights_f8* w, int32_t transposed, int32_t T, int32_t coded, const bsp_f8_adapters* adapters, int64_t* bytes) {
  int rc = bytes ? check_adapters(adapters) : BSP_ERR_NULL;
  if (rc != BSP_OK) return rc;
  const F8Adapters d = f8_adapters_of(adapters);
  rc = bsp_f8_fc_workspace(w, transposed, T, coded && !sorts(d, T), bytes);
  if (rc == BSP_OK) *bytes = in16(*bytes) + low_bytes(d, T, transposed ? w->O : w->I, false);
  return rc;
}

int bsp_f8_fc_adapted(const bsp_weights_f8* w, int32_t transposed, const bsp_codes* X, const void* values, int32_t x_dtype, int64_t ldx, int32_t T,
                      int32_t code, const bsp_f8_adapters* adapters, const bsp_f8_requests* requests, const float* bias, const void* residual,
                      int32_t relu, const bsp_codes* gate, void* Y, int32_t y_dtype, void* workspace, int64_t workspace_bytes, void* stream) {
  F8Epilogue q;
  int rc = check_product(w, transposed, T, bias, residual, relu, gate, Y, y_dtype, &q);
  if (rc == BSP_OK) rc = check_adapters(adapters);
  if (rc == BSP_OK) rc = check_requests(requests);
  if (rc != BSP_OK) return rc;
  const int K = transposed ? w->O : w->I;
  if (T < 0 || requests->T != T || requests->N != adapters->N || adapters->I != w->I || adapters->O != w->O) return BSP_ERR_SHAPE;
  if (X) {
    rc = check_codes(X);
    if (rc != BSP_OK) return rc;
    if (X->T != T || X->K != K) return BSP_ERR_SHAPE;
  } else {
    if (!code_type(code)) return BSP_ERR_DTYPE;
    rc = check_values(values, x_dtype, ldx, T, K, true);
    if (rc != BSP_OK) return rc;
  }
  if (T == 0) return BSP_OK;
  const F8Rows rows = rows_of(w, transposed != 0);
  const F8Adapters d = f8_adapters_of(adapters);
  const int64_t sums = sums_bytes(rows, T), codes = (X && !sorts(d, T)) || (!X && in_kernel(values, x_dtype, ldx, T, K)) ? 0 : codes_bytes(T, K);
  rc = check_workspace(workspace, workspace_bytes, in16(sums + codes) + low_bytes(d, T, K, false));
  if (rc != BSP_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  const F8Requests who = f8_requests_of(requests);
  float* u = (float*)((uint8_t*)workspace + in16(sums + codes));
  const int64_t ld = (int64_t)f8_blocks(K) * F8_BLOCK;
  const F8Input given = X ? F8Input{X->codes, X->scale, X->dtype, X->dtype == BSP_E5M2, ld} : F8Input{values, nullptr, x_dtype, code == BSP_E5M2, ldx};
  // values that the product wants as codes become them where they are read for u, where codes that it wants in another order are copied, too
  uint8_t *to = codes ? (uint8_t*)workspace + sums : nullptr, *to_scale = codes ? to + T * ld : nullptr;
  rc = f8_launch_down(d, transposed != 0, given, T, who, u, to, to_scale, sorts(d, T), st);
  if (rc != BSP_OK) return rc;
  F8Low low{who.which, u, transposed ? d.a_t : d.b, (int64_t)d.Rp * (transposed ? d.Ip : d.Op), (int64_t)T * d.Rp, d.Rp, f8_down_slices(T, d.N, K, false)};
  if (sorts(d, T)) low.mixed = who.tiles + 2, low.order = who.order, low.codes = to, low.scale = to_scale;
  return multiply(rows, !X && codes ? F8Input{to, to_scale, code, code == BSP_E5M2, ld} : given, T, low, q, y_dtype, workspace, st);
}

int bsp_f8_adapters_grad_workspace(const bsp_f8_adapters* adapters, int32_t T, int64_t* bytes) {
  if (!bytes) return BSP_ERR_NULL;
  const int rc = check_adapters(adapters);
  if (rc != BSP_OK) return rc;
  if (T < 0 || T > kRequests) return BSP_ERR_SHAPE;
  const F8Adapters d = f8_adapters_of(adapters);
  *bytes = low_bytes(d, T, d.I, true) + low_bytes(d, T, d.O, true) + f8_adapt_part_bytes(d, T);
  return BSP_OK;
}

int bsp_f8_adapters_grad(const bsp_f8_adapters* adapters, const void* dY, int64_t ldy, const bsp_codes* X, const void* values, int64_t ldx, int32_t T,
                         const bsp_f8_requests* requests, float* dA, float* dB, void* workspace, int64_t workspace_bytes, void* stream) {
  int64_t need = 0;
  int rc = bsp_f8_adapters_grad_workspace(adapters, T, &need);
  if (rc == BSP_OK) rc = check_requests(requests);
  if (rc == BSP_OK) rc = check_values(dY, BSP_BF16, ldy, T, adapters->O, true);
  if (rc != BSP_OK) return rc;
  if (requests->T != T || requests->N != adapters->N) return BSP_ERR_SHAPE;
  if (X) {
    rc = check_codes(X);
    if (rc != BSP_OK) return rc;
    if (X->T != T || X->K != adapters->I) return BSP_ERR_SHAPE;
  } else {
    rc = check_values(values, BSP_BF16, ldx, T, adapters->I, true);
    if (rc != BSP_OK) return rc;
  }
  if (!dA || !dB || !requests->plan) return BSP_ERR_NULL;
  if (!aligned(dA, 4) || !aligned(dB, 4)) return BSP_ERR_ALIGN;
  rc = check_workspace(workspace, workspace_bytes, need);
  if (rc != BSP_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  const F8Adapters d = f8_adapters_of(adapters);
  const F8Requests who = f8_requests_of(requests);
  float *u = (float*)workspace, *v = u + low_bytes(d, T, d.I, true) / 4, *part = v + low_bytes(d, T, d.O, true) / 4;
  const F8Input x = X ? F8Input{X->codes, X->scale, X->dtype, X->dtype == BSP_E5M2, (int64_t)f8_blocks(X->K) * F8_BLOCK} : F8Input{values, nullptr, BSP_BF16, 0, ldx};
  if (T > 0) {
    rc = f8_launch_down_both(d, x, F8Input{dY, nullptr, BSP_BF16, 0, ldy}, T, who, u, v, st);
    if (rc != BSP_OK) return rc;
  }
  return f8_launch_adapt_grad(d, (const uint16_t*)dY, ldy, x, T, who, u, v, part, dA, dB, st);
}

int bsp_rms_norm(const void* X, int64_t ldx, const void* residual, int64_t ldr, int32_t dtype, int32_t T, int32_t D, const float* weight, float eps,
                 void* H, int64_t ldh, void* Y, int64_t ldy, const bsp_codes* codes, float* rstd, void* stream) {
  int rc = check_values(X, dtype, ldx, T, D, true);
  if (rc != BSP_OK) return rc;
  if (!(eps >= 0.f)) return BSP_ERR_SHAPE;
  if (T > 0 && ((Y != nullptr) == (codes != nullptr) || (residual != nullptr) != (H != nullptr))) return BSP_ERR_NULL;
  if (residual) {
    rc = check_values(residual, dtype, ldr, T, D, true);
    if (rc == BSP_OK) rc = check_values(H, dtype, ldh, T, D, false);
    if (rc != BSP_OK) return rc;
  }
  if (codes) {
    rc = check_codes(codes);
    if (rc != BSP_OK) return rc;
    if (codes->T != T || codes->K != D) return BSP_ERR_SHAPE;
  } else {
    rc = check_values(Y, dtype, ldy, T, D, false);
    if (rc != BSP_OK) return rc;
  }
  if (T == 0) return BSP_OK;
  if (!rstd) return BSP_ERR_NULL;
  if (!aligned(rstd, 4) || !aligned(weight, 4)) return BSP_ERR_ALIGN;
  return rms_launch_forward(X, ldx, residual, ldr, dtype == BSP_F32, T, D, weight, eps, H, ldh, Y, ldy, codes ? codes->dtype : 0,
                            codes ? codes->codes : nullptr, codes ? codes->scale : nullptr, rstd, (hipStream_t)stream);
}

int bsp_rms_norm_grad_workspace(int32_t T, int32_t D, int64_t* bytes) {
  if (!bytes) return BSP_ERR_NULL;
  if (T < 0 || T > kMost || D < 1 || D > kMost) return BSP_ERR_SHAPE;
  const int64_t parts = rms_parts(T, D);
  *bytes = parts > 1 ? parts * D * 4 : 0;
  return BSP_OK;
}

int bsp_rms_norm_grad(const void* dY, int64_t ld_dy, const void* H, int64_t ldh, const void* dH, int64_t ld_dh, int32_t dtype, int32_t T, int32_t D,
                      const float* rstd, const float* weight, void* dX, int64_t ld_dx, float* dweight, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  int64_t need = 0;
  int rc = bsp_rms_norm_grad_workspace(T, D, &need);
  if (rc == BSP_OK) rc = check_values(dY, dtype, ld_dy, T, D, true);
  if (rc == BSP_OK) rc = check_values(H, dtype, ldh, T, D, true);
  if (rc == BSP_OK && dH) rc = check_values(dH, dtype, ld_dh, T, D, true);
  if (rc == BSP_OK) rc = check_values(dX, dtype, ld_dx, T, D, false);
  if (rc != BSP_OK) return rc;
  if (T > 0 && !rstd) return BSP_ERR_NULL;
  if (!aligned(rstd, 4) || !aligned(weight, 4) || !aligned(dweight, 4)) return BSP_ERR_ALIGN;
  rc = check_workspace(workspace, workspace_bytes, need);
  if (rc != BSP_OK) return rc;
  return rms_launch_backward(dY, ld_dy, H, ldh, dH, ld_dh, dtype == BSP_F32, rstd, weight, T, D, dX, ld_dx, dweight, (float*)workspace, (hipStream_t)stream);
}

int bsp_log_probs_workspace(int32_t T, int32_t V, int32_t top, int64_t* bytes) {
  if (!bytes) return BSP_ERR_NULL;
  if (T < 0 || T > kMost || V < 1 || V > kVocabulary || top < 0 || top > kTop || top > V) return BSP_ERR_SHAPE;
  *bytes = T > 0 ? logp_workspace(T, V, top) : 0;
  return BSP_OK;
}

int bsp_log_probs(const void* X, int64_t ldx, int32_t dtype, int32_t T, int32_t V, const void* tokens, int32_t token_bytes, float scale, int32_t top,
                  float* logp, float* lse, float* entropy, float* top_logp, int32_t* top_tokens, void* workspace, int64_t workspace_bytes, void* stream) {
  int64_t need = 0;
  int rc = bsp_log_probs_workspace(T, V, top, &need);
  if (rc == BSP_OK) rc = check_values(X, dtype, ldx, T, V, true);
  if (rc != BSP_OK) return rc;
  if (token_bytes != 4 && token_bytes != 8) return BSP_ERR_DTYPE;
  if (!(scale > 0.f) || scale > kSharpest) return BSP_ERR_SHAPE;
  if (T == 0) return BSP_OK;
  if (!tokens || !logp || !lse || !entropy || (top && (!top_logp || !top_tokens))) return BSP_ERR_NULL;
  if (!aligned(tokens, token_bytes) || !aligned(logp, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(top_logp, 4) || !aligned(top_tokens, 4)) return BSP_ERR_ALIGN;
  rc = check_workspace(workspace, workspace_bytes, need);
  if (rc != BSP_OK) return rc;
  return logp_launch(X, dtype == BSP_F32, ldx, T, V, tokens, token_bytes == 8, scale, top, logp, lse, entropy, top_logp, top_tokens, workspace, (hipStream_t)stream);
}

int bsp_log_probs_grad(const void* X, int64_t ldx, int32_t dtype, int32_t T, int32_t V, const void* tokens, int32_t token_bytes, float scale,
                       const float* lse, const float* entropy, const float* dlogp, const float* dentropy, void* dX, int64_t ld_dx, void* stream) {
  int64_t none = 0;
  int rc = bsp_log_probs_workspace(T, V, 0, &none);
  if (rc == BSP_OK) rc = check_values(X, dtype, ldx, T, V, true);
  if (rc == BSP_OK) rc = check_values(dX, dtype, ld_dx, T, V, false);
  if (rc != BSP_OK) return rc;
  if (token_bytes != 4 && token_bytes != 8) return BSP_ERR_DTYPE;
  if (!(scale > 0.f) || scale > kSharpest) return BSP_ERR_SHAPE;
  if (T == 0) return BSP_OK;
  if (!tokens || !lse || !entropy) return BSP_ERR_NULL;
  if (!aligned(tokens, token_bytes) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(dlogp, 4) || !aligned(dentropy, 4)) return BSP_ERR_ALIGN;
  if (X == dX && ldx != ld_dx && T > 1) return BSP_ERR_SHAPE;  // in place row for row
  return logp_launch_grad(X, dtype == BSP_F32, ldx, T, V, tokens, token_bytes == 8, scale, lse, entropy, dlogp, dentropy, dX, ld_dx, (hipStream_t)stream);
}

int bsp_f8_call_packed(int32_t call, const int64_t* w) {
  if (!w) return BSP_ERR_NULL;
  auto ptr = [&](int i) { return (void*)(intptr_t)w[i]; };
  auto num = [&](int i) { return w[i] == (int32_t)w[i] ? (int32_t)w[i] : -1; };  // (no type has that number)
  // sizes that do not fit 32 bits are as wrong as negative ones
  auto size = [&](int i) { return w[i] < 0 || w[i] > INT32_MAX ? -1 : (int32_t)w[i]; };
  auto codes = [&](int i) { return bsp_codes{size(i), size(i + 1), num(i + 2), (uint8_t*)ptr(i + 3), (uint8_t*)ptr(i + 4)}; };
  auto none = [&](int i) { return !(w[i] | w[i + 1] | w[i + 2] | w[i + 3] | w[i + 4]); };
  auto real = [&](int i) {
    double v;
    memcpy(&v, &w[i], sizeof v);
    return v;
  };
  switch (call) {
    case BSP_F8_CALL_SAVE: {
      const bsp_codes c = codes(3);
      return bsp_f8_save(ptr(0), num(1), w[2], &c, ptr(8));
    }
    case BSP_F8_CALL_LOAD: {
      const bsp_codes c = codes(0);
      return bsp_f8_load(&c, ptr(5), num(6), w[7], ptr(8));
    }
    case BSP_F8_CALL_FC: {
      const bsp_codes x = codes(2), g = codes(10);
      return bsp_f8_fc((const bsp_weights_f8*)ptr(0), num(1), &x, (const float*)ptr(7), ptr(8), num(9), none(10) ? nullptr : &g, ptr(15), num(16), ptr(17), w[18], ptr(19));
    }
    case BSP_F8_CALL_VALUES: {
      const bsp_codes g = codes(10);
      return bsp_f8_fc_values((const bsp_weights_f8*)ptr(0), num(1), ptr(2), num(3), w[4], size(5), num(6), (const float*)ptr(7), ptr(8), num(9),
                              none(10) ? nullptr : &g, ptr(15), num(16), ptr(17), w[18], ptr(19));
    }
    case BSP_F8_CALL_GRAD: {
      const bsp_codes x = codes(3);
      return bsp_f8_fc_grad((const bsp_weights_f8*)ptr(0), ptr(1), w[2], &x, (float*)ptr(8), (float*)ptr(9), ptr(10), w[11], ptr(12));
    }
    case BSP_F8_CALL_NORM: {
      const bsp_codes c = codes(10);
      return bsp_layer_norm(ptr(0), num(1), w[2], size(3), size(4), (const float*)ptr(5), (const float*)ptr(6), (float)real(7), ptr(8), w[9],
                            none(10) ? nullptr : &c, (float*)ptr(15), (float*)ptr(16), ptr(17));
    }
    case BSP_F8_CALL_NORM_GRAD:
      return bsp_layer_norm_grad(ptr(0), w[1], ptr(2), w[3], num(4), size(5), size(6), (const float*)ptr(7), (const float*)ptr(8), (const float*)ptr(9),
                                 ptr(10), w[11], (float*)ptr(12), (float*)ptr(13), ptr(14), w[15], ptr(16));
    case BSP_F8_CALL_ADAPTED: {
      const bsp_codes x = codes(2), g = codes(17);
      return bsp_f8_fc_adapted((const bsp_weights_f8*)ptr(0), num(1), none(2) ? nullptr : &x, ptr(7), num(8), w[9], size(10), num(11),
                               (const bsp_f8_adapters*)ptr(12), (const bsp_f8_requests*)ptr(13), (const float*)ptr(14), ptr(15), num(16),
                               none(17) ? nullptr : &g, ptr(22), num(23), ptr(24), w[25], ptr(26));
    }
    case BSP_F8_CALL_ADAPTERS_GRAD: {
      const bsp_codes x = codes(3);
      return bsp_f8_adapters_grad((const bsp_f8_adapters*)ptr(0), ptr(1), w[2], none(3) ? nullptr : &x, ptr(8), w[9], size(10), (const bsp_f8_requests*)ptr(11),
                                  (float*)ptr(12), (float*)ptr(13), ptr(14), w[15], ptr(16));
    }
    case BSP_F8_CALL_RMS_NORM: {
      const bsp_codes c = codes(13);
      return bsp_rms_norm(ptr(0), w[1], ptr(2), w[3], num(4), size(5), size(6), (const float*)ptr(7), (float)real(8), ptr(9), w[10], ptr(11), w[12],
                          none(13) ? nullptr : &c, (float*)ptr(18), ptr(19));
    }
    case BSP_F8_CALL_RMS_NORM_GRAD:
      return bsp_rms_norm_grad(ptr(0), w[1], ptr(2), w[3], ptr(4), w[5], num(6), size(7), size(8), (const float*)ptr(9), (const float*)ptr(10), ptr(11), w[12],
                               (float*)ptr(13), ptr(14), w[15], ptr(16));
    case BSP_F8_CALL_LOG_PROBS:
      return bsp_log_probs(ptr(0), w[1], num(2), size(3), size(4), ptr(5), num(6), (float)real(7), num(8), (float*)ptr(9), (float*)ptr(10), (float*)ptr(11),
                           (float*)ptr(12), (int32_t*)ptr(13), ptr(14), w[15], ptr(16));
    case BSP_F8_CALL_LOG_PROBS_GRAD:
      return bsp_log_probs_grad(ptr(0), w[1], num(2), size(3), size(4), ptr(5), num(6), (float)real(7), (const float*)ptr(8), (const float*)ptr(9),
                                (const float*)ptr(10), (const float*)ptr(11), ptr(12), w[13], ptr(14));
  }
  return BSP_ERR_SHAPE;
}

}  // extern "C"
