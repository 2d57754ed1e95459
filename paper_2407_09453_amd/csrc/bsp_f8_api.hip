// extern "C" entry points of the 8-bit floating-point layers and of layer norm: argument checks and dispatch.
#include "bsp_f8.h"

#include <string.h>

namespace {

inline bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool value_type(int d) { return d == BSP_F32 || d == BSP_BF16; }
inline bool code_type(int d) { return d == BSP_E4M3 || d == BSP_E5M2; }
inline unsigned size_of(int d) { return d == BSP_F32 ? 4 : 2; }
constexpr int32_t kMost = INT32_MAX - 65536;  // rows and columns: sizes rounded up stay in 32 bits
constexpr int32_t kWide = 1 << 24;            // columns of codes: 256 rows' offsets stay in 32 bits

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

int multiply(const F8Rows& rows, const F8Input& x, int T, const F8Epilogue& q, int32_t y_dtype, void* sums, hipStream_t st) {
  const bool f32 = y_dtype == BSP_F32;
  const int rc = T <= kFewRows ? f8_launch_few(rows, x, T, q, f32, (float*)sums, st) : f8_launch_tile(rows, x, T, q, f32, (float*)sums, st);
  if (rc != BSP_OK) return rc;
  const int split = split_of(rows, T, f32);
  return split > 1 ? f8_launch_join((const float*)sums, split, T, rows.out, q, f32, st) : BSP_OK;
}

int check_workspace(const void* workspace, int64_t bytes, int64_t need) {
  if (bytes < need) return BSP_ERR_CAPACITY;
  if (need > 0 && !workspace) return BSP_ERR_NULL;
  return aligned(workspace, 16) ? BSP_OK : BSP_ERR_ALIGN;
}

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
  return rc != BSP_OK ? rc : multiply(rows, x, X->T, q, y_dtype, workspace, (hipStream_t)stream);
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
  const bool inside = in_kernel(X, x_dtype, ldx, T, K);
  rc = check_workspace(workspace, workspace_bytes, sums + (inside ? 0 : codes_bytes(T, K)));
  if (rc != BSP_OK) return rc;
  if (inside) return multiply(rows, F8Input{X, nullptr, x_dtype, e5, ldx}, T, q, y_dtype, workspace, st);
  const int64_t ld = (int64_t)f8_blocks(K) * F8_BLOCK;
  uint8_t *codes = (uint8_t*)workspace + sums, *scale = codes + T * ld;
  rc = f8_launch_save(X, x_dtype == BSP_F32, ldx, T, K, e5, codes, scale, st);
  if (rc != BSP_OK) return rc;
  return multiply(rows, F8Input{codes, scale, code, e5, ld}, T, q, y_dtype, workspace, st);
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

int bsp_f8_call_packed(int32_t call, const int64_t* w) {
  if (!w) return BSP_ERR_NULL;
  auto ptr = [&](int i) { return (void*)(intptr_t)w[i]; };
  auto num = [&](int i) { return w[i] == (int32_t)w[i] ? (int32_t)w[i] : -1; };  // (no type has that number)
  // sizes that do not fit 32 bits are as wrong as negative ones
  auto size = [&](int i) { return w[i] < 0 || w[i] > INT32_MAX ? -1 : (int32_t)w[i]; };
  auto codes = [&](int i) { return bsp_codes{size(i), size(i + 1), num(i + 2), (uint8_t*)ptr(i + 3), (uint8_t*)ptr(i + 4)}; };
  auto none = [&](int i) { return !(w[i] | w[i + 1] | w[i + 2] | w[i + 3] | w[i + 4]); };
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
      double eps;
      memcpy(&eps, &w[7], sizeof eps);
      return bsp_layer_norm(ptr(0), num(1), w[2], size(3), size(4), (const float*)ptr(5), (const float*)ptr(6), (float)eps, ptr(8), w[9],
                            none(10) ? nullptr : &c, (float*)ptr(15), (float*)ptr(16), ptr(17));
    }
    case BSP_F8_CALL_NORM_GRAD:
      return bsp_layer_norm_grad(ptr(0), w[1], ptr(2), w[3], num(4), size(5), size(6), (const float*)ptr(7), (const float*)ptr(8), (const float*)ptr(9),
                                 ptr(10), w[11], (float*)ptr(12), (float*)ptr(13), ptr(14), w[15], ptr(16));
  }
  return BSP_ERR_SHAPE;
}

}  // extern "C"
