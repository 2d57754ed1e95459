// Host side of the 8-bit floating-point layers: index arrays of a mask over 128x128 blocks, by rows and by columns.
#include "bsp.h"

namespace {

int64_t blocks(int32_t n) { return ((int64_t)n + 127) / 128; }

int count(const uint8_t* gamma, int32_t O, int32_t I, int64_t* nnzb) {
  if (!gamma || !nnzb) return BSP_ERR_NULL;
  if (O < 1 || I < 1 || blocks(O) * blocks(I) > INT32_MAX) return BSP_ERR_SHAPE;
  int64_t n = 0;
  for (int64_t b = 0; b < blocks(O) * blocks(I); ++b) {
    if (gamma[b] > 1) return BSP_ERR_MASK;
    n += gamma[b];
  }
  *nnzb = n;
  return BSP_OK;
}

}  // namespace

extern "C" {

int bsp_f8_count(const uint8_t* gamma, int32_t O, int32_t I, int64_t* nnzb) { return count(gamma, O, I, nnzb); }

int bsp_f8_index(const uint8_t* gamma, int32_t O, int32_t I, int64_t capacity,
                 int32_t* row_ptr, int32_t* col_idx, int32_t* col_ptr, int32_t* row_idx) {
  int64_t nnzb = 0;
  const int rc = count(gamma, O, I, &nnzb);
  if (rc != BSP_OK) return rc;
  if (!row_ptr || !col_ptr || (nnzb > 0 && (!col_idx || !row_idx))) return BSP_ERR_NULL;
  if (capacity < nnzb) return BSP_ERR_CAPACITY;
  const int64_t R = blocks(O), C = blocks(I);
  int32_t n = 0;
  for (int64_t r = 0; r < R; ++r) {
    row_ptr[r] = n;
    for (int64_t c = 0; c < C; ++c)
      if (gamma[r * C + c]) col_idx[n++] = (int32_t)c;
  }
  row_ptr[R] = n;
  n = 0;
  for (int64_t c = 0; c < C; ++c) {
    col_ptr[c] = n;
    for (int64_t r = 0; r < R; ++r)
      if (gamma[r * C + c]) row_idx[n++] = (int32_t)r;
  }
  col_ptr[C] = n;
  return BSP_OK;
}

}  // extern "C"
