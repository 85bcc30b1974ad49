// C ABI of the microscaled 4-bit format and of distillation: argument checking and dispatch.
#include <cmath>

#include "common.h"

namespace lcd {

namespace {

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool known(lcd_dtype t) { return t == LCD_DTYPE_F32 || t == LCD_DTYPE_F16 || t == LCD_DTYPE_BF16; }
size_t size_of(lcd_dtype t) { return t == LCD_DTYPE_F32 ? 4 : 2; }
constexpr int64_t kMostRows = 0x7fffffffLL, kMostColumns = 1LL << 30;
int64_t blocks_of(int64_t K) { return (K + 31) / 32; }
int64_t on_16(int64_t v) { return (v + 15) / 16 * 16; }
// Bytes of a row of codes in a workspace.  Long rows begin on cache lines, which the product's copies of 128 bytes would straddle
// otherwise (333 x 5003 x 5001 16.6 us, 15.0 so; 2048 x 5120 x 5024 41.9 and 37.7); for short ones that would be much more memory.
int64_t code_row(int64_t K) {
  const int64_t bytes = 16 * blocks_of(K);
  return bytes < 512 ? bytes : (bytes + 127) / 128 * 128;
}

// Rows of codes and scales of a matrix with K columns.
bool mx_rows(const void* codes, int64_t ldc, const void* scales, int64_t lds, int64_t rows, int64_t K) {
  return codes && scales && rows >= 1 && rows <= kMostRows && K >= 1 && K <= kMostColumns && aligned(codes, 16) && aligned(scales, 16) &&
         ldc % 16 == 0 && lds % 16 == 0 && ldc >= 16 * blocks_of(K) && lds >= blocks_of(K);
}
bool dense_rows(const void* p, lcd_dtype t, int64_t rows, int64_t columns, int64_t ld) {
  return p && known(t) && rows >= 1 && rows <= kMostRows && columns >= 1 && columns <= kMostColumns && ld >= columns && aligned(p, size_of(t));
}

lcd_status distillation(const Distillation& d) {
  if (!dense_rows(d.logits, d.type, d.T, d.V, d.ldz) || !d.teacher_idx || !known(d.teacher_type) || d.k < 1) return LCD_ERR_INVALID_ARG;
  if (!dense_rows(d.teacher_logits, d.teacher_type, d.T, d.k, d.ldt) || d.ldi < d.k) return LCD_ERR_INVALID_ARG;
  if ((d.idx_bytes != 4 && d.idx_bytes != 8) || !aligned(d.teacher_idx, (size_t)d.idx_bytes)) return LCD_ERR_INVALID_ARG;
  if (!(d.temperature > 0.0f) || !std::isfinite(d.temperature) || !std::isfinite(1.5f / d.temperature)) return LCD_ERR_INVALID_ARG;
  if (!aligned(d.teacher_lse, 4) || !aligned(d.weight, 4) || !aligned(d.loss, 4) || !aligned(d.stats, 4)) return LCD_ERR_INVALID_ARG;
  if (d.dlogits && !dense_rows(d.dlogits, d.type, d.T, d.V, d.ldd)) return LCD_ERR_INVALID_ARG;
  if (d.dlogits == d.logits && d.ldd != d.ldz && d.T > 1) return LCD_ERR_INVALID_ARG;
  if (d.k > 1024) return LCD_ERR_UNSUPPORTED;
  return LCD_OK;
}

}  // namespace

}  // namespace lcd

using namespace lcd;

extern "C" lcd_status lcd_mx_quantize(const void* x, lcd_dtype x_type, int64_t M, int64_t K, int64_t ldx, const float* inv_smooth,
                                      uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds, void* cuda_stream) {
  if (!dense_rows(x, x_type, M, K, ldx) || !mx_rows(codes, ldc, scales, lds, M, K) || !aligned(inv_smooth, 4)) return LCD_ERR_INVALID_ARG;
  return launch_mx_quantize(x, x_type, M, K, ldx, inv_smooth, codes, ldc, scales, lds, cuda_stream);
}

extern "C" lcd_status lcd_mx_dequantize(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int64_t M, int64_t K,
                                        void* out, lcd_dtype out_type, int64_t ldo, void* cuda_stream) {
  if (!dense_rows(out, out_type, M, K, ldo) || !mx_rows(codes, ldc, scales, lds, M, K)) return LCD_ERR_INVALID_ARG;
  return launch_mx_dequantize(codes, ldc, scales, lds, M, K, out, out_type, ldo, cuda_stream);
}

extern "C" lcd_status lcd_mx_linear(const uint8_t* w_codes, int64_t ldwc, const uint8_t* w_scales, int64_t ldws, int64_t N, int64_t K,
                                    const uint8_t* x_codes, int64_t ldxc, const uint8_t* x_scales, int64_t ldxs, int64_t M, void* y,
                                    lcd_dtype y_type, int64_t ldy, int32_t* status_word_dev, void* cuda_stream) {
  if (!mx_rows(w_codes, ldwc, w_scales, ldws, N, K) || !mx_rows(x_codes, ldxc, x_scales, ldxs, M, K) ||
      !dense_rows(y, y_type, M, N, ldy) || !aligned(status_word_dev, 4))
    return LCD_ERR_INVALID_ARG;
  return launch_mx_linear({w_codes, w_scales, x_codes, x_scales, ldwc, ldws, ldxc, ldxs, N, K, M, y, y_type, ldy}, false,
                          status_word_dev, cuda_stream);
}

extern "C" lcd_status lcd_mx_linear_fused_workspace_bytes(int64_t M, int64_t K, size_t* bytes) {
  if (!bytes || M < 1 || M > kMostRows || K < 1 || K > kMostColumns) return LCD_ERR_INVALID_ARG;
  *bytes = mx_linear_quantizes(M, K) ? 0 : (size_t)M * (size_t)(code_row(K) + on_16(blocks_of(K)));
  return LCD_OK;
}

extern "C" lcd_status lcd_mx_linear_fused(const uint8_t* w_codes, int64_t ldwc, const uint8_t* w_scales, int64_t ldws, int64_t N,
                                          int64_t K, const void* x, lcd_dtype x_type, int64_t ldx, const float* inv_smooth, int64_t M,
                                          void* y, lcd_dtype y_type, int64_t ldy, void* workspace, size_t workspace_bytes,
                                          int32_t* status_word_dev, void* cuda_stream) {
  size_t need = 0;
  if (!mx_rows(w_codes, ldwc, w_scales, ldws, N, K) || !dense_rows(x, x_type, M, K, ldx) || !dense_rows(y, y_type, M, N, ldy) ||
      !aligned(inv_smooth, 4) || !aligned(workspace, 16) || !aligned(status_word_dev, 4) ||
      lcd_mx_linear_fused_workspace_bytes(M, K, &need) != LCD_OK)
    return LCD_ERR_INVALID_ARG;
  if (need > 0 && (!workspace || workspace_bytes < need)) return LCD_ERR_BUFFER_TOO_SMALL;
  if (mx_linear_quantizes(M, K))
    return launch_mx_linear({w_codes, w_scales, nullptr, nullptr, ldwc, ldws, 0, 0, N, K, M, y, y_type, ldy, x, x_type, ldx, inv_smooth},
                            false, status_word_dev, cuda_stream);
  const int64_t ldc = code_row(K), lds = on_16(blocks_of(K));
  uint8_t* codes = static_cast<uint8_t*>(workspace);
  uint8_t* scales = codes + M * ldc;
  const lcd_status st = launch_mx_quantize(x, x_type, M, K, ldx, inv_smooth, codes, ldc, scales, lds, cuda_stream);
  if (st != LCD_OK) return st;
  return launch_mx_linear({w_codes, w_scales, codes, scales, ldwc, ldws, ldc, lds, N, K, M, y, y_type, ldy}, true, status_word_dev,
                          cuda_stream);
}

extern "C" lcd_status lcd_distill_loss(const void* logits, lcd_dtype type, int64_t T, int64_t V, int64_t ldz, const void* teacher_idx,
                                       int idx_bytes, int64_t ldi, const void* teacher_logits, lcd_dtype teacher_type, int64_t ldt,
                                       int64_t k, float temperature, const float* teacher_lse, const float* weight, float* loss,
                                       float* stats, void* dlogits, int64_t ldd, void* cuda_stream) {
  const Distillation d = {logits, type, T, V, ldz, teacher_idx, idx_bytes, ldi, teacher_logits, teacher_type, ldt, k, temperature,
                          teacher_lse, weight, loss, stats, dlogits, ldd};
  if (!loss) return LCD_ERR_INVALID_ARG;
  const lcd_status st = distillation(d);
  return st == LCD_OK ? launch_distill(d, cuda_stream) : st;
}

extern "C" lcd_status lcd_distill_grad(const void* logits, lcd_dtype type, int64_t T, int64_t V, int64_t ldz, const void* teacher_idx,
                                       int idx_bytes, int64_t ldi, const void* teacher_logits, lcd_dtype teacher_type, int64_t ldt,
                                       int64_t k, float temperature, const float* teacher_lse, const float* weight, const float* stats,
                                       void* dlogits, int64_t ldd, void* cuda_stream) {
  const Distillation d = {logits, type, T, V, ldz, teacher_idx, idx_bytes, ldi, teacher_logits, teacher_type, ldt, k, temperature,
                          teacher_lse, weight, nullptr, const_cast<float*>(stats), dlogits, ldd};
  if (!stats || !dlogits) return LCD_ERR_INVALID_ARG;
  const lcd_status st = distillation(d);
  return st == LCD_OK ? launch_distill(d, cuda_stream) : st;
}
