// C ABI of the calls on batches whose rows go to different weights: argument checking and dispatch.
#include "adapters_down.cuh"
#include "adapters_launch.h"
#include "common.h"

namespace lcd {

namespace {

constexpr int64_t kMostCount = 1LL << 30, kMostColumns = 1LL << 30, kMostRows = 0x7fffffffLL;

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool known(lcd_dtype t) { return t == LCD_DTYPE_F32 || t == LCD_DTYPE_F16 || t == LCD_DTYPE_BF16; }
size_t size_of(lcd_dtype t) { return t == LCD_DTYPE_F32 ? 4 : 2; }
int64_t blocks_of(int64_t K) { return (K + 31) / 32; }
int64_t on(int64_t v, int64_t step) { return (v + step - 1) / step * step; }
// Rows of codes in the workspace begin on cache lines where they are long, as lcd_mx_linear_fused's do.
int64_t code_row(int64_t K) { return 16 * blocks_of(K) < 512 ? 16 * blocks_of(K) : on(16 * blocks_of(K), 128); }

bool counted(int64_t count) { return count >= 1 && count <= kMostCount; }
bool planned(const lcd_row_groups* rows) {
  return rows && rows->order && rows->groups && rows->offsets && aligned(rows->order, 4) && aligned(rows->groups, 4) && aligned(rows->offsets, 4) &&
         counted(rows->count);
}
bool dense_rows(const void* p, lcd_dtype t, int64_t columns, int64_t ld) {
  return p && known(t) && columns >= 1 && columns <= kMostColumns && ld >= columns && aligned(p, size_t(size_of(t)));
}
bool experts_matrix(const void* p, int64_t ld, int64_t row, int64_t distance, int64_t rows, int64_t G) {
  return p && aligned(p, 16) && ld % 16 == 0 && ld >= row && (G == 1 || (distance % 16 == 0 && distance >= (rows - 1) * ld + row));
}

int64_t padded_rank(int64_t r) { return 16 * rank_tiles(r); }

// The adapters' shapes; types are looked at by types_go.
bool adapters_there(const lcd_adapter_weights* w) {
  if (!w || w->G < 1 || w->rank < 1 || !known(w->type)) return false;
  if (!dense_rows(w->a, w->type, w->K, w->lda) || !dense_rows(w->b, w->type, w->rank, w->ldb)) return false;
  if (w->N < 1 || w->N > kMostColumns || !aligned(w->scale, 4)) return false;
  return w->G == 1 || (w->adapter_a >= (w->rank - 1) * w->lda + w->K && w->adapter_b >= (w->N - 1) * w->ldb + w->rank);
}
bool types_go(lcd_dtype x, lcd_dtype w) { return x == w || x == LCD_DTYPE_F32 || w == LCD_DTYPE_F32; }

AdapterArgs args_of(const lcd_adapter_weights& w, const lcd_row_groups& rows, bool second) {
  AdapterArgs a = {};
  a.order = rows.order;
  a.groups = rows.groups;
  a.offsets = rows.offsets;
  a.rows = (int)rows.count;
  a.G = (int)w.G;
  a.r = (int)w.rank;
  a.K = second ? w.N : w.K;
  a.w = second ? w.b : w.a;
  a.ldw = second ? w.ldb : w.lda;
  a.sw = w.G == 1 ? 0 : second ? w.adapter_b : w.adapter_a;
  return a;
}
lcd_status down(const DownArgs& d, lcd_dtype x_type, lcd_dtype w_type, bool backward, void* stream) {
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (adapters_down_tc_takes(d, x_type, w_type)) return launch_adapters_down_tc(d, x_type, backward, s);
  if (adapters_down_parts_takes(d, x_type, w_type)) return launch_adapters_down_parts(d, x_type, w_type, backward, s);
  switch (x_type) {
    case LCD_DTYPE_F32: return launch_adapters_down_f32(d, w_type, backward, s);
    case LCD_DTYPE_F16: return launch_adapters_down_f16(d, w_type, backward, s);
    default: return launch_adapters_down_bf16(d, w_type, backward, s);
  }
}

lcd_status up(const UpArgs& u, lcd_dtype w_type, lcd_dtype y_type, bool transposed, void* stream) {
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool tc = u.t_parts != nullptr;
  switch (w_type) {
    case LCD_DTYPE_F32: return tc ? launch_adapters_up_tc_f32(u, y_type, transposed, s) : launch_adapters_up_f32(u, y_type, transposed, s);
    case LCD_DTYPE_F16: return tc ? launch_adapters_up_tc_f16(u, y_type, transposed, s) : launch_adapters_up_f16(u, y_type, transposed, s);
    default: return tc ? launch_adapters_up_tc_bf16(u, y_type, transposed, s) : launch_adapters_up_bf16(u, y_type, transposed, s);
  }
}
// Whether the products for many rows run, which take t in bf16 parts.
bool takes_parts_of_t(const UpArgs& u, lcd_dtype w_type, lcd_dtype y_type) {
  if (u.a.rows < kManyRows || ((int64_t)u.a.rows / 128 + u.a.G + 1) * ((u.a.K + 63) / 64) > 0x7fffffff) return false;
  if (u.a.r > 64 && (w_type != LCD_DTYPE_BF16 || y_type == LCD_DTYPE_F32)) return false;      // the parts do not fit into shared memory
  const int64_t size = size_of(y_type);
  return u.a.rows >= 2 * kManyRows || (on_bytes(u.y, u.ldy, u.a.K, size, 16) && on_bytes(u.base, u.ldbase, u.a.K, size, 16));
}

}  // namespace

}  // namespace lcd

using namespace lcd;

extern "C" lcd_status lcd_group_rows(const void* group, int idx_bytes, int64_t count, int64_t G, int32_t* order, int32_t* groups, int32_t* offsets,
                                     void* cuda_stream) {
  if (!group || (idx_bytes != 4 && idx_bytes != 8) || !aligned(group, (size_t)idx_bytes) || !counted(count) || G < 1 || !order || !groups || !offsets ||
      !aligned(order, 4) || !aligned(groups, 4) || !aligned(offsets, 4))
    return LCD_ERR_INVALID_ARG;
  return launch_group_rows(group, idx_bytes, count, G, order, groups, offsets, cuda_stream);
}

extern "C" lcd_status lcd_mx_linear_grouped_workspace_bytes(int64_t count, int64_t K, size_t* bytes) {
  if (!bytes || !counted(count) || K < 1 || K > kMostColumns) return LCD_ERR_INVALID_ARG;
  *bytes = (size_t)count * (size_t)(code_row(K) + on(blocks_of(K), 16) + 4);       // codes, scales and where they are
  return LCD_OK;
}

extern "C" lcd_status lcd_mx_linear_grouped_resolve(int64_t count, int64_t G, int64_t N, int64_t K, int* tile_tokens, int* split, int* paired) {
  if (!counted(count) || G < 1 || N < 1 || N > kMostColumns || K < 1 || K > kMostColumns || !tile_tokens || !split || !paired) return LCD_ERR_INVALID_ARG;
  if (G > kMostExperts) return LCD_ERR_UNSUPPORTED;
  const MxGroupedShape s = mx_grouped_shape(count, G, N, K);
  *tile_tokens = s.width;
  *split = s.split;
  *paired = s.pair;
  return LCD_OK;
}

extern "C" lcd_status lcd_mx_linear_grouped(const uint8_t* w_codes, int64_t ldwc, int64_t expert_codes, const uint8_t* w_scales, int64_t ldws,
                                            int64_t expert_scales, int64_t G, int64_t N, int64_t K, const void* x, lcd_dtype x_type, int64_t T,
                                            int64_t ldx, const float* inv_smooth, const lcd_row_groups* rows, void* y, lcd_dtype y_type,
                                            int64_t ldy, void* workspace, size_t workspace_bytes, int32_t* status_word_dev, void* cuda_stream) {
  size_t need = 0;
  if (!planned(rows) || G < 1 || N < 1 || N > kMostRows || K < 1 || K > kMostColumns || T < 1 || rows->count % T != 0 ||
      !experts_matrix(w_codes, ldwc, 16 * blocks_of(K), expert_codes, N, G) || !experts_matrix(w_scales, ldws, blocks_of(K), expert_scales, N, G) ||
      !dense_rows(x, x_type, K, ldx) || !dense_rows(y, y_type, N, ldy) || !aligned(inv_smooth, 4) || !aligned(workspace, 16) ||
      !aligned(status_word_dev, 4) || lcd_mx_linear_grouped_workspace_bytes(rows->count, K, &need) != LCD_OK)
    return LCD_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < need) return LCD_ERR_BUFFER_TOO_SMALL;
  if (G > kMostExperts) return LCD_ERR_UNSUPPORTED;
  const int64_t ldc = code_row(K), lds = on(blocks_of(K), 16);
  uint8_t* codes = static_cast<uint8_t*>(workspace);
  uint8_t* scales = codes + rows->count * ldc;
  const lcd_status st = launch_mx_quantize_rows(x, x_type, T, K, ldx, inv_smooth, *rows, G, codes, ldc, scales, lds,
                                                reinterpret_cast<int32_t*>(scales + rows->count * lds), cuda_stream);
  if (st != LCD_OK) return st;
  // one expert needs no distance, but the copies' description does
  const int64_t dwc = G == 1 ? N * ldwc : expert_codes, dws = G == 1 ? N * ldws : expert_scales;
  return launch_mx_grouped({w_codes, w_scales, codes, scales, ldwc, dwc, ldws, dws, ldc, lds, G, N, K, *rows, y, y_type, ldy}, status_word_dev,
                           cuda_stream);
}

extern "C" lcd_status lcd_adapters_workspace_bytes(int64_t count, int64_t rank, size_t* bytes) {
  if (!bytes || !counted(count) || rank < 1) return LCD_ERR_INVALID_ARG;
  if (rank > kMostRank) return LCD_ERR_UNSUPPORTED;
  // t or dt, and for many rows its bf16 parts
  *bytes = (size_t)count * (size_t)padded_rank(rank) * (count >= kManyRows ? 10 : 4);
  return LCD_OK;
}

extern "C" lcd_status lcd_adapters(const lcd_adapter_weights* weights, const void* x, lcd_dtype x_type, int64_t ldx, const lcd_row_groups* rows,
                                   const void* base, int64_t ldbase, void* y, lcd_dtype y_type, int64_t ldy, float* t, int64_t ldt, void* workspace,
                                   size_t workspace_bytes, int32_t* status_word_dev, void* cuda_stream) {
  if (!planned(rows) || !adapters_there(weights) || !dense_rows(x, x_type, weights->K, ldx) || !dense_rows(y, y_type, weights->N, ldy) ||
      (base && !dense_rows(base, y_type, weights->N, ldbase)) || (base == y && ldbase != ldy && rows->count > 1) ||
      (t && (ldt < weights->rank || !aligned(t, 4))) || !aligned(workspace, 16) || !aligned(status_word_dev, 4))
    return LCD_ERR_INVALID_ARG;
  if (weights->rank > kMostRank || weights->G > kMostGroups || !types_go(x_type, weights->type)) return LCD_ERR_UNSUPPORTED;
  size_t need = 0;
  lcd_status st = lcd_adapters_workspace_bytes(rows->count, weights->rank, &need);
  if (st != LCD_OK) return st;
  if (!workspace || workspace_bytes < need) return LCD_ERR_BUFFER_TOO_SMALL;
  if (rows->count == 1) ldx = ldbase = ldy = 0;          // a single row has no pitch to be off 16 bytes
  DownArgs d = {};
  d.a = args_of(*weights, *rows, false);
  d.x = x;
  d.ldx = ldx;
  d.t = static_cast<float*>(workspace);
  d.t_rows = t;
  d.ldt_rows = ldt;
  d.status = status_word_dev;
  UpArgs u = {};
  u.a = args_of(*weights, *rows, true);
  u.a.scale = weights->scale;
  u.t = d.t;
  u.base = base;
  u.y = y;
  u.ldbase = ldbase;
  u.ldy = ldy;
  u.early = 1;
  u.status = status_word_dev;
  u.t_parts = d.t_parts = takes_parts_of_t(u, weights->type, y_type) ? d.t + rows->count * padded_rank(weights->rank) : nullptr;
  st = down(d, x_type, weights->type, false, cuda_stream);
  if (st != LCD_OK) return st;
  return up(u, weights->type, y_type, false, cuda_stream);
}

extern "C" lcd_status lcd_adapters_grad(const lcd_adapter_weights* weights, const void* dy, int64_t lddy, const void* x, int64_t ldx, lcd_dtype type,
                                        const float* t, int64_t ldt, const lcd_row_groups* rows, const void* base, int64_t ldbase, void* dx,
                                        int64_t lddx, void* da, void* db, lcd_dtype grad_type, void* workspace, size_t workspace_bytes,
                                        int32_t* status_word_dev, void* cuda_stream) {
  if (!planned(rows) || !adapters_there(weights) || !dense_rows(dy, type, weights->N, lddy) || (!dx && !da && !db) ||
      (da && !dense_rows(x, type, weights->K, ldx)) || (db && (!t || ldt < weights->rank || !aligned(t, 4))) ||
      (dx && (!dense_rows(dx, type, weights->K, lddx) || (base && !dense_rows(base, type, weights->K, ldbase)) ||
              (base == dx && ldbase != lddx && rows->count > 1) || dx == dy || dx == x)) ||
      ((da || db) && (!known(grad_type) || !aligned(da, size_of(grad_type)) || !aligned(db, size_of(grad_type)))) || !aligned(workspace, 16) ||
      !aligned(status_word_dev, 4))
    return LCD_ERR_INVALID_ARG;
  if (weights->rank > kMostRank || weights->G > kMostGroups || !types_go(type, weights->type)) return LCD_ERR_UNSUPPORTED;
  size_t need = 0;
  lcd_status st = lcd_adapters_workspace_bytes(rows->count, weights->rank, &need);
  if (st != LCD_OK) return st;
  if (!workspace || workspace_bytes < need) return LCD_ERR_BUFFER_TOO_SMALL;
  if (rows->count == 1) lddy = ldx = ldt = ldbase = lddx = 0;
  float* dt = static_cast<float*>(workspace);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  UpArgs u = {};
  if (dx) {
    u.a = args_of(*weights, *rows, false);
    u.t = dt;
    u.base = base;
    u.y = dx;
    u.ldbase = ldbase;
    u.ldy = lddx;
    u.early = 1;
    u.status = status_word_dev;
  }
  if (dx || da) {
    DownArgs d = {};
    d.a = args_of(*weights, *rows, true);
    d.a.scale = weights->scale;
    d.x = dy;
    d.ldx = lddy;
    d.t = dt;
    d.status = status_word_dev;
    u.t_parts = d.t_parts = dx && takes_parts_of_t(u, weights->type, type) ? dt + rows->count * padded_rank(weights->rank) : nullptr;
    st = down(d, type, weights->type, true, cuda_stream);
    if (st != LCD_OK) return st;
  }
  if (dx) {
    st = up(u, weights->type, type, true, cuda_stream);
    if (st != LCD_OK) return st;
  }
  if (!da && !db) return LCD_OK;
  OuterArgs o = {};
  o.order = rows->order;
  o.offsets = rows->offsets;
  o.rows = (int)rows->count;
  o.G = (int)weights->G;
  o.r = (int)weights->rank;
  o.out_type = (int)grad_type;
  o.status = status_word_dev;
  if (da) o.side[o.sides++] = {dt, padded_rank(weights->rank), 1, 0, x, ldx, 0, weights->K, nullptr, da, 0};
  if (db) o.side[o.sides++] = {t, ldt, 0, 0, dy, lddy, 0, weights->N, weights->scale, db, 1};
  return launch_adapters_outer(o, type, s);
}
