// The launches of the adapters' kernels (arguments are checked and laid out by api_groups.cu).
#ifndef LCD_ADAPTERS_LAUNCH_H_
#define LCD_ADAPTERS_LAUNCH_H_

#include "adapters.cuh"

namespace lcd {

struct UpArgs {
  AdapterArgs a;
  const float* t;              // by place, 16 * RT values a row
  const void* t_parts;         // the same as bf16 parts, [rows][kPartsT][16 * RT]: the products for many rows run
  const void* base;            // or null
  void* y;
  long long ldbase, ldy;
  int window, wide_base, wide_y;
  int in_place;                // y is base: rows without an adapter are left alone
  int32_t* status;
  int early;                   // the kernel before this one wrote t and nothing else that is read here, and began when all before it was done
};
lcd_status launch_adapters_up_f32(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s);
lcd_status launch_adapters_up_f16(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s);
lcd_status launch_adapters_up_bf16(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s);

// The same on tcgen05, for many rows, from t_parts.
lcd_status launch_adapters_up_tc_f32(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s);
lcd_status launch_adapters_up_tc_f16(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s);
lcd_status launch_adapters_up_tc_bf16(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s);

struct DownArgs;
lcd_status launch_adapters_down_f32(const DownArgs& P, lcd_dtype w_type, bool backward, cudaStream_t s);
lcd_status launch_adapters_down_f16(const DownArgs& P, lcd_dtype w_type, bool backward, cudaStream_t s);
lcd_status launch_adapters_down_bf16(const DownArgs& P, lcd_dtype w_type, bool backward, cudaStream_t s);

bool adapters_down_tc_takes(const DownArgs& P, lcd_dtype x_type, lcd_dtype w_type);
lcd_status launch_adapters_down_tc(const DownArgs& P, lcd_dtype type, bool backward, cudaStream_t s);
bool adapters_down_parts_takes(const DownArgs& P, lcd_dtype x_type, lcd_dtype w_type);
lcd_status launch_adapters_down_parts(const DownArgs& P, lcd_dtype x_type, lcd_dtype w_type, bool backward, cudaStream_t s);

// The gradient of one adapter matrix: [r] x columns of z's, sums over an adapter's rows of u (r values a row, fp32) times z.
struct OuterSide {
  const float* u;              // [rows][ldu], by place or by row
  long long ldu;
  int u_by_place, wide_u;
  const void* z;               // [rows][ldz]
  long long ldz;
  int wide_z;
  long long columns;
  const float* scale;          // [G] or null
  void* out;                   // [G][r][columns], or [G][columns][r]
  int by_column, wide_out;
};
struct OuterArgs {
  const int32_t *order, *offsets;
  int rows, G, r, out_type, sides;
  OuterSide side[2];
  long long slabs[2];
  int32_t* status;
};
lcd_status launch_adapters_outer(const OuterArgs& P, lcd_dtype z_type, cudaStream_t s);
bool adapters_outer_tc_takes(const OuterArgs& P);
lcd_status launch_adapters_outer_tc(const OuterArgs& P, lcd_dtype z_type, cudaStream_t s);

}  // namespace lcd
#endif
