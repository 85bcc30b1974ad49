// Rows of this type (adapters_down.cuh) with the adapters' types that they go with.
#include "adapters_down.cuh"

namespace lcd {

lcd_status launch_adapters_down_bf16(const DownArgs& P, lcd_dtype w_type, bool backward, cudaStream_t s) {
  switch (w_type) {
    case LCD_DTYPE_F32: return backward ? launch_down_types<__nv_bfloat16, float, true>(P, s) : launch_down_types<__nv_bfloat16, float, false>(P, s);
    case LCD_DTYPE_BF16: return backward ? launch_down_types<__nv_bfloat16, __nv_bfloat16, true>(P, s) : launch_down_types<__nv_bfloat16, __nv_bfloat16, false>(P, s);
    default: return LCD_ERR_UNSUPPORTED;
  }
}

}  // namespace lcd
