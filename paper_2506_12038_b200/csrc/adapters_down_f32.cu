// Rows of this type (adapters_down.cuh) with the adapters' types that they go with.
#include "adapters_down.cuh"

namespace lcd {

lcd_status launch_adapters_down_f32(const DownArgs& P, lcd_dtype w_type, bool backward, cudaStream_t s) {
  switch (w_type) {
    case LCD_DTYPE_F32: return backward ? launch_down_types<float, float, true>(P, s) : launch_down_types<float, float, false>(P, s);
    case LCD_DTYPE_F16: return backward ? launch_down_types<float, __half, true>(P, s) : launch_down_types<float, __half, false>(P, s);
    default: return backward ? launch_down_types<float, __nv_bfloat16, true>(P, s) : launch_down_types<float, __nv_bfloat16, false>(P, s);
  }
}

}  // namespace lcd
