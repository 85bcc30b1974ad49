// Rows of this type (adapters_down.cuh) with the adapters' types that they go with.
#include "adapters_down.cuh"

namespace lcd {

lcd_status launch_adapters_down_f16(const DownArgs& P, lcd_dtype w_type, bool backward, cudaStream_t s) {
  switch (w_type) {
    case LCD_DTYPE_F32: return backward ? launch_down_types<__half, float, true>(P, s) : launch_down_types<__half, float, false>(P, s);
    case LCD_DTYPE_F16: return backward ? launch_down_types<__half, __half, true>(P, s) : launch_down_types<__half, __half, false>(P, s);
    default: return LCD_ERR_UNSUPPORTED;
  }
}

}  // namespace lcd
