// Adapters of this type (adapters_up_tc.cuh).
#include "adapters_up_tc.cuh"

namespace lcd {

lcd_status launch_adapters_up_tc_f16(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s) {
  return launch_up_tc_weights<__half>(P, y_type, transposed, s);
}

}  // namespace lcd
