// Adapters of this type (adapters_up.cuh).
#include "adapters_up.cuh"

namespace lcd {

lcd_status launch_adapters_up_f16(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s) {
  return launch_up_weights<__half>(P, y_type, transposed, s);
}

}  // namespace lcd
