// The plan of a batch whose rows go to different weights (lcd_group_rows): a stable counting sort of the rows by group.
//
// Every warp of a CTA, or of a cluster of eight where there are many rows, has one contiguous piece of the rows.  It counts its rows by
// group in a column of its own in shared memory (match.any finds a group's rows among 32, one lane adds them, so there are no
// atomics); the columns are summed over the warps of all CTAs, in their order, and over the groups; then every warp walks its piece
// again and gives its rows their places.  What bounds it is latency: a dozen dependent steps (256 rows of 32 groups 3.0 us, 8192 in a
// cluster of eight 7, 65536 of 128 groups 17; host and device together 5.7 and 19).
#include "common.h"
#include "device_util.h"

namespace lcd {

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32, kMostCtas = 8;


template <typename I>
__device__ __forceinline__ int group_of(const I* group, int64_t row, int64_t rows, int G) {
  if (row >= rows) return -1;                                    // beside the rows, in no column
  const I v = group[row];
  return v >= 0 && v < (I)G ? (int)v : G;
}

template <typename I>
__global__ void __launch_bounds__(kThreads)
group_rows_kernel(const I* group, int64_t rows, int G, int64_t piece, int32_t* order, int32_t* groups, int32_t* offsets) {
  extern __shared__ int s_count[];                               // [warps][G + 1], then a total for every group
  __shared__ int s_scan[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, bins = G + 1;
  uint32_t rank, ctas;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
  int* total = s_count + warps * bins;
  for (int i = threadIdx.x; i < warps * bins; i += blockDim.x) s_count[i] = 0;
  begin_after_previous();
  __syncthreads();
  const int64_t from = ((int64_t)rank * warps + warp) * piece, to = min(rows, from + piece);
  int* mine = s_count + warp * bins;
  for (int64_t r = from; r < to; r += 32) {
    const int g = group_of(group, r + lane, to, G);
    const unsigned same = __match_any_sync(0xffffffffu, g);
    if (g >= 0 && (int)(__ffs(same) - 1) == lane) mine[g] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  // a group's count before every warp of this CTA
  for (int g = threadIdx.x; g < bins; g += blockDim.x) {
    int sum = 0;
    for (int w = 0; w < warps; ++w) {
      const int c = s_count[w * bins + g];
      s_count[w * bins + g] = sum;
      sum += c;
    }
    total[g] = sum;
  }
  if (ctas > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  } else {
    __syncthreads();
  }
  // the groups' sizes over all CTAs, in front of this one, and summed over the groups: thread i has groups i, i + blockDim.x, ...
  int before_all = 0;
  for (int g0 = 0; g0 < bins; g0 += blockDim.x) {
    const int g = g0 + threadIdx.x;
    int size = 0, ahead = 0;
    if (g < bins) {
      if (ctas > 1) {
        const uint32_t at = (uint32_t)__cvta_generic_to_shared(total + g);
        int c[kMostCtas];
#pragma unroll
        for (int i = 0; i < kMostCtas; ++i) {
          c[i] = 0;
          if (i < (int)ctas) {
            uint32_t there;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(i));
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(c[i]) : "r"(there) : "memory");
          }
        }
#pragma unroll
        for (int i = 0; i < kMostCtas; ++i) {
          size += c[i];
          if (i < (int)rank) ahead += c[i];
        }
      } else {
        size = total[g];
      }
    }
    int sum = size;                                              // over the warp, then over the warps
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += v;
    }
    if (lane == 31) s_scan[warp] = sum;
    __syncthreads();
    int before = before_all, all = 0;
    for (int w = 0; w < warps; ++w) {
      if (w < warp) before += s_scan[w];
      all += s_scan[w];
    }
    __syncthreads();
    const int start = before + sum - size;
    if (g < bins) {
      if (rank == 0) offsets[g] = start;                         // bin G: the rows without a group begin where the others end
      for (int w = 0; w < warps; ++w) s_count[w * bins + g] += start + ahead;
    }
    before_all += all;
  }
  __syncthreads();
  for (int64_t r = from; r < to; r += 32) {
    const int g = group_of(group, r + lane, to, G);
    const unsigned same = __match_any_sync(0xffffffffu, g);
    const int at = g >= 0 ? mine[g] + __popc(same & ((1u << lane) - 1u)) : 0;
    __syncwarp();
    if (g >= 0) {
      order[at] = (int32_t)(r + lane);
      groups[at] = g < G ? g : -1;
      if ((int)(__ffs(same) - 1) == lane) mine[g] += __popc(same);
    }
    __syncwarp();
  }
  if (ctas > 1) {                                                // no CTA leaves while another may read its totals
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
}

template <typename I>
lcd_status launch(const void* group, int64_t rows, int G, int32_t* order, int32_t* groups, int32_t* offsets, cudaStream_t s) {
  auto kern = group_rows_kernel<I>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (kWarps + 1) * (kMostGroups + 1) * 4);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  const unsigned ctas = rows > 4096 ? kMostCtas : 1;
  const int64_t most = (int64_t)kWarps * 32;
  const int warps = (int)(rows >= most ? kWarps : (rows + 31) / 32 < 4 ? 4 : (rows + 31) / 32);
  const int64_t piece = ((rows + ctas * warps - 1) / (ctas * warps) + 31) / 32 * 32;
  const cudaError_t e = launch_overlapping(kern, dim3(ctas), dim3(32 * warps), (size_t)(warps + 1) * (G + 1) * 4, ctas, s,
                                           static_cast<const I*>(group), rows, G, piece, order, groups, offsets);
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

}  // namespace

lcd_status launch_group_rows(const void* group, int idx_bytes, int64_t rows, int64_t G, int32_t* order, int32_t* groups, int32_t* offsets,
                             void* stream) {
  if (G > kMostGroups) return LCD_ERR_UNSUPPORTED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return idx_bytes == 4 ? launch<int32_t>(group, rows, (int)G, order, groups, offsets, s)
                        : launch<int64_t>(group, rows, (int)G, order, groups, offsets, s);
}

}  // namespace lcd
