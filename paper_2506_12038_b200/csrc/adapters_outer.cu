// The adapters' gradients: da = sum over an adapter's rows of dt^T x, db = s sum of dy^T t.  One kernel, both sides in a launch.
//
// A CTA has a slab of 8 CT columns of z (x or dy) and one adapter; its warps, and the CTAs of a cluster where there are few slabs, take
// sixteen of the adapter's rows in turn.  The ranks are the 16 rows of mma.sync, the columns its 8, the sum runs over the batch's rows:
// a lane loads CT consecutive columns and 2 RT consecutive ranks of four rows and pairs rows up with byte permutes.  Tile j's column c stands for
// column CT c + j, m-tile i's rows c and c + 8 for ranks 2 RT c + 2 i and + 1.  t and dt go in as terms (adapters.cuh).
// The warps' sums meet in shared memory, the cluster's in distributed shared memory, in a fixed order.  Reading z bounds it.
// For fewer rows than adapters_outer_tc.cu takes.
#include "adapters.cuh"
#include "adapters_launch.h"

namespace lcd {

namespace {

constexpr int kOuterWarps = 8, kOuterSplit = 8;
template <typename Z, int RT> constexpr int kOuterTiles = RT == 4 ? 4 : 8;

template <typename Z, int RT>
__global__ void __launch_bounds__(32 * kOuterWarps) adapters_outer_kernel(const __grid_constant__ OuterArgs P) {
  constexpr int CT = kOuterTiles<Z, RT>, R = 16 * RT, kColumns = 8 * CT;
  constexpr bool kBf16 = std::is_same<Z, __nv_bfloat16>::value;
  extern __shared__ float s_part[];                                    // [warps][R][columns]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint32_t rank, split;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
  begin_after_previous();
  // slabs of the first side, then of the second; a rank above 64 takes two CTAs a slab
  const int halves = (P.r + R - 1) / R;
  long long slab = blockIdx.x / split;
  const int group = blockIdx.y, side = slab >= P.slabs[0] * halves;
  if (side) slab -= P.slabs[0] * halves;
  const OuterSide S = P.side[side];
  const int r0 = (int)(slab % halves) * R;
  const long long col0 = slab / halves * kColumns;
  const int from = max(0, min(P.rows, P.offsets[group])), to = max(from, min(P.rows, P.offsets[group + 1]));
  const int columns = (int)max(0ll, min((long long)CT, S.columns - col0 - CT * g)), ranks = max(0, min(2 * RT, P.r - r0 - 2 * RT * g));

  float acc[RT][CT][4];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[i][j][c] = 0.0f;
  struct Frag {
    Words<Z, CT> z[4];
    Words<float, 2 * RT> u[4];
  };
  auto load = [&](Frag& f, int at) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int place = at + 4 * t + q;
      const int row = place < to ? row_of(P.order, place, P.rows) : -1;
      const long long z_row = row >= 0 ? row : 0, u_row = S.u_by_place ? (row >= 0 ? place : 0) : z_row;
      load_words(f.z[q], static_cast<const Z*>(S.z) + z_row * S.ldz + col0 + CT * g, row >= 0 ? columns : 0, S.wide_z && (columns <= 0 || columns >= CT));
      load_words(f.u[q], S.u + u_row * S.ldu + r0 + 2 * RT * g, row >= 0 ? ranks : 0, S.wide_u && (ranks <= 0 || ranks >= 2 * RT));
    }
  };
  auto multiply = [&](const Frag& f) {
    if constexpr (kBf16) {
      uint32_t b[CT][2];
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        b[j][0] = pair_of(f.z[0], f.z[1], j);
        b[j][1] = pair_of(f.z[2], f.z[3], j);
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        uint32_t a[kPartsT][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x0 = value_of(f.u[2 * (q / 2)], 2 * i + q % 2), x1 = value_of(f.u[2 * (q / 2) + 1], 2 * i + q % 2);
#pragma unroll
          for (int term = 0; term < kPartsT - 1; ++term) {
            a[term][q] = pair_upper(x0, x1);
            x0 = rest_of(x0, upper_bf16(x0));
            x1 = rest_of(x1, upper_bf16(x1));
          }
          a[kPartsT - 1][q] = pair_rounded(x0, x1);
        }
#pragma unroll
        for (int term = 0; term < kPartsT; ++term)
#pragma unroll
          for (int j = 0; j < CT; ++j) mma16<Z>(acc[i][j], a[term][0], a[term][1], a[term][2], a[term][3], b[j][0], b[j][1]);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {                                    // rows 4 t + 2 s and + 1
        float a[RT][4], a_rest[RT][4];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float x = value_of(f.u[2 * s + q / 2], 2 * i + q % 2);
            a[i][q] = upper_tf32(x);
            a_rest[i][q] = rest_tf32(x, a[i][q]);
          }
#pragma unroll
        for (int j = 0; j < CT; ++j) {
          float b[2], b_rest[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float x = value_of(f.z[2 * s + q], j);
            b[q] = kIs16<Z> ? x : upper_tf32(x);
            b_rest[q] = kIs16<Z> ? 0.0f : rest_tf32(x, b[q]);
          }
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            mma_tf32(acc[i][j], a[i][0], a[i][1], a[i][2], a[i][3], b[0], b[1]);
            mma_tf32(acc[i][j], a_rest[i][0], a_rest[i][1], a_rest[i][2], a_rest[i][3], b[0], b[1]);
            if constexpr (!kIs16<Z>) mma_tf32(acc[i][j], a[i][0], a[i][1], a[i][2], a[i][3], b_rest[0], b_rest[1]);
          }
        }
      }
    }
  };
  constexpr bool kAhead = RT * sizeof(Z) <= 8;                         // the next rows are on their way while these are multiplied
  const int step = 16 * kOuterWarps * (int)split, first = from + 16 * (int)(rank * kOuterWarps + warp);
  if (kAhead) {
    Frag now = {}, next = {};
    if (first < to) load(now, first);
    for (int at = first; at < to; at += step) {
      if (to - at > step) load(next, at + step);
      multiply(now);
      now = next;
      if (to - at <= step) break;
    }
  } else {
    for (int at = first; at < to; at += step) {
      Frag f;
      load(f, at);
      multiply(f);
      if (to - at <= step) break;
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int r = 2 * RT * g + 2 * i + (c >> 1);
#pragma unroll
      for (int j = 0; j < CT; ++j) s_part[(warp * R + r) * kColumns + CT * (2 * t + (c & 1)) + j] = acc[i][j][c];
    }
  __syncthreads();
  for (int e = threadIdx.x; e < R * kColumns; e += blockDim.x) {
    float sum = s_part[e];
#pragma unroll
    for (int w = 1; w < kOuterWarps; ++w) sum += s_part[w * R * kColumns + e];
    s_part[e] = sum;                                                   // nobody else reads this one
  }
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  } else {
    __syncthreads();
  }
  const float factor = S.scale ? S.scale[group] : 1.0f;
  for (int e = rank * blockDim.x + threadIdx.x; e < R * kColumns; e += split * blockDim.x) {
    // consecutive threads: consecutive places of the output
    const int r = S.by_column ? e % R : e / kColumns, c = S.by_column ? e / R : e % kColumns;
    if (r0 + r >= P.r || col0 + c >= S.columns) continue;
    float sum = 0.0f;
    if (split > 1) {
      const uint32_t at = (uint32_t)__cvta_generic_to_shared(s_part + r * kColumns + c);
      float v[kOuterSplit];
#pragma unroll
      for (int i = 0; i < kOuterSplit; ++i) {
        v[i] = 0.0f;
        if (i < (int)split) {
          uint32_t there;
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(i));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[i]) : "r"(there) : "memory");
        }
      }
#pragma unroll
      for (int i = 0; i < kOuterSplit; ++i) sum += v[i];
    } else {
      sum = s_part[r * kColumns + c];
    }
    sum = to > from ? sum * factor : 0.0f;
    const long long at = S.by_column ? ((long long)group * S.columns + col0 + c) * P.r + r0 + r : ((long long)group * P.r + r0 + r) * S.columns + col0 + c;
    if (P.out_type == LCD_DTYPE_F32) static_cast<float*>(S.out)[at] = sum;
    else if (P.out_type == LCD_DTYPE_F16) static_cast<__half*>(S.out)[at] = from_f32<__half>(sum);
    else static_cast<__nv_bfloat16*>(S.out)[at] = from_f32<__nv_bfloat16>(sum);
  }
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
}

template <typename Z, int RT>
lcd_status launch_outer(OuterArgs P, cudaStream_t s) {
  constexpr int CT = kOuterTiles<Z, RT>, kSmem = kOuterWarps * 16 * RT * 8 * CT * 4;
  auto kern = adapters_outer_kernel<Z, RT>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  const int halves = (P.r + 16 * RT - 1) / (16 * RT);
  long long slabs = 0;
  for (int i = 0; i < 2; ++i) {
    P.slabs[i] = i < P.sides ? (P.side[i].columns + 8 * CT - 1) / (8 * CT) : 0;
    slabs += P.slabs[i] * halves;
    const int piece = CT * (int)sizeof(Z) < 16 ? CT * (int)sizeof(Z) : 16;
    P.side[i].wide_z = on_bytes(P.side[i].z, P.side[i].ldz, 0, sizeof(Z), piece);
    P.side[i].wide_u = on_bytes(P.side[i].u, P.side[i].ldu, 0, 4, 8 * RT < 16 ? 8 * RT : 16);
  }
  if (slabs > 0x7fffffff / kOuterSplit) return LCD_ERR_UNSUPPORTED;
  // CTAs that share an adapter's rows: until there are two for every SM, while each warp has 32 of them
  const int sms = current_sm_count(), mean = P.rows / (P.G < P.rows ? P.G : P.rows);
  unsigned split = 1;
  while (split < kOuterSplit && slabs * P.G * split < 2 * sms && mean > 32 * kOuterWarps * (int)split) split *= 2;
  return adapter_launched(launch_overlapping(kern, dim3((unsigned)(slabs * split), (unsigned)P.G), dim3(32 * kOuterWarps), kSmem, split, s, P));
}

}  // namespace

lcd_status launch_adapters_outer(const OuterArgs& P, lcd_dtype z_type, cudaStream_t s) {
  if (adapters_outer_tc_takes(P)) return launch_adapters_outer_tc(P, z_type, s);
  return by_dtype(z_type, [&](auto z) {
    using Z = typename decltype(z)::type;
    switch (rank_tiles(P.r)) {
      case 1: return launch_outer<Z, 1>(P, s);
      case 2: return launch_outer<Z, 2>(P, s);
      default: return launch_outer<Z, 4>(P, s);
    }
  });
}

}  // namespace lcd
