// x a^T of the adapters' forward pass, and dy b of the backward pass: from rows of K columns to rows of the rank.
//
// A CTA takes a window of consecutive places of the plan (rows sorted by adapter) and a share of the columns; its warps take chunks of 32
// columns in turn.  The adapter's rows (ranks) are the 16 rows of mma.sync, the batch's rows its 8 columns.  Windows with rows of several
// adapters go through the columns once for each.  Sums: over the warps in shared memory, over a cluster's CTAs (which share the
// columns) in distributed shared memory, in a fixed order.
// Latency bounds it: a CTA takes 4.4 us (the plan .6, its first loads 1.2, two chunks a warp, sums .9, the cluster's .7), and 64 rows of 48
// adapters, 4096 columns, rank 16, bf16, are 512 CTAs, three an SM (12 us with cold caches, where the bytes alone take 1).
// TRANSPOSED: the adapter matrix is b [K][r], the sum runs over its rows, which the lane pairs up with byte permutes; a lane then has 2 RT
// consecutive ranks in place of ranks 8 apart.
#ifndef LCD_ADAPTERS_DOWN_CUH_
#define LCD_ADAPTERS_DOWN_CUH_

#include "adapters.cuh"

namespace lcd {

struct DownArgs {
  AdapterArgs a;
  const void* x;
  long long ldx;
  int window;
  float *t, *t_rows;           // by place, 16 * RT values a row; by row (may be null)
  long long ldt_rows;
  void* t_parts;               // by place, [rows][kPartsT][16 * RT] bf16 (may be null)
  int32_t* status;
};

// Four values of t, with their bf16 parts: all but the last cut off, that one rounded.
__device__ __forceinline__ void store_t4(const DownArgs& P, int R, long long place, int r, const float (&v)[4]) {
  *reinterpret_cast<float4*>(P.t + place * R + r) = make_float4(v[0], v[1], v[2], v[3]);
  if (!P.t_parts) return;
  uint2* to = reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(P.t_parts) + place * kPartsT * R + r);
  float w[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
  for (int p = 0; p < kPartsT; ++p) {
    const bool last = p + 1 == kPartsT;
    to[p * R / 4] = last ? make_uint2(pair_rounded(w[0], w[1]), pair_rounded(w[2], w[3])) : make_uint2(pair_upper(w[0], w[1]), pair_upper(w[2], w[3]));
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = rest_of(w[i], upper_bf16(w[i]));
  }
}

constexpr int kDownWarps = 8;
template <int RT> constexpr int kDownTokens = RT == 8 ? 2 : 4;              // groups of eight rows in the widest window
constexpr int kDownSplit = 8;                                       // most CTAs that share the columns

// NT: groups of eight rows of the widest window; one for windows of up to eight rows, whose many CTAs then have registers to share an SM.
template <typename X, typename W, int RT, int NT, bool TRANSPOSED>
__global__ void __launch_bounds__(32 * kDownWarps, NT == 1 && RT * sizeof(W) <= 4 ? 3 : NT == 1 && RT * sizeof(W) <= 8 ? 2 : 1) adapters_down_kernel(const DownArgs P) {
  constexpr int R = 16 * RT;
  constexpr bool kNative = kIs16<X> && std::is_same<X, W>::value;
  using WWords = Words<W, TRANSPOSED ? 2 * RT : 8>;
  constexpr int kW = TRANSPOSED ? 8 : 2 * RT;
  extern __shared__ float s_sum[];                                  // [warps][window][R]
  __shared__ int s_group[8 * NT], s_row[8 * NT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint32_t rank, split;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
  const int place0 = (int)(blockIdx.x / split) * P.window, count = min(P.window, P.a.rows - place0);
  begin_after_previous();
  if ((int)threadIdx.x < 8 * NT) {
    int group = -1, row = -1;
    if ((int)threadIdx.x < count) {
      group = P.a.groups[place0 + threadIdx.x];
      row = row_of(P.a.order, place0 + threadIdx.x, P.a.rows);
      if ((unsigned)group >= (unsigned)P.a.G || row < 0) group = -1;
    }
    s_group[threadIdx.x] = group;
    s_row[threadIdx.x] = row;
  }
  __syncthreads();
  const int chunks = (int)((P.a.K + 31) / 32);
  const int c0 = (int)((long long)chunks * rank / split), c1 = (int)((long long)chunks * (rank + 1) / split);

  for (int i0 = 0, i1; i0 < count; i0 = i1) {
    const int group = s_group[i0];
    for (i1 = i0 + 1; i1 < count && s_group[i1] == group; ++i1) {}
    if (group < 0) continue;
    const X* xrow[NT];
    bool mine[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int at = 8 * n + g;
      mine[n] = at >= i0 && at < i1;
      xrow[n] = static_cast<const X*>(P.x) + (mine[n] ? (long long)s_row[at] * P.ldx : 0) + 8 * t;
    }
    const W* w = static_cast<const W*>(P.a.w) + group * P.a.sw + (TRANSPOSED ? 8 * t * P.a.ldw + g * 2 * RT : g * P.a.ldw + 8 * t);
    float acc[RT][NT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][n][c] = 0.0f;
    struct Frag {
      WWords w[kW];
      Words<X, 8> x[NT];
    };
    auto load = [&](Frag& f, int c) {
      const long long k = (long long)c * 32;
      const int have = (int)min((long long)8, P.a.K - k - 8 * t);
      // chunks with another on either side: rows at any alignment in aligned words, all rows' loads on their way together (of large ranks
      // four rows' at a time)
      const bool within = k >= 32 && k + 64 <= P.a.K, shift_w = !TRANSPOSED && !P.a.wide_w && within, shift_x = !P.a.wide_x && within;
      constexpr int kBatch = kW <= 4 ? kW : 4;
      Around<W, TRANSPOSED ? 2 * RT : 8> around_w[kBatch];
      Around<X, 8> around_x[NT];
      auto row_w = [&](int i) { return w + 8 * i * P.a.ldw + k; };
      if (shift_w) {
#pragma unroll
        for (int i0 = 0; i0 < kW; i0 += kBatch) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) load_around(around_w[i], row_w(i0 + i), 8 * (i0 + i) + g < P.a.r);
          if (kW > kBatch) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) shift_words(f.w[i0 + i], around_w[i], row_w(i0 + i));
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < kW; ++i) {
          if (TRANSPOSED) {
            const int ranks = min(2 * RT, P.a.r - g * 2 * RT);
            load_words(f.w[i], w + (k + i) * P.a.ldw, i < have ? ranks : 0, P.a.wide_w && (ranks <= 0 || ranks >= 2 * RT));
          } else {
            load_words(f.w[i], row_w(i), 8 * i + g < P.a.r ? have : 0, P.a.wide_w && (have <= 0 || have >= 8));
          }
        }
      }
      if (shift_x) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (8 * n < i1 && 8 * n + 8 > i0) load_around(around_x[n], xrow[n] + k, mine[n]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (8 * n < i1 && 8 * n + 8 > i0) shift_words(f.x[n], around_x[n], xrow[n] + k);
      } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (8 * n < i1 && 8 * n + 8 > i0) load_words(f.x[n], xrow[n] + k, mine[n] ? have : 0, P.a.wide_x && (have <= 0 || have >= 8));
      }
      if (shift_w && kW <= kBatch) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) shift_words(f.w[i], around_w[i], row_w(i));
      }
    };
    // value e (column 8 t + e of the chunk) of the lane's rank q: row 8 q + g, or g * 2 RT + q
    auto value_w = [&](const Frag& f, int q, int e) { return TRANSPOSED ? value_of(f.w[TRANSPOSED ? e : 0], q) : value_of(f.w[TRANSPOSED ? 0 : q], e); };
    auto multiply = [&](const Frag& f) {
      if constexpr (kNative) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            uint32_t a[4];
            if constexpr (TRANSPOSED) {
#pragma unroll
              for (int j = 0; j < 4; ++j) a[j] = pair_of(f.w[4 * s + 2 * (j / 2)], f.w[4 * s + 2 * (j / 2) + 1], 2 * i + j % 2);
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) a[j] = f.w[2 * i + j % 2].w[2 * s + j / 2];
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
              if (8 * n < i1 && 8 * n + 8 > i0) mma16<X>(acc[i][n], a[0], a[1], a[2], a[3], f.x[n].w[2 * s], f.x[n].w[2 * s + 1]);
          }
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          float b[NT][2], b_rest[NT][2], b_finite[NT][2];         // (an infinite x has its say in the first product alone, which keeps its sign)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float v = value_of(f.x[n], 2 * s + j);
              b[n][j] = kIs16<X> ? v : upper_tf32(v);
              b_rest[n][j] = kIs16<X> ? 0.0f : rest_tf32(v, b[n][j]);
              b_finite[n][j] = kIs16<W> || fabsf(b[n][j]) != __uint_as_float(0x7f800000u) ? b[n][j] : 0.0f;
            }
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            float a[4], a_rest[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float v = value_w(f, 2 * i + j % 2, 2 * s + j / 2);
              a[j] = kIs16<W> ? v : upper_tf32(v);
              a_rest[j] = kIs16<W> ? 0.0f : rest_tf32(v, a[j]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
              if (8 * n < i1 && 8 * n + 8 > i0) {
                mma_tf32(acc[i][n], a[0], a[1], a[2], a[3], b[n][0], b[n][1]);
                if constexpr (!kIs16<X>) mma_tf32(acc[i][n], a[0], a[1], a[2], a[3], b_rest[n][0], b_rest[n][1]);
                if constexpr (!kIs16<W>) mma_tf32(acc[i][n], a_rest[0], a_rest[1], a_rest[2], a_rest[3], b_finite[n][0], b_finite[n][1]);
              }
          }
        }
      }
    };
    Frag now = {}, next = {};
    if (c0 + warp < c1) load(now, c0 + warp);
    for (int c = c0 + warp; c < c1; c += kDownWarps) {
      if (c + kDownWarps < c1) load(next, c + kDownWarps);
      multiply(now);
      now = next;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int at = 8 * n + 2 * t + (c & 1);
        if (at < i0 || at >= i1) continue;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const int r = TRANSPOSED ? g * 2 * RT + 2 * i + (c >> 1) : 16 * i + g + 8 * (c >> 1);
          s_sum[(warp * P.window + at) * R + r] = acc[i][n][c];
        }
      }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < count * R; e += blockDim.x) {
    float sum = 0.0f;
    if (s_group[e / R] >= 0) {
      sum = s_sum[e];
#pragma unroll
      for (int w = 1; w < kDownWarps; ++w) sum += s_sum[w * P.window * R + e];
    }
    s_sum[e] = sum;                                                 // nobody else reads this one
  }
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  } else {
    __syncthreads();
  }
  for (int e = 4 * (rank * blockDim.x + threadIdx.x); e < count * R; e += 4 * split * blockDim.x) {
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (split > 1) {
      const uint32_t at = (uint32_t)__cvta_generic_to_shared(s_sum + e);
      float4 part[kDownSplit];
#pragma unroll
      for (int i = 0; i < kDownSplit; ++i) {
        part[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (i < (int)split) {
          uint32_t there;
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(i));
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(part[i].x), "=f"(part[i].y), "=f"(part[i].z), "=f"(part[i].w) : "r"(there));
        }
      }
#pragma unroll
      for (int i = 0; i < kDownSplit; ++i) {
        v[0] += part[i].x;
        v[1] += part[i].y;
        v[2] += part[i].z;
        v[3] += part[i].w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = s_sum[e + i];
    }
    const int at = e / R, r = e % R, group = s_group[at];
    const float factor = P.a.scale && group >= 0 ? P.a.scale[group] : 1.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = r + i < P.a.r ? v[i] * factor : 0.0f;
    store_t4(P, R, place0 + at, r, v);
    if (P.t_rows && s_row[at] >= 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (r + i < P.a.r) P.t_rows[(long long)s_row[at] * P.ldt_rows + r + i] = v[i];
    }
  }
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
}

template <typename X, typename W, bool TRANSPOSED>
lcd_status launch_down_types(DownArgs P, cudaStream_t s) {
  P.a.wide_x = on_bytes(P.x, P.ldx, 0, sizeof(X), 16);
  return by_rank(P.a.r, [&](auto rt) {
    constexpr int RT = decltype(rt)::value, MOST = kDownTokens<RT>;
    constexpr int kWide = TRANSPOSED && 2 * RT * (int)sizeof(W) < 16 ? 2 * RT * (int)sizeof(W) : 16;
    P.a.wide_w = on_bytes(P.a.w, P.a.ldw, P.a.sw, sizeof(W), kWide);
    // Rows of a window: as many as a group has on average if all groups occur, so that few windows have rows of several.  CTAs that share its
    // columns: until there are two for every SM (four of the small ones), while each warp has a chunk.
    const int mean = P.a.rows / (P.a.G < P.a.rows ? P.a.G : P.a.rows), sms = current_sm_count();
    P.window = mean < 2 ? 1 : mean < 4 ? 2 : mean < 8 ? 4 : mean < 16 ? 8 : mean < 32 || MOST == 2 ? 16 : 8 * MOST;
    const int windows = (P.a.rows + P.window - 1) / P.window;
    unsigned split = 1;
    while (split < kDownSplit && (long long)windows * split < (P.window <= 8 ? 3 : 2) * sms && (P.a.K + 31) / 32 > (long long)split * kDownWarps) split *= 2;
    auto go = [&](auto nt) {
      constexpr int NT = decltype(nt)::value, kMostSmem = kDownWarps * 8 * NT * 16 * RT * 4;
      auto kern = adapters_down_kernel<X, W, RT, NT, TRANSPOSED>;
      static PerDeviceFlag attr_set;
      int dev;
      if (attr_set.first(&dev)) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
        if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
        attr_set.done(dev);
      }
      return adapter_launched(launch_overlapping(kern, dim3((unsigned)windows * split), dim3(32 * kDownWarps),
                                                 (size_t)kDownWarps * P.window * 16 * RT * 4, split, s, P));
    };
    return P.window <= 8 ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, MOST>{});
  });
}

}  // namespace lcd
#endif
