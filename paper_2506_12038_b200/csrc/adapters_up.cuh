// From rows of the rank to rows of columns, added to what a shared layer gave: y = base + s t b^T, and dx = base + dt a in the backward pass.
//
// A warp has 8 CT columns (eight MMA tiles of eight, four or two where the rank is large) of a window of consecutive places of the plan.
// It keeps its part of the adapter matrix in registers as the MMAs' B operand for all rows of an adapter; rows are the A operand, 16 at a
// time, t in terms (adapters.cuh).  Tile j's column c stands for column CT c + j, so that a lane ends up with 2 CT consecutive
// columns of two rows, which it adds to the base's and stores.  The next rows' base and t are on their way meanwhile.
// Reading base, writing y bounds it, with few rows latency: the plan, then the matrix and base, then t (64 rows of 48 adapters to 11008 columns,
// rank 16, bf16: 14 us with cold caches, bytes 3).  It begins while the kernel that makes t ends: the adapter matrix and the first base are loaded before.
// TRANSPOSED: the adapter matrix is a [r][K]; rows are paired up with byte permutes.
#ifndef LCD_ADAPTERS_UP_CUH_
#define LCD_ADAPTERS_UP_CUH_

#include "adapters.cuh"
#include "adapters_launch.h"

namespace lcd {

namespace {

constexpr int kUpWarps = 4;

template <typename W, int RT>
constexpr int kUpTiles = sizeof(W) == 2 ? (RT <= 4 ? 8 : 4) : (RT <= 2 ? 8 : RT == 4 ? 4 : 2);

// N consecutive values of a row, of which `have` lie inside it; wide: on 16 bytes.
template <typename Y, int N>
__device__ __forceinline__ void store_values(Y* p, const float (&v)[N], int have, bool wide) {
  if (wide && have >= N) {
    if constexpr (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 8) {
        const float part[8] = {v[i], v[i + 1], v[i + 2], v[i + 3], v[i + 4], v[i + 5], v[i + 6], v[i + 7]};
        store8(p + i, part);
      }
    } else {
      static_assert(N == 4, "four or eights");
      if constexpr (sizeof(Y) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
        const float part[8] = {v[0], v[1], v[2], v[3], 0, 0, 0, 0};
        const uint4 w = pack8<Y>(part);
        *reinterpret_cast<uint2*>(p) = make_uint2(w.x, w.y);
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < have) p[i] = from_f32<Y>(v[i]);
}

// ONE: windows of at most sixteen rows, so an adapter has its rows in one go; no registers for a next one, and more warps an SM.
template <typename W, typename Y, int RT, bool TRANSPOSED, bool ONE>
__global__ void __launch_bounds__(32 * kUpWarps, ONE && RT == 1 ? 4 : ONE && RT == 2 ? 3 : 1) adapters_up_kernel(const UpArgs P) {
  constexpr int CT = kUpTiles<W, RT>, R = 16 * RT, kOwn = 2 * CT;       // columns of a lane
  constexpr bool kBf16 = std::is_same<W, __nv_bfloat16>::value;
  __shared__ float s_out[kUpWarps][16][8 * CT + 1];
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long long col0 = ((long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)) * 8 * CT;
  const long long own0 = col0 + kOwn * t;
  const int have = (int)max(0ll, min((long long)kOwn, P.a.K - own0));
  constexpr int kSide = 16 / sizeof(Y);
  const bool inside = have >= kOwn && own0 >= kSide && own0 + Around<Y, kOwn>::kCount * 4 / (int)sizeof(Y) <= P.a.K;
  const int place0 = blockIdx.y * P.window, end = min(P.a.rows, place0 + P.window);
  if (!P.early) begin_after_previous();
  bool waited = !P.early;

  // b as words of two ranks (16-bit types) or values: tile j, ranks t 4 RT + i
  constexpr int kWordsR = kIs16<W> ? 2 * RT : 4 * RT;
  uint32_t b[CT][kWordsR];
  auto load_b = [&](int group) {
    const W* w = static_cast<const W*>(P.a.w) + group * P.a.sw;
    const int ranks = max(0, min(4 * RT, P.a.r - t * 4 * RT));
    if constexpr (TRANSPOSED) {
      const long long c = col0 + CT * g;
      const int columns = (int)max(0ll, min((long long)CT, P.a.K - c));
      Words<W, CT> row[4];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          load_words(row[q], w + (long long)(t * 4 * RT + 4 * i + q) * P.a.ldw + c, 4 * i + q < ranks ? columns : 0,
                     P.a.wide_w && (columns <= 0 || columns >= CT));
#pragma unroll
        for (int j = 0; j < CT; ++j) {
          if constexpr (kIs16<W>) {
            b[j][2 * i] = pair_of(row[0], row[1], j);
            b[j][2 * i + 1] = pair_of(row[2], row[3], j);
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) b[j][4 * i + q] = row[q].w[j];
          }
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        const long long c = col0 + CT * g + j;
        Words<W, 4 * RT> row;
        load_words(row, w + c * P.a.ldw + t * 4 * RT, c < P.a.K ? ranks : 0, P.a.wide_w && (ranks <= 0 || ranks >= 4 * RT));
#pragma unroll
        for (int i = 0; i < kWordsR; ++i) b[j][i] = row.w[i];
      }
    }
  };
  struct Rows {                     // 16 rows: base, and where they are
    Words<Y, kOwn> base[2];
    int row[2];
  };
  // The plan, 32 places at a time: lane l has place chunk + l; the next 32 are asked for ahead.
  int my_group, my_row, next_group = -1, next_row = -1, loaded = -1;
  auto look = [&](int chunk) {
    next_group = chunk + lane < end ? P.a.groups[chunk + lane] : -1;
    next_row = chunk + lane < end ? P.a.order[chunk + lane] : -1;
  };
  auto load_rows = [&](Rows& f, int at, int to) {
    const Y* from[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = __shfl_sync(0xffffffffu, my_row, (at + g + 8 * h) & 31);
      f.row[h] = at + g + 8 * h < to ? row : -1;
      from[h] = static_cast<const Y*>(P.base) + (long long)max(f.row[h], 0) * P.ldbase + own0;
    }
    if (P.base && !P.wide_base && inside) {
      Around<Y, kOwn> around[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) load_around(around[h], from[h], f.row[h] >= 0);
#pragma unroll
      for (int h = 0; h < 2; ++h) shift_words(f.base[h], around[h], from[h]);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) load_words(f.base[h], from[h], P.base && f.row[h] >= 0 ? have : 0, P.wide_base && (have <= 0 || have >= kOwn));
    }
  };
  look(place0);
  for (int chunk = place0; chunk < end; chunk += 32) {
    my_group = next_group;
    my_row = checked_row(next_row, P.a.rows);
    if (!ONE && chunk + 32 < end) look(chunk + 32);
    const int places = min(32, end - chunk);
    for (int at0 = 0, at1; at0 < places; at0 = at1) {
      int group = __shfl_sync(0xffffffffu, my_group, at0);
      const unsigned other = __ballot_sync(0xffffffffu, my_group != group || lane >= places) & (0xffffffffu << at0);
      at1 = other ? __ffs(other) - 1 : 32;
      if ((unsigned)group >= (unsigned)P.a.G) group = -1;
      if (group < 0 && P.in_place) continue;
      Rows now, next = {};
      load_rows(now, at0, at1);
      float factor = 1.0f;
      if (group >= 0) {
        if (P.a.scale) factor = P.a.scale[group];
        if (group != loaded) load_b(group);
        loaded = group;
      }
      if (!waited) {
        begin_after_previous();
        waited = true;
      }
      for (int at = at0; at < at1; at += 16) {
        float d[CT][4];
#pragma unroll
        for (int j = 0; j < CT; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c) d[j][c] = 0.0f;
        float v[2][4 * RT];
        if (group >= 0) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < RT; ++i) {
              const int place = chunk + min(at + g + 8 * h, at1 - 1);
              const float4 q = *reinterpret_cast<const float4*>(P.t + (long long)place * R + t * 4 * RT + 4 * i);
              v[h][4 * i] = q.x; v[h][4 * i + 1] = q.y; v[h][4 * i + 2] = q.z; v[h][4 * i + 3] = q.w;
            }
        }
        if (!ONE && at + 16 < at1) load_rows(next, at + 16, at1);
        if (group >= 0) {
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            if constexpr (kBf16) {
              // words of ranks (4 i, 4 i + 1) of both rows, then (4 i + 2, 4 i + 3)
              uint32_t a[kPartsT][4];
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                float x0 = v[q % 2][4 * i + 2 * (q / 2)], x1 = v[q % 2][4 * i + 2 * (q / 2) + 1];
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
                for (int j = 0; j < CT; ++j) mma16<__nv_bfloat16>(d[j], a[term][0], a[term][1], a[term][2], a[term][3], b[j][2 * i], b[j][2 * i + 1]);
            } else {
#pragma unroll
              for (int s = 0; s < 2; ++s) {
                float a[4], a_rest[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                  const float x = v[q % 2][4 * i + 2 * s + q / 2];
                  a[q] = upper_tf32(x);
                  a_rest[q] = rest_tf32(x, a[q]);
                }
#pragma unroll
                for (int j = 0; j < CT; ++j) {
                  float w[2], w_rest[2];
#pragma unroll
                  for (int q = 0; q < 2; ++q) {
                    if constexpr (kIs16<W>) {
                      const __half2 h2 = *reinterpret_cast<const __half2*>(&b[j][2 * i + s]);
                      w[q] = q ? __high2float(h2) : __low2float(h2);
                    } else {
                      const float x = __uint_as_float(b[j][4 * i + 2 * s + q]);
                      w[q] = upper_tf32(x);
                      w_rest[q] = rest_tf32(x, w[q]);
                    }
                  }
                  mma_tf32(d[j], a[0], a[1], a[2], a[3], w[0], w[1]);
                  mma_tf32(d[j], a_rest[0], a_rest[1], a_rest[2], a_rest[3], w[0], w[1]);
                  if constexpr (!kIs16<W>) mma_tf32(d[j], a[0], a[1], a[2], a[3], w_rest[0], w_rest[1]);
                }
              }
            }
          }
        }
        // rows that do not start on 16 bytes go through shared memory, so that neighbouring lanes store neighbouring columns
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (now.row[h] < 0) continue;
          float out[kOwn];
#pragma unroll
          for (int j = 0; j < CT; ++j) {
            out[j] = value_of(now.base[h], j);
            out[CT + j] = value_of(now.base[h], CT + j);
            if (group >= 0) {
              out[j] = __fmaf_rn(factor, d[j][2 * h], out[j]);
              out[CT + j] = __fmaf_rn(factor, d[j][2 * h + 1], out[CT + j]);
            }
          }
          if (P.wide_y) {
            store_values(static_cast<Y*>(P.y) + (long long)now.row[h] * P.ldy + own0, out, have, true);
          } else {
#pragma unroll
            for (int j = 0; j < kOwn; ++j) s_out[threadIdx.x >> 5][g + 8 * h][kOwn * t + j] = out[j];
          }
        }
        if (!P.wide_y) {
          __syncwarp();
          const int columns = (int)max(0ll, min((long long)(8 * CT), P.a.K - col0));
#pragma unroll 4
          for (int r = 0; r < 16; ++r) {
            const int row = __shfl_sync(0xffffffffu, r < 8 ? now.row[0] : now.row[1], r % 8 * 4);
            if (row < 0) continue;
            Y* to = static_cast<Y*>(P.y) + (long long)row * P.ldy + col0;
            for (int c = lane; c < columns; c += 32) to[c] = from_f32<Y>(s_out[threadIdx.x >> 5][r][c]);
          }
          __syncwarp();
        }
        if (ONE) break;
        now = next;
      }
    }
  }
  if (!waited) begin_after_previous();
}

template <typename W, typename Y, bool TRANSPOSED>
lcd_status launch_up_types(UpArgs P, cudaStream_t s) {
  P.wide_base = on_bytes(P.base, P.ldbase, 0, sizeof(Y), 16);
  P.wide_y = on_bytes(P.y, P.ldy, 0, sizeof(Y), 16);
  P.in_place = P.base == P.y && P.ldbase == P.ldy;
  return by_rank(P.a.r, [&](auto rt) {
    constexpr int RT = decltype(rt)::value, CT = kUpTiles<W, RT>, kPiece = (TRANSPOSED ? CT : 4 * RT) * (int)sizeof(W);
    P.a.wide_w = on_bytes(P.a.w, P.a.ldw, P.a.sw, sizeof(W), kPiece < 16 ? kPiece : 16);
    const long long warps = (P.a.K + 8 * CT - 1) / (8 * CT);
    const int sms = current_sm_count();
    const int threads = warps * 32 / sms >= 32 * kUpWarps ? 32 * kUpWarps : 64;
    const long long columns = (warps * 32 + threads - 1) / threads;
    // windows: as long as leaves every SM some CTAs, and not many more rows than a group has on average if all groups occur
    int window = 256;
    while (window > 16 && columns * ((P.a.rows + window - 1) / window) * threads < 2048ll * sms) window /= 2;
    const int mean = P.a.rows / (P.a.G < P.a.rows ? P.a.G : P.a.rows);
    while (window > 1 && window > 2 * mean) window /= 2;
    if ((P.a.rows + window - 1) / window > 65535) window = (P.a.rows + 65534) / 65535;
    P.window = window;
    auto kern = window <= 16 ? adapters_up_kernel<W, Y, RT, TRANSPOSED, true> : adapters_up_kernel<W, Y, RT, TRANSPOSED, false>;
    return adapter_launched(launch_overlapping(kern, dim3((unsigned)columns, (unsigned)((P.a.rows + window - 1) / window)), dim3(threads), 0, 1, s, P));
  });
}

}  // namespace

template <typename W>
lcd_status launch_up_weights(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s) {
  return by_dtype(y_type, [&](auto y) {
    using Y = typename decltype(y)::type;
    return transposed ? launch_up_types<W, Y, true>(P, s) : launch_up_types<W, Y, false>(P, s);
  });
}

}  // namespace lcd
#endif
