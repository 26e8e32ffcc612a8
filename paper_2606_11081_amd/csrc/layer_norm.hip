// Layer norm of every worker's rows and its gradients.
//   out = (x - mean) rstd gain + bias
//   dx  = rstd (h - mean(h) - xh mean(h xh)),  h = dout gain,  xh = (x - mean) rstd
//   dgain = sum_t dout xh,  dbias = sum_t dout
// HBM-bound: a row is read once into registers, where its mean, its variance
// (from the differences to the mean, not from squares) and the backward
// pass's two means are taken.  One wave per row up to 2048 columns, then a
// workgroup of 4 or 8 waves; a workgroup takes tile_rows rows of one worker
// with that worker's gain and bias in registers.
//
// Measured (n = 16, 65536 rows of 1024, bf16 rows, fp32 weights): forward 52 us
// (269 MB, 5.2 TB/s), backward 87 us (403 MB, 4.6 TB/s), 5 of them the join of
// the partial sums; n = 7, 5003 rows of 1023, fp32: backward 22 us (2.8 TB/s).
#pragma clang fp contract(off)

#include <type_traits>

#include "layers_device.h"

namespace gasloc {
namespace {

// Sums over the waves that share a row, the same in each of them.  `slot`:
// alternates between calls, so that no wave overwrites what another still reads.
template <int WAVES, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], int slot) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_sum_f32(v[k]);
  if constexpr (WAVES > 1) {
    __shared__ float part[2][WAVES][K];
    const int wave = threadIdx.x / kWave;
    if (lane_id() == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) part[slot][wave][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v[k] += part[slot][w][k];
    }
  }
}

// E columns per thread, V consecutive ones at a time; WHOLE: rows are whole vectors.
template <int PT, int AT, int V, int E, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES* kWave) void k_layer_norm(NormArgs a) {
  constexpr int N = E / V, kStep = WAVES * kWave * V;
  constexpr int kRowsAtOnce = WAVES == 1 ? 4 : 1;
  const int i = find_worker(a.tiles, a.n, blockIdx.x);
  const int first = a.rows.begin[i] + (static_cast<int>(blockIdx.x) - a.tiles.begin[i]) * a.tile_rows;
  const int stop = min(first + a.tile_rows, a.rows.begin[i + 1]);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c0 = (WAVES == 1 ? lane_id() : static_cast<int>(threadIdx.x)) * V;
  const void* row = live_row<PT>(a.w, i);
  const auto left = [&](int j) { return WHOLE ? V : a.width - (c0 + j * kStep); };
  const float inv = 1.0f / static_cast<float>(a.width);
  float gain[E], bias[E];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float g[V] = {}, b[V] = {};
    if (c0 + j * kStep < a.width) {
      load_row<PT, V, false>(row, a.gain + c0 + j * kStep, left(j), g);
      if (a.bias >= 0) load_row<PT, V, false>(row, a.bias + c0 + j * kStep, left(j), b);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      gain[j * V + e] = g[e];
      bias[j * V + e] = b[e];
    }
  }
  for (int t = first + (WAVES == 1 ? wave : 0); t < stop; t += kRowsAtOnce) {
    float x[E];
    float sum[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float v[V] = {};
      if (c0 + j * kStep < a.width)
        load_row<AT, V, true>(a.x, static_cast<int64_t>(t) * a.x_ld + c0 + j * kStep, left(j), v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[j * V + e] = v[e];
        sum[0] += v[e];
      }
    }
    row_sums<WAVES, 1>(sum, 0);
    const float mean = sum[0] * inv;
    float sq[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int inside = a.width - (c0 + j * kStep);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = x[j * V + e] - mean;
        x[j * V + e] = d;
        if ((WHOLE ? 0 : e) < inside) sq[0] = fmaf(d, d, sq[0]);
      }
    }
    row_sums<WAVES, 1>(sq, 1);
    const float rstd = 1.0f / sqrtf(sq[0] * inv + a.eps);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = fmaf(x[j * V + e] * rstd, gain[j * V + e], bias[j * V + e]);
      if (c0 + j * kStep < a.width)
        store_row<AT, V>(a.out, static_cast<int64_t>(t) * a.out_ld + c0 + j * kStep, left(j), o);
    }
    if (a.stats && c0 == 0) {
      a.stats[2 * static_cast<int64_t>(t)] = mean;
      a.stats[2 * static_cast<int64_t>(t) + 1] = rstd;
    }
  }
}

template <int PT, int AT, int V, int E, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES* kWave) void k_layer_norm_grad(NormGradArgs a) {
  constexpr int N = E / V, kStep = WAVES * kWave * V;
  constexpr int kRowsAtOnce = WAVES == 1 ? 4 : 1;
  const int i = find_worker(a.tiles, a.n, blockIdx.x);
  const int first = a.rows.begin[i] + (static_cast<int>(blockIdx.x) - a.tiles.begin[i]) * a.tile_rows;
  const int stop = min(first + a.tile_rows, a.rows.begin[i + 1]);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c0 = (WAVES == 1 ? lane_id() : static_cast<int>(threadIdx.x)) * V;
  const void* row = live_row<PT>(a.w, i);
  const auto left = [&](int j) { return WHOLE ? V : a.width - (c0 + j * kStep); };
  const float inv = 1.0f / static_cast<float>(a.width);
  float gain[E], dgain[E] = {}, dbias[E] = {};
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float g[V] = {};
    if (c0 + j * kStep < a.width) load_row<PT, V, false>(row, a.gain + c0 + j * kStep, left(j), g);
#pragma unroll
    for (int e = 0; e < V; ++e) gain[j * V + e] = g[e];
  }
  int slot = 0;
  for (int t = first + (WAVES == 1 ? wave : 0); t < stop; t += kRowsAtOnce) {
    float x[E], h[E];
    const float mean = a.stats[2 * static_cast<int64_t>(t)], rstd = a.stats[2 * static_cast<int64_t>(t) + 1];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float v[V] = {}, d[V] = {};
      if (c0 + j * kStep < a.width) {
        load_row<AT, V, true>(a.x, static_cast<int64_t>(t) * a.x_ld + c0 + j * kStep, left(j), v);
        load_row<AT, V, true>(a.dout, static_cast<int64_t>(t) * a.dout_ld + c0 + j * kStep, left(j), d);
      }
      // Columns behind the row count nothing: h and xh are zero there (0 * xh would be NaN if mean * rstd overflowed).
      const int inside = a.width - (c0 + j * kStep);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[j * V + e] = (WHOLE ? 0 : e) < inside ? v[e] : mean;
        h[j * V + e] = d[e];
      }
    }
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < E; ++k) {
      x[k] = (x[k] - mean) * rstd;
      dgain[k] = fmaf(h[k], x[k], dgain[k]);
      dbias[k] += h[k];
      h[k] *= gain[k];
      sum[0] += h[k];
      sum[1] = fmaf(h[k], x[k], sum[1]);
    }
    row_sums<WAVES, 2>(sum, slot);
    slot ^= 1;
    const float m1 = sum[0] * inv, m2 = sum[1] * inv;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = rstd * ((h[j * V + e] - m1) - x[j * V + e] * m2);
      if (c0 + j * kStep < a.width)
        store_row<AT, V>(a.dx, static_cast<int64_t>(t) * a.dx_ld + c0 + j * kStep, left(j), o);
    }
  }
  float* part = a.partial + 2 * static_cast<int64_t>(blockIdx.x) * a.width;
  if constexpr (WAVES == 1) {
    // the four waves' sums over their rows, added in the order of the waves
    __shared__ float s_sum[2][kWave * E];
    for (int w = 0; w < 4; ++w) {
      if (wave == w) {
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const int at = k * kWave + lane_id();
          if (w > 0) {
            dgain[k] += s_sum[0][at];
            dbias[k] += s_sum[1][at];
          }
          s_sum[0][at] = dgain[k];
          s_sum[1][at] = dbias[k];
        }
      }
      __syncthreads();
    }
    if (wave != 3) return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float g[V], b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      g[e] = dgain[j * V + e];
      b[e] = dbias[j * V + e];
    }
    if (c0 + j * kStep < a.width) {
      store_row<GASLOC_F32, V>(part, c0 + j * kStep, left(j), g);
      store_row<GASLOC_F32, V>(part, a.width + c0 + j * kStep, left(j), b);
    }
  }
}

// Adds the tiles' sums of one worker, in sixteen stretches of tiles that are
// then added in order: thread (g, l) takes stretch g of column 64 b + l.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves* kWave) void k_layer_norm_join(NormGradArgs a) {
  __shared__ float s_sum[kJoinWaves][kWave];
  const int i = blockIdx.y;
  const int64_t begin = a.tiles.begin[i], count = a.tiles.begin[i + 1] - begin;
  const int lane = lane_id(), g = threadIdx.x / kWave;
  const int c = blockIdx.x * kWave + lane;
  const bool in = c < 2 * a.width;
  float sum = 0.0f;
  if (in) {
    const float* p = a.partial + 2 * begin * a.width + c;
    const int64_t stride = 2 * static_cast<int64_t>(a.width);
#pragma unroll 8
    for (int64_t q = count * g / kJoinWaves; q < count * (g + 1) / kJoinWaves; ++q) sum += p[q * stride];
  }
  s_sum[g][lane] = sum;
  __syncthreads();
  if (g != 0 || !in) return;
  sum = s_sum[0][lane];
#pragma unroll
  for (int k = 1; k < kJoinWaves; ++k) sum += s_sum[k][lane];
  const int64_t to = c < a.width ? a.gain + c : a.bias < 0 ? -1 : a.bias + (c - a.width);
  if (to < 0) return;
  float* out = a.grads + static_cast<int64_t>(i) * a.grad_ld + to;
  *out = a.accumulate ? *out + sum : sum;
}

// Elements per thread and waves per row for a width: the fewest waves whose
// threads hold the row, at most 32 elements each.
struct NormShape {
  int e, waves;
};
NormShape norm_shape(int width) {
  const int per = (width + kWave - 1) / kWave;
  if (per <= 8) return {8, 1};
  if (per <= 16) return {16, 1};
  if (per <= 32) return {32, 1};
  if (per <= 128) return {32, 4};
  return {32, 8};
}

template <int PT, int AT, bool WHOLE>
hipError_t forward(const NormArgs& a, hipStream_t stream) {
  constexpr int V = AT == GASLOC_BF16 ? 8 : 4;
  const NormShape s = norm_shape(a.width);
  const dim3 grid(a.tiles.begin[a.n]);
  const int threads = s.waves == 1 ? 256 : s.waves * kWave;
  return launch_kernel(s.waves == 8   ? k_layer_norm<PT, AT, V, 32, 8, WHOLE>
                       : s.waves == 4 ? k_layer_norm<PT, AT, V, 32, 4, WHOLE>
                       : s.e == 32    ? k_layer_norm<PT, AT, V, 32, 1, WHOLE>
                       : s.e == 16    ? k_layer_norm<PT, AT, V, 16, 1, WHOLE>
                                      : k_layer_norm<PT, AT, V, 8, 1, WHOLE>,
                       grid, threads, 0, stream, a);
}

template <int PT, int AT, bool WHOLE>
hipError_t backward(const NormGradArgs& a, hipStream_t stream) {
  constexpr int V = AT == GASLOC_BF16 ? 8 : 4;
  const NormShape s = norm_shape(a.width);
  const dim3 grid(a.tiles.begin[a.n]);
  const int threads = s.waves == 1 ? 256 : s.waves * kWave;
  return launch_kernel(s.waves == 8   ? k_layer_norm_grad<PT, AT, V, 32, 8, WHOLE>
                       : s.waves == 4 ? k_layer_norm_grad<PT, AT, V, 32, 4, WHOLE>
                       : s.e == 32    ? k_layer_norm_grad<PT, AT, V, 32, 1, WHOLE>
                       : s.e == 16    ? k_layer_norm_grad<PT, AT, V, 16, 1, WHOLE>
                                      : k_layer_norm_grad<PT, AT, V, 8, 1, WHOLE>,
                       grid, threads, 0, stream, a);
}

}  // namespace

int norm_waves(int width) { return norm_shape(width).waves; }

hipError_t launch_layer_norm(const NormArgs& a, int params, int act, bool whole, hipStream_t stream) {
  if (params == GASLOC_BF16)
    return whole ? forward<GASLOC_BF16, GASLOC_BF16, true>(a, stream)
                 : forward<GASLOC_BF16, GASLOC_BF16, false>(a, stream);
  if (act == GASLOC_BF16)
    return whole ? forward<GASLOC_F32, GASLOC_BF16, true>(a, stream)
                 : forward<GASLOC_F32, GASLOC_BF16, false>(a, stream);
  return whole ? forward<GASLOC_F32, GASLOC_F32, true>(a, stream) : forward<GASLOC_F32, GASLOC_F32, false>(a, stream);
}

hipError_t launch_layer_norm_grad(const NormGradArgs& a, int params, int act, bool whole, hipStream_t stream) {
  if (params == GASLOC_BF16)
    return whole ? backward<GASLOC_BF16, GASLOC_BF16, true>(a, stream)
                 : backward<GASLOC_BF16, GASLOC_BF16, false>(a, stream);
  if (act == GASLOC_BF16)
    return whole ? backward<GASLOC_F32, GASLOC_BF16, true>(a, stream)
                 : backward<GASLOC_F32, GASLOC_BF16, false>(a, stream);
  return whole ? backward<GASLOC_F32, GASLOC_F32, true>(a, stream) : backward<GASLOC_F32, GASLOC_F32, false>(a, stream);
}

hipError_t launch_layer_norm_join(const NormGradArgs& a, hipStream_t stream) {
  return launch_kernel(k_layer_norm_join, dim3((2 * a.width + kWave - 1) / kWave, a.n), kJoinWaves * kWave, 0,
                       stream, a);
}

}  // namespace gasloc
