// Linear layers of every worker: products of its token rows with its weight
// and, backward, of the gradients with the weight and with the rows.
#pragma clang fp contract(off)

#include "layers_device.h"

namespace gasloc {
namespace {

template <int DT>
__device__ __forceinline__ float at(const void* base, int64_t idx) {
  if constexpr (DT == GASLOC_BF16)
    return bf16_to_f32(static_cast<const uint16_t*>(base)[idx]);
  else
    return static_cast<const float*>(base)[idx];
}

// 64 x 64 outputs per workgroup of 256 threads, 4 x 4 each; 16 k at a time in LDS.
template <int PASS, int PT, int AT>
__global__ __launch_bounds__(256) void k_linear(LinearArgs a) {
  constexpr int T = kLinearTile, K = 16;
  __shared__ float s_a[K][T + 4], s_b[K][T + 4];
  const int i = find_worker(a.tiles, a.n, blockIdx.x);
  const int tile = static_cast<int>(blockIdx.x) - a.tiles.begin[i];
  const int64_t r0 = a.rows.begin[i], count = a.rows.begin[i + 1] - r0;
  const int64_t M = PASS == kLinearWeight ? a.out_features : count;
  const int64_t N = PASS == kLinearForward ? a.out_features : a.in_features;
  const int64_t depth = PASS == kLinearForward ? a.in_features : PASS == kLinearInput ? a.out_features : count;
  const int64_t across = (N + T - 1) / T;
  const int64_t m0 = tile / across * T, n0 = tile % across * T;
  const void* w = live_row<PT>(a.w, i);
  const int tm = threadIdx.x / 16 * 4, tn = threadIdx.x % 16 * 4;
  float c[4][4] = {};
  for (int64_t k0 = 0; k0 < depth; k0 += K) {
    for (int e = threadIdx.x; e < K * T; e += 256) {
      // neighbours in memory for neighbouring threads: k first where rows run along k
      const int ka = PASS == kLinearWeight ? e / T : e % K, ma = PASS == kLinearWeight ? e % T : e / K;
      float v = 0.0f;
      if (k0 + ka < depth && m0 + ma < M) {
        if constexpr (PASS == kLinearForward)
          v = at<AT>(a.x, (r0 + m0 + ma) * a.x_ld + k0 + ka);
        else if constexpr (PASS == kLinearInput)
          v = at<AT>(a.dout, (r0 + m0 + ma) * a.dout_ld + k0 + ka);
        else
          v = at<AT>(a.dout, (r0 + k0 + ka) * a.dout_ld + m0 + ma);
      }
      s_a[ka][ma] = v;
      const int kb = PASS == kLinearForward ? e % K : e / T, nb = PASS == kLinearForward ? e / K : e % T;
      v = 0.0f;
      if (k0 + kb < depth && n0 + nb < N) {
        if constexpr (PASS == kLinearForward)
          v = as_stored<AT>(at<PT>(w, a.weight + (n0 + nb) * depth + k0 + kb));
        else if constexpr (PASS == kLinearInput)
          v = as_stored<AT>(at<PT>(w, a.weight + (k0 + kb) * N + n0 + nb));
        else
          v = at<AT>(a.x, (r0 + k0 + kb) * a.x_ld + n0 + nb);
      }
      s_b[kb][nb] = v;
    }
    __syncthreads();
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
#pragma unroll
        for (int q = 0; q < 4; ++q) c[p][q] = fmaf(s_a[k][tm + p], s_b[k][tn + q], c[p][q]);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t m = m0 + tm + p, n = n0 + tn + q;
      if (m >= M || n >= N) continue;
      if constexpr (PASS == kLinearWeight) {
        float* g = a.grads + static_cast<int64_t>(i) * a.grad_ld + a.weight + m * N + n;
        *g = a.accumulate ? *g + c[p][q] : c[p][q];
      } else if constexpr (AT == GASLOC_BF16) {
        static_cast<uint16_t*>(a.out)[(r0 + m) * a.out_ld + n] =
            static_cast<uint16_t>(f32x2_to_bf16x2(c[p][q], 0.0f) & 0xffffu);
      } else {
        static_cast<float*>(a.out)[(r0 + m) * a.out_ld + n] = c[p][q];
      }
    }
  }
}

template <int PASS>
hipError_t launch(const LinearArgs& a, int params, int act, hipStream_t stream) {
  return launch_kernel(params == GASLOC_BF16 ? k_linear<PASS, GASLOC_BF16, GASLOC_BF16>
                       : act == GASLOC_BF16  ? k_linear<PASS, GASLOC_F32, GASLOC_BF16>
                                             : k_linear<PASS, GASLOC_F32, GASLOC_F32>,
                       dim3(a.tiles.begin[a.n]), 256, 0, stream, a);
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, LinearPass pass, int params, int act, hipStream_t stream) {
  if (pass == kLinearForward) return launch<kLinearForward>(a, params, act, stream);
  if (pass == kLinearInput) return launch<kLinearInput>(a, params, act, stream);
  return launch<kLinearWeight>(a, params, act, stream);
}

}  // namespace gasloc
