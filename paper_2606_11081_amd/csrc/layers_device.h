// Device helpers of the layer kernels (embedding.hip, layer_norm.hip,
// linear.hip): which worker a tile belongs to, typed vector accesses through
// the caches, fp32 sums over a wave.  Not installed.
#pragma once

#include "device_common.h"
#include "layers.h"

namespace gasloc {
namespace {

__device__ __forceinline__ int lane_id() { return threadIdx.x % kWave; }

// The worker whose part of the list holds item t (t the same in every lane,
// begin[0] <= t < begin[n]): the last i with begin[i] <= t.  One load per lane
// and a ballot instead of a search.
__device__ __forceinline__ int find_worker(const Spans& s, int n, int t) {
  const int lane = lane_id();
  const int b = s.begin[lane < n ? lane : n];
  return __popcll(__ballot(lane < n && b <= t)) - 1;
}

// Element 0 of worker i's live row.
template <int PT>
__device__ __forceinline__ const void* live_row(const LiveRows& w, int i) {
  const void* base = (w.stepped >> i) & 1ull ? w.y : w.x;
  return static_cast<const char*>(base) + static_cast<int64_t>(i) * w.ld * (PT == GASLOC_BF16 ? 2 : 4);
}

// V consecutive elements through the caches (16-byte aligned where V elements are 16 bytes or more).
template <int DT, int V>
__device__ __forceinline__ void load_cached(const void* base, int64_t idx, float (&o)[V]) {
  if constexpr (DT == GASLOC_BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + idx;
    if constexpr (V == 8) {
      const u32x4 t = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        o[2 * k] = __uint_as_float(t[k] << 16);
        o[2 * k + 1] = __uint_as_float(t[k] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = bf16_to_f32(p[k]);
    }
  } else {
    const float* p = static_cast<const float*>(base) + idx;
    if constexpr (V % 4 == 0) {
#pragma unroll
      for (int k = 0; k < V; k += 4) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(p + k);
        o[k] = t.x; o[k + 1] = t.y; o[k + 2] = t.z; o[k + 3] = t.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = p[k];
    }
  }
}

// The same with the streaming hint: data that is read once.
template <int DT, int V>
__device__ __forceinline__ void load_once(const void* base, int64_t idx, float (&o)[V]) {
  if constexpr (DT == GASLOC_F32 && V == 8) {
    float a[4], b[4];
    load_f32<4>(static_cast<const float*>(base) + idx, 4, a);
    load_f32<4>(static_cast<const float*>(base) + idx + 4, 4, b);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      o[k] = a[k];
      o[4 + k] = b[k];
    }
  } else {
    load_params<DT, V>(base, idx, V, o);
  }
}

template <int DT, int V>
__device__ __forceinline__ void store_out(void* base, int64_t idx, const float (&o)[V]) {
  if constexpr (DT == GASLOC_F32 && V == 8) {
    float a[4], b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      a[k] = o[k];
      b[k] = o[4 + k];
    }
    store_f32<4>(static_cast<float*>(base) + idx, 4, a);
    store_f32<4>(static_cast<float*>(base) + idx + 4, 4, b);
  } else {
    float kept[V];
    store_params<DT, V>(base, idx, V, o, kept);
  }
}

// Sum over the wave, the same in every lane: DPP shifts inside each row of 16
// lanes, then the four row sums in order.
__device__ __forceinline__ float wave_sum_f32(float v) {
  const auto shifted = [](float x, auto k) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x110 + decltype(k)::value, 0xf, 0xf, true));
  };
  v += shifted(v, std::integral_constant<int, 1>{});
  v += shifted(v, std::integral_constant<int, 2>{});
  v += shifted(v, std::integral_constant<int, 4>{});
  v += shifted(v, std::integral_constant<int, 8>{});
  const auto lane = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return ((lane(15) + lane(31)) + lane(47)) + lane(63);
}

}  // namespace
}  // namespace gasloc
