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

// ---------------------------------------------------------------------------
// V consecutive elements (4 or 8) of a row, at any alignment of the element:
// the memory instructions of gfx950 take 16 bytes at any address.  `left`:
// elements of the row from the first one on; those behind it are left out
// (read as zero).  Whole rows of vectors pass left = V.
// ---------------------------------------------------------------------------

// Four or two words at an address of any alignment of two bytes; STREAM: data that is touched once.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

template <bool STREAM>
__device__ __forceinline__ u32x4 load_words4(const void* p) {
  const u32x4_any* q = static_cast<const u32x4_any*>(p);
  if constexpr (STREAM && GASLOC_NONTEMPORAL)
    return __builtin_nontemporal_load(q);
  else
    return *q;
}
template <bool STREAM>
__device__ __forceinline__ u32x2 load_words2(const void* p) {
  const u32x2_any* q = static_cast<const u32x2_any*>(p);
  if constexpr (STREAM && GASLOC_NONTEMPORAL)
    return __builtin_nontemporal_load(q);
  else
    return *q;
}
__device__ __forceinline__ void store_words4(void* p, u32x4 v) {
  u32x4_any* q = static_cast<u32x4_any*>(p);
#if GASLOC_NONTEMPORAL
  __builtin_nontemporal_store(v, q);
#else
  *q = v;
#endif
}
__device__ __forceinline__ void store_words2(void* p, u32x2 v) {
  u32x2_any* q = static_cast<u32x2_any*>(p);
#if GASLOC_NONTEMPORAL
  __builtin_nontemporal_store(v, q);
#else
  *q = v;
#endif
}

template <int DT, int V, bool STREAM>
__device__ __forceinline__ void load_row(const void* base, int64_t idx, int left, float (&o)[V]) {
  static_assert(V == 4 || V == 8, "");
  if constexpr (DT == GASLOC_BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + idx;
    if (left >= V) {
      uint32_t t[V / 2];
      if constexpr (V == 8) {
        const u32x4 v = load_words4<STREAM>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = v[k];
      } else {
        const u32x2 v = load_words2<STREAM>(p);
        t[0] = v.x;
        t[1] = v.y;
      }
#pragma unroll
      for (int k = 0; k < V / 2; ++k) {
        o[2 * k] = __uint_as_float(t[k] << 16);
        o[2 * k + 1] = __uint_as_float(t[k] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = k < left ? bf16_to_f32(p[k]) : 0.0f;
    }
  } else {
    const float* p = static_cast<const float*>(base) + idx;
#pragma unroll
    for (int k = 0; k < V; k += 4) {
      if (left >= k + 4) {
        const f32x4 t = __builtin_bit_cast(f32x4, load_words4<STREAM>(p + k));
        o[k] = t.x; o[k + 1] = t.y; o[k + 2] = t.z; o[k + 3] = t.w;
      } else {
#pragma unroll
        for (int e = k; e < k + 4; ++e) o[e] = e < left ? p[e] : 0.0f;
      }
    }
  }
}

template <int DT, int V>
__device__ __forceinline__ void store_row(void* base, int64_t idx, int left, const float (&o)[V]) {
  if constexpr (DT == GASLOC_BF16) {
    uint16_t* p = static_cast<uint16_t*>(base) + idx;
    uint32_t h[V / 2];
#pragma unroll
    for (int k = 0; k < V / 2; ++k) h[k] = f32x2_to_bf16x2(o[2 * k], o[2 * k + 1]);
    if (left >= V) {
      if constexpr (V == 8)
        store_words4(p, u32x4{h[0], h[1], h[2], h[3]});
      else
        store_words2(p, u32x2{h[0], h[1]});
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (k < left) p[k] = static_cast<uint16_t>(h[k / 2] >> (16 * (k & 1)));
    }
  } else {
    float* p = static_cast<float*>(base) + idx;
#pragma unroll
    for (int k = 0; k < V; k += 4) {
      if (left >= k + 4) {
        store_words4(p + k, __builtin_bit_cast(u32x4, f32x4{o[k], o[k + 1], o[k + 2], o[k + 3]}));
      } else {
#pragma unroll
        for (int e = k; e < k + 4; ++e)
          if (e < left) p[e] = o[e];
      }
    }
  }
}

// Sum over the wave, the same in every lane: DPP shifts inside each row of 16
// lanes, then the four row sums in order.
__device__ __forceinline__ float wave_sum_f32(float v) {
  const auto shifted = [](float x, auto k) {
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x110 + decltype(k)::value, 0xf, 0xf, true));
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
