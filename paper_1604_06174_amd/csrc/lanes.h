// Exchanges between the lanes of a wavefront in the vector unit itself (DPP and
// the row swaps of gfx950): a few cycles each, where a lane permutation through
// LDS takes about a hundred.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace ckpt {

// a's rows (OFF = 16: of sixteen lanes; 32: halves) of odd number and b's of even
// number change places
template <int OFF>
__device__ __forceinline__ void swap_rows(float &a, float &b) {
  static_assert(OFF == 16 || OFF == 32, "rows of 16 or 32 lanes");
  if (OFF == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
  } else {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
  }
}

// v of lane ^ OFF, OFF = 1, 2, 4 or 8
template <int OFF>
__device__ __forceinline__ float lane_xor(float v) {
  static_assert(OFF == 1 || OFF == 2 || OFF == 4 || OFF == 8, "within a row of sixteen lanes");
  const int x = __float_as_int(v);
  if (OFF == 1) return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true));  // quad [1, 0, 3, 2]
  if (OFF == 2) return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true));  // quad [2, 3, 0, 1]
  if (OFF == 8) return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, true));  // rotated by 8
  // four to the left for the even quads, to the right for the odd ones
  const int l = __builtin_amdgcn_update_dpp(x, x, 0x104, 0xf, 0x5, false);
  return __int_as_float(__builtin_amdgcn_update_dpp(l, x, 0x114, 0xf, 0xa, false));
}

// v + v of lane ^ OFF, the same bits in both
template <int OFF>
__device__ __forceinline__ float xor_add(float v) {
  if constexpr (OFF >= 16) {
    float w = v;
    swap_rows<OFF>(v, w);
    return v + w;
  } else {
    return v + lane_xor<OFF>(v);
  }
}

// The sums over the lanes that differ in the bits from `low` (a power of two) up, and
// in those below `high`.  Every step is taken and selected: a few cycles, where a
// branch may wait for the instruction cache.
template <int N>
__device__ __forceinline__ void add_from(int low, float (&v)[N]) {
  auto step = [&](auto off) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float t = xor_add<decltype(off)::value>(v[k]);
      v[k] = low <= off ? t : v[k];
    }
  };
  step(std::integral_constant<int, 32>());
  step(std::integral_constant<int, 16>());
  step(std::integral_constant<int, 8>());
  step(std::integral_constant<int, 4>());
  step(std::integral_constant<int, 2>());
  step(std::integral_constant<int, 1>());
}

template <int N>
__device__ __forceinline__ void add_below(int high, float (&v)[N]) {
  auto step = [&](auto off) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float t = xor_add<decltype(off)::value>(v[k]);
      v[k] = high > off ? t : v[k];
    }
  };
  step(std::integral_constant<int, 1>());
  step(std::integral_constant<int, 2>());
  step(std::integral_constant<int, 4>());
  step(std::integral_constant<int, 8>());
  step(std::integral_constant<int, 16>());
  step(std::integral_constant<int, 32>());
}

// One step of wave_columns: the values' halves change sides, so that each lane
// goes on with half of them.  id: the number of the first value a lane holds.
template <int NVAL, int OFF>
__device__ __forceinline__ void halve(float (&val)[NVAL], int &cnt, int &id, int lane, int VC) {
  constexpr int DONE = OFF == 32 ? 1 : OFF == 16 ? 2 : OFF == 8 ? 4 : OFF == 4 ? 8 : OFF == 2 ? 16 : 32;
  constexpr int C = NVAL / DONE > 1 ? NVAL / DONE : 1;  // values held before this step
  if (VC > OFF) return;
  if constexpr (C == 1) {
    val[0] = xor_add<OFF>(val[0]);
  } else {
    const bool up = lane & OFF;
#pragma unroll
    for (int k = 0; k < C / 2; ++k) {
      if constexpr (OFF >= 16) {
        float a = val[k], b = val[C / 2 + k];
        swap_rows<OFF>(a, b);
        val[k] = a + b;
      } else {
        const float keep = up ? val[C / 2 + k] : val[k], give = up ? val[k] : val[C / 2 + k];
        val[k] = keep + lane_xor<OFF>(give);
      }
    }
    cnt = C / 2;
    id += up ? C / 2 : 0;
  }
}

// Sums of a wavefront's rows (VC a power of two), NVAL = 1, 2, 4, 8 or 16 values a
// thread: value k of column tx goes to out[k VC + tx].
template <int NVAL>
__device__ __forceinline__ void wave_columns(float (&val)[NVAL], int lane, int VC, int tx, float *out) {
  int cnt = NVAL, id = 0;
  halve<NVAL, 32>(val, cnt, id, lane, VC);
  halve<NVAL, 16>(val, cnt, id, lane, VC);
  halve<NVAL, 8>(val, cnt, id, lane, VC);
  halve<NVAL, 4>(val, cnt, id, lane, VC);
  halve<NVAL, 2>(val, cnt, id, lane, VC);
  halve<NVAL, 1>(val, cnt, id, lane, VC);
  // lanes that hold the same value write the same sum
#pragma unroll
  for (int k = 0; k < NVAL; ++k)
    if (k < cnt) out[(id + k) * VC + tx] = val[k];
}

}  // namespace ckpt
