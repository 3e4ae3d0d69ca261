// Lines of a cache between memory and a wave's registers, 16 values to a lane.
#pragma once

#include "pbz_cache_internal.h"
#include "pbz_device.h"
#include "pbz_line_transform.h"

namespace pbz {

// 16 neighbouring elements of bfloat16 or FP16 as T; `wide`: the address is a multiple of 16 bytes
template <typename T>
__device__ __forceinline__ void load_run_16(const void* p, int type, int64_t at, bool wide, T (&v)[16]) {
  const uint16_t* x = static_cast<const uint16_t*>(p) + at;
  uint32_t w[8];
  if (wide) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const uint4 u = *reinterpret_cast<const uint4*>(x + 2 * i);
      w[i] = u.x;
      w[i + 1] = u.y;
      w[i + 2] = u.z;
      w[i + 3] = u.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = uint32_t(x[2 * i]) | (uint32_t(x[2 * i + 1]) << 16);
  }
  if (type == PBZ_BF16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[2 * i] = T(__uint_as_float(w[i] << 16));
      v[2 * i + 1] = T(__uint_as_float(w[i] & 0xffff0000u));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[2 * i] = T(float(__builtin_bit_cast(_Float16, uint16_t(w[i]))));
      v[2 * i + 1] = T(float(__builtin_bit_cast(_Float16, uint16_t(w[i] >> 16))));
    }
  }
}

// and of any type
template <typename T>
__device__ __forceinline__ void load_run(const void* p, int type, int64_t at, bool wide, T (&v)[16]) {
  if (type == PBZ_F64) {
    const double* x = static_cast<const double*>(p) + at;
    if (wide) {
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const double2 u = *reinterpret_cast<const double2*>(x + i);
        v[i] = T(u.x);
        v[i + 1] = T(u.y);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = T(x[i]);
    }
  } else if (type == PBZ_F32) {
    const float* x = static_cast<const float*>(p) + at;
    if (wide) {
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float4 u = *reinterpret_cast<const float4*>(x + i);
        v[i] = T(u.x);
        v[i + 1] = T(u.y);
        v[i + 2] = T(u.z);
        v[i + 3] = T(u.w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = T(x[i]);
    }
  } else {
    load_run_16(p, type, at, wide, v);
  }
}

// The largest of L lanes' values, in all of them: register moves to another lane of the pair, of four, and the mirrored ones of 8 and 16
template <int L, typename T>
__device__ __forceinline__ T lanes_max(T v) {
  if constexpr (L >= 2) v = fmax(v, line::moved<0xB1>(v));
  if constexpr (L >= 4) v = fmax(v, line::moved<0x4E>(v));
  if constexpr (L >= 8) v = fmax(v, line::moved<0x141>(v));
  if constexpr (L >= 16) v = fmax(v, line::moved<0x140>(v));
  return v;
}

// The largest magnitude of a line, the same in its L lanes; infinite if a value is not finite.
template <typename T, int L>
__device__ __forceinline__ T line_max(const T (&v)[16]) {
  T most = T(0), nought = T(0);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    most = fmax(most, fabs(v[i]));
    nought = fma(v[i], T(0), nought);      // not a number if some value is not, or is infinite
  }
  return lanes_max<L>(nought == T(0) ? most : T(__builtin_huge_valf()));
}

// 16 neighbouring elements of bfloat16 or FP16; `wide` as above
__device__ __forceinline__ void store_run(uint16_t* out, int type, bool wide, const float (&v)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    uint16_t x, y;
    if (type == PBZ_BF16) {
      x = float_to_bf16_bits(v[2 * k]);
      y = float_to_bf16_bits(v[2 * k + 1]);
    } else {
      x = __builtin_bit_cast(uint16_t, _Float16(v[2 * k]));
      y = __builtin_bit_cast(uint16_t, _Float16(v[2 * k + 1]));
    }
    w[k] = uint32_t(x) | (uint32_t(y) << 16);
  }
  if (wide) {
#pragma unroll
    for (int i = 0; i < 2; ++i) reinterpret_cast<uint4*>(out)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      out[2 * k] = uint16_t(w[k]);
      out[2 * k + 1] = uint16_t(w[k] >> 16);
    }
  }
}

}  // namespace pbz
