// The orthonormal transforms of a line of 32 L values that L neighbouring lanes hold, 32 consecutive values each.
//
// A DCT-II of n values splits into two of n / 2 (unnormalised: c_n[q] = sum_m x[m] cos(pi (2m+1) q / (2n))):
//   s[m] = x[m] + x[n-1-m]:                          c_n[2k]   = c_{n/2}(s)[k]
//   d[m] = (x[m] - x[n-1-m]) / (2 cos(pi (2m+1) / (2n))):  c_n[2k+1] = c_{n/2}(d)[k] + c_{n/2}(d)[k+1]
// the latter because 2 cos(t) cos((2k+1) t) = cos(2k t) + cos(2(k+1) t).  With lane l holding x[32 l ..], x[n-1-m] is in the
// mirrored lane, so a split is one exchange with it, after which the lower half of the lanes has s and the upper half, in mirrored
// order, has d; log2(L) splits leave every lane a line of 32, which the in-register transform of pbz_dct.h takes.  The sums over
// k and k + 1 are again with one neighbour each.  All exchanges stay within eight lanes: register moves, no LDS.  The inverse is
// the transpose, step by step in reverse.  Cost per lane and split: 32 exchanges, additions and multiplications, against 64 / 128 /
// 256 multiply-adds a value for the product with the matrix.  The factors reach n / pi, which costs that many roundings'
// accuracy at worst: nothing in FP64, and in FP32 for n = 256 still 2^-17 of the line's norm.
//
// Haar: 32 values within a lane, then the lanes' sums among each other.
#pragma once

#include "pbz_dct.h"
#include "pbz_haar.h"

namespace pbz {
namespace line {

template <int kControl>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(0, int(__float_as_uint(v)), kControl, 0xf, 0xf, true)));
}
template <int kControl>
__device__ __forceinline__ double moved(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(u)), kControl, 0xf, 0xf, true));
  const uint32_t hi = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(u >> 32)), kControl, 0xf, 0xf, true));
  return __builtin_bit_cast(double, uint64_t(lo) | (uint64_t(hi) << 32));
}

// DPP controls: the mirrored lane among n lanes, and in the upper half of n lanes the one that holds the next / previous index
template <int n> struct Mirror { static constexpr int control = n == 2 ? 0xB1 : n == 4 ? 0x1B : 0x141; };
template <int n> struct Next { static constexpr int control = n == 4 ? 0xB1 : 0x1E; };
template <int n> struct Previous { static constexpr int control = n == 4 ? 0xB1 : 0x4B; };

// 1 / (2 cos(pi (2m+1) / (2n))) for m < n / 2, n = 64, 128, 256 one after the other
template <typename T>
struct alignas(32) Secants {
  T v[32 + 64 + 128];
  constexpr Secants() : v() {
    int at = 0;
    for (int n = 64; n <= 256; n *= 2)
      for (int m = 0; m < n / 2; ++m) v[at++] = T(0.5 / dct::cos_frac(2 * m + 1, n));
  }
};
static __device__ const Secants<float> kSecantsF32 = Secants<float>();
static __device__ const Secants<double> kSecantsF64 = Secants<double>();
__device__ __forceinline__ const float* secants(float) { return kSecantsF32.v; }
__device__ __forceinline__ const double* secants(double) { return kSecantsF64.v; }

// a lane's part in the splits: position in its half at every split, and which half
template <int L>
struct Path {
  int place[4] = {0, 0, 0, 0};     // after split i: position among the L >> (i + 1) lanes of its half
  int half[3] = {0, 0, 0};
  __device__ __forceinline__ explicit Path(int lane) {
    int p = lane;
#pragma unroll
    for (int n = L, i = 0; n > 1; n >>= 1, ++i) {
      half[i] = p >= n / 2;
      p = half[i] ? n - 1 - p : p;
      place[i] = p;
    }
  }
};

// the 32 factors of a lane at the split of n lanes (1 where it has the sums), read all at once
template <typename T, int n>
__device__ __forceinline__ void factors(T (&f)[32], int half, int place) {
  typedef T Four __attribute__((ext_vector_type(4)));
  const Four* table = reinterpret_cast<const Four*>(secants(T()) + (n == 2 ? 0 : n == 4 ? 32 : 96) + 32 * place);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const Four u = table[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) f[4 * i + j] = half ? u[j] : T(1);
  }
}

template <typename T, int n>       // n lanes
__device__ __forceinline__ void split(T (&v)[32], int half, int place) {
  T f[32];
  factors<T, n>(f, half, place);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int j = 31 - i;
    const T ti = moved<Mirror<n>::control>(v[i]), tj = moved<Mirror<n>::control>(v[j]);
    const T si = v[i] + tj, sj = v[j] + ti, di = ti - v[j], dj = tj - v[i];
    v[i] = (half ? di : si) * f[i];
    v[j] = (half ? dj : sj) * f[j];
  }
}
template <typename T, int n>
__device__ __forceinline__ void unsplit(T (&v)[32], int half, int place) {
  T f[32];
  factors<T, n>(f, half, place);
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] *= f[i];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int j = 31 - i;
    const T ti = moved<Mirror<n>::control>(v[i]), tj = moved<Mirror<n>::control>(v[j]);
    const T si = v[i] + ti, sj = v[j] + tj, di = tj - v[j], dj = ti - v[i];
    v[i] = half ? di : si;
    v[j] = half ? dj : sj;
  }
}

// index among the coefficients of its half: k (n / 2) + t
template <typename T, int n>
__device__ __forceinline__ void join(T (&v)[32], int half, int t) {
  const T r = T(dct::kInvSqrt2), first = t == 0 ? T(1) : r;      // sqrt(2) times r at index 0
  T next = T(0);
  if constexpr (n > 2) next = moved<Next<n>::control>(v[0]);
#pragma unroll
  for (int k = 0; k < 32; ++k) {
    T after = T(0);
    if (k < 31) {
      if constexpr (n > 2) after = moved<Next<n>::control>(v[k + 1]);
      else after = v[k + 1];
    }
    const T other = n > 2 && t != n / 2 - 1 ? next : after;
    const T own = k == 0 ? v[k] * first : v[k] * r;
    v[k] = half ? own + other * r : v[k] * r;
    next = after;
  }
}
template <typename T, int n>
__device__ __forceinline__ void unjoin(T (&v)[32], int half, int t) {
  const T r = T(dct::kInvSqrt2), first = t == 0 ? T(1) : r;
  T previous = T(0);
  if constexpr (n > 2) previous = moved<Previous<n>::control>(v[31]);
#pragma unroll
  for (int k = 31; k >= 0; --k) {
    T before = T(0);
    if (k > 0) {
      if constexpr (n > 2) before = moved<Previous<n>::control>(v[k - 1]);
      else before = v[k - 1];
    }
    const T other = n > 2 && t != 0 ? previous : before;
    const T own = k == 0 ? v[k] * first : v[k] * r;
    v[k] = half ? own + other * r : v[k] * r;
    previous = before;
  }
}

template <int kTf, int L>
__device__ __forceinline__ int coefficient(int lane, int k) {     // which one v[k] is after forward()
  if constexpr (kTf == kTfDct) {
    const Path<L> path(lane);
    return k * L + path.half[0] + 2 * path.half[1] + 4 * path.half[2];
  } else {
    if (k == 0) {
      if (lane == 0) return 0;
      const int bit = lane & -lane;
      return L / (2 * bit) + lane / (2 * bit);
    }
    const int run = 1 << (31 - __builtin_clz(unsigned(k)));
    return run * L + lane * run + (k - run);
  }
}

template <int kTf, typename T, int L>
__device__ __forceinline__ void forward(T (&v)[32], int lane) {
  if constexpr (kTf == kTfDct) {
    const Path<L> path(lane);
    if constexpr (L >= 8) split<T, 8>(v, path.half[0], path.place[0]);
    if constexpr (L >= 4) split<T, 4>(v, path.half[L >= 8 ? 1 : 0], path.place[L >= 8 ? 1 : 0]);
    if constexpr (L >= 2) split<T, 2>(v, path.half[L >= 8 ? 2 : L >= 4 ? 1 : 0], path.place[L >= 8 ? 2 : L >= 4 ? 1 : 0]);
    dct::forward<T, 32, 1>(v);
    if constexpr (L >= 2) join<T, 2>(v, path.half[L >= 8 ? 2 : L >= 4 ? 1 : 0], 0);
    if constexpr (L >= 4) join<T, 4>(v, path.half[L >= 8 ? 1 : 0], path.half[L >= 8 ? 2 : 1]);
    if constexpr (L >= 8) join<T, 8>(v, path.half[0], path.half[1] + 2 * path.half[2]);
  } else {
    haar::forward<T, 32, 1>(v);
    T sum = v[0];
    v[0] = T(0);
#pragma unroll
    for (int bit = 1; bit < L; bit <<= 1) {
      const T other = __shfl_xor(sum, bit);
      if ((lane & (2 * bit - 1)) == bit) v[0] = (other - sum) * T(dct::kInvSqrt2);
      sum = (sum + other) * T(dct::kInvSqrt2);
    }
    if (lane == 0) v[0] = sum;
  }
}
template <int kTf, typename T, int L>
__device__ __forceinline__ void inverse(T (&v)[32], int lane) {
  if constexpr (kTf == kTfDct) {
    const Path<L> path(lane);
    if constexpr (L >= 8) unjoin<T, 8>(v, path.half[0], path.half[1] + 2 * path.half[2]);
    if constexpr (L >= 4) unjoin<T, 4>(v, path.half[L >= 8 ? 1 : 0], path.half[L >= 8 ? 2 : 1]);
    if constexpr (L >= 2) unjoin<T, 2>(v, path.half[L >= 8 ? 2 : L >= 4 ? 1 : 0], 0);
    dct::inverse<T, 32, 1, 32>(v);
    if constexpr (L >= 2) unsplit<T, 2>(v, path.half[L >= 8 ? 2 : L >= 4 ? 1 : 0], path.place[L >= 8 ? 2 : L >= 4 ? 1 : 0]);
    if constexpr (L >= 4) unsplit<T, 4>(v, path.half[L >= 8 ? 1 : 0], path.place[L >= 8 ? 1 : 0]);
    if constexpr (L >= 8) unsplit<T, 8>(v, path.half[0], path.place[0]);
  } else {
    T value = v[0];
#pragma unroll
    for (int bit = L / 2; bit > 0; bit >>= 1) {
      const T other = __shfl_xor(value, bit);
      const int place = lane & (2 * bit - 1);
      if (place == 0) value = (value + other) * T(dct::kInvSqrt2);
      if (place == bit) value = (other - value) * T(dct::kInvSqrt2);
    }
    v[0] = value;
    haar::inverse<T, 32, 1, 32>(v);
  }
}

}  // namespace line
}  // namespace pbz
