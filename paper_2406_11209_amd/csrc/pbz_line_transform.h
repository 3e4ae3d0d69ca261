// The orthonormal transforms of a line of 16 L values that L neighbouring lanes hold, 16 consecutive values each.
//
// A DCT-II of n values splits into two of n / 2 (unnormalised: c_n[q] = sum_m x[m] cos(pi (2m+1) q / (2n))):
//   s[m] = x[m] + x[n-1-m]:                          c_n[2k]   = c_{n/2}(s)[k]
//   d[m] = (x[m] - x[n-1-m]) / (2 cos(pi (2m+1) / (2n))):  c_n[2k+1] = c_{n/2}(d)[k] + c_{n/2}(d)[k+1]
// the latter because 2 cos(t) cos((2k+1) t) = cos(2k t) + cos(2(k+1) t).  With lane l holding x[16 l ..], x[n-1-m] is in the
// mirrored lane, so a split is one exchange with it, after which the lower half of the lanes has s and the upper half, in mirrored
// order, has d; log2(L) splits leave every lane a line of 16, which the in-register transform of pbz_dct.h takes.  The sums over
// k and k + 1 are again with one neighbour each.  Exchanges among up to eight lanes are register moves (the neighbours' sums of 16 lanes
// go through LDS).  The inverse is the transpose, step by step in reverse.  The factors reach n / pi, which costs that many
// roundings' accuracy at worst: nothing in FP64, and in FP32 for n = 256 still 2^-17 of the line's norm.
// 16 values to a lane: with 32, one split less, but an in-register transform of 341 multiply-adds instead of 85 and twice the code, which a
// launch over few lines fetches for nearly as long as it computes (128 keys and values of 64 tokens: 9.2 us, 6.7 with 16; over many lines the two
// are the same).
//
// Haar: 16 values within a lane, then the lanes' sums among each other.
#pragma once

#include "pbz_dct.h"
#include "pbz_haar.h"

namespace pbz {
namespace line {

constexpr int kRun = 16;      // values to a lane

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

// DPP control of the mirrored lane among n lanes
template <int n> struct Mirror { static constexpr int control = n == 2 ? 0xB1 : n == 4 ? 0x1B : n == 8 ? 0x141 : 0x140; };

// A lane's part in the splits.  Split i is of L >> i lanes: which half of them the lane is in, its place among that half, and the index
// that its results have among the half's, modulo the half's lanes.
template <int L>
struct Path {
  int half[4] = {0, 0, 0, 0}, place[4] = {0, 0, 0, 0}, index[5] = {0, 0, 0, 0, 0};
  __device__ __forceinline__ explicit Path(int lane) {
    int p = lane;
#pragma unroll
    for (int n = L, i = 0; n > 1; n >>= 1, ++i) {
      half[i] = p >= n / 2;
      p = half[i] ? n - 1 - p : p;
      place[i] = p;
    }
#pragma unroll
    for (int i = 3; i >= 0; --i) index[i] = i + 1 < 4 ? half[i + 1] + 2 * index[i + 1] : 0;
  }
  __device__ __forceinline__ int all() const { return half[0] + 2 * index[0]; }
};

// v of the upper half's lane with the next (kStep 1) or the previous (-1) index, of a split of n lanes of L; what the lower half gets does
// not matter.  (The second eight of 16 lanes are mirrored, where next and previous change places.)
template <int n, int L, int kStep, typename T>
__device__ __forceinline__ T neighbour(T v, int source, int lane) {
  if constexpr (n == 4) return moved<0xB1>(v);
  else if constexpr (n == 8 && L == 8) return moved<(kStep > 0 ? 0x1E : 0x4B)>(v);
  else if constexpr (n == 8) {
    const T up = moved<(kStep > 0 ? 0x1E : 0x4B)>(v), down = moved<(kStep > 0 ? 0x4B : 0x1E)>(v);
    return lane & 8 ? down : up;
  } else return __shfl(v, source);
}
// That lane among 16: of the upper eight, by the index that it should have.  (The places 0 .. 7 (lanes 15 .. 8) have indices 0, 4, 6, 2, 3, 7, 5, 1.)
__device__ __forceinline__ int lane_of_index(int lane, int index) {
  return (lane & ~15) + 15 - int((0x52614370u >> (4 * (index & 7))) & 7);
}

// 1 / (2 cos(pi (2m+1) / (2n))) for m < n / 2, n = 32, 64, 128, 256 one after the other
template <typename T>
struct alignas(32) Secants {
  T v[16 + 32 + 64 + 128];
  constexpr Secants() : v() {
    int at = 0;
    for (int n = 32; n <= 256; n *= 2)
      for (int m = 0; m < n / 2; ++m) v[at++] = T(0.5 / dct::cos_frac(2 * m + 1, n));
  }
};
static __device__ const Secants<float> kSecantsF32 = Secants<float>();
static __device__ const Secants<double> kSecantsF64 = Secants<double>();
__device__ __forceinline__ const float* secants(float) { return kSecantsF32.v; }
__device__ __forceinline__ const double* secants(double) { return kSecantsF64.v; }

// the factors of a lane at the split of n lanes (1 where it has the sums), read all at once
template <typename T, int n>
__device__ __forceinline__ void factors(T (&f)[kRun], int half, int place) {
  typedef T Four __attribute__((ext_vector_type(4)));
  const Four* table = reinterpret_cast<const Four*>(secants(T()) + (n / 2 - 1) * kRun + kRun * place);
#pragma unroll
  for (int i = 0; i < kRun / 4; ++i) {
    const Four u = table[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) f[4 * i + j] = half ? u[j] : T(1);
  }
}

template <typename T, int n>       // n lanes
__device__ __forceinline__ void split(T (&v)[kRun], int half, int place) {
  T f[kRun];
  factors<T, n>(f, half, place);
#pragma unroll
  for (int i = 0; i < kRun / 2; ++i) {
    const int j = kRun - 1 - i;
    const T ti = moved<Mirror<n>::control>(v[i]), tj = moved<Mirror<n>::control>(v[j]);
    const T si = v[i] + tj, sj = v[j] + ti, di = ti - v[j], dj = tj - v[i];
    v[i] = (half ? di : si) * f[i];
    v[j] = (half ? dj : sj) * f[j];
  }
}
template <typename T, int n>
__device__ __forceinline__ void unsplit(T (&v)[kRun], int half, int place) {
  T f[kRun];
  factors<T, n>(f, half, place);
#pragma unroll
  for (int i = 0; i < kRun; ++i) v[i] *= f[i];
#pragma unroll
  for (int i = 0; i < kRun / 2; ++i) {
    const int j = kRun - 1 - i;
    const T ti = moved<Mirror<n>::control>(v[i]), tj = moved<Mirror<n>::control>(v[j]);
    const T si = v[i] + ti, sj = v[j] + tj, di = tj - v[j], dj = ti - v[i];
    v[i] = half ? di : si;
    v[j] = half ? dj : sj;
  }
}

// index among the coefficients of the half: k (n / 2) + t
template <typename T, int n, int L>
__device__ __forceinline__ void join(T (&v)[kRun], int half, int t, int lane) {
  const T r = T(dct::kInvSqrt2), first = t == 0 ? T(1) : r;      // sqrt(2) times r at index 0
  const int source = n == 16 ? lane_of_index(lane, t + 1) : 0;
  T next = T(0);
  if constexpr (n > 2) next = neighbour<n, L, 1>(v[0], source, lane);
#pragma unroll
  for (int k = 0; k < kRun; ++k) {
    T after = T(0);
    if (k < kRun - 1) {
      if constexpr (n > 2) after = neighbour<n, L, 1>(v[k + 1], source, lane);
      else after = v[k + 1];
    }
    const T other = n > 2 && t != n / 2 - 1 ? next : after;
    const T own = k == 0 ? v[k] * first : v[k] * r;
    v[k] = half ? own + other * r : v[k] * r;
    next = after;
  }
}
template <typename T, int n, int L>
__device__ __forceinline__ void unjoin(T (&v)[kRun], int half, int t, int lane) {
  const T r = T(dct::kInvSqrt2), first = t == 0 ? T(1) : r;
  const int source = n == 16 ? lane_of_index(lane, t - 1) : 0;
  T previous = T(0);
  if constexpr (n > 2) previous = neighbour<n, L, -1>(v[kRun - 1], source, lane);
#pragma unroll
  for (int k = kRun - 1; k >= 0; --k) {
    T before = T(0);
    if (k > 0) {
      if constexpr (n > 2) before = neighbour<n, L, -1>(v[k - 1], source, lane);
      else before = v[k - 1];
    }
    const T other = n > 2 && t != 0 ? previous : before;
    const T own = k == 0 ? v[k] * first : v[k] * r;
    v[k] = half ? own + other * r : v[k] * r;
    previous = before;
  }
}

template <int kTf, int L>
__device__ __forceinline__ int coefficient(int lane, int k) {     // which one v[k] is after forward(); lane: of the line's
  if constexpr (kTf == kTfDct) {
    return k * L + Path<L>(lane).all();
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

template <int n, int L>
constexpr int kLevel = L / n >= 8 ? 3 : L / n >= 4 ? 2 : L / n >= 2 ? 1 : 0;      // which split the one of n lanes is

// lane: of the wave; a line's lanes start at a multiple of L
template <int kTf, typename T, int L>
__device__ __forceinline__ void forward(T (&v)[kRun], int lane) {
  const int part = lane % L;
  if constexpr (kTf == kTfDct) {
    const Path<L> path(part);
    if constexpr (L >= 16) split<T, 16>(v, path.half[0], path.place[0]);
    if constexpr (L >= 8) split<T, 8>(v, path.half[kLevel<8, L>], path.place[kLevel<8, L>]);
    if constexpr (L >= 4) split<T, 4>(v, path.half[kLevel<4, L>], path.place[kLevel<4, L>]);
    split<T, 2>(v, path.half[kLevel<2, L>], path.place[kLevel<2, L>]);
    dct::forward<T, kRun, 1>(v);
    join<T, 2, L>(v, path.half[kLevel<2, L>], path.index[kLevel<2, L>], lane);
    if constexpr (L >= 4) join<T, 4, L>(v, path.half[kLevel<4, L>], path.index[kLevel<4, L>], lane);
    if constexpr (L >= 8) join<T, 8, L>(v, path.half[kLevel<8, L>], path.index[kLevel<8, L>], lane);
    if constexpr (L >= 16) join<T, 16, L>(v, path.half[0], path.index[0], lane);
  } else {
    haar::forward<T, kRun, 1>(v);
    T sum = v[0];
    v[0] = T(0);
#pragma unroll
    for (int bit = 1; bit < L; bit <<= 1) {
      const T other = __shfl_xor(sum, bit);
      if ((part & (2 * bit - 1)) == bit) v[0] = (other - sum) * T(dct::kInvSqrt2);
      sum = (sum + other) * T(dct::kInvSqrt2);
    }
    if (part == 0) v[0] = sum;
  }
}
template <int kTf, typename T, int L>
__device__ __forceinline__ void inverse(T (&v)[kRun], int lane) {
  const int part = lane % L;
  if constexpr (kTf == kTfDct) {
    const Path<L> path(part);
    if constexpr (L >= 16) unjoin<T, 16, L>(v, path.half[0], path.index[0], lane);
    if constexpr (L >= 8) unjoin<T, 8, L>(v, path.half[kLevel<8, L>], path.index[kLevel<8, L>], lane);
    if constexpr (L >= 4) unjoin<T, 4, L>(v, path.half[kLevel<4, L>], path.index[kLevel<4, L>], lane);
    unjoin<T, 2, L>(v, path.half[kLevel<2, L>], path.index[kLevel<2, L>], lane);
    dct::inverse<T, kRun, 1, kRun>(v);
    unsplit<T, 2>(v, path.half[kLevel<2, L>], path.place[kLevel<2, L>]);
    if constexpr (L >= 4) unsplit<T, 4>(v, path.half[kLevel<4, L>], path.place[kLevel<4, L>]);
    if constexpr (L >= 8) unsplit<T, 8>(v, path.half[kLevel<8, L>], path.place[kLevel<8, L>]);
    if constexpr (L >= 16) unsplit<T, 16>(v, path.half[0], path.place[0]);
  } else {
    T value = v[0];
#pragma unroll
    for (int bit = L / 2; bit > 0; bit >>= 1) {
      const T other = __shfl_xor(value, bit);
      const int place = part & (2 * bit - 1);
      if (place == 0) value = (value + other) * T(dct::kInvSqrt2);
      if (place == bit) value = (other - value) * T(dct::kInvSqrt2);
    }
    v[0] = value;
    haar::inverse<T, kRun, 1, kRun>(v);
  }
}

}  // namespace line
}  // namespace pbz
