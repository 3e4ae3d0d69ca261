// The orthonormal transforms of a line of 16 L values that L neighbouring lanes hold, 16 consecutive values each.
//
// A DCT-II of n values splits into two of n / 2 (unnormalised: c_n[q] = sum_m x[m] cos(pi (2m+1) q / (2n))):
//   s[m] = x[m] + x[n-1-m]:                          c_n[2k]   = c_{n/2}(s)[k]
//   d[m] = (x[m] - x[n-1-m]) / (2 cos(pi (2m+1) / (2n))):  c_n[2k+1] = c_{n/2}(d)[k] + c_{n/2}(d)[k+1]
// the latter because 2 cos(t) cos((2k+1) t) = cos(2k t) + cos(2(k+1) t).  With lane l holding x[16 l ..], x[n-1-m] is in the
// mirrored lane, so a split is one exchange with it, after which the lower half of the lanes has s and the upper half d: a value, plus or minus
// the mirrored lane's, times a lane's factor.  Then the upper half's lanes are in mirrored order, and so are the values within each.  log2(L)
// splits leave every lane a line of 16, which the in-register transform of pbz_dct.h takes; where the 16 are in mirrored order, the
// coefficients of odd index change their sign.  The sums over k and k + 1 are again with one neighbour each.  All of that is without the
// orthonormal transform's factors: sqrt(1/2) for every split is in the lanes' factors, and the first coefficient's is set right before and after
// the sums.  Exchanges among up to eight lanes are register moves (the neighbours' sums of 16 lanes
// go through LDS).  The inverse is the transpose, step by step in reverse.  The factors reach n / pi, which costs that many
// roundings' accuracy at worst: nothing in FP64, and in FP32 for n = 256 still 2^-17 of the line's norm.
// (With selects between sums and differences, and the orthonormal factors at every step: FP64 as 9 instructions a value and split and 9 a value
// and sum, 4 and 4 now.)
// 16 values to a lane: with 32, one split less, but an in-register transform of 341 multiply-adds instead of 85 and twice the code, which a
// launch over few lines fetches for nearly as long as it computes (keys and values of 64 tokens, before the splits were as they are: 9.2 us, 6.7 with
// 16; over many lines the two were the same).
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

// A lane's part in the splits.  Split i is of L >> i lanes: which half of them the lane is in, and the index
// that its results have among the half's, modulo the half's lanes.
template <int L>
struct Path {
  int half[4] = {0, 0, 0, 0}, index[5] = {0, 0, 0, 0, 0};
  __device__ __forceinline__ explicit Path(int lane) {
    int p = lane;
#pragma unroll
    for (int n = L, i = 0; n > 1; n >>= 1, ++i) {
      half[i] = p >= n / 2;
      p = half[i] ? n - 1 - p : p;
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

// What the lanes' values are multiplied by at each split: sqrt(1/2), in the upper half over 2 cos(pi (2m+1) / (2n)), and negative, since it is the
// mirrored lane's value minus its own that is wanted.
template <typename T, int L>
struct alignas(32) Factors {
  static constexpr int kSplits = L == 16 ? 4 : L == 8 ? 3 : L == 4 ? 2 : 1;
  static constexpr int kWide = 16 / sizeof(T);      // to a load; the lanes' side by side
  T v[kSplits * L * kRun];
  constexpr Factors() : v() {
    for (int lane = 0; lane < L; ++lane) {
      int place = lane;
      bool mirrored = false;
      for (int split = 0, n = L; split < kSplits; ++split, n /= 2) {
        const bool upper = place >= n / 2;
        if (upper) {
          place = n - 1 - place;
          mirrored = !mirrored;
        }
        for (int i = 0; i < kRun; ++i) {
          const int m = place * kRun + (mirrored ? kRun - 1 - i : i);
          v[((split * (kRun / kWide) + i / kWide) * L + lane) * kWide + i % kWide] = T(upper ? -dct::kInvSqrt2 * 0.5 / dct::cos_frac(2 * m + 1, n * kRun) : dct::kInvSqrt2);
        }
      }
    }
  }
};
template <typename T, int L>
static __device__ const Factors<T, L> kFactors = Factors<T, L>();

// a lane's factors at a split, read all at once
template <typename T, int L>
__device__ __forceinline__ void factors(T (&f)[kRun], int split, int lane) {
  constexpr int kWide = Factors<T, L>::kWide;
  typedef T Wide __attribute__((ext_vector_type(kWide)));
  const Wide* table = reinterpret_cast<const Wide*>(kFactors<T, L>.v) + split * (kRun / kWide) * L + lane;
#pragma unroll
  for (int i = 0; i < kRun / kWide; ++i) {
    const Wide u = table[i * L];
#pragma unroll
    for (int j = 0; j < kWide; ++j) f[kWide * i + j] = u[j];
  }
}

template <typename T, int n, int L>       // n lanes of L
__device__ __forceinline__ void split(T (&v)[kRun], int which, int half, int lane) {
  T f[kRun];
  factors<T, L>(f, which, lane);
  const T side = half ? T(-1) : T(1);
#pragma unroll
  for (int i = 0; i < kRun / 2; ++i) {
    const int j = kRun - 1 - i;
    const T ti = moved<Mirror<n>::control>(v[i]), tj = moved<Mirror<n>::control>(v[j]);
    v[i] = (v[i] + tj * side) * f[i];
    v[j] = (v[j] + ti * side) * f[j];
  }
}
template <typename T, int n, int L>
__device__ __forceinline__ void unsplit(T (&v)[kRun], int which, int half, int lane) {
  T f[kRun];
  factors<T, L>(f, which, lane);
  const T side = half ? T(1) : T(-1);                     // the mirrored lane's
#pragma unroll
  for (int i = 0; i < kRun; ++i) v[i] *= f[i];
#pragma unroll
  for (int i = 0; i < kRun / 2; ++i) {
    const int j = kRun - 1 - i;
    const T ti = moved<Mirror<n>::control>(v[i]), tj = moved<Mirror<n>::control>(v[j]);
    v[i] = v[i] + tj * side;
    v[j] = v[j] + ti * side;
  }
}

// Coefficients from those of the halves: the upper half's are sums with the next one's, index k (n / 2) + t of the half's, which the lane with
// t + 1 has, and for the last t the one with t = 0 under k + 1.
template <typename T, int n, int L>
__device__ __forceinline__ void join(T (&v)[kRun], int half, int t, int lane) {
  if constexpr (n == 2) {
    const T with = half ? T(1) : T(0);
#pragma unroll
    for (int k = 0; k < kRun - 1; ++k) v[k] = v[k] + v[k + 1] * with;
  } else {
    const int source = n == 16 ? lane_of_index(lane, t + 1) : 0;
    const bool last = t == n / 2 - 1;
    const T same = half && !last ? T(1) : T(0), above = half && last ? T(1) : T(0);
    T next = neighbour<n, L, 1>(v[0], source, lane);
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
      v[k] = v[k] + next * same;
      if (k < kRun - 1) {
        next = neighbour<n, L, 1>(v[k + 1], source, lane);
        v[k] = v[k] + next * above;
      }
    }
  }
}
template <typename T, int n, int L>
__device__ __forceinline__ void unjoin(T (&v)[kRun], int half, int t, int lane) {
  if constexpr (n == 2) {
    const T with = half ? T(1) : T(0);
#pragma unroll
    for (int k = kRun - 1; k > 0; --k) v[k] = v[k] + v[k - 1] * with;
  } else {
    const int source = n == 16 ? lane_of_index(lane, t - 1) : 0;
    const T same = half && t != 0 ? T(1) : T(0), below = half && t == 0 ? T(1) : T(0);
    T previous = neighbour<n, L, -1>(v[kRun - 1], source, lane);
#pragma unroll
    for (int k = kRun - 1; k >= 0; --k) {
      v[k] = v[k] + previous * same;
      if (k > 0) {
        previous = neighbour<n, L, -1>(v[k - 1], source, lane);
        v[k] = v[k] + previous * below;
      }
    }
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

// of values in mirrored order
template <typename T, int L>
__device__ __forceinline__ void odd_signs(T (&v)[kRun], const Path<L>& path) {
  const T sign = (path.half[0] + path.half[1] + path.half[2] + path.half[3]) & 1 ? T(-1) : T(1);
#pragma unroll
  for (int k = 1; k < kRun; k += 2) v[k] *= sign;
}

// lane: of the wave; a line's lanes start at a multiple of L
template <int kTf, typename T, int L>
__device__ __forceinline__ void forward(T (&v)[kRun], int lane) {
  const int part = lane % L;
  if constexpr (kTf == kTfDct) {
    const Path<L> path(part);
    if constexpr (L >= 16) split<T, 16, L>(v, 0, path.half[0], part);
    if constexpr (L >= 8) split<T, 8, L>(v, kLevel<8, L>, path.half[kLevel<8, L>], part);
    if constexpr (L >= 4) split<T, 4, L>(v, kLevel<4, L>, path.half[kLevel<4, L>], part);
    split<T, 2, L>(v, kLevel<2, L>, path.half[kLevel<2, L>], part);
    dct::forward<T, kRun, 1>(v);
    odd_signs<T, L>(v, path);
    v[0] *= T(2.0 * dct::kInvSqrt2);
    join<T, 2, L>(v, path.half[kLevel<2, L>], path.index[kLevel<2, L>], lane);
    if constexpr (L >= 4) join<T, 4, L>(v, path.half[kLevel<4, L>], path.index[kLevel<4, L>], lane);
    if constexpr (L >= 8) join<T, 8, L>(v, path.half[kLevel<8, L>], path.index[kLevel<8, L>], lane);
    if constexpr (L >= 16) join<T, 16, L>(v, path.half[0], path.index[0], lane);
    v[0] *= part == 0 ? T(dct::kInvSqrt2) : T(1);
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
    v[0] *= part == 0 ? T(dct::kInvSqrt2) : T(1);
    if constexpr (L >= 16) unjoin<T, 16, L>(v, path.half[0], path.index[0], lane);
    if constexpr (L >= 8) unjoin<T, 8, L>(v, path.half[kLevel<8, L>], path.index[kLevel<8, L>], lane);
    if constexpr (L >= 4) unjoin<T, 4, L>(v, path.half[kLevel<4, L>], path.index[kLevel<4, L>], lane);
    unjoin<T, 2, L>(v, path.half[kLevel<2, L>], path.index[kLevel<2, L>], lane);
    odd_signs<T, L>(v, path);
    v[0] *= T(2.0 * dct::kInvSqrt2);
    dct::inverse<T, kRun, 1, kRun>(v);
    unsplit<T, 2, L>(v, kLevel<2, L>, path.half[kLevel<2, L>], part);
    if constexpr (L >= 4) unsplit<T, 4, L>(v, kLevel<4, L>, path.half[kLevel<4, L>], part);
    if constexpr (L >= 8) unsplit<T, 8, L>(v, kLevel<8, L>, path.half[kLevel<8, L>], part);
    if constexpr (L >= 16) unsplit<T, 16, L>(v, 0, path.half[0], part);
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
