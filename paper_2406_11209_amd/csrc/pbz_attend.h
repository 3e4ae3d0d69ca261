// Attention over a paged compressed cache: the pass over keys and values (pbz_cache.h has the definition; pbz_cache.hip transforms the
// queries before, and joins the records after where positions are split).
//
// A wave takes 16 R query rows of one head of the cache and a run of positions, 16 positions to a matrix tile.
//   scores   S^T = K q^T on the integer matrix cores: K's indices go from memory to the operand as they are, 16 bytes a lane; a row
//            of q is 16-bit fixed point in two bytes, two products, 256 times the first plus the second, exact.  N and the row's
//            scale are applied to the sum, so a key costs no conversion.
//   softmax  with the running maximum and sum of its row.  A lane has 4 positions of one row per tile, so the maximum over
//            positions is across four lanes; it is only taken when some score passes the old maximum by 8 (a weight by 2^8),
//            which the wave votes on, so the usual tile exchanges nothing.  The sums stay per lane to the end.
//   values   O^T += V^T P^T in FP16 with FP32 sums: the weights, times N over the largest N so far (a power of two) and 2^7, are in
//            the registers where the product wants them (the order of positions within a product is free, as long as both operands
//            have the same); the largest is 2^15, and what is 2^-29 of it is still a normal FP16 number.  V's bytes become FP16 by a
//            permute and a multiply-add of two.
//   range    The largest N so far may be of a line that a row does not see, or sees with no weight, and then all of its weights would be
//            lost in FP16.  So it is checked that each row has a weight of 1 at least, where the references or the largest N change, which is
//            seldom.  While some row has none, the rows' largest weights are found at every step, and such rows have a factor of their own, a
//            power of two.  The check costs a prompt 0.5 % (712 -> 715 us), a single token of 300 positions 6 % (10.9 -> 11.6 us: code that is read
//            once); as one branch with the change that asks for it, and with nothing held in registers for it in the usual steps.
// Lanes 16 apart share a position's line: a line of 128 is one 128-byte read of 8 (keys) or 16 lanes (values).
#pragma once

#include "pbz_cache_lines.h"

namespace pbz {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kSlack = 8.f;          // by how much (in log2) a score may pass the maximum that the weights refer to

// N of values is taken relative to the next power of two of the largest so far, between these: what a row's own factor does not reach (below) is then
// 2^-71 and less, whatever N other rows see.
constexpr uint32_t kLeastWide = 0x33800000u, kMostWide = 0x4f800000u;      // 2^-24, 2^32
__device__ __forceinline__ float wide_unit(float wide) {
  const uint32_t up = (__float_as_uint(wide) + 0x7fffffu) & 0x7f800000u;
  return __uint_as_float(up > kMostWide ? kMostWide : up < kLeastWide ? kLeastWide : up);
}

// The exponent of a row's own factor, by its largest weight so far (or less): none from 1 to 2^15, where what is below FP16's normal numbers is off by
// 2^-25 of the largest at most.  Otherwise the largest becomes 2^10, or 2^14 where it is more, so that a row's total, which has the factor, too, keeps what
// weights of 2^-29 add to it.
__device__ __forceinline__ int fitting(float largest) {
  if (largest == 0.f || (largest >= 1.f && largest <= 32768.f)) return 0;
  const int exponent = int(__float_as_uint(largest) >> 23) - 127;
  return exponent > 0 ? 14 - exponent : exponent < -86 ? 96 : 10 - exponent;
}

// N of four neighbouring positions, as stored
template <int kN> struct Scales { using Raw = uint2; };
template <> struct Scales<PBZ_F32> { using Raw = f32x4; };
template <int kN>
__device__ __forceinline__ f32x4 scales(typename Scales<kN>::Raw u) {
  if constexpr (kN == PBZ_F32) {
    return u;
  } else if constexpr (kN == PBZ_BF16) {
    return f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                 __uint_as_float(u.y & 0xffff0000u)};
  } else {
    const f16x2 a = __builtin_bit_cast(f16x2, u.x), b = __builtin_bit_cast(f16x2, u.y);
    return f32x4{float(a[0]), float(a[1]), float(b[0]), float(b[1])};
  }
}

template <int kN>
__device__ __forceinline__ typename Scales<kN>::Raw load_N(const void* N, int64_t line, int quarter) {
  constexpr int kBytes = kN == PBZ_F32 ? 4 : 2;
  return *reinterpret_cast<const typename Scales<kN>::Raw*>(static_cast<const char*>(N) + line * kBytes + uint32_t(quarter * 4 * kBytes));
}

// the bytes of one position's values that a lane holds: D / 16 neighbouring coefficients
template <int D>
__device__ __forceinline__ void load_values(const int8_t* p, uint32_t (&w)[D >= 64 ? D / 64 : 1]) {
  if constexpr (D == 32) {
    w[0] = *reinterpret_cast<const uint16_t*>(p);
  } else if constexpr (D == 64) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (D == 128) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x;
    w[1] = u.y;
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x;
    w[1] = u.y;
    w[2] = u.z;
    w[3] = u.w;
  }
}

// Byte kByte of two words, biased by 128, as FP16: the bias off, and over 2^9.  A byte by itself is an FP16 subnormal, F + 128 times 2^-24; the
// product with 2^15, minus 128 times 2^-9, is exact.
constexpr float kValueUnit = 512.f;
template <int kByte>
__device__ __forceinline__ uint32_t two_values(uint32_t w0, uint32_t w1) {
  const f16x2 biased = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(w1, w0, 0x0c000c00u | ((4u + kByte) << 16) | kByte));
  const _Float16 up = _Float16(32768.f), down = _Float16(-0.25f);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(biased, f16x2{up, up}, f16x2{down, down}));
}

// What a workgroup works on: a sequence's rows and positions, cut to what the arrays have, and a head of the cache.
struct Part {
  int head, split, record;
  uint32_t row_block;
  int64_t seq, first;      // sequence, its first row of q
  int fresh, length;       // new tokens, positions
  uint32_t rows;           // query rows: new tokens times query heads of the head
  // (the constant address space: uniform reads through the scalar cache)
  const __attribute__((address_space(4))) int32_t* table;

  // The workgroup's number among `units`, of every head and split; heads in turn, then splits.  Neighbouring workgroups are on dies in turn, so with 8
  // heads the workgroups with the same keys share a die's cache, and with any number the long sequences and the long rows of a causal prompt
  // spread over the dies.  (In runs of a head's units to a die, which keeps a head's keys to one or two dies' caches with other numbers of heads,
  // too: a prompt of 4096 with 1, 4, 5, 12 and 32 heads of 128 259, 320, 193, 383 and 258 us, in turn 154, 238, 142, 329 and 241; single tokens of
  // 64 uneven sequences 35, 74, 118, 198 and 444, in turn 35, 81, 94, 174 and 430.)
  __device__ __forceinline__ uint32_t number(const AttendCall& a) {
    const uint32_t heads = uint32_t(a.cache.heads), work = blockIdx.x / heads;
    head = int(blockIdx.x % heads);
    record = int(work % a.split_blocks);
    return work / a.split_blocks;
  }
  // the rest, of a sequence
  __device__ __forceinline__ void look_at(const AttendCall& a, int64_t sequence, int wave) {
    seq = sequence;
    split = record * (4 / a.waves_rows) + wave / a.waves_rows;
    int64_t last = seq + 1;
    first = seq;
    if (a.starts) {
      first = a.starts[seq];
      last = a.starts[seq + 1];
      first = first < 0 ? 0 : first;
      last = last > a.n_tokens ? a.n_tokens : last;
    }
    fresh = last > first ? int(last - first) : 0;
    const int64_t asked = a.lengths[seq];
    length = int(asked < 0 ? 0 : asked > a.table_tokens ? a.table_tokens : asked);
    rows = uint32_t(fresh) * uint32_t(a.groups);             // (fewer than 2^31 rows of q altogether)
    table = (const __attribute__((address_space(4))) int32_t*)(a.table + seq * a.table_stride);
  }
  // Units: row_blocks to every sequence.
  __device__ __forceinline__ void find(const AttendCall& a, int wave) {
    const uint32_t unit = number(a);
    row_block = unit % a.row_blocks;
    look_at(a, unit / a.row_blocks, wave);
  }
  // Units: as many to a sequence as it has runs of `block` rows, by the sums over the sequences before; 64 of them at a time.  (With as many to all
  // as the longest has, a batch of 63 single tokens and a chunk of 512 spent most of its 690 us on workgroups with nothing to do.)
  __device__ __forceinline__ bool find_run(const AttendCall& a, uint32_t block, int lane) {
    uint32_t unit = number(a);
    if (!a.starts) {
      const uint32_t each = (uint32_t(a.groups) + block - 1) / block;
      if (unit / each >= uint64_t(a.n_seqs)) return false;
      row_block = each - 1 - unit % each;
      look_at(a, unit / each, 0);
      return true;
    }
    for (int64_t base = 0; base < a.n_seqs; base += 64) {
      uint32_t runs = 0;
      if (base + lane < a.n_seqs) {
        int64_t from = a.starts[base + lane], to = a.starts[base + lane + 1];
        from = from < 0 ? 0 : from;
        to = to > a.n_tokens ? a.n_tokens : to;
        if (to > from) runs = (uint32_t(to - from) * uint32_t(a.groups) + block - 1) / block;
      }
      uint32_t sum = runs;
      for (int apart = 1; apart < 64; apart <<= 1) {
        const uint32_t other = __shfl_up(sum, apart);
        if (lane >= apart) sum += other;
      }
      const uint64_t behind = __ballot(sum > unit);
      if (behind) {
        const int at = __ffsll((long long)behind) - 1;
        const uint32_t own = uint32_t(__builtin_amdgcn_readlane(int(runs), at));
        const uint32_t before = uint32_t(__builtin_amdgcn_readlane(int(sum), at)) - own;
        row_block = own - 1 - (unit - before);               // the longest rows of a causal prompt first
        look_at(a, base + at, 0);
        return true;
      }
      unit -= uint32_t(__builtin_amdgcn_readlane(int(sum), 63));
    }
    return false;
  }
};

// The first position that a token sees.  (The token may be before position 0, and the window as wide as 32 bits say.)
__device__ __forceinline__ int window_from(int position, int window) { return window > 0 && position >= window ? position - window + 1 : 0; }

// The positions that rows see: any of them from .. to, all of them all_from .. all_to (each cut to what there is).
struct Range {
  int from, to, all_from, all_to;
  __device__ __forceinline__ Range(const AttendCall& a, const Part& part, uint32_t first_row, uint32_t rows) {
    const int groups = a.groups, before = part.length - part.fresh;
    const int first_at = before + int(first_row / groups), last_at = before + int((first_row + rows - 1) / groups);
    const int window = int(a.window);
    from = window_from(first_at, window);
    to = a.causal && last_at + 1 < part.length ? last_at + 1 : part.length;
    all_from = window_from(last_at, window);
    all_to = a.causal && first_at + 1 < part.length ? first_at + 1 : part.length;
  }
};

// The lines of 16 positions: the first one's index, and how many there are; a page outside the pool has none.  Looked up in two steps, the
// table's entry well before it is needed (a miss of the scalar cache lasts as long as a step).
__device__ __forceinline__ int entry(const AttendCall& a, const Part& part, int at, int end) {
  return part.table[(at < end ? at : end - 1) >> a.cache.page_shift];
}
struct Lines16 {
  int64_t line;
  int there;
  __device__ __forceinline__ void find(const AttendCall& a, const Part& part, int page, int at, int end) {
    const bool valid = at < end && page >= 0 && page < a.cache.n_pages;
    there = valid ? (part.length - at < 16 ? part.length - at : 16) : 0;
    line = (int64_t(valid ? page : 0) * a.cache.heads + part.head) * a.cache.page_size +
           (valid ? at & (a.cache.page_size - 1) : 0);
  }
};

// Keys of 16 positions as a lane holds them, and the N of keys and values.
template <int D, int kN>
struct Keys {
  static constexpr int KS = D >= 64 ? D / 64 : 1;       // integer products to a line
  i32x4 F[KS];
  typename Scales<kN>::Raw N, value_N;
  __device__ __forceinline__ void load(const AttendCall& a, int64_t line, int c, int quarter) {
    const int8_t* k = a.cache.k_F + line * D;
    const uint32_t offset = c * D + (D == 32 ? (quarter & 1) * 16 : quarter * 16);
#pragma unroll
    for (int s = 0; s < KS; ++s) F[s] = *reinterpret_cast<const i32x4*>(k + (offset + s * 64));
    N = load_N<kN>(a.cache.k_N, line, quarter);
    value_N = load_N<kN>(a.cache.v_N, line, quarter);
  }
};

// The lane, of which the compiler must not know that it is the same every time: what is derived from it before and after the pass over the
// positions would otherwise be kept in registers during it, where there are none to spare.
__device__ __forceinline__ int this_lane() {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}

// Results of 16 rows, first ..: a wave's coefficients, from LDS, transformed back and written.
template <int D>
constexpr int kResultPitch = D + 4;
template <int D>
__device__ __forceinline__ void write_results(const AttendCall& a, const Part& part, uint32_t first, const float* staged) {
  constexpr int L = D / 16, kLines = 64 / L < 16 ? 64 / L : 16;
  const int lane = this_lane(), in_line = lane % L;
  const uint32_t groups = uint32_t(a.groups);
#pragma unroll 1
  for (int base = 0; base < 16 && first + base < part.rows; base += kLines) {
    const int line = base + lane / L < 16 ? base + lane / L : 15;
    float v[16];
    if (a.transform == PBZ_TRANSFORM_HAAR) {
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = staged[line * kResultPitch<D> + line::coefficient<kTfHaar, L>(in_line, k)];
      line::inverse<kTfHaar, float, L>(v, lane);
    } else {
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = staged[line * kResultPitch<D> + line::coefficient<kTfDct, L>(in_line, k)];
      line::inverse<kTfDct, float, L>(v, lane);
    }
    const uint32_t row = first + line, token = row / groups;
    if (row < part.rows && base + lane / L < 16)
      store_run(static_cast<uint16_t*>(a.out) + (part.first + token) * a.out_token_stride +
                    (int64_t(part.head) * groups + (row - token * groups)) * a.out_head_stride + in_line * 16, a.type, a.out_wide != 0, v);
  }
}

// A wave's 16 R rows of one head: what it keeps of them while positions go by, 32 to a step.
template <int D, int R, bool kFine, int kN>
struct Rows {
  static constexpr int KS = Keys<D, kN>::KS;
  static constexpr int DT = D / 16;                      // value tiles
  int64_t place[R];                                      // [token][query head]; -1: none
  int low[R], high[R];                                   // positions that a row sees
  i32x4 q_high[R][KS], q_low[R][KS];
  float q_scale[R];
  float top[R], reference[R], total[R];                  // reference: of weights and total, the top but for the row's own factor
  f32x4 sum[R][DT];
  float widest, narrow;      // the largest N of the values so far (rounded up to a power of two); 2^7 over it
  f16x8 p[R], p_low[R];      // weights of a step

  __device__ __forceinline__ void begin(const AttendCall& a, const Part& part, uint32_t first_row, int c, int quarter, float* largest) {
    const uint32_t groups = uint32_t(a.groups);
    const int before = part.length - part.fresh;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t asked = first_row + r * 16 + c;
      const bool there = asked < part.rows;
      const uint32_t row = there ? asked : part.rows - 1;
      const uint32_t token = row / groups;
      const int64_t at = (part.first + token) * a.q_heads + int64_t(part.head) * a.groups + (row - token * groups);
      place[r] = there ? at : -1;
      const int position = before + int(token);
      high[r] = !there ? -1 : a.causal ? position : part.length - 1;
      low[r] = window_from(position, int(a.window));
      q_scale[r] = a.space.q_scale[at];
      if (q_scale[r] == 0.f) q_scale[r] = 0x1p-100f;     // all of the row's products are zero; a hidden one stays -infinity
      const int8_t* q = a.space.q + at * (2 * D);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int offset = D == 32 ? (quarter & 1) * 16 : s * 64 + quarter * 16;
        q_high[r][s] = *reinterpret_cast<const i32x4*>(q + offset);
        q_low[r][s] = *reinterpret_cast<const i32x4*>(q + D + offset);
        if (D == 32 && quarter >= 2) q_high[r][s] = q_low[r][s] = i32x4{0, 0, 0, 0};     // half of the product is not used
      }
      top[r] = kNegInf;
      reference[r] = 0.f;
      total[r] = 0.f;
      largest[64 * r] = 0.f;
#pragma unroll
      for (int t = 0; t < DT; ++t) sum[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    widest = narrow = 0.f;
  }

  // scores of 16 positions, over the row's scale, in units of ln 2
  __device__ __forceinline__ void scores(const Keys<D, kN>& key, int u, float (&x)[R][2][4]) const {
    f32x4 N = scales<kN>(key.N);
#pragma unroll
    for (int i = 0; i < 4; ++i) N[i] = fmaf(N[i], 0.f, N[i]);      // an infinity is a NaN: no score is -infinity but a hidden one's
#pragma unroll
    for (int r = 0; r < R; ++r) {
      i32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < KS; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(key.F[s], q_high[r][s], acc, 0, 0, 0);
      acc = acc << 8;
#pragma unroll
      for (int s = 0; s < KS; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(key.F[s], q_low[r][s], acc, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[r][u][i] = float(acc[i]) * N[i];
    }
  }

  // What the weights refer to grows; seldom.  largest: in LDS, 64 apart, the largest weights so far, or less; of a lane's positions, and while some
  // row is unfit, of all the row's.
  __device__ __forceinline__ void grow(const f32x4 (&N)[2], const float (&most)[R], float* largest, bool unfit) {
    float wide = 0.f;                        // of what is finite
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) wide = fmaxf(wide, fabsf(N[u][i]) < __builtin_huge_valf() ? fabsf(N[u][i]) : 0.f);
    for (int apart = 1; apart < 64; apart <<= 1) wide = fmaxf(wide, __shfl_xor(wide, apart));
    const float wider = wide > widest ? wide_unit(wide) : widest;
    const float shrink = wider > 0.f ? widest / wider : 1.f;
    widest = wider;
    narrow = wider > 0.f ? 128.f / wider : 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float m = fmaxf(top[r], most[r]);
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float factor = m == kNegInf ? 1.f : __builtin_amdgcn_exp2f(top[r] - m);
      const float had = largest[64 * r], has = had * factor * shrink;
      const int now = unfit ? fitting(has) : 0;
      const float by = __builtin_amdgcn_ldexpf(factor, unfit ? now - fitting(had) : 0);
      top[r] = m;
      reference[r] = m == kNegInf ? 0.f : m - float(now);
      largest[64 * r] = has;
      total[r] *= by;
#pragma unroll
      for (int t = 0; t < DT; ++t) sum[r][t] *= by * shrink;
    }
  }

  // Rows that see something, and among whose positions none has a weight that is surely large enough; and whether one may be too large
  __device__ __forceinline__ bool wanting(int r, float most) const {
    const uint64_t fits = __ballot(most >= 1.f), seeing = __ballot(place[r] >= 0 && top[r] != kNegInf);
    return ((seeing & ~(fits | (fits >> 16) | (fits >> 32) | (fits >> 48)) & 0xffffu) | __ballot(most > 32768.f)) != 0;
  }
  // a lane's largest weight of a step; N: over the largest so far and times 2^7
  __device__ __forceinline__ float largest_of(int r, const float (&x)[R][2][4], const f32x4 (&N)[2]) const {
    float most = 0.f, minus = top[r] == kNegInf ? 0.f : -top[r];
    asm volatile("" : "+v"(minus));              // otherwise the exponentials are kept for the usual steps' use, in registers that those want
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(__builtin_amdgcn_exp2f(fmaf(x[r][u][i], q_scale[r], minus)) * N[u][i]));
    return place[r] < 0 ? 0.f : most;
  }
  // After a change of what weights refer to, and while some row is unfit: whether one is.  Has a factor of its own, or may need one, that is.
  __device__ __forceinline__ bool fit(const float (&x)[R][2][4], const f32x4 (&N)[2], float* largest, bool unfit) {
    float most[R];
    bool any = unfit;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      most[r] = fmaxf(largest[64 * r], largest_of(r, x, N));
      any = any || wanting(r, most[r]);
    }
    if (__builtin_expect(!any, 1)) {
#pragma unroll
      for (int r = 0; r < R; ++r) largest[64 * r] = most[r];
      return false;
    }
    bool own = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float m = most[r];
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float had = unfit ? largest[64 * r] : 0.f, has = m < __builtin_huge_valf() ? m : had;      // (infinite: so is the row's result)
      largest[64 * r] = has;
      const int now = fitting(has);
      const int change = now - fitting(had);
      const float by = __builtin_amdgcn_ldexpf(1.f, change);       // (0 below 2^-126: so much less is what the sums held)
      if (top[r] != kNegInf) reference[r] = top[r] - float(now);
      total[r] = __builtin_amdgcn_ldexpf(total[r], change);
#pragma unroll
      for (int t = 0; t < DT; ++t) sum[r][t] *= by;
      // (a row that has seen nothing but N of zero may come to need a factor without its reference changing)
      own = own || now != 0 || (has == 0.f && top[r] != kNegInf && place[r] >= 0);
    }
    return __any(own);
  }
  // Scores to weights, of 32 positions.  whole: all of them are there, and every row sees them.
  __device__ __forceinline__ void weigh(float (&x)[R][2][4], f32x4 (&N)[2], int at, bool whole, int there0, int there1, int quarter, float* largest, bool& unfit) {
    bool odd = false;
    if (!whole) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = at + 16 * u + quarter * 4 + i;
          const bool is = quarter * 4 + i < (u ? there1 : there0);
          if (!is) N[u][i] = 0.f;
          odd = odd || !(fabsf(N[u][i]) < __builtin_huge_valf());
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (!is || j > high[r] || j < low[r]) x[r][u][i] = kNegInf;
        }
      odd = __any(odd);
    }
    float wide = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) wide = fmaxf(wide, fabsf(N[u][i]));
    float most[R];
    bool more = wide > widest;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      most[r] = x[r][0][0];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) most[r] = fmaxf(most[r], x[r][u][i]);
      most[r] *= q_scale[r];
      more = more || most[r] > top[r] + kSlack;
    }
    const bool grown = __any(more);
    if (grown) grow(N, most, largest, unfit);
    const f32x4 n[2] = {N[0] * narrow, N[1] * narrow};
    if (grown || unfit) unfit = fit(x, n, largest, unfit);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(fmaf(x[r][u][i], q_scale[r], -reference[r]));
          total[r] += e;
          const float w = e * n[u][i];
          const _Float16 h = _Float16(w);
          p[r][u * 4 + i] = h;
          if constexpr (kFine) p_low[r][u * 4 + i] = _Float16(w - float(h));
        }
    }
    if (odd) {                               // zero times an N that is not finite
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (x[r][i / 4][i % 4] == kNegInf) {
            p[r][i] = _Float16(0);
            if constexpr (kFine) p_low[r][i] = _Float16(0);
          }
    }
  }

  // the weighted values of coefficient tile t
  __device__ __forceinline__ void add(int t, f16x8 v) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sum[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[r], sum[r][t], 0, 0, 0);
      if constexpr (kFine) sum[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p_low[r], sum[r][t], 0, 0, 0);
    }
  }

  // What a wave leaves for another with the same rows: per lane references, totals, sums in one unit; the lanes of a wave side by side.
  static constexpr int kLeft = R * (2 + 4 * DT);
  __device__ __forceinline__ float unit_of(int r, const float* largest, bool unfit) const {
    return __builtin_amdgcn_ldexpf(widest * (kValueUnit / (128.f * 127.f)) / kSumUnit, unfit ? -fitting(largest[64 * r]) : 0);
  }
  __device__ __forceinline__ void leave(float* left, int lane, const float* largest, bool unfit) const {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float unit = unit_of(r, largest, unfit);
      left[(2 * r) * 64 + lane] = top[r];
      left[(2 * r + 1) * 64 + lane] = __builtin_amdgcn_ldexpf(total[r], unfit ? -fitting(largest[64 * r]) : 0);
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) left[(2 * R + (r * DT + t) * 4 + i) * 64 + lane] = sum[r][t][i] * unit;
    }
  }
  __device__ __forceinline__ void into_unit(const float* largest, bool unfit) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float unit = unit_of(r, largest, unfit);
      total[r] = __builtin_amdgcn_ldexpf(total[r], unfit ? -fitting(largest[64 * r]) : 0);
#pragma unroll
      for (int t = 0; t < DT; ++t) sum[r][t] *= unit;
    }
  }
  __device__ __forceinline__ void take(const float* left, int lane) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float other = left[(2 * r) * 64 + lane], both = fmaxf(top[r], other);
      const float mine = both == kNegInf ? 1.f : __builtin_amdgcn_exp2f(top[r] - both);
      const float theirs = both == kNegInf ? 1.f : __builtin_amdgcn_exp2f(other - both);
      top[r] = both;
      total[r] = total[r] * mine + left[(2 * r + 1) * 64 + lane] * theirs;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[r][t][i] = sum[r][t][i] * mine + left[(2 * R + (r * DT + t) * 4 + i) * 64 + lane] * theirs;
    }
  }

  // a lane has coefficients (4 quarter + i) DT + t of its rows: a record, or where there are no splits the result, by way of the wave's
  // room in LDS
  __device__ __forceinline__ void store(const AttendCall& a, const Part& part, uint32_t first_row, float* staged, int c, int quarter) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float l = total[r];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (l != l) top[r] = 0.f;            // a row that sees a NaN is one, also where it sees nothing else
      if (a.records == 1) {
        if (a.lse && quarter == 0 && place[r] >= 0) a.lse[place[r]] = (top[r] + __builtin_amdgcn_logf(l)) * 0.693147180559945309f;
        const float by = top[r] == kNegInf ? 0.f : kSumUnit / l;
        float* to = staged + c * kResultPitch<D> + quarter * 4 * DT;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int t = 0; t < DT; ++t) to[i * DT + t] = sum[r][t][i] * by;
        wave_lds_sync();
        write_results<D>(a, part, first_row + r * 16, staged);
        wave_lds_sync();
        continue;
      }
      if (place[r] < 0) continue;
      const int64_t to = int64_t(part.record) * a.n_tokens * a.q_heads + place[r];
      if (quarter == 0) a.space.state[to] = make_float2(top[r], l);
      if (top[r] == kNegInf) continue;
      float* out = a.space.sums + to * D + quarter * 4 * DT;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (DT >= 4) {
#pragma unroll
          for (int t = 0; t < DT; t += 4) {
            const f32x4 v = {sum[r][t][i], sum[r][t + 1][i], sum[r][t + 2][i], sum[r][t + 3][i]};
            *reinterpret_cast<f32x4*>(out + i * DT + t) = v;
          }
        } else {
          *reinterpret_cast<float2*>(out + i * DT) = make_float2(sum[r][0][i], sum[r][1][i]);
        }
      }
    }
  }
};

// The values of four neighbouring coefficients at 8 positions (their words w) as operands: tiles[t], coefficient t of the four
__device__ __forceinline__ void value_tiles(const uint32_t (&w)[8], u32x4 (&tiles)[4]) {
#pragma unroll
  for (int pair = 0; pair < 4; ++pair) {
    const uint32_t w0 = w[2 * pair] ^ 0x80808080u, w1 = w[2 * pair + 1] ^ 0x80808080u;
    tiles[0][pair] = two_values<0>(w0, w1);
    tiles[1][pair] = two_values<1>(w0, w1);
    tiles[2][pair] = two_values<2>(w0, w1);
    tiles[3][pair] = two_values<3>(w0, w1);
  }
}

// Few rows: every wave by itself, positions of its own split; waves with the same rows join what they have before it is stored.  Keys are read a
// step ahead, into the registers that the products before them have left; values while the scores are taken.
// Bound by memory: waves wait for loads in two thirds of their cycles.  One token each of 256 sequences of 4096 positions, 32 query heads on 8 of
// 128: 372 us a call, 5.85 TB/s; of 64 sequences 105 us, 5.2 TB/s; one of 131072 positions 45 us, 6.1 TB/s.  Three waves a SIMD where the
// registers allow: with two, and values read a step ahead as well, the last one takes 41 us, but 256 sequences of 512 67 us instead of 56.
template <int D, int R, bool kFine, int kN>
__global__ __launch_bounds__(256, D == 256 ? (R == 1 ? 2 : 1) : R == 1 ? 3 : 2) void k_attend(const AttendCall a) {
  constexpr int VW = D >= 64 ? D / 64 : 1;       // 32-bit words of values a lane has of a position
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, quarter = lane >> 4;
  Part part;
  part.find(a, wave);
  const int sharing = 4 / a.waves_rows;          // waves with the same rows, whose splits become one record
  Rows<D, R, kFine, kN> rows;
  __shared__ float left[D == 32 ? 4 : 3][Rows<D, R, kFine, kN>::kLeft * 64];      // (with more columns, at most two waves have rows)
  __shared__ float largest[4][R * 64];
  const uint32_t together = uint32_t(a.waves_rows) * (16 * R);
  for (uint32_t base = part.row_block * together; base < part.rows; base += a.row_blocks * together) {
    const uint32_t first = base + uint32_t(wave % a.waves_rows) * (16 * R);
    const bool any = first < part.rows;
    rows.begin(a, part, first, c, quarter, largest[wave] + lane);
    bool unfit = false;                          // some row's weights have a factor of its own, or may need one
    const Range sees(a, part, any ? first : base, any && part.rows - first < 16 * R ? part.rows - first : any ? 16 * R : 1);
    const int64_t start = (sees.from & ~63) + int64_t(part.split) * a.chunk;
    const int begin = start < sees.to ? int(start) : sees.to;
    const int end = !any || part.split >= a.n_splits ? begin : part.split == a.n_splits - 1 || start + a.chunk > sees.to ? sees.to : int(start + a.chunk);
    Lines16 now[2], next[2];
    int page[2] = {0, 0};
    Keys<D, kN> key[2];
    if (begin < end) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        now[u].find(a, part, entry(a, part, begin + 16 * u, end), begin + 16 * u, end);
        key[u].load(a, now[u].line, c, quarter);
        page[u] = entry(a, part, begin + 32 + 16 * u, end);
      }
    }
    for (int at = begin; at < end; at += 32) {
      uint32_t value[VW][8];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int8_t* v = a.cache.v_F + now[u].line * D;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t w[VW];
          load_values<D>(v + uint32_t((quarter * 4 + i) * D + c * (D / 16)), w);
#pragma unroll
          for (int h = 0; h < VW; ++h) value[h][u * 4 + i] = w[h];
        }
      }
      f32x4 N[2] = {scales<kN>(key[0].value_N), scales<kN>(key[1].value_N)};
      float x[R][2][4];
      rows.scores(key[0], 0, x);
      rows.scores(key[1], 1, x);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        next[u].find(a, part, page[u], at + 32 + 16 * u, end);
        page[u] = entry(a, part, at + 64 + 16 * u, end);
        if (at + 32 < end) key[u].load(a, next[u].line, c, quarter);
      }
      const bool whole = at >= sees.all_from && at + 32 <= sees.all_to && now[0].there == 16 && now[1].there == 16;
      rows.weigh(x, N, at, whole, now[0].there, now[1].there, quarter, largest[wave] + lane, unfit);
#pragma unroll
      for (int h = 0; h < VW; ++h) {
        u32x4 tiles[4];
        value_tiles(value[h], tiles);
#pragma unroll
        for (int t = 0; t < (D == 32 ? 2 : 4); ++t) rows.add(4 * h + t, __builtin_bit_cast(f16x8, tiles[t]));
      }
      now[0] = next[0];
      now[1] = next[1];
    }
    const int turn = wave / a.waves_rows;
    if (sharing > 1) {
      if (turn > 0) rows.leave(left[wave - a.waves_rows], lane, largest[wave] + lane, unfit);
      __syncthreads();
    }
    if (turn == 0) {
      rows.into_unit(largest[wave] + lane, unfit);
      for (int w = 1; w < sharing; ++w) rows.take(left[wave + (w - 1) * a.waves_rows], lane);
      wave_lds_sync();
      const int at_end = this_lane();
      rows.store(a, part, first, left[wave], at_end & 15, at_end >> 4);
    }
    if (sharing > 1) __syncthreads();
  }
}

// In LDS: the largest weight so far of a lane's positions, or less, and the exponent of the row's own factor.
struct Fitting {
  float largest;
  int own;
};

// A wave's 32 rows of one head in tiles of 32: the same as Rows, a lane having one row and 16 of a step's 32 positions,
// 8 (i / 4) + 4 half + i % 4.  Whether the weights' reference has to grow shows in their sum, which is taken anyway: a lane's part of it
// may reach 2^8, and is infinite or no number while there is no reference.
template <int D, bool kFine>
struct TallRows {
  static constexpr int KS = D / 32, DT = D / 32;
  int low, high;
  i32x4 q_high[KS], q_low[KS];
  float q_scale, minus_top, total, widest;
  f32x16 sum[DT];
  f16x8 p[2], p_low[2];

  __device__ __forceinline__ void begin(const AttendCall& a, const Part& part, uint32_t first_row, int c, int half, Fitting* fitted) {
    fitted->largest = 0.f;
    const uint32_t groups = uint32_t(a.groups);
    const uint32_t asked = first_row + c;
    const bool there = asked < part.rows;
    const uint32_t row = there ? asked : part.rows - 1;
    const uint32_t token = row / groups;
    const int64_t at = (part.first + token) * a.q_heads + int64_t(part.head) * a.groups + (row - token * groups);
    const int position = part.length - part.fresh + int(token);
    high = !there ? -1 : a.causal ? position : part.length - 1;
    low = window_from(position, int(a.window));
    q_scale = a.space.q_scale[at];
    if (q_scale == 0.f) q_scale = 0x1p-100f;             // all of the row's products are zero; a hidden one stays -infinity
    const int8_t* q = a.space.q + at * (2 * D) + half * 16;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q_high[s] = *reinterpret_cast<const i32x4*>(q + s * 32);
      q_low[s] = *reinterpret_cast<const i32x4*>(q + D + s * 32);
    }
    minus_top = there ? -kNegInf : 0.f;
    total = widest = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[t][i] = 0.f;
  }

  // products of 32 positions' indices with the row's fixed-point coefficients: the high bytes, then the low ones added to 256 times that
  __device__ __forceinline__ void products_high(const i32x4 (&key)[KS], i32x16& acc) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(key[s], q_high[s], acc, 0, 0, 0);
  }
  __device__ __forceinline__ void products_low(const i32x4 (&key)[KS], i32x16& acc) const {
    acc = acc << 8;
#pragma unroll
    for (int s = 0; s < KS; ++s) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(key[s], q_low[s], acc, 0, 0, 0);
  }

  // After a change of what weights refer to, by which the sums change, and while some row is unfit (as in Rows): whether one is.  e is brought to
  // where FP16 can hold what becomes of it.  beyond: some N is more than 2^7.
  __device__ __forceinline__ bool wanting(float most) const {
    const uint64_t fits = __ballot(most >= 1.f), seeing = __ballot(high >= 0 && minus_top != -kNegInf);
    return (seeing & ~(fits | (fits >> 32)) & 0xffffffffu) != 0;
  }
  __device__ __forceinline__ bool fit(float (&e)[16], const f32x4 (&N)[4], float by, bool beyond, Fitting* fitted, bool unfit) {
    float most = fitted->largest * by;
    int before = 0, now = 0;
    bool rows = unfit || beyond || wanting(most);
    if (rows) {
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(e[i] * N[i / 4][i % 4]));
      rows = unfit || beyond || wanting(most);
    }
    if (__builtin_expect(rows, 0)) {
      const bool seeing = high >= 0 && minus_top != -kNegInf;
      before = unfit ? fitted->own : 0;
      most = fmaxf(most, __shfl_xor(most, 32));
      most = seeing && most < __builtin_huge_valf() ? most : 0.f;                  // (infinite: so is the row's result)
      now = fitting(most);
      fitted->own = now;
      const float own = __builtin_amdgcn_ldexpf(1.f, now);
#pragma unroll
      for (int i = 0; i < 16; ++i) e[i] *= own;
      // (a row that has seen nothing but N of zero may come to need a factor without its reference changing)
      rows = beyond || __any(now != 0 || (most == 0.f && seeing));
    }
    fitted->largest = most;
    by = __builtin_amdgcn_ldexpf(by, now - before);
#pragma unroll
    for (int t = 0; t < DT; ++t) sum[t] *= by;
    return rows;
  }

  // exponentials against the reference; their sum
  __device__ __forceinline__ float exponentials(const float (&x)[16], float minus, float (&e)[16]) const {
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      e[i] = __builtin_amdgcn_exp2f(fmaf(x[i], q_scale, minus));
      part[i % 4] += e[i];
    }
    return (part[0] + part[1]) + (part[2] + part[3]);
  }

  // Scores over the row's scale, in units of ln 2; hidden ones are -infinity where not the whole step is seen.
  __device__ __forceinline__ void scores(const i32x16& acc, const f32x4 (&key_N)[4], int at, bool whole, uint32_t there, int half,
                                         float (&x)[16]) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = float(acc[i]) * key_N[i / 4][i % 4];
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int place32 = 8 * (i / 4) + 4 * half + i % 4;
        if (!((there >> place32) & 1) || at + place32 > high || at + place32 < low) x[i] = kNegInf;
      }
    }
  }
  // e: the exponentials against the reference; more: their sum.  Where that does not do, a new reference and exponentials against that;
  // by: what the sums have to be multiplied by.
  __device__ __forceinline__ bool refer(const float (&x)[16], float (&e)[16], float& more, const f32x4 (&N)[4], float by, bool beyond, Fitting* fitted,
                                        bool unfit) {
    if (__any(!(more <= 256.f))) {
      float most = x[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) most = fmaxf(most, x[i]);
      most *= q_scale;
      most = fmaxf(most, __shfl_xor(most, 32));
      most = fmaxf(most, -minus_top);
      const float factor = most == kNegInf ? 1.f : __builtin_amdgcn_exp2f(-minus_top - most);
      minus_top = -most;
      total *= factor;
      by *= factor;
      more = exponentials(x, most == kNegInf ? 0.f : minus_top, e);
    }
    return fit(e, N, by, beyond, fitted, unfit);
  }
  // The weights.  N: of values, over the largest so far and times 2^7; odd: some are hidden, and some N are not finite.
  __device__ __forceinline__ void weights(const float (&x)[16], const float (&e)[16], const f32x4 (&N)[4], bool odd) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float w = e[i] * N[i / 4][i % 4];
      const _Float16 h = _Float16(w);
      p[i / 8][i % 8] = h;
      if constexpr (kFine) p_low[i / 8][i % 8] = _Float16(w - float(h));
    }
    if (odd) {                               // zero times an N that is not finite
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (x[i] == kNegInf) {
          p[i / 8][i % 8] = _Float16(0);
          if constexpr (kFine) p_low[i / 8][i % 8] = _Float16(0);
        }
    }
  }

  __device__ __forceinline__ void add(int b, int t, f16x8 v) {
    sum[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[b], sum[t], 0, 0, 0);
    if constexpr (kFine) sum[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p_low[b], sum[t], 0, 0, 0);
  }

  // A lane has coefficients (8 (i / 4) + 4 half + i % 4) DT + t of its row: a record, or where there are no splits the result, by way of the
  // wave's room in LDS.
  __device__ __forceinline__ void store(const AttendCall& a, const Part& part, uint32_t first_row, float* staged, int c, int half, int own) {
    const float l = total + __shfl_xor(total, 32);
    const float top = l != l ? 0.f : -minus_top;         // a row that sees a NaN is one, also where it sees nothing else
    const float unit = __builtin_amdgcn_ldexpf(widest * (kValueUnit / (128.f * 127.f)) / kSumUnit, -own);
    const bool there = first_row + c < part.rows;
    const uint32_t row = there ? first_row + c : part.rows - 1, token = row / uint32_t(a.groups);
    const int64_t place = (part.first + token) * a.q_heads + int64_t(part.head) * a.groups + (row - token * uint32_t(a.groups));
    if (a.records == 1) {
      if (a.lse && half == 0 && there) a.lse[place] = (top + __builtin_amdgcn_logf(l)) * 0.693147180559945309f;
      const float by = top == kNegInf ? 0.f : unit * (kSumUnit / l);
#pragma unroll 1
      for (int pass = 0; pass < 2; ++pass) {
        if (c / 16 == pass) {
          float* to = staged + c % 16 * kResultPitch<D> + half * 4 * DT;
#pragma unroll
          for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int t = 0; t < DT; ++t) to[(8 * (i / 4) + i % 4) * DT + t] = sum[t][i] * by;
        }
        wave_lds_sync();
        write_results<D>(a, part, first_row + pass * 16, staged);
        wave_lds_sync();
      }
      return;
    }
    if (!there) return;
    const int64_t to = int64_t(part.record) * a.n_tokens * a.q_heads + place;
    if (half == 0) a.space.state[to] = make_float2(top, l);
    if (top == kNegInf) return;
    float* out = a.space.sums + to * D + half * 4 * DT;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float* o = out + (8 * (i / 4) + i % 4) * DT;
      if constexpr (DT >= 4) {
#pragma unroll
        for (int t = 0; t < DT; t += 4) {
          const f32x4 v = {sum[t][i], sum[t + 1][i], sum[t + 2][i], sum[t + 3][i]};
          *reinterpret_cast<f32x4*>(o + t) = v * unit;
        }
      } else {
        *reinterpret_cast<float2*>(o) = make_float2(sum[0][i] * unit, sum[1][i] * unit);
      }
    }
  }
};

// The largest over a wave's lanes, in all of them; register moves only.
__device__ __forceinline__ float wave_max(float v) {
  const auto shifted = [](float x, auto control, auto rows) {
    return __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(int(__float_as_uint(x)), int(__float_as_uint(x)), decltype(control)::value,
                                                                decltype(rows)::value, 0xf, false)));
  };
  v = fmaxf(v, shifted(v, std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>()));
  v = fmaxf(v, shifted(v, std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>()));
  v = fmaxf(v, shifted(v, std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>()));
  v = fmaxf(v, shifted(v, std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>()));
  v = fmaxf(v, shifted(v, std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>()));
  v = fmaxf(v, shifted(v, std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>()));
  return __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(v)), 63)));
}

// A stage of 64 positions: a lane's line (its first one where there is none), and which positions there are.
struct Stage {
  int64_t line;
  uint64_t there;
  __device__ __forceinline__ void find(const AttendCall& a, const Part& part, int page, int at, int end, int lane) {
    const int j = at + lane;
    const bool valid = (j & ~15) < end && j < part.length && page >= 0 && page < a.cache.n_pages;
    line = (int64_t(valid ? page : 0) * a.cache.heads + part.head) * a.cache.page_size + (valid ? j & (a.cache.page_size - 1) : 0);
    there = __ballot(valid);
  }
  // the first line of 16 positions: those behind the end may be of another page, or none, but there are as many lines to read
  __device__ __forceinline__ int64_t first(int of) const {
    const uint32_t lo = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(line)), 16 * of));
    const uint32_t hi = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(uint64_t(line) >> 32)), 16 * of));
    return int64_t(uint64_t(lo) | (uint64_t(hi) << 32));
  }
};

// Many rows: a workgroup's four waves have neighbouring row tiles and go through the positions together, 64 to a stage.  Each wave
// converts the values of 16 of them into LDS, where every wave finds its operands, and N of all lies there, too; two buffers, so one
// barrier to a stage.  Every load is made whether or not it will be used (behind the end: of the pool's first line), so that
// the waits between loads and their uses count exactly.
// Bound by vector instructions, of which there are 223 to 32 positions of 32 rows of 128, 16 of them exponentials at a quarter of the rate; they
// are issued in 71 % of the time, and the matrix cores are busy in 38 %.  A prompt of 8192, 32 query heads on 8 of 128: 680 to 740 us on different
// cards, 0.74 to 0.8 PFLOP/s.  (Wave by wave with tiles of 16, as k_attend: 1022 us.)
template <int D, bool kFine, int kN>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void k_attend_tall(const AttendCall a) {
  constexpr int DT = D / 32, KS = D / 32, VW = D >= 128 ? D / 128 : 1;
  constexpr int kChunks = D / 16, kKeyLoads = D / 64;      // 16-byte pieces of a line; loads of 64 of them for a wave's 16 lines
  // LDS: stages, and in the end the waves' rooms for their results
  struct Stages {
    u32x4 operands[2][4][DT][64];
    i32x4 keys[3][64][kChunks];                  // piece p of line l at p ^ (l >> s), so that a read of 32 lines has 8 lanes on every bank
  };
  constexpr int kRoom = 16 * kResultPitch<D>;
  __shared__ alignas(16) uint8_t memory[int(sizeof(Stages)) > 16 * kRoom ? int(sizeof(Stages)) : 16 * kRoom];
  auto& operands = reinterpret_cast<Stages*>(memory)->operands;
  auto& keys = reinterpret_cast<Stages*>(memory)->keys;
  __shared__ alignas(16) float scale_of[2][2][64];           // keys, values (over the largest so far, times 2^7)
  __shared__ float2 reach[2];                    // the largest N of values so far, up to the next power of two; 1: some N is not finite, 2: some is beyond
  __shared__ Fitting fitted[256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, half = lane >> 5;
  Part part;
  if (!part.find_run(a, 128, lane)) return;
  TallRows<D, kFine> rows;
  {
    const uint32_t first = part.row_block * 128;
    const Range all(a, part, first, part.rows - first < 128 ? part.rows - first : 128);
    const int64_t start = (all.from & ~63) + int64_t(part.split) * a.chunk;
    const int begin = start < all.to ? int(start) : all.to;
    const int end = part.split == a.n_splits - 1 || start + a.chunk > all.to ? all.to : int(start + a.chunk);
    const uint32_t own = first + wave * 32;
    const int at_first = this_lane();
    bool unfit = false;                      // some row's weights have a factor of its own, or may need one
    rows.begin(a, part, own, at_first & 31, at_first >> 5, fitted + threadIdx.x);
    const Range sees(a, part, own < part.rows ? own : first, own < part.rows ? (part.rows - own < 32 ? part.rows - own : 32) : 1);
    if (begin < end) {
      const int32_t* table = a.table + part.seq * a.table_stride;
      // a stage's 64 positions: this wave's 16 of the values, one N a lane; and the 32 positions of a step's keys
      int page;                              // the table's entry for the lane's position (a vector load: waits for LDS wait for
                                             // scalar loads, too)
      uint32_t word[VW][8];
      float N_next = 0.f, widest = 0.f;
      i32x4 key_word[kKeyLoads];
      const auto look_up = [&](int at) {
        const int j = at + lane;
        page = table[(j < end ? j : end - 1) >> a.cache.page_shift];
      };
      const auto load_values_of = [&](const Stage& stage) {
        const int8_t* v = a.cache.v_F + stage.first(wave) * D;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t offset = (8 * (i / 4) + 4 * half + i % 4) * D + c * (D / 32);
          if constexpr (D == 64) word[0][i] = *reinterpret_cast<const uint16_t*>(v + offset);
          else if constexpr (D == 128) word[0][i] = *reinterpret_cast<const uint32_t*>(v + offset);
          else {
            const uint2 u = *reinterpret_cast<const uint2*>(v + offset);
            word[0][i] = u.x;
            word[VW - 1][i] = u.y;
          }
        }
        // waves 0 and 2 read the keys' N, the others the values'
        const void* N = wave & 1 ? a.cache.v_N : a.cache.k_N;
        if constexpr (kN == PBZ_F32) N_next = static_cast<const float*>(N)[stage.line];
        else if constexpr (kN == PBZ_BF16) N_next = bf16_bits_to_float(static_cast<const uint16_t*>(N)[stage.line]);
        else N_next = float(static_cast<const _Float16*>(N)[stage.line]);
      };
      const auto convert = [&](int buffer, uint64_t there) {
#pragma unroll
        for (int h = 0; h < VW; ++h) {
          u32x4 tiles[4];
          value_tiles(word[h], tiles);
#pragma unroll
          for (int t = 0; t < (D == 64 ? 2 : 4); ++t) operands[buffer][wave][4 * h + t][lane] = tiles[t];
        }
        if (wave == 0) scale_of[buffer][0][lane] = fmaf(N_next, 0.f, N_next);      // an infinity is a NaN: no score is -infinity but a hidden one's
        if (wave == 1) {
          const float N = (there >> lane) & 1 ? N_next : 0.f;
          const bool finite = fabsf(N) < __builtin_huge_valf();
          const float wide = wave_max(finite ? fabsf(N) : 0.f);
          if (wide > widest) widest = wide_unit(wide);
          scale_of[buffer][1][lane] = widest > 0.f ? N * (128.f / widest) : N;
          const bool odd = __any(!finite);
          if (lane == 0) reach[buffer] = make_float2(widest, (odd ? 1.f : 0.f) + (wide > widest ? 2.f : 0.f));
        }
      };
      const auto load_keys = [&](const Stage& stage) {
        const i32x4* k = reinterpret_cast<const i32x4*>(a.cache.k_F + stage.first(wave) * D);
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) key_word[i] = k[i * 64 + lane];
      };
      constexpr int kShift = D == 64 ? 2 : D == 128 ? 1 : 0;
      const auto put_keys = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) {
          const int l = 16 * wave + (i * 64 + lane) / kChunks, piece = lane % kChunks;
          keys[buffer][l][piece ^ ((l >> kShift) & (kChunks - 1))] = key_word[i];
        }
      };
      const auto read_keys = [&](int buffer, int b, i32x4 (&key)[KS]) {
        const int l = 32 * b + c;
#pragma unroll
        for (int s = 0; s < KS; ++s) key[s] = keys[buffer][l][(2 * s + half) ^ ((l >> kShift) & (kChunks - 1))];
      };
      // A step: its weights and weighted values, and meanwhile the products of the next one (of keys 32 next_b .. of a buffer), so that
      // the matrix cores have work while exponentials are taken.
      const auto step = [&](i32x16& acc, int at, int buffer, int b, int next_keys, int next_b, uint32_t there, bool odd, float shrink, bool renew, bool beyond) {
        const bool whole = at >= sees.all_from && at + 32 <= sees.all_to && there == ~0u;
        f32x4 key_N[4], N[4];
        i32x4 key[KS];
        float x[16], e[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) key_N[g] = *reinterpret_cast<const f32x4*>(&scale_of[buffer][0][32 * b + 8 * g + 4 * half]);
        read_keys(next_keys, next_b, key);
#pragma unroll
        for (int g = 0; g < 4; ++g) N[g] = *reinterpret_cast<const f32x4*>(&scale_of[buffer][1][32 * b + 8 * g + 4 * half]);
        rows.scores(acc, key_N, at, whole, there, half, x);
        rows.products_high(key, acc);
        float more = rows.exponentials(x, rows.minus_top, e);
#pragma unroll
        for (int s = 0; s < KS; ++s) {       // a product, then a share of the exponentials
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, 48 / KS, 0);
        }
        if (__any(!(more <= 256.f)) || renew || unfit) unfit = rows.refer(x, e, more, N, shrink, beyond, fitted + threadIdx.x, unfit);
        rows.total += more;
        u32x4 tile[DT];
#pragma unroll
        for (int t = 0; t < DT; ++t) tile[t] = operands[buffer][2 * b][t][lane];
        rows.products_low(key, acc);
        rows.weights(x, e, N, !whole && odd);
#pragma unroll
        for (int t = 0; t < DT; ++t) rows.add(0, t, __builtin_bit_cast(f16x8, tile[t]));
#pragma unroll
        for (int t = 0; t < DT; ++t) rows.add(1, t, __builtin_bit_cast(f16x8, operands[buffer][2 * b + 1][t][lane]));
      };
      // Keys are a stage further ahead than values: the products of a step are taken while the weights of the one before are.
      Stage now, after;
      look_up(begin);
      now.find(a, part, page, begin, end, lane);
      load_keys(now);
      load_values_of(now);
      look_up(begin + 64);
      put_keys(0);
      convert(0, now.there);
      after.find(a, part, page, begin + 64, end, lane);
      load_keys(after);
      look_up(begin + 128);
      put_keys(1);
      __syncthreads();
      i32x16 acc;
      {
        i32x4 key[KS];
        read_keys(0, 0, key);
        rows.products_high(key, acc);
        rows.products_low(key, acc);
      }
      int buffer = 0, key_buffer = 0;
      for (int stage = begin; stage < end; stage += 64) {
        const int next_buffer = key_buffer == 2 ? 0 : key_buffer + 1, free_buffer = next_buffer == 2 ? 0 : next_buffer + 1;
        const float2 reached = reach[buffer];
        const bool wider = reached.x > rows.widest, beyond = reached.y >= 2.f, odd = reached.y != 0.f && reached.y != 2.f;
        float shrink = 1.f;                  // the values' largest N so far is another one, by whose share the sums shrink
        if (wider) {
          shrink = rows.widest / reached.x;
          rows.widest = reached.x;
        }
        const uint64_t there = now.there;
        now = after;
        load_values_of(now);
        after.find(a, part, page, stage + 128, end, lane);
        load_keys(after);
        look_up(stage + 192);
        step(acc, stage, buffer, 0, key_buffer, 1, uint32_t(there), odd, shrink, wider || beyond, beyond);
        step(acc, stage + 32, buffer, 1, next_buffer, 0, uint32_t(there >> 32), odd, 1.f, beyond, beyond);
        buffer ^= 1;
        key_buffer = next_buffer;
        put_keys(free_buffer);
        convert(buffer, now.there);
        __syncthreads();
      }
    }
    const int at_end = this_lane();
    rows.store(a, part, own, reinterpret_cast<float*>(memory) + wave * kRoom, at_end & 31, at_end >> 5, unfit ? fitted[threadIdx.x].own : 0);
  }
}

template <int D, int kN>
int launch(bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s) {
  const dim3 grid(call.units * call.split_blocks * uint32_t(call.cache.heads)), block(256);
  if (tall) {
    if constexpr (D >= 64) {
      if (fine) k_attend_tall<D, true, kN><<<grid, block, 0, s>>>(call);
      else k_attend_tall<D, false, kN><<<grid, block, 0, s>>>(call);
    }
  } else if (rows == 16) {
    if (fine) k_attend<D, 1, true, kN><<<grid, block, 0, s>>>(call);
    else k_attend<D, 1, false, kN><<<grid, block, 0, s>>>(call);
  } else {
    if (fine) k_attend<D, 2, true, kN><<<grid, block, 0, s>>>(call);
    else k_attend<D, 2, false, kN><<<grid, block, 0, s>>>(call);
  }
  return hip_status(hipGetLastError());
}
template <int D>
int launch(bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s) {
  switch (call.cache.n_type) {
    case PBZ_F32: return launch<D, PBZ_F32>(tall, rows, fine, call, s);
    case PBZ_BF16: return launch<D, PBZ_BF16>(tall, rows, fine, call, s);
    default: return launch<D, PBZ_F16>(tall, rows, fine, call, s);
  }
}

}  // namespace
}  // namespace pbz
