// The paged compressed cache (pbz_cache.h): checks and launches, the kernels that append lines and copy pages, and what an
// attention call does before and after its pass over keys and values (pbz_attend.h).
#include <algorithm>
#include <cmath>
#include <vector>

#include "pbz_cache_lines.h"

namespace pbz {
namespace {

constexpr int kMaxSplits = 256;
// Workgroups of 256 threads to a launch: HIP counts a dimension's threads modulo 2^32, and leaves out the others without an error.
constexpr int64_t kMaxBlocks = (int64_t(1) << 24) - 1;
// of a sequence: the kernels look up to 256 positions ahead, in 32 bits
constexpr int64_t kMaxPositions = (int64_t(1) << 31) - 1024;
constexpr int64_t kBusyWaves = 2048;         // waves that keep the chip busy: two to a SIMD
// Pairs of pages to a launch: 3.5 KiB of its 4 KiB of arguments; twice as many where 16 bits hold a page's number.
constexpr int kPairsPerLaunch = 448;

// ---- append ----------------------------------------------------------------------------------------------------------

struct AppendCall {
  CacheGeom cache;
  pbz_lines x[2];          // keys, values
  const int64_t* slots;
  int64_t lines;           // tokens * 2 * heads
  int32_t type;
  int32_t wide;
};

// L = D / 16 lanes to a line; a wave's indices go through LDS, where a lane's coefficients, L apart, become 16 neighbouring bytes.
// Bound by FP64 instructions: 8192 tokens of 8 heads of 128, bfloat16, take 26 us (2.0 TB/s), of which 21 are their issue (800 to a wave's 8 lines).  64
// tokens take 4.7 us, a launch's latencies.
template <int kTf, int D>
__global__ __launch_bounds__(256) void k_append(const AppendCall a) {
  constexpr int L = D / 16, kLines = 64 / L, kPitch = D + 4;      // the pitch keeps lines off one bank
  __shared__ uint32_t staged[4][kLines * kPitch / 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane % L, in_wave = lane / L;
  const int64_t asked = (int64_t(blockIdx.x) * 4 + wave) * kLines + in_wave;
  const bool there = asked < a.lines;
  const int64_t line = there ? asked : a.lines - 1;
  const uint32_t heads = uint32_t(a.cache.heads);
  const int64_t pair = line / heads;                              // [token][keys, values]
  const int head = int(line - pair * heads);
  const int64_t token = pair >> 1;
  const bool values = pair & 1;
  const pbz_lines& x = a.x[values];
  double v[16];
  load_run(x.data, a.type, token * x.token_stride + head * x.head_stride + part * 16, a.wide != 0, v);
  const int64_t slot = a.slots[token];
  line::forward<kTf, double, L>(v, lane);
  const double N = line_max<double, L>(v);
  const bool finite = N < __builtin_huge_val();
  // Quotients as products with a reciprocal, off by some 2^-45 at most; next to a border between two indices the quotient itself decides, and where N is
  // so small that the reciprocal is infinite.  Adding 1.5 * 2^52 leaves the nearest integer in the sum's lowest bits.
  const double reciprocal = N > 0.0 && finite ? 127.0 / N : 0.0;
  int r[16];
  bool close = !(reciprocal < __builtin_huge_val());
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    v[k] = finite ? v[k] : 0.0;
    const double sum = fma(v[k], reciprocal, 0x1.8p52);
    r[k] = int(uint32_t(__builtin_bit_cast(uint64_t, sum)));
    close = close || fabs(fma(v[k], reciprocal, 0x1.8p52 - sum)) > 0.5 - 0x1p-30;
  }
  if (close) {
#pragma unroll 1
    for (int k = 0; k < 16; ++k) r[k] = reciprocal > 0.0 ? int(rint(127.0 * v[k] / N)) : 0;
  }
  uint8_t* bytes = reinterpret_cast<uint8_t*>(staged[wave]) + in_wave * kPitch;
#pragma unroll
  for (int k = 0; k < 16; ++k) bytes[line::coefficient<kTf, L>(part, k)] = uint8_t(r[k]);
  wave_lds_sync();
  const int64_t page = slot >> a.cache.page_shift;
  if (!there || slot < 0 || page >= a.cache.n_pages) return;
  const int64_t to = (page * heads + head) * a.cache.page_size + (slot & (a.cache.page_size - 1));
  const uint32_t* from = staged[wave] + (in_wave * kPitch + part * 16) / 4;
  *reinterpret_cast<uint4*>(const_cast<int8_t*>(values ? a.cache.v_F : a.cache.k_F) + to * D + part * 16) =
      make_uint4(from[0], from[1], from[2], from[3]);
  if (part == 0)
    store_float(const_cast<void*>(values ? a.cache.v_N : a.cache.k_N), a.cache.n_type, to, finite ? N : __builtin_nan(""));
}

// ---- copies of pages ---------------------------------------------------------------------------------------------------

constexpr int kPiece = 16384;      // bytes of a page's part to a workgroup

template <typename Page, int kPairs>
struct CopyCall {
  char* pool[4];
  int64_t bytes[4];            // of a page's part; a multiple of 16
  int32_t pieces[4];           // of a page, up to and with this part
  Page pairs[2 * kPairs];
};

// Bound by memory, and by the ramp and the end of each launch: 2048 pages of 64 tokens of 8 heads of 128 126 us in three launches of 16-bit page
// numbers, 4.4 TB/s, 137 us in five of 32-bit ones (and with these in pieces of 8 KiB 143, of 32 KiB 161).
// The pairs travel with the launch: no copy to the device, nothing to keep alive, and a captured graph holds them.
template <typename Page, int kPairs>
__global__ __launch_bounds__(256) void k_copy_pages(const CopyCall<Page, kPairs> a) {
  const int64_t from = a.pairs[2 * blockIdx.y], to = a.pairs[2 * blockIdx.y + 1];
  const int x = int(blockIdx.x);
  const int part = (x >= a.pieces[0]) + (x >= a.pieces[1]) + (x >= a.pieces[2]);
  char* const pool = part == 0 ? a.pool[0] : part == 1 ? a.pool[1] : part == 2 ? a.pool[2] : a.pool[3];
  const int64_t bytes = part == 0 ? a.bytes[0] : part == 1 ? a.bytes[1] : part == 2 ? a.bytes[2] : a.bytes[3];
  const int before = part == 0 ? 0 : part == 1 ? a.pieces[0] : part == 2 ? a.pieces[1] : a.pieces[2];
  const int64_t at = int64_t(x - before) * kPiece;
  const uint4* const source = reinterpret_cast<const uint4*>(pool + from * bytes + at);
  uint4* const target = reinterpret_cast<uint4*>(pool + to * bytes + at);
  const int count = int((bytes - at < kPiece ? bytes - at : kPiece) / 16);
  if (count == kPiece / 16) {
    uint4 held[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) held[i] = source[i * 256 + threadIdx.x];
#pragma unroll
    for (int i = 0; i < 4; ++i) target[i * 256 + threadIdx.x] = held[i];
  } else {
    for (int i = threadIdx.x; i < count; i += 256) target[i] = source[i];
  }
}

// ---- attention: queries before, results after ----------------------------------------------------------------------------

struct QueryCall {
  const void* q;
  int64_t token_stride, head_stride;
  int64_t rows;            // tokens * query heads
  int32_t q_heads;
  int32_t type;
  int32_t wide;
  float scale;             // scale log2(e) / 127
  AttendSpace space;
  // Where nothing joins records, rows of no sequence are zeroed here, each by the lanes that have its query (by a head's first workgroup of the
  // pass, in turn, one token beside 8191 such rows of 32 heads of 128 took 1070 us, now 46); otherwise last_bound is 0
  void* out;
  float* lse;
  int64_t out_token_stride, out_head_stride;
  const int32_t* bounds;
  int64_t last_bound;
  int32_t out_wide;
};

// Transformed, and held relative to the row's largest coefficient in 16 bits, +-32639 = 127 * 256 + 127, high and low byte signed.
// 262144 rows of 128: 37 us (3.6 TB/s), 30 of them the issue of its 573 instructions to a wave's 8 rows.
template <int kTf, int D>
__global__ __launch_bounds__(256) void k_queries(const QueryCall a) {
  constexpr int L = D / 16, kLines = 64 / L, kPitch = D + 2;      // in coefficients of 16 bits
  __shared__ uint32_t staged[4][kLines * kPitch / 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane % L, in_wave = lane / L;
  const int64_t asked = (int64_t(blockIdx.x) * 4 + wave) * kLines + in_wave;
  const bool there = asked < a.rows;
  const int64_t row = there ? asked : a.rows - 1;
  const int64_t token = row / a.q_heads;
  const int32_t begin = a.bounds[0], end = a.bounds[a.last_bound];      // of the tokens that sequences have, read before they are needed
  float v[16];
  load_run_16(a.q, a.type, token * a.token_stride + (row - token * a.q_heads) * a.head_stride + part * 16, a.wide != 0, v);
  line::forward<kTf, float, L>(v, lane);
  const float most = line_max<float, L>(v);
  const bool finite = most < __builtin_huge_valf();
  const float scale = finite ? most * (1.f / 32639.f) * fabsf(a.scale) : __builtin_nanf("");
  float up = scale > 0.f ? 32639.f / most : 0.f;         // a row whose scale is 0 is taken for one of zeros
  up = up < __builtin_huge_valf() ? a.scale < 0.f ? -up : up : 0.f;
  // Adding 1.5 * 2^23 leaves the nearest integer in the sum's lowest bits; and 128, for the high byte to be signed's and the low one's bit 7 the
  // other way round.
  uint16_t* both = reinterpret_cast<uint16_t*>(staged[wave]) + in_wave * kPitch;
#pragma unroll
  for (int k = 0; k < 16; ++k) both[line::coefficient<kTf, L>(part, k)] = uint16_t(__float_as_uint(fmaf(v[k], up, 0x1.8p23f + 128.f)));
  wave_lds_sync();
  if (!there) return;
  const uint32_t* from = staged[wave] + (in_wave * kPitch + part * 16) / 2;
  uint32_t high[4], low[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w0 = from[2 * i], w1 = from[2 * i + 1];
    high[i] = __builtin_amdgcn_perm(w1, w0, 0x07050301u);
    low[i] = __builtin_amdgcn_perm(w1, w0, 0x06040200u) ^ 0x80808080u;
  }
  int8_t* const q = a.space.q + row * (2 * D) + part * 16;
  *reinterpret_cast<uint4*>(q) = make_uint4(high[0], high[1], high[2], high[3]);
  *reinterpret_cast<uint4*>(q + D) = make_uint4(low[0], low[1], low[2], low[3]);
  if (part == 0) a.space.q_scale[row] = scale;
  if (a.last_bound && (token < begin || token >= end)) {
    const float none[16] = {};
    store_run(static_cast<uint16_t*>(a.out) + token * a.out_token_stride + (row - token * a.q_heads) * a.out_head_stride + part * 16, a.type,
              a.out_wide != 0, none);
    if (part == 0 && a.lse) a.lse[row] = -__builtin_huge_valf();
  }
}

struct FinishCall {
  AttendSpace space;
  void* out;
  float* lse;
  int64_t token_stride, head_stride;
  int64_t rows;
  const int32_t* starts;
  int64_t n_seqs;
  int32_t q_heads;
  int32_t type;
  int32_t wide;
  int32_t n_splits;
};

// Joins the splits of a row, divides by the sum and transforms back.  64 records of 32 rows of 128: 5.5 us; 3 of 25408 rows: 12.7 us, 3.6 TB/s.
// A launch of its own, since the caches of two dies do not see each other's stores: with the last workgroup of a unit joining its records, written
// through to memory and read from there, the calls of those two took 76 and 127 us instead of 68 and 91.  kRows rows to a workgroup: with one, the threads share its splits;
// with more, every thread takes four columns of a row through all of them.
template <int kTf, int D, int kRows>
__global__ __launch_bounds__(256) void k_finish(const FinishCall a) {
  constexpr int L = D / 16, kColumns = D / 4, kPitch = D + 4, kGroups = kRows == 1 ? 256 / kColumns : 1;
  constexpr float kNone = -__builtin_huge_valf();
  __shared__ alignas(16) float staged[kRows * kGroups * kPitch];
  __shared__ float weight[kRows == 1 ? kMaxSplits : 1];
  __shared__ float joined[8];
  const int64_t first = int64_t(blockIdx.x) * kRows;
  const int tid = threadIdx.x;
  int64_t begin = 0, end = a.rows;           // of the rows that sequences have; the others' records have not been written
  if (a.starts) {
    begin = int64_t(a.starts[0]) * a.q_heads;
    end = int64_t(a.starts[a.n_seqs]) * a.q_heads;
  }
  if constexpr (kRows == 1) {
    const int column = tid % kColumns, group = tid / kColumns;
    const float* const sums = a.space.sums + first * D + column * 4;
    const int64_t apart_records = a.rows * D;
    // the first eight of a thread's records on their way while the weights are found: 64 records of 32 rows of 128 8.1 -> 5.5 us
    float4 ahead[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = group + i * kGroups;
      ahead[i] = *reinterpret_cast<const float4*>(sums + (s < a.n_splits ? s : 0) * apart_records);
    }
    float2 state = make_float2(kNone, 0.f);
    if (tid < a.n_splits) state = a.space.state[int64_t(tid) * a.rows + first];
    float most = state.x;
    for (int apart = 1; apart < 64; apart <<= 1) most = fmaxf(most, __shfl_xor(most, apart));
    if ((tid & 63) == 0) joined[tid >> 6] = most;
    __syncthreads();
    most = fmaxf(fmaxf(joined[0], joined[1]), fmaxf(joined[2], joined[3]));
    const float w = state.x == kNone ? 0.f : __builtin_amdgcn_exp2f(state.x - most);
    weight[tid] = state.x == kNone ? -1.f : w;           // (its sums have not been written)
    float total = state.x == kNone ? 0.f : w * state.y;
    for (int apart = 1; apart < 64; apart <<= 1) total += __shfl_xor(total, apart);
    if ((tid & 63) == 0) joined[4 + (tid >> 6)] = total;
    __syncthreads();
    total = (joined[4] + joined[5]) + (joined[6] + joined[7]);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto add = [&](int s, const float4& u) {
      const float f = weight[s];
      sum.x += f < 0.f ? 0.f : f * u.x;
      sum.y += f < 0.f ? 0.f : f * u.y;
      sum.z += f < 0.f ? 0.f : f * u.z;
      sum.w += f < 0.f ? 0.f : f * u.w;
    };
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (group + i * kGroups < a.n_splits) add(group + i * kGroups, ahead[i]);
#pragma unroll 8
    for (int s = group + 8 * kGroups; s < a.n_splits && first >= begin && first < end; s += kGroups) add(s, *reinterpret_cast<const float4*>(sums + s * apart_records));
    const float by = most == kNone ? 0.f : kSumUnit / total;
    *reinterpret_cast<float4*>(staged + group * kPitch + column * 4) = make_float4(sum.x * by, sum.y * by, sum.z * by, sum.w * by);
    __syncthreads();
    if (tid < D) {
      float s = 0.f;
      for (int g = 0; g < kGroups; ++g) s += staged[g * kPitch + tid];
      staged[tid] = s;                       // this thread's own column: nobody else reads it before the barrier
    }
    if (tid == 0 && a.lse) a.lse[first] = (most + __builtin_amdgcn_logf(total)) * 0.693147180559945309f;
  } else {
    for (int item = tid; item < kRows * kColumns; item += 256) {
      const int64_t row = first + item / kColumns;
      const int column = item % kColumns;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row < a.rows) {
        float most = kNone, total = 0.f;
#pragma unroll 4
        for (int s = 0; s < a.n_splits; ++s) most = fmaxf(most, a.space.state[int64_t(s) * a.rows + row].x);
        const int splits = row >= begin && row < end ? a.n_splits : 0;
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
          const float2 state = a.space.state[int64_t(s) * a.rows + row];
          const float4 u = *reinterpret_cast<const float4*>(a.space.sums + (int64_t(s) * a.rows + row) * D + column * 4);
          const bool none = state.x == kNone;            // (its sums have not been written)
          const float f = none ? 0.f : __builtin_amdgcn_exp2f(state.x - most);
          total += none ? 0.f : f * state.y;
          sum.x += none ? 0.f : f * u.x;
          sum.y += none ? 0.f : f * u.y;
          sum.z += none ? 0.f : f * u.z;
          sum.w += none ? 0.f : f * u.w;
        }
        const float by = most == kNone ? 0.f : kSumUnit / total;
        sum = make_float4(sum.x * by, sum.y * by, sum.z * by, sum.w * by);
        if (column == 0 && a.lse) a.lse[row] = (most + __builtin_amdgcn_logf(total)) * 0.693147180559945309f;
      }
      *reinterpret_cast<float4*>(staged + (item / kColumns) * kPitch + column * 4) = sum;
    }
  }
  __syncthreads();
  if (tid >= kRows * L) return;              // whole lines
  const int part = tid % L, in_block = tid / L;
  const int64_t row = first + in_block;
  const int64_t token = row / a.q_heads;
  const int64_t head = row - token * a.q_heads;
  float v[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = staged[in_block * kPitch + line::coefficient<kTf, L>(part, k)];
  line::inverse<kTf, float, L>(v, tid & 63);
  if (row >= a.rows) return;
  if (row < begin || row >= end) {           // a row of no sequence
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = 0.f;
    if (part == 0 && a.lse) a.lse[row] = kNone;
  }
  store_run(static_cast<uint16_t*>(a.out) + token * a.token_stride + head * a.head_stride + part * 16, a.type, a.wide != 0, v);
}

// ---- host ------------------------------------------------------------------------------------------------------------

// f(transform, D) with both as types
template <typename F>
void for_line(int transform, int dim, F&& f) {
  const auto sized = [&](auto tf) {
    if (dim == 32) f(tf, std::integral_constant<int, 32>());
    else if (dim == 64) f(tf, std::integral_constant<int, 64>());
    else if (dim == 128) f(tf, std::integral_constant<int, 128>());
    else f(tf, std::integral_constant<int, 256>());
  };
  if (transform == PBZ_TRANSFORM_HAAR) sized(std::integral_constant<int, kTfHaar>());
  else sized(std::integral_constant<int, kTfDct>());
}

bool aligned(const void* p, uintptr_t to = 16) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_geometry(const pbz_codec* c, const pbz_cache* cache) {
  if (!c || !cache) return PBZ_ERR_NULL;
  if (c->ndim != 1 || (c->vol != 32 && c->vol != 64 && c->vol != 128 && c->vol != 256)) return PBZ_ERR_BLOCK_SHAPE;
  if (c->itype != PBZ_I8 || c->ftype == PBZ_F64) return PBZ_ERR_TYPE;
  if (c->kept != c->vol) return PBZ_ERR_MASK;
  const int64_t size = cache->page_size;
  if (size < 16 || size > 1024 || (size & (size - 1)) || cache->heads < 1 || cache->heads > 65535 || cache->n_pages < 1 ||
      cache->n_pages > INT32_MAX || cache->n_pages > (int64_t(1) << 40) / (int64_t(cache->heads) * size * c->vol))
    return PBZ_ERR_SHAPE;
  return PBZ_OK;
}

int check_cache(const pbz_codec* c, const pbz_cache* cache, CacheGeom* g) {
  const int st = check_geometry(c, cache);
  if (st != PBZ_OK) return st;
  if (!cache->k_N || !cache->k_F || !cache->v_N || !cache->v_F) return PBZ_ERR_NULL;
  if (!aligned(cache->k_N) || !aligned(cache->k_F) || !aligned(cache->v_N) || !aligned(cache->v_F)) return PBZ_ERR_ALIGNMENT;
  g->n_pages = cache->n_pages;
  g->heads = cache->heads;
  g->page_size = cache->page_size;
  g->page_shift = __builtin_ctz(unsigned(cache->page_size));
  g->n_type = c->ftype;
  g->k_N = cache->k_N;
  g->k_F = static_cast<const int8_t*>(cache->k_F);
  g->v_N = cache->v_N;
  g->v_F = static_cast<const int8_t*>(cache->v_F);
  return PBZ_OK;
}

constexpr int64_t kMaxElements = int64_t(1) << 40;

bool stride_ok(int64_t stride, int64_t count) { return stride >= 0 && (count < 2 || stride <= kMaxElements / (count - 1)); }

// how an attention call is dealt out; every field follows from sizes that the host has
struct AttendPlan {
  int64_t rows;            // of q
  int tile;                // query rows to a wave
  int waves_rows;
  int64_t row_blocks, split_blocks, units;
  int64_t n_splits, chunk;
  int64_t records;         // splits as they are left to be joined
  int finish_rows;         // rows to a workgroup there
  bool tall;               // the kernel for many rows
  bool whole() const { return records == 1; }       // the pass over the positions writes the results itself
  size_t q_bytes, scale_bytes, state_bytes, sum_bytes;
  size_t total() const { return q_bytes + scale_bytes + state_bytes + sum_bytes; }
};

size_t padded(uint64_t n) { return size_t((n + 255) / 256 * 256); }

int plan_attend(const pbz_codec* c, const pbz_cache* cache, const pbz_attention* a, AttendPlan* p) {
  const int st = check_geometry(c, cache);
  if (st != PBZ_OK) return st;
  if (!a) return PBZ_ERR_NULL;
  if (a->type != PBZ_BF16 && a->type != PBZ_F16) return PBZ_ERR_TYPE;
  if (a->q_heads < 1 || a->q_heads % cache->heads || a->n_tokens < 1 || a->n_seqs < 1 || a->n_seqs > INT32_MAX ||
      a->max_pages < 1 || a->max_pages > kMaxPositions / cache->page_size || a->table_stride < a->max_pages ||
      a->table_stride > kMaxElements / a->n_seqs || a->max_new < 1 || a->max_length < 0 || a->window < 0 ||
      a->window > INT32_MAX || a->n_tokens > INT32_MAX / a->q_heads || (!a->starts && a->n_tokens != a->n_seqs))
    return PBZ_ERR_SHAPE;
  if (!std::isfinite(a->scale)) return PBZ_ERR_SCALAR;
  const int groups = a->q_heads / cache->heads;
  const int64_t fresh = a->starts ? std::min(a->max_new, a->n_tokens) : 1;
  const int64_t rows = fresh * groups;
  p->rows = a->n_tokens * a->q_heads;
  // Row tiles of 16, or of 32 where they would be more than half empty otherwise: 8 heads of 128 over 16 x 4096 positions with 16 rows
  // each 35 us in tiles of 16 and 37 in tiles of 32, with 24 rows 43 and 38, with 48 71 and 50.  Lines of 256 leave the tiles of 32
  // half the waves: with 32 rows 74 and 82 us, with 48 117 and 109.
  p->tile = rows <= 16 || (c->vol == 256 && rows <= 32) ? 16 : 32;
  const int64_t tiles = (rows + p->tile - 1) / p->tile;
  // A workgroup's waves share what they can of the positions: three or four row tiles go through them together (128 rows as above: 76 us,
  // 85 wave by wave), fewer leave waves for other splits, which are joined before they are stored.
  p->waves_rows = tiles >= 3 ? 4 : tiles == 2 ? 2 : 1;
  p->tall = c->vol >= 64 && p->tile == 32 && p->waves_rows == 4;
  const int waves_splits = 4 / p->waves_rows;
  int64_t length = a->max_pages * cache->page_size;
  if (a->max_length > 0) length = std::min(length, a->max_length);
  if (a->window > 0) length = std::min(length, a->window + fresh + 63);
  // Splits of the positions, where rows alone do not fill the chip, for 1400, 2048 and 3000 waves: chunks of 10 to 387 after up to 3528 95, 87 and 107
  // us, one token of 131072 71, 65 and 70, of 64 uneven sequences to 8200 128, 128 and 191; the tall kernel for lines of 256 has one wave to a SIMD
  // (32 new tokens of 4 query heads, 128 rows, after 16 x 4096: 153 us with 1024, 172 with 2048; 128 new tokens after 4 x 4096 140 and 159).  Down to 64
  // positions: one token after 8000, lines of 128, takes 18 us, 21 with at least 128 and 23 with 256.
  // (max_new bounds the tiles of every sequence, all rows together those of all)
  const int64_t some = std::min(a->n_seqs * tiles, (a->n_tokens * groups + p->tile - 1) / p->tile + a->n_seqs);
  const int64_t alone = some * cache->heads, busy = p->tall && c->vol == 256 ? kBusyWaves / 2 : kBusyWaves;
  int64_t splits = std::max<int64_t>((busy + alone - 1) / alone, waves_splits);
  splits = std::max<int64_t>(1, std::min<int64_t>({splits, kMaxSplits * waves_splits, length / 64}));
  p->chunk = ((length + splits - 1) / splits + 63) / 64 * 64;
  p->n_splits = (length + p->chunk - 1) / p->chunk;
  p->row_blocks = (tiles + p->waves_rows - 1) / p->waves_rows;
  p->split_blocks = (p->n_splits + waves_splits - 1) / waves_splits;
  p->records = p->split_blocks;
  // Joining: few rows of many records have a workgroup each, whose threads share the records (32 rows of 131072 positions, the same call over and
  // over: 54 us in all, 64 with several rows to a workgroup); with 4096 rows of 16 records that is the slower way (58 and 52), and with 2048 (41 and 38).
  p->finish_rows = p->records >= 8 && p->rows < 2048 ? 1 : 64 / (c->vol / 16);
  // the kernel for many rows finds runs of 128 rows of every sequence; there are no more of them than
  const int64_t most = kMaxBlocks / cache->heads / p->split_blocks;
  if (!p->tall) p->row_blocks = std::max<int64_t>(1, std::min(p->row_blocks, most / a->n_seqs));      // (a workgroup takes rows in turn)
  p->units = p->tall ? a->n_tokens * groups / 128 + a->n_seqs : a->n_seqs * p->row_blocks;
  if (p->units > most || p->rows > kMaxBlocks * (4096 / c->vol) || (!p->whole() && p->rows > kMaxBlocks * p->finish_rows)) return PBZ_ERR_SHAPE;
  p->q_bytes = padded(uint64_t(p->rows) * 2 * c->vol);
  p->scale_bytes = padded(uint64_t(p->rows) * sizeof(float));
  p->state_bytes = p->whole() ? 0 : padded(uint64_t(p->rows) * p->records * sizeof(float2));
  p->sum_bytes = p->whole() ? 0 : padded(uint64_t(p->rows) * p->records * c->vol * sizeof(float));
  return PBZ_OK;
}

// As many launches as the pairs need
template <typename Page, int kPairs>
int copy_pages(const pbz_codec* c, const pbz_cache* cache, int64_t n_pairs, const int32_t* pairs, hipStream_t stream) {
  CopyCall<Page, kPairs> call;
  const int64_t lines = int64_t(cache->heads) * cache->page_size;
  void* const pools[4] = {cache->k_F, cache->v_F, cache->k_N, cache->v_N};
  int64_t pieces = 0;
  for (int i = 0; i < 4; ++i) {
    call.pool[i] = static_cast<char*>(pools[i]);
    call.bytes[i] = lines * (i < 2 ? c->vol : ftype_bytes(c->ftype));
    pieces += (call.bytes[i] + kPiece - 1) / kPiece;
    call.pieces[i] = int32_t(pieces);
  }
  for (int64_t at = 0; at < n_pairs; at += kPairs) {
    const int64_t n = std::min<int64_t>(kPairs, n_pairs - at);
    std::copy(pairs + 2 * at, pairs + 2 * (at + n), call.pairs);
    k_copy_pages<Page, kPairs><<<dim3(unsigned(pieces), unsigned(n)), 256, 0, stream>>>(call);
    const int st = hip_status(hipGetLastError());
    if (st != PBZ_OK) return st;
  }
  return PBZ_OK;
}

}  // namespace
}  // namespace pbz

using namespace pbz;

extern "C" {

int pbz_cache_layout(const pbz_codec* c, const pbz_cache* cache, size_t* n_bytes, size_t* f_bytes) {
  const int st = check_geometry(c, cache);
  if (st != PBZ_OK) return st;
  const size_t lines = size_t(cache->n_pages) * size_t(cache->heads) * size_t(cache->page_size);
  if (n_bytes) *n_bytes = lines * size_t(ftype_bytes(c->ftype));
  if (f_bytes) *f_bytes = lines * size_t(c->vol);
  return PBZ_OK;
}

int pbz_cache_append(const pbz_codec* c, const pbz_cache* cache, int64_t n_tokens, const pbz_lines* k, const pbz_lines* v,
                     pbz_ftype type, const int64_t* slots, void* stream) {
  AppendCall call;
  const int st = check_cache(c, cache, &call.cache);
  if (st != PBZ_OK) return st;
  if (!k || !v || !k->data || !v->data || !slots) return PBZ_ERR_NULL;
  if (type != PBZ_F64 && type != PBZ_F32 && type != PBZ_BF16 && type != PBZ_F16) return PBZ_ERR_TYPE;
  const int bytes = ftype_bytes(type);
  call.wide = 1;
  int i = 0;
  for (const pbz_lines* x : {k, v}) {
    if (n_tokens < 1 || n_tokens > INT32_MAX / cache->heads || !stride_ok(x->token_stride, n_tokens) ||
        !stride_ok(x->head_stride, cache->heads))
      return PBZ_ERR_SHAPE;
    if (!aligned(x->data) || x->token_stride * bytes % 16 || x->head_stride * bytes % 16) call.wide = 0;
    call.x[i++] = *x;
  }
  call.slots = slots;
  call.lines = n_tokens * 2 * cache->heads;
  call.type = type;
  const int64_t lines = 256 / (c->vol / 16), blocks = (call.lines + lines - 1) / lines;
  if (blocks > kMaxBlocks) return PBZ_ERR_SHAPE;
  c->used.store(true);
  const dim3 grid{unsigned(blocks)};
  for_line(c->transform, c->vol, [&](auto tf, auto dim) {
    k_append<decltype(tf)::value, decltype(dim)::value><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(call);
  });
  return hip_status(hipGetLastError());
}

int pbz_cache_copy_pages(const pbz_codec* c, const pbz_cache* cache, int64_t n_pairs, const int32_t* pairs, void* stream) {
  CacheGeom g;
  const int st = check_cache(c, cache, &g);
  if (st != PBZ_OK) return st;
  if (!pairs) return PBZ_ERR_NULL;
  if (n_pairs < 1 || n_pairs > cache->n_pages) return PBZ_ERR_SHAPE;
  // every page in the pool, written at most once, and not read as well
  for (int64_t i = 0; i < 2 * n_pairs; ++i)
    if (pairs[i] < 0 || pairs[i] >= cache->n_pages) return PBZ_ERR_PAGES;
  if (n_pairs <= 32) {
    for (int64_t i = 0; i < n_pairs; ++i)
      for (int64_t j = 0; j < n_pairs; ++j)
        if (pairs[2 * i + 1] == pairs[2 * j] || (i != j && pairs[2 * i + 1] == pairs[2 * j + 1])) return PBZ_ERR_PAGES;
  } else {
    try {
      std::vector<uint8_t> role(size_t(cache->n_pages), 0);      // 1 read, 2 written
      for (int64_t i = 0; i < n_pairs; ++i) role[size_t(pairs[2 * i])] = 1;
      for (int64_t i = 0; i < n_pairs; ++i) {
        uint8_t& to = role[size_t(pairs[2 * i + 1])];
        if (to) return PBZ_ERR_PAGES;
        to = 2;
      }
    } catch (...) {
      return PBZ_ERR_ALLOC;
    }
  }
  const auto stream_ = static_cast<hipStream_t>(stream);
  if (cache->n_pages <= 65536) return copy_pages<uint16_t, 2 * kPairsPerLaunch>(c, cache, n_pairs, pairs, stream_);
  return copy_pages<int32_t, kPairsPerLaunch>(c, cache, n_pairs, pairs, stream_);
}

int pbz_cache_attend_workspace(const pbz_codec* c, const pbz_cache* cache, const pbz_attention* a, size_t* bytes) {
  if (!bytes) return PBZ_ERR_NULL;
  AttendPlan p;
  const int st = plan_attend(c, cache, a, &p);
  if (st != PBZ_OK) return st;
  *bytes = p.total();
  return PBZ_OK;
}

int pbz_cache_attend(const pbz_codec* c, const pbz_cache* cache, const pbz_attention* a, void* workspace,
                     size_t workspace_bytes, void* stream) {
  AttendCall call;
  int st = check_cache(c, cache, &call.cache);
  if (st != PBZ_OK) return st;
  AttendPlan p;
  st = plan_attend(c, cache, a, &p);
  if (st != PBZ_OK) return st;
  if (!a->q || !a->out || !a->lengths || !a->table || !workspace) return PBZ_ERR_NULL;
  for (int64_t stride : {a->q_token_stride, a->out_token_stride})
    if (!stride_ok(stride, a->n_tokens)) return PBZ_ERR_SHAPE;
  for (int64_t stride : {a->q_head_stride, a->out_head_stride})
    if (!stride_ok(stride, a->q_heads)) return PBZ_ERR_SHAPE;
  if (workspace_bytes < p.total() || !aligned(workspace)) return PBZ_ERR_WORKSPACE;
  char* at = static_cast<char*>(workspace);
  AttendSpace& space = call.space;
  space.q = reinterpret_cast<int8_t*>(at);
  space.q_scale = reinterpret_cast<float*>(at += p.q_bytes);
  space.state = reinterpret_cast<float2*>(at += p.scale_bytes);
  space.sums = reinterpret_cast<float*>(at += p.state_bytes);
  c->used.store(true);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int L = c->vol / 16;

  QueryCall query;
  query.q = a->q;
  query.token_stride = a->q_token_stride;
  query.head_stride = a->q_head_stride;
  query.rows = p.rows;
  query.q_heads = a->q_heads;
  query.type = a->type;
  query.wide = aligned(a->q) && a->q_token_stride % 8 == 0 && a->q_head_stride % 8 == 0;
  query.scale = a->scale * float(1.4426950408889634074 / 127.0);
  query.space = space;
  query.out = a->out;
  query.lse = a->lse;
  query.out_token_stride = a->out_token_stride;
  query.out_head_stride = a->out_head_stride;
  const bool bounded = p.whole() && a->starts;
  query.bounds = bounded ? a->starts : a->lengths;      // (any address that can be read)
  query.last_bound = bounded ? a->n_seqs : 0;
  query.out_wide = aligned(a->out) && a->out_token_stride % 8 == 0 && a->out_head_stride % 8 == 0;
  const dim3 query_grid(unsigned((p.rows + 256 / L - 1) / (256 / L)));
  for_line(c->transform, c->vol, [&](auto tf, auto dim) {
    k_queries<decltype(tf)::value, decltype(dim)::value><<<query_grid, 256, 0, s>>>(query);
  });
  st = hip_status(hipGetLastError());
  if (st != PBZ_OK) return st;

  call.out = a->out;
  call.lse = a->lse;
  call.out_token_stride = a->out_token_stride;
  call.out_head_stride = a->out_head_stride;
  call.type = a->type;
  call.transform = c->transform;
  call.out_wide = query.out_wide;
  call.records = int32_t(p.records);
  call.starts = a->starts;
  call.lengths = a->lengths;
  call.table = a->table;
  call.table_stride = a->table_stride;
  call.n_tokens = a->n_tokens;
  call.n_seqs = a->n_seqs;
  call.table_tokens = a->max_pages * cache->page_size;
  call.window = a->window;
  call.chunk = p.chunk;
  call.causal = a->causal != 0;
  call.q_heads = a->q_heads;
  call.groups = a->q_heads / cache->heads;
  call.n_splits = int32_t(p.n_splits);
  call.waves_rows = p.waves_rows;
  call.row_blocks = uint32_t(p.row_blocks);
  call.split_blocks = uint32_t(p.split_blocks);
  call.units = uint32_t(p.units);
  st = launch_attend(c->vol, p.tall, p.tile, a->type == PBZ_F16, call, s);
  if (st != PBZ_OK || p.whole()) return st;

  FinishCall finish;
  finish.space = space;
  finish.out = a->out;
  finish.lse = a->lse;
  finish.token_stride = a->out_token_stride;
  finish.head_stride = a->out_head_stride;
  finish.rows = p.rows;
  finish.starts = a->starts;
  finish.n_seqs = a->n_seqs;
  finish.q_heads = a->q_heads;
  finish.type = a->type;
  finish.wide = call.out_wide;
  finish.n_splits = int32_t(p.records);
  for_line(c->transform, c->vol, [&](auto tf, auto dim) {
    constexpr int kTf = decltype(tf)::value, D = decltype(dim)::value, kWave = 64 / (D / 16);
    if (p.finish_rows == 1) k_finish<kTf, D, 1><<<dim3(unsigned(p.rows)), 256, 0, s>>>(finish);
    else k_finish<kTf, D, kWave><<<dim3(unsigned((p.rows + kWave - 1) / kWave)), 256, 0, s>>>(finish);
  });
  return hip_status(hipGetLastError());
}

}  // extern "C"
