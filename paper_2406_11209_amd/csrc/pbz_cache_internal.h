// What the cache's translation units share: geometry, the attention call as the kernels see it.
#pragma once

#include "pbz_cache.h"
#include "pbz_internal.h"

namespace pbz {

struct CacheGeom {
  int64_t n_pages;
  int32_t heads;
  int32_t page_size;
  int32_t page_shift;
  int32_t n_type;          // pbz_ftype of N
  const void* k_N;
  const int8_t* k_F;
  const void* v_N;
  const int8_t* v_F;
};

// Sums of values whose mean is a FP32 number need not be one.
constexpr float kSumUnit = 0x1p24f;

// Workspace of an attention call, [row] = [token][query head]
struct AttendSpace {
  int8_t* q;               // [row][2][D]: a coefficient is (256 high + low) times the row's scale
  float* q_scale;          // [row], times scale log2(e) / 127
  float2* state;           // [record][row]: running maximum (of scores in units of ln 2) and sum
  float* sums;             // [record][row][D]: coefficients of the weighted sum over kSumUnit; not written where the maximum is -infinity
};

struct AttendCall {
  CacheGeom cache;
  AttendSpace space;
  void* out;
  float* lse;
  int64_t out_token_stride, out_head_stride;
  int32_t type, transform, out_wide;
  int32_t records;         // splits that are left to be joined
  const int32_t* starts;
  const int32_t* lengths;
  const int32_t* table;
  int64_t table_stride;
  int64_t n_tokens;
  int64_t n_seqs;
  int64_t table_tokens;    // positions that the table has room for
  int64_t window;
  int64_t chunk;           // positions to a split, a multiple of 64
  int32_t causal;
  int32_t q_heads;
  int32_t groups;
  int32_t n_splits;
  int32_t waves_rows;      // of a workgroup's four waves: so many take row tiles, the others splits
  uint32_t row_blocks, split_blocks;
  uint32_t units;          // workgroups of a head and a split
};

// tall: the kernel for many rows; rows: query rows to a wave, 16 or 32; a translation unit per D
int launch_attend_32(bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s);
int launch_attend_64(bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s);
int launch_attend_128(bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s);
int launch_attend_256(bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s);
inline int launch_attend(int dim, bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s) {
  switch (dim) {
    case 32: return launch_attend_32(tall, rows, fine, call, s);
    case 64: return launch_attend_64(tall, rows, fine, call, s);
    case 128: return launch_attend_128(tall, rows, fine, call, s);
    default: return launch_attend_256(tall, rows, fine, call, s);
  }
}

}  // namespace pbz
