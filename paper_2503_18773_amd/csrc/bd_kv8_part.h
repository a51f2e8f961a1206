// Partial results of splits, and the instances of the attention kernels over the paged 8-bit cache.
#pragma once

#include "bd_kv8_device.h"

namespace bd {

// Few rows: the launch merges its splits' partial results itself, in up to kMostSplits of them, with a counter for each of up to
// kCounters units (sequence, KV head, tile of 16 rows, or 32 where a sequence may have more than 16).  Workspace: the counters, then [unit][split][rows][D] unnormalised outputs and [unit][split]
// [rows][2] maxima (base 2) and sums.
constexpr int kMostSplits = 128;
constexpr long kCounters = BD_PAGED8_COUNTER_BYTES / 4;
constexpr long few_rows(long rows) { return rows <= 16 ? 16 : 32; }   // of a tile
constexpr long few_tiles(long rows) { return (rows + few_rows(rows) - 1) / few_rows(rows); }
struct Parts8 {
  uint32_t* counters;
  float* data;
};
hipError_t launch_kv8_few(const Step8& s, int head_dim, int code, int elem, const Rows8& q, const Scores8& sc, int splits, void* ws, void* out,
                          hipStream_t st);
constexpr int many_rows(int head_dim) { return head_dim == 64 ? 128 : 256; }   // of a workgroup of launch_kv8_many's
hipError_t launch_kv8_many(const Step8& s, int head_dim, int code, int elem, const Rows8& q, const Scores8& sc, int splits, float* part,
                           void* out, hipStream_t st);

#define BD_KV8_INSTANCES(head_dim, code, elem, RUN)                   \
  if (head_dim == 64) {                                               \
    if (code == BD_CODE_INT8 && elem == BD_ELEM_F16) RUN(64, BD_CODE_INT8, BD_ELEM_F16);        \
    else if (code == BD_CODE_INT8) RUN(64, BD_CODE_INT8, BD_ELEM_BF16);                         \
    else if (elem == BD_ELEM_F16) RUN(64, BD_CODE_E4M3, BD_ELEM_F16);                           \
    else RUN(64, BD_CODE_E4M3, BD_ELEM_BF16);                                                   \
  } else {                                                            \
    if (code == BD_CODE_INT8 && elem == BD_ELEM_F16) RUN(128, BD_CODE_INT8, BD_ELEM_F16);       \
    else if (code == BD_CODE_INT8) RUN(128, BD_CODE_INT8, BD_ELEM_BF16);                        \
    else if (elem == BD_ELEM_F16) RUN(128, BD_CODE_E4M3, BD_ELEM_F16);                          \
    else RUN(128, BD_CODE_E4M3, BD_ELEM_BF16);                                                  \
  }

namespace {

// Many rows: behind the counters, [splits][rows][D] unnormalised outputs, then [splits][rows][2] maxima (base 2) and sums; a row is (token, query head).
template <int D, int N>
__device__ __forceinline__ void store_part(float* part, int splits, size_t rows, int split, size_t row, int d, const float* o, float unit,
                                           float m, float l) {
  float* to = part + ((size_t)split * rows + row) * D + d;
#pragma unroll
  for (int e = 0; e < N; e += 4) *(f4_t*)(to + e) = f4_t{o[e] * unit, o[e + 1] * unit, o[e + 2] * unit, o[e + 3] * unit};
  if (d == 0) {
    float* ml = part + (size_t)splits * rows * D + ((size_t)split * rows + row) * 2;
    ml[0] = m;
    ml[1] = l;
  }
}

}  // namespace
}  // namespace bd
