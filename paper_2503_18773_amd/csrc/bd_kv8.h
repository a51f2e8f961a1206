// What the kernels of the paged 8-bit cache share (gfx950 only).
#pragma once

#include "bd_common.h"

namespace bd {

constexpr int kStatusRead = 1, kStatusWrite = 2, kStatusRows = 4, kStatusPosition = 8;

struct Rows8 {
  uint16_t* data;
  int64_t token, head;   // strides, elements
};

// A cache and the rows of a step, as kernels take them.
struct Step8 {
  uint8_t *k_codes, *v_codes;
  float *k_scales, *v_scales;
  uint16_t *k_res, *v_res;
  const int32_t *block_table, *cu;
  int32_t *seq_lens, *status;
  int batch, n_q_heads, n_kv_heads, gq, num_pages, max_pages, total, max_tokens;
};

// What a workgroup's first loads wait for, as scalars ahead of a kernel's structures: those are in registers when it starts
// (build.py), the structures have to be fetched first.
#define BD_KV8_HOT_PARAMS \
  const int32_t *hot_table, const int32_t *hot_lens, const int32_t *hot_cu, int hot_max_pages, int hot_total, int hot_max_tokens
#define BD_KV8_HOT_ARGS(s) (s).block_table, (s).seq_lens, (s).cu, (s).max_pages, (s).total, (s).max_tokens
#define BD_KV8_HOT(s)                             \
  (s).block_table = hot_table;                    \
  (s).seq_lens = const_cast<int32_t*>(hot_lens);  \
  (s).cu = hot_cu;                                \
  (s).max_pages = hot_max_pages;                  \
  (s).total = hot_total;                          \
  (s).max_tokens = hot_max_tokens

struct Rotate8 {
  const float* table;
  const int32_t* positions;
  int n_positions, dim, interleaved;
};

struct Scores8 {
  float scale, cap;
  const float* slopes;
  const int32_t* prefix;
  int window;
};

hipError_t launch_kv8_append(const Step8& s, int head_dim, int code, int elem, const Rows8& k, const Rows8& v, const Rows8& q,
                             const Rows8& q_out, const Rotate8& rot, hipStream_t st);
hipError_t launch_kv8_advance(const Step8& s, hipStream_t st);
hipError_t launch_kv8_attn(const Step8& s, bool few, int head_dim, int code, int elem, const Rows8& q, const Scores8& sc, int splits, void* ws,
                           void* out, hipStream_t st);
int kv8_splits(const bd_paged8_cache* c, int max_tokens, int max_len);

#ifdef __HIPCC__
namespace {

// Where the step's rows of sequence b are and what it holds before them; false: it is to be left out (or has no rows).  every_thread: b is the thread's own.
struct Seq8 {
  int len, row, n;   // tokens before the step, first row, rows
};
struct PlainLoad {
  __device__ __forceinline__ int32_t operator()(const int32_t* p) const { return *p; }
};
template <class Load = PlainLoad>
__device__ __forceinline__ bool step_rows(const Step8& s, int b, Seq8& q, bool every_thread = false, Load load = Load()) {
  q.len = load(s.seq_lens + b);
  q.row = s.cu ? load(s.cu + b) : b;
  const int end = s.cu ? load(s.cu + b + 1) : b + 1;
  const bool rows = q.row >= 0 && end >= q.row && end <= s.total;
  q.n = rows ? end - q.row : 0;
  const bool fits = rows && q.n <= s.max_tokens && q.len >= 0 && q.len <= 0x7fffffff - q.n;
  if (!fits && s.status && (every_thread || threadIdx.x == 0)) atomicOr(s.status, kStatusRows);
  return fits && q.n > 0;
}

__device__ __forceinline__ int page_of(const Step8& s, int b, int block) {
  const int page = block < s.max_pages ? s.block_table[(size_t)b * s.max_pages + block] : -1;
  return page >= 0 && page < s.num_pages ? page : -1;
}

}  // namespace
#endif

}  // namespace bd
