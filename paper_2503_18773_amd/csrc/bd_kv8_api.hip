// C-ABI entry points of the paged 8-bit cache: argument validation, launches, and the merge of splits.
#include <algorithm>
#include <cmath>

#include "bd_kv8_part.h"

namespace bd {
namespace {

// A wave a row.
template <int D, int ELEM>
__global__ __launch_bounds__(256) void kv8_merge_kernel(Step8 s, int splits, const float* part, uint16_t* out) {
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  Seq8 sq;
  if (!queries_of(s, b, sq)) return;
  const long i = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= (long)sq.n * s.n_q_heads) return;
  const size_t rows = (size_t)s.total * s.n_q_heads, row = (size_t)sq.row * s.n_q_heads + i;
  const float* ml = part + (size_t)splits * rows * D + row * 2;
  float top = -INFINITY;
  for (int k = lane; k < splits; k += 64) top = fmaxf(top, ml[(size_t)k * rows * 2]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  constexpr int kPer = D / 64;
  float o[kPer] = {}, l = 0.f;
  if (top != -INFINITY) {
    for (int k = 0; k < splits; ++k) {
      const float fac = __builtin_amdgcn_exp2f(ml[(size_t)k * rows * 2] - top);
      l += fac * ml[(size_t)k * rows * 2 + 1];
      const float* from = part + ((size_t)k * rows + row) * D + lane * kPer;
#pragma unroll
      for (int e = 0; e < kPer; ++e) o[e] += fac * from[e];
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if (kPer == 2)
    *(uint32_t*)(out + row * D + 2 * lane) = elem2<ELEM>(o[0] * inv, o[kPer - 1] * inv);
  else
    out[row * D + lane] = (uint16_t)elem2<ELEM>(o[0] * inv, 0.f);
}

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bd_status hip_status(hipError_t e) {
  if (e == hipSuccess) return BD_OK;
  note_hip_error(e);
  return BD_ERR_HIP;
}

bd_status check_shape8(const bd_paged8_cache* c) {
  if (!c) return BD_ERR_INVALID_ARG;
  if (c->batch <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->num_pages <= 0 || c->max_pages_per_seq <= 0) return BD_ERR_INVALID_ARG;
  if (c->n_q_heads % c->n_kv_heads != 0) return BD_ERR_INVALID_ARG;
  if (c->code_type != BD_CODE_INT8 && c->code_type != BD_CODE_E4M3) return BD_ERR_INVALID_ARG;
  if (c->elem_type != BD_ELEM_F16 && c->elem_type != BD_ELEM_BF16) return BD_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return BD_ERR_UNSUPPORTED;
  if (c->batch > 65535 || c->n_q_heads > 32767) return BD_ERR_UNSUPPORTED;   // launch grid dimensions
  return BD_OK;
}

bd_status check_buffers8(const bd_paged8_cache* c) {
  const void* need[8] = {c->k_codes, c->v_codes, c->k_res, c->v_res, c->k_scales, c->v_scales, c->block_table, c->seq_lens};
  for (int i = 0; i < 8; ++i) {
    if (!need[i]) return BD_ERR_INVALID_ARG;
    if (!aligned(need[i], i < 4 ? 16 : 4)) return BD_ERR_ALIGNMENT;
  }
  return aligned(c->status, 4) ? BD_OK : BD_ERR_ALIGNMENT;
}

bd_status check_rows(const bd_rows* r) {
  if (!r || !r->data || r->token_stride < 0 || r->head_stride < 0) return BD_ERR_INVALID_ARG;
  if (!aligned(r->data, 16) || r->token_stride % 8 != 0 || r->head_stride % 8 != 0) return BD_ERR_ALIGNMENT;
  return BD_OK;
}

// The step's rows: whose they are.
bd_status check_step(const bd_paged8_cache* c, const int32_t* cu, int32_t total, int32_t max_tokens) {
  if (total < 0 || max_tokens < 1) return BD_ERR_INVALID_ARG;
  if (!cu && total != c->batch) return BD_ERR_INVALID_ARG;
  return aligned(cu, 4) ? BD_OK : BD_ERR_ALIGNMENT;
}

Step8 step_of(const bd_paged8_cache* c, const int32_t* cu, int32_t total, int32_t max_tokens) {
  Step8 s{};
  s.k_codes = (uint8_t*)c->k_codes;
  s.v_codes = (uint8_t*)c->v_codes;
  s.k_scales = c->k_scales;
  s.v_scales = c->v_scales;
  s.k_res = (uint16_t*)c->k_res;
  s.v_res = (uint16_t*)c->v_res;
  s.block_table = c->block_table;
  s.cu = cu;
  s.seq_lens = c->seq_lens;
  s.status = c->status;
  s.batch = c->batch;
  s.n_q_heads = c->n_q_heads;
  s.n_kv_heads = c->n_kv_heads;
  s.gq = c->n_q_heads / c->n_kv_heads;
  s.num_pages = c->num_pages;
  s.max_pages = c->max_pages_per_seq;
  s.total = total;
  s.max_tokens = cu ? std::min(max_tokens, total) : 1;
  return s;
}

Rows8 rows_of(const bd_rows* r) { return r ? Rows8{(uint16_t*)r->data, r->token_stride, r->head_stride} : Rows8{nullptr, 0, 0}; }

// Which kernel a call of up to `rows` rows (tokens times query heads) of a KV head takes: tiles of 16 or 32 rows whose waves have
// blocks of their own (launch_kv8_few), or tiles of many_rows() whose waves share blocks (launch_kv8_many).  The latter do twice as much with a
// block's codes, but leave compute units idle that the former's tiles, or splits of those, would fill:
// - up to 64 rows, and up to 256 where two splits of each tile find units (8 KV heads, behind 8192 tokens: 64 tokens of one sequence 36 us against
//   50, 17 of four 44 / 49; 64 of four, 256 tiles, 72 / 55);
// - one split, which is what kv8_splits chooses for short sequences, and one round and a half of tiles (prompts, one split: 1000 tokens of 2 KV heads, 250
//   tiles, 17 / 38; 256 of 8 KV heads, 256 tiles, 12 / 17.5; 100 of four sequences, 416 tiles, 13.4 / 15; 600 of 8 KV heads, 600 tiles, 31.6 / 29.6).
bool takes_few(const bd_paged8_cache* c, long rows, int num_splits) {
  const long tiles = (long)c->batch * c->n_kv_heads * few_tiles(rows);
  return rows <= 64 || (rows <= 256 && tiles <= 128) || (num_splits == 1 && tiles <= 448);
}

}  // namespace

// Few rows: one workgroup on a compute unit at most (it asks for as much as the unit can draw; 32 splits of 8 KV heads at 128K
// tokens 57 us, 64 splits 73).  Of those, a split takes some 0.6 us off for each of its blocks that it shares out, and costs its merge 0.02 us for each
// row: sqrt(30 blocks / rows) is best (4 rows, 8 units: 4095 tokens, 8 / 16 / 32 splits 12.7 / 11.6 / 14.3 us; 2047 tokens 4 / 8 / 16 splits
// 12.1 / 10.4 / 11.1; one unit, 60000 tokens 32 / 64 / 128 splits 24.9 / 21.7 / 24.4; 24 rows, one unit, 16000 tokens 62 splits 48.5, 13 splits 32.6).
// Up to four blocks are a wave's each in one workgroup, which spares the merge.
// Many rows: as many workgroups as compute units hold (of head dimension 64 two, of 128 one), eight blocks in each at least.
int kv8_splits(const bd_paged8_cache* c, int max_tokens, int max_len) {
  const long rows = (long)max_tokens * (c->n_q_heads / c->n_kv_heads);
  const long blocks = (std::max(max_len, 1) - 1L) / kBlock + 1;
  if (takes_few(c, rows, blocks <= 24 ? 1 : 2)) {
    const long held = std::min(rows, few_rows(rows)), units = (long)c->batch * c->n_kv_heads * few_tiles(rows);
    const long want = blocks <= 4 ? 1 : std::min((long)std::lround(std::sqrt(30. * blocks / held)), blocks);
    const long splits = std::max(1L, std::min(want, 256 / units));
    if (splits == 1 || takes_few(c, rows, 2)) return (int)splits;
    return 1;
  }
  const long units = (long)c->batch * c->n_kv_heads * ((rows + many_rows(c->head_dim) - 1) / many_rows(c->head_dim));
  return (int)std::max(1L, std::min((blocks + 7) / 8, (c->head_dim == 64 ? 512 : 256) / units));
}

hipError_t launch_kv8_attn(const Step8& s, bool few, int head_dim, int code, int elem, const Rows8& q, const Scores8& sc, int splits, void* ws,
                           void* out, hipStream_t st) {
  if (few) return launch_kv8_few(s, head_dim, code, elem, q, sc, splits, ws, out, st);
  float* part = (float*)((char*)ws + BD_PAGED8_COUNTER_BYTES);
  const hipError_t e = launch_kv8_many(s, head_dim, code, elem, q, sc, splits, part, out, st);
  if (e != hipSuccess || splits == 1) return e;
  const dim3 grid((unsigned)(((long)s.max_tokens * s.n_q_heads + 3) / 4), s.batch);
#define BD_RUN(D, E) hipLaunchKernelGGL((kv8_merge_kernel<D, E>), grid, dim3(256), 0, st, s, splits, part, (uint16_t*)out)
  if (head_dim == 64) {
    if (elem == BD_ELEM_F16) BD_RUN(64, BD_ELEM_F16);
    else BD_RUN(64, BD_ELEM_BF16);
  } else {
    if (elem == BD_ELEM_F16) BD_RUN(128, BD_ELEM_F16);
    else BD_RUN(128, BD_ELEM_BF16);
  }
#undef BD_RUN
  return hipGetLastError();
}

}  // namespace bd

using namespace bd;

extern "C" {

size_t bd_paged8_cache_bytes(const bd_paged8_cache* c, int which) {
  if (check_shape8(c) != BD_OK || which < 0 || which > 7) return 0;
  const size_t pool = (size_t)c->num_pages * c->n_kv_heads;
  switch (which) {
    case 0: case 1: return pool * kBlock * c->head_dim;
    case 2: case 3: return pool * 4;
    case 4: case 5: return (size_t)c->batch * c->n_kv_heads * kBlock * c->head_dim * 2;
    case 6: return (size_t)c->batch * c->max_pages_per_seq * 4;
    default: return (size_t)c->batch * 4;
  }
}

bd_status bd_paged8_append(const bd_paged8_cache* c, const bd_rows* k_new, const bd_rows* v_new, const bd_rows* q, const bd_rows* q_out,
                           const int32_t* cu_tokens, int32_t total, int32_t max_tokens, const bd_rotation* rot, void* stream) {
  bd_status s = check_shape8(c);
  if (s != BD_OK) return s;
  if ((s = check_buffers8(c)) != BD_OK || (s = check_step(c, cu_tokens, total, max_tokens)) != BD_OK) return s;
  if ((q == nullptr) != (q_out == nullptr) || (q && !rot)) return BD_ERR_INVALID_ARG;
  Rotate8 r{nullptr, nullptr, 1, 0, 0};
  if (rot) {
    if (!rot->cos_sin || rot->n_positions < 1 || rot->rotary_dim < 16 || rot->rotary_dim > c->head_dim || rot->rotary_dim % 16 != 0 ||
        (rot->interleaved != 0 && rot->interleaved != 1))
      return BD_ERR_INVALID_ARG;
    if (!aligned(rot->cos_sin, 16) || !aligned(rot->positions, 4)) return BD_ERR_ALIGNMENT;
    r = Rotate8{rot->cos_sin, rot->positions, rot->n_positions, rot->rotary_dim, rot->interleaved};
  }
  if (total == 0) return BD_OK;
  if ((s = check_rows(k_new)) != BD_OK || (s = check_rows(v_new)) != BD_OK) return s;
  if (q && ((s = check_rows(q)) != BD_OK || (s = check_rows(q_out)) != BD_OK)) return s;
  if (q && (q_out->token_stride < c->head_dim || q_out->head_stride < c->head_dim)) return BD_ERR_INVALID_ARG;   // rows on top of each other
  const Step8 st = step_of(c, cu_tokens, total, max_tokens);
  // a launch's threads, of which up to 512 are a workgroup: fewer than 2^32
  if (((long)st.max_tokens * (c->n_q_heads + 2 * c->n_kv_heads) * (c->head_dim / 16) + 255) / 256 + 2L * c->n_kv_heads * ((st.max_tokens - 1L) / kBlock + 1) > (1L << 23) - 1)
    return BD_ERR_UNSUPPORTED;
  return hip_status(launch_kv8_append(st, c->head_dim, c->code_type, c->elem_type, rows_of(k_new), rows_of(v_new), rows_of(q), rows_of(q_out),
                                      r, (hipStream_t)stream));
}

int32_t bd_paged8_choose_splits(const bd_paged8_cache* c, int32_t max_tokens, int32_t max_len) {
  if (check_shape8(c) != BD_OK || max_tokens < 1 || max_len < 1) return 1;
  return kv8_splits(c, max_tokens, max_len);
}

size_t bd_paged8_workspace_bytes(const bd_paged8_cache* c, int32_t total, int32_t max_tokens, int32_t num_splits) {
  if (check_shape8(c) != BD_OK || total < 1 || max_tokens < 1 || num_splits < 2) return 0;
  const long gq = c->n_q_heads / c->n_kv_heads;
  // (256: where splits are dealt by length there are as many as compute units)
  auto few = [&](long rows) {
    return std::max((size_t)std::min(num_splits, kMostSplits) * c->batch * c->n_kv_heads * few_tiles(rows), c->batch > 1 ? (size_t)256 : 0) * std::min(rows, few_rows(rows));
  };
  const long rows = std::min(max_tokens, total) * gq;
  size_t filed = takes_few(c, rows, num_splits) ? few(rows) : (size_t)num_splits * total * c->n_q_heads;
  if (takes_few(c, gq, num_splits)) filed = std::max(filed, few(gq));   // (a call without cu_tokens, whatever its max_tokens)
  return BD_PAGED8_COUNTER_BYTES + filed * (c->head_dim + 2) * sizeof(float);
}

bd_status bd_paged8_attn(const bd_paged8_cache* c, const bd_rows* q, const int32_t* cu_tokens, int32_t total, int32_t max_tokens,
                         const bd_scores* scores, int32_t num_splits, void* workspace, void* out, void* stream) {
  bd_status s = check_shape8(c);
  if (s != BD_OK) return s;
  if ((s = check_buffers8(c)) != BD_OK || (s = check_step(c, cu_tokens, total, max_tokens)) != BD_OK) return s;
  if (!scores || num_splits < 1 || scores->window < 0 || !(scores->softcap >= 0.f)) return BD_ERR_INVALID_ARG;
  if (scores->softcap > 1024.f) return BD_ERR_UNSUPPORTED;
  if (!aligned(scores->slopes, 4) || !aligned(scores->prefix_lens, 4)) return BD_ERR_ALIGNMENT;
  if (total == 0) return BD_OK;
  if ((s = check_rows(q)) != BD_OK) return s;
  if (!out || (num_splits > 1 && !workspace)) return BD_ERR_INVALID_ARG;
  if (!aligned(out, 16) || !aligned(workspace, 16)) return BD_ERR_ALIGNMENT;
  const Step8 st = step_of(c, cu_tokens, total, max_tokens);
  const long rows = (long)st.max_tokens * st.gq;
  const bool few = takes_few(c, rows, num_splits);
  // launch grid dimensions: KV heads x tiles of rows, tiles x splits; the merge's rows
  if (num_splits > 65535 || (few ? few_tiles(rows) * c->n_kv_heads : (rows + many_rows(c->head_dim) - 1) / many_rows(c->head_dim) * num_splits) > 65535 ||
      ((long)st.max_tokens * c->n_q_heads + 3) / 4 > (1L << 24) - 1)
    return BD_ERR_UNSUPPORTED;
  const Scores8 sc{scores->softmax_scale, scores->softcap, scores->slopes, scores->prefix_lens, scores->window};
  return hip_status(launch_kv8_attn(st, few, c->head_dim, c->code_type, c->elem_type, rows_of(q), sc, num_splits, workspace, out,
                                    (hipStream_t)stream));
}

bd_status bd_paged8_advance(const bd_paged8_cache* c, const int32_t* cu_tokens, int32_t total, int32_t max_tokens, void* stream) {
  bd_status s = check_shape8(c);
  if (s != BD_OK) return s;
  if ((s = check_buffers8(c)) != BD_OK || (s = check_step(c, cu_tokens, total, max_tokens)) != BD_OK) return s;
  if (total == 0) return BD_OK;
  return hip_status(launch_kv8_advance(step_of(c, cu_tokens, total, max_tokens), (hipStream_t)stream));
}

}  // extern "C"
