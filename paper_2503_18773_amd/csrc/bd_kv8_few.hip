// Attention over the paged 8-bit cache of few query rows: decoding, and a few tokens a sequence at once.
#include "bd_kv8_device.h"
#include "bd_kv8_part.h"

namespace bd {
namespace {

// Sixteen rows (a token's query head each, token by token) of one KV head against blocks of 128 tokens, a wave a block.
// Per block  S^T = K Q^T  and  O^T += V^T P^T  with 16 x 16 x 32 products, tokens x rows and channels x rows: a lane holds
// scores and outputs of one row, and its scores are, as they come, the eight tokens that the second product wants of the lane.
// The order of tokens inside of the products is free, and chosen so that a lane's codes are 16 adjacent bytes: S^T's row 4 a + i of
// tile t is token 32 a + 4 t + i, so lane group g has tokens 32 g .. 32 g + 31; likewise the channels of K.
template <int D, int CODE, int ELEM>
struct Few {
  static constexpr int kChunks = D / 64, kSteps = D / 32, kTiles = D / 16;
  int lane, col, grp;
  h8_t q[kSteps];
  float c;       // scores in natural units per product and K scale
  RowView view;
  float m, l;    // running maximum (base 2, scale included) and sum of the lane's row
  f4_t acc[kTiles];

  __device__ __forceinline__ void scores(f4_t* s, int n, float ck, int from, int stride, int per_tile, bool masked, int end, const Scores8& sc) const {
    // s[t][i] is token from + stride * grp + per_tile * t + i
    const bool plain = !(sc.cap > 0.f) && !sc.slopes;
    const float inv_cap = sc.cap > 0.f ? 1.f / sc.cap : 0.f;
#pragma unroll
    for (int t = 0; t < n; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = from + stride * grp + per_tile * t + i;
        float x = s[t][i] * (plain ? ck * kLog2e : ck);
        if (!plain) {
          if (sc.cap > 0.f) x = capped(x, sc.cap, inv_cap);
          if (sc.slopes) x -= view.slope * (float)abs(view.pos - j);
          x *= kLog2e;
        }
        if (masked && !(j < end && view.sees(j))) x = -INFINITY;
        s[t][i] = x;
      }
  }
  // weights in place of scores; lv: the block's V scale, ref: the reference scale, both as logarithms
  __device__ __forceinline__ void weights(f4_t* s, int n, float lv, float ref) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < n; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
    top = join_groups(top, Max()) + lv;
    const float now = fmaxf(m, top), base = now == -INFINITY ? 0.f : now;
    const float was = __builtin_amdgcn_exp2f(m - base), off = lv - base + kShift;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < n; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[t][i] = __builtin_amdgcn_exp2f(s[t][i] + off);
        sum += s[t][i];
      }
    l = l * was + join_groups(sum, Add()) * __builtin_amdgcn_exp2f(fminf(fmaxf(ref - lv, -100.f), 100.f));
    m = now;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[dt][i] *= was;
  }
};

template <int D, int CODE, int ELEM>
__global__ __launch_bounds__(256, 2) void kv8_few_kernel(Step8 s, Rows8 q, Scores8 sc, int splits, float* part, uint16_t* out) {
  typedef Few<D, CODE, ELEM> F;
  __shared__ float lds[4 * 16 * (D + 4) + 4 * 16 * 2];
  const int b = blockIdx.z, h = blockIdx.y % s.n_kv_heads, tile = blockIdx.y / s.n_kv_heads, split = blockIdx.x;
  Seq8 sq;
  if (!step_rows(s, b, sq)) return;
  const int rows = sq.n * s.gq;
  if (16 * tile >= rows) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  F f;
  f.lane = threadIdx.x & 63;
  f.col = f.lane & 15;
  f.grp = f.lane >> 4;
  const int row = min(16 * tile + f.col, rows - 1), token = row / s.gq, head = h * s.gq + row % s.gq;
  const int length = sq.len + sq.n, lo = sq.len + 16 * tile / s.gq, hi = sq.len + min(16 * tile + 15, rows - 1) / s.gq;
  f.view.pos = sq.len + token;
  f.view.prefix = sc.prefix ? min(max(sc.prefix[b], 0), length) : 0;
  f.view.window = sc.window;
  f.view.slope = sc.slopes ? sc.slopes[head] : 0.f;
  const uint16_t* q_row = q.data + (sq.row + token) * q.token + head * q.head;
  us8_t raw[F::kSteps];
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < F::kSteps; ++k) {
    raw[k] = *(const us8_t*)(q_row + 64 * (k / 2) + 16 * f.grp + 8 * (k % 2));
    most = max(most, most_of(raw[k]));
  }
  int shift = 0;
  if (ELEM == BD_ELEM_BF16) {
    most = __float_as_uint(join_groups(__uint_as_float(most), Max()));   // (bit patterns of positive numbers)
    shift = bf16_shift(most);
  }
#pragma unroll
  for (int k = 0; k < F::kSteps; ++k) f.q[k] = query8<ELEM>(raw[k], shift);
  f.c = ldexpf(sc.scale, -shift);
  f.m = -INFINITY;
  f.l = 0.f;
#pragma unroll
  for (int dt = 0; dt < F::kTiles; ++dt) f.acc[dt] = f4_t{0.f, 0.f, 0.f, 0.f};

  const Blocks blocks(lo, hi, length, f.view.prefix, sc.window, s.max_pages);
  const float ref = scale_reference(s, blocks, b, h, f.lane);
  bool missing = blocks.lacks;
  for (int it = 4 * split + wave; it < blocks.count; it += 4 * splits) {
    const int block = blocks[it], page = __builtin_amdgcn_readfirstlane(page_of(s, b, block));
    if (page < 0) {
      missing = true;
      continue;
    }
    const size_t unit = (size_t)page * s.n_kv_heads + h;
    const uint8_t* kc = s.k_codes + unit * (kBlock * D) + (32 * (f.col >> 2) + (f.col & 3)) * D + 16 * f.grp;
    const uint8_t* vc = s.v_codes + unit * (kBlock * D) + f.col * kBlock + 32 * f.grp;
    u4_t kw[8][F::kChunks], vw[F::kTiles][2];
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int p = 0; p < F::kChunks; ++p) kw[t][p] = *(const u4_t*)(kc + 4 * t * D + 64 * p);
#pragma unroll
    for (int dt = 0; dt < F::kTiles; ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u) vw[dt][u] = *(const u4_t*)(vc + 16 * dt * kBlock + 16 * u);
    const float ks = s.k_scales[unit], vs = s.v_scales[unit];
    f4_t x[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      x[t] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < F::kChunks; ++p) {
        x[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<CODE>(kw[t][p][0], kw[t][p][1]), f.q[2 * p], x[t], 0, 0, 0);
        x[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<CODE>(kw[t][p][2], kw[t][p][3]), f.q[2 * p + 1], x[t], 0, 0, 0);
      }
    }
    f.scores(x, 8, f.c * ks, block * kBlock, 32, 4, !all_seen(block * kBlock, lo, hi, f.view.prefix, sc.window), 0x7fffffff, sc);
    f.weights(x, 8, vs > 0.f ? log2f(vs) : ref, ref);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      h8_t p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (_Float16)x[2 * k + e / 4][e % 4];
#pragma unroll
      for (int dt = 0; dt < F::kTiles; ++dt)
        f.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8<CODE>(vw[dt][k / 2][2 * (k % 2)], vw[dt][k / 2][2 * (k % 2) + 1]), p, f.acc[dt], 0, 0, 0);
    }
  }
  if (missing && s.status && f.lane == 0) atomicOr(s.status, kStatusRead);

  // the residual: 32 tokens a wave, of the workgroup whose waves would be next
  const int tail = length % kBlock, from = 32 * wave;
  if (blocks.tail && split == (blocks.count + 3) / 4 % splits && from < tail) {
    const size_t unit = (size_t)b * s.n_kv_heads + h;
    const uint16_t* kr = s.k_res + unit * (kBlock * D) + (from + 8 * (f.col >> 2) + (f.col & 3)) * D + 16 * f.grp;
    const uint16_t* vr = s.v_res + unit * (kBlock * D) + (from + 8 * f.grp) * D + f.col;
    us8_t kx[2][F::kSteps], vx[F::kTiles];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int k = 0; k < F::kSteps; ++k) kx[t][k] = *(const us8_t*)(kr + 4 * t * D + 64 * (k / 2) + 8 * (k % 2));
#pragma unroll
    for (int dt = 0; dt < F::kTiles; ++dt)
#pragma unroll
      for (int e = 0; e < 8; ++e) vx[dt][e] = from + 8 * f.grp + e < tail ? vr[e * D + 16 * dt] : (uint16_t)0;   // (rows behind the last are anything)
    f4_t x[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      x[t] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < F::kSteps; ++k) {
        if (ELEM == BD_ELEM_F16)
          x[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, kx[t][k]), f.q[k], x[t], 0, 0, 0);
        else
          x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, kx[t][k]), __builtin_bit_cast(bf8_t, raw[k]), x[t], 0, 0, 0);
      }
    }
    f.scores(x, 2, sc.scale, length - tail + from, 8, 4, true, length, sc);
    f.weights(x, 2, 0.f, ref);
    if (ELEM == BD_ELEM_F16) {
      h8_t p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (_Float16)x[e / 4][e % 4];
#pragma unroll
      for (int dt = 0; dt < F::kTiles; ++dt)
        f.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, vx[dt]), p, f.acc[dt], 0, 0, 0);
    } else {
      // bf16 values want bf16 weights: in two pieces, 16 bits of them
      bf8_t p, p2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = (__bf16)x[e / 4][e % 4];
        p2[e] = (__bf16)(x[e / 4][e % 4] - (float)p[e]);
      }
#pragma unroll
      for (int dt = 0; dt < F::kTiles; ++dt) {
        f.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, vx[dt]), p, f.acc[dt], 0, 0, 0);
        f.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, vx[dt]), p2, f.acc[dt], 0, 0, 0);
      }
    }
  }

  // the four waves' results, in units of 2^(m - kShift) and, the sums, of 2^ref
  float* ml = lds + 4 * 16 * (D + 4);
  if (f.grp == 0) {
    ml[(wave * 16 + f.col) * 2] = f.m;
    ml[(wave * 16 + f.col) * 2 + 1] = f.l;
  }
#pragma unroll
  for (int dt = 0; dt < F::kTiles; ++dt) *(f4_t*)(lds + (wave * 16 + f.col) * (D + 4) + 16 * dt + 4 * f.grp) = f.acc[dt];
  __syncthreads();
  constexpr int kPer = D / 16;   // channels a thread
  const int r = threadIdx.x / 16, d = threadIdx.x % 16 * kPer;
  if (16 * tile + r >= rows) return;
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[(w * 16 + r) * 2]);
  float o[kPer] = {}, sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float fac = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[(w * 16 + r) * 2] - top);
    sum += fac * ml[(w * 16 + r) * 2 + 1];
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] += fac * lds[(w * 16 + r) * (D + 4) + d + e];
  }
  const float unit = __builtin_amdgcn_exp2f(ref);
  const int tk = (16 * tile + r) / s.gq, hd = h * s.gq + (16 * tile + r) % s.gq;
  const size_t at = (size_t)(sq.row + tk) * s.n_q_heads + hd;
  if (splits > 1) {
    store_part<D, kPer>(part, splits, (size_t)s.total * s.n_q_heads, split, at, d, o, unit, top, sum);
    return;
  }
  const float inv = sum > 0.f ? unit / sum : 0.f;
#pragma unroll
  for (int e = 0; e < kPer; e += 2) *(uint32_t*)(out + at * D + d + e) = elem2<ELEM>(o[e] * inv, o[e + 1] * inv);
}

}  // namespace

hipError_t launch_kv8_few(const Step8& s, int head_dim, int code, int elem, const Rows8& q, const Scores8& sc, int splits, float* part,
                          void* out, hipStream_t st) {
  const int tiles = (int)(((long)s.max_tokens * s.gq + 15) / 16);
  const dim3 grid(splits, s.n_kv_heads * tiles, s.batch);
#define BD_RUN(D, C, E) hipLaunchKernelGGL((kv8_few_kernel<D, C, E>), grid, dim3(256), 0, st, s, q, sc, splits, part, (uint16_t*)out)
  BD_KV8_INSTANCES(head_dim, code, elem, BD_RUN)
#undef BD_RUN
  return hipGetLastError();
}

}  // namespace bd
