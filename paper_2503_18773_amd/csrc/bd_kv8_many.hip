// Attention over the paged 8-bit cache of many query rows: prompts and pieces of prompts.
#include "bd_kv8_device.h"
#include "bd_kv8_part.h"

namespace bd {
namespace {

constexpr int kManyRows = 128;   // rows of a workgroup, 32 of each wave

// 128 rows (a token's query head each, token by token) of one KV head against blocks of 128 tokens, one after the other.  A block's
// codes come through registers, requested a block ahead, and are put into LDS as fp16, once for all waves.  Per block
// S^T = K Q^T  and  O^T += V^T P^T  with 32 x 32 x 16 products: a lane holds scores and outputs of one row, and its scores are, as they
// come, the tokens that the second product wants of the lane, if row m of K's tile is token m with bits 2 and 3 exchanged.
template <int D, int CODE, int ELEM>
__global__ __launch_bounds__(256, 2) void kv8_many_kernel(Step8 s, Rows8 q, Scores8 sc, int splits, float* part, uint16_t* out) {
  constexpr int kSteps = D / 16, kTiles = D / 32, kUnits = kBlock * D / 16 / 256;   // 16-code units of a thread, of K and of V
  constexpr int kRowChunks = D / 8, kKMask = kRowChunks - 1;   // chunks of 8 elements, exchanged by the row's low bits against bank conflicts
  __shared__ __align__(16) uint16_t lds_k[kBlock * D], lds_v[kBlock * D];
  const int h = blockIdx.x, b = blockIdx.z;
  const int tile = (int)(gridDim.y / splits - 1 - blockIdx.y / splits), split = blockIdx.y % splits;   // (the longest first)
  Seq8 sq;
  if (!queries_of(s, b, sq)) return;
  const int rows = sq.n * s.gq;
  if (kManyRows * tile >= rows) return;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first_row = kManyRows * tile + 32 * wave;
  const int row = min(first_row + col, rows - 1), token = row / s.gq, head = h * s.gq + row % s.gq;
  const int length = sq.len + sq.n;
  const int lo = sq.len + kManyRows * tile / s.gq, hi = sq.len + min(kManyRows * tile + kManyRows - 1, rows - 1) / s.gq;   // positions of the workgroup's rows
  const int wave_lo = sq.len + min(first_row, rows - 1) / s.gq, wave_hi = sq.len + min(first_row + 31, rows - 1) / s.gq;
  RowView view;
  view.pos = sq.len + token;
  view.prefix = sc.prefix ? min(max(scalar_load(sc.prefix + b), 0), length) : 0;
  view.window = window_of(sc.window);
  view.slope = sc.slopes ? sc.slopes[head] : 0.f;

  const uint16_t* q_row = q.data + (sq.row + token) * q.token + head * q.head + 8 * half;
  h8_t qf[kSteps];
  int shift = 0;
  {
    us8_t raw[kSteps];
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      raw[k] = *(const us8_t*)(q_row + 16 * k);
      most = max(most, most_of(raw[k]));
    }
    if (ELEM == BD_ELEM_BF16) shift = bf16_shift(__float_as_uint(join_xor32(__uint_as_float(most), Max())));
#pragma unroll
    for (int k = 0; k < kSteps; ++k) qf[k] = query8<ELEM>(raw[k], shift);
  }
  const float c = ldexpf(sc.scale, -shift);

  const Blocks blocks(lo, hi, length, view.prefix, sc.window, s.max_pages);
  const int32_t* table = s.block_table + (size_t)b * s.max_pages;
  const float ref = scale_reference(s, table, blocks, h);
  float m = -INFINITY, l = 0.f;
  f16x_t acc[kTiles];
#pragma unroll
  for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;

  const int at_k = ((col & 0x13) | (col & 4) << 1 | (col & 8) >> 1);   // K's row of this lane in a tile of 32
  auto frag_k = [&](int t, int k) {
    const int r = 32 * t + at_k;
    return *(const h8_t*)(lds_k + r * D + 8 * ((2 * k + half) ^ (r & kKMask)));
  };
  auto frag_v = [&](int dt, int chunk) {
    const int r = 32 * dt + col;
    return *(const h8_t*)(lds_v + r * kBlock + 8 * (chunk ^ (r & 15)));
  };
  // scores to weights; returns nothing, changes m, l, acc
  f16x_t x[4];
  auto weigh = [&](int from, float ck, bool masked, bool gone, float lv) {
    finish_scores<f16x_t, 4>(x, ck, sc, view, masked, from + 8 * half, [](int t, int i) { return 32 * t + 16 * (i / 8) + i % 8; });
    if (gone) no_scores<f16x_t, 4>(x);
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[t][i]);
    top = join_xor32(top, Max()) + lv;
    const float now = fmaxf(m, top), base = now == -INFINITY ? 0.f : now;
    const float was = __builtin_amdgcn_exp2f(m - base), off = lv - base + kShift;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[t][i] = __builtin_amdgcn_exp2f(x[t][i] + off);
        sum += x[t][i];
      }
    l = l * was + join_xor32(sum, Add()) * __builtin_amdgcn_exp2f(fminf(fmaxf(ref - lv, -100.f), 100.f));
    m = now;
    if (__any(was != 1.f)) {
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] *= was;
    }
  };

  // this split's blocks, the residual with the last split
  const int begin = (int)((long)blocks.count * split / splits), end = (int)((long)blocks.count * (split + 1) / splits);
  u4_t kw[kUnits], vw[kUnits];
  bool missing = blocks.lacks;
  auto request = [&](int page) {   // (a block that is not there: any page's bytes, and none of its tokens seen)
    const size_t unit = (size_t)max(page, 0) * s.n_kv_heads + h;
    const u4_t* kc = (const u4_t*)(s.k_codes + unit * (kBlock * D));
    const u4_t* vc = (const u4_t*)(s.v_codes + unit * (kBlock * D));
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
      kw[n] = kc[n * 256 + threadIdx.x];
      vw[n] = vc[n * 256 + threadIdx.x];
    }
  };
  int next_page = page_in(s, table, blocks, begin);
  if (begin < end) request(next_page);
  for (int it = begin; it < end; ++it) {
    const int page = next_page, from = blocks[it] * kBlock;
    const bool gone = page < 0;
    missing |= gone;
    next_page = page_in(s, table, blocks, it + 1);
    const size_t unit = (size_t)max(page, 0) * s.n_kv_heads + h;
    const float ks = scalar_scale(s.k_scales + unit), vs = scalar_scale(s.v_scales + unit);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
      const int u = n * 256 + threadIdx.x;
      const int kr = u / (D / 16), kx = 2 * (u % (D / 16)), vr = u / 8, vx = 2 * (u % 8);
      *(h8_t*)(lds_k + kr * D + 8 * (kx ^ (kr & kKMask))) = codes8<CODE>(kw[n][0], kw[n][1]);
      *(h8_t*)(lds_k + kr * D + 8 * ((kx + 1) ^ (kr & kKMask))) = codes8<CODE>(kw[n][2], kw[n][3]);
      *(h8_t*)(lds_v + vr * kBlock + 8 * (vx ^ (vr & 15))) = codes8<CODE>(vw[n][0], vw[n][1]);
      *(h8_t*)(lds_v + vr * kBlock + 8 * ((vx + 1) ^ (vr & 15))) = codes8<CODE>(vw[n][2], vw[n][3]);
    }
    __syncthreads();
    if (it + 1 < end) request(next_page);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(frag_k(t, k), qf[k], x[t], 0, 0, 0);
    }
    weigh(from, c * ks, !all_seen(from, wave_lo, wave_hi, view.prefix, sc.window), gone, vs > 0.f ? log2f(vs) : ref);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        h8_t p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (_Float16)x[t][8 * u + e];
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(frag_v(dt, 4 * t + 2 * u + half), p, acc[dt], 0, 0, 0);
      }
  }
  if (missing && s.status && threadIdx.x == 0) atomicOr(s.status, kStatusRead);

  if (blocks.tail && split == splits - 1) {
    const int tail = length % kBlock;
    const size_t unit = (size_t)b * s.n_kv_heads + h;
    const uint16_t* kr = s.k_res + unit * (kBlock * D);
    const uint16_t* vr = s.v_res + unit * (kBlock * D);
    __syncthreads();
    for (int u = threadIdx.x; u < kBlock * kRowChunks; u += 256) {
      const int t = u / kRowChunks, ch = u % kRowChunks;
      // (rows behind the last are anything)
      us8_t kv = {}, vv = {};
      if (t < tail) {
        kv = *(const us8_t*)(kr + t * D + 8 * ch);
        vv = *(const us8_t*)(vr + t * D + 8 * ch);
      }
      *(us8_t*)(lds_k + t * D + 8 * (ch ^ (t & kKMask))) = kv;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = 8 * ch + e;
        lds_v[d * kBlock + 8 * ((t / 8) ^ (d & 15)) + t % 8] = vv[e];
      }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        if (ELEM == BD_ELEM_F16)
          x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(frag_k(t, k), qf[k], x[t], 0, 0, 0);
        else
          x[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, frag_k(t, k)), *(const bf8_t*)(q_row + 16 * k), x[t], 0, 0, 0);
      }
    }
    weigh(length - tail, sc.scale, true, false, 0.f);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (ELEM == BD_ELEM_F16) {
          h8_t p;
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = (_Float16)x[t][8 * u + e];
#pragma unroll
          for (int dt = 0; dt < kTiles; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(frag_v(dt, 4 * t + 2 * u + half), p, acc[dt], 0, 0, 0);
        } else {
          // bf16 values want bf16 weights: in two pieces, 16 bits of them
          bf8_t p, p2;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] = (__bf16)x[t][8 * u + e];
            p2[e] = (__bf16)(x[t][8 * u + e] - (float)p[e]);
          }
#pragma unroll
          for (int dt = 0; dt < kTiles; ++dt) {
            const bf8_t v = __builtin_bit_cast(bf8_t, frag_v(dt, 4 * t + 2 * u + half));
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p, acc[dt], 0, 0, 0);
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p2, acc[dt], 0, 0, 0);
          }
        }
      }
  }

  if (first_row + col >= rows) return;
  const float unit = __builtin_amdgcn_exp2f(ref);
  const size_t at = (size_t)(sq.row + token) * s.n_q_heads + head;
  const float inv = l > 0.f ? unit / l : 0.f;
#pragma unroll
  for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * dt + 8 * g + 4 * half;
      const float o[4] = {acc[dt][4 * g], acc[dt][4 * g + 1], acc[dt][4 * g + 2], acc[dt][4 * g + 3]};
      if (splits > 1)
        store_part<D, 4>(part, splits, (size_t)s.total * s.n_q_heads, split, at, d, o, unit, m, l);
      else
        *(u2_t*)(out + at * D + d) = u2_t{elem2<ELEM>(o[0] * inv, o[1] * inv), elem2<ELEM>(o[2] * inv, o[3] * inv)};
    }
}

}  // namespace

hipError_t launch_kv8_many(const Step8& s, int head_dim, int code, int elem, const Rows8& q, const Scores8& sc, int splits, float* part,
                           void* out, hipStream_t st) {
  const int tiles = (int)(((long)s.max_tokens * s.gq + kManyRows - 1) / kManyRows);
  const dim3 grid(s.n_kv_heads, tiles * splits, s.batch);
#define BD_RUN(D, C, E) hipLaunchKernelGGL((kv8_many_kernel<D, C, E>), grid, dim3(256), 0, st, s, q, sc, splits, part, (uint16_t*)out)
  BD_KV8_INSTANCES(head_dim, code, elem, BD_RUN)
#undef BD_RUN
  return hipGetLastError();
}

}  // namespace bd
