// Attention over the paged 8-bit cache of many query rows: prompts and pieces of prompts.
#include "bd_kv8_device.h"
#include "bd_kv8_part.h"

namespace bd {
namespace {

// 256 rows (a token's query head each, token by token) of one KV head against blocks of 128 tokens, one after the other.  A block's
// codes come through registers and are put into LDS as fp16, once for all waves.  Per block
// S^T = K Q^T  and  O^T += V^T P^T  with 32 x 32 x 16 products: a lane holds scores and outputs of one row, and its scores are, as they
// come, the tokens that the second product wants of the lane, if row m of K's tile is token m with bits 2 and 3 exchanged.
//
// Both products of a block take the matrix unit as long as its weights (an exponential each) take the vector unit, so the two waves of
// a SIMD are kept half a block apart: in every phase, between two barriers, one has products and the other weights.
//   phase          2 i             2 i + 1         2 i + 2             2 i + 3
//   waves 0 .. 3   ..., K_i        weights i       V_i, K_i+1          weights i + 1
//   waves 4 .. 7   weights i - 1   V_i-1, K_i      weights i           V_i, K_i+1
// With the weights a wave puts its share of codes into LDS, where two blocks' keys and two blocks' values have room: waves 0 .. 3 with
// weights i those of K_i+1 and V_i, waves 4 .. 7 those of K_i+2 and V_i+1, which is after the last use of the block that was there before
// and ahead of the first of the new one; and requests the next ones.
template <int D, int CODE, int ELEM, int WAVES, bool PHASED>
__global__ __launch_bounds__(64 * WAVES, 2) void kv8_many_kernel(Step8 s, Rows8 q, Scores8 sc, int splits, float* part, uint16_t* out) {
  constexpr int kSteps = D / 16, kTiles = D / 32, kThreads = 64 * WAVES, kManyRows = 32 * WAVES, kUnits = kBlock * D / 16 / kThreads;   // 16-code units of a thread, of K and of V
  constexpr int kRowChunks = D / 8;
  constexpr int kPitchK = D + 8, kPitchV = kBlock + 8;   // (16 bytes more than a row: 16 rows then lie in all of the banks)
  constexpr int kSizeK = kBlock * kPitchK, kSizeV = D * kPitchV;
  __shared__ __align__(16) uint16_t lds_k[2 * kSizeK], lds_v[2 * kSizeV];
  const int h = blockIdx.x, b = blockIdx.z;
  const int tile = (int)(gridDim.y / splits - 1 - blockIdx.y / splits), split = blockIdx.y % splits;   // (the longest first)
  Seq8 sq;
  if (!queries_of(s, b, sq)) return;
  const int rows = sq.n * s.gq;
  if (kManyRows * tile >= rows) return;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool early = wave < 4;
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

  const int32_t* table = s.block_table + (size_t)b * s.max_pages;
  const Blocks blocks(lo, hi, length, view.prefix, sc.window, s.max_pages);
  // this split's blocks, the residual with the last split
  const int begin = (int)((long)blocks.count * split / splits), count = (int)((long)blocks.count * (split + 1) / splits) - begin;
  bool missing = blocks.lacks;
  auto page_of_block = [&](int i) { return i < count ? page_in(s, table, blocks, begin + i) : -1; };
  u4_t kw[kUnits], vw[kUnits];
  const uint32_t at = 16 * threadIdx.x;
  // (a block that is not there: any page's bytes, and none of its tokens seen)
  auto request = [&](u4_t* w, const uint8_t* codes, int page) {
    const uint8_t* from = codes + ((size_t)max(page, 0) * s.n_kv_heads + h) * (kBlock * D);
#pragma unroll
    for (int n = 0; n < kUnits; ++n) w[n] = *(const u4_t*)(from + 16 * kThreads * n + at);
  };
  constexpr int kPer = D / 16;   // units of a token's channels
  uint16_t* const k_to = lds_k + (threadIdx.x / kPer) * kPitchK + 16 * (threadIdx.x % kPer);
  uint16_t* const v_to = lds_v + (threadIdx.x / 8) * kPitchV + 16 * (threadIdx.x % 8);
  auto put_k = [&](int slot) {
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
      h8_t* to = (h8_t*)(k_to + slot * kSizeK + n * (kThreads / kPer) * kPitchK);
      to[0] = codes8<CODE>(kw[n][0], kw[n][1]);
      to[1] = codes8<CODE>(kw[n][2], kw[n][3]);
    }
  };
  auto put_v = [&](int slot) {
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
      h8_t* to = (h8_t*)(v_to + slot * kSizeV + n * (kThreads / 8) * kPitchV);
      to[0] = codes8<CODE>(vw[n][0], vw[n][1]);
      to[1] = codes8<CODE>(vw[n][2], vw[n][3]);
    }
  };
  int pages[3] = {page_of_block(0), page_of_block(1), page_of_block(2)};   // of blocks i, i + 1, i + 2
  if (count > 0) {
    request(kw, s.k_codes, pages[0]);
    request(vw, s.v_codes, pages[0]);
  }

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
    for (int k = 0; k < kSteps; ++k) {
      if (sc.scale < 0.f) raw[k] ^= (uint16_t)0x8000;
      qf[k] = query8<ELEM>(raw[k], shift);
    }
  }
  const float c = ldexpf(fabsf(sc.scale), -shift);   // (the queries have its sign)
  const float ref = scale_reference(s, table, blocks, h);
  float m = -INFINITY, l = 0.f;
  f16x_t acc[kTiles];
#pragma unroll
  for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;

  const int at_k = ((col & 0x13) | (col & 4) << 1 | (col & 8) >> 1);   // K's row of this lane in a tile of 32
  const uint16_t* const k_from = lds_k + at_k * kPitchK + 8 * half;
  const uint16_t* const v_from = lds_v + col * kPitchV + 8 * half;
  f16x_t x[4];
  h8_t p[8];
  // (a step's operands are read from LDS during the one before; the fences keep the compiler from reading all of them at once,
  // for which there are no registers)
  auto products = [&](int slot) {
    const uint16_t* const from = k_from + slot * kSizeK;
    h8_t now[4], next[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
      now[t] = *(const h8_t*)(from + 32 * t * kPitchK);
    }
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      if (k + 1 < kSteps)
#pragma unroll
        for (int t = 0; t < 4; ++t) next[t] = *(const h8_t*)(from + 32 * t * kPitchK + 16 * (k + 1));
#pragma unroll
      for (int t = 0; t < 4; ++t) x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[t], qf[k], x[t], 0, 0, 0);
#pragma unroll
      for (int t = 0; t < 4; ++t) now[t] = next[t];
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto outputs = [&](int slot) {
    const uint16_t* const from = v_from + slot * kSizeV;
    h8_t now[kTiles], next[kTiles];
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) now[dt] = *(const h8_t*)(from + 32 * dt * kPitchV);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (u < 7)
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) next[dt] = *(const h8_t*)(from + 32 * dt * kPitchV + 16 * (u + 1));
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[dt], p[u], acc[dt], 0, 0, 0);
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) now[dt] = next[dt];
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Scores to weights, relative to a reference m that follows a row's largest score when that is 2^6 past it, which few blocks after
  // the first are: kShift leaves the weights' fp16 room for that.
  auto weigh = [&](Linear s_of, float lv) {
    float top = x[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[t][i]);
    top = fmaf(join_xor32(top, Max()), s_of.by, s_of.plus + lv);
    if (__any(top > m + 6.f)) {
      const float now = fmaxf(m, top), was = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= was;
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] *= was;
    }
    const float off = s_of.plus + lv - (m == -INFINITY ? 0.f : m) + kShift;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = __builtin_amdgcn_exp2f(fmaf(x[t][i], s_of.by, off));
  };
  // the row sum of this lane's tokens, in units of 2^ref
  auto add_up = [&](float sum, float lv) { l += sum * __builtin_amdgcn_exp2f(fminf(fmaxf(ref - lv, -100.f), 100.f)); };
  // A block's scales, requested a block ahead.  (By vector loads: they come in order with the codes' and behind nothing else, where a scalar load
  // would have to be waited for with the next operand from LDS.)
  float scale_k = 0.f, scale_v = 0.f;
  auto request_scales = [&](int page) {
    const size_t unit = (size_t)max(page, 0) * s.n_kv_heads + h;
    uint32_t zero = 0;
    asm("" : "+v"(zero));
    scale_k = (s.k_scales + unit)[zero];
    scale_v = (s.v_scales + unit)[zero];
  };
  auto weights = [&](int i, int page) {
    const int from = blocks[begin + i] * kBlock;
    const float ks = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(scale_k)));
    const float vs = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(scale_v)));
    request_scales(pages[1]);
    const float lv = vs > 0.f ? log2f(vs) : ref;
    missing |= page < 0;
    const Linear s_of = finish_scores<f16x_t, 4>(x, c * ks, sc, view, !all_seen(from, wave_lo, wave_hi, view.prefix, sc.window), from + 8 * half,
                                                 [](int t, int i) { return 32 * t + 16 * (i / 8) + i % 8; });
    if (page < 0) no_scores<f16x_t, 4>(x);
    weigh(s_of, lv);
    float sum = 0.f;
    const h2_t one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const h2_t w = {(_Float16)x[u / 2][8 * (u % 2) + e], (_Float16)x[u / 2][8 * (u % 2) + e + 1]};
        sum = __builtin_amdgcn_fdot2(w, one, sum, false);   // (of the weights as the product takes them)
        p[u][e] = w[0];
        p[u][e + 1] = w[1];
      }
    add_up(sum, lv);
  };

  if (count > 0) {
    put_k(0);
    request_scales(pages[0]);
    if (PHASED && !early) {
      request(kw, s.k_codes, pages[1]);
      put_v(0);
      request(vw, s.v_codes, pages[1]);
      put_k(1);
      request(kw, s.k_codes, pages[2]);
      __syncthreads();
      __syncthreads();
      for (int i = 0; i < count; ++i) {
        if (i > 0) outputs((i - 1) & 1);
        products(i & 1);
        __syncthreads();
        const int ahead = page_of_block(i + 3);
        weights(i, pages[0]);
        put_k(i & 1);
        put_v((i + 1) & 1);
        request(kw, s.k_codes, ahead);
        request(vw, s.v_codes, pages[2]);
        pages[0] = pages[1];
        pages[1] = pages[2];
        pages[2] = ahead;
        __syncthreads();
      }
      outputs((count - 1) & 1);
    } else {
      request(kw, s.k_codes, pages[1]);
      __syncthreads();
      products(0);
      if (PHASED) __syncthreads();
      for (int i = 0; i < count; ++i) {
        const int ahead = page_of_block(i + 3);
        weights(i, pages[0]);
        put_k((i + 1) & 1);
        put_v(i & 1);
        request(kw, s.k_codes, pages[2]);
        request(vw, s.v_codes, pages[1]);
        __syncthreads();
        outputs(i & 1);
        if (i + 1 < count) products((i + 1) & 1);
        pages[0] = pages[1];
        pages[1] = pages[2];
        pages[2] = ahead;
        if (PHASED) __syncthreads();
      }
    }
  }
  if (missing && s.status && lane == 0) atomicOr(s.status, kStatusRead);

  if (blocks.tail && split == splits - 1) {
    const int tail = length % kBlock;
    const size_t unit = (size_t)b * s.n_kv_heads + h;
    const uint16_t* kr = s.k_res + unit * (kBlock * D);
    const uint16_t* vr = s.v_res + unit * (kBlock * D);
    __syncthreads();
    for (int u = threadIdx.x; u < kBlock * kRowChunks; u += kThreads) {
      const int t = u / kRowChunks, ch = u % kRowChunks;
      // (rows behind the last are anything)
      us8_t kv = {}, vv = {};
      if (t < tail) {
        kv = *(const us8_t*)(kr + t * D + 8 * ch);
        vv = *(const us8_t*)(vr + t * D + 8 * ch);
      }
      *(us8_t*)(lds_k + t * kPitchK + 8 * ch) = kv;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lds_v[(8 * ch + e) * kPitchV + t] = vv[e];
      }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const h8_t kf = *(const h8_t*)(k_from + 32 * t * kPitchK + 16 * k);
        if (ELEM == BD_ELEM_F16)
          x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[k], x[t], 0, 0, 0);
        else
          x[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, kf), *(const bf8_t*)(q_row + 16 * k), x[t], 0, 0, 0);
      }
    }
    if (ELEM == BD_ELEM_BF16 && sc.scale < 0.f)   // (qf has its sign)
      for (int t = 0; t < 4; ++t) x[t] = -x[t];
    const Linear s_of = finish_scores<f16x_t, 4>(x, fabsf(sc.scale), sc, view, true, length - tail + 8 * half,
                                                 [](int t, int i) { return 32 * t + 16 * (i / 8) + i % 8; });
    weigh(s_of, 0.f);
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      h8_t p0;
      bf8_t p1, p2;   // bf16 values want bf16 weights: in two pieces, 16 bits of them
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = x[u / 2][8 * (u % 2) + e];
        sum += y;
        p0[e] = (_Float16)y;
        p1[e] = (__bf16)y;
        p2[e] = (__bf16)(y - (float)p1[e]);
      }
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) {
        const h8_t vf = *(const h8_t*)(v_from + 32 * dt * kPitchV + 16 * u);
        if (ELEM == BD_ELEM_F16) {
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, p0, acc[dt], 0, 0, 0);
        } else {
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, vf), p1, acc[dt], 0, 0, 0);
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, vf), p2, acc[dt], 0, 0, 0);
        }
      }
    }
    add_up(sum, 0.f);
  }

  l = join_xor32(l, Add());
  if (first_row + col >= rows) return;
  const float unit = __builtin_amdgcn_exp2f(ref);
  const size_t out_row = (size_t)(sq.row + token) * s.n_q_heads + head;
  const float inv = l > 0.f ? unit / l : 0.f;
#pragma unroll
  for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * dt + 8 * g + 4 * half;
      const float o[4] = {acc[dt][4 * g], acc[dt][4 * g + 1], acc[dt][4 * g + 2], acc[dt][4 * g + 3]};
      if (splits > 1)
        store_part<D, 4>(part, splits, (size_t)s.total * s.n_q_heads, split, out_row, d, o, unit, m, l);
      else
        *(u2_t*)(out + out_row * D + d) = u2_t{elem2<ELEM>(o[0] * inv, o[1] * inv), elem2<ELEM>(o[2] * inv, o[3] * inv)};
    }
}

// Head dimension 128: eight waves in phases, one workgroup on a compute unit (its LDS).  A prompt of 8192 tokens, 32 over 8 heads 652 us, in one phase
// 748, unphased with a barrier a block 666; 1024 tokens behind 31744, a window and a cap 354 / 437 / 387.
// 64: half the products to as many weights, so that there is less to put beside them: four waves, unphased, two workgroups on a unit.  Six prompts of up to 1333
// tokens, 16 heads and a bias 37 us, eight waves in phases 49 (unphased 40 against 31 without a bias); only a long prompt is better off with those, 8192
// tokens 457 / 430.  (Kernel times after a pause; 8192 tokens of head dimension 128 in a row of passes: 527 to 538 us, 1.02 to 1.04 PFLOP/s.)
template <int D, int CODE, int ELEM>
void run(const Step8& s, const Rows8& q, const Scores8& sc, int splits, float* part, void* out, hipStream_t st) {
  constexpr int kWaves = many_rows(D) / 32;
  const int tiles = (int)(((long)s.max_tokens * s.gq + many_rows(D) - 1) / many_rows(D));
  hipLaunchKernelGGL((kv8_many_kernel<D, CODE, ELEM, kWaves, kWaves == 8>), dim3(s.n_kv_heads, tiles * splits, s.batch), dim3(64 * kWaves), 0, st, s, q,
                     sc, splits, part, (uint16_t*)out);
}

}  // namespace

hipError_t launch_kv8_many(const Step8& s, int head_dim, int code, int elem, const Rows8& q, const Scores8& sc, int splits, float* part,
                           void* out, hipStream_t st) {
#define BD_RUN(D, C, E) run<D, C, E>(s, q, sc, splits, part, out, st)
  BD_KV8_INSTANCES(head_dim, code, elem, BD_RUN)
#undef BD_RUN
  return hipGetLastError();
}

}  // namespace bd
