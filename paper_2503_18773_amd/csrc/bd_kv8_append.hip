// Appending a step's tokens to the paged 8-bit cache, with the position rotation on the way.
#include "bd_kv8.h"

namespace bd {
namespace {

typedef _Float16 half_t;
typedef __bf16 bf_t;
typedef uint16_t us8_t __attribute__((ext_vector_type(8)));

template <int ELEM>
__device__ __forceinline__ float to_f32(uint16_t b) {
  if (ELEM == BD_ELEM_BF16) return __uint_as_float((uint32_t)b << 16);
  return (float)__builtin_bit_cast(half_t, b);
}
template <int ELEM>
__device__ __forceinline__ uint16_t from_f32(float f) {
  if (ELEM == BD_ELEM_BF16) return __builtin_bit_cast(uint16_t, (bf_t)f);
  return __builtin_bit_cast(uint16_t, (half_t)f);
}

// A head's channels in vectors of 8, two of them (a, b) to a thread, so that a rotation's pairs meet in one: pair vector p
// has rotation pairs 8 p .. 8 p + 7.
struct PairVec {
  int a, b;
  bool turns;
  __device__ __forceinline__ PairVec(const Rotate8& r, int p) {
    turns = 16 * p < r.dim;
    const bool halves = turns && !r.interleaved;
    a = halves ? p : 2 * p;
    b = halves ? p + r.dim / 16 : 2 * p + 1;
  }
};

// cos and sin of a token's pairs 8 p .. 8 p + 7
struct Angles {
  float c[8], s[8];
  __device__ __forceinline__ void load(const Rotate8& r, int position, int p) {
    const float* at = r.table + (size_t)position * r.dim + 8 * p;
    const f4_t c0 = *(const f4_t*)at, c1 = *(const f4_t*)(at + 4);
    const f4_t s0 = *(const f4_t*)(at + r.dim / 2), s1 = *(const f4_t*)(at + r.dim / 2 + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c[e] = c0[e];
      c[e + 4] = c1[e];
      s[e] = s0[e];
      s[e + 4] = s1[e];
    }
  }
};
__device__ __forceinline__ int position_of(const Rotate8& r, const Step8& s, int row, int index) {
  int p = r.positions ? r.positions[row] : index;
  if (p < 0 || p >= r.n_positions) {
    if (s.status) atomicOr(s.status, kStatusPosition);
    p = p < 0 ? 0 : r.n_positions - 1;
  }
  return p;
}

// (x cos - y sin, x sin + y cos).  In 64 bits, where the products of a half and an fp32 number are exact and the sum's one
// rounding is far below the two that follow, to fp32 and to the element type: the keys are what their codes are chosen from,
// and a key that came out a step off would be another code.
template <int ELEM>
__device__ __forceinline__ void turn(uint16_t& x, uint16_t& y, float c, float s) {
  const double dx = to_f32<ELEM>(x), dy = to_f32<ELEM>(y), dc = c, ds = s;
  float fx = (float)(dx * dc - dy * ds), fy = (float)(dx * ds + dy * dc);
  asm("" : "+v"(fx), "+v"(fy));   // (the compiler would make one rounding of the two, by a long way round)
  x = from_f32<ELEM>(fx);
  y = from_f32<ELEM>(fy);
}
template <int ELEM>
__device__ __forceinline__ void turn_pair(us8_t& a, us8_t& b, const Angles& w, int interleaved) {
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint16_t x = a[2 * e], y = a[2 * e + 1];
      turn<ELEM>(x, y, w.c[e], w.s[e]);
      a[2 * e] = x;
      a[2 * e + 1] = y;
      x = b[2 * e];
      y = b[2 * e + 1];
      turn<ELEM>(x, y, w.c[4 + e], w.s[4 + e]);
      b[2 * e] = x;
      b[2 * e + 1] = y;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint16_t x = a[e], y = b[e];
      turn<ELEM>(x, y, w.c[e], w.s[e]);
      a[e] = x;
      b[e] = y;
    }
  }
}

__device__ __forceinline__ us8_t load8(const uint16_t* p) { return *(const us8_t*)p; }
__device__ __forceinline__ void store8(uint16_t* p, us8_t v) { *(us8_t*)p = v; }

// The largest magnitude of a workgroup's values, given each thread's largest bit pattern (magnitudes of a half type order as
// their bits do).
template <int WAVES>
__device__ __forceinline__ uint32_t group_max(uint32_t m, uint32_t* lds) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) m = max(m, lds[w]);
  return m;
}

// code = x / scale, the quotient rounded as IEEE division rounds it, so that the codes follow from the values alone, to the nearest.
// q = x r with r = 1 / scale rounded correctly is within a step of the quotient, and q + (x - q scale) r then is the quotient rounded correctly
// (Markstein's theorem; what the residue loses below 2^-149 is of quotients far below the smallest code).  Scales below 2^-90 are divided by.
struct Divisor {
  float scale, r;
  __device__ __forceinline__ Divisor(float s) : scale(s), r(s >= 0x1p-90f ? 1.f / s : 0.f) {}
  __device__ __forceinline__ float operator()(float x) const {
    const float q = x * r;
    return fmaf(fmaf(-q, scale, x), r, q);
  }
};
template <int CODE>
__device__ __forceinline__ uint32_t code4(const float* x, const Divisor& by) {
  constexpr float kMost = CODE == BD_CODE_INT8 ? 127.f : 448.f;
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = by(x[e]);
  if (by.r == 0.f) {   // (of the whole block)
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = by.scale > 0.f ? x[e] / by.scale : 0.f;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (CODE == BD_CODE_INT8) y[e] = rintf(y[e]);
    y[e] = fminf(fmaxf(y[e], -kMost), kMost);
  }
  if (CODE == BD_CODE_INT8)
    return ((uint32_t)(int)y[0] & 255u) | ((uint32_t)(int)y[1] & 255u) << 8 | ((uint32_t)(int)y[2] & 255u) << 16 | (uint32_t)(int)y[3] << 24;
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
}

// Two kinds of workgroups.  The first 2 H * blocks, which take longest: one block that the step completes, of one KV head's keys or
// values.  The first block of a sequence takes its older tokens from the residual, and its workgroup files what the step leaves behind
// the last block there afterwards: nobody else touches that head's residual.  The others: rows that stay in the element type, rotated
// queries and, if the step completes no block of the sequence, keys and values on their way to the residual; a thread has
// one pair vector of up to `heads` heads of a token.
template <int D, int CODE, int ELEM>
__global__ __launch_bounds__(4 * D) void kv8_append_kernel(BD_KV8_HOT_PARAMS, int heads, int blocks, Step8 s, Rows8 k, Rows8 v, Rows8 q, Rows8 q_out,
                                                           Rotate8 rot) {
  BD_KV8_HOT(s);
  constexpr int kThreads = 4 * D;
  constexpr int kPairs = D / 16;
  constexpr float kMost = CODE == BD_CODE_INT8 ? 127.f : 448.f;
  __shared__ uint32_t lds[8 + D * 33];
  const int b = blockIdx.y;
  Seq8 sq;
  if (!step_rows(s, b, sq)) return;
  const int done = (int)(((unsigned)sq.len + (unsigned)sq.n) / kBlock) - sq.len / kBlock;   // blocks that the step completes
  const int H = s.n_kv_heads;
  const int r0 = sq.len % kBlock;

  const int block_groups = 2 * H * blocks;
  if ((int)blockIdx.x >= block_groups) {
    const int units = s.n_q_heads + 2 * H, groups = (units + heads - 1) / heads;
    const uint32_t task = (blockIdx.x - block_groups) * kThreads + threadIdx.x;   // (fewer than 2^32: bd_paged8_append)
    const int p = task % kPairs;
    const int g = (int)(task / kPairs % groups), i = (int)(task / kPairs / groups);
    if (i >= sq.n) return;
    const int row = sq.row + i;
    const PairVec at(rot, p);
    Angles w;
    if (at.turns) w.load(rot, position_of(rot, s, row, sq.len + i), p);
    for (int u = g; u < units; u += groups) {
      const bool is_q = u < s.n_q_heads, is_v = u >= s.n_q_heads + H;
      const int h = is_q ? u : is_v ? u - s.n_q_heads - H : u - s.n_q_heads;
      if (is_q ? !q.data : done > 0) continue;
      const Rows8& from = is_q ? q : is_v ? v : k;
      const uint16_t* src = from.data + row * from.token + h * from.head;
      us8_t x = load8(src + 8 * at.a), y = load8(src + 8 * at.b);
      if (at.turns && !is_v) turn_pair<ELEM>(x, y, w, rot.interleaved);
      uint16_t* dst = is_q ? q_out.data + row * q_out.token + h * q_out.head
                           : (is_v ? s.v_res : s.k_res) + (((size_t)b * H + h) * kBlock + r0 + i) * D;
      store8(dst + 8 * at.a, x);
      store8(dst + 8 * at.b, y);
    }
    return;
  }

  const int block = (int)blockIdx.x % blocks, unit = (int)blockIdx.x / blocks;   // unit: K heads, then V heads
  if (block >= done) return;
  const bool is_v = unit >= H;
  const int h = is_v ? unit - H : unit;
  const int page = page_of(s, b, sq.len / kBlock + block);
  uint16_t* res = (is_v ? s.v_res : s.k_res) + ((size_t)b * H + h) * kBlock * D;
  const Rows8& from = is_v ? v : k;
  const uint16_t* src = from.data + h * from.head;
  if (page < 0 && s.status && threadIdx.x == 0) atomicOr(s.status, kStatusWrite);
  const int t0 = block * kBlock - r0;   // index in the step of the block's first token, negative: in the residual

  if (!is_v) {
    // keys: [token][channel], a thread's pair vectors; values at hand until the block's largest is known
    constexpr int kTasks = kBlock * kPairs / kThreads;
    us8_t x[kTasks], y[kTasks];
    uint32_t most = 0;
#pragma unroll
    for (int n = 0; n < kTasks; ++n) {
      const int task = n * kThreads + threadIdx.x, p = task % kPairs, i = t0 + task / kPairs;
      const PairVec at(rot, p);
      const uint16_t* row = i < 0 ? res + (size_t)(task / kPairs) * D : src + (sq.row + i) * from.token;
      x[n] = load8(row + 8 * at.a);
      y[n] = load8(row + 8 * at.b);
      if (i >= 0 && at.turns) {
        Angles w;
        w.load(rot, position_of(rot, s, sq.row + i, sq.len + i), p);
        turn_pair<ELEM>(x[n], y[n], w, rot.interleaved);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, max((uint32_t)x[n][e] & 0x7fffu, (uint32_t)y[n][e] & 0x7fffu));
    }
    const float scale = to_f32<ELEM>((uint16_t)group_max<kThreads / 64>(most, lds)) / kMost;
    const Divisor by(scale);
    if (page >= 0) {
      uint8_t* out = s.k_codes + ((size_t)page * H + h) * kBlock * D;
      if (threadIdx.x == 0) s.k_scales[(size_t)page * H + h] = scale;
#pragma unroll
      for (int n = 0; n < kTasks; ++n) {
        const int task = n * kThreads + threadIdx.x;
        const PairVec at(rot, task % kPairs);
        float f[16];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f[e] = to_f32<ELEM>(x[n][e]);
          f[8 + e] = to_f32<ELEM>(y[n][e]);
        }
        uint8_t* row = out + (size_t)(task / kPairs) * D;
        *(u2_t*)(row + 8 * at.a) = u2_t{code4<CODE>(f, by), code4<CODE>(f + 4, by)};
        *(u2_t*)(row + 8 * at.b) = u2_t{code4<CODE>(f + 8, by), code4<CODE>(f + 12, by)};
      }
    }
  } else {
    // values: to [channel][token] through LDS, a word of four tokens' codes at a time
    constexpr int kVecs = D / 8, kTasks = kBlock / 4 * kVecs / kThreads;
    us8_t x[kTasks][4];
    uint32_t most = 0;
#pragma unroll
    for (int n = 0; n < kTasks; ++n) {
      const int task = n * kThreads + threadIdx.x, c = task % kVecs;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = task / kVecs * 4 + j, i = t0 + t;
        x[n][j] = load8((i < 0 ? res + (size_t)t * D : src + (sq.row + i) * from.token) + 8 * c);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max(most, (uint32_t)x[n][j][e] & 0x7fffu);
      }
    }
    const float scale = to_f32<ELEM>((uint16_t)group_max<kThreads / 64>(most, lds)) / kMost;
    const Divisor by(scale);
    if (page >= 0) {
      uint8_t* out = s.v_codes + ((size_t)page * H + h) * kBlock * D;
      if (threadIdx.x == 0) s.v_scales[(size_t)page * H + h] = scale;
#pragma unroll
      for (int n = 0; n < kTasks; ++n) {
        const int task = n * kThreads + threadIdx.x, c = task % kVecs;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float f[4] = {to_f32<ELEM>(x[n][0][e]), to_f32<ELEM>(x[n][1][e]), to_f32<ELEM>(x[n][2][e]), to_f32<ELEM>(x[n][3][e])};
          lds[8 + (8 * c + e) * 33 + task / kVecs] = code4<CODE>(f, by);
        }
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < D * 8 / kThreads; ++n) {
        const int task = n * kThreads + threadIdx.x;
        const uint32_t* w = lds + 8 + (task / 8) * 33 + (task % 8) * 4;
        *(u4_t*)(out + 16 * (size_t)task) = u4_t{w[0], w[1], w[2], w[3]};
      }
    }
  }
  if (block > 0) return;

  // (every thread's loads from the residual were used before the barrier in group_max)
  const int left = (int)(((unsigned)sq.len + (unsigned)sq.n) % kBlock);
  for (int task = threadIdx.x; task < left * kPairs; task += kThreads) {
    const int p = task % kPairs, t = task / kPairs, i = sq.n - left + t;
    const PairVec at(rot, p);
    const uint16_t* row = src + (sq.row + i) * from.token;
    us8_t x = load8(row + 8 * at.a), y = load8(row + 8 * at.b);
    if (!is_v && at.turns) {
      Angles w;
      w.load(rot, position_of(rot, s, sq.row + i, sq.len + i), p);
      turn_pair<ELEM>(x, y, w, rot.interleaved);
    }
    store8(res + (size_t)t * D + 8 * at.a, x);
    store8(res + (size_t)t * D + 8 * at.b, y);
  }
}

__global__ __launch_bounds__(256) void kv8_advance_kernel(Step8 s) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= s.batch) return;
  Seq8 q;
  if (step_rows(s, b, q, true)) s.seq_lens[b] = q.len + q.n;
}

}  // namespace

hipError_t launch_kv8_append(const Step8& s, int head_dim, int code, int elem, const Rows8& k, const Rows8& v, const Rows8& q,
                             const Rows8& q_out, const Rotate8& rot, hipStream_t st) {
  const int units = s.n_q_heads + 2 * s.n_kv_heads, pairs = head_dim / 16;
  // Eight heads to a thread share a token's cosines and sines where there are threads enough (16384 tokens, 2 / 4 / 8 heads 101 / 90 / 88
  // us, 9 prompts of up to 1333 56 / 50 / 50); a few tokens' heads are a thread's each.
  const int heads = (long)s.total * units * pairs > 256 * 2048 ? 8 : 1;
  const int groups = (units + heads - 1) / heads;
  const int threads = 4 * head_dim;
  const long row_groups = ((long)s.max_tokens * groups * pairs + threads - 1) / threads;
  const int blocks = (int)(((long)s.max_tokens + kBlock - 1) / kBlock);   // the most that a step of so many tokens completes
  const dim3 grid((unsigned)(row_groups + 2L * s.n_kv_heads * blocks), s.batch);
#define BD_RUN(D, C, E) \
  hipLaunchKernelGGL((kv8_append_kernel<D, C, E>), grid, dim3(threads), 0, st, BD_KV8_HOT_ARGS(s), heads, blocks, s, k, v, q, q_out, rot)
#define BD_RUN_TYPES(D)                                          \
  if (code == BD_CODE_INT8) {                                    \
    if (elem == BD_ELEM_F16) BD_RUN(D, BD_CODE_INT8, BD_ELEM_F16); \
    else BD_RUN(D, BD_CODE_INT8, BD_ELEM_BF16);                  \
  } else {                                                       \
    if (elem == BD_ELEM_F16) BD_RUN(D, BD_CODE_E4M3, BD_ELEM_F16); \
    else BD_RUN(D, BD_CODE_E4M3, BD_ELEM_BF16);                  \
  }
  if (head_dim == 64) {
    BD_RUN_TYPES(64)
  } else {
    BD_RUN_TYPES(128)
  }
#undef BD_RUN_TYPES
#undef BD_RUN
  return hipGetLastError();
}

hipError_t launch_kv8_advance(const Step8& s, hipStream_t st) {
  hipLaunchKernelGGL(kv8_advance_kernel, dim3((s.batch + 255) / 256), dim3(256), 0, st, s);
  return hipGetLastError();
}

}  // namespace bd
