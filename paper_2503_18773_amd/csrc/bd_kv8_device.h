// Device helpers of attention over the paged 8-bit cache (gfx950, wave64).
#pragma once

#include "bd_device.h"
#include "bd_kv8.h"

namespace bd {
namespace {

typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
typedef float f16x_t __attribute__((ext_vector_type(16)));
typedef uint16_t us8_t __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f;
// A row's weights are held as 2^kShift times what they are relative to the largest one's: the matrix unit takes them in fp16, whose
// subnormals then begin 2^-22 below the largest.
constexpr float kShift = 8.f;

// Four codes as fp16, exactly.  Integers: the byte, moved to 0 .. 255, is put below 0x64 as an fp16 number's mantissa (1024 + byte),
// and 1024 + 128 taken off.
template <int CODE>
__device__ __forceinline__ void codes4(uint32_t w, h2_t& lo, h2_t& hi) {
  if (CODE == BD_CODE_INT8) {
    const uint32_t u = w ^ 0x80808080u;
    const h2_t off = {(_Float16)-1152.f, (_Float16)-1152.f};
    lo = __builtin_bit_cast(h2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off;
    hi = __builtin_bit_cast(h2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off;
  } else {
    lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
  }
}
template <int CODE>
__device__ __forceinline__ h8_t codes8(uint32_t w0, uint32_t w1) {
  h2_t a, b, c, d;
  codes4<CODE>(w0, a, b);
  codes4<CODE>(w1, c, d);
  return h8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight channels of a query as fp16.  bf16 queries are brought to below 2^7 by a power of two, the row's own (`shift`, from the row's
// largest magnitude): exact but for what is 2^-22 and less of the largest.
__device__ __forceinline__ uint32_t most_of(us8_t x) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, (uint32_t)x[e] & 0x7fffu);
  return m;
}
__device__ __forceinline__ int bf16_shift(uint32_t most) { return 133 - (int)(most >> 7); }
template <int ELEM>
__device__ __forceinline__ h8_t query8(us8_t x, int shift) {
  if (ELEM == BD_ELEM_F16) return __builtin_bit_cast(h8_t, x);
  h8_t r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (_Float16)ldexpf(__uint_as_float((uint32_t)x[e] << 16), shift);
  return r;
}

// step_rows for launches that write neither lengths nor lists, through the scalar cache
struct ScalarLoad {
  __device__ __forceinline__ int32_t operator()(const int32_t* p) const { return scalar_load(p); }
};
__device__ __forceinline__ bool queries_of(const Step8& s, int b, Seq8& q) { return step_rows(s, b, q, false, ScalarLoad()); }

// What a query row sees, and what is done to its scores, by how far a token is before it (behind it: negative).  No token behind the
// sequence's end is seen: rows and prefix end with it.
struct RowView {
  int pos;           // index in the sequence
  int prefix;        // of the sequence, at most its length
  uint32_t window;   // 2^31: none
  float slope;
};
__device__ __forceinline__ uint32_t window_of(int window) { return window ? (uint32_t)window : 0x80000000u; }

// The blocks of a sequence that queries at positions lo .. hi can see: [0, pre) and [first, ...), `count` in all that the table has room
// for; whether it lacks some; and whether they can see the residual behind the whole blocks.
struct Blocks {
  int pre, first, count;
  bool lacks, tail;
  __device__ __forceinline__ Blocks(int lo, int hi, int length, int prefix, int window, int max_pages) {
    const int full = length / kBlock;
    pre = min((int)(((unsigned)prefix + kBlock - 1) / kBlock), full);
    first = max(pre, window && lo >= window ? (lo - window + 1) / kBlock : 0);
    const int end = min(hi / kBlock + 1, full);
    lacks = max(pre, end) > max_pages;
    pre = min(pre, max_pages);
    first = min(first, max_pages);
    count = pre + max(0, min(end, max_pages) - first);
    tail = length > full * kBlock && (hi >= full * kBlock || prefix > full * kBlock);
  }
  __device__ __forceinline__ int operator[](int i) const { return i < pre ? i : first + i - pre; }
};
// whether all of tokens from .. from + 127 are seen from everywhere in lo .. hi
__device__ __forceinline__ bool all_seen(int from, int lo, int hi, int prefix, int window) {
  return from + kBlock <= prefix || (from + kBlock - 1 <= lo && (window == 0 || hi - from < window));
}

// A score in units of log2 e is x * by + plus, of what finish_scores leaves in x: its multiplication is one with what the exponential's
// argument needs anyway, and the largest x is the largest score (by > 0).
struct Linear {
  float by, plus;
};

// N x 4 (or 16) products of a row to scores, -infinity for tokens that the row does not see.  c >= 0: what a product is worth, in natural
// units; from + offset(t, i): the token.  Every pass is decided on once for all of them.
// The cap: cap tanh(y) = cap + 2 cap r with r = -1 / (1 + e^2y), r within 2^-23 absolutely: the score within 2^-22 cap, which for caps of up to 1024
// (bd_paged8_attn takes no larger ones) is less than what rounding a weight to 11 bits is.
template <class X, int N, class Offset>
__device__ __forceinline__ Linear finish_scores(X* x, float c, const Scores8& sc, const RowView& view, bool masked, int from, Offset offset) {
  constexpr int K = sizeof(X) / 4;
  Linear f{fmaxf(c * kLog2e, 1e-30f), 0.f};   // (0 times -infinity is no score)
  if (sc.cap > 0.f) {
    const float twice = fminf(2.f * kLog2e * c / sc.cap, 1e30f);   // (nor is 0 times infinity)
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < K; ++i) x[t][i] = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(x[t][i] * twice));
    f = Linear{2.f * kLog2e * sc.cap, kLog2e * sc.cap};
  }
  // (how far the tokens are before the row, in each pass for itself: for both the compiler would keep them all in registers)
  int before = view.pos - from;
  if (sc.slopes) {
    const float distance = (float)before, slope = view.slope * kLog2e;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < K; ++i) x[t][i] = fmaf(-slope, fabsf(distance - (float)offset(t, i)), fmaf(x[t][i], f.by, f.plus));
    f = Linear{1.f, 0.f};
  }
  asm volatile("" : "+v"(before));
  if (masked) {
    const int prefix = view.pos - view.prefix;   // (how far a row is behind the prefix's end)
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int y = before - offset(t, i);
        x[t][i] = ((y <= prefix) & ((uint32_t)y >= view.window)) ? -INFINITY : x[t][i];
      }
  }
  return f;
}
template <class X, int N>
__device__ __forceinline__ void no_scores(X* x) {
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int i = 0; i < (int)(sizeof(X) / 4); ++i) x[t][i] = -INFINITY;
}

// A page's number, -1 where the table has none, through the scalar cache: nothing of the launch writes the table, and a load that the
// wave's vector loads need not be waited for with.
__device__ __forceinline__ int page_in(const Step8& s, const int32_t* table, const Blocks& bl, int i) {
  const int page = i < bl.count ? scalar_load(table + bl[i]) : -1;
  return page < s.num_pages ? page : -1;   // (negative as it is)
}
__device__ __forceinline__ float scalar_scale(const float* p) { return __int_as_float(scalar_load((const int32_t*)p)); }

// Logarithm (base 2) of the scale that the row sums are kept in units of: that of the first of the visible blocks (of up to 64)
// with a scale.  A weight enters the product with V's codes times its block's scale, as an addend of its exponent, and the row sum
// times 2^(reference - own): blocks whose values differ in size cost nothing, and a block of zeros counts as any other.
__device__ __forceinline__ float scale_reference(const Step8& s, const int32_t* table, const Blocks& bl, int h) {
  for (int i = 0; i < min(bl.count, 64); ++i) {
    const int page = page_in(s, table, bl, i);
    const float v = page >= 0 ? scalar_scale(s.v_scales + (size_t)page * s.n_kv_heads + h) : 0.f;
    if (v > 0.f) return log2f(v);
  }
  return 0.f;
}

template <int ELEM>
__device__ __forceinline__ uint32_t elem2(float a, float b) {
  if (ELEM == BD_ELEM_BF16) return __builtin_bit_cast(uint32_t, bf2_t{(__bf16)a, (__bf16)b});
  return __builtin_bit_cast(uint32_t, h2_t{(_Float16)a, (_Float16)b});
}

}  // namespace
}  // namespace bd
