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

// What a query row sees, and what is done to its scores.
struct RowView {
  int pos;      // index in the sequence
  int prefix;   // of the sequence, at most its length
  int window;   // 0: none
  float slope;
  __device__ __forceinline__ bool sees(int j) const { return j < prefix || (j <= pos && (window == 0 || pos - j < window)); }
};
// natural units
__device__ __forceinline__ float capped(float x, float cap, float inv_cap) {
  // tanh(y) = 1 - 2 / (1 + e^2y): within 2^-23 of it absolutely, which is what a score needs
  const float e = __builtin_amdgcn_exp2f(x * inv_cap * (2.f * kLog2e));
  return cap - 2.f * cap * __builtin_amdgcn_rcpf(1.f + e);
}

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

// Logarithm (base 2) of the scale that the row sums are kept in units of: that of the first of the visible blocks (of up to 64)
// with a scale.  A weight enters the product with V's codes times its block's scale, as an addend of its exponent, and the row sum
// times 2^(reference - own): blocks whose values differ in size cost nothing, and a block of zeros counts as any other.
__device__ __forceinline__ float scale_reference(const Step8& s, const Blocks& bl, int b, int h, int lane) {
  float v = 0.f;
  if (lane < bl.count) {
    const int page = page_of(s, b, bl[lane]);
    if (page >= 0) v = s.v_scales[(size_t)page * s.n_kv_heads + h];
  }
  const uint64_t some = __ballot(v > 0.f);
  if (some == 0) return 0.f;
  return log2f(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), __builtin_ctzll(some))));
}

template <int ELEM>
__device__ __forceinline__ uint32_t elem2(float a, float b) {
  if (ELEM == BD_ELEM_BF16) return __builtin_bit_cast(uint32_t, bf2_t{(__bf16)a, (__bf16)b});
  return __builtin_bit_cast(uint32_t, h2_t{(_Float16)a, (_Float16)b});
}

}  // namespace
}  // namespace bd
