// Attention over the paged 8-bit cache of few query rows: decoding, and a few tokens a sequence at once.
#include "bd_kv8_device.h"
#include "bd_kv8_part.h"

namespace bd {
namespace {

// Sixteen rows (a token's query head each, token by token), or twice that, of one KV head against blocks of 128 tokens, a wave a block.
// Per block  S^T = K Q^T  and  O^T += V^T P^T  with 16 x 16 x 32 products, tokens x rows and channels x rows: a lane holds
// scores and outputs of one row of each sixteen, and its scores are, as they come, the eight tokens that the second product wants of the lane.
// The order of tokens inside of the products is free, and chosen so that a lane's codes are 16 adjacent bytes: S^T's row 4 a + i of
// tile t is token 64 (t / 4) + 16 a + 4 (t % 4) + i, so lane group g has tokens 16 g .. 16 g + 15 of each half; likewise the channels of K.
template <int D, int CODE, int ELEM>
struct Few {
  static constexpr int kChunks = D / 64, kSteps = D / 32, kTiles = D / 16;
  h8_t q[kSteps];
  float c;       // scores in natural units per product and K scale
  RowView view;
  float m, l;    // running maximum (base 2, scale included) and sum of the lane's row
  f4_t acc[kTiles];

  // weights in place of N tiles' scores; lv: the block's V scale, ref: the reference scale, both as logarithms
  template <int N>
  __device__ __forceinline__ void weights(f4_t* s, Linear s_of, float lv, float ref) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
    top = fmaf(join_groups(top, Max()), s_of.by, s_of.plus + lv);
    const float now = fmaxf(m, top), base = now == -INFINITY ? 0.f : now;
    const float was = __builtin_amdgcn_exp2f(m - base), off = s_of.plus + lv - base + kShift;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], s_of.by, off));
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

// Two floats past the L2 cache, to and from other XCDs' workgroups.
__device__ __forceinline__ void put2(float* p, float a, float b) {
  __hip_atomic_store((unsigned long long*)p, (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void get2(const float* p, float& a, float& b) {
  const unsigned long long x = __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  a = __uint_as_float((uint32_t)x);
  b = __uint_as_float((uint32_t)(x >> 32));
}

// The weight of a partial result, given the largest maximum.
__device__ __forceinline__ float merge_weight(float m, float top) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top); }

// A ragged batch's workgroups, dealt by length: of the `room` that there are for a head's tile, a sequence gets one for so many blocks each
// (six at least, and no more than twice `splits` in all) that all of them find room.  This workgroup's sequence, its number among that one's, how many those are, and the first one's
// number; false: it is left over.  (Lengths as they are before the step, whatever lists and prefixes make of them.)  Against as many splits for
// each: 4 sequences of 20000 down to 6700 tokens 31.8 -> 28.6 us, 3 of up to 60000 60.5 -> 52.0, 24 of up to 5000 and 4 KV heads 27.0 -> 22.8; it
// takes a microsecond, which short ones do not make up for (16 of up to 4000, five queries each, 34.3 / 35.8, 2 of 700 9.6 / 10.6): the
// table's width is what the host knows of the lengths.
struct Share {
  int b, split, splits, first;
};
__device__ __forceinline__ bool fair_share(const Step8& s, int lane, int room, int most, int window, Share& share) {
  int blocks = lane < s.batch ? max(s.seq_lens[lane], 0) / kBlock + 1 : 0;
  if (window) blocks = min(blocks, window / kBlock + 2);
  const float mine = (float)blocks;
  float each = ceilf(fmaxf(join_groups(row_sum16(mine), Add()) / (float)max(1, room - s.batch / 2), 6.f)), wanted;
  for (int i = 0;; ++i) {
    wanted = fminf(ceilf(mine / each), (float)most);
    const float need = join_groups(row_sum16(wanted), Add());
    if (need <= (float)room) break;
    if (i == 8) {   // (not seen; one for each has room: launch_kv8_few)
      wanted = lane < s.batch ? 1.f : 0.f;
      break;
    }
    each = ceilf(each * fmaxf(need / (float)room, 1.02f));
  }
  int to = (int)wanted;   // running sum over the lanes
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int other = __shfl_up(to, d);
    to += lane >= d ? other : 0;
  }
  const uint64_t found = __ballot((int)blockIdx.x < to);
  if (!found) return false;
  const int at = __builtin_ctzll(found);
  share.b = at;
  share.splits = __builtin_amdgcn_readlane((int)wanted, at);
  share.first = __builtin_amdgcn_readlane(to, at) - share.splits;
  share.split = (int)blockIdx.x - share.first;
  return true;
}

template <int D, int CODE, int ELEM, int NT>
__global__ __launch_bounds__(256, 1) void kv8_few_kernel(BD_KV8_HOT_PARAMS, int splits, int order, int room, Step8 s, Rows8 q, Scores8 sc, Parts8 parts, uint16_t* out) {
  BD_KV8_HOT(s);
  typedef Few<D, CODE, ELEM> F;
  constexpr int kPitch = D + 4, kTileRows = 16 * NT;
  __shared__ float lds[4 * kTileRows * kPitch + 4 * kTileRows * 2];
  const int h = blockIdx.y % s.n_kv_heads, tile = blockIdx.y / s.n_kv_heads;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, split = blockIdx.x, slot = 0;   // slot: where the sequence's partial results begin, of its head's tile
  if (room) {
    Share share;
    if (!fair_share(s, lane, room, min(2 * splits, kMostSplits), sc.window, share)) return;
    b = share.b;
    split = share.split;
    splits = share.splits;
    slot = share.first;
  } else {
    int before;
    b = __builtin_amdgcn_readfirstlane(paged_sequence<false>(s.seq_lens, lane, before, order, 0, 0));
  }
  // (requested with the length, for where the wave's first block turns out to be the one of that number)
  const int32_t* table = s.block_table + (size_t)b * s.max_pages;
  const int guessed = split + splits * wave;
  const int guess = guessed < s.max_pages ? scalar_load(table + guessed) : -1;
  Seq8 sq;
  if (!queries_of(s, b, sq)) return;
  const int rows = sq.n * s.gq;
  if (kTileRows * tile >= rows) return;
  const int here = min(kTileRows, rows - kTileRows * tile);   // of the tile
  const int length = sq.len + sq.n, lo = sq.len + kTileRows * tile / s.gq, hi = sq.len + min(kTileRows * tile + kTileRows - 1, rows - 1) / s.gq;
  const int prefix = sc.prefix ? min(max(scalar_load(sc.prefix + b), 0), length) : 0;
  F f[NT];
  const uint16_t* q_row[NT];
  us8_t raw[NT][F::kSteps];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = min(kTileRows * tile + 16 * n + col, rows - 1), token = row / s.gq, head = h * s.gq + row % s.gq;
    f[n].view.pos = sq.len + token;
    f[n].view.prefix = prefix;
    f[n].view.window = window_of(sc.window);
    f[n].view.slope = sc.slopes ? sc.slopes[head] : 0.f;
    q_row[n] = q.data + (sq.row + token) * q.token + head * q.head + 16 * grp;
#pragma unroll
    for (int k = 0; k < F::kSteps; ++k) raw[n][k] = *(const us8_t*)(q_row[n] + 64 * (k / 2) + 8 * (k % 2));
  }

  // Blocks are dealt to the splits in turn, and a split's to its waves: a few blocks are one to a workgroup, on compute units of their own, since
  // one of those draws some 35 GB/s whatever it asks for.  The residual goes, 32 tokens a wave, where the next block would.  No more splits
  // than that are at work.
  const Blocks blocks(lo, hi, length, prefix, sc.window, s.max_pages);
  const int active = max(1, min(splits, blocks.count + blocks.tail));
  if (split >= active) return;
  const int begin = split + active * wave;
  bool missing = blocks.lacks;
  // (a block that is not there: any page's bytes, and none of its tokens seen)
  u4_t kw[8][F::kChunks], vw[F::kTiles][2];
  float ks, vs;
  const uint32_t lane_k = (16 * (col >> 2) + (col & 3)) * D + 16 * grp, lane_v = col * kBlock + 16 * grp;
  auto request_k = [&](int page) {
    const size_t unit = (size_t)max(page, 0) * s.n_kv_heads + h;
    const uint8_t* kc = s.k_codes + unit * (kBlock * D);
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int p = 0; p < F::kChunks; ++p) kw[t][p] = *(const u4_t*)(kc + (64 * (t / 4) + 4 * (t % 4)) * D + 64 * p + lane_k);
    ks = scalar_scale(s.k_scales + unit);
  };
  auto request_v = [&](int page) {
    const size_t unit = (size_t)max(page, 0) * s.n_kv_heads + h;
    const uint8_t* vc = s.v_codes + unit * (kBlock * D);
#pragma unroll
    for (int dt = 0; dt < F::kTiles; ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u) vw[dt][u] = *(const u4_t*)(vc + 16 * dt * kBlock + 64 * u + lane_v);
    vs = scalar_scale(s.v_scales + unit);
  };
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    f[n].m = -INFINITY;
    f[n].l = 0.f;
#pragma unroll
    for (int dt = 0; dt < F::kTiles; ++dt) f[n].acc[dt] = f4_t{0.f, 0.f, 0.f, 0.f};
  }
  float ref;
  auto prepare = [&]() {   // (behind the first requests)
    ref = scale_reference(s, table, blocks, h);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      int shift = 0;
      if (ELEM == BD_ELEM_BF16) {
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < F::kSteps; ++k) most = max(most, most_of(raw[n][k]));
        shift = bf16_shift(__float_as_uint(join_groups(__uint_as_float(most), Max())));   // (bit patterns of positive numbers)
      }
#pragma unroll
      for (int k = 0; k < F::kSteps; ++k) f[n].q[k] = query8<ELEM>(sc.scale < 0.f ? raw[n][k] ^ (uint16_t)0x8000 : raw[n][k], shift);
      f[n].c = ldexpf(fabsf(sc.scale), -shift);   // (the queries have its sign)
    }
  };
  const int tail = length % kBlock, first = 32 * wave;
  const bool rest = blocks.tail && split == blocks.count % active && first < tail;
  us8_t kx[2][F::kSteps], vx[F::kTiles];
  auto request_rest = [&]() {
    const size_t unit = ((size_t)b * s.n_kv_heads + h) * (kBlock * D);
    const uint16_t* kr = s.k_res + unit + (first + 8 * (col >> 2) + (col & 3)) * D + 16 * grp;
    const uint16_t* vr = s.v_res + unit + (first + 8 * grp) * D + col;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int k = 0; k < F::kSteps; ++k) kx[t][k] = *(const us8_t*)(kr + 4 * t * D + 64 * (k / 2) + 8 * (k % 2));
#pragma unroll
    for (int dt = 0; dt < F::kTiles; ++dt)
#pragma unroll
      for (int e = 0; e < 8; ++e) vx[dt][e] = first + 8 * grp + e < tail ? vr[e * D + 16 * dt] : (uint16_t)0;   // (rows behind the last are anything)
  };
  if (begin < blocks.count) {
    int it = begin, page = blocks.pre == 0 && blocks.first == 0 && begin == guessed ? (guess < s.num_pages ? guess : -1) : page_in(s, table, blocks, begin);
    request_k(page);
    request_v(page);
    int next_page = page_in(s, table, blocks, it + 4 * active);
    prepare();
    f4_t x[NT][8];
    int from;
    float block_k, lv;
    bool gone;
    auto products = [&]() {
      from = blocks[it] * kBlock;
      gone = page < 0;
      missing |= gone;
      block_k = ks;
      lv = vs > 0.f ? log2f(vs) : ref;
#pragma unroll
      for (int t = 0; t < 8; ++t) {
#pragma unroll
        for (int n = 0; n < NT; ++n) x[n][t] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < F::kChunks; ++p) {
          const h8_t k0 = codes8<CODE>(kw[t][p][0], kw[t][p][1]), k1 = codes8<CODE>(kw[t][p][2], kw[t][p][3]);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            x[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, f[n].q[2 * p], x[n][t], 0, 0, 0);
            x[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, f[n].q[2 * p + 1], x[n][t], 0, 0, 0);
          }
        }
      }
    };
    auto outputs = [&]() {
      const bool masked = !all_seen(from, lo, hi, prefix, sc.window);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const Linear s_of = finish_scores<f4_t, 8>(x[n], f[n].c * block_k, sc, f[n].view, masked, from + 16 * grp,
                                                   [](int t, int i) { return 64 * (t / 4) + 4 * (t % 4) + i; });
        if (gone) no_scores<f4_t, 8>(x[n]);
        f[n].template weights<8>(x[n], s_of, lv, ref);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        h8_t p[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) p[n][e] = (_Float16)x[n][2 * k + e / 4][e % 4];
#pragma unroll
        for (int dt = 0; dt < F::kTiles; ++dt) {
          const h8_t v = codes8<CODE>(vw[dt][k / 2][2 * (k % 2)], vw[dt][k / 2][2 * (k % 2) + 1]);
#pragma unroll
          for (int n = 0; n < NT; ++n) f[n].acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[n], f[n].acc[dt], 0, 0, 0);
        }
      }
    };
    // The next block's keys are on their way while the scores and values are dealt with, its values behind them.  (The last block is
    // written out once more: with the requests under a condition in the loop, the compiler waits for a block's values before its first product.)
    products();
    while (it + 4 * active < blocks.count) {
      page = next_page;
      request_k(page);
      outputs();
      request_v(page);
      it += 4 * active;
      next_page = page_in(s, table, blocks, it + 4 * active);
      products();
    }
    outputs();
    if (rest) request_rest();
  } else {
    if (rest) request_rest();
    prepare();
  }
  if (missing && s.status && lane == 0) atomicOr(s.status, kStatusRead);

  if (rest) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      f4_t x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        x[t] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < F::kSteps; ++k) {
          if (ELEM == BD_ELEM_F16)
            x[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, kx[t][k]), f[n].q[k], x[t], 0, 0, 0);
          else
            x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, kx[t][k]), *(const bf8_t*)(q_row[n] + 64 * (k / 2) + 8 * (k % 2)), x[t], 0, 0, 0);
        }
        if (ELEM == BD_ELEM_BF16 && sc.scale < 0.f) x[t] = -x[t];   // (f.q has its sign)
      }
      const Linear s_of = finish_scores<f4_t, 2>(x, fabsf(sc.scale), sc, f[n].view, true, length - tail + first + 8 * grp, [](int t, int i) { return 4 * t + i; });
      f[n].template weights<2>(x, s_of, 0.f, ref);
      h8_t p;
      bf8_t p1, p2;   // bf16 values want bf16 weights: in two pieces, 16 bits of them
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = x[e / 4][e % 4];
        p[e] = (_Float16)y;
        p1[e] = (__bf16)y;
        p2[e] = (__bf16)(y - (float)p1[e]);
      }
#pragma unroll
      for (int dt = 0; dt < F::kTiles; ++dt) {
        if (ELEM == BD_ELEM_F16) {
          f[n].acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, vx[dt]), p, f[n].acc[dt], 0, 0, 0);
        } else {
          f[n].acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, vx[dt]), p1, f[n].acc[dt], 0, 0, 0);
          f[n].acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, vx[dt]), p2, f[n].acc[dt], 0, 0, 0);
        }
      }
    }
  }

  // the four waves' results, in units of 2^(m - kShift) and, the sums, of 2^ref
  float* ml = lds + 4 * kTileRows * kPitch;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 16 * n + col;
    if (r < here) {
      if (grp == 0) {
        ml[(wave * kTileRows + r) * 2] = f[n].m;
        ml[(wave * kTileRows + r) * 2 + 1] = f[n].l;
      }
#pragma unroll
      for (int dt = 0; dt < F::kTiles; ++dt) *(f4_t*)(lds + (wave * kTileRows + r) * kPitch + 16 * dt + 4 * grp) = f[n].acc[dt];
    }
  }
  __syncthreads();
  constexpr int kPer = D / 16;   // channels a thread
  const int d = threadIdx.x % 16 * kPer;
  const float unit = __builtin_amdgcn_exp2f(ref);
  const int at = b * (int)gridDim.y + blockIdx.y;   // of the counters
  const int slots = (room ? room : s.batch * splits) * (int)gridDim.y, first_slot = room ? (int)blockIdx.y * room + slot : at * splits;
  const int filed = min(kTileRows, s.max_tokens * s.gq);   // rows of a partial result
  float* po = parts.data + (size_t)first_slot * filed * D;
  float* pml = parts.data + (size_t)slots * filed * D + (size_t)first_slot * filed * 2;
  auto to_out = [&](int r, const float* o, float sum) {
    const int i = kTileRows * tile + r;
    const size_t out_row = sq.row * (size_t)s.n_q_heads + (size_t)(i / s.gq) * s.n_q_heads + h * s.gq + i % s.gq;
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int e = 0; e < kPer; e += 2) *(uint32_t*)(out + out_row * D + d + e) = elem2<ELEM>(o[e] * inv, o[e + 1] * inv);
  };
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 16 * n + threadIdx.x / 16;
    if (r >= here) continue;
    float o[kPer] = {}, sum = 0.f, top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[(w * kTileRows + r) * 2]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float fac = merge_weight(ml[(w * kTileRows + r) * 2], top);
      sum += fac * ml[(w * kTileRows + r) * 2 + 1];
#pragma unroll
      for (int e = 0; e < kPer; ++e) o[e] += fac * lds[(w * kTileRows + r) * kPitch + d + e];
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] *= unit;
    if (active == 1) {
      to_out(r, o, sum);
    } else {
#pragma unroll
      for (int e = 0; e < kPer; e += 2) put2(po + (split * filed + r) * D + d + e, o[e], o[e + 1]);
      if (d == 0) put2(pml + (split * filed + r) * 2, top, sum);
    }
  }
  if (active == 1) return;

  // The workgroup that files the last of the partial results merges them, which spares a launch.  They pass between XCDs, whose L2
  // caches do not know of each other: device-scope stores and loads, which go through those, so that no cache has to be written back or emptied
  // (as a release and an acquire at that scope would); a store is waited for before it is counted.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  uint32_t* seen = (uint32_t*)lds;
  if (threadIdx.x == 0) {
    const uint32_t n = __hip_atomic_fetch_add(parts.counters + at, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
    if (n == (uint32_t)active) __hip_atomic_store(parts.counters + at, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *seen = n;
  }
  __syncthreads();
  if (*seen != (uint32_t)active) return;
  float* fac = lds;                            // [16][kMostSplits] weights of the partial results
  float* sums = lds + 16 * kMostSplits;        // [16]
  float* slices_o = sums + 16;                 // [slice][row][D]
  for (int n = 0; n < NT && 16 * n < here; ++n) {
    __syncthreads();
    const int r = threadIdx.x / 16, left = min(16, here - 16 * n);
    const float* from_o = po + 16 * n * D;
    const float* from_ml = pml + 16 * n * 2;
    // outputs: rows x slices of the splits fill the workgroup; a thread's first ones are on their way with the maxima and sums
    const int held = left > 8 ? 16 : left > 4 ? 8 : left > 2 ? 4 : left, slices = 16 / held, mr = r % held, slice = r / held;
    constexpr int kAhead = 8;
    float ahead[kAhead][kPer];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int e = 0; e < kPer; e += 2) {
        ahead[i][e] = ahead[i][e + 1] = 0.f;
        if (slice + i * slices < active && mr < left) get2(from_o + ((slice + i * slices) * filed + mr) * D + d + e, ahead[i][e], ahead[i][e + 1]);
      }
    // a row's maxima and sums by 16 threads
    const int lane16 = threadIdx.x % 16;
    float all = -INFINITY, mm[kMostSplits / 16], ll[kMostSplits / 16];
#pragma unroll
    for (int i = 0; i < kMostSplits / 16; ++i) {
      mm[i] = -INFINITY;
      ll[i] = 0.f;
      if (16 * i + lane16 < active && r < left) get2(from_ml + ((16 * i + lane16) * filed + r) * 2, mm[i], ll[i]);
      all = fmaxf(all, mm[i]);
    }
#pragma unroll
    for (int x = 1; x < 16; x *= 2) all = fmaxf(all, __shfl_xor(all, x));
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < kMostSplits / 16; ++i) {
      const float w = merge_weight(mm[i], all);
      l += w * ll[i];
      fac[r * kMostSplits + 16 * i + lane16] = w;
    }
#pragma unroll
    for (int x = 1; x < 16; x *= 2) l += __shfl_xor(l, x);
    if (lane16 == 0) sums[r] = l;
    __syncthreads();
    float acc[kPer] = {};
    if (mr < left) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (slice + i * slices >= active) break;
        const float w = fac[mr * kMostSplits + slice + i * slices];
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] += w * ahead[i][e];
      }
#pragma unroll 8
      for (int k = slice + kAhead * slices; k < active; k += slices) {
        const float w = fac[mr * kMostSplits + k];
#pragma unroll
        for (int e = 0; e < kPer; e += 2) {
          float y0, y1;
          get2(from_o + (k * filed + mr) * D + d + e, y0, y1);
          acc[e] += w * y0;
          acc[e + 1] += w * y1;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < kPer; e += 4) *(f4_t*)(slices_o + r * kPitch + d + e) = f4_t{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
    __syncthreads();
    if (r < left) {
      float o[kPer] = {};
      for (int k = 0; k < slices; ++k)
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] += slices_o[(k * held + r) * kPitch + d + e];
      to_out(16 * n + r, o, sums[r]);
    }
  }
}

}  // namespace

hipError_t launch_kv8_few(const Step8& s, int head_dim, int code, int elem, const Rows8& q, const Scores8& sc, int splits, void* ws, void* out,
                          hipStream_t st) {
  const long rows = (long)s.max_tokens * s.gq, tiles = few_tiles(rows);
  if (s.n_kv_heads * tiles * s.batch > kCounters) splits = 1;   // (far more workgroups than the chip holds)
  splits = splits < kMostSplits ? splits : kMostSplits;
  const Parts8 parts{(uint32_t*)ws, (float*)((char*)ws + BD_PAGED8_COUNTER_BYTES)};
  // Ragged batches: where there are compute units for several splits of a sequence, those are dealt by length; where there are
  // fewer units than sequences, the longest come first.
  const long units = s.n_kv_heads * tiles;
  const bool ragged = s.batch >= 2 && s.batch <= 64;
  const int room = ragged && splits > 1 && units * s.batch <= 128 && s.max_pages >= 40 ? (int)(256 / units) : 0;
  const int order = ragged && !room && units * s.batch > 256 ? s.batch : 0;
  const dim3 grid(room ? room : splits, (unsigned)units, room ? 1 : s.batch);
#define BD_RUN_N(D, C, E, N) \
  hipLaunchKernelGGL((kv8_few_kernel<D, C, E, N>), grid, dim3(256), 0, st, BD_KV8_HOT_ARGS(s), splits, order, room, s, q, sc, parts, (uint16_t*)out)
#define BD_RUN(D, C, E)                       \
  do {                                        \
    if (rows <= 16) BD_RUN_N(D, C, E, 1);     \
    else BD_RUN_N(D, C, E, 2);                \
  } while (0)
  BD_KV8_INSTANCES(head_dim, code, elem, BD_RUN)
#undef BD_RUN
#undef BD_RUN_N
  return hipGetLastError();
}

}  // namespace bd
