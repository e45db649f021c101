// Device code of both key/value caches' kernels (cache.hip, cache4.hip): which
// sequence a work item belongs to, and the merge of partial results of an
// attention whose sequences are split.  C is a batch (CacheBatch or
// Cache4Batch), Args an attention's arguments.
#pragma once

#include "cache.h"
#include "device.h"

namespace w4a8 {

namespace {

// ---- the batch

struct Sequence {
  int b;     // -1: none
  int row0;  // first row of its new tokens
  int n;     // new tokens
  int len;   // tokens held, the new ones the last of them
  int item;  // the item's number within the sequence
};

// Rows and length of sequence b; whatever the arrays hold, the rows lie in
// [0, T) and the length within the table.
template <class C>
__device__ __forceinline__ void sequence(const C& c, int b, int& row0, int& n, int& len) {
  row0 = min(max(c.starts[b], 0), c.T);
  n = min(max(c.starts[b + 1], row0), c.T) - row0;
  len = min(max(c.lengths[b], 0), c.max_blocks * kCacheBlock);
}

// Inclusive sum over the wave's lanes, by lane moves in the vector unit: within
// rows of 16, then each row's total into the rows after it.
__device__ __forceinline__ int wave_scan(int v) {
  constexpr int kRowShr = 0x110, kRowBcast15 = 0x142, kRowBcast31 = 0x143;
  auto step = [&](auto ctrl, auto rows) {  // lanes without a source add 0
    v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
  };
  using std::integral_constant;
  step(integral_constant<int, kRowShr + 1>{}, integral_constant<int, 0xF>{});
  step(integral_constant<int, kRowShr + 2>{}, integral_constant<int, 0xF>{});
  step(integral_constant<int, kRowShr + 4>{}, integral_constant<int, 0xF>{});
  step(integral_constant<int, kRowShr + 8>{}, integral_constant<int, 0xF>{});
  step(integral_constant<int, kRowBcast15>{}, integral_constant<int, 0xA>{});
  step(integral_constant<int, kRowBcast31>{}, integral_constant<int, 0xC>{});
  return v;
}

// The sequence that work item `item` belongs to, when sequence b has
// count(n, len) items and they are numbered through the batch.  Every wave
// finds it by itself, 64 sequences at a time.
template <class C, class F>
__device__ __forceinline__ Sequence find_sequence(const C& c, int item, F count) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int b0 = 0; b0 < c.B; b0 += 64) {
    const int b = b0 + lane;
    int row0 = 0, n = 0, len = 0, cnt = 0;
    if (b < c.B) {
      sequence(c, b, row0, n, len);
      cnt = count(n, len);
    }
    const int upto = wave_scan(cnt);
    const uint64_t past = __ballot(base + upto > item);
    if (past) {
      const int l = __builtin_ctzll(past);
      Sequence s;
      s.b = b0 + l;
      s.row0 = __builtin_amdgcn_readlane(row0, l);
      s.n = __builtin_amdgcn_readlane(n, l);
      s.len = __builtin_amdgcn_readlane(len, l);
      s.item = item - base - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(cnt, l));
      return s;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
  return Sequence{-1, 0, 0, 0, 0};
}

// ---- partial results

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The total of a row's weights is held times 2^-15 (where the smallest scales of
// the 8-bit cache's values need it).
constexpr float kTotalUnit = 0x1p-15f;
constexpr float kFar = 100.0f;

// Two weights to fp16, round to nearest even.
__device__ __forceinline__ uint32_t f16x2_bits(float lo, float hi) {
  const float2_t v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// Eight elements of a row's output from its sums and total.  A row that sees
// nothing is 0 (0 * 0), NaN stays.
__device__ __forceinline__ uint4 output8(const float (&o)[8], float total) {
  const float inv = total > 0.0f ? 1.0f / total : total;
  auto two = [&](int e) { return bf16x2_bits(o[e] * kTotalUnit * inv, o[e + 1] * kTotalUnit * inv); };
  return make_uint4(two(0), two(2), two(4), two(6));
}

// A total moved by the factor 2^d, d <= 0: by one product, or, where that would
// vanish while the total (which may be as large as 2^127) does not, by two.
__device__ __forceinline__ float rescaled(float total, float d) {
  const float half = __builtin_amdgcn_exp2f(0.5f * d);
  return d < -kFar ? total * half * half : total * __builtin_amdgcn_exp2f(d);
}

// The larger (sum) of the values of lanes l, l ^ 16, l ^ 32 and l ^ 48.
template <class F>
__device__ __forceinline__ float fold_groups(float x, F op) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

// Merge of the splits' partial results, [S][T][H]: P threads for 8 d of a
// (token, head), each folding every P-th split, their results meeting by lane
// moves and, from four waves, in LDS.  (One thread for all of 64 splits took
// 36 us of the 79 that one token over 100000 took: its reads wait for each
// other.)  Tokens of no sequence are left as they are.
template <int P, class Args>
__global__ __launch_bounds__(256) void cache_attention_merge(const Args a) {
  constexpr int kD = kCacheD, kChunks = kD / 8, kRowsHere = 256 / (kChunks * P);
  static_assert(P == 4 || P == 16, "parts of a row are the four 16-lane groups of one or four waves");
  struct Partial {
    float mx, sum, o[8];
  };
  constexpr int kWords = sizeof(Partial) / 4;
  struct Words {
    uint32_t w[kWords];
  };
  __shared__ uint32_t l_part[P == 16 ? 4 : 1][kWords][kChunks];
  const int tid = threadIdx.x, c = tid % kChunks, part = tid / kChunks % P;
  const int64_t row = (int64_t)blockIdx.x * kRowsHere + tid / (kChunks * P), rows = (int64_t)a.c.T * a.H;
  const int64_t tok = row / a.H;
  const int first = a.c.starts[0], end = a.c.starts[a.c.B];
  auto fold = [](const Partial& x, const Partial& y) {
    Partial r;
    r.mx = fmaxf(x.mx, y.mx);
    const float base = r.mx == -INFINITY ? 0.0f : r.mx;
    const float f0 = __builtin_amdgcn_exp2f(x.mx - base), f1 = __builtin_amdgcn_exp2f(y.mx - base);
    r.sum = rescaled(x.sum, x.mx - base) + rescaled(y.sum, y.mx - base);
#pragma unroll
    for (int e = 0; e < 8; ++e) r.o[e] = x.o[e] * f0 + y.o[e] * f1;
    return r;
  };
  Partial mine{-INFINITY, 0.0f, {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
  if (row < rows)
    for (int s = part; s < a.S; s += P) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (s * rows + row) * 2);
      const float4* p = reinterpret_cast<const float4*>(a.part_o + (s * rows + row) * kD + 8 * c);
      const float4 u = p[0], v = p[1];
      mine = fold(mine, Partial{ml.x, ml.y, {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w}});
    }
#pragma unroll
  for (int half = 0; half < 2; ++half) {  // lane groups 16, then 32 apart: a swap yields both values
    const Words w = __builtin_bit_cast(Words, mine);
    Words x, y;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const auto r = half == 0 ? __builtin_amdgcn_permlane16_swap(w.w[i], w.w[i], false, false)
                               : __builtin_amdgcn_permlane32_swap(w.w[i], w.w[i], false, false);
      x.w[i] = r[0];
      y.w[i] = r[1];
    }
    mine = fold(__builtin_bit_cast(Partial, x), __builtin_bit_cast(Partial, y));
  }
  if constexpr (P == 16) {
    if ((tid & 63) < kChunks) {
      const Words w = __builtin_bit_cast(Words, mine);
#pragma unroll
      for (int i = 0; i < kWords; ++i) l_part[tid >> 6][i][c] = w.w[i];
    }
    lds_barrier();
    if (tid >= kChunks) return;
#pragma unroll
    for (int q = 1; q < 4; ++q) {
      Words w;
#pragma unroll
      for (int i = 0; i < kWords; ++i) w.w[i] = l_part[q][i][c];
      mine = fold(mine, __builtin_bit_cast(Partial, w));
    }
  } else if (part != 0) {
    return;
  }
  if (row >= rows || tok < first || tok >= end) return;
  *reinterpret_cast<uint4*>(a.o.p + tok * a.o.row + (row % a.H) * a.o.head + 8 * c) = output8(mine.o, mine.sum);
}

}  // namespace

}  // namespace w4a8
