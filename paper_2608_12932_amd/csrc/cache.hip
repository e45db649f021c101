// The 8-bit key/value cache: appending to it and attending over it.
//
// A sequence's cache is a list of blocks of 64 tokens, each a page of a pool
// (the table names them).  A page holds, for each kv head, the keys' and the
// values' int8 codes and one fp32 scale for either:
//     s = max |x| / 127 over the block's tokens,  code = round_half_even(x / s),
// the keys being rotated at their positions first (rounded to bf16, as a bf16
// model holds them).  A block that is not full yet is quantized anew at every
// append, always from the exact bf16 values, which a ring of the last two
// blocks keeps for every sequence: no value is rounded twice, so the codes do
// not depend on how many tokens came at a time, and a draft's rejected tokens
// can be taken back by a smaller length.
#include <algorithm>
#include <climits>

#include "cache.h"
#include "device.h"
#include "kernels.h"

namespace w4a8 {

namespace {

constexpr int kD = kCacheD, kHalf = kD / 2, kBlock = kCacheBlock, kRecent = kCacheRecent;
constexpr int kPageBytes = kBlock * kD;  // one head's codes of a page, keys or values

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
__device__ __forceinline__ void sequence(const CacheBatch& c, int b, int& row0, int& n, int& len) {
  row0 = min(max(c.starts[b], 0), c.T);
  n = min(max(c.starts[b + 1], row0), c.T) - row0;
  len = min(max(c.lengths[b], 0), c.max_blocks * kBlock);
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
template <class F>
__device__ __forceinline__ Sequence find_sequence(const CacheBatch& c, int item, F count) {
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

__device__ __forceinline__ int clamp_pos(int p, int n_pos) { return p < 0 ? 0 : (p >= n_pos ? n_pos - 1 : p); }

// ---- append

// The rotated pair of chunks (8 values each at d and d + 64): lo = a cos -
// b sin, hi = b cos + a sin, each product and sum rounded in fp32 (no
// contraction), then to bf16.
__device__ __forceinline__ void rotate_pair(uint4& a8, uint4& b8, const float* cs, const float* sn) {
#pragma clang fp contract(off)
  uint32_t aw[4] = {a8.x, a8.y, a8.z, a8.w}, bw[4] = {b8.x, b8.y, b8.z, b8.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float a0 = bf16_lo(aw[e]), a1 = bf16_hi(aw[e]), b0 = bf16_lo(bw[e]), b1 = bf16_hi(bw[e]);
    const float c0 = cs[2 * e], c1 = cs[2 * e + 1], s0 = sn[2 * e], s1 = sn[2 * e + 1];
    aw[e] = bf16x2_bits(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
    bw[e] = bf16x2_bits(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
  }
  a8 = make_uint4(aw[0], aw[1], aw[2], aw[3]);
  b8 = make_uint4(bw[0], bw[1], bw[2], bw[3]);
}

constexpr int kAppendThreads = 512;  // a block in one pass
constexpr int kTokensPerPass = kAppendThreads / 8;  // 8 threads to a token: chunks c and c + 8
constexpr int kPasses = kBlock / kTokensPerPass;
constexpr int kCodePitch = kD + 4;                  // bytes of a token's codes in LDS, off the banks' period

// One workgroup per (touched block, kv head, keys or values): the block's
// tokens from the new rows and, where older ones lie in front of them, from
// the ring; the codes and the scale; the ring's new entries.
//
// The ring keeps the last two blocks, so block w lies where block w - 2 was.
// A call that starts inside a block fb and reaches past block fb + 1 would
// have one workgroup read the old tokens of fb while another overwrites them:
// there the workgroup of fb, once it has read them, writes the ring for the
// block that takes their place.
//
// Bound by its chain of reads, each of which waits for the one before, not by
// bytes: the batch, the slot, rows and positions, the tables, and (the compiler
// puts it right before the barrier) the page.  5.3 us for 16 sequences' single
// tokens at 8 kv heads, 6.7 us for 1024 tokens (6.8 MB, 1.3 us at a copy's
// rate); with 256 threads in two passes 6.0 and 6.8.
__global__ __launch_bounds__(kAppendThreads) void cache_append(const CacheAppendArgs a) {
  __shared__ uint32_t l_max[kAppendThreads / 64];
  __shared__ uint8_t l_codes[kBlock * kCodePitch];
  const CacheBatch& cb = a.c;
  const int tid = threadIdx.x, hk = blockIdx.y;
  const bool keys = blockIdx.z == 0;
  const Sequence s = find_sequence(cb, blockIdx.x, [](int n, int len) {
    return n > 0 && len > 0 ? (len - 1) / kBlock - max(len - n, 0) / kBlock + 1 : 0;
  });
  if (s.b < 0) return;
  const int first = max(s.len - s.n, 0);  // the first new token that has a place
  const int fb = first / kBlock, last = (s.len - 1) / kBlock, blk = fb + s.item;
  const int slot = a.slots ? a.slots[s.b] : s.b;
  const int page = cb.table[(int64_t)s.b * cb.max_blocks + blk];
  const bool slot_ok = slot >= 0 && slot < a.n_slots;
  const TokenRows rows = keys ? a.k : a.v;
  uint16_t* ring = (keys ? a.k_recent : a.v_recent) + ((int64_t)(slot_ok ? slot : 0) * cb.Hkv + hk) * (kRecent * kD);
  const int c = tid & 7;

  // Chunks c and c + 8 of token t: rotated if it is a new key.  A lane without
  // a token loads the call's last one.
  auto load = [&](int t, uint4& lo, uint4& hi) {
    const bool held = t < first, there = t < s.len && (!held || slot_ok);
    const int row = s.row0 + (there && !held ? t - (s.len - s.n) : s.n - 1);
    const uint16_t* src = there && held ? ring + (t & (kRecent - 1)) * kD : rows.p + row * rows.row + hk * rows.head;
    lo = *reinterpret_cast<const uint4*>(src + 8 * c);
    hi = *reinterpret_cast<const uint4*>(src + kHalf + 8 * c);
    if (keys) {
      const int64_t at = (int64_t)clamp_pos(cb.pos[row], cb.n_pos) * kHalf + 8 * c;
      float cs[8], sn[8];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        *reinterpret_cast<float4*>(cs + 4 * e) = *reinterpret_cast<const float4*>(cb.rope_cos + at + 4 * e);
        *reinterpret_cast<float4*>(sn + 4 * e) = *reinterpret_cast<const float4*>(cb.rope_sin + at + 4 * e);
      }
      if (!held) rotate_pair(lo, hi, cs, sn);
    }
    if (!there) lo = hi = make_uint4(0u, 0u, 0u, 0u);
  };
  auto keep = [&](int t, const uint4& lo, const uint4& hi) {
    uint16_t* dst = ring + (t & (kRecent - 1)) * kD;
    *reinterpret_cast<uint4*>(dst + 8 * c) = lo;
    *reinterpret_cast<uint4*>(dst + kHalf + 8 * c) = hi;
  };

  uint4 lo[kPasses], hi[kPasses];
  uint32_t m = 0;
#pragma unroll
  for (int u = 0; u < kPasses; ++u) load(blk * kBlock + u * kTokensPerPass + (tid >> 3), lo[u], hi[u]);
#pragma unroll
  for (int u = 0; u < kPasses; ++u) m = absmax_chunk(absmax_chunk(m, lo[u]), hi[u]);
  m = wave_max_u32(fold_pair_max(m));
  if ((tid & 63) == 0) l_max[tid >> 6] = m;
  lds_barrier();  // and every old token has been read
  m = l_max[0];
#pragma unroll
  for (int w = 1; w < kAppendThreads / 64; ++w) m = max(m, l_max[w]);

  // ---- the ring
  const bool old = first % kBlock != 0;  // block fb has older tokens
  auto replaced = [&](int w) { return old && w > fb && ((w - fb) & 1) == 0; };  // w lies where fb does
  if (slot_ok) {
    if (blk >= last - 1 && !replaced(blk)) {
#pragma unroll
      for (int u = 0; u < kPasses; ++u) {
        const int t = blk * kBlock + u * kTokensPerPass + (tid >> 3);
        if (t >= first && t < s.len) keep(t, lo[u], hi[u]);
      }
    }
    if (blk == fb)
      for (int w = max(last - 1, fb); w <= last; ++w)
        if (replaced(w))
          for (int u = 0; u < kPasses; ++u) {
            const int t = w * kBlock + u * kTokensPerPass + (tid >> 3);
            uint4 x, y;
            load(t, x, y);
            if (t < s.len) keep(t, x, y);
          }
  }

  // ---- codes and scale (magnitudes below 2^-90 count as zero, which keeps
  // the scale and its reciprocal ordinary fp32 values).  A block whose older
  // tokens are in no ring keeps what it has.
  if (page < 0 || page >= cb.n_pages || (old && blk == fb && !slot_ok)) return;
  const float top = bf16_lo(__builtin_amdgcn_readfirstlane(m));
  const QScale qs = qscale_from_absmax(top < 0x1p-90f ? 0.0f : top);
  const int64_t head = (int64_t)page * cb.Hkv + hk;
  if (tid == 0) cb.scales[head * 2 + (keys ? 0 : 1)] = qs.s;
  int8_t* dst = (keys ? cb.k_codes : cb.v_codes) + head * kPageBytes;
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int tok = u * kTokensPerPass + (tid >> 3);
    const uint2 q0 = quant_chunk(lo[u], qs.s, qs.inv, qs.mode), q1 = quant_chunk(hi[u], qs.s, qs.inv, qs.mode);
    if (keys) {
      *reinterpret_cast<uint2*>(dst + tok * kD + 8 * c) = q0;
      *reinterpret_cast<uint2*>(dst + tok * kD + kHalf + 8 * c) = q1;
    } else {
      uint32_t* l = reinterpret_cast<uint32_t*>(l_codes + tok * kCodePitch);
      l[2 * c] = q0.x;
      l[2 * c + 1] = q0.y;
      l[16 + 2 * c] = q1.x;
      l[16 + 2 * c + 1] = q1.y;
    }
  }
  if (keys) return;
  // the values' codes are held [d][token]: a thread turns 4 d of 8 tokens
  lds_barrier();
  if (tid >= kD / 4 * (kBlock / 8)) return;
  const int d4 = tid & 31, t8 = tid >> 5;
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint32_t*>(l_codes + (8 * t8 + e) * kCodePitch + 4 * d4);
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    uint2 o;
    o.x = pack4(w[0] >> (8 * d), w[1] >> (8 * d), w[2] >> (8 * d), w[3] >> (8 * d));
    o.y = pack4(w[4] >> (8 * d), w[5] >> (8 * d), w[6] >> (8 * d), w[7] >> (8 * d));
    *reinterpret_cast<uint2*>(dst + (4 * d4 + d) * kBlock + 8 * t8) = o;
  }
}

// ---- attention

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Weights are exp2(score - offset) 2^12.  The offset follows the running maximum
// only where that has outgrown it by more than 3, so that the sums are hardly
// ever rescaled: weights reach 2^15 at most, and fp16 holds those down to
// 2^-26 of the offset's in full precision.
constexpr float kWeightShift = 12.0f, kSlack = 3.0f;
// A weight carries its block's scale of the values.  As long as the scales lie
// in [kLowScale, kHighScale], a weight that vanishes in fp32 (below 2^-126)
// counts for less than 2^-58 of the total: it lies 2^138 below a weight at the
// offset, and two scales are 2^80 apart at most.  Past that range a block whose
// largest weight lies more than kFar below the offset adds to the total apart
// from its weights, in rows that have seen such a scale.
constexpr float kLowScale = 0x1p-60f, kHighScale = 0x1p20f, kLowLog2 = -60.0f, kHighLog2 = 20.0f, kFar = 100.0f;
// stand-in scale of a values' block of zeros: its weights still count
constexpr float kZeroLog2 = kLowLog2, kZeroInv = 1.0f / kLowScale;
// Exponents are score factor + (log2 of the values' scale + 12 - offset), one
// multiply-add a weight; with offsets from here on that sum's rounding (2^-7)
// would show, and soon pass fp16's range: there the offset is subtracted from
// the rounded score, which is exact where it counts.
constexpr float kLarge = 0x1p16f;
// The total is held times 2^-15: a token whose weight is at the offset then adds
// 2^-3 / scale, up to 2^97 with the smallest scale there is and the slack, so
// that 2^30 of them stay below 2^128, and 2^-103 with a scale of 2^100.
constexpr float kTotalUnit = 0x1p-15f, kTotalShift = kWeightShift - 15.0f;

__device__ __forceinline__ f16x2 as_f16x2(uint32_t u) { return __builtin_bit_cast(f16x2, u); }

// Four signed codes as fp16, exactly: the byte code + 128 under the exponent
// of 1024 is 1152 + code.
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& a, uint32_t& b) {
  const uint32_t u = w ^ 0x80808080u;
  const f16x2 bias = {(_Float16)-1152.0f, (_Float16)-1152.0f};
  a = __builtin_bit_cast(uint32_t, as_f16x2(__builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + bias);
  b = __builtin_bit_cast(uint32_t, as_f16x2(__builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + bias);
}
__device__ __forceinline__ f16x8 codes_to_f16x8(uint32_t w0, uint32_t w1) {
  uint4 r;
  codes_to_f16(w0, r.x, r.y);
  codes_to_f16(w1, r.z, r.w);
  return __builtin_bit_cast(f16x8, r);
}
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

// One workgroup per (rows of one sequence's kv head, split of its blocks).
// A row is a (new token, query head of the kv head) pair, row i G + g; a wave
// holds R tiles of 16 rows.  Of NW waves KW hold the same rows and take every
// KW-th block each, meeting in LDS at the end; the NW / KW of them that go
// through the same blocks hold different rows.
//
// Per block of 64 tokens:
//   - the rotated query is two int8 digits of a 16-bit number on its row's
//     scale, so S^T = K Q^T is exact int8 MFMAs on the codes as they lie in
//     the page;
//   - lane group g (16 lanes) holds tokens 16 g .. 16 g + 15 of its row's
//     scores, which is what 16 bytes of a value row [d][token] give it;
//   - weights exp2(score + log2(values' scale) - offset) in fp16 with the
//     values' codes in fp16 (exact) for O^T += V^T P^T: the values' scale is
//     inside the weight, and comes out of the weights' total through its
//     reciprocal;
//   - the next block's scores are formed under this block's exponentials.
//
// Waves that share their blocks bring each through LDS, a block ahead of its
// use: 64 lanes that fetch operands straight from a page touch 16 rows 64
// bytes at a time, in the page's own order an instruction covers 1 KiB.  Each
// wave loads its share; chunk c (16 bytes) of token j's keys lies at
// c ^ (2 (j / 16) + j / 2 % 2), so that the 16 rows that an operand read
// touches at once are on distinct banks, and it converts its share of the
// values to fp16 on the way, a quarter of the vector instructions (at R = 2
// they were a third of all).  A wave that has its blocks to itself (KW = NW)
// reads its operands from memory: no barrier, and a shorter way to the first
// of them.
template <int R, int KW, int NW, int AUX = kCacheDefault>
__global__ __launch_bounds__(NW * 64, 2) void cache_attention(const CacheAttnArgs a) {
  constexpr int kWaveRows = 16 * R, kSame = NW / KW, kRows = kSame * kWaveRows;
  constexpr bool kDirect = kSame == 1;
  constexpr int kPitch = kD + 4;  // floats of a row in the merge
  // LDS of the waves on one block: two stages of keys, then two of values
  constexpr int kValues = 2 * kPageBytes, kValueStage = 2 * kPageBytes;
  constexpr int kGroupBytes = kDirect ? 0 : kValues + 2 * kValueStage, kMergeBytes = KW > 1 ? NW * kWaveRows * kPitch * 4 : 0;
  __shared__ __align__(16) uint8_t lds[std::max(KW * kGroupBytes, kMergeBytes)];
  __shared__ float2 l_ml[KW > 1 ? NW * kWaveRows : 1];
  __shared__ float l_scale[kRows];  // of a row's scores, in base-2 units, before the block's

  const CacheBatch& cb = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int G = a.G, kw = wave / kSame, same = wave % kSame;
  // Workgroups of neighbouring kv heads go to the XCDs in turn, so that all of
  // a head's row blocks find its pages in one L2.
  const int hk = blockIdx.x;
  int split = blockIdx.y, item = blockIdx.z;
  if ((int)gridDim.y > a.S) {  // more row blocks than one axis of a launch holds
    item += (split / a.S) * gridDim.z;
    split %= a.S;
  }

  // ---- the workgroup's place.  A row's number wg_row0 + x is token i0 + (r0 +
  // x) / G: one division for the workgroup, and a product for the small numbers
  // (below 2^13, where the half keeps it clear of the integers by more than its
  // rounding).
  const Sequence s =
      find_sequence(cb, item, [&](int n, int) { return (int)(((uint32_t)(n * G) + kRows - 1) / kRows); });
  if (s.b < 0) return;
  const int n_rows = s.n * G, wg_row0 = s.item * kRows, i0 = a.by_g.divide(wg_row0), r0 = wg_row0 - i0 * G;
  auto token_of = [&](int x) { return i0 + (int)(((float)(r0 + x) + 0.5f) * a.inv_g); };
  // this split's blocks of those that the workgroup's last row sees
  const int seen = s.len - s.n + token_of(min(wg_row0 + kRows, n_rows) - 1 - wg_row0) + 1;
  const int blocks = (max(seen, 0) + kBlock - 1) / kBlock, per = a.by_s.divide(blocks + a.S - 1);
  const int p_begin = split * per, p_end = min(p_begin + per, blocks);

  // ---- the wave's blocks p_first + KW i < p_end; all waves of a workgroup
  // that meet at barriers make the same number of rounds.  Lane j of page_l
  // and scales_l holds what block 64 (i / 64) + j needs.
  const int p_first = p_begin + kw;
  const int rounds = max(p_end - (kDirect ? p_first : p_begin) + KW - 1, 0) / KW;
  int page_l = -1;
  float2 scales_l;
  auto fetch_pages = [&](int i0) {
    const int p = p_first + KW * (i0 + lane);
    page_l = p < p_end ? cb.table[(int64_t)s.b * cb.max_blocks + p] : -1;
    if (page_l >= cb.n_pages) page_l = -1;  // no page (as below 0): tokens that no row sees
  };
  auto fetch_scales = [&] {
    scales_l = make_float2(0.0f, 0.0f);
    if (page_l >= 0) scales_l = *reinterpret_cast<const float2*>(cb.scales + ((int64_t)page_l * cb.Hkv + hk) * 2);
  };
  fetch_pages(0);
  // the positions of the rows that this wave rotates, four at a time, 16 lanes
  // to a row (past the sequence's rows the last one again)
  constexpr int kTurns = kRows / NW / 4;
  int pos_l[kTurns];
  auto turn_row = [&](int t) { return (wave * kTurns + t) * 4 + g; };
  auto turn_token = [&](int t) { return token_of(min(turn_row(t), n_rows - 1 - wg_row0)); };
#pragma unroll
  for (int t = 0; t < kTurns; ++t) pos_l[t] = cb.pos[s.row0 + turn_token(t)];

  // ---- the blocks' codes.  Operand order: keys, row m of tile t is token
  // 16 (m / 4) + 4 t + m % 4, so that lane group g gets the scores of tokens
  // 16 g + 4 t ..; values, row d of a tile of 16, tokens 16 g ..
  auto page_bytes = [&](int page) { return page < 0 ? 0u : (uint32_t)kPageBytes; };  // nothing is read where there is no page
  auto page_base = [&](const int8_t* codes, int page) {
    return uniform_ptr(codes + ((int64_t)max(page, 0) * cb.Hkv + hk) * kPageBytes);
  };
  uint8_t* l_group = lds + kw * kGroupBytes;
  const uint32_t lds_group = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)l_group;
  constexpr int kLoads = 8 / kSame;  // KiB of a block's keys (and values) that this wave loads
  // direct: operands
  const uint32_t k_own = (uint32_t)((16 * (l16 >> 2) + (l16 & 3)) * kD + 16 * g), v_own = (uint32_t)(l16 * kBlock + 16 * g);
  v4i kr[kDirect ? 4 : 1][2];
  // through LDS: 8 tokens' keys an instruction
  const uint32_t k_chunk = (uint32_t)((lane & 7) ^ ((lane >> 4) & 1)), k_row = (uint32_t)(lane >> 3) * kD;
  auto load_keys = [&](int i, int page) {  // block i's, through LDS: to stage i % 2
    if constexpr (kDirect) {
      const __amdgpu_buffer_rsrc_t r = make_rsrc(page_base(cb.k_codes, page), page_bytes(page));
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) kr[t][h] = as_v4i(buf_load16<AUX>(r, k_own + (uint32_t)(4 * t * kD + 64 * h)));
    } else {
      const u32x4 r = make_rsrc_words(page_base(cb.k_codes, page), page_bytes(page));
      const uint32_t dst = lds_group + (uint32_t)((i & 1) * kPageBytes);
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        const int m = same * kLoads + n;  // tokens 8 m ..
        lds_dma16(r, uniform_u32(dst + (uint32_t)(m * 1024)), k_row + ((k_chunk ^ (uint32_t)(2 * (m >> 1))) << 4) + (uint32_t)(m * 1024), 0);
      }
    }
  };
  // values: to registers, direct as operands, else in the page's order, and
  // then as fp16 to LDS: the two MFMA operands (8 tokens of a lane group each)
  // of tile d at 2 d and 2 d + 1, lane group g's row r at 16 g + (r ^ 4 g)
  uint4 vr[kLoads];
  auto load_values = [&](int page) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(page_base(cb.v_codes, page), page_bytes(page));
#pragma unroll
    for (int d = 0; d < kLoads; ++d)
      vr[d] = buf_load16<AUX>(r, (uint32_t)((same * kLoads + d) * 1024) + (kDirect ? v_own : (uint32_t)(lane * 16)));
  };
  const int v_put = (lane & 3) * 256 + (((lane >> 2) ^ (4 * (lane & 3))) << 4);
  auto stage_values = [&](int i) {
    uint8_t* dst = l_group + kValues + (i & 1) * kValueStage + 2 * same * kLoads * 1024 + v_put;
#pragma unroll
    for (int d = 0; d < kLoads; ++d) {
      *reinterpret_cast<f16x8*>(dst + 2048 * d) = codes_to_f16x8(vr[d].x, vr[d].y);
      *reinterpret_cast<f16x8*>(dst + 2048 * d + 1024) = codes_to_f16x8(vr[d].z, vr[d].w);
    }
  };
  const int k_get = (16 * (l16 >> 2) + (l16 & 3)) * kD + ((g ^ (2 * (l16 >> 2) + ((l16 >> 1) & 1))) << 4);
  const int v_get = g * 256 + ((l16 ^ (4 * g)) << 4);

  // Pages of the block at hand and the ones after it.
  int page0 = __builtin_amdgcn_readlane(page_l, 0), page1 = __builtin_amdgcn_readlane(page_l, 1),
      page2 = __builtin_amdgcn_readlane(page_l, 2);
  load_keys(0, page0);

  // ---- the queries: lane l16 has d = 4 l16 .. and 64 + 4 l16 .. of a row.
  // The workgroup rotates each row once and hands the digits round through
  // LDS; rotated by every wave that needs it, a row took four times the vector
  // instructions and loads of 16 rows each.
  uint2 q_lo[kTurns], q_hi[kTurns];
  float4 cs4[kTurns], sn4[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int i = turn_token(t), row = min(turn_row(t) + wg_row0, n_rows - 1);
    const uint16_t* src = a.q.p + (s.row0 + i) * a.q.row + (hk * G + row - i * G) * a.q.head + 4 * l16;
    const int64_t at = (int64_t)clamp_pos(pos_l[t], cb.n_pos) * kHalf + 4 * l16;
    q_lo[t] = *reinterpret_cast<const uint2*>(src);
    q_hi[t] = *reinterpret_cast<const uint2*>(src + kHalf);
    cs4[t] = *reinterpret_cast<const float4*>(cb.rope_cos + at);
    sn4[t] = *reinterpret_cast<const float4*>(cb.rope_sin + at);
  }
  fetch_scales();
  load_values(page0);
  if constexpr (!kDirect) load_keys(1, page1);

  // A row's digits in LDS: 16 chunks of 16 bytes, the high digits of d = 16 c ..
  // in chunk c, the low ones in 8 + c, chunk c of row r at c ^ (r % 16); where
  // the merge comes later, or the values' second stages.
  auto digits = [&](int row) {
    return lds + (kDirect ? row * 256 : (row >> 6) * kGroupBytes + kValues + kValueStage + (row & 63) * 256);
  };
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const uint32_t pw[2] = {q_lo[t].x, q_lo[t].y}, rw[2] = {q_hi[t].x, q_hi[t].y};
    const float cs[4] = {cs4[t].x, cs4[t].y, cs4[t].z, cs4[t].w}, sn[4] = {sn4[t].x, sn4[t].y, sn4[t].z, sn4[t].w};
    float x[2][4];
    uint32_t mag = 0;  // the largest magnitude, as bits, which order like the numbers, infinity and NaN above them
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = (e & 1) ? bf16_hi(pw[e / 2]) : bf16_lo(pw[e / 2]);
      const float r = (e & 1) ? bf16_hi(rw[e / 2]) : bf16_lo(rw[e / 2]);
      x[0][e] = p * cs[e] - r * sn[e];
      x[1][e] = r * cs[e] + p * sn[e];
      mag = max(mag, max(__float_as_uint(x[0][e]) & 0x7FFFFFFFu, __float_as_uint(x[1][e]) & 0x7FFFFFFFu));
    }
    auto fold = [&](auto ctrl) { mag = max(mag, lane_move<decltype(ctrl)::value>(mag)); };
    fold(std::integral_constant<int, kXor1>{});  // over the row's 16 lanes
    fold(std::integral_constant<int, kXor2>{});
    fold(std::integral_constant<int, kMirror8>{});
    fold(std::integral_constant<int, kMirror16>{});
    const float top = __uint_as_float(mag);
    // 16 bits: |x| / sq <= 32512 = 127 * 256, half a step is 2^-16 of the row's
    // largest.  The number v is rounded by an addition that leaves v + 128 in
    // the low 16 bits: its high byte is the high digit, its low byte the low
    // digit + 128.
    const float inv = top < 0x1p-100f ? 0.0f : 32512.0f / top * a.q_sign;
    const int row = turn_row(t);
    uint32_t* dst = reinterpret_cast<uint32_t*>(digits(row)) + (l16 & 3);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(fmaf(x[h][e], inv, 12582912.0f + 128.0f));
      const uint32_t p01 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), p23 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u);
      const int c = 4 * h + (l16 >> 2);
      dst[4 * (c ^ (row & 15))] = __builtin_amdgcn_perm(p23, p01, 0x07060302u);
      dst[4 * ((c + 8) ^ (row & 15))] = __builtin_amdgcn_perm(p23, p01, 0x05040100u) ^ 0x80808080u;
    }
    if (l16 == 0) l_scale[row] = top * (1.0f / 32512.0f) * a.scale_log2e;
  }
  lds_barrier();

  // ---- this lane's rows (row l16 of each of the wave's tiles): digits, the B
  // operand of the int8 MFMAs, d = 16 g .. and 64 + 16 g ..
  v4i qh[R][2], ql[R][2];
  float row_scale[R];
  int last_key[R];  // the last token that the row sees, -1 for a row past the end
#pragma unroll
  for (int t = 0; t < R; ++t) {
    const int row = same * kWaveRows + 16 * t + l16;
    const uint8_t* src = digits(row);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      qh[t][h] = *reinterpret_cast<const v4i*>(src + (((4 * h + g) ^ l16) << 4));
      ql[t][h] = *reinterpret_cast<const v4i*>(src + (((4 * h + g + 8) ^ l16) << 4));
    }
    row_scale[t] = l_scale[row];
    last_key[t] = wg_row0 + row < n_rows ? s.len - s.n + token_of(row) : -1;
  }

  f32x4 acc[R][8];
  float m[R], l[R];
#pragma unroll
  for (int t = 0; t < R; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.0f;
#pragma unroll
    for (int d = 0; d < 8; ++d) acc[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // Scores of block i: the high digits' sum, times 256, plus the low digits',
  // in passes over several tiles, whose products do not wait for each other.
  v4i sc[R][4];
  auto score = [&](int i) {
    const uint8_t* src = l_group + (i & 1) * kPageBytes;
    constexpr int kPass = R == 1 ? 4 : 2;  // token tiles at a time: the operands' registers
#pragma unroll
    for (int u0 = 0; u0 < 4; u0 += kPass) {
      v4i kf[kPass][2];
#pragma unroll
      for (int u = 0; u < kPass; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)  // the second half of d is 4 chunks on
          kf[u][h] = kDirect ? kr[kDirect ? u0 + u : 0][h] : *reinterpret_cast<const v4i*>(src + (k_get ^ (64 * h)) + 4 * (u0 + u) * kD);
#pragma unroll
      for (int p = 0; p < 4; ++p)  // high digits of both halves of d, then low digits
#pragma unroll
        for (int t = 0; t < R; ++t)
#pragma unroll
          for (int u = 0; u < kPass; ++u) {
            v4i& x = sc[t][u0 + u];
            x = mfma16(kf[u][p & 1], p < 2 ? qh[t][p & 1] : ql[t][p & 1], p == 0 ? v4i{0, 0, 0, 0} : p == 2 ? x << 8 : x);
          }
    }
  };
  // Everything that this wave has loaded into LDS is there, and what it has
  // read from LDS has arrived; the asm keeps later accesses behind it.
  auto arrived = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); };

  if constexpr (!kDirect) {
    arrived();  // (the digits, too: the values' second stages are free after the barrier)
    stage_values(0);
    load_values(page1);
    lds_barrier();
  }
  score(0);
  if constexpr (kDirect)
    load_keys(1, page1);
  else
    lds_barrier();  // the first round loads over block 0's keys
  float vlog_l = 0.0f, vinv_l = 0.0f;
  bool careful = false;  // the wave has come to a scale of values out of the range, or to a large offset
  bool wild[R] = {};     // the row has seen such a scale
  for (int i = 0; i < rounds; ++i) {
    const int j = i & 63;
    if (j == 0) {  // the values' scales as they go into weights and total
      vlog_l = scales_l.y == 0.0f ? kZeroLog2 : __log2f(scales_l.y);
      vinv_l = scales_l.y == 0.0f ? kZeroInv * kTotalUnit : kTotalUnit / scales_l.y;
      careful = careful || __any(scales_l.y != 0.0f && !(scales_l.y >= kLowScale && scales_l.y <= kHighScale));
    }
    const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scales_l.x), j));
    const float vlog = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vlog_l), j));
    const float vinv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vinv_l), j));
    if (j == 61) fetch_pages(i + 3);  // the next 64; their scales once this block's have been read
    if (j == 63) fetch_scales();
    const int page3 = __builtin_amdgcn_readlane(page_l, (i + 3) & 63);
    const int key0 = (p_first + KW * i) * kBlock;

    // Block i's values and block i + 1's keys are in LDS, and block i's keys
    // and block i - 1's values are no longer read, as the barrier at the end
    // of the last round (before the first round, the one behind block 0's
    // scores) says: their places are free.
    if constexpr (!kDirect) {
      stage_values(i + 1);
      load_values(page2);
      load_keys(i + 2, page2);
    }

    // ---- the rows' largest scores, and what turns a score into an exponent:
    // f is the base-2 factor, above 0 so that a masked -inf stays -inf
    float x[R][16], f[R], vl[R], vi[R], top[R];
    bool all = true;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      int mx = sc[t][0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = max(mx, sc[t][e >> 2][e & 3]);
      top[t] = (float)mx;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][e] = (float)sc[t][e >> 2][e & 3];
      f[t] = row_scale[t] * ks;
      f[t] = f[t] < 0x1p-126f ? 0x1p-126f : f[t];
      vl[t] = vlog;
      vi[t] = vinv;
      all = all && last_key[t] >= key0 + kBlock - 1;
    }
    if (!__all(all) || page0 < 0) {
#pragma unroll
      for (int t = 0; t < R; ++t) {
        const int lim = page0 >= 0 ? last_key[t] - key0 - 16 * g : INT_MIN;  // tokens of this lane past it are not seen
        top[t] = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[t][e] = e <= lim ? x[t][e] : -INFINITY;
          top[t] = fmaxf(top[t], x[t][e]);
        }
        if (page0 < 0 || last_key[t] < key0) {  // nothing of the block is seen, whatever its scales hold
          f[t] = 1.0f;
          vl[t] = vi[t] = 0.0f;
        }
      }
    }
    bool outgrown = false;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      top[t] = fold_groups(fmaf(top[t], f[t], vl[t]), [](float p, float r) { return fmaxf(p, r); });
      outgrown = outgrown || top[t] - m[t] > kSlack;
    }
    if (__any(outgrown)) {
      bool large = false;
#pragma unroll
      for (int t = 0; t < R; ++t) {
        // a row's own maximum alone moves its offset: its result does not
        // depend on the rows that share the wave
        const bool up = top[t] - m[t] > kSlack;
        l[t] = rescaled(l[t], up ? m[t] - top[t] : 0.0f);
        const float alpha = up ? __builtin_amdgcn_exp2f(m[t] - top[t]) : 1.0f;
        m[t] = up ? top[t] : m[t];
        large = large || (fabsf(m[t]) >= kLarge && m[t] != -INFINITY);
#pragma unroll
        for (int d = 0; d < 8; ++d) acc[t][d] *= alpha;
      }
      careful = careful || __any(large);
    }
    // Rows with a large offset, and rows far above a block after a scale out of
    // the range (kFar): the weights from the rounded score less the offset, the
    // total from the scores alone.  That the loop has this way at all costs 1 - 2 %
    // of a call (1024 over 8192: 150 us without it, 153 with it).
    if (__builtin_expect(careful, 0)) {
#pragma unroll
      for (int t = 0; t < R; ++t) {
        wild[t] = wild[t] || (top[t] > -INFINITY && !(vlog >= kLowLog2 && vlog <= kHighLog2));
        const bool apart = (fabsf(m[t]) >= kLarge && m[t] != -INFINITY) || (wild[t] && top[t] < m[t] - kFar);
        const float shift = m[t] + kWeightShift - m[t];  // what the offset below becomes: 12, and m's rounding
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float y = fmaf(x[t][e], f[t], vl[t]) - m[t];
          sum += __builtin_amdgcn_exp2f(y - vl[t] + kTotalShift);
          x[t][e] = apart ? y + (kWeightShift - shift) : x[t][e];
        }
        l[t] += apart ? sum : 0.0f;
        f[t] = apart ? 1.0f : f[t];
        vl[t] = apart ? m[t] : vl[t];
        vi[t] = apart ? 0.0f : vi[t];
      }
    }

    // ---- weights, the next block's scores under them
    f16x8 pw[R][2];
    score(i + 1);
    if constexpr (kDirect) load_keys(i + 2, page2);
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const float off = vl[t] + kWeightShift - (m[t] == -INFINITY ? 0.0f : m[t]);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][e] = __builtin_amdgcn_exp2f(fmaf(x[t][e], f[t], off));
#pragma unroll
      for (int h = 0; h < 2; ++h)
        pw[t][h] = __builtin_bit_cast(
            f16x8, make_uint4(f16x2_bits(x[t][8 * h], x[t][8 * h + 1]), f16x2_bits(x[t][8 * h + 2], x[t][8 * h + 3]),
                              f16x2_bits(x[t][8 * h + 4], x[t][8 * h + 5]), f16x2_bits(x[t][8 * h + 6], x[t][8 * h + 7])));
      // the total takes the weights before their rounding to fp16, where those
      // of a block with small values have vanished
      float sum[4] = {x[t][0], x[t][1], x[t][2], x[t][3]};
#pragma unroll
      for (int e = 4; e < 16; ++e) sum[e & 3] += x[t][e];
      l[t] = fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), vi[t], l[t]);
    }

    // ---- O^T += V^T P^T
    const uint8_t* src = l_group + kValues + (i & 1) * kValueStage + v_get;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      f16x8 v0, v1;
      if constexpr (kDirect) {
        v0 = codes_to_f16x8(vr[d].x, vr[d].y);
        v1 = codes_to_f16x8(vr[d].z, vr[d].w);
      } else {
        v0 = *reinterpret_cast<const f16x8*>(src + 2048 * d);
        v1 = *reinterpret_cast<const f16x8*>(src + 2048 * d + 1024);
      }
#pragma unroll
      for (int t = 0; t < R; ++t) acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pw[t][0], acc[t][d], 0, 0, 0);
#pragma unroll
      for (int t = 0; t < R; ++t) acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pw[t][1], acc[t][d], 0, 0, 0);
    }
    if constexpr (kDirect) {
      load_values(page1);
    } else {
      arrived();
      lds_barrier();
    }
    page0 = page1;
    page1 = page2;
    page2 = page3;
  }
#pragma unroll
  for (int t = 0; t < R; ++t) l[t] = fold_groups(l[t], [](float p, float r) { return p + r; });

  // Where a row's result goes: its partial sums, or the output.
  auto write8 = [&](int row, int d, const float (&o)[8], float mx, float lsum) {
    const int i = token_of(row - wg_row0), h = hk * G + row - i * G;
    const int64_t tok = s.row0 + i;
    if (a.S > 1) {
      const int64_t at = ((int64_t)split * cb.T + tok) * a.H + h;
      float* po = a.part_o + at * kD + d;
      *reinterpret_cast<float4*>(po) = make_float4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<float4*>(po + 4) = make_float4(o[4], o[5], o[6], o[7]);
      if (d == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(mx, lsum);
    } else {
      *reinterpret_cast<uint4*>(a.o.p + tok * a.o.row + h * a.o.head + d) = output8(o, lsum);
    }
  };

  if constexpr (KW > 1) {
    // the KW waves' partial results of the same rows meet in LDS, where the
    // stages were
    float* l_o = reinterpret_cast<float*>(lds);
    arrived();
    lds_barrier();
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const int r = wave * kWaveRows + 16 * t + l16;
#pragma unroll
      for (int d = 0; d < 8; ++d)
        *reinterpret_cast<float4*>(&l_o[r * kPitch + 16 * d + 4 * g]) = make_float4(acc[t][d][0], acc[t][d][1], acc[t][d][2], acc[t][d][3]);
      if (g == 0) l_ml[r] = make_float2(m[t], l[t]);
    }
    lds_barrier();
    for (int i = tid; i < kRows * 16; i += NW * 64) {
      const int r = i >> 4, d = (i & 15) * 8, row = wg_row0 + r;  // row r lies r + kRows w rows from the first wave's
      if (row >= n_rows) continue;
      float mx = -INFINITY, lsum = 0.0f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KW; ++w) mx = fmaxf(mx, l_ml[r + w * kRows].x);
      const float base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float2 ml = l_ml[r + w * kRows];
        const float f = __builtin_amdgcn_exp2f(ml.x - base);
        lsum += rescaled(ml.y, ml.x - base);
        const float* p = &l_o[(r + w * kRows) * kPitch + d];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(p[e], f, o[e]);
      }
      write8(row, d, o, mx, lsum);
    }
  } else {
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const int row = wg_row0 + same * kWaveRows + 16 * t + l16;
      // lane groups g and g ^ 1 trade halves, so that a lane has 8 d in a row
#pragma unroll
      for (int d = 0; d < 8; d += 2) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool odd = g & 1;
          const float got = __shfl_xor(odd ? acc[t][d][e] : acc[t][d + 1][e], 16, 64), own = odd ? acc[t][d + 1][e] : acc[t][d][e];
          o[e] = odd ? got : own;
          o[4 + e] = odd ? own : got;
        }
        if (row < n_rows) write8(row, 16 * (d + (g & 1)) + 8 * (g >> 1), o, m[t], l[t]);
      }
    }
  }
}

// Merge of the splits' partial results, [S][T][H]: P threads for 8 d of a
// (token, head), each folding every P-th split, their results meeting by lane
// moves and, from four waves, in LDS.  (One thread for all of 64 splits took
// 36 us of the 79 that one token over 100000 took: its reads wait for each
// other.)  Tokens of no sequence are left as they are.
template <int P>
__global__ __launch_bounds__(256) void cache_attention_merge(const CacheAttnArgs a) {
  constexpr int kChunks = kD / 8, kRowsHere = 256 / (kChunks * P);
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

// The forms of a call, and what one of its workgroups costs in ns: alone on a
// CU lat + lat_round a round (a block of each of the KW groups of waves); in
// a full chip each of the ceil(workgroups / 256) that a CU runs adds thr +
// thr_round a round.  Fitted, with the merge's 1820 + 0.21 a (split, token,
// head), to 138 calls (B 1 - 64, 1 - 1024 new tokens, 1 - 100000 long, six head
// layouts) at 12 numbers of splits: what the rule picks is 0.8 % above the best
// of all forms and splits on average, 9 % at most; 32 rows a workgroup, 64 in
// four waves times two and 128 in four waves, tried too, would take off under
// 1 %.  us of 16 / 64 / 128 rows, at its best splits each: 8 x 16 tokens over
// 2500 20.4 23.2 27.6, 23 x 27 over 478 30.5 20.8 19.1, 1024 over 8192 326 195
// 155.
//   The calls were of one kind of sequence each.  A batch is taken as B
// sequences of max_len with the average number of new tokens, so one that mixes
// kinds gets the form and splits of neither.  us of the batch, and of its two
// parts as calls of their own: one token over 100000 among 63 over 200 673, 41 +
// 10; a chunk of 1024 among 8 single tokens, all over 8192, 249, 153 + 27; among
// 32 343, 153 + 83; a chunk of 193 among 63 251, 53 + 160.
typedef void (*AttnFn)(const CacheAttnArgs);
struct AttnForm {
  int rows, KW, threads;
  int64_t lat, lat_round, thr, thr_round;
  AttnFn fn;
};
const AttnForm kForms[] = {
    {16, 4, 256, 800, 970, 860, 990, cache_attention<1, 4, 4>},
    {64, 1, 256, 1570, 1010, 1840, 720, cache_attention<1, 1, 4>},
    {128, 2, 512, 3010, 50, 8830, 1600, cache_attention<2, 2, 8>},
};
// A cache that is read once (by the average of new tokens, as above) and is
// larger than this does not stay in the memory-side cache (256 MB) until the
// next call: it is read past it.  us with / without: 64 sequences of 4096 (537 MB)
// 84 / 99, one of 100000 (205 MB) 39 / 44; of 131 MB, when called again and again,
// 28.4 / 27.7.
constexpr int64_t kStreamBytes = int64_t(160) << 20;
const AttnFn kStreamFn = cache_attention<1, 4, 4, kCacheStream>;
constexpr int64_t kMaxAxis = 65535;  // workgroups along the second and third axis of a launch

struct AttnPlan {
  int form = 0, S = 1;
  bool stream = false;
  int64_t tiles = 0;  // the most row blocks that the batch can have
};

// On the host's path of every call: 60 ns, 250 with divisions.  Rows and KW are
// powers of two and the loop over the splits is unrolled, so nearly all
// divisions are shifts and products.
AttnPlan plan_attention(int B, int T, int H, int Hkv, int max_len) {
  const int64_t G = H / Hkv, n = (T + B - 1) / B, blocks = (max_len + kBlock - 1) / kBlock;
  const int64_t most = (int64_t)T * H <= (1 << 22) ? blocks : 1;  // splits
  constexpr int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
  AttnPlan p;
  int64_t least = INT64_MAX;
  for (int f = 0; f < (int)(sizeof kForms / sizeof kForms[0]); ++f) {
    const AttnForm& k = kForms[f];
    const int by_rows = __builtin_ctz(k.rows), by_kw = __builtin_ctz(k.KW);
    const int64_t tiles = B * ((n * G + k.rows - 1) >> by_rows) * Hkv;
#pragma unroll
    for (int S : kSplits) {
      if (S > 1 && S > most) break;
      const int64_t rounds = ((uint64_t)(blocks + S - 1) / S + k.KW - 1) >> by_kw;
      const int64_t cost = std::max(k.lat + rounds * k.lat_round, ((tiles * S + 255) >> 8) * (k.thr + rounds * k.thr_round)) +
                           (S > 1 ? 1820 + (int64_t)((uint64_t)S * T * H * 21 / 100) : 0);
      if (cost < least) {
        least = cost;
        p.form = f;
        p.S = S;
      }
    }
  }
  const int64_t rows = kForms[p.form].rows;
  // every sequence's last row block may be partial, but each has a row
  p.tiles = std::min<int64_t>(T * G / rows + B, T * ((G + rows - 1) / rows));
  p.stream = p.form == 0 && n * G <= rows && (int64_t)B * max_len >= kStreamBytes / (2 * kD) / Hkv;
  return p;
}

size_t workspace_of(const AttnPlan& p, int T, int H) {
  return p.S > 1 ? kCounterRegionBytes + (size_t)p.S * T * H * (kD + 2) * sizeof(float) : 0;
}

}  // namespace

hipError_t launch_cache_append(const CacheAppendArgs& a, hipStream_t stream) {
  if (a.c.T == 0 || a.c.B == 0) return hipSuccess;
  // touched blocks: (n + 126) / 64 of a sequence with n new tokens at most, and no more than its tokens
  const int64_t most = std::min<int64_t>(a.c.T, ((int64_t)a.c.T + 126ll * std::min(a.c.B, a.c.T)) / kBlock);
  cache_append<<<dim3((unsigned)most, (unsigned)a.c.Hkv, 2), dim3(kAppendThreads), 0, stream>>>(a);
  return hipGetLastError();
}

// 2^28 rows of a kv head: the row blocks of 64 sequences, each of which may
// claim all rows (whatever the arrays hold), then add up within 32 bits, and
// two axes of a launch hold the row blocks of a call.
bool cache_attention_fits(int T, int H, int Hkv) { return (int64_t)T * (H / Hkv) <= int64_t(1) << 28; }

size_t cache_attention_workspace(int B, int T, int H, int Hkv, int max_len) {
  return workspace_of(plan_attention(B, T, H, Hkv, max_len), T, H);
}

bool launch_cache_attention(const CacheAttnArgs& a0, void* workspace, size_t bytes, hipStream_t stream, hipError_t& error) {
  CacheAttnArgs a = a0;
  const AttnPlan p = plan_attention(a.c.B, a.c.T, a.H, a.c.Hkv, a.max_len);
  const size_t need = workspace_of(p, a.c.T, a.H);
  if (need && (bytes < need || !workspace || (uintptr_t)workspace % 256)) return false;
  a.G = a.H / a.c.Hkv;
  a.S = p.S;
  a.inv_g = 1.0f / (float)a.G;
  a.by_g = Divisor(a.G);
  a.by_s = Divisor(a.S);
  if (a.S > 1) {
    a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kCounterRegionBytes);
    a.part_ml = a.part_o + (size_t)a.S * a.c.T * a.H * kD;
  }
  const AttnForm& k = kForms[p.form];
  const unsigned z = (unsigned)std::min<int64_t>(p.tiles, kMaxAxis), y = (unsigned)((p.tiles + z - 1) / z) * (unsigned)a.S;
  (p.stream ? kStreamFn : k.fn)<<<dim3((unsigned)a.c.Hkv, y, z), dim3(k.threads), 0, stream>>>(a);
  if (a.S > 1) {
    const int P = a.S <= 16 ? 4 : 16;
    const int64_t threads = (int64_t)a.c.T * a.H * (kD / 8) * P;
    const AttnFn merge = P == 4 ? cache_attention_merge<4> : cache_attention_merge<16>;
    merge<<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream>>>(a);
  }
  error = hipGetLastError();
  return true;
}

}  // namespace w4a8
