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

constexpr int kAppendThreads = 256;
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
  const bool slot_ok = slot >= 0 && slot < a.n_slots;
  const TokenRows rows = keys ? a.k : a.v;
  uint16_t* ring = (keys ? a.k_recent : a.v_recent) + ((int64_t)(slot_ok ? slot : 0) * cb.Hkv + hk) * (kRecent * kD);
  const int c = tid & 7;

  // chunks c and c + 8 of token t: rotated if it is a new key
  auto load = [&](int t, uint4& lo, uint4& hi) {
    lo = hi = make_uint4(0u, 0u, 0u, 0u);
    if (t >= s.len) return;
    if (t < first) {
      if (!slot_ok) return;
      const uint16_t* src = ring + (t & (kRecent - 1)) * kD;
      lo = *reinterpret_cast<const uint4*>(src + 8 * c);
      hi = *reinterpret_cast<const uint4*>(src + kHalf + 8 * c);
      return;
    }
    const int row = s.row0 + t - (s.len - s.n);
    const uint16_t* src = rows.p + row * rows.row + hk * rows.head;
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
      rotate_pair(lo, hi, cs, sn);
    }
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
  // the scale and its reciprocal ordinary fp32 values)
  const int page = cb.table[(int64_t)s.b * cb.max_blocks + blk];
  if (page < 0 || page >= cb.n_pages) return;
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

constexpr int kAttnWaves = 4;
// log2 of the factor on all weights: fp16 then holds weights down to 2^-29 of
// the largest in full precision
constexpr float kWeightShift = 15.0f;
// stand-in scale of a values' block of zeros (2^-80): its weights still count
constexpr float kZeroLog2 = -80.0f, kZeroInv = 0x1p80f;

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
// holds R tiles of 16 rows.  KW waves hold the same rows and take every KW-th
// block each, meeting in LDS at the end; the 4 / KW groups of waves hold
// different rows.
//
// Per block of 64 tokens, with everything in registers (the page's layout is
// the operands'):
//   - the rotated query is two int8 digits of a 16-bit number on its row's
//     scale, so S^T = K Q^T is exact int8 MFMAs on the codes as they lie in
//     the page;
//   - lane group g (16 lanes) holds tokens 16 g .. 16 g + 15 of its row's
//     scores, which is what a 16-byte load of a value row [d][token] gives it;
//   - weights exp2(score + log2(values' scale) - running maximum) in fp16
//     with the values' codes in fp16 (exact) for O^T += V^T P^T: the values'
//     scale is inside the weight, and comes out of the weights' total through
//     its reciprocal.
template <int R, int KW>
__global__ __launch_bounds__(kAttnWaves * 64, 2) void cache_attention(const CacheAttnArgs a) {
  constexpr int kWaveRows = 16 * R, kRows = kAttnWaves / KW * kWaveRows;
  constexpr int kPitch = kD + 4;  // floats of a row in the merge
  __shared__ __align__(16) float l_o[KW > 1 ? kAttnWaves * kWaveRows * kPitch : 4];
  __shared__ float2 l_ml[KW > 1 ? kAttnWaves * kWaveRows : 1];

  const CacheBatch& cb = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % cb.Hkv, rest = blockIdx.x / cb.Hkv, split = rest % a.S;
  const int G = a.G;
  const Sequence s =
      find_sequence(cb, rest / a.S, [&](int n, int) { return (int)(((int64_t)n * G + kRows - 1) / kRows); });
  if (s.b < 0) return;
  const int kw = wave % KW, n_rows = s.n * G, row0 = s.item * kRows + wave / KW * kWaveRows;
  // tokens that the workgroup's (the wave's) last row sees
  auto seen_by = [&](int row) { return s.len - s.n + min(row, n_rows - 1) / G + 1; };
  const int blocks_wg = (max(seen_by(s.item * kRows + kRows - 1), 0) + kBlock - 1) / kBlock;
  const int per = (blocks_wg + a.S - 1) / a.S;
  const int seen = row0 < n_rows ? max(seen_by(row0 + kWaveRows - 1), 0) : 0;
  const int p_begin = split * per, p_end = min(p_begin + per, (seen + kBlock - 1) / kBlock);

  // ---- the wave's blocks p = p_first + KW i, i < count; lane j of the
  // registers below holds what block 64 (i / 64) + j needs
  const int p_first = p_begin + kw;
  const int count = p_end > p_first ? (p_end - p_first + KW - 1) / KW : 0;
  int page_l = -1;
  float2 scales_l;
  auto fetch_pages = [&](int i0) {
    const int i = i0 + lane;
    page_l = i < count ? cb.table[(int64_t)s.b * cb.max_blocks + p_first + KW * i] : -1;
    if (page_l >= cb.n_pages) page_l = -1;  // no page (as below 0): tokens that no row sees
  };
  auto fetch_scales = [&] {
    scales_l = make_float2(0.0f, 0.0f);
    if (page_l >= 0) scales_l = *reinterpret_cast<const float2*>(cb.scales + ((int64_t)page_l * cb.Hkv + hk) * 2);
  };
  auto resource = [&](const int8_t* codes, int page) {  // an empty one where there is no page
    return make_rsrc(codes + ((int64_t)max(page, 0) * cb.Hkv + hk) * kPageBytes, page < 0 ? 0u : (uint32_t)kPageBytes);
  };
  // K: row m of tile t is token 16 (m / 4) + 4 t + m % 4, so that lane group g
  // gets the scores of tokens 16 g + 4 t ..; V: row d, tokens 16 g ..
  const uint32_t k_off = (uint32_t)((16 * (l16 >> 2) + (l16 & 3)) * kD + 16 * g);
  const uint32_t v_off = (uint32_t)(l16 * kBlock + 16 * g);
  uint4 kr[4][2], vr[8];
  auto load_keys = [&](int page) {
    const __amdgpu_buffer_rsrc_t r = resource(cb.k_codes, page);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) kr[t][h] = buf_load16(r, k_off + (uint32_t)(4 * t * kD + 64 * h));
  };
  auto load_values = [&](int page) {
    const __amdgpu_buffer_rsrc_t r = resource(cb.v_codes, page);
#pragma unroll
    for (int d = 0; d < 8; ++d) vr[d] = buf_load16(r, v_off + (uint32_t)(16 * d * kBlock));
  };
  fetch_pages(0);

  // ---- this lane's rows (row l16 of each tile): the query's d = 16 g .. and
  // 64 + 16 g .. and the table row, requested before the first block's codes
  uint4 qr[R][4];
  float4 cs4[R][4], sn4[R][4];
  int last_key[R];  // the last token that the row sees, -1 for a row past the end
#pragma unroll
  for (int t = 0; t < R; ++t) {
    const int row = row0 + 16 * t + l16;
    const bool ok = row < n_rows;
    const int i = ok ? row / G : 0, tok = s.row0 + i;  // a row past the end reads the sequence's first
    last_key[t] = ok ? s.len - s.n + i : -1;
    const uint16_t* src = a.q.p + tok * a.q.row + (hk * G + (ok ? row - i * G : 0)) * a.q.head + 16 * g;
    const int64_t at = (int64_t)clamp_pos(cb.pos[tok], cb.n_pos) * kHalf + 16 * g;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      qr[t][e] = *reinterpret_cast<const uint4*>(src + (e >> 1) * kHalf + (e & 1) * 8);
      cs4[t][e] = *reinterpret_cast<const float4*>(cb.rope_cos + at + 4 * e);
      sn4[t][e] = *reinterpret_cast<const float4*>(cb.rope_sin + at + 4 * e);
    }
  }
  int page = __builtin_amdgcn_readlane(page_l, 0);
  load_keys(page);
  fetch_scales();
  load_values(page);

  // ---- the rotated queries' digits, the B operand of the int8 MFMAs
  v4i qh[R][2], ql[R][2];
  float row_scale[R];  // of a score, in base-2 units, before the block's
#pragma unroll
  for (int t = 0; t < R; ++t) {
    float x[2][16];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float cs[4] = {cs4[t][e].x, cs4[t][e].y, cs4[t][e].z, cs4[t][e].w};
      const float sn[4] = {sn4[t][e].x, sn4[t][e].y, sn4[t][e].z, sn4[t][e].w};
      const uint4 u = qr[t][e >> 1], v = qr[t][2 + (e >> 1)];
      const uint32_t uw[2] = {(e & 1) ? u.z : u.x, (e & 1) ? u.w : u.y}, vw[2] = {(e & 1) ? v.z : v.x, (e & 1) ? v.w : v.y};
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const float p = (f & 1) ? bf16_hi(uw[f / 2]) : bf16_lo(uw[f / 2]);
        const float r = (f & 1) ? bf16_hi(vw[f / 2]) : bf16_lo(vw[f / 2]);
        x[0][4 * e + f] = p * cs[f] - r * sn[f];
        x[1][4 * e + f] = r * cs[f] + p * sn[f];
      }
    }
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, fmaxf(fabsf(x[0][e]), fabsf(x[1][e])));
    top = fold_groups(top, [](float p, float r) { return fmaxf(p, r); });
    // 16 bits: |x| / sq <= 32512 = 127 * 256, half a step is 2^-16 of the row's largest
    const bool zero = top < 0x1p-100f;
    const float inv = zero ? 0.0f : 32512.0f / top * a.q_sign;
    row_scale[t] = top * (1.0f / 32512.0f) * a.scale_log2e;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int v = (int)rintf(x[h][4 * w + e] * inv);
          const int d = (v + 128) >> 8;
          hi[e] = (uint32_t)d;
          lo[e] = (uint32_t)(v - 256 * d);
        }
        qh[t][h][w] = (int)pack4(hi[0], hi[1], hi[2], hi[3]);
        ql[t][h][w] = (int)pack4(lo[0], lo[1], lo[2], lo[3]);
      }
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

  float vlog_l = 0.0f, vinv_l = 0.0f;
  for (int i = 0; i < count; ++i) {
    const int j = i & 63;
    if (j == 0) {  // the values' scales as they go into weights and total
      vlog_l = scales_l.y == 0.0f ? kZeroLog2 : __log2f(scales_l.y);
      vinv_l = scales_l.y == 0.0f ? kZeroInv : 1.0f / scales_l.y;
    }
    const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scales_l.x), j));
    const float vlog = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vlog_l), j));
    const float vinv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vinv_l), j));
    const bool held = page >= 0;
    if (j == 63) {
      fetch_pages(i + 1);
      fetch_scales();
    }
    const int next = i + 1 < count ? __builtin_amdgcn_readlane(page_l, (i + 1) & 63) : -1;
    const int key0 = (p_first + KW * i) * kBlock;

    // ---- scores: the high digits' sum, times 256, plus the low digits'
    v4i sc[R][4];
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v4i x = mfma16(as_v4i(kr[u][0]), qh[t][0], v4i{0, 0, 0, 0});
        x = mfma16(as_v4i(kr[u][1]), qh[t][1], x);
        x = x << 8;
        x = mfma16(as_v4i(kr[u][0]), ql[t][0], x);
        sc[t][u] = mfma16(as_v4i(kr[u][1]), ql[t][1], x);
      }
    load_keys(next);

    // ---- weights
    f16x8 pw[R][2];
#pragma unroll
    for (int t = 0; t < R; ++t) {
      float x[16];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[4 * u + r] = (float)sc[t][u][r];
      // base-2 factor of the scores, above 0 so that a masked -inf stays -inf
      float f = row_scale[t] * ks, vl = vlog, vi = vinv;
      f = f < 0x1p-126f ? 0x1p-126f : f;
      const int lim = held ? last_key[t] - key0 - 16 * g : INT_MIN;  // tokens of this lane past it are not seen
      if (__any(lim < 15)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = e <= lim ? x[e] : -INFINITY;
        if (lim < 0) {  // nothing of the block is seen, whatever its scales hold
          f = 1.0f;
          vl = vi = 0.0f;
        }
      }
      float top = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
      top = fold_groups(fmaf(top, f, vl), [](float p, float r) { return fmaxf(p, r); });
      if (__any(top > m[t])) {
        const float mn = fmaxf(m[t], top);
        const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[t] - mn);
        m[t] = mn;
        l[t] *= alpha;
#pragma unroll
        for (int d = 0; d < 8; ++d) acc[t][d] *= alpha;
      }
      const float off = vl + kWeightShift - (m[t] == -INFINITY ? 0.0f : m[t]);
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], f, off));
        sum += x[e];
      }
      l[t] = fmaf(sum, vi, l[t]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        pw[t][h] = __builtin_bit_cast(f16x8, make_uint4(f16x2_bits(x[8 * h], x[8 * h + 1]), f16x2_bits(x[8 * h + 2], x[8 * h + 3]),
                                                        f16x2_bits(x[8 * h + 4], x[8 * h + 5]), f16x2_bits(x[8 * h + 6], x[8 * h + 7])));
    }

    // ---- O^T += V^T P^T
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const f16x8 v0 = codes_to_f16x8(vr[d].x, vr[d].y), v1 = codes_to_f16x8(vr[d].z, vr[d].w);
#pragma unroll
      for (int t = 0; t < R; ++t) {
        acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pw[t][0], acc[t][d], 0, 0, 0);
        acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pw[t][1], acc[t][d], 0, 0, 0);
      }
    }
    load_values(next);
    page = next;
  }
#pragma unroll
  for (int t = 0; t < R; ++t) l[t] = fold_groups(l[t], [](float p, float r) { return p + r; });

  // Where a row's result goes: its partial sums, or the output.
  auto write8 = [&](int row, int d, const float (&o)[8], float mx, float lsum) {
    const int64_t tok = s.row0 + row / G;
    const int h = hk * G + row % G;
    if (a.S > 1) {
      const int64_t at = ((int64_t)split * cb.T + tok) * a.H + h;
      float* po = a.part_o + at * kD + d;
      *reinterpret_cast<float4*>(po) = make_float4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<float4*>(po + 4) = make_float4(o[4], o[5], o[6], o[7]);
      if (d == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(mx, lsum);
    } else {
      const float inv = lsum > 0.0f ? 1.0f / lsum : lsum;  // a row that sees nothing is 0 (0 * 0), NaN stays
      *reinterpret_cast<uint4*>(a.o.p + tok * a.o.row + h * a.o.head + d) =
          make_uint4(bf16x2_bits(o[0] * inv, o[1] * inv), bf16x2_bits(o[2] * inv, o[3] * inv),
                     bf16x2_bits(o[4] * inv, o[5] * inv), bf16x2_bits(o[6] * inv, o[7] * inv));
    }
  };

  if constexpr (KW > 1) {
    // the KW waves' partial results of the same rows meet in LDS
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const int r = wave * kWaveRows + 16 * t + l16;
#pragma unroll
      for (int d = 0; d < 8; ++d)
        *reinterpret_cast<float4*>(&l_o[r * kPitch + 16 * d + 4 * g]) = make_float4(acc[t][d][0], acc[t][d][1], acc[t][d][2], acc[t][d][3]);
      if (g == 0) l_ml[r] = make_float2(m[t], l[t]);
    }
    lds_barrier();
    for (int i = tid; i < kRows * 16; i += kAttnWaves * 64) {
      const int r = i >> 4, d = (i & 15) * 8, row = s.item * kRows + r;
      if (row >= n_rows) continue;
      const int first = r / kWaveRows * KW * kWaveRows + r % kWaveRows;  // the row in the first of its waves
      float mx = -INFINITY, lsum = 0.0f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KW; ++w) mx = fmaxf(mx, l_ml[first + w * kWaveRows].x);
      const float base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float2 ml = l_ml[first + w * kWaveRows];
        const float f = __builtin_amdgcn_exp2f(ml.x - base);
        lsum = fmaf(ml.y, f, lsum);
        const float* p = &l_o[(first + w * kWaveRows) * kPitch + d];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(p[e], f, o[e]);
      }
      write8(row, d, o, mx, lsum);
    }
  } else {
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const int row = row0 + 16 * t + l16;
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
// (token, head), each folding every P-th split, their results meeting in LDS.
// (One thread for all of 64 splits took 36 us of the 79 that one token over
// 100000 took: its reads wait for each other.)  Tokens of no sequence are
// left as they are.
template <int P>
__global__ __launch_bounds__(256) void cache_attention_merge(const CacheAttnArgs a) {
  constexpr int kChunks = kD / 8, kRowsHere = 256 / (kChunks * P);
  __shared__ float l_part[P > 1 ? 256 * 11 : 1];  // a thread's maximum, total and 8 sums
  const int tid = threadIdx.x, c = tid % kChunks, part = tid / kChunks % P;
  const int64_t row = (int64_t)blockIdx.x * kRowsHere + tid / (kChunks * P), rows = (int64_t)a.c.T * a.H;
  const int64_t tok = row / a.H;
  const bool ok = row < rows && tok >= a.c.starts[0] && tok < a.c.starts[a.c.B];
  float mx = -INFINITY, lsum = 0.0f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto fold = [&](float m2, float l2, const float* w) {  // one more partial result
    const float top = fmaxf(mx, m2), base = top == -INFINITY ? 0.0f : top;
    const float f0 = __builtin_amdgcn_exp2f(mx - base), f1 = __builtin_amdgcn_exp2f(m2 - base);
    lsum = lsum * f0 + l2 * f1;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = o[e] * f0 + w[e] * f1;
    mx = top;
  };
  if (ok)
    for (int s = part; s < a.S; s += P) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (s * rows + row) * 2);
      const float4* p = reinterpret_cast<const float4*>(a.part_o + (s * rows + row) * kD + 8 * c);
      const float4 u = p[0], v = p[1];
      const float w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
      fold(ml.x, ml.y, w);
    }
  if constexpr (P > 1) {
    float* mine = l_part + tid * 11;
    mine[0] = mx;
    mine[1] = lsum;
#pragma unroll
    for (int e = 0; e < 8; ++e) mine[2 + e] = o[e];
    lds_barrier();
    if (part != 0) return;
    for (int q = 1; q < P; ++q) {
      const float* p = mine + q * kChunks * 11;
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = p[2 + e];
      fold(p[0], p[1], w);
    }
  }
  if (!ok) return;
  const float inv = lsum > 0.0f ? 1.0f / lsum : lsum;
  *reinterpret_cast<uint4*>(a.o.p + tok * a.o.row + (row % a.H) * a.o.head + 8 * c) =
      make_uint4(bf16x2_bits(o[0] * inv, o[1] * inv), bf16x2_bits(o[2] * inv, o[3] * inv),
                 bf16x2_bits(o[4] * inv, o[5] * inv), bf16x2_bits(o[6] * inv, o[7] * inv));
}

// The form of a call: row tiles a wave, waves that share rows, the
// workgroup's rows, the most row blocks that the batch can have, and the
// splits of the blocks.
struct AttnPlan {
  int R, KW, rows;
  int64_t tiles;
  int S;
};

constexpr int kPlanLeast = 4, kPlanWgs = 512;
AttnPlan plan_attention(int B, int T, int H, int Hkv, int max_len) {
  AttnPlan p;
  const int64_t G = H / Hkv, all = (int64_t)T * G, mean = (all + B - 1) / B;
  p.R = mean <= 16 ? 1 : 2;
  p.KW = mean <= 32 ? 4 : mean <= 64 ? 2 : 1;
  p.rows = kAttnWaves / p.KW * 16 * p.R;
  // every sequence's last row block may be partial, but each has a row
  p.tiles = std::min<int64_t>(all / p.rows + B, T * ((G + p.rows - 1) / p.rows));
  const int64_t blocks = (max_len + kBlock - 1) / kBlock, items = std::max<int64_t>(p.tiles * Hkv, 1);
  const int64_t least = kPlanLeast;  // blocks of a split
  p.S = (int)std::max<int64_t>(1, std::min<int64_t>({(kPlanWgs + items - 1) / items, blocks / least, 64}));
  return p;
}

}  // namespace

hipError_t launch_cache_append(const CacheAppendArgs& a, hipStream_t stream) {
  if (a.c.T == 0 || a.c.B == 0) return hipSuccess;
  // touched blocks: (n + 126) / 64 of a sequence with n new tokens at most, and no more than its tokens
  const int64_t most = std::min<int64_t>(a.c.T, ((int64_t)a.c.T + 126ll * std::min(a.c.B, a.c.T)) / kBlock);
  cache_append<<<dim3((unsigned)most, (unsigned)a.c.Hkv, 2), dim3(kAppendThreads), 0, stream>>>(a);
  return hipGetLastError();
}

size_t cache_attention_workspace(int B, int T, int H, int Hkv, int max_len) {
  const AttnPlan p = plan_attention(B, T, H, Hkv, max_len);
  return p.S > 1 ? kCounterRegionBytes + (size_t)p.S * T * H * (kD + 2) * sizeof(float) : 0;
}

hipError_t launch_cache_attention(const CacheAttnArgs& a0, hipStream_t stream) {
  if (a0.c.T == 0 || a0.c.B == 0) return hipSuccess;
  CacheAttnArgs a = a0;
  const AttnPlan p = plan_attention(a.c.B, a.c.T, a.H, a.c.Hkv, a.max_len);
  a.G = a.H / a.c.Hkv;
  a.S = p.S;
  if (a.S > 1) {
    a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + kCounterRegionBytes);
    a.part_ml = a.part_o + (size_t)a.S * a.c.T * a.H * kD;
  }
  const int64_t grid = p.tiles * a.c.Hkv * a.S;
  if (grid > kMaxGrid) return hipErrorInvalidValue;
  typedef void (*Fn)(const CacheAttnArgs);
  const Fn k = p.R == 1 ? (Fn)cache_attention<1, 4>
               : p.KW == 4 ? (Fn)cache_attention<2, 4>
               : p.KW == 2 ? (Fn)cache_attention<2, 2>
                           : (Fn)cache_attention<2, 1>;
  k<<<dim3((unsigned)grid), dim3(kAttnWaves * 64), 0, stream>>>(a);
  if (a.S > 1) {
    const int64_t threads = (int64_t)a.c.T * a.H * (kD / 8);
    if (a.S <= 4)
      cache_attention_merge<1><<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream>>>(a);
    else
      cache_attention_merge<16><<<dim3((unsigned)(threads / 16)), dim3(256), 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace w4a8
