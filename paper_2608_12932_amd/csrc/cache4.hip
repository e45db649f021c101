// The 4-bit key/value cache: appending to it, reading it back and attending
// over it.
//
// A sequence's cache is a list of blocks of 64 tokens, each a page of a pool
// (the table names them).  Each token's keys and values of a kv head are held
// by themselves, in two groups of 64 elements with an fp16 scale s and offset b:
//     s = fp16((hi - lo) / 15),  b = fp16(lo - 16 s),
//     code = min(max(round_half_even((x - b) / s - 16), 0), 15)  (0 where s = 0),
// and stand for fp16(s (16 + code) + b).  A token's codes depend on nothing but
// the token, so an append writes its tokens' codes and leaves all others.
//
// The sum 16 + code is what four bits in the mantissa of 16.0 in fp16 are, so a
// value takes one masked insertion and one multiply-add in fp16, two at a time.
#include <algorithm>
#include <climits>

#include "cache4.h"
#include "cache_device.h"
#include "kernels.h"

namespace w4a8 {

namespace {

constexpr int kD = kCacheD, kBlock = kCacheBlock;
constexpr int kCodeBytes = kBlock * kD / 2, kCodeWords = kCodeBytes / 4;  // one head's codes of a page, keys or values
constexpr int kParams = 4 * kBlock, kParamBytes = 2 * kParams;            // and its scales and offsets
constexpr float kClamp = 16384.0f;  // 16 s and b stay within fp16 up to here

__device__ __forceinline__ f16x2 as_f16x2(uint32_t u) { return __builtin_bit_cast(f16x2, u); }

// Eight values from a word: element 2 i in bits 4 i .., element 2 i + 1 in bits
// 16 + 4 i ..; s[i] and b[i] are the scales and offsets of elements 2 i, 2 i + 1.
__device__ __forceinline__ f16x8 values8(uint32_t w, const f16x2 (&s)[4], const f16x2 (&b)[4]) {
  uint32_t mask = 0x03C003C0u, sixteen = 0x4C004C00u;
  asm("" : "+s"(mask));  // in registers: as literals they cannot share the instruction that masks and inserts
  asm("" : "+v"(sixteen));
  const uint32_t f[4] = {((w << 6) & mask) | sixteen, ((w << 2) & mask) | sixteen, ((w >> 2) & mask) | sixteen,
                         ((w >> 6) & mask) | sixteen};
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(as_f16x2(f[0]), s[0], b[0]));
  r.y = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(as_f16x2(f[1]), s[1], b[1]));
  r.z = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(as_f16x2(f[2]), s[2], b[2]));
  r.w = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(as_f16x2(f[3]), s[3], b[3]));
  return __builtin_bit_cast(f16x8, r);
}
// Eight keys: a word of one token, whose scale and offset are the halves of sb.
__device__ __forceinline__ f16x8 keys8(uint32_t w, uint32_t sb) {
  const f16x2 p = as_f16x2(sb), s2 = {p[0], p[0]}, b2 = {p[1], p[1]};
  const f16x2 s[4] = {s2, s2, s2, s2}, b[4] = {b2, b2, b2, b2};
  return values8(w, s, b);
}
// A value of eight tokens.
__device__ __forceinline__ f16x8 values8(uint32_t w, const uint4& s4, const uint4& b4) {
  const f16x2 s[4] = {as_f16x2(s4.x), as_f16x2(s4.y), as_f16x2(s4.z), as_f16x2(s4.w)};
  const f16x2 b[4] = {as_f16x2(b4.x), as_f16x2(b4.y), as_f16x2(b4.z), as_f16x2(b4.w)};
  return values8(w, s, b);
}
__device__ __forceinline__ int nibble(int e) { return 4 * (e >> 1) + 16 * (e & 1); }  // bits of element e

// The aligned groups of Size tokens that a sequence's last n tokens touch: the
// items of append (eight tokens, those of a word of values) and read (blocks).
constexpr int kEight = 8;
template <int Size>
__device__ __forceinline__ int touched(int n, int len) {
  return n > 0 && len > 0 ? (len - 1) / Size - max(len - n, 0) / Size + 1 : 0;
}

// ---- append

constexpr int64_t kResident = 256 * 8;  // workgroups of 256 threads that the chip holds

// One workgroup per (eight tokens, N kv heads): half of its threads take the
// keys, half the values, 16 threads to a token, with the loads of all N heads in
// flight together.  Bound by a chain of reads (batch, page, words) and, with many
// tokens, by the vector unit beside it: 16 single tokens of 8 heads 3.5 us, 3288
// tokens 8.9 (17 MB; 9.6 with one head a workgroup, 10.3 with four; 11.3 with
// whole divisions).
template <int N>
__global__ __launch_bounds__(256) void cache4_append(const Cache4RowsArgs a) {
  constexpr int kPitch = kD + 4;  // bytes of a token's codes in LDS, off the banks' period
  __shared__ __align__(16) uint8_t l_codes[N][kEight * kPitch];
  const Cache4Batch& cb = a.c;
  const int tid = threadIdx.x & 127, h0 = blockIdx.y * N;
  const bool keys = __builtin_amdgcn_readfirstlane(threadIdx.x >> 7) == 0;
  const Sequence s = find_sequence(cb, blockIdx.x, [](int n, int len) { return touched<kEight>(n, len); });
  if (s.b < 0) return;
  const int first = max(s.len - s.n, 0);  // the first new token that has a place
  const int t8 = first / kEight + s.item, page = cb.table[(int64_t)s.b * cb.max_blocks + t8 / (kBlock / kEight)];
  const int c = tid & 15, t = t8 * kEight + (tid >> 4), at = t & (kBlock - 1);
  const bool there = t >= first && t < s.len, held = page >= 0 && page < cb.n_pages;

  // ---- the token's eight elements of each head; one outside the call takes its
  // last, one past the heads the last of them
  const TokenRows rows = keys ? a.k : a.v;
  const int64_t row = s.row0 + (there ? t - (s.len - s.n) : s.n - 1);
  uint4 x4[N];
#pragma unroll
  for (int u = 0; u < N; ++u)
    x4[u] = *reinterpret_cast<const uint4*>(rows.p + row * rows.row + min(h0 + u, cb.Hkv - 1) * rows.head + 8 * c);
  // values: a thread turns eight tokens' codes of one d into a word
  auto head_of = [&](int u) { return (int64_t)(held ? page : 0) * cb.Hkv + min(h0 + u, cb.Hkv - 1); };
  auto word_of = [&](int u) { return cb.v_codes + head_of(u) * kCodeWords + (t8 & 7) * kD + tid; };
  uint32_t mask = 0, old[N];  // the new tokens' bits, and what else the words hold
#pragma unroll
  for (int e = 0; e < kEight; ++e) mask |= t8 * kEight + e >= first && t8 * kEight + e < s.len ? 15u << nibble(e) : 0u;
#pragma unroll
  for (int u = 0; u < N; ++u) old[u] = !keys && held && mask != ~0u ? *word_of(u) & ~mask : 0u;

#pragma unroll
  for (int u = 0; u < N; ++u) {
    const uint32_t xw[4] = {x4[u].x, x4[u].y, x4[u].z, x4[u].w};
    float x[8], lo, hi;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = (e & 1) ? bf16_hi(xw[e / 2]) : bf16_lo(xw[e / 2]);
      x[e] = v != v ? 0.0f : fminf(fmaxf(v, -kClamp), kClamp);
      lo = e ? fminf(lo, x[e]) : x[e];
      hi = e ? fmaxf(hi, x[e]) : x[e];
    }
    auto fold = [&](auto ctrl) {  // over the group's 8 lanes
      lo = fminf(lo, __uint_as_float(lane_move<decltype(ctrl)::value>(__float_as_uint(lo))));
      hi = fmaxf(hi, __uint_as_float(lane_move<decltype(ctrl)::value>(__float_as_uint(hi))));
    };
    fold(std::integral_constant<int, kXor1>{});
    fold(std::integral_constant<int, kXor2>{});
    fold(std::integral_constant<int, kMirror8>{});
    const _Float16 s16 = (_Float16)((hi - lo) / 15.0f);
    const float sf = (float)s16;
    const _Float16 b16 = (_Float16)(lo - 16.0f * sf);  // (16 s is exact, so a fused difference is the same)
    const float bf = (float)b16;
    // The quotient by one product and a correction (Markstein's step): q = a y with
    // y = 1 / s rounded is off by at most 1.5 ulp, the residual a - s q is exact
    // (some 12 bits), and q + (a - s q) y lies within 1.5 2^-24 ulp of a / s; that
    // is never so close to a midpoint of two fp32 numbers (a has 24 bits and s
    // 11: 2^-12 ulp at least), so that it rounds to the quotient itself.
    const float safe = sf > 0.0f ? sf : 1.0f, y = 1.0f / safe;
    uint32_t code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = x[e] - bf, q = a * y;
      const float r = fmaf(fmaf(-safe, q, a), y, q);
      code[e] = sf > 0.0f ? (uint32_t)fminf(fmaxf(rintf(r - 16.0f), 0.0f), 15.0f) : 0u;
    }
    const uint32_t s_bits = __builtin_bit_cast(uint16_t, s16), b_bits = __builtin_bit_cast(uint16_t, b16);
    const bool write = held && there && h0 + u < cb.Hkv;
    if (keys) {
      uint32_t w = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) w |= code[e] << nibble(e);
      if (write) cb.k_codes[head_of(u) * kCodeWords + ((at & 3) * 16 + (at >> 2)) * 16 + c] = w;
      if (write && (c & 7) == 0)
        reinterpret_cast<uint32_t*>(cb.k_params)[head_of(u) * (kParams / 2) + (c >> 3) * kBlock + at] = s_bits | b_bits << 16;
    } else {
      uint32_t* l = reinterpret_cast<uint32_t*>(l_codes[u] + (tid >> 4) * kPitch) + 2 * c;
      l[0] = code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24;
      l[1] = code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24;
      if (write && (c & 7) == 0) {
        uint16_t* p = cb.v_params + head_of(u) * kParams + (c >> 3) * (2 * kBlock) + at;
        p[0] = (uint16_t)s_bits;
        p[kBlock] = (uint16_t)b_bits;
      }
    }
  }
  lds_barrier();
  if (keys || !held) return;
  const int d = 8 * (tid >> 2 & 15) + 4 * (tid >> 6) + (tid & 3);
#pragma unroll
  for (int u = 0; u < N; ++u) {
    if (h0 + u >= cb.Hkv) break;
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < kEight; ++e) w |= (uint32_t)l_codes[u][e * kPitch + d] << nibble(e);
    *word_of(u) = old[u] | (w & mask);
  }
}

// ---- read

// One workgroup per (block, kv head): half of its threads take the keys, half
// the values, eight elements of eight tokens each: a word of either is eight
// tokens' (values) or one token's (keys).  So every code is read once, and a
// thread has all of its loads in flight together.
__global__ __launch_bounds__(256) void cache4_read(const Cache4RowsArgs a) {
  const Cache4Batch& cb = a.c;
  const int tid = threadIdx.x & 127, hk = blockIdx.y;
  const bool keys = __builtin_amdgcn_readfirstlane(threadIdx.x >> 7) == 0;
  const TokenRows rows = keys ? a.k : a.v;
  if (!rows.p) return;
  const Sequence s = find_sequence(cb, blockIdx.x, [](int n, int len) { return touched<kBlock>(n, len); });
  if (s.b < 0) return;
  const int first = max(s.len - s.n, 0), blk = first / kBlock + s.item;
  const int page = cb.table[(int64_t)s.b * cb.max_blocks + blk];
  const int c = tid & 15, t8 = tid >> 4, t0 = blk * kBlock + t8 * kEight;
  const bool held = page >= 0 && page < cb.n_pages;
  const int64_t head = (int64_t)(held ? page : 0) * cb.Hkv + hk;
  uint32_t out[8][4];  // eight elements of each token, as bf16
  if (keys) {
    const uint32_t* w = cb.k_codes + head * kCodeWords + 2 * t8 * 16 + c;  // tokens 8 t8 + 4 i + j in rows 16 j + 2 t8 + i
    const uint4* p = reinterpret_cast<const uint4*>(cb.k_params + head * kParams + (c >> 3) * (2 * kBlock) + 16 * t8);
    const uint4 p0 = p[0], p1 = p[1];
    const uint32_t sb[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
    uint32_t code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) code[e] = w[((e & 3) * 16 + (e >> 2)) * 16];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const f16x8 v = keys8(code[e], sb[e]);
#pragma unroll
      for (int d = 0; d < 4; ++d) out[e][d] = bf16x2_bits((float)v[2 * d], (float)v[2 * d + 1]);
    }
  } else {
    const uint32_t* w = cb.v_codes + head * kCodeWords + t8 * kD + 4 * c;
    const uint4 w0 = *reinterpret_cast<const uint4*>(w), w1 = *reinterpret_cast<const uint4*>(w + kBlock);
    const uint4* p = reinterpret_cast<const uint4*>(cb.v_params + head * kParams + (c >> 3) * (2 * kBlock) + 8 * t8);
    const uint4 s4 = p[0], b4 = p[kBlock / 8];
    const uint32_t ww[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const f16x8 x = values8(ww[2 * d], s4, b4), y = values8(ww[2 * d + 1], s4, b4);
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e][d] = bf16x2_bits((float)x[e], (float)y[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int t = t0 + e;
    if (t < first || t >= s.len) continue;
    const uint4 v = held ? make_uint4(out[e][0], out[e][1], out[e][2], out[e][3]) : make_uint4(0u, 0u, 0u, 0u);
    stg_nt(reinterpret_cast<uint4*>(rows.p + (int64_t)(s.row0 + t - (s.len - s.n)) * rows.row + hk * rows.head + 8 * c), v);
  }
}

// ---- attention

// Weights are exp2(score - offset).  The offset is the score of the row's
// largest less 12, and follows the maximum only where that has outgrown it by
// more than 3, so that the sums are hardly ever rescaled: weights reach 2^15,
// and fp16 holds those down to 2^-14, 2^-26 of the largest, in full precision,
// smaller ones to 2^-24.
constexpr float kWeightShift = 12.0f, kSlack = 3.0f, kLog2e = 1.4426950408889634f;
// A score's exponent is one multiply-add, score factor - offset.  From here on
// its rounding to fp32 could lift it past fp16's range: there the offset is the
// rounded score itself and is subtracted from rounded scores.
constexpr float kLarge = 0x1p23f;

// One workgroup per (rows of one sequence's kv head, split of its blocks).
// A row is a (new token, query head of the kv head) pair, row i G + g; a wave
// holds R tiles of 16 rows.
//
// Per block of 64 tokens, S^T = K Q^T and O^T += V^T P^T in fp16 MFMAs of
// 16 x 16 x 32:
//   - row m of key tile u is token 4 m + u, and a lane's part of the sum over d
//     is d = 32 g .. 32 g + 31 (lane group g): 16 bytes of a token's codes,
//     all of one group;
//   - so lane group g holds the scores of tokens 16 g + 4 r + u, 16 in a row,
//     which is what P^T wants of it when V^T brings tokens 16 g + 8 h .. in its
//     step h: a word of codes a lane and row;
//   - row m of value tile t is d = 8 m + t, so that a lane's rows share a group
//     and its eight outputs are 16 bytes of a row.
//
// Of NW waves KW groups hold the same rows and take every KW-th block each,
// meeting in LDS at the end; the waves of a group hold different rows of the same
// blocks.  A group of one wave reads its operands straight from the page (a load
// instruction covers 1 KiB of keys).  A larger one turns a share of each block a
// wave into fp16 operands and hands them round through LDS, a block ahead of
// their use; operand order, 1 KiB an operand, so no access meets a bank twice.
//
// 64 single tokens over 4096: 51 us, 5.9 TB/s of cache, bound by HBM and, behind
// it, by the vector unit (384 of some 500 instructions a block turn codes into
// fp16).  1024 tokens over 8192: 145 us in a graph (0.89 PFLOP/s), 173 behind other
// kernels in a trace, bound by vector and matrix instructions, which share a
// SIMD's issue: a wave's vector instructions beside another's MFMAs take half of
// the MFMAs' time on top of their own (8 MFMAs 175 cycles, 32 multiply-adds 189,
// both together 278).  Some of the vector work is done over: each of a head's row
// blocks (32 of 128 rows there) turns the same codes into fp16.
template <int R, int KW, int NW, int AUX = kCacheDefault>
__global__ __launch_bounds__(NW * 64, 2) void cache4_attention(const Cache4AttnArgs a) {
  constexpr int kWaveRows = 16 * R, kSame = NW / KW, kRows = kSame * kWaveRows;
  constexpr bool kDirect = kSame == 1;
  constexpr int kPitch = kD + 4;     // floats of a row in the merge
  constexpr int kStage = 32 * 1024;  // a block's operands
  constexpr int kMergeBytes = KW > 1 ? NW * kWaveRows * kPitch * 4 : 0;
  static_assert(kDirect || kSame == 4 || kSame == 8, "shares of a block's 16 + 16 operands");
  __shared__ __align__(16) uint8_t lds[std::max(kDirect ? 0 : KW * 2 * kStage, kMergeBytes)];
  __shared__ float2 l_ml[KW > 1 ? NW * kWaveRows : 1];

  const Cache4Batch& cb = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int G = a.G, kw = wave / kSame, same = wave % kSame;
  // Workgroups of neighbouring kv heads go to the XCDs in turn, so that with a
  // multiple of 8 of them all of a head's row blocks find its pages in one L2 (with
  // 4 in two, with an odd number in all).
  const int hk = blockIdx.x;
  int split = blockIdx.y, item = blockIdx.z;
  if ((int)gridDim.y > a.S) {  // more row blocks than one axis of a launch holds
    item += (split / a.S) * gridDim.z;
    split %= a.S;
  }
  // Row blocks that see more go first: of a chunk the last ones.  (Nine ragged
  // sequences of up to 433 tokens over up to 764 56 -> 52 us.)
  item = (int)(gridDim.z * (gridDim.y / a.S)) - 1 - item;

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
  // the wave's blocks p_first + KW i < p_end; waves that meet at barriers make the same number of rounds
  const int p_first = p_begin + kw, rounds = max(p_end - (kDirect ? p_first : p_begin) + KW - 1, 0) / KW;

  // The page of block i, -1: none (past the split's, or out of the pool: tokens that no row sees)
  typedef const __attribute__((address_space(4))) int32_t* ConstTable;
  const ConstTable table = (ConstTable)(uintptr_t)(cb.table + (int64_t)s.b * cb.max_blocks);
  auto page_of = [&](int i) {
    const int p = p_first + KW * i;
    const int page = table[max(min(p, p_end - 1), 0)];
    return p < p_end && page >= 0 && page < cb.n_pages ? page : -1;
  };
  int page0 = page_of(0), page1 = page_of(1), page2 = page_of(2);

  // ---- this lane's rows (row l16 of each of the wave's tiles): 32 elements of
  // each, in fp16 at the row's own power of two, the largest in [2^14, 2^15), so
  // that elements down to 2^-28 of it are exact
  f16x8 qf[R][4];
  float f[R];       // a score's factor, in base-2 units
  int last_key[R];  // the last token that the row sees, -1 for a row past the end
#pragma unroll
  for (int t = 0; t < R; ++t) {
    const int x = same * kWaveRows + 16 * t + l16, row = min(x, n_rows - 1 - wg_row0), i = token_of(row);
    const uint16_t* src = a.q.p + (int64_t)(s.row0 + i) * a.q.row + (int64_t)(hk * G + wg_row0 + row - i * G) * a.q.head + 32 * g;
    uint32_t w[16], mag = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint4 v = *reinterpret_cast<const uint4*>(src + 8 * e);
      w[4 * e] = v.x;
      w[4 * e + 1] = v.y;
      w[4 * e + 2] = v.z;
      w[4 * e + 3] = v.w;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) mag = absmax_pairs(mag, w[e]);
    mag = fold_pair_max(mag);
    mag = __float_as_uint(fold_groups(__uint_as_float(mag), [](float p, float r) { return __uint_as_float(max(__float_as_uint(p), __float_as_uint(r))); }));
    const int up = min(141 - (int)(mag >> 7), 126);  // mag holds a bf16's bits
    const float to = __uint_as_float((uint32_t)(127 + up) << 23) * a.q_sign;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      qf[t][e] = __builtin_bit_cast(
          f16x8, make_uint4(f16x2_bits(bf16_lo(w[4 * e]) * to, bf16_hi(w[4 * e]) * to),
                            f16x2_bits(bf16_lo(w[4 * e + 1]) * to, bf16_hi(w[4 * e + 1]) * to),
                            f16x2_bits(bf16_lo(w[4 * e + 2]) * to, bf16_hi(w[4 * e + 2]) * to),
                            f16x2_bits(bf16_lo(w[4 * e + 3]) * to, bf16_hi(w[4 * e + 3]) * to)));
    // the row's power of two first: the scale times log2(e) may lie past fp32; above 0: a masked -inf stays
    f[t] = fmaxf(__uint_as_float((uint32_t)(127 - up) << 23) * a.scale * kLog2e, 0x1p-126f);
    last_key[t] = wg_row0 + x < n_rows ? s.len - s.n + i : -1;
  }

  // ---- a block's codes and parameters as they lie in the page
  auto bytes = [&](int page, int n) { return page < 0 ? 0u : (uint32_t)n; };  // nothing is read where there is no page
  auto rsrc = [&](const void* base, int page, int n) {
    return make_rsrc(uniform_ptr(static_cast<const uint8_t*>(base) + ((int64_t)max(page, 0) * cb.Hkv + hk) * n), bytes(page, n));
  };
  // keys: tile u's rows 1 KiB on; a token's params of this lane group's half of d, four tokens 16 bytes
  const uint32_t k_at = (uint32_t)(l16 * 64 + 16 * g), kp_at = (uint32_t)((g >> 1) * 256 + l16 * 16);
  // values: step h, half j of a lane's rows
  const uint32_t v_at = (uint32_t)(g * 1024 + l16 * 16), vp_at = (uint32_t)((l16 >> 3) * 256 + 32 * g);
  // (not direct) a wave's share of its group's blocks: of four waves each a tile of keys and a quarter of
  // the values, of eight the first four the keys, the others the values
  const bool my_keys = kSame < 8 || same < 4, my_values = kSame < 8 || same >= 4;
  const int piece = same & 3;
  struct Keys {
    uint4 codes[kDirect ? 4 : 1], params;
  };
  struct Values {
    uint4 codes[kDirect ? 4 : 1], s[kDirect ? 2 : 1], b[kDirect ? 2 : 1];
  };
  auto load_keys = [&](int page, Keys& k) {
    const __amdgpu_buffer_rsrc_t r = rsrc(cb.k_codes, page, kCodeBytes), p = rsrc(cb.k_params, page, kParamBytes);
    if constexpr (kDirect) {
      k.params = buf_load16<AUX>(p, kp_at);
#pragma unroll
      for (int u = 0; u < 4; ++u) k.codes[u] = buf_load16<AUX>(r, k_at + 1024 * u);
    } else {
      k.params.x = buf_load4<AUX>(p, kp_at + 4 * piece);
      k.codes[0] = buf_load16<AUX>(r, k_at + 1024 * piece);
    }
  };
  auto load_values = [&](int page, Values& v) {
    const __amdgpu_buffer_rsrc_t r = rsrc(cb.v_codes, page, kCodeBytes), p = rsrc(cb.v_params, page, kParamBytes);
    if constexpr (kDirect) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v.s[h] = buf_load16<AUX>(p, vp_at + 16 * h);
        v.b[h] = buf_load16<AUX>(p, vp_at + 128 + 16 * h);
        v.codes[2 * h] = buf_load16<AUX>(r, v_at + 512 * h);
        v.codes[2 * h + 1] = buf_load16<AUX>(r, v_at + 512 * h + 256);
      }
    } else {
      v.s[0] = buf_load16<AUX>(p, vp_at + 16 * (piece >> 1));
      v.b[0] = buf_load16<AUX>(p, vp_at + 128 + 16 * (piece >> 1));
      v.codes[0] = buf_load16<AUX>(r, v_at + 256 * piece);
    }
  };
  // Values of tokens that the sequence does not hold are zeros, whatever lies
  // there: their weights are 0, but 0 times infinity is not.
  auto clean = [&](uint4& x, int token0) {  // of tokens token0 ..
    uint32_t* w = &x.x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] &= (token0 + 2 * i < s.len ? 0xFFFFu : 0u) | (token0 + 2 * i + 1 < s.len ? 0xFFFF0000u : 0u);
  };
  auto key0_of = [&](int i) { return (p_first + KW * i) * kBlock; };
  auto clean_values = [&](int i, Values& v) {
    if (key0_of(i) + kBlock <= s.len) return;
#pragma unroll
    for (int h = 0; h < (kDirect ? 2 : 1); ++h) {
      const int token0 = key0_of(i) + 16 * g + 8 * (kDirect ? h : piece >> 1);
      clean(v.s[h], token0);
      clean(v.b[h], token0);
    }
  };
  auto word = [](const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; };

  // The weights' total is one more row of values, of ones: every lane of a row
  // holds it, in all four of its elements.
  f32x4 acc[R][8], total[R], sc[R][4];
  float m[R];  // the offset
  const f16x8 ones = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
  for (int t = 0; t < R; ++t) {
    m[t] = -INFINITY;
    total[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int d = 0; d < 8; ++d) acc[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // ---- the steps of a block
  // scores, from operands that `key` gives for (tile, step)
  auto score = [&](auto key) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f16x8 kf = key(u, e);
#pragma unroll
        for (int t = 0; t < R; ++t)
          sc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[t][e], e == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : sc[t][u], 0, 0, 0);
      }
  };
  // masks, the rows' largest, the offsets; token 16 g + e is element e / 4 of tile e % 4
  float x[R][16], by[R], off[R];
  auto look = [&](int i, int page) {
    const int key0 = key0_of(i);
    float top[R];
    bool all = true;
#pragma unroll
    for (int t = 0; t < R; ++t) {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][e] = sc[t][e & 3][e >> 2];
      all = all && last_key[t] >= key0 + kBlock - 1;
    }
    if (!__all(all) || page < 0) {
#pragma unroll
      for (int t = 0; t < R; ++t) {
        const int lim = page >= 0 ? last_key[t] - key0 - 16 * g : INT_MIN;  // tokens of this lane past it are not seen
#pragma unroll
        for (int e = 0; e < 16; ++e) x[t][e] = e <= lim ? x[t][e] : -INFINITY;
      }
    }
    bool outgrown = false;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      top[t] = x[t][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top[t] = fmaxf(top[t], x[t][e]);
      top[t] = fold_groups(top[t], [](float p, float r) { return fmaxf(p, r); }) * f[t];
      top[t] = fabsf(top[t]) >= kLarge ? top[t] : top[t] - kWeightShift;  // the offset that it asks for
      outgrown = outgrown || top[t] - m[t] > kSlack;
    }
    if (__any(outgrown)) {
#pragma unroll
      for (int t = 0; t < R; ++t) {
        // a row's own maximum alone moves its offset: its result does not
        // depend on the rows that share the wave
        const bool up = top[t] - m[t] > kSlack;
        const float alpha = up ? __builtin_amdgcn_exp2f(m[t] - top[t]) : 1.0f;
        m[t] = up ? top[t] : m[t];
        total[t] *= alpha;
#pragma unroll
        for (int d = 0; d < 8; ++d) acc[t][d] *= alpha;
      }
    }
    bool large = false;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      by[t] = f[t];
      off[t] = m[t] == -INFINITY ? 0.0f : -m[t];
      large = large || fabsf(off[t]) >= kLarge - 16.0f;
    }
    if (__builtin_expect(__any(large), 0)) {
#pragma unroll
      for (int t = 0; t < R; ++t) {
        const bool rounded = fabsf(off[t]) >= kLarge - 16.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[t][e] = rounded ? x[t][e] * by[t] : x[t][e];
        by[t] = rounded ? 1.0f : by[t];
      }
    }
  };
  f16x8 pw[R][2];
  auto weigh = [&] {
#pragma unroll
    for (int t = 0; t < R; ++t) {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][e] = __builtin_amdgcn_exp2f(fmaf(x[t][e], by[t], off[t]));
#pragma unroll
      for (int h = 0; h < 2; ++h)
        pw[t][h] = __builtin_bit_cast(
            f16x8, make_uint4(f16x2_bits(x[t][8 * h], x[t][8 * h + 1]), f16x2_bits(x[t][8 * h + 2], x[t][8 * h + 3]),
                              f16x2_bits(x[t][8 * h + 4], x[t][8 * h + 5]), f16x2_bits(x[t][8 * h + 6], x[t][8 * h + 7])));
    }
  };
  // O^T += V^T P^T, from operands that `value` gives for (step, tile)
  auto add = [&](auto value) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        const f16x8 vf = value(h, d);
#pragma unroll
        for (int t = 0; t < R; ++t) acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pw[t][h], acc[t][d], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < R; ++t) total[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pw[t][h], total[t], 0, 0, 0);
    }
  };

  if constexpr (kDirect) {
    // With one tile of rows a block's codes are loaded while the block before it
    // is worked on, into registers of their own: 9 KiB a wave in flight.  (With
    // two tiles those registers would cost the second wave of a SIMD: there the
    // next keys are loaded behind the scores, the next values at the end.)
    constexpr bool kAhead = R == 1;
    Keys keys[2];
    Values vals[2];
    load_keys(page0, keys[0]);
    load_values(page0, vals[0]);
    auto round = [&](int i, Keys& k, Values& v, Keys& k_next, Values& v_next) {
      const int page3 = page_of(i + 3);
      if constexpr (kAhead) {
        load_keys(page1, k_next);
        load_values(page1, v_next);
      }
      score([&](int u, int e) { return keys8(word(k.codes[u], e), word(k.params, u)); });
      if constexpr (!kAhead) load_keys(page1, k);
      look(i, page0);
      weigh();
      clean_values(i, v);
      add([&](int h, int d) { return values8(word(v.codes[2 * h + d / 4], d % 4), v.s[h], v.b[h]); });
      if constexpr (!kAhead) load_values(page1, v);
      page0 = page1;
      page1 = page2;
      page2 = page3;
    };
    int i = 0;
    if constexpr (kAhead) {
      for (; i + 1 < rounds; i += 2) {  // (a way from the first to the loop's head would make it wait for all loads)
        round(i, keys[0], vals[0], keys[1], vals[1]);
        round(i + 1, keys[1], vals[1], keys[0], vals[0]);
      }
      if (i < rounds) round(i, keys[0], vals[0], keys[1], vals[1]);
    } else {
      for (; i < rounds; ++i) round(i, keys[0], vals[0], keys[0], vals[0]);
    }
  } else {
    uint8_t* l_group = lds + kw * 2 * kStage;
    // A block's codes are loaded two rounds before they become operands, which
    // is a round before their use.
    auto stage_keys = [&](int i, const Keys& k) {  // operand (u, step) at 4 u + step
      if (!my_keys) return;
      uint8_t* dst = l_group + (i & 1) * kStage + lane * 16 + piece * 4096;
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<f16x8*>(dst + e * 1024) = keys8(word(k.codes[0], e), k.params.x);
    };
    auto stage_values = [&](int i, Values& v) {  // operand (h, d) at 16 + 8 h + d
      if (!my_values) return;
      uint8_t* dst = l_group + (i & 1) * kStage + kStage / 2 + lane * 16 + piece * 4096;
      clean_values(i, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<f16x8*>(dst + e * 1024) = values8(word(v.codes[0], e), v.s[0], v.b[0]);
    };
    auto load = [&](int page, Keys& k, Values& v) {
      if (my_keys) load_keys(page, k);
      if (my_values) load_values(page, v);
    };
    Keys k[2];
    Values v[2];
    load(page0, k[0], v[0]);
    load(page1, k[1], v[1]);
    stage_keys(0, k[0]);
    stage_values(0, v[0]);
    load(page2, k[0], v[0]);
    lds_barrier();
    int page3 = page_of(3);
    auto round = [&](int i, Keys& k, Values& v) {
      const int page4 = page_of(i + 4);
      // The next block's operands go where block i - 1's were, which were last read
      // before the barrier: its values beside this block's scores, its keys beside
      // the products with the values, vector work for either.
      stage_values(i + 1, v);
      if (my_values) load_values(page3, v);
      const uint8_t* src = l_group + (i & 1) * kStage + lane * 16;
      score([&](int u, int e) { return *reinterpret_cast<const f16x8*>(src + (4 * u + e) * 1024); });
      look(i, page0);
      weigh();
      stage_keys(i + 1, k);
      if (my_keys) load_keys(page3, k);
      add([&](int h, int d) { return *reinterpret_cast<const f16x8*>(src + (16 + 8 * h + d) * 1024); });
      lds_barrier();
      page0 = page1;
      page1 = page2;
      page2 = page3;
      page3 = page4;
    };
    int i = 0;
    for (; i + 1 < rounds; i += 2) {  // (a way from the first to the loop's head would make it wait for all loads)
      round(i, k[1], v[1]);
      round(i + 1, k[0], v[0]);
    }
    if (i < rounds) round(i, k[1], v[1]);
  }
  float l[R];
#pragma unroll
  for (int t = 0; t < R; ++t) l[t] = total[t][0] * kTotalUnit;

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
    // the partial results of the waves with the same rows meet in LDS
    if constexpr (!kDirect) lds_barrier();  // (where the stages were)
    float* l_o = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const int r = wave * kWaveRows + 16 * t + l16;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int d = 0; d < 8; d += 4)
          *reinterpret_cast<float4*>(&l_o[r * kPitch + 32 * g + 8 * e + d]) =
              make_float4(acc[t][d][e], acc[t][d + 1][e], acc[t][d + 2][e], acc[t][d + 3][e]);
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
        const float by = __builtin_amdgcn_exp2f(ml.x - base);
        lsum = fmaf(ml.y, by, lsum);
        const float* p = &l_o[(r + w * kRows) * kPitch + d];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(p[e], by, o[e]);
      }
      write8(row, d, o, mx, lsum);
    }
  } else {
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const int row = wg_row0 + same * kWaveRows + 16 * t + l16;
      if (row >= n_rows) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float o[8];
#pragma unroll
        for (int d = 0; d < 8; ++d) o[d] = acc[t][d][e];
        write8(row, 32 * g + 8 * e, o, m[t], l[t]);
      }
    }
  }
}

// The forms of a call, and what one of its workgroups costs in ns: alone on a
// CU lat + lat_round a round (a block of each of the KW groups of waves); in a
// full chip each of the ceil(workgroups / 256) that a CU runs adds thr +
// thr_round a round.  Fitted, with the merge's 3430 + 0.24 a (split, token,
// head), to 95 calls (B 1 - 64, 1 - 1024 new tokens, 60 - 90000 long, five head
// layouts) at up to 12 numbers of splits: what the rule picks is 0.2 % above the
// best of all forms and splits on average, 6 % at most.  Without the three
// shared forms the best would be 1.9 % slower on average and 39 % at most,
// without the last 0.2 % and 15 %.  64 and 128 rows in four waves (one a SIMD),
// and 16 and 32 rows in eight, tried too, took nothing off.  us of the five, at
// its best splits each, as they are now: 12 ragged sequences of up to 33 tokens
// over up to 1900 22 20 28 36 29; 256 over 4096 45 34 40 44 37; 1024 over 8192 277
// 176 162 161 145.
//   The calls were of one kind of sequence each.  A batch is taken as B
// sequences of max_len with the average number of new tokens, so one that mixes
// kinds gets the form and splits of neither, and a call for each kind is faster:
// one token each of 63 sequences of 1000 and one of 100000, 32 heads on 8: 495 us
// in one call (no splits), 17 + 28 in two; 63 single tokens beside a chunk of 1024,
// all over 8192: 313, 96 + 144.  Beside a chunk of 512 over 4096, 16 heads on 16, it
// makes no difference: 138, 99 + 37.
typedef void (*Attn4Fn)(const Cache4AttnArgs);
struct Attn4Form {
  int rows, KW, threads;
  int64_t lat, lat_round, thr, thr_round;
  Attn4Fn fn;
};
const Attn4Form kForms[] = {
    {16, 4, 256, 2420, 1140, 1200, 1030, cache4_attention<1, 4, 4>},
    {32, 4, 256, 3240, 1650, 1550, 1470, cache4_attention<2, 4, 4>},
    {128, 1, 512, 3310, 1370, 2820, 1370, cache4_attention<1, 1, 8>},
    {256, 1, 512, 3510, 1690, 4700, 2120, cache4_attention<2, 1, 8>},
    {128, 2, 512, 7240, 830, 5420, 2310, cache4_attention<2, 2, 8>},
};
constexpr int64_t kMergeCost = 3430, kMergePart = 24;  // ns, ns for 100 (split, token, head)
// Where the rows of an average sequence's kv head are one row block, pages are read
// past the caches, as each is read once: of 13 calls from 1 MB to 300 MB, on another
// cache each time (another layer's), none was slower so, and 64 sequences of 4096
// take 52 us instead of 61.  On the same cache again, of which the memory-side one
// still holds some, two from 150 MB on were (29.3 -> 31.0 us, 55 -> 60).  A longer
// chunk among single tokens reads its pages so once for each of its row blocks.
const Attn4Fn kStreamFn = cache4_attention<1, 4, 4, kCacheStream>;
constexpr int64_t kMaxAxis = 65535;  // workgroups along the second and third axis of a launch

struct Attn4Plan {
  int form = 0, S = 1;
  bool stream = false;
  int64_t tiles = 0;  // the most row blocks that the batch can have
};

Attn4Plan plan_attention(int B, int T, int H, int Hkv, int max_len) {
  const int64_t G = H / Hkv, n = (T + B - 1) / B, blocks = (max_len + kBlock - 1) / kBlock;
  const int64_t most = (int64_t)T * H <= (1 << 22) ? blocks : 1;  // splits
  constexpr int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
  Attn4Plan p;
  int64_t least = INT64_MAX;
  for (int f = 0; f < (int)(sizeof kForms / sizeof kForms[0]); ++f) {
    const Attn4Form& k = kForms[f];
    const int by_rows = __builtin_ctz(k.rows), by_kw = __builtin_ctz(k.KW);
    const int64_t tiles = B * ((n * G + k.rows - 1) >> by_rows) * Hkv;
#pragma unroll
    for (int S : kSplits) {
      if (S > 1 && S > most) break;
      const int64_t rounds = ((uint64_t)(blocks + S - 1) / S + k.KW - 1) >> by_kw;
      const int64_t cost = std::max(k.lat + rounds * k.lat_round, ((tiles * S + 255) >> 8) * (k.thr + rounds * k.thr_round)) +
                           (S > 1 ? kMergeCost + (int64_t)((uint64_t)S * T * H * kMergePart / 100) : 0);
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
  p.stream = p.form == 0 && n * G <= rows;
  return p;
}

size_t workspace_of(const Attn4Plan& p, int T, int H) {
  return p.S > 1 ? kCounterRegionBytes + (size_t)p.S * T * H * (kD + 2) * sizeof(float) : 0;
}

// Groups of `size` tokens that a batch's rows touch at most: (n + 2 size - 2) /
// size of a sequence with n rows, and no more than its rows.
unsigned most_touched(const Cache4Batch& c, int size) {
  return (unsigned)std::min<int64_t>(c.T, (c.T + (2ll * size - 2) * std::min(c.B, c.T)) / size);
}

}  // namespace

hipError_t launch_cache4_append(const Cache4RowsArgs& a, hipStream_t stream) {
  const unsigned groups = most_touched(a.c, kEight);
  constexpr int N = 2;
  if ((int64_t)groups * a.c.Hkv > kResident)  // more than one round of workgroups
    cache4_append<N><<<dim3(groups, (unsigned)(a.c.Hkv + N - 1) / N), dim3(256), 0, stream>>>(a);
  else
    cache4_append<1><<<dim3(groups, (unsigned)a.c.Hkv), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache4_read(const Cache4RowsArgs& a, hipStream_t stream) {
  cache4_read<<<dim3(most_touched(a.c, kBlock), (unsigned)a.c.Hkv), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

size_t cache4_attention_workspace(int B, int T, int H, int Hkv, int max_len) {
  return workspace_of(plan_attention(B, T, H, Hkv, max_len), T, H);
}

bool launch_cache4_attention(const Cache4AttnArgs& a0, void* workspace, size_t bytes, hipStream_t stream, hipError_t& error) {
  Cache4AttnArgs a = a0;
  const Attn4Plan p = plan_attention(a.c.B, a.c.T, a.H, a.c.Hkv, a.max_len);
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
  const Attn4Form& k = kForms[p.form];
  const unsigned z = (unsigned)std::min<int64_t>(p.tiles, kMaxAxis), y = (unsigned)((p.tiles + z - 1) / z) * (unsigned)a.S;
  (p.stream ? kStreamFn : k.fn)<<<dim3((unsigned)a.c.Hkv, y, z), dim3(k.threads), 0, stream>>>(a);
  if (a.S > 1) {
    const int P = a.S <= 16 ? 4 : 16;
    const int64_t threads = (int64_t)a.c.T * a.H * (kD / 8) * P;
    const Attn4Fn merge = P == 4 ? cache_attention_merge<4, Cache4AttnArgs> : cache_attention_merge<16, Cache4AttnArgs>;
    merge<<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream>>>(a);
  }
  error = hipGetLastError();
  return true;
}

}  // namespace w4a8
