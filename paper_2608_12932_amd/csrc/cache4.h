// Launch interface of the 4-bit key/value cache (cache4.hip: its append, the
// read and the attention over it) and of the head norms with the rotation
// (heads.hip) for the C ABI (api.cpp).
#pragma once

#include "cache.h"

namespace w4a8 {

constexpr int kCache4Group = 64;  // elements with a scale and an offset of their own

// The batch and the cache, as all three calls are given them; the batch as in
// CacheBatch.
struct Cache4Batch {
  uint32_t* k_codes;      // [n_pages][Hkv][4][16][16]: token 4 i + j in row [j][i], 8 elements a word
  uint32_t* v_codes;      // [n_pages][Hkv][8][2][16][4]: 8 tokens a word, d = 8 i + 4 j + l in [j][i][l]
  uint16_t* k_params;     // fp16 [n_pages][Hkv][2][64][2]: scale, offset of a token's group
  uint16_t* v_params;     // fp16 [n_pages][Hkv][2][2][64]: scales, then offsets of a group's tokens
  int64_t n_pages;
  const int32_t* starts;  // [B + 1]
  const int32_t* lengths; // [B]
  const int32_t* table;   // [B][max_blocks]
  int max_blocks;
  int B, T, Hkv;
};

struct Cache4RowsArgs {
  Cache4Batch c;
  TokenRows k, v;  // the append's input, the read's output (p may be nullptr there)
};
hipError_t launch_cache4_append(const Cache4RowsArgs& a, hipStream_t stream);
hipError_t launch_cache4_read(const Cache4RowsArgs& a, hipStream_t stream);

struct Cache4AttnArgs {
  Cache4Batch c;
  TokenRows q, o;
  int H, G;               // query heads, and how many share a kv head
  float scale;            // |score scale| (1 for a scale of 0)
  float q_sign;           // the scale's sign, 0 for a scale of 0
  int max_len;            // the longest sequence, for the choice of splits alone
  // set by the launcher
  int S;                  // splits of a sequence's blocks
  float inv_g;            // 1 / G
  Divisor by_g, by_s;
  float* part_o;          // [S][T][H][128] unnormalized partial sums
  float* part_ml;         // [S][T][H][2] offset (base 2) and weight total
};
// false: the workspace is none for this call, and nothing was launched
bool launch_cache4_attention(const Cache4AttnArgs& a, void* workspace, size_t bytes, hipStream_t stream, hipError_t& error);
size_t cache4_attention_workspace(int B, int T, int H, int Hkv, int max_len);

// Heads of one kind: their rows in and out, and the norm's gain (nullptr: none).
struct HeadRows {
  TokenRows x, out;
  const uint16_t* gamma;
  int n;
};
struct QkNormRopeArgs {
  HeadRows q, k;
  int T;
  float eps;
  const int32_t* pos;     // [axes][T], nullptr: no rotation
  const float* rope_cos;  // [n_pos][64]
  const float* rope_sin;
  int n_pos, axes;
  uint64_t axis_lo, axis_hi;  // bits 0 and 1 of each pair's axis
};
hipError_t launch_qk_norm_rope(const QkNormRopeArgs& a, hipStream_t stream);

}  // namespace w4a8
