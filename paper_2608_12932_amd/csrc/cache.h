// Launch interface of the 8-bit key/value cache (cache.hip: its append and
// the attention that reads it) for the C ABI (api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace w4a8 {

constexpr int kCacheD = 128;      // head dimension
constexpr int kCacheBlock = 64;   // tokens of a block, one page of the table
constexpr int kCacheRecent = 128; // tokens of a sequence's ring of exact values: two blocks

// Rows of the new tokens, [T][heads][128] with any row and head stride.
struct TokenRows {
  uint16_t* p;
  int64_t row, head;  // strides in elements, multiples of 8
};

// The batch and the cache, as both calls are given them.  Rows starts[b] ..
// starts[b + 1] are the new tokens of sequence b, the last of the lengths[b]
// that it holds; its block i is page table[b][i].
struct CacheBatch {
  int8_t* k_codes;        // [n_pages][Hkv][64][128]
  int8_t* v_codes;        // [n_pages][Hkv][128][64]
  float* scales;          // [n_pages][Hkv][2]: keys', values'
  int64_t n_pages;
  const int32_t* starts;  // [B + 1]
  const int32_t* lengths; // [B]
  const int32_t* table;   // [B][max_blocks]
  int max_blocks;
  int B, T, Hkv;
  const int32_t* pos;     // [T]
  const float* rope_cos;  // [n_pos][64]
  const float* rope_sin;
  int n_pos;
};

struct CacheAppendArgs {
  CacheBatch c;
  TokenRows k, v;
  uint16_t* k_recent;     // bf16 [n_slots][Hkv][128][128]
  uint16_t* v_recent;
  int64_t n_slots;
  const int32_t* slots;   // [B], or nullptr: sequence b has slot b
};
hipError_t launch_cache_append(const CacheAppendArgs& a, hipStream_t stream);

// Division of numbers 0 <= n < 2^31 by a fixed d >= 1 as a product: with
// l = ceil(log2 d), m = ceil(2^(31 + l) / d) < 2^32 exceeds the quotient by less
// than 1, so n m / 2^(31 + l) exceeds n / d by less than 2^-l <= 1 / d.
struct Divisor {
  uint32_t d = 1, m = 0, shift = 0;
  Divisor() = default;
  explicit Divisor(uint32_t by) : d(by) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < by) ++l;
    if (by > 1) {
      m = (uint32_t)(((uint64_t(1) << (31 + l)) + by - 1) / by);
      shift = l - 1;
    }
  }
  __host__ __device__ int divide(int n) const {
    return d == 1 ? n : (int)((uint32_t)(((uint64_t)(uint32_t)n * m) >> 32) >> shift);
  }
};

struct CacheAttnArgs {
  CacheBatch c;
  TokenRows q, o;
  int H, G;               // query heads, and how many share a kv head
  float scale_log2e;      // |score scale| times log2(e)
  float q_sign;           // the scale's sign, 0 for a scale of 0
  int max_len;            // the longest sequence, for the choice of splits alone
  // set by the launcher
  int S;                  // splits of a sequence's blocks
  float inv_g;            // 1 / G
  Divisor by_g, by_s;
  float* part_o;          // [S][T][H][128] unnormalized partial sums
  float* part_ml;         // [S][T][H][2] running maximum (base 2) and weight total
};
// false: the workspace is none for this call, and nothing was launched
bool launch_cache_attention(const CacheAttnArgs& a, void* workspace, size_t bytes, hipStream_t stream, hipError_t& error);
size_t cache_attention_workspace(int B, int T, int H, int Hkv, int max_len);
bool cache_attention_fits(int T, int H, int Hkv);  // one launch takes the work

}  // namespace w4a8
