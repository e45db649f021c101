// What stands between the fused QKV projection and the cache: RMSNorm of each
// query and key head and its rotation, at positions of one axis or several, in
// one pass.  Per head x of 128:
//     r = 1 / sqrt(sum x^2 / 128 + eps),  h = (x r) gamma
//     y_d = h_d cos_d - h_{d+64} sin_d,  y_{d+64} = h_{d+64} cos_d + h_d sin_d,
// cos_d = cos[p][d] with p the token's position in the axis of pair d; all in
// fp32, rounded once, to bf16.
#include <algorithm>

#include "cache4.h"
#include "device.h"

namespace w4a8 {

namespace {

constexpr int kD = kCacheD, kHalf = kD / 2;
constexpr int kSlots = 8;  // heads of a wave at a time: 8 lanes to a head, chunks c and c + 8 of it a lane

__device__ __forceinline__ int clamped(int p, int n_pos) { return p < 0 ? 0 : (p >= n_pos ? n_pos - 1 : p); }

// A wave takes 8 U heads of one token, so that a lane's eight pairs of the
// tables are read once for U heads.
template <int U>
__global__ __launch_bounds__(256) void qk_norm_rope(const QkNormRopeArgs a) {
  const int tid = threadIdx.x, c = tid & 7, slot = (tid >> 3) & 7;
  const int64_t t = (int64_t)blockIdx.x * 4 + (tid >> 6);
  if (t >= a.T) return;
  const int n = a.q.n + a.k.n, base = blockIdx.y * (kSlots * U) + slot;

  uint4 lo[U], hi[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = min(base + kSlots * u, n - 1);  // (past the last head: that one again)
    const bool k = h >= a.q.n;
    const uint16_t* src = (k ? a.k.x.p : a.q.x.p) + t * (k ? a.k.x.row : a.q.x.row) + (h - (k ? a.q.n : 0)) * (k ? a.k.x.head : a.q.x.head);
    lo[u] = *reinterpret_cast<const uint4*>(src + 8 * c);
    hi[u] = *reinterpret_cast<const uint4*>(src + kHalf + 8 * c);
  }

  float cs[8], sn[8];
  if (a.pos) {
    auto position = [&](int x) { return x < a.axes ? clamped(a.pos[(int64_t)x * a.T + t], a.n_pos) : 0; };
    const int p0 = position(0), p1 = position(1), p2 = position(2), p3 = position(3);
    const uint32_t b0 = (uint32_t)(a.axis_lo >> (8 * c)), b1 = (uint32_t)(a.axis_hi >> (8 * c));
    auto at = [&](int e) {  // of pair 8 c + e
      const int x = (b1 >> e) & 1 ? ((b0 >> e) & 1 ? p3 : p2) : ((b0 >> e) & 1 ? p1 : p0);
      return (int64_t)x * kHalf + 8 * c + e;
    };
    if (a.whole) {
      const int64_t i = at(0);
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        *reinterpret_cast<float4*>(cs + e) = *reinterpret_cast<const float4*>(a.rope_cos + i + e);
        *reinterpret_cast<float4*>(sn + e) = *reinterpret_cast<const float4*>(a.rope_sin + i + e);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int64_t i = at(e);
        cs[e] = a.rope_cos[i];
        sn[e] = a.rope_sin[i];
      }
    }
  }

#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = base + kSlots * u;
    const bool k = h >= a.q.n;
    const uint32_t lw[4] = {lo[u].x, lo[u].y, lo[u].z, lo[u].w}, hw[4] = {hi[u].x, hi[u].y, hi[u].z, hi[u].w};
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = (e & 1) ? bf16_hi(lw[e / 2]) : bf16_lo(lw[e / 2]);
      y[e] = (e & 1) ? bf16_hi(hw[e / 2]) : bf16_lo(hw[e / 2]);
    }
    const uint16_t* gamma = k ? a.k.gamma : a.q.gamma;
    if (gamma) {  // (both heads' kinds may share a wave, of which one has no norm)
      float ss = 0.0f;  // of x^2 / 128, which is finite where the mean is
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e] * (1.0f / kD), x[e], fmaf(y[e] * (1.0f / kD), y[e], ss));
      auto add = [&](auto ctrl) { ss += __uint_as_float(lane_move<decltype(ctrl)::value>(__float_as_uint(ss))); };
      add(std::integral_constant<int, kXor1>{});  // over the head's 8 lanes
      add(std::integral_constant<int, kXor2>{});
      add(std::integral_constant<int, kMirror8>{});
      const float r = 1.0f / sqrtf(ss + a.eps);
      const uint4 g0 = *reinterpret_cast<const uint4*>(gamma + 8 * c), g1 = *reinterpret_cast<const uint4*>(gamma + kHalf + 8 * c);
      const uint32_t w0[4] = {g0.x, g0.y, g0.z, g0.w}, w1[4] = {g1.x, g1.y, g1.z, g1.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = x[e] * r * ((e & 1) ? bf16_hi(w0[e / 2]) : bf16_lo(w0[e / 2]));
        y[e] = y[e] * r * ((e & 1) ? bf16_hi(w1[e / 2]) : bf16_lo(w1[e / 2]));
      }
    }
    if (a.pos) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = x[e], q = y[e];
        x[e] = p * cs[e] - q * sn[e];
        y[e] = q * cs[e] + p * sn[e];
      }
    }
    if (h < n) {
      uint16_t* dst = (k ? a.k.out.p : a.q.out.p) + t * (k ? a.k.out.row : a.q.out.row) + (h - (k ? a.q.n : 0)) * (k ? a.k.out.head : a.q.out.head);
      *reinterpret_cast<uint4*>(dst + 8 * c) =
          make_uint4(bf16x2_bits(x[0], x[1]), bf16x2_bits(x[2], x[3]), bf16x2_bits(x[4], x[5]), bf16x2_bits(x[6], x[7]));
      *reinterpret_cast<uint4*>(dst + kHalf + 8 * c) =
          make_uint4(bf16x2_bits(y[0], y[1]), bf16x2_bits(y[2], y[3]), bf16x2_bits(y[4], y[5]), bf16x2_bits(y[6], y[7]));
    }
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkNormRopeArgs& a, hipStream_t stream) {
  const int groups = (a.q.n + a.k.n + kSlots - 1) / kSlots;  // of eight heads
  typedef void (*Fn)(const QkNormRopeArgs);
  constexpr Fn kFns[] = {qk_norm_rope<1>, qk_norm_rope<2>, qk_norm_rope<3>, qk_norm_rope<4>, qk_norm_rope<5>};
  // one token's tables serve as many heads as a wave takes, once there are waves enough
  int U = 1;
  if ((int64_t)a.T * groups > 4096)
    for (int u = 2; u <= 5; ++u)
      if ((groups + u - 1) / u * u <= (groups + U - 1) / U * U || U == 1) U = u;
  kFns[U - 1]<<<dim3((unsigned)((a.T + 3) / 4), (unsigned)((groups + U - 1) / U)), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace w4a8
