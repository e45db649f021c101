// What stands between the fused QKV projection and the cache: RMSNorm of each
// query and key head and its rotation, at positions of one axis or several, in
// one pass.  Per head x of 128:
//     r = 1 / sqrt(sum x^2 / 128 + eps),  h = (x r) gamma
//     y_d = h_d cos_d - h_{d+64} sin_d,  y_{d+64} = h_{d+64} cos_d + h_d sin_d,
// cos_d = cos[p][d] with p the token's position in the axis of pair d; all in
// fp32, rounded once, to bf16.
#include "cache4.h"
#include "device.h"

namespace w4a8 {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kD = kCacheD, kHalf = kD / 2;
constexpr int kSlots = 8;  // heads of a wave: 8 lanes to a head, chunks c and c + 8 of it a lane

// One of two values, as a select: a conditional between variables is an lvalue,
// for which the compiler puts them into memory (16 us a call).
template <class T>
__device__ __forceinline__ T pick(bool first, T x, T y) {
  return first ? x : y;
}

// A wave takes 8 heads of one token.  Its 64 lanes look up the token's 64 pairs
// of the tables, one each, whichever axis turns it, and hand them round through
// LDS: read by every lane that needs them, eight pairs of interleaved axes are
// 16 loads a lane, which took half as long again as all the rest.
//
// Bound by HBM where there are tokens enough, else by two reads behind each
// other (positions, tables) and the launch.  8192 tokens of 40 heads (168 MB):
// 31 us, 5.4 TB/s, whether or not the last call's rows are still in the memory-
// side cache; with stores through the second-level caches 29 and 42 us, 2048
// tokens 9.2 us instead of 6.5.
__global__ __launch_bounds__(256) void qk_norm_rope(const QkNormRopeArgs a) {
  __shared__ __align__(16) float l_table[4][2][kHalf];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 7, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t = blockIdx.x * 4 + wave;
  if (t >= a.T) return;
  const int n = a.q.n + a.k.n, head = blockIdx.y * kSlots + (lane >> 3), h = min(head, n - 1);  // (past the last head: that one again)
  const bool k = h >= a.q.n;
  const int of_kind = h - (k ? a.q.n : 0);
  const uint16_t* src = pick(k, a.k.x.p, a.q.x.p) + t * pick(k, a.k.x.row, a.q.x.row) + of_kind * pick(k, a.k.x.head, a.q.x.head) + 8 * c;
  const uint4 lo = *reinterpret_cast<const uint4*>(src), hi = *reinterpret_cast<const uint4*>(src + kHalf);

  float cos_l = 0.0f, sin_l = 0.0f;  // of pair `lane`
  if (a.pos) {
    // the axes' positions, the same in all lanes; an axis too many reads the first one's, so that no load waits for another
    typedef const __attribute__((address_space(4))) int32_t* ConstPos;
    const ConstPos pos = (ConstPos)(uintptr_t)a.pos;
    auto position = [&](int x) { return min(max(pos[(x < a.axes ? x : 0) * (int64_t)a.T + t], 0), a.n_pos - 1); };
    const int p0 = position(0), p1 = position(1), p2 = position(2), p3 = position(3);
    const bool b0 = a.axis_lo >> lane & 1, b1 = a.axis_hi >> lane & 1;
    const int64_t at = (int64_t)pick(b1, pick(b0, p3, p2), pick(b0, p1, p0)) * kHalf + lane;
    cos_l = a.rope_cos[at];
    sin_l = a.rope_sin[at];
  }

  const uint32_t lw[4] = {lo.x, lo.y, lo.z, lo.w}, hw[4] = {hi.x, hi.y, hi.z, hi.w};
  float x[8], y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = (e & 1) ? bf16_hi(lw[e / 2]) : bf16_lo(lw[e / 2]);
    y[e] = (e & 1) ? bf16_hi(hw[e / 2]) : bf16_lo(hw[e / 2]);
  }
  const uint16_t* gamma = pick(k, a.k.gamma, a.q.gamma);
  if (gamma) {  // (both kinds of heads may share a wave, of which one has no norm)
    const uint4 g0 = *reinterpret_cast<const uint4*>(gamma + 8 * c), g1 = *reinterpret_cast<const uint4*>(gamma + kHalf + 8 * c);
    float ss = 0.0f;  // of x^2 / 128, which is finite where the mean is
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e] * (1.0f / kD), x[e], fmaf(y[e] * (1.0f / kD), y[e], ss));
    auto add = [&](auto ctrl) { ss += __uint_as_float(lane_move<decltype(ctrl)::value>(__float_as_uint(ss))); };
    add(std::integral_constant<int, kXor1>{});  // over the head's 8 lanes
    add(std::integral_constant<int, kXor2>{});
    add(std::integral_constant<int, kMirror8>{});
    const float r = 1.0f / sqrtf(ss + a.eps);
    const uint32_t w0[4] = {g0.x, g0.y, g0.z, g0.w}, w1[4] = {g1.x, g1.y, g1.z, g1.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = x[e] * r * ((e & 1) ? bf16_hi(w0[e / 2]) : bf16_lo(w0[e / 2]));
      y[e] = y[e] * r * ((e & 1) ? bf16_hi(w1[e / 2]) : bf16_lo(w1[e / 2]));
    }
  }
  if (a.pos) {
    l_table[wave][0][lane] = cos_l;
    l_table[wave][1][lane] = sin_l;
    wave_order();
    const f32x4* l = reinterpret_cast<const f32x4*>(&l_table[wave][0][8 * c]);
    const f32x4 cs[2] = {l[0], l[1]}, sn[2] = {l[kHalf / 4], l[kHalf / 4 + 1]};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = x[e], q = y[e], cs_e = cs[e / 4][e % 4], sn_e = sn[e / 4][e % 4];
      x[e] = p * cs_e - q * sn_e;
      y[e] = q * cs_e + p * sn_e;
    }
  }
  if (head < n) {
    uint16_t* dst = pick(k, a.k.out.p, a.q.out.p) + t * pick(k, a.k.out.row, a.q.out.row) + of_kind * pick(k, a.k.out.head, a.q.out.head) + 8 * c;
    stg_nt(reinterpret_cast<uint4*>(dst),
           make_uint4(bf16x2_bits(x[0], x[1]), bf16x2_bits(x[2], x[3]), bf16x2_bits(x[4], x[5]), bf16x2_bits(x[6], x[7])));
    stg_nt(reinterpret_cast<uint4*>(dst + kHalf),
           make_uint4(bf16x2_bits(y[0], y[1]), bf16x2_bits(y[2], y[3]), bf16x2_bits(y[4], y[5]), bf16x2_bits(y[6], y[7])));
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkNormRopeArgs& a, hipStream_t stream) {
  const int groups = (a.q.n + a.k.n + kSlots - 1) / kSlots;
  qk_norm_rope<<<dim3((unsigned)((a.T + 3) / 4), (unsigned)groups), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace w4a8
