// Rotary positions with several axes: pairs of a head's channels are turned by angles that a token's positions give.
//
//   y1 = x1 cos t - x2 sin t,  y2 = x2 cos t + x1 sin t,   t = position on the pair's axis * the pair's frequency
//
// The gradient is the same with -t.  Angles are taken in 64 bits as turns (t / 2 pi), of which only the fraction goes on in 32: a product
// of a position below 2^31 and a frequency of 1 is off by 2^-24 of a turn there at most, where 32 bits would lose everything from 2^24 on.
#include "internal.h"
#include "common.h"

namespace lv {

namespace {

struct RopeCall {
  const int32_t *pos;      // [n][axes]
  const uint16_t *x[2];    // q, k
  uint16_t *y[2];
  int64_t x_stride[2], y_stride[2];
  int heads, all;          // of q; of both
  int n, axes, head_dim;
  int parts, per;          // the heads are taken in so many parts of `per`
  int rotated;             // channels that are; the others are copied
  float sign;              // of the sine
};

// What a lane does with its eight channels: channel e turns with pair `pair`, its partner lies `dist` channels away (below: it is the second of
// the pair, whose first is its partner)
struct Lane {
  int pair, axis, dist;
};

// By how the channels of a pair lie: next to each other; as many apart as an axis has pairs; as many as there are in all
__device__ __forceinline__ Lane lane_of(const RopePairs &r, int c) {
  Lane l = {0, 0, 0};
  if (c >= 2 * r.first[r.axes]) return l;
  if (r.pairing == LV_ROPE_ADJACENT) {
    l.pair = c >> 1;
    l.dist = c & 1 ? -1 : 1;
  } else if (r.pairing == LV_ROPE_HEAD_HALVES) {
    const int all = r.first[r.axes];
    l.pair = c < all ? c : c - all;
    l.dist = c < all ? all : -all;
  } else {
    int a = 0;
    while (c >= 2 * r.first[a + 1]) ++a;
    const int p = r.first[a + 1] - r.first[a], j = c - 2 * r.first[a];
    l.pair = r.first[a] + (j < p ? j : j - p);
    l.dist = j < p ? p : -p;
  }
  while (l.pair >= r.first[l.axis + 1]) ++l.axis;
  return l;
}

}  // namespace

// D / 8 lanes take the heads of one token in turn, 16 bytes of each, so that a lane works its angles out once for all of them.  The partners
// come from memory as well, where the first read of the line has just brought them: as 16 bytes where they lie so (WIDE: an axis has a
// multiple of 8 pairs), else one by one; adjacent pairs lie in the lane's own bytes.  All that a head needs has been read before any of it is
// written, so the output may take the input's place.
template <int D, int MODE>      // 0: adjacent pairs, 1: partners in 16 bytes, 2: one by one
__global__ __launch_bounds__(256) void k_rope(RopeCall a, RopePairs r) {
  constexpr int L = D / 8;
  const int64_t unit = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const int c0 = threadIdx.x % L * 8;
  const int tok = (int)(unit / a.parts), part = (int)(unit - (int64_t)tok * a.parts);
  if (tok >= a.n) return;
  float cs[8], sn[8];
  int dist[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const Lane l = lane_of(r, c0 + e);
    dist[e] = l.dist;
    double turns = (double)a.pos[(int64_t)tok * a.axes + l.axis] * r.turns[l.pair];
    turns -= __builtin_floor(turns);
    const float f = (float)turns;
    cs[e] = l.dist ? __builtin_amdgcn_cosf(f) : 1.0f;
    sn[e] = l.dist ? __builtin_amdgcn_sinf(f) * (l.dist < 0 ? a.sign : -a.sign) : 0.0f;
  }
  const int end = min((part + 1) * a.per, a.all);
  for (int h = part * a.per; h < end; ++h) {
    const int which = h >= a.heads, head = which ? h - a.heads : h;
    const uint16_t *x = a.x[which] + (int64_t)tok * a.x_stride[which] + head * D + c0;
    const u32x4 w = *(const u32x4 *)x;
    float v[8] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y), bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)}, p[8];
    if constexpr (MODE == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = v[e ^ 1];
    } else if constexpr (MODE == 1) {
      const u32x4 o = *(const u32x4 *)(x + dist[0]);
      p[0] = bf16_lo(o.x), p[1] = bf16_hi(o.x), p[2] = bf16_lo(o.y), p[3] = bf16_hi(o.y);
      p[4] = bf16_lo(o.z), p[5] = bf16_hi(o.z), p[6] = bf16_lo(o.w), p[7] = bf16_hi(o.w);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = bf16_to_f32(x[e + dist[e]]);
    }
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = v[e] * cs[e] + p[e] * sn[e];
    if (c0 + 8 > a.rotated) {      // channels that are copied: also what is not finite there
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = c0 + e < a.rotated ? y[e] : v[e];
    }
    *(u32x4 *)(a.y[which] + (int64_t)tok * a.y_stride[which] + head * D + c0) =
        u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
  }
}

int launch_rope(const RopePairs &pairs, const int32_t *pos, int n, int heads, int kv_heads, int head_dim, bool inverse, const uint16_t *q,
                int64_t q_stride, const uint16_t *k, int64_t k_stride, uint16_t *q_out, int64_t q_out_stride, uint16_t *k_out,
                int64_t k_out_stride, hipStream_t st) {
  RopeCall a;
  a.pos = pos;
  a.x[0] = q, a.x[1] = k;
  a.y[0] = q_out, a.y[1] = k_out;
  a.x_stride[0] = q_stride, a.x_stride[1] = k_stride;
  a.y_stride[0] = q_out_stride, a.y_stride[1] = k_out_stride;
  a.heads = heads;
  a.all = heads + kv_heads;
  a.n = n;
  a.axes = pairs.axes;
  a.head_dim = head_dim;
  a.rotated = 2 * pairs.first[pairs.axes];
  a.sign = inverse ? -1.0f : 1.0f;
  a.per = 8;
  a.parts = (a.all + a.per - 1) / a.per;
  const int per_group = 256 / (head_dim / 8);
  const uint32_t grid = (uint32_t)(((int64_t)n * a.parts + per_group - 1) / per_group);
  bool wide = true;
  for (int i = 1; i <= pairs.axes; ++i) wide = wide && pairs.first[i] % 8 == 0;
  const int mode = pairs.pairing == LV_ROPE_ADJACENT ? 0 : wide ? 1 : 2;
  auto go = [&](auto kernel) { kernel<<<dim3(grid), 256, 0, st>>>(a, pairs); };
  if (head_dim == 64) mode == 0 ? go(k_rope<64, 0>) : mode == 1 ? go(k_rope<64, 1>) : go(k_rope<64, 2>);
  else mode == 0 ? go(k_rope<128, 0>) : mode == 1 ? go(k_rope<128, 1>) : go(k_rope<128, 2>);
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

}  // namespace lv
