// Rotary positions with several axes: pairs of a head's channels are turned by angles that a token's positions give.
//
//   y1 = x1 cos t - x2 sin t,  y2 = x2 cos t + x1 sin t,   t = position on the pair's axis * the pair's frequency
//
// The gradient is the same with -t.  Angles are taken in 64 bits as turns (t / 2 pi), of which only the fraction goes on in 32: a product
// of a position below 2^31 and a frequency of 1 is off by 2^-24 of a turn there at most, where 32 bits would lose everything from 2^24 on.
//
// Bound by HBM: every row is read and written once.  43,968 tokens of 16 + 16 heads of 64 in 63 us, 5.7 TB/s (a copy of 4 GB reaches 4.8 on the same
// card); one head after the other behind the angles, as it was first, 97.  20,011 tokens of 16 + 4 heads of 128 in 38 us, 60 before.
// Axes whose pairs are no multiple of 8 fetch partners by two bytes: the former 177 us with halves of an axis paired (10, 11, 11 pairs), 126 with a
// head's, 67 with neighbours.  A single token takes 3 us of the GPU.  Rounded to bf16: the result, once.
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
  int n, axes;
  int parts;               // the heads are taken in so many
  int rotated;             // channels that are; the others are copied
  float sign;              // of the sine
};

// Channel c's axis (its channels lie in [2 first, 2 first + 2 pairs) where an axis' halves are paired), pair and the distance of its partner, below 0
// where it is the pair's second; 0: not turned
struct Channel {
  int axis, pair, dist;
};
__device__ __forceinline__ int axis_of(const RopePairs &r, int pair) {
  return (pair >= r.first[1] && r.axes > 1) + (pair >= r.first[2] && r.axes > 2) + (pair >= r.first[3] && r.axes > 3);
}
__device__ __forceinline__ Channel channel_of(const RopePairs &r, int all, int c) {
  Channel l = {0, 0, 0};
  if (c >= 2 * all) return l;
  if (r.pairing == LV_ROPE_ADJACENT) {
    l.pair = c >> 1;
    l.dist = c & 1 ? -1 : 1;
    l.axis = axis_of(r, l.pair);
  } else if (r.pairing == LV_ROPE_HEAD_HALVES) {
    l.pair = c < all ? c : c - all;
    l.dist = c < all ? all : -all;
    l.axis = axis_of(r, l.pair);
  } else {
    l.axis = axis_of(r, c >> 1);
    const int lo = l.axis == 0 ? 0 : l.axis == 1 ? r.first[1] : l.axis == 2 ? r.first[2] : r.first[3];
    const int hi = l.axis == 0 ? r.first[1] : l.axis == 1 ? r.first[2] : l.axis == 2 ? r.first[3] : r.first[4];
    const int j = c - 2 * lo, p = hi - lo;
    l.pair = lo + (j < p ? j : j - p);
    l.dist = j < p ? p : -p;
  }
  return l;
}

}  // namespace

// D / 8 lanes take heads of one token, 16 bytes of each, so that a lane works its angles out once for PER of them.  The partners come from
// memory as well, where the first read of the line has just brought them: as 16 bytes where they lie so (an axis has a multiple
// of 8 pairs), else one by one; adjacent pairs lie in the lane's own bytes.  All reads of a lane's heads are on the way before its angles are
// worked out, and all that a head needs has been read before any of it is written, so the output may take the input's place.
template <int D, int MODE, int PER>      // 0: adjacent pairs, 1: partners in 16 bytes, 2: one by one
__global__ __launch_bounds__(256) void k_rope(RopeCall a, RopePairs r) {
  constexpr int L = D / 8;
  const uint32_t unit = blockIdx.x * (256 / L) + threadIdx.x / L;
  const int c0 = threadIdx.x % L * 8;
  const int tok = (int)(unit / (uint32_t)a.parts), h0 = (int)(unit - (uint32_t)tok * a.parts) * PER;
  if (tok >= a.n) return;
  const int all = a.rotated >> 1;
  int dist[8];
  Channel ch = channel_of(r, all, c0);
  if constexpr (MODE == 1) dist[0] = ch.dist;
  if constexpr (MODE == 2) {
#pragma unroll
    for (int e = 0; e < 8; ++e) dist[e] = channel_of(r, all, c0 + e).dist;
  }
  u32x4 w[PER];
  uint32_t o[PER][4];      // the partners: two bf16 to a word
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int h = min(h0 + i, a.all - 1), which = h >= a.heads, head = which ? h - a.heads : h;
    const uint16_t *x = (which ? a.x[1] : a.x[0]) + (int64_t)tok * (which ? a.x_stride[1] : a.x_stride[0]) + head * D + c0;
    w[i] = *(const u32x4 *)x;
    if constexpr (MODE == 1) {
      const u32x4 y = *(const u32x4 *)(x + dist[0]);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = y[e];
    }
    if constexpr (MODE == 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = (uint32_t)x[2 * e + dist[2 * e]] | (uint32_t)x[2 * e + 1 + dist[2 * e + 1]] << 16;
    }
  }
  float cs[8], sn[8];
  const int32_t *pos = a.pos + (int64_t)tok * a.axes;
  int at = pos[ch.axis];
#pragma unroll
  for (int e = 0; e < (MODE == 0 ? 4 : 8); ++e) {
    if constexpr (MODE == 1) {
      ch.pair += e ? 1 : 0;
    } else {
      ch = channel_of(r, all, MODE == 0 ? c0 + 2 * e : c0 + e);
      at = pos[ch.axis];
    }
    double turns = (double)at * r.turns[ch.pair];
    turns -= __builtin_floor(turns);
    const float f = (float)turns, co = __builtin_amdgcn_cosf(f), si = __builtin_amdgcn_sinf(f) * a.sign;
    if constexpr (MODE == 0) {
      cs[2 * e] = cs[2 * e + 1] = co;
      sn[2 * e] = -si;
      sn[2 * e + 1] = si;
    } else {
      cs[e] = co;
      sn[e] = ch.dist < 0 ? si : -si;
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int h = h0 + i, which = h >= a.heads, head = which ? h - a.heads : h;
    const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
    uint32_t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x0 = bf16_lo(v[e]), x1 = bf16_hi(v[e]);
      const float p0 = MODE == 0 ? x1 : bf16_lo(o[i][e]), p1 = MODE == 0 ? x0 : bf16_hi(o[i][e]);
      y[e] = pack_bf16(x0 * cs[2 * e] + p0 * sn[2 * e], x1 * cs[2 * e + 1] + p1 * sn[2 * e + 1]);
      if (c0 + 8 > a.rotated) {      // channels that are copied, bit by bit
        const uint32_t keep = (c0 + 2 * e < a.rotated ? 0u : 0xffffu) | (c0 + 2 * e + 1 < a.rotated ? 0u : 0xffff0000u);
        y[e] = (y[e] & ~keep) | (v[e] & keep);
      }
    }
    if (h < a.all)
      *(u32x4 *)((which ? a.y[1] : a.y[0]) + (int64_t)tok * (which ? a.y_stride[1] : a.y_stride[0]) + head * D + c0) = u32x4{y[0], y[1], y[2], y[3]};
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
  a.rotated = 2 * pairs.first[pairs.axes];
  a.sign = inverse ? -1.0f : 1.0f;
  const int per_group = 256 / (head_dim / 8);
  // four heads to a lane, so that the angles are worked out once for all of them; one where the chip would not be full so (32 heads of 64: 1 token
  // 2.8 us with one and 3.3 with four, 256 3.8 and 4.6; 5496 tokens 12.8 and 10)
  const bool few = (int64_t)n * a.all <= 8192;
  const int per = few ? 1 : 4;
  a.parts = (a.all + per - 1) / per;
  const uint32_t grid = (uint32_t)(((int64_t)n * a.parts + per_group - 1) / per_group);
  bool wide = true;
  for (int i = 1; i <= pairs.axes; ++i) wide = wide && pairs.first[i] % 8 == 0;
  const int mode = pairs.pairing == LV_ROPE_ADJACENT ? 0 : wide ? 1 : 2;
  auto go = [&](auto kernel) { kernel<<<dim3(grid), 256, 0, st>>>(a, pairs); };
  auto by_mode = [&](auto dim, auto p) {
    constexpr int D = decltype(dim)::value, PER = decltype(p)::value;
    mode == 0 ? go(k_rope<D, 0, PER>) : mode == 1 ? go(k_rope<D, 1, PER>) : go(k_rope<D, 2, PER>);
  };
  auto by_per = [&](auto dim) { few ? by_mode(dim, std::integral_constant<int, 1>{}) : by_mode(dim, std::integral_constant<int, 4>{}); };
  head_dim == 64 ? by_per(std::integral_constant<int, 64>{}) : by_per(std::integral_constant<int, 128>{});
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

}  // namespace lv
