// The paged cache of K and V: rows of new tokens are written into its pages, quantised to E4M3 or E2M1 on the way when the cache
// holds that, and ranges of positions are read back as bf16 rows.
//
// A page holds page_tokens consecutive positions of one sequence, [kv head][position][channel], so that what attention
// reads of one head is one piece of memory.  Both kernels are bound by HBM: a token's row is read once and written once.
// 43,968 tokens of 16 heads of 64 written as E4M3: 59 us, 4.6 TB/s; 137,400 read back: 166 us, 5.1 TB/s (a copy of 4 GB reaches 4.8 on
// the same card).  As E2M1 57 us, and 40 to read these back.  A single token takes 3 us of the GPU and twice that of the host.
#include "internal.h"
#include "common.h"

namespace lv {

namespace {

// The sequence of token `tok` by its offsets (off[s] <= tok < off[s + 1]), -1 for a token of none.  All lanes of the wave call it
// with the same tok.
__device__ __forceinline__ int seq_of(const int32_t *off, int n_seq, int tok, int lane, int &start) {
  const int s = __builtin_amdgcn_readfirstlane(last_at_most(off, n_seq, tok, lane));
  if (s < 0) return -1;
  start = __builtin_amdgcn_readfirstlane(off[s]);
  return tok < __builtin_amdgcn_readfirstlane(off[s + 1]) ? s : -1;
}

// Bytes of the pool up to position `place` of page `id`, counted in rows
__device__ __forceinline__ int64_t row_of(const CacheView &cv, int id, int head, int place) {
  return (((int64_t)id * cv.kv_heads + head) << cv.page_shift) + place;
}

// The page of position pos of a sequence; -1: not held
__device__ __forceinline__ int page_of(const CacheView &cv, int seq, int64_t pos) {
  if (pos < 0 || (pos >> cv.page_shift) >= cv.max_pages) return -1;
  const int id = cv.table[(int64_t)seq * cv.max_pages + (pos >> cv.page_shift)];
  return (uint32_t)id < (uint32_t)cv.n_pages ? id : -1;
}

template <int LANES>   // largest over the 8 or 16 lanes of a row
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dpp_take<0xB1, 0xF>(v));    // quad_perm [1,0,3,2]
  v = fmaxf(v, dpp_take<0x4E, 0xF>(v));    // quad_perm [2,3,0,1]
  v = fmaxf(v, dpp_take<0x141, 0xF>(v));   // row_half_mirror
  if (LANES == 16) v = fmaxf(v, dpp_take<0x140, 0xF>(v));   // row_mirror
  return v;
}
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_take<0xB1, 0xF>(v);
  v += dpp_take<0x4E, 0xF>(v);
  v += dpp_take<0x141, 0xF>(v);
  if (LANES == 16) v += dpp_take<0x140, 0xF>(v);
  return v;
}

// Eight channels of a row as E4M3 codes and the row's exponent byte.  The scale is the smallest power of two that brings
// the row's largest finite |value| to 448 or less (448 = 1.75 * 2^8): codes times a power of two are exact in bf16, so
// what is read back is what attention uses.  Infinities saturate, NaN stays.
template <int LANES>
__device__ __forceinline__ u32x2 quant_row8(const u32x4 w, uint32_t &exp_byte) {
  float x[8] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y), bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)};
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float m = fabsf(x[i]);
    a = fmaxf(a, m < INFINITY ? m : 0.f);
  }
  a = row_max<LANES>(a);
  const uint32_t bits = __float_as_uint(a);
  // biased exponent of a, less 8, one more for a mantissa over 1.75; at least 2^-126, 2^0 for a row of zeros
  int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = bits == 0u ? 127 : max(e, 1);
  exp_byte = (uint32_t)e;
  const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = clamp448(x[i] * inv);
    x[i] = x[i] != x[i] ? x[i] : y;
  }
  return u32x2{cvt4_fp8(x[0], x[1], x[2], x[3]), cvt4_fp8(x[4], x[5], x[6], x[7])};
}

// Eight channels of a row as E2M1 codes, and the exponent byte of the 32 channels that they are a quarter of: the smallest power of two
// that brings the largest finite |value| to 6 or less (6 = 1.5 * 2^2).  E2M1 has no NaN: a byte of 255 makes all 32 NaN, and one among
// them sets it.
__device__ __forceinline__ uint32_t quant_block8(u32x4 w, uint32_t &exp_byte) {
  // the largest magnitude by its bits, two values to a word
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  auto mag = [](uint32_t v) { return __builtin_bit_cast(u16x2, v & 0x7fff7fffu); };
  auto larger = [](u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); };
  auto largest = [&](const u32x4 v) {
    u16x2 m = larger(larger(mag(v.x), mag(v.y)), larger(mag(v.z), mag(v.w)));
    m = larger(m, __builtin_bit_cast(u16x2, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, m), 0xB1, 0xF, 0xF, false)));
    m = larger(m, __builtin_bit_cast(u16x2, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, m), 0x4E, 0xF, 0xF, false)));
    return (uint32_t)max(m.x, m.y);
  };
  uint32_t top = largest(w);
  bool wild = false;      // the block has a NaN
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(top >= 0x7f80u) != 0, 0)) {
    wild = top > 0x7f80u;
    // the scale is that of the finite values; infinities saturate
    u32x4 f = w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] &= (f[i] & 0x7f80u) == 0x7f80u ? 0xffff0000u : ~0u;
      f[i] &= (f[i] & 0x7f800000u) == 0x7f800000u ? 0xffffu : ~0u;
    }
    top = largest(f);
  }
  // biased exponent of the largest, less 2, one more for a mantissa over 1.5; at least 2^-126, 2^0 for a block of zeros
  const int e = top == 0u ? 127 : max((int)(top >> 7) - 2 + ((top & 0x7fu) > 0x40u ? 1 : 0), 1);
  exp_byte = wild ? 255u : (uint32_t)e;
  return wild ? 0u : cvt8_fp4(w, __uint_as_float((uint32_t)e << 23));
}

}  // namespace

// A wave takes eight (64 channels) or four (128) consecutive tokens of one head, 16 bytes of K and of V per lane: what it
// writes is one piece of a page, what it reads are whole 128-byte lines.  Waves of neighbouring heads stand side by side, so
// a workgroup reads longer pieces of the tokens' rows.
template <int D, int DTYPE>
__global__ __launch_bounds__(256) void k_cache_write(CacheView cv, char *kp, char *vp, uint8_t *ksc, uint8_t *vsc,
                                                     const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride,
                                                     const int32_t *off, const int32_t *pos0, int n, int64_t units, int qk_norm) {
  constexpr int L = D / 8, T = 64 / L;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= units) return;
  const int head = __builtin_amdgcn_readfirstlane((int)(unit % cv.kv_heads));
  const int tok0 = __builtin_amdgcn_readfirstlane((int)(unit / cv.kv_heads) * T);
  const int sub = lane / L, tok = tok0 + sub;
  u32x4 wk = {0, 0, 0, 0}, wv = {0, 0, 0, 0};
  if (tok < n) {
    wk = *(const u32x4 *)(k + tok * k_stride + head * D + (lane % L) * 8);
    wv = *(const u32x4 *)(v + tok * v_stride + head * D + (lane % L) * 8);
  }
  int id = -1;
  int64_t pos = 0;
#pragma unroll 1
  for (int j = 0; j < T; ++j) {     // where each token goes; mostly all to the first one's sequence
    if (tok0 + j >= n) break;
    int start = 0;
    const int s = seq_of(off, cv.n_seq, tok0 + j, lane, start);
    if (s < 0) continue;
    const int end = __builtin_amdgcn_readfirstlane(off[s + 1]);
    const int64_t first = (int64_t)pos0[s] - start;
    if (tok >= tok0 + j && tok < end) {
      pos = first + tok;
      id = page_of(cv, s, pos);
    }
    j = max(j, min(j + T, end - tok0) - 1);   // (never back, whatever the offsets hold)
  }
  if (qk_norm) {
    const float r = 1.0f / sqrtf(row_sum<L>(sumsq8(wk)) * (1.0f / D) + kQkEps);
    wk = scale8(wk, r);
  }
  if constexpr (DTYPE == LV_CACHE_E2M1) {
    uint32_t ek, ev;
    const uint32_t ck = quant_block8(wk, ek), cw = quant_block8(wv, ev);
    if (tok < n && id >= 0) {
      const int64_t row = row_of(cv, id, head, (int)(pos & ((1 << cv.page_shift) - 1)));
      *(uint32_t *)(kp + row * (D / 2) + (lane % L) * 4) = ck;
      *(uint32_t *)(vp + row * (D / 2) + (lane % L) * 4) = cw;
      if (lane % 4 == 0) {
        ksc[row * (D / 32) + lane % L / 4] = (uint8_t)ek;
        vsc[row * (D / 32) + lane % L / 4] = (uint8_t)ev;
      }
    }
  } else if constexpr (DTYPE == LV_CACHE_E4M3) {
    uint32_t ek, ev;
    const u32x2 ck = quant_row8<L>(wk, ek), cw = quant_row8<L>(wv, ev);
    if (tok < n && id >= 0) {
      const int64_t row = row_of(cv, id, head, (int)(pos & ((1 << cv.page_shift) - 1)));
      *(u32x2 *)(kp + row * D + (lane % L) * 8) = ck;
      *(u32x2 *)(vp + row * D + (lane % L) * 8) = cw;
      if (lane % L == 0) {
        ksc[row] = (uint8_t)ek;
        vsc[row] = (uint8_t)ev;
      }
    }
  } else if (tok < n && id >= 0) {
    const int64_t row = row_of(cv, id, head, (int)(pos & ((1 << cv.page_shift) - 1)));
    *(u32x4 *)(kp + row * (2 * D) + (lane % L) * 16) = wk;
    *(u32x4 *)(vp + row * (2 * D) + (lane % L) * 16) = wv;
  }
}

// The reverse; positions that are not held read as zeros.
template <int D, int DTYPE>
__global__ __launch_bounds__(256) void k_cache_read(CacheView cv, const char *kp, const char *vp, const uint8_t *ksc,
                                                    const uint8_t *vsc, const int32_t *first, const int32_t *off, uint16_t *k,
                                                    int64_t k_stride, uint16_t *v, int64_t v_stride, int n, int64_t units) {
  constexpr int L = D / 8, T = 64 / L;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= units) return;
  const int head = __builtin_amdgcn_readfirstlane((int)(unit % cv.kv_heads));
  const int tok0 = __builtin_amdgcn_readfirstlane((int)(unit / cv.kv_heads) * T);
  const int tok = tok0 + lane / L;
  int id = -1;
  int64_t pos = 0;
  bool live = false;
#pragma unroll 1
  for (int j = 0; j < T; ++j) {
    if (tok0 + j >= n) break;
    int start = 0;
    const int s = seq_of(off, cv.n_seq, tok0 + j, lane, start);
    if (s < 0) continue;
    const int end = __builtin_amdgcn_readfirstlane(off[s + 1]);
    if (tok >= tok0 + j && tok < end) {
      live = tok < n;
      pos = (int64_t)first[s] - start + tok;
      id = page_of(cv, s, pos);
    }
    j = max(j, min(j + T, end - tok0) - 1);   // (never back, whatever the offsets hold)
  }
  if (!live) return;
  u32x4 wk = {0, 0, 0, 0}, wv = {0, 0, 0, 0};
  if (id >= 0) {
    const int64_t row = row_of(cv, id, head, (int)(pos & ((1 << cv.page_shift) - 1)));
    if constexpr (DTYPE == LV_CACHE_E2M1) {
      const uint32_t ck = *(const uint32_t *)(kp + row * (D / 2) + (lane % L) * 4), cw = *(const uint32_t *)(vp + row * (D / 2) + (lane % L) * 4);
      wk = dequant8(ck, __uint_as_float((uint32_t)ksc[row * (D / 32) + lane % L / 4] << 23));
      wv = dequant8(cw, __uint_as_float((uint32_t)vsc[row * (D / 32) + lane % L / 4] << 23));
    } else if constexpr (DTYPE == LV_CACHE_E4M3) {
      const u32x2 ck = *(const u32x2 *)(kp + row * D + (lane % L) * 8), cw = *(const u32x2 *)(vp + row * D + (lane % L) * 8);
      wk = dequant8(ck, __uint_as_float((uint32_t)ksc[row] << 23));
      wv = dequant8(cw, __uint_as_float((uint32_t)vsc[row] << 23));
    } else {
      wk = *(const u32x4 *)(kp + row * (2 * D) + (lane % L) * 16);
      wv = *(const u32x4 *)(vp + row * (2 * D) + (lane % L) * 16);
    }
  }
  *(u32x4 *)(k + tok * k_stride + head * D + (lane % L) * 8) = wk;
  *(u32x4 *)(v + tok * v_stride + head * D + (lane % L) * 8) = wv;
}

int launch_cache_write(const CacheView &cv, const litevggt_cache &c, const uint16_t *k, int64_t k_stride, const uint16_t *v,
                       int64_t v_stride, const int32_t *off, const int32_t *pos, int n, int qk_norm, hipStream_t st) {
  const int t = 64 / (cv.head_dim / 8);
  const int64_t units = ((int64_t)n + t - 1) / t * cv.kv_heads;
  auto go = [&](auto kernel) {
    kernel<<<dim3((uint32_t)((units + 3) / 4)), 256, 0, st>>>(cv, (char *)c.k, (char *)c.v, c.k_scale, c.v_scale, k, k_stride, v, v_stride,
                                                              off, pos, n, units, qk_norm);
  };
  if (cv.dtype == LV_CACHE_E2M1) cv.head_dim == 64 ? go(k_cache_write<64, LV_CACHE_E2M1>) : go(k_cache_write<128, LV_CACHE_E2M1>);
  else if (cv.dtype == LV_CACHE_E4M3) cv.head_dim == 64 ? go(k_cache_write<64, LV_CACHE_E4M3>) : go(k_cache_write<128, LV_CACHE_E4M3>);
  else cv.head_dim == 64 ? go(k_cache_write<64, LV_CACHE_BF16>) : go(k_cache_write<128, LV_CACHE_BF16>);
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

int launch_cache_read(const CacheView &cv, const litevggt_cache &c, const int32_t *first, const int32_t *off, uint16_t *k,
                      int64_t k_stride, uint16_t *v, int64_t v_stride, int n, hipStream_t st) {
  const int t = 64 / (cv.head_dim / 8);
  const int64_t units = ((int64_t)n + t - 1) / t * cv.kv_heads;
  auto go = [&](auto kernel) {
    kernel<<<dim3((uint32_t)((units + 3) / 4)), 256, 0, st>>>(cv, (const char *)c.k, (const char *)c.v, c.k_scale, c.v_scale, first, off, k,
                                                              k_stride, v, v_stride, n, units);
  };
  if (cv.dtype == LV_CACHE_E2M1) cv.head_dim == 64 ? go(k_cache_read<64, LV_CACHE_E2M1>) : go(k_cache_read<128, LV_CACHE_E2M1>);
  else if (cv.dtype == LV_CACHE_E4M3) cv.head_dim == 64 ? go(k_cache_read<64, LV_CACHE_E4M3>) : go(k_cache_read<128, LV_CACHE_E4M3>);
  else cv.head_dim == 64 ? go(k_cache_read<64, LV_CACHE_BF16>) : go(k_cache_read<128, LV_CACHE_BF16>);
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

}  // namespace lv
