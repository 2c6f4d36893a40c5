// The attention weight that the positions of a cache draw: what the rows of new tokens give each of them, added to what it had.
//
//   mass_t += sum over rows r of w_rt / sum over t' of w_rt',   w_rt = exp2(c q_r.k_t - R_r),   c = scale * log2(e)
//
// A weight's divisor is known when the row's last key has been seen, so the keys are walked twice: k_mass_rows* sums each row's weights
// (pieces of the key axis by different waves, k_mass_join puts them together), k_mass_keys sums each key's.  V is not read.  In all of them a
// wave holds a chunk of keys in registers as bf16, fetched and decoded once, and walks the rows that see them: 32 x 32 tiles of MFMA, no LDS,
// no barrier, and nobody waits for another wave.  Which channels a lane holds is free as long as q and k agree: a half wave takes half a
// row's channels in one piece, so its loads are 16 bytes wide in every kind of cache.
//
// Up to 32 rows: bound by reading K and writing the scores, from which the second walk is made, in bf16 (5 rows over 137,405 positions of 16 heads
// of 64: 61 to 68 us for 281 MB and 44, 5 to join, 14 to add; K twice was 48 and 54); over codes by chains of dependent loads and three launches (5
// rows over 60,000: 48 us in bf16, 34 in E4M3, 29 in E2M1, whose bytes take 27, 15 and 8).  More: a tile of 32 x 32 scores takes 16
// exponentials, 16 multiply-adds and 16 sums of a lane, twice, some 400 cycles each time with what goes around them, against 128 of MFMA at 64
// channels: four frames of 1374 tokens over 2748 to 41,220 positions of an E2M1 cache 441 us for the rows' sums and 395 for the keys', 20 to join
// (VALU 62 and 71 % busy, 1.5 and 1.6 of two waves resident to a SIMD, CUs busy 84 and 89 %).
// (Tried and level: a tile's products ahead of or among the weights of the one before, keys in chunks of 5 tiles: 926, for want of registers.)
//
// References, sums and masses are fp32; sums over rows and pieces have a fixed order.  q is rounded to bf16 after its normalisation, as
// K was before it was stored; nothing else is rounded below fp32.
#include <algorithm>

#include "internal.h"
#include "common.h"
#include "mass_plan.h"

namespace lv {

using namespace mass;

namespace {

// (A reference is c times the largest score, rounded: by 16 at most where scores, times the scale, stay below 2^28, so that all of a row's
// weights are 2^16 times too large or too small at most, which the division takes out.  From 2^31 on they would leave fp32's range.)
constexpr float kUnset = -1e30f;             // reference of a row that has seen no key
constexpr float kRaise = 1.0995116e12f;      // 2^40: a sum beyond it raises the reference
constexpr int kNoKey = 0x7fff0000;           // the position of a key that is not there: beyond all that rows see

enum class Kind { BF16, E4M3, E2M1 };

struct Call {
  const uint16_t *q;
  int64_t q_stride;        // 0: rows lie as their numbers count (k_mass_pack)
  const int32_t *q_off, *kv_len;
  int n_q, n_seq, kv_heads, group, frame;
  float c;
  const char *k;
  const uint8_t *k_scale;
  const int32_t *table;
  int page_shift, n_pages, max_pages;
  Cut cut;
  int splits;              // of the rows
  const float *mass_in;
  float *mass;
  float2 *part;            // [piece][kv head][token, head of the group]: reference, sum of weights
  float2 *stat;            // [kv head][token, head of the group]: reference, 1 / sum of weights
  Cut rows_cut;            // k_mass_add: that of the rows' sums
  float *scores;           // [kv head][token, head of the group][position], where there are few rows; else null
};

struct Seq {
  int q0, nq, nk, p0;      // its queries, its keys, the position of its first query
};

__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
// One number for all lanes, by a scalar load
__device__ __forceinline__ int uniform_at(const int32_t *p, int i) { return ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)p)[i]; }

__device__ __forceinline__ Seq seq_of_numbers(const Call &a, int off, int next, int kv_len) {
  Seq r;
  const int len = max(kv_len, 0);
  r.q0 = min(max(off, 0), a.n_q);
  r.nq = min(max(next, r.q0), a.n_q) - r.q0;
  r.nk = (int)min((int64_t)len, (int64_t)a.max_pages << a.page_shift);
  r.p0 = len - r.nq;
  return r;
}
__device__ __forceinline__ Seq seq_at(const Call &a, int s) { return seq_of_numbers(a, uniform_at(a.q_off, s), uniform_at(a.q_off, s + 1), uniform_at(a.kv_len, s)); }

// Keys that query i sees (all up to this one); it does not fall from query to query
__device__ __forceinline__ int limit_of(const Call &a, const Seq &s, int i) {
  if (a.frame <= 0) return s.nk;
  const int p = s.p0 + i;
  if (p < 0) return 0;
  return (int)min((uint32_t)s.nk, ((uint32_t)p / (uint32_t)a.frame + 1u) * (uint32_t)a.frame);   // (below 2^32)
}
// The first query that sees a key
__device__ __forceinline__ int first_query(const Call &a, const Seq &s, int key) {
  if (a.frame <= 0) return 0;
  return max((int)((uint32_t)key / (uint32_t)a.frame * (uint32_t)a.frame) - s.p0, 0);
}

// ---------------------------------------------------------------------------------------
// A lane's half row (D / 2 channels from (lane / 32) D / 2 on) of one key as it is stored
template <Kind K, int D>
struct Half {
  static constexpr int kBytes = K == Kind::BF16 ? D : K == Kind::E4M3 ? D / 2 : D / 4;
  static constexpr int kLoads = kBytes / 16, kScales = K == Kind::E2M1 ? D / 64 : 1;
  u32x4 w[kLoads];
  uint32_t e[kScales];
  __device__ __forceinline__ void load(const Call &a, int64_t row, int lane) {
    const char *p = a.k + row * (2 * kBytes) + (lane >> 5) * kBytes;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) w[i] = *(const u32x4 *)(p + i * 16);
    if constexpr (K == Kind::E4M3) e[0] = a.k_scale[row];
    if constexpr (K == Kind::E2M1) {
#pragma unroll
      for (int i = 0; i < kScales; ++i) e[i] = a.k_scale[row * (D / 32) + (lane >> 5) * kScales + i];
    }
  }
  // channels 8 j .. of it
  __device__ __forceinline__ bf16x8 fragment(int j) const {
    if constexpr (K == Kind::BF16) return __builtin_bit_cast(bf16x8, w[j]);
    if constexpr (K == Kind::E4M3)
      return __builtin_bit_cast(bf16x8, dequant8(u32x2{w[j / 2][j % 2 * 2], w[j / 2][j % 2 * 2 + 1]}, __uint_as_float(e[0] << 23)));
    if constexpr (K == Kind::E2M1) return __builtin_bit_cast(bf16x8, dequant8((uint32_t)w[j / 4][j % 4], __uint_as_float(e[j / 4] << 23)));
  }
};

// The pool's row of a lane's key, -1 if the key is not held or not the sequence's.  What is beyond the end looks at the table's last column.
__device__ __forceinline__ int64_t row_of(const Call &a, int seq, int head, int key, int nk) {
  const int id = a.table[(int64_t)seq * a.max_pages + min((uint32_t)key >> a.page_shift, (uint32_t)a.max_pages - 1u)];
  const bool held = key < nk && (uint32_t)id < (uint32_t)a.n_pages;
  return held ? (((int64_t)id * a.kv_heads + head) << a.page_shift) + (key & ((1 << a.page_shift) - 1)) : -1;
}

__device__ __forceinline__ int64_t row_number(const Call &a, int head, const Seq &s) { return ((int64_t)head * a.n_q + s.q0) * a.group; }

template <int D>
struct Query {
  bf16x8 f[D / 16];
  __device__ __forceinline__ void load(const Call &a, const Seq &s, int head, int row, int n_rows, int lane) {
    const int r = min(row, n_rows - 1);
    const uint16_t *p;
    if (a.q_stride == 0) {
      p = a.q + (row_number(a, head, s) + r) * D;
    } else {
      const int i = (int)((uint32_t)r / (uint32_t)a.group), g = r - i * a.group;
      p = a.q + (int64_t)(s.q0 + i) * a.q_stride + (int64_t)(head * a.group + g) * D;
    }
    p += (lane >> 5) * (D / 2);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) f[j] = *(const bf16x8 *)(p + 8 * j);
  }
};

template <int D>
__device__ __forceinline__ f32x16 product(const bf16x8 (&x)[D / 16], const bf16x8 (&y)[D / 16]) {
  f32x16 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < D / 16; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[j], y[j], acc, 0, 0, 0);
  return acc;
}

struct Work {
  int seq, head, piece, split;
  int c0, c1;      // its chunks
};

// What all chunks of a sequence cost
__device__ __forceinline__ float cost_of_all(const Call &a, const Cut &c, const Seq &s) {
  return has_pieces(c, s.nq, s.nk) ? chunk_cost(c, s.nq * a.group) * (float)quotient_up(s.nk, c.chunk) : 0.f;
}
__device__ __forceinline__ int chunks_of_piece(const Call &a, const Cut &c, const Seq &s, float work) { return mass::chunks_of_piece(c, s.nq * a.group, s.nk, work); }
__device__ __forceinline__ int units_of(const Call &a, const Cut &c, const Seq &s, float work) {
  return has_pieces(c, s.nq, s.nk) ? quotient_up(quotient_up(s.nk, c.chunk), chunks_of_piece(a, c, s, work)) * a.kv_heads * a.splits : 0;
}
// The work of a piece, worked out by every wave (the same in all of them) or once
__device__ __forceinline__ Seq lane_seq(const Call &a) {
  const int i = min((int)(threadIdx.x & 63), a.n_seq - 1);
  return seq_of_numbers(a, a.q_off[i], a.q_off[i + 1], a.kv_len[i]);
}
__device__ __forceinline__ float work_of(const Call &a, const Cut &c, const Seq &mine) {
  if (c.starts) return __builtin_bit_cast(float, uniform_at(c.starts, a.n_seq + 1));
  return piece_work(c, a.kv_heads, wave_sum_ordered((int)(threadIdx.x & 63) < a.n_seq ? cost_of_all(a, c, mine) : 0.f));
}

// up to the lane (row_shr 1, 2, 4, 8 inside rows of 16 lanes; the rows' last lanes to the rows behind)
__device__ __forceinline__ int wave_prefix(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

// The wave's part of the call: the units of the sequences one after the other, those that are not there behind them all.  (Workgroups go to
// the parts of an XCD in turn, whether these have room or not: where every pair had the same number of units, a third of them empty, the
// parts that got the full ones held the others up, and 5 of 8 waves ran: four frames over 2748 to 41,220 positions 737 us
// for the rows' sums and 896 for the keys', 505 and 633 so.)
__device__ __forceinline__ bool find_work(const Call &a, int unit, Work &w, Seq &s) {
  const int lane = threadIdx.x & 63;
  const Cut &c = a.cut;
  int local;
  float work;
  if (c.starts) {
    if (unit >= uniform_at(c.starts, a.n_seq)) return false;
    w.seq = scalar(max(last_at_most(c.starts, a.n_seq, unit, lane), 0));
    local = unit - uniform_at(c.starts, w.seq);
    s = seq_at(a, w.seq);
    work = work_of(a, c, s);
  } else {
    const Seq mine = lane_seq(a);
    work = work_of(a, c, mine);
    const int units = lane < a.n_seq ? units_of(a, c, mine, work) : 0, end = wave_prefix(units);
    if (unit >= __builtin_amdgcn_readlane(end, 63)) return false;
    w.seq = scalar(__popcll(__builtin_amdgcn_ballot_w64(end <= unit)));
    local = unit - __builtin_amdgcn_readlane(end - units, w.seq);
    s.q0 = __builtin_amdgcn_readlane(mine.q0, w.seq);
    s.nq = __builtin_amdgcn_readlane(mine.nq, w.seq);
    s.nk = __builtin_amdgcn_readlane(mine.nk, w.seq);
    s.p0 = __builtin_amdgcn_readlane(mine.p0, w.seq);
  }
  if (!has_pieces(c, s.nq, s.nk)) return false;      // (lengths that changed meanwhile)
  const int chunks = quotient_up(s.nk, c.chunk), per = scalar(chunks_of_piece(a, c, s, work)), pieces = scalar(quotient_up(chunks, per));
  const int x = scalar((int)((uint32_t)local / (uint32_t)pieces));
  w.piece = scalar(local - x * pieces);
  w.head = scalar((int)((uint32_t)x / (uint32_t)a.splits));
  w.split = scalar(x - w.head * a.splits);
  if (w.head >= a.kv_heads) return false;
  w.c0 = w.piece * per;
  w.c1 = min(w.c0 + per, chunks);
  return w.c0 < w.c1;
}

}  // namespace

// More than 64 sequences: the work of a piece and the units before each sequence, worked out once.  (Twice: for the rows' sums, then, with
// `b`, for the keys'.)  Sums in a fixed order.
__global__ __launch_bounds__(1024) void k_mass_plan(Call a, Call b, int *starts_a, int *starts_b) {
  const int tid = threadIdx.x, lane = tid & 63, wave = scalar(tid >> 6);
  __shared__ int sums[2][16];
  __shared__ float works[16];
  for (int which = 0; which < 2; ++which) {
    const Call &c = which ? b : a;
    int *const starts = which ? starts_b : starts_a;
    auto seq = [&](int i) { return seq_of_numbers(c, c.q_off[i], c.q_off[i + 1], c.kv_len[i]); };
    float all = 0.f;
    for (int i = tid; i < c.n_seq; i += 1024) all += cost_of_all(c, c.cut, seq(i));
    all = wave_sum_ordered(all);
    if (lane == 0) works[wave] = all;
    __syncthreads();
    all = 0.f;
    for (int x = 0; x < 16; ++x) all += works[x];
    const float work = piece_work(c.cut, c.kv_heads, all);
    int before = 0;
    for (int i0 = 0; i0 < c.n_seq; i0 += 1024) {
      const int i = i0 + tid, turn = i0 >> 10 & 1;
      const int units = i < c.n_seq ? units_of(c, c.cut, seq(i), work) : 0, end = wave_prefix(units);
      if (lane == 63) sums[turn][wave] = end;
      __syncthreads();      // (the other of the two is read by nobody any more behind it)
      int at = before + end - units;
      for (int x = 0; x < 16; ++x) {
        at += x < wave ? sums[turn][x] : 0;
        before += sums[turn][x];
      }
      if (i < c.n_seq) starts[i] = at;
    }
    if (tid == 0) {
      starts[c.n_seq] = before;
      starts[c.n_seq + 1] = __builtin_bit_cast(int, work);
    }
    __syncthreads();
  }
}

// Rows by kv head, normalised if they are to be: [kv head][token, head of the group][D].  As they come, the rows of one head lie the width of a
// token apart, and many waves that walk the same head would all wait for the few channels of L2 that such lines are in.
template <int D>
__global__ __launch_bounds__(256) void k_mass_pack(const uint16_t *q, int64_t stride, int n_q, int kv_heads, int group, int qk_norm, uint16_t *out) {
  constexpr int L = D / 8;
  const int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L, rows = (int64_t)n_q * kv_heads * group;
  const int p = threadIdx.x % L;
  const uint32_t rr = (uint32_t)(r < rows ? r : rows - 1), heads = (uint32_t)(kv_heads * group);
  const uint32_t tok = rr / heads, head = rr - tok * heads, kv = head / (uint32_t)group;
  u32x4 w = *(const u32x4 *)(q + tok * stride + head * D + p * 8);
  if (qk_norm) {
    float ss = sumsq8(w);
#pragma unroll
    for (int o = 1; o < L; o <<= 1) ss += __shfl_xor(ss, o, 64);
    w = scale8(w, 1.0f / sqrtf(ss * (1.0f / D) + kQkEps));
  }
  if (r < rows) *(u32x4 *)(out + (((int64_t)kv * n_q + tok) * group + (head - kv * group)) * D + p * 8) = w;
}

// ---------------------------------------------------------------------------------------
// Rows' sums, many rows: S^T = K Q^T, a lane has one row and 16 of a tile's keys.  NT tiles of 32 keys stay in registers.  A row's sum over
// the keys of a wave's piece is kept in `part`: chunks after the first add to it.  Blocks of rows that do not all see the whole chunk come
// first; the others look at no position.
template <Kind K, int D, int NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_mass_rows(Call a) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  Work w;
  Seq s;
  if (!find_work(a, scalar((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), w, s)) return;
  const int n_rows = s.nq * a.group;
  // rows of this split, in blocks of 32, from the first that sees the piece's first key
  const int blocks = (n_rows + 31) / 32, per = scalar(quotient_up(blocks, a.splits));
  const int b1 = min((w.split + 1) * per, blocks);
  float2 *part = a.part + (int64_t)w.piece * a.kv_heads * a.n_q * a.group + row_number(a, w.head, s);
  bool fresh = true;
  for (int ch = w.c0; ch < w.c1; ++ch) {
    const int key0 = ch * (32 * NT);
    bf16x8 kf[NT][D / 16];
    uint32_t there = 0;      // bit 2 t + g: group g of 16 keys of tile t is held
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int64_t row = row_of(a, w.seq, w.head, key0 + t * 32 + (lane & 31), s.nk);
      const uint64_t held = __builtin_amdgcn_ballot_w64(row >= 0);
      there |= (held & 1 ? 1u : 0u) << (2 * t) | (held >> 16 & 1 ? 2u : 0u) << (2 * t);
      Half<K, D> x;
      x.load(a, max(row, (int64_t)0), lane);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) kf[t][j] = x.fragment(j);
    }
    there = (uint32_t)scalar((int)there);
    if (there == 0 && !(fresh && ch == w.c1 - 1)) continue;
    const int b0 = max(scalar(first_query(a, s, fresh ? w.c0 * (32 * NT) : key0)) * a.group / 32, w.split * per);
    // the first block whose rows all see the chunk
    const int end = min(key0 + 32 * NT, s.nk);
    const int whole = (int)min((uint32_t)(scalar(first_query(a, s, end - 1)) * a.group + 31) / 32u, (uint32_t)blocks);
    if (b0 >= b1) {
      fresh = false;
      continue;
    }
    Query<D> next;
    next.load(a, s, w.head, b0 * 32 + (lane & 31), n_rows, lane);
    auto block = [&](auto cut, int b) __attribute__((always_inline)) {
      constexpr bool kCut = decltype(cut)::value;
      const int row = b * 32 + (lane & 31);
      const Query<D> q = next;
      next.load(a, s, w.head, row + 32, n_rows, lane);
      const int lim = kCut ? limit_of(a, s, min(row, n_rows - 1) / a.group) : end;
      float ref = kUnset, l = 0.f;

#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t held = there >> (2 * t) & 3u;
        f32x16 x = product<D>(kf[t], q.f);

        if (t > 0 && held == 0) continue;
        const int k0 = key0 + t * 32;
        if (kCut || held != 3u || k0 + 32 > end) {
          int seen = lim;
          asm volatile("" : "+v"(seen));      // (known ahead of the loop, 128 comparisons would be kept in scalar registers that are not there)
          const int t0 = seen - (held & 1u ? k0 : kNoKey) - 4 * h, t1 = seen - (held & 2u ? k0 + 16 : kNoKey) - 4 * h;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((r >> 2 & 1) * 8 + (r & 3) >= (r < 8 ? t0 : t1)) x[r] = -INFINITY;
        }
        float sum;
        auto weights = [&]() __attribute__((always_inline)) {
          float s0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[0], a.c, -ref)), s1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[1], a.c, -ref));
#pragma unroll
          for (int r = 2; r < 16; r += 2) {
            s0 += __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.c, -ref));
            s1 += __builtin_amdgcn_exp2f(__builtin_fmaf(x[r + 1], a.c, -ref));
          }
          sum = s0 + s1;
        };
        auto raise = [&]() __attribute__((always_inline)) {
          float top = x[0];
#pragma unroll
          for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float to = fmaxf(ref, top * a.c);
          l *= __builtin_amdgcn_exp2f(ref - to);
          ref = to;
        };
        if (t == 0) raise();
        weights();
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(l + sum <= kRaise)) != 0, 0)) {
          raise();
          weights();
        }
        l += sum;
      }
      l += __shfl_xor(l, 32, 64);
      if (lane < 32 && row < n_rows) {
        if (!fresh) {
          const float2 o = part[row];
          const float to = fmaxf(ref, o.x);
          l = l * __builtin_amdgcn_exp2f(ref - to) + o.y * __builtin_amdgcn_exp2f(o.x - to);
          ref = to;
        }
        part[row] = float2{ref, l};
      }
    };
    int b = b0;
    for (; b < min(whole, b1); ++b) block(std::true_type{}, b);
    for (; b < b1; ++b) block(std::false_type{}, b);
    fresh = false;
  }
}

// ---------------------------------------------------------------------------------------
// Rows' sums, up to 32 rows: S = Q K^T, a lane has one key of a tile and 4 RG of the rows, and sums of its own until the piece's end.  The next
// tile is on its way, and the page of the one behind it known, while one is computed with.  SCORES: they are kept, so that K is not
// read again.
template <Kind K, int D, int RG, bool SCORES>
__global__ __launch_bounds__(256) void k_mass_rows_few(Call a) {
  constexpr int R = 4 * RG;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  Work w;
  Seq s;
  if (!find_work(a, scalar((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), w, s)) return;
  const int n_rows = s.nq * a.group;
  const int64_t room = (int64_t)a.max_pages << a.page_shift;
  // 8 RG rows at a time (more than once where sequences are of unlike lengths)
  for (int row0 = 0; row0 < n_rows; row0 += 8 * RG) {
    Half<K, D> coming;
    int64_t at = row_of(a, w.seq, w.head, w.c0 * 32 + (lane & 31), s.nk);
    int64_t at1 = row_of(a, w.seq, w.head, (w.c0 + 1) * 32 + (lane & 31), s.nk);
    coming.load(a, max(at, (int64_t)0), lane);
    Query<D> q;
    q.load(a, s, w.head, row0 + (lane & 31), n_rows, lane);
    const int64_t number = row_number(a, w.head, s) + row0;
    float l[R], ref[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      l[r] = 0.f;
      ref[r] = kUnset;
    }
    for (int ch = w.c0; ch < w.c1; ++ch) {
      const int key = ch * 32 + (lane & 31);
      const Half<K, D> x = coming;
      const bool held = at >= 0;
      at = at1;
      coming.load(a, max(at, (int64_t)0), lane);
      at1 = row_of(a, w.seq, w.head, key + 64, s.nk);
      if (__builtin_amdgcn_ballot_w64(held) == 0) continue;
      bf16x8 kf[D / 16];
#pragma unroll
      for (int j = 0; j < D / 16; ++j) kf[j] = x.fragment(j);
      const f32x16 y = product<D>(q.f, kf);
      // the lane's key counts for rows from this one on
      const int from = held ? first_query(a, s, key) * a.group - row0 - 4 * h : kNoKey;
      float v[R], p[R];
      bool high = false;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int row = 8 * (r >> 2) + (r & 3);
        if constexpr (SCORES) {
          if (key < s.nk && row0 + row + 4 * h < n_rows) a.scores[(number + row + 4 * h) * room + key] = y[r];
        }
        v[r] = row >= from ? y[r] : -INFINITY;
        p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(v[r], a.c, -ref[r]));
        high = high || !(l[r] + p[r] <= kRaise);
      }
      if (__builtin_amdgcn_ballot_w64(high) != 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float to = fmaxf(ref[r], v[r] * a.c);
          l[r] *= __builtin_amdgcn_exp2f(ref[r] - to);
          ref[r] = to;
          p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(v[r], a.c, -to));
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) l[r] += p[r];
    }
    float2 *part = a.part + (int64_t)w.piece * a.kv_heads * a.n_q * a.group + number;
    // over the 32 lanes of a half: at each step a lane gives half of its rows away and takes the other lane's share of the half it keeps, until
    // lane r has row r of R; then the lanes that have the same row
    auto join = [&](int r, float other, float sum) __attribute__((always_inline)) {
      const float to = fmaxf(ref[r], other);
      l[r] = l[r] * __builtin_amdgcn_exp2f(ref[r] - to) + sum * __builtin_amdgcn_exp2f(other - to);
      ref[r] = to;
    };
    auto halve = [&](auto step) __attribute__((always_inline)) {
      constexpr int kBit = decltype(step)::value;
      const bool up = lane & kBit;
      if constexpr (kBit < R) {
#pragma unroll
        for (int r = 0; r < kBit; ++r) {
          float a0 = ref[r], a1 = ref[r + kBit], b0 = l[r], b1 = l[r + kBit];
          asm("" : "+v"(a0), "+v"(a1), "+v"(b0), "+v"(b1));
          ref[r] = up ? a1 : a0;
          l[r] = up ? b1 : b0;
          join(r, __shfl_xor(up ? a0 : a1, kBit, 64), __shfl_xor(up ? b0 : b1, kBit, 64));
        }
      } else {
        join(0, __shfl_xor(ref[0], kBit, 64), __shfl_xor(l[0], kBit, 64));
      }
    };
    if constexpr (R == 16) {
      halve(std::integral_constant<int, 8>{});
      halve(std::integral_constant<int, 4>{});
    }
    halve(std::integral_constant<int, 2>{});
    halve(std::integral_constant<int, 1>{});
    if constexpr (R == 4) {
      halve(std::integral_constant<int, 4>{});
      halve(std::integral_constant<int, 8>{});
    }
    halve(std::integral_constant<int, 16>{});
    const int r = lane & (R - 1), row = 8 * (r >> 2) + (r & 3) + 4 * h;
    if ((lane & 31) < R && row0 + row < n_rows) part[row] = float2{ref[0], l[0]};
  }
}

// Keys' sums from scores that were kept: four keys to a thread, a workgroup to a unit.  OWN: the pieces of 64 rows at a time are put together by
// every workgroup for itself (a wave to a row, its lanes to the pieces), which is less than another launch where there are few of them
// (5 rows over 137,405 positions, 2147 workgroups: 21 us so, 17 with the launch).
template <bool OWN>
__global__ __launch_bounds__(256) void k_mass_add(Call a) {
  Work w;
  Seq s;
  if (!find_work(a, (int)blockIdx.x, w, s)) return;
  const int n_rows = s.nq * a.group, lane = threadIdx.x & 63, wave = scalar((int)(threadIdx.x >> 6));
  const int64_t room = (int64_t)a.max_pages << a.page_shift, base = ((int64_t)w.seq * a.kv_heads + w.head) * room, number = row_number(a, w.head, s);
  const int64_t all = (int64_t)a.kv_heads * a.n_q * a.group;
  const int of_piece = OWN ? chunks_of_piece(a, a.rows_cut, s, work_of(a, a.rows_cut, lane_seq(a))) * a.rows_cut.chunk : 1;      // keys
  __shared__ float2 stat[64];
  for (int ch = w.c0; ch < w.c1; ++ch) {
    const int64_t key = (int64_t)ch * 1024 + threadIdx.x * 4;
    const int id = key < s.nk ? a.table[(int64_t)w.seq * a.max_pages + (key >> a.page_shift)] : -1;
    const bool held = (uint32_t)id < (uint32_t)a.n_pages;
    int from[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) from[e] = first_query(a, s, (int)min(key, (int64_t)s.nk) + e) * a.group;
    f32x4 had = {0.f, 0.f, 0.f, 0.f}, drawn = {0.f, 0.f, 0.f, 0.f};
    if (held && a.mass_in) had = *(const f32x4 *)(a.mass_in + base + key);
    for (int r0 = 0; r0 < n_rows; r0 += 64) {
      const int rows = min(n_rows - r0, 64);
      if (OWN && (n_rows > 64 || ch == w.c0)) {      // (the same for all)
        __syncthreads();
        for (int r = wave; r < rows; r += 4) {
          const int seen = quotient_up(limit_of(a, s, (r0 + r) / a.group), of_piece);
          float ref = kUnset, l = 0.f;
          for (int p = lane; p < seen; p += 64) {
            const float2 o = a.part[p * all + number + r0 + r];
            const float to = fmaxf(ref, o.x);
            l = l * __builtin_amdgcn_exp2f(ref - to) + o.y * __builtin_amdgcn_exp2f(o.x - to);
            ref = to;
          }
          float to = ref;
#pragma unroll
          for (int o = 32; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor(to, o, 64));
          l = wave_sum(l * __builtin_amdgcn_exp2f(ref - to));
          if (lane == 0) stat[r] = float2{to, l == 0.f ? 0.f : 1.0f / l};
        }
        __syncthreads();
      }
      if (held) {
#pragma unroll 4
        for (int r = 0; r < rows; ++r) {
          const f32x4 v = *(const f32x4 *)(a.scores + (number + r0 + r) * room + key);
          const float2 o = OWN ? stat[r] : a.stat[number + r0 + r];
#pragma unroll
          for (int e = 0; e < 4; ++e) drawn[e] += r0 + r >= from[e] ? __builtin_amdgcn_exp2f(__builtin_fmaf(v[e], a.c, -o.x)) * o.y : 0.f;
        }
      }
    }
    f32x4 sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = had[e] + drawn[e];
    float *p = a.mass + base + key;
    if (key + 4 <= s.nk) {
      *(f32x4 *)p = sum;
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (key + e < s.nk) p[e] = sum[e];
    }
  }
}

// ---------------------------------------------------------------------------------------
// The sums of a row's pieces put together, always in the same order.  ROWS of them to a workgroup (64: a lane each, the pieces by turns to
// the four waves; 4: a wave each, a lane's pieces 64 apart), four pieces' loads on the way together.
template <int ROWS>
__global__ __launch_bounds__(256) void k_mass_join(Call a, int side) {
  constexpr int kSlices = 256 / ROWS;
  const int pair = scalar((int)(blockIdx.x / (uint32_t)side)), turn = scalar((int)(blockIdx.x - pair * (uint32_t)side));
  const int seq = scalar((int)((uint32_t)pair / (uint32_t)a.kv_heads)), head = scalar(pair - seq * a.kv_heads);
  const Seq s = seq_at(a, seq);
  const int n_rows = s.nq * a.group, mine = ROWS == 64 ? threadIdx.x & 63 : threadIdx.x >> 6, slice = ROWS == 64 ? threadIdx.x >> 6 : threadIdx.x & 63;
  const int of_piece = chunks_of_piece(a, a.cut, s, work_of(a, a.cut, lane_seq(a))) * a.cut.chunk;      // keys
  const int64_t all = (int64_t)a.kv_heads * a.n_q * a.group, base = row_number(a, head, s);
  __shared__ float2 sums[4][64];
  for (int row0 = turn * ROWS; row0 < n_rows; row0 += side * ROWS) {
    const int row = min(row0 + mine, n_rows - 1);
    const int lim = limit_of(a, s, row / a.group);
    const int seen = quotient_up(lim, of_piece);      // pieces that it sees
    float ref = kUnset, l = 0.f;
    for (int p0 = slice; p0 < seen; p0 += 4 * kSlices) {
      float2 o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = a.part[min(p0 + i * kSlices, seen - 1) * all + base + row];
      float to = ref;
#pragma unroll
      for (int i = 0; i < 4; ++i) to = fmaxf(to, o[i].x);
      l *= __builtin_amdgcn_exp2f(ref - to);
#pragma unroll
      for (int i = 0; i < 4; ++i) l += p0 + i * kSlices < seen ? o[i].y * __builtin_amdgcn_exp2f(o[i].x - to) : 0.f;
      ref = to;
    }
    if constexpr (ROWS == 64) {
      sums[slice][mine] = float2{ref, l};
      __syncthreads();
      if (slice == 0) {
        float to = ref;
#pragma unroll
        for (int i = 1; i < 4; ++i) to = fmaxf(to, sums[i][mine].x);
        l *= __builtin_amdgcn_exp2f(ref - to);
#pragma unroll
        for (int i = 1; i < 4; ++i) l += sums[i][mine].y * __builtin_amdgcn_exp2f(sums[i][mine].x - to);
        ref = to;
      }
      __syncthreads();
    } else {
      float to = ref;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor(to, o, 64));
      l = wave_sum(l * __builtin_amdgcn_exp2f(ref - to));
      ref = to;
    }
    if (slice == 0 && row0 + mine < n_rows) a.stat[base + row] = float2{ref, l == 0.f ? 0.f : 1.0f / l};
  }
}

// ---------------------------------------------------------------------------------------
// Keys' sums, up to 32 rows whose scores are not kept: S = Q K^T, a lane has one key of each of NT tiles and 4 RG of a block's rows, whose references and divisors are in its
// registers, the same for all lanes of a half.
template <Kind K, int D, int NT, int RG>
__global__ __launch_bounds__(256) void k_mass_keys_few(Call a) {
  constexpr int R = 4 * RG;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  Work w;
  Seq s;
  if (!find_work(a, scalar((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), w, s)) return;
  const int n_rows = s.nq * a.group;
  const float2 *stat = a.stat + row_number(a, w.head, s);
  const int64_t base = (int64_t)(w.seq * a.kv_heads + w.head) * ((int64_t)a.max_pages << a.page_shift);
  for (int ch = w.c0; ch < w.c1; ++ch) {
    const int key0 = ch * (32 * NT);
    bf16x8 kf[NT][D / 16];
    float acc[NT];
    int from[NT];      // the first row that sees the lane's key
    uint32_t mine = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int key = key0 + t * 32 + (lane & 31);
      const int64_t row = row_of(a, w.seq, w.head, key, s.nk);
      mine |= (row >= 0 ? 1u : 0u) << t;
      from[t] = first_query(a, s, key) * a.group;
      acc[t] = 0.f;
      Half<K, D> x;
      x.load(a, max(row, (int64_t)0), lane);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) kf[t][j] = x.fragment(j);
    }
    if (__builtin_amdgcn_ballot_w64(mine != 0) != 0) {
      // (a chunk's last key decides where blocks begin that all its keys are seen by)
      const int all_from = scalar(first_query(a, s, min(key0 + 32 * NT, s.nk) - 1)) * a.group;
      const int b0 = scalar(first_query(a, s, key0)) * a.group / (8 * RG);
      Query<D> next;
      if (b0 * (8 * RG) < n_rows) next.load(a, s, w.head, b0 * (8 * RG) + (lane & 31), n_rows, lane);
      for (int b = b0; b * (8 * RG) < n_rows; ++b) {
        const int row0 = b * (8 * RG);
        const Query<D> q = next;
        next.load(a, s, w.head, row0 + 8 * RG + (lane & 31), n_rows, lane);
        float ref[R], inv[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float2 o = stat[min(row0 + 8 * (r >> 2) + (r & 3) + 4 * h, n_rows - 1)];
          ref[r] = o.x;
          inv[r] = o.y;
        }
        if (row0 < all_from || row0 + 8 * RG > n_rows) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const f32x16 x = product<D>(q.f, kf[t]);
            const int lo = from[t] - row0 - 4 * h, hi = n_rows - row0 - 4 * h;
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const int i = 8 * (r >> 2) + (r & 3);
              const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.c, -ref[r])) * inv[r];
              acc[t] += i >= lo && i < hi ? p : 0.f;
            }
          }
        } else {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const f32x16 x = product<D>(q.f, kf[t]);
            float a0 = 0.f, a1 = 0.f;
#pragma unroll
            for (int r = 0; r < R; r += 2) {
              a0 = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.c, -ref[r])), inv[r], a0);
              a1 = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(x[r + 1], a.c, -ref[r + 1])), inv[r + 1], a1);
            }
            acc[t] += a0 + a1;
          }
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float sum = acc[t] + __shfl_xor(acc[t], 32, 64);
      const int key = key0 + t * 32 + (lane & 31);
      if (lane < 32 && key < s.nk) {
        const float had = a.mass_in ? a.mass_in[base + key] : 0.f;
        a.mass[base + key] = mine >> t & 1 ? had + sum : 0.f;
      }
    }
  }
}

// Keys' sums, many rows: S^T = K Q^T as in k_mass_rows, with the rows' references and divisors one to a lane and a sum for each of a lane's 16
// keys, which the lanes of a half put together when the last row is done.
template <Kind K, int D, int NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_mass_keys(Call a) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  Work w;
  Seq s;
  if (!find_work(a, scalar((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), w, s)) return;
  const int n_rows = s.nq * a.group;
  const float2 *stat = a.stat + row_number(a, w.head, s);
  const int64_t base = (int64_t)(w.seq * a.kv_heads + w.head) * ((int64_t)a.max_pages << a.page_shift);
  for (int ch = w.c0; ch < w.c1; ++ch) {
    const int key0 = ch * (32 * NT);
    bf16x8 kf[NT][D / 16];
    f32x16 acc[NT];
    uint64_t held[NT];      // by lanes, the first 32 of which have a key each
    uint32_t any = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int64_t row = row_of(a, w.seq, w.head, key0 + t * 32 + (lane & 31), s.nk);
      held[t] = __builtin_amdgcn_ballot_w64(row >= 0);
      any |= held[t] ? 1u << t : 0u;
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;
      Half<K, D> x;
      x.load(a, max(row, (int64_t)0), lane);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) kf[t][j] = x.fragment(j);
    }
    const int b0 = scalar(first_query(a, s, key0)) * a.group / 32, blocks = n_rows / 32;      // (whole ones)
    if (any && b0 * 32 < n_rows) {
      const int whole = (int)min((uint32_t)(scalar(first_query(a, s, min(key0 + 32 * NT, s.nk) - 1)) * a.group + 31) / 32u, (uint32_t)blocks + 1u);
      Query<D> next;
      float2 next_stat = stat[min(b0 * 32 + (lane & 31), n_rows - 1)];
      next.load(a, s, w.head, b0 * 32 + (lane & 31), n_rows, lane);
      auto block = [&](auto cut, int b) __attribute__((always_inline)) {
        const int row = b * 32 + (lane & 31);
        const Query<D> q = next;
        const float ref = next_stat.x, inv = next_stat.y;
        next_stat = stat[min(row + 32, n_rows - 1)];
        next.load(a, s, w.head, row + 32, n_rows, lane);
        const int lim = decltype(cut)::value && row < n_rows ? limit_of(a, s, row / a.group) : 0;      // keys that the lane's row sees

#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const f32x16 x = product<D>(kf[t], q.f);

          if (!(any >> t & 1)) continue;
          if constexpr (!decltype(cut)::value) {
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[t][r] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.c, -ref)), inv, acc[t][r]);
          } else {
            const int t0 = lim - (key0 + t * 32) - 4 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.c, -ref)) * inv;
              acc[t][r] += (r >> 2) * 8 + (r & 3) < t0 ? p : 0.f;
            }
          }
        }
      };
      int b = b0;
      for (; b < min(whole, blocks); ++b) block(std::true_type{}, b);
      for (; b < blocks; ++b) block(std::false_type{}, b);
      if (b * 32 < n_rows) block(std::true_type{}, b);      // (rows beyond the last see nothing)
    }
    // over the 32 lanes of a half: at each step a lane gives one half of its sums away and adds the other lane's to the half it keeps, so that
    // lane r of 16 ends with sum r
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x16 v = acc[t];
      auto halve = [&](auto step) __attribute__((always_inline)) {
        constexpr int kBit = decltype(step)::value;
        const bool up = lane & kBit;
#pragma unroll
        for (int r = 0; r < kBit; ++r) {
          float low = v[r], high = v[r + kBit];
          asm("" : "+v"(low), "+v"(high));      // (else one is taken by an index that the lane chooses: sixteen selections)
          v[r] = (up ? high : low) + __shfl_xor(up ? low : high, kBit, 64);
        }
      };
      halve(std::integral_constant<int, 8>{});
      halve(std::integral_constant<int, 4>{});
      halve(std::integral_constant<int, 2>{});
      halve(std::integral_constant<int, 1>{});
      const float sum = v[0] + __shfl_xor(v[0], 16, 64);
      const int r = lane & 15, i = 16 * (r >> 3) + 8 * (r >> 2 & 1) + 4 * h + (r & 3), key = key0 + t * 32 + i;
      if (!(lane & 16) && key < s.nk) {
        const float had = a.mass_in ? a.mass_in[base + key] : 0.f;
        a.mass[base + key] = held[t] >> i & 1 ? had + sum : 0.f;
      }
    }
  }
}

// ---------------------------------------------------------------------------------------
// Parts, divisors, normalised rows, scores: each as much as any call of up to n_q tokens takes, so that scratch for more serves fewer
static size_t parts_bytes(int64_t rows, int kv_heads, int64_t most_keys) {
  return align_up((size_t)std::min(rows * most_pieces(kv_heads, most_keys), std::max(kMostParts, rows)) * sizeof(float2), 256);
}
static size_t plan_bytes(int n_seq) { return n_seq > 64 ? 2 * align_up((size_t)(n_seq + 2) * sizeof(int), 256) : 0; }
static size_t packed_bytes(int64_t rows, int head_dim) { return align_up((size_t)rows * head_dim * 2, 256); }
static size_t stat_bytes(int64_t rows) { return align_up((size_t)rows * sizeof(float2), 256); }

size_t mass_ws_bytes(int n_q, int n_seq, int heads, int kv_heads, int head_dim, int dtype, int64_t most_keys) {
  const int64_t rows = (int64_t)n_q * heads, kept = std::min((int64_t)n_q, kept_tokens(n_seq, heads, kv_heads, head_dim, dtype, most_keys));
  return plan_bytes(n_seq) + parts_bytes(rows, kv_heads, most_keys) + stat_bytes(rows) + packed_bytes(rows, head_dim) +
         align_up((size_t)kept * heads * most_keys * sizeof(float), 256);
}

template <Kind K, int D>
static int launch_kind(const MassArgs &x, const Call &c, const Form &f, int *plan, hipStream_t st) {
  const double rows = (double)x.n_q * c.group / c.n_seq;
  const int64_t pairs = (int64_t)c.n_seq * c.kv_heads;
  constexpr int NR = D == 64 ? 8 : 4, NK = D == 64 ? 4 : 2;      // tiles of a chunk of the many rows' kernels (Form's cuts)
  const int64_t most = (int64_t)c.max_pages << c.page_shift;
  Call by_rows = c, by_keys = c;
  by_rows.cut = f.rows;
  by_rows.splits = f.splits;
  by_keys.cut = f.keys;
  by_keys.splits = 1;
  if (c.n_seq > 64) {
    int *const starts = plan, *const starts_keys = (int *)((char *)plan + plan_bytes(c.n_seq) / 2);
    k_mass_plan<<<dim3(1), 1024, 0, st>>>(by_rows, by_keys, starts, starts_keys);
    by_rows.cut.starts = starts;
    by_keys.cut.starts = starts_keys;
  }
  by_keys.rows_cut = by_rows.cut;
  // units at most: those aimed at and one for each sequence and head, and no more than there are chunks
  auto units = [&](const Call &y) {
    return std::min(y.cut.aim + pairs, pairs * ((most + y.cut.chunk - 1) / y.cut.chunk)) * y.splits;
  };
  // a wave to a unit
  auto walk = [&](auto kernel, const Call &y) {
    kernel<<<dim3((uint32_t)((units(y) + 3) / 4)), 256, 0, st>>>(y);
  };
  if (x.n_q > 0) {
    if (f.keep) f.eight ? walk(k_mass_rows_few<K, D, 1, true>, by_rows) : walk(k_mass_rows_few<K, D, 4, true>, by_rows);
    else if (f.few && f.eight) walk(k_mass_rows_few<K, D, 1, false>, by_rows);
    else if (f.few) {
      if constexpr (D == 128) walk(k_mass_rows_few<K, D, 4, false>, by_rows);
    } else {
      walk(k_mass_rows<K, D, NR>, by_rows);
    }
    const int64_t per_pair = std::max((int64_t)1, kAim / pairs);
    auto join = [&](auto kernel, int at_once) {
      const int side = (int)std::min(per_pair, ((int64_t)x.n_q * c.group + at_once - 1) / at_once);
      kernel<<<dim3((uint32_t)(pairs * side)), 256, 0, st>>>(by_rows, side);
    };
    if (!f.own) rows <= 64.0 ? join(k_mass_join<4>, 4) : join(k_mass_join<64>, 64);
  }
  const dim3 blocks((uint32_t)units(by_keys));
  if (f.own) {
    k_mass_add<true><<<blocks, 256, 0, st>>>(by_keys);
  } else if (f.keep) {
    k_mass_add<false><<<blocks, 256, 0, st>>>(by_keys);
  } else if (f.few && f.eight) {
    walk(k_mass_keys_few<K, D, 2, 1>, by_keys);
  } else if (f.few) {
    if constexpr (D == 128) walk(k_mass_keys_few<K, D, 2, 4>, by_keys);
  } else if (f.small_chunks) {
    walk(k_mass_keys<K, D, 1>, by_keys);
  } else {
    walk(k_mass_keys<K, D, NK>, by_keys);
  }
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

int launch_mass(const MassArgs &x, void *ws, hipStream_t st) {
  const int64_t most = (int64_t)x.cv.max_pages << x.cv.page_shift, rows = (int64_t)x.n_q * x.heads;
  const Form f = form_of(x.n_q, x.cv.n_seq, x.heads, x.cv.kv_heads, x.cv.head_dim, x.cv.dtype, most);
  Call c = {};
  char *at = (char *)ws;
  int *const plan = (int *)at;
  at += plan_bytes(x.cv.n_seq);
  c.part = (float2 *)at;
  at += parts_bytes(rows, x.cv.kv_heads, most);
  c.stat = (float2 *)at;
  at += stat_bytes(rows);
  c.q = x.q;
  c.q_stride = x.q_stride;
  c.kv_heads = x.cv.kv_heads;
  c.group = x.heads / x.cv.kv_heads;
  if (x.n_q > 0 && (x.qk_norm || !f.few)) {
    uint16_t *packed = (uint16_t *)at;
    const uint32_t grid = (uint32_t)((rows * (x.cv.head_dim / 8) + 255) / 256);
    if (x.cv.head_dim == 64) k_mass_pack<64><<<dim3(grid), 256, 0, st>>>(x.q, x.q_stride, x.n_q, c.kv_heads, c.group, x.qk_norm, packed);
    else k_mass_pack<128><<<dim3(grid), 256, 0, st>>>(x.q, x.q_stride, x.n_q, c.kv_heads, c.group, x.qk_norm, packed);
    c.q = packed;
    c.q_stride = 0;
  }
  at += packed_bytes(rows, x.cv.head_dim);
  if (f.scores) c.scores = (float *)at;
  c.q_off = x.q_off;
  c.kv_len = x.kv_len;
  c.n_q = x.n_q;
  c.n_seq = x.cv.n_seq;
  c.frame = x.frame;
  c.c = x.scale * 1.4426950408889634f;
  c.k = (const char *)x.k;
  c.k_scale = x.k_scale;
  c.table = x.cv.table;
  c.page_shift = x.cv.page_shift;
  c.n_pages = x.cv.n_pages;
  c.max_pages = x.cv.max_pages;
  c.mass_in = x.mass_in;
  c.mass = x.mass;
  auto by_dim = [&](auto kind) {
    constexpr Kind K = decltype(kind)::value;
    return x.cv.head_dim == 64 ? launch_kind<K, 64>(x, c, f, plan, st) : launch_kind<K, 128>(x, c, f, plan, st);
  };
  if (x.cv.dtype == LV_CACHE_BF16) return by_dim(std::integral_constant<Kind, Kind::BF16>{});
  if (x.cv.dtype == LV_CACHE_E4M3) return by_dim(std::integral_constant<Kind, Kind::E4M3>{});
  return by_dim(std::integral_constant<Kind, Kind::E2M1>{});
}

}  // namespace lv
