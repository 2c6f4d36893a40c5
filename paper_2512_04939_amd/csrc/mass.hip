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
// References, sums and masses are fp32; sums over rows and pieces have a fixed order.  q is rounded to bf16 after its normalisation, as
// K was before it was stored; nothing else is rounded below fp32.
#include <algorithm>

#include "internal.h"
#include "common.h"

namespace lv {

namespace {

constexpr float kUnset = -1e30f;             // reference of a row that has seen no key
constexpr float kRaise = 1.0995116e12f;      // 2^40: a sum beyond it raises the reference
constexpr int kNoKey = 0x7fff0000;           // the position of a key that is not there: beyond all that rows see

enum class Kind { BF16, E4M3, E2M1 };

struct Call {
  const uint16_t *q;
  int64_t q_stride;
  const int32_t *q_off, *kv_len;
  int n_q, n_seq, kv_heads, group, frame;
  float c;
  const char *k;
  const uint8_t *k_scale;
  const int32_t *table;
  int page_shift, n_pages, max_pages;
  int pieces, splits;      // of the key axis; of the rows
  int units;
  const float *mass_in;
  float *mass;
  float2 *part;            // [piece][kv head][token, head of the group]: reference, sum of weights
  float2 *stat;            // [kv head][token, head of the group]: reference, 1 / sum of weights
};

struct Seq {
  int q0, nq, nk, p0;      // its queries, its keys, the position of its first query
};

__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
// One number for all lanes, by a scalar load
__device__ __forceinline__ int uniform_at(const int32_t *p, int i) { return ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)p)[i]; }

__device__ __forceinline__ Seq seq_at(const Call &a, int s) {
  Seq r;
  const int len = max(uniform_at(a.kv_len, s), 0);
  r.q0 = min(max(uniform_at(a.q_off, s), 0), a.n_q);
  r.nq = min(max(uniform_at(a.q_off, s + 1), r.q0), a.n_q) - r.q0;
  r.nk = (int)min((int64_t)len, (int64_t)a.max_pages << a.page_shift);
  r.p0 = len - r.nq;
  return r;
}

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

template <int D>
struct Query {
  bf16x8 f[D / 16];
  __device__ __forceinline__ void load(const Call &a, const Seq &s, int head, int row, int n_rows, int lane) {
    const int r = min(row, n_rows - 1);
    const int i = (int)((uint32_t)r / (uint32_t)a.group), g = r - i * a.group;
    const uint16_t *p = a.q + (int64_t)(s.q0 + i) * a.q_stride + (int64_t)(head * a.group + g) * D + (lane >> 5) * (D / 2);
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

// The wave's part of the call: chunks of kc keys, `pieces` runs of them as long as the sequence's length makes them
__device__ __forceinline__ bool find_work(const Call &a, int unit, int kc, Work &w, Seq &s) {
  if (unit >= a.units) return false;
  const int x = scalar((int)((uint32_t)unit / (uint32_t)a.splits));
  w.split = scalar(unit - x * a.splits);
  const int y = scalar((int)((uint32_t)x / (uint32_t)a.pieces));
  w.piece = scalar(x - y * a.pieces);
  w.seq = scalar((int)((uint32_t)y / (uint32_t)a.kv_heads));
  w.head = scalar(y - w.seq * a.kv_heads);
  s = seq_at(a, w.seq);
  const int chunks = scalar((int)(((uint32_t)s.nk + kc - 1) / (uint32_t)kc)), per = scalar((int)((uint32_t)(chunks + a.pieces - 1) / (uint32_t)a.pieces));
  w.c0 = min(w.piece * per, chunks);
  w.c1 = min(w.c0 + per, chunks);
  return w.c0 < w.c1;
}

__device__ __forceinline__ int64_t row_number(const Call &a, int head, const Seq &s) { return ((int64_t)head * a.n_q + s.q0) * a.group; }

}  // namespace

// ---------------------------------------------------------------------------------------
// Rows' sums, many rows: S^T = K Q^T, a lane has one row and 16 of a tile's keys.  NT tiles of 32 keys stay in registers.  A row's sum over
// the keys of a wave's piece is kept in `part`: chunks after the first add to it.
template <Kind K, int D, int NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_mass_rows(Call a) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  Work w;
  Seq s;
  if (!find_work(a, scalar((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), 32 * NT, w, s)) return;
  const int n_rows = s.nq * a.group;
  if (n_rows == 0) return;
  // rows of this split, in blocks of 32, from the first that sees the piece's first key
  const int blocks = (n_rows + 31) / 32, per = scalar((int)((uint32_t)(blocks + a.splits - 1) / (uint32_t)a.splits));
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
    const int from = first_query(a, s, fresh ? w.c0 * (32 * NT) : key0) * a.group / 32;
    for (int b = max(from, w.split * per); b < b1; ++b) {
      const int row = b * 32 + (lane & 31);
      Query<D> q;
      q.load(a, s, w.head, row, n_rows, lane);
      const int lim = limit_of(a, s, min(row, n_rows - 1) / a.group);
      const int first = scalar(limit_of(a, s, b * 32 / a.group));      // keys that every row of the block sees
      float ref = kUnset, l = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t held = there >> (2 * t) & 3u;
        if (held == 0) continue;
        f32x16 x = product<D>(kf[t], q.f);
        const int k0 = key0 + t * 32;
        if (held != 3u || k0 + 32 > first) {
          const int t0 = lim - (held & 1u ? k0 : kNoKey) - 4 * h, t1 = lim - (held & 2u ? k0 + 16 : kNoKey) - 4 * h;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((r >> 2 & 1) * 8 + (r & 3) >= (r < 8 ? t0 : t1)) x[r] = -INFINITY;
        }
        float sum;
        auto weights = [&]() __attribute__((always_inline)) {
          float s0 = 0.f, s1 = 0.f;
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
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
    }
    fresh = false;
  }
}

// ---------------------------------------------------------------------------------------
// Rows' sums, up to 32 rows: S = Q K^T, a lane has one key of a tile and 4 RG of the rows, and sums of its own until the piece's end.
template <Kind K, int D, int RG>
__global__ __launch_bounds__(256) void k_mass_rows_few(Call a) {
  constexpr int R = 4 * RG;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  Work w;
  Seq s;
  if (!find_work(a, scalar((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), 32, w, s)) return;
  const int n_rows = s.nq * a.group;
  if (n_rows == 0) return;
  // blocks of 32 rows (8 RG of which are looked at; more than one block where sequences are of unlike lengths)
  for (int row0 = 0; row0 < n_rows; row0 += 8 * RG) {
    Query<D> q;
    q.load(a, s, w.head, row0 + (lane & 31), n_rows, lane);
    float l[R], ref[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      l[r] = 0.f;
      ref[r] = kUnset;
    }
    for (int ch = w.c0; ch < w.c1; ++ch) {
      const int key = ch * 32 + (lane & 31);
      const int64_t at = row_of(a, w.seq, w.head, key, s.nk);
      if (__builtin_amdgcn_ballot_w64(at >= 0) == 0) continue;
      Half<K, D> x;
      x.load(a, max(at, (int64_t)0), lane);
      bf16x8 kf[D / 16];
#pragma unroll
      for (int j = 0; j < D / 16; ++j) kf[j] = x.fragment(j);
      const f32x16 y = product<D>(q.f, kf);
      // the lane's key counts for rows from this one on
      const int from = at >= 0 ? first_query(a, s, key) * a.group - row0 - 4 * h : kNoKey;
      float v[R], top = 0.f;
      bool high = false;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        v[r] = 8 * (r >> 2) + (r & 3) >= from ? y[r] : -INFINITY;
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(v[r], a.c, -ref[r]));
        top = l[r] + p;
        high = high || !(top <= kRaise);
      }
      if (__builtin_amdgcn_ballot_w64(high) != 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float to = fmaxf(ref[r], v[r] * a.c);
          l[r] *= __builtin_amdgcn_exp2f(ref[r] - to);
          ref[r] = to;
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) l[r] += __builtin_amdgcn_exp2f(__builtin_fmaf(v[r], a.c, -ref[r]));
    }
    float2 *part = a.part + (int64_t)w.piece * a.kv_heads * a.n_q * a.group + row_number(a, w.head, s) + row0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float to = ref[r];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor(to, o, 64));
      float sum = l[r] * __builtin_amdgcn_exp2f(ref[r] - to);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      const int row = 8 * (r >> 2) + (r & 3) + 4 * h;
      if ((lane & 31) == 0 && row0 + row < n_rows) part[row] = float2{to, sum};
    }
  }
}

// ---------------------------------------------------------------------------------------
// The sums of a row's pieces put together, always in the same order; LANES of them take every LANES-th piece.
template <int LANES>
__global__ __launch_bounds__(256) void k_mass_join(Call a, int kc, int side) {
  const int pair = scalar((int)(blockIdx.x / (uint32_t)side)), turn = scalar((int)(blockIdx.x - pair * (uint32_t)side));
  const int seq = scalar((int)((uint32_t)pair / (uint32_t)a.kv_heads)), head = scalar(pair - seq * a.kv_heads);
  const Seq s = seq_at(a, seq);
  const int n_rows = s.nq * a.group, lane = threadIdx.x % LANES;
  const int chunks = (int)(((uint32_t)s.nk + kc - 1) / (uint32_t)kc), per = (int)((uint32_t)(chunks + a.pieces - 1) / (uint32_t)a.pieces);
  const int64_t all = (int64_t)a.kv_heads * a.n_q * a.group, base = row_number(a, head, s);
  for (int row = turn * (256 / LANES) + threadIdx.x / LANES; row < n_rows; row += side * (256 / LANES)) {
    const int lim = limit_of(a, s, row / a.group);
    const int seen = per ? (int)(((uint32_t)lim + (uint32_t)(per * kc) - 1) / (uint32_t)(per * kc)) : 0;      // pieces that it sees
    float ref = kUnset, l = 0.f;
    for (int p = lane; p < seen; p += LANES) {
      const float2 o = a.part[p * all + base + row];
      const float to = fmaxf(ref, o.x);
      l = l * __builtin_amdgcn_exp2f(ref - to) + o.y * __builtin_amdgcn_exp2f(o.x - to);
      ref = to;
    }
    if constexpr (LANES == 64) {
      float to = ref;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor(to, o, 64));
      l = wave_sum(l * __builtin_amdgcn_exp2f(ref - to));
      ref = to;
    }
    if (lane == 0) a.stat[base + row] = float2{ref, l == 0.f ? 0.f : 1.0f / l};
  }
}

// ---------------------------------------------------------------------------------------
// Keys' sums: S = Q K^T, a lane has one key of each of NT tiles and 4 RG of a block's rows, whose references and divisors are in its
// registers, the same for all lanes of a half.
template <Kind K, int D, int NT, int RG>
__global__ __launch_bounds__(256) void k_mass_keys(Call a) {
  constexpr int R = 4 * RG;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  Work w;
  Seq s;
  if (!find_work(a, scalar((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), 32 * NT, w, s)) return;
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
      for (int b = scalar(first_query(a, s, key0)) * a.group / (8 * RG); b * (8 * RG) < n_rows; ++b) {
        const int row0 = b * (8 * RG);
        Query<D> q;
        q.load(a, s, w.head, row0 + (lane & 31), n_rows, lane);
        float ref[R], inv[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float2 o = stat[min(row0 + 8 * (r >> 2) + (r & 3) + 4 * h, n_rows - 1)];
          ref[r] = o.x;
          inv[r] = o.y;
        }
        const bool cut = row0 < all_from || row0 + 8 * RG > n_rows;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const f32x16 x = product<D>(q.f, kf[t]);
          float p[R];
#pragma unroll
          for (int r = 0; r < R; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.c, -ref[r])) * inv[r];
          if (cut) {
            const int lo = from[t] - row0 - 4 * h, hi = n_rows - row0 - 4 * h;
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const int i = 8 * (r >> 2) + (r & 3);
              p[r] = i >= lo && i < hi ? p[r] : 0.f;
            }
          }
#pragma unroll
          for (int r = 0; r < R; ++r) acc[t] += p[r];
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

// ---------------------------------------------------------------------------------------
namespace {

constexpr int kAim = 4096;                             // waves to aim at: two rounds of eight a CU
constexpr int64_t kMostParts = (int64_t)1 << 24;       // (row, piece) pairs in the workspace, where rows leave a choice

struct Form {
  int pieces, splits;      // k_mass_rows*
  int key_pieces;          // k_mass_keys
};
Form form_of(int n_q, int n_seq, int heads, int kv_heads, int64_t most_keys) {
  Form f;
  const int64_t pairs = (int64_t)n_seq * kv_heads, rows = std::max((int64_t)n_q, (int64_t)1) * heads;
  const int64_t most = (most_keys + 31) / 32;
  const int64_t aim = std::max((int64_t)1, std::min((kAim + pairs - 1) / pairs, most));
  f.key_pieces = (int)aim;
  f.pieces = (int)std::max((int64_t)1, std::min(aim, kMostParts / rows));
  f.splits = (int)std::max((int64_t)1, kAim / (pairs * f.pieces));
  return f;
}
size_t parts_bytes(int64_t rows, int64_t aim) { return (size_t)std::min(rows * aim, std::max(kMostParts, rows)) * sizeof(float2); }

}  // namespace

size_t mass_ws_bytes(int n_q, int n_seq, int heads, int kv_heads, int head_dim, int64_t most_keys) {
  const Form f = form_of(n_q, n_seq, heads, kv_heads, most_keys);
  const int64_t rows = (int64_t)n_q * heads;
  return align_up(parts_bytes(rows, f.key_pieces), 256) + align_up((size_t)rows * sizeof(float2), 256) + align_up((size_t)rows * head_dim * 2, 256);
}

template <Kind K, int D>
static int launch_kind(const MassArgs &x, Call c, const Form &f, hipStream_t st) {
  const double rows = (double)x.n_q * c.group / c.n_seq;
  const int64_t pairs = (int64_t)c.n_seq * c.kv_heads;
  auto grid = [&]() { return dim3((uint32_t)((c.units + 3) / 4)); };
  constexpr int NR = D == 64 ? 8 : 4, NK = D == 64 ? 4 : 2;
  auto keys = [&]() -> int {
    c.pieces = f.key_pieces;
    c.splits = 1;
    c.units = (int)(pairs * c.pieces);
    if (rows <= 8.0) k_mass_keys<K, D, 2, 1><<<grid(), 256, 0, st>>>(c);
    else k_mass_keys<K, D, NK, 4><<<grid(), 256, 0, st>>>(c);
    LV_HIP_CHECK_LAUNCH();
    return LV_OK;
  };
  c.pieces = f.pieces;
  int kc = 32;
  if (x.n_q == 0) return keys();
  if (rows <= 32.0) {
    c.splits = 1;
    c.units = (int)(pairs * c.pieces);
    if (rows <= 8.0) k_mass_rows_few<K, D, 1><<<grid(), 256, 0, st>>>(c);
    else k_mass_rows_few<K, D, 4><<<grid(), 256, 0, st>>>(c);
  } else {
    kc = 32 * NR;
    c.splits = f.splits;
    c.units = (int)(pairs * c.pieces * c.splits);
    k_mass_rows<K, D, NR><<<grid(), 256, 0, st>>>(c);
  }
  const int64_t per_pair = std::max((int64_t)1, kAim / pairs);
  auto join = [&](auto kernel, int rows_at_once) {
    const int side = (int)std::min(per_pair, ((int64_t)x.n_q * c.group + rows_at_once - 1) / rows_at_once);
    kernel<<<dim3((uint32_t)(pairs * side)), 256, 0, st>>>(c, kc, side);
  };
  if (rows <= 64.0) join(k_mass_join<64>, 4);
  else join(k_mass_join<1>, 256);
  return keys();
}

int launch_mass(const MassArgs &x, void *ws, hipStream_t st) {
  const int64_t most = (int64_t)x.cv.max_pages << x.cv.page_shift, rows = (int64_t)x.n_q * x.heads;
  const Form f = form_of(x.n_q, x.cv.n_seq, x.heads, x.cv.kv_heads, most);
  Call c = {};
  c.part = (float2 *)ws;
  c.stat = (float2 *)((char *)ws + align_up(parts_bytes(rows, f.key_pieces), 256));
  c.q = x.q;
  c.q_stride = x.q_stride;
  if (x.qk_norm) {
    uint16_t *qn = (uint16_t *)((char *)c.stat + align_up((size_t)rows * sizeof(float2), 256));
    const int rc = launch_norm_rows(x.q, x.q_stride, x.n_q, x.heads, x.cv.head_dim, qn, st);
    if (rc) return rc;
    c.q = qn;
    c.q_stride = (int64_t)x.heads * x.cv.head_dim;
  }
  c.q_off = x.q_off;
  c.kv_len = x.kv_len;
  c.n_q = x.n_q;
  c.n_seq = x.cv.n_seq;
  c.kv_heads = x.cv.kv_heads;
  c.group = x.heads / x.cv.kv_heads;
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
    return x.cv.head_dim == 64 ? launch_kind<K, 64>(x, c, f, st) : launch_kind<K, 128>(x, c, f, st);
  };
  if (x.cv.dtype == LV_CACHE_BF16) return by_dim(std::integral_constant<Kind, Kind::BF16>{});
  if (x.cv.dtype == LV_CACHE_E4M3) return by_dim(std::integral_constant<Kind, Kind::E4M3>{});
  return by_dim(std::integral_constant<Kind, Kind::E2M1>{});
}

}  // namespace lv
