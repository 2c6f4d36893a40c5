// Eviction from a paged cache: of each sequence the pages that have drawn the least attention weight leave.
//
// Two kernels.  k_evict_sums reads the masses once, which bounds it (4 bytes per kv head and position), and sums them by page in 64 bits, so
// that no order of the sums makes two pages change places that are not equal to 2^-50.  k_evict_select finds, with one workgroup to
// a sequence, the page up to which they leave: by the bits of their sums, eleven at a time, until few are left.  32 sequences of up to 8588 pages of
// 16, 16 heads: 24 us for the sums (156 MB), 18 to select, where each step waits for the one before; 46 with all bits by turns.
#include <algorithm>

#include "internal.h"
#include "common.h"

namespace lv {

namespace {

constexpr int kSpan = 256;       // positions that a workgroup sums at a time
constexpr int kBins = 2048;
constexpr int kList = 128;       // keys that are compared one by one
constexpr int kOwnSums = 128;    // masses of a page (heads times positions) up to which k_evict_select sums them by itself, a thread to a page
constexpr int kLdsKeys = 16384;  // columns whose keys lie in LDS

__device__ __forceinline__ int used_columns(const EvictArgs &a, int s) {
  const int64_t len = max(a.kv_len[s], 0);
  return (int)min((len + (1 << a.page_shift) - 1) >> a.page_shift, (int64_t)a.max_pages);
}

// Doubles in their order as whole numbers, NaN above all others (a page whose mass is not known stays), and below the mark of a column that
// may not leave
__device__ __forceinline__ uint64_t key_of(double v) {
  if (v != v) return ~(uint64_t)1;
  v = v == 0.0 ? 0.0 : v;       // (-0)
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return b >> 63 ? ~b : b | (uint64_t)1 << 63;
}

}  // namespace

// A span's positions: four to a lane, heads by turns to the four waves, put together in a fixed order.  Pages of more than a span have
// several sums.
__global__ __launch_bounds__(256) void k_evict_sums(EvictArgs a, double *sums, int side) {
  const int s = blockIdx.x / (uint32_t)side, turn = blockIdx.x - s * (uint32_t)side;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t room = (int64_t)a.max_pages << a.page_shift, len = min((int64_t)max(a.kv_len[s], 0), room);
  const int per = max(1 << a.page_shift >> 8, 1);            // sums of a page
  const int pages = max(kSpan >> a.page_shift, 1);           // pages of a span
  __shared__ double part[4][64];
  for (int64_t p0 = (int64_t)turn * kSpan; p0 < len; p0 += (int64_t)side * kSpan) {
    const int64_t at = p0 + lane * 4;
    double sum = 0.0;
    if (at < len)
      for (int h = wave; h < a.kv_heads; h += 4) {
        const f32x4 v = *(const f32x4 *)(a.mass + ((int64_t)s * a.kv_heads + h) * room + at);
        sum += ((double)v.x + (at + 1 < len ? (double)v.y : 0.0)) + ((at + 2 < len ? (double)v.z : 0.0) + (at + 3 < len ? (double)v.w : 0.0));
      }
    part[wave][lane] = sum;
    __syncthreads();
    if (threadIdx.x < 64) part[0][lane] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    __syncthreads();
    const int lanes = 64 / pages;
    if ((int)threadIdx.x < pages && p0 + threadIdx.x * lanes * 4 < len) {
      double all = 0.0;
      for (int i = 0; i < lanes; ++i) all += part[0][threadIdx.x * lanes + i];
      // (a span that begins inside a page: one page, and one of its sums)
      sums[((int64_t)s * a.max_pages * per) + (per > 1 ? p0 >> 8 : (p0 >> a.page_shift) + threadIdx.x)] = all;
    }
    __syncthreads();
  }
}

namespace {

__device__ __forceinline__ int wave_prefix(int v, int lane) {     // up to the lane
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(v, o, 64);
    v += lane >= o ? x : 0;
  }
  return v;
}
__device__ __forceinline__ uint64_t lower(uint64_t a, uint64_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint64_t higher(uint64_t a, uint64_t b) { return a > b ? a : b; }

}  // namespace

// LDS: the keys lie there and not in the workspace.  OWN: it sums the masses itself.
template <bool LDS, bool OWN>
__global__ __launch_bounds__(1024) void k_evict_select(EvictArgs a, const double *sums, uint64_t *room) {
  extern __shared__ uint64_t keys_lds[];
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int used = used_columns(a, s), per = max(1 << a.page_shift >> 8, 1);
  const int64_t len = min((int64_t)max(a.kv_len[s], 0), (int64_t)a.max_pages << a.page_shift);
  const int32_t *table = a.table + (int64_t)s * a.max_pages;
  sums += (int64_t)s * a.max_pages * per;
  uint64_t *const keys = LDS ? keys_lds : room + (int64_t)s * a.max_pages;
  __shared__ uint32_t bins[kBins];
  __shared__ int counts[16][2], found[2], listed;
  __shared__ uint64_t ends[16][2], list[kList], at_last;
  const int lo_col = min(a.first_pages, used), hi_col = max(used - min(a.last_pages, used), lo_col);

  // keys of the pages that may leave (all bits set: may not), how many these are, how many are held, the least and the largest key.  Four
  // columns' loads are on the way together.
  int held = 0, open = 0;
  uint64_t lo = ~(uint64_t)0, hi = 0;
  for (int j0 = tid; j0 < used; j0 += 4 * 1024) {
    int ids[4];
    double mass[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = min(j0 + i * 1024, used - 1);
      ids[i] = table[j];
      if constexpr (!OWN) mass[i] = sums[(int64_t)j * per];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = j0 + i * 1024;
      if (j >= used) break;
      const bool is_held = (uint32_t)ids[i] < (uint32_t)a.n_pages, is_open = is_held && j >= lo_col && j < hi_col;
      uint64_t k = ~(uint64_t)0;
      held += is_held;
      if (is_open) {
        double sum = 0.0;
        if constexpr (OWN) {
          const int64_t room = (int64_t)a.max_pages << a.page_shift, first = (int64_t)j << a.page_shift;
          const int n = (int)min(len - first, (int64_t)1 << a.page_shift);
          for (int h = 0; h < a.kv_heads; ++h) {
            const float *p = a.mass + ((int64_t)s * a.kv_heads + h) * room + first;
#pragma unroll 4
            for (int x = 0; x < 1 << a.page_shift; x += 4) {
              const f32x4 v = *(const f32x4 *)(p + x);
              sum += ((x < n ? (double)v.x : 0.0) + (x + 1 < n ? (double)v.y : 0.0)) + ((x + 2 < n ? (double)v.z : 0.0) + (x + 3 < n ? (double)v.w : 0.0));
            }
          }
        } else {
          sum = mass[i];
          for (int x = 1; x < per; ++x)
            if (((int64_t)j << a.page_shift) + x * kSpan < len) sum += sums[(int64_t)j * per + x];
        }
        k = key_of(sum);
        lo = lower(lo, k);
        hi = higher(hi, k);
        ++open;
      }
      keys[j] = k;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    held += __shfl_xor(held, o, 64);
    open += __shfl_xor(open, o, 64);
    lo = lower(lo, (uint64_t)__shfl_xor((unsigned long long)lo, o, 64));
    hi = higher(hi, (uint64_t)__shfl_xor((unsigned long long)hi, o, 64));
  }
  if (lane == 0) {
    counts[wave][0] = held;
    counts[wave][1] = open;
    ends[wave][0] = lo;
    ends[wave][1] = hi;
  }
  if (tid == 0) listed = 0;
  __syncthreads();
  held = open = 0;
  for (int i = 0; i < 16; ++i) {
    held += counts[i][0];
    open += counts[i][1];
    lo = lower(lo, ends[i][0]);
    hi = higher(hi, ends[i][1]);
  }
  const int leave = max(min(held - max(a.keep[s], 0), open), 0);
  __syncthreads();

  // the key up to which they leave: below `lo` all do, of those equal to it the first `ties`.  A turn leaves a 2048th of the range; once
  // its keys fit a list, each is compared with all others there.
  int ties = leave, inside = open;      // keys in lo .. hi
  if (leave > 0) {
    while (lo < hi && inside > kList) {
      const int shift = max(64 - __builtin_clzll(hi - lo) - 11, 0);
      for (int i = tid; i < kBins; i += 1024) bins[i] = 0;
      __syncthreads();
      for (int j = lo_col + tid; j < hi_col; j += 1024) {
        const uint64_t k = keys[j];
        if (k >= lo && k <= hi) atomicAdd(&bins[(k - lo) >> shift], 1u);
      }
      __syncthreads();
      // two bins to a thread; the one in which the count passes `ties`
      const int b0 = (int)bins[2 * tid], b1 = (int)bins[2 * tid + 1];
      const int upto = wave_prefix(b0 + b1, lane);
      if (lane == 63) counts[wave][0] = upto;
      __syncthreads();
      int before = upto - b0 - b1;
      for (int i = 0; i < wave; ++i) before += counts[i][0];
      if (before < ties && ties <= before + b0 + b1) {
        const bool second = ties > before + b0;
        found[0] = 2 * tid + second;
        found[1] = second ? before + b0 : before;
      }
      __syncthreads();
      inside = (int)bins[found[0]];
      ties -= found[1];
      lo += (uint64_t)found[0] << shift;
      const uint64_t rest = ((uint64_t)1 << shift) - 1;
      hi = hi - lo < rest ? hi : lo + rest;
      __syncthreads();
    }
    if (lo < hi) {
      for (int j = lo_col + tid; j < hi_col; j += 1024) {
        const uint64_t k = keys[j];
        if (k >= lo && k <= hi) list[atomicAdd(&listed, 1)] = k;
      }
      __syncthreads();
      if (tid < inside) {
        const uint64_t k = list[tid];
        int less = 0, same = 0;
        for (int i = 0; i < inside; ++i) {
          less += list[i] < k;
          same += list[i] == k;
        }
        if (less < ties && ties <= less + same) {      // (all that are equal write the same)
          at_last = k;
          found[1] = less;
        }
      }
      __syncthreads();
      lo = at_last;
      ties -= found[1];
    }
  }

  // columns in their order: a wave has a run of them, and counts first
  const int32_t *const from = table;
  int32_t *const to = a.table_out + (int64_t)s * a.max_pages, *const freed = a.freed + (int64_t)s * a.max_pages;
  if (leave > 0) {
    const int run = (used + 1023) / 1024 * 64, j0 = wave * run;
    int less = 0, same = 0;
    for (int j = j0 + lane; j < j0 + run; j += 64) {
      const uint64_t k = j < used ? keys[j] : ~(uint64_t)0;
      less += __popcll(__builtin_amdgcn_ballot_w64(k < lo));
      same += __popcll(__builtin_amdgcn_ballot_w64(k == lo));
    }
    if (lane == 0) {
      counts[wave][0] = less;
      counts[wave][1] = same;
    }
    __syncthreads();
    int tied = 0, gone = 0;
    for (int i = 0; i < wave; ++i) {
      gone += counts[i][0] + min(max(ties - tied, 0), counts[i][1]);
      tied += counts[i][1];
    }
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    for (int jj = j0 + lane; jj < j0 + run; jj += 4 * 64) {
      int ids[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) ids[i] = from[min(jj + i * 64, used - 1)];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = jj + i * 64;
        const uint64_t k = j < min(j0 + run, used) ? keys[j] : ~(uint64_t)0;
        const uint64_t equal = __builtin_amdgcn_ballot_w64(k == lo);
        const bool leaves = k < lo || (k == lo && tied + __popcll(equal & below) < ties);
        const uint64_t out = __builtin_amdgcn_ballot_w64(leaves);
        if (leaves) freed[gone + __popcll(out & below)] = ids[i];
        if (j < min(j0 + run, used)) to[j] = leaves ? -1 : ids[i];
        tied += __popcll(equal);
        gone += __popcll(out);
      }
    }
  }
  for (int j = (leave > 0 ? used : 0) + tid; j < a.max_pages; j += 1024) to[j] = from[j];
  for (int j = leave + tid; j < a.max_pages; j += 1024) freed[j] = -1;
  if (tid == 0) a.n_freed[s] = leave;
}

size_t evict_ws_bytes(int n_seq, int page_shift, int max_pages) {
  const int per = std::max(1 << page_shift >> 8, 1);
  return align_up((size_t)n_seq * max_pages * per * sizeof(double), 256) + align_up((size_t)n_seq * max_pages * sizeof(uint64_t), 256);
}

int launch_evict(const EvictArgs &a, void *ws, hipStream_t st) {
  const int per = std::max(1 << a.page_shift >> 8, 1);
  double *sums = (double *)ws;
  uint64_t *keys = (uint64_t *)((char *)ws + align_up((size_t)a.n_seq * a.max_pages * per * sizeof(double), 256));
  // one kernel for short caches (30 pages of 16, 8 heads 9.2 us, two kernels 11.5; 1000 pages 17.3 and 14.6)
  const bool own = a.max_pages <= 256 && (a.kv_heads << a.page_shift) <= kOwnSums;
  if (!own) {
    const int64_t spans = (((int64_t)a.max_pages << a.page_shift) + kSpan - 1) / kSpan;
    const int side = (int)std::max((int64_t)1, std::min(spans, (int64_t)(8192 / a.n_seq)));
    k_evict_sums<<<dim3((uint32_t)(side * (int64_t)a.n_seq)), 256, 0, st>>>(a, sums, side);
  }
  const size_t lds = (size_t)a.max_pages * sizeof(uint64_t);
  if (own) {
    k_evict_select<true, true><<<dim3((uint32_t)a.n_seq), 1024, lds, st>>>(a, sums, keys);
  } else if (a.max_pages <= kLdsKeys) {
    static std::atomic<uint64_t> done{0};
    const int rc = allow_dynamic_lds<kLdsKeys * sizeof(uint64_t)>((const void *)k_evict_select<true, false>, done);
    if (rc) return rc;
    k_evict_select<true, false><<<dim3((uint32_t)a.n_seq), 1024, lds, st>>>(a, sums, keys);
  } else {
    k_evict_select<false, false><<<dim3((uint32_t)a.n_seq), 1024, 0, st>>>(a, sums, keys);
  }
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

}  // namespace lv
