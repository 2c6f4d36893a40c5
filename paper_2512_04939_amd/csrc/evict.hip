// Eviction from a paged cache: of each sequence the pages that have drawn the least attention weight leave.
//
// Two kernels.  k_evict_sums reads the masses once, which bounds it (4 bytes per kv head and position), and sums them by page in 64 bits, so
// that no order of the sums makes two pages change places that are not equal to 2^-50.  k_evict_select finds, with one workgroup to
// a sequence, the page up to which they leave: by the bits of their sums, eleven at a time.
#include <algorithm>

#include "internal.h"
#include "common.h"

namespace lv {

namespace {

constexpr int kSpan = 256;       // positions that a workgroup sums at a time
constexpr int kBins = 2048;

__device__ __forceinline__ int used_columns(const EvictArgs &a, int s) {
  const int64_t len = max(a.kv_len[s], 0);
  return (int)min((len + (1 << a.page_shift) - 1) >> a.page_shift, (int64_t)a.max_pages);
}

// Doubles in their order as whole numbers, NaN above all others (a page whose mass is not known stays)
__device__ __forceinline__ uint64_t key_of(double v) {
  if (v != v) return ~(uint64_t)0;
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

}  // namespace

__global__ __launch_bounds__(1024) void k_evict_select(EvictArgs a, double *sums, uint64_t *keys) {
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int used = used_columns(a, s), per = max(1 << a.page_shift >> 8, 1);
  const int64_t len = min((int64_t)max(a.kv_len[s], 0), (int64_t)a.max_pages << a.page_shift);
  const int32_t *table = a.table + (int64_t)s * a.max_pages;
  sums += (int64_t)s * a.max_pages * per;
  keys += (int64_t)s * a.max_pages;
  __shared__ uint32_t bins[kBins];
  __shared__ int counts[16][2];
  __shared__ uint64_t ends[16][2];
  __shared__ int found[2];
  const int lo_col = min(a.first_pages, used), hi_col = max(used - min(a.last_pages, used), lo_col);

  // keys of the pages that may leave, how many these are, how many are held, the least and the largest key
  auto held_at = [&](int j) { return (uint32_t)table[j] < (uint32_t)a.n_pages; };
  int held = 0, open = 0;
  uint64_t lo = ~(uint64_t)0, hi = 0;
  for (int j = tid; j < used; j += 1024) {
    if (!held_at(j)) continue;
    ++held;
    if (j < lo_col || j >= hi_col) continue;
    ++open;
    double sum = 0.0;
    for (int i = 0; i < per; ++i)
      if (((int64_t)j << a.page_shift) + i * kSpan < len) sum += sums[(int64_t)j * per + i];
    const uint64_t k = key_of(sum);
    keys[j] = k;
    lo = min(lo, k);
    hi = max(hi, k);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    held += __shfl_xor(held, o, 64);
    open += __shfl_xor(open, o, 64);
    lo = min(lo, (uint64_t)__shfl_xor((unsigned long long)lo, o, 64));
    hi = max(hi, (uint64_t)__shfl_xor((unsigned long long)hi, o, 64));
  }
  if (lane == 0) {
    counts[wave][0] = held;
    counts[wave][1] = open;
    ends[wave][0] = lo;
    ends[wave][1] = hi;
  }
  __syncthreads();
  held = open = 0;
  for (int i = 0; i < 16; ++i) {
    held += counts[i][0];
    open += counts[i][1];
    lo = min(lo, ends[i][0]);
    hi = max(hi, ends[i][1]);
  }
  const int leave = max(min(held - max(a.keep[s], 0), open), 0);

  // the key up to which they leave: below `lo` all do, of those equal to it the first `ties`.  Every turn leaves a 2048th of the range.
  int ties = leave;
  if (leave > 0) {
    while (lo < hi) {
      const int width = 64 - __builtin_clzll(hi - lo), shift = max(width - 11, 0);
      for (int i = tid; i < kBins; i += 1024) bins[i] = 0;
      __syncthreads();
      for (int j = lo_col + tid; j < hi_col; j += 1024) {
        if (!held_at(j)) continue;
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
      if (before < ties && ties <= before + b0) {
        found[0] = 2 * tid;
        found[1] = before;
      } else if (before + b0 < ties && ties <= before + b0 + b1) {
        found[0] = 2 * tid + 1;
        found[1] = before + b0;
      }
      __syncthreads();
      const uint64_t at = lo + ((uint64_t)found[0] << shift);
      ties -= found[1];
      const uint64_t rest = ((uint64_t)1 << shift) - 1;
      hi = hi - at < rest ? hi : at + rest;
      lo = at;
      __syncthreads();
    }
  }

  __syncthreads();

  // columns in their order
  int tied = 0, gone = 0;
  int32_t *freed = a.freed + (int64_t)s * a.max_pages;
  for (int j0 = 0; j0 < a.max_pages; j0 += 1024) {
    const int j = j0 + tid;
    const bool mine = j < a.max_pages;
    const int id = mine ? table[j] : -1;
    bool leaves = false;
    if (j0 < hi_col && leave > 0) {       // (the same for all)
      const bool is_open = j >= lo_col && j < hi_col && (uint32_t)id < (uint32_t)a.n_pages;
      const uint64_t k = is_open ? keys[j] : ~(uint64_t)0;
      const uint64_t same = __builtin_amdgcn_ballot_w64(is_open && k == lo);
      if (lane == 0) counts[wave][0] = __popcll(same);
      __syncthreads();
      int t = tied + __popcll(same & (((uint64_t)1 << lane) - 1));
      for (int i = 0; i < 16; ++i) {
        t += i < wave ? counts[i][0] : 0;
        tied += counts[i][0];
      }
      leaves = is_open && (k < lo || (k == lo && t < ties));
      const uint64_t out = __builtin_amdgcn_ballot_w64(leaves);
      if (lane == 0) counts[wave][1] = __popcll(out);
      __syncthreads();
      int at = gone + __popcll(out & (((uint64_t)1 << lane) - 1));
      for (int i = 0; i < 16; ++i) {
        at += i < wave ? counts[i][1] : 0;
        gone += counts[i][1];
      }
      if (leaves) freed[at] = id;
    }
    if (mine) a.table_out[(int64_t)s * a.max_pages + j] = leaves ? -1 : id;
    if (mine && j >= leave) freed[j] = -1;
  }
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
  const int64_t spans = (((int64_t)a.max_pages << a.page_shift) + kSpan - 1) / kSpan;
  const int side = (int)std::max((int64_t)1, std::min(spans, (int64_t)(8192 / a.n_seq)));
  k_evict_sums<<<dim3((uint32_t)(side * (int64_t)a.n_seq)), 256, 0, st>>>(a, sums, side);
  k_evict_select<<<dim3((uint32_t)a.n_seq), 1024, 0, st>>>(a, sums, keys);
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

}  // namespace lv
