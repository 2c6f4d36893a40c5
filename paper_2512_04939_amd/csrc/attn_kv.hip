// Attention of the rows of one set over the keys of another: new tokens over a paged cache, queries over an encoder's states.
//
//   o_r = sum_t w_rt v_t / sum_t w_rt,   w_rt = exp2(c q_r.k_t - R_r),   c = scale * log2(e)
//
// for any reference R_r, in one pass over the keys: the reference of a row is raised, and what has been summed so far is
// scaled, when a sum passes 2^40 (a score lies 40 binades above the reference).  Sums and references are per row and fp32.
//
// A row is a (query token, head) pair; the heads that share a kv head are rows of one block, so K and V are read once for
// all of them.  Two kernels.  k_kv_attn_few: blocks of 32 or 64 rows whose four waves take 32 of every 128 keys each; bound by
// reading K and V (5.2 TB/s of 5.9 that a read alone reaches here, over 32 ragged sequences of an E4M3 cache).  k_kv_attn_many: blocks of
// 256 rows that walk the keys in stages of 64, which all waves read from LDS.  1.0 PFLOP/s for equal lengths, at 64 and at 128 channels (a
// library's product of 8192^3 reaches 1.37 on the same card), where MFMA is busy 55 and 56 % of the time.  At 64 channels a tile of 32 x 32
// costs 256 cycles of exp2 and some 170 of multiply-adds, sums and roundings against 256 of MFMA: instructions of the VALU, the
// products' issue among them, are active 80 % of a SIMD's cycles, and its two waves wait 37 % of theirs for a turn to issue and 13 % for data
// and barriers.  At 128 channels the VALU is active 56 %, the waves wait 36 and 25 %.  In
// both kernels a long key axis is cut into pieces that different workgroups take; k_kv_attn_join puts their sums together.
//
// Scores are computed transposed, S^T = K Q^T (32x32x16 MFMA, K as A operand): a lane owns one row's scores, and the
// weights already lie as the B operand of O^T += V^T P^T.  K and V lie in LDS as rows; V's fragments come out by transposing reads.
//
// Rounded to bf16: the weights, for the second product (their sum is that of the unrounded ones), q after its normalisation
// (as K was before it), and the result.  An E4M3 or E2M1 code times a power of two is a bf16 value: nothing is rounded there.  The scale is
// multiplied to the fp32 scores and not into q, where it would cost a rounding (7 % of the time at 64 channels).
#include <algorithm>

#include "internal.h"
#include "common.h"
#include "kv_plan.h"

namespace lv {

namespace {

constexpr int kGrp = 16;                 // rows of K or V that are fetched together; a page holds a multiple of it
constexpr int kUncut = 0x7fffffff;       // tiles of a piece where nothing is cut
constexpr int kNoKey = 0x7fff0000;       // the position of a key that is not there: beyond all that rows see
constexpr float kUnset = -1e30f;         // reference of a row that has seen no key
constexpr float kRowRaise = 1.0995116e12f;   // 2^40
constexpr int kCus = 256;
constexpr int kWholeTiles = 8;           // no call is cut whose sequences have fewer tiles: joining is a launch (8 or 16: level)
constexpr int kSide = 16;                // units side by side that one XCD takes, at most (find_work)
constexpr int kRounds = 3;               // a call's pieces fill the chip's slots at most so often

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

enum class Kv { ROWS, PAGES, E4M3, E2M1 };     // rows of another set; pages of bf16, of codes
template <Kv KV> constexpr bool kCoded = KV == Kv::E4M3 || KV == Kv::E2M1;                // codes that become bf16 on their way into LDS
template <Kv KV, int D> constexpr int kRowBytes = KV == Kv::E2M1 ? D / 2 : KV == Kv::E4M3 ? D : 2 * D;

template <Kv KV, int D, int QB> constexpr int kFewWaves = KV == Kv::E2M1 && D == 64 && QB == 1 ? 4 : 2;      // waves of a SIMD, few rows (by registers)

// What a kernel needs of the call, by value
struct Call {
  const uint16_t *q;
  uint16_t *o;
  int64_t q_stride, o_stride;
  const int32_t *q_off, *k_begin, *k_end;
  int n_q, n_seq, kv_heads, group, qk_norm, frame, n_kv;
  float c;
  const char *k, *v;
  int64_t k_stride, v_stride;            // bytes
  const uint8_t *k_scale, *v_scale;
  const int32_t *table;
  int page_shift, n_pages, max_pages;
  int rows_per_block, tile;              // rows of a block, keys of a tile (the unit of cutting): powers of two
  int block_shift, tile_shift;
  int target;                            // pieces to aim at; 0: nothing is cut
  int most_units;                        // units that there is room for
  int resident;                          // workgroups that the chip holds at once
  int *chosen;                           // tiles of a piece, units of the call: for the kernels that come after who works them out
  int *starts, *taken;                   // more than 64 sequences: units, slots before each (k_kv_attn_plan); else null
  float *part;                           // [slot][rows_per_block][D] sums
  float2 *part_ml;                       // [slot][rows_per_block] reference, sum of weights
  int slots;
};

__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct SeqInfo {
  int q0, nq, k0, nk;      // its queries, its keys
  int p0;                  // position of its first query
  int blocks, tiles;
};

__device__ __forceinline__ SeqInfo seq_of_numbers(const Call &a, int off, int next, int begin, int end) {
  SeqInfo r;
  r.q0 = min(max(off, 0), a.n_q);
  r.nq = min(max(next, r.q0), a.n_q) - r.q0;
  if (a.table) {
    const int64_t most = (int64_t)a.max_pages << a.page_shift;
    r.k0 = 0;
    r.nk = (int)min((int64_t)max(end, 0), most);
    r.p0 = max(end, 0) - r.nq;
  } else {
    r.k0 = min(max(begin, 0), a.n_kv);
    r.nk = min(max(end, r.k0), a.n_kv) - r.k0;
    r.p0 = 0;
  }
  r.blocks = (int)(((uint32_t)(r.nq * a.group) + a.rows_per_block - 1) >> a.block_shift);
  r.tiles = (int)(((uint32_t)r.nk + a.tile - 1) >> a.tile_shift);
  return r;
}
__device__ __forceinline__ SeqInfo seq_info(const Call &a, int s) {
  return seq_of_numbers(a, a.q_off[s], a.q_off[s + 1], a.table ? 0 : a.k_begin[s], a.k_end[s]);
}
// One number for all lanes, in a scalar register: it comes by a scalar load (what a vector load brings drags all that hangs on it into
// vector registers)
__device__ __forceinline__ int uniform_at(const int32_t *p, int i) { return ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)p)[i]; }
__device__ __forceinline__ SeqInfo uniform_seq(const Call &a, int s) {
  return seq_of_numbers(a, uniform_at(a.q_off, s), uniform_at(a.q_off, s + 1), a.table ? 0 : uniform_at(a.k_begin, s), uniform_at(a.k_end, s));
}

// Keys that the row of query i of a sequence sees (all up to this one)
__device__ __forceinline__ int limit_of(const Call &a, const SeqInfo &q, int i) {
  if (a.frame <= 0) return q.nk;
  const int p = q.p0 + i;
  if (p < 0) return 0;
  return (int)min((uint32_t)q.nk, ((uint32_t)p / (uint32_t)a.frame + 1u) * (uint32_t)a.frame);   // (below 2^32)
}

// Over the lanes by moves inside rows of 16 lanes, then from row to row: shuffles are LDS round trips, and a call's first 2 us were
// six of them for each reduction (cross attention of 4 x 16 rows over 1000 to 1500 keys: 13.1 us with shuffles, 11.1 so)
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t old, uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, kCtrl, 0xF, 0xF, false);
}
__device__ __forceinline__ uint32_t wave_min_u32(uint32_t v) {
  v = min(v, dpp_u32<0x128>(v, v));   // row_ror:8
  v = min(v, dpp_u32<0x124>(v, v));   // row_ror:4
  v = min(v, dpp_u32<0x4E>(v, v));    // quad_perm [2,3,0,1]
  v = min(v, dpp_u32<0xB1>(v, v));    // quad_perm [1,0,3,2]
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = min((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return (uint32_t)scalar((int)min((uint32_t)b[0], (uint32_t)b[1]));
}
// (sums up to the lane: row_shr 1, 2, 4, 8 where the lane there is one of the row; the rows' last lanes to the rows behind)
__device__ __forceinline__ int wave_prefix(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast:31 into rows 2 and 3
  return v;
}

// The sequence of the call that this lane looks at, of the first 64
__device__ __forceinline__ SeqInfo lane_seq(const Call &a, int lane) {
  SeqInfo q = {0, 0, 0, 0, 0, 0, 0};
  if (lane < a.n_seq) q = seq_info(a, lane);
  return q;
}

// One sequence whose blocks fill the chip's slots once or more: the blocks of its first heads, as many as fill whole rounds, are not
// cut, those of the others are, so that the last round is as full.
__device__ __forceinline__ int whole_heads(const Call &a, int blocks) {
  if (a.n_seq > 1 || blocks == 0 || a.target == 0) return 0;
  return min((int)((uint32_t)(blocks * a.kv_heads / a.resident * a.resident) / (uint32_t)blocks), a.kv_heads);
}

// How the keys are cut: the tiles of a piece.  Up to 64 sequences every wave works it out from the lengths, the same in all of them.  A
// candidate per lane: its pieces' number, and from that how long the call would take in tiles (rounds of the
// chip's slots, each as long as a piece and what a workgroup costs to start and end).  `me`: lane_seq(0); work: blocks times tiles of all
// sequences, most: the most tiles.
__device__ __forceinline__ int piece_tiles(const Call &a, int lane, const SeqInfo &me, float work, int most) {
  const int heads = a.n_seq > 1 ? a.kv_heads : scalar(a.kv_heads - whole_heads(a, me.blocks));
  work *= (float)heads;
  if (most <= 1 || work == 0.f) return kUncut;
  static_assert(kRounds == 3, "candidates");
  // lane 63: uncut; the others: 1 .. kRounds rounds, 21 steps of 4 % less pieces in each.  (A hair longer than the quotient: the
  // pieces are at most as many as were aimed at and one for each block, whatever the roundings.)
  const float pieces = (float)a.target * (float)(1 + lane / 21) / kRounds * (1.0f - 0.04f * (float)(lane % 21));
  const int s = lane == 63 ? most : (int)fminf((float)most, fmaxf(1.0f, ceilf(work / pieces * 1.0001f)));
  float units = 0.f;
  const float inv = 1.0f / (float)s;
  if (a.n_seq <= 16) {
    for (int i = 0; i < a.n_seq; ++i) {
      const int tiles = __builtin_amdgcn_readlane(me.tiles, i);
      units += (float)__builtin_amdgcn_readlane(me.blocks, i) * fmaxf(ceilf((float)tiles * inv - 1e-4f), 1.0f);
    }
    units *= (float)heads;
  } else {
    units = work * inv + 0.5f * (float)a.n_seq * (float)a.kv_heads;
  }
  // (a piece's sums are written and read: 8 tiles of many rows' time for the slots' 512 of 64 KB; 3 to 11 make no difference to speak of)
  const float cost = ceilf(units * (1.0f / (float)a.resident)) * (float)(min(s, most) + (s < most && a.rows_per_block > 64 ? 11 : 3)) + (s < most ? 6.f : 0.f);
  // the least, of equal ones the later (longer pieces)
  return __builtin_amdgcn_readlane(s, candidate_of(wave_min_u32(cost_key(cost, lane))));
}

__device__ __forceinline__ int piece_tiles(const Call &a, int lane, const SeqInfo &me) {
  if (a.target == 0) return kUncut;
  float work = (float)me.blocks * (float)me.tiles;
  int most = me.blocks ? me.tiles : 0;
  if (a.n_seq > 1) {
    work = wave_sum_ordered(work);
    most = (int)~wave_min_u32(~(uint32_t)most);
  } else {
    work = __builtin_bit_cast(float, scalar(__builtin_bit_cast(int, work)));
    most = scalar(most);
  }
  return piece_tiles(a, lane, me, work, most);
}

__device__ __forceinline__ int pieces_of(int tiles, int s) { return s == kUncut ? 1 : max((int)((uint32_t)(tiles + s - 1) / (uint32_t)s), 1); }
__device__ __forceinline__ int units_of(const Call &a, const SeqInfo &q, int s) { return q.blocks * a.kv_heads * pieces_of(q.tiles, s); }

// The slots of the workspace that a sequence takes: those of its pieces, if it is cut.  They are at most twice the pieces aimed at,
// however many sequences there are: who is cut has more tiles than a piece, so at most twice as many pieces as the quotient.
__device__ __forceinline__ int slots_taken(const Call &a, const SeqInfo &q, int s) { return pieces_of(q.tiles, s) > 1 ? units_of(a, q, s) : 0; }

struct Work {
  int seq, head, block, pieces;
  int t0, t1;      // its tiles
  int slot;
};

// Sum over the lanes before this one; total: over all
__device__ __forceinline__ int wave_scan(int v, int &total) {
  const int x = wave_prefix(v);
  total = __builtin_amdgcn_readlane(x, 63);
  return x - v;
}

// A lane's sequence, in all lanes
__device__ __forceinline__ SeqInfo from_lane(const SeqInfo &q, int j) {
  SeqInfo r;
  r.q0 = __builtin_amdgcn_readlane(q.q0, j);
  r.nq = __builtin_amdgcn_readlane(q.nq, j);
  r.k0 = __builtin_amdgcn_readlane(q.k0, j);
  r.nk = __builtin_amdgcn_readlane(q.nk, j);
  r.p0 = __builtin_amdgcn_readlane(q.p0, j);
  r.blocks = __builtin_amdgcn_readlane(q.blocks, j);
  r.tiles = __builtin_amdgcn_readlane(q.tiles, j);
  return r;
}

// The workgroup's piece of the call, in the order (sequence, head, piece, block): workgroups that read the same keys stand side by
// side, and up to 8 (several sequences) or 16 of them go to one XCD, whose L2 then brings K and V once.  (Many rows; each of
// them by itself in turn: 1374 queries over 138,774 keys 871 us against 835, 32 x 2000 over 4000 1109 against 1046, both 16 heads of 64;
// 1374 over 30,000 in pages, 16 heads of 128, 439 against 407.)
__device__ __forceinline__ bool find_work(const Call &a, int lane, Work &w, SeqInfo &info) {
  SeqInfo me;
  int s, total, whole = 0, start = 0, cut = 0, mine = 0, none;     // units of the call, and of these, ahead of the others, those that are not cut
  if (a.starts) {
    s = uniform_at(a.chosen, 0);
    total = uniform_at(a.chosen, 1);
  } else {
    me = lane_seq(a, lane);
    s = piece_tiles(a, lane, me);
    if (a.target && blockIdx.x == 0 && threadIdx.x == 0) *a.chosen = s;
    if (a.n_seq > 1) {
      mine = units_of(a, me, s);
      if (a.rows_per_block > 64 && a.n_seq <= 16) {
        // the sequences of the longest pieces first, so that short ones fill the last round (12 of 100 to 2000 queries over 100 to 15,000
        // keys 459 -> 449 us, 6 of 261 to 2088 over up to 20,097 417 -> 408; 64 of 70 to 400 over 100 to 2000 143 -> 160, by the loop itself)
        const int n = pieces_of(me.tiles, s), len = (int)((uint32_t)(me.tiles + n - 1) / (uint32_t)n);
        total = 0;
        for (int j = 0; j < a.n_seq; ++j) {
          const int units = __builtin_amdgcn_readlane(mine, j), longer = __builtin_amdgcn_readlane(len, j);
          start += longer > len || (longer == len && j < lane) ? units : 0;
          total += units;
        }
      } else {
        start = wave_scan(mine, total);
      }
      if (a.target) cut = wave_scan(slots_taken(a, me, s), none);
    } else {
      whole = scalar(whole_heads(a, me.blocks)) * scalar(me.blocks);
      total = scalar(whole + (me.blocks * a.kv_heads - whole) * pieces_of(me.tiles, s));
    }
  }
  // XCDs take turns with a few units that stand side by side
  const int side = a.rows_per_block <= 64 ? 1 : a.n_seq > 1 ? 8 : min(max(scalar(me.blocks), 1), kSide);
  const uint32_t y = blockIdx.x / kXcd, turn = y / (uint32_t)side;
  const int u = (int)((turn * kXcd + blockIdx.x % kXcd) * side + (y - turn * side));
  if (u >= total || u >= a.most_units) return false;
  int local = u;
  w.seq = 0;
  w.slot = u - whole;
  if (a.starts) {
    w.seq = scalar(max(last_at_most(a.starts, a.n_seq, u, lane), 0));
    info = uniform_seq(a, w.seq);
    local = u - uniform_at(a.starts, w.seq);
    w.slot = local + uniform_at(a.taken, w.seq);
  } else if (a.n_seq > 1) {
    const uint64_t hit = __builtin_amdgcn_ballot_w64(u >= start && u < start + mine);
    w.seq = scalar(__ffsll((unsigned long long)hit) - 1);
    info = from_lane(me, w.seq);
    local = u - __builtin_amdgcn_readlane(start, w.seq);
    w.slot = local + __builtin_amdgcn_readlane(cut, w.seq);
  } else {
    info = from_lane(me, 0);
  }
  w.pieces = u < whole ? 1 : scalar(pieces_of(info.tiles, s));
  // (offsets that do not ascend, lengths that changed meanwhile.  A second way out of the branches above costs four registers.)
  if (!unit_there(local, info.blocks * a.kv_heads * w.pieces, w.pieces > 1, w.slot, a.slots)) return false;
  const int skip = u < whole ? 0 : whole / info.blocks;     // heads
  local -= skip * info.blocks;
  const int len = w.pieces == 1 ? info.tiles : (int)((uint32_t)(info.tiles + w.pieces - 1) / (uint32_t)w.pieces);
  const int hp = (int)((uint32_t)local / (uint32_t)info.blocks);      // head and piece
  w.block = scalar(local - hp * info.blocks);
  const int head = w.pieces == 1 ? hp : (int)((uint32_t)hp / (uint32_t)w.pieces), piece = hp - head * w.pieces;
  w.head = skip + scalar(head);
  w.t0 = scalar(min(piece * len, info.tiles));
  w.t1 = min(w.t0 + scalar(len), info.tiles);
  return true;
}

// More than 64 sequences: one workgroup works out what the others would take long to, each for itself (one token for each of 1024
// sequences of 1000 keys, 16 heads on 4 of 128: 390 us so, 623 with every wave looking at all lengths; of 4096 of 250: 593 and
// 5204; of 256 of 1000: 107 and 121).  Sums in a fixed order.
__global__ __launch_bounds__(1024) void k_kv_attn_plan(Call a) {
  const int tid = threadIdx.x, lane = tid & 63, wave = scalar(tid >> 6);
  __shared__ float works[16];
  __shared__ int mosts[16], units[2][16], slots[2][16];
  int s = kUncut;
  if (a.target) {
    float work = 0.f;
    int most = 0;
    for (int i = tid; i < a.n_seq; i += 1024) {
      const SeqInfo q = seq_info(a, i);
      work += (float)q.blocks * (float)q.tiles;
      most = max(most, q.blocks ? q.tiles : 0);
    }
    work = wave_sum_ordered(work);
    most = (int)~wave_min_u32(~(uint32_t)most);
    if (lane == 0) {
      works[wave] = work;
      mosts[wave] = most;
    }
    __syncthreads();
    work = 0.f;
    most = 0;
    for (int i = 0; i < 16; ++i) {
      work += works[i];
      most = max(most, mosts[i]);
    }
    const SeqInfo none = {0, 0, 0, 0, 0, 0, 0};      // (read for 16 sequences and fewer only)
    s = piece_tiles(a, lane, none, work, most);
  }
  int before = 0, taken = 0;
  for (int b = 0; b < a.n_seq; b += 1024) {
    const int i = b + tid, turn = b >> 10 & 1;
    SeqInfo q = {0, 0, 0, 0, 0, 0, 0};
    if (i < a.n_seq) q = seq_info(a, i);
    int u, t;
    int at = wave_scan(share_of(units_of(a, q, s), a.most_units), u), slot = wave_scan(share_of(slots_taken(a, q, s), a.slots), t);
    if (lane == 0) {
      units[turn][wave] = share_of(u, a.most_units);
      slots[turn][wave] = share_of(t, a.slots);
    }
    __syncthreads();      // (the other of the two is read by nobody any more behind it)
    for (int x = 0; x < 16; ++x) {
      at += x < wave ? units[turn][x] : 0;
      slot += x < wave ? slots[turn][x] : 0;
    }
    if (i < a.n_seq) {
      a.starts[i] = start_of(before, at, a.most_units);
      a.taken[i] = start_of(taken, slot, a.slots);
    }
    for (int x = 0; x < 16; ++x) {
      before = start_of(before, units[turn][x], a.most_units);
      taken = start_of(taken, slots[turn][x], a.slots);
    }
  }
  if (tid == 0) {
    a.chosen[0] = s;
    a.chosen[1] = before;
  }
}

// ---------------------------------------------------------------------------------------
// Tiles in LDS: 32 keys, rows of D bf16 channels as they lie, their 16-byte pieces moved by an exclusive or with bits of
// the row so that neither the rows that 16 lanes read K fragments from nor the four that V's transposing reads take
// 64 bytes each from share banks.
template <int D>
struct Tile {
  static constexpr int kRow = D * 2;                  // bytes
  static constexpr int kPieces = D / 8;               // 16-byte pieces of a row
  static constexpr int kRowsPer = 64 / kPieces;       // rows that one fetch of a wave brings (1 KB)
  static constexpr int kFetches = kGrp / kRowsPer;    // fetches of a group of 16 rows
  static __device__ __forceinline__ int k_xor(int row) { return D == 64 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int v_xor(int row) { return D == 64 ? (row >> 1 & 1) * 4 : (row & 3) * 4; }
};

// 16-byte pieces from global memory straight into LDS at `lds` + 16 * lane.  What lies beyond the range of `rsrc` arrives
// as zeros.  Not waited for: vmcnt.  (The wait states are for a scalar register that a VALU instruction has just written.  The compiler
// takes no declaration of m0, which it keeps for itself: nothing else in these kernels may use it.)
__device__ __forceinline__ void fetch_lds(u32x4 rsrc, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane((int)lds)),
               "v"(off), "s"(rsrc)
               : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ u32x4 uniform_rsrc(const char *base, int bytes) {
  const uint64_t b = (uint64_t)base;
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b), (uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)),
               (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

// Where a group of 16 keys of one head lies: the first row of K and V, and the bytes of each that exist (0: none)
struct Group {
  const char *k, *v;
  int k_bytes, v_bytes;
  int64_t row;   // pages: rows before it
};

template <Kv KV, int D>
__device__ __forceinline__ Group group_at(const Call &a, int head, int k0, int key, int end, int page) {
  constexpr int row_bytes = kRowBytes<KV, D>;
  const int rows = min(scalar(max(end - key, 0)), kGrp);     // (in one they become a vector instruction, and all that hangs on it)
  Group g;
  if constexpr (KV == Kv::ROWS) {
    g.row = (int64_t)k0 + key;
    g.k = a.k + g.row * a.k_stride + head * row_bytes;
    g.v = a.v + g.row * a.v_stride + head * row_bytes;
    g.k_bytes = rows ? (int)((rows - 1) * a.k_stride) + row_bytes : 0;
    g.v_bytes = rows ? (int)((rows - 1) * a.v_stride) + row_bytes : 0;
  } else {
    const int64_t id = max(page, 0);
    g.row = ((id * a.kv_heads + head) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
    g.k = a.k + g.row * row_bytes;
    g.v = a.v + g.row * row_bytes;
    g.k_bytes = g.v_bytes = page >= 0 ? rows * row_bytes : 0;
  }
  return g;
}

// The page of position `key` (of a sequence's keys, which end before position `end`): -1 where it is none.  No branches: what is
// beyond the end looks at the table's last column.
__device__ __forceinline__ int page_at(const Call &a, int seq, uint32_t key, int end) {
  const int32_t *row = a.table + (int64_t)seq * a.max_pages;
  const int id = row[min(key >> a.page_shift, (uint32_t)a.max_pages - 1u)];
  return key < (uint32_t)end && (uint32_t)id < (uint32_t)a.n_pages ? id : -1;
}

// A lane's offsets from a group's first row (of K or of V) in its fetches, bf16: fetch j brings rows kRowsPer j .. and piece p ^ x(row), where
// x(row) = x(lane's row of fetch 0) ^ turn j.  They are worked out where they are used: kept, they cost the registers that 128
// channels have not got.
template <int D>
struct Offsets {
  uint32_t at;             // the row's bytes (a multiple of 16), and the number of the piece in the lowest four bits
  int step, turn;
  __device__ __forceinline__ void init(int lane, int64_t stride, bool of_v) {
    using T = Tile<D>;
    const int r = lane / T::kPieces, p = lane % T::kPieces;
    at = (uint32_t)(r * (int)stride) | (uint32_t)(p ^ (of_v ? T::v_xor(r) : T::k_xor(r)));
    step = T::kRowsPer * (int)stride;
    turn = of_v ? 0 : 4;
  }
};

// The group's rows on their way into LDS (bf16)
template <int D>
__device__ __forceinline__ void fetch_group(const char *p, int bytes, const Offsets<D> &off, uint32_t lds) {
  const u32x4 r = uniform_rsrc(p, bytes);
  uint32_t at = off.at;
  asm volatile("" : "+v"(at));
  const uint32_t row = at & ~15u, piece = at & 15u;
#pragma unroll
  for (int j = 0; j < Tile<D>::kFetches; ++j) fetch_lds(r, row + (uint32_t)(j * off.step) + (piece ^ (uint32_t)(j * off.turn)) * 16u, lds + j * 1024);
}

// A scalar buffer resource (in vector registers it becomes a loop over the lanes)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t scalar_rsrc(const void *p, int bytes) {
  const uint64_t b = (uint64_t)p;
  const uint64_t u = (uint32_t)scalar((int)(uint32_t)b) | (uint64_t)(uint32_t)scalar((int)(b >> 32)) << 32;
  return __builtin_amdgcn_make_buffer_rsrc((void *)u, 0, scalar(bytes), 0x00020000);
}

// E4M3: a group's codes and exponents (of K or of V) in registers, then as bf16 in LDS.  D = 64: one load of a wave has all 16 rows.
template <Kv KV, int D>
struct Codes {
  static constexpr int kLoads = D / 64, kPer = D / 16, kRows = 64 / kPer;   // loads; 16-byte pieces of a row, rows of a load
  u32x4 c[kLoads];
  uint32_t e[kLoads];
  __device__ __forceinline__ void load(const char *codes, const uint8_t *scales, const Group &g, int lane) {
    const __amdgpu_buffer_rsrc_t rc = scalar_rsrc(codes, g.k_bytes), rs = scalar_rsrc(scales + g.row, g.k_bytes / D);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      c[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, j * 1024 + lane * 16, 0, 0));
      e[j] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rs, j * kRows + lane / kPer, 0, 0);
    }
  }
  __device__ __forceinline__ void store(char *lds, bool of_v, int lane) const {
    using T = Tile<D>;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = j * kRows + lane / kPer, p = 2 * (lane % kPer), x = of_v ? T::v_xor(row) : T::k_xor(row);
      const float f = __uint_as_float(e[j] << 23);
      *(u32x4 *)(lds + row * T::kRow + ((p ^ x) * 16)) = dequant8(u32x2{c[j].x, c[j].y}, f);
      *(u32x4 *)(lds + row * T::kRow + (((p + 1) ^ x) * 16)) = dequant8(u32x2{c[j].z, c[j].w}, f);
    }
  }
};

// E2M1: four lanes to a row, all 16 rows in one load.  A lane has 16 (64 channels) or 32 consecutive channels, which share a scale.
template <int D>
struct Codes<Kv::E2M1, D> {
  static constexpr int kWords = D / 32;     // of codes; 16-byte pieces of bf16 that they become
  uint32_t c[kWords];
  uint32_t e;
  __device__ __forceinline__ void load(const char *codes, const uint8_t *scales, const Group &g, int lane) {
    const __amdgpu_buffer_rsrc_t rc = scalar_rsrc(codes, g.k_bytes), rs = scalar_rsrc(scales + g.row * (D / 32), g.k_bytes / 16);
    if constexpr (D == 64) {
      const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rc, lane * 8, 0, 0));
      c[0] = w.x;
      c[1] = w.y;
    } else {
      const u32x4 w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, lane * 16, 0, 0));
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = w[i];
    }
    e = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rs, D == 64 ? lane / 2 : lane, 0, 0);
  }
  __device__ __forceinline__ void store(char *lds, bool of_v, int lane) const {
    using T = Tile<D>;
    const int row = lane / 4, p = kWords * (lane % 4), x = of_v ? T::v_xor(row) : T::k_xor(row);
    const float f = __uint_as_float(e << 23);
    // In which order a lane writes its pieces: such that the eight lanes that write at once are in different banks
    const int turn = D == 64 ? row & 1 : (row & 1) * 2 | (lane >> 1 & 1);
    uint32_t w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; i += 2) {
      const uint32_t even = c[i], odd = c[i + 1], mask = turn & 1 ? even ^ odd : 0u;
      w[i] = even ^ mask;
      w[i + 1] = odd ^ mask;
    }
    if constexpr (kWords == 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t mask = turn & 2 ? w[i] ^ w[i + 2] : 0u;
        w[i] ^= mask;
        w[i + 2] ^= mask;
      }
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) *(u32x4 *)(lds + row * T::kRow + (((p + (i ^ turn)) ^ x) * 16)) = dequant8(w[i], f);
  }
};

// E2M1, few rows: codes and scales lie in LDS as they are held, in a ring of kSlots tiles of 32 keys a wave, on their way straight from memory.
// A slot: K's codes, V's, 256 bytes of K's scales, 256 of V's.  (A tile's codes are a quarter of bf16's bytes and take as long to compute with: waves
// count more than what each has on the way.  A token over 137,405 positions of 16 heads of 64: 61 us with the next tile's codes in registers and
// two waves to a SIMD, 57 with the ring, 50 with three waves, 46.5 with four; 32 over 301 to 30,011, 16 heads on 4 of 128, two waves: 76 and 73.)
template <int D>
struct Ring {
  static constexpr int kSlots = 2, kCodes = 32 * (D / 2), kScales = 32 * (D / 32);      // bytes of a tile's K or V
  static constexpr int kSlot = 2 * kCodes + 512, kBytes = kSlots * kSlot;
  static constexpr int kWhole = 2 * (D / 64) + 2, kApart = 8;      // fetches of a tile that lies in one page, and in two
};
// fetch_lds of 4 bytes a lane
__device__ __forceinline__ void fetch_lds4(u32x4 rsrc, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(off),
               "s"(rsrc)
               : "memory");
}

// ---------------------------------------------------------------------------------------
// A tile's K as E2M1 codes and scales: of the lane's key (lane % 32) half of the channels, (lane / 32) D / 2 on
template <int D, bool RAW>
struct RawKeys {};
template <int D>
struct RawKeys<D, true> {
  u32x4 kw[D / 64];
  uint32_t ke[D / 64];
};

// QB blocks of 32 rows of a wave.  RAW: K's fragments come from codes in registers, with the channels in the order in which a lane has them
// (any order will do that q has as well).
template <int D, int QB, bool RAW = false>
struct Rows : RawKeys<D, RAW> {
  bf16x8 q[QB][D / 16];
  f32x16 o[QB][D / 32];     // O^T: a lane's row, channels 32 dt + 8 (r / 4) + 4 h + r % 4
  float l[QB], ref[QB];     // sum of this lane half's weights, the row's reference (both halves the same)
  int lim[QB];              // keys the row sees

  // rows first .. first + 32 QB - 1 of the (sequence, kv head); those beyond n_rows repeat the last
  __device__ __forceinline__ void load(const Call &a, const SeqInfo &s, int head, int first, int lane) {
    const int n_rows = s.nq * a.group;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
      const int r = min(first + b * 32 + (lane & 31), n_rows - 1);
      const int i = (int)((uint32_t)r / (uint32_t)a.group), g = r - i * a.group;
      const uint16_t *p = a.q + (int64_t)(s.q0 + i) * a.q_stride + (int64_t)(head * a.group + g) * D + (lane >> 5) * (RAW ? D / 2 : 8);
      u32x4 w[D / 16];
#pragma unroll
      for (int j = 0; j < D / 16; ++j) w[j] = *(const u32x4 *)(p + (RAW ? 8 : 16) * j);
      if (a.qk_norm) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) ss += sumsq8(w[j]);
        ss += __shfl_xor(ss, 32, 64);
        const float f = 1.0f / sqrtf(ss * (1.0f / D) + kQkEps);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) w[j] = scale8(w[j], f);
      }
#pragma unroll
      for (int j = 0; j < D / 16; ++j) q[b][j] = __builtin_bit_cast(bf16x8, w[j]);
      lim[b] = limit_of(a, s, i);
      l[b] = 0.f;
      ref[b] = kUnset;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[b][dt][e] = 0.f;
    }
  }

  // block b's references are raised to the largest of a tile's scores, and what has been summed is scaled
  __device__ __forceinline__ void raise(int b, const f32x16 &s, float c) {
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float to = fmaxf(ref[b], top * c), f = __builtin_amdgcn_exp2f(ref[b] - to);
    ref[b] = to;
    l[b] *= f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[b][dt][r] *= f;
  }

  // one tile of 32 keys, 16 from key0 and 16 from key1 on, K and V rows at k_lds and v_lds; what is not held is zeros, its
  // keys are kNoKey.  cut: some row does not see some of the keys.
  __device__ __forceinline__ void tile(const char *k_lds, const char *v_lds, float c, int key0, int key1, bool cut, int lane) {
    using T = Tile<D>;
    const int h = lane >> 5, kr = lane & 31;
    f32x16 s[QB];
    {
      bf16x8 kf[D / 16];
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        if constexpr (RAW) kf[j] = __builtin_bit_cast(bf16x8, dequant8((uint32_t)this->kw[j / 4][j % 4], __uint_as_float(this->ke[j / 4] << 23)));
        else kf[j] = __builtin_bit_cast(bf16x8, *(const u32x4 *)(k_lds + kr * T::kRow + (((2 * j + h) ^ T::k_xor(kr)) * 16)));
      }
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        f32x16 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < D / 16; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j], q[b][j], acc, 0, 0, 0);
        s[b] = acc;
      }
    }
    // V fragments: [16 keys][32 channels], two halves of 8 keys each
    u32x4 vf[2][D / 32];
    {
      const int row = 4 * h + (lane >> 2 & 3);
      const char *p = v_lds + row * T::kRow + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        const char *pd = p + ((dt * 64) ^ (T::v_xor(row) * 16));
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(pd + u * 16 * T::kRow)));
          const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(pd + u * 16 * T::kRow + 8 * T::kRow)));
          vf[u][dt] = u32x4{x.x, x.y, y.x, y.y};
        }
      }
    }
    if (cut) {
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        const int t0 = lim[b] - key0 - 4 * h, t1 = lim[b] - key1 - 4 * h;       // the lane's keys below these count
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((r >> 2 & 1) * 8 + (r & 3) >= (r < 8 ? t0 : t1)) s[b][r] = -INFINITY;
      }
      // a weight of 0 times an infinity or NaN would reach rows that do not see that key: such entries are taken out
      // here and added to the rows that do
      typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
      u16x2 top = {0, 0};
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[u][dt][i] & 0x7fff7fffu));
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(top.x >= 0x7f80 || top.y >= 0x7f80) != 0, 0)) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t w = vf[u][dt][i];
              vf[u][dt][i] = w & ~(((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u));
            }
        add_wild(s, c, v_lds, key0, key1, lane);
      }
    }
#pragma unroll
    for (int b = 0; b < QB; ++b) {
      uint32_t w[8];
      float sum0, sum1;
      auto weights = [&]() __attribute__((always_inline)) {
        sum0 = sum1 = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][2 * e], c, -ref[b]));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][2 * e + 1], c, -ref[b]));
          w[e] = pack_bf16(p0, p1);
          asm("" : "+v"(w[e]));      // (where paths meet the pair would be carried unpacked, in twice the registers)
          sum0 += p0;
          sum1 += p1;
        }
      };
      weights();
      if (__builtin_amdgcn_ballot_w64(!(l[b] + (sum0 + sum1) <= kRowRaise)) != 0) {
        raise(b, s[b], c);
        weights();
      }
      l[b] += sum0 + sum1;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 p = __builtin_bit_cast(bf16x8, u32x4{w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]});
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          o[b][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[u][dt]), p, o[b][dt], 0, 0, 0);
      }
    }
  }

  // Entries of V that are not finite, to the rows that see their keys.  The references are raised before: to raise one scales what has
  // been summed, at a row's first tile by 0, and an infinity would become NaN.  (In the loop: ahead of it the compiler works it out for
  // every tile that is cut, and the loops around lose their registers to it.)
  __device__ __forceinline__ void add_wild(const f32x16 (&s)[QB], float c, const char *v_lds, int key0, int key1, int lane) {
    using T = Tile<D>;
    const int h = lane >> 5;
#pragma unroll 1
    for (int t = 0; t < 32; ++t) {
      if (t == 0) {
#pragma unroll
        for (int b = 0; b < QB; ++b) raise(b, s[b], c);
      }
      const int key = t < 16 ? key0 + t : key1 + t - 16;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int byte = (dt * 64 + i * 16 + h * 8) ^ (T::v_xor(t) * 16);
          const u32x2 w = *(const u32x2 *)(v_lds + t * T::kRow + byte);
          const float x[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = (__float_as_uint(x[e]) & 0x7f800000u) == 0x7f800000u ? x[e] : 0.f;
#pragma unroll
            for (int b = 0; b < QB; ++b) o[b][dt][4 * i + e] += key < lim[b] ? y : 0.f;
          }
        }
    }
  }
};

// ---------------------------------------------------------------------------------------
// Few rows.  A workgroup has 32 or 64 rows of a (sequence, kv head) and a piece of its keys, in tiles of 128: wave w takes the w-th 32
// keys of each, through LDS of its own, so nobody waits for anybody before the end.  bf16: two
// tiles in LDS, the next one on its way while one is computed with; E4M3: the next tile's codes on their way in registers, turned
// into bf16 in LDS.  Two workgroups per CU where LDS allows.  5 queries over 137,405 keys, 16 heads of 64, bf16: 99 us, 5.7 TB/s, and 5 to
// join; 32 tokens over 301 to 30,011 keys, 16 heads on 4 of 128, E4M3: 97 us, 5.2 TB/s, and 5 to join.  (Eight waves to a
// workgroup where there are few of them: 34.1 us against 32.0 for 24 rows over 30,000 keys, 17.2 against 14.4 for 48 over 2000.)
template <Kv KV, int D, int QB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kFewWaves<KV, D, QB>, kFewWaves<KV, D, QB>))) void k_kv_attn_few(Call a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  using T = Tile<D>;
  constexpr int kRows = 32 * QB;
  constexpr int kTile = 32 * T::kRow;          // bytes of a tile's K or V
  constexpr int kStages = kCoded<KV> ? 1 : 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Work w;
  SeqInfo s;
  if (!find_work(a, lane, w, s)) return;
  const int n_rows = s.nq * a.group, row0 = w.block * kRows;
  const int last = scalar(limit_of(a, s, min(row0 + kRows - 1, n_rows - 1) / a.group));     // keys that some row sees
  const int first = scalar(limit_of(a, s, row0 / a.group));                          // keys that every row sees
  const int begin = w.t0 * 128 + wave * 32, end = (int)min((uint32_t)w.t1 * 128u, (uint32_t)last);
  const int n = __builtin_amdgcn_readfirstlane(end > begin ? (end - begin + 127) / 128 : 0);     // the wave's tiles

  char *const mine = lds + wave * (2 * kStages * kTile);
  const uint32_t mine_at = __builtin_amdgcn_readfirstlane(lds_addr(mine));
  Offsets<D> ko, vo;
  if constexpr (!kCoded<KV>) {
    ko.init(lane, KV == Kv::ROWS ? a.k_stride : T::kRow, false);
    vo.init(lane, KV == Kv::ROWS ? a.v_stride : T::kRow, true);
  }
  int ids[2] = {0, 0};               // lane j: the pages of the two groups of tile j of 64
  uint64_t holes = 0;
  auto look_up = [&](int i) {        // tiles i .. i + 63
    if constexpr (KV != Kv::ROWS) {
      const uint32_t key = (uint32_t)begin + (uint32_t)(i + lane) * 128u;
      ids[0] = page_at(a, w.seq, key, end);
      ids[1] = page_at(a, w.seq, key + kGrp, end);
      holes = __builtin_amdgcn_ballot_w64((key < (uint32_t)end && ids[0] < 0) || (key + kGrp < (uint32_t)end && ids[1] < 0));
    }
  };
  Codes<KV, D> kc[2], vc[2];
  auto fetch = [&](int i) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int key = begin + i * 128 + g * kGrp;
      const int page = KV == Kv::ROWS ? 0 : __builtin_amdgcn_readlane(ids[g], i & 63);
      const Group at = group_at<KV, D>(a, w.head, s.k0, key, i < n ? end : 0, page);
      if constexpr (kCoded<KV>) {
        kc[g].load(at.k, a.k_scale, at, lane);
        vc[g].load(at.v, a.v_scale, at, lane);
      } else {
        const uint32_t to = mine_at + (i % kStages) * (2 * kTile) + g * kGrp * T::kRow;
        fetch_group<D>(at.k, at.k_bytes, ko, to);
        fetch_group<D>(at.v, at.v_bytes, vo, to + kTile);
      }
    }
  };
  Rows<D, QB, KV == Kv::E2M1> rows;
  if constexpr (KV == Kv::E2M1) {
    using R = Ring<D>;
    char *const ring = lds + wave * (R::kBytes + kTile), *const vt = ring + R::kBytes;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_addr(ring));
    uint32_t there = 0;       // bits 2 slot + g: group g of the slot's tile is held
    // What is not held arrives as zeros, and its keys are nobody's.  (Scales by words: with the last row's those of the row behind, in the same
    // page.)  Pages of 32 positions and more: a tile lies in one; else a half of the lanes
    // takes a group.
    const bool whole = a.page_shift > 4;
    auto fetch_raw = [&](int i) __attribute__((always_inline)) {
      if (i % 64 == 0) look_up(i);
      const int slot = i % R::kSlots, key = begin + i * 128;
      const uint32_t to = ring_at + slot * R::kSlot;
      int id[2], rows_of[2];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        id[g] = i < n ? __builtin_amdgcn_readlane(ids[g], i & 63) : -1;
        rows_of[g] = id[g] < 0 ? 0 : min(end - key - g * kGrp, kGrp);
      }
      there = (there & ~(3u << 2 * slot)) | ((id[0] < 0 ? 0u : 1u) | (id[1] < 0 ? 0u : 2u)) << 2 * slot;
      auto at = [&](int g) __attribute__((always_inline)) {
        return (((int64_t)max(id[g], 0) * a.kv_heads + w.head) << a.page_shift) + ((key + g * kGrp) & ((1 << a.page_shift) - 1));
      };
      if (whole) {
        const int64_t row = at(0);
        const int rows = rows_of[0] + rows_of[1];
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const u32x4 r = uniform_rsrc((v ? a.v : a.k) + row * (D / 2), rows * (D / 2));
#pragma unroll
          for (int x = 0; x < D / 64; ++x) fetch_lds(r, x * 1024 + lane * 16, to + v * R::kCodes + x * 1024);
          fetch_lds4(uniform_rsrc((const char *)(v ? a.v_scale : a.k_scale) + row * (D / 32), (rows * (D / 32) + 3) & ~3), lane * 4, to + 2 * R::kCodes + v * 256);
        }
      } else {
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const int64_t row = at(g);
            const u32x4 r = uniform_rsrc((v ? a.v : a.k) + row * (D / 2), rows_of[g] * (D / 2));
            const u32x4 rs = uniform_rsrc((const char *)(v ? a.v_scale : a.k_scale) + row * (D / 32), (rows_of[g] * (D / 32) + 3) & ~3);
            if constexpr (D == 64) {
              if (lane >> 5 == g) fetch_lds(r, (lane & 31) * 16, to + v * R::kCodes);
            } else {
              fetch_lds(r, lane * 16, to + v * R::kCodes + g * 1024);
            }
            if (lane / (D / 8) == g) fetch_lds4(rs, lane % (D / 8) * 4, to + 2 * R::kCodes + v * 256);
          }
      }
    };
    if (n > 0) {
#pragma unroll
      for (int i = 0; i < R::kSlots; ++i) fetch_raw(i);
    }
    rows.load(a, s, w.head, row0, lane);
    for (int i = 0; i < n; ++i) {
      const int slot = i % R::kSlots, kr = lane & 31, h = lane >> 5;
      const char *const at = ring + slot * R::kSlot, *const scales = at + 2 * R::kCodes;
      if (whole) wait_vm<(R::kSlots - 1) * R::kWhole>();
      else wait_vm<(R::kSlots - 1) * R::kApart>();
#pragma unroll
      for (int x = 0; x < D / 64; ++x) {
        rows.kw[x] = *(const u32x4 *)(at + kr * (D / 2) + h * (D / 4) + x * 16);
        rows.ke[x] = *(const uint8_t *)(scales + kr * (D / 32) + h * (D / 64) + x);
      }
      Codes<KV, D> vc[2];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int x = 0; x < D / 32; ++x) vc[g].c[x] = *(const uint32_t *)(at + R::kCodes + g * (kGrp * D / 2) + lane * (D / 8) + x * 4);
        vc[g].e = *(const uint8_t *)(scales + 256 + g * (R::kScales / 2) + (D == 64 ? lane / 2 : lane));
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      const uint32_t open = there >> 2 * slot & 3u;
      fetch_raw(i + R::kSlots);
      if (open == 0) continue;
#pragma unroll
      for (int g = 0; g < 2; ++g) vc[g].store(vt + g * kGrp * T::kRow, true, lane);
      const int key0 = begin + i * 128;
      rows.tile(nullptr, vt, a.c, open & 1u ? key0 : kNoKey, open & 2u ? key0 + kGrp : kNoKey, open != 3u || key0 + 32 > first, lane);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the tile has been read: its place may be filled again
    }
    wait_vm<0>();      // nothing may land where the sums will lie
  } else {
    if (n > 0) {      // (on its way while the rows come)
      look_up(0);
      fetch(0);
    }
    rows.load(a, s, w.head, row0, lane);
    if (n > 0) {
      uint64_t shut_now = holes;
      for (int i = 0; i < n; ++i) {
        char *kt = mine + (i % kStages) * (2 * kTile);
        int shut = 0;
        if (KV != Kv::ROWS && (shut_now >> (i & 63) & 1))
          shut = (__builtin_amdgcn_readlane(ids[0], i & 63) < 0 ? 1 : 0) | (__builtin_amdgcn_readlane(ids[1], i & 63) < 0 ? 2 : 0);
        if constexpr (kCoded<KV>) {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            kc[g].store(kt + g * kGrp * T::kRow, false, lane);
            vc[g].store(kt + kTile + g * kGrp * T::kRow, true, lane);
          }
        }
        if (i + 1 < n) {
          if ((i + 1) % 64 == 0) look_up(i + 1);
          fetch(i + 1);
          if constexpr (!kCoded<KV>) wait_vm<4 * T::kFetches>();
        } else if constexpr (!kCoded<KV>) {
          wait_vm<0>();
        }
        const int key0 = begin + i * 128;
        if (shut != 3)
          rows.tile(kt, kt + kTile, a.c, shut & 1 ? kNoKey : key0, shut & 2 ? kNoKey : key0 + kGrp, shut || key0 + 32 > first, lane);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the tile has been read: its place may be filled again
        shut_now = holes;
      }
    }
  }

  // the four waves' sums: [wave][row][D] and their references and sums of weights
  __syncthreads();
  float *po = (float *)lds;
  __shared__ float2 ml[4][kRows];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int r = b * 32 + (lane & 31);
    const float l = rows.l[b] + __shfl_xor(rows.l[b], 32, 64);
    if (lane < 32) ml[wave][r] = float2{rows.ref[b], l};
    float *p = po + (wave * kRows + r) * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = dt * 32 + i * 8 + (lane >> 5) * 4;
        *(f32x4 *)(p + (ch ^ ((lane & 15) * 4))) = f32x4{rows.o[b][dt][4 * i], rows.o[b][dt][4 * i + 1], rows.o[b][dt][4 * i + 2], rows.o[b][dt][4 * i + 3]};
      }
  }
  __syncthreads();
  for (int i = tid; i < kRows * (D / 4); i += 256) {
    const int r = i / (D / 4), ch = i % (D / 4) * 4;
    if (row0 + r >= n_rows) break;
    float top = ml[0][r].x;
#pragma unroll
    for (int x = 1; x < 4; ++x) top = fmaxf(top, ml[x][r].x);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = __builtin_amdgcn_exp2f(ml[x][r].x - top);
      const f32x4 y = *(const f32x4 *)(po + (x * kRows + r) * D + (ch ^ ((r & 15) * 4)));
      l += ml[x][r].y * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += y[e] * f;
    }
    if (w.pieces > 1) {
      const int64_t at = (int64_t)w.slot * kRows + r;
      *(f32x4 *)(a.part + at * D + ch) = sum;
      if (ch == 0) a.part_ml[at] = float2{top, l};
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;     // no key seen: zeros
      const int rr = row0 + r, tok = rr / a.group;
      uint16_t *p = a.o + (int64_t)(s.q0 + tok) * a.o_stride + (w.head * a.group + rr - tok * a.group) * D + ch;
      *(u32x2 *)p = u32x2{pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
    }
  }
}

// ---------------------------------------------------------------------------------------
// Many rows.  A workgroup has 256 rows and walks a piece of the keys in stages of 64 (four groups of 16).  bf16: a ring of four
// stages in LDS, filled straight from memory; E4M3: three stages of bf16 in LDS, the codes of the next one in registers.
//
// 64 channels: four waves of 64 rows, of which wave w fetches the w-th group of a stage.  A wave's two blocks of 32 rows run half a step
// apart, so that one's weights (VALU) are taken while the other's products (MFMA) run:
//   A(t): scores of block 1 (tile t) | K(t + 1) is read | output of block 1 (t - 1) | V(t) is read;  weights of block 0 (t)
//   B(t): scores of block 0 (t + 1), output of block 0 (t);                                          weights of block 1 (t)
// K's and V's fragments are read once for both blocks, half a phase before their first use, into the registers that the products
// before have just been issued from.
//
// 128 channels: a block of 32 rows fills the registers that two waves per SIMD have (64 rows and one wave per SIMD: 304 and more
// of 512, which the compiler does not divide without copies and spills).  Eight waves of 32 rows; wave w fetches K's (w even) or V's rows of group w / 2.
// Tiles take turns as the blocks do above:
//   C(t): scores (t + 1) | K(t + 2) is read | output (t - 1) | V(t) is read;  weights (t)
//
// No register may go to scratch in the loops: reading it back waits for the fetches (three times the time).
//
// Whole calls: 13,740 queries over 14,316 states, 16 heads of 64: 782 to 805 us (1.00 to 1.03 PFLOP/s), 28 of them to join; 1374 over 138,774
// keys in pages 835 (0.93), 19 to join; six chunks of 261 to 2088 over up to 20,097 keys in E4M3 pages, every seventh given back, 408 to 413
// (0.80), 17 to join; 3 to 701 queries over up to 6007 states, 16 heads on 2 of 128, 134 (0.57): 6 for K's normalisation, 14 to join.  16
// heads of 128: 32 x 2000 over 4000 2045 (1.03), 1374 over 30,000 keys in pages 407 to 418 (0.81 to 0.83), 457 in E4M3 pages (0.74).
template <int D>
struct Many {
  static constexpr int QB = D == 64 ? 2 : 1, kWaves = 8 / QB, kRows = 32 * QB;
};
template <Kv KV, int D>
__global__ __launch_bounds__(64 * Many<D>::kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_kv_attn_many(Call a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  using T = Tile<D>;
  constexpr int QB = Many<D>::QB, kWaves = Many<D>::kWaves, kRows = Many<D>::kRows;
  constexpr int kHalf = 64 * T::kRow;                     // bytes of a stage's K or V
  constexpr int kStages = kCoded<KV> ? 3 : 4;
  constexpr int kFetch = (kWaves == 4 ? 2 : 1) * T::kFetches;     // fetches of a wave and stage
  constexpr int KF = D / 16, DT = D / 32;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Work w;
  SeqInfo s;
  if (!find_work(a, lane, w, s)) return;
  const int n_rows = s.nq * a.group, block0 = w.block * 256, row0 = block0 + wave * kRows;
  const int last = scalar(limit_of(a, s, min(block0 + 255, n_rows - 1) / a.group));
  const bool live = row0 < n_rows;
  const int first = live ? scalar(limit_of(a, s, row0 / a.group)) : 0;       // keys that every row of the wave sees
  const int begin = w.t0 * 64, end = (int)min((uint32_t)w.t1 * 64u, (uint32_t)last);

  // what the wave fetches: its group, K's rows and (four waves) V's
  const int group = kWaves == 4 ? wave : wave >> 1;
  const bool only_v = kWaves == 8 && (wave & 1);
  Offsets<D> off, off_v;
  if constexpr (!kCoded<KV>) {
    off.init(lane, KV != Kv::ROWS ? T::kRow : only_v ? a.v_stride : a.k_stride, only_v);
    if constexpr (kWaves == 4) off_v.init(lane, KV != Kv::ROWS ? T::kRow : a.v_stride, true);
  }
  const uint32_t to = (only_v ? kHalf : 0) + group * (kGrp * T::kRow), base = __builtin_amdgcn_readfirstlane(lds_addr(lds)) + to;
  // Pages: stages are made of the groups that are held.  The numbers and pages of 256 of them, 64 stages, are listed at a time, and
  // stages are fetched three ahead: a list serves the computation of stages from .. from + 60.  Lane j, of stage from + j: group and page
  // that this wave fetches.
  __shared__ int list[KV == Kv::ROWS ? 1 : kWaves][2][KV == Kv::ROWS ? 1 : 256];
  int n = KV == Kv::ROWS ? scalar(end > begin ? (end - begin + 63) / 64 : 0) : 0x7fffffff;    // stages (pages: once it is known)
  // Of a group: rows before it in the pool, and how many of its 16 exist, in the bits from 24 of the upper word on.
  int from = 0, listed = 0;
  uint32_t own = 0, own_hi = 0;
  int plain = KV == Kv::ROWS ? (first > begin ? (first - begin) >> 6 : 0) : 0;     // stages up to this one hold 64 keys that every row sees
  auto look_up = [&](int i) __attribute__((always_inline)) {
    if constexpr (KV != Kv::ROWS) {
      int *const ids = list[wave][0], *const groups = list[wave][1];
      int at = i ? scalar(groups[4 * (i - from)]) : begin >> 4, count = 0;
      const int last_group = (end + kGrp - 1) >> 4;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      from = i;
#pragma unroll 1
      do {
        int id[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) id[p] = page_at(a, w.seq, (uint32_t)(at + p * 64 + lane) * kGrp, end);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const uint64_t held = __builtin_amdgcn_ballot_w64(id[p] >= 0);
          const int to = count + __builtin_amdgcn_mbcnt_hi((uint32_t)(held >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)held, 0u));
          if (id[p] >= 0 && to < 256) {
            ids[to] = id[p];
            groups[to] = at + p * 64 + lane;
          }
          count += scalar(__popcll(held));
        }
        at += 256;
      } while (count < 256 && at < last_group);
      if (count <= 256 && at >= last_group) n = i + (count + 3) / 4;
      listed = min(count, 256);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      const bool there = 4 * lane + group < count;
      const int key = there ? groups[4 * lane + group] * kGrp : 0, id = there ? ids[4 * lane + group] : 0;
      const int64_t row = (((int64_t)id * a.kv_heads + w.head) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
      own = (uint32_t)row;
      own_hi = (uint32_t)(row >> 32) | (there ? (uint32_t)min(end - key, kGrp) << 24 : 0u);
      const bool whole = 4 * lane + 3 < count && groups[4 * lane + 3] * kGrp + kGrp <= first;
      const uint64_t ragged = __builtin_amdgcn_ballot_w64(!whole);
      plain = i + (ragged ? __ffsll((unsigned long long)ragged) - 1 : 64);
    }
  };
  Codes<KV, D> codes, codes_v;
  // Rows: what the next fetch brings, and the rows that are left of it on
  const int64_t row_first = (int64_t)s.k0 + begin + group * kGrp;
  const char *next_k = a.k + row_first * a.k_stride + w.head * T::kRow, *next_v = a.v + row_first * a.v_stride + w.head * T::kRow;
  if (only_v) next_k = next_v;
  const int64_t step_k = 64 * (only_v ? a.v_stride : a.k_stride), step_v = 64 * a.v_stride;
  const int stride_k = (int)(only_v ? a.v_stride : a.k_stride), stride_v = (int)a.v_stride;
  int left = end - begin - group * kGrp;
  uint32_t ring = base;          // where it goes
  // the stages in their order; beyond the last one nothing is read, the counts stay
  auto fetch = [&](int i) __attribute__((always_inline)) {
    if constexpr (KV == Kv::ROWS) {
      int bytes_k = (kGrp - 1) * stride_k + T::kRow, bytes_v = (kGrp - 1) * stride_v + T::kRow;
      if (__builtin_expect(left < kGrp, 0)) {
        bytes_k = left > 0 ? (left - 1) * stride_k + T::kRow : 0;
        bytes_v = left > 0 ? (left - 1) * stride_v + T::kRow : 0;
      }
      fetch_group<D>(next_k, bytes_k, off, ring);
      if constexpr (kWaves == 4) fetch_group<D>(next_v, bytes_v, off_v, ring + kHalf);
      next_k += step_k;
      next_v += step_v;
      left -= 64;
    } else {
      constexpr int kBytes = kRowBytes<KV, D>;
      const uint32_t lo = __builtin_amdgcn_readlane(own, i - from), hi = __builtin_amdgcn_readlane(own_hi, i - from);
      Group at;
      at.row = (int64_t)((uint64_t)(hi & 0xffffffu) << 32 | lo);
      at.k_bytes = at.v_bytes = (int)(hi >> 24) * kBytes;
      if constexpr (kCoded<KV>) {
        codes.load((only_v ? a.v : a.k) + at.row * kBytes, only_v ? a.v_scale : a.k_scale, at, lane);
        if constexpr (kWaves == 4) codes_v.load(a.v + at.row * kBytes, a.v_scale, at, lane);
      } else {
        fetch_group<D>((only_v ? a.v : a.k) + at.row * kBytes, at.k_bytes, off, ring);
        if constexpr (kWaves == 4) fetch_group<D>(a.v + at.row * kBytes, at.k_bytes, off_v, ring + kHalf);
      }
    }
    if constexpr (!kCoded<KV>) ring = ring == base + (kStages - 1) * (2 * kHalf) ? base : ring + 2 * kHalf;
  };
  auto put = [&](int i) __attribute__((always_inline)) {
    char *p = lds + ((uint32_t)i % kStages) * (2 * kHalf) + to;
    codes.store(p, only_v, lane);
    if constexpr (kWaves == 4) codes_v.store(p + kHalf, true, lane);
  };
  // this wave's part of stage i + 1 has landed; behind the barrier all of it, and nobody reads stage i - 1 any more
  auto publish = [&](int i) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!kCoded<KV>) wait_vm<(kStages - 3) * kFetch>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (kCoded<KV>) put(i + 2);
    fetch(i + 3);
  };
  auto start = [&]() __attribute__((always_inline)) {
    fetch(0);
    if constexpr (kCoded<KV>) {
      put(0);
      fetch(1);
      put(1);
      fetch(2);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    } else {
      fetch(1);
      fetch(2);
      wait_vm<2 * kFetch>();
    }
    __builtin_amdgcn_s_barrier();
  };
  if (end > begin) look_up(0);
  else n = 0;
  if (!live) {      // no rows: the wave moves its share of the stages
    if (n > 0) {
      start();
      for (int i = 0; i < n; ++i) {
        if (KV != Kv::ROWS && i - from > 60) {
          look_up(i);
          if (i >= n) break;
        }
        publish(i);
      }
      wait_vm<0>();
    }
    return;
  }
  Rows<D, QB> rows;
  rows.load(a, s, w.head, row0, lane);
  if (n > 0) {
    start();
    f32x16 sacc[2];              // scores: of the two blocks, or of even and odd tiles
    uint32_t pb[2][8];
    u32x4 fk[KF], fv[2][DT];     // 64 channels
    constexpr int kF4 = QB == 1 ? 4 : 1;
    u32x4 f0[kF4], f1[kF4], g0[kF4], g1[kF4];      // 128 channels: K's and V's fragments
    const uint32_t lds0 = lds_addr(lds);
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    const int kr = lane & 31, vr = 4 * h + (lane >> 2 & 3);
    auto tile_at = [&](int t) __attribute__((always_inline)) { return ((uint32_t)(t >> 1) % kStages) * (2 * kHalf) + (uint32_t)(t & 1) * (32 * T::kRow); };
    const uint32_t k_lane = kr * T::kRow + ((h ^ T::k_xor(kr)) * 16);                       // piece 2 j + h: ^ 32 j
    const uint32_t v_lane = kHalf + vr * T::kRow + T::v_xor(vr) * 16 + (lane >> 4 & 1) * 32 + (lane & 3) * 8;   // channels 32 dt: ^ 64 dt
    uint32_t lanes = k_lane | v_lane << 16;      // (128 channels: in one register)
    auto k_at = [&](int t) __attribute__((always_inline)) {
      if constexpr (QB == 2) return k_lane + (lds0 + tile_at(t));
      asm volatile("" : "+v"(lanes));
      return (lanes & 0xffffu) + (lds0 + tile_at(t));
    };
    auto v_at = [&](int t) __attribute__((always_inline)) {
      if constexpr (QB == 2) return v_lane + (lds0 + tile_at(t));
      asm volatile("" : "+v"(lanes));
      return (lanes >> 16) + (lds0 + tile_at(t));
    };
    auto read_k = [&](int t) __attribute__((always_inline)) {
      const uint32_t p = k_at(t);
#pragma unroll
      for (int j = 0; j < KF; ++j) fk[j] = *(lds_u32x4 *)(uintptr_t)(p ^ (j * 32));
    };
    auto read_v = [&](int t) __attribute__((always_inline)) {
      const uint32_t p = v_at(t);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t q = (p ^ (dt * 64)) + u * 16 * T::kRow;
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)q));
          const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(q + 8 * T::kRow)));
          fv[u][dt] = u32x4{x.x, x.y, y.x, y.y};
        }
    };
    // 128 channels: four fragments at a time
    auto read_k4 = [&](int t, int half, u32x4(&f)[kF4]) __attribute__((always_inline)) {
      const uint32_t p = k_at(t);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = *(lds_u32x4 *)(uintptr_t)(p ^ ((4 * half + j) * 32));
    };
    auto read_v4 = [&](int t, int u, u32x4(&f)[kF4]) __attribute__((always_inline)) {
      const uint32_t p = v_at(t) + u * 16 * T::kRow;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const uint32_t q = p ^ (dt * 64);
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)q));
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(q + 8 * T::kRow)));
        f[dt] = u32x4{x.x, x.y, y.x, y.y};
      }
    };
    // product number m of a phase: scores of bs (the first half), output of bo
    auto product = [&](auto scores, auto output, int m, int bs, int bo) __attribute__((always_inline)) {
      if (m < KF) {
        if constexpr (decltype(scores)::value) {
          const u32x4 f = QB == 2 ? fk[m % KF] : m < 4 ? f0[m % kF4] : f1[m % kF4];
          f32x16 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          if (m) acc = sacc[bs];
          sacc[bs] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f), rows.q[QB == 2 ? bs : 0][m], acc, 0, 0, 0);
        }
      } else if constexpr (decltype(output)::value) {
        const int u = (m - KF) / DT, dt = (m - KF) % DT;
        const u32x4 f = QB == 2 ? fv[u][dt] : u == 0 ? g0[dt % kF4] : g1[dt % kF4];
        const bf16x8 w = __builtin_bit_cast(bf16x8, u32x4{pb[bo][4 * u], pb[bo][4 * u + 1], pb[bo][4 * u + 2], pb[bo][4 * u + 3]});
        f32x16 &o = rows.o[QB == 2 ? bo : 0][dt];
        o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f), w, o, 0, 0, 0);
      }
    };
    float sum0, sum1;
    auto weight = [&](int b, int e, float p0, float p1) __attribute__((always_inline)) {
      pb[b][e] = pack_bf16(p0, p1);
      asm("" : "+v"(pb[b][e]));      // (where paths meet the pair would be carried unpacked, in twice the registers)
      sum0 += p0;
      sum1 += p1;
    };
    auto weights = [&](int b) __attribute__((always_inline)) {
      const float ref = rows.ref[QB == 2 ? b : 0];
      sum0 = sum1 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        weight(b, e, __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[b][2 * e], a.c, -ref)), __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[b][2 * e + 1], a.c, -ref)));
    };
    // A phase: 2 KF products, and the weights of block bw among them, a pair of them to one or two products, each in three
    // steps that stand next to the other pairs' (the exponent of the next, exp2 of this, sum and rounding of the last).  `then` follows
    // product m (reads of fragments).
    // Rows (no pages) of 128 channels: all weights, then the products, ahead of the other wave's weights: 32 x 2000 queries over 4000
    // keys, 16 heads 2070 us, weights among the products 2092; of 64 channels 1080 and 1057.  Where calls are small or in pages the sides lie
    // close, and not always so: 9 sets of 3 to 701 over up to 6007 134 and 127, 1374 over 30,000 keys in pages 407 and 414, in E4M3 pages level.
    auto phase = [&](auto scores, auto output, int bw, int bs, int bo, auto &&then) __attribute__((always_inline)) {
      if constexpr (QB == 1 && KV == Kv::ROWS) {
        __builtin_amdgcn_sched_barrier(0);
        weights(bw);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int m = 0; m < 2 * KF; ++m) {
          product(scores, output, m, bs, bo);
          then(m);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        return;
      }
      constexpr int kPer = 2 * KF / 8;
      const float ref = rows.ref[QB == 2 ? bw : 0];
      sum0 = sum1 = 0.f;
      float x0 = __builtin_fmaf(sacc[bw][0], a.c, -ref), x1 = __builtin_fmaf(sacc[bw][1], a.c, -ref), y0 = 0.f, y1 = 0.f;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 2 * KF; ++m) {
        product(scores, output, m, bs, bo);
        const int e = m / kPer;
        if (m % kPer == 0) {
          const float z0 = y0, z1 = y1;
          y0 = __builtin_amdgcn_exp2f(x0);
          y1 = __builtin_amdgcn_exp2f(x1);
          if (kPer == 1 && e) weight(bw, e - 1, z0, z1);
          if (kPer == 1 && e < 7) {
            x0 = __builtin_fmaf(sacc[bw][2 * e + 2], a.c, -ref);
            x1 = __builtin_fmaf(sacc[bw][2 * e + 3], a.c, -ref);
          }
        } else {
          weight(bw, e, y0, y1);
          if (e < 7) {
            x0 = __builtin_fmaf(sacc[bw][2 * e + 2], a.c, -ref);
            x1 = __builtin_fmaf(sacc[bw][2 * e + 3], a.c, -ref);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        then(m);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (kPer == 1) weight(bw, 7, y0, y1);
    };
    // block b's weights become part of its sums, with the references raised first where a sum went past 2^40
    auto settle = [&](int b) __attribute__((always_inline)) {
      constexpr int kOne = QB == 2 ? 1 : 0;
      const int r = b * kOne;
      __builtin_amdgcn_sched_barrier(0);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(rows.l[r] + (sum0 + sum1) <= kRowRaise)) != 0, 0)) {
        float top = sacc[b][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(top, sacc[b][e]);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float to = fmaxf(rows.ref[r], top * a.c), f = __builtin_amdgcn_exp2f(rows.ref[r] - to);
        rows.ref[r] = to;
        rows.l[r] *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) rows.o[r][dt][e] *= f;
        weights(b);
      }
      rows.l[r] += sum0 + sum1;
      __builtin_amdgcn_sched_barrier(0);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    auto phase_a = [&](auto head, auto tail, int t) __attribute__((always_inline)) {
      phase(Yes{}, std::bool_constant<!decltype(head)::value>{}, 0, 1, 1, [&](int m) __attribute__((always_inline)) {
        if (m == KF - 1 && !decltype(tail)::value) read_k(t + 1);
        if (m == 2 * KF - 1) read_v(t);
      });
      settle(0);
    };
    auto phase_b = [&](auto tail) __attribute__((always_inline)) {
      phase(std::bool_constant<!decltype(tail)::value>{}, Yes{}, 1, 0, 0, [](int) {});
      settle(1);
    };
    // head: nothing of a tile before; tail: no tile after; pub: stage t / 2 + 1 is needed and t / 2 - 1 no more
    auto phase_c = [&](auto head, auto tail, auto pub, int b, int t) __attribute__((always_inline)) {
      constexpr bool kHead = decltype(head)::value, kTail = decltype(tail)::value;
      phase(std::bool_constant<!kTail>{}, std::bool_constant<!kHead>{}, b, b ^ 1, b ^ 1, [&](int m) __attribute__((always_inline)) {
        if (m == 7) {
          if constexpr (decltype(pub)::value) publish(t >> 1);
          if (!kTail) {
            read_k4(t + 2, 0, f0);
            read_k4(t + 2, 1, f1);
          }
        }
        if (m == 15) {
          read_v4(t, 0, g0);
          read_v4(t, 1, g1);
        }
      });
      settle(b);
    };
    int i = 0;
    while (i < n) {
      // the stages from i on whose keys are all there and seen
      if (KV != Kv::ROWS && i - from > 60) {
        look_up(i);
        if (i >= n) break;
      }
      const int j = scalar(min(plain, KV == Kv::ROWS ? n : min(n, from + 61)));
      if (j > i) {
        if constexpr (QB == 2) {
          read_k(2 * i);
#pragma unroll
          for (int m = 0; m < KF; ++m) product(Yes{}, No{}, m, 0, 0);
          phase_a(Yes{}, No{}, 2 * i);
          if (i < j - 1) do {
            asm volatile("" : "+v"(sacc[1]));   // (the same phase follows the loop: its instructions would be drawn before the branch)
            phase_b(No{});
            publish(i);
            phase_a(No{}, No{}, 2 * i + 1);
            phase_b(No{});
            phase_a(No{}, No{}, 2 * i + 2);
            ++i;
          } while (i < j - 1);
          phase_b(No{});
          publish(i);
          phase_a(No{}, Yes{}, 2 * i + 1);
          phase_b(Yes{});
#pragma unroll
          for (int m = KF; m < 2 * KF; ++m) product(No{}, Yes{}, m, 1, 1);
        } else {
          read_k4(2 * i, 0, f0);
          read_k4(2 * i, 1, f1);
#pragma unroll
          for (int m = 0; m < KF; ++m) product(Yes{}, No{}, m, 0, 0);
          read_k4(2 * i + 1, 0, f0);
          read_k4(2 * i + 1, 1, f1);
          if (i < j - 1) {
            phase_c(Yes{}, No{}, Yes{}, 0, 2 * i);
            phase_c(No{}, No{}, No{}, 1, 2 * i + 1);
            ++i;
            if (i < j - 1) do {
              asm volatile("" : "+v"(sacc[0]));
              phase_c(No{}, No{}, Yes{}, 0, 2 * i);
              phase_c(No{}, No{}, No{}, 1, 2 * i + 1);
              ++i;
            } while (i < j - 1);
            phase_c(No{}, No{}, Yes{}, 0, 2 * i);      // (its reads of a tile beyond the run are of a stage that is there or arriving, and not used)
          } else {
            phase_c(Yes{}, No{}, Yes{}, 0, 2 * i);
          }
          phase_c(No{}, Yes{}, No{}, 1, 2 * i + 1);
#pragma unroll
          for (int m = KF; m < 2 * KF; ++m) product(No{}, Yes{}, m, 1, 1);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
      } else {
        const char *kt = lds + ((uint32_t)i % kStages) * (2 * kHalf);
#pragma unroll 1
        for (int t = 0; t < 2; ++t) {
          int key0 = begin + i * 64 + t * 32, key1 = key0 + kGrp;
          if constexpr (KV != Kv::ROWS) {
            const int *const groups = list[wave][1] + 4 * (i - from) + 2 * t;
            const int known = 4 * (i - from) + 2 * t;
            key0 = known < listed ? scalar(groups[0]) * kGrp : kNoKey;
            key1 = known + 1 < listed ? scalar(groups[1]) * kGrp : kNoKey;
          }
          if (key0 < end)
            rows.tile(kt + t * 32 * T::kRow, kt + kHalf + t * 32 * T::kRow, a.c, key0, key1, key1 + kGrp > first, lane);
        }
        publish(i);
      }
      ++i;
    }
    wait_vm<0>();     // nothing may land after the workgroup ends
  }
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int r = wave * kRows + b * 32 + (lane & 31);
    const int rr = block0 + r, tok = rr / a.group;
    const float l = rows.l[b] + __shfl_xor(rows.l[b], 32, 64);
    if (rr >= n_rows) continue;
    if (w.pieces > 1) {
      const int64_t at = (int64_t)w.slot * 256 + r;
      if (lane < 32) a.part_ml[at] = float2{rows.ref[b], l};
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4 *)(a.part + at * D + dt * 32 + i * 8 + h * 4) =
              f32x4{rows.o[b][dt][4 * i], rows.o[b][dt][4 * i + 1], rows.o[b][dt][4 * i + 2], rows.o[b][dt][4 * i + 3]};
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      uint16_t *p = a.o + (int64_t)(s.q0 + tok) * a.o_stride + (w.head * a.group + rr - tok * a.group) * D + h * 4;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(u32x2 *)(p + dt * 32 + i * 8) = u32x2{pack_bf16(rows.o[b][dt][4 * i] * inv, rows.o[b][dt][4 * i + 1] * inv),
                                                  pack_bf16(rows.o[b][dt][4 * i + 2] * inv, rows.o[b][dt][4 * i + 3] * inv)};
    }
  }
}

// ---------------------------------------------------------------------------------------
// The sums of a row's pieces put together, always in the same order.  A row has D / 4 lanes times SL: each of
// these takes every SL-th piece (few rows, many pieces), and they meet in LDS.  SL = 1: 16 or 8 consecutive rows of one kv head, whose sums lie
// side by side in a slot, mostly of one sequence (otherwise one after the other).  Bound by the way from the lengths to the sums and
// by reading the latter: 4 pieces of 7 heads of 13,740 rows in 28 us, 4.0 TB/s.  (A token with all its
// heads to a workgroup instead: 16 pieces of 1374 rows 24 us against 18, ragged rows of heads that share 12.2 against 13.7.)
template <int D, int SL>
__global__ __launch_bounds__(256) void k_kv_attn_join(Call a) {
  constexpr int kCh = D / 4, kRowsWg = 256 / (kCh * SL);
  static_assert(SL == 1 || kRowsWg == 1, "one sequence");
  const int tid = threadIdx.x, lane = tid & 63;
  const int in_wg = tid / kCh / SL, sl = tid / kCh % SL, ch = tid % kCh * 4;
  const int head = blockIdx.y;
  const uint32_t row = blockIdx.x * kRowsWg + in_wg;
  const int tok = (int)(row / (uint32_t)a.group), g = (int)row - tok * a.group;
  const int piece_len = uniform_at(a.chosen, 0);
  SeqInfo q;
  int start = 0;
  if (!a.starts) {
    q = lane_seq(a, lane);
    int none;
    if (a.n_seq > 1) start = wave_scan(slots_taken(a, q, piece_len), none);
  }
  bool open = tok < a.n_q;
  uint64_t left;
#pragma unroll 1
  while ((left = __builtin_amdgcn_ballot_w64(open)) != 0) {
    // the sequence of the first row that is left, the number of its first slot
    const int first = __builtin_amdgcn_readlane(tok, __ffsll((unsigned long long)left) - 1);
    SeqInfo s = {0, 0, 0, 0, 0, 0, 0};
    int before = 0;
    if (a.starts) {
      const int seq = scalar(last_at_most(a.q_off, a.n_seq, first, lane));
      if (seq >= 0) {
        s = uniform_seq(a, seq);
        before = uniform_at(a.taken, seq);
      }
    } else {
      const uint64_t hit = __builtin_amdgcn_ballot_w64(first >= q.q0 && first < q.q0 + q.nq);
      if (hit) {
        const int j = scalar(__ffsll((unsigned long long)hit) - 1);
        s = from_lane(q, j);
        before = __builtin_amdgcn_readlane(start, j);
      }
    }
    const bool its = open && tok >= s.q0 && tok < s.q0 + s.nq;
    open = open && !its && tok != first;
    const int pieces = pieces_of(s.tiles, piece_len), whole = whole_heads(a, s.blocks);
    if (s.nq == 0 || pieces == 1 || head < whole) continue;          // of no sequence; written already
    const int r = (tok - s.q0) * a.group + g;
    const int block = r >> a.block_shift, in_block = r & (a.rows_per_block - 1);
    const int64_t slot0 = before + (int64_t)(head - whole) * pieces * s.blocks + block;
    const int n = its && slot0 + (int64_t)(pieces - 1) * s.blocks < a.slots ? pieces : 0;
    auto at = [&](int x) { return (slot0 + (int64_t)x * s.blocks) * a.rows_per_block + in_block; };
    // four pieces at a time: their loads are on the way together
    float top = kUnset, l = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int x0 = sl; x0 < n; x0 += 4 * SL) {
      float2 ml[4];
      f32x4 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t from = at(min(x0 + i * SL, n - 1));
        ml[i] = a.part_ml[from];
        y[i] = *(const f32x4 *)(a.part + from * D + ch);
      }
      float to = top;
#pragma unroll
      for (int i = 0; i < 4; ++i) to = fmaxf(to, ml[i].x);
      const float f0 = __builtin_amdgcn_exp2f(top - to);
      top = to;
      l *= f0;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] *= f0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (x0 + i * SL >= n) break;
        const float f = __builtin_amdgcn_exp2f(ml[i].x - to);
        l += ml[i].y * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += y[i][e] * f;
      }
    }
    if constexpr (SL > 1) {      // (one row in the workgroup: all of it comes here, and once)
      __shared__ float tops[SL], ls[SL];
      __shared__ f32x4 sums[SL][kCh];
      if (ch == 0) {
        tops[sl] = top;
        ls[sl] = l;
      }
      sums[sl][ch / 4] = sum;
      __syncthreads();
      if (sl) return;
      for (int x = 1; x < SL; ++x) top = fmaxf(top, tops[x]);
      l = 0.f;
      sum = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int x = 0; x < SL; ++x) {
        const float f = __builtin_amdgcn_exp2f(tops[x] - top);
        const f32x4 y = sums[x][ch / 4];
        l += ls[x] * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += y[e] * f;
      }
    }
    if (n == 0) continue;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    *(u32x2 *)(a.o + (int64_t)tok * a.o_stride + (head * a.group + g) * D + ch) =
        u32x2{pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
  }
}

// K's rows normalised per head, for cross attention with qk_norm: once for all blocks that read them.  Bound by HBM: 27,216 states
// of 2 heads of 128 in 6.2 us.
template <int D>
__global__ __launch_bounds__(256) void k_norm_rows(const uint16_t *k, int64_t stride, int64_t n_rows, int kv_heads, uint16_t *out) {
  constexpr int L = D / 8;
  const int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const int p = threadIdx.x % L;
  const int64_t rr = min(r, n_rows - 1);
  const u32x4 w = *(const u32x4 *)(k + rr / kv_heads * stride + rr % kv_heads * D + p * 8);
  float ss = sumsq8(w);
#pragma unroll
  for (int o = 1; o < L; o <<= 1) ss += __shfl_xor(ss, o, 64);
  const u32x4 y = scale8(w, 1.0f / sqrtf(ss * (1.0f / D) + kQkEps));
  if (r < n_rows) *(u32x4 *)(out + r * D + p * 8) = y;
}

// ---------------------------------------------------------------------------------------
struct Form {
  bool few;
  int rows, tile;
  int resident;      // workgroups that the chip holds at once
  int64_t units;     // blocks of the call at most, all heads
  int target;        // pieces beside these at most
};

// Which kernel: by the rows that a (sequence, kv head) has on average.  64 channels, 16 heads of one sequence: 24 rows over 30,000
// keys 29 us in blocks of 32 rows, 41 in those of 256; 48 rows 31 us in blocks of 64, 46 of 32, 41 of 256 (over 2000 keys 12.6, 12.1, 17);
// 100 rows 51 of 64, 84 of 32, 49 of 256.  128 channels, 8 sequences over 4000 keys: 24 rows 54 us in blocks of 32, 61 of 256; 48 rows 90 and 63
// (64 do not fit the registers).
Form form_of(int n_q, int n_seq, int heads, int kv_heads, int head_dim, int dtype, int64_t most_keys) {
  Form f;
  const int group = heads / kv_heads;
  const double rows = (double)n_q * group / n_seq;
  f.few = rows <= (head_dim == 64 ? 64.0 : 32.0);
  f.rows = f.few ? (rows <= 32.0 ? 32 : 64) : 256;
  f.tile = f.few ? 128 : 64;
  // (by LDS; 128 channels, many rows: 8 waves each)
  f.resident = kCus * (head_dim == 64 || (f.few && dtype != LV_CACHE_BF16) ? 2 : 1);
  if (f.few && dtype == LV_CACHE_E2M1 && head_dim == 64 && f.rows == 32) f.resident = kCus * kFewWaves<Kv::E2M1, 64, 1>;
  f.units = ((int64_t)n_q * group / f.rows + n_seq) * kv_heads;
  const int64_t tiles = (most_keys + f.tile - 1) / f.tile;
  // (Blocks of several sequences that fill the chip four times over are not cut: 32 x 2000 queries over 4000 keys, 16 heads of 64
  // 1043 us against 1089 cut, of 128 2045 against 2177, 64 sequences of 100 to 2000 over 100 to 4000 608 against 650.  One sequence: whole_heads.)
  const int64_t target = f.units >= 4 * f.resident && !f.few && n_seq > 1 ? 0 : tiles < kWholeTiles ? 0 : kRounds * f.resident;
  f.target = (int)(target < f.units * tiles ? target : f.units * tiles);
  return f;
}
// Blocks that are cut take a piece each beside those aimed at, and at most twice as many as were aimed at (slots_taken)
int64_t slots_of(const Form &f) { return std::min(f.units + f.target, 2 * (int64_t)f.target); }
size_t sums_bytes(const Form &f, int head_dim) { return align_up((size_t)slots_of(f) * f.rows * (head_dim + 2) * sizeof(float), 256); }
// In front of the sums: 256 bytes, and the plan of more than 64 sequences
size_t plan_bytes(int n_seq) { return 256 + (n_seq > 64 ? 2 * align_up((size_t)n_seq * sizeof(int), 256) : 0); }

}  // namespace

size_t kv_attn_ws_bytes(int n_q, int n_seq, int heads, int kv_heads, int head_dim, int dtype, int64_t most_keys) {
  // What the call needs grows with n_q inside a form only.  The size is the largest up to n_q, so that scratch for a
  // longer call serves the shorter ones.
  const int group = heads / kv_heads;
  const int64_t cut = (4 * kCus * (head_dim == 64 ? 2 : 1) - 1) / kv_heads - n_seq;     // most blocks of many rows that are cut (form_of)
  size_t most = 0;
  for (int64_t n : {(int64_t)n_q, (int64_t)32 * n_seq / group, (int64_t)64 * n_seq / group, (256 * cut + 255) / group})
    if (n > 0 && n <= n_q) most = std::max(most, sums_bytes(form_of((int)n, n_seq, heads, kv_heads, head_dim, dtype, most_keys), head_dim));
  return most || n_seq > 64 ? plan_bytes(n_seq) + most : 0;
}

// LDS that a kernel has of its own beside what its launch asks for, at most: the lists of pages of eight waves (k_kv_attn_many)
constexpr size_t kStaticLds = 8 * 2 * 256 * sizeof(int);

template <typename K, size_t LDS>
static int go(K kernel, std::atomic<uint64_t> &done, std::integral_constant<size_t, LDS>, const Call &c, uint32_t grid, int threads, hipStream_t st) {
  if constexpr (LDS + kStaticLds > 65536) {     // (what a launch may take of its own accord)
    const int rc = allow_dynamic_lds<LDS>((const void *)kernel, done);
    if (rc) return rc;
  }
  kernel<<<dim3(grid), threads, LDS, st>>>(c);
  return LV_OK;
}

template <Kv KV, int D>
static int launch_form(const Form &f, const Call &c, uint32_t grid, hipStream_t st) {
  constexpr size_t tile = 64 * D * 2 * 2;      // 64 keys of K and V as bf16
  static std::atomic<uint64_t> d0{0}, d1{0}, d2{0};
  // (the ring of four waves' tiles, and room for their sums at the end)
  constexpr size_t ring = KV == Kv::E2M1 ? 4 * (Ring<D>::kBytes + tile / 4) : kCoded<KV> ? 2 * tile : 4 * tile, sums = 4 * 32 * D * sizeof(float);
  if (f.few && f.rows == 32) return go(k_kv_attn_few<KV, D, 1>, d0, std::integral_constant<size_t, std::max(ring, sums)>{}, c, grid, 256, st);
  if constexpr (D == 64)
    if (f.few) return go(k_kv_attn_few<KV, D, 2>, d1, std::integral_constant<size_t, std::max(ring, 2 * sums)>{}, c, grid, 256, st);
  return go(k_kv_attn_many<KV, D>, d2, std::integral_constant<size_t, kCoded<KV> ? 3 * tile : 4 * tile>{}, c, grid,
            64 * Many<D>::kWaves, st);
}

int launch_kv_attn(const KvAttnArgs &x, void *ws, hipStream_t st) {
  const int64_t most = x.paged ? (int64_t)x.cv.max_pages << x.cv.page_shift : x.n_kv;
  const Form f = form_of(x.n_q, x.n_seq, x.heads, x.kv_heads, x.head_dim, x.paged ? x.cv.dtype : LV_CACHE_BF16, most);
  Call c;
  c.q = x.q;
  c.o = x.o;
  c.q_stride = x.q_stride;
  c.o_stride = x.o_stride;
  c.q_off = x.q_off;
  c.k_begin = x.k_begin;
  c.k_end = x.k_end;
  c.n_q = x.n_q;
  c.n_seq = x.n_seq;
  c.kv_heads = x.kv_heads;
  c.group = x.heads / x.kv_heads;
  c.qk_norm = x.qk_norm;
  c.frame = x.frame;
  c.n_kv = x.n_kv;
  c.c = x.scale * 1.4426950408889634f;
  c.k = (const char *)x.k;
  c.v = (const char *)x.v;
  c.k_stride = x.k_stride * 2;
  c.v_stride = x.v_stride * 2;
  c.k_scale = x.k_scale;
  c.v_scale = x.v_scale;
  c.table = x.paged ? x.cv.table : nullptr;
  c.page_shift = x.cv.page_shift;
  c.n_pages = x.cv.n_pages;
  c.max_pages = x.cv.max_pages;
  c.rows_per_block = f.rows;
  c.tile = f.tile;
  c.block_shift = __builtin_ctz(f.rows);
  c.tile_shift = __builtin_ctz(f.tile);
  c.target = f.target;
  c.slots = (int)slots_of(f);
  c.resident = f.resident;
  c.most_units = (int)(f.units + f.target);
  c.chosen = (int *)ws;
  c.starts = x.n_seq > 64 ? (int *)((char *)ws + 256) : nullptr;
  c.taken = x.n_seq > 64 ? (int *)((char *)c.starts + align_up((size_t)x.n_seq * sizeof(int), 256)) : nullptr;
  c.part = f.target ? (float *)((char *)ws + plan_bytes(x.n_seq)) : nullptr;
  c.part_ml = f.target ? (float2 *)(c.part + (size_t)c.slots * f.rows * x.head_dim) : nullptr;
  const int side = f.few ? 1 : x.n_seq > 1 ? 8 : kSide;
  const uint32_t grid = (uint32_t)((f.units + f.target) / kXcd * kXcd + kXcd * (side + 1));     // (whole turns of units side by side)
  auto by_kv = [&](auto kv) {
    constexpr Kv KV = decltype(kv)::value;
    return x.head_dim == 64 ? launch_form<KV, 64>(f, c, grid, st) : launch_form<KV, 128>(f, c, grid, st);
  };
  if (c.starts) k_kv_attn_plan<<<dim3(1), 1024, 0, st>>>(c);
  int rc;
  if (!x.paged) rc = by_kv(std::integral_constant<Kv, Kv::ROWS>{});
  else if (x.cv.dtype == LV_CACHE_BF16) rc = by_kv(std::integral_constant<Kv, Kv::PAGES>{});
  else if (x.cv.dtype == LV_CACHE_E4M3) rc = by_kv(std::integral_constant<Kv, Kv::E4M3>{});
  else rc = by_kv(std::integral_constant<Kv, Kv::E2M1>{});
  if (rc) return rc;
  if (f.target) {
    auto join = [&](auto kernel, int rows) {
      kernel<<<dim3((uint32_t)(((int64_t)x.n_q * c.group + rows - 1) / rows), (uint32_t)x.kv_heads), 256, 0, st>>>(c);
    };
    if (x.head_dim == 64) f.few ? join(k_kv_attn_join<64, 16>, 1) : join(k_kv_attn_join<64, 1>, 16);
    else f.few ? join(k_kv_attn_join<128, 8>, 1) : join(k_kv_attn_join<128, 1>, 8);
  }
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

int launch_norm_rows(const uint16_t *k, int64_t k_stride, int n, int kv_heads, int head_dim, uint16_t *out, hipStream_t st) {
  const int64_t rows = (int64_t)n * kv_heads;
  const uint32_t grid = (uint32_t)((rows * (head_dim / 8) + 255) / 256);
  if (head_dim == 64) k_norm_rows<64><<<dim3(grid), 256, 0, st>>>(k, k_stride, rows, kv_heads, out);
  else k_norm_rows<128><<<dim3(grid), 256, 0, st>>>(k, k_stride, rows, kv_heads, out);
  LV_HIP_CHECK_LAUNCH();
  return LV_OK;
}

}  // namespace lv
