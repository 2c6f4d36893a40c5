// Which kernels a call of the drawn weight takes and how its keys are cut (mass.hip): arithmetic that is the same on the host, where it is tested.
#pragma once
#include <hip/hip_runtime.h>
#include <algorithm>
#include <stdint.h>

#include "../../include/litevggt.h"

namespace lv {
namespace mass {

__host__ __device__ inline int larger(int a, int b) { return a > b ? a : b; }
__host__ __device__ inline int quotient_up(int a, int b) { return (int)(((uint32_t)a + (uint32_t)b - 1u) / (uint32_t)b); }

// How the keys of a call are cut: into chunks of so many, and these into pieces, about `aim` of them in all, so that pieces of sequences with
// many rows are shorter and all take about as long
struct Cut {
  int chunk, aim;
  int most;                // pieces of a sequence
  int block;               // rows that a wave takes at a time
  bool of_rows;            // sequences without queries have no pieces
  const int *starts;       // more than 64 sequences: units before each, in all, and the work of a piece (k_mass_plan); else null
};

__host__ __device__ inline bool has_pieces(const Cut &c, int queries, int keys) { return keys > 0 && (!c.of_rows || queries > 0); }
// What a chunk of a sequence with so many rows costs
__host__ __device__ inline float chunk_cost(const Cut &c, int rows) {
  return (float)larger(quotient_up(rows, c.block), 1);
}
// The work of a piece, from that of all sequences and heads (a hair more, so that there are not more pieces than were aimed at and one for each
// sequence and head)
__host__ __device__ inline float piece_work(const Cut &c, int kv_heads, float all) { return all * (float)kv_heads / (float)c.aim * 1.0001f; }
__host__ __device__ inline int chunks_of_piece(const Cut &c, int rows, int keys, float work) {
  const int chunks = quotient_up(keys, c.chunk);
  return larger(larger((int)fminf(ceilf(work / chunk_cost(c, rows)), (float)chunks), quotient_up(chunks, c.most)), 1);
}

constexpr int kAim = 4096;                             // waves of the few rows' kernels: two rounds of eight a CU
constexpr int kAimMany = 32768;                        // of the many rows', whose chunks are longer work
constexpr int kUnits = 6144;                           // three rounds of two waves a SIMD
constexpr int64_t kMostParts = (int64_t)1 << 25;       // (row, piece) pairs in the workspace, where rows leave a choice
constexpr int64_t kMostScores = (int64_t)1 << 27;      // scores there

struct Form {
  bool few, scores;        // lanes with a key each; the call's scores fit and would be kept
  bool keep, own;          // they are; the adding kernel joins the rows' pieces itself
  bool eight;              // few: rows in blocks of 8, else of 32
  bool small_chunks;       // many: the keys' sums by chunks of 32
  int splits;              // of the rows
  Cut rows, keys;          // for the rows' sums; for the keys'
};

// Pieces of the only sequence that has many keys, at most
inline int64_t most_pieces(int kv_heads, int64_t most_keys) {
  return std::max((int64_t)1, std::min((int64_t)(kAimMany + kv_heads - 1) / kv_heads, (most_keys + 31) / 32));
}
// Tokens up to which scores are kept: where writing and reading them costs less than reading K and taking the products again, and they fit.  Over
// 60,000 positions, 16 heads of 64, kept and not: bf16 16 rows 67 us and 81, 24 77 and 82, 32 87 and 81; E4M3 12 57 and 61, 24 71 and 62; E2M1 12 53 and
// 58, 16 60 and 58; of 128, bf16 32 115 and 144, E2M1 16 65 and 75.
inline int64_t kept_tokens(int n_seq, int heads, int kv_heads, int head_dim, int dtype, int64_t most_keys) {
  const int64_t row_bytes = dtype == LV_CACHE_BF16 ? 2 * head_dim : dtype == LV_CACHE_E4M3 ? head_dim : head_dim / 2;
  const int64_t rows = std::min(row_bytes / 8 + 8, (int64_t)32);
  return std::min(rows * n_seq / (heads / kv_heads), kMostScores / (most_keys * heads));
}
inline Form form_of(int n_q, int n_seq, int heads, int kv_heads, int head_dim, int dtype, int64_t most_keys) {
  Form f;
  const int group = heads / kv_heads;
  const int64_t pairs = (int64_t)n_seq * kv_heads, rows = std::max((int64_t)n_q, (int64_t)1) * heads;
  const double mean = (double)n_q * group / n_seq;
  f.scores = n_q <= kept_tokens(n_seq, heads, kv_heads, head_dim, dtype, most_keys);
  // (not kept, E2M1: 32 rows of 128 channels 75 us so, 86 in the other form; 16 of 64 64 and 58)
  f.few = f.scores || mean <= (head_dim == 128 ? 32.0 : 8.0);
  f.keep = n_q > 0 && f.few && f.scores;
  // as many workgroups as there are CUs or fewer join their rows themselves
  f.own = f.keep && pairs * ((most_keys + 1023) / 1024) <= 256;
  f.eight = mean <= 8.0;
  const int aim = f.few ? kAim : kAimMany;
  const int most = (int)std::max((int64_t)1, std::min(most_pieces(kv_heads, most_keys), kMostParts / rows));
  // Many rows: where the chunks are too few to fill the chip a few times over, rows are split too, down to four blocks of 32.  (The sums by
  // keys cannot be: they take chunks of 32 keys then.)
  const int64_t blocks = ((int64_t)n_q * group / n_seq + 31) / 32;
  const int many = head_dim == 64 ? 256 : 128;
  const int64_t units = std::min(pairs * ((most_keys + many - 1) / many), (int64_t)aim);
  f.splits = f.few ? 1 : (int)std::max((int64_t)1, std::min(std::min((kUnits + units - 1) / units, blocks / 4), (int64_t)64));
  f.small_chunks = pairs * ((most_keys + many / 2 - 1) / (many / 2)) < kUnits / 4;
  const int block = f.few && f.eight ? 8 : 32;
  f.rows = Cut{f.few ? 32 : many, aim, most, block, true, nullptr};
  f.keys = Cut{f.keep ? 1024 : f.few ? 64 : f.small_chunks ? 32 : many / 2, aim, 0x7fffffff, block, false, nullptr};
  return f;
}

}  // namespace mass
}  // namespace lv
