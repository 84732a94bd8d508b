// The plan of a batch whose requests share prefixes: which rows meet which keys, in which workgroup (include/hydra_step.h).
//
// The rows of a set are the (new token, query head of a KV head) pairs of consecutive tokens, row = token * group + head in group.  A
// group of requests that shares keys is one set of all its tokens against the shared keys; every request is a set of
// its own tokens against the rest of its context, or against all of it where its group shares nothing.  A set is cut into blocks of
// rows and into parts of its keys; a piece is one block with one part, for every KV head, and a workgroup's work.  Where a row meets its
// keys in several pieces, each leaves a partial result (maximum, sum, unnormalised output), and the merge puts them together.
//
// One workgroup plans: lengths and offsets of the whole batch lie in its LDS.  All sums are of whole numbers, so a batch has one plan.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wave_ops.hpp"

namespace hydra {
namespace prefix {

constexpr int kMostRequests = 2048;
constexpr int kPlanThreads = 1024;
constexpr int kTileKeys = 64;    // keys are cut at multiples of this behind a set's first one
constexpr int kMostParts = 64;   // of a set's keys
constexpr int kSlots = 512;      // workgroups that the chip holds at once, two to a compute unit

// How a piece is computed.
enum Form : int32_t { kKeySplit = 1 };
__host__ __device__ inline constexpr int rows_of_form(int) { return 32; }
// Cost of a tile of keys, for one block of rows.
__host__ __device__ inline constexpr int cost_of_form(int) { return 6; }
constexpr int kLeastCost = 12;  // of a piece: less is not worth a partial result

struct Piece {
  int32_t table_row;            // request whose row of the block table the keys are found by
  int32_t key_begin, key_end;
  int32_t limit;                // the set's token i sees keys up to limit + i
  int32_t first_token;          // of the set
  int32_t first_row;            // of the block, in the set
  int32_t form_rows;            // form * 256 + rows of the block
  int32_t partial;              // first row of its partial results; -1: the result is final
};
static_assert(sizeof(Piece) == 32, "two loads");

// A token's partial results: of its own request's set and of its group's.  Rows r of a set: block r / rows, whose `parts` results are
// rows of partial results first + (block * parts + part) * rows + r % rows.
struct TokenPart {
  int32_t first, parts, rows, token;  // token: number in the set; parts 0: none
};
struct Token {
  TokenPart own, shared;
};
static_assert(sizeof(Token) == 32, "two loads");

struct PlanHeader {
  int32_t n_pieces;
  int32_t reserved[31];
};

// Workspace: header, pieces, tokens, row statistics (maximum, sum), row outputs.
struct Layout {
  int64_t pieces, rows;  // capacity: pieces for each KV head, rows of partial results of a KV head
  size_t pieces_at, tokens_at, stats_at, out_at, total;
};
inline Layout layout_of(int32_t batch, int32_t n_groups, int32_t total_q, int32_t group, int32_t n_kv_heads, int32_t head_dim) {
  Layout l;
  const int64_t sets = (int64_t)batch + n_groups, rows = 2 * (int64_t)total_q * group;  // (of a group's set and of its requests' own)
  const int64_t cuts = kSlots / n_kv_heads + 1;  // pieces that cutting keys adds at most
  l.pieces = sets + rows / 32 + cuts;
  const int64_t wide = sets < rows / 64 ? sets : rows / 64;  // sets of more than 64 rows
  l.rows = rows + 32 * sets + 128 * wide + 128 * cuts;
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  l.pieces_at = sizeof(PlanHeader);
  l.tokens_at = l.pieces_at + up((size_t)l.pieces * sizeof(Piece));
  l.stats_at = l.tokens_at + up((size_t)total_q * sizeof(Token));
  l.out_at = l.stats_at + up((size_t)l.rows * n_kv_heads * 2 * sizeof(float));
  l.total = l.out_at + (size_t)l.rows * n_kv_heads * head_dim * sizeof(float);
  return l;
}

struct PlanArgs {
  const int32_t* cu_seqlens_q;
  const int32_t* kv_lens;
  const int32_t* cu_groups;
  const int32_t* shared_lens;
  PlanHeader* header;
  Piece* pieces;
  Token* tokens;
  int32_t batch, n_groups, total_q, group, n_kv_heads, table_keys;
  int32_t pieces_capacity, rows_capacity;
};
// LDS of the plan, in words: per request offset, context, group, per group first request, keys, blocks, leader, per set end of pieces, first partial row, parts.
inline size_t plan_lds_bytes(int32_t batch, int32_t n_groups) { return ((size_t)3 * batch + 1 + (size_t)4 * n_groups + 1 + (size_t)3 * (batch + n_groups)) * sizeof(int32_t); }

#if defined(__HIP_DEVICE_COMPILE__)

struct Set {
  int rows, keys, begin;  // rows 0: no set
  int form, blocks, tiles;
};

#endif

__global__ __launch_bounds__(kPlanThreads) void prefix_plan_kernel(const PlanArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ int32_t lds[];
  const int batch = a.batch, groups = a.n_groups, sets = batch + groups;
  int32_t* const s_cu = lds;                    // [batch + 1]
  int32_t* const s_kv = s_cu + batch + 1;       // [batch], 0: the request has no output
  int32_t* const s_group = s_kv + batch;        // [batch]
  int32_t* const s_first = s_group + batch;     // [groups + 1]
  int32_t* const s_keys = s_first + groups + 1; // [groups] shared keys
  int32_t* const s_blocks = s_keys + groups;    // [groups] blocks of 128 rows of its requests one by one
  int32_t* const s_lead = s_blocks + groups;    // [groups] first request that has output
  int32_t* const s_end = s_lead + groups;       // [sets] end of the set's pieces
  int32_t* const s_partial = s_end + sets;      // [sets] first row of its partial results, -1: final results
  int32_t* const s_parts = s_partial + sets;    // [sets]
  __shared__ int32_t s_wave[2][kPlanThreads / 64];
  __shared__ unsigned long long s_cost;
  const int thread = (int)threadIdx.x, lane = thread & 63, wave = thread >> 6;

  for (int i = thread; i <= batch; i += kPlanThreads) {
    const int at = a.cu_seqlens_q[i];
    s_cu[i] = at < 0 ? 0 : (at > a.total_q ? a.total_q : at);
    if (i < batch) {
      const int kv = a.kv_lens[i], end = a.cu_seqlens_q[i + 1], q = end - at;
      s_kv[i] = q > 0 && kv >= q ? (kv < a.table_keys ? kv : a.table_keys) : 0;
    }
  }
  for (int g = thread; g <= groups; g += kPlanThreads) {
    const int at = a.cu_groups[g];
    s_first[g] = at < 0 ? 0 : (at > batch ? batch : at);
    if (g < groups) {
      s_keys[g] = a.shared_lens[g];
      s_blocks[g] = 0;
      s_lead[g] = 0x7fffffff;
    }
  }
  if (thread == 0) s_cost = 0;
  __syncthreads();
  // what all of a group's requests have in common, and what its tokens can all see
  for (int b = thread; b < batch; b += kPlanThreads) {
    int lo = 0, hi = groups - 1;  // the last group that begins at or before b
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_first[mid] <= b) lo = mid;
      else hi = mid - 1;
    }
    s_group[b] = lo;
    const int q = s_cu[b + 1] - s_cu[b];
    if (s_kv[b] > 0) {
      atomicMin(&s_keys[lo], s_kv[b] - q + 1);
      atomicAdd(&s_blocks[lo], (q * a.group + 127) / 128);
      atomicMin(&s_lead[lo], b);
    }
  }
  __syncthreads();
  for (int g = thread; g < groups; g += kPlanThreads) {
    const int first = s_first[g], end = s_first[g + 1] < first ? first : s_first[g + 1];
    const int rows = (s_cu[end] - s_cu[first]) * a.group;
    // (worth it where packing the rows of several requests saves blocks of rows; a chunk of many rows fills its own)
    const bool worth = s_lead[g] < end && 4 * s_blocks[g] >= 5 * ((rows + 127) / 128);
    s_keys[g] = worth && s_keys[g] > 0 ? s_keys[g] / kTileKeys * kTileKeys : 0;
  }
  __syncthreads();

  auto set_of = [&](int i) {
    Set s;
    int end;
    if (i < groups) {
      const int first = s_first[i], last = s_first[i + 1] < first ? first : s_first[i + 1];
      s.begin = 0;
      end = s_keys[i];
      s.rows = end > 0 ? (s_cu[last] - s_cu[first]) * a.group : 0;
    } else {
      const int b = i - groups;
      s.begin = s_kv[b] > 0 ? s_keys[s_group[b]] : 0;
      end = s_kv[b];
      s.rows = end > s.begin ? (s_cu[b + 1] - s_cu[b]) * a.group : 0;
    }
    s.keys = end - s.begin;
    s.form = kKeySplit;
    const int per = rows_of_form(s.form);
    s.blocks = (s.rows + per - 1) / per;
    s.tiles = s.rows > 0 ? (s.keys + kTileKeys - 1) / kTileKeys : 0;
    return s;
  };
  // The cost of everything, and what a piece may cost so that the chip's workgroups have equal shares of it.  (Longer parts by as much
  // as the last tile costs, so cutting adds at most as many pieces as there are shares.)
  {
    int64_t cost = 0;
    for (int i = thread; i < sets; i += kPlanThreads) {
      const Set s = set_of(i);
      cost += (int64_t)s.blocks * s.tiles * cost_of_form(s.form);
    }
    if (cost > 0) atomicAdd(&s_cost, (unsigned long long)cost);
  }
  __syncthreads();
  const int slots = kSlots / a.n_kv_heads > 0 ? kSlots / a.n_kv_heads : 1;
  int64_t share = ((int64_t)s_cost + slots - 1) / slots;
  if (share < kLeastCost) share = kLeastCost;
  auto parts_of = [&](const Set& s) {
    if (s.tiles == 0) return 0;
    const int64_t fair = (share + cost_of_form(s.form) - 1) / cost_of_form(s.form);
    int per = fair < s.tiles ? (int)fair : s.tiles;  // tiles of a part
    const int least = (s.tiles + kMostParts - 1) / kMostParts;
    if (per < least) per = least;
    return (s.tiles + per - 1) / per;
  };

  int pieces_before = 0, rows_before = 0;
  for (int first = 0; first < sets; first += kPlanThreads) {
    const int i = first + thread;
    int pieces = 0, partial_rows = 0, parts = 0;
    bool final = false;
    if (i < sets) {
      const Set s = set_of(i);
      parts = parts_of(s);
      pieces = s.blocks * parts;
      final = i >= groups && parts == 1 && s.begin == 0;
      partial_rows = final ? 0 : pieces * rows_of_form(s.form);
    }
    int pieces_end = wave_scan_add(pieces), rows_end = wave_scan_add(partial_rows);
    if (lane == 63) {
      s_wave[0][wave] = pieces_end;
      s_wave[1][wave] = rows_end;
    }
    __syncthreads();
    int pieces_round = 0, rows_round = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      const int pw = s_wave[0][w], rw = s_wave[1][w];
      pieces_end += w < wave ? pw : 0;
      rows_end += w < wave ? rw : 0;
      pieces_round += pw;
      rows_round += rw;
    }
    if (i < sets) {
      s_end[i] = pieces_before + pieces_end;
      s_partial[i] = final ? -1 : rows_before + rows_end - partial_rows;
      s_parts[i] = parts;
    }
    pieces_before += pieces_round;
    rows_before += rows_round;
    __syncthreads();
  }
  // (cannot be more than there is room for, unless offsets decrease)
  const int n_pieces = pieces_before <= a.pieces_capacity && rows_before <= a.rows_capacity ? pieces_before : 0;
  if (thread == 0) a.header->n_pieces = n_pieces;

  for (int p = thread; p < n_pieces; p += kPlanThreads) {
    int lo = 0, hi = sets - 1;  // the first set that ends behind piece p
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_end[mid] > p) hi = mid;
      else lo = mid + 1;
    }
    const Set s = set_of(lo);
    const int parts = s_parts[lo], number = p - (s_end[lo] - s.blocks * parts), block = number / parts, part = number - block * parts;
    const int per = (s.tiles + parts - 1) / parts * kTileKeys, block_rows = rows_of_form(s.form);
    const int rows = s.rows - block * block_rows < block_rows ? s.rows - block * block_rows : block_rows;
    const bool shared = lo < groups;
    const int request = shared ? s_lead[lo] : lo - groups;
    Piece piece;
    piece.table_row = request;
    piece.key_begin = s.begin + part * per;
    piece.key_end = part * per + per < s.keys ? piece.key_begin + per : s.begin + s.keys;
    piece.limit = shared ? 0x3fffffff : s_kv[request] - (s_cu[request + 1] - s_cu[request]);  // (every token of a group sees all shared keys)
    piece.first_token = shared ? s_cu[s_first[lo]] : s_cu[request];
    piece.first_row = block * block_rows;
    piece.form_rows = s.form * 256 + rows;
    piece.partial = s_partial[lo] < 0 ? -1 : s_partial[lo] + number * block_rows;
    a.pieces[p] = piece;
  }
  for (int t = thread; t < a.total_q; t += kPlanThreads) {
    int lo = 0, hi = batch - 1;  // the first request that ends behind token t
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_cu[mid + 1] > t) hi = mid;
      else lo = mid + 1;
    }
    Token token = {};
    if (n_pieces > 0 && s_kv[lo] > 0 && t >= s_cu[lo] && t < s_cu[lo + 1]) {
      auto part_of = [&](int set, int first_token) {
        TokenPart part = {};
        if (s_parts[set] == 0 || s_partial[set] < 0) return part;
        part.first = s_partial[set];
        part.parts = s_parts[set];
        part.rows = rows_of_form(set_of(set).form);
        part.token = t - first_token;
        return part;
      };
      token.own = part_of(groups + lo, s_cu[lo]);
      const int g = s_group[lo];
      if (s_keys[g] > 0) token.shared = part_of(g, s_cu[s_first[g]]);
    }
    a.tokens[t] = token;
  }
#else
  (void)a;
#endif
}

}  // namespace prefix
}  // namespace hydra
