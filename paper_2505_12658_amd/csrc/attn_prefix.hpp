// Attention over the paged cache of requests that share prefixes: the pieces of a plan (prefix_plan.hpp), and the merge of their
// partial results.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_paged.hpp"
#include "prefix_plan.hpp"

namespace hydra {
namespace prefix {

struct Args {
  paged::PagedArgs paged;  // queries, output, cache and table as in the paged call; its lengths and shares are not used
  const PlanHeader* header;
  const Piece* pieces;
  const Token* tokens;
  float* stats;        // [n_kv_heads][rows] maximum, sum
  float* partial_out;  // [n_kv_heads][rows][D]
  int64_t rows;        // of partial results of a KV head
  int32_t total_q;
};

#if defined(__HIP_DEVICE_COMPILE__)

// A block of up to 32 rows; the four waves split the keys: wave w takes the blocks of 32 keys w, w + 4, .. of the piece through a stage of its
// own, and the four partial results are merged through LDS.
template <int D>
__device__ __forceinline__ void run_key_split(const Args& args, const Piece& piece, int kv_head, unsigned char* smem, float* s_stats) {
  using G = paged::StageGeom<D>;
  using W = paged::WaveTile<D, 1>;
  constexpr int kHalfKeys = kKvTileRows / 2, kWaves = paged::kWavesPerGroup;
  const paged::PagedArgs& a = args.paged;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 31;
  const int n_rows = piece.form_rows & 255;

  W w;
  w.init(lane, a.scale_log2);
  const bool valid = m < n_rows;
  const int row = piece.first_row + (valid ? m : n_rows - 1);
  const int token = row / a.group, head = kv_head * a.group + (row - token * a.group);
  w.load_q(0, a.q + (int64_t)(piece.first_token + token) * a.q_stride + head * D, piece.limit + token);
  const int first_limit = piece.limit + piece.first_row / a.group;  // of the block's first row: keys up to it need no mask

  const int32_t* table = a.block_tables + (int64_t)piece.table_row * a.max_blocks_per_seq;
  unsigned char* stage = smem + wave * G::kSlotBytes;
  const int end = piece.key_end;
  int key = piece.key_begin + wave * kHalfKeys;
  constexpr int kStep = kWaves * kHalfKeys;
  paged::TileSlots<D, kHalfKeys, 1> slots;
  paged::TileRegs<D, kHalfKeys> regs;
  if (key < end) {
    paged::fetch_tile_slots(slots, a, table, 0, lane, end, key);
    paged::load_tile_regs(regs, slots, a, lane, kv_head);
    if (key + kStep < end) paged::request_tile_blocks(slots, a, table, 0, lane, end, key + kStep);
  }
  for (; key < end; key += kStep) {
    paged::store_tile_regs(regs, stage, lane);
    if (key + kStep < end) {
      paged::slots_from_blocks(slots, a, 0, lane, end, key + kStep);
      paged::load_tile_regs(regs, slots, a, lane, kv_head);
      if (key + 2 * kStep < end) paged::request_tile_blocks(slots, a, table, 0, lane, end, key + 2 * kStep);
    }
    __builtin_amdgcn_sched_barrier(0);  // (the loads go out before the arithmetic)
    w.template tile<1>(stage, key, key + kHalfKeys - 1 > first_limit || key + kHalfKeys > end);
  }

  // ---- merge of the waves (see run_packed_rows) ----
  s_stats[wave * 64 + lane] = w.row_max[0];
  s_stats[256 + wave * 64 + lane] = w.row_sum[0];
  float* mine = reinterpret_cast<float*>(stage);
#pragma unroll
  for (int cc = 0; cc < W::CC; ++cc)
#pragma unroll
    for (int i = 0; i < 16; ++i) mine[(cc * 16 + i) * 64 + lane] = w.o_acc[0][cc][i];
  __syncthreads();
  if (wave != 0) return;
  float scale_of[kWaves];
  float top = s_stats[lane];
#pragma unroll
  for (int o = 1; o < kWaves; ++o) top = fmaxf(top, s_stats[o * 64 + lane]);
  float total = 0.f;
#pragma unroll
  for (int o = 0; o < kWaves; ++o) {
    scale_of[o] = fast_exp2((s_stats[o * 64 + lane] - top) * w.c);
    total += scale_of[o] * s_stats[256 + o * 64 + lane];
  }
#pragma unroll
  for (int cc = 0; cc < W::CC; ++cc)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float acc = 0.f;
#pragma unroll
      for (int o = 0; o < kWaves; ++o) acc += scale_of[o] * reinterpret_cast<const float*>(smem + o * G::kSlotBytes)[(cc * 16 + i) * 64 + lane];
      w.o_acc[0][cc][i] = acc;
    }
  w.row_sum[0] = total;
  if (piece.partial < 0) {
    w.store_row(0, valid ? a.out + ((int64_t)(piece.first_token + token) * a.n_q_heads + head) * D : nullptr);
    return;
  }
  const float sum = sum_with_other_half(total);
  const int64_t at = kv_head * args.rows + piece.partial + m;
  if (valid) {
    if (w.hf == 0) *reinterpret_cast<f32x2_t*>(args.stats + 2 * at) = f32x2_t{top, sum};
#pragma unroll
    for (int cc = 0; cc < W::CC; ++cc)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const int col = 32 * cc + 8 * g4 + 4 * w.hf;
        if (col < D)
          *reinterpret_cast<f32x4_t*>(args.partial_out + at * D + col) =
              f32x4_t{w.o_acc[0][cc][4 * g4], w.o_acc[0][cc][4 * g4 + 1], w.o_acc[0][cc][4 * g4 + 2], w.o_acc[0][cc][4 * g4 + 3]};
      }
  }
}

#endif  // __HIP_DEVICE_COMPILE__

// grid: a workgroup per piece (of the plan's capacity) and KV head
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_prefix_kernel(const Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) unsigned char smem[paged::StageGeom<D>::kLdsBytes];
  __shared__ float s_stats[2 * 4 * 64];
  const int number = (int)blockIdx.x / a.paged.n_kv_heads, kv_head = (int)blockIdx.x - number * a.paged.n_kv_heads;
  if (number >= a.header->n_pieces) return;
  const Piece piece = a.pieces[number];
  run_key_split<D>(a, piece, kv_head, smem, s_stats);
#else
  (void)a;
#endif
}

// Merge: a wave per (token, query head); a row's columns are dealt four to a lane, and D / 4 lanes that have them all take every
// kStreams-th partial result.
constexpr int kMergeWaves = 4;
template <int D>
__global__ __launch_bounds__(64 * kMergeWaves) void prefix_merge_kernel(const Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kLanes = D / 4, kStreams = 64 / kLanes, kEach = 2 * kMostParts / 64;
  const int lane = (int)threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * kMergeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = (int)(unit / a.paged.n_q_heads), head = (int)(unit - (int64_t)t * a.paged.n_q_heads);
  if (t >= a.total_q) return;
  const Token token = a.tokens[t];
  const int n = token.own.parts + token.shared.parts;
  if (n == 0) return;  // written by its one piece, or a token without output
  const int kv_head = head / a.paged.group, in_group = head - kv_head * a.paged.group;
  // row of partial results of this row's part number i (the request's own ones first), and the distance to the next one's
  auto first_of = [&](const TokenPart& p) {
    if (p.parts == 0) return 0;
    const int row = p.token * a.paged.group + in_group, block = row / p.rows;
    return p.first + block * p.parts * p.rows + (row - block * p.rows);
  };
  const int own = first_of(token.own), shared = first_of(token.shared);
  const int64_t base = kv_head * a.rows;
  auto row_of = [&](int i) { return base + (i < token.own.parts ? own + i * token.own.rows : shared + (i - token.own.parts) * token.shared.rows); };
  // lane i: statistics of parts i and i + 64
  f32x2_t stat[kEach];
  float top = kLowest;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int i = e * 64 + lane;
    stat[e] = f32x2_t{kLowest, 0.f};
    if (i < n) stat[e] = *reinterpret_cast<const f32x2_t*>(a.stats + 2 * row_of(i));
    top = fmaxf(top, stat[e][0]);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  float total = 0.f, weight[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    weight[e] = fast_exp2((stat[e][0] - top) * a.paged.scale_log2);
    total += weight[e] * stat[e][1];
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
  const int stream = lane / kLanes, col = (lane - stream * kLanes) * 4;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < n; i0 += kStreams) {
    const int i = i0 + stream;
    const float w0 = __shfl(weight[0], i & 63), w1 = __shfl(weight[1], i & 63), w = i < 64 ? w0 : w1;
    if (stream < kStreams && i < n) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.partial_out + row_of(i) * D + col);
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[x] += w * v[x];
    }
  }
  // the streams' sums, all in the first one's lanes
  f32x4_t sum = acc;
#pragma unroll
  for (int s = 1; s < kStreams; ++s)
#pragma unroll
    for (int x = 0; x < 4; ++x) sum[x] += __shfl(acc[x], (lane + s * kLanes) & 63);
  if (stream != 0) return;
  const float inv = 1.0f / total;
  const f32x2_t a0 = {sum[0] * inv, sum[1] * inv}, a1 = {sum[2] * inv, sum[3] * inv};
  const u32x2_t pk = {__builtin_bit_cast(uint32_t, __builtin_convertvector(a0, bf16x2_t)), __builtin_bit_cast(uint32_t, __builtin_convertvector(a1, bf16x2_t))};
  *reinterpret_cast<u32x2_t*>(a.paged.out + ((int64_t)t * a.paged.n_q_heads + head) * D + col) = pk;
#else
  (void)a;
#endif
}

}  // namespace prefix
}  // namespace hydra
