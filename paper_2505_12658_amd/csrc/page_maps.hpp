// Page maps of a step: blocks off the free list, block tables, slots, positions, offsets and context lengths (include/hydra_step.h).
//
// Two sums run over the requests, of new tokens and of new blocks; everything else follows from a request's place in them.  Every
// workgroup takes both sums over the batch, some requests per thread and round, until its own tokens are past, and keeps the round that they lie in;
// a token then finds its request in LDS.  So one launch does, without a second one that would wait for the sums of a first: the
// lengths are some KB that every workgroup after the first finds in L2.
//
// What bounds it: latency, of the lengths, the barriers and the table.  us: 96 decode steps 2.9, 700 3.7, 2000 5.9; prefills of 610 tokens, 100 3.5, 400
// 5.4, 1024 (8 MB written) 8.2.  (Workgroups of 1024 threads with four tokens each: 4.6, 5.1, 9.9; 6.0, 8.0, 9.7.)
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wave_ops.hpp"

namespace hydra {
namespace maps {

constexpr int kThreads = 256;         // of a workgroup
constexpr int kMostTokens = 1 << 20;  // per step: the sums of a round of 1024 lengths that are held to one more than this fit 31 bits, behind as many before them

struct Args {
  const int32_t* q_lens;
  const int32_t* context_lens;
  int32_t* block_tables;
  const int32_t* free_blocks;
  const int32_t* n_free;
  const int32_t* position_deltas;
  int32_t* cu_seqlens_q;
  int32_t* kv_lens;
  int64_t* slot_mapping;
  int32_t* positions;
  int32_t* next_context;
  int32_t* pool;
  int32_t free_capacity, max_blocks_per_seq, batch, total_tokens, tokens_each, block_shift, num_blocks;
};

// grid: a workgroup per tokens_each tokens.  EACH: requests of a thread in a round, next to each other.  TOKENS: tokens, tables and what a request gets; STATE: next_context and pool.
// Both in one launch unless several workgroups would still read what they overwrite (the same arrays as context_lens and n_free).
template <int EACH, bool TOKENS, bool STATE>
__global__ __launch_bounds__(kThreads) void page_maps_kernel(const Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kWaves = kThreads / 64, kRound = kThreads * EACH, kGroup = kRound / 64;
  static_assert(EACH <= 4, "see kMostTokens");
  __shared__ int32_t s_end[kRound], s_context[kRound], s_first[kRound];  // per request: end of its tokens, context, place of its first new block on the list
  __shared__ int32_t s_wave[2][kWaves];
  __shared__ int32_t s_taken, s_wanted;  // blocks off the list, and blocks that all the requests of the step need
  const int thread = (int)threadIdx.x, lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const int n_free_given = *a.n_free;
  const int n_free = n_free_given < 0 ? 0 : (n_free_given > a.free_capacity ? a.free_capacity : n_free_given);
  const int in_block = (1 << a.block_shift) - 1;
  auto least = [](int x, int y) { return y < x ? y : x; };
  const int begin = (int)blockIdx.x * a.tokens_each;
  const int end = least(begin + a.tokens_each, a.total_tokens);
  if (thread == 0) s_taken = s_wanted = 0;
  int tokens_before = 0, blocks_before = 0;  // of the requests of earlier rounds
  int q[EACH], context[EACH];
  auto lengths_of = [&](int first) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int b = first + EACH * thread + e;
      q[e] = context[e] = 0;
      if (b < a.batch) {
        q[e] = a.q_lens[b];
        context[e] = a.context_lens[b];
      }
    }
  };
  lengths_of(0);
  for (int first = 0; first < a.batch; first += kRound) {
    int need[EACH], q_sum = 0, need_sum = 0;
    bool fits_row[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      q[e] = q[e] < 0 ? 0 : (q[e] > kMostTokens ? kMostTokens + 1 : q[e]);
      fits_row[e] = context[e] >= 0 && (int64_t)context[e] + q[e] <= (int64_t)a.max_blocks_per_seq << a.block_shift;
      const int held = fits_row[e] ? (int)(((int64_t)context[e] + in_block) >> a.block_shift) : 0;
      need[e] = fits_row[e] ? (int)(((int64_t)context[e] + q[e] + in_block) >> a.block_shift) - held : 0;  // (no more than q)
      q_sum += q[e];
      need_sum += need[e];
    }
    int q_end = wave_scan_add(q_sum), need_end = wave_scan_add(need_sum);
    if (lane == 63) {
      s_wave[0][wave] = q_end;
      s_wave[1][wave] = need_end;
    }
    __syncthreads();
    int q_round = 0, need_round = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int qw = s_wave[0][w], nw = s_wave[1][w];
      q_end += w < wave ? qw : 0;
      need_end += w < wave ? nw : 0;
      q_round += qw;
      need_round += nw;
    }
    q_end += tokens_before - q_sum;
    need_end += blocks_before - need_sum;
    int taken = -1, wanted = -1;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int b = first + EACH * thread + e;
      q_end += q[e];
      need_end += need[e];
      const bool in_step = q[e] == 0 || q_end <= a.total_tokens;
      const bool served = fits_row[e] && in_step && (need[e] == 0 || need_end <= n_free);
      const int token_end = q_end < a.total_tokens ? q_end : a.total_tokens;
      if (STATE) {
        taken = need[e] > 0 && served ? need_end : taken;
        wanted = need[e] > 0 && in_step ? need_end : wanted;
        if (a.next_context && blockIdx.x == 0 && b < a.batch) a.next_context[b] = served ? context[e] + q[e] : context[e];
      }
      if (TOKENS) {
        if (blockIdx.x == 0 && b < a.batch) {
          a.cu_seqlens_q[b + 1] = token_end;
          a.kv_lens[b] = served ? context[e] + q[e] : 0;
          if (b == 0) a.cu_seqlens_q[0] = 0;
        }
        s_end[EACH * thread + e] = token_end;
        s_context[EACH * thread + e] = context[e];
        s_first[EACH * thread + e] = served ? n_free - 1 - (need_end - need[e]) : -1 - (1 << 30);
      }
    }
    if (STATE && blockIdx.x == 0) {
      // (sums only grow, and those that are served with new blocks come before those that are not)
      auto last = [&](int sum, int32_t* most) {
        const uint64_t lanes = __builtin_amdgcn_ballot_w64(sum >= 0);
        if (lanes != 0 && lane == 63 - __builtin_clzll(lanes)) atomicMax(most, sum);
      };
      last(taken, &s_taken);
      last(wanted, &s_wanted);
    }
    __syncthreads();
    if (first + kRound < a.batch) lengths_of(first + kRound);  // (on their way while this round's tokens are written)
    if (TOKENS) {
      const int round_begin = tokens_before > begin ? tokens_before : begin;
      int round_end = tokens_before + q_round;
      round_end = round_end < end ? round_end : end;
      const int in_round = least(a.batch - first, kRound);
      const bool long_ones = q_round > 16 * in_round;
      for (int t0 = round_begin + 64 * wave; t0 < round_end; t0 += kThreads) {
        const int t = t0 + lane < round_end ? t0 + lane : round_end - 1;
        // The token's request, the first one that ends behind it: where requests have many tokens, that of the wave's first token (of 64
        // groups, and then of one's members), which is mostly all the others' too; otherwise by a search of each lane's own.
        int lo = 0, hi = in_round - 1;
        if (long_ones) {
          const int group_end = least(kGroup * lane + kGroup - 1, hi);
          lo = kGroup * __builtin_popcountll(__builtin_amdgcn_ballot_w64(kGroup * lane <= hi && s_end[group_end] <= t0));
          lo += __builtin_ctzll(__builtin_amdgcn_ballot_w64(s_end[least(lo + lane % kGroup, hi)] > t0));
          if (s_end[lo] > t0 + 63) hi = lo;
        }
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (s_end[mid] > t) hi = mid;
          else lo = mid + 1;
        }
        const int start = lo > 0 ? s_end[lo - 1] : tokens_before;
        const int of = first + lo, held_tokens = s_context[lo], at = s_first[lo];
        const int position = (int)((uint32_t)held_tokens + (uint32_t)(t - start));
        int64_t slot = -1;
        if (at >= -1 - kMostTokens) {  // served  (the place may be below 0 only where no new block is needed)
          const int page = position >> a.block_shift, held_pages = (int)(((int64_t)held_tokens + in_block) >> a.block_shift);
          int32_t* entry = a.block_tables + (int64_t)of * a.max_blocks_per_seq + page;
          int block;
          if (page >= held_pages) {
            block = a.free_blocks[at - (page - held_pages)];
            if ((position & in_block) == 0) *entry = block;  // (every new block begins with a new token)
          } else {
            block = *entry;
          }
          if (block >= 0 && block < a.num_blocks) slot = ((int64_t)block << a.block_shift) + (position & in_block);
        }
        a.slot_mapping[t] = slot;
        if (a.positions) a.positions[t] = (int)((uint32_t)position + (a.position_deltas ? (uint32_t)a.position_deltas[of] : 0u));
      }
    }
    tokens_before += q_round;
    tokens_before = tokens_before < a.total_tokens ? tokens_before : a.total_tokens;
    blocks_before += need_round;
    blocks_before = blocks_before < 1 << 29 ? blocks_before : 1 << 29;  // (more only where the tokens are beyond total_tokens)
    if (blockIdx.x != 0 && tokens_before >= end) return;  // (the first workgroup has every request's results to write)
    __syncthreads();
  }
  if (TOKENS) {
    for (int t = (tokens_before > begin ? tokens_before : begin) + thread; t < end; t += kThreads) {
      a.slot_mapping[t] = -1;
      if (a.positions) a.positions[t] = 0;
    }
  }
  if (STATE && blockIdx.x == 0 && thread == 0) {
    a.pool[0] = n_free - s_taken;
    a.pool[1] = s_wanted > n_free ? s_wanted - n_free : 0;
  }
#else
  (void)a;
#endif
}

}  // namespace maps
}  // namespace hydra
