// Block tables of a step, from the lengths on the device: blocks taken from a ring of free ones and given back to it,
// offsets and lengths of the sequences, position and slot of every new token.
//
//   len_b = kv_len_b + new_b        need_b = ceil(len_b / 16)
//   take_b = max(0, need_b - held_b)        give_b = max(0, held_b - max(need_b, shared_b))
//
// The i-th block taken (by sequence, then by place in the row) is ring[head + i], the i-th given goes to
// ring[head + count + i]: neither depends on the order in which threads run, and what one part of the step reads no
// other part writes.  The sums over the sequences are scans by one CTA, which also finds out whether the step can be
// made at all; a second kernel writes what the sums are the offsets of.
//
// Bound by latency in a step of single tokens, by the 12 bytes a token in a round of prompts.
#include <algorithm>

#include "kv.h"
#include "rotary.cuh"

using namespace misat;

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanEach = 4;  // sequences of a thread a round
constexpr int kThreads = 256;
constexpr int kRun = 128;     // tokens, or blocks given back, of a warp at a time

struct TableArgs {
  int32_t n, n_tokens, max_q, columns, ring_size;
  int64_t stride;
  const int32_t* fresh;  // new tokens
  const int32_t* kv_len;
  const int32_t* shared;
  const int32_t* state;
  int32_t* table;
  int32_t* ring;
  int32_t* state_out;
  int32_t* q_off;
  int32_t* kv_len_out;
  int32_t* positions;
  int64_t* slots;
  int32_t* err;
  // What the second kernel needs of the first: per sequence blocks held before, blocks taken and given before it, first
  // block given; then Head.
  int32_t *held, *take_off, *give_off, *give_from, *head;
};
enum Head { kOk, kRingHead, kGiveBase, kGiven, kHeadWords };

// Sums that stay at the largest number where they would pass it: malformed counts cannot wrap around.
__device__ __forceinline__ uint32_t sat(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }
struct Sums {
  uint32_t fresh, take, give;
  __device__ __forceinline__ void add(const Sums& r) {
    fresh = sat(fresh, r.fresh);
    take = sat(take, r.take);
    give = sat(give, r.give);
  }
};

struct Row {
  int fresh, len, held, from;  // from: first block that may be given back
  bool ok;
  __device__ __forceinline__ int need() const { return (len + kBlockTokens - 1) / kBlockTokens; }
  __device__ __forceinline__ Sums sums() const {
    return {(uint32_t)fresh, (uint32_t)max(need() - held, 0), (uint32_t)max(held - from, 0)};
  }
};
__device__ __forceinline__ Row load_row(const TableArgs& a, int b) {
  if (b >= a.n) return {0, 0, 0, 0, true};
  const int fresh = __ldcg(a.fresh + b), before = __ldcg(a.kv_len + b), held = __ldcg(a.state + b);
  const int shared = a.shared ? __ldcg(a.shared + b) : 0;
  // A row holds blocks for the tokens that are there, and has room for those to come.
  const bool ok = fresh >= 0 && fresh <= a.max_q && before >= 0 && before <= kMaxLen && fresh <= kMaxLen - before &&
                  held >= 0 && held <= a.columns && (int64_t)before <= (int64_t)held * kBlockTokens && shared >= 0 &&
                  shared <= held && (int64_t)before + fresh <= (int64_t)a.columns * kBlockTokens;
  if (!ok) return {0, 0, 0, 0, false};
  Row r{fresh, before + fresh, held, 0, true};
  r.from = max(r.need(), shared);
  return r;
}

__global__ void __launch_bounds__(kPlanThreads) k_table_plan(const __grid_constant__ TableArgs a) {
  __shared__ Sums part[kPlanThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  chain_wait();
  // Sum over the threads before this one (returned), and over all (in `all`).
  auto scan = [&](Sums v, Sums& all) {
    Sums inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Sums t{__shfl_up_sync(0xffffffffu, inc.fresh, o), __shfl_up_sync(0xffffffffu, inc.take, o),
                   __shfl_up_sync(0xffffffffu, inc.give, o)};
      if (lane >= o) inc.add(t);
    }
    __syncthreads();
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    Sums before{0, 0, 0};
    all = Sums{0, 0, 0};
#pragma unroll 1
    for (int i = 0; i < kPlanThreads / 32; ++i) {
      if (i == warp) before = all;
      all.add(part[i]);
    }
    const Sums left{__shfl_up_sync(0xffffffffu, inc.fresh, 1), __shfl_up_sync(0xffffffffu, inc.take, 1),
                    __shfl_up_sync(0xffffffffu, inc.give, 1)};
    if (lane > 0) before.add(left);
    return before;
  };
  constexpr int kRound = kPlanThreads * kPlanEach;
  Sums total{0, 0, 0};
  bool ok = true;
  for (int b0 = 0; b0 < a.n; b0 += kRound) {
    Sums mine{0, 0, 0}, all;
#pragma unroll
    for (int i = 0; i < kPlanEach; ++i) {
      const Row r = load_row(a, b0 + tid * kPlanEach + i);
      ok = ok && r.ok;
      mine.add(r.sums());
    }
    scan(mine, all);
    total.add(all);
  }
  const int head = __ldcg(a.state + a.n), count = __ldcg(a.state + a.n + 1);
  ok = ok && total.fresh == (uint32_t)a.n_tokens && head >= 0 && head < a.ring_size && count >= 0 &&
       count <= a.ring_size && (int64_t)count + total.give <= a.ring_size;
  const bool sound = __syncthreads_and(ok);
  const bool enough = total.take <= (uint32_t)max(count, 0), go = sound && enough;
  Sums base{0, 0, 0};
  for (int b0 = 0; b0 < a.n; b0 += kRound) {
    Row r[kPlanEach];
    Sums mine{0, 0, 0}, all;
#pragma unroll
    for (int i = 0; i < kPlanEach; ++i) {
      r[i] = load_row(a, b0 + tid * kPlanEach + i);
      mine.add(r[i].sums());
    }
    Sums at = base;
    at.add(scan(mine, all));
    base.add(all);
#pragma unroll
    for (int i = 0; i < kPlanEach; ++i) {
      const int b = b0 + tid * kPlanEach + i;
      if (b >= a.n) break;
      if (go) {
        a.held[b] = r[i].held;
        a.take_off[b] = (int)at.take;
        a.give_off[b] = (int)at.give;
        a.give_from[b] = r[i].from;
        a.q_off[b] = (int)at.fresh;
        a.kv_len_out[b] = r[i].len;
        a.state_out[b] = r[i].need();
      } else {
        a.q_off[b] = 0;
        if (a.kv_len_out != a.kv_len) a.kv_len_out[b] = __ldcg(a.kv_len + b);
        if (a.state_out != a.state) a.state_out[b] = __ldcg(a.state + b);
      }
      at.add(r[i].sums());
    }
  }
  if (tid == 0) {
    a.q_off[a.n] = go ? a.n_tokens : 0;
    a.give_off[a.n] = (int)total.give;
    a.head[kOk] = go;
    if (go) {
      const int take = (int)total.take, give = (int)total.give;
      a.head[kRingHead] = head;
      a.head[kGiveBase] = (int)(((int64_t)head + count) % a.ring_size);
      a.head[kGiven] = give;
      a.state_out[a.n] = (int)(((int64_t)head + take) % a.ring_size);
      a.state_out[a.n + 1] = count - take + give;
    } else {
      set_error(a.err, sound ? MISAT_ERR_OOM : MISAT_ERR_INVALID_ARG);
      a.state_out[a.n] = head;
      a.state_out[a.n + 1] = count;
    }
  }
}

__global__ void __launch_bounds__(kThreads) k_table_fill(const __grid_constant__ TableArgs a) {
  const int lane = threadIdx.x & 31;
  const int warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kThreads / 32);
  chain_wait();
  const bool go = __ldcg(a.head + kOk) != 0;
  const int runs = (a.n_tokens + kRun - 1) / kRun;
  if (!go) {
    for (int r = warp; r < runs; r += warps)
      for (int t = r * kRun + lane; t < min((r + 1) * kRun, a.n_tokens); t += 32) {
        a.positions[t] = -1;
        a.slots[t] = -1;
      }
    return;
  }
  const int ring_head = __ldcg(a.head + kRingHead), base = __ldcg(a.head + kGiveBase), given = __ldcg(a.head + kGiven);
  auto place = [&](int first, int i) {  // of the ring
    const int64_t p = (int64_t)first + i;
    return (int)(p >= a.ring_size ? p - a.ring_size : p);
  };
  for (int r = warp; r < runs; r += warps) {
    const int t0 = r * kRun;
    OffsetFinder find(a.q_off, a.n, t0);
#pragma unroll 1
    for (int i = 0; i < kRun && t0 + i < a.n_tokens; i += 32) {
      const int t = min(t0 + i + lane, a.n_tokens - 1);
      const int b = find(t);
      const int pos = __ldcg(a.kv_len_out + b) - __ldcg(a.q_off + b + 1) + t, col = pos / kBlockTokens;
      const int held = __ldcg(a.held + b);
      int blk = -1;
      if (pos >= 0 && col < a.columns) {
        int32_t* row = a.table + (int64_t)b * a.stride;
        if (col < held) {
          blk = __ldcg(row + col);
        } else {
          const int k = __ldcg(a.take_off + b) + col - held;
          if (k >= 0 && k < a.ring_size) {
            blk = __ldcg(a.ring + place(ring_head, k));
            if (pos % kBlockTokens == 0) row[col] = blk;
          }
        }
      }
      if (t0 + i + lane < a.n_tokens) {
        a.positions[t] = pos;
        a.slots[t] = (int64_t)blk * kBlockTokens + pos % kBlockTokens;
      }
    }
  }
  for (int r = warp; r < (given + kRun - 1) / kRun; r += warps) {
    const int j0 = r * kRun;
    OffsetFinder find(a.give_off, a.n, j0);
#pragma unroll 1
    for (int i = 0; i < kRun && j0 + i < given; i += 32) {
      const int j = min(j0 + i + lane, given - 1);
      const int b = find(j);
      const int col = __ldcg(a.give_from + b) + j - __ldcg(a.give_off + b);
      if (j0 + i + lane < given && col >= 0 && col < a.columns)
        a.ring[place(base, j)] = __ldcg(a.table + (int64_t)b * a.stride + col);
    }
  }
}

}  // namespace

extern "C" {

int misat_kv_tables(misat_kv* kv, const misat_kv_step* s, void* work, int64_t work_bytes, void* cuda_stream) {
  if (!kv || !s || s->n < 0 || s->n > kv->max_batch || s->n_tokens < 0 || s->n_tokens == INT32_MAX || s->max_q < 0 ||
      s->columns < 0 || s->table_stride < s->columns || s->ring_size < 1 || (s->n == 0 && s->n_tokens > 0))
    return MISAT_ERR_INVALID_ARG;
  if (!s->q_off || !s->state || !s->state_out || !s->ring ||
      (s->n > 0 && (!s->new_tokens || !s->kv_len || !s->kv_len_out || (!s->block_table && s->columns > 0))) ||
      (s->n_tokens > 0 && (!s->positions || !s->slots)) || !work || (reinterpret_cast<uintptr_t>(work) & 3) ||
      work_bytes < MISAT_KV_TABLES_WORK(s->n) || !on_device(kv->device))
    return MISAT_ERR_INVALID_ARG;
  TableArgs a{};
  a.n = s->n;
  a.n_tokens = s->n_tokens;
  a.max_q = s->max_q;
  a.columns = s->columns;
  a.ring_size = s->ring_size;
  a.stride = s->table_stride;
  a.fresh = s->new_tokens;
  a.kv_len = s->kv_len;
  a.shared = s->shared;
  a.state = s->state;
  a.table = s->block_table;
  a.ring = s->ring;
  a.state_out = s->state_out;
  a.q_off = s->q_off;
  a.kv_len_out = s->kv_len_out;
  a.positions = s->positions;
  a.slots = s->slots;
  a.err = kv->err;
  int32_t* w = static_cast<int32_t*>(work);
  a.head = w;
  a.held = w + 4;
  a.take_off = a.held + s->n;
  a.give_from = a.take_off + s->n;
  a.give_off = a.give_from + s->n;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  launch_chained(k_table_plan, 1, kPlanThreads, 0, st, a);
  // Warps for the tokens, and for blocks given back (as many as a sequence may have, at most).
  const int64_t warps = std::max<int64_t>(((int64_t)s->n_tokens + kRun - 1) / kRun, (s->n + 1) / 2);
  const int64_t most = (int64_t)kv->num_sms * 8;
  if (warps > 0)
    launch_chained(k_table_fill, (int)std::min((warps + kThreads / 32 - 1) / (kThreads / 32), most), kThreads, 0, st, a);
  return launch_status();
}

}  // extern "C"
