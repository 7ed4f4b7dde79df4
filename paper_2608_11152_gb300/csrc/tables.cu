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
constexpr int kThreads = 256;
constexpr int kEach = 4;                   // tokens of a lane side by side
constexpr int kAhead = 4;                  // times that many tokens of a warp on their way together
constexpr int kRun = 32 * kEach * kAhead;  // tokens of a warp at a time
constexpr int kGiveRun = 128;              // blocks given back
constexpr int kFillTokens = 4096;          // most tokens of a step that one CTA makes

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
  bool whole;  // positions and slots at 16-byte boundaries
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

// What the tokens' places follow from, in memory between two kernels or in shared memory.
struct Plan {
  const int32_t *q_off, *len, *held, *take_off, *give_off, *give_from;
  int ring_head, give_base, given;
};

__device__ __forceinline__ int ring_place(const TableArgs& a, int first, int i) {
  const int64_t p = (int64_t)first + i;
  return (int)(p >= a.ring_size ? p - a.ring_size : p);
}
// Block of a position of sequence b, of whose row `held` places were filled before the step: from the row, or from the
// ring (not from the row, into which the token that begins the block puts it).
struct Place {
  const int32_t* from;
  int32_t* row;
};
__device__ __forceinline__ Place place_of(const TableArgs& a, int b, int col, int held, int take_off, int ring_head) {
  int32_t* row = a.table + (int64_t)b * a.stride + col;
  const int k = take_off + col - held;
  if (col < 0 || col >= a.columns || k >= a.ring_size) return {nullptr, nullptr};
  if (col < held) return {row, nullptr};
  return {a.ring + ring_place(a, ring_head, k), row};
}
// One block given back: the j-th of all.
__device__ __forceinline__ void give(const TableArgs& a, const Plan& p, int b, int j, int from, int off) {
  const int col = from + j - off;
  if (col >= 0 && col < a.columns)
    a.ring[ring_place(a, p.give_base, j)] = __ldcg(a.table + (int64_t)b * a.stride + col);
}

// The last i with off[i] <= t, off in shared memory with off[n] > t.
__device__ __forceinline__ int search(const int32_t* off, int n, int t) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (off[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

// EACH: sequences of a thread a round; up to EACH x 1,024 of them stay in registers between the sums and the writes.
// FILL: one round, and this CTA writes the tokens' places too, from shared memory.
template <int EACH, bool FILL>
__global__ void __launch_bounds__(kPlanThreads) k_table_plan(const __grid_constant__ TableArgs a) {
  constexpr int kWarps = kPlanThreads / 32, kRound = kPlanThreads * EACH, kSeqs = FILL ? kRound : 1;
  __shared__ Sums part[kWarps];
  __shared__ int32_t s_q[kSeqs + 1], s_len[kSeqs], s_held[kSeqs], s_take[kSeqs], s_give[kSeqs + 1], s_from[kSeqs];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  chain_wait();
  auto shuffled = [](const Sums& v, int from) {
    return Sums{__shfl_sync(0xffffffffu, v.fresh, from), __shfl_sync(0xffffffffu, v.take, from),
                __shfl_sync(0xffffffffu, v.give, from)};
  };
  auto scan_warp = [&](Sums v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Sums t = shuffled(v, lane - o);
      if (lane >= o) v.add(t);
    }
    return v;
  };
  // Sum over the threads before this one (returned), and over all (in `all`).
  auto scan = [&](Sums v, Sums& all) {
    const Sums inc = scan_warp(v);
    __syncthreads();
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    const Sums warps = scan_warp(part[lane]);
    all = shuffled(warps, kWarps - 1);
    const Sums ahead = shuffled(warps, max(warp - 1, 0)), left = shuffled(inc, max(lane - 1, 0));
    Sums before{0, 0, 0};
    if (warp > 0) before.add(ahead);
    if (lane > 0) before.add(left);
    return before;
  };
  Row r[EACH];
  auto load = [&](int b0) {
    Sums mine{0, 0, 0};
#pragma unroll
    for (int i = 0; i < EACH; ++i) r[i] = load_row(a, b0 + tid * EACH + i);
#pragma unroll
    for (int i = 0; i < EACH; ++i) mine.add(r[i].sums());
    return mine;
  };
  const int head = __ldcg(a.state + a.n), count = __ldcg(a.state + a.n + 1);
  Sums total{0, 0, 0}, at{0, 0, 0}, all;
  bool ok = true;
  for (int b0 = 0; b0 == 0 || b0 < a.n; b0 += kRound) {
    const Sums mine = load(b0);
#pragma unroll
    for (int i = 0; i < EACH; ++i) ok = ok && r[i].ok;
    at = scan(mine, all);
    total.add(all);
  }
  ok = ok && total.fresh == (uint32_t)a.n_tokens && head >= 0 && head < a.ring_size && count >= 0 &&
       count <= a.ring_size && (int64_t)count + total.give <= a.ring_size;
  const bool sound = __syncthreads_and(ok);
  const bool enough = total.take <= (uint32_t)max(count, 0), go = sound && enough;
  Sums base{0, 0, 0};
  for (int b0 = 0; b0 == 0 || b0 < a.n; b0 += kRound) {
    if (a.n > kRound) {
      at = scan(load(b0), all);
      at.add(base);
      base.add(all);
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int b = b0 + tid * EACH + i;
      if (b >= a.n) break;
      if (go) {
        if constexpr (FILL) {
          s_q[b] = (int)at.fresh;
          s_len[b] = r[i].len;
          s_held[b] = r[i].held;
          s_take[b] = (int)at.take;
          s_give[b] = (int)at.give;
          s_from[b] = r[i].from;
        } else {
          a.held[b] = r[i].held;
          a.take_off[b] = (int)at.take;
          a.give_off[b] = (int)at.give;
          a.give_from[b] = r[i].from;
        }
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
  Plan p{s_q, s_len, s_held, s_take, s_give, s_from, head, 0, (int)total.give};
  if (go) p.give_base = ring_place(a, head, count);
  if (tid == 0) {
    a.q_off[a.n] = go ? a.n_tokens : 0;
    if (!go) set_error(a.err, sound ? MISAT_ERR_OOM : MISAT_ERR_INVALID_ARG);
    a.state_out[a.n] = go ? ring_place(a, head, (int)total.take) : head;
    a.state_out[a.n + 1] = go ? count - (int)total.take + (int)total.give : count;
    if constexpr (FILL) {
      s_q[a.n] = a.n_tokens;
      s_give[a.n] = (int)total.give;
    } else {
      a.give_off[a.n] = (int)total.give;
      a.head[kOk] = go;
      a.head[kRingHead] = p.ring_head;
      a.head[kGiveBase] = p.give_base;
      a.head[kGiven] = p.given;
    }
  }
  if constexpr (FILL) {
    __syncthreads();
    for (int t = tid; t < a.n_tokens; t += kPlanThreads) {
      int pos = -1;
      int64_t slot = -1;
      if (go) {
        const int b = search(s_q, a.n, t);
        pos = s_len[b] - s_q[b + 1] + t;
        const Place at = place_of(a, b, pos / kBlockTokens, s_held[b], s_take[b], p.ring_head);
        const int blk = at.from ? __ldcg(at.from) : -1;
        if (at.row && pos % kBlockTokens == 0) *at.row = blk;
        slot = (int64_t)blk * kBlockTokens + pos % kBlockTokens;
      }
      a.positions[t] = pos;
      a.slots[t] = slot;
    }
    if (go)
      for (int j = tid; j < p.given; j += kPlanThreads) {
        const int b = search(s_give, a.n, j);
        give(a, p, b, j, s_from[b], s_give[b]);
      }
  }
}

__global__ void __launch_bounds__(kThreads) k_table_fill(const __grid_constant__ TableArgs a) {
  const int lane = threadIdx.x & 31;
  const int warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kThreads / 32);
  chain_wait();
  const bool go = __ldcg(a.head + kOk) != 0;
  const int64_t n = a.n_tokens;
  if (!go) {
    for (int64_t t = (int64_t)warp * 32 + lane; t < n; t += (int64_t)warps * 32) {
      a.positions[t] = -1;
      a.slots[t] = -1;
    }
    return;
  }
  const Plan p{a.q_off,     a.kv_len_out, a.held, a.take_off, a.give_off, a.give_from, __ldcg(a.head + kRingHead),
               __ldcg(a.head + kGiveBase), __ldcg(a.head + kGiven)};
  for (int64_t t0 = (int64_t)warp * kRun; t0 < n; t0 += (int64_t)warps * kRun) {
    // A lane's first token of each part of the run, then the sequence's numbers, then the blocks: each step's loads are
    // on their way together.
    OffsetFinder find(p.q_off, a.n, (int)t0);
    int b[kAhead], to[kAhead], pos[kAhead], held[kAhead], take[kAhead], blk[kAhead];
    Place at[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      int from;
      b[i] = find((int)min(t0 + (i * 32 + lane) * kEach, n - 1), from, to[i]);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      pos[i] = __ldcg(p.len + b[i]) - to[i] + (int)min(t0 + (i * 32 + lane) * kEach, n - 1);
      held[i] = __ldcg(p.held + b[i]);
      take[i] = __ldcg(p.take_off + b[i]);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      at[i] = place_of(a, b[i], pos[i] / kBlockTokens, held[i], take[i], p.ring_head);
      blk[i] = at[i].from ? __ldcg(at[i].from) : -1;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t first = t0 + (i * 32 + lane) * kEach;
      if (first >= n) continue;
      int32_t x[kEach];
      int64_t y[kEach];
      int s = b[i], q = pos[i], end = to[i], h = held[i], k = take[i], block = blk[i];
      Place place = at[i];
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        x[e] = q;
        y[e] = (int64_t)block * kBlockTokens + q % kBlockTokens;
        if (place.row && q % kBlockTokens == 0) *place.row = block;
        ++q;
        if (e + 1 == kEach || first + e + 1 >= n) continue;
        const bool next = first + e + 1 >= end;
        if (next) {  // the next sequence with tokens
          do {
            ++s;
            end = __ldcg(p.q_off + min(s, a.n - 1) + 1);
          } while (first + e + 1 >= end && s + 1 < a.n);
          s = min(s, a.n - 1);
          q = __ldcg(p.len + s) - end + (int)first + e + 1;
          h = __ldcg(p.held + s);
          k = __ldcg(p.take_off + s);
        }
        if (next || q % kBlockTokens == 0) {
          place = place_of(a, s, q / kBlockTokens, h, k, p.ring_head);
          block = place.from ? __ldcg(place.from) : -1;
        }
      }
      if (a.whole && first + kEach <= n) {
        *reinterpret_cast<int4*>(a.positions + first) = make_int4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<longlong2*>(a.slots + first) = make_longlong2(y[0], y[1]);
        *reinterpret_cast<longlong2*>(a.slots + first + 2) = make_longlong2(y[2], y[3]);
      } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          if (first + e < n) {
            a.positions[first + e] = x[e];
            a.slots[first + e] = y[e];
          }
      }
    }
  }
  for (int64_t j0 = (int64_t)warp * kGiveRun; j0 < p.given; j0 += (int64_t)warps * kGiveRun) {
    OffsetFinder find(p.give_off, a.n, (int)j0);
#pragma unroll 1
    for (int i = 0; i < kGiveRun && j0 + i < p.given; i += 32) {
      const int j = (int)min(j0 + i + lane, (int64_t)p.given - 1);
      int off, end;
      const int b = find(j, off, end);
      if (j0 + i + lane < p.given) give(a, p, b, j, __ldcg(p.give_from + b), off);
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
  a.whole = ((reinterpret_cast<uintptr_t>(s->positions) | reinterpret_cast<uintptr_t>(s->slots)) & 15) == 0;
  // A small step is one CTA's.
  if (s->n <= kPlanThreads && s->n_tokens <= kFillTokens) {
    launch_chained(k_table_plan<1, true>, 1, kPlanThreads, 0, st, a);
    return launch_status();
  }
  if (s->n <= kPlanThreads) launch_chained(k_table_plan<1, false>, 1, kPlanThreads, 0, st, a);
  else launch_chained(k_table_plan<4, false>, 1, kPlanThreads, 0, st, a);
  // Warps for the tokens, and for blocks given back.
  const int64_t warps = std::max<int64_t>((s->n_tokens - 1) / kRun + 1, s->n / 2);
  const int64_t most = (int64_t)kv->num_sms * 8;
  launch_chained(k_table_fill, (int)std::min((warps - 1) / (kThreads / 32) + 1, most), kThreads, 0, st, a);
  return launch_status();
}

}  // extern "C"
