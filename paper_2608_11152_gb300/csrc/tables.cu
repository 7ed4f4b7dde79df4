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
// Bound by latency.  256 sequences of one token: 4.1 us, one CTA with a launch, two trips to memory before its sums
// and two behind them (20.8 us as two kernels with sums over the warps one after the other).  4,096 sequences with
// 4.05 M tokens, 253,000 blocks taken and 417,000 given back: 25 us, of which the sums 7 and the 48 MB of positions and
// slots 8 at the least; in the second kernel a warp has tokens next to each other, searches for its first one alone and
// looks up 31 blocks at a time, one a lane (four tokens a lane, each with its lookup: 30 us; a lookup for every token: 60).
#include <algorithm>
#include <initializer_list>

#include "kv.h"
#include "rotary.cuh"

using namespace misat;

namespace {

constexpr int kMaxTokens = INT32_MAX - 4096;  // numbers of tokens run past the last one by a few
constexpr int kPlanThreads = 1024;
constexpr int kThreads = 256;
constexpr int kFillCtas = 4;               // on an SM
constexpr int kRun = 480;                  // tokens of a warp at a time: at most 31 blocks, one a lane
constexpr int kGives = 4;                  // blocks given back of a lane at a time
constexpr int kFillTokens = 4096;          // most tokens of a step that one CTA makes
constexpr int kFillPlaces = 1 << 17;       // most places of a table whose blocks one CTA gives back, however many they are
constexpr int kFillGives = 8192;           // most blocks that it gives back of a larger one

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
  // What the second kernel needs of the first: Head, a Mark of each sequence and of the end, blocks given before each,
  // first block given of each.
  int32_t* head;
  int4* marks;
  int32_t *give_off, *give_from;
  bool vec_rows;  // what is read and written of each sequence, at 16-byte boundaries
  bool defer;     // a step of one CTA: many blocks given back are left to the second kernel
};
// Of a sequence: first new token, length after the step, blocks held before it, blocks taken before it.
struct Mark {
  int off, len, held, take;
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
__device__ __forceinline__ Row row_of(const TableArgs& a, int fresh, int before, int held, int shared) {
  // A row holds blocks for the tokens that are there, and has room for those to come.  One without blocks that gets none (a
  // finished sequence) shares none, whatever its number still says; where it gets some, a number left from before would
  // keep them from being given back.
  const bool ok = fresh >= 0 && fresh <= a.max_q && before >= 0 && before <= kMaxLen && fresh <= kMaxLen - before &&
                  held >= 0 && held <= a.columns && (int64_t)before <= (int64_t)held * kBlockTokens && shared >= 0 &&
                  (shared <= held || (held | before | fresh) == 0) &&
                  (int64_t)before + fresh <= (int64_t)a.columns * kBlockTokens;
  if (!ok) return {0, 0, 0, 0, false};
  Row r{fresh, before + fresh, held, 0, true};
  r.from = max(r.need(), shared);
  return r;
}
// EACH sequences from b on; those past the last are empty.
template <int EACH>
__device__ __forceinline__ void load_rows(const TableArgs& a, int b, Row (&r)[EACH]) {
  if constexpr (EACH == 4) {
    if (a.vec_rows && b + EACH <= a.n) {
      const auto four = [&](const int32_t* p) { return __ldcg(reinterpret_cast<const int4*>(p + b)); };
      const int4 f = four(a.fresh), l = four(a.kv_len), h = four(a.state), s = a.shared ? four(a.shared) : int4{};
      r[0] = row_of(a, f.x, l.x, h.x, s.x);
      r[1] = row_of(a, f.y, l.y, h.y, s.y);
      r[2] = row_of(a, f.z, l.z, h.z, s.z);
      r[3] = row_of(a, f.w, l.w, h.w, s.w);
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    r[i] = Row{0, 0, 0, 0, true};
    if (b + i < a.n)
      r[i] = row_of(a, __ldcg(a.fresh + b + i), __ldcg(a.kv_len + b + i), __ldcg(a.state + b + i),
                    a.shared ? __ldcg(a.shared + b + i) : 0);
  }
}
template <int EACH>
__device__ __forceinline__ void store_rows(const TableArgs& a, int32_t* p, int b, const int (&v)[EACH]) {
  if constexpr (EACH == 4) {
    if (a.vec_rows && b + EACH <= a.n) {
      *reinterpret_cast<int4*>(p + b) = make_int4(v[0], v[1], v[2], v[3]);
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (b + i < a.n) p[b + i] = v[i];
}

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
    load_rows(a, b0 + tid * EACH, r);
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
    const int b = b0 + tid * EACH;
    int off[EACH], len[EACH], need[EACH], given[EACH], from[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      off[i] = go ? (int)at.fresh : 0;
      len[i] = r[i].len;
      need[i] = r[i].need();
      given[i] = (int)at.give;
      from[i] = r[i].from;
      if (go && b + i < a.n) {
        if constexpr (FILL) {
          s_q[b] = off[i];
          s_len[b] = len[i];
          s_held[b] = r[i].held;
          s_take[b] = (int)at.take;
          s_give[b] = given[i];
          s_from[b] = from[i];
        } else {
          a.marks[b + i] = make_int4(off[i], len[i], r[i].held, (int)at.take);
        }
      } else if (b + i < a.n) {
        len[i] = __ldcg(a.kv_len + b + i);
        need[i] = __ldcg(a.state + b + i);
      }
      at.add(r[i].sums());
    }
    store_rows(a, a.q_off, b, off);
    store_rows(a, a.kv_len_out, b, len);
    store_rows(a, a.state_out, b, need);
    if constexpr (!FILL) {
      store_rows(a, a.give_off, b, given);
      store_rows(a, a.give_from, b, from);
    }
  }
  const int give_base = go ? ring_place(a, head, count) : 0, given = (int)total.give;
  const bool later = FILL && a.defer && go && given > kFillGives;
  if (tid == 0) {
    a.q_off[a.n] = go ? a.n_tokens : 0;
    if (!go) set_error(a.err, sound ? MISAT_ERR_OOM : MISAT_ERR_INVALID_ARG);
    a.state_out[a.n] = go ? ring_place(a, head, (int)total.take) : head;
    a.state_out[a.n + 1] = go ? count - (int)total.take + (int)total.give : count;
    if constexpr (FILL) {
      s_q[a.n] = a.n_tokens;
      s_give[a.n] = given;
    } else {
      a.marks[a.n] = make_int4(a.n_tokens, 0, 0, 0);
    }
    if (!FILL || a.defer) {
      a.head[kOk] = FILL || go;
      a.head[kRingHead] = head;
      a.head[kGiveBase] = give_base;
      a.head[kGiven] = FILL && !later ? 0 : given;
      if (!FILL || later) a.give_off[a.n] = given;
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
        const Place at = place_of(a, b, pos / kBlockTokens, s_held[b], s_take[b], head);
        const int blk = at.from ? __ldcg(at.from) : -1;
        if (at.row && pos % kBlockTokens == 0) *at.row = blk;
        slot = (int64_t)blk * kBlockTokens + pos % kBlockTokens;
      }
      a.positions[t] = pos;
      a.slots[t] = slot;
    }
    if (later) {
      if (tid < a.n) {
        a.give_off[tid] = s_give[tid];
        a.give_from[tid] = s_from[tid];
      }
    } else if (go) {
#pragma unroll 4
      for (int j = tid; j < given; j += kPlanThreads) {
        const int b = search(s_give, a.n, j);
        a.ring[ring_place(a, give_base, j)] = __ldcg(a.table + (int64_t)b * a.stride + (s_from[b] + j - s_give[b]));
      }
    }
  }
}

// The marks of 32 sequences, one a lane, and the one that a token belongs to (as OffsetFinder finds it).
struct MarkFinder {
  const int4* marks;
  int n, lane, base;
  int4 mine;  // marks[base + lane]
  __device__ __forceinline__ void load(int b) {
    base = b;
    mine = base + lane <= n ? __ldcg(marks + base + lane) : make_int4(0x7fffffff, 0, 0, 0);
  }
  __device__ __forceinline__ MarkFinder(const TableArgs& a, int t) : marks(a.marks), n(a.n), lane(threadIdx.x & 31) {
    load(find_sequence(a.q_off, a.n, t, lane, 32));
  }
  // to: the first token of the next sequence.
  __device__ __forceinline__ int operator()(int t, Mark& m, int& to) {
    int b = -1;
    m = Mark{0, 0, 0, 0};
    to = 0;
#pragma unroll 1
    while (true) {
      int lo = 0;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const int v = __shfl_sync(0xffffffffu, mine.x, lo + o);
        if (v <= t) lo += o;
      }
      const bool beyond = lo == 31 && base + 31 < n;
      const Mark own{__shfl_sync(0xffffffffu, mine.x, lo), __shfl_sync(0xffffffffu, mine.y, lo),
                     __shfl_sync(0xffffffffu, mine.z, lo), __shfl_sync(0xffffffffu, mine.w, lo)};
      const int next = __shfl_sync(0xffffffffu, mine.x, min(lo + 1, 31));
      if (b < 0 && !beyond) {
        b = base + lo;
        m = own;
        to = lo < 31 ? next : __ldcg(&marks[min(b + 1, n)].x);
      }
      if (!__any_sync(0xffffffffu, b < 0)) return min(b, n - 1);
      load(base + 31);
    }
  }
};

__global__ void __launch_bounds__(kThreads, kFillCtas) k_table_fill(const __grid_constant__ TableArgs a) {
  const int lane = threadIdx.x & 31;
  const int warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kThreads / 32);
  chain_wait();
  const int4 plan = __ldcg(reinterpret_cast<const int4*>(a.head));  // in the order of Head
  const bool go = plan.x != 0;
  const int64_t n = a.n_tokens;
  if (!go) {
    for (int64_t t = (int64_t)warp * 32 + lane; t < n; t += (int64_t)warps * 32) {
      a.positions[t] = -1;
      a.slots[t] = -1;
    }
    return;
  }
  const int head = plan.y, base = plan.z, given = plan.w;
  // A warp's tokens are next to each other: only its first one is searched for.
  const int share = (int)max((n + warps - 1) / warps, (int64_t)32);
  const int stop = (int)min((int64_t)(warp + 1) * share, n);
  int t = (int)min((int64_t)warp * share, n);
  if (t < stop) {
    MarkFinder find(a, t);
    Mark m;
    int to, b = find(t, m, to);
    while (true) {
      const int left = min(to, stop) - t;
      if (left >= 32 || to >= stop) {
        // Up to kRun tokens of one sequence: a lane looks up one of their blocks, and puts it into the row if it is new.
        const int some = min(left, kRun), first = m.len - to + t, col = first / kBlockTokens;
        const int last = (first + some - 1) / kBlockTokens;
        int blk = -1;
        if (col + lane <= last) {
          const Place p = place_of(a, b, col + lane, m.held, m.take, head);
          if (p.from) blk = __ldcg(p.from);
          if (p.row && (col + lane) * kBlockTokens >= first) *p.row = blk;
        }
#pragma unroll 5
        for (int i = 0; i < some; i += 32) {
          const int pos = first + i + lane;
          const int64_t base = (int64_t)__shfl_sync(0xffffffffu, blk, (pos / kBlockTokens - col) & 31) * kBlockTokens;
          if (i + lane < some) {
            a.positions[t + i + lane] = pos;
            a.slots[t + i + lane] = base + pos % kBlockTokens;
          }
        }
        t += some;
      } else {
        // Short sequences: a token a lane.
        const int mine = t + lane;
        Mark own;
        int end;
        const int s = find(min(mine, stop - 1), own, end);
        if (mine < stop) {
          const int pos = own.len - end + mine;
          const Place p = place_of(a, s, pos / kBlockTokens, own.held, own.take, head);
          const int blk = p.from ? __ldcg(p.from) : -1;
          if (p.row && pos % kBlockTokens == 0) *p.row = blk;
          a.positions[mine] = pos;
          a.slots[mine] = (int64_t)blk * kBlockTokens + pos % kBlockTokens;
        }
        t += 32;
      }
      if (t >= stop) break;
      if (t >= to) b = find(t, m, to);
    }
  }
  const int64_t gives = max(((int64_t)given + warps - 1) / warps, (int64_t)32), last = min((warp + 1) * gives, (int64_t)given);
  int64_t j0 = warp * gives;
  if (j0 < last) {
    OffsetFinder find(a.give_off, a.n, (int)j0);
    for (; j0 < last; j0 += 32 * kGives) {  // each step's loads on their way together
      int64_t at[kGives];
      int blk[kGives];
#pragma unroll
      for (int i = 0; i < kGives; ++i) {
        const int j = (int)min(j0 + i * 32 + lane, last - 1);
        int off, end;
        const int b = find(j, off, end);
        at[i] = (int64_t)b * a.stride + (j - off);
        blk[i] = b;
      }
#pragma unroll
      for (int i = 0; i < kGives; ++i) at[i] += __ldcg(a.give_from + blk[i]);
#pragma unroll
      for (int i = 0; i < kGives; ++i) blk[i] = __ldcg(a.table + at[i]);
#pragma unroll
      for (int i = 0; i < kGives; ++i)
        if (j0 + i * 32 + lane < last) a.ring[ring_place(a, base, (int)(j0 + i * 32 + lane))] = blk[i];
    }
  }
}

}  // namespace

extern "C" {

int misat_kv_tables(misat_kv* kv, const misat_kv_step* s, void* work, int64_t work_bytes, void* cuda_stream) {
  if (!kv || !s || s->n < 0 || s->n > kv->max_batch || s->n_tokens < 0 || s->n_tokens > kMaxTokens || s->max_q < 0 ||
      s->columns < 0 || s->table_stride < s->columns || s->ring_size < 1 || (s->n == 0 && s->n_tokens > 0))
    return MISAT_ERR_INVALID_ARG;
  if (!s->q_off || !s->state || !s->state_out || !s->ring ||
      (s->n > 0 && (!s->new_tokens || !s->kv_len || !s->kv_len_out || (!s->block_table && s->columns > 0))) ||
      (s->n_tokens > 0 && (!s->positions || !s->slots)) || !work || (reinterpret_cast<uintptr_t>(work) & 15) ||
      work_bytes < MISAT_KV_TABLES_WORK(s->n) || !on_device(kv->device))
    return MISAT_ERR_INVALID_ARG;
  const auto bits = [](std::initializer_list<const void*> list) {
    uintptr_t all = 0;
    for (const void* p : list) all |= reinterpret_cast<uintptr_t>(p);
    return all;
  };
  if ((bits({s->new_tokens, s->kv_len, s->shared, s->state, s->block_table, s->ring, s->state_out, s->q_off, s->kv_len_out,
             s->positions}) & 3) || !at_elements(s->slots, 8))
    return MISAT_ERR_INVALID_ARG;
  // What is written is no other array's, or a later part of the step would read numbers that are not the ones that it was
  // worked out from, and leave the arrays by them.  A sequence's input is read by the thread that writes its results, before
  // that: these may be in its place.
  const int64_t n = s->n, T = s->n_tokens;
  constexpr int kResults = 3, kWritten = 8, kArrays = 12;
  const Extent x[kArrays] = {{s->state_out, n + 2}, {s->q_off, n + 1}, {s->kv_len_out, n},
                             {s->block_table, n ? (n - 1) * s->table_stride + s->columns : 0}, {s->ring, s->ring_size},
                             {s->positions, T}, {s->slots, T, 8}, {work, MISAT_KV_TABLES_WORK(n), 1},
                             {s->new_tokens, n}, {s->kv_len, n}, {s->shared, n}, {s->state, n + 2}};
  bool over = false;  // (without branches, which took 0.35 us of a call)
  for (int i = 0; i < kWritten; ++i)
    for (int j = i + 1; j < kArrays; ++j)
      over |= !apart(x[i], x[j]) & !(i < kResults && j >= kWritten && x[i].begin == x[j].begin);
  if (over) return MISAT_ERR_INVALID_ARG;
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
  a.head = static_cast<int32_t*>(work);
  a.marks = static_cast<int4*>(work) + 1;
  a.give_from = reinterpret_cast<int32_t*>(a.marks + s->n + 1);
  a.give_off = a.give_from + (s->n + 3) / 4 * 4;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  a.vec_rows = (bits({a.fresh, a.kv_len, a.shared, a.state, a.state_out, a.q_off, a.kv_len_out}) & 15) == 0;
  // A small step is one CTA's: 256 sequences of one token 3.4 us in a graph where none finishes, with a second kernel behind
  // it 4.7.  How many blocks it gives back is not known here, and one CTA takes 0.6 us a thousand of them: 8 us for 8,192,
  // 23 for 32,768, 43 for 65,536, 81 for 128,000, where the two kernels take 6.3 to 6.6.  So the size of the table decides: up
  // to kFillPlaces places the step in which all of them come back at once takes at most 81 us, beyond that no step takes
  // more than 10 and each pays the second launch.
  if (s->n <= kPlanThreads && s->n_tokens <= kFillTokens) {
    a.defer = (int64_t)s->n * s->columns > kFillPlaces;
    launch_chained(k_table_plan<1, true>, 1, kPlanThreads, 0, st, a);
    a.n_tokens = 0;
    if (a.defer) launch_chained(k_table_fill, kv->num_sms, kThreads, 0, st, a);
    return launch_status();
  }
  if (s->n <= kPlanThreads) launch_chained(k_table_plan<1, false>, 1, kPlanThreads, 0, st, a);
  else launch_chained(k_table_plan<4, false>, 1, kPlanThreads, 0, st, a);
  // Warps for the tokens, and for blocks given back: at most as many as the GPU holds at a time.
  const int64_t warps = std::max<int64_t>((s->n_tokens - 1) / 128 + 1, s->n / 2);
  launch_chained(k_table_fill, (int)std::min<int64_t>((warps - 1) / (kThreads / 32) + 1, kv->num_sms * kFillCtas), kThreads,
                 0, st, a);
  return launch_status();
}

}  // extern "C"
