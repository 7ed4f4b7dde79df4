// What the attention kernel has to do, the run of it that each CTA takes, and the warps that work out its parts
// and load keys, values and queries.
#pragma once

#ifdef __CUDACC__  // (compiled for the host, the includer defines what these do)
#include "kv.h"
#include "tensor.cuh"
#endif

namespace misat {
namespace runs {

constexpr int kKeys = 128;     // keys of a block
constexpr int kPages = kKeys / kBlockTokens;
constexpr int kTile = 128;     // rows of a stream's tile
constexpr int kThreads = 384;
constexpr int kRing = 160 * 1024;  // bytes of the ring of key and value tiles

struct AttendArgs {
  KvBatch b;
  Heads q, out;
  float* lse;
  float scale, c;  // c = scale * log2(e)
  int32_t group, hkv, d, n_blocks, window, tok, rows;  // tok: tokens of a stream's tile; rows: of the fullest tile
  bool small;           // find_run_small's conditions hold
  bool map_q, vec_out, vec32;  // queries through a tensor map; output rows at 16- and 32-byte boundaries
  float4* ws_o;  // [slots][DP / 4][128 rows]
  float2* ws_ml; // [slots][128 rows]: m, l
  unsigned* ctr; // [2 x CTAs] arrivals of split items, zero between calls
  int32_t* err;
  const uint32_t* bits;  // of a tree's nodes, [tokens][words]; nullptr: tokens in a row
  const int32_t* depth;
  int32_t words;
};

// ---- what there is to do ----
//
// Lengths and offsets are read more than once, and a call whose lengths change while it runs still has to stay
// inside the buffers.  Every read is checked by itself (load_seq); what was worked out from an earlier read (the
// place of a run, the items before a sequence, the last CTA of an item) is checked against the later one where it is
// used.  Such a call's run ends early, with an error recorded.

struct Seq {
  int begin, n, len;  // first new token, new tokens, tokens in all
};

__device__ __forceinline__ Seq load_seq(const AttendArgs& a, int b) {
  const int begin = __ldcg(a.b.q_off + b), end = __ldcg(a.b.q_off + b + 1), len = __ldcg(a.b.kv_len + b);
  const bool ok = begin >= 0 && end >= begin && end <= a.b.n_tokens && end - begin <= a.b.max_q && len >= 0 &&
                  len <= kMaxLen && len <= a.b.stride * kBlockTokens;
  if (!ok) set_error(a.err, MISAT_ERR_INVALID_ARG);
  return {begin, ok ? end - begin : 0, len};
}

// Keys of the item of a sequence's tokens [t0, t0 + nt), in blocks.
struct Span {
  int from, to;    // keys [from, to) that some row sees
  int jb, blocks;  // first block, number of blocks (0: no row sees a key)
};
__device__ __forceinline__ Span span_of(const AttendArgs& a, const Seq& s, int t0, int nt) {
  const int p0 = s.len - s.n + t0, to = max(p0 + nt, 0);
  const int first = a.bits ? p0 - t0 : p0;  // the first position: any node of a tree may be a root
  const int from = a.window > 0 && first >= a.window ? first - a.window + 1 : 0;
  const int jb = from / kKeys;
  return {from, to, jb, to > 0 ? (to + kKeys - 1) / kKeys - jb : 0};
}
__device__ __forceinline__ int item_cost(const AttendArgs& a, const Seq& s, int tile) {
  const int t0 = tile * 2 * a.tok;
  return max(span_of(a, s, t0, min(2 * a.tok, s.n - t0)).blocks, 1);
}
__device__ __forceinline__ int n_items(const AttendArgs& a, const Seq& s) {
  return (uint32_t)(s.n + 2 * a.tok - 1) / (uint32_t)(2 * a.tok);
}

// A CTA's part of one item.
struct Segment {
  Seq s;
  Span k;
  int b, h;
  int t0, nt;          // tokens of the item
  int j0, nb;          // first block (of the sequence) and blocks of this part
  bool pair;           // both streams have rows of their own, and read the same keys
  bool twin;           // both streams have an item of their own: the same rows of kv heads h and h + 1
  bool whole;          // the part is the item
  int64_t first, last; // the item's blocks in the order of all blocks
  __device__ __forceinline__ bool both() const { return pair || twin; }  // each stream takes all blocks
  __device__ __forceinline__ int head(int st) const { return h + (twin ? st : 0); }
  __device__ __forceinline__ int stream_blocks(int st) const { return both() ? nb : (nb + 1 - st) / 2; }
  // The products of a part in the order of issue: step x is stream x & 1's next block.  A stream's
  // scores are formed two steps ahead of its product with the values, so the loops over the steps
  // run from -2 to steps() - 1: values of step x, then scores of step x + 2.
  __device__ __forceinline__ int steps() const { return both() ? 2 * nb : nb; }
  __device__ __forceinline__ int block(int step) const { return j0 + (both() ? step / 2 : step); }
};

// x / d.  Counts of blocks fit 31 bits but for the wildest batches; those take 63 steps instead of the
// hundreds of instructions that a 64-bit division is at every place of use.
__device__ __forceinline__ int64_t div_down(int64_t x, int64_t d) {
  if ((x >> 31) == 0 && (d >> 31) == 0) return (uint32_t)x / (uint32_t)d;
  uint64_t q = 0, r = 0;
#pragma unroll 1
  for (int i = 62; i >= 0; --i) {
    r = r << 1 | ((uint64_t)x >> i & 1);
    if (r >= (uint64_t)d) {
      r -= (uint64_t)d;
      q |= (uint64_t)1 << i;
    }
  }
  return (int64_t)q;
}

// The CTAs that have parts of a split item, from the length of a run.
struct Parts {
  int first, last;
};
__device__ __forceinline__ Parts parts_of(const AttendArgs& a, const Segment& g, int64_t per) {
  const int64_t last = div_down(g.last - 1, per);
  if (last >= gridDim.x) set_error(a.err, MISAT_ERR_INVALID_ARG);  // more blocks than were counted
  return {(int)div_down(g.first, per), (int)min(last, (int64_t)gridDim.x - 1)};
}

// The items in the order in which their blocks are dealt out.  Natural: by sequence, kv head, tile.
// In columns (`cols` > 0): item i is in row i / cols and column i % cols of a table with as many rows as
// a CTA has items, and the order is down the columns.  A CTA's run is about one column, so the CTAs work
// on the same row at about the same time: on neighbouring items, which read the same keys, and these
// come from the L2 cache instead of memory.  (Natural order gives a CTA the tiles of one head one after
// the other, each CTA another head: 16 sequences of 1,000 to 30,000 tokens, 2,200 items: 4.0 ms
// against 3.1 ms.)
constexpr int kMaxSeqs = 256;         // sequences in a batch whose items are taken in columns
constexpr int kMaxItems = 1 << 20;

// The run of blocks of one CTA, item by item.
struct Walk {
  int b, h, tile, off;
  int pad;   // what an item counts, where items are not split (0: its blocks)
  int cols;  // columns, 0: natural order
  int item, items;  // in columns: the item's number, all items
  int64_t left, at;
  Seq s;
  // The lengths are not the ones that the run was worked out from.
  __device__ __forceinline__ void stop(const AttendArgs& a) {
    set_error(a.err, MISAT_ERR_INVALID_ARG);
    left = 0;
  }
  // In columns: the sequence, head and tile of the item, from the number of items before each sequence.
  __device__ __forceinline__ void locate(const AttendArgs& a, const int* before) {
    int lo = 0, hi = a.b.n;
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (before[mid] <= item) lo = mid;
      else hi = mid;
    }
    b = lo;
    s = load_seq(a, b);
    const int tiles = n_items(a, s), i = item - before[b];
    h = i / max(tiles, 1);
    tile = i - h * tiles;
    if (tiles == 0 || h >= a.hkv || off >= item_cost(a, s, tile)) stop(a);
  }
  __device__ __forceinline__ bool next(const AttendArgs& a, const int* before, Segment& g) {
    if (left <= 0) return false;
    g.s = s;
    g.b = b;
    g.h = h;
    g.t0 = tile * 2 * a.tok;
    g.nt = min(2 * a.tok, s.n - g.t0);
    g.pair = g.nt > a.tok;
    g.k = span_of(a, s, g.t0, g.nt);
    const int cost = pad ? pad : max(g.k.blocks, 1);
    const int take = (int)min(left, (int64_t)(cost - off));
    g.j0 = g.k.jb + off;
    g.nb = pad || g.k.blocks == 0 ? g.k.blocks : take;
    g.whole = take == cost;
    g.first = at - off;
    g.last = g.first + cost;
    at += take;
    left -= take;
    off = 0;
    // Two heads of an item at a time, where the run has both whole: they have equally many blocks, and
    // neither waits for the other (single tokens of 256 sequences, 8 kv heads of 128, 10 to 100 cached tokens: 73.5
    // us one by one, 38.6 in twos; 63 to 511 tokens: 108 and 77; 512 to 16,000 tokens: 1,285 and 1,275).
    g.twin = !g.pair && g.whole && pad == 0 && cols == 0 && g.nt == s.n && h + 1 < a.hkv && left >= cost;
    if (g.twin) {
      at += cost;
      left -= cost;
      ++h;
    }
    if (left <= 0) return true;
    if (cols > 0) {
      const int next_row = item + cols, next_col = item % cols + 1;
      item = next_row < items ? next_row : next_col;
      if (next_row >= items && next_col == cols) stop(a);
      else locate(a, before);
    } else if (++tile * 2 * a.tok >= s.n) {
      tile = 0;
      if (++h == a.hkv) {
        h = 0;
        do {
          if (b + 1 >= a.b.n) {  // fewer blocks than were counted
            stop(a);
            break;
          }
          s = load_seq(a, ++b);
        } while (s.n == 0);
      }
    }
    return true;
  }
};

// Blocks, items and longest item of a sequence and one kv head, or of several.
struct Cost {
  int64_t blocks;
  int items, longest;
  __device__ __forceinline__ void add(const Cost& r) {
    blocks += r.blocks;
    items += r.items;
    longest = max(longest, r.longest);
  }
};

// ---- shared memory ----

constexpr int kSegs = 4;

template <int DP>
struct Layout {
  static constexpr int kHalf = kKeys * 128;                 // 128 rows of 64 elements
  static constexpr int kStage = kHalf * (DP / 64);          // a tile of keys, values or queries
  static constexpr int kStages = kRing / kStage;
  static constexpr int kQ = 0;                              // two tiles of queries
  static constexpr int kKv = 2 * kStage;
  static constexpr int kCtl = kKv + kStages * kStage;
};

struct Control {
  Segment seg[kSegs];  // the run, a few items ahead
  uint64_t seg_full[kSegs], seg_empty[kSegs];
  uint64_t kv_full[10], kv_empty[10];
  uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_full[2];
  uint64_t ml_full, ml_free, wg[2], drain;
  uint64_t s_free[2], pv_done[2];  // where weights and scores are apart
  float2 ml[kTile];  // m and l of stream 1 for the join
  int before[kMaxSeqs];  // items before each sequence, where they are taken in columns
  Cost sum[kThreads / 32];
  Walk start;
  int64_t per;  // length of a run
  int last[2];
  int abort;
  uint32_t tmem;
};
template <int DP>
constexpr int smem_bytes() { return Layout<DP>::kCtl + (int)sizeof(Control); }
static_assert(smem_bytes<128>() <= 227 * 1024, "shared memory of a CTA");
static_assert(Layout<64>::kStages <= 10 && Layout<128>::kStages <= 10, "ring barriers");

// A counter through a ring or a pair of phases.
struct Ring {
  int at = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step(int n) {
    if (++at == n) {
      at = 0;
      phase ^= 1;
    }
  }
};

// ---- the parts of a run, from the warp that works them out to the others ----
constexpr int kItemLimit = 64;  // limit of waits that last as long as an item: 2^30 keys take some 15 seconds
constexpr int kReaders = 11;  // 8 softmax warps, keys and values, matrix instructions, queries
struct Feed {
  Control* c;
  Ring ring;
  // The next part, or nullptr: the end, or gave up.  (It may wait for a reader that is an item behind.)
  __device__ __forceinline__ const Segment* next() {
    if (!mbar_wait(smem_u32(&c->seg_full[ring.at]), ring.phase, &c->abort, kItemLimit)) return nullptr;
    const Segment* g = &c->seg[ring.at];
    return g->nb < 0 ? nullptr : g;
  }
  __device__ __forceinline__ void done() {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&c->seg_empty[ring.at]));
    ring.step(kSegs);
  }
};
__device__ __forceinline__ void feed(const AttendArgs& a, Control* c, Walk w) {
  Ring ring;
  const bool lead = (threadIdx.x & 31) == 0;
  for (bool more = true; more; ring.step(kSegs)) {
    Segment g;
    more = w.next(a, c->before, g);
    if (!more) g.nb = -1;
    if (!mbar_wait(smem_u32(&c->seg_empty[ring.at]), ring.phase ^ 1, &c->abort, kItemLimit)) return;
    if (lead) {
      c->seg[ring.at] = g;
      mbar_arrive(smem_u32(&c->seg_full[ring.at]));
    }
    __syncwarp();
  }
}

// ---- the run of each CTA ----
__device__ __forceinline__ Cost cost_of(const AttendArgs& a, const Seq& s) {
  Cost r{0, n_items(a, s), 0};
#pragma unroll 1
  for (int t = 0; t < r.items; ++t) {
    const int k = item_cost(a, s, t);
    r.blocks += k;
    r.longest = max(r.longest, k);
  }
  return r;
}
__device__ __forceinline__ void warp_sum(Cost& r) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.blocks += __shfl_xor_sync(0xffffffffu, r.blocks, o);
  r.items = __reduce_add_sync(0xffffffffu, r.items);
  r.longest = __reduce_max_sync(0xffffffffu, r.longest);
}
__device__ __forceinline__ int64_t warp_scan(int64_t v) {  // sum over this lane and those before it
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t t = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += t;
  }
  return v;
}

// How the blocks are dealt out, from their sum over the batch.
//
// With at most one item per CTA, an item is split only where that saves more than kSplit blocks of the
// longest one: writing, announcing and joining the parts takes about as long as kSplit blocks
// (4 sequences of 17 to 640 tokens, 8 kv heads: 14.8 us split evenly, 14.1 us whole).  Whole items then count
// as equally long.
//
// A part has two blocks at least, which the streams take at the same time, and no fewer than make the
// parts' time and the time to join them even: n blocks in p parts take n / p block times, and the join
// p / kJoin block times for up to 8 rows, in proportion more for more of them (2 sequences of 6,400 tokens
// with 280 new ones, 2 heads of 128: 63 us with kJoin = 112, 51 with 28, 46 with 14 and 7, 59 with 1.75;
// one of 30,000 tokens with 64 new ones, 8 heads: 101, 73, 68, 73 and 98).
constexpr int kSplit = 8;
constexpr float kJoin = 14.f;
__device__ __forceinline__ int least_part(const AttendArgs& a, int longest) {
  return (int)max(2.f, sqrtf((float)longest * (float)max(a.rows, 8) / (8.f * kJoin)));
}
struct Deal {
  int64_t total, items, per;
  int longest;
  bool whole;
  __device__ __forceinline__ Deal(const AttendArgs& a, const Cost& sum)
      : total(sum.blocks * a.hkv), items((int64_t)sum.items * a.hkv), longest(sum.longest) {
    per = div_down(total + gridDim.x - 1, gridDim.x);
    whole = items <= gridDim.x && longest <= per + kSplit;
    if (whole) {
      per = longest;
      total = items * longest;
    } else {
      per = max(per, (int64_t)least_part(a, longest));
    }
  }
  __device__ __forceinline__ int64_t lo() const { return per * blockIdx.x; }
};

// The place of block `lo` in sequence b, whose blocks are [before, before + v).
__device__ __forceinline__ Walk place(const AttendArgs& a, const Deal& d, int b, const Seq& s, int64_t before,
                                      int64_t v) {
  const int64_t head = div_down(v, a.hkv), h = div_down(d.lo() - before, head);
  int64_t rest = d.lo() - before - h * head;
  int t = 0;
  if (d.whole) {
    t = (int)div_down(rest, d.longest);
    rest = 0;
  } else {
#pragma unroll 1
    for (int cost; rest >= (cost = item_cost(a, s, t)); ++t) rest -= cost;
  }
  return {b, (int)h, t, (int)rest, d.whole ? d.longest : 0, 0, 0, 0, min(d.per, d.total - d.lo()), d.lo(), s};
}

// Where this CTA's run begins and how long it is, for at most 32 sequences with at most one item per CTA:
// by one warp, a lane per sequence, while the others set out.  The deal is Deal's, in 32 bits: fewer items
// than CTAs, of at most 2^23 blocks.
__device__ __forceinline__ bool find_run_small(const AttendArgs& a, Control* c, Walk& w) {
  const int lane = threadIdx.x & 31;
  const Seq s = lane < a.b.n ? load_seq(a, lane) : Seq{0, 0, 0};
  const Cost mine = cost_of(a, s);
  const int own = (int)mine.blocks;
  const int total = __reduce_add_sync(0xffffffffu, own) * a.hkv;
  const int items = __reduce_add_sync(0xffffffffu, mine.items) * a.hkv;
  const int longest = __reduce_max_sync(0xffffffffu, mine.longest), grid = (int)gridDim.x;
  int per = (uint32_t)(total + grid - 1) / (uint32_t)grid;
  const bool whole = longest <= per + kSplit;
  if (!whole) per = max(per, least_part(a, longest));
  // Counted in items where they stay whole, else in blocks.
  const int head = whole ? mine.items : own, v = head * a.hkv;
  const int lo = whole ? (int)blockIdx.x : per * (int)blockIdx.x;
  if (lo >= (whole ? items : total)) return false;
  int before = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += t;
  }
  before -= v;
  const bool mine_begins = before <= lo && lo < before + v;
  if (!__any_sync(0xffffffffu, mine_begins)) {  // (offsets that overlap: sums beyond 32 bits)
    set_error(a.err, MISAT_ERR_INVALID_ARG);
    return false;
  }
  if (mine_begins) {
    const int h = (uint32_t)(lo - before) / (uint32_t)head;
    int rest = lo - before - h * head, t = 0;
    if (whole) {
      t = rest;
      rest = 0;
    } else {
#pragma unroll 1
      for (int cost; rest >= (cost = item_cost(a, s, t)); ++t) rest -= cost;
    }
    c->start = Walk{lane, h, t, rest, whole ? longest : 0, 0, 0, 0, whole ? longest : min(per, total - lo),
                    whole ? (int64_t)longest * lo : lo, s};
    c->per = whole ? longest : per;
  }
  __syncwarp();
  w = c->start;
  return true;
}

// The same by all threads, for any batch.
__device__ __forceinline__ bool find_run(const AttendArgs& a, Control* c, Seq* seqs, Walk& w) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kWarps = kThreads / 32;
  const Seq mine = tid < a.b.n ? load_seq(a, tid) : Seq{0, 0, 0};
  const Cost first = cost_of(a, mine);
  Cost sum = first;
#pragma unroll 1
  for (int b = tid + kThreads; b < a.b.n; b += kThreads) sum.add(cost_of(a, load_seq(a, b)));
  warp_sum(sum);
  if (lane == 0) c->sum[warp] = sum;
  __syncthreads();
  sum = Cost{0, 0, 0};
#pragma unroll
  for (int i = 0; i < kWarps; ++i) sum.add(c->sum[i]);
  const Deal d(a, sum);
  const int64_t lo = d.lo();
  if (lo >= d.total) return false;
  auto scan = [&](int64_t v, int64_t& all) {  // sum over the threads before this one, and over all
    const int64_t inc = warp_scan(v);
    __syncthreads();
    if (lane == 31) c->sum[warp].blocks = inc;
    __syncthreads();
    int64_t before = inc - v;
    all = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) before += c->sum[i].blocks;
      all += c->sum[i].blocks;
    }
    return before;
  };
  int64_t all;
  const int rows = (int)div_down(d.items + gridDim.x - 1, gridDim.x);
  if (rows > 1 && a.b.max_q > 2 * a.tok && a.b.n <= kMaxSeqs && d.items <= kMaxItems) {
    // Items before each sequence, the cost of each column, and the place in the column.
    const int64_t mine_before = scan((int64_t)first.items * a.hkv, all);
    if (tid < a.b.n) {
      c->before[tid] = (int)mine_before;
      seqs[tid] = mine;
    }
    __syncthreads();
    const int items = (int)d.items, cols = (items + rows - 1) / rows;
    auto cost_at = [&](int item) {
      int x = 0, y = a.b.n;
#pragma unroll 1
      while (y - x > 1) {
        const int mid = (x + y) / 2;
        if (c->before[mid] <= item) x = mid;
        else y = mid;
      }
      const Seq s = seqs[x];
      return item_cost(a, s, (item - c->before[x]) % n_items(a, s));
    };
    int64_t v = 0;
    if (tid < cols)
#pragma unroll 1
      for (int i = tid; i < items; i += cols) v += cost_at(i);
    const int64_t before = scan(v, all);
    if (before <= lo && lo < before + v) {
      int64_t rest = lo - before;
      int i = tid;
#pragma unroll 1
      for (int cost; rest >= (cost = cost_at(i)); i += cols) rest -= cost;
      c->start = Walk{0, 0, 0, (int)rest, 0, cols, i, items, min(d.per, d.total - lo), lo, {0, 0, 0}};
      c->per = d.per;
    }
    fence_async_shared();  // `seqs` lies where keys are going to land
    __syncthreads();
    w = c->start;
    w.locate(a, c->before);
    return true;
  }
  if (tid == 0) c->start.left = 0;
  int64_t base = 0;
#pragma unroll 1
  for (int b0 = 0; base <= lo && b0 < a.b.n; b0 += kThreads) {
    const Seq s = b0 == 0 ? mine : b0 + tid < a.b.n ? load_seq(a, b0 + tid) : Seq{0, 0, 0};
    const int64_t v =
        (d.whole ? (int64_t)n_items(a, s) * d.longest : b0 == 0 ? first.blocks : cost_of(a, s).blocks) * a.hkv;
    const int64_t before = base + scan(v, all);
    base += all;
    if (before <= lo && lo < before + v) {
      c->start = place(a, d, b0 + tid, s, before, v);
      c->per = d.per;
    }
  }
  __syncthreads();
  w = c->start;
  if (w.left == 0 && tid == 0) set_error(a.err, MISAT_ERR_INVALID_ARG);  // fewer blocks than were counted
  return w.left > 0;
}

// ---- keys and values ----
template <int DP>
struct Loader {
  using L = Layout<DP>;
  const AttendArgs& a;
  const CUtensorMap* map_k;
  const CUtensorMap* map_v;
  Control* c;
  uint32_t kv;
  Ring ring;

  // Pages [lo, hi) of key block j hold keys that some row of the item sees; a lane has one box of one page.
  static __device__ __forceinline__ int lo_page(const Segment& g, int j) {
    return max(g.k.from / kBlockTokens - j * kPages, 0);
  }
  static __device__ __forceinline__ int hi_page(const Segment& g, int j) {
    return min((g.k.to + kBlockTokens - 1) / kBlockTokens - j * kPages, kPages);
  }
  // The table's entry for this lane's page; read a block ahead of its use, and checked there.
  __device__ __forceinline__ int page(const Segment& g, int j) const {
    const int i = (threadIdx.x & 31) / (DP / 64);
    return i >= lo_page(g, j) && i < hi_page(g, j)
               ? __ldcg(a.b.table + (int64_t)g.b * a.b.stride + j * kPages + i)
               : 0;
  }
  __device__ __forceinline__ bool load(const Segment& g, const CUtensorMap* map, int head, int j, int blk) {
    const int lane = threadIdx.x & 31, lo = lo_page(g, j), hi = hi_page(g, j);
    const uint32_t full = smem_u32(&c->kv_full[ring.at]);
    if (!mbar_wait(smem_u32(&c->kv_empty[ring.at]), ring.phase ^ 1, &c->abort)) return false;
    if (lane == 0) mbar_expect(full, (hi - lo) * (DP / 64) * kBlockTokens * 128);
    __syncwarp();
    const int i = lane / (DP / 64), half = lane % (DP / 64);
    if (i >= lo && i < hi) {
      int row = blk * a.hkv + head;
      if (blk < 0 || blk >= a.n_blocks) {
        set_error(a.err, MISAT_ERR_INVALID_ARG);
        row = a.n_blocks * a.hkv;  // past the tensor: the box is filled with zeros
      }
      tma_load_3d(kv + ring.at * L::kStage + half * L::kHalf + i * kBlockTokens * 128, map, full, half * 64, 0, row);
    }
    ring.step(L::kStages);
    return true;
  }
  __device__ __forceinline__ void run() {
    Feed feed{c};
    for (; const Segment* p = feed.next(); feed.done()) {
      const Segment g = *p;
      if (g.nb == 0) continue;
      // Keys are loaded two steps ahead of values; a pair's two steps use one tile.  Table entries of the steps
      // between, and of one more.
      const int n = g.pair ? g.nb : g.steps(), lead = g.pair ? 1 : 2;
      auto block = [&](int x) { return g.j0 + (g.twin ? x / 2 : x); };
      int now = 0, next = 0, ahead = page(g, g.j0);
#pragma unroll 1
      for (int x = -lead; x < n; ++x) {
        const int y = x + lead, head = g.head(x & 1);  // x and x + 2: the same stream
        const int fetched = y + 1 < n ? page(g, block(y + 1)) : 0;
        if (x >= 0 && !load(g, map_v, head, block(x), now)) return;
        if (y < n && !load(g, map_k, head, block(y), ahead)) return;
        now = g.pair ? ahead : next;
        next = ahead;
        ahead = fetched;
      }
    }
  }
  // After a wait that ran out: the copies still in flight are waited for, again for a bounded time.
  __device__ __forceinline__ void drain() {
    int go_on = 0;
    for (int i = 0; i < L::kStages; ++i)
      mbar_wait(smem_u32(&c->kv_full[i]), i < ring.at ? ring.phase : ring.phase ^ 1, &go_on);
  }
};

// ---- queries ----
// Which of the two query tiles a stream of a segment uses: both streams of a pair their own, else
// the one tile that was not used last, so that the next item's queries load early.
struct QuerySlots {
  uint32_t phases = 0;  // bit per tile (phases that are chosen at run time are bits: an array would be memory)
  int turn = 0;
  __device__ __forceinline__ int slot(const Segment& g, int st) const { return g.both() ? st : turn; }
  __device__ __forceinline__ uint32_t phase(int slot) const { return phases >> slot & 1; }
  __device__ __forceinline__ void step(const Segment& g) {
    phases ^= g.both() ? 3 : 1 << turn;
    turn ^= !g.both();
  }
};

template <int DP>
struct QueryLoader {
  using L = Layout<DP>;
  const AttendArgs& a;
  const CUtensorMap* map;
  char* smem;
  Control* c;
  uint32_t issued = 0;  // bit per tile: the parity of the copies issued to it

  __device__ __forceinline__ void run() {
    const int lane = threadIdx.x & 31;
    QuerySlots qs;
    Feed feed{c};
    for (; const Segment* g = feed.next(); feed.done()) {
      if (g->nb == 0) continue;
      for (int st = 0; st < (g->both() ? 2 : 1); ++st) {
        const int slot = qs.slot(*g, st);
        const uint32_t full = smem_u32(&c->q_full[slot]);
        if (!mbar_wait(smem_u32(&c->q_empty[slot]), qs.phase(slot) ^ 1, &c->abort, kItemLimit)) return;
        const int first = g->pair ? st * a.tok : 0;  // token of the item
        const int token = g->s.begin + g->t0 + first, head = g->head(st) * a.group;
        char* dst = smem + L::kQ + slot * L::kStage;
        issued ^= 1u << slot;
        // Row r of a tile is token r / group and head r % group: the order of a box of heads and tokens.
        if (a.map_q) {
          if (elect_one()) {
            mbar_expect(full, DP * 2 * a.group * a.tok);
            for (int x = 0; x < DP; x += 64)
              tma_load_3d(smem_u32(dst) + x / 64 * L::kHalf, map, full, x, head, token);
          }
          continue;
        }
        // Rows that no map can describe: an element at a time; elements past d are zeros.
        const int rows = min(a.tok, g->nt - first) * a.group;
        for (int i = lane; i < rows * DP; i += 32) {
          const int r = i / DP, e = i % DP, t = r / a.group;
          const uint16_t* q = static_cast<const uint16_t*>(a.q.p) + (int64_t)(token + t) * a.q.ts +
                              (int64_t)(head + r - t * a.group) * a.q.hs;
          *reinterpret_cast<uint16_t*>(dst + e / 64 * L::kHalf + r * 128 + ((e / 8 & 7) ^ (r & 7)) * 16 + e % 8 * 2) =
              e < a.d ? q[e] : 0;
        }
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(full);
      }
      qs.step(*g);
    }
  }
  // After a wait that ran out: the copies still in flight land before the CTA's shared memory is given back; they are
  // waited for, again for a bounded time.
  __device__ __forceinline__ void drain() {
    int go_on = 0;
    for (int i = 0; i < 2; ++i) mbar_wait(smem_u32(&c->q_full[i]), (issued >> i & 1) ^ 1, &go_on);
  }
};

}  // namespace runs
}  // namespace misat
