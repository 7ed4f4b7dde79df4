// Attention of new tokens over a paged cache (one token, or a chunk), on the tensor cores.
//
//   out_r = sum_j p_rj v_j / l_r,  p_rj = 2^(c (s_rj - m_r)),  s = q k^T,  c = scale log2 e,  l_r = sum_j p_rj
//
// One pass over the keys.  A tile is 128 rows: 128 / group tokens times the `group` query heads that
// share a kv head, so the keys and values are read once for all of them.  Per 128 keys the matrix
// instructions form S = Q K^T in tensor memory, a thread per row reads its 128 scores, takes them to
// weights and writes these back as the 16-bit operand of O += P V, which stays in tensor memory.
// The running maximum m is a reference, not the maximum: O and l are rescaled only when a score
// passes it by more than a bound (Weights), and the sums are in 32 bits.
// Scores, m, l and O are 32 bits throughout.  The weights are rounded once, to the 16 bits of the values that they
// multiply (the matrix instruction takes one type); l adds them unrounded.  The result is rounded once.
//
// What bounds it, and what it does: a step of single tokens reads the cache once, at 7.0 TB/s (256 sequences
// of 512 to 16,000 tokens, 8 kv heads of 128: 1.19 to 1.23 ms for 8.4 GB); a chunk is the products and the
// chain of scores, exponentials and product of each stream, at 1,260 to 1,440 TFLOP/s of 1,887 (2,048 tokens
// over 129,024, 32 heads: 3.03 to 3.45 ms on different GPUs, power-capped at some 1.55 GHz).
//
// Two streams of such tiles share a CTA, so that one's matrix products run under the other's
// exponentials.  An item of more than 128 rows gives each stream half of its rows, and both read the same
// keys; a smaller item (a step of single tokens) gives each stream every other block of 128 keys, and
// the first stream joins the two at the end; and two such items of neighbouring heads are taken together,
// a stream each.
//
// One CTA per SM.  The blocks of all items, in order, are dealt out in equal contiguous runs, so
// long and short sequences, and the triangle of a chunk, load every SM alike.  An item that
// crosses runs leaves partial sums (O, m, l in 32 bits) in the workspace; the last CTA to arrive
// adds them, always in the order of the keys, so the result has the same bits on every call.
//
// Warps: 0-3 and 4-7 softmax of stream 0 and 1; 8 loads queries; 9 issues the matrix instructions; 10 loads
// keys and values (a page of 16 tokens is one or two boxes, 2 KB each); 11 works out the parts.  Warps
// 0, 4 and 8 share a scheduler, and a step of single tokens has rows for warps 0 and 4 alone: with the keys
// loaded by warp 8 beside them, 256 sequences took 1,274 us instead of 1,209.
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "kv.h"
#include "tensor.cuh"

using namespace misat;

namespace {

constexpr int kKeys = 128;     // keys of a block
constexpr int kPages = kKeys / kBlockTokens;
constexpr int kTile = 128;     // rows of a stream's tile
constexpr int kThreads = 384;
constexpr int kRing = 160 * 1024;  // bytes of the ring of key and value tiles
constexpr int kRegsIssue = 88, kRegsSoftmax = 208;  // 128 * 88 + 256 * 208 = 384 * 168 registers

// The weights in 16 bits are 2^(kFactor + c (s - m)): O and l carry the factor 2^kFactor, which the result does not
// see and the log-sum-exp takes off; O and l are rescaled when a score passes m by more than 2^kRescale.
// bfloat16 has the exponents of 32 bits and needs no factor.  float16 holds 2^-14 to 2^16 in full precision and
// rounds to zero below 2^-25: with 65,000 as the largest weight, one that is 2^-25 of its row's reference keeps its
// 11 bits, and zero is what is below 2^-36 of it.  (With 2^8 as the largest weight and no factor, 131,072 keys 18
// below one that takes most of the weight added up to 1.4% too little.)  The narrower range means more rescales: 97
// prompts of 512 to 2,048 tokens under a window, scores of standard deviation 1, take 954 us, 940 with a factor of
// 2^10, 934 with 2^9, 930 with 2^8; one token over 131,072, 91 us with each.
template <class T>
struct Weights {
  static constexpr float kRescale = 8.f, kFactor = 0.f, kOff = 1.f;
};
template <>
struct Weights<__half> {
  static constexpr float kRescale = 4.99f, kFactor = 11.f, kOff = 0x1p-11f;
};

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
};

// ---- what there is to do ----

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
  const int from = a.window > 0 && p0 >= a.window ? p0 - a.window + 1 : 0;
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
    const int tiles = n_items(a, s);
    h = (item - before[b]) / tiles;
    tile = item - before[b] - h * tiles;
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
      item = item + cols < items ? item + cols : item % cols + 1;
      locate(a, before);
    } else if (++tile * 2 * a.tok >= s.n) {
      tile = 0;
      if (++h == a.hkv) {
        h = 0;
        do {
          if (b + 1 >= a.b.n) {  // fewer blocks than were counted: the lengths changed under the call
            left = 0;
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
  if (before <= lo && lo < before + v) {
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
  return true;
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

template <class T, int DP>
__device__ __forceinline__ void load_queries(const AttendArgs& a, const CUtensorMap* map, char* smem, Control* c) {
  using L = Layout<DP>;
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

// ---- matrix instructions ----
// Tensor memory: S of stream 0 and 1 (128 columns each; the weights replace the scores in the first
// 64), O of stream 0 and 1 (DP columns each).  Instructions of one thread execute in order, so S of
// the next block may be issued right behind the product that reads the weights in its place.
__device__ __forceinline__ uint32_t col_s(int st) { return st * 128; }
template <int DP>
__device__ __forceinline__ uint32_t col_o(int st) { return 256 + st * DP; }

template <class T, int DP>
struct Issuer {
  using L = Layout<DP>;
  static constexpr bool kBf16 = std::is_same_v<T, __nv_bfloat16>;
  const AttendArgs& a;
  Control* c;
  char* smem;
  uint32_t base, ctl, tmem;
  Ring ring;
  int k_stage = 0, v_stage = 0;
  uint32_t p_phases = 0;  // bit per stream

  // Address of a barrier of the control block.
  __device__ __forceinline__ uint32_t bar(size_t offset, int i = 0) const { return ctl + (uint32_t)offset + i * 8; }
#define MISAT_BAR(name, ...) bar(offsetof(Control, name), ##__VA_ARGS__)

  __device__ __forceinline__ void scores(int st, int slot, int stage) const {
    const uint32_t q = desc_lo(base + L::kQ + slot * L::kStage, 16), k = desc_lo(base + L::kKv + stage * L::kStage, 16);
    const uint32_t d = tmem + col_s(st);
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      const uint32_t at = ((i / 4) * L::kHalf + (i % 4) * 32) / 16;
      mma_ss(d, q + at, k + at, desc_hi(1024), mma_desc(kBf16, 128, kKeys, false), i > 0);
    }
  }
  // O of the stream (+)= weights times values, over the pages of the block that hold visible keys.
  __device__ __forceinline__ void product(const Segment& g, int st, int stage, int j, bool fresh) const {
    const uint32_t v = desc_lo(base + L::kKv + stage * L::kStage, L::kHalf);
    const uint32_t d = tmem + col_o<DP>(st), p = tmem + col_s(st);
    constexpr uint32_t id = mma_desc(kBf16, 128, DP, true);
    if (j * kKeys >= g.k.from && (j + 1) * kKeys <= g.k.to) {
#pragma unroll
      for (int i = 0; i < kPages; ++i)
        mma_ts(d, p + i * 8, v + i * kBlockTokens * 128 / 16, desc_hi(1024), id, !fresh || i > 0);
    } else {
      const int lo = Loader<DP>::lo_page(g, j), hi = Loader<DP>::hi_page(g, j);
#pragma unroll 1
      for (int i = lo; i < hi; ++i)
        mma_ts(d, p + i * 8, v + i * kBlockTokens * 128 / 16, desc_hi(1024), id, !fresh || i > lo);
    }
  }
  // Keys of block j that no row of the item sees but that share a page with one that is seen: their
  // values may be anything (a sequence's last page is filled to its length only), and are cleared.
  __device__ __forceinline__ bool ragged(const Segment& g, int j) const {
    return ((g.k.from > j * kKeys && g.k.from % kBlockTokens) ||
            (g.k.to < (j + 1) * kKeys && g.k.to % kBlockTokens));
  }
  __device__ __forceinline__ void clear(const Segment& g, int stage, int j) {
    const int lane = threadIdx.x & 31, from = g.k.from - j * kKeys, to = g.k.to - j * kKeys;
    char* v = smem + L::kKv + stage * L::kStage;
    auto zero = [&](int r0, int r1) {
      for (int i = r0 * (DP / 8) + lane; i < r1 * (DP / 8); i += 32) {
        const int row = i / (DP / 8), ch = i % (DP / 8);
        *reinterpret_cast<uint4*>(v + (ch / 8) * L::kHalf + row * 128 + (ch & 7) * 16) = make_uint4(0, 0, 0, 0);
      }
    };
    if (from > 0) zero(from / kBlockTokens * kBlockTokens, from);
    if (to < kKeys) zero(to, (to + kBlockTokens - 1) / kBlockTokens * kBlockTokens);
    fence_async_shared();
    __syncwarp();
  }
  // Step x, by one thread.  The ring's next tile is the values of step x, then the keys of step x + 2;
  // in a pair the second stream uses the first one's.
  __device__ __forceinline__ bool step(const Segment& g, int x, int n, int slot0, int slot1) {
    const int st = x & 1, slot = st ? slot1 : slot0;
    const bool has_v = x >= 0, has_k = x + 2 < n;
    const bool first_use = !g.pair || st == 0, last_use = !g.pair || st == 1;
    if (has_v) {
      if (first_use) {
        v_stage = ring.at;
        if (!mbar_wait_one(MISAT_BAR(kv_full, v_stage), ring.phase, &c->abort)) return false;
        ring.step(L::kStages);
      }
      if (!mbar_wait_one(MISAT_BAR(p_full, st), p_phases >> st & 1, &c->abort)) return false;
      p_phases ^= 1 << st;
      tc_fence_after();
      product(g, st, v_stage, g.block(x), x < 2);
      if (last_use) mma_commit(MISAT_BAR(kv_empty, v_stage));
      if (!has_k) mma_commit(MISAT_BAR(o_full, st));
    }
    if (has_k) {
      if (first_use) {
        k_stage = ring.at;
        if (!mbar_wait_one(MISAT_BAR(kv_full, k_stage), ring.phase, &c->abort)) return false;
        ring.step(L::kStages);
      }
      scores(st, slot, k_stage);
      mma_commit(MISAT_BAR(s_full, st));
      if (last_use) mma_commit(MISAT_BAR(kv_empty, k_stage));
      if (x + 3 == n) {  // the last scores: the queries have been read
        mma_commit(MISAT_BAR(q_empty, slot0));
        if (g.both()) mma_commit(MISAT_BAR(q_empty, 1));
      }
    }
    return true;
  }
  __device__ __forceinline__ void run() {
    QuerySlots qs;
    Feed feed{c};
    for (; const Segment* p = feed.next(); feed.done()) {
      const Segment g = *p;
      const int n = g.steps();
      if (n == 0) continue;
      for (int st = 0; st < (g.both() ? 2 : 1); ++st) {
        const int slot = qs.slot(g, st);
        if (!mbar_wait(smem_u32(&c->q_full[slot]), qs.phase(slot), &c->abort)) return;
      }
      tc_fence_after();
      // Steps in runs: one thread waits and issues without a vote or an election in between, which left the
      // tensor cores idle; the warp meets where values have to be cleared, at the ends of the item's keys.
      const int slot0 = qs.slot(g, 0), slot1 = qs.slot(g, 1), by = g.pair ? 2 : 1;
      const int tail = ragged(g, g.j0 + g.nb - 1) ? n - (g.both() ? 2 : 1) : n;
#pragma unroll 1
      for (int x = -2; x < n;) {
        int end = x < 0 ? 0 : x < tail ? tail : n;
        if (x >= 0 && ragged(g, g.block(x))) {
          end = x + by;
          if (!mbar_wait(MISAT_BAR(kv_full, ring.at), ring.phase, &c->abort)) return;
          clear(g, ring.at, g.block(x));
        }
        int state = 0;
        uint32_t lead;
        if (elect_one(lead)) {
          bool ok = true;
#pragma unroll 1
          for (int y = x; y < min(end, n) && ok; ++y)
            ok = step(g, y, n, slot0, slot1);
          state = ring.at | (int)ring.phase << 8 | (int)p_phases << 9 | (int)ok << 11;
        }
        state = __shfl_sync(0xffffffffu, state, lead);
        ring.at = state & 0xff;
        ring.phase = state >> 8 & 1;
        p_phases = state >> 9 & 3;
        if (!(state >> 11 & 1)) return;
        x = end;
      }
      qs.step(g);
    }
  }
  // The instructions issued and their arrivals are waited for (for a bounded time) before tensor memory is
  // freed and the CTA's shared memory with it.
  __device__ __forceinline__ void drain() {
    int go_on = 0;
    if (elect_one()) mma_commit(smem_u32(&c->drain));
    __syncwarp();
    mbar_wait(smem_u32(&c->drain), 0, &go_on);
  }
};

// ---- softmax ----
template <class T>
__device__ __forceinline__ uint32_t pack16(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack16<__nv_bfloat16>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <>
__device__ __forceinline__ uint32_t pack16<__half>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <class T, int DP>
struct Softmax {
  const AttendArgs& a;
  Control* c;
  uint32_t tmem;  // with the warp's lanes
  int st;         // stream
  int row;        // row of the tile = lane of tensor memory
  uint32_t s_phase = 0, o_phase = 0, o1_phase = 0, wg_phase = 0, ml_phase = 0;  // o1: of stream 1, kept by stream 0
  bool joined = false;  // stream 1: its last item was joined by stream 0

  // The scores outside [lo, hi) become -infinity, in tensor memory: few blocks need it, and the loops over
  // the scores stay small (the kernel's code does not fit the instruction cache otherwise).
  __device__ __forceinline__ void hide(int lo, int hi) {
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
      uint32_t r[32];
      __syncwarp();
      tmem_ld32(r, tmem + col_s(st) + q * 32);
      const int from = lo - q * 32, to = hi - q * 32;
      const uint32_t seen = (from >= 32 ? 0u : ~0u << max(from, 0)) & (to >= 32 ? ~0u : (1u << max(to, 0)) - 1);
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (!(seen & 1u << i)) r[i] = 0xff800000u;
      tmem_st32(tmem + col_s(st) + q * 32, r);
    }
    tc_wait_st();
  }
  static __device__ __forceinline__ void top_of(const uint32_t (&r)[32], float (&mx)[4]) {
#pragma unroll
    for (int i = 0; i < 32; i += 8)
#pragma unroll
      for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], __uint_as_float(r[i + k]), __uint_as_float(r[i + 4 + k]));
  }

  // One block: scores to weights, with the running reference m and sum l.
  __device__ __forceinline__ void block(int lo, int hi, bool mask, bool fresh, float& m, float& l) {
    if (mask) hide(lo, hi);
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    uint32_t r[4][32];
#pragma unroll
    for (int q = 0; q < 4; ++q) tmem_ld32_issue(r[q], tmem + col_s(st) + q * 32);
    tmem_landed();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      tmem_tie(r[q]);
      top_of(r[q], mx);
    }
    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
    // While a row has seen no key (a window that begins inside the block), its O and l are zeros of any scale.
    if (fresh || m == -INFINITY) m = top;
    if (!fresh) {
      const bool need = top > m && !((top - m) * a.c <= Weights<T>::kRescale);
      if (__any_sync(0xffffffffu, need)) {
        const float f = need ? exp2_approx((m - top) * a.c) : 1.f;
        const uint64_t f2 = pack2(f, f);
#pragma unroll 1
        for (int q = 0; q < DP / 16; ++q) {
          uint32_t o[16];
          __syncwarp();
          tmem_ld16(o, tmem + col_o<DP>(st) + q * 16);
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            float x, y;
            unpack2(mul2(pack2(__uint_as_float(o[i]), __uint_as_float(o[i + 1])), f2), x, y);
            o[i] = __float_as_uint(x);
            o[i + 1] = __float_as_uint(y);
          }
          tmem_st16(tmem + col_o<DP>(st) + q * 16, o);
        }
        l *= f;
        if (need) m = top;
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32_issue(r[q], tmem + col_s(st) + q * 32);
        tmem_landed();
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_tie(r[q]);
      }
    }
    const float ref = m == -INFINITY ? 0.f : fmaf(-m, a.c, Weights<T>::kFactor);
    const uint64_t c2 = pack2(a.c, a.c), ref2 = pack2(ref, ref);
    uint64_t sum[4] = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t(&s)[32] = r[q];
        float x, y;
        unpack2(fma2(pack2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c2, ref2), x, y);
        x = exp2_approx(x);
        y = exp2_approx(y);
        sum[i & 3] = add2(sum[i & 3], pack2(x, y));
        p[i] = pack16<T>(x, y);
      }
      // Over the first scores, which have been read.
      tmem_st16(tmem + col_s(st) + q * 16, p);
    }
    float x, y;
    unpack2(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), x, y);
    l += x + y;
  }

  __device__ __forceinline__ bool wg_sync() {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&c->wg[st]));
    const bool ok = mbar_wait(smem_u32(&c->wg[st]), wg_phase, &c->abort);
    wg_phase ^= 1;
    return ok;
  }

  __device__ __forceinline__ int position(const Segment& g, int t0, int r) const {
    return g.s.len - g.s.n + g.t0 + t0 + r / a.group;
  }
  __device__ __forceinline__ T* out_row(const Segment& g, int t0, int r) const {
    const int t = r / a.group;
    return static_cast<T*>(a.out.p) + (int64_t)(g.s.begin + g.t0 + t0 + t) * a.out.ts +
           (int64_t)(g.head(st) * a.group + r - t * a.group) * a.out.hs;
  }
  __device__ __forceinline__ void put_lse(const Segment& g, int t0, int r, float m, float l) const {
    if (!a.lse) return;
    const int t = r / a.group;
    a.lse[(int64_t)(g.s.begin + g.t0 + t0 + t) * (a.group * a.hkv) + g.head(st) * a.group + r - t * a.group] =
        l > 0.f || l != l ? m * a.scale + logf(l * Weights<T>::kOff) : -INFINITY;
  }
  // Eight elements of an output row.
  __device__ __forceinline__ void put8(T* p, const float (&x)[8]) const {
    const uint4 v = make_uint4(pack16<T>(x[0], x[1]), pack16<T>(x[2], x[3]), pack16<T>(x[4], x[5]),
                               pack16<T>(x[6], x[7]));
    if (a.vec_out) {
      *reinterpret_cast<uint4*>(p) = v;
    } else {
      uint16_t* e = reinterpret_cast<uint16_t*>(p);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
  }

  // Results of a tile, or its partial sums.  join: O, m and l of stream 1 belong to the same rows.
  // seen: the row sees a key (where it does and l is zero all its scores are -infinity, and 0 / 0 is the result).
  // out: the row's first element.
  __device__ __forceinline__ void finish(const Segment& g, int t0, int rows, bool join, bool seen, float m, float l,
                                         T* out) {
    const bool whole = g.whole;
    float w0 = 1.f, w1 = 0.f;
    if (join) {
      const float2 o = c->ml[row];
      const float top = fmaxf(m, o.x);
      w0 = m == top ? 1.f : exp2_approx((m - top) * a.c);  // equal also when both are -infinity
      w1 = o.x == top ? 1.f : exp2_approx((o.x - top) * a.c);
      l = l * w0 + o.y * w1;
      m = top;
    }
    const bool mine = row < rows;
    const int warp_rows = rows - (row & ~31);
    int slot = 0;
    if (!whole) slot = (blockIdx.x * 2 + (g.first >= c->per * blockIdx.x)) * 2 + st;
    if (whole) {
      const float inv = seen ? 1.f / l : 0.f;
      w0 *= inv;
      w1 *= inv;
    }
    const int d = a.d;
    const bool vec32 = a.vec32;
    if (warp_rows > 0) {
#pragma unroll 1
      for (int q = 0; q < DP; q += 16) {
        uint32_t o[16], o1[16];
        __syncwarp();
        tmem_ld16(o, tmem + col_o<DP>(st) + q);
        if (join) tmem_ld16(o1, tmem + col_o<DP>(1) + q);
        float x[2][8];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          x[i / 8][i % 8] = __uint_as_float(o[i]) * w0;
          if (join) x[i / 8][i % 8] += __uint_as_float(o1[i]) * w1;
        }
        if (!mine) continue;
        if (whole) {
          if (vec32 && q + 16 <= d) {
            store32(out + q, pack16<T>(x[0][0], x[0][1]), pack16<T>(x[0][2], x[0][3]), pack16<T>(x[0][4], x[0][5]),
                    pack16<T>(x[0][6], x[0][7]), pack16<T>(x[1][0], x[1][1]), pack16<T>(x[1][2], x[1][3]),
                    pack16<T>(x[1][4], x[1][5]), pack16<T>(x[1][6], x[1][7]));
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (q + e * 8 < d) put8(out + q + e * 8, x[e]);
          }
        } else {
          float4* p = a.ws_o + ((int64_t)slot * (DP / 4) + q / 4) * kTile + row;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            p[e * kTile] = make_float4(x[e / 2][e % 2 * 4], x[e / 2][e % 2 * 4 + 1], x[e / 2][e % 2 * 4 + 2],
                                       x[e / 2][e % 2 * 4 + 3]);
        }
      }
    }
    if (mine) {
      if (whole) put_lse(g, t0, row, m, l);
      else a.ws_ml[slot * kTile + row] = make_float2(m, l);
    }
  }

  // The item is split between CTAs c0..c1: the last of them to arrive adds the parts.
  __device__ __forceinline__ bool arrive(const Segment& g, int t0, int rows) {
    const int64_t per = c->per;
    const int c0 = (int)div_down(g.first, per), c1 = (int)div_down(g.last - 1, per);
    const int wt = threadIdx.x & 127;
    __threadfence();
    if (!wg_sync()) return false;
    if (wt == 0) {
      const unsigned before = atomicAdd(a.ctr + c0 * 2 + st, 1u);
      c->last[st] = before == (unsigned)(c1 - c0);
    }
    if (!wg_sync()) return false;
    if (!c->last[st]) return true;
    __threadfence();
    if (wt == 0) a.ctr[c0 * 2 + st] = 0;
    // A thread has eight columns of a row, and goes through the parts with a running maximum, kAhead of
    // them loaded at a time: each round of loads is a trip to the L2 cache.
    constexpr int kAhead = 8;
    const int n = rows * (a.d / 8);
#pragma unroll 1
    for (int i = wt; i < n; i += 128) {
      const int r = i % rows, g8 = i / rows;
      float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, sum = 0.f, top = -INFINITY;
#pragma unroll 1
      for (int p0 = c0; p0 <= c1; p0 += kAhead) {
        float2 ml[kAhead];
        float4 u[kAhead], v[kAhead];
        float next = top;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int p = p0 + k, slot = (p * 2 + (p == c0)) * 2 + st;
          ml[k] = make_float2(-INFINITY, 0.f);
          u[k] = v[k] = make_float4(0, 0, 0, 0);
          if (p <= c1) {
            ml[k] = __ldcg(a.ws_ml + slot * kTile + r);
            const float4* o = a.ws_o + ((int64_t)slot * (DP / 4) + g8 * 2) * kTile + r;
            u[k] = __ldcg(o);
            v[k] = __ldcg(o + kTile);
          }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) next = fmaxf(next, ml[k].x);
        const float old = top == next ? 1.f : exp2_approx((top - next) * a.c);
        sum *= old;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= old;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const float f = ml[k].x == next ? 1.f : exp2_approx((ml[k].x - next) * a.c);
          sum += ml[k].y * f;
          x[0] += u[k].x * f;
          x[1] += u[k].y * f;
          x[2] += u[k].z * f;
          x[3] += u[k].w * f;
          x[4] += v[k].x * f;
          x[5] += v[k].y * f;
          x[6] += v[k].z * f;
          x[7] += v[k].w * f;
        }
        top = next;
      }
      const float inv = position(g, t0, r) >= 0 ? 1.f / sum : 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= inv;
      put8(out_row(g, t0, r) + g8 * 8, x);
      if (g8 == 0) put_lse(g, t0, r, top, sum);
    }
    return true;
  }

  __device__ __forceinline__ void run() {
    Feed feed{c};
    for (; const Segment* p = feed.next(); feed.done()) {
      const Segment& g = *p;
      const int t0 = g.pair ? st * a.tok : 0;
      const int rows = min(a.tok, g.nt - t0) * a.group;
      if (g.nb == 0) {  // no row sees a key
        if ((g.both() || st == 0) && row < rows) {
          T* out = out_row(g, t0, row);
          const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
          for (int e = 0; e < a.d; e += 8) put8(out + e, zero);
          put_lse(g, t0, row, 0.f, 0.f);
        }
        continue;
      }
      const bool active = (row & ~31) < rows;
      const int p0 = g.s.len - g.s.n + g.t0 + t0;        // position of the tile's first token
      const int p1 = p0 + min(a.tok, g.nt - t0) - 1;     // and of its last
      const int pos = row < rows ? p0 + row / a.group : -1;
      float m = -INFINITY, l = 0.f;
      const bool both = g.both(), join = !both && g.nb > 1;
      const int nb = g.stream_blocks(st), window = a.window;
      int k0 = (g.j0 + (both ? 0 : st)) * kKeys;  // first key of the stream's next block
      for (int i = 0; i < nb; ++i, k0 += both ? kKeys : 2 * kKeys) {
        if (!mbar_wait(smem_u32(&c->s_full[st]), s_phase, &c->abort)) return;
        s_phase ^= 1;
        if (active) {
          tc_fence_after();
          const bool mask = k0 + kKeys > p0 + 1 || (window > 0 && p1 - k0 >= window);
          const int hi = max(pos + 1 - k0, 0), lo = window > 0 && pos - k0 >= window ? pos - k0 - window + 1 : 0;
          block(lo, hi, mask, i == 0, m, l);
          tc_wait_st();
          tc_fence_before();
        }
        // the join of the item before has to have read this stream's O before it is overwritten
        if (joined) {
          if (!mbar_wait(smem_u32(&c->ml_free), ml_phase ^ 1, &c->abort)) return;
          joined = false;
          tc_fence_after();
          tc_fence_before();
        }
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&c->p_full[st]));
      }
      T* out = row < rows ? out_row(g, t0, row) : nullptr;  // (while the last product runs)
      if (nb > 0) {
        if (!mbar_wait(smem_u32(&c->o_full[st]), o_phase, &c->abort)) return;
        o_phase ^= 1;
      }
      if (join && st == 1) {
        c->ml[row] = make_float2(m, l);
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&c->ml_full));
        ml_phase ^= 1;
        joined = true;
        continue;
      }
      if (st == 1 && !both) continue;
      if (join) {
        // In this order: o_full[1] may be a phase behind until stream 1 says that its item is done.
        if (!mbar_wait(smem_u32(&c->ml_full), ml_phase, &c->abort)) return;
        if (!mbar_wait(smem_u32(&c->o_full[1]), o1_phase, &c->abort)) return;
        ml_phase ^= 1;
      }
      if (st == 0 && (join || both)) o1_phase ^= 1;
      tc_fence_after();
      finish(g, t0, rows, join, pos >= 0, m, l, out);
      tc_fence_before();
      if (join) {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&c->ml_free));
      }
      if (!g.whole && !arrive(g, t0, rows)) return;
    }
  }
};

template <class T, int DP>
__global__ void __launch_bounds__(kThreads, 1)
    k_attend(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map_k,
             const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q) {
  using L = Layout<DP>;
  extern __shared__ __align__(1024) char smem[];
  Control* c = reinterpret_cast<Control*>(smem + L::kCtl);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < L::kStages; ++i) {
      mbar_init(smem_u32(&c->kv_full[i]), 1);
      mbar_init(smem_u32(&c->kv_empty[i]), 1);
    }
    for (int i = 0; i < kSegs; ++i) {
      mbar_init(smem_u32(&c->seg_full[i]), 1);
      mbar_init(smem_u32(&c->seg_empty[i]), kReaders);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&c->q_full[i]), 1);
      mbar_init(smem_u32(&c->q_empty[i]), 1);
      mbar_init(smem_u32(&c->s_full[i]), 1);
      mbar_init(smem_u32(&c->p_full[i]), 4);
      mbar_init(smem_u32(&c->o_full[i]), 1);
      mbar_init(smem_u32(&c->wg[i]), 4);
    }
    mbar_init(smem_u32(&c->ml_full), 4);
    mbar_init(smem_u32(&c->ml_free), 4);
    mbar_init(smem_u32(&c->drain), 1);
    c->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  if (warp == 9) tmem_alloc(smem_u32(&c->tmem), 512);
  if (warp == 10 && elect_one()) {
    prefetch_map(&map_k);
    prefetch_map(&map_v);
    if (a.map_q) prefetch_map(&map_q);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = c->tmem;
  chain_wait();
  // Tokens before the first sequence and behind the last are in none: their rows are not written.
  if (blockIdx.x == 0 && threadIdx.x == 256 && (__ldcg(a.b.q_off) != 0 || __ldcg(a.b.q_off + a.b.n) != a.b.n_tokens))
    set_error(a.err, MISAT_ERR_INVALID_ARG);
  Walk w;
  if (a.small || find_run(a, c, reinterpret_cast<Seq*>(smem + L::kKv), w)) {
    if (warp < 8) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
      Softmax<T, DP> s{a, c, tmem + ((uint32_t)(warp & 3) << 21), warp / 4, (int)(threadIdx.x & 127)};
      s.run();
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
      if (warp == 10) {
        Loader<DP> ld{a, &map_k, &map_v, c, smem_u32(smem) + L::kKv};
        ld.run();
        if (*(volatile int*)&c->abort) ld.drain();
      } else if (warp == 9) {
        Issuer<T, DP> is{a, c, smem, smem_u32(smem), smem_u32(smem) + L::kCtl, tmem};
        is.run();
        is.drain();
      } else if (warp == 8) {
        load_queries<T, DP>(a, &map_q, smem, c);
      } else if (warp == 11) {
        if (a.small && !find_run_small(a, c, w)) w.left = 0;
        feed(a, c, w);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 9) tmem_free(tmem, 512);
  if (threadIdx.x == 0 && c->abort) set_error(a.err, MISAT_ERR_INTERNAL);
}

template <class T, int DP>
int allow_smem() {
  return cudaFuncSetAttribute(k_attend<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<DP>()) ==
                 cudaSuccess
             ? MISAT_OK
             : MISAT_ERR_CUDA;
}

template <class T, int DP>
void launch(const misat_kv* kv, const AttendArgs& a, const CUtensorMap& map_q, cudaStream_t st) {
  launch_chained(k_attend<T, DP>, kv->num_sms, kThreads, smem_bytes<DP>(), st, a, kv->map_k, kv->map_v, map_q);
}

// Map of [n2][n1][d] 16-bit elements, strides in bytes, for boxes of 64 elements x b1 x b2.
bool encode_map(const misat_kv* kv, CUtensorMap* map, void* p, cuuint64_t n1, cuuint64_t stride1, cuuint64_t n2,
                cuuint64_t stride2, cuuint32_t b1, cuuint32_t b2) {
  const cuuint64_t dims[3] = {(cuuint64_t)kv->d, n1, n2}, strides[2] = {stride1, stride2};
  const cuuint32_t box[3] = {64, b1, b2}, unit[3] = {1, 1, 1};
  return kv->encode(map, kv->dtype == MISAT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                    3, p, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

namespace misat {

int attend_prepare(misat_kv* kv) {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) !=
          cudaSuccess ||
      found != cudaDriverEntryPointSuccess)
    return MISAT_ERR_CUDA;
  kv->encode = reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(fn);
  // [blocks x kv heads][16][d]; a box is 64 elements of the 16 tokens of one block and head.  Elements past d
  // are filled with zeros, so a head of any size up to 64 or 128 uses the whole tile.
  const cuuint64_t rows = (cuuint64_t)kv->n_blocks * kv->hkv, row = (cuuint64_t)kv->d * 2;
  if (!encode_map(kv, &kv->map_k, kv->kb, kBlockTokens, row, rows, row * kBlockTokens, kBlockTokens, 1) ||
      !encode_map(kv, &kv->map_v, kv->vb, kBlockTokens, row, rows, row * kBlockTokens, kBlockTokens, 1))
    return MISAT_ERR_CUDA;
  const bool bf = kv->dtype == MISAT_BF16;
  const int dp = kv->d > 64 ? 128 : 64;
  const int rc = dp == 128 ? (bf ? allow_smem<__nv_bfloat16, 128>() : allow_smem<__half, 128>())
                           : (bf ? allow_smem<__nv_bfloat16, 64>() : allow_smem<__half, 64>());
  if (rc != MISAT_OK) return rc;
  // Error word and arrivals (zero between calls), statistics and sums of the parts: four slots a CTA.
  const size_t slots = (size_t)kv->num_sms * 4, head = 256 + (kv->num_sms * 2 * sizeof(unsigned) + 255) / 256 * 256;
  char* p = nullptr;
  if (cudaMalloc(&p, head + slots * kTile * (sizeof(float2) + dp * sizeof(float))) != cudaSuccess) return MISAT_ERR_OOM;
  kv->err = reinterpret_cast<int32_t*>(p);
  kv->ctr = reinterpret_cast<unsigned*>(p + 256);
  kv->head = head;
  kv->ws_ml = reinterpret_cast<float2*>(p + head);
  kv->ws_o = reinterpret_cast<float4*>(p + head + slots * kTile * sizeof(float2));
  return cudaMemset(p, 0, head) == cudaSuccess ? MISAT_OK : MISAT_ERR_CUDA;
}

void launch_attend(misat_kv* kv, const KvBatch& b, const Heads& q, const Heads& out, float* lse, int32_t window,
                   cudaStream_t st) {
  const int group = kv->hq / kv->hkv;
  AttendArgs a{};
  a.b = b;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.scale = kv->scale;
  a.c = kv->scale * 1.4426950408889634f;
  a.group = group;
  a.hkv = kv->hkv;
  a.d = kv->d;
  a.n_blocks = kv->n_blocks;
  a.window = window;
  a.tok = kTile / group;
  a.rows = (int)std::min<int64_t>((int64_t)b.max_q * group, a.tok * group);
  a.vec_out = aligned16(out, 2);
  a.vec32 = ((reinterpret_cast<uintptr_t>(out.p) | (uintptr_t)(out.ts * 2) | (uintptr_t)(out.hs * 2)) & 31) == 0;
  a.ws_o = kv->ws_o;
  a.ws_ml = kv->ws_ml;
  a.ctr = kv->ctr;
  a.err = kv->err;
  a.small = b.n <= 32 && (b.n_tokens / (2 * a.tok) + (int64_t)b.n) * kv->hkv <= kv->num_sms;
  // Queries come through a map where rows start at 16-byte boundaries (a head or token that is read as
  // several has a stride of zero, which a map cannot have); the strides of single heads and tokens are free.
  CUtensorMap map_q{};
  const int64_t hs = kv->hq > 1 ? q.hs : kv->d, ts = b.n_tokens > 1 ? q.ts : (int64_t)kv->hq * kv->d;
  if (aligned16({q.p, ts, hs}, 2) && hs > 0 && ts > 0)
    a.map_q = encode_map(kv, &map_q, q.p, kv->hq, hs * 2, b.n_tokens, ts * 2, group, a.tok);
  const bool bf = kv->dtype == MISAT_BF16;
  if (kv->d > 64) bf ? launch<__nv_bfloat16, 128>(kv, a, map_q, st) : launch<__half, 128>(kv, a, map_q, st);
  else bf ? launch<__nv_bfloat16, 64>(kv, a, map_q, st) : launch<__half, 64>(kv, a, map_q, st);
}

}  // namespace misat
