// Trees of drafted tokens on a pool's blocks: the plan of a step's trees, and what is kept of them.
//
// Plan: node i of a sequence has a parent before it, or follows the tokens before the tree.  Depth and ancestors of a
// node come from walking up, a thread per node, in shared memory: parents are smaller numbers, so the walk ends, and
// its ancestors come in falling order, so the bits of a word are complete before the next lower word begins.
//
// Keep: the keys and values of the accepted nodes move from slot P + path[i] to P + i.  The path rises, so path[i] >= i,
// and a thread that owns 16 bytes of a row's elements and goes through the path in order reads every row before it is
// written, also where it has several rows in flight.
//
// Both are bound by latency: a few dependent reads a sequence, then one pass over the rows.  The plan of 64 trees of 16 to
// 32 nodes takes 1.8 us, of 1,024 trees of 129 nodes 4.8; paths of 64 such trees (8 kv heads of 128) 3.3 us.  1,024 paths of
// up to 64 rows of 8 x 64 elements move 95 MB in 21.7 us, 0.64 of the copy rate: 128 bytes at a place.  Sixteen rows of a
// column are in flight (8: 27.4 us, 24: 22.7, 32: 21.9).
#include <algorithm>

#include "kv.h"

using namespace misat;

namespace {

constexpr int kThreads = 128;    // of k_keep
constexpr int kMaxNodes = 512;   // threads of k_tree: one a node up to here
constexpr int kRoot = -1, kAbsent = -2;

struct TreeArgs {
  KvBatch b;
  const int32_t* parent;
  int32_t* depth;
  uint32_t* bits;
  int32_t words, window;
  int32_t* err;
};

// New tokens of sequence b and its place in the batch; n = 0 where it is malformed (its tokens are then [begin, end),
// wherever that leads).
struct Range {
  int begin, n, len, end;
};
__device__ __forceinline__ Range load_range(const KvBatch& k, int b, int32_t* err) {
  const int begin = __ldcg(k.q_off + b), end = __ldcg(k.q_off + b + 1), len = __ldcg(k.kv_len + b);
  const bool ok = begin >= 0 && end >= begin && end <= k.n_tokens && end - begin <= k.max_q && len >= end - begin &&
                  len <= kMaxLen && len <= k.stride * kBlockTokens;
  if (!ok && threadIdx.x == 0) set_error(err, MISAT_ERR_INVALID_ARG);
  return {begin, ok ? end - begin : 0, len, end};
}

// Tokens [from, to) of the batch, as far as it has them: nodes that are not there.
__device__ __forceinline__ void put_absent(const TreeArgs& a, int from, int to) {
  to = min(to, a.b.n_tokens);
  for (int64_t t = max(from, 0) + (int64_t)threadIdx.x; t < to; t += blockDim.x) {
    a.depth[t] = 0;
    for (int w = 0; w < a.words; ++w) a.bits[t * a.words + w] = 0;
  }
}

__global__ void __launch_bounds__(kMaxNodes) k_tree(const __grid_constant__ TreeArgs a) {
  __shared__ int32_t up[MISAT_KV_TREE_NODES];
  chain_wait();
  // Every token of the batch gets a depth and bits: it is before the first sequence, behind the last, or between two
  // neighbouring offsets, and absent where these are malformed.
  if (blockIdx.x == 0) {
    const int first = __ldcg(a.b.q_off), last = __ldcg(a.b.q_off + a.b.n);
    if (first != 0 || last != a.b.n_tokens) {
      if (threadIdx.x == 0) set_error(a.err, MISAT_ERR_INVALID_ARG);
      put_absent(a, 0, first);
      put_absent(a, last, a.b.n_tokens);
    }
  }
  const Range s = load_range(a.b, blockIdx.x, a.err);
  if (s.n == 0) put_absent(a, s.begin, s.end);
  for (int i = (int)threadIdx.x; i < s.n; i += blockDim.x) {
    const int p = __ldcg(a.parent + s.begin + i);
    up[i] = p < i && p >= kAbsent ? p : kAbsent - 1;  // (neither a parent nor one of the two marks)
  }
  __syncthreads();
  for (int i = (int)threadIdx.x; i < s.n; i += blockDim.x) {
    // Up to the tokens before the tree, with the bits of the first `window` nodes.
    uint32_t* row = a.bits + (int64_t)(s.begin + i) * a.words;
    int at = i, nodes = 0;
    const int most = a.window > 0 ? a.window : MISAT_KV_TREE_NODES;
    for (int w = a.words - 1; w >= 0; --w) {
      uint32_t word = 0;
      for (; at >= w * 32 && nodes < most; ++nodes) {
        word |= 1u << (at & 31);
        at = up[at];
      }
      row[w] = word;
    }
    for (; at >= 0; ++nodes) at = up[at];
    const bool there = at == kRoot;
    a.depth[s.begin + i] = there ? nodes - 1 : 0;
    if (!there) {
      if (at != kAbsent || nodes > 1) set_error(a.err, MISAT_ERR_INVALID_ARG);
      for (int w = 0; w < a.words; ++w) row[w] = 0;
    }
  }
}

struct KeepArgs {
  KvBatch b;
  const int32_t* path;
  int64_t path_stride;
  const int32_t* n_keep;
  int32_t* len_out;
  uint4* kb;
  uint4* vb;
  int32_t hkv, vecs, n_blocks, split, width;  // vecs: of 16 bytes a row; split: CTAs of a sequence; width: longest path
  int32_t* err;
};

__global__ void __launch_bounds__(kThreads) k_keep(const __grid_constant__ KeepArgs a) {
  constexpr int kAhead = 16;
  extern __shared__ __align__(16) longlong2 moves[];  // rows of kv head 0: from and to, from = -1: stays
  const int b = blockIdx.x, tid = threadIdx.x;
  chain_wait();
  const int32_t* path = a.path + (int64_t)b * a.path_stride;
  // The path is read beside the lengths that say how much of it counts.
  int p = tid < a.width ? __ldcg(path + tid) : 0, last = tid > 0 && tid < a.width ? __ldcg(path + tid - 1) : -1;
  const int m = __ldcg(a.n_keep + b);
  const Range s = load_range(a.b, b, a.err);
  bool ok = m >= 0 && m <= s.n && m <= a.width && s.len >= s.n;
  const int before = s.len - s.n;
  auto row_of = [&](int pos) {
    const int blk = __ldcg(a.b.table + (int64_t)b * a.b.stride + pos / kBlockTokens);
    return blk >= 0 && blk < a.n_blocks ? ((int64_t)blk * a.hkv * kBlockTokens + pos % kBlockTokens) * a.vecs : -1;
  };
  if (ok) {
    for (int i = tid; i < m; i += kThreads) {
      if (i != tid) {
        p = __ldcg(path + i);
        last = __ldcg(path + i - 1);
      }
      const bool fits = p > last && p < s.n && p >= i;
      longlong2 move = make_longlong2(-1, -1);
      if (fits && p != i) move = make_longlong2(row_of(before + p), row_of(before + i));
      moves[i] = move;
      ok = ok && fits && (p == i || (move.x >= 0 && move.y >= 0));
    }
  }
  ok = __syncthreads_and(ok);
  if (blockIdx.y == 0 && tid == 0) {
    if (!ok) set_error(a.err, MISAT_ERR_INVALID_ARG);
    a.len_out[b] = ok ? before + m : __ldcg(a.b.kv_len + b);
  }
  if (!ok) return;
  // A column: 16 bytes of the rows of a kv head, of the keys or the values.
  const int heads = a.hkv * a.vecs, cols = 2 * heads;
  for (int c = blockIdx.y * kThreads + tid; c < cols; c += a.split * kThreads) {
    uint4* rows = c < heads ? a.kb : a.vb;
    const int k = c < heads ? c : c - heads, head = k / a.vecs;
    rows += (int64_t)head * kBlockTokens * a.vecs + (k - head * a.vecs);
#pragma unroll 1
    for (int i = 0; i < m; i += kAhead) {
      uint4 v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < m && moves[i + j].x >= 0) v[j] = rows[moves[i + j].x];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < m && moves[i + j].x >= 0) rows[moves[i + j].y] = v[j];
    }
  }
}

}  // namespace

extern "C" {

int misat_kv_tree(misat_kv* kv, const misat_kv_batch* batch, const int32_t* parents, int32_t window, int32_t* depth,
                  uint32_t* bits, int32_t words, void* cuda_stream) {
  if (!batch_ok(kv, batch) || window < 0 || batch->max_q > MISAT_KV_TREE_NODES || words < 0 ||
      words != (batch->max_q + 31) / 32)
    return MISAT_ERR_INVALID_ARG;
  if (batch->n_tokens == 0) return MISAT_OK;
  if (!parents || !depth || !bits || batch->max_q == 0 || !on_device(kv->device)) return MISAT_ERR_INVALID_ARG;
  if (!at_elements(parents) || !at_elements(depth) || !at_elements(bits)) return MISAT_ERR_INVALID_ARG;
  // A CTA reads its sequence's parents and lengths while others write.
  const int64_t n = batch->n, T = batch->n_tokens;
  const Extent d(depth, T), m(bits, T * words);
  if (!apart(d, m)) return MISAT_ERR_INVALID_ARG;
  for (const Extent& x : {Extent(batch->kv_len, n), Extent(batch->q_off, n + 1), Extent(parents, T)})
    if (!apart(d, x) || !apart(m, x)) return MISAT_ERR_INVALID_ARG;
  const TreeArgs a{batch_view(batch), parents, depth, bits, words, window, kv->err};
  const int threads = std::min((batch->max_q + 31) / 32 * 32, kMaxNodes);
  launch_chained(k_tree, batch->n, threads, 0, static_cast<cudaStream_t>(cuda_stream), a);
  return launch_status();
}

int misat_kv_keep(misat_kv* kv, const misat_kv_batch* batch, const int32_t* path, int64_t path_stride,
                  const int32_t* n_keep, int32_t* kv_len_out, void* cuda_stream) {
  if (!batch_ok(kv, batch) || batch->max_q > MISAT_KV_TREE_NODES || path_stride < 0) return MISAT_ERR_INVALID_ARG;
  if (batch->n == 0) return MISAT_OK;
  if (!batch->q_off || !batch->kv_len || (!batch->block_table && batch->table_stride > 0) ||
      (!path && path_stride > 0) || !n_keep || !kv_len_out || !on_device(kv->device))
    return MISAT_ERR_INVALID_ARG;
  if (!at_elements(path) || !at_elements(n_keep) || !at_elements(kv_len_out)) return MISAT_ERR_INVALID_ARG;
  // Several CTAs read what there is of a sequence, and one of them writes its length.  (The last row of several may be shorter
  // than their distance.)
  const int64_t n = batch->n, table = n == 1 ? batch->table_stride : (n - 1) * batch->table_stride + 1;
  const Extent out(kv_len_out, n);
  for (const Extent& x : {Extent(batch->kv_len, n), Extent(batch->q_off, n + 1), Extent(batch->block_table, table),
                          Extent(n_keep, n), Extent(path, n * path_stride)})
    if (!apart(out, x)) return MISAT_ERR_INVALID_ARG;
  KeepArgs a{};
  a.b = batch_view(batch);
  a.path = path;
  a.path_stride = path_stride;
  a.n_keep = n_keep;
  a.len_out = kv_len_out;
  a.kb = static_cast<uint4*>(kv->kb);
  a.vb = static_cast<uint4*>(kv->vb);
  a.hkv = kv->hkv;
  a.vecs = kv->d / 8;
  a.n_blocks = kv->n_blocks;
  a.width = (int)std::min<int64_t>(path_stride, MISAT_KV_TREE_NODES);
  a.err = kv->err;
  const int cols = (2 * kv->hkv * a.vecs + kThreads - 1) / kThreads;
  a.split = std::max(1, std::min(cols, kv->num_sms * 8 / batch->n));
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3(batch->n, a.split);
  lc.blockDim = dim3(kThreads);
  lc.dynamicSmemBytes = sizeof(longlong2) * a.width;
  lc.stream = static_cast<cudaStream_t>(cuda_stream);
  lc.attrs = &at;
  lc.numAttrs = 1;
  cudaLaunchKernelEx(&lc, k_keep, a);
  return launch_status();
}

}  // extern "C"
