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
// over 129,024, 32 heads: 3.03 to 3.47 ms on different GPUs, power-capped at some 1.55 GHz).
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
#include "runs.cuh"
#include "tensor.cuh"

using namespace misat;
using namespace misat::runs;

namespace {

constexpr int kRegsIssue = 88, kRegsSoftmax = 208;  // 128 * 88 + 256 * 208 = 384 * 168 registers

// The weights in 16 bits are 2^(kFactor + c (s - m)): O and l carry the factor 2^kFactor, which the result does not
// see and the log-sum-exp takes off; O and l are rescaled when a score passes m by more than 2^kRescale.
// bfloat16 has the exponents of 32 bits and needs no factor.  float16 holds 2^-14 to 2^16 in full precision and
// rounds to zero below 2^-25: with 61,000 as the largest weight, one that is 2^-25 of its row's reference keeps its
// 11 bits, and zero is what is below 2^-36 of it.  (With 2^8 as the largest weight and no factor, 131,072 keys 18
// below one that takes most of the weight added up to 1.4% too little.)  The narrower range means more rescales: 97
// prompts of 512 to 2,048 tokens under a window, scores of standard deviation 1, took 954 us with it, 940 with a factor
// of 2^10, 934 with 2^9, 930 with 2^8; one token over 131,072, 91 us with each.
template <class T>
struct Weights {
  static constexpr float kRescale = 8.f, kFactor = 0.f, kOff = 1.f;
};
template <>
struct Weights<__half> {
  static constexpr float kRescale = 4.9f, kFactor = 11.f, kOff = 0x1p-11f;
};

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
    const bool need = !fresh && top > m && !((top - m) * a.c <= Weights<T>::kRescale);
    const float from = m;
    if (need) m = top;
    float ref = m == -INFINITY ? 0.f : fmaf(-m, a.c, Weights<T>::kFactor);
    // Where c m has few bits behind the point, the weights' exponents do not come out of c s - c m: m is taken off the
    // scores first, which is exact near it.  (The rounding of c m would pass float16's largest weight.)
    const bool far = fabsf(ref) >= 0x1p20f;
    if (__any_sync(0xffffffffu, need || far)) {
      if (!fresh) {
        const float f = need ? exp2_approx((from - top) * a.c) : 1.f;
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
      }
      const float off = far ? m : 0.f;
#pragma unroll 1
      for (int q = __any_sync(0xffffffffu, far) ? 0 : 4; q < 4; ++q) {
        uint32_t x[32];
        __syncwarp();
        tmem_ld32(x, tmem + col_s(st) + q * 32);
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) - off);
        tmem_st32(tmem + col_s(st) + q * 32, x);
      }
      tc_wait_st();
      if (far) ref = Weights<T>::kFactor;
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_ld32_issue(r[q], tmem + col_s(st) + q * 32);
      tmem_landed();
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_tie(r[q]);
    }
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
    const Parts parts = parts_of(a, g, c->per);
    const int c0 = parts.first, c1 = parts.last;
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
        QueryLoader<DP> ql{a, &map_q, smem, c};
        ql.run();
        if (*(volatile int*)&c->abort) ql.drain();
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
