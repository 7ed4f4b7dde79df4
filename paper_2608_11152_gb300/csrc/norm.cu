// Norm of each head with the rotation behind it, forward (into a tensor, or into blocks) and backward.
//
//   y = R_p (x r w),  r = 1 / sqrt(mean x^2 + eps)
//   g = R_p^T dy,  a = g w,  dx = r (a - x r mean(a x r)),  dw = sum g x r          (w with its offset)
//
// One pass: a group of lanes holds a head of a token, so the sums over its elements are shuffles within the group and
// the elements are read once.  A lane has the same unit of the same head (rotary's units: in the half layout two vectors
// rot/2 apart or one past the rotated part, else one vector of whole pairs) of one token after the other: the weight,
// and backward its gradient, stay in registers, and the tokens' cosines and sines come from shared memory, where they
// are worked out once for all heads of the CTA.  Squares, sums and products are in 32 bits, results are rounded once.
//
// Bound by memory where there are many tokens: 65,536 x 32 heads of 128 in bf16 forward 162 us for 1.07 GB (6.6 TB/s,
// 0.97 of a plain copy), backward 241 us for 1.61 GB (0.98); by latency and issue where there are few: 64 tokens 2.3 us,
// 5,003 tokens of 28 heads of 96 12.4 us (floor 7.9).  With the next token in registers instead of shared memory
// these two were 411 and 24.8 us.
//
// The weight's gradient is a sum over tokens (and heads): each CTA of a fixed grid writes the sum of its tokens, and a
// second kernel adds these in order.  Of few tokens the CTAs are one cluster, and add the sums in each other's shared
// memory: one launch instead of two.
#include <algorithm>
#include <cmath>

#include "kv.h"
#include "rotary.cuh"
#include "tensor.cuh"

using namespace misat;

namespace {

constexpr int kMaxTile = 32;   // tokens of a CTA at a time: their places are found by one warp
constexpr int kMaxHead = 256;  // elements
constexpr int kCluster = 8, kClusterRounds = 3;  // CTAs of a cluster, and rounds of tokens of each
constexpr int kMaxTokens = INT32_MAX - 4096;  // numbers of tokens run past the last one by a few rounds
constexpr int kShared = 47 * 1024;  // dynamic bytes of a CTA, at most 48 KiB with the places of its tokens

// By the elements of a lane and the bytes of its part of a token: threads of a CTA, CTAs on an SM, copies in flight.
struct Shape {
  int threads, ctas, depth;
};
constexpr Shape shape_of(int elements, int bytes, bool backward) {
  if (backward) {
    if (elements > 16) return {128, 3, 3};
    if (bytes > 64) return {128, 3, 2};
    return {256, 2, 128 / bytes};
  }
  if (elements > 16) return {256, 3, 3};
  if (bytes > 48) return {128, 6, 2};
  return {256, 4, 96 / bytes};
}

struct HeadWeight {
  const void* p;  // nullptr: no norm
  int64_t hs;
  float eps, offset;
  bool wide;   // 32 bits, else the tensor's type
  bool whole;  // heads at 16-byte boundaries
};

struct NormArgs {
  int32_t n_tokens, hq, hkv, d, rot;  // hkv = 0: plain rotation of hq heads
  int32_t heads, first;               // rows of a token, and the first of them (queries, keys, values)
  int32_t units, lane_bits, chunk, side;  // lanes of a head; heads of a CTA, tokens side by side
  int32_t per, tile;                  // tokens of a CTA, and of those at a time
  int32_t turns;                      // 32-bit numbers of a token's cosines
  FastDiv by_chunk;
  const uint64_t* freq;
  float attn, inv_d;
  Heads x, out, k, v, dy;
  HeadWeight wq, wk;
  const int32_t* positions;
  const int32_t* depth;
  KvBatch b;
  void* kb;
  void* vb;
  int32_t n_blocks;
  int32_t* err;
  float* parts;
  // Backward in one kernel: the weight's gradient, its rows' distance and type.
  bool fused;
  void* dw;
  int64_t dw_hs;
  int32_t dw_type;
};

__device__ __forceinline__ void put_weight(void* out, int32_t type, int64_t at, float v) {
  if (type == MISAT_F32) static_cast<float*>(out)[at] = v;
  else if (type == MISAT_BF16) static_cast<__nv_bfloat16*>(out)[at] = from_f<__nv_bfloat16>(v);
  else static_cast<__half*>(out)[at] = from_f<__half>(v);
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A number in the shared memory of the cluster's CTA of a rank, at the place that it has in this one's.
__device__ __forceinline__ float of_rank(const float* p, int rank) {
  uint32_t at;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// Two elements rounded in one instruction.
__device__ __forceinline__ void narrow2(float a, float b, __nv_bfloat16* out) {
  *reinterpret_cast<__nv_bfloat162*>(out) = __floats2bfloat162_rn(a, b);
}
__device__ __forceinline__ void narrow2(float a, float b, __half* out) {
  *reinterpret_cast<__half2*>(out) = __floats2half2_rn(a, b);
}

// A lane's part of a head: UPL units of up to two vectors.
template <class T, int VEC, bool HALF, int UPL>
struct Part {
  using V = Vec<T, VEC>;
  static constexpr bool kPair = !HALF && VEC == 1;           // a unit is two neighbouring elements, moved one by one
  static constexpr bool kTwo = HALF || kPair;                // a unit has a second vector
  static constexpr int kStep = kPair ? 2 : VEC;              // elements a unit steps over
  static constexpr int kPairs = HALF ? VEC : kPair ? 1 : VEC / 2;  // pairs of a unit
  static constexpr int kElems = kTwo ? 2 * VEC : VEC;        // elements of a unit
  static constexpr int kBytes = UPL * kElems * (int)sizeof(T);
  static constexpr Shape shape(bool backward) {
    return VEC == 1 ? Shape{256, backward ? 1 : 2, 1} : shape_of(UPL * kElems, kBytes * (backward ? 2 : 1), backward);
  }

  int half, paired, units, d, lane, lanes;
  __device__ __forceinline__ Part(const NormArgs& a, int lane)
      : half(a.rot / 2), paired(HALF ? a.rot / 2 / VEC : (a.rot / 2 + kPairs - 1) / kPairs), units(a.units), d(a.d),
        lane(lane), lanes(1 << a.lane_bits) {}

  __device__ __forceinline__ int unit(int j) const { return lane + j * lanes; }
  __device__ __forceinline__ bool has(int j) const { return unit(j) < units; }
  // First element of a unit, and of its second vector.
  __device__ __forceinline__ int first(int j) const {
    return HALF && unit(j) >= paired ? (unit(j) + paired) * VEC : unit(j) * kStep;
  }
  __device__ __forceinline__ int second(int j) const { return HALF ? unit(j) * VEC + half : unit(j) * 2 + 1; }
  __device__ __forceinline__ bool has_second(int j) const {
    return HALF ? unit(j) < paired : kPair && unit(j) * 2 + 1 < d;
  }
  // Element i of a unit: the first vector's, then the second's.
  __device__ __forceinline__ int element(int j, int i) const { return i < VEC ? first(j) + i : second(j) + i - VEC; }
  __device__ __forceinline__ bool has_element(int j, int i) const { return has(j) && (i < VEC || has_second(j)); }

  struct Raw {
    V lo[UPL], hi[kTwo ? UPL : 1];
    __device__ __forceinline__ V& vec(int v) { return kTwo && v % 2 ? hi[v / 2] : lo[kTwo ? v / 2 : v]; }
  };
  // Each vector with its number, its first element, and whether it is there.
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int j = 0; j < UPL; ++j) {
      f(kTwo ? 2 * j : j, first(j), has(j));
      if constexpr (kTwo) f(2 * j + 1, second(j), has(j) && has_second(j));
    }
  }
  __device__ __forceinline__ void fetch(const T* p, Raw& r) const {
#pragma unroll
    for (int j = 0; j < UPL; ++j) {
      if (has(j)) r.lo[j] = *reinterpret_cast<const V*>(p + first(j));
      if constexpr (kTwo)
        if (has(j) && has_second(j)) r.hi[j] = *reinterpret_cast<const V*>(p + second(j));
    }
  }
  __device__ __forceinline__ void put(T* p, const Raw& r) const {
#pragma unroll
    for (int j = 0; j < UPL; ++j) {
      if (has(j)) *reinterpret_cast<V*>(p + first(j)) = r.lo[j];
      if constexpr (kTwo)
        if (has(j) && has_second(j)) *reinterpret_cast<V*>(p + second(j)) = r.hi[j];
    }
  }
  // In 32 bits, and back.
  __device__ __forceinline__ void widen(const Raw& r, float (&x)[UPL][kElems]) const {
#pragma unroll
    for (int j = 0; j < UPL; ++j)
#pragma unroll
      for (int i = 0; i < kElems; ++i)
        x[j][i] = to_f(i < VEC ? r.lo[j].e[i] : r.hi[kTwo ? j : 0].e[i < VEC ? 0 : i - VEC]);
  }
  __device__ __forceinline__ void narrow(const float (&x)[UPL][kElems], Raw& r) const {
#pragma unroll
    for (int j = 0; j < UPL; ++j)
#pragma unroll
      for (int i = 0; i < kElems; i += VEC) {
        V& v = i < VEC ? r.lo[j] : r.hi[kTwo ? j : 0];
        if constexpr (VEC > 1 && sizeof(T) == 2) {
#pragma unroll
          for (int e = 0; e < VEC; e += 2) narrow2(x[j][i + e], x[j][i + e + 1], v.e + e);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) v.e[e] = from_f<T>(x[j][i + e]);
        }
      }
  }

  // Where pair p of a token's cosines is: eight of a unit are kept as two runs of four, so that neighbouring lanes
  // read neighbouring 16 bytes.
  static __device__ __forceinline__ int place(int p, int paired) {
    if constexpr (kPairs == 8) return ((p % 8 / 4) * paired + p / 8) * 4 + p % 4;
    else return p;
  }
  template <bool BACK>
  __device__ __forceinline__ void turn_all(const float* cosines, const float* sines, float (&x)[UPL][kElems]) const {
#pragma unroll
    for (int j = 0; j < UPL; ++j) {
      if (unit(j) >= paired) continue;
      alignas(16) float c[kPairs], s[kPairs];
      if constexpr (kPairs >= 4) {
#pragma unroll
        for (int k = 0; k < kPairs; k += 4) {
          const int at = place(unit(j) * kPairs + k, paired);
          *reinterpret_cast<float4*>(c + k) = *reinterpret_cast<const float4*>(cosines + at);
          *reinterpret_cast<float4*>(s + k) = *reinterpret_cast<const float4*>(sines + at);
        }
      } else {
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
          c[k] = cosines[unit(j) * kPairs + k];
          s[k] = sines[unit(j) * kPairs + k];
        }
      }
      if constexpr (kTwo && kPairs > 1) {  // two pairs at a time
#pragma unroll
        for (int k = 0; k < kPairs; k += 2) {
          const uint64_t u = pack2(x[j][k], x[j][k + 1]), w = pack2(x[j][VEC + k], x[j][VEC + k + 1]);
          const uint64_t cc = pack2(c[k], c[k + 1]), ss = pack2(s[k], s[k + 1]);
          const uint64_t first = BACK ? fma2(w, ss, mul2(u, cc)) : sub2(mul2(u, cc), mul2(w, ss));
          const uint64_t second = BACK ? sub2(mul2(w, cc), mul2(u, ss)) : fma2(u, ss, mul2(w, cc));
          unpack2(first, x[j][k], x[j][k + 1]);
          unpack2(second, x[j][VEC + k], x[j][VEC + k + 1]);
        }
        continue;
      }
      auto pairs = [&](bool ends) {
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
          if (ends && unit(j) * kPairs + k >= half) continue;
          float& u = x[j][kTwo ? k : 2 * k];
          float& w = x[j][kTwo ? VEC + k : 2 * k + 1];
          const float a = u, b = w, sn = BACK ? -s[k] : s[k];
          u = a * c[k] - b * sn;
          w = a * sn + b * c[k];
        }
      };
      // The rotated part may end inside a vector: what is behind stays as it is (a product with zero would make NaN of
      // an infinity).
      if (HALF || kPairs == 1 || half % kPairs == 0) pairs(false);
      else pairs(true);
    }
  }
  template <class W>
  __device__ __forceinline__ void load_weight(const W* w, bool whole, float offset, float (&out)[UPL][kElems]) const {
    constexpr int N = VEC * (int)sizeof(W) > 16 ? 16 / (int)sizeof(W) : VEC;  // of a vector
#pragma unroll
    for (int j = 0; j < UPL; ++j)
#pragma unroll
      for (int i = 0; i < kElems; i += N) {
        Vec<W, N> v{};
        if (N > 1 && whole) {
          if (has_element(j, i)) v = *reinterpret_cast<const Vec<W, N>*>(w + element(j, i));
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (has_element(j, i + e)) v.e[e] = w[element(j, i + e)];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) out[j][i + e] = offset + to_f(v.e[e]);
      }
  }
  __device__ __forceinline__ void load_weight(const HeadWeight& w, int head, float (&out)[UPL][kElems]) const {
    const int64_t at = (int64_t)head * w.hs;
    if (w.wide) load_weight(static_cast<const float*>(w.p) + at, w.whole, w.offset, out);
    else load_weight(static_cast<const T*>(w.p) + at, w.whole, w.offset, out);
  }
  // The sum over the head's lanes.
  __device__ __forceinline__ float sum(float v) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (lanes > o) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
};

// Sum of products of a lane's elements.
template <int U, int E>
__device__ __forceinline__ float dot(const float (&x)[U][E], const float (&y)[U][E]) {
  uint64_t sum = 0;
#pragma unroll
  for (int j = 0; j < U; ++j)
#pragma unroll
    for (int i = 0; i < E; i += 2)
      sum = fma2(pack2(x[j][i], x[j][i + 1]), pack2(y[j][i], y[j][i + 1]), sum);
  float a, b;
  unpack2(sum, a, b);
  return a + b;
}

// cos and sin of (pos * freq / 2^64) turns.  The nearest quarter turn is taken off in whole numbers; what is left is
// x half turns, |x| <= 1/4, where the power series of sin(pi x) to x^9 and of cos(pi x) to x^10 are off by less than
// 2^-28 of the result.  (Over all heads a token's turns are as many instructions as a head or two; sincospif, which
// takes any x, is twice that: 40,000 tokens of 1 and of 8 heads of 128 took 19.6 and 36.5 us with it, 12.4 and 33.5 now.)
__device__ __forceinline__ float2 short_turn(int32_t pos, uint64_t freq, float attn) {
  const uint32_t ph = (uint32_t)(((uint64_t)(int64_t)pos * freq) >> 32);
  const uint32_t quarter = (ph + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(ph - (quarter << 30)) * 0x1p-31f, y = x * x;
  // pi^k / k!, the first one in two parts
  float s = fmaf(y, 0.0821458866f, -0.599264529f);
  s = fmaf(y, s, 2.55016404f);
  s = fmaf(y, s, -5.16771278f);
  s = fmaf(y, s, -8.74227766e-8f);
  s = fmaf(x, 3.14159274f, x * s);
  float c = fmaf(y, -0.0258068913f, 0.235330630f);
  c = fmaf(y, c, -1.33526277f);
  c = fmaf(y, c, 4.05871213f);
  c = fmaf(y, c, -4.93480220f);
  c = fmaf(y, c, 1.f);
  const float u = quarter & 1 ? -s : c, v = quarter & 1 ? c : s;
  const float f = quarter & 2 ? -attn : attn;
  return make_float2(u * f, v * f);
}

// The tile's cosines and sines: [tokens][2][turns].  A thread has one pair of every so many tokens.
template <class P>
struct Turns {
  int pair, token, step;
  uint64_t freq;
  float* out;
  __device__ __forceinline__ Turns(const NormArgs& a, int paired, float* smem) {
    const int half = a.rot / 2, tid = threadIdx.x;
    step = half > 0 ? (int)blockDim.x / half : 0;
    token = half > 0 ? tid / half : 0;
    pair = tid - token * half;
    if (token >= step) token = kMaxTile;
    else freq = __ldg(a.freq + pair);
    out = smem + P::place(pair, paired);
  }
  __device__ __forceinline__ void fill(const NormArgs& a, int nt, const int32_t* pos) const {
    for (int t = token; t < nt; t += step) {
      const float2 cs = short_turn(pos[t], freq, a.attn);
      float* o = out + t * 2 * a.turns;
      o[0] = cs.x;
      o[a.turns] = cs.y;
    }
  }
};

// A lane's parts of the next tokens on their way: asynchronous copies into shared memory that no other lane reads, so
// that many are in flight without registers; where a part is no whole vectors, the next one in registers.
template <class P, class T, bool WHOLE, int TENSORS>
struct Stages {
  static constexpr int kThreads = P::shape(TENSORS == 2).threads;
  static constexpr int kDepth = P::shape(TENSORS == 2).depth;
  static constexpr int kSize = WHOLE ? kDepth * TENSORS * P::kBytes * kThreads : 0;  // shared memory
  static constexpr int kVec = sizeof(typename P::V);  // bytes
  const P& part;
  const char* smem;  // this thread's first vector
  uint32_t base;
  typename P::Raw next[WHOLE ? 1 : TENSORS];

  __device__ __forceinline__ Stages(const P& part, void* smem)
      : part(part), smem(static_cast<const char*>(smem) + threadIdx.x * kVec),
        base((uint32_t)__cvta_generic_to_shared(smem) + threadIdx.x * kVec) {
    // Vectors that are not there are zeros from the start, and no copy touches them: they add nothing to the sums.
    if constexpr (WHOLE) {
      char* mine = static_cast<char*>(smem) + threadIdx.x * kVec;
      for (int i = 0; i < kDepth * TENSORS; ++i)
        part.each([&](int v, int, bool there) {
          if (!there) *reinterpret_cast<typename P::V*>(mine + (i * (P::kBytes / kVec) + v) * kThreads * kVec) = {};
        });
    } else {
      for (int i = 0; i < TENSORS; ++i) part.each([&](int v, int, bool) { next[i].vec(v) = {}; });
    }
  }
  __device__ __forceinline__ uint32_t at(int stage, int tensor, int vec) const {
    return base + ((stage * TENSORS + tensor) * (P::kBytes / kVec) + vec) * kThreads * kVec;
  }
  __device__ __forceinline__ void issue(int stage, int tensor, const T* p, bool ok) {
    if constexpr (WHOLE) {
      part.each([&](int v, int e, bool there) {
        if (!ok || !there) return;
        if constexpr (kVec == 16)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at(stage, tensor, v)), "l"(p + e) : "memory");
        else
          asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at(stage, tensor, v)), "l"(p + e), "n"(kVec)
                       : "memory");
      });
      if (tensor + 1 == TENSORS) asm volatile("cp.async.commit_group;" ::: "memory");
    } else {
      if (ok) part.fetch(p, next[tensor]);
    }
  }
  __device__ __forceinline__ void wait() const {
    if constexpr (WHOLE) asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
  }
  __device__ __forceinline__ void take(int stage, int tensor, typename P::Raw& r) const {
    if constexpr (WHOLE) {
      part.each([&](int v, int e, bool) {
        r.vec(v) = *reinterpret_cast<const typename P::V*>(smem + (at(stage, tensor, v) - at(0, 0, 0)));
      });
    } else {
      r = next[tensor];
    }
  }
};

template <class T, int VEC, bool HALF, int UPL>
__global__ void __launch_bounds__(Part<T, VEC, HALF, UPL>::shape(false).threads,
                                  Part<T, VEC, HALF, UPL>::shape(false).ctas)
    k_norm_rotate(const __grid_constant__ NormArgs a) {
  extern __shared__ __align__(16) float s_mem[];
  __shared__ int32_t s_pos[kMaxTile];
  // Element offsets of a token's row in the queries' result and of its row of kv head 0 in the blocks, -1: skip.
  __shared__ int64_t s_row[kMaxTile][2];
  using P = Part<T, VEC, HALF, UPL>;
  using S = Stages<P, T, VEC != 1, 1>;
  float* s_turn = s_mem + S::kSize / 4;
  const int tid = threadIdx.x, group = tid >> a.lane_bits, side = a.by_chunk.div(group);
  const P part(a, tid & ((1 << a.lane_bits) - 1));
  S stages(part, s_mem);
  const int h = a.first + blockIdx.y * a.chunk + group - side * a.chunk;
  const bool mine = side < a.side && h < a.first + a.heads;
  const bool works = __any_sync(0xffffffffu, mine);  // the warp has a head at all
  const bool q = h < a.hq, k = h < a.hq + a.hkv;
  const Heads& src = q ? a.x : k ? a.k : a.v;
  const int hh = q ? h : k ? h - a.hq : h - a.hq - a.hkv;
  const int begin = blockIdx.x * a.per, end = (int)min((int64_t)begin + a.per, (int64_t)a.n_tokens);
  const T* in = static_cast<const T*>(src.p) + (int64_t)hh * src.hs + (int64_t)(begin + side) * src.ts;
  const int64_t step = (int64_t)a.side * src.ts;
  // A token's row is at its number's place in the queries' result, or at its slot of the blocks.
  T* const base_out = q ? static_cast<T*>(a.out.p) + (int64_t)h * a.out.hs
                        : static_cast<T*>(k ? a.kb : a.vb) + (int64_t)hh * kBlockTokens * a.d;
  chain_wait();
  int ahead = mine ? begin + side : end;  // the next token to copy
  int put_at = 0, take_at = 0;            // its stage, and that of the next one to work on
  auto issue = [&]() {
    stages.issue(put_at, 0, in, ahead < end);
    ahead += a.side;
    in += step;
    put_at = put_at + 1 == S::kDepth ? 0 : put_at + 1;
  };
#pragma unroll
  for (int i = 0; i < (S::kDepth > 1 ? S::kDepth - 1 : 1); ++i) issue();
  int32_t ahead_pos = a.hkv == 0 && tid < a.tile && begin + tid < end ? __ldcg(a.positions + begin + tid) : 0;
  const Turns<P> turns(a, part.paired, s_turn);
  const HeadWeight& hw = q ? a.wq : a.wk;
  const bool normed = k && hw.p;
  float w[UPL][P::kElems];
  if (normed && mine) part.load_weight(hw, hh, w);
  for (int t0 = begin; t0 < end; t0 += a.tile) {
    const int nt = min(a.tile, end - t0);
    if (t0 > begin) __syncthreads();  // the last tile's turns have been read
    int64_t pos = 0;
    int blk = -1;
    if (a.hkv == 0) {
      if (tid < nt) {
        s_pos[tid] = ahead_pos;
        s_row[tid][0] = (int64_t)(t0 + tid) * a.out.ts;
      }
      if (tid < a.tile && t0 + a.tile + tid < end) ahead_pos = __ldcg(a.positions + t0 + a.tile + tid);
    } else if (tid < 32) {
      const int t = t0 + min(tid, nt - 1), depth = a.depth ? __ldcg(a.depth + t) : 0;
      OffsetFinder find(a.b.q_off, a.b.n, t0);
      int from, to;
      const int b = find(t, from, to), len = __ldcg(a.b.kv_len + b);
      pos = (int64_t)len - to + t;
      const bool ok = from <= t && t < to && to - from <= a.b.max_q && len >= to - from && pos >= 0 &&
                      len <= kMaxLen && pos < a.b.stride * kBlockTokens;
      if (ok) blk = __ldcg(a.b.table + (int64_t)b * a.b.stride + pos / kBlockTokens);
      if (tid < nt) s_pos[tid] = a.depth ? len - (to - from) + depth : (int32_t)pos;
    }
    __syncthreads();
    turns.fill(a, nt, s_pos);
    if (a.hkv > 0 && tid < nt) {  // (the block's number arrives meanwhile)
      const bool ok = blk >= 0 && blk < a.n_blocks;
      if (!ok) set_error(a.err, MISAT_ERR_INVALID_ARG);
      s_row[tid][0] = ok ? (int64_t)(t0 + tid) * a.out.ts : -1;
      s_row[tid][1] = ok ? ((int64_t)blk * a.hkv * kBlockTokens + pos % kBlockTokens) * a.d : -1;
    }
    __syncthreads();
    for (int base = works ? 0 : nt; base < nt; base += a.side) {
      const int t = base + side;
      const bool ok = mine && t < nt;
      typename P::Raw raw;
      if constexpr (S::kDepth > 1) {
        issue();
        stages.wait();
        stages.take(take_at, 0, raw);
        take_at = take_at + 1 == S::kDepth ? 0 : take_at + 1;
      } else {
        stages.take(0, 0, raw);
        issue();
      }
      float x[UPL][P::kElems];
      part.widen(raw, x);
      const float sum = part.sum(dot(x, x));
      const int64_t row = s_row[t < nt ? t : 0][q ? 0 : 1];
      if (!ok || row < 0) continue;
      if (k) {
        if (normed) {
          const float r = rsqrtf(fmaf(sum, a.inv_d, hw.eps));
          const uint64_t r2 = pack2(r, r);
#pragma unroll
          for (int j = 0; j < UPL; ++j)
#pragma unroll
            for (int i = 0; i < P::kElems; i += 2)
              unpack2(mul2(mul2(pack2(x[j][i], x[j][i + 1]), r2), pack2(w[j][i], w[j][i + 1])), x[j][i], x[j][i + 1]);
        }
        const float* cs = s_turn + t * 2 * a.turns;
        part.template turn_all<false>(cs, cs + a.turns, x);
        part.narrow(x, raw);
      }
      part.put(base_out + row, raw);
    }
  }
}

template <class T, int VEC, bool HALF, int UPL>
__global__ void __launch_bounds__(Part<T, VEC, HALF, UPL>::shape(true).threads,
                                  Part<T, VEC, HALF, UPL>::shape(true).ctas)
    k_norm_backward(const __grid_constant__ NormArgs a) {
  extern __shared__ __align__(16) float s_mem[];
  __shared__ int32_t s_pos[kMaxTile];
  using P = Part<T, VEC, HALF, UPL>;
  using S = Stages<P, T, VEC != 1, 2>;
  float* s_turn = s_mem + S::kSize / 4;
  const int tid = threadIdx.x, group = tid >> a.lane_bits, side = a.by_chunk.div(group);
  const P part(a, tid & ((1 << a.lane_bits) - 1));
  S stages(part, s_mem);
  const int h = blockIdx.y * a.chunk + group - side * a.chunk;
  const bool mine = side < a.side && h < a.heads;
  const bool works = __any_sync(0xffffffffu, mine);
  const int begin = blockIdx.x * a.per, end = (int)min((int64_t)begin + a.per, (int64_t)a.n_tokens);
  const T* x_in = static_cast<const T*>(a.x.p) + (int64_t)h * a.x.hs + (int64_t)(begin + side) * a.x.ts;
  const T* g_in = static_cast<const T*>(a.dy.p) + (int64_t)h * a.dy.hs + (int64_t)(begin + side) * a.dy.ts;
  T* out = static_cast<T*>(a.out.p) + (int64_t)h * a.out.hs + (int64_t)(begin + side) * a.out.ts;
  const int64_t x_step = (int64_t)a.side * a.x.ts, g_step = (int64_t)a.side * a.dy.ts, step = (int64_t)a.side * a.out.ts;
  chain_wait();
  int ahead = mine ? begin + side : end, put_at = 0, take_at = 0;
  auto issue = [&]() {
    stages.issue(put_at, 0, x_in, ahead < end);
    stages.issue(put_at, 1, g_in, ahead < end);
    ahead += a.side;
    x_in += x_step;
    g_in += g_step;
    put_at = put_at + 1 == S::kDepth ? 0 : put_at + 1;
  };
#pragma unroll
  for (int i = 0; i < (S::kDepth > 1 ? S::kDepth - 1 : 1); ++i) issue();
  int32_t ahead_pos = tid < a.tile && begin + tid < end ? __ldcg(a.positions + begin + tid) : 0;
  const Turns<P> turns(a, part.paired, s_turn);
  float w[UPL][P::kElems], dw[UPL][P::kElems];
#pragma unroll
  for (int j = 0; j < UPL; ++j)
#pragma unroll
    for (int i = 0; i < P::kElems; ++i) dw[j][i] = 0.f;
  if (mine) part.load_weight(a.wq, h, w);
  for (int t0 = begin; t0 < end; t0 += a.tile) {
    const int nt = min(a.tile, end - t0);
    if (tid < nt) s_pos[tid] = ahead_pos;
    if (tid < a.tile && t0 + a.tile + tid < end) ahead_pos = __ldcg(a.positions + t0 + a.tile + tid);
    __syncthreads();
    turns.fill(a, nt, s_pos);
    __syncthreads();
    for (int base = works ? 0 : nt; base < nt; base += a.side) {
      const int t = base + side;
      const bool ok = mine && t < nt;
      typename P::Raw raw_x, raw_g;
      if constexpr (S::kDepth > 1) {
        issue();
        stages.wait();
        stages.take(take_at, 0, raw_x);
        stages.take(take_at, 1, raw_g);
        take_at = take_at + 1 == S::kDepth ? 0 : take_at + 1;
      } else {
        stages.take(0, 0, raw_x);
        stages.take(0, 1, raw_g);
        issue();
      }
      float x[UPL][P::kElems], g[UPL][P::kElems];
      part.widen(raw_x, x);
      part.widen(raw_g, g);
      const float* cs = s_turn + (ok ? t : 0) * 2 * a.turns;
      part.template turn_all<true>(cs, cs + a.turns, g);
      const float squares = part.sum(dot(x, x));
      float aw[UPL][P::kElems];  // g w
#pragma unroll
      for (int j = 0; j < UPL; ++j)
#pragma unroll
        for (int i = 0; i < P::kElems; i += 2)
          unpack2(mul2(pack2(g[j][i], g[j][i + 1]), pack2(w[j][i], w[j][i + 1])), aw[j][i], aw[j][i + 1]);
      const float along = part.sum(dot(aw, x));
      if (!ok) continue;
      const float r = rsqrtf(fmaf(squares, a.inv_d, a.wq.eps)), m = r * along * a.inv_d;
      const uint64_t r2 = pack2(r, r), m2 = pack2(-m, -m);
#pragma unroll
      for (int j = 0; j < UPL; ++j)
#pragma unroll
        for (int i = 0; i < P::kElems; i += 2) {
          const uint64_t u = mul2(pack2(x[j][i], x[j][i + 1]), r2);
          unpack2(fma2(pack2(g[j][i], g[j][i + 1]), u, pack2(dw[j][i], dw[j][i + 1])), dw[j][i], dw[j][i + 1]);
          unpack2(mul2(r2, fma2(u, m2, pack2(aw[j][i], aw[j][i + 1]))), x[j][i], x[j][i + 1]);
        }
      part.narrow(x, raw_x);
      part.put(out, raw_x);
      out += step;
    }
    __syncthreads();  // the next tile's turns come where these were read
  }
  // The CTA's sum: over its tokens side by side, and over its heads where they share the weight.
  if constexpr (S::kDepth > 1) asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  float* red = s_mem;  // [groups][d]
  if (mine) {
#pragma unroll
    for (int j = 0; j < UPL; ++j)
#pragma unroll
      for (int i = 0; i < P::kElems; ++i)
        if (part.has_element(j, i)) red[group * a.d + part.element(j, i)] = dw[j][i];
  }
  __syncthreads();
  const int heads = min(a.chunk, a.heads - (int)blockIdx.y * a.chunk);  // of this CTA
  const bool shared = a.wq.hs == 0;
  const int cols = shared ? a.d : heads * a.d;
  float* parts = shared ? a.parts + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.d
                        : a.parts + (int64_t)blockIdx.x * a.heads * a.d + (int64_t)blockIdx.y * a.chunk * a.d;
  if (a.fused) parts = red;  // (a thread's first group of its column is read before it is written)
  for (int i = tid; i < cols; i += blockDim.x) {
    float v = 0.f;
    for (int s = 0; s < a.side; ++s)
      for (int h = 0; h < (shared ? heads : 1); ++h) v += red[(s * a.chunk + h) * a.d + i];
    parts[i] = v;
  }
  if (a.fused) {
    const int ranks = gridDim.x * (shared ? gridDim.y : 1);
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    cluster_barrier();
    for (int i = rank * blockDim.x + tid; i < cols; i += ranks * blockDim.x) {
      float v = 0.f;
      for (int r = 0; r < ranks; ++r) v += of_rank(red + i, r);
      put_weight(a.dw, a.dw_type, shared ? i : (int64_t)(blockIdx.y * a.chunk + i / a.d) * a.dw_hs + i % a.d, v);
    }
    cluster_barrier();  // (no CTA ends while its sums are read)
  }
}

// The weight's gradient: the parts of each element, in order.
constexpr int kSumCols = 32, kSumRows = 32;
struct SumArgs {
  const float* parts;
  void* out;
  int64_t hs;
  int32_t n_parts, cols, d, dtype;
};
__global__ void __launch_bounds__(kSumCols * kSumRows) k_norm_weight(const __grid_constant__ SumArgs a) {
  __shared__ float s[kSumRows][kSumCols];
  chain_wait();
  const int c = blockIdx.x * kSumCols + threadIdx.x % kSumCols, row = threadIdx.x / kSumCols;
  float v = 0.f;
  if (c < a.cols)
#pragma unroll 8
    for (int p = row; p < a.n_parts; p += kSumRows) v += __ldcg(a.parts + (int64_t)p * a.cols + c);
  s[row][threadIdx.x % kSumCols] = v;
  __syncthreads();
  if (row == 0 && c < a.cols) {
#pragma unroll
    for (int i = 1; i < kSumRows; ++i) v += s[i][threadIdx.x];
    const int64_t at = (int64_t)(c / a.d) * a.hs + c % a.d;
    put_weight(a.out, a.dtype, at, v);
  }
}

struct Grid {
  int x, y, threads;
  size_t smem;
  dim3 cluster;
  int vec;  // elements of a vector, 1: one by one
  int upl;
};

// How heads and tokens are laid over lanes and CTAs.
Grid plan(NormArgs& a, int elem, bool half_layout, int vec, bool backward, int num_sms) {
  const int n = vec > 1 ? vec : 1;
  Grid g{};
  g.vec = vec;
  if (vec > 1) a.units = half_layout ? a.rot / 2 / n + (a.d - a.rot) / n : a.d / n;
  else a.units = half_layout ? a.d - a.rot / 2 : (a.d + 1) / 2;
  const auto lanes_for = [&](int upl) {
    int bits = 0;
    while ((upl << bits) < a.units) ++bits;
    return bits;
  };
  // Units of a lane: one of the half layout's, as they are 16 elements (in 32 bits 8: two where a warp is too small);
  // else two or three, whichever leaves fewer places of the lanes empty.
  if (vec <= 2) g.upl = vec == 2 && half_layout ? 4 : 8;
  else if (half_layout) g.upl = a.units > 32 ? 2 : 1;
  else g.upl = 3 << lanes_for(3) < 2 << lanes_for(2) ? 3 : 2;
  a.lane_bits = lanes_for(g.upl);
  const int pairs = vec > 1 ? (half_layout ? n : n / 2) : 1;
  a.turns = (a.rot / 2 + pairs - 1) / pairs * pairs;
  // What the copies in flight leave of the shared memory holds the turns of a tile's tokens.
  const int elements = vec > 1 ? g.upl * n * (half_layout ? 2 : 1) : 0, bytes = elements * elem * (backward ? 2 : 1);
  const Shape shape = vec > 1 ? shape_of(elements, bytes, backward) : Shape{256, backward ? 1 : 2, 1};
  const int threads = shape.threads, turn = 8 * a.turns;
  const int ring = shape.depth * bytes * threads;
  const int room = turn ? std::min(kMaxTile, (kShared - ring) / turn) : kMaxTile;
  // All heads of a token in one CTA where they fit, else equal parts of them; the rest of the CTA takes other tokens.
  const int slots = threads >> a.lane_bits, chunks = (a.heads + slots - 1) / slots;
  a.chunk = (a.heads + chunks - 1) / chunks;
  a.side = std::min(slots / a.chunk, room);
  a.by_chunk.set(a.chunk);
  g.y = (a.heads + a.chunk - 1) / a.chunk;
  g.threads = vec > 1 ? threads : ((a.side * a.chunk << a.lane_bits) + 31) / 32 * 32;
  // As many CTAs as the GPU holds at a time, with equally many rounds of tokens each; forward, several times as many where
  // that would be many rounds: they then work on neighbouring rows at any time (65,536 x 32 heads of 128 in bf16: 192 us
  // with one wave of CTAs, 173 with 32 rounds a CTA, 166 with 24, 163 with 16; the append of 70,000 tokens, which looks up
  // their places: 280, 258, 256, 262).  A little more than one wave would be two (40,000 x 8 heads: 33.5 us with 17
  // rounds, 38.3 with 16).  Element by element a CTA's first steps cost more than that gains (10,000 x 32 heads of 154
  // when this was measured: 100 us, 126 with 32 rounds).
  const int rounds = (a.n_tokens - 1) / a.side + 1, most = std::max(1, num_sms * shape.ctas / g.y);
  a.per = (rounds - 1) / std::min(rounds, most) + 1;
  const int most_rounds = a.hkv ? 24 : 16;
  if (!backward && vec > 1 && a.per > 3 * most_rounds) a.per = most_rounds;
  g.x = (rounds - 1) / a.per + 1;
  if (backward) {
    // The CTAs whose sums belong together are a cluster where few rounds are left for each: a call of 8 tokens of 32 heads
    // takes 4.5 to 5.7 us from the host (on different machines) and 3.8 in a graph, as two kernels 7.3 and 4.2; of 32 tokens,
    // which are too many rounds, 6.3 to 7.2 and 4.4.
    const int most_x = kCluster / (a.wq.hs == 0 ? g.y : 1);
    a.fused = rounds <= most_x * kClusterRounds;
    if (a.fused) {
      a.per = (rounds - 1) / std::min(rounds, most_x) + 1;
      g.x = (rounds - 1) / a.per + 1;
      g.cluster = dim3(g.x, a.wq.hs == 0 ? g.y : 1, 1);
    }
  }
  a.per *= a.side;
  a.tile = std::min(a.per, room / a.side * a.side);
  g.smem = ring + turn * a.tile;
  if (backward) g.smem = std::max(g.smem, sizeof(float) * a.side * a.chunk * a.d);
  return g;
}

// Elements of the vectors that every row is made of: 16 bytes, or two elements, where every row starts on such a
// boundary and no vector straddles the end of a head or (half layout) of the rotated halves; else one by one.
int vector_of(const NormArgs& a, int elem, bool half_layout) {
  uintptr_t at = 0;
  for (const Heads* h : {&a.x, &a.out, &a.k, &a.v, &a.dy})
    if (h->p) at |= reinterpret_cast<uintptr_t>(h->p) | (uintptr_t)(h->ts * elem) | (uintptr_t)(h->hs * elem);
  for (const int n : {16 / elem, 2})
    if (at % (n * elem) == 0 && a.d % n == 0 && (!half_layout || a.rot / 2 % n == 0)) return n;
  return 1;
}

template <class... P, class... A>
void launch(void (*kernel)(P...), const Grid& g, cudaStream_t st, A&&... args) {
  cudaLaunchAttribute at[2]{};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = g.cluster.x;
  at[1].val.clusterDim.y = g.cluster.y;
  at[1].val.clusterDim.z = g.cluster.z;
  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3(g.x, g.y);
  lc.blockDim = dim3(g.threads);
  lc.dynamicSmemBytes = g.smem;
  lc.stream = st;
  lc.attrs = at;
  lc.numAttrs = g.cluster.x * g.cluster.y > 1 ? 2 : 1;
  cudaLaunchKernelEx(&lc, kernel, static_cast<P>(args)...);
}

template <class T, int VEC, bool HALF, int UPL>
void launch_part(const NormArgs& a, const Grid& g, bool backward, cudaStream_t st) {
  if (backward) launch(k_norm_backward<T, VEC, HALF, UPL>, g, st, a);
  else launch(k_norm_rotate<T, VEC, HALF, UPL>, g, st, a);
}
template <class T>
void launch_t(const NormArgs& a, const Grid& g, bool half_layout, bool backward, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  if (g.vec == 1) return half_layout ? launch_part<T, 1, true, 8>(a, g, backward, st)
                                     : launch_part<T, 1, false, 8>(a, g, backward, st);
  if (g.vec == 2) return half_layout ? launch_part<T, 2, true, 4>(a, g, backward, st)
                                     : launch_part<T, 2, false, 8>(a, g, backward, st);
  if (!half_layout) return g.upl == 3 ? launch_part<T, VEC, false, 3>(a, g, backward, st)
                                      : launch_part<T, VEC, false, 2>(a, g, backward, st);
  if constexpr (sizeof(T) == 4)
    if (g.upl == 2) return launch_part<T, VEC, true, 2>(a, g, backward, st);
  launch_part<T, VEC, true, 1>(a, g, backward, st);
}
void launch_norm(const NormArgs& a, const Grid& g, int dtype, bool half_layout, bool backward, cudaStream_t st) {
  if (dtype == MISAT_BF16) launch_t<__nv_bfloat16>(a, g, half_layout, backward, st);
  else if (dtype == MISAT_F16) launch_t<__half>(a, g, half_layout, backward, st);
  else launch_t<float>(a, g, half_layout, backward, st);
}

bool norm_ok(const misat_head_norm* n, int dtype, int heads, int d) {
  if (!n) return false;
  const bool empty = n->head_stride != 0 && heads == 0;
  return (n->weight || empty) && (n->dtype == dtype || n->dtype == MISAT_F32) &&
         (n->head_stride == 0 || n->head_stride >= d) && n->eps > 0 && std::isfinite(n->eps) && std::isfinite(n->offset) &&
         reinterpret_cast<uintptr_t>(n->weight) % (n->dtype == MISAT_F32 ? 4 : 2) == 0;
}
HeadWeight weight_of(const misat_head_norm* n) {
  if (!n) return {};
  const int elem = n->dtype == MISAT_F32 ? 4 : 2;
  return {n->weight, n->head_stride, n->eps, n->offset, elem == 4,
          ((reinterpret_cast<uintptr_t>(n->weight) | (uintptr_t)(n->head_stride * elem)) & 15) == 0};
}

bool sizes_ok(const misat_rope* r, const misat_head_norm* norm, int32_t dtype, int32_t n_tokens, int32_t n_heads,
              int32_t head_dim) {
  return r && dtype >= MISAT_BF16 && dtype <= MISAT_F32 && n_tokens >= 0 && n_tokens <= kMaxTokens && n_heads >= 0 &&
         n_heads <= 65535 && head_dim >= r->rot && head_dim <= kMaxHead && norm_ok(norm, dtype, n_heads, head_dim);
}
NormArgs rotary_args(const misat_rope* r, const misat_head_norm* norm, int32_t n_tokens, int32_t n_heads,
                     int32_t head_dim) {
  NormArgs a{};
  a.n_tokens = n_tokens;
  a.hq = a.heads = n_heads;
  a.d = head_dim;
  a.inv_d = 1.f / (float)head_dim;
  a.rot = r->rot;
  a.freq = r->freq;
  a.attn = r->attn;
  a.wq = weight_of(norm);
  return a;
}
// Parts of the weight's gradient, and elements of one.
int64_t parts_of(const NormArgs& a, const Grid& g) { return a.fused ? 0 : a.wq.hs == 0 ? (int64_t)g.x * g.y : g.x; }
int64_t part_size(const NormArgs& a) { return a.wq.hs == 0 ? a.d : (int64_t)a.heads * a.d; }

}  // namespace

extern "C" {

int misat_norm_rotary(const misat_rope* r, const misat_head_norm* norm, int32_t dtype, int32_t n_tokens,
                      int32_t n_heads, int32_t head_dim, const void* x, int64_t x_ts, int64_t x_hs,
                      const int32_t* positions, void* out, int64_t o_ts, int64_t o_hs, void* cuda_stream) {
  if (!sizes_ok(r, norm, dtype, n_tokens, n_heads, head_dim)) return MISAT_ERR_INVALID_ARG;
  if (n_tokens == 0 || n_heads == 0) return MISAT_OK;
  const int elem = dtype == MISAT_F32 ? 4 : 2;
  if (!heads_ok(x, x_ts, x_hs, elem) || !result_ok(out, o_ts, o_hs, elem, n_tokens, n_heads) || !positions ||
      !at_elements(positions) ||
      !in_place_ok(x, x_ts, x_hs, out, o_ts, o_hs, n_tokens, n_heads) || !on_device(r->device))
    return MISAT_ERR_INVALID_ARG;
  NormArgs a = rotary_args(r, norm, n_tokens, n_heads, head_dim);
  a.x = {const_cast<void*>(x), x_ts, x_hs};
  a.out = {out, o_ts, o_hs};
  a.positions = positions;
  const bool half = r->layout == MISAT_ROPE_HALF;
  const Grid g = plan(a, elem, half, vector_of(a, elem, half), false, r->num_sms);
  launch_norm(a, g, dtype, half, false, static_cast<cudaStream_t>(cuda_stream));
  return launch_status();
}

int misat_norm_rotary_work(const misat_rope* r, const misat_head_norm* norm, int32_t dtype, int32_t n_tokens,
                           int32_t n_heads, int32_t head_dim, int64_t* bytes) {
  if (!sizes_ok(r, norm, dtype, n_tokens, n_heads, head_dim) || !bytes) return MISAT_ERR_INVALID_ARG;
  *bytes = 0;
  if (n_tokens == 0 || n_heads == 0) return MISAT_OK;
  // The largest of what they may be: it depends on the tensors' addresses.
  const int elem = dtype == MISAT_F32 ? 4 : 2;
  for (const int vec : {1, 2, 16 / elem}) {
    NormArgs a = rotary_args(r, norm, n_tokens, n_heads, head_dim);
    const bool half = r->layout == MISAT_ROPE_HALF;
    if (vec > vector_of(a, elem, half)) continue;
    const Grid g = plan(a, elem, half, vec, true, r->num_sms);
    *bytes = std::max(*bytes, parts_of(a, g) * part_size(a) * (int64_t)sizeof(float));
  }
  return MISAT_OK;
}

int misat_norm_rotary_backward(const misat_rope* r, const misat_head_norm* norm, int32_t dtype, int32_t n_tokens,
                               int32_t n_heads, int32_t head_dim, const void* x, int64_t x_ts, int64_t x_hs,
                               const void* grad, int64_t g_ts, int64_t g_hs, const int32_t* positions, void* dx,
                               int64_t dx_ts, int64_t dx_hs, void* dweight, int64_t dw_hs, void* work,
                               int64_t work_bytes, void* cuda_stream) {
  if (!sizes_ok(r, norm, dtype, n_tokens, n_heads, head_dim) ||
      (!dweight && (n_heads > 0 || norm->head_stride == 0)) || (norm->head_stride && dw_hs < head_dim) ||
      reinterpret_cast<uintptr_t>(dweight) % (norm->dtype == MISAT_F32 ? 4 : 2) || !on_device(r->device))
    return MISAT_ERR_INVALID_ARG;
  const int elem = dtype == MISAT_F32 ? 4 : 2;
  const bool none = n_tokens == 0 || n_heads == 0;
  if (!none && (!heads_ok(x, x_ts, x_hs, elem) || !heads_ok(grad, g_ts, g_hs, elem) ||
                !result_ok(dx, dx_ts, dx_hs, elem, n_tokens, n_heads) || !positions ||
                !at_elements(positions) ||
                !in_place_ok(x, x_ts, x_hs, dx, dx_ts, dx_hs, n_tokens, n_heads) ||
                !in_place_ok(grad, g_ts, g_hs, dx, dx_ts, dx_hs, n_tokens, n_heads) ||
                (reinterpret_cast<uintptr_t>(work) & 15)))
    return MISAT_ERR_INVALID_ARG;
  NormArgs a = rotary_args(r, norm, n_tokens, n_heads, head_dim);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  SumArgs s{static_cast<const float*>(work), dweight, norm->head_stride ? dw_hs : 0, 0, (int32_t)part_size(a), head_dim,
            norm->dtype};
  if (!none) {
    a.x = {const_cast<void*>(x), x_ts, x_hs};
    a.dy = {const_cast<void*>(grad), g_ts, g_hs};
    a.out = {dx, dx_ts, dx_hs};
    a.positions = positions;
    a.parts = static_cast<float*>(work);
    const bool half = r->layout == MISAT_ROPE_HALF;
    const Grid g = plan(a, elem, half, vector_of(a, elem, half), true, r->num_sms);
    s.n_parts = (int32_t)parts_of(a, g);
    if (!a.fused && (!work || work_bytes < s.n_parts * part_size(a) * (int64_t)sizeof(float)))
      return MISAT_ERR_INVALID_ARG;
    a.dw = dweight;
    a.dw_hs = dw_hs;
    a.dw_type = norm->dtype;
    launch_norm(a, g, dtype, half, true, st);
    if (a.fused) return launch_status();
  }
  if (s.cols > 0) launch_chained(k_norm_weight, (s.cols + kSumCols - 1) / kSumCols, kSumCols * kSumRows, 0, st, s);
  return launch_status();
}

int misat_kv_append_norm(misat_kv* kv, const misat_kv_batch* batch, const misat_head_norm* q_norm,
                         const misat_head_norm* k_norm, const misat_kv_draft* draft, const void* k, int64_t k_ts,
                         int64_t k_hs, const void* v, int64_t v_ts, int64_t v_hs, const void* q, int64_t q_ts,
                         int64_t q_hs, void* q_out, int64_t qo_ts, int64_t qo_hs, void* cuda_stream) {
  if (!batch_ok(kv, batch) || batch->n_tokens > kMaxTokens || (q_norm && !norm_ok(q_norm, kv->dtype, kv->hq, kv->d)) ||
      (k_norm && !norm_ok(k_norm, kv->dtype, kv->hkv, kv->d)))
    return MISAT_ERR_INVALID_ARG;
  if (batch->n_tokens == 0) return MISAT_OK;
  if (!heads_ok(k, k_ts, k_hs, 2) || !heads_ok(v, v_ts, v_hs, 2) || (draft && (!draft->depth || !at_elements(draft->depth))))
    return MISAT_ERR_INVALID_ARG;
  if (q && (!heads_ok(q, q_ts, q_hs, 2) || !result_ok(q_out, qo_ts, qo_hs, 2, batch->n_tokens, kv->hq) ||
            !in_place_ok(q, q_ts, q_hs, q_out, qo_ts, qo_hs, batch->n_tokens, kv->hq)))
    return MISAT_ERR_INVALID_ARG;
  if (!on_device(kv->device)) return MISAT_ERR_INVALID_ARG;
  NormArgs a{};
  a.n_tokens = batch->n_tokens;
  a.hq = kv->hq;
  a.hkv = kv->hkv;
  a.first = q ? 0 : kv->hq;
  a.heads = (q ? kv->hq : 0) + 2 * kv->hkv;
  a.d = kv->d;
  a.inv_d = 1.f / (float)kv->d;
  a.attn = 1.f;
  a.x = {const_cast<void*>(q), q_ts, q_hs};
  if (q) a.out = {q_out, qo_ts, qo_hs};
  a.k = {const_cast<void*>(k), k_ts, k_hs};
  a.v = {const_cast<void*>(v), v_ts, v_hs};
  a.wq = weight_of(q_norm);
  a.wk = weight_of(k_norm);
  bool half = true;
  if (kv->rope) {
    a.rot = kv->rope->rot;
    a.freq = kv->rope->freq;
    a.attn = kv->rope->attn;
    half = kv->rope->layout == MISAT_ROPE_HALF;
  }
  a.depth = draft ? draft->depth : nullptr;
  a.b = batch_view(batch);
  a.kb = kv->kb;
  a.vb = kv->vb;
  a.n_blocks = kv->n_blocks;
  a.err = kv->err;
  const Grid g = plan(a, 2, half, vector_of(a, 2, half), false, kv->num_sms);
  launch_norm(a, g, kv->dtype, half, false, static_cast<cudaStream_t>(cuda_stream));
  return launch_status();
}

}  // extern "C"
