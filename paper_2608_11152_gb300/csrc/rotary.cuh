// Pieces of the kernels that rotate heads and fill tables: conversions, the turn of a pair, the sequence of a token.
#pragma once

#include "kv.h"

namespace misat {

// n / d for n * d < 2^32: m = ceil(2^32 / d) (d = 1 would need 33 bits and is the identity).
struct FastDiv {
  uint32_t d, m;
  void set(uint32_t v) {
    d = v;
    m = v > 1 ? (uint32_t)((((uint64_t)1 << 32) + v - 1) / v) : 0;
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return d == 1 ? n : __umulhi(n, m); }
};

template <class T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f(float x) { return x; }
template <>
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f(float x) { return x; }
template <>
__device__ __forceinline__ __half from_f(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f(float x) { return __float2bfloat16_rn(x); }

// cos and sin of (pos * freq / 2^64) turns.  The nearest quarter turn is taken off in whole
// numbers; what is left, within an eighth of a turn, goes to a 32-bit float with 24 good bits.
__device__ __forceinline__ float2 turn(int32_t pos, uint64_t freq, float attn, bool backward) {
  const uint32_t ph = (uint32_t)(((uint64_t)(int64_t)pos * freq) >> 32);
  const uint32_t quarter = (ph + 0x20000000u) >> 30;
  const int32_t rest = (int32_t)(ph - (quarter << 30));
  float s, c;
  sincospif((float)rest * 0x1p-31f, &s, &c);
  if (quarter & 1) {
    const float t = c;
    c = -s;
    s = t;
  }
  if (quarter & 2) {
    c = -c;
    s = -s;
  }
  if (backward) s = -s;
  return make_float2(c * attn, s * attn);
}

// The sequence of token t: the last b in [0, n) with q_off[b] <= t, found by a warp 32 offsets at
// a time (two rounds for 1,024 sequences; each round is one memory latency).  Bounded for
// malformed offsets: the range shrinks in every round.  many: stops where that many are left, and returns the first.
__device__ __forceinline__ int find_sequence(const int32_t* q_off, int n, int t, int lane, int many = 1) {
  int lo = 0, hi = n;  // the answer is in [lo, hi)
  while (hi - lo > many) {
    const int step = (hi - lo + 31) / 32;
    const int i = lo + lane * step;
    const bool le = i < hi && (i == lo || __ldcg(q_off + i) <= t);
    const unsigned m = __ballot_sync(0xffffffffu, le);
    const int last = 31 - __clz(m);  // lane 0 always holds
    lo += last * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// The sequence of item t of a warp's run: the last b with off[b] <= t.  A warp holds 32 offsets at a time.
struct OffsetFinder {
  const int32_t* off;
  int n, lane, base, mine;  // mine: off[base + lane]
  __device__ __forceinline__ void load(int b) {
    base = b;
    mine = base + lane <= n ? __ldcg(off + base + lane) : 0x7fffffff;
  }
  __device__ __forceinline__ OffsetFinder(const int32_t* off, int n, int t) : off(off), n(n), lane(threadIdx.x & 31) {
    load(find_sequence(off, n, t, lane, 32));
  }
  // All lanes call it, each with its item, in rising order over the lanes and the calls.  from, to:
  // off[b] and off[b + 1].
  __device__ __forceinline__ int operator()(int t) {
    int from, to;
    return operator()(t, from, to);
  }
  __device__ __forceinline__ int operator()(int t, int& from, int& to) {
    int b = -1;
    from = to = 0;
#pragma unroll 1
    while (true) {
      int lo = 0;  // the last of the 32 offsets that is at most t
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const int v = __shfl_sync(0xffffffffu, mine, lo + o);
        if (v <= t) lo += o;
      }
      const bool beyond = lo == 31 && base + 31 < n;  // the next offsets may be at most t too
      const int first = __shfl_sync(0xffffffffu, mine, lo), second = __shfl_sync(0xffffffffu, mine, min(lo + 1, 31));
      if (b < 0 && !beyond) {
        b = base + lo;
        from = first;
        to = lo < 31 ? second : __ldcg(off + min(b + 1, n));  // (b = n: an item behind the last sequence)
      }
      if (!__any_sync(0xffffffffu, b < 0)) return min(b, n - 1);
      load(base + 31);
    }
  }
};

// VEC elements of T in one access, at an address that is a multiple of their size, at most 16 bytes.
template <class T, int VEC>
struct alignas(VEC * sizeof(T)) Vec {
  T e[VEC];
};

}  // namespace misat
