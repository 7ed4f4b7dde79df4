// Rotary positions, and the append of new tokens to a paged cache with the rotation on the way.
//
// Both are one pass over their data: a CTA takes a few tokens, finds each token's position (and,
// for the append, its slot) and computes the cosines and sines of the tokens' pairs once, into
// shared memory.  A thread has one unit of a head -- in the half layout two vectors rot/2 apart (or
// one vector past the rotated part), in the interleaved layout one vector of whole pairs -- of one
// token, takes the unit's cosines and sines to registers, and goes through heads of the token with
// them: all heads share the angles, so the trigonometry and the reads of shared memory are a
// fraction of an item, and the next head is one addition away.  Elements are turned in 32 bits and rounded
// once.
//
// Bound by memory: 65,536 tokens x 32 heads of 128 in bf16 take 175 us for 1.07 GB (6.1 TB/s, 0.90 of a
// plain copy), the append of 70,000 tokens with 32 + 2 x 8 heads 290 us for 1.75 GB; the same rotation in 32 bits takes 311 us
// for 2.15 GB (6.9 TB/s), and in the interleaved layout 192 and 328.  One head in flight
// per thread and five CTAs on an SM: four heads in flight with three CTAs took 297 us for the former, two
// with three 231 us.
#include <cmath>
#include <new>

#include "kv.h"

using namespace misat;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTok = 8;    // tokens of a CTA, a warp each
constexpr int kHeads = 4;     // heads of a token that a thread goes through, at least, where there are many tokens

// n / d for n * d < 2^32: m = ceil(2^32 / d) (d = 1 would need 33 bits and is the identity).
struct FastDiv {
  uint32_t d, m;
  void set(uint32_t v) {
    d = v;
    m = v > 1 ? (uint32_t)((((uint64_t)1 << 32) + v - 1) / v) : 0;
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return d == 1 ? n : __umulhi(n, m); }
};

struct RotArgs {
  int32_t n_tokens, hq, hkv, d, rot;  // hkv = 0: plain rotation of hq heads
  int32_t tok_per_cta, heads_per_cta, backward;
  int32_t units;                 // of a head
  FastDiv unit_threads, groups;  // threads of a head's units, heads of a token side by side
  const uint64_t* freq;
  float attn;
  Heads x, out, k, v;  // x: queries
  const int32_t* positions;
  KvBatch b;
  void* kb;
  void* vb;
  int32_t n_blocks;
  int32_t* err;
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
// malformed offsets: the range shrinks in every round.
__device__ __forceinline__ int find_sequence(const int32_t* q_off, int n, int t, int lane) {
  int lo = 0, hi = n;  // the answer is in [lo, hi)
  while (hi - lo > 1) {
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

// VEC elements of T at p; VEC * sizeof(T) is 16 and p aligned to it, or VEC is 1.
template <class T, int VEC>
struct alignas(VEC * sizeof(T)) Vec {
  T e[VEC];
};

template <class T, int VEC, bool HALF>
__global__ void __launch_bounds__(kThreads, HALF ? 5 : 7) k_rotate(const __grid_constant__ RotArgs a) {
  extern __shared__ float2 s_turn[];  // [tok_per_cta][rot / 2]
  __shared__ int32_t s_pos[kMaxTok];
  __shared__ int64_t s_slot[kMaxTok];  // element offset of the token's row of kv head 0, -1: skip
  using V = Vec<T, VEC>;
  constexpr bool PAIR = !HALF && VEC == 1;        // a unit is two neighbouring elements, moved one by one
  constexpr int W = PAIR ? 2 : VEC;               // elements a unit steps over
  constexpr int N = HALF ? VEC : PAIR ? 1 : VEC / 2;  // pairs of a unit
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t0 = blockIdx.x * a.tok_per_cta;
  const int nt = min(a.tok_per_cta, a.n_tokens - t0);
  const int h0 = blockIdx.y * a.heads_per_cta + (a.x.p ? 0 : a.hq);
  const int h1 = min(h0 + a.heads_per_cta, a.hq + 2 * a.hkv);
  const int half = a.rot / 2, paired = HALF ? half / W : 0;  // paired: units of two vectors
  const int slot = a.unit_threads.div(tid), tok = a.groups.div(slot), group = slot - tok * a.groups.d;
  const int u0 = tid - slot * a.unit_threads.d;
  const bool active = tok < nt;

  // First element of a unit, and of its second vector (-1: it has none).
  auto first = [&](int u) { return HALF && u >= paired ? (u + paired) * W : u * W; };
  auto second = [&](int u) {
    return HALF ? (u < paired ? u * W + half : -1) : PAIR && u * 2 + 1 < a.d ? u * 2 + 1 : -1;
  };
  auto fetch = [&](int h, int u, V& lo, V& hi) {
    const bool q = h < a.hq, k = h < a.hq + a.hkv;
    const Heads& src = q ? a.x : k ? a.k : a.v;
    const int hh = q ? h : k ? h - a.hq : h - a.hq - a.hkv;
    const T* s = static_cast<const T*>(src.p) + (int64_t)(t0 + tok) * src.ts + (int64_t)hh * src.hs;
    lo = *reinterpret_cast<const V*>(s + first(u));
    const int e2 = second(u);
    if (e2 >= 0) hi = *reinterpret_cast<const V*>(s + e2);
  };
  auto put = [&](int h, int u, const float2 (&cs)[N], V& lo, V& hi) {
    const bool q = h < a.hq, k = h < a.hq + a.hkv;
    T* o = q ? static_cast<T*>(a.out.p) + (int64_t)(t0 + tok) * a.out.ts + (int64_t)h * a.out.hs
             : static_cast<T*>(k ? a.kb : a.vb) + s_slot[tok] +
                   (int64_t)(h - a.hq - (k ? 0 : a.hkv)) * kBlockTokens * a.d;
    const int el = first(u), e2 = second(u);
    if (k && el < a.rot) {
      if constexpr (HALF || PAIR) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float x = to_f(lo.e[e]), y = to_f(hi.e[e]);
          lo.e[e] = from_f<T>(x * cs[e].x - y * cs[e].y);
          hi.e[e] = from_f<T>(x * cs[e].y + y * cs[e].x);
        }
      } else {
        auto pairs = [&](bool ends) {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            if (ends && el + 2 * e >= a.rot) continue;
            const float x = to_f(lo.e[2 * e]), y = to_f(lo.e[2 * e + 1]);
            lo.e[2 * e] = from_f<T>(x * cs[e].x - y * cs[e].y);
            lo.e[2 * e + 1] = from_f<T>(x * cs[e].y + y * cs[e].x);
          }
        };
        // A vector in which the rotated part ends keeps the rest as it is: x * 1 - y * 0 is NaN where y is
        // infinite.  The test in every vector took 315 us instead of 308 (append of 28 + 8 heads of 64).
        if (el + W <= a.rot) pairs(false);
        else pairs(true);
      }
    }
    *reinterpret_cast<V*>(o + el) = lo;
    if (e2 >= 0) *reinterpret_cast<V*>(o + e2) = hi;
  };

  chain_wait();
  // The first head is on its way before the positions are looked up.
  V lo, hi;
  const int begin = h0 + group;
  if (active && begin < h1) fetch(begin, u0, lo, hi);
  if (a.hkv == 0) {
    if (tid < nt) {
      s_pos[tid] = __ldcg(a.positions + t0 + tid);
      s_slot[tid] = 0;
    }
  } else if (warp < nt) {
    const int t = t0 + warp;
    const int b = find_sequence(a.b.q_off, a.b.n, t, lane);
    const int from = __ldcg(a.b.q_off + b), end = __ldcg(a.b.q_off + b + 1), len = __ldcg(a.b.kv_len + b);
    const int64_t pos = (int64_t)len - end + t;
    const bool ok = from <= t && t < end && end - from <= a.b.max_q && len >= end - from && pos >= 0 &&
                    len <= kMaxLen && pos < a.b.stride * kBlockTokens;
    int64_t at = -1;
    if (ok) {
      const int blk = __ldcg(a.b.table + (int64_t)b * a.b.stride + pos / kBlockTokens);
      if (blk >= 0 && blk < a.n_blocks) at = ((int64_t)blk * a.hkv * kBlockTokens + pos % kBlockTokens) * a.d;
    }
    if (lane == 0) {
      if (at < 0) set_error(a.err, MISAT_ERR_INVALID_ARG);
      s_pos[warp] = (int32_t)pos;
      s_slot[warp] = at;
    }
  }
  __syncthreads();
  for (int i = tid; i < nt * half; i += kThreads) {
    const int t = i / half, p = i - t * half;
    s_turn[i] = turn(s_pos[t], __ldg(a.freq + p), a.attn, a.backward);
  }
  __syncthreads();
  if (!active || s_slot[tok] < 0) return;
  bool loaded = true;
  for (int u = u0; u < a.units; u += a.unit_threads.d) {
    float2 cs[N];
    const int pair = HALF ? first(u) : first(u) / 2;
#pragma unroll
    for (int e = 0; e < N; ++e) cs[e] = pair + e < half ? s_turn[tok * half + pair + e] : make_float2(1.f, 0.f);
    for (int h = begin; h < h1; h += a.groups.d) {
      if (!loaded) fetch(h, u, lo, hi);
      loaded = false;
      put(h, u, cs, lo, hi);
    }
  }
}

template <class T>
void launch_rotate_t(RotArgs& a, int layout, int num_sms, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  const bool half_layout = layout == MISAT_ROPE_HALF;
  // Whole 16-byte vectors wherever every row starts on such a boundary and no vector straddles the
  // end of a head or (half layout) of the rotated halves; else element by element.
  const bool vec = aligned16(a.x, sizeof(T)) && aligned16(a.out, sizeof(T)) && aligned16(a.k, sizeof(T)) &&
                   aligned16(a.v, sizeof(T)) && a.d % VEC == 0 && (!half_layout || (a.rot / 2) % VEC == 0);
  int units;
  if (vec)
    units = half_layout ? a.rot / 2 / VEC + (a.d - a.rot) / VEC : a.d / VEC;
  else
    units = half_layout ? a.d - a.rot / 2 : (a.d + 1) / 2;
  const int heads = (a.x.p ? a.hq : 0) + 2 * a.hkv;
  // The CTA's threads beyond one head's units take other heads of the token (`groups` of them) and other
  // tokens.  One head per thread while all CTAs of that shape fit the GPU at once: a step of a few
  // sequences is latency.  Else kHeads heads or more per thread.
  const int unit_threads = units < kThreads ? units : kThreads, slots = kThreads / unit_threads;
  const bool few = (int64_t)a.n_tokens * heads * units <= (int64_t)num_sms * 8 * kThreads;
  int groups = heads;
  if (!few)
    for (groups = 1; groups * 2 * kHeads <= heads;) groups *= 2;
  if (groups > slots) groups = slots;
  int tok = slots / groups;
  if (tok > kMaxTok) tok = kMaxTok;
  const int hpc = few ? groups : heads;
  a.units = units;
  a.tok_per_cta = tok;
  a.heads_per_cta = hpc;
  a.unit_threads.set(unit_threads);
  a.groups.set(groups);
  const dim3 grid((a.n_tokens - 1) / tok + 1, (heads - 1) / hpc + 1);
  const size_t smem = sizeof(float2) * tok * (a.rot / 2);
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc{};
  lc.gridDim = grid;
  lc.blockDim = dim3(kThreads);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  lc.attrs = &at;
  lc.numAttrs = 1;
  if (vec && half_layout) cudaLaunchKernelEx(&lc, k_rotate<T, VEC, true>, a);
  else if (vec) cudaLaunchKernelEx(&lc, k_rotate<T, VEC, false>, a);
  else if (half_layout) cudaLaunchKernelEx(&lc, k_rotate<T, 1, true>, a);
  else cudaLaunchKernelEx(&lc, k_rotate<T, 1, false>, a);
}

void launch_rotate(RotArgs& a, int dtype, int layout, int num_sms, cudaStream_t st) {
  if (dtype == MISAT_BF16) launch_rotate_t<__nv_bfloat16>(a, layout, num_sms, st);
  else if (dtype == MISAT_F16) launch_rotate_t<__half>(a, layout, num_sms, st);
  else launch_rotate_t<float>(a, layout, num_sms, st);
}

}  // namespace

extern "C" {

int misat_rope_create(const misat_rope_config* c, misat_rope** out) {
  if (!c || !out) return MISAT_ERR_INVALID_ARG;
  const bool parts = c->scaling == MISAT_ROPE_SCALE_BY_PARTS;
  if (c->rot_dim < 2 || c->rot_dim > 1024 || c->rot_dim % 2 ||
      (c->layout != MISAT_ROPE_HALF && c->layout != MISAT_ROPE_INTERLEAVED) || c->scaling < 0 ||
      c->scaling > MISAT_ROPE_SCALE_BY_PARTS || !(c->base > 1) || !std::isfinite(c->base) || !(c->attn_factor > 0) ||
      !std::isfinite(c->attn_factor))
    return MISAT_ERR_INVALID_ARG;
  if (c->scaling != MISAT_ROPE_SCALE_NONE && !(c->factor > 0 && std::isfinite(c->factor)))
    return MISAT_ERR_INVALID_ARG;
  if (parts && !(c->orig_len > 0 && std::isfinite(c->orig_len) && c->beta_slow >= 0 && c->beta_fast > c->beta_slow &&
                 std::isfinite(c->beta_fast)))
    return MISAT_ERR_INVALID_ARG;
  const double tau = 6.283185307179586476925286766559;
  uint64_t freq[512];
  const int n = c->rot_dim / 2;
  for (int i = 0; i < n; ++i) {
    double f = std::pow(c->base, -2.0 * i / c->rot_dim);
    if (c->scaling == MISAT_ROPE_SCALE_LINEAR) {
      f /= c->factor;
    } else if (parts) {
      double g = (c->orig_len * f / tau - c->beta_slow) / (c->beta_fast - c->beta_slow);
      g = g < 0 ? 0 : g > 1 ? 1 : g;
      f *= g + (1 - g) / c->factor;
    }
    const double turns = f / tau;
    freq[i] = (uint64_t)std::ldexp(turns - std::floor(turns), 64);  // below 2^64: the fraction is below 1
  }
  misat_rope* r = new (std::nothrow) misat_rope{};
  if (!r) return MISAT_ERR_OOM;
  r->rot = c->rot_dim;
  r->layout = c->layout;
  r->attn = (float)c->attn_factor;
  if (cudaGetDevice(&r->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&r->num_sms, cudaDevAttrMultiProcessorCount, r->device) != cudaSuccess) {
    cudaGetLastError();
    delete r;
    return MISAT_ERR_CUDA;
  }
  if (cudaMalloc(&r->freq, sizeof(uint64_t) * n) != cudaSuccess) {
    cudaGetLastError();
    delete r;
    return MISAT_ERR_OOM;
  }
  if (cudaMemcpy(r->freq, freq, sizeof(uint64_t) * n, cudaMemcpyHostToDevice) != cudaSuccess) {
    cudaGetLastError();
    cudaFree(r->freq);
    delete r;
    return MISAT_ERR_CUDA;
  }
  *out = r;
  return MISAT_OK;
}

int misat_rope_destroy(misat_rope* r) {
  if (!r) return MISAT_ERR_INVALID_ARG;
  cudaFree(r->freq);
  delete r;
  return MISAT_OK;
}

int misat_rotary(const misat_rope* r, int32_t dtype, int32_t n_tokens, int32_t n_heads, int32_t head_dim,
                 const void* x, int64_t x_ts, int64_t x_hs, const int32_t* positions, void* out, int64_t o_ts,
                 int64_t o_hs, int32_t backward, void* cuda_stream) {
  if (!r || dtype < MISAT_BF16 || dtype > MISAT_F32 || n_tokens < 0 || n_heads < 0 || n_heads > 65535 ||
      head_dim < r->rot || head_dim > 1024)
    return MISAT_ERR_INVALID_ARG;
  if (n_tokens == 0 || n_heads == 0) return MISAT_OK;
  const int elem = dtype == MISAT_F32 ? 4 : 2;
  if (!heads_ok(x, x_ts, x_hs, elem) || !result_ok(out, o_ts, o_hs, elem, n_tokens, n_heads) || !positions)
    return MISAT_ERR_INVALID_ARG;
  if (!in_place_ok(x, x_ts, x_hs, out, o_ts, o_hs, n_tokens, n_heads)) return MISAT_ERR_INVALID_ARG;
  if (!on_device(r->device)) return MISAT_ERR_INVALID_ARG;
  RotArgs a{};
  a.n_tokens = n_tokens;
  a.hq = n_heads;
  a.d = head_dim;
  a.rot = r->rot;
  a.backward = backward != 0;
  a.freq = r->freq;
  a.attn = r->attn;
  a.x = {const_cast<void*>(x), x_ts, x_hs};
  a.out = {out, o_ts, o_hs};
  a.positions = positions;
  launch_rotate(a, dtype, r->layout, r->num_sms, static_cast<cudaStream_t>(cuda_stream));
  return launch_status();
}

int misat_kv_append(misat_kv* kv, const misat_kv_batch* batch, const void* k, int64_t k_ts, int64_t k_hs,
                    const void* v, int64_t v_ts, int64_t v_hs, const void* q, int64_t q_ts, int64_t q_hs, void* q_out,
                    int64_t qo_ts, int64_t qo_hs, void* cuda_stream) {
  if (!batch_ok(kv, batch)) return MISAT_ERR_INVALID_ARG;
  if (batch->n_tokens == 0) return MISAT_OK;
  if (!heads_ok(k, k_ts, k_hs, 2) || !heads_ok(v, v_ts, v_hs, 2)) return MISAT_ERR_INVALID_ARG;
  if (q && (!heads_ok(q, q_ts, q_hs, 2) || !result_ok(q_out, qo_ts, qo_hs, 2, batch->n_tokens, kv->hq) ||
            !in_place_ok(q, q_ts, q_hs, q_out, qo_ts, qo_hs, batch->n_tokens, kv->hq)))
    return MISAT_ERR_INVALID_ARG;
  if (!on_device(kv->device)) return MISAT_ERR_INVALID_ARG;
  RotArgs a{};
  a.n_tokens = batch->n_tokens;
  a.hq = kv->hq;
  a.hkv = kv->hkv;
  a.d = kv->d;
  a.x = {const_cast<void*>(q), q_ts, q_hs};
  if (q) a.out = {q_out, qo_ts, qo_hs};
  a.k = {const_cast<void*>(k), k_ts, k_hs};
  a.v = {const_cast<void*>(v), v_ts, v_hs};
  a.attn = 1.f;
  int layout = MISAT_ROPE_HALF;
  if (kv->rope) {
    a.rot = kv->rope->rot;
    a.freq = kv->rope->freq;
    a.attn = kv->rope->attn;
    layout = kv->rope->layout;
  }
  a.b = batch_view(batch);
  a.kb = kv->kb;
  a.vb = kv->vb;
  a.n_blocks = kv->n_blocks;
  a.err = kv->err;
  launch_rotate(a, kv->dtype, layout, kv->num_sms, static_cast<cudaStream_t>(cuda_stream));
  return launch_status();
}

}  // extern "C"
