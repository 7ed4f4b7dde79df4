// Rotary positions, and the append of new tokens to a paged cache with the rotation on the way.
//
// Both are one pass over their data: a CTA takes a few tokens, finds each token's position (and,
// for the append, its slot), computes the cosines and sines of the tokens' pairs once into shared
// memory, and then moves heads: an item is one unit of one head of one token, a unit is the piece
// of a head that a thread holds -- in the half layout two vectors rot/2 apart (or one vector past
// the rotated part), in the interleaved layout one vector of whole pairs.  All heads of a token
// share its angles, so the trigonometry is 1/heads of an item.
#include <cmath>
#include <new>

#include "kv.h"

using namespace misat;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTok = 8;    // tokens of a CTA, a warp each
constexpr int kInFlight = 4;  // items a thread loads before it stores the first

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
  FastDiv units, per_tok;  // units of a head, units of heads_per_cta heads
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

// One item of a CTA: a unit of a head of a token.
struct Item {
  uint32_t tok, head, unit;  // token of the CTA; head of all heads (queries, keys, values); unit of the head
};
__device__ __forceinline__ Item item_of(const RotArgs& a, uint32_t i, int h0) {
  const uint32_t t = a.per_tok.div(i), r = i - t * a.per_tok.d, h = a.units.div(r);
  return {t, h0 + h, r - h * a.units.d};
}

template <class T, int VEC, bool HALF>
__global__ void __launch_bounds__(kThreads, 3) k_rotate(const __grid_constant__ RotArgs a) {
  extern __shared__ float2 s_turn[];  // [tok_per_cta][rot / 2]
  __shared__ int32_t s_pos[kMaxTok];
  __shared__ int64_t s_slot[kMaxTok];  // element offset of the token's row of kv head 0, -1: skip
  using V = Vec<T, VEC>;
  constexpr int W = (HALF || VEC > 1) ? VEC : 2;  // elements of a unit's vector (a scalar interleaved unit: a pair)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t0 = blockIdx.x * a.tok_per_cta;
  const int nt = min(a.tok_per_cta, a.n_tokens - t0);
  const int heads = a.hq + 2 * a.hkv;
  const int h0 = blockIdx.y * a.heads_per_cta + (a.x.p ? 0 : a.hq);
  const int nh = min(a.heads_per_cta, heads - h0);
  const int half = a.rot / 2, paired = HALF ? half / W : 0;  // paired: units of two vectors
  const int n_items = nt * nh * (int)a.units.d;
  // First element of the unit's vector, and of its second one (-1: none).
  auto element = [&](uint32_t u) { return HALF ? ((int)u < paired ? u * W : (u + paired) * W) : u * W; };
  auto second = [&](uint32_t u) -> int {
    if constexpr (HALF) return (int)u < paired ? u * W + half : -1;
    else if constexpr (VEC > 1) return -1;
    else return (int)(u * 2 + 1) < a.d ? u * 2 + 1 : -1;
  };
  auto fetch = [&](uint32_t i, V& lo, V& hi) {
    const Item it = item_of(a, i, h0);
    int h = it.head;
    const Heads& src = h < a.hq ? a.x : h < a.hq + a.hkv ? a.k : a.v;
    if (h >= a.hq) h -= h < a.hq + a.hkv ? a.hq : a.hq + a.hkv;
    const T* s = static_cast<const T*>(src.p) + (int64_t)(t0 + it.tok) * src.ts + (int64_t)h * src.hs;
    lo = *reinterpret_cast<const V*>(s + element(it.unit));
    const int e2 = second(it.unit);
    if (e2 >= 0) hi = *reinterpret_cast<const V*>(s + e2);
  };
  auto put = [&](uint32_t i, V& lo, V& hi) {
    const Item it = item_of(a, i, h0);
    int h = it.head;
    const int64_t slot = s_slot[it.tok];
    if (slot < 0) return;
    const bool turns = h < a.hq + a.hkv;
    T* o;
    if (h < a.hq) {
      o = static_cast<T*>(a.out.p) + (int64_t)(t0 + it.tok) * a.out.ts + (int64_t)h * a.out.hs;
    } else {
      h -= turns ? a.hq : a.hq + a.hkv;
      o = static_cast<T*>(turns ? a.kb : a.vb) + slot + (int64_t)h * kBlockTokens * a.d;
    }
    const int el = element(it.unit), e2 = second(it.unit);
    const float2* tr = s_turn + it.tok * half;
    if constexpr (HALF) {
      if (turns && e2 >= 0) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2 cs = tr[el + e];
          const float x = to_f(lo.e[e]), y = to_f(hi.e[e]);
          lo.e[e] = from_f<T>(x * cs.x - y * cs.y);
          hi.e[e] = from_f<T>(x * cs.y + y * cs.x);
        }
      }
    } else if constexpr (VEC > 1) {
      if (turns) {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          if (el + e < a.rot) {
            const float2 cs = tr[(el + e) / 2];
            const float x = to_f(lo.e[e]), y = to_f(lo.e[e + 1]);
            lo.e[e] = from_f<T>(x * cs.x - y * cs.y);
            lo.e[e + 1] = from_f<T>(x * cs.y + y * cs.x);
          }
        }
      }
    } else {
      if (turns && el < a.rot) {
        const float2 cs = tr[el / 2];
        const float x = to_f(lo.e[0]), y = to_f(hi.e[0]);
        lo.e[0] = from_f<T>(x * cs.x - y * cs.y);
        hi.e[0] = from_f<T>(x * cs.y + y * cs.x);
      }
    }
    *reinterpret_cast<V*>(o + el) = lo;
    if (e2 >= 0) *reinterpret_cast<V*>(o + e2) = hi;
  };

  chain_wait();
  // The first items are on their way before the positions are looked up: a CTA has one round of items
  // as a rule, and its time is two memory latencies, not three.
  V lo[kInFlight], hi[kInFlight];
#pragma unroll
  for (int j = 0; j < kInFlight; ++j)
    if (tid + j * kThreads < n_items) fetch(tid + j * kThreads, lo[j], hi[j]);
  if (a.hkv == 0) {
    if (tid < nt) {
      s_pos[tid] = __ldcg(a.positions + t0 + tid);
      s_slot[tid] = 0;
    }
  } else if (warp < nt) {
    const int t = t0 + warp;
    const int b = find_sequence(a.b.q_off, a.b.n, t, lane);
    const int begin = __ldcg(a.b.q_off + b), end = __ldcg(a.b.q_off + b + 1), len = __ldcg(a.b.kv_len + b);
    const int64_t pos = (int64_t)len - end + t;
    const bool ok = begin <= t && t < end && end - begin <= a.b.max_q && len >= end - begin && pos >= 0 &&
                    pos < a.b.stride * kBlockTokens;
    int64_t slot = -1;
    if (ok) {
      const int blk = __ldcg(a.b.table + (int64_t)b * a.b.stride + pos / kBlockTokens);
      if (blk >= 0 && blk < a.n_blocks)
        slot = ((int64_t)blk * a.hkv * kBlockTokens + pos % kBlockTokens) * a.d;
    }
    if (lane == 0) {
      if (slot < 0) set_error(a.err, MISAT_ERR_INVALID_ARG);
      s_pos[warp] = (int32_t)pos;
      s_slot[warp] = slot;
    }
  }
  __syncthreads();
  for (int i = tid; i < nt * half; i += kThreads) {
    const int t = i / half, p = i - t * half;
    s_turn[i] = turn(s_pos[t], __ldg(a.freq + p), a.attn, a.backward);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kInFlight; ++j)
    if (tid + j * kThreads < n_items) put(tid + j * kThreads, lo[j], hi[j]);
  for (int base = tid + kInFlight * kThreads; base < n_items; base += kThreads * kInFlight) {
#pragma unroll
    for (int j = 0; j < kInFlight; ++j)
      if (base + j * kThreads < n_items) fetch(base + j * kThreads, lo[j], hi[j]);
#pragma unroll
    for (int j = 0; j < kInFlight; ++j)
      if (base + j * kThreads < n_items) put(base + j * kThreads, lo[j], hi[j]);
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
  // A CTA's items: one per thread while all CTAs of that size fit the GPU at once (a step of a few
  // sequences is latency: more CTAs, each with one round of loads), else kInFlight per thread.
  const int64_t per_tok = (int64_t)heads * units;
  const int target = (int64_t)a.n_tokens * per_tok <= (int64_t)num_sms * 8 * kThreads ? kThreads : kThreads * kInFlight;
  int tok = 1, hpc = heads;
  if (per_tok >= target)
    hpc = target / units < 1 ? 1 : target / units;
  else
    tok = (int)(target / per_tok) < kMaxTok ? (int)(target / per_tok) : kMaxTok;
  a.tok_per_cta = tok;
  a.heads_per_cta = hpc;
  a.units.set(units);
  a.per_tok.set(units * hpc);
  const dim3 grid((a.n_tokens + tok - 1) / tok, (heads + hpc - 1) / hpc);
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
  if (!heads_ok(x, x_ts, x_hs, elem) || !heads_ok(out, o_ts, o_hs, elem) || !positions) return MISAT_ERR_INVALID_ARG;
  if (x == out && (x_ts != o_ts || x_hs != o_hs)) return MISAT_ERR_INVALID_ARG;
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
  if (q && (!heads_ok(q, q_ts, q_hs, 2) || !heads_ok(q_out, qo_ts, qo_hs, 2) ||
            (q == q_out && (q_ts != qo_ts || q_hs != qo_hs))))
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
