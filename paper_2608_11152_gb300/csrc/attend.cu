// Attention of new tokens over a paged cache: a warp per (token, query head), one key at a time.
#include "kv.h"

using namespace misat;

namespace {

struct AttendArgs {
  KvBatch b;
  Heads q, out;
  const void* kb;
  const void* vb;
  float* lse;
  float scale;
  int32_t hq, group, hkv, d, n_blocks, window;
  int32_t* err;
};

__device__ __forceinline__ float ldf(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float ldf(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void stf(__half* p, float x) { *p = __float2half_rn(x); }
__device__ __forceinline__ void stf(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <class T>
__global__ void __launch_bounds__(128) k_attend(const __grid_constant__ AttendArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  chain_wait();
  if (id >= (int64_t)a.b.n_tokens * a.hq) return;
  const int t = (int)(id / a.hq), h = (int)(id % a.hq), hk = h / a.group;
  int lo = 0, hi = a.b.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.b.q_off[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int begin = a.b.q_off[lo], end = a.b.q_off[lo + 1], len = a.b.kv_len[lo];
  const bool ok = begin <= t && t < end && end - begin <= a.b.max_q && len >= 0 && len <= a.b.stride * kBlockTokens;
  if (!ok && lane == 0) set_error(a.err, MISAT_ERR_INVALID_ARG);
  const int64_t pos = ok ? (int64_t)len - end + t : -1;
  const int64_t from = a.window > 0 && pos + 1 > a.window ? pos + 1 - a.window : 0;
  const T* q = static_cast<const T*>(a.q.p) + (int64_t)t * a.q.ts + (int64_t)h * a.q.hs;
  float qr[4], o[4] = {0, 0, 0, 0};
  for (int i = 0; i < 4; ++i) qr[i] = lane + 32 * i < a.d ? ldf(q + lane + 32 * i) * a.scale : 0.f;
  float m = -INFINITY, l = 0.f;
  for (int64_t j = from; j <= pos; ++j) {
    const int blk = a.b.table[(int64_t)lo * a.b.stride + j / kBlockTokens];
    if (blk < 0 || blk >= a.n_blocks) {
      if (lane == 0) set_error(a.err, MISAT_ERR_INVALID_ARG);
      continue;
    }
    const int64_t at = (((int64_t)blk * a.hkv + hk) * kBlockTokens + j % kBlockTokens) * a.d;
    const T* kr = static_cast<const T*>(a.kb) + at;
    const T* vr = static_cast<const T*>(a.vb) + at;
    float s = 0.f;
    for (int i = 0; i < 4; ++i)
      if (lane + 32 * i < a.d) s += qr[i] * ldf(kr + lane + 32 * i);
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    const float mn = fmaxf(m, s);
    const float c = m == -INFINITY ? 0.f : __expf(m - mn), p = __expf(s - mn);
    l = l * c + p;
    for (int i = 0; i < 4; ++i)
      if (lane + 32 * i < a.d) o[i] = o[i] * c + p * ldf(vr + lane + 32 * i);
    m = mn;
  }
  T* out = static_cast<T*>(a.out.p) + (int64_t)t * a.out.ts + (int64_t)h * a.out.hs;
  for (int i = 0; i < 4; ++i)
    if (lane + 32 * i < a.d) stf(out + lane + 32 * i, l > 0 ? o[i] / l : 0.f);
  if (a.lse && lane == 0) a.lse[id] = l > 0 ? m + logf(l) : -INFINITY;
}

}  // namespace

namespace misat {

void launch_attend(misat_kv* kv, const KvBatch& b, const Heads& q, const Heads& out, float* lse, int32_t window,
                   cudaStream_t st) {
  AttendArgs a{b, q, out, kv->kb, kv->vb, lse, kv->scale, kv->hq, kv->hq / kv->hkv, kv->hkv, kv->d, kv->n_blocks,
               window, kv->err};
  const int64_t warps = (int64_t)b.n_tokens * kv->hq;
  const int grid = (int)((warps + 3) / 4);
  if (kv->dtype == MISAT_BF16) launch_chained(k_attend<__nv_bfloat16>, grid, 128, 0, st, a);
  else launch_chained(k_attend<__half>, grid, 128, 0, st, a);
}

}  // namespace misat
