// Pools of KV blocks: the handle behind misat_kv_* and the checks of the attention call.
#include <cmath>
#include <memory>
#include <new>

#include "kv.h"

using namespace misat;

extern "C" {

int misat_kv_create(const misat_kv_config* c, misat_kv** out) {
  if (!c || !out) return MISAT_ERR_INVALID_ARG;
  if (c->n_blocks < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_q_heads < c->n_kv_heads ||
      c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > 128 || c->n_q_heads > 32768 ||
      (int64_t)c->n_blocks * c->n_kv_heads >= ((int64_t)1 << 31) || c->head_dim < 8 || c->head_dim > 128 ||
      c->head_dim % 8 || (c->dtype != MISAT_BF16 && c->dtype != MISAT_F16) || c->max_batch < 1 ||
      c->max_batch > (1 << 20) || !(c->scale >= 0) || !std::isfinite(c->scale) || !c->k_blocks || !c->v_blocks ||
      c->k_blocks == c->v_blocks ||
      ((reinterpret_cast<uintptr_t>(c->k_blocks) | reinterpret_cast<uintptr_t>(c->v_blocks)) & 15))
    return MISAT_ERR_INVALID_ARG;
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return MISAT_ERR_CUDA;
  if (c->rope && (c->rope->rot > c->head_dim || c->rope->device != device)) return MISAT_ERR_INVALID_ARG;
  misat_kv* kv = new (std::nothrow) misat_kv{};
  if (!kv) return MISAT_ERR_OOM;
  kv->device = device;
  kv->n_blocks = c->n_blocks;
  kv->hkv = c->n_kv_heads;
  kv->hq = c->n_q_heads;
  kv->d = c->head_dim;
  kv->dtype = c->dtype;
  kv->max_batch = c->max_batch;
  kv->scale = c->scale > 0 ? c->scale : (float)(1.0 / std::sqrt((double)c->head_dim));
  kv->rope = c->rope;
  kv->kb = c->k_blocks;
  kv->vb = c->v_blocks;
  int rc = MISAT_OK;
  if (cudaDeviceGetAttribute(&kv->num_sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
    rc = MISAT_ERR_CUDA;
  if (rc == MISAT_OK) rc = attend_prepare(kv);
  if (rc == MISAT_OK && cudaDeviceSynchronize() != cudaSuccess) rc = MISAT_ERR_CUDA;
  if (rc != MISAT_OK) {
    cudaGetLastError();
    misat_kv_destroy(kv);
    return rc;
  }
  *out = kv;
  return MISAT_OK;
}

int misat_kv_destroy(misat_kv* kv) {
  if (!kv) return MISAT_ERR_INVALID_ARG;
  cudaFree(kv->err);  // with the workspace behind it
  delete kv;
  return MISAT_OK;
}

int misat_kv_attend(misat_kv* kv, const misat_kv_batch* batch, const void* q, int64_t q_ts, int64_t q_hs, void* out,
                    int64_t o_ts, int64_t o_hs, float* lse, int32_t window, void* cuda_stream) {
  if (!batch_ok(kv, batch) || window < 0) return MISAT_ERR_INVALID_ARG;
  if (batch->n_tokens == 0) return MISAT_OK;
  if (!heads_ok(q, q_ts, q_hs, 2) || !result_ok(out, o_ts, o_hs, 2, batch->n_tokens, kv->hq) ||
      !in_place_ok(q, q_ts, q_hs, out, o_ts, o_hs, batch->n_tokens, kv->hq) || (reinterpret_cast<uintptr_t>(lse) & 3) || !on_device(kv->device))
    return MISAT_ERR_INVALID_ARG;
  launch_attend(kv, batch_view(batch), {const_cast<void*>(q), q_ts, q_hs}, {out, o_ts, o_hs}, lse, window,
                static_cast<cudaStream_t>(cuda_stream));
  return launch_status();
}

int misat_kv_sync(misat_kv* kv, void* cuda_stream) {
  if (!kv || !on_device(kv->device)) return MISAT_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  // The error word, and the arrivals behind it: zero between calls, unless one gave up inside or saw lengths
  // change, whatever error the word holds of an earlier call.
  std::unique_ptr<int32_t[]> head(new (std::nothrow) int32_t[kv->head / sizeof(int32_t)]);
  if (!head) return MISAT_ERR_OOM;
  if (cudaMemcpyAsync(head.get(), kv->err, kv->head, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaStreamSynchronize(st) != cudaSuccess)
    return MISAT_ERR_CUDA;
  const size_t arrivals = reinterpret_cast<char*>(kv->ctr) - reinterpret_cast<char*>(kv->err);
  int32_t err = head[0];
  for (size_t i = arrivals / sizeof(int32_t); err == 0 && i < kv->head / sizeof(int32_t); ++i)
    if (head[i]) err = MISAT_ERR_INTERNAL;
  if (err && (cudaMemsetAsync(kv->err, 0, kv->head, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess))
    return MISAT_ERR_CUDA;
  return err;
}

}  // extern "C"
