// Internal definitions of the KV block operators: handles and the launches behind the C ABI.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

// Frequencies of a rotation as fractions of a turn in 64-bit fixed point: the angle at position p
// is (p * freq[i] mod 2^64) / 2^64 turns.  The product wraps at whole turns, so nothing is lost in the
// reduction: the angle is off by the frequency's own rounding in 64 bits (2^-54 turns times the position)
// and the cut to 32 bits (2^-32 turns), below 2^-31 turns at any position below 2^20, where a 32-bit product of
// position and frequency has lost all but a few bits.
struct misat_rope {
  int device, num_sms;
  int32_t rot, layout;
  float attn;
  uint64_t* freq;  // device [rot / 2]
};

struct misat_kv {
  int device, num_sms;
  int32_t n_blocks, hkv, hq, d, dtype, max_batch;
  float scale;
  const misat_rope* rope;
  void* kb;
  void* vb;
  // of the attention kernel: maps of the blocks, partial sums of split items, their arrivals
  decltype(&cuTensorMapEncodeTiled) encode;
  CUtensorMap map_k, map_v;
  float4* ws_o;
  float2* ws_ml;
  unsigned* ctr;
  size_t head;   // bytes of the error word and the arrivals
  int32_t* err;  // sticky; in front of the workspace above, which is one allocation with it
};

namespace misat {

// A tensor of heads; strides in elements.
struct Heads {
  void* p;
  int64_t ts, hs;
};

// Device view of a misat_kv_batch.
struct KvBatch {
  int32_t n, n_tokens, max_q;
  const int32_t* q_off;
  const int32_t* kv_len;
  const int32_t* table;
  int64_t stride;
};

constexpr int kMaxLen = 1 << 30;  // tokens of a sequence

// Checks of the arguments that both pool calls share.  A tensor's pointer has to be aligned to its
// elements; strides may be anything non-negative.
inline bool heads_ok(const void* p, int64_t ts, int64_t hs, int elem) {
  return p && ts >= 0 && hs >= 0 && (reinterpret_cast<uintptr_t>(p) % elem) == 0;
}
// A tensor that is written: no two tokens or heads in one place.
inline bool result_ok(const void* p, int64_t ts, int64_t hs, int elem, int n_tokens, int n_heads) {
  return heads_ok(p, ts, hs, elem) && (n_tokens <= 1 || ts > 0) && (n_heads <= 1 || hs > 0);
}
// A result at its input's address is the input itself: the same strides, where there is more than one to step over.
inline bool in_place_ok(const void* x, int64_t ts, int64_t hs, const void* out, int64_t o_ts, int64_t o_hs, int n_tokens,
                        int n_heads) {
  return x != out || ((n_tokens <= 1 || ts == o_ts) && (n_heads <= 1 || hs == o_hs));
}
inline bool batch_ok(const misat_kv* kv, const misat_kv_batch* b) {
  if (!kv || !b || b->n < 0 || b->n > kv->max_batch || b->n_tokens < 0 || b->max_q < 0 || b->table_stride < 0)
    return false;
  if (b->n_tokens > 0 && b->n == 0) return false;
  return b->n_tokens == 0 || (b->q_off && b->kv_len && (b->block_table || b->table_stride == 0));
}
inline KvBatch batch_view(const misat_kv_batch* b) {
  return {b->n, b->n_tokens, b->max_q, b->q_off, b->kv_len, b->block_table, b->table_stride};
}

inline bool aligned16(const Heads& h, int elem) {
  return !h.p || ((reinterpret_cast<uintptr_t>(h.p) | (uintptr_t)(h.ts * elem) | (uintptr_t)(h.hs * elem)) & 15) == 0;
}

// The handle's device is the current one.
inline bool on_device(int device) {
  int d = -1;
  return cudaGetDevice(&d) == cudaSuccess && d == device;
}

// Return code of the launches just made.
inline int launch_status() { return cudaGetLastError() == cudaSuccess ? MISAT_OK : MISAT_ERR_CUDA; }

// Maps of the attention kernel, and the pool's device memory; MISAT_OK or an error code.
int attend_prepare(misat_kv* kv);
void launch_attend(misat_kv* kv, const KvBatch& b, const Heads& q, const Heads& out, float* lse, int32_t window,
                   cudaStream_t st);

}  // namespace misat
