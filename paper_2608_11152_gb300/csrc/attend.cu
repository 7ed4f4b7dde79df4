// Attention of new tokens over a paged cache: the pool's maps and workspace, and the launch.  The kernel is in attend.cuh.
#include "attend.cuh"

namespace misat {
namespace {

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
  const int dp = kv->d > 64 ? 128 : 64;
  int rc = allow_pool<false>(kv);
  if (rc == MISAT_OK) rc = attend_tree_prepare(kv);
  if (rc != MISAT_OK) return rc;
  // Error word and arrivals (zero between calls), statistics and sums of the parts: four slots a CTA.
  const size_t slots = (size_t)kv->num_sms * 4, head = 256 + (kv->num_sms * 2 * sizeof(unsigned) + 255) / 256 * 256;
  char* p = nullptr;
  if (cudaMalloc(&p, head + slots * runs::kTile * (sizeof(float2) + dp * sizeof(float))) != cudaSuccess) return MISAT_ERR_OOM;
  kv->err = reinterpret_cast<int32_t*>(p);
  kv->ctr = reinterpret_cast<unsigned*>(p + 256);
  kv->head = head;
  kv->ws_ml = reinterpret_cast<float2*>(p + head);
  kv->ws_o = reinterpret_cast<float4*>(p + head + slots * runs::kTile * sizeof(float2));
  return cudaMemset(p, 0, head) == cudaSuccess ? MISAT_OK : MISAT_ERR_CUDA;
}

void launch_attend(misat_kv* kv, const KvBatch& b, const Heads& q, const Heads& out, float* lse, int32_t window,
                   const misat_kv_draft* draft, cudaStream_t st) {
  const int group = kv->hq / kv->hkv;
  runs::AttendArgs a{};
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
  a.tok = runs::kTile / group;
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
  if (draft) {
    a.bits = draft->bits;
    a.depth = draft->depth;
    a.words = draft->words;
    launch_attend_tree(kv, a, map_q, st);
  } else {
    launch_pool<false>(kv, a, map_q, st);
  }
}

}  // namespace misat
