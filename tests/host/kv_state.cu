// What a pool keeps between calls, for a test that plants it.
#include "kv.h"

extern "C" int kv_plant(misat_kv* kv, int32_t error, unsigned arrivals) {
  const int n = kv->num_sms * 2;
  unsigned* v = new unsigned[n];
  for (int i = 0; i < n; ++i) v[i] = arrivals;
  int rc = cudaMemcpy(kv->ctr, v, n * sizeof(unsigned), cudaMemcpyHostToDevice);
  delete[] v;
  return rc ? rc : cudaMemcpy(kv->err, &error, sizeof(error), cudaMemcpyHostToDevice);
}
