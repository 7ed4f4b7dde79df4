// The attention's deal of work (csrc/runs.cuh) on the host, a thread per CUDA thread, with lengths that change
// after a given number of reads.  Every part that a CTA would take is checked against the buffers.
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>
#include <barrier>
#include <memory>
#include <thread>
#include <vector>

#define __device__
#define __host__
#define __forceinline__ inline
#define __restrict__

struct float2 { float x, y; };
struct float4 { float x, y, z, w; };
struct CUtensorMap { char c[128]; };
struct Dim { unsigned x, y, z; };
struct Warp {
  std::barrier<> bar{32};
  int64_t slot[32];
};
static thread_local Dim threadIdx, blockIdx;
static Dim gridDim;
static thread_local Warp* warp_;
static thread_local std::barrier<>* block_;

// Two versions of every array; a read takes the second one once `switch_at` reads have been made.
struct Memory {
  std::vector<int32_t> a, b;
};
static std::vector<Memory*> g_mem;
static std::atomic<int64_t> g_reads, g_switch;
static std::atomic<int> g_outside;
static int32_t __ldcg(const int32_t* p) {
  for (Memory* m : g_mem)
    if (p >= m->a.data() && p < m->a.data() + m->a.size())
      return (g_reads.fetch_add(1) < g_switch.load() ? m->a : m->b)[p - m->a.data()];
  ++g_outside;
  return 0;
}
static void set_error(int32_t* err, int32_t code) {
  __atomic_store_n(err, code, __ATOMIC_RELAXED);
}
template <class A, class B>
static auto min(A a, B b) -> decltype(a + b) { return a < b ? a : b; }
template <class A, class B>
static auto max(A a, B b) -> decltype(a + b) { return a > b ? a : b; }
static void __syncthreads() { block_->arrive_and_wait(); }
static void __syncwarp() { warp_->bar.arrive_and_wait(); }
template <class F>
static int64_t exchange(int64_t v, F f) {
  warp_->slot[threadIdx.x & 31] = v;
  __syncwarp();
  const int64_t r = f(warp_->slot);
  __syncwarp();
  return r;
}
template <class T>
static T __shfl_xor_sync(unsigned, T v, int o) {
  return (T)exchange(v, [&](int64_t* s) { return s[(threadIdx.x & 31) ^ o]; });
}
template <class T>
static T __shfl_up_sync(unsigned, T v, int o) {
  const int lane = threadIdx.x & 31;
  return (T)exchange(v, [&](int64_t* s) { return s[lane >= o ? lane - o : lane]; });
}
static int __reduce_add_sync(unsigned, int v) {
  return (int)exchange(v, [](int64_t* s) {
    uint32_t t = 0;
    for (int i = 0; i < 32; ++i) t += (uint32_t)s[i];
    return (int64_t)(int32_t)t;
  });
}
static bool __any_sync(unsigned, bool v) {
  return exchange(v, [](int64_t* s) {
    int64_t t = 0;
    for (int i = 0; i < 32; ++i) t |= s[i];
    return t;
  });
}
static int __reduce_max_sync(unsigned, int v) {
  return (int)exchange(v, [](int64_t* s) {
    int64_t t = s[0];
    for (int i = 1; i < 32; ++i) t = s[i] > t ? s[i] : t;
    return t;
  });
}

#define MISAT_ERR_INVALID_ARG -1
#define MISAT_ERR_INTERNAL -7
namespace misat {
constexpr int kBlockTokens = 16, kMaxLen = 1 << 30;
struct Heads { void* p; int64_t ts, hs; };
struct KvBatch {
  int32_t n, n_tokens, max_q;
  const int32_t* q_off;
  const int32_t* kv_len;
  const int32_t* table;
  int64_t stride;
};

// ---- barriers and copies, for the warp that loads queries: waits that pass until one runs out ----
struct Copies {
  uint32_t bar;
  int issued;  // phases that copies were issued for
  bool flying;
};
static Copies g_copies[2];
static thread_local int t_waits;
static int g_passes;  // waits of the warp that pass
static volatile int* g_abort;
static uint32_t smem_u32(const void* p) { return (uint32_t)(uintptr_t)p; }
static bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort, int = 1) {
  if (abort == g_abort && t_waits++ >= g_passes) {
    *abort = 1;
    return false;
  }
  for (Copies& c : g_copies)  // the copies of phase k land before a wait for its parity, k & 1, returns
    if (c.bar == bar && c.issued > 0 && (((c.issued - 1) & 1) == (int)parity)) c.flying = false;
  return true;
}
static void mbar_arrive(uint32_t) {}
static void mbar_expect(uint32_t bar, uint32_t) {
  for (Copies& c : g_copies)
    if (c.bar == bar) ++c.issued;
}
static bool elect_one() { return (threadIdx.x & 31) == 0; }
static void fence_async_shared() {}
static void tma_load_3d(uint32_t, const void*, uint32_t bar, int, int, int) {
  for (Copies& c : g_copies)
    if (c.bar == bar) c.flying = true;
}
}  // namespace misat
using namespace misat;
#include "runs.cuh"
using namespace misat::runs;

namespace {

struct Check {
  int bad = 0, parts = 0;
  void part(const AttendArgs& a, const Segment& g, int64_t per) {
    ++parts;
    const int heads = g.twin ? 2 : 1;
    bool ok = g.b >= 0 && g.b < a.b.n && g.h >= 0 && g.h + heads <= a.hkv && g.nt > 0 && g.t0 >= 0 &&
              g.t0 + g.nt <= g.s.n && g.s.begin >= 0 && g.s.begin + g.s.n <= a.b.n_tokens && g.nb >= 0 &&
              (int64_t)g.k.to <= a.b.stride * kBlockTokens && (g.nb == 0 || (g.j0 >= g.k.jb && g.j0 + g.nb <= g.k.jb + g.k.blocks));
    if (!g.whole) {
      const Parts p = parts_of(a, g, per);
      ok = ok && p.first >= 0 && p.first <= (int)blockIdx.x && p.last >= p.first && p.last < (int)gridDim.x;
    }
    bad += !ok;
  }
};

}  // namespace

// One call over `n` sequences: offsets and lengths `x` before, `y` after `switch_at` reads.  Returns the parts that
// are outside the buffers or never end; *seen: the parts, *error: the sticky error.
extern "C" int deal(int n, const int32_t* off_x, const int32_t* off_y, const int32_t* len_x, const int32_t* len_y,
                    int n_tokens, int max_q, int64_t stride, int group, int hkv, int window, int grid, int64_t switch_at,
                    int* seen, int* error) {
  Memory off{{off_x, off_x + n + 1}, {off_y, off_y + n + 1}}, len{{len_x, len_x + n}, {len_y, len_y + n}};
  g_mem = {&off, &len};
  g_reads = 0;
  g_switch = switch_at;
  g_outside = 0;
  int32_t err = 0;
  AttendArgs a{};
  a.b = {n, n_tokens, max_q, off.a.data(), len.a.data(), nullptr, stride};
  a.group = group;
  a.hkv = hkv;
  a.window = window;
  a.tok = kTile / group;
  a.rows = min((int64_t)max_q * group, (int64_t)a.tok * group);
  a.small = n <= 32 && (n_tokens / (2 * a.tok) + (int64_t)n) * hkv <= grid;
  a.err = &err;
  gridDim = {(unsigned)grid, 1, 1};
  Check check;
  for (int block = 0; block < grid; ++block) {
    auto c = std::make_unique<Control>();
    memset((void*)c.get(), 0x5a, sizeof(Control));  // whatever an earlier kernel left
    std::vector<Seq> seqs(kMaxSeqs);
    std::barrier<> bar(a.small ? 32 : kThreads);
    std::vector<std::unique_ptr<Warp>> warps;
    for (int w = 0; w < kThreads / 32; ++w) warps.push_back(std::make_unique<Warp>());
    std::vector<std::thread> threads;
    const int nt = a.small ? 32 : kThreads;
    for (int t = 0; t < nt; ++t)
      threads.emplace_back([&, t] {
        threadIdx = {(unsigned)t, 0, 0};
        blockIdx = {(unsigned)block, 0, 0};
        block_ = &bar;
        warp_ = warps[t / 32].get();
        Walk w;
        const bool found = a.small ? find_run_small(a, c.get(), w) : find_run(a, c.get(), seqs.data(), w);
        if (!found || t != 0) return;
        Segment g;
        int rounds = 0;
        while (w.next(a, c->before, g)) {
          check.part(a, g, c->per);
          if (check.bad > 100 || ++rounds > 1000000) {
            ++check.bad;
            break;
          }
        }
      });
    for (auto& t : threads) t.join();
  }
  *seen = check.parts;
  *error = err;
  return check.bad + g_outside;
}

// The warp that loads queries, where its wait after `passes` others runs out; part k is a pair, one of two heads or
// neither by digit k of `kinds` (base 3), and the tiles are free when they are asked for.  Returns the tiles whose
// copies are in flight when it ends.
extern "C" int queries(int passes, int kinds) {
  auto c = std::make_unique<Control>();
  memset((void*)c.get(), 0, sizeof(Control));
  AttendArgs a{};
  a.map_q = true;
  a.group = 4;
  a.tok = 32;
  for (int k = 0; k < kSegs; ++k, kinds /= 3) {
    Segment& g = c->seg[k];
    g.nb = 3;
    g.nt = 1;
    g.pair = kinds % 3 == 1;
    g.twin = kinds % 3 == 2;
  }
  for (int i = 0; i < 2; ++i) g_copies[i] = {smem_u32(&c->q_full[i]), 0, false};
  g_passes = passes;
  g_abort = &c->abort;
  Warp warp;
  CUtensorMap map;
  std::vector<char> smem(Layout<128>::kCtl);
  std::vector<std::thread> threads;
  for (int t = 0; t < 32; ++t)
    threads.emplace_back([&, t] {
      threadIdx = {256u + t, 0, 0};
      warp_ = &warp;
      t_waits = 0;
      QueryLoader<128> ql{a, &map, smem.data(), c.get()};
      ql.run();
      __syncwarp();
      if (*g_abort) ql.drain();
    });
  for (auto& t : threads) t.join();
  return g_copies[0].flying + g_copies[1].flying;
}
