// Runs a CUDA kernel's own source on the host, a block at a time: every thread is a fibre, block barriers and warp
// exchanges are where fibres wait for one another.  Enough for kernels of plain loads and stores, one block at a time (no
// clusters); PTX is taken out of the source beforehand (tests/host_cuda.py).  Test infrastructure only.
// Arrays come from `guarded`: they end (or begin) where memory that may not be touched begins, so that a read or write
// beside them ends the process.
#pragma once
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <sys/mman.h>
#include <ucontext.h>

#include <functional>
#include <vector>

#ifndef __grid_constant__
#define __grid_constant__
#endif
#undef __launch_bounds__
#define __launch_bounds__(...)
#undef __shared__
#define __shared__ static
#undef __forceinline__
#define __forceinline__ inline

namespace host_cuda {

constexpr int kMostThreads = 1024;
struct Fibre {
  ucontext_t at;
  std::vector<char> stack;
  int waits = 0;            // 0: runs, 1: for its warp, 2: for its block, 3: done
  unsigned long long value = 0, peers[32];
};
inline Fibre fibres[kMostThreads];
inline ucontext_t scheduler;
inline int now = 0;
inline std::function<void()> body;
inline void yield(int why) {
  fibres[now].waits = why;
  swapcontext(&fibres[now].at, &scheduler);
}
inline void entry() {
  body();
  fibres[now].waits = 3;
}

}  // namespace host_cuda

inline dim3 gridDim, blockDim;
inline uint3 blockIdx, threadIdx;

namespace host_cuda {

inline void run_block(int threads) {
  for (int t = 0; t < threads; ++t) {
    Fibre& f = fibres[t];
    f.stack.resize(64 << 10), f.waits = 0;
    getcontext(&f.at);
    f.at.uc_stack.ss_sp = f.stack.data(), f.at.uc_stack.ss_size = f.stack.size(), f.at.uc_link = &scheduler;
    makecontext(&f.at, entry, 0);
  }
  for (;;) {
    for (int t = 0; t < threads; ++t)
      if (fibres[t].waits == 0) now = t, threadIdx.x = t, swapcontext(&scheduler, &fibres[t].at);
    int done = 0, at_block = 0;
    bool moved = false;
    for (int w = 0; w < threads; w += 32) {
      int n = 0;
      for (int l = 0; l < 32; ++l) n += fibres[w + l].waits == 1, done += fibres[w + l].waits == 3, at_block += fibres[w + l].waits == 2;
      if (n == 32) {        // all of the warp are at an exchange
        for (int l = 0; l < 32; ++l)
          for (int k = 0; k < 32; ++k) fibres[w + l].peers[k] = fibres[w + k].value;
        for (int l = 0; l < 32; ++l) fibres[w + l].waits = 0;
        moved = true;
      }
    }
    if (done == threads) return;
    if (at_block && done + at_block == threads) {
      for (int t = 0; t < threads; ++t)
        if (fibres[t].waits == 2) fibres[t].waits = 0;
      moved = true;
    }
    if (!moved) fprintf(stderr, "threads wait for others that never come\n"), exit(3);
  }
}
inline const unsigned long long* exchange(unsigned mask, unsigned long long value) {
  if (mask != 0xffffffffu) fprintf(stderr, "exchanges of part of a warp are not covered\n"), exit(3);
  fibres[now].value = value;
  yield(1);
  return fibres[now].peers;
}

// An array that ends where memory that may not be touched begins (or begins where such memory ends).
inline void* guarded(size_t bytes, bool at_end = true) {
  const size_t page = 4096, guard = 16 << 20, room = (bytes + page - 1) / page * page;
  char* p = (char*)mmap(nullptr, room + 2 * guard, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
  if (p == MAP_FAILED || mprotect(p + guard, room, PROT_READ | PROT_WRITE)) perror("mmap"), exit(3);
  return p + guard + (at_end ? room - bytes : 0);
}

}  // namespace host_cuda

inline void __syncthreads() { host_cuda::yield(2); }
inline void __syncwarp() { host_cuda::exchange(0xffffffffu, 0); }
inline void __threadfence() {}
inline unsigned __ballot_sync(unsigned mask, bool x) {
  const unsigned long long* all = host_cuda::exchange(mask, x);
  unsigned r = 0;
  for (int l = 0; l < 32; ++l) r |= (unsigned)(all[l] & 1) << l;
  return r;
}
inline bool __any_sync(unsigned mask, bool x) { return __ballot_sync(mask, x) != 0; }
template <class T>
T host_shuffle(unsigned mask, T x, int from) {
  static_assert(sizeof(T) <= 8, "one word");
  unsigned long long u = 0;
  memcpy(&u, &x, sizeof(T));
  u = host_cuda::exchange(mask, u)[from];
  memcpy(&x, &u, sizeof(T));
  return x;
}
template <class T>
T __shfl_sync(unsigned mask, T x, int from) { return host_shuffle(mask, x, from & 31); }
template <class T>
T __shfl_xor_sync(unsigned mask, T x, int m) { return host_shuffle(mask, x, (host_cuda::now & 31) ^ m); }
template <class T>
T __shfl_up_sync(unsigned mask, T x, int d) {
  const int lane = host_cuda::now & 31;
  return host_shuffle(mask, x, lane >= d ? lane - d : lane);
}
inline int __reduce_max_sync(unsigned mask, int x) {
  const unsigned long long* all = host_cuda::exchange(mask, (unsigned)x);
  int r = x;
  for (int l = 0; l < 32; ++l) r = (int)(unsigned)all[l] > r ? (int)(unsigned)all[l] : r;
  return r;
}
inline int __ffs(unsigned x) { return __builtin_ffs(x); }
inline float __uint_as_float(unsigned u) {
  float f;
  memcpy(&f, &u, 4);
  return f;
}
inline unsigned __float_as_uint(float f) {
  unsigned u;
  memcpy(&u, &f, 4);
  return u;
}
inline int __popc(unsigned x) { return __builtin_popcount(x); }
template <class T>
T __ldg(const T* p) { return *p; }
inline int atomicCAS(int* p, int expect, int x) {
  const int was = *p;
  if (was == expect) *p = x;
  return was;
}
inline void sincospif(float x, float* s, float* c) { *s = (float)sin(M_PI * (double)x), *c = (float)cos(M_PI * (double)x); }
template <class T>
T min(T a, T b) { return a < b ? a : b; }
template <class T>
T max(T a, T b) { return a > b ? a : b; }

template <class... P, class... A>
cudaError_t host_launch(const cudaLaunchConfig_t* cfg, void (*kernel)(P...), A... args) {
  for (unsigned i = 0; i < cfg->numAttrs; ++i)
    if (cfg->attrs[i].id == cudaLaunchAttributeClusterDimension) fprintf(stderr, "clusters are not covered\n"), exit(3);
  gridDim = cfg->gridDim, blockDim = cfg->blockDim;
  host_cuda::body = [=] { kernel(P(args)...); };
  for (unsigned y = 0; y < gridDim.y; ++y)
    for (unsigned x = 0; x < gridDim.x; ++x) {
      blockIdx.x = x, blockIdx.y = y;
      host_cuda::run_block(blockDim.x);
    }
  return cudaSuccess;
}
#define cudaLaunchKernelEx host_launch
#define cudaGetLastError() cudaSuccess
