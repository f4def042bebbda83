// What the kernels around the paged cache share: row addressing, error reports and the work schedule of the attention.
#pragma once
#include <atomic>

#include "ckv_common.cuh"

namespace ckv {

constexpr int kStatusMagicWord = 63;        // word of the status section that says words 0..7 are meaningful
constexpr int kStatusMagic = 0x434b5631;
constexpr int kStatusPage = 4096;           // status code: a page or row index outside its buffer was met

// Work space of the paged calls (byte offsets from the 256-byte aligned base).
struct PagedWs {
  size_t status;   // 64 x int32 as in WsLayout
  size_t split;    // int32 [workers][4]                    what each worker left in its two slots for partial results
  size_t ml;       // float2 [workers][2][rows]             running maximum (base 2) and sum of a partial result
  size_t o;        // float [workers][2][rows][128]         its unnormalised output
  size_t total;
};
PagedWs paged_ws(const ckv_paged& pg);   // of ckv_paged_attend
PagedWs tree_ws(const ckv_paged& pg);    // of ckv_tree_attend: no less

// Records a code in the status word of a work space that no call may have cleared yet; the first code stays until it is
// read.  (Two reporters may both find a fresh work space: they then store the same kind of code.)
__device__ __forceinline__ void report_status(int* status, int code) {
  volatile int* s = status;
  if (s[kStatusMagicWord] != kStatusMagic) {
    for (int i = 1; i < 8; ++i) s[i] = 0;
    s[0] = code;
    __threadfence();
    s[kStatusMagicWord] = kStatusMagic;
  } else {
    atomicCAS(status, 0, code);
  }
}

// Tokens of unit u: clamped, so that a table of starts that is not ascending or leaves [0, T] is never followed outside it.
__device__ __forceinline__ void unit_tokens(const int32_t* starts, int u, int T, int& first, int& count) {
  first = min(max(starts[u], 0), T);
  count = max(min(starts[u + 1], T) - first, 0);
}

// A kernel's attributes are set once on each device.
struct PerDevice {
  std::atomic<bool> done[kMaxDevices] = {};
  template <class F>
  cudaError_t once(F&& f) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < kMaxDevices && done[dev].load(std::memory_order_acquire)) return cudaSuccess;
    const cudaError_t r = f();
    if (r == cudaSuccess && dev < kMaxDevices) done[dev].store(true, std::memory_order_release);
    return r;
  }
};

// Launchers (each returns cudaGetLastError() after queuing its kernels).
cudaError_t launch_rotate(const ckv_paged& pg, const ckv_rotary* rot, const void* q, const void* k, const void* v,
                          const int32_t* positions, const int32_t* starts, void* q_out, void* k_out,
                          const int32_t* lengths, const int32_t* table, void* k_pages, void* v_pages,
                          int32_t* new_lengths, int* status, cudaStream_t st);
cudaError_t launch_gather_pages(const ckv_shape& s, const ckv_params& p, const ckv_paged& pg, const void* k, const void* v,
                                const int32_t* indices, const int32_t* budgets, const int32_t* offsets,
                                const int32_t* table, void* k_pages, void* v_pages, int32_t* lengths, int* status,
                                cudaStream_t st);
cudaError_t launch_paged_attend(const ckv_paged& pg, const void* q, const void* k_pages, const void* v_pages,
                                const int32_t* table, const int32_t* lengths, const int32_t* starts, void* out, float* lse,
                                char* ws, cudaStream_t st);
constexpr int kMaxTreeWords = 32;     // of ckv_tree_masks: 1024 tokens of a unit
cudaError_t launch_tree_masks(int Nu, int T, int words, const int32_t* parents, const int32_t* starts,
                              const int32_t* first_positions, uint32_t* masks, int32_t* positions, int* status, cudaStream_t st);
cudaError_t launch_tree_attend(const ckv_paged& pg, const void* q, const void* k_pages, const void* v_pages,
                               const int32_t* table, const int32_t* lengths, const int32_t* starts, const uint32_t* tree,
                               int tree_words, void* out, float* lse, char* ws, cudaStream_t st);

}  // namespace ckv
