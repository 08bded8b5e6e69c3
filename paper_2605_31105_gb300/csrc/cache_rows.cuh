// What the entry points and kernels that work on a cache's pages share: host checks, tables
// and their rows on the device, the status word.
#pragma once

#include <initializer_list>

#include "cache_args.cuh"

namespace grkv {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int cuda_rc(cudaError_t e) { return e == cudaSuccess ? GRKV_OK : GRKV_ERR_CUDA; }

#define GRKV_TRY(expr)              \
  do {                              \
    const int rc_ = (expr);         \
    if (rc_ != GRKV_OK) return rc_; \
  } while (0)

// Non-null, and aligned to `align` bytes: 16 for row data and the workspace (moved 16 bytes
// at a time), an element for the integer arrays, so that a slice of a table or of the
// lengths (one layer's units) can be passed as it is.
inline int check_ptrs(std::initializer_list<const void*> ptrs, uintptr_t align) {
  for (const void* p : ptrs)
    if (!p) return GRKV_ERR_INVALID_ARG;
  for (const void* p : ptrs)
    if ((uintptr_t)p & (align - 1)) return GRKV_ERR_MISALIGNED;
  return GRKV_OK;
}
// The same for a pointer that may be null.
inline int check_optional(const void* p, uintptr_t align) {
  return ((uintptr_t)p & (align - 1)) ? GRKV_ERR_MISALIGNED : GRKV_OK;
}

// Checks that every cache call makes before its own: parameters, workspace.
int cache_begin(const grkv_cache_params* p, const void* ws, size_t ws_bytes, CacheShape* s, CacheWs* L);

inline int clear_status(char* ws, const CacheWs& L, cudaStream_t st) {
  return cuda_rc(cudaMemsetAsync(ws + L.status, 0, 4, st));
}

struct Table {
  int U, cols, P, shift;
  __host__ __device__ int page() const { return 1 << shift; }
  // Length clamped to what the table can hold; a length outside sets the status.
  __device__ int clamped(int len, int* status) const {
    const int cap = cols << shift;
    if (len < 0 || len > cap) set_status(status, GRKV_ERR_INVALID_ARG);
    return min(max(len, 0), cap);
  }
};

// The status of a call whose only block writes it whole (solo), which saves the call a memset,
// or of one whose blocks add their faults to a cleared word.
struct Status {
  int* word;
  int* at;   // where faults go
  bool solo;
  __device__ Status(int* word_, int* shared, bool solo_) : word(word_), at(solo_ ? shared : word_), solo(solo_) {
    if (!solo) return;
    if (threadIdx.x == 0) *at = 0;
    __syncthreads();
  }
  __device__ void end() const {   // all threads of the block
    if (!solo) return;
    __syncthreads();
    if (threadIdx.x == 0) *word = *at;
  }
};

// The status of a call of one kernel.  `solo` blocks, up to kMaxSolo, are one cluster, of which the
// first writes the word whole, without a memset in front (a decoding step's append 3.8 us for 6.2).  More
// blocks (solo 0) add their faults to a word that a memset has cleared, or that k_clear_status clears
// while they run (launch_call).  Every thread of the block runs to end().
constexpr int kMaxSolo = 8;
struct CallStatus {
  struct Smem {
    int err, all[kMaxSolo];
  };
  int* word;
  Smem* sm;
  int solo;
  __device__ CallStatus(int* word_, Smem* sm_, int solo_) : word(word_), sm(sm_), solo(solo_) {
    if (threadIdx.x == 0) sm->err = 0;
    __syncthreads();
    // every block has started once this is waited for, in end()
    if (solo > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  }
  __device__ int* at() const { return &sm->err; }   // where faults go
  __device__ void end() const {
    __syncthreads();
    if (solo <= 1) {
      if (solo == 0) chain_wait();
      if (threadIdx.x == 0) {
        if (solo == 1) *word = sm->err;
        else if (sm->err) set_status(word, sm->err);
      }
      return;
    }
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (threadIdx.x == 0) {
      uint32_t to;   // this block's word in the first block's shared memory
      asm("mapa.shared::cluster.u32 %0, %1, 0;"
          : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(&sm->all[blockIdx.x])));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(sm->err) : "memory");
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      int err = 0;
      for (int x = 0; x < solo; ++x) err = min(err, sm->all[x]);
      *word = err;
    }
  }
};

// Clears the status word; the kernel behind it may start at once.
cudaError_t launch_clear_status(int* word, cudaStream_t st);

// Launches a kernel of `blocks` blocks (a grid of one dimension) whose last parameters are the status
// word and `solo`, for a call that moves `bytes`.  Long calls clear the word beside their kernel, 2 us less
// on the GPU (an append of 50 MB 8.6 us for 10.6) and 0.5 to 1 us more on the host, which they hide;
// short ones, which wait for the host, by a memset (trees of 1024 units 9.0 us a call of the host for 9.9).
constexpr size_t kLongCall = (size_t)16 << 20;
template <typename... Params, typename... Args>
cudaError_t launch_call(void (*kern)(Params...), int64_t blocks, int threads, size_t bytes, int* word,
                        cudaStream_t st, Args&&... args) {
  int solo = blocks <= kMaxSolo ? (int)blocks : 0;
  if (solo > 1 && !cluster_fits(solo, kern, threads, 0)) solo = 0;
  const bool beside = !solo && bytes >= kLongCall;
  if (!solo) {
    const cudaError_t e = beside ? launch_clear_status(word, st) : cudaMemsetAsync(word, 0, 4, st);
    if (e != cudaSuccess) return e;
  }
  count_launches(1);
  return launch_kernel(beside, solo, kern, dim3((unsigned)blocks), threads, 0, st, std::forward<Args>(args)...,
                       word, solo);
}

inline Table table_of(const CacheShape& s) { return Table{s.U, s.cols, s.P, s.shift}; }

struct RowMove {
  Table tb;
  int t;                     // rows per unit
  const int32_t* count;      // rows of a unit, or null: t
  const int32_t* len;        // slots of a unit
  int* status;
};

// Row index of slot `slot` of unit u in the pool; -1 (and the status) where the table has no page.
__device__ __forceinline__ long long pool_row(const Table& tb, const int32_t* table, int u,
                                              int slot, int* status) {
  const int e = table[(size_t)u * tb.cols + (slot >> tb.shift)];
  if ((unsigned)e >= (unsigned)tb.P) {
    set_status(status, GRKV_ERR_INVALID_ARG);
    return -1;
  }
  return ((long long)e << tb.shift) + (slot & (tb.page() - 1));
}
__device__ __forceinline__ int rows_of(const RowMove& m, int u) {
  if (!m.count) return m.t;
  const int n = m.count[u];
  if (n < 0 || n > m.t) set_status(m.status, GRKV_ERR_INVALID_ARG);
  return min(max(n, 0), m.t);
}

// Where row i of unit u's kept rows comes from and goes to; false (and the status) if the
// call's contract is broken there.
__device__ __forceinline__ bool kept_row(const RowMove& m, const int32_t* idx,
                                         const int32_t* table_in, int len, const int32_t* table_out,
                                         const int32_t* first, bool in_place, int u, int i,
                                         long long* from, long long* to) {
  const int cap = m.tb.cols << m.tb.shift, f = first ? first[u] : 0, src = idx[(size_t)u * m.t + i];
  const int dst = min(max(f, 0), cap) + i;
  if (src < 0 || src >= len || f < 0 || dst >= cap ||
      (in_place && src < dst)) {
    set_status(m.status, GRKV_ERR_INVALID_ARG);
    return false;
  }
  *from = pool_row(m.tb, table_in, u, src, m.status);
  *to = pool_row(m.tb, table_out, u, dst, m.status);
  return *from >= 0 && *to >= 0;
}

}  // namespace grkv
