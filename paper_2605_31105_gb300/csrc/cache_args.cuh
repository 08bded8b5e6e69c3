// Validated sizes of the paged cache and the launchers behind its entry points.
#pragma once

#include "grkv_internal.cuh"

namespace grkv {

constexpr int kMaxCacheGroup = 64;   // query heads per KV head of the attention
constexpr int kMaxTree = 256;        // drafted nodes per unit
constexpr int kMaxAttendSms = 160;   // SMs whose CTAs' partial results the workspace holds
constexpr int64_t kMaxAttendTiles = (int64_t)1 << 36;   // of a call: a CTA counts its own in 32 bits

struct CacheShape {
  int U, g, t;
  int P, page, shift, cols;   // pool pages, slots per page (1 << shift), table columns
  int W, s;                   // window (0: every earlier slot) and sinks
  int dtype, simt;
  int test_timeout;           // GRKV_TEST_TIMEOUT (tests of the bounded-wait exit)
  float scale;
};

struct AttendIo {
  const void *q, *k, *v;
  const int32_t *table, *len, *qlen, *parent;   // qlen, parent may be null
  void* out;
  float* lse;   // may be null
  bool cross;   // every row sees every slot of its unit
};

// Workspace regions of the cache calls (byte offsets, 256-byte aligned).
struct CacheWs {
  size_t status;
  size_t rec;    // AttendRec [2 kMaxAttendSms]
  size_t pml;    // float2 [2 CTAs][rows] reference and sum of a partial row
  size_t po;     // float  [2 CTAs][rows][d] its unnormalised output
  size_t list;   // int    [P] free pages found by a reserve
  size_t jobs;   // int4   [U] its copies: old page, new page, slots
  size_t total;
};

size_t attend_part_rows(const CacheShape& s);      // rows of the partial results of all CTAs
int64_t attend_tiles(const CacheShape& s);         // key tiles of a call at most
cudaError_t launch_attend(const CacheShape& s, const AttendIo& io, char* ws, const CacheWs& L,
                          cudaStream_t st);

}  // namespace grkv
