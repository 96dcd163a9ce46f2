// Launch interface between the C ABI (t2v_api.hip) and the kernels of attention over a paged cache.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/t2vattn.h"
#include "t2v_paged.h"

namespace t2v {

struct PagedCall {
  const void* q;
  int64_t q_stride;
  int heads;
  const int32_t* cu;
  int64_t tokens;
  t2v_pages cache;
  float scale;
  void* out;
  float* lse;
  unsigned long long* trace;
};

// One kernel's part of a call: the sequences that it takes, its workgroups, and its place in the workspace.
struct PagedPart {
  PagedClass cls;
  bool few;          // the kernel of 32-row tiles, or that of 128
  int shares;        // workgroups
  int64_t at;        // bytes into the workspace
};
int paged_tile_rows(bool few);
// The kernel's workgroups on a GPU of ncu CUs.
int paged_workgroups(bool few, int head_dim, int ncu);
int paged_least_share(bool few);  // keys
int64_t paged_part_bytes(const PagedPart& p, int head_dim);

hipError_t launch_paged_fwd(const PagedCall& c, const PagedPart& p, void* ws, hipStream_t s);
hipError_t launch_paged_join(const PagedCall& c, const PagedPart* parts, int n, void* ws, hipStream_t s);

#if T2V_CHECKED
hipError_t paged_fwd_check_take(unsigned int* rec, unsigned int canary);
#endif

}  // namespace t2v
