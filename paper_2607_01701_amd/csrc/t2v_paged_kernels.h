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

int paged_few_rows();
int paged_many_rows();
int paged_least_share();  // keys
// Workgroups that a GPU of ncu CUs holds at once.
int paged_groups(int head_dim, int ncu);
// only_few: no sequence can have more than few rows.
int64_t paged_workspace(int groups, bool only_few, int head_dim);

hipError_t launch_paged_fwd(const PagedCall& c, int groups, void* ws, hipStream_t s);
hipError_t launch_paged_join(const PagedCall& c, int groups, void* ws, hipStream_t s);

#if T2V_CHECKED
hipError_t paged_fwd_check_take(unsigned int* rec, unsigned int canary);
#endif

}  // namespace t2v
