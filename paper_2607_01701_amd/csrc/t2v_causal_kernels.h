// Launch interface between the C ABI (t2v_api.hip) and the causal attention kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "t2v_causal.h"

namespace t2v {

struct CausalArgs {
  const void* q;
  const void* k;
  const void* v;
  int64_t q_stride, k_stride, v_stride;  // elements between tokens of q, k and v
  const void* dout;                      // [Tq, H, D], as out and dq
  void* out;                             // written by the forward kernels, read by the dQ kernel, as lse
  float* lse;                            // [H, Tq]
  float* delta;  // [2, H, Tq]: -Delta, then lse * log2(e); the dQ kernel's for the dK/dV kernels
  void* dq;
  void* dk;  // [Tk, Hk, D], as dv
  void* dv;
  int heads, kv_heads, head_dim;
  int64_t tq;
  float scale;
  float* partial;  // slots of cut loops
  unsigned long long* trace;
};

int causal_fwd_rows(bool narrow);
int causal_fwd_few_rows();  // the kernel for at most so many rows of a (sequence, key head)
int causal_dq_rows(bool narrow);
// dK/dV: at head_dim 128 tiles of 256 keys (wide) or 128, at 64 of 256; the loop counted in stages of so many
// queries.
int causal_dkdv_keys(int head_dim, bool wide);
int causal_dkdv_stage(int head_dim, int keys);
int causal_dkdv_wide_keys();
int causal_dkdv_wide_stage();
// Bytes of one partial slot: fp32 rows and, forward, their running maximum and sum; dK and dV.
int64_t causal_fwd_slot_bytes(int rows, int head_dim);
int64_t causal_dq_slot_bytes(int rows, int head_dim);
int64_t causal_dkdv_slot_bytes(int keys, int head_dim);

hipError_t launch_causal_fwd(const CausalArgs& a, int rows, const CausalItem* items, int n, hipStream_t s);
hipError_t launch_causal_fwd_join(const CausalArgs& a, int rows, const CausalItem* tiles, int n, hipStream_t s);
hipError_t launch_causal_dkdv(const CausalArgs& a, int keys, const CausalItem* items, int n, hipStream_t s);
hipError_t launch_causal_dkdv_wide(const CausalArgs& a, const CausalItem* items, int n, hipStream_t s);
hipError_t launch_causal_dkdv_join(const CausalArgs& a, int keys, const CausalItem* tiles, int n, hipStream_t s);
hipError_t launch_causal_dq(const CausalArgs& a, int rows, const CausalItem* items, int n, hipStream_t s);
hipError_t launch_causal_dq_join(const CausalArgs& a, int rows, const CausalItem* tiles, int n, hipStream_t s);

#if T2V_CHECKED
hipError_t causal_fwd_check_take(unsigned int* rec, unsigned int canary);
hipError_t causal_dkdv_check_take(unsigned int* rec, unsigned int canary);
hipError_t causal_dkdv_wide_check_take(unsigned int* rec, unsigned int canary);
hipError_t causal_dq_check_take(unsigned int* rec, unsigned int canary);
#endif

}  // namespace t2v
