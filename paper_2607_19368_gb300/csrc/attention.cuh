// What the attention calls share: the kernels' view of the paged cache and of
// packed rows, and the sequence of a packed token.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace sls {

struct RowsView {
  char* data;
  int64_t token_b, head_b;  // strides in bytes
};

struct CacheView {
  char* k;
  char* v;
  int64_t page_b, slot_b, head_b;  // strides in bytes
  int64_t num_pages;
  int page_shift;                  // log2(page_size)
  int kv_heads, head_dim;
  const int32_t* table;
  int64_t table_ld;
  int max_pages;
  const int32_t* kv_lens;
  int B;
};

// Cached tokens of sequence s, cut to what its page table can hold.
SLS_DEV int64_t cache_len(const CacheView& c, int s) {
  const int64_t m = c.kv_lens[s], cap = (int64_t)c.max_pages << c.page_shift;
  return m < 0 ? 0 : (m < cap ? m : cap);
}

// Packed rows [q0, q1) of sequence s, cut to [0, T).
SLS_DEV void seq_rows(const int32_t* cu, int s, int64_t T, int64_t& q0, int64_t& q1) {
  q0 = min(max((int64_t)cu[s], (int64_t)0), T);
  q1 = min(max((int64_t)cu[s + 1], q0), T);
}

// 16-bit elements in pairs, as float32
template <typename T>
struct Half2;
template <>
struct Half2<__nv_bfloat16> {
  SLS_DEV static float2 widen(uint32_t u) {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  }
  SLS_DEV static uint32_t narrow(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <>
struct Half2<__half> {
  SLS_DEV static float2 widen(uint32_t u) {
    return __half22float2(*reinterpret_cast<const __half2*>(&u));
  }
  SLS_DEV static uint32_t narrow(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

template <typename T>
SLS_DEV void widen8(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = Half2<T>::widen(w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

template <typename T>
SLS_DEV uint4 narrow8(const float (&x)[8]) {
  return make_uint4(Half2<T>::narrow(x[0], x[1]), Half2<T>::narrow(x[2], x[3]),
                    Half2<T>::narrow(x[4], x[5]), Half2<T>::narrow(x[6], x[7]));
}

// The attention launches overlap their edges: each may start its preamble before what is
// ahead of it in the stream has finished, and every thread of it waits until then
// (at_wait_ahead) before it reads or writes global memory or leaves: what has finished
// then implies that all before it has.  The small launches let their follower start once
// all of their CTAs run (at_go); from the large ones, whose followers would wait for
// whole SMs, that costs more than it gives (8 ragged prompts 165 us, 184 with it).
SLS_DEV void at_go() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
SLS_DEV void at_wait_ahead() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
int at_launch(void (*kern)(P...), dim3 grid, int threads, size_t smem, int cluster,
              cudaStream_t stream, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  SLS_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, args...));
  SLS_LAUNCH_CHECK();
  return SLS_OK;
}

// ---- launchers ----------------------------------------------------------------
struct AppendArgs {
  RowsView q, k, v, out;
  CacheView c;
  int64_t T;
  int q_heads;
  const int32_t* cu;         // NULL: token t belongs to sequence t
  const int32_t* positions;  // NULL: the cache index
  const void* q_weight;
  const void* k_weight;
  float eps;
  const float* inv_freq;
  int pairs;
  int interleaved;
  float rope_scale;
};
int launch_qkv_append(const AppendArgs& a, int dtype, cudaStream_t stream);

struct AttnArgs {
  RowsView q, out;
  CacheView c;
  int64_t T;
  int q_heads;
  const int32_t* cu;  // NULL: token t belongs to sequence t
  int causal;
  float scale;
};
// Prefill; workspace: attention_prefill_workspace() bytes.
size_t attention_prefill_workspace(const CacheView& c, int64_t T, int q_heads);
int launch_attention_prefill(const AttnArgs& a, int dtype, void* workspace, cudaStream_t stream);
// The single-token form (cu NULL); workspace: attention_decode_workspace() bytes.
size_t attention_decode_workspace(const CacheView& c, int q_heads);
int launch_attention_decode(const AttnArgs& a, int dtype, void* workspace, cudaStream_t stream);
// Device addresses of the current device's status words, set when a device-side
// wait of the kernel gives up.
int prefill_status_word(int** word);
int decode_status_word(int** word);

}  // namespace sls
