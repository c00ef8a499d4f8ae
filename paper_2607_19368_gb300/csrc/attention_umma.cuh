// tcgen05 products of 128-byte-swizzled shared-memory tiles, and loads of tensor memory, that the
// attention kernels share.
#pragma once

#include "attention_tma.cuh"

namespace sls {

// 128-byte swizzle matrix descriptor (stride between eight-row groups 1024 bytes):
// the high word is fixed, the low word holds the address and the leading offset, the
// bytes between 64-element blocks along N for an operand whose N runs along the rows
// (unused otherwise), both in units of 16 bytes.
constexpr uint32_t AP_DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
SLS_DEV uint32_t ap_desc(uint32_t smem_addr, uint32_t lead) {
  return ((smem_addr & 0x3FFFFu) >> 4) | ((lead >> 4) << 16);
}

// D (+)= A B with A in shared memory / in tensor memory
SLS_DEV void ap_mma_ss(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .b64 x, y;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %6, 0;\n"
      " mov.b64 x, {%1, %5};\n mov.b64 y, {%2, %5};\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(AP_DESC_HI), "r"(lead)
      : "memory");
}
SLS_DEV void ap_commit(uint32_t lead, uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n"
      " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(
          smem_u32(bar)), "r"(lead)
      : "memory");
}
SLS_DEV void ap_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
SLS_DEV void ap_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

SLS_DEV void ap_ld32(uint32_t addr, float* v) {
  uint32_t* u = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]),
        "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]),
        "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]),
        "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]),
        "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(addr));
}
// Loads before this are in their registers after it; the empty statements keep
// the compiler from using a register earlier.
template <int N>
SLS_DEV void ap_wait_ld(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}
SLS_DEV float ap_max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

}  // namespace sls
