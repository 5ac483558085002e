// Wrappers of gfx950 instructions and scheduling hints shared by the kernel files.
#pragma once
#include <atomic>

#include "common.h"

// Kernels that need more than the default 64 KiB of dynamic LDS have that limit raised once per device; `done` is the
// kernel's own mask of the devices where that has happened.
template <class F>
static hipError_t raise_dynamic_lds(std::atomic<unsigned long long>& done, int device, F* kernel, size_t bytes) {
  const unsigned long long bit = 1ull << (device & 63);
  if (device < 64 && (done.load(std::memory_order_acquire) & bit)) return hipSuccess;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == hipSuccess && device < 64) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// ------------------------------------------------------------------------------------------------
// device-only intrinsics (hipcc also parses kernels in its host pass, where these do not exist)
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ int wave_uniform(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_readfirstlane(v);
#else
  return v;
#endif
}
// 16 bytes per lane from global memory straight into LDS: lane l lands at lds_wave_base + 16 l
__device__ __forceinline__ void global_to_lds_16(const uint4* gsrc, uint4* lds_wave_base) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(gsrc, lds_wave_base, 16, 0, 0);
#else
  (void)gsrc;
  (void)lds_wave_base;
#endif
}
// scheduling hint: the next SIZE instructions of class MASK (0x008 matrix, 0x100 LDS read) form one
// group; consecutive groups are issued in the order the hints are written
template <int MASK, int SIZE>
__device__ __forceinline__ void sched_group() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_sched_group_barrier(MASK, SIZE, 0);
#endif
}
// 4 bytes per lane from global memory straight into LDS: lane l lands at lds_wave_base + 4 l
__device__ __forceinline__ void global_to_lds_4(const uint32_t* gsrc, uint32_t* lds_wave_base) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(gsrc, lds_wave_base, 4, 0, 0);
#else
  (void)gsrc;
  (void)lds_wave_base;
#endif
}
// streaming load: the line is not kept in the caches once read (weights are read once per product)
typedef unsigned int esp_u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_stream_16(const uint4* p) {
  const esp_u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const esp_u32x4*>(p));
  return uint4{v.x, v.y, v.z, v.w};
}
// 16 and 8 bytes to an address of any alignment of two, past the caches: a kernel that writes much more than the L2 holds and reads none of it again is
// up to twice as fast with them (values read back from 4 bits, 11008 x 13824: 118 -> 57 us, 6.8 TB/s)
typedef unsigned int esp_u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int esp_u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void store_stream_16(void* p, const void* v) {
  esp_u32x4_any q;
  __builtin_memcpy(&q, v, 16);
  __builtin_nontemporal_store(q, reinterpret_cast<esp_u32x4_any*>(p));
}
__device__ __forceinline__ void store_stream_8(void* p, const void* v) {
  esp_u32x2_any q;
  __builtin_memcpy(&q, v, 8);
  __builtin_nontemporal_store(q, reinterpret_cast<esp_u32x2_any*>(p));
}
__device__ __forceinline__ uint32_t load_stream_4(const uint32_t* p) { return __builtin_nontemporal_load(p); }
__device__ __forceinline__ void sched_fence() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_sched_barrier(0);
#endif
}
// NM matrix instructions with ND copies into LDS and NA LDS reads spread evenly among them: after each multiply one copy
// and a share of the reads.  A matrix instruction occupies its pipe for 16 or 32 clocks, during which the wave can issue
// other work; issued in bursts (all multiplies, then all copies, then all reads) the copies queue up at the
// vector-memory issue while the matrix pipe runs dry - measured 5-6 % slower on the prefill shapes.  READS_FIRST: the
// reads ahead of the copy in each slot (same-box comparisons: 2 % faster for the 8-wave 32x32x32 kernel, 4-8 % slower
// for the 4-wave kernel with its deeper operand read-ahead, no difference for the other 8-wave kernels).
template <int NM, int ND, int NA, bool READS_FIRST = false>
__device__ __forceinline__ void sched_spread() {
  constexpr int AP = (NA + NM - 1) / NM;
#pragma unroll
  for (int p = 0; p < NM; p++) {
    sched_group<0x008, 1>();
    if (READS_FIRST && AP > 0) sched_group<0x100, AP>();
    if (p < ND) sched_group<0x010, 1>();
    if (!READS_FIRST && AP > 0) sched_group<0x100, AP>();
  }
  if (ND > NM) sched_group<0x010, ND - NM>();
}

// 16 x 16 outputs, 32 channels: lane l = 16 g + c holds channels 8 g .. 8 g + 7 of row c (A) and of column c (B)
template <int DT>
__device__ __forceinline__ floatx4_t mfma16(uint4 a, uint4 b, floatx4_t c) {
  if (DT == ESPARSE_F16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  }
}
