// Reads and writes of rows at any alignment, and their element types.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <tuple>

#include "internal.h"

namespace archead {
namespace rows {

// 16 / 8 bytes at any address: one load or store (global memory takes
// misaligned vector accesses on gfx950).
template <typename V>
__device__ __forceinline__ V load_any(const void* p) {
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
template <typename V>
__device__ __forceinline__ void store_any(void* p, V v) {
  __builtin_memcpy(p, &v, sizeof(V));
}

// Eight consecutive elements of a row as they lie in memory.  DT: archead_dtype.
template <int DT>
struct Eight {
  static constexpr int kBytes = DT == ARCHEAD_F32 ? 4 : 2;
  uint4 w[kBytes / 2];
  // elements [j, j + 8) of a row of n elements at p; those past n are `fill`
  // (bits of an element)
  __device__ __forceinline__ void load(const uint8_t* p, int64_t j, int64_t n, uint32_t fill) {
    const uint8_t* q = p + j * kBytes;
    if (j + 8 <= n) {
      w[0] = load_any<uint4>(q);
      if constexpr (kBytes == 4) w[1] = load_any<uint4>(q + 16);
      return;
    }
    uint32_t d[2 * kBytes];
#pragma unroll
    for (int i = 0; i < 2 * kBytes; ++i) d[i] = kBytes == 4 ? fill : fill * 0x10001u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (j + i >= n) continue;
      if constexpr (kBytes == 4) {
        d[i] = *reinterpret_cast<const uint32_t*>(q + 4 * i);
      } else {
        const uint32_t h = *reinterpret_cast<const uint16_t*>(q + 2 * i);
        d[i / 2] = i & 1 ? (d[i / 2] & 0xffffu) | h << 16 : (d[i / 2] & 0xffff0000u) | h;
      }
    }
#pragma unroll
    for (int i = 0; i < kBytes / 2; ++i) w[i] = uint4{d[4 * i], d[4 * i + 1], d[4 * i + 2], d[4 * i + 3]};
  }
  __device__ __forceinline__ float at(int i) const {
    const uint4& u = w[kBytes == 4 ? i / 4 : 0];
    const int k = kBytes == 4 ? i % 4 : i / 2;
    const uint32_t d = k == 0 ? u.x : k == 1 ? u.y : k == 2 ? u.z : u.w;
    if constexpr (kBytes == 4) return __uint_as_float(d);
    else if constexpr (DT == ARCHEAD_BF16) return __uint_as_float(i & 1 ? d & 0xffff0000u : d << 16);
    else {
      const uint16_t h = uint16_t(i & 1 ? d >> 16 : d);
      _Float16 f;
      __builtin_memcpy(&f, &h, 2);
      return float(f);
    }
  }
};

// fn<<<grid, block, lds, s>>>(args...), its own status returned (the thread's last
// error may be another call's)
template <typename... P, typename... A>
hipError_t launch_kernel(void (*fn)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t s, const A&... args) {
  std::tuple<P...> held(args...);
  return std::apply(
      [&](P&... h) {
        void* ptrs[] = {static_cast<void*>(&h)...};
        return hipLaunchKernel(reinterpret_cast<const void*>(fn), grid, block, ptrs, lds, s);
      },
      held);
}
// the same with more than 64 KB of LDS
template <typename... P, typename... A>
hipError_t launch_kernel_lds(void (*fn)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t s, const A&... args) {
  const hipError_t e =
      hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
  return e == hipSuccess ? launch_kernel(fn, grid, block, lds, s, args...) : e;
}

inline bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline int dtype_bytes(archead_dtype t) { return t == ARCHEAD_F32 ? 4 : 2; }
inline bool float_dtype(archead_dtype t) { return t == ARCHEAD_F32 || t == ARCHEAD_BF16 || t == ARCHEAD_F16; }
inline archead_status launch_status(hipError_t e, const char* what) {
  return e == hipSuccess ? ARCHEAD_OK : fail(ARCHEAD_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace rows
}  // namespace archead
