// What the serving operators' sources share: 16-bit types, strided rows, the
// status word and the host-side argument checks.
#ifndef LUMEN_ATTN_COMMON_H
#define LUMEN_ATTN_COMMON_H

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <atomic>

#include "lumen_attn.h"

namespace lumen_attn_detail {

constexpr int kWave = 64;

// --------------------------------------------------------- 16-bit values

__device__ __forceinline__ uint16_t bits(_Float16 x) {
  return __builtin_bit_cast(uint16_t, x);
}

__device__ __forceinline__ _Float16 half_of(uint32_t x) {
  return __builtin_bit_cast(_Float16, uint16_t(x));
}

template <bool kBf16>
__device__ __forceinline__ float value(uint16_t x) {
  if (kBf16) return __builtin_bit_cast(float, uint32_t(x) << 16);
  return float(half_of(x));
}

// Rounded to nearest even.
template <bool kBf16>
__device__ __forceinline__ uint16_t rounded(float x) {
  if (kBf16) return __builtin_bit_cast(uint16_t, __bf16(x));
  return bits(_Float16(x));
}

template <bool kBf16>
__device__ __forceinline__ void unpack8(const uint4 &r, float *x) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = value<kBf16>(uint16_t(w[i]));
    x[2 * i + 1] = value<kBf16>(uint16_t(w[i] >> 16));
  }
}

template <bool kBf16>
__device__ __forceinline__ uint4 pack8(const float *x) {
  uint32_t w[4];
  for (int i = 0; i < 4; ++i)
    w[i] = uint32_t(rounded<kBf16>(x[2 * i])) |
           uint32_t(rounded<kBf16>(x[2 * i + 1])) << 16;
  return uint4{w[0], w[1], w[2], w[3]};
}

// ------------------------------------------------------------ other parts

// x of lane l and of lane l ^ kLanes (16 or 32), in the same order for both.
// (The elements are copied out before they are cast: a cast of a vector's
// element in place reads its first.)
template <int kLanes>
__device__ __forceinline__ void both(float x, float *a, float *b) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = kLanes == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false)
                              : __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t r0 = r[0], r1 = r[1];
  *a = __builtin_bit_cast(float, r0);
  *b = __builtin_bit_cast(float, r1);
}

// Starts a load of 16 bytes a lane from the lane's address into LDS, at byte
// `to` + 16 * lane (`to` the wavefront's), not to be kept in caches.  `to` goes
// through m0, which the compiler writes, since it uses m0 itself.  The load is
// counted like any load, but the compiler does not know of it: wait_loads<n> waits
// until at most the last n are still under way, and keeps reads of the LDS behind
// it.  That, unlike the builtin, lets a read wait for its own block alone.
__device__ __forceinline__ void load_to_lds(const void *from, uint32_t to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt"
               :: "{m0}"(to), "v"(from) : "memory");
}
// The same from byte `at` of the lane on, of memory at `from`, kept in caches.
__device__ __forceinline__ void load_to_lds(const void *from, uint32_t at, uint32_t to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "{m0}"(to), "v"(at), "s"(from) : "memory");
}
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" :: "i"(kLeft) : "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}
// A barrier after the wavefront's own LDS reads, with loads under way.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T *)(p))

// A value that is the same in all lanes, in scalar registers.
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return uint64_t(__builtin_amdgcn_readfirstlane(uint32_t(x))) |
         uint64_t(__builtin_amdgcn_readfirstlane(uint32_t(x >> 32))) << 32;
}

// lumen_attn_rows, typed.
struct Rows {
  uint16_t *base;
  int64_t token, head;
};

// Lowers the status word to the least code of the wavefront's lanes: one
// atomic a wavefront that has an error, none otherwise.
__device__ __forceinline__ void record_wave(int32_t *status, int err) {
  for (int code = LUMEN_ERR_TOO_MANY; code < LUMEN_OK; ++code)
    if (__any(err == code)) {
      if ((threadIdx.x & (kWave - 1)) == 0) atomicMin(status, code);
      return;
    }
}

inline bool aligned(const void *p, uintptr_t n) {
  return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0;
}

inline int check_dtype(int32_t dtype) {
  return dtype == LUMEN_ATTN_BF16 || dtype == LUMEN_ATTN_FP16
             ? LUMEN_OK
             : LUMEN_ERR_UNSUPPORTED;
}

inline int check_status(const int32_t *d_status) {
  if (!d_status) return LUMEN_ERR_INVALID_ARG;
  return aligned(d_status, 4) ? LUMEN_OK : LUMEN_ERR_MISALIGNED;
}

inline int check_rows(const lumen_attn_rows *r, int64_t tokens) {
  if (!r || r->token_stride < 0 || r->head_stride < 0)
    return LUMEN_ERR_INVALID_ARG;
  if (tokens == 0) return LUMEN_OK;
  if (!r->d_base) return LUMEN_ERR_INVALID_ARG;
  if (!aligned(r->d_base, 16) || r->token_stride % 8 || r->head_stride % 8)
    return LUMEN_ERR_MISALIGNED;
  return LUMEN_OK;
}

inline float scale_log2(float scale) { return scale * 1.44269504088896341f; }

inline int check_scale(float scale) {
  return scale > 0.0f && scale_log2(scale) < INFINITY ? LUMEN_OK : LUMEN_ERR_INVALID_ARG;
}

// The rows from token `first` on.
inline Rows rows_of(const lumen_attn_rows *r, int64_t first) {
  return Rows{static_cast<uint16_t *>(r->d_base) + first * r->token_stride,
              r->token_stride, r->head_stride};
}

// Compute units of the current device.
inline int compute_units(int *out) {
  static std::atomic<int> known[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return LUMEN_ERR_HIP;
  }
  int n = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) !=
            hipSuccess ||
        n < 1) {
      (void)hipGetLastError();
      return LUMEN_ERR_HIP;
    }
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
  }
  *out = n;
  return LUMEN_OK;
}

}  // namespace lumen_attn_detail

#endif  // LUMEN_ATTN_COMMON_H
