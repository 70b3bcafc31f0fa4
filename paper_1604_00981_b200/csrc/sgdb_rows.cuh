// Rows of fp32 or bf16 elements as 16-byte chunks or single elements: loads that stream
// past L1, widening to fp32, one rounding (to nearest even) on the way back.
#pragma once

#include <cuda_bf16.h>

#include "sgdb_device.cuh"

namespace sgdb {

// Programmatic dependent launch, device side.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename T>
__device__ __forceinline__ float widen(T x) {
  return GradTraits<T>::widen(x);
}

template <typename T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ BF16 narrow<BF16>(float x) {
  return BF16{__bfloat16_as_ushort(__float2bfloat16_rn(x))};
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// V elements of type T, 16 bytes, that are read and written together.
template <typename T, int V>
struct Chunk;

template <typename T>
struct Chunk16 {
  using Raw = uint4;
  static __device__ __forceinline__ Raw zero() { return make_uint4(0, 0, 0, 0); }
  static __device__ __forceinline__ void store_raw(T* p, const Raw& r) { __stcs(reinterpret_cast<uint4*>(p), r); }
};
template <>
struct Chunk<float, 4> : Chunk16<float> {
  static __device__ __forceinline__ void unpack(const uint4& r, float (&out)[4]) { GradTraits<float>::unpack(r, out); }
  static __device__ __forceinline__ uint4 pack(const float (&in)[4]) {
    return make_uint4(__float_as_uint(in[0]), __float_as_uint(in[1]), __float_as_uint(in[2]), __float_as_uint(in[3]));
  }
};
template <>
struct Chunk<BF16, 8> : Chunk16<BF16> {
  static __device__ __forceinline__ void unpack(const uint4& r, float (&out)[8]) { GradTraits<BF16>::unpack(r, out); }
  static __device__ __forceinline__ uint4 pack(const float (&in)[8]) {
    return make_uint4(pack_bf16(in[0], in[1]), pack_bf16(in[2], in[3]), pack_bf16(in[4], in[5]), pack_bf16(in[6], in[7]));
  }
};

// Copies of 16 bytes from global to shared memory that the thread itself waits for: a thread that reads only what it has
// copied needs no barrier.
__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(__cvta_generic_to_global(src)) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {  // all but the last N groups are there
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The elements first .. last - 1 of a chunk to its place p on a 16-byte boundary: the rest of the chunk belongs to others.
// From one end of the chunk on it takes at most one store of 8, 4 and 2 bytes.
template <typename T>
__device__ __forceinline__ void store_part(T* p, const uint4& v, int first, int last) {
  constexpr int V = 16 / static_cast<int>(sizeof(T));
  uint32_t* words = reinterpret_cast<uint32_t*>(p);
  if (first > 0 && last < V) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e >= first && e < last) {
        if constexpr (sizeof(T) == 4)
          words[e] = w[e];
        else
          reinterpret_cast<uint16_t*>(p)[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
      }
    return;
  }
  const bool at_end = first > 0;  // the chunk's end, or its beginning
  const int bytes = (last - first) * static_cast<int>(sizeof(T));
  if (bytes & 8) *reinterpret_cast<uint2*>(words + (at_end ? 2 : 0)) = at_end ? make_uint2(v.z, v.w) : make_uint2(v.x, v.y);
  if (bytes & 4) {
    const bool second = (bytes & 8) != 0;  // from that end
    const int at = at_end ? (second ? 1 : 3) : (second ? 2 : 0);
    words[at] = at == 0 ? v.x : at == 1 ? v.y : at == 2 ? v.z : v.w;
  }
  if (sizeof(T) == 2 && (bytes & 2)) {
    const int at = at_end ? (16 - bytes) / 4 : bytes / 4;  // the word that has the last one
    const uint32_t w = at == 0 ? v.x : at == 1 ? v.y : at == 2 ? v.z : v.w;
    reinterpret_cast<uint16_t*>(words + at)[at_end ? 1 : 0] = static_cast<uint16_t>(at_end ? w >> 16 : w);
  }
}

// Elements between the 16-byte boundary before p and p.
template <typename T>
__device__ __forceinline__ int shift_of(const T* p) {
  return static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
}

template <typename T>
constexpr int kChunk16 = 16 / static_cast<int>(sizeof(T));  // elements per 16 bytes

// One element of an array whose type is known at run time (parameters, which are few).
__device__ __forceinline__ float load_any(const void* p, int dt, long long i) {
  return dt == SGDB_BF16 ? widen<BF16>(static_cast<const BF16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_any(void* p, int dt, long long i, float v) {
  if (dt == SGDB_BF16)
    static_cast<BF16*>(p)[i] = narrow<BF16>(v);
  else
    static_cast<float*>(p)[i] = v;
}

// Two fp32 numbers in a pair of registers, and instructions that work on both, each rounded as the scalar one is.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi) {
  Pair d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ Pair pair(float both) { return pair(both, both); }
__device__ __forceinline__ float2 split(Pair a) {
  float2 d;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(a));
  return d;
}
__device__ __forceinline__ float total(Pair a) {
  const float2 d = split(a);
  return d.x + d.y;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace sgdb
