// Element types of the operators around the convolutions (group norm, adapters, distillation): vectors of
// 16 bytes at any element's address, to and from 32-bit floats.
#pragma once
#include "sfc_device.hpp"

namespace sfc {

typedef __bf16 bf16;
typedef _Float16 f16;

// Elements in 16 bytes, which is what a lane loads and stores at once.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

// A load or store of 16 (8) bytes at an address that is aligned to its elements alone: gfx950 takes any byte
// address, and rows of odd lengths need no path of their own.
template <typename T>
using raw16 = unsigned __attribute__((ext_vector_type(4), aligned(sizeof(T))));
typedef unsigned raw4 __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ raw4 load16(const T* p) {
  return *reinterpret_cast<const raw16<T>*>(p);
}

// The first `valid` elements at p, zeros behind them (none is read past the last one).
template <typename T>
__device__ __forceinline__ raw4 load_part(const T* p, int valid) {
  if (valid >= kVec<T>) return load16(p);
  raw4 r = {0u, 0u, 0u, 0u};
  constexpr int per = 4 / (int)sizeof(T);  // elements of a dword
#pragma unroll
  for (int j = 0; j < kVec<T>; ++j) {
    if (j < valid) {
      if constexpr (sizeof(T) == 4)
        r[j] = reinterpret_cast<const unsigned*>(p)[j];
      else
        r[j / per] |= (unsigned)reinterpret_cast<const unsigned short*>(p)[j] << (16 * (j % per));
    }
  }
  return r;
}

// The first `valid` elements at p and `fill` behind them; `room` elements lie between p and the end of the tensor,
// and the vector is read whole unless it ends before.
template <typename T>
__device__ __forceinline__ raw4 load_cut(const T* p, int valid, int64_t room, unsigned fill = 0u) {
  if (valid >= kVec<T>) return load16(p);
  raw4 r = room < kVec<T> ? load_part(p, valid) : load16(p);
  constexpr int per = 4 / (int)sizeof(T);
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    if constexpr (per == 1) {
      if (d >= valid) r[d] = fill;
    } else {
      if (2 * d >= valid) r[d] = fill;
      else if (2 * d + 1 >= valid) r[d] = (r[d] & 0xffffu) | (fill & 0xffff0000u);
    }
  }
  return r;
}

// Element j of a loaded vector as a float.
template <typename T>
__device__ __forceinline__ float element(const raw4& r, int j) {
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(r[j]);
  } else if constexpr (__is_same(T, bf16)) {
    const unsigned w = r[j / 2];
    return __uint_as_float(j % 2 ? w & 0xffff0000u : w << 16);
  } else {
    const unsigned short h = (unsigned short)(j % 2 ? r[j / 2] >> 16 : r[j / 2] & 0xffffu);
    return (float)__builtin_bit_cast(f16, h);
  }
}

// Floats rounded to nearest even, as T, in the dwords that are stored.  STREAM: past the caches (kStreamBytes).
template <typename T, int V, bool STREAM = false>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V], int valid) {
  typedef T pack __attribute__((ext_vector_type(V)));
  if constexpr (sizeof(T) * V == 16 || sizeof(T) * V == 8 || sizeof(T) * V == 4) {
    if (valid >= V) {
      pack o;
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = (T)v[j];
      typedef T loose __attribute__((ext_vector_type(V), aligned(sizeof(T))));
      if constexpr (STREAM) {
        // (fenced in: where both stores are arms of one branch they would be made one, which is not streamed)
        asm volatile("");
        __builtin_nontemporal_store(o, reinterpret_cast<loose*>(p));
        asm volatile("");
      } else {
        *reinterpret_cast<loose*>(p) = o;
      }
      return;
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (j < valid) p[j] = (T)v[j];
}

// Results of this many bytes and more, twice the L2 caches, are stored past them: what the next kernel reads first would
// wait for them to be written back (group norm, channels last, 32 224x224 maps of 64 channels in bfloat16: the two
// kernels 134 us, 116 stored so).  Smaller ones stay where their reader finds them.
constexpr int64_t kStreamBytes = (int64_t)64 << 20;

// Sum over the lanes of a wave whose numbers agree modulo `group` (a power of two below 64; 1: all lanes),
// in every one of them.
__device__ __forceinline__ float wave_sum(float v, int group = 1) {
  for (int m = 32; m >= group; m >>= 1) v += __shfl_xor(v, m, 64);
  return v;
}

}  // namespace sfc
