// Helpers of the memory-bound operators: division by a launch constant, vectors of 1 to 8 elements.
#pragma once

#include "common.cuh"

// n / d for 0 <= n < 2^31 by one high product, an addition and a shift (Granlund and Montgomery 1994): with l = ceil(log2 d)
// and m = floor(2^32 (2^l - d) / d) + 1, the quotient is (high(n m) + n) >> l.
struct FastDiv {
  uint32_t d, m, l;
  FastDiv() : d(1), m(1), l(0) {}
  explicit FastDiv(uint32_t div) : d(div), l(0) {
    while (((uint64_t)1 << l) < div) ++l;
    m = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - div)) / div + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, m) + n) >> l; }
  __device__ __forceinline__ uint32_t mod(uint32_t n, uint32_t q) const { return n - q * d; }
};

// N consecutive elements of T in memory (aligned to their size up to 16 bytes), in registers as floats or as raw words.
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
  T e[N];
};
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) { return *reinterpret_cast<const Pack<T, N>*>(p); }
template <typename T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& v) { *reinterpret_cast<Pack<T, N>*>(p) = v; }

// Whether rows that start at p, ld elements of `elem` bytes apart, all start at a multiple of `bytes`.
static inline bool fax_rows_aligned(const void* p, int64_t ld, size_t elem, size_t bytes) {
  return fax_aligned(p, bytes) && (ld * (int64_t)elem) % (int64_t)bytes == 0;
}
