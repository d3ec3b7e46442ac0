// Which columns of a row a thread of the norm kernels has, and which vectors it may read whole.  Host code too, so that every
// access can be enumerated without a GPU.
#pragma once
#include <cstdint>

namespace sl {

// the columns of a thread: K pieces of E, the first of them `lead` columns before the row where rows are shifted
template <int E, int K, bool SHIFT>
struct Columns {
  uint32_t first, step, parts, d, lead;
  __host__ __device__ __forceinline__ uint32_t part(int k) const { return first + k * step; }
  __host__ __device__ __forceinline__ bool any(int k) const { return part(k) < parts; }
  // where a thread without a k-th piece loads, so that no load needs a condition
  __host__ __device__ __forceinline__ int safe(int k) const { return any(k) ? col(k) : -(SHIFT ? (int)lead : 0); }
  __host__ __device__ __forceinline__ int col(int k) const { return (int)(part(k) * E) - (SHIFT ? (int)lead : 0); }
  __host__ __device__ __forceinline__ bool whole(int k) const { return !SHIFT || (col(k) >= 0 && col(k) + E <= (int)d); }
  __host__ __device__ __forceinline__ bool has(int k, int e) const { return !SHIFT || (uint32_t)(col(k) + e) < d; }
  // the k-th piece is read as one vector, from safe(k); otherwise element by element, those of the row only
  __host__ __device__ __forceinline__ bool by_vector(int k, bool near_end) const { return !SHIFT || !near_end || (any(k) && whole(k)); }
};

template <int E, int K, bool SHIFT>
__host__ __device__ __forceinline__ Columns<E, K, SHIFT> columns_of(uint64_t row, uint32_t lane, uint32_t lanes, uint32_t d) {
  Columns<E, K, SHIFT> c;
  c.first = lane;
  c.step = lanes;
  c.d = d;
  c.lead = SHIFT ? (uint32_t)(row * d % E) : 0;
  c.parts = (d + c.lead + E - 1) / E;
  return c;
}

// A vector with the end of a row reaches up to 7 elements past it; so many rows from the last one on have fewer than 7 behind them
// (one from d = 7 on, up to seven below; rows that lie further apart leave more room).
__host__ __device__ __forceinline__ uint32_t rows_near_end(uint32_t d) { return 6 / d + 1; }
__host__ __device__ __forceinline__ bool near_array_end(uint64_t row, uint32_t n, uint32_t near) { return row + near >= n; }

}  // namespace sl
