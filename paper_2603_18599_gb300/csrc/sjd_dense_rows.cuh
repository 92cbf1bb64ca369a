// Which features of a row each thread of its group takes (sjd_dense.cu).
#pragma once

#include <cuda_runtime.h>

namespace sjd_dense_ops {

// A thread's features of a row: pieces of 8 neighbours, `step` apart, where a row
// can be accessed 16 bytes at a time (`W`). Else a warp's pieces follow one
// another and a piece's features lie 32 apart, so that a warp's accesses of single elements are side by
// side, at distances that are known beforehand.
struct Place {
  int first, step;
};
template <bool W>
__host__ __device__ __forceinline__ Place place_of(int lane, int G, int pieces) {
  return W ? Place{8 * lane, 8 * G} : Place{lane / 32 * 256 * pieces + lane % 32, 256};
}
// Feature j of piece i; whether it is one of the row's.
template <bool W>
__host__ __device__ __forceinline__ int feature(int i, int j, Place at) {
  return W ? at.first + i * at.step + j : at.first + i * 256 + j * 32;
}
template <bool W>
__host__ __device__ __forceinline__ bool is_there(int i, int j, Place at, int D) {
  return W ? feature<true>(i, 0, at) < D : i * 256 + j * 32 < D - at.first;   // (pieces are there as a whole, or not)
}

// Pieces of a thread where G of them take a row of any length, and whether a thread has
// a piece i, in loops that take several at a time: without `W` the features behind its
// last piece are the next warp's.
__host__ __device__ __forceinline__ int pieces_of(int D, int G) { return (D + 8 * G - 1) / (8 * G); }
template <bool W>
__host__ __device__ __forceinline__ bool is_mine(int i, int pieces) {
  return W || i < pieces;
}

}  // namespace sjd_dense_ops
