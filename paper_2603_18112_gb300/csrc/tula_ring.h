// What copies of rows off 16-byte boundaries bring: on the host too.
#pragma once

#ifdef __CUDACC__
#define TULA_RING_FN __host__ __device__ __forceinline__
#else
#define TULA_RING_FN inline
#endif

namespace tula {

// Bytes from the 16-byte boundary at or below an address, `off` bytes on from there, to the one at or above the end
// of `bytes` from it.
TULA_RING_FN unsigned bytes_copied(unsigned off, int bytes) { return (off + (unsigned)bytes + 15) / 16 * 16; }

// The last row that a round of `per` rows, each of `bytes` or more, may begin with to be copied so; nor may the first
// one: up to 15 bytes that come along lie before its first row and behind its last one, and there the matrix has to
// go on.  Before any round but the first there are `per` rows, which are 32 bytes or more; behind it there may be one
// row of a few.
inline long long last_round_copied(long long rows, int per, int bytes) { return rows - per - (15 + bytes - 1) / bytes; }

}  // namespace tula
