// How many tiles cover the rows or columns of the 8-bit linear layer, for every extent up to 2^31 - 1.  Without CUDA in it, so that a CPU test
// can compile it: nobody waits for a call of that size in a test.
#pragma once
#ifdef __CUDACC__
#define LINEAR_FN __host__ __device__ __forceinline__
#else
#define LINEAR_FN inline
#endif

// (tiles are powers of two, so that an index inside the last one stays below 2^31 too)
LINEAR_FN long long linear_tiles(int extent, int tile) { return ((long long)extent + tile - 1) / tile; }
