// Which warps of a block of the cache's append work together on K or V of one head of one page, and which 16-byte pieces each of their lanes
// takes.  Without CUDA in it, so that a CPU test can compile it and see every piece taken once at every size.
#pragma once
#ifdef __CUDACC__
#define APPEND_FN __host__ __device__ __forceinline__
#else
#define APPEND_FN inline
#endif

constexpr int kAppThreads = 256;
constexpr int kHold = 8;          // pieces that a lane holds in registers

// Warps of a team.  A power of two, so that teams divide the block and masks give a lane's place: the most with which a full page's
// lanes (min(page, T) rows of 2^row_shift pieces) have kHold pieces each, so that few have more than those to read twice.
APPEND_FN int append_team(int page, int T, int row_shift) {
    const int wide = ((page < T ? page : T) << row_shift) / (32 * kHold), most = wide < 1 ? 1 : wide > 8 ? 8 : wide;
    return most & 8 ? 8 : most & 4 ? 4 : most & 2 ? 2 : 1;
}
// A lane's place in its team: it takes pieces `place`, `place + 32 team`, ...
APPEND_FN int append_place(int warp, int lane, int team) { return ((warp & (team - 1)) << 5) + lane; }
