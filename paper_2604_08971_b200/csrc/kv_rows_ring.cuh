// The ring of tiles of serving attention for few rows: how many, and why.  Without CUDA in it, so that a CPU test can compile it and walk the ring.
//
// One warp fills the slots in order, kRowsWarps others take the tiles in turn: tile n lies in slot n % stages and is warp n % kRowsWarps's.  A wait
// on a barrier knows its phase by one bit, so that a warp must never come to a slot whose phase before the one it waits for is still open:
// the wait would end at once, on the tile of before.  Copies land in any order, so what a warp knows to have landed is what it took itself.  With
// a multiple of kRowsWarps slots every slot is one warp's, and the phase before is one that it has waited for.  (Six slots for four
// warps let tile n's warp come while tile n - 6 was on its way, once copies came from memory rather than the L2: on
// 17 samples of 7961 keys at d 128 results were wrong and waits ran out.)
#pragma once

constexpr int kRowsWarps = 4, kRowsKeys = 32;      // warps that compute; keys of a tile

// Tiles of the ring, by the bytes of one (of K or V): two for each warp, three where they are small; one where 16-bit rows of 128 make them 8 KB,
// so that two blocks fit an SM (a row of 64 samples, 16 heads on 4, on 7874 keys, 1032 MB: 174 us; eight slots and one block 223; two rows of
// 64 samples, 14 heads on 2, on 2979 keys, 195 MB: 59 against 53).
constexpr int rows_stages(int tile_bytes) { return (tile_bytes > 4096 ? 1 : tile_bytes > 2048 ? 2 : 3) * kRowsWarps; }
