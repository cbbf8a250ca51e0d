// The order in which the blocks of a grouped product take its tiles.  Plain functions of whole numbers, so that a host program can walk through a launch.
#pragma once

#ifdef __HIP__
#define MOE_ORDER __host__ __device__ inline __attribute__((always_inline))
#else
#define MOE_ORDER inline
#endif

namespace moe {

// row tiles per band of the XCD-aware tile order of the LDS-DMA path
constexpr int kBandRows = 4;
// Launches of at most so many rounds of 256 row tiles deal them to the XCDs in short runs.  (Long runs above this line against short
// ones everywhere, training steps of d = d_ff = 4096, 8 experts, whose gate/up launch has twice the rounds given: 6.5 rounds 6475 and
// 6445 us, 7 6818 and 6846, 8 7711 and 7798, 9 8631 and 8726, 10 9576 and 9691; for launches below it see row_gemm_block.)
constexpr int kFineRounds = 6;

// The tile of block `block`, one of `total` or beyond them, in the order of band_tile.  Blocks go round the eight XCDs; a full round of 256 gives each XCD runs of
// consecutive tiles, a last one that is not full deals them one by one.
MOE_ORDER int dealt_tile(int block, int total) {
  const int rounds = total >> 8, xcd = block & 7, round = block >> 8, i = (block >> 3) & 31;
  int q = round << 8;
  if (round < rounds) q += rounds > kFineRounds && round < rounds - 1 ? (xcd << 5) + i : ((i >> 3) << 6) + (xcd << 3) + (i & 7);
  else q += (i << 3) + xcd;
  return q;
}

// Tile q: bands of kBandRows row tiles one behind the other, within a band column by column.  from_back > 0: of the first 3 * from_back bands' places every third is
// taken by one from the back (the last whole band first), the others by those from the front.  (The last band may have fewer rows.)
struct TilePlace {
  int mt, nt;
};
MOE_ORDER TilePlace band_tile(int q, int n_mt, int ntn, int from_back) {
  const int per_band = kBandRows * ntn, at = q / per_band, r = q - at * per_band, bands = n_mt / kBandRows, mixed = 3 * from_back;
  const int band = at >= bands ? at : at >= mixed ? at - from_back : at % 3 == 2 ? bands - 1 - at / 3 : at / 3 * 2 + at % 3;
  const int left = n_mt - band * kBandRows, high = left < kBandRows ? left : kBandRows;
  return {band * kBandRows + r % high, r / high};
}

// A product of one group in tiles of one height, those of a last round that is not full cut into `tail` lower ones: tile q >= total for blocks beyond.
struct CutTile {
  int q, piece, pieces;
};
MOE_ORDER CutTile cut_tile(int block, int total, int tail) {
  const int full = total >> 8 << 8;
  if (block < full) return {dealt_tile(block, total), 0, 1};
  return {full + (block - full) / tail, (block - full) % tail, tail};
}
MOE_ORDER int cut_tile_blocks(int total, int tail) {
  const int full = total >> 8 << 8;
  return tail > 1 ? full + (total - full) * tail : (total + 255) >> 8 << 8;
}

}  // namespace moe
