// How the norms' launches divide their rows.  Plain functions of whole numbers, so that a host program can walk through the plans.
#pragma once

#include <stdint.h>

#include "../../include/moe_hip.h"

namespace moe {

// A team's next row is an index, too, which may be as many rows further on as a launch has teams: 2048 blocks of sixteen at most (where rows are many).
constexpr int kNormMaxD = 16384, kNormMaxRows = INT32_MAX - (1 << 15);

// TEAM: who works on a row.  Sixteen or thirty-two lanes; a wavefront; the block; or (rows of more than 8192 values) a block of up to sixteen wavefronts, whose lanes have
// too few registers to hold the next row as well, or, in the backward pass, this one.
enum { kWaveTeam = 0, kBlockTeam = 1, kLongTeam = 2, kLanes16Team = 3, kLanes32Team = 4 };
constexpr bool wide_team(int team) { return team == kBlockTeam || team == kLongTeam; }
constexpr int lanes_of(int team) { return team == kLanes16Team ? 16 : team == kLanes32Team ? 32 : 64; }

// Pieces of a lane, wavefronts of a row, blocks.  Measured (T rows of d, bf16 unless it says otherwise):
//  - rows of up to 1024 values take a wavefront (16384 x 768 backward: 18.5 us, with a block of two wavefronts 20.2), four a block; in the backward pass eight, whose sums of
//    the weights' gradients are one, in as many blocks as the registers of 256 units hold at once (65536 x 256: 512 blocks 27.5 us, 384 34.7, 768 30.3, blocks of four 31.5;
//    6000 x 1000 fp32: 256 blocks 16.8, 384 20.4, 512 20.1, of four 19.9);
//  - longer ones a block whose lanes hold one piece, or two where rows of bf16 are long and many: half as many wavefronts take part in a row's barriers (forward 8192 x 7168:
//    44.0 us for 49.6, 8000 x 5000 33 for 62, 8192 x 2048 20.4 for 18.5, 500 x 4096 5.9 for 5.1).  In the backward pass only rows of full pieces, long enough for seven or eight
//    wavefronts a unit, without dropout (8000 x 6000 60 us for 62.5, 8000 x 4096 35.8 for 35.3; with dropout 8000 x 5000 95 for 75, 8000 x 7168 99 for 95, rows of 3500 64 for
//    55, of 2200 without dropout 32 for 26); nor in fp32, where a piece is 32 bytes (4000 x 5000 37 + 43 us for 31.5 + 41.3);
//  - 16 wavefronts a unit, each with the next row's loads under way, reach the copy's rate, in the backward pass with two pieces a lane eight.  The backward pass takes fewer
//    blocks where they would get less than four rows: their sums of the weights' gradients are written and read again (2000 x 2048: 512 blocks 9.7 + 3.4 us, 1024 11.0 + 5.0,
//    256 12.2 + 4.1).  Blocks of five wavefronts are two a unit there: of three, 15 wavefronts at four a SIMD, the last does not find its place (8000 x 2200 fp32 37.8 us for
//    46.3, with dropout 38 for 47; bf16 without, whose registers allow five a SIMD, 28.8 for 25.7);
//  - where blocks of columns have sixteen rows a lane at most, in 8 MB, they are in the same launch as the rows (256 x 4096: 5.2 us for 6.8 + 3.3, 1000 x 4096 13.0 for 11.6 + 4.4,
//    512 x 1000 6.3 for 5.8 + 3.2; 1000 x 512 8.5 for 4.6 + 2.9, 2000 x 333 fp32 18.2 for 5.6 + 3.0).  The blocks of eight wavefronts, beside rows of up to 1024
//    values, count as half their size (with eight rows a lane 777 x 333 fp32 takes 8.1 us, with sixteen, in blocks of four, 11.0).
// With two pieces a lane bf16 rows take a short piece value by value in the forward pass (8000 x 5001: 43 us for 53, backward settled 91 for 99); so do rows of more than 8192
// values, for their registers.
struct NormPlan {
  int V, team, waves, blocks;
  int columns;  // blocks for the weights' gradients, in the same launch; 0: a launch of their own, from the blocks' sums
};
// in_place: an output is an input whose columns would be read beside it.
inline NormPlan norm_plan(const moe_norm_t* n, bool backward, bool drop, bool in_place) {
  const int pieces = (n->d + 7) / 8, rows = n->n_rows;
  const auto at_most = [](int x, int most) { return x < most ? x : most; };
  const auto evenly = [&](int64_t teams, int blocks) {  // no more blocks of so many teams than give the same number of rounds
    if (rows == 0) return 0;
    const int64_t per = (rows + teams * blocks - 1) / (teams * blocks);  // (a block's rows are many where all are: the sums pass 2^31)
    return (int)((rows + teams * per - 1) / (teams * per));
  };
  NormPlan p = {};
  const int elem = n->dtype == MOE_F32 ? 4 : 2;
  const auto own_columns = [&](int waves) {
    const int side = n->dtype == MOE_F32 ? 4 : 8;  // pieces of 128 bytes
    if (backward && !in_place && rows <= 16 * (64 * waves / side) && (int64_t)rows * n->d * elem <= 1 << 23) p.columns = (pieces + side - 1) / side;
  };
  if (pieces <= 128) {
    p.V = pieces <= 64 ? 1 : 2;
    p.team = pieces <= 16 ? kLanes16Team : pieces <= 32 ? kLanes32Team : kWaveTeam;
    own_columns(4);
    p.waves = backward ? 8 : 4;
    const int teams = p.waves * (64 / lanes_of(p.team));
    p.blocks = at_most((rows + teams - 1) / teams, 2048);
    if (backward && !p.columns) p.blocks = evenly(teams, at_most(p.blocks, 512 / p.V));
    return p;
  }
  const bool two = pieces > 1024 || (pieces > 256 && rows > 1024 && n->dtype == MOE_BF16 && !(backward && (drop || n->d % 8 || pieces <= 448)));
  p.V = two ? 2 : 1;
  p.team = pieces > 1024 ? kLongTeam : kBlockTeam;
  p.waves = (pieces + 64 * p.V - 1) / (64 * p.V);
  if (!two) own_columns(p.waves);
  p.blocks = (backward && two && p.team == kBlockTeam ? 2048 : 4096) / p.waves / 256 * 256;  // 256 units, the same number of blocks each: one at least, of 16 wavefronts, or of 8
  if (p.blocks > 2048) p.blocks = 2048;
  if (backward && p.waves == 5) p.blocks = at_most(p.blocks, 512);
  if (backward && !p.columns) p.blocks = evenly(1, at_most(p.blocks, rows / 4 + 64));
  p.blocks = at_most(p.blocks, rows);
  return p;
}

}  // namespace moe
