// How the scan's and the norms' launches are cut, from a call's extents and types
// alone: host arithmetic, which the launchers and the tests share.
#pragma once
#include "seq_internal.h"

namespace seqops {

constexpr int kChunk = SEQ_SCAN_CHUNK;  // 16 lanes of 8 steps
constexpr int kFlatMax = 15;  // lengths below 16: norms over a sequence's whole block

struct ScanShape {
  int per, rows, waves, blks, segs, seg_chunks, chunks;  // rows: channels of a wave
  int steps;  // a lane's in a pass
  int fine, fine_chunks;
  int64_t wgs;
};
inline ScanShape scan_shape(const seq_scan_t& p, bool bwd) {
  ScanShape s = {};
  s.per = p.D / p.G;
  s.chunks = int(ceil_div(p.L, kChunk));
  const int64_t waves4 = int64_t(p.N) * p.G * ceil_div(s.per, 4);
  s.rows = 4, s.steps = 8;
  if (bwd) {
    // Larger workgroups leave fewer parts of dB and dC, smaller ones spread few
    // channels further.  Backward at four and at eight waves, us: 2 x 520 x 260 fp32,
    // 8 states, 28.0 and 29.5; 2 x 520 x 1500 47.6 and 47.1; 1 x 64 x 1000 bf16, 16
    // states, 29.7 and 33.9; 1 x 1024 x 2048 75 and 56; 8 x 2048 x 500 215 and 143.
    // (With 16 states eight are faster below nine chunks, too, where the channels are
    // not few: 2 x 520 x 1001 69 and 51.)
    s.waves = s.per > 16 && (waves4 > 1024 || s.chunks > 8) ? 8 : 4;
  } else {
    // Few and short rows: a channel has a whole wave, 512 steps a pass (which
    // fits in LDS for up to 16 states).  2 x 520 x 1001: 15 us, against 22 in
    // segments; 1 x 1024 x 16384: 176 us, against 145.
    if (waves4 <= 1024 && p.L > 256 && p.L <= 2048 && p.S <= 16) s.rows = 1;
    s.waves = p.S > 32 ? 8 : 4;
  }
  s.blks = int(ceil_div(s.per, s.waves * s.rows));
  // Segments where the chip is less than half full: as many as its 2048 places
  // for waves (two a SIMD) take at once.
  const int64_t wgs = int64_t(p.N) * p.G * s.blks, places = 2048 / s.waves;
  int64_t want = wgs * s.waves <= (bwd || s.rows == 1 ? 1024 : 512) ? places / wgs : 1;
  // 16 steps a lane are a sixth less work, but a pass may waste twice as many,
  // and two waves fit on a SIMD instead of three: for a chip that two a SIMD fill
  // at once (4 x 2048 x 2048, forward and backward, 348 us against 355; 1 x 1024 x
  // 16384 150 against 160), and long rows (ragged 6 x 1536 x 4000 155 against 173;
  // ragged 12 x 4096 x 700, however, 164 against 131).
  if (!bwd && s.rows == 4 && p.S <= 16 && ceil_div(p.L, 256) * 12 <= ceil_div(p.L, 128) * 7 && want * 256 <= p.L &&
      (wgs * s.waves * want <= 2048 || p.L > 2048))
    s.steps = 16;
  const int per = 64 / s.rows * s.steps / kChunk;  // chunks a pass
  const int64_t passes = ceil_div(s.chunks, per);
  if (want > passes) want = passes;
  s.seg_chunks = int(ceil_div(passes, want)) * per;
  s.segs = int(ceil_div(s.chunks, s.seg_chunks));
  s.wgs = wgs * s.segs;
  // (pieces of 256 steps at least, up to 4096 waves of them)
  s.fine = 1;
  while (s.fine < 4 && waves4 * (s.segs - 1) * s.fine * 2 <= 4096 && s.seg_chunks >= 4 * s.fine) s.fine *= 2;
  s.fine_chunks = int(ceil_div(s.seg_chunks, s.fine));
  return s;
}
// As many as LDS holds beside what S states need: an exchange is two barriers.
inline int scan_batch(int S) { return S > 32 ? 4 : S > 16 || S <= 8 ? 8 : 16; }

struct NormShape {
  bool flat;
  int nt, cl;
  int64_t tiles, row_tiles;  // (flat: sequences)
  int parts, part;           // 0: the channels are not cut
  int wgs;                   // backward: with a part of the parameters' gradients each
};
// Channels of a thread that stay in registers (bytes of up to four tensors' eight columns).
inline int norm_held(const seq_norm_t& p) { return p.res_dtype == CONV_DTYPE_BF16 ? 4 : 2; }
inline NormShape norm_shape(const seq_norm_t& p) {
  NormShape s = {};
  s.flat = p.L <= kFlatMax;
  if (s.flat) {
    s.tiles = p.N;
    s.nt = int64_t(p.D) * p.L > 2048 ? 1024 : 256;
    s.part = 256 / p.L * 8;
  } else {
    const auto tile = [&](int cl) {
      s.cl = cl;
      s.row_tiles = ceil_div(p.L, cl * 8);
      s.tiles = s.row_tiles * p.N;
      s.part = 256 / cl * norm_held(p);
    };
    // Whole channels at once where each CU has a tile of at least 32 columns (half a
    // cache line of bf16; the next tile's workgroup is of the same XCD) and at least
    // half of its channels (fp32 residual: a quarter) stay in registers over the
    // backward pass; else cut.  Forward and backward after a block, gated, us for
    // N x D x 2048, whole and cut, with a bf16 residual | an fp32 one (x in bf16):
    //   4 x 1024   44,  52 |  48,  62     16 x 1024  165, 192 |  218,  240
    //   4 x 1536   60,  80 |  79,  95     16 x 1536  290, 301 |  363,  366
    //   4 x 2048  100, 103 | 116, 129     16 x 2048  390, 388 |  522,  496
    //   4 x 2560  126, 133 | 151, 163     16 x 2560  520, 488 |  623,  642
    // The bound on D CL, 8192, lies where the two meet; over many tiles they do a
    // little before it, over few a little behind.  Too few tiles to be whole:  fp32
    // 3 x 1000 x 1333 66 and 59, bf16 9 x 2816 x 53 110 and 45.
    tile(p.L > 32 ? 8 : p.L > 16 ? 4 : 2);
    const auto whole = [&] { return s.tiles >= 256 && int64_t(p.D) * s.cl <= 8192; };
    if (!whole() && s.cl == 8) {
      tile(4);
      if (!whole()) tile(8);
    }
    s.nt = int64_t(p.D) * s.cl > 512 ? 1024 : 256;
    if (whole()) {
      s.wgs = 256;
      return s;
    }
  }
  if (p.D >= 2 * s.part && (!s.flat || s.tiles < 128)) {
    s.nt = 256;
    s.parts = int(ceil_div(p.D, s.part));
  } else {
    while (s.cl > 2 && s.tiles < 256) {
      s.cl /= 2;
      s.row_tiles = ceil_div(p.L, s.cl * 8);
      s.tiles = s.row_tiles * p.N;
    }
  }
  s.wgs = int(s.parts ? s.tiles : s.flat ? (s.tiles < 512 ? s.tiles : 512) : s.tiles < 256 ? s.tiles : 256);
  return s;
}

}  // namespace seqops
