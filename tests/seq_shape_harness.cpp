// The launches' shapes (csrc/seq_shape.h) for the tests, on the CPU.
#include "seq_shape.h"

extern "C" void t_scan(int N, int D, int L, int S, int G, int bwd, int64_t* o) {
  seq_scan_t p = {};
  p.N = N, p.D = D, p.L = L, p.S = S, p.G = G;
  const seqops::ScanShape s = seqops::scan_shape(p, bwd);
  const int64_t v[] = {s.rows, s.waves, s.steps, s.segs, s.seg_chunks, s.fine, s.fine_chunks, s.chunks, s.blks,
                       seqops::scan_batch(S)};
  for (int i = 0; i < int(sizeof(v) / sizeof(v[0])); ++i) o[i] = v[i];
}

extern "C" void t_norm(int N, int D, int L, int res_dtype, int64_t* o) {
  seq_norm_t p = {};
  p.N = N, p.D = D, p.L = L, p.res_dtype = res_dtype;
  const seqops::NormShape s = seqops::norm_shape(p);
  const int64_t v[] = {s.flat, s.nt, s.cl, s.tiles, s.parts, s.part, s.wgs, seqops::norm_held(p)};
  for (int i = 0; i < int(sizeof(v) / sizeof(v[0])); ++i) o[i] = v[i];
}
