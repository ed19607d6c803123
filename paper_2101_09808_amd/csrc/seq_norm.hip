// Root-mean-square norms over the channels of [N, D, L], before and after a
// block, forward and backward:
//
//   before:  r = residual + scale x,                    out = w r rstd(r)
//   after:   v = x gate sigmoid(gate),  out = residual + scale w v rstd(v)
//
// with rstd(v) = 1 / sqrt(mean_d v^2 + eps).  Backward, with n = v rstd and h
// the gradient that reaches n:  dv = rstd (h - n mean_d(h n)).  A handful of
// operations an element: bound by memory.
//
// The length is innermost, so a column's channels lie L apart: a workgroup
// takes all channels of a tile of 8 CL columns, CL lanes of eight columns a
// channel, and goes over it twice (statistics, results).  The first H channels
// of a thread stay in registers between the two (forward what is normed,
// backward what was loaded); what is more is read again.  Loads go out before
// anything waits for them: a tile that lies whole inside the row has no
// conditions on the way.  bf16 4 x 2048 x 2048 with gate and residual: forward 43
// us (134 MB, 3.1 TB/s), backward 50 (168 MB, 3.4 TB/s); a CU has one workgroup,
// whose reading, sums and writing follow one another.
#include <type_traits>

#include "seq_device.h"
#include "seq_internal.h"
#include "seq_shape.h"

namespace seqops {
namespace {

template <typename T, typename R, bool POST>
struct NormTypes {  // of out and dout
  using Out = T;
};
template <typename T, typename R>
struct NormTypes<T, R, true> {
  using Out = R;
};

struct NormArgs {
  int N, D, L;
  float eps, inv_d;
  int64_t x_n, x_d, gate_n, gate_d, res_n, res_d, dout_n, dout_d, dsum_n, dsum_d;
  const void* x;
  const float *weight, *scale;
  const void *gate, *residual;
  void *out, *sum;
  const void *dout, *dsum;
  void *dx, *dgate, *dresidual;
  float *partial;  // backward: [workgroups][2][D]
  uint32_t tiles, row_tiles;  // in all, of one n
  int parts, part;  // of the channels; a part's channels
  float *stats;     // [tiles][parts][sums]
};

// What a launch does: everything, a part's sums, or what follows them.
enum Phase { kWhole, kSums, kRest };

__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }

// Sums s[0..7] (NS sets) over the workgroup's threads of the same tid % CL; every
// thread gets its own position's sums.  Rows of sixteen lanes by DPP, the rows'
// sums through LDS in two steps.
template <int NT, int CL, int NS>
struct ColumnSums {
  static constexpr int C = NS * CL * 8, ROWS = NT / 16, PARTS = ROWS < NT / C ? ROWS : NT / C;
  float part[ROWS][C], some[PARTS][C], total[C];
  __device__ __forceinline__ void run(float (*s)[8]) {
    const int tid = threadIdx.x, tl = tid & 15;
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v = s[k][j];
        if (CL <= 2) v += dpp0<kRowShr + 2>(v);
        if (CL <= 4) v += dpp0<kRowShr + 4>(v);
        v += dpp0<kRowShr + 8>(v);
        s[k][j] = v;
      }
    if (tl >= 16 - CL) {
#pragma unroll
      for (int k = 0; k < NS; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) part[tid >> 4][(k * CL + tl - (16 - CL)) * 8 + j] = s[k][j];
    }
    __syncthreads();
    const int c = tid % C, q = tid / C;
    if (q < PARTS) {
      float v = 0.f;
#pragma unroll
      for (int r = 0; r < ROWS / PARTS; ++r) v += part[q * (ROWS / PARTS) + r][c];
      some[q][c] = v;
    }
    __syncthreads();
    if (tid < C) {
      float v = 0.f;
#pragma unroll
      for (int r = 0; r < PARTS; ++r) v += some[r][tid];
      total[tid] = v;
    }
    __syncthreads();
    share(s);
  }
  __device__ __forceinline__ void share(float (*s)[8]) const {
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[k][j] = total[(k * CL + int(threadIdx.x) % CL) * 8 + j];
  }
  // The sums of `parts` launched workgroups, from [parts][C]; to it, one's own.
  __device__ __forceinline__ void take(const float* stats, int parts, float (*s)[8]) {
    const int tid = threadIdx.x;
    if (tid < C) {
      float v = 0.f;
#pragma unroll 8
      for (int r = 0; r < parts; ++r) v += stats[r * C + tid];
      total[tid] = v;
    }
    __syncthreads();
    share(s);
  }
  __device__ __forceinline__ void give(float* stats) const {
    if (threadIdx.x < C) stats[threadIdx.x] = total[threadIdx.x];
  }
};

// Neighbouring tiles share cache lines: they go to workgroups of the same XCD
// (those of equal index modulo 8).
__device__ __forceinline__ uint32_t tile_of(uint32_t b, uint32_t tiles) {
  const uint32_t per = tiles / 8, whole = per * 8;
  return b < whole ? (b % 8) * per + b / 8 : b;
}

// The same value, which the compiler may not compute addresses from beforehand:
// kept over a whole workgroup's work they cost more registers than there are.
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Eight columns of channel d of a tensor.
template <bool IN, typename T>
__device__ __forceinline__ Raw8<T> cols(const void* base, int64_t d, int64_t stride, int nv) {
  return load8(static_cast<const T*>(base) + d * stride, IN ? 8 : nv);
}
// Where a thread's columns start in sequence n of a tensor.
template <typename T>
__device__ __forceinline__ const void* at_cols(const void* base, int n, int64_t n_stride, int col) {
  return base ? static_cast<const T*>(base) + n * n_stride + col : nullptr;
}

template <typename T, typename R, bool POST, int PHASE, int NT, int CL, int H>
__global__ __launch_bounds__(NT) void norm_fwd_kernel(const NormArgs a) {
  using Out = typename NormTypes<T, R, POST>::Out;
  __shared__ ColumnSums<NT, CL, 1> sums;
  constexpr int RS = NT / CL;
  const uint32_t part = PHASE ? blockIdx.x % a.parts : 0;
  const uint32_t tile = PHASE ? blockIdx.x / a.parts : tile_of(blockIdx.x, a.tiles);
  const int rows = PHASE && int(part + 1) * a.part < a.D ? int(part + 1) * a.part : a.D;  // (the part's end)
  float* const stats = PHASE ? a.stats + (int64_t(tile) * a.parts + (PHASE == kSums ? part : 0)) * (CL * 8) : nullptr;
  const int n = int(tile / a.row_tiles);
  const int col0 = int(tile - n * a.row_tiles) * (CL * 8), col = col0 + int(threadIdx.x) % CL * 8, nv = a.L - col;
  const void* const xp = at_cols<T>(a.x, n, a.x_n, col);
  const void* const gp = POST ? at_cols<T>(a.gate, n, a.gate_n, col) : nullptr;
  const void* const rp = at_cols<R>(a.residual, n, a.res_n, col);
  const bool has_g = POST && a.gate, has_r = a.residual;
  const int64_t base = int64_t(n) * a.D * a.L + col;
  auto body = [&](auto inside) {
    constexpr bool IN = decltype(inside)::value;
    float s[1][8] = {};
    int d0 = int(threadIdx.x) / CL + (PHASE ? int(part) * a.part : 0);
    // x and gate (before: the residual) of a channel, its r or v
    auto terms = [&](const Raw8<T>& x, const Raw8<T>& g, const Raw8<R>& r, int d, float* v) {
      unpack8(x, v);
      float o[8];
      if (POST) {
        if (has_g) {
          unpack8(g, o);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= silu(o[j]);
        }
      } else {
        const float sc = a.scale ? a.scale[d] : 1.f;
        unpack8(r, o);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf(sc, v[j], o[j]);
      }
    };
    auto first = [&](const float* v, int d) {
      if (!POST && a.sum) store8(static_cast<R*>(a.sum) + base + int64_t(d) * a.L, IN ? 8 : nv, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[0][j] = __builtin_fmaf(v[j], v[j], s[0][j]);
    };
    auto second = [&](const float* v, const Raw8<R>& r, int d) {
      const float w = a.weight[d];
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = w * (v[j] * s[0][j]);
      if (POST) {
        const float sc = a.scale ? a.scale[d] : 1.f;
        float q[8];
        unpack8(r, q);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = __builtin_fmaf(sc, o[j], q[j]);
      }
      store8(static_cast<Out*>(a.out) + base + int64_t(d) * a.L, IN ? 8 : nv, o);
    };
    // (of the residual what the first pass needs: before a block)
    Raw8<T> x[H], g[H];
    Raw8<R> r[H];
#pragma unroll
    for (int k = 0; k < H; ++k) {
      const int d = d0 + k * RS, dc = d < rows ? d : rows - 1;
      x[k] = cols<IN, T>(xp, dc, a.x_d, nv);
      g[k] = has_g ? cols<IN, T>(gp, dc, a.gate_d, nv) : Raw8<T>{};
      r[k] = !POST && has_r ? cols<IN, R>(rp, dc, a.res_d, nv) : Raw8<R>{};
    }
    float held[H][8];
#pragma unroll
    for (int k = 0; k < H; ++k) {
      const int d = d0 + k * RS;
      if (d < rows) {
        terms(x[k], g[k], r[k], d, held[k]);
        if (PHASE != kRest) first(held[k], d);
      }
      __builtin_amdgcn_sched_barrier(0);  // (one channel's registers at a time)
    }
    auto again_at = [&](int d, float* v, Raw8<R>& rr) {
      const Raw8<T> xx = cols<IN, T>(xp, d, a.x_d, nv), gg = has_g ? cols<IN, T>(gp, d, a.gate_d, nv) : Raw8<T>{};
      rr = has_r ? cols<IN, R>(rp, d, a.res_d, nv) : Raw8<R>{};
      terms(xx, gg, rr, d, v);
    };
    for (int d = d0 + H * RS; PHASE != kRest && d < rows; d += RS) {
      float v[8];
      Raw8<R> rr;
      again_at(d, v, rr);
      first(v, d);
    }
    // (after a block: the residual, on its way while the sums are formed)
    if (POST && PHASE != kSums) {
      d0 = fresh(d0);
#pragma unroll
      for (int k = 0; k < H; ++k) {
        const int d = d0 + k * RS;
        r[k] = has_r ? cols<IN, R>(rp, d < rows ? d : rows - 1, a.res_d, nv) : Raw8<R>{};
      }
    }
    if (PHASE == kRest)
      sums.take(stats, a.parts, s);
    else
      sums.run(s);
    if (PHASE == kSums) {
      sums.give(stats);
      return;
    }
    d0 = fresh(d0);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[0][j] = __builtin_amdgcn_rsqf(__builtin_fmaf(s[0][j], a.inv_d, a.eps));
#pragma unroll
    for (int k = 0; k < H; ++k) {
      const int d = d0 + k * RS;
      if (d < rows) second(held[k], r[k], d);
      __builtin_amdgcn_sched_barrier(0);
    }
    for (int d = d0 + H * RS; d < rows; d += RS) {
      float v[8];
      Raw8<R> rr;
      again_at(d, v, rr);
      second(v, rr, d);
    }
  };
  if (col0 + CL * 8 <= a.L)
    body(std::true_type{});
  else
    body(std::false_type{});
}

// One element of the backward pass: x, the gate z, v (before: r) and g = dout.
struct Elem {
  float v, h;  // v or r; gradient that reaches n
  float x, z, g;
};
template <bool POST>
__device__ __forceinline__ void finish(const Elem& e, float rstd, float m, float sc, bool gated, float dsum, float* dx,
                                       float* dgate, float* dres, float* dw, float* dsc) {
  const float n = e.v * rstd, dv = rstd * __builtin_fmaf(-n, m, e.h);
  if (POST) {
    const float gn = e.g * n;
    *dw += sc * gn;
    *dsc += gn;  // (times w: a row's common factor)
    const float s = gated ? sigmoid(e.z) : 1.f;
    *dx = gated ? dv * (e.z * s) : dv;
    *dgate = gated ? dv * e.x * (s * (1.f + e.z * (1.f - s))) : 0.f;
  } else {
    const float dr = dsum + dv;
    *dw += e.g * n;
    *dsc += dr * e.x;
    *dx = sc * dr;
    *dres = dr;
  }
}

// A workgroup takes tiles blockIdx.x, blockIdx.x + gridDim.x, ... and adds each
// channel's parameter gradients over its columns and tiles, in registers for the
// channels that stay there, the others in its own part of `partial` (always the
// same thread, so in order); norm_sum_kernel adds the parts.
template <typename T, typename R, bool POST, int PHASE, int NT, int CL, int H>
__global__ __launch_bounds__(NT) void norm_bwd_kernel(const NormArgs a) {
  using Out = typename NormTypes<T, R, POST>::Out;
  using V = typename std::conditional<POST, T, R>::type;  // of x (before: of sum)
  __shared__ ColumnSums<NT, CL, 2> sums;
  constexpr int RS = NT / CL;
  const uint32_t part = PHASE ? blockIdx.x % a.parts : 0, wg = PHASE ? blockIdx.x / a.parts : blockIdx.x;
  const int rows = PHASE && int(part + 1) * a.part < a.D ? int(part + 1) * a.part : a.D;  // (the part's end)
  const int row0 = PHASE ? int(part) * a.part : 0;
  float* const stats = PHASE ? a.stats + (int64_t(wg) * a.parts + (PHASE == kSums ? part : 0)) * (CL * 16) : nullptr;
  float* pw = a.partial + int64_t(wg) * 2 * a.D;
  float* ps = pw + a.D;
  float dws[H] = {}, dscs[H] = {};
  for (uint32_t b = wg; b < a.tiles; b += PHASE ? a.tiles : gridDim.x) {
    const uint32_t tile = PHASE ? b : tile_of(b, a.tiles);
    const int n = int(tile / a.row_tiles);
    const int col0 = int(tile - n * a.row_tiles) * (CL * 8), col = col0 + int(threadIdx.x) % CL * 8, nv = a.L - col;
    const int64_t v_d = POST ? a.x_d : a.res_d, base = int64_t(n) * a.D * a.L + col;
    const void* const vp = POST ? at_cols<T>(a.x, n, a.x_n, col) : at_cols<R>(a.sum, n, a.res_n, col);
    const void* const dp = at_cols<Out>(a.dout, n, a.dout_n, col);
    // before: x takes the gate's place, and it and dsum are only the second pass's
    const void* const gp = POST ? at_cols<T>(a.gate, n, a.gate_n, col)
                                : a.scale ? at_cols<T>(a.x, n, a.x_n, col) : nullptr;
    const int64_t g_d = POST ? a.gate_d : a.x_d;
    const bool has_g = POST ? a.gate != nullptr : a.scale != nullptr, has_s = !POST && a.dsum;
    const void* const sp = POST ? nullptr : at_cols<R>(a.dsum, n, a.dsum_n, col);
    auto body = [&](auto inside) {
      constexpr bool IN = decltype(inside)::value;
      float s[2][8] = {};
      int d0 = fresh(threadIdx.x / CL) + row0;
      auto first = [&](const Raw8<V>& vr, const Raw8<T>& zr, const Raw8<Out>& gr, int d) {
        float v[8], z[8], g[8];
        unpack8(vr, v);
        unpack8(gr, g);
        if (POST && has_g) {
          unpack8(zr, z);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= silu(z[j]);
        }
        const float w = POST && a.scale ? a.weight[d] * a.scale[d] : a.weight[d];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          s[0][j] = __builtin_fmaf(v[j], v[j], s[0][j]);
          s[1][j] = __builtin_fmaf(w * g[j], v[j], s[1][j]);
        }
      };
      auto second = [&](const Raw8<V>& vr, const Raw8<T>& zr, const Raw8<Out>& gr, const Raw8<R>& dsr, int d, float& dw,
                        float& dsc) {
        float v[8], x[8], z[8] = {}, g[8], ds[8] = {}, dx[8], dg[8], dr[8];
        if (!POST) {
          unpack8(zr, x);
          unpack8(dsr, ds);
        }
        unpack8(vr, v);
        unpack8(gr, g);
        const float w = a.weight[d], sc = a.scale ? a.scale[d] : 1.f, h = POST ? sc * w : w;
        if (POST) {
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = v[j];
          if (has_g) {
            unpack8(zr, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = x[j] * silu(z[j]);
          }
        }
        float dwr = 0.f, dscr = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const Elem e = {v[j], h * g[j], x[j], z[j], g[j]};
          finish<POST>(e, s[0][j], s[1][j], sc, POST && has_g, ds[j], &dx[j], &dg[j], &dr[j], &dwr, &dscr);
        }
        const int64_t at = base + int64_t(d) * a.L;
        store8(static_cast<T*>(a.dx) + at, IN ? 8 : nv, dx);
        if (POST && has_g) store8(static_cast<T*>(a.dgate) + at, IN ? 8 : nv, dg);
        if (!POST && a.dresidual) store8(static_cast<R*>(a.dresidual) + at, IN ? 8 : nv, dr);
        dw += dwr;
        dsc += POST ? dscr * w : dscr;
      };
      Raw8<V> v[H];
      Raw8<T> z[H];  // gate (before: x)
      Raw8<Out> g[H];
      Raw8<R> ds[H];
      auto gate_or_x = [&](int d) { return has_g ? cols<IN, T>(gp, d, g_d, nv) : Raw8<T>{}; };
      auto dsum = [&](int d) { return has_s ? cols<IN, R>(sp, d, a.dsum_d, nv) : Raw8<R>{}; };
#pragma unroll
      for (int k = 0; k < H; ++k) {
        const int d = d0 + k * RS, dc = d < rows ? d : rows - 1;
        v[k] = cols<IN, V>(vp, dc, v_d, nv);
        g[k] = cols<IN, Out>(dp, dc, a.dout_d, nv);
        z[k] = gate_or_x(dc);
        ds[k] = dsum(dc);
      }
#pragma unroll
      for (int k = 0; k < H; ++k) {
        if (PHASE != kRest && d0 + k * RS < rows) first(v[k], z[k], g[k], d0 + k * RS);
        __builtin_amdgcn_sched_barrier(0);
      }
      for (int d = d0 + H * RS; PHASE != kRest && d < rows; d += RS)
        first(cols<IN, V>(vp, d, v_d, nv), POST ? gate_or_x(d) : Raw8<T>{}, cols<IN, Out>(dp, d, a.dout_d, nv), d);
      if (PHASE == kRest)
        sums.take(stats, a.parts, s);
      else
        sums.run(s);
      if (PHASE == kSums) {
        sums.give(stats);
        return;
      }
      d0 = fresh(d0);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (columns behind the row's end: zeros, also with eps = 0)
        s[0][j] = IN || j < nv ? __builtin_amdgcn_rsqf(__builtin_fmaf(s[0][j], a.inv_d, a.eps)) : 0.f;
        s[1][j] *= s[0][j] * a.inv_d;  // mean of h n
      }
#pragma unroll
      for (int k = 0; k < H; ++k) {
        if (d0 + k * RS < rows)
          second(again(v[k]), again(z[k]), again(g[k]), ds[k], d0 + k * RS, dws[k], dscs[k]);
        __builtin_amdgcn_sched_barrier(0);  // (one channel's registers at a time)
      }
      for (int d = d0 + H * RS; d < rows; d += RS) {
        float dw = 0.f, dsc = 0.f;
        second(cols<IN, V>(vp, d, v_d, nv), gate_or_x(d), cols<IN, Out>(dp, d, a.dout_d, nv), dsum(d), d, dw, dsc);
#pragma unroll
        for (int m = 1; m < CL; m <<= 1) dw += __shfl_xor(dw, m), dsc += __shfl_xor(dsc, m);
        if (threadIdx.x % CL == 0) {
          const bool more = b != wg;
          pw[d] = more ? pw[d] + dw : dw;
          ps[d] = more ? ps[d] + dsc : dsc;
        }
      }
    };
    if (col0 + CL * 8 <= a.L)
      body(std::true_type{});
    else
      body(std::false_type{});
  }
  if (PHASE == kSums) return;
#pragma unroll
  for (int k = 0; k < H; ++k) {
    const int d = int(threadIdx.x) / CL + row0 + k * RS;
#pragma unroll
    for (int m = 1; m < CL; m <<= 1) dws[k] += __shfl_xor(dws[k], m), dscs[k] += __shfl_xor(dscs[k], m);
    if (threadIdx.x % CL == 0 && d < rows) pw[d] = dws[k], ps[d] = dscs[k];
  }
}

// Short lengths (up to kFlatMax): a sequence's [D, L] block as one run of
// elements.  A thread keeps its column: the threads in use are a multiple of L.

// PHASE: as for the tiles; `stats` has [parts][NS][L] of the sequence.
template <int PHASE, int NT, int NS>
__device__ __forceinline__ void flat_sums(float* s, int L, int used, float* lds, float* stats, int part, int parts) {
  const int tid = threadIdx.x;
  float* some = lds + NS * NT;  // [NS][16][L]
  float* total = some + NS * 16 * (kFlatMax + 1);
  if (PHASE == kRest) {
    if (tid < NS * L) {
      float v = 0.f;
#pragma unroll 8
      for (int r = 0; r < parts; ++r) v += stats[r * NS * L + tid];
      total[tid] = v;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NS; ++k) s[k] = total[k * L + tid % L];
    return;
  }
#pragma unroll
  for (int k = 0; k < NS; ++k) lds[k * NT + tid] = tid < used ? s[k] : 0.f;
  __syncthreads();
  if (tid < 16 * L) {
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      float v = 0.f;
      for (int i = tid; i < used; i += 16 * L) v += lds[k * NT + i];
      some[k * 16 * L + tid] = v;
    }
  }
  __syncthreads();
  if (tid < L) {
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      float v = 0.f;
      for (int i = 0; i < 16; ++i) v += some[k * 16 * L + i * L + tid];
      if (PHASE == kSums)
        stats[(part * NS + k) * L + tid] = v;
      else
        total[k * L + tid] = v;
    }
  }
  if (PHASE == kSums) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NS; ++k) s[k] = total[k * L + tid % L];
}
template <int NT, int NS>
constexpr int flat_lds() {
  return NS * NT + NS * 16 * (kFlatMax + 1) + NS * (kFlatMax + 1);
}

template <typename T, typename R, bool POST>
__device__ __forceinline__ float normed1(const NormArgs& a, int n, int d, int l) {
  const float x = to_f(static_cast<const T*>(a.x)[n * a.x_n + d * a.x_d + l]);
  if (POST) return a.gate ? x * silu(to_f(static_cast<const T*>(a.gate)[n * a.gate_n + d * a.gate_d + l])) : x;
  const float r = a.residual ? to_f(static_cast<const R*>(a.residual)[n * a.res_n + d * a.res_d + l]) : 0.f;
  return __builtin_fmaf(a.scale ? a.scale[d] : 1.f, x, r);
}

template <typename T, typename R, bool POST, int PHASE, int NT>
__global__ __launch_bounds__(NT) void norm_fwd_flat_kernel(const NormArgs a) {
  using Out = typename NormTypes<T, R, POST>::Out;
  __shared__ float lds[flat_lds<NT, 1>()];
  const int part = PHASE ? int(blockIdx.x) % a.parts : 0, n = PHASE ? int(blockIdx.x) / a.parts : int(blockIdx.x);
  const int rows = PHASE && (part + 1) * a.part < a.D ? (part + 1) * a.part : a.D;
  float* const stats = PHASE ? a.stats + int64_t(n) * a.parts * a.L : nullptr;
  const int tid = threadIdx.x, per = NT / a.L, used = per * a.L, l = tid % a.L, d0 = tid / a.L + part * a.part;
  const int64_t base = int64_t(n) * a.D * a.L + l;
  float s[1] = {0.f};
  if (PHASE != kRest && tid < used) {
    for (int d = d0; d < rows; d += per) {
      const float v = normed1<T, R, POST>(a, n, d, l);
      if (!POST && a.sum) static_cast<R*>(a.sum)[base + int64_t(d) * a.L] = from_f<R>(v);
      s[0] = __builtin_fmaf(v, v, s[0]);
    }
  }
  flat_sums<PHASE, NT, 1>(s, a.L, used, lds, stats, part, a.parts);
  if (PHASE == kSums || tid >= used) return;
  const float rstd = __builtin_amdgcn_rsqf(__builtin_fmaf(s[0], a.inv_d, a.eps));
  for (int d = d0; d < rows; d += per) {
    float o = a.weight[d] * (normed1<T, R, POST>(a, n, d, l) * rstd);
    if (POST) {
      const float r = a.residual ? to_f(static_cast<const R*>(a.residual)[n * a.res_n + d * a.res_d + l]) : 0.f;
      o = __builtin_fmaf(a.scale ? a.scale[d] : 1.f, o, r);
    }
    static_cast<Out*>(a.out)[base + int64_t(d) * a.L] = from_f<Out>(o);
  }
}

// (a column has a part of its own in `partial`: [workgroups][L][2][D])
template <typename T, typename R, bool POST, int PHASE, int NT>
__global__ __launch_bounds__(NT) void norm_bwd_flat_kernel(const NormArgs a) {
  using Out = typename NormTypes<T, R, POST>::Out;
  __shared__ float lds[flat_lds<NT, 2>()];
  const int part = PHASE ? int(blockIdx.x) % a.parts : 0, wg = PHASE ? int(blockIdx.x) / a.parts : int(blockIdx.x);
  const int rows = PHASE && (part + 1) * a.part < a.D ? (part + 1) * a.part : a.D;
  float* const stats = PHASE ? a.stats + int64_t(wg) * a.parts * 2 * a.L : nullptr;
  const int tid = threadIdx.x, per = NT / a.L, used = per * a.L, l = tid % a.L, d0 = tid / a.L + part * a.part;
  float* pw = a.partial + (int64_t(wg) * a.L + l) * 2 * a.D;
  float* ps = pw + a.D;
  for (int n = wg; n < a.N; n += PHASE ? a.N : int(gridDim.x)) {
    const int64_t base = int64_t(n) * a.D * a.L + l;
    auto read = [&](int d) {
      Elem e = {};
      if (POST || a.scale) e.x = to_f(static_cast<const T*>(a.x)[n * a.x_n + d * a.x_d + l]);
      if (POST) {
        if (a.gate) e.z = to_f(static_cast<const T*>(a.gate)[n * a.gate_n + d * a.gate_d + l]);
        e.v = a.gate ? e.x * silu(e.z) : e.x;
      } else {
        e.v = to_f(static_cast<const R*>(a.sum)[n * a.res_n + d * a.res_d + l]);
      }
      e.g = to_f(static_cast<const Out*>(a.dout)[n * a.dout_n + d * a.dout_d + l]);
      e.h = (POST && a.scale ? a.scale[d] * a.weight[d] : a.weight[d]) * e.g;
      return e;
    };
    float s[2] = {0.f, 0.f};
    if (PHASE != kRest && tid < used) {
      for (int d = d0; d < rows; d += per) {
        const Elem e = read(d);
        s[0] = __builtin_fmaf(e.v, e.v, s[0]);
        s[1] = __builtin_fmaf(e.h, e.v, s[1]);
      }
    }
    flat_sums<PHASE, NT, 2>(s, a.L, used, lds, stats, part, a.parts);
    if (PHASE == kSums) return;
    if (tid < used) {
      const float rstd = __builtin_amdgcn_rsqf(__builtin_fmaf(s[0], a.inv_d, a.eps));
      const float m = s[1] * rstd * a.inv_d;
      for (int d = d0; d < rows; d += per) {
        const Elem e = read(d);
        const int64_t at = base + int64_t(d) * a.L;
        const float ds = !POST && a.dsum ? to_f(static_cast<const R*>(a.dsum)[n * a.dsum_n + d * a.dsum_d + l]) : 0.f;
        float dx, dg, dr, dw = 0.f, dsc = 0.f;
        finish<POST>(e, rstd, m, a.scale ? a.scale[d] : 1.f, POST && a.gate, ds, &dx, &dg, &dr, &dw, &dsc);
        static_cast<T*>(a.dx)[at] = from_f<T>(dx);
        if (POST && a.gate) static_cast<T*>(a.dgate)[at] = from_f<T>(dg);
        if (!POST && a.dresidual) static_cast<R*>(a.dresidual)[at] = from_f<R>(dr);
        if (POST) dsc *= a.weight[d];
        const bool more = n != wg;
        pw[d] = more ? pw[d] + dw : dw;
        ps[d] = more ? ps[d] + dsc : dsc;
      }
    }
    __syncthreads();
  }
}

// Adds the parts in order: a workgroup takes 64 channels of one gradient, its
// sixteen waves a sixteenth of the parts each.
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* partial, int parts, int D, float* dweight,
                                                        float* dscale) {
  __shared__ float lds[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (d < D)
#pragma unroll 8
    for (int p = wave; p < parts; p += 16) s += partial[(int64_t(p) * 2 + blockIdx.y) * D + d];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && d < D) {
#pragma unroll
    for (int w = 1; w < 16; ++w) s += lds[w][lane];
    (blockIdx.y ? dscale : dweight)[d] = s;
  }
}

int64_t stats_floats(const seq_norm_t& p, const NormShape& s, int sums) {
  return s.parts ? s.tiles * s.parts * (s.flat ? p.L : s.cl * 8) * sums : 0;
}
int64_t partial_floats(const seq_norm_t& p, const NormShape& s) {
  return (int64_t(s.wgs) * (s.flat ? p.L : 1) * 2 * p.D + 3) / 4 * 4;
}

template <typename T, typename R, bool POST, int PHASE, int NT, int CL>
void launch_cl(const NormArgs& a, const NormShape& sh, bool bwd, hipStream_t s) {
  constexpr int H = sizeof(R) == 2 ? 4 : 2;
  const uint32_t wgs = uint32_t(PHASE ? sh.tiles * sh.parts : bwd ? sh.wgs : sh.tiles);
  if (bwd)
    norm_bwd_kernel<T, R, POST, PHASE, NT, CL, H><<<dim3(wgs), NT, 0, s>>>(a);
  else
    norm_fwd_kernel<T, R, POST, PHASE, NT, CL, PHASE ? H : 2 * H><<<dim3(wgs), NT, 0, s>>>(a);
}
template <typename T, typename R, bool POST, int PHASE, int NT>
void launch_nt(const NormArgs& a, const NormShape& sh, bool bwd, hipStream_t s) {
  if (sh.flat) {
    const uint32_t wgs = uint32_t(PHASE ? sh.tiles * sh.parts : bwd ? sh.wgs : sh.tiles);
    if (bwd)
      norm_bwd_flat_kernel<T, R, POST, PHASE, NT><<<dim3(wgs), NT, 0, s>>>(a);
    else
      norm_fwd_flat_kernel<T, R, POST, PHASE, NT><<<dim3(wgs), NT, 0, s>>>(a);
    return;
  }
  switch (sh.cl) {
    case 2: launch_cl<T, R, POST, PHASE, NT, 2>(a, sh, bwd, s); break;
    case 4: launch_cl<T, R, POST, PHASE, NT, 4>(a, sh, bwd, s); break;
    default: launch_cl<T, R, POST, PHASE, NT, 8>(a, sh, bwd, s); break;
  }
}
template <typename T, typename R, bool POST>
int run(const seq_norm_t& p, bool bwd, hipStream_t s) {
  const NormShape sh = norm_shape(p);
  if (sh.tiles * (sh.parts ? sh.parts : 1) * sh.nt > kMaxThreads) return CONV_ERANGE;
  NormArgs a = {};
  a.N = p.N, a.D = p.D, a.L = p.L, a.eps = p.eps, a.inv_d = 1.f / float(p.D);
  a.x_n = p.x_n, a.x_d = p.x_d, a.gate_n = p.gate_n, a.gate_d = p.gate_d, a.res_n = p.res_n, a.res_d = p.res_d;
  a.dout_n = p.dout_n, a.dout_d = p.dout_d, a.dsum_n = p.dsum_n, a.dsum_d = p.dsum_d;
  a.x = p.x, a.weight = p.weight, a.scale = p.scale, a.gate = p.gate, a.residual = p.residual;
  a.out = p.out, a.sum = p.sum, a.dout = p.dout, a.dsum = p.dsum;
  a.dx = p.dx, a.dgate = p.dgate, a.dresidual = p.dresidual;
  a.tiles = uint32_t(sh.tiles), a.row_tiles = uint32_t(sh.row_tiles), a.parts = sh.parts, a.part = sh.part;
  const int64_t need = bwd ? norm_bwd_workspace(p) : norm_fwd_workspace(p);
  if (need) {
    if (!p.workspace) return CONV_ENULL;
    if (p.workspace_bytes < need) return CONV_ESCRATCH;
  }
  a.partial = static_cast<float*>(p.workspace);
  a.stats = a.partial + (bwd ? partial_floats(p, sh) : 0);
  if (sh.parts) {
    launch_nt<T, R, POST, kSums, 256>(a, sh, bwd, s);
    if (hipGetLastError() != hipSuccess) return CONV_EHIP;
    launch_nt<T, R, POST, kRest, 256>(a, sh, bwd, s);
  } else if (sh.nt == 1024) {
    launch_nt<T, R, POST, kWhole, 1024>(a, sh, bwd, s);
  } else {
    launch_nt<T, R, POST, kWhole, 256>(a, sh, bwd, s);
  }
  if (hipGetLastError() != hipSuccess) return CONV_EHIP;
  if (!bwd) return CONV_OK;
  const int parts = sh.wgs * (sh.flat ? p.L : 1);
  norm_sum_kernel<<<dim3(uint32_t(ceil_div(p.D, 64)), p.scale ? 2 : 1), 1024, 0, s>>>(a.partial, parts, p.D, p.dweight,
                                                                                      p.dscale);
  return hipGetLastError() == hipSuccess ? CONV_OK : CONV_EHIP;
}
template <bool POST>
int run_types(const seq_norm_t& p, bool bwd, hipStream_t s) {
  if (p.dtype == CONV_DTYPE_F32) return run<float, float, POST>(p, bwd, s);
  return p.res_dtype == CONV_DTYPE_F32 ? run<bf16, float, POST>(p, bwd, s) : run<bf16, bf16, POST>(p, bwd, s);
}
}  // namespace

int64_t norm_fwd_workspace(const seq_norm_t& p) {
  return stats_floats(p, norm_shape(p), 1) * int64_t(sizeof(float));
}
int64_t norm_bwd_workspace(const seq_norm_t& p) {
  const NormShape sh = norm_shape(p);
  return (partial_floats(p, sh) + stats_floats(p, sh, 2)) * int64_t(sizeof(float));
}
int launch_norm_fwd(const seq_norm_t& p, bool post, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return post ? run_types<true>(p, false, s) : run_types<false>(p, false, s);
}
int launch_norm_bwd(const seq_norm_t& p, bool post, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return post ? run_types<true>(p, true, s) : run_types<false>(p, true, s);
}

}  // namespace seqops
