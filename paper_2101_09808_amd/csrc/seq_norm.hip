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
// channel, and goes over it twice (statistics, results).
#include "seq_device.h"
#include "seq_internal.h"

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
};

__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }

// Sums s[0..7] (and more of them: NS sets) over the workgroup's threads of the
// same lane group position tid % CL; every thread gets its own position's sums.
template <int NT, int CL, int NS>
__device__ __forceinline__ void column_sums(float (*s)[8], float* lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int W = NT / 64, C = CL * 8;
#pragma unroll
  for (int k = 0; k < NS; ++k) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v = s[k][j];
#pragma unroll
      for (int m = CL; m < 64; m <<= 1) v += __shfl_xor(v, m);
      s[k][j] = v;
    }
  }
  float* part = lds;                 // [W][NS][C]
  float* total = lds + W * NS * C;   // [NS][C]
  if (lane < CL) {
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) part[(wave * NS + k) * C + lane * 8 + j] = s[k][j];
  }
  __syncthreads();
  for (int i = tid; i < NS * C; i += NT) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += part[w * NS * C + i];
    total[i] = v;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NS; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) s[k][j] = total[k * C + (tid % CL) * 8 + j];
}

// A row's terms at eight columns: r or v.
template <typename T, typename R, bool POST>
__device__ __forceinline__ void normed8(const NormArgs& a, int n, int d, int col, int nv, float* v) {
  unpack8(load8(static_cast<const T*>(a.x) + n * a.x_n + d * a.x_d + col, nv), v);
  if (POST) {
    if (a.gate) {
      float g[8];
      unpack8(load8(static_cast<const T*>(a.gate) + n * a.gate_n + d * a.gate_d + col, nv), g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= silu(g[j]);
    }
  } else {
    const float sc = a.scale ? a.scale[d] : 1.f;
    float r[8] = {};
    if (a.residual) unpack8(load8(static_cast<const R*>(a.residual) + n * a.res_n + d * a.res_d + col, nv), r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf(sc, v[j], r[j]);
  }
}

// HOLD > 0: a thread's rows (at most HOLD) stay in registers between the passes.
template <typename T, typename R, bool POST, int NT, int CL, int HOLD>
__global__ __launch_bounds__(NT) void norm_fwd_kernel(const NormArgs a) {
  using Out = typename NormTypes<T, R, POST>::Out;
  __shared__ float lds[(NT / 64 + 1) * CL * 8];
  const int n = blockIdx.x / a.row_tiles, tid = threadIdx.x;
  const int col = int(blockIdx.x - n * a.row_tiles) * (CL * 8) + (tid % CL) * 8, nv = a.L - col;
  constexpr int RS = NT / CL;
  float s[1][8] = {}, held[HOLD > 0 ? HOLD : 1][8];
  auto first = [&](int d, float* v) {
    normed8<T, R, POST>(a, n, d, col, nv, v);
    if (!POST && a.sum) store8(static_cast<R*>(a.sum) + (int64_t(n) * a.D + d) * a.L + col, nv, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[0][j] = __builtin_fmaf(v[j], v[j], s[0][j]);
  };
  if (nv > 0) {
    if (HOLD > 0) {
#pragma unroll
      for (int k = 0; k < HOLD; ++k) {
        const int d = tid / CL + k * RS;
        if (d < a.D) first(d, held[k]);
      }
    } else {
      for (int d = tid / CL; d < a.D; d += RS) {
        float v[8];
        first(d, v);
      }
    }
  }
  column_sums<NT, CL, 1>(s, lds);
  if (nv <= 0) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) s[0][j] = __builtin_amdgcn_rsqf(__builtin_fmaf(s[0][j], a.inv_d, a.eps));
  auto second = [&](int d, const float* v) {
    const float w = a.weight[d];
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = w * (v[j] * s[0][j]);
    if (POST) {
      const float sc = a.scale ? a.scale[d] : 1.f;
      float r[8] = {};
      if (a.residual) unpack8(load8(static_cast<const R*>(a.residual) + n * a.res_n + d * a.res_d + col, nv), r);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = __builtin_fmaf(sc, o[j], r[j]);
    }
    store8(static_cast<Out*>(a.out) + (int64_t(n) * a.D + d) * a.L + col, nv, o);
  };
  if (HOLD > 0) {
#pragma unroll
    for (int k = 0; k < HOLD; ++k) {
      const int d = tid / CL + k * RS;
      if (d < a.D) second(d, held[k]);
    }
  } else {
    for (int d = tid / CL; d < a.D; d += RS) {
      float v[8];
      normed8<T, R, POST>(a, n, d, col, nv, v);
      second(d, v);
    }
  }
}

// One element of the backward pass: x, the gate z, r (before) and g = dout.
struct Elem {
  float v, h;       // v or r; gradient that reaches n
  float x, z, g;
};
template <typename T, typename R, bool POST>
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
// row's parameter gradients over its columns and tiles in its own part of
// `partial` (always the same thread, so in order); norm_sum_kernel adds the parts.
template <typename T, typename R, bool POST, int NT, int CL>
__global__ __launch_bounds__(NT) void norm_bwd_kernel(const NormArgs a) {
  using Out = typename NormTypes<T, R, POST>::Out;
  __shared__ float lds[(NT / 64 + 1) * CL * 16];
  const int tid = threadIdx.x;
  constexpr int RS = NT / CL;
  float* pw = a.partial + int64_t(blockIdx.x) * 2 * a.D;
  float* ps = pw + a.D;
  for (uint32_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const int n = tile / a.row_tiles;
    const int col = int(tile - n * a.row_tiles) * (CL * 8) + (tid % CL) * 8, nv = a.L - col;
    const Out* dout = static_cast<const Out*>(a.dout) + n * a.dout_n + col;
    auto read = [&](int d, float* v, float* x, float* z, float* g) {
      if (POST || (a.scale && x)) unpack8(load8(static_cast<const T*>(a.x) + n * a.x_n + d * a.x_d + col, nv), x);
      if (POST) {
        if (a.gate) unpack8(load8(static_cast<const T*>(a.gate) + n * a.gate_n + d * a.gate_d + col, nv), z);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = a.gate ? x[j] * silu(z[j]) : x[j];
      } else {
        unpack8(load8(static_cast<const R*>(a.sum) + n * a.res_n + d * a.res_d + col, nv), v);
      }
      unpack8(load8(dout + d * a.dout_d, nv), g);
    };
    float s[2][8] = {};
    if (nv > 0) {
      for (int d = tid / CL; d < a.D; d += RS) {
        float v[8], x[8], z[8], g[8];
        read(d, v, POST ? x : nullptr, z, g);
        const float w = POST && a.scale ? a.weight[d] * a.scale[d] : a.weight[d];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          s[0][j] = __builtin_fmaf(v[j], v[j], s[0][j]);
          s[1][j] = __builtin_fmaf(w * g[j], v[j], s[1][j]);
        }
      }
    }
    column_sums<NT, CL, 2>(s, lds);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // (columns behind the row's end: zeros, also with eps = 0)
      s[0][j] = j < nv ? __builtin_amdgcn_rsqf(__builtin_fmaf(s[0][j], a.inv_d, a.eps)) : 0.f;
      s[1][j] *= s[0][j] * a.inv_d;  // mean of h n
    }
    for (int d = tid / CL; d < a.D; d += RS) {
      float dw = 0.f, dsc = 0.f;
      const float w = a.weight[d], sc = a.scale ? a.scale[d] : 1.f;
      if (nv > 0) {
        float v[8], x[8] = {}, z[8] = {}, g[8], ds[8] = {}, dx[8], dg[8], dr[8];
        read(d, v, x, z, g);
        if (!POST && a.dsum) unpack8(load8(static_cast<const R*>(a.dsum) + n * a.dsum_n + d * a.dsum_d + col, nv), ds);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const Elem e = {v[j], (POST ? sc * w : w) * g[j], x[j], z[j], g[j]};
          finish<T, R, POST>(e, s[0][j], s[1][j], sc, POST && a.gate, ds[j], &dx[j], &dg[j], &dr[j], &dw, &dsc);
        }
        const int64_t at = (int64_t(n) * a.D + d) * a.L + col;
        store8(static_cast<T*>(a.dx) + at, nv, dx);
        if (POST && a.gate) store8(static_cast<T*>(a.dgate) + at, nv, dg);
        if (!POST && a.dresidual) store8(static_cast<R*>(a.dresidual) + at, nv, dr);
      }
#pragma unroll
      for (int m = 1; m < CL; m <<= 1) {
        dw += __shfl_xor(dw, m);
        dsc += __shfl_xor(dsc, m);
      }
      if (tid % CL == 0) {
        if (POST) dsc *= w;
        const bool more = tile != blockIdx.x;
        pw[d] = more ? pw[d] + dw : dw;
        ps[d] = more ? ps[d] + dsc : dsc;
      }
    }
    __syncthreads();
  }
}

// Short lengths (L < 16): a sequence's [D, L] block as one run of elements.  A
// thread keeps its column: the threads in use are a multiple of L.
constexpr int kFlatMax = 15;

template <int NT, int NS>
__device__ __forceinline__ void flat_sums(float* s, int L, int used, float* lds) {
  const int tid = threadIdx.x;
  float* part = lds + NS * NT;      // [NS][16][L]
  float* total = part + NS * 16 * (kFlatMax + 1);
#pragma unroll
  for (int k = 0; k < NS; ++k) lds[k * NT + tid] = tid < used ? s[k] : 0.f;
  __syncthreads();
  if (tid < 16 * L) {
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      float v = 0.f;
      for (int i = tid; i < used; i += 16 * L) v += lds[k * NT + i];
      part[k * 16 * L + tid] = v;
    }
  }
  __syncthreads();
  if (tid < L) {
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      float v = 0.f;
      for (int i = 0; i < 16; ++i) v += part[k * 16 * L + i * L + tid];
      total[k * L + tid] = v;
    }
  }
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

template <typename T, typename R, bool POST, int NT>
__global__ __launch_bounds__(NT) void norm_fwd_flat_kernel(const NormArgs a) {
  using Out = typename NormTypes<T, R, POST>::Out;
  __shared__ float lds[flat_lds<NT, 1>()];
  const int n = blockIdx.x, tid = threadIdx.x, per = NT / a.L, used = per * a.L, l = tid % a.L, d0 = tid / a.L;
  const int64_t base = int64_t(n) * a.D * a.L + l;
  float s[1] = {0.f};
  if (tid < used) {
    for (int d = d0; d < a.D; d += per) {
      const float v = normed1<T, R, POST>(a, n, d, l);
      if (!POST && a.sum) static_cast<R*>(a.sum)[base + int64_t(d) * a.L] = from_f<R>(v);
      s[0] = __builtin_fmaf(v, v, s[0]);
    }
  }
  flat_sums<NT, 1>(s, a.L, used, lds);
  if (tid >= used) return;
  const float rstd = __builtin_amdgcn_rsqf(__builtin_fmaf(s[0], a.inv_d, a.eps));
  for (int d = d0; d < a.D; d += per) {
    float o = a.weight[d] * (normed1<T, R, POST>(a, n, d, l) * rstd);
    if (POST) {
      const float r = a.residual ? to_f(static_cast<const R*>(a.residual)[n * a.res_n + d * a.res_d + l]) : 0.f;
      o = __builtin_fmaf(a.scale ? a.scale[d] : 1.f, o, r);
    }
    static_cast<Out*>(a.out)[base + int64_t(d) * a.L] = from_f<Out>(o);
  }
}

// (a column has a part of its own in `partial`: [workgroups][L][2][D])
template <typename T, typename R, bool POST, int NT>
__global__ __launch_bounds__(NT) void norm_bwd_flat_kernel(const NormArgs a) {
  using Out = typename NormTypes<T, R, POST>::Out;
  __shared__ float lds[flat_lds<NT, 2>()];
  const int tid = threadIdx.x, per = NT / a.L, used = per * a.L, l = tid % a.L, d0 = tid / a.L;
  float* pw = a.partial + (int64_t(blockIdx.x) * a.L + l) * 2 * a.D;
  float* ps = pw + a.D;
  for (int n = blockIdx.x; n < a.N; n += gridDim.x) {
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
    if (tid < used) {
      for (int d = d0; d < a.D; d += per) {
        const Elem e = read(d);
        s[0] = __builtin_fmaf(e.v, e.v, s[0]);
        s[1] = __builtin_fmaf(e.h, e.v, s[1]);
      }
    }
    flat_sums<NT, 2>(s, a.L, used, lds);
    if (tid < used) {
      const float rstd = __builtin_amdgcn_rsqf(__builtin_fmaf(s[0], a.inv_d, a.eps));
      const float m = s[1] * rstd * a.inv_d;
      for (int d = d0; d < a.D; d += per) {
        const Elem e = read(d);
        const int64_t at = base + int64_t(d) * a.L;
        const float ds = !POST && a.dsum ? to_f(static_cast<const R*>(a.dsum)[n * a.dsum_n + d * a.dsum_d + l]) : 0.f;
        float dx, dg, dr, dw = 0.f, dsc = 0.f;
        finish<T, R, POST>(e, rstd, m, a.scale ? a.scale[d] : 1.f, POST && a.gate, ds, &dx, &dg, &dr, &dw, &dsc);
        static_cast<T*>(a.dx)[at] = from_f<T>(dx);
        if (POST && a.gate) static_cast<T*>(a.dgate)[at] = from_f<T>(dg);
        if (!POST && a.dresidual) static_cast<R*>(a.dresidual)[at] = from_f<R>(dr);
        if (POST) dsc *= a.weight[d];
        const bool more = n != int(blockIdx.x);
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
    for (int p = wave; p < parts; p += 16) s += partial[(int64_t(p) * 2 + blockIdx.y) * D + d];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && d < D) {
#pragma unroll
    for (int w = 1; w < 16; ++w) s += lds[w][lane];
    (blockIdx.y ? dscale : dweight)[d] = s;
  }
}

struct Shape {
  bool flat;
  int nt, cl, hold;
  int64_t tiles, row_tiles;
  int wgs;  // backward
};
Shape shape_of(const seq_norm_t& p) {
  Shape s = {};
  s.flat = p.L <= kFlatMax;
  if (s.flat) {
    s.nt = int64_t(p.D) * p.L > 2048 ? 1024 : 256;
    s.wgs = p.N < 512 ? p.N : 512;
    return s;
  }
  s.cl = 8;
  while (s.cl > 2 && (p.L <= s.cl * 4 || p.N * ceil_div(p.L, s.cl * 8) < 256)) s.cl /= 2;
  s.nt = int64_t(p.D) * s.cl > 2048 ? 1024 : 256;
  s.hold = ceil_div(int64_t(p.D) * s.cl, s.nt) <= 8 ? 8 : 0;
  s.row_tiles = ceil_div(p.L, s.cl * 8);
  s.tiles = s.row_tiles * p.N;
  s.wgs = int(s.tiles < 512 ? s.tiles : 512);
  return s;
}

template <typename T, typename R, bool POST, int NT, int CL>
void launch_cl(const NormArgs& a, const Shape& sh, bool bwd, hipStream_t s) {
  if (bwd)
    norm_bwd_kernel<T, R, POST, NT, CL><<<dim3(sh.wgs), NT, 0, s>>>(a);
  else if (sh.hold)
    norm_fwd_kernel<T, R, POST, NT, CL, 8><<<dim3(uint32_t(sh.tiles)), NT, 0, s>>>(a);
  else
    norm_fwd_kernel<T, R, POST, NT, CL, 0><<<dim3(uint32_t(sh.tiles)), NT, 0, s>>>(a);
}
template <typename T, typename R, bool POST, int NT>
void launch_nt(const NormArgs& a, const Shape& sh, bool bwd, hipStream_t s) {
  if (sh.flat) {
    if (bwd)
      norm_bwd_flat_kernel<T, R, POST, NT><<<dim3(sh.wgs), NT, 0, s>>>(a);
    else
      norm_fwd_flat_kernel<T, R, POST, NT><<<dim3(a.N), NT, 0, s>>>(a);
    return;
  }
  switch (sh.cl) {
    case 2: launch_cl<T, R, POST, NT, 2>(a, sh, bwd, s); break;
    case 4: launch_cl<T, R, POST, NT, 4>(a, sh, bwd, s); break;
    default: launch_cl<T, R, POST, NT, 8>(a, sh, bwd, s); break;
  }
}
template <typename T, typename R, bool POST>
int run(const seq_norm_t& p, bool bwd, hipStream_t s) {
  const Shape sh = shape_of(p);
  if ((sh.flat ? int64_t(p.N) : sh.tiles) * sh.nt > kMaxThreads) return CONV_ERANGE;
  NormArgs a = {};
  a.N = p.N, a.D = p.D, a.L = p.L, a.eps = p.eps, a.inv_d = 1.f / float(p.D);
  a.x_n = p.x_n, a.x_d = p.x_d, a.gate_n = p.gate_n, a.gate_d = p.gate_d, a.res_n = p.res_n, a.res_d = p.res_d;
  a.dout_n = p.dout_n, a.dout_d = p.dout_d, a.dsum_n = p.dsum_n, a.dsum_d = p.dsum_d;
  a.x = p.x, a.weight = p.weight, a.scale = p.scale, a.gate = p.gate, a.residual = p.residual;
  a.out = p.out, a.sum = p.sum, a.dout = p.dout, a.dsum = p.dsum;
  a.dx = p.dx, a.dgate = p.dgate, a.dresidual = p.dresidual;
  a.partial = static_cast<float*>(p.workspace);
  a.tiles = uint32_t(sh.tiles), a.row_tiles = uint32_t(sh.row_tiles);
  if (bwd) {
    if (!p.workspace) return CONV_ENULL;
    if (p.workspace_bytes < norm_bwd_workspace(p)) return CONV_ESCRATCH;
  }
  if (sh.nt == 1024)
    launch_nt<T, R, POST, 1024>(a, sh, bwd, s);
  else
    launch_nt<T, R, POST, 256>(a, sh, bwd, s);
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

int64_t norm_bwd_workspace(const seq_norm_t& p) {
  const Shape sh = shape_of(p);
  return int64_t(sh.wgs) * (sh.flat ? p.L : 1) * 2 * p.D * int64_t(sizeof(float));
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
