// The short causal convolution of each channel: forward, backward, one token.
//
//   p(t) = bias + sum_r w[r] e(t - (R-1) + r),   out = p or p sigmoid(p)
//
// with e = (initial state, x).  R <= 8 products an output leave it bound by
// memory: every tensor goes through once.  bf16 8 x 2048 x 2048, R = 4: forward
// 27 us (134 MB, 5.0 TB/s), backward 50 us (201 MB, 4.0 TB/s); a copy of this
// size from memory reaches 5.3 TB/s.
#include <type_traits>

#include "seq_device.h"
#include "seq_internal.h"

namespace seqops {
namespace {

// x / d for x < 2^32 by a multiplication: m = floor(2^(32+s) / d) + 1 - 2^32
// with s = ceil(log2 d) (Granlund and Montgomery, division by invariants).
struct FastDiv {
  uint32_t d, m, s;
};
FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while ((uint64_t(1) << s) < d) ++s;
  return {d, uint32_t((((uint64_t(1) << 32) * ((uint64_t(1) << s) - d)) / d) + 1), s};
}
__device__ __forceinline__ uint32_t quot(FastDiv f, uint32_t x) {
  const uint32_t h = __umulhi(f.m, x);
  return f.s ? (h + ((x - h) >> 1)) >> (f.s - 1) : x;
}

template <typename T>
struct ConvArgs {
  int N, D, L;
  int silu;
  int64_t x_n, x_d, dout_n, dout_d;
  const T* x;
  const float *weight, *bias;
  const T* initial;
  const int32_t* lengths;
  T *out, *final_state;
  const T *dout, *dfinal;
  T* dx;
  float *dweight, *dbias;
  T* dinitial;
  FastDiv tiles;   // threads (backward: segments) a row
  FastDiv dim;     // D
  uint32_t items;  // threads in all; backward: segments of a channel
  int parts, seg_tiles;  // backward
  float* partial;
};

// e(t) for a t that may lie before the sequence.
template <typename T, int R>
__device__ __forceinline__ T entry(const T* x, const T* init, int t) {
  if (t >= 0) return x[t];
  return R > 1 && init ? init[t + R - 1] : T{};
}

// The entries t0 - 8 .. t0 - 1 (of which the last R - 1 count); t0 is a
// multiple of 8.
template <typename T, int R>
__device__ __forceinline__ void before8(const T* x, const T* init, int t0, int len, float* e) {
  if (t0 > 0) {
    unpack8(load8(x + t0 - 8, len - (t0 - 8)), e);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) e[j] = R > 1 && init && j >= 9 - R ? to_f(init[j + R - 9]) : 0.f;
}

// A thread makes eight outputs of one row: it reads their entries and the eight
// before them (the neighbour's, from L1), both as single loads.
template <typename T, int R>
__global__ __launch_bounds__(256) void conv_fwd_kernel(const ConvArgs<T> a) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.items) return;
  const uint32_t row = quot(a.tiles, i);
  const int t0 = int(i - row * a.tiles.d) * 8;
  const uint32_t n = quot(a.dim, row), d = row - n * a.dim.d;
  const int len = seq_len(a.lengths, n, a.L);
  const T* x = a.x + n * a.x_n + d * a.x_d;
  const T* init = a.initial ? a.initial + int64_t(row) * (R - 1) : nullptr;
  float v[8];
  if (t0 < len) {
    float e[16], w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = a.weight[int64_t(d) * R + r];
    const float b = a.bias ? a.bias[d] : 0.f;
    const Raw8<T> cur = load8(x + t0, len - t0);
    if (R > 1) before8<T, R>(x, init, t0, len, e);
    unpack8(cur, e + 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float p = b;
#pragma unroll
      for (int r = 0; r < R; ++r) p = __builtin_fmaf(w[r], e[j + r + 9 - R], p);
      v[j] = t0 + j < len ? (a.silu ? p * sigmoid(p) : p) : 0.f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
  }
  store8<true>(a.out + int64_t(row) * a.L + t0, a.L - t0, v);
  // the thread of the last step (of an empty sequence: the first thread)
  const int last = len > 0 ? len - 1 : 0;
  if (R > 1 && a.final_state && t0 == last / 8 * 8) {
#pragma unroll
    for (int k = 0; k < R - 1; ++k)
      a.final_state[int64_t(row) * (R - 1) + k] = entry<T, R>(x, init, len - (R - 1) + k);
  }
}

template <typename T, int R>
__global__ __launch_bounds__(256) void conv_step_kernel(const ConvArgs<T> a) {
  const uint32_t row = blockIdx.x * 256 + threadIdx.x;
  if (row >= a.items) return;
  const uint32_t n = quot(a.dim, row), d = row - n * a.dim.d;
  T e[R];
#pragma unroll
  for (int k = 0; k < R - 1; ++k) e[k] = a.initial[int64_t(row) * (R - 1) + k];
  e[R - 1] = a.x[n * a.x_n + d * a.x_d];
  float p = a.bias ? a.bias[d] : 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) p = __builtin_fmaf(a.weight[int64_t(d) * R + r], to_f(e[r]), p);
  a.out[row] = from_f<T>(a.silu ? p * sigmoid(p) : p);
  if (a.final_state) {
#pragma unroll
    for (int k = 0; k < R - 1; ++k) a.final_state[int64_t(row) * (R - 1) + k] = e[k + 1];
  }
}

// Backward.  With q(t) = dout(t) act'(p(t)) (zero outside 0..len-1),
//
//   de(j) = sum_r w[r] q(j + R-1 - r) + dfinal(j - len + R-1),
//   dw[r] = sum q(t) e(t - (R-1) + r),  db = sum q.
//
// A wave takes a row's segment from right to left, 512 steps at a time: the q
// that a lane's last gradients need are its right neighbour's first, and the
// last lane's are the first lane's of the step before, so q is formed once.
// The weights' sums stay in registers over all the wave's rows; a workgroup
// belongs to one channel, its four waves' sums are added in order, and where a
// channel has several workgroups (`parts`: few channels) a second kernel adds
// theirs in order.
template <typename T, int R>
__global__ __launch_bounds__(256) void conv_bwd_kernel(const ConvArgs<T> a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t part = quot(a.dim, blockIdx.x), d = blockIdx.x - part * a.dim.d;
  float w[R], dw[R], db = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    w[r] = a.weight[int64_t(d) * R + r];
    dw[r] = 0.f;
  }
  const float b = a.bias ? a.bias[d] : 0.f;
  for (uint32_t item = part * 4 + wave; item < a.items; item += a.parts * 4) {
    const uint32_t n = quot(a.tiles, item), seg = item - n * a.tiles.d;
    const int len = seq_len(a.lengths, n, a.L);
    const int64_t row = int64_t(n) * a.D + d;
    const T* x = a.x + n * a.x_n + d * a.x_d;
    const T* dout = a.dout + n * a.dout_n + d * a.dout_d;
    const T* init = a.initial ? a.initial + row * (R - 1) : nullptr;
    const T* dfin = R > 1 && a.dfinal ? a.dfinal + row * (R - 1) : nullptr;
    T* dx = a.dx + row * a.L;
    const int64_t seg_steps = int64_t(a.seg_tiles) * 512;
    const int lo = int(int(seg) * seg_steps);  // (below L: no segment is empty)
    const int hi = int(lo + seg_steps < a.L ? lo + seg_steps : a.L);
    // the q behind the segment: lane i makes the i-th
    float next[8];
    {
      float q = 0.f;
      const int t = hi + lane;
      if (lane < R - 1 && t < len) {
        float p = b;
#pragma unroll
        for (int r = 0; r < R; ++r) p = __builtin_fmaf(w[r], to_f(entry<T, R>(x, init, t - (R - 1) + r)), p);
        q = to_f(dout[t]);
        if (a.silu) {
          const float s = sigmoid(p);
          q *= s * (1.f + p * (1.f - s));
        }
      }
#pragma unroll
      for (int k = 0; k < R - 1; ++k) next[k] = __shfl(q, k);
    }
    // (a tile inside the sequence needs no masks)
    auto step = [&](int tile, auto inside) {
      constexpr bool kInside = decltype(inside)::value;
      const int t0 = tile + lane * 8;
      float e[16], q[16];
      unpack8(load8(x + t0, len - t0), e + 8);
      if (R > 1) {
        if (kInside || t0 < len + 8)
          before8<T, R>(x, init, t0, len, e);
        else
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = 0.f;
      }
      unpack8(load8(dout + t0, len - t0), q);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool ok = kInside || t0 + j < len;
        if (a.silu) {
          float p = b;
#pragma unroll
          for (int r = 0; r < R; ++r) p = __builtin_fmaf(w[r], e[j + r + 9 - R], p);
          const float s = sigmoid(p);
          q[j] *= s * (1.f + p * (1.f - s));
        }
        q[j] = ok ? q[j] : 0.f;
        db += q[j];
#pragma unroll
        for (int r = 0; r < R; ++r) dw[r] = __builtin_fmaf(q[j], ok ? e[j + r + 9 - R] : 0.f, dw[r]);
      }
#pragma unroll
      for (int k = 0; k < R - 1; ++k) {
        q[8 + k] = dpp<kWaveShl1>(next[k], q[k]);
        next[k] = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(q[k])));
      }
      float g[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        g[j] = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) g[j] = __builtin_fmaf(w[r], q[j + R - 1 - r], g[j]);
        const int k = t0 + j - len + R - 1;
        if (dfin && k >= 0 && k < R - 1) g[j] += to_f(dfin[k]);
        if (!kInside && t0 + j >= len) g[j] = 0.f;
      }
      store8<true>(dx + t0, a.L - t0, g);
      if (R > 1 && t0 == 0 && a.dinitial) {
#pragma unroll
        for (int i = 0; i < R - 1; ++i) {
          float s = 0.f;
#pragma unroll
          for (int r = 0; r <= i; ++r) s = __builtin_fmaf(w[r], q[i - r], s);
          if (dfin && i >= len) s += to_f(dfin[i - len]);
          a.dinitial[row * (R - 1) + i] = from_f<T>(s);
        }
      }
    };
    for (int tile = (hi - 1) / 512 * 512; tile >= lo; tile -= 512) {
      if (tile + 512 <= len)
        step(tile, std::true_type{});
      else
        step(tile, std::false_type{});
    }
  }
  __shared__ float sums[4][R + 1];
#pragma unroll
  for (int r = 0; r <= R; ++r) {
    float s = r < R ? dw[r < R ? r : 0] : db;
    for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
    if (lane == 0) sums[wave][r] = s;
  }
  __syncthreads();
  if (threadIdx.x <= R) {
    const int r = threadIdx.x;
    const float s = (sums[0][r] + sums[1][r]) + (sums[2][r] + sums[3][r]);
    if (a.parts > 1)
      a.partial[(int64_t(part) * a.D + d) * (R + 1) + r] = s;
    else if (r < R)
      a.dweight[int64_t(d) * R + r] = s;
    else if (a.dbias)
      a.dbias[d] = s;
  }
}

// Adds the parts' sums in order.
__global__ __launch_bounds__(64) void conv_sum_kernel(const float* partial, int parts, int D, int R, float* dweight,
                                                      float* dbias) {
  const int64_t i = int64_t(blockIdx.x) * 64 + threadIdx.x;
  if (i >= int64_t(D) * (R + 1)) return;
  float s = 0.f;
  for (int p = 0; p < parts; ++p) s += partial[p * int64_t(D) * (R + 1) + i];
  const int64_t d = i / (R + 1);
  const int r = int(i - d * (R + 1));
  if (r < R)
    dweight[d * R + r] = s;
  else if (dbias)
    dbias[d] = s;
}

struct BwdSplit {
  int parts, segs, seg_tiles;
};
// Workgroups a channel: one while there are 1024 channels or more (four waves
// each fill the chip's 1024 SIMDs four times); fewer channels are split, down
// to one tile of 512 steps a wave.
BwdSplit bwd_split(const seq_conv_t& p) {
  const int64_t tiles = ceil_div(p.L, 512);
  int64_t parts = ceil_div(1024, p.D);
  const int64_t most = ceil_div(p.N * tiles, 4);
  if (parts > most) parts = most;
  int64_t segs = ceil_div(parts * 4, p.N);
  if (segs > tiles) segs = tiles;
  const int64_t seg_tiles = ceil_div(tiles, segs);
  return {int(parts), int(ceil_div(tiles, seg_tiles)), int(seg_tiles)};
}

template <typename T>
ConvArgs<T> args_of(const seq_conv_t& p) {
  ConvArgs<T> a = {};
  a.N = p.N, a.D = p.D, a.L = p.L, a.silu = p.activation == SEQ_ACT_SILU;
  a.x_n = p.x_n, a.x_d = p.x_d, a.dout_n = p.dout_n, a.dout_d = p.dout_d;
  a.x = static_cast<const T*>(p.x), a.weight = p.weight, a.bias = p.bias;
  a.initial = static_cast<const T*>(p.initial_state), a.lengths = p.lengths;
  a.out = static_cast<T*>(p.out), a.final_state = static_cast<T*>(p.final_state);
  a.dout = static_cast<const T*>(p.dout), a.dfinal = static_cast<const T*>(p.dfinal_state);
  a.dx = static_cast<T*>(p.dx), a.dweight = p.dweight, a.dbias = p.dbias;
  a.dinitial = static_cast<T*>(p.dinitial_state);
  a.dim = fast_div(uint32_t(p.D));
  return a;
}

enum Kind { kFwd, kBwd, kStep };
template <typename T, int R>
void launch_r(Kind kind, const ConvArgs<T>& a, hipStream_t s) {
  if (kind == kBwd)
    conv_bwd_kernel<T, R><<<dim3(uint32_t(int64_t(a.D) * a.parts)), 256, 0, s>>>(a);
  else if (kind == kFwd)
    conv_fwd_kernel<T, R><<<dim3((a.items - 1) / 256 + 1), 256, 0, s>>>(a);
  else
    conv_step_kernel<T, R><<<dim3((a.items - 1) / 256 + 1), 256, 0, s>>>(a);
}
template <typename T>
int launch_t(Kind kind, int R, const ConvArgs<T>& a, hipStream_t s) {
  switch (R) {
    case 1: launch_r<T, 1>(kind, a, s); break;
    case 2: launch_r<T, 2>(kind, a, s); break;
    case 3: launch_r<T, 3>(kind, a, s); break;
    case 4: launch_r<T, 4>(kind, a, s); break;
    case 5: launch_r<T, 5>(kind, a, s); break;
    case 6: launch_r<T, 6>(kind, a, s); break;
    case 7: launch_r<T, 7>(kind, a, s); break;
    default: launch_r<T, 8>(kind, a, s); break;
  }
  return hipGetLastError() == hipSuccess ? CONV_OK : CONV_EHIP;
}

template <typename T>
int fwd(const seq_conv_t& p, hipStream_t s) {
  ConvArgs<T> a = args_of<T>(p);
  const int64_t tiles = ceil_div(p.L, 8), items = int64_t(p.N) * p.D * tiles;
  if (items > kMaxThreads - 255) return CONV_ERANGE;
  a.tiles = fast_div(uint32_t(tiles));
  a.items = uint32_t(items);
  return launch_t(kFwd, p.R, a, s);
}
template <typename T>
int step(const seq_conv_t& p, hipStream_t s) {
  ConvArgs<T> a = args_of<T>(p);
  const int64_t items = int64_t(p.N) * p.D;
  if (items > kMaxThreads - 255) return CONV_ERANGE;
  a.items = uint32_t(items);
  return launch_t(kStep, p.R, a, s);
}
template <typename T>
int bwd(const seq_conv_t& p, hipStream_t s) {
  ConvArgs<T> a = args_of<T>(p);
  const BwdSplit sp = bwd_split(p);
  const int64_t items = int64_t(p.N) * sp.segs;
  if (int64_t(p.D) * sp.parts * 256 > kMaxThreads || items >= int64_t(1) << 31) return CONV_ERANGE;
  if (sp.parts > 1 && p.workspace_bytes < conv_bwd_workspace(p)) return CONV_ESCRATCH;
  if (sp.parts > 1 && !p.workspace) return CONV_ENULL;
  a.parts = sp.parts, a.seg_tiles = sp.seg_tiles;
  a.tiles = fast_div(uint32_t(sp.segs)), a.items = uint32_t(items);
  a.partial = static_cast<float*>(p.workspace);
  const int rc = launch_t(kBwd, p.R, a, s);
  if (rc != CONV_OK || sp.parts == 1) return rc;
  conv_sum_kernel<<<dim3(uint32_t(ceil_div(int64_t(p.D) * (p.R + 1), 64))), 64, 0, s>>>(
      a.partial, sp.parts, p.D, p.R, p.dweight, p.dbias);
  return hipGetLastError() == hipSuccess ? CONV_OK : CONV_EHIP;
}
}  // namespace

int64_t conv_bwd_workspace(const seq_conv_t& p) {
  const int parts = bwd_split(p).parts;
  return parts > 1 ? int64_t(parts) * p.D * (p.R + 1) * int64_t(sizeof(float)) : 0;
}
int launch_conv_fwd(const seq_conv_t& p, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p.dtype == CONV_DTYPE_BF16 ? fwd<bf16>(p, s) : fwd<float>(p, s);
}
int launch_conv_bwd(const seq_conv_t& p, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p.dtype == CONV_DTYPE_BF16 ? bwd<bf16>(p, s) : bwd<float>(p, s);
}
int launch_conv_step(const seq_conv_t& p, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p.dtype == CONV_DTYPE_BF16 ? step<bf16>(p, s) : step<float>(p, s);
}

}  // namespace seqops
