// The selective scan: forward, backward, one token.
//
//   h[s](t) = a[s](t) h[s](t-1) + x(t) B[s](t),  a = exp(dt A[s]),  x = dt u
//   y(t) = sum_s C[s](t) h[s](t) + Dskip u(t),   out = y z sigmoid(z)
//
// A step of a state is an exponential (two issue slots) and five products and
// multiply-adds, S of them for every element read: bound by the vector ALU.
// The recurrence is composed along the length.  A row of sixteen lanes takes a
// channel, 8 or 16 steps a lane; each lane folds its steps (state from zero,
// and the decay over them), the pairs (decay, state) are scanned over the row
// by DPP in four levels, and each lane runs its steps again from the state that
// reaches it.  So a step's exponential and products are formed once, the scan
// costs a lane eight instructions, and only dt, x and y of the lane's steps are
// held over the states, which go two at a time.  A wave is four channels; a
// workgroup's channels are of one group and share B and C, staged in LDS as
// fp32, the next pass's under way meanwhile.  Workgroups walk along the length.
// Where rows are too few to fill the chip, a channel has all 64 lanes (short
// lengths), or the length is cut into segments: a first launch finds what each
// segment alone makes of a zero state, the second composes those before its own.
//
// Forward, bf16, 4 x 2048 x 2048 with 16 states and gate (2^28 steps of states):
// 89 us, 10.4 issue slots a step of a state (7 of them the recurrence itself),
// slots in use 82% of the time.  1 x 1024 x 16384 (2^28 too, cut into 8): 146 us.
#include <type_traits>

#include "seq_device.h"
#include "seq_internal.h"
#include "seq_shape.h"

namespace seqops {
namespace {

template <typename T>
struct ScanArgs {
  int N, D, L, S, G, per;  // per: channels of a group
  int softplus;
  int blks, segs, seg_chunks, chunks;
  int run_segs, run_first;  // the segments that a launch works on
  int batch;  // backward: states between two exchanges of dB and dC, a power of 2
  int64_t u_n, u_d, delta_n, delta_d, z_n, z_d, dout_n, dout_d, B_n, B_g, B_s, C_n, C_g, C_s;
  const T *u, *delta, *z, *B, *C;
  const float *A, *Dskip, *bias, *initial;
  const int32_t* lengths;
  T* out;
  float *final_state, *checkpoints;
  const T* dout;
  const float* dfinal;
  T *du, *ddelta, *dz, *dB, *dC;
  float *dA, *dD, *dbias, *dinitial;
  // scratch
  int fine, fine_chunks;   // pieces of a segment whose ends are found; their chunks
  float *ends, *end_dt;    // [N][segs * fine][D][S], [N][segs * fine][D]
  float* part_bc;          // [N][G][blks][S][2][chunks * 128], a chunk's steps as in LDS
  float *part_A, *part_D;  // [N][segs][D][S], [N][segs][D][2] (Dskip, delta_bias)
};

// Where a thread stands: a wave of RW channels, 64 / RW lanes each.
struct Place {
  int lane, wave, row, tl;
  int n, g, blk, seg;
  int d0;    // the wave's first channel
  int held;  // how many of its channels there are (may be none)
  int d;     // the row's channel; one that exists, if its own does not
  bool ok;
};
template <int RW, typename T>
__device__ __forceinline__ Place place(const ScanArgs<T>& a) {
  Place p;
  p.lane = threadIdx.x & 63;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  p.row = p.lane / (64 / RW), p.tl = p.lane % (64 / RW);
  uint32_t b = blockIdx.x;
  p.blk = int(b % a.blks), b /= a.blks;
  p.g = int(b % a.G), b /= a.G;
  p.seg = int(b % a.run_segs) + a.run_first, p.n = int(b / a.run_segs);
  const int cw = (p.blk * int(blockDim.x >> 6) + p.wave) * RW, left = a.per - cw;
  p.held = left < 0 ? 0 : left < RW ? left : RW;
  p.d0 = p.g * a.per + cw;
  p.ok = p.row < left;
  p.d = p.ok ? p.d0 + p.row : p.g * a.per + a.per - 1;
  return p;
}

// B (and C) of the steps that a workgroup works on, TS for each of the LN lanes
// of a channel, in LDS: a state's steps in runs of 4 LN, four of every lane, so
// that a lane's reads are whole 16-byte banks next to its neighbours'.
template <typename T, int LN, int TS, int NB>
struct Stage {
  Raw8<T> raw[NB];
  // rows 0..S-1 are first's states, the others second's
  __device__ __forceinline__ void load(const T* first, int64_t first_s, const T* second, int64_t second_s, int S,
                                       int rows, int t0, int len) {
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int i = threadIdx.x + k * blockDim.x, r = i / (LN * TS / 8), t = t0 + i % (LN * TS / 8) * 8;
      if (r < rows) raw[k] = load8((r < S ? first + r * first_s : second + (r - S) * second_s) + t, len - t);
    }
  }
  __device__ __forceinline__ void store(float* lds, int rows) const {
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int i = threadIdx.x + k * blockDim.x, r = i / (LN * TS / 8), e = i % (LN * TS / 8);
      if (r < rows) {
        float v[8];
        unpack8(raw[k], v);
        float* at = lds + r * (LN * TS) + (TS == 8 ? e * 4 : (e & 1) * (8 * LN) + (e >> 1) * 4);
        *reinterpret_cast<f32x4*>(at) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(at + 4 * LN) = f32x4{v[4], v[5], v[6], v[7]};
      }
    }
  }
};
template <int LN, int TS>
__device__ __forceinline__ void lds_steps(const float* lds, int tl, float* v) {
#pragma unroll
  for (int k = 0; k < TS / 4; ++k) {
    const f32x4 q = *reinterpret_cast<const f32x4*>(lds + k * 4 * LN + tl * 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[k * 4 + j] = q[j];
  }
}

// The states that reach each lane, for two states at once: H (a lane's steps
// from zero; lane 0 has its incoming state in them) and P (their decay) are
// composed in levels of 1, 2, 4 and 8 lanes, then from row to row where a channel
// has the whole wave.  (So P is of kChunk steps at most: decays that overflow over
// more of them stay out.)  A lane without a source is left as it is.  H
// becomes the state behind each lane, `in` the one before it (lane 0: kept).
// Written as DPP operands, which the compiler makes moves of; a DPP source has
// to be two instructions old, which the two chains are to one another.
#define SEQ_DPP2(OP, X, Y, CTRL)                \
  OP " %" #X ", %" #X ", %2 " CTRL "\n" OP " %" #Y ", %" #Y ", %3 " CTRL "\n"
#define SEQ_LEVEL(CTRL) SEQ_DPP2("v_fmac_f32_dpp", 0, 1, CTRL) SEQ_DPP2("v_mul_f32_dpp", 2, 3, CTRL)
#define SEQ_ROW(DIR, K) DIR ":" #K " row_mask:0xf bank_mask:0xf"
#define SEQ_ROW_LEVELS(DIR) \
  "s_nop 1\n" SEQ_LEVEL(SEQ_ROW(DIR, 1)) SEQ_LEVEL(SEQ_ROW(DIR, 2)) SEQ_LEVEL(SEQ_ROW(DIR, 4))
#define SEQ_SHIFT(CTRL)                                   \
  "s_nop 0\n"                                             \
  "v_mov_b32_dpp %4, %0 " CTRL " row_mask:0xf bank_mask:0xf\n" \
  "v_mov_b32_dpp %5, %1 " CTRL " row_mask:0xf bank_mask:0xf\n" \
  "s_nop 1\n"
#define SEQ_SCAN_OPERANDS "+v"(H[0]), "+v"(H[1]), "+v"(P[0]), "+v"(P[1]), "+v"(in[0]), "+v"(in[1])
template <int LN>
__device__ __forceinline__ void scan_lanes(float* H, float* P, float* in) {
  if constexpr (LN == 16)
    asm volatile(SEQ_ROW_LEVELS("row_shr") SEQ_DPP2("v_fmac_f32_dpp", 0, 1, SEQ_ROW("row_shr", 8))
                     SEQ_SHIFT("row_shr:1")
                 : SEQ_SCAN_OPERANDS);
  else
    asm volatile(SEQ_ROW_LEVELS("row_shr") SEQ_LEVEL(SEQ_ROW("row_shr", 8))
                     SEQ_DPP2("v_fmac_f32_dpp", 0, 1, "row_bcast:15 row_mask:0x2 bank_mask:0xf")
                         "s_nop 0\n" SEQ_DPP2("v_fmac_f32_dpp", 0, 1, "row_bcast:15 row_mask:0x4 bank_mask:0xf")
                             "s_nop 0\n" SEQ_DPP2("v_fmac_f32_dpp", 0, 1, "row_bcast:15 row_mask:0x8 bank_mask:0xf")
                                 SEQ_SHIFT("wave_shr:1")
                 : SEQ_SCAN_OPERANDS);
}
// The same from right to left (lane 15 keeps its `in`), rows of sixteen.
__device__ __forceinline__ void scan_lanes_back(float* H, float* P, float* in) {
  asm volatile(SEQ_ROW_LEVELS("row_shl") SEQ_DPP2("v_fmac_f32_dpp", 0, 1, SEQ_ROW("row_shl", 8))
                   SEQ_SHIFT("row_shl:1")
               : SEQ_SCAN_OPERANDS);
}
// A row's sum in its lane 15.
__device__ __forceinline__ float row_sum(float v) {
  v += dpp0<kRowShr + 1>(v);
  v += dpp0<kRowShr + 2>(v);
  v += dpp0<kRowShr + 4>(v);
  v += dpp0<kRowShr + 8>(v);
  return v;
}

// h (or a gradient) as the pieces of segments from `from` to before `to` in turn
// leave it; `at` is the state's place in a piece's `ends`, d its channel.
template <typename T>
__device__ __forceinline__ float through(const ScanArgs<T>& a, int n, int from, int to, int step, int64_t at, int d,
                                         float A2, float h) {
  const int64_t first = int64_t(n) * a.segs * a.fine + from;
  const float *dt = a.end_dt + first * a.D + d, *end = a.ends + first * a.D * a.S + at;
  const int64_t dt_step = int64_t(step) * a.D, end_step = dt_step * a.S;
#pragma unroll 4
  for (int k = from; k != to; k += step, dt += dt_step, end += end_step)
    h = times_exp2(h, A2 * *dt) + *end;
  return h;
}

// A as the exponent of 2.  Minus infinity (a state without memory) becomes the
// lowest finite number, so that a step of length zero leaves the state as it is.
__device__ __forceinline__ float decay2(float A) {
  const float A2 = kLog2e * A;
  return A2 < -__FLT_MAX__ ? -__FLT_MAX__ : A2;  // (NaN: kept)
}

// dt of a lane's steps and its sum.  `full`: no step of the workgroup's is
// behind the end; else those have dt = 0 (the state stands still).
template <typename T, int TS>
__device__ __forceinline__ float steps(const Raw8<T>* raw, float bias, bool soft, bool full, int valid, float* dt) {
#pragma unroll
  for (int k = 0; k < TS / 8; ++k) unpack8(raw[k], dt + 8 * k);
#pragma unroll
  for (int j = 0; j < TS; ++j) dt[j] += bias;
  if (soft) {
#pragma unroll
    for (int j = 0; j < TS; ++j) dt[j] = softplus(dt[j]);
  }
  if (!full) {
    branch();
#pragma unroll
    for (int j = 0; j < TS; ++j) dt[j] = j < valid ? dt[j] : 0.f;
  }
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < TS; ++j) sum += dt[j];
  return sum;
}

// A wave's values of four channels' states: [channel][S] in LDS as in memory,
// so entry e belongs to channel e / S.
template <typename T>
__device__ __forceinline__ int64_t state_at(const ScanArgs<T>& a, const Place& p, int64_t outer) {
  return (outer * a.D + p.d0) * a.S;
}

// RW channels a wave, LN = 64 / RW lanes each; TS steps a lane, LN TS a pass.
template <typename T, int RW, int TS, int NB>
__global__ __launch_bounds__(512) void scan_fwd_kernel(const ScanArgs<T> a) {
  extern __shared__ float lds[];
  constexpr int LN = 64 / RW, kSteps = LN * TS;
  constexpr int kPer = kSteps / kChunk, kLanes = kChunk / TS;  // checkpoints a pass, lanes to one
  const Place p = place<RW>(a);
  const int S = a.S, Se = (S + 1) & ~1, rows = 2 * S, lane = p.lane, row = p.row, tl = p.tl;
  const int len = seq_len(a.lengths, p.n, a.L), held = p.held;
  // (a segment is of whole passes)
  const int first = p.seg * a.seg_chunks * kChunk;
  const int stop = p.seg == a.segs - 1 ? a.L : first + a.seg_chunks * kChunk, end = len < stop ? len : stop;
  float* bc = lds;  // [2][rows], a row of zeros behind them
  float* zeros = bc + 2 * rows * kSteps;
  float* hs = zeros + kSteps + p.wave * (1 + kPer) * RW * Se;
  float *as = hs + RW * Se, *mid = as + RW * Se;  // mid: states at the checkpoints inside a pass
  for (int e = lane; e < RW * Se; e += 64) {
    const int r = e / Se, s = e - r * Se;
    float A2 = 0.f, h = 0.f;
    if (r < held) {
      const int64_t at = state_at(a, p, 0) + int64_t(r) * S + s;
      A2 = decay2(a.A[s < S ? at : at - 1]);
      if (s < S && a.initial) h = a.initial[int64_t(p.n) * a.D * S + at];
      if (s < S && p.seg) h = through(a, p.n, 0, p.seg * a.fine, 1, at, p.d0 + r, A2, h);
    }
    as[e] = A2;
    hs[e] = h;
  }
  for (int e = threadIdx.x; e < kSteps; e += blockDim.x) zeros[e] = 0.f;
  // entry e of [channel][S] in memory, from an array of [channel][Se]
  auto put = [&](float* to, const float* from) {
    for (int e = lane; e < held * S; e += 64) to[e] = from[e + e / S * (Se - S)];
  };
  const T* up = a.u + p.n * a.u_n + p.d * a.u_d + tl * TS;
  const T* dp = a.delta + p.n * a.delta_n + p.d * a.delta_d + tl * TS;
  const T* zp = a.z ? a.z + p.n * a.z_n + p.d * a.z_d + tl * TS : nullptr;
  const T* Bp = a.B + p.n * a.B_n + p.g * a.B_g;
  const T* Cp = a.C + p.n * a.C_n + p.g * a.C_g;
  const float skip = a.Dskip ? a.Dskip[p.d] : 0.f, bias = a.bias ? a.bias[p.d] : 0.f;
  T* op = a.out + (int64_t(p.n) * a.D + p.d) * a.L + tl * TS;
  Stage<T, LN, TS, NB> st;
  Raw8<T> ru[TS / 8] = {}, rd[TS / 8] = {}, rz[TS / 8] = {};
  auto fetch = [&](const T* from, int t0, Raw8<T>* r) {
#pragma unroll
    for (int k = 0; k < TS / 8; ++k) r[k] = load8(from + t0 + 8 * k, len - t0 - tl * TS - 8 * k);
  };
  if (first < end) {
    st.load(Bp, a.B_s, Cp, a.C_s, S, rows, first, len);
    fetch(up, first, ru);
    fetch(dp, first, rd);
    st.store(bc, rows);
  }
  __syncthreads();
  int buf = 0;
  for (int t0 = first; t0 < end; t0 += kSteps) {
    const int valid = len - t0 - tl * TS;
    const float* cur = bc + buf * rows * kSteps;
    const bool more = t0 + kSteps < end, full = t0 + kSteps <= len;
    if (a.checkpoints)
      put(a.checkpoints + state_at(a, p, int64_t(p.n) * a.chunks + t0 / kChunk), hs);
    float dt[TS], x[TS], y[TS];
    const float sum = steps<T, TS>(rd, bias, a.softplus, full, valid, dt);
#pragma unroll
    for (int k = 0; k < TS / 8; ++k) unpack8(ru[k], x + 8 * k);
#pragma unroll
    for (int j = 0; j < TS; ++j) {
      y[j] = skip * x[j];
      x[j] *= dt[j];
    }
    if (more) {
      st.load(Bp, a.B_s, Cp, a.C_s, S, rows, t0 + kSteps, len);
      fetch(up, t0 + kSteps, ru);
      fetch(dp, t0 + kSteps, rd);
    }
    if (zp) fetch(zp, t0, rz);
    for (int s = 0; s < S; s += 2) {
      // (with S odd the last state's pair has its decay and reads zeros: it is not
      // finite only where that state is not)
      const bool two = s + 1 < S;
      const float *b0 = cur + s * kSteps, *b1 = two ? b0 + kSteps : zeros;
      float w[2][TS], b[2][TS], A2[2], in[2], H[2], P[2];
      lds_steps<LN, TS>(b0, tl, b[0]);
      lds_steps<LN, TS>(b1, tl, b[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        A2[i] = as[row * Se + s + i];
        in[i] = hs[row * Se + s + i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) P[i] = exp2_fast(sum * A2[i]);
#pragma unroll
      for (int j = 0; j < TS; ++j) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          w[i][j] = exp2_fast(dt[j] * A2[i]);
          b[i][j] *= x[j];
          H[i] = j ? __builtin_fmaf(w[i][j], H[i], b[i][j]) : b[i][j];
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) H[i] = __builtin_fmaf(P[i], tl == 0 ? in[i] : 0.f, H[i]);
      scan_lanes<LN>(H, P, in);
      float c[2][TS];
      lds_steps<LN, TS>(b0 + S * kSteps, tl, c[0]);
      lds_steps<LN, TS>(two ? b0 + (S + 1) * kSteps : zeros, tl, c[1]);
#pragma unroll
      for (int j = 0; j < TS; ++j) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          in[i] = __builtin_fmaf(w[i][j], in[i], b[i][j]);
          y[j] = __builtin_fmaf(in[i], c[i][j], y[j]);
        }
      }
      if (tl % kLanes == kLanes - 1) {
        float* to = (tl == LN - 1 ? hs : mid + tl / kLanes * RW * Se) + row * Se + s;
        to[0] = in[0], to[1] = in[1];
      }
    }
    if (kPer > 1 && a.checkpoints) {
      wave_sync();
      for (int k = 1; k < kPer && t0 + k * kChunk < end; ++k)
        put(a.checkpoints + state_at(a, p, int64_t(p.n) * a.chunks + t0 / kChunk + k), mid + (k - 1) * RW * Se);
    }
    if (p.ok) {
#pragma unroll
      for (int k = 0; k < TS / 8; ++k) {
        float* yk = y + 8 * k;
        if (zp) {
          float z[8];
          unpack8(rz[k], z);
#pragma unroll
          for (int j = 0; j < 8; ++j) yk[j] *= z[j] * sigmoid(z[j]);
        }
        if (!full) {
          branch();
#pragma unroll
          for (int j = 0; j < 8; ++j) yk[j] = 8 * k + j < valid ? yk[j] : 0.f;
        }
        store8(op + t0 + 8 * k, a.L - t0 - tl * TS - 8 * k, yk);
      }
    }
    if (more) st.store(bc + (buf ^ 1) * rows * kSteps, rows);
    buf ^= 1;
    __syncthreads();
  }
  if (a.final_state && p.seg == a.segs - 1) put(a.final_state + state_at(a, p, p.n), hs);
  if (p.ok) {  // (passes behind the end)
    const float zero[8] = {};
    int t0 = first;
    if (end > first) t0 += (end - first + kSteps - 1) / kSteps * kSteps;
    for (; t0 < stop; t0 += kSteps)
#pragma unroll
      for (int k = 0; k < TS / 8; ++k) store8(op + t0 + 8 * k, stop - t0 - tl * TS - 8 * k, zero);
  }
}

// What a piece of a segment alone makes of a zero state, and its sum of dt: forward, h at
// its right end, the sum of x(t) B(t) exp(A (dt behind t)); BACK, r at its left
// end, the sum of dy(t) C(t) exp(A (dt up to and with t)).  The steps stand side
// by side, weighted with their decay to that end, so a state needs no scan, only
// a sum over the row; the decays' exponents are sums of dt, taken along as the
// passes walk away from the end.  Where those decays may grow (some A is positive, or
// without softplus a step negative) they can be past fp32 over a piece when they are
// not over kChunk steps, and go into each product without being formed.  A segment is
// cut further (`fine`), for more waves than the scan's registers allow: 1 x 1024 x
// 16384, 16 states, seven segments of eight, 63 us whole and 59 in two pieces each.
template <typename T, int TS, int NB, bool BACK>
__global__ __launch_bounds__(512) void scan_ends_kernel(const ScanArgs<T> a) {
  extern __shared__ float lds[];
  constexpr int kSteps = 16 * TS;
  const Place p = place<4>(a);
  const int S = a.S, Se = (S + 1) & ~1, lane = p.lane, row = p.row, tl = p.tl;
  const int len = seq_len(a.lengths, p.n, a.L);
  const int seg = p.seg / a.fine, piece = p.seg - seg * a.fine;  // (p.seg: of the pieces)
  const int c0 = seg * a.seg_chunks + piece * a.fine_chunks;
  const int cs = seg == a.segs - 1 ? a.chunks : (seg + 1) * a.seg_chunks;
  const int c1 = c0 + a.fine_chunks < cs ? c0 + a.fine_chunks : cs;
  const int64_t stop64 = int64_t(c1) * kChunk;
  const int first = c0 * kChunk, end = len < stop64 ? len : int(stop64);
  const int passes = end > first ? (end - first + kSteps - 1) / kSteps : 0;
  float* bc = lds;  // [2][S], a row of zeros behind them
  float* zeros = bc + 2 * S * kSteps;
  float* hs = zeros + kSteps + p.wave * 8 * Se;
  float* as = hs + 4 * Se;
  bool grow = false;  // (the wave's)
  for (int e = lane; e < 4 * Se; e += 64) {
    const int r = e / Se, s = e - r * Se;
    const float A2 = r < p.held && s < S ? decay2(a.A[state_at(a, p, 0) + int64_t(r) * S + s]) : 0.f;
    as[e] = A2;
    hs[e] = 0.f;
    grow |= A2 > 0.f;
  }
  grow = __any(grow);
  for (int e = threadIdx.x; e < kSteps; e += blockDim.x) zeros[e] = 0.f;
  const bool gate = BACK && a.z;
  const T* dp = a.delta + p.n * a.delta_n + p.d * a.delta_d + tl * TS;
  const T* vp = BACK ? a.dout + p.n * a.dout_n + p.d * a.dout_d + tl * TS : a.u + p.n * a.u_n + p.d * a.u_d + tl * TS;
  const T* zp = gate ? a.z + p.n * a.z_n + p.d * a.z_d + tl * TS : nullptr;
  const T* Mp = BACK ? a.C + p.n * a.C_n + p.g * a.C_g : a.B + p.n * a.B_n + p.g * a.B_g;
  const int64_t M_s = BACK ? a.C_s : a.B_s;
  const float bias = a.bias ? a.bias[p.d] : 0.f;
  Stage<T, 16, TS, NB> st;
  Raw8<T> rd[TS / 8] = {}, rv[TS / 8] = {}, rz[TS / 8] = {};
  auto at_pass = [&](int k) { return first + (BACK ? k : passes - 1 - k) * kSteps; };
  auto fetch = [&](int t0) {
    st.load(Mp, M_s, Mp, M_s, S, S, t0, end);
#pragma unroll
    for (int k = 0; k < TS / 8; ++k) {
      const int valid = end - t0 - tl * TS - 8 * k;
      rd[k] = load8(dp + t0 + 8 * k, valid);
      rv[k] = load8(vp + t0 + 8 * k, valid);
      if (gate) rz[k] = load8(zp + t0 + 8 * k, valid);
    }
  };
  if (passes) {
    fetch(at_pass(0));
    st.store(bc, S);
  }
  __syncthreads();
  float total = 0.f;  // dt of the passes behind
  for (int k = 0; k < passes; ++k) {
    const int t0 = at_pass(k);
    const float* cur = bc + (k & 1) * S * kSteps;
    float dt[TS], v[TS];
    const float sum = steps<T, TS>(rd, bias, a.softplus, t0 + kSteps <= end, end - t0 - tl * TS, dt);
#pragma unroll
    for (int i = 0; i < TS / 8; ++i) {
      unpack8(rv[i], v + 8 * i);
      if (gate) {
        float z[8];
        unpack8(rz[i], z);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * i + j] *= z[j] * sigmoid(z[j]);
      }
    }
    if (!BACK) {
#pragma unroll
      for (int j = 0; j < TS; ++j) v[j] *= dt[j];
    }
    if (!a.softplus && !grow) {
      bool negative = false;
#pragma unroll
      for (int j = 0; j < TS; ++j) negative |= dt[j] < 0.f;
      grow = __any(negative);
    }
    if (k + 1 < passes) fetch(at_pass(k + 1));
    // dt becomes each step's distance from the end: the lanes' sums first
    float lanes = sum;
    if (BACK) {
      lanes += dpp0<kRowShr + 1>(lanes);
      lanes += dpp0<kRowShr + 2>(lanes);
      lanes += dpp0<kRowShr + 4>(lanes);
      lanes += dpp0<kRowShr + 8>(lanes);
    } else {
      lanes += dpp0<kRowShl + 1>(lanes);
      lanes += dpp0<kRowShl + 2>(lanes);
      lanes += dpp0<kRowShl + 4>(lanes);
      lanes += dpp0<kRowShl + 8>(lanes);
    }
    float far = total + (BACK ? dpp0<kRowShr + 1>(lanes) : dpp0<kRowShl + 1>(lanes));
    total += __shfl(lanes, (lane & 48) + (BACK ? 15 : 0));
    if (BACK) {
#pragma unroll
      for (int j = 0; j < TS; ++j) dt[j] = far += dt[j];
    } else {
#pragma unroll
      for (int j = TS - 1; j >= 0; --j) {
        const float own = dt[j];
        dt[j] = far;
        far += own;
      }
    }
    if (grow) {  // (one state at a time: no more registers than below)
      for (int s = 0; s < S; ++s) {
        float m[TS], H = 0.f;
        const float A2 = as[row * Se + s];
        lds_steps<16, TS>(cur + s * kSteps, tl, m);
#pragma unroll
        for (int j = 0; j < TS; ++j) H += times_exp2(v[j] * m[j], dt[j] * A2);
        H = row_sum(H);
        if (tl == 15) hs[row * Se + s] += H;
      }
    } else {
      for (int s = 0; s < S; s += 2) {
        const float *m0 = cur + s * kSteps, *m1 = s + 1 < S ? m0 + kSteps : zeros;
        float m[2][TS], H[2] = {0.f, 0.f};
        const float A2[2] = {as[row * Se + s], as[row * Se + s + 1]};
        lds_steps<16, TS>(m0, tl, m[0]);
        lds_steps<16, TS>(m1, tl, m[1]);
#pragma unroll
        for (int j = 0; j < TS; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) H[i] = __builtin_fmaf(exp2_fast(dt[j] * A2[i]), v[j] * m[i][j], H[i]);
        H[0] = row_sum(H[0]), H[1] = row_sum(H[1]);
        if (tl == 15) hs[row * Se + s] += H[0], hs[row * Se + s + 1] += H[1];
      }
    }
    if (k + 1 < passes) st.store(bc + ((k + 1) & 1) * S * kSteps, S);
    __syncthreads();
  }
  const int64_t at = int64_t(p.n) * a.segs * a.fine + p.seg;
  float* to = a.ends + state_at(a, p, at);
  for (int e = lane; e < p.held * S; e += 64) to[e] = hs[e + e / S * (Se - S)];
  if (tl == 0 && p.ok) a.end_dt[at * a.D + p.d] = total;
}

// Sums sixteen values over the four rows: lane (row, tl) gets, of position tl,
// values 0-3, 4-7 of lo in rows 0, 1 and of hi in rows 2, 3.
__device__ __forceinline__ f32x4 sum_rows(const float* lo, const float* hi) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(lo[j]), __float_as_uint(hi[j]), false, false);
    v[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  f32x4 o;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[j]), __float_as_uint(v[j + 4]), false, false);
    o[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return o;
}

// Backward.  With e(t) the gradient of h(t) and r(t) = a(t) e(t) what goes on to
// h(t-1):
//
//   e(t) = dy(t) C(t) + r(t+1)        (r behind the end: dfinal_state)
//   dC = sum_d dy h,  dB = sum_d e x,  dx = sum_s e B,  k = r h(t-1)
//   ddt = u dx + sum_s A k,  dA = sum k dt,  du = dt dx + Dskip dy
//
// The walk is from right to left.  In a chunk the states come again from the
// checkpoint (the forward pass's scan), then the gradients by the same scan the
// other way; nothing of a chunk but eight steps' sums outlives a state.  dB and
// dC are sums over channels: over a wave's four by permlane swaps, over the
// workgroup's waves through LDS (two states at a time), over workgroups and
// segments by scan_sum_kernel from `part_bc`, always in the same order.
//
// 4 x 2048 x 2048 with 16 states: 250 us, 28 issue slots a step of a state
// (in use 87% of the time): 17 the formulas, 4 the scans, 3 the sums over the
// wave, the rest an element's functions shared by its 16 states; the parts of
// dB and dC are another 14 us.
template <typename T, int NB, bool GATE>
__global__ __launch_bounds__(512) void scan_bwd_kernel(const ScanArgs<T> a) {
  extern __shared__ float lds[];
  const Place p = place<4>(a);
  const int S = a.S, Se = (S + 1) & ~1, rows = 2 * S, lane = p.lane, row = p.row, tl = p.tl;
  const int nw = blockDim.x >> 6, batch = a.batch;
  const int len = seq_len(a.lengths, p.n, a.L);
  const int c0 = p.seg * a.seg_chunks, c1 = c0 + a.seg_chunks < a.chunks ? c0 + a.seg_chunks : a.chunks;
  const int used = (len + kChunk - 1) / kChunk, cend = used < c1 ? used : c1;
  float* bc = lds;                     // B then C, a row of zeros behind them
  float* zeros = bc + rows * kChunk;
  float* ex = zeros + kChunk;          // [batch][waves][256]
  float* as = ex + batch * nw * 256 + p.wave * 16 * Se;
  float *rs = as + 4 * Se, *hs = rs + 4 * Se, *dAs = hs + 4 * Se;
  const int held = p.held;
  for (int e = lane; e < 4 * Se; e += 64) {
    const int r0 = e / Se, s = e - r0 * Se;
    float A2 = 0.f, r = 0.f;
    if (r0 < held) {
      const int64_t at = state_at(a, p, 0) + int64_t(r0) * S + s;
      A2 = decay2(a.A[s < S ? at : at - 1]);
      if (s < S && a.dfinal) r = a.dfinal[int64_t(p.n) * a.D * S + at];
      if (s < S && p.seg < a.segs - 1)
        r = through(a, p.n, a.segs * a.fine - 1, (p.seg + 1) * a.fine - 1, -1, at, p.d0 + r0, A2, r);
    }
    as[e] = A2;
    rs[e] = r;
    hs[e] = dAs[e] = 0.f;
  }
  for (int e = threadIdx.x; e < kChunk; e += blockDim.x) zeros[e] = 0.f;
  const T* up = a.u + p.n * a.u_n + p.d * a.u_d + tl * 8;
  const T* dp = a.delta + p.n * a.delta_n + p.d * a.delta_d + tl * 8;
  const T* zp = GATE ? a.z + p.n * a.z_n + p.d * a.z_d + tl * 8 : nullptr;
  const T* gp = a.dout + p.n * a.dout_n + p.d * a.dout_d + tl * 8;
  const T* Bp = a.B + p.n * a.B_n + p.g * a.B_g;
  const T* Cp = a.C + p.n * a.C_n + p.g * a.C_g;
  const float skip = a.Dskip ? a.Dskip[p.d] : 0.f, bias = a.bias ? a.bias[p.d] : 0.f;
  const int64_t at_row = (int64_t(p.n) * a.D + p.d) * a.L + tl * 8;
  // (the steps of a row without a channel are all behind its end: they add nothing)
  const int row_len = p.ok ? len - tl * 8 : 0;
  float dD = 0.f, dbias = 0.f;
  Stage<T, 16, 8, NB> st;
  Raw8<T> ru = {}, rd = {}, rz = {}, rg = {};
  float ck[4];  // the chunk's checkpoint: entries lane, lane + 64, ... of [channel][S]
  auto fetch = [&](int c) {
    const int t0 = c * kChunk, valid = row_len - t0;
    st.load(Bp, a.B_s, Cp, a.C_s, S, rows, t0, len);
    ru = load8(up + t0, valid);
    rd = load8(dp + t0, valid);
    rg = load8(gp + t0, valid);
    if (GATE) rz = load8(zp + t0, valid);
    const float* from = a.checkpoints + state_at(a, p, int64_t(p.n) * a.chunks + c);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + k * 64 < held * S) ck[k] = from[lane + k * 64];
  };
  int ck_at[4];  // where they belong in [channel][Se]
#pragma unroll
  for (int k = 0; k < 4; ++k) ck_at[k] = lane + k * 64 + (lane + k * 64) / S * (Se - S);
  // dB and dC of the batch of states from s0 on, over the waves
  auto sum_batch = [&](int s0, int c) {
    float* to = a.part_bc + ((int64_t(p.n) * a.G + p.g) * a.blks + p.blk) * S * 2 * a.chunks * kChunk;
    for (int o = threadIdx.x; o < batch * 64; o += blockDim.x) {
      const int i = o >> 6, q = (o & 63) * 4;
      if (s0 + i < S) {
        const float* from = ex + i * nw * 256 + q;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < nw; w += 4, from += 1024)
#pragma unroll
          for (int k = 0; k < 4; ++k) v += *reinterpret_cast<const f32x4*>(from + k * 256);
        *reinterpret_cast<f32x4*>(to + ((int64_t(s0 + i) * 2 + (q >> 7)) * a.chunks + c) * kChunk + (q & 127)) = v;
      }
    }
  };
  const int last = (S - 1) & -batch;  // the last batch: summed when the next chunk begins
  if (c0 < cend) fetch(cend - 1);
  for (int c = cend - 1; c >= c0; --c) {
    const int t0 = c * kChunk, valid = row_len - t0;
    const bool full = t0 + kChunk <= len;
    __syncthreads();  // (the chunk before has been read, its last batch written)
    if (c + 1 < cend) sum_batch(last, c + 1);
    st.store(bc, rows);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + k * 64 < held * S) hs[ck_at[k]] = ck[k];
    float dt[8], x[8], dy[8], dx[8], ddt[8], y[8];
    const float sum = steps<T, 8>(&rd, bias, a.softplus, full, valid, dt);
    const Raw8<T> ku = again(ru), kd = again(rd), kg = again(rg), kz = again(rz);
    {
      float z[8], u[8];
      unpack8(rg, dy);
      if (GATE) {
        unpack8(rz, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) dy[j] *= z[j] * sigmoid(z[j]);
      }
      unpack8(ru, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = dt[j] * u[j];
        dx[j] = ddt[j] = 0.f;
        y[j] = skip * u[j];
      }
    }
    __syncthreads();
    if (c > c0) fetch(c - 1);
    // Two states at a time (with S odd the last one's pair has its decay and reads
    // zeros), `batch` between two exchanges.
    for (int s = 0; s < S; s += 2) {
      const bool two = s + 1 < S;
      const float* b0 = bc + s * kChunk;
      const float* q0 = b0 + S * kChunk;
      float b[2][8], cc[2][8], w[2][8], A2[2], rin[2], R[2] = {0.f, 0.f}, P[2], Q[2];
      lds_steps<16, 8>(q0, tl, cc[0]);
      lds_steps<16, 8>(two ? q0 + kChunk : zeros, tl, cc[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        A2[i] = as[row * Se + s + i];
        rin[i] = rs[row * Se + s + i];
        P[i] = Q[i] = exp2_fast(sum * A2[i]);
      }
#pragma unroll
      for (int j = 7; j >= 0; --j) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          w[i][j] = exp2_fast(dt[j] * A2[i]);
          R[i] = w[i][j] * __builtin_fmaf(dy[j], cc[i][j], R[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) R[i] = __builtin_fmaf(P[i], tl == 15 ? rin[i] : 0.f, R[i]);
      scan_lanes_back(R, P, rin);
      float* exb = ex + (s & (batch - 1)) * nw * 256 + p.wave * 256 + lane * 4;
      float h[2][8], hin[2], H[2] = {0.f, 0.f}, dA[2] = {0.f, 0.f};
      lds_steps<16, 8>(b0, tl, b[0]);
      lds_steps<16, 8>(two ? b0 + kChunk : zeros, tl, b[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) hin[i] = hs[row * Se + s + i];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          h[i][j] = x[j] * b[i][j];
          H[i] = __builtin_fmaf(w[i][j], H[i], h[i][j]);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) H[i] = __builtin_fmaf(Q[i], tl == 0 ? hin[i] : 0.f, H[i]);
      scan_lanes<16>(H, Q, hin);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          h[i][j] = __builtin_fmaf(w[i][j], j ? h[i][j ? j - 1 : 0] : hin[i], h[i][j]);
          if (GATE) y[j] = __builtin_fmaf(h[i][j], cc[i][j], y[j]);
        }
      }
      float dB[2][8], dC[2][8];
#pragma unroll
      for (int j = 7; j >= 0; --j) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float e = __builtin_fmaf(dy[j], cc[i][j], rin[i]);
          dC[i][j] = dy[j] * h[i][j];
          dB[i][j] = e * x[j];
          dx[j] = __builtin_fmaf(e, b[i][j], dx[j]);
          rin[i] = w[i][j] * e;
          const float k = rin[i] * (j ? h[i][j ? j - 1 : 0] : hin[i]);
          ddt[j] = __builtin_fmaf(A2[i], k, ddt[j]);
          dA[i] = __builtin_fmaf(k, dt[j], dA[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        *reinterpret_cast<f32x4*>(exb + i * nw * 256) = sum_rows(dB[i], dC[i]);
        dA[i] = row_sum(dA[i]);
      }
      if (tl == 15) dAs[row * Se + s] += dA[0], dAs[row * Se + s + 1] += dA[1];
      if (tl == 0) rs[row * Se + s] = rin[0], rs[row * Se + s + 1] = rin[1];
      if ((s + 2 & (batch - 1)) == 0 && s + 2 < S) {
        __syncthreads();
        sum_batch(s & -batch, c);
        __syncthreads();  // (the next batch overwrites it)
      }
    }
    if (p.ok) {
      float u[8], raw[8], o[8], od[8], oz[8];
      unpack8(ku, u);
      unpack8(kd, raw);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        od[j] = __builtin_fmaf(dx[j], u[j], kLn2 * ddt[j]);
        if (a.softplus) od[j] *= sigmoid(raw[j] + bias);  // (of an infinite step: 1)
        o[j] = __builtin_fmaf(dx[j], dt[j], skip * dy[j]);
      }
      if (GATE) {
        float g[8], z[8];
        unpack8(kg, g);
        unpack8(kz, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float sg = sigmoid(z[j]);
          oz[j] = g[j] * y[j] * (sg * (1.f + z[j] * (1.f - sg)));
        }
      }
      if (!full) {
        branch();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j >= valid) o[j] = od[j] = oz[j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dD = __builtin_fmaf(dy[j], u[j], dD);
        dbias += od[j];
      }
      const int room = a.L - t0 - tl * 8;
      store8(a.du + at_row + t0, room, o);
      store8(a.ddelta + at_row + t0, room, od);
      if (GATE) store8(a.dz + at_row + t0, room, oz);
    }
  }
  if (c0 < cend) {
    __syncthreads();
    sum_batch(last, c0);
  }
  wave_sync();  // (nothing to sum: dAs and rs as they were cleared)
  const int64_t at = int64_t(p.n) * a.segs + p.seg;
  const auto put = [&](float* to, const float* from) {
    for (int e = lane; e < held * S; e += 64) to[e] = from[e + e / S * (Se - S)];
  };
  put(a.part_A + state_at(a, p, at), dAs);
  if (a.dinitial && p.seg == 0) put(a.dinitial + state_at(a, p, p.n), rs);
  dD = row_sum(dD), dbias = row_sum(dbias);
  if (!p.ok) return;
  if (tl == 15) {
    float* to = a.part_D + (at * a.D + p.d) * 2;
    to[0] = dD, to[1] = dbias;
  }
  const float zero[8] = {};
  for (int c = c0 > used ? c0 : used; c < c1; ++c) {
    const int t0 = c * kChunk, room = a.L - t0 - tl * 8;
    store8(a.du + at_row + t0, room, zero);
    store8(a.ddelta + at_row + t0, room, zero);
    if (GATE) store8(a.dz + at_row + t0, room, zero);
  }
}

// Adds the backward pass's parts in order.  The first `bc_wgs` workgroups: four
// steps of dB or dC a thread, over the channel blocks; the others: an element of
// dA, dDskip or ddelta_bias, over sequences and segments.
template <typename T>
__global__ __launch_bounds__(256) void scan_sum_kernel(const ScanArgs<T> a, uint32_t bc_wgs) {
  if (blockIdx.x < bc_wgs) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int quads = a.chunks * (kChunk / 4);
    const int64_t r = i / quads;  // (n, g, s, which)
    if (r >= int64_t(a.N) * a.G * a.S * 2) return;
    const int q = int(i - r * quads), c = q / 32, t = c * kChunk + (q & 15) * 8 + (q >> 4 & 1) * 4;
    if (t >= a.L) return;
    const int which = int(r & 1);
    const int64_t ng = r / (2 * a.S), ngs = r >> 1;
    const int s = int(ngs - ng * a.S), len = seq_len(a.lengths, int(ng / a.G), a.L);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (c * kChunk < len) {
      const int64_t step = int64_t(a.S) * 2 * a.chunks * kChunk;
      const float* from =
          a.part_bc + ng * a.blks * step + (int64_t(s) * 2 + which) * a.chunks * kChunk + int64_t(q) * 4;
#pragma unroll 16
      for (int b = 0; b < a.blks; ++b) v += *reinterpret_cast<const f32x4*>(from + b * step);
    }
    T* to = (which ? a.dC : a.dB) + ngs * a.L + t;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (t + j < a.L) to[j] = from_f<T>(t + j < len ? v[j] : 0.f);
    return;
  }
  const int64_t i = int64_t(blockIdx.x - bc_wgs) * 256 + threadIdx.x, states = int64_t(a.D) * a.S;
  const int parts = a.N * a.segs;
  if (i < states) {
    float v = 0.f;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) v += a.part_A[k * states + i];
    a.dA[i] = v;
  } else if (i < states + int64_t(a.D) * 2) {
    const int64_t e = i - states;
    float v = 0.f;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) v += a.part_D[k * int64_t(a.D) * 2 + e];
    float* to = e & 1 ? a.dbias : a.dD;
    if (to) to[e >> 1] = v;
  }
}

// One token: bound by the states, which go through memory once, as they lie:
// four states a lane, GL lanes a channel, so that a wave's store covers whole
// cache lines.  A group of GL lanes has up to four channels, 64 / GL apart; each
// lane forms one's step and gate (a softplus is as much work as three states)
// and hands them round, and keeps its A for all the sequences that it works on.
template <typename T>
struct StepArgs {
  int N, D, S, per, G, softplus;
  int blks, seqs;  // waves of a channel group; sequences of a wave
  uint32_t waves;
  int64_t u_n, u_d, delta_n, delta_d, z_n, z_d, B_n, B_g, B_s, C_n, C_g, C_s;
  const T *u, *delta, *z, *B, *C;
  const float *A, *Dskip, *bias, *initial;
  T* out;
  float* final_state;
};

// Lane c's value of a group of GL lanes.
template <int GL, int c>
__device__ __forceinline__ float from_lane(float v) {
  if constexpr (GL == 1) return v;
  if constexpr (GL == 2) return dpp0<(c ? 0xF5 : 0xA0)>(v);
  if constexpr (GL == 4) return dpp0<c * 0x55>(v);
  return __shfl(v, (threadIdx.x & 63 & -GL) + c);
}
// The sum over the group.
template <int GL>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (GL >= 2) v += dpp0<0xB1>(v);  // (quads: 1 0 3 2)
  if constexpr (GL >= 4) v += dpp0<0x4E>(v);  // (2 3 0 1)
  for (int m = 4; m < GL; m <<= 1) v += __shfl_xor(v, m);
  return v;
}
template <int I = 0, int N, typename F>
__device__ __forceinline__ void each(std::integral_constant<int, N> n, F f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<I + 1>(n, f);
  }
}

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
// The first m of four floats.  STREAM: past the caches, for what is read once.
template <bool STREAM>
__device__ __forceinline__ void load4(const float* p, int m, float* v) {
  if (m == 4) {
    const f32x4u* q = reinterpret_cast<const f32x4u*>(p);
    const f32x4u r = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = r[j];
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (j < m) v[j] = p[j];
  }
}

template <typename T, int GL>
__global__ __launch_bounds__(256) void scan_step_kernel(const StepArgs<T> a) {
  constexpr int CH = GL < 4 ? GL : 4, W = 64 / GL;  // channels of a lane group, lane groups
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (wave >= a.waves) return;
  const int lane = threadIdx.x & 63, li = lane % GL, s0 = li * 4, m = a.S - s0 < 0 ? 0 : a.S - s0 < 4 ? a.S - s0 : 4;
  const uint32_t q = wave / uint32_t(a.blks), blk = wave - q * a.blks;
  const int g = int(q % uint32_t(a.G)), n0 = int(q / uint32_t(a.G)) * a.seqs;
  const int n1 = n0 + a.seqs < a.N ? n0 + a.seqs : a.N;
  const int c0 = int(blk) * (CH * W) + lane / GL, left = (a.per - c0 + W - 1) / W, have = left < CH ? left : CH;
  if (have <= 0) return;  // (a whole lane group)
  const int d0 = g * a.per + c0;
  const int mine = li < have ? li : have - 1, d = d0 + mine * W;  // whose scalars this lane forms
  float A2[CH][4] = {};
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (c < have) load4<false>(a.A + int64_t(d0 + c * W) * a.S + s0, m, A2[c]);
#pragma unroll
    for (int j = 0; j < 4; ++j) A2[c][j] = decay2(A2[c][j]);
  }
  const float bias = a.bias ? a.bias[d] : 0.f, skip = a.Dskip ? a.Dskip[d] : 0.f;
  struct Token {
    float h[CH][4], u, delta, z, B[4], C[4];
  };
  auto load = [&](int n) {
    Token t = {};
    const int64_t at = (int64_t(n) * a.D + d0) * a.S + s0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (c < have) load4<true>(a.initial + at + int64_t(c * W) * a.S, m, t.h[c]);
    t.u = to_f(a.u[n * a.u_n + d * a.u_d]);
    t.delta = to_f(a.delta[n * a.delta_n + d * a.delta_d]);
    if (a.z) t.z = to_f(a.z[n * a.z_n + d * a.z_d]);
    const T* Bp = a.B + n * a.B_n + g * a.B_g + s0 * a.B_s;
    const T* Cp = a.C + n * a.C_n + g * a.C_g + s0 * a.C_s;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < m) t.B[j] = to_f(Bp[j * a.B_s]), t.C[j] = to_f(Cp[j * a.C_s]);
    return t;
  };
  Token next = load(n0);
  for (int n = n0; n < n1; ++n) {
    Token t = next;
    if (n + 1 < n1) next = load(n + 1);
    const int64_t at = (int64_t(n) * a.D + d0) * a.S + s0;
    auto &h = t.h;
    auto &B = t.B, &C = t.C;
    const float u = t.u, z = t.z;
    float y[CH], dt = t.delta + bias;
    if (a.softplus) dt = softplus(dt);
    const float x = dt * u;
    each(std::integral_constant<int, CH>{}, [&](auto ic) {
      constexpr int c = decltype(ic)::value;
      const float dtc = from_lane<GL, c>(dt), xc = from_lane<GL, c>(x);
      y[c] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        h[c][j] = __builtin_fmaf(exp2_fast(A2[c][j] * dtc), h[c][j], xc * B[j]);
        y[c] = __builtin_fmaf(C[j], h[c][j], y[c]);
      }
      if (c < have) {
        float* to = a.final_state + at + int64_t(c * W) * a.S;
        if (m == 4) {
          __builtin_nontemporal_store(f32x4u{h[c][0], h[c][1], h[c][2], h[c][3]}, reinterpret_cast<f32x4u*>(to));
        } else {
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (j < m) to[j] = h[c][j];
        }
      }
      y[c] = group_sum<GL>(y[c]);
    });
    float o = y[0];
#pragma unroll
    for (int c = 1; c < CH; ++c) o = mine == c ? y[c] : o;
    o = __builtin_fmaf(skip, u, o);
    if (a.z) o *= z * sigmoid(z);
    if (li < have) a.out[int64_t(n) * a.D + d] = from_f<T>(o);
  }
}

int64_t pad4(int64_t n) { return (n + 3) / 4 * 4; }
int64_t ends_floats(const seq_scan_t& p, const ScanShape& s) {
  const int64_t pieces = int64_t(p.N) * s.segs * s.fine;
  return s.segs > 1 ? pad4(pieces * p.D * p.S) + pad4(pieces * p.D) : 0;
}

template <typename T>
ScanArgs<T> args_of(const seq_scan_t& p, const ScanShape& s) {
  ScanArgs<T> a = {};
  a.N = p.N, a.D = p.D, a.L = p.L, a.S = p.S, a.G = p.G, a.per = s.per, a.softplus = p.delta_softplus;
  a.blks = s.blks, a.segs = a.run_segs = s.segs, a.seg_chunks = s.seg_chunks, a.chunks = s.chunks;
  a.fine = s.fine, a.fine_chunks = s.fine_chunks;
  a.u_n = p.u_n, a.u_d = p.u_d, a.delta_n = p.delta_n, a.delta_d = p.delta_d, a.z_n = p.z_n, a.z_d = p.z_d;
  a.dout_n = p.dout_n, a.dout_d = p.dout_d;
  a.B_n = p.B_n, a.B_g = p.B_g, a.B_s = p.B_s, a.C_n = p.C_n, a.C_g = p.C_g, a.C_s = p.C_s;
  const auto t = [](const void* v) { return static_cast<const T*>(v); };
  const auto w = [](void* v) { return static_cast<T*>(v); };
  a.u = t(p.u), a.delta = t(p.delta), a.z = t(p.z), a.B = t(p.B), a.C = t(p.C);
  a.A = p.A, a.Dskip = p.Dskip, a.bias = p.delta_bias, a.initial = p.initial_state, a.lengths = p.lengths;
  a.out = w(p.out), a.final_state = p.final_state, a.checkpoints = p.checkpoints;
  a.dout = t(p.dout), a.dfinal = p.dfinal_state;
  a.du = w(p.du), a.ddelta = w(p.ddelta), a.dz = w(p.dz), a.dB = w(p.dB), a.dC = w(p.dC);
  a.dA = p.dA, a.dD = p.dDskip, a.dbias = p.ddelta_bias, a.dinitial = p.dinitial_state;
  return a;
}

template <typename K, typename A>
int launch(K kernel, int64_t wgs, int threads, int64_t lds, hipStream_t s, const A& a) {
  if (lds > 65536 && hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                         hipFuncAttributeMaxDynamicSharedMemorySize, int(lds)) != hipSuccess)
    return CONV_EHIP;
  kernel<<<dim3(uint32_t(wgs)), threads, uint32_t(lds), s>>>(a);
  return hipGetLastError() == hipSuccess ? CONV_OK : CONV_EHIP;
}
// Staging loads of 16 bytes (fp32: 32) a thread holds for the next pass: 1, 2, 4
// or 8, at most MOST.
template <int MOST, int NB = 1, typename F>
int with_loads(int rows, int pass, int waves, F f) {
  if (ceil_div(rows * pass / 8, waves * 64) > NB) {
    if constexpr (NB < MOST) return with_loads<MOST, 2 * NB>(rows, pass, waves, f);
    return CONV_ENOPLAN;
  }
  return f(std::integral_constant<int, NB>{});
}

template <typename T, int TS, bool BACK>
int ends_steps(const seq_scan_t& p, const ScanShape& s, const ScanArgs<T>& a, int64_t wgs, hipStream_t st) {
  const int64_t lds = ((2 * p.S + 1) * int64_t(16 * TS) + 4 * 8 * ((p.S + 1) & ~1)) * 4;
  return with_loads<4>(p.S, 16 * TS, 4, [&](auto nb) {
    return launch(scan_ends_kernel<T, TS, decltype(nb)::value, BACK>, wgs, 256, lds, st, a);
  });
}
// The ends of all segments but the last (BACK: the first), which nothing comes after.
template <typename T, bool BACK>
int ends_pass(const seq_scan_t& p, const ScanShape& s, ScanArgs<T> a, hipStream_t st) {
  a.blks = int(ceil_div(s.per, 16));
  a.run_segs = (s.segs - 1) * s.fine, a.run_first = BACK ? s.fine : 0;
  const int64_t wgs = int64_t(p.N) * p.G * a.blks * a.run_segs;
  if (wgs * 256 > kMaxThreads) return CONV_ERANGE;
  return p.S <= 32 ? ends_steps<T, 16, BACK>(p, s, a, wgs, st) : ends_steps<T, 8, BACK>(p, s, a, wgs, st);
}

template <typename T, int RW, int TS>
int fwd_pass(const seq_scan_t& p, const ScanShape& s, const ScanArgs<T>& a, hipStream_t st) {
  constexpr int pass = 64 / RW * TS, per = pass / kChunk;
  const int64_t lds = ((4 * p.S + 1) * int64_t(pass) + s.waves * (1 + per) * RW * ((p.S + 1) & ~1)) * 4;
  // (512 steps of 32 rows by 4 waves; else 256 of 32 or 128 of 64 by 4, 128 of 128 by 8)
  return with_loads<RW == 1 ? 8 : 4>(2 * p.S, pass, s.waves, [&](auto nb) {
    return launch(scan_fwd_kernel<T, RW, TS, decltype(nb)::value>, s.wgs, s.waves * 64, lds, st, a);
  });
}
template <typename T>
int fwd(const seq_scan_t& p, hipStream_t st) {
  const ScanShape s = scan_shape(p, false);
  if (s.wgs * s.waves * 64 > kMaxThreads) return CONV_ERANGE;
  if (s.segs > 1 && !p.workspace) return CONV_ENULL;
  if (s.segs > 1 && p.workspace_bytes < scan_fwd_workspace(p)) return CONV_ESCRATCH;
  ScanArgs<T> a = args_of<T>(p, s);
  a.ends = static_cast<float*>(p.workspace);
  a.end_dt = a.ends + pad4(int64_t(p.N) * s.segs * s.fine * p.D * p.S);
  if (s.segs > 1) {
    const int rc = ends_pass<T, false>(p, s, a, st);
    if (rc != CONV_OK) return rc;
  }
  if (s.rows == 1) return fwd_pass<T, 1, 8>(p, s, a, st);
  return s.steps == 16 ? fwd_pass<T, 4, 16>(p, s, a, st) : fwd_pass<T, 4, 8>(p, s, a, st);
}

template <typename T, bool GATE>
int bwd_pass(const seq_scan_t& p, const ScanShape& s, const ScanArgs<T>& a, hipStream_t st) {
  const int rows = 2 * p.S, Se = (p.S + 1) & ~1;
  const int64_t lds = ((rows + 1) * int64_t(kChunk) + a.batch * s.waves * 256 + s.waves * 16 * Se) * 4;
  return with_loads<8>(rows, kChunk, s.waves, [&](auto nb) {
    return launch(scan_bwd_kernel<T, decltype(nb)::value, GATE>, s.wgs, s.waves * 64, lds, st, a);
  });
}
template <typename T>
int bwd(const seq_scan_t& p, hipStream_t st) {
  const ScanShape s = scan_shape(p, true);
  const int64_t bc_wgs = ceil_div(int64_t(p.N) * p.G * p.S * 2 * s.chunks * (kChunk / 4), 256);
  const int64_t sum_wgs = bc_wgs + ceil_div(int64_t(p.D) * (p.S + 2), 256);
  if (s.wgs * s.waves * 64 > kMaxThreads || sum_wgs * 256 > kMaxThreads) return CONV_ERANGE;
  if (!p.workspace) return CONV_ENULL;
  if (p.workspace_bytes < scan_bwd_workspace(p)) return CONV_ESCRATCH;
  ScanArgs<T> a = args_of<T>(p, s);
  a.batch = scan_batch(p.S);
  a.part_bc = static_cast<float*>(p.workspace);
  a.part_A = a.part_bc + int64_t(p.N) * p.G * s.blks * p.S * 2 * s.chunks * kChunk;
  a.part_D = a.part_A + pad4(int64_t(p.N) * s.segs * p.D * p.S);
  a.ends = a.part_D + pad4(int64_t(p.N) * s.segs * p.D * 2);
  a.end_dt = a.ends + pad4(int64_t(p.N) * s.segs * s.fine * p.D * p.S);
  int rc = s.segs > 1 ? ends_pass<T, true>(p, s, a, st) : CONV_OK;
  if (rc == CONV_OK) rc = p.z ? bwd_pass<T, true>(p, s, a, st) : bwd_pass<T, false>(p, s, a, st);
  if (rc != CONV_OK) return rc;
  scan_sum_kernel<T><<<dim3(uint32_t(sum_wgs)), 256, 0, st>>>(a, uint32_t(bc_wgs));
  return hipGetLastError() == hipSuccess ? CONV_OK : CONV_EHIP;
}

template <typename T, int GL>
int step_launch(const StepArgs<T>& a, hipStream_t st) {
  scan_step_kernel<T, GL><<<dim3((a.waves - 1) / 4 + 1), 256, 0, st>>>(a);
  return hipGetLastError() == hipSuccess ? CONV_OK : CONV_EHIP;
}
template <typename T>
int step(const seq_scan_t& p, hipStream_t st) {
  StepArgs<T> a = {};
  a.N = p.N, a.D = p.D, a.S = p.S, a.G = p.G, a.per = p.D / p.G, a.softplus = p.delta_softplus;
  int lanes = 1;
  while (lanes * 4 < p.S) lanes *= 2;
  a.blks = int(ceil_div(a.per, 64 / lanes * (lanes < 4 ? lanes : 4)));
  // A wave takes up to four sequences (A is read once for them) while 4096 waves
  // are left.  256 x 4096 x 16 states, from memory: 33 us at one, 32 at two, 31 at
  // four, 33 at eight (140 MB: 4.5 TB/s).
  const int64_t waves = int64_t(p.N) * p.G * a.blks;
  a.seqs = waves >= 4 * 4096 ? 4 : waves >= 2 * 4096 ? 2 : 1;
  const int64_t used = ceil_div(p.N, a.seqs) * p.G * a.blks;
  if ((used + 3) * 64 > kMaxThreads) return CONV_ERANGE;
  a.waves = uint32_t(used);
  a.u_n = p.u_n, a.u_d = p.u_d, a.delta_n = p.delta_n, a.delta_d = p.delta_d, a.z_n = p.z_n, a.z_d = p.z_d;
  a.B_n = p.B_n, a.B_g = p.B_g, a.B_s = p.B_s, a.C_n = p.C_n, a.C_g = p.C_g, a.C_s = p.C_s;
  const auto t = [](const void* v) { return static_cast<const T*>(v); };
  a.u = t(p.u), a.delta = t(p.delta), a.z = t(p.z), a.B = t(p.B), a.C = t(p.C);
  a.A = p.A, a.Dskip = p.Dskip, a.bias = p.delta_bias, a.initial = p.initial_state;
  a.out = static_cast<T*>(p.out), a.final_state = p.final_state;
  switch (lanes) {
    case 1: return step_launch<T, 1>(a, st);
    case 2: return step_launch<T, 2>(a, st);
    case 4: return step_launch<T, 4>(a, st);
    case 8: return step_launch<T, 8>(a, st);
    default: return step_launch<T, 16>(a, st);
  }
}
}  // namespace

int64_t scan_fwd_workspace(const seq_scan_t& p) {
  return ends_floats(p, scan_shape(p, false)) * int64_t(sizeof(float));
}
int64_t scan_bwd_workspace(const seq_scan_t& p) {
  const ScanShape s = scan_shape(p, true);
  const int64_t rows = int64_t(p.N) * s.segs * p.D;
  return (int64_t(p.N) * p.G * s.blks * p.S * 2 * s.chunks * kChunk + pad4(rows * p.S) + pad4(rows * 2) +
          ends_floats(p, s)) * int64_t(sizeof(float));
}
int launch_scan_fwd(const seq_scan_t& p, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p.dtype == CONV_DTYPE_BF16 ? fwd<bf16>(p, s) : fwd<float>(p, s);
}
int launch_scan_bwd(const seq_scan_t& p, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p.dtype == CONV_DTYPE_BF16 ? bwd<bf16>(p, s) : bwd<float>(p, s);
}
int launch_scan_step(const seq_scan_t& p, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p.dtype == CONV_DTYPE_BF16 ? step<bf16>(p, s) : step<float>(p, s);
}

}  // namespace seqops
