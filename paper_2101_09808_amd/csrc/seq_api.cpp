// C ABI of the sequence operators (seq_ops.h): argument checks, then the
// launchers of seq_*.hip.  Nothing here allocates or throws.
#include "seq_internal.h"

namespace {
using namespace seqops;

constexpr int32_t kMaxLen = 1 << 30;  // (a step index plus a tile stays in 32 bits)
constexpr int32_t kMaxDim = 1 << 30;  // (and a channel plus a workgroup's: scan and norms)

bool bad_dtype(int32_t t) { return t != CONV_DTYPE_F32 && t != CONV_DTYPE_BF16; }

// Extents that every operator shares.  N D is a row index of 32 bits.
int check_extents(int32_t N, int32_t D, int32_t L) {
  if (N <= 0 || D <= 0 || L <= 0) return CONV_EINVAL;
  if (L > kMaxLen || int64_t(N) * D >= int64_t(1) << 31) return CONV_ERANGE;
  return CONV_OK;
}

int check_conv(const seq_conv_t* p) {
  if (!p) return CONV_ENULL;
  if (const int rc = check_extents(p->N, p->D, p->L)) return rc;
  if (p->R < 1 || p->R > SEQ_CONV_MAX_TAPS || bad_dtype(p->dtype)) return CONV_EINVAL;
  if (p->activation != SEQ_ACT_NONE && p->activation != SEQ_ACT_SILU) return CONV_EINVAL;
  return CONV_OK;
}

int check_scan(const seq_scan_t* p) {
  if (!p) return CONV_ENULL;
  if (const int rc = check_extents(p->N, p->D, p->L)) return rc;
  if (p->S < 1 || p->S > SEQ_SCAN_MAX_STATE || p->G < 1 || p->D % p->G || bad_dtype(p->dtype) || p->reserved)
    return CONV_EINVAL;
  return p->D > kMaxDim ? CONV_ERANGE : CONV_OK;
}

int check_norm(const seq_norm_t* p) {
  if (!p) return CONV_ENULL;
  if (const int rc = check_extents(p->N, p->D, p->L)) return rc;
  if (bad_dtype(p->dtype) || (p->res_dtype != p->dtype && p->res_dtype != CONV_DTYPE_F32)) return CONV_EINVAL;
  if (!(p->eps >= 0.f)) return CONV_EINVAL;
  return p->D > kMaxDim ? CONV_ERANGE : CONV_OK;
}

bool scan_inputs(const seq_scan_t* p) { return p->u && p->delta && p->A && p->B && p->C; }
}  // namespace

extern "C" {

int seq_causal_conv_fwd(const seq_conv_t* p, void* stream) {
  if (const int rc = check_conv(p)) return rc;
  if (!p->x || !p->weight || !p->out) return CONV_ENULL;
  return launch_conv_fwd(*p, stream);
}
int seq_causal_conv_bwd(const seq_conv_t* p, void* stream) {
  if (const int rc = check_conv(p)) return rc;
  if (!p->x || !p->weight || !p->dout || !p->dx || !p->dweight) return CONV_ENULL;
  return launch_conv_bwd(*p, stream);
}
int64_t seq_causal_conv_bwd_workspace(const seq_conv_t* p) {
  const int rc = check_conv(p);
  return rc ? rc : conv_bwd_workspace(*p);
}
int seq_causal_conv_step(const seq_conv_t* p, void* stream) {
  if (const int rc = check_conv(p)) return rc;
  if (p->L != 1 || p->lengths) return CONV_EINVAL;
  if (!p->x || !p->weight || !p->out || (p->R > 1 && !(p->initial_state && p->final_state))) return CONV_ENULL;
  return launch_conv_step(*p, stream);
}

int seq_selective_scan_fwd(const seq_scan_t* p, void* stream) {
  if (const int rc = check_scan(p)) return rc;
  if (!scan_inputs(p) || !p->out) return CONV_ENULL;
  return launch_scan_fwd(*p, stream);
}
int64_t seq_selective_scan_fwd_workspace(const seq_scan_t* p) {
  const int rc = check_scan(p);
  return rc ? rc : scan_fwd_workspace(*p);
}
int seq_selective_scan_bwd(const seq_scan_t* p, void* stream) {
  if (const int rc = check_scan(p)) return rc;
  if (!scan_inputs(p) || !p->checkpoints || !p->dout || !p->du || !p->ddelta || !p->dA || !p->dB || !p->dC ||
      (p->z && !p->dz) || (p->Dskip && !p->dDskip) || (p->delta_bias && !p->ddelta_bias))
    return CONV_ENULL;
  return launch_scan_bwd(*p, stream);
}
int64_t seq_selective_scan_bwd_workspace(const seq_scan_t* p) {
  const int rc = check_scan(p);
  return rc ? rc : scan_bwd_workspace(*p);
}
int seq_selective_scan_step(const seq_scan_t* p, void* stream) {
  if (const int rc = check_scan(p)) return rc;
  if (p->L != 1 || p->lengths || p->checkpoints) return CONV_EINVAL;
  if (!scan_inputs(p) || !p->out || !p->initial_state || !p->final_state) return CONV_ENULL;
  return launch_scan_step(*p, stream);
}

int seq_norm_pre_fwd(const seq_norm_t* p, void* stream) {
  if (const int rc = check_norm(p)) return rc;
  if (p->gate) return CONV_EINVAL;
  if (!p->x || !p->weight || !p->out) return CONV_ENULL;
  return launch_norm_fwd(*p, false, stream);
}
int seq_norm_post_fwd(const seq_norm_t* p, void* stream) {
  if (const int rc = check_norm(p)) return rc;
  if (p->sum) return CONV_EINVAL;
  if (!p->x || !p->weight || !p->out) return CONV_ENULL;
  return launch_norm_fwd(*p, true, stream);
}
int seq_norm_pre_bwd(const seq_norm_t* p, void* stream) {
  if (const int rc = check_norm(p)) return rc;
  if (p->gate || p->dgate) return CONV_EINVAL;
  if (!p->sum || !p->weight || !p->dout || !p->dx || !p->dweight || (p->scale && !(p->x && p->dscale)))
    return CONV_ENULL;
  return launch_norm_bwd(*p, false, stream);
}
int seq_norm_post_bwd(const seq_norm_t* p, void* stream) {
  if (const int rc = check_norm(p)) return rc;
  if (p->sum || p->dsum || p->dresidual) return CONV_EINVAL;
  if (!p->x || !p->weight || !p->dout || !p->dx || !p->dweight || (p->scale && !p->dscale) ||
      (p->gate && !p->dgate))
    return CONV_ENULL;
  return launch_norm_bwd(*p, true, stream);
}
int64_t seq_norm_fwd_workspace(const seq_norm_t* p) {
  const int rc = check_norm(p);
  return rc ? rc : norm_fwd_workspace(*p);
}
int64_t seq_norm_bwd_workspace(const seq_norm_t* p) {
  const int rc = check_norm(p);
  return rc ? rc : norm_bwd_workspace(*p);
}

}  // extern "C"
