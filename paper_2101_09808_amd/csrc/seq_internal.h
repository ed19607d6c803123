// Host side of the sequence operators: what seq_api.cpp checks and
// the launchers of seq_*.hip take.
#pragma once
#include <stdint.h>

#include "seq_ops.h"

namespace seqops {

// Every launch is below these, so 32-bit workgroup arithmetic holds; the HIP
// runtime takes fewer than 2^32 threads a launch.
constexpr int64_t kMaxThreads = (int64_t(1) << 32) - 1;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int64_t conv_bwd_workspace(const seq_conv_t& p);
int launch_conv_fwd(const seq_conv_t& p, void* stream);
int launch_conv_bwd(const seq_conv_t& p, void* stream);
int launch_conv_step(const seq_conv_t& p, void* stream);

int64_t scan_fwd_workspace(const seq_scan_t& p);
int64_t scan_bwd_workspace(const seq_scan_t& p);
int launch_scan_fwd(const seq_scan_t& p, void* stream);
int launch_scan_bwd(const seq_scan_t& p, void* stream);
int launch_scan_step(const seq_scan_t& p, void* stream);

int64_t norm_fwd_workspace(const seq_norm_t& p);
int64_t norm_bwd_workspace(const seq_norm_t& p);
int launch_norm_fwd(const seq_norm_t& p, bool post, void* stream);
int launch_norm_bwd(const seq_norm_t& p, bool post, void* stream);

}  // namespace seqops
