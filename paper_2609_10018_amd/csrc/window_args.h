// Launchers of the windowed attention (host-side declarations).
#pragma once

#include <hip/hip_runtime.h>

#include "layout.h"
#include "window.h"

namespace elasto {

struct WindowTensors {
  View q, k, v, o, dout, dq, dk, dv;  // byte strides
  float* lse;
};

// Bytes of scratch a launch of this description uses (0: none).
int64_t window_fwd_workspace(const elasto_window_t& a);
int64_t window_bwd_workspace(const elasto_window_t& a);

// The description has been checked; batch, tokens and heads are at least 1.
hipError_t launch_window_fwd(const elasto_window_t& a, const WindowTensors& t, void* ws, hipStream_t s);
hipError_t launch_window_bwd(const elasto_window_t& a, const WindowTensors& t, void* ws, hipStream_t s);

// A launch holds fewer than 2^32 threads, 256 a workgroup.
constexpr int64_t kMaxBlocks = 1 << 24;

// Largest sinks: the keys of the first tile of the backward pass's key kernel
// must hold them all.
constexpr int kMaxSinks = 64;

}  // namespace elasto
