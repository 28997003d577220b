// launch_packed.h -- internal interface between the C-ABI layer (api.cpp) and
// the kernels of softmax attention over packed sequences (window.hip).
// Arguments arrive here already validated.
#pragma once

#include "launch.h"

namespace hyb {

// s.B sequences one after the other in N rows: sequence b is rows token_start[b] ..
// token_start[b + 1] - 1 (device, clamped to the rows there are; the first starts at
// row 0).  Of the base T (the sequences' mean length, for choices of the host only) and
// seq_lens (null) say nothing of the rows; lse is [Hq][N].
struct PackedArgs : WindowArgs {
  const int32_t* token_start;
  int N;
  long q_stride, k_stride, v_stride;  // elements from a row of q, k, v to the next
};

hipError_t launch_packed_prefill(const PackedArgs& a, hipStream_t st);
hipError_t launch_packed_backward(const PackedArgs& a, hipStream_t st);
double packed_threads(const Shape& s, int N);  // of the largest launch
size_t packed_backward_ws_bytes(const Shape& s, int N);

}  // namespace hyb
