// Backward passes that are captured into a graph, as the native nodes see them.
#pragma once

#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime_api.h>
#include <torch/csrc/autograd/function.h>

namespace tb {

// A leaf's gradient is accumulated by one node as long as any graph holds it, on the stream of the graph that came first.
// Where that is the default stream and another one is being captured, the engine would make the default stream wait for
// a captured event, which HIP refuses in a place that ends the process.
inline bool leaves_capture(const torch::autograd::Node* next) {
  if (!next) return false;
  const auto to = const_cast<torch::autograd::Node*>(next)->stream();
  if (!to || to->id() != 0) return false;
  const hipStream_t now = c10::hip::getCurrentHIPStream(to->device_index()).stream();
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  return now && hipStreamIsCapturing(now, &status) == hipSuccess && status == hipStreamCaptureStatusActive;
}
constexpr const char* kLeavesCapture =
    "a backward pass is being captured while a graph from outside the capture holds the same leaf: let go of that graph "
    "(or capture with a detached leaf)";
inline bool leaves_capture(const torch::autograd::edge_list& edges) {
  for (const auto& e : edges)
    if (leaves_capture(e.function.get())) return true;
  return false;
}

}  // namespace tb
