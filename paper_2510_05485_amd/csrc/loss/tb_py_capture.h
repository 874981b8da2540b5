// Backward passes that are captured into a graph, as the native nodes see them.
#pragma once

#include <unordered_set>
#include <vector>

#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime_api.h>
#include <torch/csrc/autograd/function.h>

namespace tb {

// A leaf's gradient is accumulated by one node as long as any graph holds it, on the stream of the graph that came first.
// Where that is the default stream and another one is being captured, the engine would make the default stream wait for
// a captured event, which HIP refuses in a place that ends the process.  So would any other node of the default stream.
// Looked for among all that this backward pass goes on to from `node`, whose turn it is: a leaf is mostly the end of a
// chain (a cast table, a model behind its logits), and what torch.autograd.grad stops before is not executed.
inline bool leaves_capture(torch::autograd::Node* node) {
  const hipStream_t now = c10::hip::getCurrentHIPStream().stream();
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (!node || !now || hipStreamIsCapturing(now, &status) != hipSuccess || status != hipStreamCaptureStatusActive) return false;
  std::vector<torch::autograd::Node*> left = {node};
  std::unordered_set<torch::autograd::Node*> seen;
  while (!left.empty()) {
    torch::autograd::Node* from = left.back();
    left.pop_back();
    for (size_t i = 0; i < from->num_outputs(); ++i) {
      if (!from->task_should_compute_output(i)) continue;
      torch::autograd::Node* next = from->next_edge(i).function.get();
      if (!seen.insert(next).second) continue;
      const auto stream = next->stream();
      if (stream && stream->id() == 0) return true;
      left.push_back(next);
    }
  }
  return false;
}
constexpr const char* kLeavesCapture =
    "a backward pass is being captured while a graph from outside the capture holds a leaf that it goes on to: let go of "
    "that graph (or capture with a detached leaf)";

}  // namespace tb
