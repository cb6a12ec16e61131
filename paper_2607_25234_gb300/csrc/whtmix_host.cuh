// whtmix_host.cuh -- what the C entry points share on the host (whtmix_capi.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

#include <mutex>

namespace whtmix {
namespace host {

int fail(cudaError_t e);  // remembers e for whtmix_last_cuda_error
int device(int* dev, int* sms);
int workspace(int dev, cudaStream_t stream, size_t bytes, int slot, void** out);
// A word of device memory that is there as long as the library, for kernels whose waits may give up; read by whtmix_sync.
int error_word(int dev, unsigned int** err);

// The scratch of one call.  On a stream that is being captured it is allocated and freed by nodes of the graph, so that no other
// graph, no later call and no growing workspace shares or ends it; on the per-thread default stream, one handle for a stream of each host
// thread, it is allocated and freed on that stream.  Elsewhere it is the stream's workspace of slot 2, and calls of several host threads on
// one stream are let through one after another, whole.
class Scratch {
 public:
  Scratch() = default;
  Scratch(const Scratch&) = delete;
  Scratch& operator=(const Scratch&) = delete;
  ~Scratch() { (void)give_back(); }
  int take(int dev, cudaStream_t stream, size_t bytes);
  int give_back();  // behind the call's last launch (the destructor's, where a launch has failed)
  void* get() const { return p_; }

 private:
  void* p_ = nullptr;
  cudaStream_t stream_ = nullptr;
  bool own_ = false;  // allocated for this call
  std::unique_lock<std::mutex> turn_;
};

}  // namespace host
}  // namespace whtmix
