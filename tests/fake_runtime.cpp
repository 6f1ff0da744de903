// A CUDA runtime in host memory, for what the host code does when a call fails or when nothing orders a copy before a launch: no
// device is touched.  Allocations are host blocks that are tracked, the nth one from now can be made to fail; a host-to-device copy from
// pageable memory can be made to land only when its device is next waited for, which the runtime's documentation allows; kernels do nothing, but an AdamW launch is
// remembered with its list, moves its clock on when its device is next waited for, and is checked at every launch and replay: the list
// and every buffer that it names have to be there, with no copy still under way.  The products and the other kernels are empty.
#include <cuda_runtime.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <functional>
#include <map>
#include <vector>

#include "conv.h"
#include "kernels.h"

namespace {

struct Copy { void* dst; std::vector<char> bytes; };
struct AdamWLaunch { const char* tensors; const int* first; int count; char* clock; int dev; };
struct Graph { std::vector<AdamWLaunch> launches; };

std::map<char*, size_t> blocks;
std::vector<Copy> copies[2];
std::vector<std::function<void()>> under_way[2];
int current = 0, fail_in = -1;
bool late = false;
long long violations = 0, adamw_launches = 0;
int masters = 0;              // in the list of the last AdamW launch
Graph* capture = nullptr;
std::vector<Graph*> executables;

bool live(const void* p) {
  const char* at = static_cast<const char*>(p);
  auto it = blocks.upper_bound(const_cast<char*>(at));
  if (it == blocks.begin()) return false;
  --it;
  return at < it->first + it->second;
}

void wait(int dev) {
  for (const Copy& c : copies[dev]) memcpy(c.dst, c.bytes.data(), c.bytes.size());
  copies[dev].clear();
  for (auto& f : under_way[dev]) f();
  under_way[dev].clear();
}

// The list's entries begin with the six or seven pointers of a tensor (weights, master, gradient, moments, scales); null where there is none.
void launch(const AdamWLaunch& l) {
  ++adamw_launches;
  if (!live(l.tensors) || !live(l.first) || !live(l.clock) || !copies[l.dev].empty()) { ++violations; return; }
  const size_t entry = (reinterpret_cast<const char*>(l.first) - l.tensors) / l.count;
  masters = 0;
  for (int i = 0; i < l.count; ++i)
    for (int k = 0; k < 7; ++k) {
      const void* p;
      memcpy(&p, l.tensors + i * entry + k * sizeof(void*), sizeof(p));
      if (p && !live(p)) ++violations;
      if (p && k == 1) ++masters;
    }
  char* clock = l.clock;
  under_way[l.dev].push_back([clock] { if (live(clock)) ++*reinterpret_cast<long long*>(clock + 16); });
}

}  // namespace

extern "C" {
__attribute__((visibility("default"))) void fake_fail_in(int n) { fail_in = n; }                   // the nth allocation from now on, 0: the next
__attribute__((visibility("default"))) void fake_late_copies(int on) { late = on != 0; }
__attribute__((visibility("default"))) int fake_copies_under_way() { return static_cast<int>(copies[0].size() + copies[1].size()); }
__attribute__((visibility("default"))) int fake_blocks() { return static_cast<int>(blocks.size()); }
__attribute__((visibility("default"))) long long fake_violations() { return violations; }
__attribute__((visibility("default"))) long long fake_adamw_launches() { return adamw_launches; }
__attribute__((visibility("default"))) int fake_adamw_masters() { return masters; }
__attribute__((visibility("default"))) void fake_set_device(int dev) { current = dev; }
__attribute__((visibility("default"))) int fake_device() { return current; }

cudaError_t cudaMalloc(void** p, size_t bytes) {
  if (fail_in >= 0 && fail_in-- == 0) { *p = nullptr; return cudaErrorMemoryAllocation; }
  *p = aligned_alloc(256, (bytes + 255) / 256 * 256);
  memset(*p, 0x5a, bytes);
  blocks[static_cast<char*>(*p)] = bytes;
  return cudaSuccess;
}
cudaError_t cudaFree(void* p) {
  if (!p) return cudaSuccess;
  wait(0); wait(1);
  if (!blocks.erase(static_cast<char*>(p))) { ++violations; return cudaErrorInvalidValue; }
  free(p);
  return cudaSuccess;
}
cudaError_t cudaMallocHost(void** p, size_t bytes) { *p = malloc(bytes); return cudaSuccess; }
cudaError_t cudaFreeHost(void* p) { free(p); return cudaSuccess; }
__attribute__((visibility("default"))) void* fake_malloc(size_t bytes) { void* p; return cudaMalloc(&p, bytes) == cudaSuccess ? p : nullptr; }
__attribute__((visibility("default"))) void fake_free(void* p) { cudaFree(p); }
cudaError_t cudaMemcpy(void* dst, const void* src, size_t bytes, cudaMemcpyKind kind) {
  for (const Copy& c : copies[current]) memcpy(c.dst, c.bytes.data(), c.bytes.size());              // copies of one stream come in order
  copies[current].clear();
  if (kind == cudaMemcpyHostToDevice && late) copies[current].push_back({dst, std::vector<char>(static_cast<const char*>(src), static_cast<const char*>(src) + bytes)});
  else memcpy(dst, src, bytes);
  return cudaSuccess;
}
cudaError_t cudaMemcpyAsync(void* dst, const void* src, size_t bytes, cudaMemcpyKind, cudaStream_t) { memcpy(dst, src, bytes); return cudaSuccess; }
cudaError_t cudaMemset(void* dst, int v, size_t bytes) { memset(dst, v, bytes); return cudaSuccess; }
cudaError_t cudaMemsetAsync(void* dst, int v, size_t bytes, cudaStream_t) { memset(dst, v, bytes); return cudaSuccess; }
cudaError_t cudaDeviceSynchronize() { wait(current); return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { wait(current); return cudaSuccess; }
cudaError_t cudaGetDevice(int* dev) { *dev = current; return cudaSuccess; }
cudaError_t cudaSetDevice(int dev) { if (dev < 0 || dev > 1) return cudaErrorInvalidDevice; current = dev; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int) { *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : 148; return cudaSuccess; }
cudaError_t cudaGetDeviceProperties_v2(cudaDeviceProp* p, int) { memset(p, 0, sizeof(*p)); p->multiProcessorCount = 148; p->major = 10; return cudaSuccess; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t* e, unsigned) { *e = reinterpret_cast<cudaEvent_t>(malloc(1)); return cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t e) { free(e); return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaStreamCreateWithFlags(cudaStream_t* s, unsigned) { *s = reinterpret_cast<cudaStream_t>(malloc(1)); return cudaSuccess; }
cudaError_t cudaStreamDestroy(cudaStream_t s) { free(s); return cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t, cudaEvent_t, unsigned) { return cudaSuccess; }
cudaError_t cudaStreamBeginCapture(cudaStream_t, cudaStreamCaptureMode) { capture = new Graph; return cudaSuccess; }
cudaError_t cudaStreamEndCapture(cudaStream_t, cudaGraph_t* g) { *g = reinterpret_cast<cudaGraph_t>(capture); capture = nullptr; return cudaSuccess; }
cudaError_t cudaGraphDestroy(cudaGraph_t g) { delete reinterpret_cast<Graph*>(g); return cudaSuccess; }
cudaError_t cudaGraphInstantiate(cudaGraphExec_t* e, cudaGraph_t g, unsigned long long) {
  *e = reinterpret_cast<cudaGraphExec_t>(new Graph(*reinterpret_cast<Graph*>(g)));
  return cudaSuccess;
}
cudaError_t cudaGraphExecDestroy(cudaGraphExec_t e) { delete reinterpret_cast<Graph*>(e); return cudaSuccess; }
cudaError_t cudaGraphLaunch(cudaGraphExec_t e, cudaStream_t) {
  for (const AdamWLaunch& l : reinterpret_cast<Graph*>(e)->launches) launch(l);
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int* n, const void*, int, size_t, unsigned) { *n = 2; return cudaSuccess; }
// the only kernel of adamw.cu: (tensors, first, count, total, lg, clock, ...)
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void** a) {
  const AdamWLaunch l{*static_cast<const char**>(a[0]), *static_cast<const int**>(a[1]), *static_cast<int*>(a[2]), *static_cast<char**>(a[5]), current};
  if (capture) capture->launches.push_back(l);
  else launch(l);
  return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaSuccess; }
void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, void*, void*, void*, void*, int*) {}
char __cudaInitModule(void**) { return 1; }
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
}

namespace mbd {
bool pdl_enabled() { return false; }
void tc_gemm_plan(TcGemm&, int, bool) {}
cudaError_t tc_gemm_prepare(TcGemm& g, const void*, int64_t, const void*, int64_t, int, const Epi*) { g.k_splits = 1; return cudaSuccess; }
cudaError_t tc_gemm_launch(const TcGemm&, cudaStream_t) { return cudaSuccess; }
cudaError_t selftest_timeout_launch(int*, int, cudaStream_t) { return cudaSuccess; }
cudaError_t simt_gemm_launch(const SimtGemm&, cudaStream_t) { return cudaSuccess; }
cudaError_t reduce_partials_launch(const float*, int, int64_t, int64_t, const Epi&, int, cudaStream_t) { return cudaSuccess; }
cudaError_t softmax_xent_launch(const float*, int64_t, int64_t, const int32_t*, void*, int, float*, cudaStream_t) { return cudaSuccess; }
cudaError_t sum_f32_launch(const float*, int64_t, float, float*, cudaStream_t) { return cudaSuccess; }
cudaError_t colsum_launch(const void*, int, int64_t, int64_t, float*, int, float*, float*, float, cudaStream_t) { return cudaSuccess; }
int colsum_row_splits(int64_t, int64_t, int) { return 1; }
int colsum_launches(int64_t, int64_t, int) { return 1; }
cudaError_t sgd_update_launch(void*, int, const float*, int64_t, float, int, cudaStream_t) { return cudaSuccess; }
cudaError_t sgd_momentum_update_launch(void* w, int, float*, float* v, const float*, int64_t, float, float, float, int, cudaStream_t) {
  if (!live(w) || !live(v)) ++violations;
  return cudaSuccess;
}
cudaError_t sgd_master_update_launch(float* w32, void*, const float*, int64_t, float, int, cudaStream_t) {
  if (!live(w32)) ++violations;
  return cudaSuccess;
}
cudaError_t widen_bf16_launch(const void*, float*, int64_t, int, cudaStream_t) { return cudaSuccess; }
void Profiler::begin(int, double, cudaStream_t) {}
void Profiler::end() {}
void Profiler::collect() {}
void Profiler::reset() {}
void Profiler::destroy() {}

// no convolutions here
mbd_status conv_create(const mbd_layer*, int, int64_t, int, int, int, int, int*, cudaStream_t, Profiler*, bool, ConvNet**) { return MBD_E_UNSUPPORTED; }
void conv_destroy(ConvNet*) {}
mbd_status conv_set_weights(ConvNet*, int, const void*) { return MBD_E_UNSUPPORTED; }
mbd_status conv_get_weights(ConvNet*, int, void*) { return MBD_E_UNSUPPORTED; }
mbd_status conv_forward(ConvNet*, const void*, float*) { return MBD_E_UNSUPPORTED; }
mbd_status conv_backward(ConvNet*, float) { return MBD_E_UNSUPPORTED; }
mbd_status conv_sgd_step(ConvNet*, float) { return MBD_E_UNSUPPORTED; }
mbd_status conv_get_tensor(ConvNet*, int, int, void*, size_t) { return MBD_E_UNSUPPORTED; }
mbd_status conv_set_tensor(ConvNet*, int, int, const void*, size_t) { return MBD_E_UNSUPPORTED; }
size_t conv_input_bytes(const ConvNet*) { return 0; }
mbd_status conv_output_to_nchw(ConvNet*, void*) { return MBD_E_UNSUPPORTED; }
mbd_status conv_top_grad_from_nchw(ConvNet*, const void*) { return MBD_E_UNSUPPORTED; }
int conv_last_relu(const ConvNet*) { return 0; }
mbd_status conv_enable_master(ConvNet*) { return MBD_E_UNSUPPORTED; }
mbd_status conv_enable_momentum(ConvNet*, float) { return MBD_E_UNSUPPORTED; }
mbd_status conv_stage_input(ConvNet*, const void*) { return MBD_E_UNSUPPORTED; }
mbd_status conv_forward_layer(ConvNet*, int, float*, int) { return MBD_E_UNSUPPORTED; }
mbd_status conv_backward_layer(ConvNet*, int, float, int) { return MBD_E_UNSUPPORTED; }
mbd_status conv_outer_rows(ConvNet*, int, int, int, void*, size_t, int) { return MBD_E_UNSUPPORTED; }
mbd_status conv_set_dw(ConvNet*, int, const void*, size_t) { return MBD_E_UNSUPPORTED; }
mbd_status conv_get_product(const ConvNet*, int, int, const TcGemm**) { return MBD_E_UNSUPPORTED; }
}  // namespace mbd
