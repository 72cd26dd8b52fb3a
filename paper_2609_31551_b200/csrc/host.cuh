// Host-side plumbing of the library's translation units: error text, tensor maps, the device check, kernel launches.
#pragma once
#include "../../include/eas_encoder.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>

#include <cstdarg>
#include <cstdio>
#include <mutex>

namespace eas {

// ------------------------------------------------------------------------------------ errors
inline thread_local char g_err[512] = "";
inline eas_status fail(eas_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return s;
}
#define CUDA_TRY(expr)                                                                              \
  do {                                                                                              \
    cudaError_t e_ = (expr);                                                                        \
    if (e_ != cudaSuccess) return fail(EAS_ERR_CUDA, "%s failed: %s", #expr, cudaGetErrorString(e_)); \
  } while (0)

#define EAS_TRY(expr)            \
  do {                           \
    eas_status s_ = (expr);      \
    if (s_ != EAS_OK) return s_; \
  } while (0)

// ------------------------------------------------------------------------------------ tensor maps
inline PFN_cuTensorMapEncodeTiled_v12000 get_encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  if (fn == nullptr) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) == cudaSuccess &&
        qres == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }
  return fn;
}

// bf16 tensor map.  dims/strides innermost first; strides (bytes) for dims 1..rank-1.
inline eas_status make_tmap(CUtensorMap* m, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
                            const uint32_t* box, CUtensorMapSwizzle swz) {
  PFN_cuTensorMapEncodeTiled_v12000 fn = get_encode_fn();
  if (fn == nullptr) return fail(EAS_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  cuuint64_t gdim[5], gstr[5];
  cuuint32_t bx[5], es[5];
  for (int i = 0; i < rank; ++i) { gdim[i] = dims[i]; bx[i] = box[i]; es[i] = 1; }
  for (int i = 0; i + 1 < rank; ++i) gstr[i] = strides[i];
  CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), gdim, gstr, bx, es,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, swz, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(EAS_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", static_cast<int>(r));
  return EAS_OK;
}

// ------------------------------------------------------------------------------------ device and launches
// Kernel attributes (the dynamic shared-memory limit) belong to a device's context: they are set once per DEVICE, the
// first time a launch site is reached with that device current.
struct OncePerDevice {
  std::mutex m;
  bool done[64] = {};
  // true until settled() has been called with this device current (always true for ordinals past the table: the
  // attribute is then set every time).  A failed attribute call returns before settled(), so the next launch retries.
  bool first() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return true;
    std::lock_guard<std::mutex> lock(m);
    return !done[dev];
  }
  void settled() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return;
    std::lock_guard<std::mutex> lock(m);
    done[dev] = true;
  }
};

// shared memory requested by the light kernels: more than half an SM's capacity, so that a second CTA
// can never be co-resident and a grid of B CTAs occupies B SMs
constexpr int kOnePerSmSmem = 120 * 1024;

inline eas_status device_check(int* sm_count, int* device = nullptr) {
  int dev = 0;
  CUDA_TRY(cudaGetDevice(&dev));
  if (device != nullptr) *device = dev;
  int major = 0, minor = 0, sms = 0;
  CUDA_TRY(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
  CUDA_TRY(cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev));
  CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  if (major != 10) return fail(EAS_ERR_ARCH, "device is compute capability %d.%d; this library is built for 10.x", major, minor);
  *sm_count = sms;
  return EAS_OK;
}

// All kernels are launched with programmatic stream serialization and wait (griddepcontrol.wait) before touching any data.
// In a call that owns the whole device they release their successor at their start, so that it sets itself up while they
// run.  A call on a SHARE of the SMs (Section 3.4) must not do that: its grids are persistent (all CTAs resident at once), so
// a dependent kernel would be released the moment its predecessor started, its CTAs would settle on SMs outside the share and
// sit there holding shared memory and tensor memory while they wait -- exactly the SMs the co-resident worker was
// promised.  There the successor is released by the exit of the predecessor's last CTA: at most `sm_budget` SMs hold a CTA
// of the call at any time, and only the completion of the predecessor (its flush, 1-2 us) overlaps the launch.  From a
// kernel's last CTA to the next one past its wait, 32 images of 577 tokens on 74 SMs: 4.0-4.9 us without the attribute, 2.0-2.3
// this way, 1.0-1.7 with the early release (on all SMs).  Set by every entry point before its first launch (per host thread).
inline thread_local bool g_overlap_launches = true;
inline thread_local int g_device_sms = 0;      // SMs of the device, set with it
template <typename Params>
inline eas_status launch_kernel(void (*kern)(Params), int grid, int block, size_t smem, cudaStream_t stream, const Params& params,
                                int cluster = 1) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
  cfg.blockDim = dim3(static_cast<unsigned>(block), 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[n].val.programmaticStreamSerializationAllowed = 1;
  ++n;
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[n].val.clusterDim.y = 1;
    attr[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  Params q = params;
  q.early_launch = g_overlap_launches ? 1 : 0;
  CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, q));
  return EAS_OK;
}

// sm_budget of a call without a handle: 0 = all SMs of the current device
inline eas_status resolve_budget(int32_t sm_budget, int* budget) {
  int sm_count = 0;
  EAS_TRY(device_check(&sm_count));
  if (sm_budget < 0 || sm_budget > sm_count) return fail(EAS_ERR_INVALID_ARG, "sm_budget %d outside 0..%d", sm_budget, sm_count);
  *budget = sm_budget == 0 ? sm_count : sm_budget;
  g_overlap_launches = *budget == sm_count;
  g_device_sms = sm_count;
  return EAS_OK;
}

}  // namespace eas
