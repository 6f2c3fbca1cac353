// What the host sides of the C ABI share: error reporting, argument checks, the
// device of a stream, TMA map encoding.  Defined in mw_abi.cu unless inline here.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>

#include "mw_bca.h"
#include "mw_internal.h"

#define MW_TRY(expr)                 \
  do {                               \
    mw_status _s = (expr);           \
    if (_s != MW_OK) return _s;      \
  } while (0)

namespace mw {

// Records the calling thread's error message and hands the status back.
mw_status fail(mw_status s, const char* fmt, ...);
// Clears it.
mw_status ok();

bool aligned16(const void* p);
// Rows of d bf16 from p all start at multiples of 32 bytes.
bool wide_rows(const void* p, int d);
mw_status check_ptr(const void* p, const char* name);

bool d_supported(int d);
int kernel_d(int d);
int mma_d(int d);
mw_status check_dims(int B, int H, int d);
mw_status check_rows(long long rows, const char* what);
mw_status check_tokens(long long BH, long long rows);

// Map over [BH, rows, d] (see encode_map in mw_abi.cu), from a small cache of the
// calling thread.
mw_status make_map(CUtensorMap* m, const void* ptr, int rows, int BH, int d, const char* name,
                   int box_rows = kTileRows, bool f32 = false, int cols = 0);
// Map over the backward's bias rows [BH, N_pad, 8] f32.
mw_status encode_bias_map(CUtensorMap* m, const float* bias, int N_pad, int BH, int box_rows);
// Map over bf16 rows [BH, rows, d] in boxes of 32 rows: x 64 columns with the 128-byte
// swizzle, or x 32 without.
mw_status encode_rows_map(CUtensorMap* m, void* ptr, int rows, int BH, int d, bool swizzle);

// The device status word of the current device `dev`.
mw_status status_ptr(int dev, unsigned** out);
// SM count of the current device, queried once per device.
int sm_count();
// Budget of a kernel's wait (option wait_budget_ms).
unsigned long long budget_ns();
// Test hook (option debug_skip_q_load): bit 0 for the even CTAs, bit 1 for the odd ones.
int debug_skip_q();

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
inline int ceil_div(long long a, long long b) { return static_cast<int>((a + b - 1) / b); }

// Makes the device of `stream` current on the calling thread for the scope
// of one entry point (binding its primary context, which driver calls such
// as cuTensorMapEncodeTiled need on threads where nothing else did), and
// restores the caller's device afterwards.
class DeviceScope {
 public:
  explicit DeviceScope(cudaStream_t stream) {
    if (cudaGetDevice(&prev_) != cudaSuccess) prev_ = -1;
    int dev = prev_;
    // (cudaStreamGetDevice is not allowed on a stream under graph capture,
    // and a capturing stream belongs to the current device anyway)
    cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
    if (stream != nullptr && cudaStreamIsCapturing(stream, &cs) == cudaSuccess &&
        cs == cudaStreamCaptureStatusNone && cudaStreamGetDevice(stream, &dev) != cudaSuccess)
      dev = prev_;
    if (dev < 0) dev = 0;
    err_ = cudaSetDevice(dev);
    dev_ = dev;
  }
  ~DeviceScope() {
    if (prev_ >= 0 && prev_ != dev_) cudaSetDevice(prev_);
  }
  mw_status status() const {
    if (err_ != cudaSuccess) return fail(MW_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(err_));
    return MW_OK;
  }
  int device() const { return dev_; }

 private:
  int prev_ = -1, dev_ = 0;
  cudaError_t err_ = cudaSuccess;
};

inline mw_status launch_status(cudaError_t e, const char* what) {
  if (e != cudaSuccess) return fail(MW_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
  return ok();
}

}  // namespace mw
