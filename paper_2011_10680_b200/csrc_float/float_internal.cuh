// Internal declarations of the operators on floating-point activations (4-bit weights with group scales, activations saved
// in 8 bits).  They live apart from csrc/, the integer-only inference pipeline, which holds no floating point.
#pragma once

#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../csrc/hq_internal.cuh"

// The three products share one shape:  out[j][i] = bias[i] + sum_r A(i, r) * B(j, r),  i contiguous in `out`, A the quantized
// operand, B the floating-point one.
//   FORWARD  A(i, r) = w[i][r]              B(j, r) = x[j][r]     (i: outputs, j: tokens, r: inputs)
//   DGRAD    A(i, r) = w[r][i]              B(j, r) = dy[j][r]    (i: inputs, j: tokens, r: outputs)
//   WGRAD    A(i, r) = saved[r][i]          B(j, r) = dy[r][j]    (i: inputs, j: outputs, r: tokens)
enum ProductKind { PRODUCT_FORWARD = 0, PRODUCT_DGRAD = 1, PRODUCT_WGRAD = 2 };

struct ProductArgs {
  const void* q;            // packed 4-bit integers [n][k/2] (FORWARD, DGRAD) or bytes [m][k] (WGRAD)
  const void* scale;        // per group of a row of q: the activations' type, or float (WGRAD)
  int32_t q_cols;           // values per row of q
  int32_t groups, group;    // scales per row of q, values per scale
  const void* b;            // floating-point operand
  long long b_stride;       // values between its rows
  const void* bias;         // per i, or NULL
  void* out;
  long long out_stride;
  int32_t i, j, r;          // extents
};

struct ActArgs {
  const void* x;  long long x_stride;       // forward: input; backward: dy
  const void* gate; long long gate_stride;  // forward, or NULL
  void* y; long long y_stride;              // forward: output or NULL; backward: dx
  void* dgate; long long dgate_stride;      // backward, or NULL
  int8_t* xq; float* xs;                    // saved input
  int8_t* gq; float* gs;                    // saved gate, or NULL
  long long rows; int32_t cols, group, groups;
  int32_t act;
  int32_t sm_count;
};

__device__ __forceinline__ float hq_to_float(float v) { return v; }
__device__ __forceinline__ float hq_to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float hq_to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T hq_from_float(float v);
template <> __device__ __forceinline__ float hq_from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half hq_from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 hq_from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Value `col` of a row of packed 4-bit integers.
__device__ __forceinline__ int hq_nibble(const uint8_t* row, int col) {
  const int v = (row[col >> 1] >> ((col & 1) * 4)) & 15;
  return (v ^ 8) - 8;
}

// Up to 16 rows of FORWARD (product_few.cu).
bool hq_product_few_supported(const ProductArgs& a, int sm_count);
hq_status hq_launch_product_few(hq_handle* h, int type, const ProductArgs& a, cudaStream_t s);
// On the tensor cores (product_tc.cu): every shape whose rows start on 16 bytes.  hq_launch_product_any takes all of them.
bool hq_product_tc_supported(ProductKind kind, const ProductArgs& a);
hq_status hq_launch_product_tc(hq_handle* h, ProductKind kind, int type, const ProductArgs& a, cudaStream_t s);
// The launch of a shape, for hq_linear_plan; false where the kernel does not take it.
bool hq_plan_product_few(const ProductArgs& a, int sm_count, hq_product_plan* plan);
bool hq_plan_product_tc(ProductKind kind, const ProductArgs& a, int sm_count, hq_product_plan* plan);
cudaError_t hq_launch_product_any(ProductKind kind, int type, const ProductArgs& a, cudaStream_t s);
// Lets a kernel have that much dynamic shared memory: at its first launch on a device (`done` is the kernel's own), not when a handle is
// made, so that a program pays for the kernels that it uses and depends on no others.  Allowed while a stream is capturing.
constexpr int kMaxDevices = 64;
template <class Kernel>
inline cudaError_t hq_allow_shared(std::atomic<bool> (&done)[kMaxDevices], int device, Kernel kernel, int bytes) {
  if (device < kMaxDevices && done[device].load()) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && device < kMaxDevices) done[device].store(true);
  return e;
}
cudaError_t hq_launch_act_save8(int type, const ActArgs& a, cudaStream_t s);
cudaError_t hq_launch_act_backward8(int type, const ActArgs& a, cudaStream_t s);
