// The three products on the CUDA cores, for every shape, stride and group: 64 x 64 outputs per block, 16 steps of the reduction
// at a time through shared memory, 32-bit multiply-adds on values restored in 32 bits.  The plain path: the shapes that the
// tensor-core kernels cannot fetch (rows whose pitch is no multiple of 16 bytes) end here.
#include "float_internal.cuh"

namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256;

template <int KIND, class T>
__device__ __forceinline__ float quantized(const ProductArgs& p, int i, int r) {
  if (KIND == PRODUCT_FORWARD) {
    const uint8_t* row = (const uint8_t*)p.q + (long long)i * (p.q_cols >> 1);
    return (float)hq_nibble(row, r) * hq_to_float(((const T*)p.scale)[(long long)i * p.groups + r / p.group]);
  }
  if (KIND == PRODUCT_DGRAD) {
    const uint8_t* row = (const uint8_t*)p.q + (long long)r * (p.q_cols >> 1);
    return (float)hq_nibble(row, i) * hq_to_float(((const T*)p.scale)[(long long)r * p.groups + i / p.group]);
  }
  return (float)((const int8_t*)p.q)[(long long)r * p.q_cols + i] * ((const float*)p.scale)[(long long)r * p.groups + i / p.group];
}

template <int KIND, class T>
__global__ void __launch_bounds__(kThreads) product_any_kernel(const ProductArgs p, int i_tiles) {
  hq_pdl_entry();
  __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
  const int i0 = (int)(blockIdx.x % (unsigned)i_tiles) * kTile, j0 = (int)(blockIdx.x / (unsigned)i_tiles) * kTile;
  const int ti = threadIdx.x % 16, tj = threadIdx.x / 16;
  float acc[4][4] = {};
  for (int r0 = 0; r0 < p.r; r0 += kStep) {
    for (int e = threadIdx.x; e < kTile * kStep; e += kThreads) {
      // neighbouring threads along the contiguous direction of each operand
      const int ai = KIND == PRODUCT_FORWARD ? e / kStep : e % kTile, ar = KIND == PRODUCT_FORWARD ? e % kStep : e / kTile;
      const int bj = KIND == PRODUCT_WGRAD ? e % kTile : e / kStep, br = KIND == PRODUCT_WGRAD ? e / kTile : e % kStep;
      sa[ar][ai] = (i0 + ai < p.i && r0 + ar < p.r) ? quantized<KIND, T>(p, i0 + ai, r0 + ar) : 0.f;
      const long long at = KIND == PRODUCT_WGRAD ? (long long)(r0 + br) * p.b_stride + j0 + bj : (long long)(j0 + bj) * p.b_stride + r0 + br;
      sb[br][bj] = (j0 + bj < p.j && r0 + br < p.r) ? hq_to_float(((const T*)p.b)[at]) : 0.f;
    }
    __syncthreads();
    const int steps = min(kStep, p.r - r0);
    for (int r = 0; r < steps; ++r) {
      float a[4], b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) { a[u] = sa[r][ti + 16 * u]; b[u] = sb[r][tj + 16 * u]; }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] = fmaf(a[u], b[v], acc[u][v]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int i = i0 + ti + 16 * u;
    if (i >= p.i) continue;
    const float add = p.bias ? hq_to_float(((const T*)p.bias)[i]) : 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int j = j0 + tj + 16 * v;
      if (j < p.j) ((T*)p.out)[(long long)j * p.out_stride + i] = hq_from_float<T>(acc[u][v] + add);
    }
  }
}

template <int KIND>
cudaError_t launch(int type, const ProductArgs& a, cudaStream_t s) {
  const long long it = (a.i + kTile - 1) / kTile, jt = (a.j + kTile - 1) / kTile;
  if (it * jt > 0x7fffffffll) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)(it * jt));
  if (type == HQ_F16) return hq_launch_pdl(product_any_kernel<KIND, __half>, grid, dim3(kThreads), 0, s, a, (int)it);
  return hq_launch_pdl(product_any_kernel<KIND, __nv_bfloat16>, grid, dim3(kThreads), 0, s, a, (int)it);
}

}  // namespace

cudaError_t hq_launch_product_any(ProductKind kind, int type, const ProductArgs& a, cudaStream_t s) {
  return kind == PRODUCT_FORWARD ? launch<PRODUCT_FORWARD>(type, a, s)
       : kind == PRODUCT_DGRAD ? launch<PRODUCT_DGRAD>(type, a, s) : launch<PRODUCT_WGRAD>(type, a, s);
}
