// Activation functions whose input is saved in 8 bits (hq_act_save8), and their backward pass from what was saved
// (hq_act_backward8).  Both are one pass over the data: a thread holds eight neighbouring values of a row, a group is held by
// group / 8 neighbouring lanes of one warp, which agree on its largest magnitude by shuffles.
#include "float_internal.cuh"

namespace {

constexpr int kThreads = 256, kVec = 8;

// Eight values from memory; `n` of them exist (n < 8 only without VEC).
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* src, int n, float (&v)[kVec]) {
  if (VEC) {
    constexpr int kWords = kVec * sizeof(T) / 16;
    uint4 w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = ((const uint4*)src)[i];
    const T* t = (const T*)w;
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = hq_to_float(t[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = i < n ? hq_to_float(src[i]) : 0.f;
  }
}
template <class T, bool VEC>
__device__ __forceinline__ void store8(T* dst, int n, const float (&v)[kVec]) {
  if (VEC) {
    constexpr int kWords = kVec * sizeof(T) / 16;
    uint4 w[kWords];
    T* t = (T*)w;
#pragma unroll
    for (int i = 0; i < kVec; ++i) t[i] = hq_from_float<T>(v[i]);
#pragma unroll
    for (int i = 0; i < kWords; ++i) ((uint4*)dst)[i] = w[i];
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) if (i < n) dst[i] = hq_from_float<T>(v[i]);
  }
}

template <int ACT>
__device__ __forceinline__ float f_of(float x) {
  if (ACT == HQ_ACT_RELU) return x < 0.f ? 0.f : x;                 // (a NaN stays one)
  if (ACT == HQ_ACT_GELU) return x * normcdff(x);
  if (ACT == HQ_ACT_SILU) return x / (1.f + expf(-x));
  return x;
}
template <int ACT>
__device__ __forceinline__ float df_of(float x) {
  if (ACT == HQ_ACT_RELU) return x > 0.f ? 1.f : 0.f;
  if (ACT == HQ_ACT_GELU) return normcdff(x) + x * (expf(-0.5f * x * x) * 0.3989422804014327f);
  if (ACT == HQ_ACT_SILU) { const float p = 1.f / (1.f + expf(-x)); return p * (1.f + x * (1.f - p)); }
  return 1.f;
}

// Scale of a group from its largest magnitude, given as the bits of a non-negative float: in that order NaN > infinity > any
// finite value, so that one integer maximum finds all three.
__device__ __forceinline__ float group_scale(unsigned amax_bits) {
  return amax_bits >= 0x7f800000u ? __int_as_float(0x7fffffff) : __fdiv_rn(__uint_as_float(amax_bits), 127.f);
}

// q = x / s rounded to the nearest integer, ties to even, of the EXACT quotient (half of a group's largest value lies next to the
// border between 63 and 64, so a rounded quotient would often end on the wrong side).  The estimate t = round(x * (1 / s)) is off
// by one at most, next to a border; x - t s is a multiple of the last place of s, below s in magnitude, hence exact in 32 bits
// (for |x| < s it is x itself or, by Sterbenz, exact again), and its comparison with s / 2 decides.
__device__ __forceinline__ int quantize(float x, float s, float inv, float half) {
  constexpr float kMagic = 12582912.f;                              // 1.5 * 2^23: the sum's low bits are the integer
  const float u = fmaf(x, inv, kMagic);
  const float t = u - kMagic;
  const float rest = fmaf(-t, s, x);
  int q = __float_as_int(u);
  if (fabsf(rest) > half || (fabsf(rest) == half && (q & 1))) q += rest > 0.f ? 1 : -1;
  return q;
}
__device__ __forceinline__ uint2 quantize8(const float (&x)[kVec], float s) {
  int q[kVec];
  if (s >= 0x1p-100f) {
    const float inv = __frcp_rn(s), half = 0.5f * s;
#pragma unroll
    for (int i = 0; i < kVec; ++i) q[i] = quantize(x[i], s, inv, half);
  } else {                                                          // 0, NaN, or so small that 1 / s leaves the 32-bit range
#pragma unroll
    for (int i = 0; i < kVec; ++i) q[i] = s > 0.f ? __double2int_rn((double)x[i] / (double)s) : 0;
  }
  uint2 w;
  w.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
  w.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
  return w;
}

// Quantizes the eight values held by each lane of a group and stores integers and scale.  Every lane of the warp takes part.
template <bool VEC>
__device__ __forceinline__ void save_group(const float (&v)[kVec], int lanes, int lane_in_group, int8_t* q, float* scale, int n) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < kVec; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  for (int d = 1; d < lanes; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
  const float s = group_scale(top);
  const uint2 w = quantize8(v, s);
  if (VEC) {
    if (n > 0) *(uint2*)q = w;
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) if (i < n) q[i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
  }
  if (lane_in_group == 0 && n > 0) *scale = s;
}

template <bool VEC>
__device__ __forceinline__ void restore8(const int8_t* q, float s, int n, float (&v)[kVec]) {
  if (VEC) {
    const uint2 w = *(const uint2*)q;
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = (float)(int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3))) * s;
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = i < n ? (float)q[i] * s : 0.f;
  }
}

// Where a thread works: slot = eight columns of a row, slots of a row filled up to whole groups.
struct Slot { long long row; int col, n; };
__device__ __forceinline__ Slot slot_of(long long slot, long long slots, int per_row, int cols) {
  Slot at;
  int in_row;
  if (slots <= 0x7fffffffll) { const unsigned r = (unsigned)slot / (unsigned)per_row; at.row = r; in_row = (int)((unsigned)slot - r * (unsigned)per_row); }
  else { at.row = slot / per_row; in_row = (int)(slot - at.row * per_row); }
  at.col = in_row * kVec;
  at.n = slot < slots ? max(0, min(kVec, cols - at.col)) : 0;
  return at;
}

template <class T, int ACT, bool VEC>
__global__ void __launch_bounds__(kThreads) act_save8_kernel(const ActArgs p, long long slots) {
  hq_pdl_entry();
  const int lanes = p.group / kVec, per_row = p.groups * lanes;
  const Slot at = slot_of((long long)blockIdx.x * kThreads + threadIdx.x, slots, per_row, p.cols);
  const int lane_in_group = threadIdx.x & (lanes - 1);
  const long long flat = at.row * p.cols + at.col;
  float x[kVec] = {}, g[kVec] = {};
  if (at.n > 0) load8<T, VEC>((const T*)p.x + at.row * p.x_stride + at.col, at.n, x);
  if (at.n > 0 && p.gate) load8<T, VEC>((const T*)p.gate + at.row * p.gate_stride + at.col, at.n, g);
  const long long group_at = at.row * p.groups + at.col / p.group;
  save_group<VEC>(x, lanes, lane_in_group, p.xq + flat, p.xs + group_at, at.n);
  if (p.gate) save_group<VEC>(g, lanes, lane_in_group, p.gq + flat, p.gs + group_at, at.n);
  if (p.y && at.n > 0) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) x[i] = f_of<ACT>(x[i]) * (p.gate ? g[i] : 1.f);
    store8<T, VEC>((T*)p.y + at.row * p.y_stride + at.col, at.n, x);
  }
}

template <class T, int ACT, bool VEC>
__global__ void __launch_bounds__(kThreads) act_backward8_kernel(const ActArgs p, long long slots) {
  hq_pdl_entry();
  const int per_row = p.groups * (p.group / kVec);
  const Slot at = slot_of((long long)blockIdx.x * kThreads + threadIdx.x, slots, per_row, p.cols);
  if (at.n == 0) return;
  const long long flat = at.row * p.cols + at.col;
  const long long group_at = at.row * p.groups + at.col / p.group;
  float dy[kVec], x[kVec], out[kVec];
  load8<T, VEC>((const T*)p.x + at.row * p.x_stride + at.col, at.n, dy);
  restore8<VEC>(p.xq + flat, p.xs[group_at], at.n, x);
  if (p.gq) {
    float g[kVec];
    restore8<VEC>(p.gq + flat, p.gs[group_at], at.n, g);
#pragma unroll
    for (int i = 0; i < kVec; ++i) out[i] = dy[i] * f_of<ACT>(x[i]);
    store8<T, VEC>((T*)p.dgate + at.row * p.dgate_stride + at.col, at.n, out);
#pragma unroll
    for (int i = 0; i < kVec; ++i) dy[i] *= g[i];
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) out[i] = dy[i] * df_of<ACT>(x[i]);
  store8<T, VEC>((T*)p.y + at.row * p.y_stride + at.col, at.n, out);
}

// Whole 16-byte pieces everywhere: pitches that keep every row on its 16 bytes, and whole eights of columns.
bool vectors(int type, const ActArgs& a) {
  const long long per16 = type == HQ_F32 ? 4 : 8;
  const bool strides = a.x_stride % per16 == 0 && (!a.gate || a.gate_stride % per16 == 0) && (!a.y || a.y_stride % per16 == 0) &&
                       (!a.dgate || a.dgate_stride % per16 == 0);
  return strides && a.cols % kVec == 0;
}

template <bool SAVE, class T, int ACT>
cudaError_t launch_act(const ActArgs& a, bool vec, cudaStream_t s) {
  const long long slots = a.rows * a.groups * (a.group / kVec);
  const long long blocks = (slots + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kThreads);
  if (SAVE) return vec ? hq_launch_pdl(act_save8_kernel<T, ACT, true>, grid, block, 0, s, a, slots)
                       : hq_launch_pdl(act_save8_kernel<T, ACT, false>, grid, block, 0, s, a, slots);
  return vec ? hq_launch_pdl(act_backward8_kernel<T, ACT, true>, grid, block, 0, s, a, slots)
             : hq_launch_pdl(act_backward8_kernel<T, ACT, false>, grid, block, 0, s, a, slots);
}
template <bool SAVE, class T>
cudaError_t launch_type(const ActArgs& a, bool vec, cudaStream_t s) {
  switch (a.act) {
    case HQ_ACT_RELU: return launch_act<SAVE, T, HQ_ACT_RELU>(a, vec, s);
    case HQ_ACT_GELU: return launch_act<SAVE, T, HQ_ACT_GELU>(a, vec, s);
    case HQ_ACT_SILU: return launch_act<SAVE, T, HQ_ACT_SILU>(a, vec, s);
    default: return launch_act<SAVE, T, HQ_ACT_NONE>(a, vec, s);
  }
}
template <bool SAVE>
cudaError_t launch(int type, const ActArgs& a, cudaStream_t s) {
  const bool vec = vectors(type, a);
  return type == HQ_F32 ? launch_type<SAVE, float>(a, vec, s)
       : type == HQ_F16 ? launch_type<SAVE, __half>(a, vec, s) : launch_type<SAVE, __nv_bfloat16>(a, vec, s);
}

}  // namespace

cudaError_t hq_launch_act_save8(int type, const ActArgs& a, cudaStream_t s) { return launch<true>(type, a, s); }
cudaError_t hq_launch_act_backward8(int type, const ActArgs& a, cudaStream_t s) { return launch<false>(type, a, s); }
