// Activation functions whose input is saved in 8 bits (hq_act_save8), and their backward pass from what was saved
// (hq_act_backward8).  Both are one pass over the data and bound by it: a thread holds eight neighbouring values of a row (of two rows,
// or four where one 16-bit tensor is read, to keep enough bytes in flight), a group is held by group / 8 neighbouring lanes of one
// warp, which agree on its largest magnitude by shuffles.  At the memory's rate a value of a gated 16-bit pass has about 40
// instruction slots, so the functions are made of the hardware's exponential and reciprocal, and an 8-bit integer of a 16-bit
// value is one multiply-add.
#include "float_internal.cuh"

namespace {

constexpr int kThreads = 256, kVec = 8;

// Eight values as they lie in memory; `n` of them exist (n < 8 only without VEC).  Kept like this until they are used: a thread then
// has several pieces on their way.
template <class T> struct Raw { uint4 w[kVec * sizeof(T) / 16]; };
template <class T, bool VEC>
__device__ __forceinline__ void fetch8(const T* src, int n, Raw<T>& v) {
#pragma unroll
  for (int i = 0; i < (int)(kVec * sizeof(T) / 16); ++i) v.w[i] = make_uint4(0, 0, 0, 0);
  if (n == 0) return;
  if (VEC) {
#pragma unroll
    for (int i = 0; i < (int)(kVec * sizeof(T) / 16); ++i) v.w[i] = ((const uint4*)src)[i];
  } else {
    T* t = (T*)v.w;
#pragma unroll
    for (int i = 0; i < kVec; ++i) if (i < n) t[i] = src[i];
  }
}
// Two 32-bit values side by side: the multiply-adds below run on pairs (one instruction for both).
struct Two { unsigned long long v; };
__device__ __forceinline__ Two two(float lo, float hi) { Two r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ Two both(float x) { return two(x, x); }
__device__ __forceinline__ float lo(Two a) { return __uint_as_float((unsigned)a.v); }
__device__ __forceinline__ float hi(Two a) { return __uint_as_float((unsigned)(a.v >> 32)); }
__device__ __forceinline__ Two add(Two a, Two b) { Two r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Two mul(Two a, Two b) { Two r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Two fma(Two a, Two b, Two c) { Two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
constexpr int kPairs = kVec / 2;

template <class T>
__device__ __forceinline__ void expand8(const Raw<T>& raw, Two (&v)[kPairs]) {
  const T* t = (const T*)raw.w;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) v[i] = two(hq_to_float(t[2 * i]), hq_to_float(t[2 * i + 1]));
}
template <bool VEC>
__device__ __forceinline__ uint2 fetch_bytes(const int8_t* src, int n) {
  uint2 w = make_uint2(0, 0);
  if (n == 0) return w;
  if (VEC) w = *(const uint2*)src;
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (!VEC && i < n) { const unsigned b = (unsigned)(uint8_t)src[i] << (8 * (i & 3)); if (i < 4) w.x |= b; else w.y |= b; }
  return w;
}
template <class T, bool VEC>
__device__ __forceinline__ void store8(T* dst, int n, const Two (&pairs)[kPairs]) {
  float v[kVec];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) { v[2 * i] = lo(pairs[i]); v[2 * i + 1] = hi(pairs[i]); }
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

// (What would be below 2^-126 becomes zero, the reciprocal of a number above 2^126 too; the forms that keep them cost several
// instructions more.  Where that would lose a result, see far_tail.)
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float reciprocal_fast(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// Phi(-a) exp(a^2 / 2) for a = |x| is smooth and falls as 1 / a: a polynomial of degree eight in t = 1 / (1 + 0.3 a), without a
// constant term, holds it to 1.4e-7 of its value for a <= 14 (least largest relative error, found by linear programming), 5e-7 in
// 32-bit arithmetic.
__device__ __forceinline__ Two tail_ratio(Two x) {
  const Two a = {x.v & 0x7fffffff7fffffffull}, d = fma(both(0.3f), a, both(1.f));
  const Two t = two(reciprocal_fast(lo(d)), reciprocal_fast(hi(d)));
  Two m = both(0.0355620074f);
  m = fma(m, t, both(-0.156766692f));
  m = fma(m, t, both(0.205662328f));
  m = fma(m, t, both(-0.0531041713f));
  m = fma(m, t, both(0.128284194f));
  m = fma(m, t, both(0.099989319f));
  m = fma(m, t, both(0.120743002f));
  m = fma(m, t, both(0.119629944f));
  return mul(m, t);
}
// Phi(x) and exp(-x^2 / 2): the tail keeps its relative accuracy, and the exponential serves the derivative too.
constexpr float kBellExponent = -0.7213475204f;                     // log2(e) / 2
__device__ __forceinline__ Two normal_cdf(Two x, Two& bell) {
  const Two e = mul(mul(x, x), both(kBellExponent));
  bell = two(exp2_fast(lo(e)), exp2_fast(hi(e)));
  const Two tail = mul(tail_ratio(x), bell), rest = fma(both(-1.f), tail, both(1.f));
  return two(lo(x) > 0.f ? lo(rest) : lo(tail), hi(x) > 0.f ? hi(rest) : hi(tail));
}
__device__ __forceinline__ Two logistic(Two x) {
  const Two e = mul(x, both(-1.4426950409f)), d = add(two(exp2_fast(lo(e)), exp2_fast(hi(e))), both(1.f));
  return two(reciprocal_fast(lo(d)), reciprocal_fast(hi(d)));
}
constexpr float kPhiSlope = 0.3989422804f;                          // 1 / sqrt(2 pi)

// f(x) and f'(x) (what is not used of them is not computed)
template <int ACT>
__device__ __forceinline__ Two f_and_slope(Two x, Two& slope) {
  if (ACT == HQ_ACT_RELU) {
    slope = two(lo(x) > 0.f ? 1.f : 0.f, hi(x) > 0.f ? 1.f : 0.f);
    return two(lo(x) < 0.f ? 0.f : lo(x), hi(x) < 0.f ? 0.f : hi(x));      // (a NaN stays one)
  }
  if (ACT == HQ_ACT_GELU) {
    Two bell;
    const Two phi = normal_cdf(x, bell);
    slope = fma(mul(x, both(kPhiSlope)), bell, phi);
    return mul(x, phi);
  }
  if (ACT == HQ_ACT_SILU) {
    const Two p = logistic(x), f = mul(x, p);
    slope = fma(f, fma(both(-1.f), p, both(1.f)), p);
    return f;
  }
  slope = both(1.f);
  return x;
}

// SiLU far to the left is x exp(x), a normal number down to x = -91.9, while the logistic function leaves the 32-bit range at -87.3.  From
// kFarFrom on the exponential is multiplied in as a square.  (GELU loses nothing above 2^-126 itself, and of its derivative what is
// below 2^-123.)
constexpr float kFarFrom = 87.f;
__device__ __forceinline__ float silu_far(float x, float& slope) {
  const float h = exp2_fast(x * 0.7213475204f), f = x * h * h;      // exp(x / 2)
  slope = fmaf(h, h, f);
  return f;
}

// Scale of a group from its largest magnitude, given as the bits of a non-negative float: in that order NaN > infinity > any
// finite value, so that one integer maximum finds all three.  top / 127, rounded correctly: a product with the rounded reciprocal,
// its remainder, which is exact, and one correction (Markstein), while nothing near the smallest floats is met.
__device__ __forceinline__ float group_scale(unsigned top_bits) {
  const float top = __uint_as_float(top_bits), c = 1.f / 127.f;
  const float s = top * c, corrected = fmaf(fmaf(-127.f, s, top), c, s);
  if (top_bits - 0x0f000000u < 0x7f800000u - 0x0f000000u) return corrected;           // 2^-97 <= top < infinity
  return top_bits >= 0x7f800000u ? __int_as_float(0x7fffffff) : __fdiv_rn(top, 127.f);
}

// q = x / s rounded to the nearest integer, ties to even, of the EXACT quotient.  Half of a group's largest value lies next to the
// border between 63 and 64, so a rounded quotient would often end on the wrong side.
//
// Any 32-bit x: the estimate t = round(x * (1 / s)) is off by one at most, next to a border; x - t s is a multiple of the last place
// of s, below s in magnitude, hence exact in 32 bits (for |x| < s it is x itself or, by Sterbenz, exact again), and its comparison
// with s / 2 decides.
//
// 16-bit x: let z = 127 x / top, top the group's largest magnitude.  With at most 11 significant bits in x and top, z is half-way
// between two integers or at least 2^-19 of itself away from it.  s is top / 127 up to 2^-24 of it: where z is no such half, x / s
// is on the same side of it, and any estimate good to 2^-19 rounds right; where it is, x / s lies below it if s was rounded up and
// above it if s was rounded down.  So 1 / s is moved by 2^-20 in that direction and one multiply-add does it (its own errors
// are below 2^-22).  s = top / 127 exactly: z = x / s may be a true tie, which goes to even; a power of two makes x / s exact,
// any other s takes the careful way.
constexpr float kMagic = 12582912.f;                                // 1.5 * 2^23: the sum's low bits are the integer
__device__ __forceinline__ int quantize(float x, float s, float inv, float half) {
  const float u = fmaf(x, inv, kMagic);
  const float t = u - kMagic;
  const float rest = fmaf(-t, s, x);
  int q = __float_as_int(u);
  if (fabsf(rest) > half || (fabsf(rest) == half && (q & 1))) q += rest > 0.f ? 1 : -1;
  return q;
}
template <class T>
__device__ __forceinline__ uint2 quantize8(const Two (&x)[kPairs], float s, float top) {
  unsigned q[kVec];
  const bool normal = s >= 0x1p-100f;
  bool direct = sizeof(T) == 2 && normal;
  float inv = reciprocal_fast(s);                                   // good to 2^-23
  if (sizeof(T) == 2) {
    const float over = fmaf(s, 127.f, -top);                        // its sign is exact
    const unsigned bits = __float_as_uint(s);
    if (over == 0.f) { direct = direct && (bits & 0x7fffffu) == 0; inv = __uint_as_float(0x7f000000u - bits); }
    else inv = fmaf(inv, over > 0.f ? -0x1p-20f : 0x1p-20f, inv);
  }
  if (direct) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const Two u = fma(x[i], both(inv), both(kMagic));
      q[2 * i] = (unsigned)u.v; q[2 * i + 1] = (unsigned)(u.v >> 32);
    }
  } else if (normal) {
    const float r = __frcp_rn(s), half = 0.5f * s;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) { q[2 * i] = quantize(lo(x[i]), s, r, half); q[2 * i + 1] = quantize(hi(x[i]), s, r, half); }
  } else {                                                          // 0, NaN, or so small that 1 / s leaves the 32-bit range
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      // (a scale of a few units of 2^-149 may be rounded down so far that the quotient passes 127: up to 190, top = 190 2^-149)
      const float v = i & 1 ? hi(x[i / 2]) : lo(x[i / 2]);
      q[i] = s > 0.f ? min(max(__double2int_rn((double)v / (double)s), -127), 127) : 0;
    }
  }
  uint2 w;
  w.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
  w.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
  return w;
}

// Largest magnitude of a thread's eight values, as the bits of a float.  (NaN wins: the 16-bit maxima hand it on.)
template <class T> __device__ __forceinline__ unsigned largest(const Raw<T>& raw);
template <> __device__ __forceinline__ unsigned largest<float>(const Raw<float>& raw) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    top = max(max(top, max(raw.w[i].x & 0x7fffffffu, raw.w[i].y & 0x7fffffffu)), max(raw.w[i].z & 0x7fffffffu, raw.w[i].w & 0x7fffffffu));
  return top;
}
template <class P>
__device__ __forceinline__ P largest_pair(const uint4& w) {
  const unsigned a = w.x & 0x7fff7fffu, b = w.y & 0x7fff7fffu, c = w.z & 0x7fff7fffu, d = w.w & 0x7fff7fffu;
  return __hmax2_nan(__hmax2_nan(*(const P*)&a, *(const P*)&b), __hmax2_nan(*(const P*)&c, *(const P*)&d));
}
template <> __device__ __forceinline__ unsigned largest<__half>(const Raw<__half>& raw) {
  const __half2 m = largest_pair<__half2>(raw.w[0]);
  return max(__float_as_uint(__low2float(m)) & 0x7fffffffu, __float_as_uint(__high2float(m)) & 0x7fffffffu);
}
template <> __device__ __forceinline__ unsigned largest<__nv_bfloat16>(const Raw<__nv_bfloat16>& raw) {
  const __nv_bfloat162 m = largest_pair<__nv_bfloat162>(raw.w[0]);
  const unsigned bits = *(const unsigned*)&m & 0x7fff7fffu;
  return max(bits << 16, bits & 0xffff0000u);
}

// Quantizes the eight values held by each lane of a group and stores integers and scale.  Every lane of the warp takes part.
// Returns the group's largest magnitude, as the bits of a float.
template <class T, bool VEC>
__device__ __forceinline__ unsigned save_group(const Raw<T>& raw, const Two (&v)[kPairs], int lanes, int lane_in_group, int8_t* q, float* scale, int n) {
  unsigned top = largest<T>(raw);
  for (int d = 1; d < lanes; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
  const float s = group_scale(top);
  const uint2 w = quantize8<T>(v, s, __uint_as_float(top));
  if (VEC) {
    if (n > 0) *(uint2*)q = w;
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) if (i < n) q[i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
  }
  if (lane_in_group == 0 && n > 0) *scale = s;
  return top;
}

__device__ __forceinline__ void restore8(uint2 w, float s, Two (&v)[kPairs]) {
  w.x ^= 0x80808080u; w.y ^= 0x80808080u;                           // 2^23 + (byte + 128) is a float whose last byte is that number
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const unsigned word = i < 2 ? w.x : w.y;
    const float a = __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7540 + 2 * (i & 1)));
    const float b = __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7541 + 2 * (i & 1)));
    v[i] = mul(add(two(a, b), both(-8388736.f)), both(s));
  }
}

// Where a thread works: slot = eight columns of a row, slots of a row filled up to whole groups.  A thread takes the same columns of
// PIECES rows, `step` rows apart: its addresses are worked out once, and all its loads are on their way together.  (Longer walks
// that fetch the next piece while they work on one were slower throughout, 8192 x 16384 gated: forward 240 us against 221.)
struct Slots { long long all, step; int per_row; uint32_t mul; };    // mul: 2^32 / per_row, rounded down
struct Slot { long long row; int col, n; };
__device__ __forceinline__ Slot slot_of(long long slot, const Slots& s, int cols) {
  Slot at;
  int in_row;
  if (s.all <= 0x7fffffffll) {
    unsigned r = __umulhi((unsigned)slot, s.mul), rest = (unsigned)slot - r * (unsigned)s.per_row;     // one too few at most
    if (rest >= (unsigned)s.per_row) { ++r; rest -= s.per_row; }
    at.row = r; in_row = (int)rest;
  } else {
    at.row = slot / s.per_row; in_row = (int)(slot - at.row * s.per_row);
  }
  at.col = in_row * kVec;
  at.n = slot < s.all ? max(0, min(kVec, cols - at.col)) : 0;
  return at;
}

// SiLU's far values among those of the calling thread, once more.  (By a walk of its own: whatever it needed of the kernel's would be kept in
// registers throughout.)
template <class T, bool GATE, int PIECES>
__device__ __noinline__ void far_forward(const ActArgs& p, const Slots& slots) {
  const Slot at = slot_of((long long)blockIdx.x * kThreads + threadIdx.x, slots, p.cols);
  for (long long row = at.row; row < p.rows && row < at.row + PIECES * slots.step; row += slots.step) {
    for (int col = at.col; col < at.col + at.n; ++col) {
      const float x = hq_to_float(((const T*)p.x)[row * p.x_stride + col]);
      if (!(x < -kFarFrom)) continue;
      float slope;
      const float f = silu_far(x, slope);
      ((T*)p.y)[row * p.y_stride + col] = hq_from_float<T>(GATE ? f * hq_to_float(((const T*)p.gate)[row * p.gate_stride + col]) : f);
    }
  }
}
template <class T, bool GATE, int PIECES>
__device__ __noinline__ void far_backward(const ActArgs& p, const Slots& slots) {
  const Slot at = slot_of((long long)blockIdx.x * kThreads + threadIdx.x, slots, p.cols);
  for (long long row = at.row; row < p.rows && row < at.row + PIECES * slots.step; row += slots.step) {
    for (int col = at.col; col < at.col + at.n; ++col) {
      const long long flat = row * p.cols + col, group = row * p.groups + col / p.group;
      const float x = (float)p.xq[flat] * p.xs[group], dy = hq_to_float(((const T*)p.x)[row * p.x_stride + col]);
      if (!(x < -kFarFrom)) continue;
      float slope;
      const float f = silu_far(x, slope);
      if (GATE) ((T*)p.dgate)[row * p.dgate_stride + col] = hq_from_float<T>(dy * f);
      ((T*)p.y)[row * p.y_stride + col] = hq_from_float<T>(GATE ? dy * ((float)p.gq[flat] * p.gs[group]) * slope : dy * slope);
    }
  }
}

// GATE: a second tensor.
template <class T, int ACT, bool VEC, bool GATE, int PIECES>
__global__ void __launch_bounds__(kThreads, 4) act_save8_kernel(const __grid_constant__ ActArgs p, const __grid_constant__ Slots slots) {
  hq_pdl_entry();
  const int lanes = p.group / kVec, group_log = 31 - __clz(p.group);
  const int lane_in_group = threadIdx.x & (lanes - 1);
  const Slot at = slot_of((long long)blockIdx.x * kThreads + threadIdx.x, slots, p.cols);
  const T* x_at = (const T*)p.x + at.row * p.x_stride + at.col;
  const T* g_at = GATE ? (const T*)p.gate + at.row * p.gate_stride + at.col : nullptr;
  T* y_at = (T*)p.y + at.row * p.y_stride + at.col;
  long long flat = at.row * p.cols + at.col, group_at = at.row * p.groups + (at.col >> group_log);
  int n[PIECES];
  Raw<T> raw_x[PIECES], raw_g[GATE ? PIECES : 1];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    n[i] = at.row + i * slots.step < p.rows ? at.n : 0;
    fetch8<T, VEC>(x_at + i * slots.step * p.x_stride, n[i], raw_x[i]);
    if (GATE) fetch8<T, VEC>(g_at + i * slots.step * p.gate_stride, n[i], raw_g[GATE ? i : 0]);
  }
  bool far = false;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    Two x[kPairs], g[kPairs];
    expand8<T>(raw_x[i], x);
    const unsigned top = save_group<T, VEC>(raw_x[i], x, lanes, lane_in_group, p.xq + flat, p.xs + group_at, n[i]);
    if (GATE) {
      expand8<T>(raw_g[GATE ? i : 0], g);
      save_group<T, VEC>(raw_g[GATE ? i : 0], g, lanes, lane_in_group, p.gq + flat, p.gs + group_at, n[i]);
    }
    if (p.y && n[i] > 0) {
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        Two slope;
        x[k] = f_and_slope<ACT>(x[k], slope);
        if (GATE) x[k] = mul(x[k], g[k]);
      }
      store8<T, VEC>(y_at + i * slots.step * p.y_stride, n[i], x);
      far = far || top >= __float_as_uint(kFarFrom);
    }
    flat += slots.step * p.cols;
    group_at += slots.step * p.groups;
  }
  if (ACT == HQ_ACT_SILU && far) far_forward<T, GATE, PIECES>(p, slots);
}

template <class T, int ACT, bool VEC, bool GATE, int PIECES>
__global__ void __launch_bounds__(kThreads, GATE ? 5 : 4) act_backward8_kernel(const __grid_constant__ ActArgs p, const __grid_constant__ Slots slots) {
  hq_pdl_entry();
  const int group_log = 31 - __clz(p.group);
  const Slot at = slot_of((long long)blockIdx.x * kThreads + threadIdx.x, slots, p.cols);
  const T* dy_at = (const T*)p.x + at.row * p.x_stride + at.col;
  T* dx_at = (T*)p.y + at.row * p.y_stride + at.col;
  T* dgate_at = GATE ? (T*)p.dgate + at.row * p.dgate_stride + at.col : nullptr;
  const long long flat = at.row * p.cols + at.col, group_at = at.row * p.groups + (at.col >> group_log);
  int n[PIECES];
  Raw<T> raw_dy[PIECES];
  uint2 xq[PIECES], gq[GATE ? PIECES : 1];
  float xs[PIECES], gs[GATE ? PIECES : 1];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    n[i] = at.row + i * slots.step < p.rows ? at.n : 0;
    fetch8<T, VEC>(dy_at + i * slots.step * p.x_stride, n[i], raw_dy[i]);
    xq[i] = fetch_bytes<VEC>(p.xq + flat + i * slots.step * p.cols, n[i]);
    xs[i] = n[i] ? p.xs[group_at + i * slots.step * p.groups] : 0.f;
    if (GATE) {
      gq[GATE ? i : 0] = fetch_bytes<VEC>(p.gq + flat + i * slots.step * p.cols, n[i]);
      gs[GATE ? i : 0] = n[i] ? p.gs[group_at + i * slots.step * p.groups] : 0.f;
    }
  }
  bool far = false;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    if (n[i] == 0) continue;
    Two dy[kPairs], x[kPairs], g[kPairs], dgate[kPairs];
    expand8<T>(raw_dy[i], dy);
    restore8(xq[i], xs[i], x);
    if (GATE) restore8(gq[GATE ? i : 0], gs[GATE ? i : 0], g);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      Two slope;
      const Two f = f_and_slope<ACT>(x[k], slope);
      if (GATE) { dgate[k] = mul(dy[k], f); dy[k] = mul(dy[k], g[k]); }
      if (ACT != HQ_ACT_NONE) dy[k] = mul(dy[k], slope);
    }
    if (GATE) store8<T, VEC>(dgate_at + i * slots.step * p.dgate_stride, n[i], dgate);
    store8<T, VEC>(dx_at + i * slots.step * p.y_stride, n[i], dy);
    far = far || xs[i] * 128.f >= kFarFrom;
  }
  if (ACT == HQ_ACT_SILU && far) far_backward<T, GATE, PIECES>(p, slots);
}

// Whole 16-byte pieces everywhere: pitches that keep every row on its 16 bytes, and whole eights of columns.
bool vectors(int type, const ActArgs& a) {
  const long long per16 = type == HQ_F32 ? 4 : 8;
  const bool strides = a.x_stride % per16 == 0 && (!a.gate || a.gate_stride % per16 == 0) && (!a.y || a.y_stride % per16 == 0) &&
                       (!a.dgate || a.dgate_stride % per16 == 0);
  return strides && a.cols % kVec == 0;
}

template <bool SAVE, class T, int ACT, bool VEC, bool GATE, int kPieces>
cudaError_t launch_pieces(const ActArgs& a, cudaStream_t s) {
  Slots slots;
  slots.per_row = a.groups * (a.group / kVec);
  slots.step = (a.rows + kPieces - 1) / kPieces;
  slots.all = slots.step * slots.per_row;
  slots.mul = (uint32_t)((1ull << 32) / (unsigned)slots.per_row);     // (a group has four slots at least)
  const long long blocks = (slots.all + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kThreads);
  if (SAVE) return hq_launch_pdl(act_save8_kernel<T, ACT, VEC, GATE, kPieces>, grid, block, 0, s, a, slots);
  return hq_launch_pdl(act_backward8_kernel<T, ACT, VEC, GATE, kPieces>, grid, block, 0, s, a, slots);
}
// Pieces per thread: what keeps enough bytes in flight (with one, forward + backward of the gated 8192 x 16384 case took 412 us, with two
// 382; ungated GELU of that size one 372, two 347, four 340), but one while that leaves SMs without a block (32 x 4096: 16 blocks of
// four pieces, 5.0 us forward + backward, 64 of one, 3.3).
template <bool SAVE, class T, int ACT, bool VEC, bool GATE>
cudaError_t launch_pieces(const ActArgs& a, cudaStream_t s) {
  constexpr int kPieces = !VEC ? 1 : GATE || sizeof(T) == 4 ? 2 : 4;
  const long long slots = a.rows * a.groups * (a.group / kVec);
  if (slots < a.sm_count * 512ll * kPieces) return launch_pieces<SAVE, T, ACT, VEC, GATE, 1>(a, s);
  return launch_pieces<SAVE, T, ACT, VEC, GATE, kPieces>(a, s);
}
template <bool SAVE, class T, int ACT>
cudaError_t launch_act(const ActArgs& a, bool vec, cudaStream_t s) {
  if (a.gq) return vec ? launch_pieces<SAVE, T, ACT, true, true>(a, s) : launch_pieces<SAVE, T, ACT, false, true>(a, s);
  return vec ? launch_pieces<SAVE, T, ACT, true, false>(a, s) : launch_pieces<SAVE, T, ACT, false, false>(a, s);
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
