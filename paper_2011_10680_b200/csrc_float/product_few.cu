// hq_linear_w4 for few rows: the matrix-vector case, one token of each of a few sequences.  The packed weights are read once
// and that is the bound, so everything else has to hide behind their stream: at the memory's rate a scheduler has about 350 cycles
// for 32 outputs x 128 inputs.
//   - Every warp has a ring of its own: one lane fetches 32 outputs x 256 inputs by TMA, the warp consumes them, and the lane
//     fetches into the same place again.  No warp waits for another until a tile's inputs are through.
//   - The integers go through the 16-bit matrix instruction (mma.m16n8k16).  A nibble masked out of a word IS a 16-bit float: the
//     subnormal u 2^-24, or 16 u 2^-24 for an upper nibble, u = integer + 8.  That takes five instructions per eight weights.
//     sum (u - 8) x is the sum with u less the same sum with u = 8 for all, which is made once per CTA by the same instructions in
//     the same order (weights of zero give exactly zero), and the sum over a group is scaled in 32 bits.
//   - x is stored in shared memory once per CTA, in the order in which the nibbles come out of a word (0 4 1 5 2 6 3 7 of every
//     eight), as 16-bit floats under a power of two per row and 128 inputs that brings the largest of them to 2^15 .. 2^16, those
//     that meet upper nibbles divided by 16.  fp16 values are held exactly from 2^-25 of the largest one up, bf16 values from 2^-28; below,
//     to 2^-36 of it, which is 2^-12 of what one addition in 32 bits rounds away.  The sum with u and the one it is corrected by
//     are up to 8 sum |x|, so the 32-bit additions round to 2^-24 of that, whatever the weights: a value 2^14 times the others' size
//     that meets a weight of zero still leaves 2^-21 of itself times the scale, some 2^-14 of a usual result.
//   - Groups shorter than 128: the eight columns of the instruction carry a row's inputs group by group, zeros elsewhere, so that
//     every group has a sum of its own ("parts"; 64: two columns per row, 32: four).
//   - Few outputs: a team of 2 .. 16 warps of a CTA splits the inputs of a tile, the CTAs of a cluster do too, and the parts are
//     added up in shared memory in a fixed order.  Teams do not wait for one another.
//   - Infinities, NaN and values of 2^73 and more, which the representation does not hold, and results that come out infinite or NaN
//     (an infinite scale): once more, value by value.
#include "../csrc/tc_common.cuh"
#include "float_internal.cuh"

namespace {

constexpr int kThreads = 512, kWarps = 16, kWarpsLog = 4, kRows = 16, kStep = 128;
constexpr int kMaxShared = 226 * 1024;
constexpr int kMaxColumns = 16;               // of the matrix instruction, for all rows: rows times parts
constexpr int kMaxInputs = 1 << 20;           // see FewArgs::group_mul
constexpr int kStageInputs = 256;             // per fetch: 128 bytes of a row, one swizzle span
constexpr int kMaxDepth = 4;

struct FewArgs {
  ProductArgs p;
  int tiles;               // along the outputs, a team's
  int splits, range;       // CTAs per tile; inputs of each (a multiple of kStageInputs)
  int along_log;           // warps of a team: 1 .. 16 (16 where CTAs share a tile)
  int parts_log;           // columns per row: 1, 2 or 4
  uint32_t group_mul;      // 2^31 / (group / 32), rounded up: the scale of input k (a multiple of 32) is the high word of (k / 16) * group_mul.
                           // Exact while (k / 32) (group / 32) < 2^31, that is up to kMaxInputs inputs
  int depth;               // stages of a warp's ring
  int pitch;               // bytes of a row of x in shared memory
  int scale_pitch;         // bytes of an output's scales per fetch: two, four or eight, and what 4-byte copies bring along
  int ring_at, scale_at, fix_at, red_at, sum_at;     // shared memory: rings of weights and scales, corrections, the warps' sums, the CTA's
  uint32_t* status;
};

struct Control {
  unsigned long long full[kWarps][kMaxDepth];
  volatile uint32_t abort_flag;
  volatile uint32_t flip;
  volatile uint32_t beyond;         // x holds something that the representation does not
  volatile uint32_t not_finite;     // a result came out like that
};

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
// Two nibbles of a word, their sign bits turned over.  (`flip`, 0x00080008, comes out of memory: with two constants in sight the
// compiler makes two instructions of this one.)
__device__ __forceinline__ uint32_t lower(uint32_t w, uint32_t flip) { return (w & 0x000f000fu) ^ flip; }
__device__ __forceinline__ uint32_t upper(uint32_t w, uint32_t flip_upper) { return (w & 0x00f000f0u) ^ flip_upper; }
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) { const __half2 v = __floats2half2_rn(lo, hi); return *(const uint32_t*)&v; }

template <class T> __device__ __forceinline__ T load_scale(uint32_t addr) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
  return *(const T*)&v;
}
template <class T> __device__ __forceinline__ void to_floats(const uint4& v, float (&f)[8]) {
  const T* t = (const T*)&v;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = hq_to_float(t[i]);
}

// Largest magnitude of eight values, as the bits of a float.  (NaN wins: the 16-bit maxima hand it on.)
template <class P>
__device__ __forceinline__ uint32_t largest_pair(const uint4& v) {
  const uint32_t a = v.x & 0x7fff7fffu, b = v.y & 0x7fff7fffu, c = v.z & 0x7fff7fffu, d = v.w & 0x7fff7fffu;
  const P m = __hmax2_nan(__hmax2_nan(*(const P*)&a, *(const P*)&b), __hmax2_nan(*(const P*)&c, *(const P*)&d));
  return *(const uint32_t*)&m;
}
template <class T> __device__ __forceinline__ uint32_t largest(const uint4& v);
template <> __device__ __forceinline__ uint32_t largest<__nv_bfloat16>(const uint4& v) {
  const uint32_t m = largest_pair<__nv_bfloat162>(v) & 0x7fff7fffu;
  return max(m << 16, m & 0xffff0000u);
}
template <> __device__ __forceinline__ uint32_t largest<__half>(const uint4& v) {
  const uint32_t m = largest_pair<__half2>(v) & 0x7fff7fffu;       // (as 16-bit integers they are in order too, NaN on top)
  const __half_raw r{(unsigned short)max(m & 0xffffu, m >> 16)};
  return __float_as_uint(__half2float(__half(r)));
}

// Results value by value, a warp on each: those that came out infinite or NaN, or all of them.  (A group's sum times an infinite scale is no
// sum of the products: an integer of zero, or terms of both signs, make a NaN of that.  Such a scale always ends in a result that is
// not finite, so nothing else has to look for it.)
template <class T, int RT>
__device__ __noinline__ void by_value(const FewArgs& a, bool all) {
  const ProductArgs& p = a.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, groups_of_ctas = gridDim.x / a.splits;
  if (a.splits > 1 && cluster_ctarank() != 0) return;              // (256 results at a time at most: the first CTA's threads have written all)
  // the tiles of the CTA's teams, one after the other
  for (int tile = blockIdx.x / a.splits; tile < a.tiles; tile += groups_of_ctas) {
    for (int e = warp; e < p.j * (16 * RT); e += kWarps) {
      const int row = e / (16 * RT), i = tile * (16 * RT) + e % (16 * RT);
      if (i >= p.i) continue;
      T* const at = (T*)p.out + row * p.out_stride + i;
      if (!all && isfinite(hq_to_float(*at))) continue;
      const T* x = (const T*)p.b + row * p.b_stride;
      const uint8_t* q = (const uint8_t*)p.q + (long long)i * (p.q_cols >> 1);
      const T* s = (const T*)p.scale + (long long)i * p.groups;
      float sum = 0.f;
      for (int k = lane * 2; k < p.r; k += 64) {
        const float scale = hq_to_float(s[k / p.group]);
        sum = fmaf(hq_to_float(x[k]), (float)hq_nibble(q, k) * scale, sum);
        sum = fmaf(hq_to_float(x[k + 1]), (float)hq_nibble(q, k + 1) * scale, sum);
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (lane == 0) *at = hq_from_float<T>(sum + (p.bias ? hq_to_float(((const T*)p.bias)[i]) : 0.f));
    }
  }
}

// NB: eights of columns; RT: sixteens of outputs per warp; WHOLE: a step has one scale per output.
template <class T, int NB, int RT, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 1) product_few_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ FewArgs a) {
  extern __shared__ uint8_t raw_shared[];
  __shared__ Control ctl;
  constexpr int kStageBytes = 16 * RT * 128;
  const uint32_t kScaleBytes = 16 * RT * a.scale_pitch;
  const ProductArgs& p = a.p;
  const uint32_t base = (smem_u32(raw_shared) + 1023u) & ~1023u;
  uint8_t* const shared = raw_shared + (base - smem_u32(raw_shared));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int row_in_8 = ((g & 1) << 2) | (g >> 1);                  // the output on fragment row g: neighbours on different banks
  const int rank = a.splits > 1 ? (int)cluster_ctarank() : 0;
  const int along = 1 << a.along_log, parts_log = WHOLE ? 0 : a.parts_log, parts = 1 << parts_log;
  const int kw = warp & (along - 1), team = warp >> a.along_log, teams = kWarps >> a.along_log;
  const int k_begin = rank * a.range, k_end = min(p.r, k_begin + a.range);
  const int stages = (k_end - k_begin + kStageInputs - 1) / kStageInputs;
  const int my_stages = kw < stages ? (stages - kw + along - 1) >> a.along_log : 0;       // of a tile, this warp's
  // consecutive tiles go to different CTAs
  const int groups_of_ctas = gridDim.x / a.splits, tile0 = blockIdx.x / a.splits + team * groups_of_ctas, tile_stride = teams * groups_of_ctas;
  const int units = (tile0 < a.tiles ? (a.tiles - tile0 + tile_stride - 1) / tile_stride : 0) * my_stages;
  const uint32_t ring = base + a.ring_at + warp * a.depth * kStageBytes;
  const uint32_t scale_ring = base + a.scale_at + warp * a.depth * kScaleBytes;

  if (lane == 0)
    for (int s = 0; s < a.depth; ++s) mbar_init(smem_u32(&ctl.full[warp][s]), 1 + 32);
  if (threadIdx.x == 0) { ctl.abort_flag = 0; ctl.beyond = 0; ctl.not_finite = 0; ctl.flip = 0x00080008u; }
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
  hq_pdl_entry();

  // The warp's fetches: stage `f_stage` of its tile `f_tile`.  (Inputs and outputs past the last arrive as zeros.)  A lane brings
  // the scales of one output, as the aligned words they lie in; those of outputs past the last are never used.
  int f_tile = tile0, f_stage = 0, f_slot = 0;
  const long long all_scales = (long long)p.i * p.groups;
  long long f_row = (long long)(tile0 * (16 * RT) + lane) * p.groups;       // first scale of this lane's output
  bool f_live = lane < 16 * RT && tile0 * (16 * RT) + lane < p.i;
  auto fetch = [&]() {
    const uint32_t bar = smem_u32(&ctl.full[warp][f_slot]);
    const int k = k_begin + ((f_stage << a.along_log) + kw) * kStageInputs, row = f_tile * (16 * RT);
    if (lane == 0) {
      mbar_expect_tx(bar, kStageBytes);
      tma_load_2d(ring + f_slot * kStageBytes, &map_q, bar, k >> 1, row);
    }
    if (f_live && k < p.r) {
      const int first = (int)__umulhi((uint32_t)k >> 4, a.group_mul), last = min(first + 2 * parts - 1, p.groups - 1);
      const uint32_t to = scale_ring + f_slot * kScaleBytes + lane * a.scale_pitch;
      const long long w0 = (f_row + first) >> 1, w1 = (f_row + last) >> 1;
#pragma unroll
      for (int w = 0; w < (WHOLE ? 2 : 5); ++w) {
        if (w0 + w <= w1) {
          const int bytes = (w0 + w) * 2 + 1 < all_scales ? 4 : 2;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 4 * w), "l"((const uint32_t*)p.scale + w0 + w), "r"(bytes) : "memory");
        }
      }
    }
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
    if (++f_slot == a.depth) f_slot = 0;
    if (++f_stage == my_stages) {
      f_stage = 0; f_tile += tile_stride;
      f_row = (long long)(f_tile * (16 * RT) + lane) * p.groups;
      f_live = lane < 16 * RT && f_tile * (16 * RT) + lane < p.i;
    }
  };

  // x, zeros behind its end up to whole stages, and a step of zeros in front, which the columns without inputs read.
  const int pieces = stages * (kStageInputs / 8), all_pieces = pieces * p.j;
  float2* const fix = (float2*)(shared + a.fix_at);               // per step and column: the power of two, and what u = 8 gives
  bool beyond = false;
  {
    constexpr int kLoads = 4;                                     // in flight per thread
    int row = 0, c = threadIdx.x;
    uint4 v[kLoads];
    int row_of[kLoads], c_of[kLoads];
    auto load_x = [&]() {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) {
        while (c >= pieces && row < p.j) { c -= pieces; ++row; }
        row_of[l] = row; c_of[l] = c;
        const int k = k_begin + c * 8;
        v[l] = make_uint4(0, 0, 0, 0);
        if (row < p.j && k < k_end) v[l] = *(const uint4*)((const T*)p.b + row * p.b_stride + k);
        c += kThreads;
      }
    };
    load_x();                                                     // (first of all: what everything else waits for)
    const int ahead = min(a.depth, units);
    for (int n = 0; n < ahead; ++n) fetch();
    for (int e = threadIdx.x; e - lane < all_pieces; e += kLoads * kThreads) {
      if (e != threadIdx.x) load_x();
#pragma unroll
      for (int l = 0; l < kLoads; ++l) {
        if (e - lane + l * kThreads >= all_pieces) break;         // (the whole warp: a row has whole warps of pieces)
        float f[8];
        to_floats<T>(v[l], f);
        uint32_t top = largest<T>(v[l]);
        beyond = beyond || top >= 0x64000000u;                    // 2^73
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
        const uint32_t e2 = max(top >> 23, 15u);                  // the largest value's exponent: 2^(e2 - 127)
        const float down = __uint_as_float(min(269u - min(e2, 255u), 254u) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= (i & 1) ? down * 0.0625f : down;
        const int st = c_of[l] >> 4, in = c_of[l] & 15;
        *(uint4*)(shared + 256 + row_of[l] * a.pitch + st * 256 + (in & 3) * 64 + (in >> 2) * 16) =
            make_uint4(half2_bits(f[0], f[4]), half2_bits(f[1], f[5]), half2_bits(f[2], f[6]), half2_bits(f[3], f[7]));
        // 2^-24 of the integers and 2^(142 - e2) of x taken back
        if (in == 0)
          for (int q = 0; q < parts; ++q) fix[st * (8 * NB) + (row_of[l] << parts_log) + q].x = __uint_as_float((e2 + 9u) << 23);
      }
    }
    if (threadIdx.x < 16) ((uint4*)shared)[threadIdx.x] = make_uint4(0, 0, 0, 0);
  }
  if (__syncthreads_or(beyond) && threadIdx.x == 0) ctl.beyond = 1;
  const uint32_t flip = ctl.flip, flip4 = flip << 4;

  // column g of every eight: its part has to be that of the thread's inputs, else it reads the zeros
  uint32_t x_at[NB], x_step[NB];                                   // first step, and bytes from one step to the next
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int col = nb * 8 + g, row = col >> parts_log;
    const bool on = row < p.j && (col & (parts - 1)) == (t << parts_log) >> 2;
    x_at[nb] = base + (on ? 256 + row * a.pitch + t * 16 : 0);
    x_step[nb] = on ? 256u : 0u;
  }
  // the sums that u = 8 gives, times the power of two
  for (int st = warp; st < pieces >> 4; st += kWarps) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float acc[4] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 b = load_shared(x_at[nb] + st * x_step[nb] + i * 64);
        mma(acc, 0x00080008u, 0x00080008u, 0x00800080u, 0x00800080u, b.x, b.y);
        mma(acc, 0x00080008u, 0x00080008u, 0x00800080u, 0x00800080u, b.z, b.w);
      }
      if (g == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float2& at = fix[st * (8 * NB) + nb * 8 + 2 * t + k];
          if (nb * 8 + 2 * t + k < p.j << parts_log) at.y = -acc[k] * at.x; else at = make_float2(0.f, 0.f);
        }
      }
    }
  }
  __syncthreads();

  // scales: column c is part c % parts of its row of x
  const int part0 = ((2 * t) & (parts - 1)) * (kStep >> parts_log), part1 = ((2 * t + 1) & (parts - 1)) * (kStep >> parts_log);
  int lost = 0, lost_slot = 0;                                     // a wait that ran out: copies in flight then, and the first one's place
  uint32_t lost_phase = 0;
  bool ok = true;
  float total[RT][NB][4] = {};
  int n = 0, slot = 0;
  uint32_t phase = 0;
  for (int tile = tile0; tile < a.tiles; tile += tile_stride) {
   for (int stage = 0; stage < my_stages; ++stage, ++n) {
    if (ok && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.full[warp][slot]), phase, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER))) {
      ok = false;
      lost = min(a.depth, units - n); lost_slot = slot; lost_phase = phase;
    }
    const uint32_t from = ring + slot * kStageBytes;
    const int st0 = ((stage << a.along_log) + kw) * 2, k0 = k_begin + st0 * kStep;
    // (with one eight of columns both halves of the stage at once: twice the chains of dependent sums)
    float acc[2][RT][NB][4] = {};
    constexpr int kTogether = NB == 1 ? 2 : 1;
#pragma unroll
    for (int half0 = 0; half0 < 2; half0 += kTogether) {
      uint4 w[kTogether][2 * RT];
#pragma unroll
      for (int y = 0; y < kTogether; ++y)
#pragma unroll
        for (int h = 0; h < 2 * RT; ++h) w[y][h] = load_shared(from + (row_in_8 + 8 * h) * 128 + ((((half0 + y) * 4 + t) ^ row_in_8) << 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 b[kTogether][NB];
#pragma unroll
        for (int y = 0; y < kTogether; ++y)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) b[y][nb] = load_shared(x_at[nb] + (st0 + half0 + y) * x_step[nb] + i * 64);
#pragma unroll
        for (int y = 0; y < kTogether; ++y) {
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const uint32_t lo = word(w[y][2 * r], i), hi = word(w[y][2 * r + 1], i), lo8 = lo >> 8, hi8 = hi >> 8;
            const uint32_t a0 = lower(lo, flip), a1 = lower(hi, flip), a2 = upper(lo, flip4), a3 = upper(hi, flip4);
            const uint32_t c0 = lower(lo8, flip), c1 = lower(hi8, flip), c2 = upper(lo8, flip4), c3 = upper(hi8, flip4);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              mma(acc[half0 + y][r][nb], a0, a1, a2, a3, b[y][nb].x, b[y][nb].y);
              mma(acc[half0 + y][r][nb], c0, c1, c2, c3, b[y][nb].z, b[y][nb].w);
            }
          }
        }
      }
    }
    const uint32_t first = __umulhi((uint32_t)k0 >> 4, a.group_mul);
    // the first scale of an output lies in the upper half of its word where its index is odd
    uint32_t s_at[2 * RT];
#pragma unroll
    for (int h = 0; h < 2 * RT; ++h) {
      const uint32_t in_tile = row_in_8 + 8 * h, row = (uint32_t)tile * (16 * RT) + in_tile;
      s_at[h] = scale_ring + slot * kScaleBytes + in_tile * a.scale_pitch + (((row * (uint32_t)p.groups + first) & 1) << 1);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      // (inputs past the last one give sums of zero; their scales, whatever is found there, must not make a NaN of it)
      const int k = k0 + half * kStep;
      const bool on0 = k + part0 < k_end, on1 = k + part1 < k_end;
      const uint32_t i0 = (__umulhi((uint32_t)(k + part0) >> 4, a.group_mul) - first) * 2;
      const uint32_t i1 = WHOLE ? i0 : (__umulhi((uint32_t)(k + part1) >> 4, a.group_mul) - first) * 2;
      float s0[2 * RT], s1[2 * RT];
#pragma unroll
      for (int h = 0; h < 2 * RT; ++h) {
        s0[h] = on0 ? hq_to_float(load_scale<T>(s_at[h] + i0)) : 0.f;
        s1[h] = WHOLE ? s0[h] : on1 ? hq_to_float(load_scale<T>(s_at[h] + i1)) : 0.f;
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const uint4 f = load_shared(base + a.fix_at + ((st0 + half) * (8 * NB) + nb * 8 + 2 * t) * 8);
        const float p0 = __uint_as_float(f.x), c0 = __uint_as_float(f.y), p1 = __uint_as_float(f.z), c1 = __uint_as_float(f.w);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float (&sum)[4] = total[r][nb];
            const float (&v)[4] = acc[half][r][nb];
            sum[2 * h] = fmaf(s0[2 * r + h], fmaf(v[2 * h], p0, c0), sum[2 * h]);
            sum[2 * h + 1] = fmaf(s1[2 * r + h], fmaf(v[2 * h + 1], p1, c1), sum[2 * h + 1]);
          }
        }
      }
    }
    __syncwarp();
    if (ok && n + a.depth < units) fetch();
    if (++slot == a.depth) { slot = 0; phase ^= 1; }
   }
    // the tile's inputs are through: add up the warps' parts, all outputs at once with one eight of columns, sixteen with two (the
    // sums of 16 outputs of a column lie together, every other pair of columns turned by eight to spread the banks)
    auto meet = [&]() {
      if (a.along_log == 0) __syncwarp();
      else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 << a.along_log) : "memory");
    };
    constexpr int kHalves = NB == 1 ? RT : 1, kSums = 16 * 8 * NB * kHalves;       // sixteens of outputs, values of a warp
#pragma unroll
    for (int r0 = 0; r0 < RT; r0 += kHalves) {
      float* mine = (float*)(shared + a.red_at) + warp * kSums;
#pragma unroll
      for (int r = r0; r < r0 + kHalves; ++r)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int k2 = 0; k2 < 4; ++k2) {
          mine[(((r - r0) * NB + nb) * 8 + 2 * t + (k2 & 1)) * 16 + ((row_in_8 + (k2 >> 1) * 8) ^ ((t & 1) << 3))] = total[r][nb][k2];
          total[r][nb][k2] = 0.f;
        }
      }
      meet();
      const float* sums = (const float*)(shared + a.red_at) + (team << a.along_log) * kSums;
      const int members = 32 << a.along_log, outputs = p.j * (16 * kHalves);
      auto output = [&](int e, float sum) {
        const int row = e / (16 * kHalves), i = tile * (16 * RT) + r0 * 16 + (e & (16 * kHalves - 1));
        if (i < p.i) {
          if (!isfinite(sum)) ctl.not_finite = 1;
          if (p.bias) sum += hq_to_float(((const T*)p.bias)[i]);
          ((T*)p.out)[row * p.out_stride + i] = hq_from_float<T>(sum);
        }
      };
      for (int e = kw * 32 + lane; e < outputs; e += members) {
        const int col = ((e / (16 * kHalves)) << parts_log) + (kHalves == 2 ? (e >> 4 & 1) * 8 : 0), turned = (e & 15) ^ ((col >> 1 & 1) << 3);
        const float* part = sums + col * 16 + turned;            // a row's columns: this one, the next, and two more, turned the other way
        const int other = 32 + (turned ^ 8) - turned;
        float sum = 0.f;
#pragma unroll 4
        for (int k2 = 0; k2 < along; ++k2, part += kSums) {
          sum += part[0];
          if (!WHOLE) sum += part[16];
          if (!WHOLE && parts == 4) { sum += part[other]; sum += part[other + 16]; }
        }
        if (a.splits == 1) output(e, sum); else ((float*)(shared + a.sum_at))[e] = sum;
      }
      if (a.splits > 1) {
        cluster_sync_all();
        if (rank != 0 && threadIdx.x == 0 && ctl.beyond)
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(smem_u32((const void*)&ctl.beyond), 0)), "r"(1) : "memory");
        for (int e = threadIdx.x + rank * kThreads; e < outputs; e += kThreads * a.splits) {
          float sum = 0.f;
          for (int c = 0; c < a.splits; ++c) {
            float v;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(in_cta(base + a.sum_at + e * 4, c)));
            sum += v;
          }
          output(e, sum);
        }
        cluster_sync_all();
      }
      meet();                                                    // the sums are read
    }
  }
  __syncthreads();                                                 // the results are written
  if (ctl.beyond || ctl.not_finite) by_value<T, RT>(a, ctl.beyond);
  if (!ok && lane == 0) {                                          // let the copies in flight land before the memory goes
    for (; lost > 0; --lost) {
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait_for(smem_u32(&ctl.full[warp][lost_slot]), lost_phase, kSuspendNs) && global_ns() - t0 < kWaitBudgetNs) {}
      if (++lost_slot == a.depth) { lost_slot = 0; lost_phase ^= 1; }
    }
  }
}

int columns_eights(int j, int parts) { return j * parts <= 8 ? 1 : 2; }

// Parts of a 128-input step that can have scales of their own.
int parts_of(const ProductArgs& a) { return a.group >= a.r || a.group % 128 == 0 ? 1 : a.group % 64 == 0 ? 2 : 4; }

template <class T, int NB, int RT, bool WHOLE>
cudaError_t launch(const CUtensorMap& map, const FewArgs& a, int grid, int shared, int device, cudaStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const cudaError_t ready = hq_allow_shared(done, device, product_few_kernel<T, NB, RT, WHOLE>, kMaxShared);
  if (ready != cudaSuccess) return ready;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)a.splits; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = (size_t)shared; cfg.stream = s;
  cfg.attrs = attr; cfg.numAttrs = a.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, product_few_kernel<T, NB, RT, WHOLE>, map, a);
}
template <class T, bool WHOLE>
cudaError_t launch_shape(int nb, int rt, const CUtensorMap& map, const FewArgs& a, int grid, int shared, int device, cudaStream_t s) {
  if (rt == 2) return nb == 1 ? launch<T, 1, 2, WHOLE>(map, a, grid, shared, device, s) : launch<T, 2, 2, WHOLE>(map, a, grid, shared, device, s);
  return nb == 1 ? launch<T, 1, 1, WHOLE>(map, a, grid, shared, device, s) : launch<T, 2, 1, WHOLE>(map, a, grid, shared, device, s);
}
template <class T>
cudaError_t launch_type(int nb, int rt, const CUtensorMap& map, const FewArgs& a, int grid, int shared, int device, cudaStream_t s) {
  return a.parts_log == 0 ? launch_shape<T, true>(nb, rt, map, a, grid, shared, device, s) : launch_shape<T, false>(nb, rt, map, a, grid, shared, device, s);
}

// The launch of a shape: sixteens of outputs per tile, cluster size, warps of a team, shared memory; false when x does not fit the
// CTAs of a cluster.
bool plan(const ProductArgs& p, int sm_count, FewArgs& a, int& rt, int& shared) {
  const int parts = parts_of(p), nb = columns_eights(p.j, parts);
  const int all = (p.r + kStageInputs - 1) / kStageInputs;
  const unsigned group32 = (unsigned)(p.group >= p.r ? kMaxInputs : p.group) / 32;
  if (p.r > kMaxInputs) return false;
  bool found = false;
  for (int splits = 1; splits <= 8; splits *= 2) {
    const int per = (all + splits - 1) / splits, clusters = sm_count / splits;
    if (clusters < 1 || (splits > 1 && (splits - 1) * per >= all)) break;     // a CTA without inputs
    const long long inputs = (long long)per * kStageInputs;
    const long long pitch = inputs * 2 + 64;                           // 64 modulo 128: eight lanes' pieces lie on different banks
    const long long x_bytes = (256 + p.j * pitch + 1023) & ~1023ll, fix_bytes = (inputs / kStep * 8 * nb * 8 + 127) & ~127ll;
    // Sixteen or 32 outputs per tile (32 share what is read of x), and teams of as many warps as leave the longest warp the least: its
    // stages times the outputs of one.
    const int scale_pitch = parts == 1 ? 8 : parts == 2 ? 12 : 20;
    long long best = 0;
    for (int r = 2; r >= 1; --r) {
      const int tiles = (p.i + 16 * r - 1) / (16 * r);
      const int at_a_time = nb == 1 ? r : 1;
      const int red_bytes = kWarps * 16 * 8 * nb * at_a_time * (int)sizeof(float), sum_bytes = splits > 1 ? 16 * at_a_time * p.j * 4 : 0;
      const long long rest = 1024 + x_bytes + fix_bytes + red_bytes + sum_bytes;
      const int stage_bytes = kWarps * 16 * r * 128, scale_bytes = kWarps * 16 * r * scale_pitch;
      int depth = rest < kMaxShared ? (int)((kMaxShared - rest) / (stage_bytes + scale_bytes)) : 0;
      if (depth > kMaxDepth) depth = kMaxDepth;
      if (depth < 1) continue;
      for (int log = splits > 1 ? kWarpsLog : 0; log <= kWarpsLog; ++log) {
        const int at_once = clusters << (kWarpsLog - log), rounds = (tiles + at_once - 1) / at_once;
        const long long stages = (per + (1 << log) - 1) >> log;
        const long long cost = rounds * (stages * (r == 2 ? 7 : 4) + (log ? 2 : 1)) * (depth == 1 ? 2 : 1);
        if (best != 0 && cost >= best) continue;
        best = cost;
        a.p = p;
        a.depth = depth; a.along_log = log; a.tiles = tiles;
        a.parts_log = parts == 4 ? 2 : parts - 1; a.splits = splits; a.range = per * kStageInputs; a.pitch = (int)pitch; a.scale_pitch = scale_pitch;
        a.ring_at = (int)x_bytes;
        a.scale_at = a.ring_at + depth * stage_bytes;
        a.fix_at = a.scale_at + depth * scale_bytes;
        a.red_at = a.fix_at + (int)fix_bytes;
        a.sum_at = a.red_at + red_bytes;
        a.group_mul = (uint32_t)(((1ull << 31) + group32 - 1) / group32);
        rt = r;
        shared = (int)(rest + depth * (stage_bytes + scale_bytes));
        found = true;
      }
    }
    if (best == 0) continue;
    // more CTAs per tile only where the GPU is not filled and every warp keeps a stage
    if (a.tiles * splits * 2 > sm_count || per < 2 * kWarps) break;
  }
  return found;
}

}  // namespace

// From hq_create.
bool hq_product_few_init() { return load_driver_entry_points(); }

bool hq_product_few_supported(const ProductArgs& p, int sm_count) {
  if (p.j > kMaxColumns || p.j * parts_of(p) > kMaxColumns || p.q_cols % 32 || (p.b_stride % 8 && p.j > 1)) return false;
  FewArgs a{};
  int rt, shared;
  return plan(p, sm_count, a, rt, shared);
}

bool hq_plan_product_few(const ProductArgs& p, int sm_count, hq_product_plan* out) {
  if (!hq_product_few_supported(p, sm_count)) return false;
  FewArgs a{};
  int rt, shared;
  plan(p, sm_count, a, rt, shared);
  const int at_once = (sm_count / a.splits) << (kWarpsLog - a.along_log);
  out->columns = 8 * columns_eights(p.j, 1 << a.parts_log); out->outputs = kRows * rt; out->splits = a.splits;
  out->steps = a.range / kStageInputs;
  out->rounds = (a.tiles + at_once - 1) / at_once;
  out->stages = a.depth; out->groups = 1 << a.along_log; out->units = 0; out->unit_stages = 0;
  return true;
}

hq_status hq_launch_product_few(hq_handle* h, int type, const ProductArgs& p, cudaStream_t s) {
  FewArgs a{};
  int rt = 1, shared = 0;
  if (!plan(p, h->sm_count, a, rt, shared)) return HQ_ERR_UNSUPPORTED;
  a.status = h->dev_status;
  const int nb = columns_eights(p.j, 1 << a.parts_log);
  const int at_once = h->sm_count / a.splits;
  const int grid = (a.tiles < at_once ? a.tiles : at_once) * a.splits;
  CUtensorMap map;
  if (!encode_rows_map(&map, p.q, p.i, p.q_cols >> 1, 128, kRows * rt, CU_TENSOR_MAP_SWIZZLE_128B)) return HQ_ERR_CUDA;
  const cudaError_t e = type == HQ_F16 ? launch_type<__half>(nb, rt, map, a, grid, shared, h->device, s)
                                       : launch_type<__nv_bfloat16>(nb, rt, map, a, grid, shared, h->device, s);
  return e == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
