// The three products on the tensor cores (tcgen05.mma kind::f16, 32-bit accumulators in tensor memory):
//   out[j][i] = bias[i] + sum_r A(i, r) * B(j, r).
// The quantized operand A lies on the 128 lanes, so that a weight matrix fills them whatever the number of tokens; B lies on
// NT <= 256 columns.  Both come by TMA as they are stored, A into a ring of its own, from which warps restore each value in the type
// of B - (integer - offset) * scale, one rounding - and write the swizzled tile the MMA reads.  FORWARD tiles are K-major; DGRAD and
// WGRAD reduce over the rows of what is stored, their tiles are MN-major, so no operand is ever transposed by hand.
// Roles: one thread fetches, one issues MMAs, four groups of four warps convert A, each every fourth stage (a stage takes a warp
// longer than its MMAs take), four warps drain the accumulators; CTAs are persistent and have two accumulators, so that a tile is
// drained while the next one is computed.  When there are too few tiles to go round, the CTAs of a cluster share a tile's
// reduction and add their parts in rank order through distributed shared memory.
#include "../csrc/tc_common.cuh"
#include "float_internal.cuh"

namespace {

constexpr int kThreads = 768;
constexpr int kStep = 64;                         // values of the reduction per stage: 128 bytes, one swizzle span
constexpr int kGroups = 4;                        // of converter warps, which take the stages in turn: one waits, the other works
constexpr int kConverterWarps = 4;                // per group
constexpr int kTileABytes = kTileC * kStep * 2;

enum Role { ROLE_FETCH = 0, ROLE_MMA = 1, ROLE_ALLOC = 2, ROLE_CONVERT = 4, ROLE_DRAIN = 20 };   // by warp

template <int NT>
struct Shape {
  static constexpr int kStages = NT == 256 ? 4 : NT == 128 ? 5 : 6;
  static constexpr int kStageBytes = kTileABytes + (NT < 64 ? 64 : NT) * kStep * 2;
  static constexpr int kRawBytes = NT == 256 ? 32 * 1024 : 64 * 1024;     // ring of the quantized operand
  static constexpr int kSharedBytes = kStages * kStageBytes + kRawBytes + 1024;
};
// One fetch of the quantized operand: FORWARD 128 rows of 128 bytes, the inputs of four stages; DGRAD 64 rows of 64 bytes and WGRAD 64
// rows of 128 bytes, one stage.
template <int KIND>
struct Unit {
  static constexpr int kStagesOf = KIND == PRODUCT_FORWARD ? 4 : 1;
  static constexpr int kRowBytes = KIND == PRODUCT_DGRAD ? 64 : 128, kRows = KIND == PRODUCT_FORWARD ? kTileC : kStep;
  static constexpr int kBytes = kRowBytes * kRows;
};
constexpr int kMaxUnits = 16;

struct Control {
  unsigned long long full_a[8], full_b[8], empty[8], raw_full[kMaxUnits], raw_empty[kMaxUnits], acc_full[2], acc_empty[2], drain;
  uint32_t tmem;
  volatile uint32_t abort_flag;
  volatile uint32_t flip;
};

struct TcArgs {
  ProductArgs p;
  int i_tiles, tiles;       // tiles along i; all tiles
  int steps;                // stages of the whole reduction
  int splits, split_steps;  // CTAs per tile, stages of each
  uint32_t group_mul;       // FORWARD: 2^31 / (group / 32), rounded up, where that divides exactly (see hq_launch_product_tc), else 0
  uint32_t* status;
};

__device__ __forceinline__ void mma_f16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
// Operand tile in 128-byte swizzled rows.  K-major: a row is 64 values of the reduction, eight rows are 1024 bytes.  MN-major: a row
// is 64 values along the lanes / columns, eight rows (steps of the reduction) are 1024 bytes (stride), the next 64 lanes follow
// after 64 rows (leading).
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, bool mn_major) {
  uint64_t d = (uint64_t)((addr >> 4) & 0x3FFF);
  d |= (uint64_t)(mn_major ? (kStep * 128) >> 4 : 1) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// Wait for work in flight before a CTA that gave up ends; bounded by itself, whatever the abort flag says.
__device__ __forceinline__ void drain_wait(uint32_t bar, uint32_t parity, uint32_t* status) {
  const unsigned long long t0 = global_ns();
  while (!mbar_try_wait_for(bar, parity, kSuspendNs)) {
    if (global_ns() - t0 > kWaitBudgetNs) { atomicCAS(status, 0u, (uint32_t)HQ_DEV_TIMEOUT_DRAIN); return; }
  }
}

__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ void store_shared(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Pairs of 16-bit values.  `kMagic4` with a 4-bit number in its low bits is kOffset - 8 + that number, exactly.
template <class T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
  using Two = __nv_bfloat162;
  static constexpr uint32_t kMagic4 = 0x43004300u, kOffset4 = 0x43084308u;     // 128, 136
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { const Two v = __floats2bfloat162_rn(lo, hi); return *(const uint32_t*)&v; }
  static __device__ __forceinline__ uint32_t twice(float s) { return pack(s, s); }
};
template <> struct Pair<__half> {
  using Two = __half2;
  static constexpr uint32_t kMagic4 = 0x64006400u, kOffset4 = 0x64086408u;     // 1024, 1032
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { const Two v = __floats2half2_rn(lo, hi); return *(const uint32_t*)&v; }
  static __device__ __forceinline__ uint32_t twice(float s) { return pack(s, s); }
};
template <class T>
__device__ __forceinline__ uint32_t scaled4(uint32_t magic, uint32_t scale2) {
  using Two = typename Pair<T>::Two;
  const uint32_t offset = Pair<T>::kOffset4;
  const Two v = __hmul2(__hsub2(*(const Two*)&magic, *(const Two*)&offset), *(const Two*)&scale2);
  return *(const uint32_t*)&v;
}
// Eight packed 4-bit integers -> eight values times the scale, in order.  The sign bit of each integer is turned over on the way
// (two's complement to offset by 8).  The subtraction is exact, the product rounds once.
// (`flip`, Pair<T>::kOffset4, comes out of memory: with both constants of the masking in sight the compiler makes two instructions of
// each.)
template <class T>
__device__ __forceinline__ void convert4(uint32_t w, uint32_t scale2, uint32_t flip, uint32_t (&out)[4]) {
  constexpr uint32_t kMask = 0x000f000fu;
  const uint32_t p0 = scaled4<T>((w & kMask) ^ flip, scale2);                  // values 0 and 4
  const uint32_t p1 = scaled4<T>(((w >> 4) & kMask) ^ flip, scale2);           // 1 and 5
  const uint32_t p2 = scaled4<T>(((w >> 8) & kMask) ^ flip, scale2);           // 2 and 6
  const uint32_t p3 = scaled4<T>(((w >> 12) & kMask) ^ flip, scale2);          // 3 and 7
  out[0] = __byte_perm(p0, p1, 0x5410);
  out[1] = __byte_perm(p2, p3, 0x5410);
  out[2] = __byte_perm(p0, p1, 0x7632);
  out[3] = __byte_perm(p2, p3, 0x7632);
}
// Four signed bytes -> four values times a 32-bit scale, rounded once.  2^23 + (byte + 128) is a float whose last byte is that number.
template <class T>
__device__ __forceinline__ void convert8(uint32_t w, float scale, uint32_t& lo, uint32_t& hi) {
  const uint32_t v = w ^ 0x80808080u;
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = (__uint_as_float(__byte_perm(v, 0x4b000000u, 0x7540 + i)) - 8388736.f) * scale;
  lo = Pair<T>::pack(f[0], f[1]);
  hi = Pair<T>::pack(f[2], f[3]);
}

// The two scales of a converter thread's 64 integers of a stage (one per half), fetched a stage of its group ahead.
template <int KIND, class T>
struct Scales {
  const ProductArgs& p;
  const int row_part, lane_part;
  const uint8_t* base;
  int limit[2];                    // FORWARD: nothing; else 1 if the half's columns exist
  int second;                      // from the first half's scale to the second's (not FORWARD)
  bool row_live;

  __device__ __forceinline__ Scales(const ProductArgs& args, int t)
      : p(args), row_part(KIND == PRODUCT_FORWARD ? t : t & 63), lane_part(KIND == PRODUCT_FORWARD ? 0 : (t >> 6) * 64) {}
  __device__ __forceinline__ void enter(int i0, bool tile_live) {
    if (KIND == PRODUCT_FORWARD) {
      const long long row = i0 + row_part;
      row_live = tile_live && row < p.i;
      base = (const uint8_t*)p.scale + row * p.groups * sizeof(T);
    } else {
      const int col = i0 + lane_part;
      row_live = tile_live;
      limit[0] = col < p.i; limit[1] = col + 32 < p.i;
      second = (col + 32) / p.group - col / p.group;
      base = (const uint8_t*)p.scale + (long long)(col / p.group) * (KIND == PRODUCT_DGRAD ? sizeof(T) : sizeof(float));
    }
  }
  // of stage `st` of the tile entered; zero for what does not exist
  __device__ __forceinline__ void load(int st, uint32_t group_mul, float (&scale)[2]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      scale[h] = 0.f;
      if (KIND == PRODUCT_FORWARD) {
        const int k = st * kStep + 32 * h;
        if (row_live && k < p.r) scale[h] = hq_to_float(((const T*)base)[group_mul ? __umulhi((uint32_t)k >> 4, group_mul) : k / p.group]);
      } else {
        const long long row = st * kStep + row_part;
        if (row_live && row < p.r && limit[h]) {
          if (KIND == PRODUCT_DGRAD) scale[h] = hq_to_float(((const T*)base)[row * p.groups + h * second]);
          else scale[h] = ((const float*)base)[row * p.groups + h * second];
        }
      }
    }
  }
};

// One thread's part of a stage: 64 integers of a row of what was fetched, to one row of the operand tile.
template <int KIND, class T>
__device__ __forceinline__ void convert_stage(uint32_t raw, int stage_of_unit, const float (&scale)[2], uint32_t tile_a, int t, uint32_t flip) {
  const int row = KIND == PRODUCT_FORWARD ? t : t & 63, half = KIND == PRODUCT_FORWARD ? 0 : t >> 6;
  const uint32_t to = tile_a + half * (kStep * 128) + row * 128;
  constexpr int kPieces = KIND == PRODUCT_WGRAD ? 4 : 2;           // of 16 bytes
  uint4 q[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int piece = (KIND == PRODUCT_FORWARD ? stage_of_unit * 2 : half * kPieces) + i;
    const uint32_t swizzled = KIND == PRODUCT_DGRAD ? piece ^ ((row >> 1) & 3) : piece ^ (row & 7);
    q[i] = load_shared(raw + row * Unit<KIND>::kRowBytes + (swizzled << 4));
  }
  const uint32_t* w = (const uint32_t*)q;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    uint32_t v[4];
    if (KIND == PRODUCT_WGRAD) {
      convert8<T>(w[2 * c], scale[c >> 2], v[0], v[1]);
      convert8<T>(w[2 * c + 1], scale[c >> 2], v[2], v[3]);
    } else {
      convert4<T>(w[c], Pair<T>::twice(scale[c >> 2]), flip, v);   // (exact: the scales have the type T)
    }
    store_shared(to + ((c ^ (row & 7)) << 4), v[0], v[1], v[2], v[3]);
  }
}

template <int KIND, class T, int NT>
__global__ void __launch_bounds__(kThreads, 1) product_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_b, const TcArgs a) {
  extern __shared__ uint8_t raw_shared[];
  __shared__ Control ctl;
  constexpr int kStages = Shape<NT>::kStages, kStageBytes = Shape<NT>::kStageBytes;
  constexpr int kBoxes = KIND == PRODUCT_WGRAD ? (NT + 63) / 64 : 1;
  constexpr int kBBytes = KIND == PRODUCT_WGRAD ? kBoxes * 64 * kStep * 2 : NT * kStep * 2;     // that a stage's copies bring
  constexpr uint32_t kColumns = NT * 2;
  constexpr int kPer = Unit<KIND>::kStagesOf, kUnits = Shape<NT>::kRawBytes / Unit<KIND>::kBytes;
  const uint32_t base = (smem_u32(raw_shared) + 1023u) & ~1023u, raw_ring = base + kStages * kStageBytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const ProductArgs& p = a.p;
  const int rank = a.splits > 1 ? (int)cluster_ctarank() : 0;
  const int first = blockIdx.x / a.splits, stride = gridDim.x / a.splits;
  const int begin = rank * a.split_steps, end = min(a.steps, begin + a.split_steps);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&ctl.full_a[s]), kConverterWarps);
      mbar_init(smem_u32(&ctl.full_b[s]), 1);
      mbar_init(smem_u32(&ctl.empty[s]), 1);
    }
    for (int u = 0; u < kUnits; ++u) { mbar_init(smem_u32(&ctl.raw_full[u]), 1); mbar_init(smem_u32(&ctl.raw_empty[u]), kPer * kConverterWarps); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctl.acc_full[b]), 1); mbar_init(smem_u32(&ctl.acc_empty[b]), 4); }
    mbar_init(smem_u32(&ctl.drain), 1);
    ctl.abort_flag = 0;
    ctl.flip = Pair<T>::kOffset4;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == ROLE_ALLOC) tmem_alloc(smem_u32(&ctl.tmem), kColumns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem;
  hq_pdl_entry();

  if (warp == ROLE_FETCH) {
    if (elect_one()) {
      int s = 0, u = 0;
      uint32_t phase = 0, u_phase = 0, issued = 0, u_issued = 0;
      bool ok = true;
      // the quantized operand of stages `st` and on
      auto fetch_unit = [&](int i0, int st) {
        if (!mbar_wait(smem_u32(&ctl.raw_empty[u]), u_phase ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER)) return false;
        const uint32_t bar = smem_u32(&ctl.raw_full[u]), dst = raw_ring + u * Unit<KIND>::kBytes;
        mbar_expect_tx(bar, Unit<KIND>::kBytes);
        if (KIND == PRODUCT_FORWARD) tma_load_2d(dst, &map_q, bar, st * (kStep / 2), i0);
        else tma_load_2d(dst, &map_q, bar, KIND == PRODUCT_DGRAD ? i0 >> 1 : i0, st * kStep);
        u_issued |= 1u << u;
        if (++u == kUnits) { u = 0; u_phase ^= 1; }
        return true;
      };
      for (int tile = first; tile < a.tiles && ok; tile += stride) {
        const int i0 = tile % a.i_tiles * kTileC, j0 = tile / a.i_tiles * NT;
        for (int st = begin; st < end; ++st) {
          if ((st - begin) % kPer == 0 && !fetch_unit(i0, st)) { ok = false; break; }
          if (!mbar_wait(smem_u32(&ctl.empty[s]), phase ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER)) { ok = false; break; }
          const uint32_t bar = smem_u32(&ctl.full_b[s]), dst = base + s * kStageBytes + kTileABytes;
          mbar_expect_tx(bar, kBBytes);
          if (KIND == PRODUCT_WGRAD) {
#pragma unroll
            for (int b = 0; b < kBoxes; ++b) tma_load_2d(dst + b * (64 * kStep * 2), &map_b, bar, j0 + b * 64, st * kStep);
          } else {
            tma_load_2d(dst, &map_b, bar, st * kStep, j0);
          }
          issued |= 1u << s;
          if (++s == kStages) { s = 0; phase ^= 1; }
        }
      }
      if (!ok) {                                                 // given up: let the copies in flight land before the memory goes
        for (int k = 0; k < kStages; ++k)
          if (issued >> k & 1) drain_wait(smem_u32(&ctl.full_b[k]), k < s ? phase : phase ^ 1, a.status);
        for (int k = 0; k < kUnits; ++k)
          if (u_issued >> k & 1) drain_wait(smem_u32(&ctl.raw_full[k]), k < u ? u_phase : u_phase ^ 1, a.status);
      }
    }
  } else if (warp == ROLE_MMA) {
    if (elect_one()) {
      constexpr bool kAMn = KIND != PRODUCT_FORWARD, kBMn = KIND == PRODUCT_WGRAD;
      constexpr uint32_t kType = sizeof(typename Pair<T>::Two) == 4 && Pair<T>::kMagic4 == 0x43004300u ? 1u : 0u;    // bf16 : fp16
      constexpr uint32_t idesc = (1u << 4) | (kType << 7) | (kType << 10) | ((uint32_t)kAMn << 15) | ((uint32_t)kBMn << 16) |
                                 ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(kTileC >> 4) << 24);
      int s = 0; uint32_t phase = 0;
      int buf = 0; uint32_t acc_phase = 0;
      bool ok = true;
      for (int tile = first; tile < a.tiles && ok; tile += stride) {
        if (!mbar_wait(smem_u32(&ctl.acc_empty[buf]), acc_phase ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_MMA)) { ok = false; break; }
        tc_fence_after();
        for (int st = begin; st < end; ++st) {
          if (!mbar_wait(smem_u32(&ctl.full_b[s]), phase, &ctl, a.status, HQ_DEV_TIMEOUT_MMA) ||
              !mbar_wait(smem_u32(&ctl.full_a[s]), phase, &ctl, a.status, HQ_DEV_TIMEOUT_MMA)) { ok = false; break; }
          tc_fence_after();
          const uint32_t tile_a = base + s * kStageBytes;
          uint64_t da = tile_desc(tile_a, kAMn), db = tile_desc(tile_a + kTileABytes, kBMn);
#pragma unroll
          for (int k = 0; k < kStep / 16; ++k) {
            mma_f16(tmem + buf * NT, da, db, idesc, (st > begin || k > 0) ? 1u : 0u);
            da += kAMn ? (16 * 128) >> 4 : 2;
            db += kBMn ? (16 * 128) >> 4 : 2;
          }
          mma_commit(smem_u32(&ctl.empty[s]));
          if (++s == kStages) { s = 0; phase ^= 1; }
        }
        if (!ok) break;
        mma_commit(smem_u32(&ctl.acc_full[buf]));
        if (++buf == 2) { buf = 0; acc_phase ^= 1; }
      }
      if (!ok) {
        mma_commit(smem_u32(&ctl.drain));
        drain_wait(smem_u32(&ctl.drain), 0, a.status);
      }
    }
  } else if (warp >= ROLE_CONVERT && warp < ROLE_CONVERT + kGroups * kConverterWarps) {
    const int group = (warp - ROLE_CONVERT) / kConverterWarps, t = threadIdx.x - (ROLE_CONVERT + group * kConverterWarps) * 32;
    const uint32_t flip = ctl.flip;
    // Stages are numbered through the CTA's tiles, a tile filled up to whole units; the group takes every kGroups-th.
    const int steps = end - begin, padded = (steps + kPer - 1) / kPer * kPer;
    Scales<KIND, T> scales(p, t);
    int tile = first, st = group, tile_no = 0;                   // stage of the tile, and how many tiles came before
    auto settle = [&]() {
      bool moved = false;
      while (st >= padded && tile < a.tiles) { st -= padded; tile += stride; ++tile_no; moved = true; }
      return moved;
    };
    settle();
    scales.enter(tile % a.i_tiles * kTileC, tile < a.tiles);
    float scale[2];
    scales.load(begin + st, a.group_mul, scale);
    bool ok = true;
    while (tile < a.tiles && ok) {
      const long long n = (long long)tile_no * steps + st, v = (long long)tile_no * padded + st;
      const bool real = st < steps;
      const unsigned unit_no = (unsigned)(v / kPer);
      const int u = unit_no % kUnits, s = (int)((unsigned)n % kStages), of_unit = (int)(v % kPer);
      const uint32_t u_phase = (unit_no / kUnits) & 1, phase = ((unsigned)n / kStages) & 1;
      ok = mbar_wait(smem_u32(&ctl.raw_full[u]), u_phase, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER);
      if (real) ok = ok && mbar_wait(smem_u32(&ctl.empty[s]), phase ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (real) {
        convert_stage<KIND, T>(raw_ring + u * Unit<KIND>::kBytes, of_unit, scale, base + s * kStageBytes, t, flip);
        fence_async_smem();
      }
      st += kGroups;
      if (settle()) scales.enter(tile % a.i_tiles * kTileC, tile < a.tiles);
      scales.load(begin + st, a.group_mul, scale);
      __syncwarp();
      if (lane == 0) {
        if (real) mbar_arrive(smem_u32(&ctl.full_a[s]));
        mbar_arrive(smem_u32(&ctl.raw_empty[u]));
      }
    }
  } else if (warp >= ROLE_DRAIN) {
    const int quad = warp & 3;
    int buf = 0; uint32_t acc_phase = 0;
    for (int tile = first; tile < a.tiles; tile += stride) {
      const int i = tile % a.i_tiles * kTileC + quad * 32 + lane;
      const int j0 = tile / a.i_tiles * NT;
      const float add = (p.bias && i < p.i) ? hq_to_float(((const T*)p.bias)[i]) : 0.f;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.acc_full[buf]), acc_phase, &ctl, a.status, HQ_DEV_TIMEOUT_EPILOGUE))) break;
      tc_fence_after();
      for (int c = 0; c < NT / 32; ++c) {
        int v[32];
        tmem_ld32_issue(tmem + buf * NT + ((uint32_t)(quad * 32) << 16) + c * 32, v);
        tmem_ld_wait();
        tie(v);
        if (a.splits > 1) {
          float* part = (float*)(raw_shared + (base - smem_u32(raw_shared)));
#pragma unroll
          for (int k = 0; k < 32; ++k) part[(c * 32 + k) * kTileC + quad * 32 + lane] = __int_as_float(v[k]);
        } else if (i < p.i) {
          T* out = (T*)p.out + (long long)(j0 + c * 32) * p.out_stride + i;
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (j0 + c * 32 + k < p.j) out[(long long)k * p.out_stride] = hq_from_float<T>(__int_as_float(v[k]) + add);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl.acc_empty[buf]));
      if (++buf == 2) { buf = 0; acc_phase ^= 1; }
    }
  }
  __syncwarp();
  if (a.splits > 1) {
    cluster_sync_all();                                          // every part is written
    const int i0 = first % a.i_tiles * kTileC, j0 = first / a.i_tiles * NT;
    const int cols = NT / a.splits;                              // columns this CTA adds up (splits divides NT)
    const uint32_t mine = base + rank * cols * kTileC * 4;
    for (int e = threadIdx.x; e < cols * kTileC; e += kThreads) {
      const int i = i0 + e % kTileC, j = j0 + rank * cols + e / kTileC;
      if (i < p.i && j < p.j) {
        float sum = 0.f;
        for (int k = 0; k < a.splits; ++k) {
          float v;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(in_cta(mine + e * 4, k)));
          sum += v;
        }
        if (p.bias) sum += hq_to_float(((const T*)p.bias)[i]);
        ((T*)p.out)[(long long)j * p.out_stride + i] = hq_from_float<T>(sum);
      }
    }
    cluster_sync_all();                                          // nobody reads a part any more
  }
  tc_fence_before();
  __syncthreads();
  if (warp == ROLE_ALLOC) { tc_fence_after(); tmem_dealloc(tmem, kColumns); }
}

// ---------------------------------------------------------------- host side ------------------
bool encode_b_map(CUtensorMap* map, int type, const ProductArgs& a, ProductKind kind, int nt) {
  const long long cols = kind == PRODUCT_WGRAD ? a.j : a.r, rows = kind == PRODUCT_WGRAD ? a.r : a.j;
  const long long stride = rows == 1 ? (cols + 7) / 8 * 8 : a.b_stride;      // (the stride of a single row means nothing)
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {kStep, (cuuint32_t)(kind == PRODUCT_WGRAD ? kStep : nt)};
  const cuuint32_t estr[2] = {1, 1};
  return g_encode_tiled(map, type == HQ_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.b), dims,
                        strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KIND, class T, int NT>
cudaError_t launch(const CUtensorMap* map, const TcArgs& a, int grid, cudaStream_t s) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)a.splits; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = Shape<NT>::kSharedBytes; cfg.stream = s;
  cfg.attrs = attr; cfg.numAttrs = a.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, product_tc_kernel<KIND, T, NT>, map[0], map[1], a);
}
template <int KIND, class T>
cudaError_t launch_width(int nt, const CUtensorMap* map, const TcArgs& a, int grid, cudaStream_t s) {
  switch (nt) {
    case 32: return launch<KIND, T, 32>(map, a, grid, s);
    case 64: return launch<KIND, T, 64>(map, a, grid, s);
    case 128: return launch<KIND, T, 128>(map, a, grid, s);
    default: return launch<KIND, T, 256>(map, a, grid, s);
  }
}
template <class T>
cudaError_t launch_kind(ProductKind kind, int nt, const CUtensorMap* map, const TcArgs& a, int grid, cudaStream_t s) {
  return kind == PRODUCT_FORWARD ? launch_width<PRODUCT_FORWARD, T>(nt, map, a, grid, s)
       : kind == PRODUCT_DGRAD ? launch_width<PRODUCT_DGRAD, T>(nt, map, a, grid, s) : launch_width<PRODUCT_WGRAD, T>(nt, map, a, grid, s);
}

template <int KIND, class T, int NT>
bool allow_shared() {
  return cudaFuncSetAttribute(product_tc_kernel<KIND, T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<NT>::kSharedBytes) == cudaSuccess;
}
template <int KIND, class T>
bool allow_widths() { return allow_shared<KIND, T, 32>() && allow_shared<KIND, T, 64>() && allow_shared<KIND, T, 128>() && allow_shared<KIND, T, 256>(); }
template <class T>
bool allow_kinds() { return allow_widths<PRODUCT_FORWARD, T>() && allow_widths<PRODUCT_DGRAD, T>() && allow_widths<PRODUCT_WGRAD, T>(); }

}  // namespace

// Once per device, from hq_create.
bool hq_product_tc_init() { return load_driver_entry_points() && allow_kinds<__half>() && allow_kinds<__nv_bfloat16>(); }

bool hq_product_tc_supported(ProductKind kind, const ProductArgs& a) {
  if (a.r < 1) return false;
  const int b_rows = kind == PRODUCT_WGRAD ? a.r : a.j;
  if (a.b_stride % 8 && b_rows > 1) return false;                          // rows of B start on 16 bytes
  return kind == PRODUCT_WGRAD ? a.q_cols % 16 == 0 : a.q_cols % 32 == 0;  // and so do those of the quantized operand
}

hq_status hq_launch_product_tc(hq_handle* h, ProductKind kind, int type, const ProductArgs& p, cudaStream_t s) {
  TcArgs a{};
  a.p = p;
  a.status = h->dev_status;
  a.i_tiles = (p.i + kTileC - 1) / kTileC;
  a.steps = (p.r + kStep - 1) / kStep;
  const int nt = p.j > 128 ? 256 : p.j > 64 ? 128 : p.j > 32 ? 64 : 32;
  const long long tiles = (long long)a.i_tiles * ((p.j + nt - 1) / nt);
  if (tiles > 0x3fffffff) return HQ_ERR_UNSUPPORTED;
  a.tiles = (int)tiles;
  a.splits = 1;
  while (a.splits < 8 && tiles * a.splits * 2 <= h->sm_count && a.steps >= a.splits * 2 * 4) a.splits *= 2;
  a.split_steps = (a.steps + a.splits - 1) / a.splits;
  while (a.splits > 1 && (a.splits - 1) * a.split_steps >= a.steps) { a.splits /= 2; a.split_steps = (a.steps + a.splits - 1) / a.splits; }
  const int grid = a.splits > 1 ? a.tiles * a.splits : (int)(tiles < h->sm_count ? tiles : h->sm_count);
  // k / group by a multiply-high, exact while (k / 32) (group / 32) < 2^31
  if (kind == PRODUCT_FORWARD && p.r <= (1 << 20)) {
    const unsigned group32 = (unsigned)(p.group >= p.r ? 1 << 20 : p.group) / 32;
    a.group_mul = (uint32_t)(((1ull << 31) + group32 - 1) / group32);
  }
  CUtensorMap map[2];
  const bool bytes = kind == PRODUCT_WGRAD;
  const int unit_row = kind == PRODUCT_DGRAD ? Unit<PRODUCT_DGRAD>::kRowBytes : 128, unit_rows = kind == PRODUCT_FORWARD ? kTileC : kStep;
  if (!encode_rows_map(&map[0], p.q, kind == PRODUCT_FORWARD ? p.i : p.r, bytes ? p.q_cols : p.q_cols >> 1, unit_row, unit_rows, swizzle_for(unit_row)) ||
      !encode_b_map(&map[1], type, p, kind, nt)) return HQ_ERR_CUDA;
  const cudaError_t e = type == HQ_F16 ? launch_kind<__half>(kind, nt, map, a, grid, s) : launch_kind<__nv_bfloat16>(kind, nt, map, a, grid, s);
  return e == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
