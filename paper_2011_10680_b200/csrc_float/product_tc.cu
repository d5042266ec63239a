// The three products on the tensor cores (tcgen05.mma kind::f16, 32-bit accumulators in tensor memory):
//   out[j][i] = bias[i] + sum_r A(i, r) * B(j, r).
// The quantized operand A lies on the 128 lanes, so that a weight matrix fills them whatever the number of tokens; B lies on
// NT <= 256 columns.  Both come by TMA as they are stored, A into a ring of its own, from which warps restore each value in the type
// of B - (integer - offset) * scale, one rounding - and write the swizzled tile the MMA reads.  FORWARD tiles are K-major; DGRAD and
// WGRAD reduce over the rows of what is stored, their tiles are MN-major, so no operand is ever transposed by hand.
// Roles: one thread fetches, one issues MMAs, groups of warps convert A, taking the stages in turn, four warps drain the accumulators;
// CTAs are persistent and have two accumulators, so that a tile is drained while the next one is computed.  With many columns two
// CTAs share their MMAs (cta_group::2).  When there are too few tiles to go round, the CTAs or pairs of a cluster share a tile's
// reduction and add their parts in rank order through distributed shared memory.
//
// What bounds it.  256 columns: the tensor cores under the power cap - 4001 tokens, 16384 x 4096 bf16 in 387 us alone (1388 TFLOP/s, 0.83
// of the measured burst, at the sustained rate), 443 us back to back; 8192 x 16384 x 4096 fp16 gradient 780 us (1410).  Few
// columns: the turn of a stage through converters and barriers, some 600 cycles (650 with 256 columns), and some 4 us before the first
// MMA and behind the last - 48 tokens, 8192 x 8192: 29 us, 1.4 TB/s.  Neither the memory nor the arithmetic is full then: of 1294 warp
// instructions a stage 544 convert (17 per eight weights), 1.6 a cycle are issued of 4, and warps wait most for loaded scales and
// at barriers.
#include <type_traits>

#include "../csrc/tc_common.cuh"
#include "float_internal.cuh"

namespace {

constexpr int kThreads = 896;
constexpr int kStep = 64;                         // values of the reduction per stage: 128 bytes, one swizzle span
constexpr int kTileABytes = kTileC * kStep * 2;

// Roles by warp.  A warp's scheduler is its number modulo four, and the threads that fetch and issue MMAs, which every stage waits
// for, share theirs with few converters or none: beside four of them each of their instructions takes some 14 cycles (48 tokens,
// 8192 x 8192, with groups of four warps: 34.3 us, apart 33.5).  Accumulator lanes 32 q .. 32 q + 31 belong to warps 4 n + q.
enum Role { ROLE_FETCH, ROLE_MMA, ROLE_ALLOC, ROLE_CONVERT, ROLE_DRAIN };
__device__ __forceinline__ Role role_of(int warp) {
  if (warp & 3) return warp < 24 ? ROLE_CONVERT : ROLE_DRAIN;
  return warp == 0 ? ROLE_FETCH : warp == 4 ? ROLE_MMA : warp == 8 ? ROLE_ALLOC : warp == 12 ? ROLE_DRAIN : ROLE_CONVERT;
}
// Converter warps by number: eighteen on schedulers of their own, and three beside the issuers, which come last (`beside_first`: first;
// with few columns a stage is bound by the converters' instructions, and a fourth scheduler helps more than it hinders: 48 tokens,
// 8192 x 8192: 30.5 us, so 29.0; 4001 tokens, 16384 x 4096, on pairs: 389 us, so 394).
constexpr int kMaxConverters = 21;
__device__ __forceinline__ int converter_number(int warp, bool beside_first) {
  if (warp & 3) return (beside_first ? 3 : 0) + (warp >> 2) * 3 + (warp & 3) - 1;
  return (beside_first ? 0 : 18) + (warp >> 2) - 4;
}

// One fetch of the quantized operand: FORWARD 128 rows of 128 bytes, the inputs of four stages (64 bytes and two stages with 128 columns
// and more, see Shape); DGRAD 64 rows of 64 bytes and WGRAD 64 rows of 128 bytes, one stage.
template <int KIND, int NT>
struct Unit {
  static constexpr int kStagesOf = KIND != PRODUCT_FORWARD ? 1 : NT >= 128 ? 2 : 4;
  static constexpr int kRowBytes = KIND == PRODUCT_FORWARD ? kStagesOf * kStep / 2 : KIND == PRODUCT_DGRAD ? 64 : 128;
  static constexpr int kRows = KIND == PRODUCT_FORWARD ? kTileC : kStep;
  static constexpr int kBytes = kRowBytes * kRows;
};
// NT = 256: two CTAs of a cluster (neighbouring SMs) share every MMA (cta_group::2), 256 lanes x 256 columns: each converts its own
// 128 lanes and fetches half of the columns.  One CTA with 256 columns of its own is bound by its shared memory: per stage (512
// cycles of MMAs) 48 KB go in and 48 KB out beside what the converters move.
// Converters work in groups, which take the stages in turn (most of a warp's time on one is waiting): two warps with two rows of 64
// integers per thread, or four with one.  A barrier tells a round of its ring by its parity, and a wait returns
// at once while the round before is still under way: whoever waits has to know that the round before is through.
//   - The ring of the quantized operand: copies land in any order, so a group knows what it has waited for itself and nothing
//     else.  The ring holds a whole number of turns of the groups: a group then finds its stages in the same places every round.
//   - The ring of stages is emptied in order.  A group knows that its own last stage, kGroups before the present one, found its place
//     empty: no more groups than stages.  FORWARD fills a tile's last unit up with stages that nobody converts, so that a group's
//     last stage may be longer ago; but the unit before in the same place is through, whose last stage is at most a whole ring of the
//     quantized operand behind: no more of those stages than stages.
template <int KIND, int NT>
struct Shape {
  static constexpr bool kPair = NT == 256, kWgrad = KIND == PRODUCT_WGRAD;
  static constexpr int kCtas = kPair ? 2 : 1, kColumnsHere = NT / kCtas;
  static constexpr int kStages = kWgrad ? 5 : NT >= 128 ? 6 : 8;    // (WGRAD with 64 columns or less: six, adapter 19.7 us against 19.3)
  static constexpr int kStageBytes = kTileABytes + (kColumnsHere < 64 ? 64 : kColumnsHere) * kStep * 2;
  static constexpr int kPer = Unit<KIND, NT>::kStagesOf;
  static constexpr int kUnits = kWgrad ? 8 : kStages / kPer;       // of the ring of the quantized operand: 64 KB, 24 or 32
  static constexpr int kRawBytes = kUnits * Unit<KIND, NT>::kBytes;
  static constexpr int kSharedBytes = kStages * kStageBytes + kRawBytes + 1024;
  static constexpr int kRowsPerThread = kWgrad ? 1 : 2, kConverterWarps = 4 / kRowsPerThread;
  static constexpr int kGroups = kWgrad ? 4 : kStages;             // (saved activations: five were no faster)
  static_assert((kPer * kUnits) % kGroups == 0 && kGroups <= kStages && (kPer == 1 || kPer * kUnits <= kStages));
  static_assert(kGroups * kConverterWarps <= kMaxConverters && kUnits <= 8 && kStages <= 8);
};

constexpr int kMaxUnits = 8;

struct Control {
  unsigned long long full[8], empty[8], raw_full[kMaxUnits], raw_empty[kMaxUnits], acc_full[2], acc_empty[2], drain;
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
__device__ __forceinline__ void mma_f16_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
// A pair's load: into this CTA's shared memory, counted on a barrier of the leading CTA (`bar`: cluster address).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
// Arrival on a barrier of the leading CTA (`bar`: cluster address).  By the letter of the memory model what is announced to another CTA is
// released at cluster scope; that instruction took 1200 to 1700 cycles.  This form releases at CTA scope.  What it announces was made
// visible where it lies before - operands, which the MMA reads from their own SM, by a proxy fence, tensor memory by a tcgen05
// fence - and a pair's arrivals are usually written like this, but that it suffices rests on observation: repeated calls of every
// shape on pairs give the same bits, and the right ones.
__device__ __forceinline__ void arrive_leading(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
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

// Pairs of 16-bit values; see convert4 for the constants (lower half, upper half): the exponent with the sign bits of both nibbles, the
// factors 1 and 1/8, and what is taken off, 128 + 8 and 16 + 8 (bf16), 1024 + 8 and 128 + 8 (fp16).
template <class T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
  using Two = __nv_bfloat162;
  static constexpr bool kBf16 = true;
  static constexpr uint32_t kFlip = 0x43404308u, kFactor = 0x3e003f80u, kOffset = 0xc1c0c308u;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { const Two v = __floats2bfloat162_rn(lo, hi); return *(const uint32_t*)&v; }
  static __device__ __forceinline__ uint32_t twice(float s) { return pack(s, s); }
};
template <> struct Pair<__half> {
  using Two = __half2;
  static constexpr bool kBf16 = false;
  static constexpr uint32_t kFlip = 0x64406408u, kFactor = 0x30003c00u, kOffset = 0xd840e408u;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { const Two v = __floats2half2_rn(lo, hi); return *(const uint32_t*)&v; }
  static __device__ __forceinline__ uint32_t twice(float s) { return pack(s, s); }
};
// Eight packed 4-bit integers -> eight values times the scale, in order.  Each byte goes to both halves of a word, the upper one
// shifted right by one: its lower nibble lands on bits 0-3 of the lower half, its upper nibble on bits 3-6 of the upper half.  Under
// the exponent of 128 (bf16; 1024 fp16) they stand for 128 + u and 128 + 8 u, u the integer + 8 (its sign bit turned over on the
// way); one exact multiply-add takes both to the integer, and the product rounds once.
// (`flip`, Pair<T>::kFlip, comes out of memory: with both constants of the masking in sight the compiler makes two instructions of it.)
template <class T>
__device__ __forceinline__ void convert4(uint32_t w, uint32_t scale2, uint32_t flip, uint32_t (&out)[4]) {
  using Two = typename Pair<T>::Two;
  const uint32_t shifted = w >> 1, factor = Pair<T>::kFactor, offset = Pair<T>::kOffset;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = (__byte_perm(w, shifted, 0x0400 + 0x1111 * i) & 0x0078000fu) ^ flip;
    const Two v = __hmul2(__hfma2(*(const Two*)&m, *(const Two*)&factor, *(const Two*)&offset), *(const Two*)&scale2);
    out[i] = *(const uint32_t*)&v;
  }
}
// Four signed bytes -> four values times a 32-bit scale, rounded once.  2^23 + (byte + 128) is a float whose last byte is that number;
// the subtraction and the product run on pairs.
template <class T>
__device__ __forceinline__ void convert8(uint32_t w, unsigned long long scale2, uint32_t& lo, uint32_t& hi) {
  const uint32_t v = w ^ 0x80808080u;
  uint32_t out[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t a = __byte_perm(v, 0x4b000000u, 0x7540 + 2 * i), b = __byte_perm(v, 0x4b000000u, 0x7541 + 2 * i);
    unsigned long long f;
    asm("{\n\t.reg .b64 t;\n\tmov.b64 t, {%1, %2};\n\tadd.rn.f32x2 t, t, %3;\n\tmul.rn.f32x2 %0, t, %4;\n\t}"
        : "=l"(f) : "r"(a), "r"(b), "l"(0xcb000080cb000080ull), "l"(scale2));      // - 8388736 twice
    out[i] = Pair<T>::pack(__uint_as_float((uint32_t)f), __uint_as_float((uint32_t)(f >> 32)));
  }
  lo = out[0];
  hi = out[1];
}

// The scales of a converter thread's rows of a stage, one per half of a row's 64 integers, fetched a turn of its group ahead.  Within a
// tile the thread's rows (not FORWARD) move on by a fixed step.
template <int KIND, class T, int ROWS>
struct Scales {
  using S = typename std::conditional<KIND == PRODUCT_WGRAD, float, T>::type;
  const ProductArgs& p;
  const uint32_t group_mul;
  const int row_part, lane_part;   // first of the rows (the second is 32 further on), and the first lane of the half (not FORWARD)
  const S* at;                     // FORWARD: of the first row; else the first scale of the stage to be loaded
  int along;                       // FORWARD: first input of the stage to be loaded; else its first row
  bool exists[2];                  // FORWARD: the rows; else the halves' columns
  int second;                      // from the first half's scale to the second's (not FORWARD)
  long long step;                  // from one turn of the group to the next (not FORWARD)

  __device__ __forceinline__ Scales(const ProductArgs& args, uint32_t mul, int row, int half, int groups)
      : p(args), group_mul(mul), row_part(row), lane_part(half * 64), step((long long)groups * kStep * args.groups) {}
  // stage `st` of the reduction, in the tile of lanes from i0
  __device__ __forceinline__ void enter(int i0, bool tile_exists, int st) {
    if (KIND == PRODUCT_FORWARD) {
      const long long row = i0 + row_part;
      exists[0] = tile_exists && row < p.i;
      exists[1] = tile_exists && row + 32 < p.i;
      at = (const S*)p.scale + row * p.groups;
      along = st * kStep;
    } else {
      const int col = i0 + lane_part, g = col / p.group;
      exists[0] = tile_exists && col < p.i;
      exists[1] = tile_exists && col + 32 < p.i;
      second = (col + 32) / p.group - g;
      along = st * kStep + row_part;
      at = (const S*)p.scale + (long long)along * p.groups + g;
    }
  }
  // zero for what does not exist; then `turns` stages on
  __device__ __forceinline__ void load(int turns, float (&scale)[ROWS][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = along + 32 * h;
      const uint32_t g = KIND != PRODUCT_FORWARD ? 0 : group_mul ? __umulhi((uint32_t)k >> 4, group_mul) : (uint32_t)k / (uint32_t)p.group;
#pragma unroll
      for (int x = 0; x < ROWS; ++x) {
        scale[x][h] = 0.f;
        if (KIND == PRODUCT_FORWARD) {
          if (exists[x] && k < p.r) scale[x][h] = hq_to_float(at[(x ? 32ll * p.groups : 0ll) + g]);
        } else if (exists[h] && along + 32 * x < p.r) {
          // (a group of both halves is fetched once: 333 rows 20.2 us against 21.4, 8191 x 4096 x 4096 weights 290 against 303; the same
          // question for FORWARD costs more than it saves, 48 tokens 29.6 us against 28.8)
          scale[x][h] = h && second == 0 ? scale[x][0] : hq_to_float(at[(x ? 32ll * p.groups : 0ll) + (h ? second : 0)]);
        }
      }
    }
    along += turns * kStep;
    if (KIND != PRODUCT_FORWARD) at += step;
  }
};

// 64 integers of a row of what was fetched (`half`: the half of the lanes, not FORWARD), restored ...
template <int KIND, class T, int ROW_BYTES>
__device__ __forceinline__ void convert_row(uint32_t raw, int stage_of_unit, const float (&scale)[2], int row, int half, uint32_t flip, uint32_t (&v)[8][4]) {
  constexpr int kPieces = KIND == PRODUCT_WGRAD ? 4 : 2;           // of 16 bytes
  uint4 q[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int piece = (KIND == PRODUCT_FORWARD ? stage_of_unit * 2 : half * kPieces) + i;
    const uint32_t swizzled = ROW_BYTES == 64 ? piece ^ ((row >> 1) & 3) : piece ^ (row & 7);
    q[i] = load_shared(raw + row * ROW_BYTES + (swizzled << 4));
  }
  const uint32_t* w = (const uint32_t*)q;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    if (KIND == PRODUCT_WGRAD) {
      const unsigned long long scale2 = (unsigned long long)__float_as_uint(scale[c >> 2]) * 0x100000001ull;
      convert8<T>(w[2 * c], scale2, v[c][0], v[c][1]);
      convert8<T>(w[2 * c + 1], scale2, v[c][2], v[c][3]);
    } else {
      convert4<T>(w[c], Pair<T>::twice(scale[c >> 2]), flip, v[c]);   // (exact: the scales have the type T)
    }
  }
}
// ... and written to a row of the operand tile.
__device__ __forceinline__ void store_row(uint32_t tile_a, int row, int half, const uint32_t (&v)[8][4]) {
  const uint32_t to = tile_a + half * (kStep * 128) + row * 128;
#pragma unroll
  for (int c = 0; c < 8; ++c) store_shared(to + ((c ^ (row & 7)) << 4), v[c][0], v[c][1], v[c][2], v[c][3]);
}

template <int KIND, class T, int NT>
__global__ void __launch_bounds__(kThreads, 1) product_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_b, const TcArgs a) {
  extern __shared__ uint8_t raw_shared[];
  __shared__ Control ctl;
  constexpr bool kPair = Shape<KIND, NT>::kPair;
  constexpr int kStages = Shape<KIND, NT>::kStages, kStageBytes = Shape<KIND, NT>::kStageBytes, kGroups = Shape<KIND, NT>::kGroups;
  constexpr int kCtas = Shape<KIND, NT>::kCtas, kColumnsHere = Shape<KIND, NT>::kColumnsHere;
  constexpr int kBoxes = KIND == PRODUCT_WGRAD ? (kColumnsHere + 63) / 64 : 1;
  constexpr int kBBytes = KIND == PRODUCT_WGRAD ? kBoxes * 64 * kStep * 2 : kColumnsHere * kStep * 2;     // that a CTA's copies bring per stage
  constexpr uint32_t kColumns = NT * 2;
  constexpr int kPer = Shape<KIND, NT>::kPer, kUnits = Shape<KIND, NT>::kUnits, kRowsPerThread = Shape<KIND, NT>::kRowsPerThread;
  constexpr int kConverterWarps = Shape<KIND, NT>::kConverterWarps;
  const uint32_t base = (smem_u32(raw_shared) + 1023u) & ~1023u, raw_ring = base + kStages * kStageBytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Role role = role_of(warp);
  const ProductArgs& p = a.p;
  // the CTAs of a cluster: the parts of a tile's reduction, each by one CTA or a pair
  const bool clustered = kPair || a.splits > 1;
  const int cta = clustered ? (int)cluster_ctarank() : 0, rank = cta / kCtas, in_pair = cta % kCtas, leader = cta - in_pair;
  const int first = blockIdx.x / (a.splits * kCtas), stride = gridDim.x / (a.splits * kCtas);
  const int begin = rank * a.split_steps, end = min(a.steps, begin + a.split_steps);
  auto i_of = [&](int tile) { return (tile % a.i_tiles * kCtas + in_pair) * kTileC; };
  auto j_of = [&](int tile) { return tile / a.i_tiles * NT; };
  // the leading CTA's barrier of that name
  auto leading = [&](unsigned long long& bar) { return kPair ? in_cta(smem_u32(&bar), leader) : smem_u32(&bar); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&ctl.full[s]), 1 + kCtas * kConverterWarps);
      mbar_init(smem_u32(&ctl.empty[s]), 1);
    }
    for (int u = 0; u < kUnits; ++u) { mbar_init(smem_u32(&ctl.raw_full[u]), 1); mbar_init(smem_u32(&ctl.raw_empty[u]), kPer * kConverterWarps); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctl.acc_full[b]), 1); mbar_init(smem_u32(&ctl.acc_empty[b]), 4 * kCtas); }
    mbar_init(smem_u32(&ctl.drain), 1);
    ctl.abort_flag = 0;
    ctl.flip = Pair<T>::kFlip;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (role == ROLE_ALLOC) { if constexpr (kPair) tmem_alloc2(smem_u32(&ctl.tmem), kColumns); else tmem_alloc(smem_u32(&ctl.tmem), kColumns); }
  tc_fence_before();
  __syncthreads();
  if (kPair) cluster_sync_all();                                   // both CTAs' barriers exist before either touches the other's
  tc_fence_after();
  const uint32_t tmem = ctl.tmem;
  hq_pdl_entry();

  if (role == ROLE_FETCH) {
    if (elect_one()) {
      int s = 0, u = 0;
      uint32_t phase = 0, u_phase = 0, issued = 0, u_issued = 0;
      bool ok = true;
      // the quantized operand of stages `st` and on
      auto fetch_unit = [&](int i0, int st) {
        if (!mbar_wait(smem_u32(&ctl.raw_empty[u]), u_phase ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER)) return false;
        const uint32_t bar = smem_u32(&ctl.raw_full[u]), dst = raw_ring + u * Unit<KIND, NT>::kBytes;
        mbar_expect_tx(bar, Unit<KIND, NT>::kBytes);
        if (KIND == PRODUCT_FORWARD) tma_load_2d(dst, &map_q, bar, st * (kStep / 2), i0);
        else tma_load_2d(dst, &map_q, bar, KIND == PRODUCT_DGRAD ? i0 >> 1 : i0, st * kStep);
        u_issued |= 1u << u;
        if (++u == kUnits) { u = 0; u_phase ^= 1; }
        return true;
      };
      for (int tile = first; tile < a.tiles && ok; tile += stride) {
        const int i0 = i_of(tile), j0 = j_of(tile) + in_pair * kColumnsHere;
        for (int st = begin; st < end; ++st) {
          if ((st - begin) % kPer == 0 && !fetch_unit(i0, st)) { ok = false; break; }
          if (!mbar_wait(smem_u32(&ctl.empty[s]), phase ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER)) { ok = false; break; }
          const uint32_t bar = leading(ctl.full[s]), dst = base + s * kStageBytes + kTileABytes;
          if (in_pair == 0) mbar_expect_tx(smem_u32(&ctl.full[s]), kCtas * kBBytes);
#pragma unroll
          for (int b = 0; b < kBoxes; ++b) {
            const int x = KIND == PRODUCT_WGRAD ? j0 + b * 64 : st * kStep, y = KIND == PRODUCT_WGRAD ? st * kStep : j0;
            if constexpr (kPair) tma_load_2d_pair(dst + b * (64 * kStep * 2), &map_b, bar, x, y);
            else tma_load_2d(dst + b * (64 * kStep * 2), &map_b, bar, x, y);
          }
          issued |= 1u << s;
          if (++s == kStages) { s = 0; phase ^= 1; }
        }
      }
      // The last stages' MMAs are done before this CTA may end: they read its memory, and in a pair the other CTA signals its barriers.
      for (int k = 0; k < kStages && ok; ++k)
        if (issued >> k & 1) ok = mbar_wait(smem_u32(&ctl.empty[k]), k < s ? phase : phase ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_DRAIN);
      if (!ok) {                                                 // given up: let the copies in flight land before the memory goes
        // (those of the odd CTA of a pair are counted on the leading one, which waits for them before the closing cluster barrier)
        for (int k = 0; k < kStages && in_pair == 0; ++k)
          if (issued >> k & 1) drain_wait(smem_u32(&ctl.full[k]), k < s ? phase : phase ^ 1, a.status);   // (or its budget: a converter may be missing)
        for (int k = 0; k < kUnits; ++k)
          if (u_issued >> k & 1) drain_wait(smem_u32(&ctl.raw_full[k]), k < u ? u_phase : u_phase ^ 1, a.status);
      }
    }
  } else if (role == ROLE_MMA) {
    if (in_pair == 0 && elect_one()) {
      constexpr bool kAMn = KIND != PRODUCT_FORWARD, kBMn = KIND == PRODUCT_WGRAD;
      constexpr uint32_t kType = Pair<T>::kBf16 ? 1u : 0u;
      constexpr uint32_t idesc = (1u << 4) | (kType << 7) | (kType << 10) | ((uint32_t)kAMn << 15) | ((uint32_t)kBMn << 16) |
                                 ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(kCtas * kTileC >> 4) << 24);
      // completion of the MMAs issued so far, signalled in this CTA and its partner (addresses of the first barrier of a row)
      struct Both { uint32_t here, there; };
      auto both = [&](unsigned long long& bar) {
        if constexpr (kPair) return Both{in_cta(smem_u32(&bar), leader), in_cta(smem_u32(&bar), leader + 1)};
        else return Both{smem_u32(&bar), 0u};
      };
      auto commit = [&](const Both& bar, int k) {
        if constexpr (kPair) { mma_commit_2cta(bar.here + 8 * k); mma_commit_2cta(bar.there + 8 * k); } else mma_commit(bar.here + 8 * k);
      };
      const Both empty = both(ctl.empty[0]), acc_full = both(ctl.acc_full[0]);
      const uint32_t full = smem_u32(&ctl.full[0]);
      int s = 0; uint32_t phase = 0;
      int buf = 0; uint32_t acc_phase = 0;
      bool ok = true;
      const uint64_t desc_a = tile_desc(base, kAMn), desc_b = tile_desc(base + kTileABytes, kBMn);    // (addresses fit: no carry)
      // (the next stage's barrier is looked at while the present stage's MMAs are issued: the look alone takes some 200 cycles)
      bool ready = false;
      for (int tile = first; tile < a.tiles && ok; tile += stride) {
        if (!mbar_wait(smem_u32(&ctl.acc_empty[buf]), acc_phase ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_MMA)) { ok = false; break; }
        tc_fence_after();
        for (int st = begin; st < end; ++st) {
          if (!ready && !mbar_wait(full + 8 * s, phase, &ctl, a.status, HQ_DEV_TIMEOUT_MMA)) { ok = false; break; }
          tc_fence_after();
          const uint64_t da = desc_a + (uint32_t)(s * (kStageBytes >> 4)), db = desc_b + (uint32_t)(s * (kStageBytes >> 4));
          const int done = s;
          if (++s == kStages) { s = 0; phase ^= 1; }
          ready = mbar_try_wait_for(full + 8 * s, phase, 0);
#pragma unroll
          for (int k = 0; k < kStep / 16; ++k) {
            const uint64_t ak = da + k * (kAMn ? (16 * 128) >> 4 : 2), bk = db + k * (kBMn ? (16 * 128) >> 4 : 2);
            const uint32_t more = (st > begin || k > 0) ? 1u : 0u;
            if constexpr (kPair) mma_f16_pair(tmem + buf * NT, ak, bk, idesc, more); else mma_f16(tmem + buf * NT, ak, bk, idesc, more);
          }
          if (st + 1 == end) commit(acc_full, buf);
          commit(empty, done);
        }
        if (!ok) break;
        if (++buf == 2) { buf = 0; acc_phase ^= 1; }
      }
      if (!ok) {
        if constexpr (kPair) mma_commit_2cta(in_cta(smem_u32(&ctl.drain), leader)); else mma_commit(smem_u32(&ctl.drain));
        drain_wait(smem_u32(&ctl.drain), 0, a.status);
      }
    }
  } else if (role == ROLE_CONVERT && converter_number(warp, !kPair) < kGroups * kConverterWarps) {
    const int number = converter_number(warp, !kPair);
    const int group = number / kConverterWarps, member = number % kConverterWarps;
    // (two warps: the halves of the lanes, or 64 rows each; four: halves and 32 rows, or 32 rows)
    const int row0 = (KIND == PRODUCT_FORWARD ? member * 32 * kRowsPerThread : kRowsPerThread == 2 ? 0 : (member & 1) * 32) + lane;
    const int half = KIND == PRODUCT_FORWARD ? 0 : kRowsPerThread == 2 ? member : member >> 1;
    const uint32_t flip = ctl.flip;
    // Stages are numbered through the CTA's tiles, a tile filled up to whole units; the group takes every kGroups-th.
    const int steps = end - begin, padded = (steps + kPer - 1) / kPer * kPer;
    int tile = first, st = group;                                // a tile, and a stage of it
    unsigned before = 0, before_padded = 0;                      // stages in the tiles before
    auto settle = [&]() {
      bool moved = false;
      while (st >= padded && tile < a.tiles) { st -= padded; tile += stride; before += steps; before_padded += padded; moved = true; }
      return moved;
    };
    Scales<KIND, T, kRowsPerThread> scales(p, a.group_mul, row0, half, kGroups);
    settle();
    scales.enter(i_of(tile), tile < a.tiles, begin + st);
    float scale[kRowsPerThread][2];
    scales.load(kGroups, scale);
    while (tile < a.tiles) {
      const unsigned n = before + st, v = before_padded + st, unit_no = v / kPer;
      const bool real = st < steps;
      const int u = unit_no % kUnits, s = (int)(n % kStages);
      const uint32_t raw = raw_ring + u * Unit<KIND, NT>::kBytes, to = base + s * kStageBytes;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.raw_full[u]), (unit_no / kUnits) & 1, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER))) break;
      if (real) {
        // the first row's values are made before the stage they go to is free
        uint32_t value[8][4];
        convert_row<KIND, T, Unit<KIND, NT>::kRowBytes>(raw, (int)(v % kPer), scale[0], row0, half, flip, value);
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.empty[s]), ((n / kStages) & 1) ^ 1, &ctl, a.status, HQ_DEV_TIMEOUT_PRODUCER))) break;
        store_row(to, row0, half, value);
        if (kRowsPerThread == 2) {
          convert_row<KIND, T, Unit<KIND, NT>::kRowBytes>(raw, (int)(v % kPer), scale[kRowsPerThread - 1], row0 + 32, half, flip, value);
          store_row(to, row0 + 32, half, value);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) { if constexpr (kPair) arrive_leading(leading(ctl.full[s])); else mbar_arrive(smem_u32(&ctl.full[s])); }
      }
      if (lane == 0) mbar_arrive(smem_u32(&ctl.raw_empty[u]));
      st += kGroups;
      if (settle()) scales.enter(i_of(tile), tile < a.tiles, begin + st);
      scales.load(kGroups, scale);                               // (behind the fence, which waits for loads too)
    }
  } else if (role == ROLE_DRAIN) {
    const int quad = warp & 3;
    int buf = 0; uint32_t acc_phase = 0;
    for (int tile = first; tile < a.tiles; tile += stride) {
      const int i = i_of(tile) + quad * 32 + lane, j0 = j_of(tile);
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
      if (lane == 0) { if constexpr (kPair) arrive_leading(leading(ctl.acc_empty[buf])); else mbar_arrive(smem_u32(&ctl.acc_empty[buf])); }
      if (++buf == 2) { buf = 0; acc_phase ^= 1; }
    }
  }
  __syncwarp();
  if (a.splits > 1) {
    cluster_sync_all();                                          // every part is written
    const int i0 = i_of(first), j0 = j_of(first);
    const int cols = NT / a.splits;                              // columns this CTA adds up (splits divides NT)
    const uint32_t mine = base + rank * cols * kTileC * 4;
    const bool whole = p.out_stride % 4 == 0;                    // four values of a row leave in one store
    for (int e = threadIdx.x; e < cols * (kTileC / 4); e += kThreads) {
      const int i = i0 + e % (kTileC / 4) * 4, j = j0 + rank * cols + e / (kTileC / 4);
      if (i >= p.i || j >= p.j) continue;
      float4 part[4], sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k0 = 0; k0 < a.splits; k0 += 4) {                 // (a remote load takes long: four on their way)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k0 + k < a.splits)
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(part[k].x), "=f"(part[k].y), "=f"(part[k].z), "=f"(part[k].w)
                         : "r"(in_cta(mine + e * 16, (k0 + k) * kCtas + in_pair)));
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k0 + k < a.splits) { sum.x += part[k].x; sum.y += part[k].y; sum.z += part[k].z; sum.w += part[k].w; }
      }
      float v[4] = {sum.x, sum.y, sum.z, sum.w};
      T* out = (T*)p.out + (long long)j * p.out_stride + i;
#pragma unroll
      for (int k = 0; k < 4; ++k) if (p.bias && i + k < p.i) v[k] += hq_to_float(((const T*)p.bias)[i + k]);
      if (whole && i + 4 <= p.i) {
        *(uint2*)out = make_uint2(Pair<T>::pack(v[0], v[1]), Pair<T>::pack(v[2], v[3]));
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) if (i + k < p.i) out[k] = hq_from_float<T>(v[k]);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  // The CTAs of a cluster leave together: nobody reads a part any more, the leading CTA has seen its MMAs complete, its partner has
  // sent its last arrival.
  if (clustered) cluster_sync_all();
  if (role == ROLE_ALLOC) { tc_fence_after(); if constexpr (kPair) tmem_dealloc2(tmem, kColumns); else tmem_dealloc(tmem, kColumns); }
}

// ---------------------------------------------------------------- host side ------------------
bool encode_b_map(CUtensorMap* map, int type, const ProductArgs& a, ProductKind kind, int nt) {
  const long long cols = kind == PRODUCT_WGRAD ? a.j : a.r, rows = kind == PRODUCT_WGRAD ? a.r : a.j;
  const long long stride = rows == 1 ? (cols + 7) / 8 * 8 : a.b_stride;      // (the stride of a single row means nothing)
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {kStep, (cuuint32_t)(kind == PRODUCT_WGRAD ? kStep : nt == 256 ? 128 : nt)};
  const cuuint32_t estr[2] = {1, 1};
  return g_encode_tiled(map, type == HQ_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.b), dims,
                        strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KIND, class T, int NT>
cudaError_t launch(const CUtensorMap* map, const TcArgs& a, int grid, int device, cudaStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const cudaError_t ready = hq_allow_shared(done, device, product_tc_kernel<KIND, T, NT>, Shape<KIND, NT>::kSharedBytes);
  if (ready != cudaSuccess) return ready;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)(a.splits * Shape<KIND, NT>::kCtas); attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = Shape<KIND, NT>::kSharedBytes; cfg.stream = s;
  cfg.attrs = attr; cfg.numAttrs = a.splits * Shape<KIND, NT>::kCtas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, product_tc_kernel<KIND, T, NT>, map[0], map[1], a);
}
template <int KIND, class T>
cudaError_t launch_width(int nt, const CUtensorMap* map, const TcArgs& a, int grid, int device, cudaStream_t s) {
  switch (nt) {
    case 32: return launch<KIND, T, 32>(map, a, grid, device, s);
    case 64: return launch<KIND, T, 64>(map, a, grid, device, s);
    case 128: return launch<KIND, T, 128>(map, a, grid, device, s);
    default: return launch<KIND, T, 256>(map, a, grid, device, s);
  }
}
template <class T>
cudaError_t launch_kind(ProductKind kind, int nt, const CUtensorMap* map, const TcArgs& a, int grid, int device, cudaStream_t s) {
  return kind == PRODUCT_FORWARD ? launch_width<PRODUCT_FORWARD, T>(nt, map, a, grid, device, s)
       : kind == PRODUCT_DGRAD ? launch_width<PRODUCT_DGRAD, T>(nt, map, a, grid, device, s) : launch_width<PRODUCT_WGRAD, T>(nt, map, a, grid, device, s);
}

}  // namespace

// From hq_create.
bool hq_product_tc_init() { return load_driver_entry_points(); }

bool hq_product_tc_supported(ProductKind kind, const ProductArgs& a) {
  if (a.r < 1) return false;
  const int b_rows = kind == PRODUCT_WGRAD ? a.r : a.j;
  if (a.b_stride % 8 && b_rows > 1) return false;                          // rows of B start on 16 bytes
  return kind == PRODUCT_WGRAD ? a.q_cols % 16 == 0 : a.q_cols % 32 == 0;  // and so do those of the quantized operand
}

namespace {

template <int KIND, int NT>
void fill_rings(hq_product_plan* plan) {
  using S = Shape<KIND, NT>;
  plan->stages = S::kStages; plan->groups = S::kGroups; plan->units = S::kUnits; plan->unit_stages = S::kPer;
}
template <int KIND>
void fill_rings(int nt, hq_product_plan* plan) {
  nt == 32 ? fill_rings<KIND, 32>(plan) : nt == 64 ? fill_rings<KIND, 64>(plan) : nt == 128 ? fill_rings<KIND, 128>(plan) : fill_rings<KIND, 256>(plan);
}

// Columns per tile and CTAs (or pairs) per tile: what is through first, by the cycles that a stage, a tile and the joining of parts
// take (a stage, counted in the kernel: 650 with 256 columns on a pair, about 600 with 64, 32 and with saved activations).
// Returns the columns, 0 for more tiles than can be counted.
int plan_tiles(const ProductArgs& p, int sm_count, TcArgs& a) {
  a.steps = (p.r + kStep - 1) / kStep;
  int nt = 0;
  long long best = 0;
  for (const int width : {32, 64, 128, 256}) {
    const int ctas = width == 256 ? 2 : 1, stage = width == 256 ? 650 : width == 128 ? 620 : 600;
    const long long i_tiles = (p.i + ctas * kTileC - 1) / (ctas * kTileC), tiles = i_tiles * ((p.j + width - 1) / width);
    if (tiles > 0x3fffffff) continue;
    for (int splits = 1; splits * ctas <= 8; splits *= 2) {
      const int split_steps = (a.steps + splits - 1) / splits;
      if (splits > 1 && ((splits - 1) * split_steps >= a.steps || split_steps < 4)) break;
      const long long at_once = sm_count / (ctas * splits);
      if (at_once < 1) break;
      const long long rounds = (tiles + at_once - 1) / at_once;
      if (splits > 1 && rounds > 1) break;
      const long long cost = rounds * ((long long)split_steps * stage + 1500) + (splits > 1 ? 3000 + 10 * width : 0);
      if (best && cost >= best) continue;
      best = cost; nt = width;
      a.i_tiles = (int)i_tiles; a.tiles = (int)tiles; a.splits = splits; a.split_steps = split_steps;
    }
  }
  return nt;
}

}  // namespace

bool hq_plan_product_tc(ProductKind kind, const ProductArgs& p, int sm_count, hq_product_plan* plan) {
  if (!hq_product_tc_supported(kind, p)) return false;
  TcArgs a{};
  const int nt = plan_tiles(p, sm_count, a);
  if (nt == 0) return false;
  kind == PRODUCT_FORWARD ? fill_rings<PRODUCT_FORWARD>(nt, plan) : kind == PRODUCT_DGRAD ? fill_rings<PRODUCT_DGRAD>(nt, plan) : fill_rings<PRODUCT_WGRAD>(nt, plan);
  const int at_once = sm_count / ((nt == 256 ? 2 : 1) * a.splits);
  plan->columns = nt; plan->outputs = (nt == 256 ? 2 : 1) * kTileC; plan->splits = a.splits; plan->steps = a.split_steps;
  plan->rounds = (a.tiles + at_once - 1) / at_once;
  return true;
}

hq_status hq_launch_product_tc(hq_handle* h, ProductKind kind, int type, const ProductArgs& p, cudaStream_t s) {
  TcArgs a{};
  const int nt = plan_tiles(p, h->sm_count, a);
  if (nt == 0) return HQ_ERR_UNSUPPORTED;
  a.p = p;
  a.status = h->dev_status;
  const int ctas = nt == 256 ? 2 : 1, at_once = h->sm_count / ctas;
  const int grid = (a.splits > 1 ? a.tiles * a.splits : a.tiles < at_once ? a.tiles : at_once) * ctas;
  // k / group by a multiply-high, exact while (k / 32) (group / 32) < 2^31
  if (kind == PRODUCT_FORWARD && p.r <= (1 << 20)) {
    const unsigned group32 = (unsigned)(p.group >= p.r ? 1 << 20 : p.group) / 32;
    a.group_mul = (uint32_t)(((1ull << 31) + group32 - 1) / group32);
  }
  CUtensorMap map[2];
  const bool bytes = kind == PRODUCT_WGRAD;
  const int unit_row = kind == PRODUCT_WGRAD ? Unit<PRODUCT_WGRAD, 32>::kRowBytes : kind == PRODUCT_DGRAD ? Unit<PRODUCT_DGRAD, 32>::kRowBytes
                     : nt >= 128 ? Unit<PRODUCT_FORWARD, 128>::kRowBytes : Unit<PRODUCT_FORWARD, 32>::kRowBytes;
  const int unit_rows = kind == PRODUCT_FORWARD ? kTileC : kStep;
  if (!encode_rows_map(&map[0], p.q, kind == PRODUCT_FORWARD ? p.i : p.r, bytes ? p.q_cols : p.q_cols >> 1, unit_row, unit_rows, swizzle_for(unit_row)) ||
      !encode_b_map(&map[1], type, p, kind, nt)) return HQ_ERR_CUDA;
  const cudaError_t e = type == HQ_F16 ? launch_kind<__half>(kind, nt, map, a, grid, h->device, s) : launch_kind<__nv_bfloat16>(kind, nt, map, a, grid, h->device, s);
  return e == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
