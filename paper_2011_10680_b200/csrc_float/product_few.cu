// hq_linear_w4 for up to 16 rows: the matrix-vector case, one token of each of a few sequences.  The packed weights are read once
// and that is the bound; everything else has to hide behind their stream.
//   - A warp takes 16 outputs x 128 inputs at a time: two 16-byte loads per thread, held in registers four steps ahead.  The
//     integers go through the 16-bit matrix instruction (mma.m16n8k16) as they are - offset by 8, which is taken off exactly - so
//     that a weight costs about 1.4 instructions whatever the number of rows; the sum over a group is scaled in 32 bits.
//   - The order of the inputs inside a step is that in which the nibbles come out of a word (0 4 1 5 2 6 3 7 of every eight, a
//     thread's 32 inputs being its own), and x is stored in shared memory in that order once per CTA.
//   - Groups shorter than 128: the eight columns of the instruction carry a row's inputs group by group, zeros elsewhere, so that
//     every group has a sum of its own ("parts"; 64: two columns per row, 32: four).
//   - The warps of a CTA split the inputs and add up in shared memory in a fixed order; few outputs: the CTAs of a cluster do too.
#include "../csrc/tc_common.cuh"
#include "float_internal.cuh"

namespace {

constexpr int kThreads = 256, kWarps = 8, kRows = 16, kStep = 128, kAhead = 4;
constexpr int kMaxShared = 200 * 1024;

struct FewArgs {
  ProductArgs p;
  int row_tiles;           // CTA tiles along the outputs
  int splits, range;       // CTAs per tile; inputs of each (a multiple of kStep)
  int along;               // warps along the inputs: 1, 2, 4 or 8; the others take more outputs
  int parts;               // columns per row: 1, 2 or 4
  int pitch;               // bytes of a row of x in shared memory
  int red_bytes;           // one of the two buffers of partial sums
};

template <class T> struct Few;
template <> struct Few<__nv_bfloat16> {
  using Two = __nv_bfloat162;
  static constexpr uint32_t kFlip = 0x43084308u, kOffset = 0x43084308u;        // 128 + 8, and 136
  static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
template <> struct Few<__half> {
  using Two = __half2;
  static constexpr uint32_t kFlip = 0x64086408u, kOffset = 0x64086408u;        // 1024 + 8, and 1032
  static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};

__device__ __forceinline__ uint4 load_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Eight 4-bit integers of a word as pairs (0 4) (1 5) (2 6) (3 7), exact.
template <class T>
__device__ __forceinline__ void integers(uint32_t w, uint32_t (&out)[4]) {
  using Two = typename Few<T>::Two;
  const uint32_t offset = Few<T>::kOffset;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = ((w >> (4 * i)) & 0x000f000fu) ^ Few<T>::kFlip;
    const Two v = __hsub2(*(const Two*)&m, *(const Two*)&offset);
    out[i] = *(const uint32_t*)&v;
  }
}

// What a thread has in flight for one step: the inputs t*32 .. t*32+31 of two outputs, and their scales (of the columns 2t, 2t+1).
template <class T> struct Unit { uint4 w[2]; T s[4]; };

template <class T, int NB>
__global__ void __launch_bounds__(kThreads, NB <= 2 ? 2 : 1) product_few_kernel(const FewArgs a) {
  extern __shared__ __align__(16) uint8_t shared[];
  const ProductArgs& p = a.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = a.splits > 1 ? (int)cluster_ctarank() : 0;
  const int kw = warp % a.along, rw = warp / a.along, wr = kWarps / a.along;
  const int k_begin = rank * a.range, k_end = min(p.r, k_begin + a.range);
  const int steps = (k_end - k_begin + kStep - 1) / kStep, my_steps = (steps + a.along - 1) / a.along;
  const int tile0 = blockIdx.x / a.splits, tile_stride = gridDim.x / a.splits;
  const long long pitch_q = p.q_cols >> 1;
  // scales: column c is part c % parts of its row of x
  const int part0 = (2 * t) % a.parts, part1 = (2 * t + 1) % a.parts, part_len = kStep / a.parts;
  hq_pdl_entry();

  int load_tile = tile0, load_step = 0;
  auto load = [&](Unit<T>& u) {
    const int k = k_begin + (load_step * a.along + kw) * kStep;
    const int row = (load_tile * wr + rw) * kRows + g;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u.w[h] = make_uint4(0, 0, 0, 0);
      u.s[2 * h] = u.s[2 * h + 1] = hq_from_float<T>(0.f);
      const int r = row + 8 * h;
      if (load_tile < a.row_tiles && r < p.i && k < k_end) {
        if (k + t * 32 < k_end) u.w[h] = load_stream((const uint8_t*)p.q + r * pitch_q + ((k + t * 32) >> 1));
        const T* s = (const T*)p.scale + (long long)r * p.groups;
        if (a.parts == 1) {
          u.s[2 * h] = u.s[2 * h + 1] = s[k / p.group];
        } else {
          if (k + part0 * part_len < k_end) u.s[2 * h] = s[(k + part0 * part_len) / p.group];
          if (k + part1 * part_len < k_end) u.s[2 * h + 1] = s[(k + part1 * part_len) / p.group];
        }
      }
    }
    if (++load_step == my_steps) { load_step = 0; load_tile += tile_stride; }
  };
  Unit<T> ring[kAhead];
#pragma unroll
  for (int d = 0; d < kAhead; ++d) load(ring[d]);

  // x in the order of the nibbles: for every step 16-byte pieces [word of a thread's four][thread of four]
  const int pieces = steps * (kStep / 8);
  for (int e = threadIdx.x; e < pieces * p.j; e += kThreads) {
    const int row = e / pieces, c = e - row * pieces, k = k_begin + c * 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (k < k_end) v = *(const uint4*)((const T*)p.b + row * p.b_stride + k);
    uint4 o;
    o.x = __byte_perm(v.x, v.z, 0x5410); o.y = __byte_perm(v.x, v.z, 0x7632);
    o.z = __byte_perm(v.y, v.w, 0x5410); o.w = __byte_perm(v.y, v.w, 0x7632);
    *(uint4*)(shared + row * a.pitch + (c >> 4) * 256 + (c & 3) * 64 + ((c >> 2) & 3) * 16) = o;
  }
  __syncthreads();

  // where this thread's columns find their inputs: column g of every eight; its part has to be that of the thread's inputs
  const uint8_t* x_at[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int col = nb * 8 + g, row = col / a.parts;
    x_at[nb] = (row < p.j && col % a.parts == t * a.parts / 4) ? shared + row * a.pitch + t * 16 : nullptr;
  }
  float* const red = (float*)(shared + ((p.j * a.pitch + 127) & ~127));
  float total[NB][4] = {};
  int step = 0, tile = tile0, parity = 0;
  const int units = (tile0 < a.row_tiles ? (a.row_tiles - tile0 + tile_stride - 1) / tile_stride : 0) * my_steps;
  for (int n = 0; n < units; n += kAhead) {
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {
      if (n + d < units) {
        Unit<T>& u = ring[d];
        const int at = (step * a.along + kw) * 256;
        float acc[NB][4] = {};
        if (step * a.along + kw < steps) {
          const uint32_t* w0 = (const uint32_t*)&u.w[0];
          const uint32_t* w1 = (const uint32_t*)&u.w[1];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t lo[4], hi[4];
            integers<T>(w0[i], lo);
            integers<T>(w1[i], hi);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint4 b = x_at[nb] ? *(const uint4*)(x_at[nb] + at + i * 64) : make_uint4(0, 0, 0, 0);
              Few<T>::mma(acc[nb], lo[0], hi[0], lo[1], hi[1], b.x, b.y);
              Few<T>::mma(acc[nb], lo[2], hi[2], lo[3], hi[3], b.z, b.w);
            }
          }
        }
        float s[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] = hq_to_float(u.s[k]);
        if (step * a.along + kw < steps) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int k = 0; k < 4; ++k) total[nb][k] = fmaf(s[k], acc[nb][k], total[nb][k]);
        }
        load(u);
        if (++step == my_steps) {                                // the tile's inputs are through: add up the warps' parts
          step = 0;
          float* mine = (float*)((uint8_t*)red + parity * a.red_bytes) + warp * (kRows * 8 * NB);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              mine[(nb * 8 + 2 * t + (k & 1)) * kRows + g + (k >> 1) * 8] = total[nb][k];
              total[nb][k] = 0.f;
            }
          }
          if (a.splits > 1) cluster_sync_all(); else __syncthreads();
          const float* parts = (const float*)((uint8_t*)red + parity * a.red_bytes);
          const int outputs = kRows * wr * p.j;
          for (int e = threadIdx.x + rank * kThreads; e < outputs; e += kThreads * a.splits) {
            const int r16 = e % kRows, w = e / kRows % wr, row = e / (kRows * wr);
            const int i = (tile * wr + w) * kRows + r16;
            if (i < p.i) {
              float sum = 0.f;
              for (int c = 0; c < a.splits; ++c) {
                for (int k = 0; k < a.along; ++k) {
                  for (int q = 0; q < a.parts; ++q) {
                    const float* from = parts + (w * a.along + k) * (kRows * 8 * NB) + (row * a.parts + q) * kRows + r16;
                    float v;
                    if (a.splits > 1) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(in_cta(smem_u32(from), c)));
                    else v = *from;
                    sum += v;
                  }
                }
              }
              if (p.bias) sum += hq_to_float(((const T*)p.bias)[i]);
              ((T*)p.out)[row * p.out_stride + i] = hq_from_float<T>(sum);
            }
          }
          parity ^= 1;                                           // (the other buffer's readers are behind the barrier above)
          tile += tile_stride;
        }
      }
    }
  }
  if (a.splits > 1) cluster_sync_all();                          // nobody reads this CTA's parts any more
}

int columns_eights(int j, int parts) { const int n = (j * parts + 7) / 8; return n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : 8; }

// Parts of a 128-input step that can have scales of their own.
int parts_of(const ProductArgs& a) { return a.group >= a.r || a.group % 128 == 0 ? 1 : a.group % 64 == 0 ? 2 : 4; }

template <class T, int NB>
cudaError_t launch(const FewArgs& a, int grid, int shared, cudaStream_t s) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)a.splits; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = (size_t)shared; cfg.stream = s;
  cfg.attrs = attr; cfg.numAttrs = a.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, product_few_kernel<T, NB>, a);
}
template <class T>
cudaError_t launch_type(int nb, const FewArgs& a, int grid, int shared, cudaStream_t s) {
  return nb == 1 ? launch<T, 1>(a, grid, shared, s) : nb == 2 ? launch<T, 2>(a, grid, shared, s)
       : nb == 4 ? launch<T, 4>(a, grid, shared, s) : launch<T, 8>(a, grid, shared, s);
}

template <class T, int NB>
bool allow_shared() { return cudaFuncSetAttribute(product_few_kernel<T, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxShared) == cudaSuccess; }
template <class T>
bool allow_type() { return allow_shared<T, 1>() && allow_shared<T, 2>() && allow_shared<T, 4>() && allow_shared<T, 8>(); }

// The launch of a shape: cluster size, warps along the inputs, shared memory; false when x does not fit the CTAs of a cluster.
bool plan(const ProductArgs& p, int sm_count, FewArgs& a, int& shared) {
  const int parts = parts_of(p), nb = columns_eights(p.j, parts);
  const int steps = (p.r + kStep - 1) / kStep, tiles16 = (p.i + kRows - 1) / kRows;
  bool found = false;
  for (int splits = 1; splits <= 8; splits *= 2) {
    const int per = (steps + splits - 1) / splits;
    if (splits > 1 && (splits - 1) * per >= steps) break;              // a CTA without inputs
    const int along = per >= 8 ? 8 : per >= 4 ? 4 : per >= 2 ? 2 : 1, wr = kWarps / along;
    const long long pitch = (long long)per * kStep * 2 + 64;           // 64 modulo 128: eight lanes' pieces lie on different banks
    const int red_bytes = kWarps * kRows * 8 * nb * (int)sizeof(float);
    const long long need = ((p.j * pitch + 127) & ~127ll) + 2 * red_bytes;
    if (need > kMaxShared) continue;
    a.p = p;
    a.parts = parts; a.splits = splits; a.range = per * kStep; a.along = along; a.pitch = (int)pitch; a.red_bytes = red_bytes;
    a.row_tiles = (tiles16 + wr - 1) / wr;
    shared = (int)need;
    found = true;
    // more CTAs per tile only while the GPU is not filled and every warp keeps two steps
    if (a.row_tiles * splits * 2 > sm_count || per < 32) break;
  }
  return found;
}

}  // namespace

bool hq_product_few_init() { return allow_type<__half>() && allow_type<__nv_bfloat16>(); }

bool hq_product_few_supported(const ProductArgs& p) {
  if (p.j > 16 || p.q_cols % 32 || (p.b_stride % 8 && p.j > 1)) return false;
  FewArgs a{};
  int shared;
  return plan(p, 148, a, shared);
}

hq_status hq_launch_product_few(hq_handle* h, int type, const ProductArgs& p, cudaStream_t s) {
  FewArgs a{};
  int shared = 0;
  if (!plan(p, h->sm_count, a, shared)) return HQ_ERR_UNSUPPORTED;
  const int nb = columns_eights(p.j, a.parts);
  const int resident = shared <= 100 * 1024 && nb <= 2 ? 2 : 1;
  const int room = h->sm_count * resident;
  const int grid = a.splits > 1 ? a.row_tiles * a.splits : a.row_tiles < room ? a.row_tiles : room;
  const cudaError_t e = type == HQ_F16 ? launch_type<__half>(nb, a, grid, shared, s) : launch_type<__nv_bfloat16>(nb, a, grid, shared, s);
  return e == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
