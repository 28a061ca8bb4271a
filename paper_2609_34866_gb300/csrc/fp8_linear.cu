// Product in 8-bit floating point (e4m3) with a scale for every 128 of K, on the tensor cores of sm_103a:
//
//   y[m, n] = sum_b sx[m, b] sw[n / block_rows, b] sum_{k in block b} qx[m, k] qw[n, k]
//
// A block's sum is an accumulator of its own: four products of K = 32, then it is read out of tensor memory, multiplied by its
// scales and added to running sums in registers, while the next block's products fill another accumulator. The output
// channels are the accumulator's 128 lanes and the tokens its columns, so that one layout serves one token and thousands: a
// lane's channel has its own scale (block_rows = 1), a column's token another, which every lane reads from shared memory.
//
// Roles of a block: a warp that issues the copies (TMA, weights and token codes in one ring), a warp that issues the
// products, eight warps that read out, scale and add up. Many tiles: persistent blocks. Few tiles: one a cluster, whose
// blocks take ranges of K and add their sums through shared memory in a fixed order.
#include <cudaTypedefs.h>

#include <algorithm>

#include "common.cuh"
#include "per_device.h"
#include "serve.h"
#include "tc.cuh"

namespace jab {
namespace {

constexpr int TM = 128, BK = 128;  // output channels of a tile; K of a stage, of a scale
constexpr int kMaxRanges = 8;      // K ranges of a tile (the portable cluster size)

struct F8Params {
  int64_t M, Mp, ldy;
  int N, stages, tiles_n, tiles_m, ranges, y_type;
  FastDiv by_n;
  const float *sx, *sw;  // sx [stages, Mp]
  void* y;
  int* status;
};

template <int NTOK>
struct Cfg {
  static constexpr int W_STAGE = TM * BK, X_STAGE = NTOK * BK, STAGE = W_STAGE + X_STAGE;
  static constexpr int ST = NTOK == 256 ? 4 : NTOK == 128 ? 6 : NTOK == 64 ? 8 : NTOK == 32 ? 9 : 11;
  static constexpr int D_COLS = NTOK < 32 ? 32 : NTOK, DST = 512 / D_COLS < 8 ? 512 / D_COLS : 8;  // accumulators
  static constexpr int HALF = NTOK / 2;                                                           // columns of a warp
  static constexpr int THREADS = 320;                                                             // (200 registers each: 128 of them sums)
  static constexpr bool SPLIT = NTOK <= 128;
  static constexpr int SMEM = ST * STAGE + 1024 + 1024 + 8 * 2 * HALF * 4;
  static_assert(!SPLIT || NTOK * TM * 4 <= ST * STAGE, "a tile's sums take the stages' place");
};

struct Bars {
  uint64_t full[11], empty[11], tfull[8], tempty[8], joined, drain;
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(Bars) <= 1024, "barrier block");

// Waits for a phase while leaving: bounded, whatever the abort flag says.
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity) {
  const uint64_t t0 = tc::globaltimer();
  while (!tc::mbar_test(bar, parity))
    if (tc::globaltimer() - t0 > tc::kWaitLimitNs) break;
}

__device__ __forceinline__ float load_cluster(uint32_t at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// N consecutive columns of 32 lanes.
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[32]) { tc::tmem_ld32(taddr, r); }
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                 "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}

__device__ __forceinline__ void put(void* y, int64_t at, float v, int type) {
  if (type == JAB_FP32) static_cast<float*>(y)[at] = v;
  else if (type == JAB_FP16) static_cast<half_t*>(y)[at] = __float2half_rn(v);
  else static_cast<bf16_t*>(y)[at] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ uint32_t pair_of(float a, float b, int type) {
  if (type == JAB_FP16) return tc::pack_half2(a, b);
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int NTOK, bool ROWS>
__global__ void __launch_bounds__(Cfg<NTOK>::THREADS, 1)
    fp8_linear_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ F8Params p) {
  using C = Cfg<NTOK>;
  constexpr int ST = C::ST, DST = C::DST, HALF = C::HALF;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Bars* bars = reinterpret_cast<Bars*>(smem + ST * C::STAGE);
  float* scales = reinterpret_cast<float*>(smem + ST * C::STAGE + 1024);
  const int warp = tc::warp_index(), lane = threadIdx.x & 31;
  const int ranges = C::SPLIT ? p.ranges : 1;
  // A block's tiles and its stages of each: [st0, st0 + stages)
  const int total = p.tiles_n * p.tiles_m, rank = ranges > 1 ? (int)tc::cluster_ctarank() : 0;
  const int unit0 = ranges > 1 ? blockIdx.x / ranges : blockIdx.x, step = ranges > 1 ? total : gridDim.x;
  const int st0 = p.stages * rank / ranges, stages = p.stages * (rank + 1) / ranges - st0;
  volatile int* abort = &bars->abort;
  auto load_w = [&](int s, int kb, int nt) {  // (past the end of K: zeros)
    tc::mbar_expect_tx(&bars->full[s], C::STAGE);
    tc::tma_load_2d(smem + s * C::STAGE, &tmW, &bars->full[s], (st0 + kb) * BK, nt * TM);
  };
  auto load_x = [&](int s, int kb, int mt) {
    tc::tma_load_2d(smem + s * C::STAGE + C::W_STAGE, &tmX, &bars->full[s], (st0 + kb) * BK, mt * NTOK);
  };
  const int early = min(ST, stages);
  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; ++s) {
      tc::mbar_init(&bars->full[s], 1);
      tc::mbar_init(&bars->empty[s], 1);
    }
    for (int d = 0; d < DST; ++d) {
      tc::mbar_init(&bars->tfull[d], 1);
      tc::mbar_init(&bars->tempty[d], 8);
    }
    tc::mbar_init(&bars->joined, 8 * ranges);
    tc::mbar_init(&bars->drain, 1);
    bars->abort = 0;
    tc::fence_mbar_init();
    // (the kernel before, which made the codes of X, did not write the weights, and all before that one is complete)
    const int mt = p.by_n.quot(unit0), nt = unit0 - mt * p.tiles_n;
    for (int i = 0; i < early; ++i) load_w(i, i, nt);
  }
  if (warp == 1) {
    tc::tmem_alloc(&bars->tmem_base, 512);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (ranges > 1) tc::cluster_sync();  // (the others' barriers are there)
  const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
  stream_order();

  if (warp < 2) {
    if (warp == 0) {
      if (tc::elect_one()) {  // ---------------- copies
        int i = 0;
        bool ok = true;
        for (int unit = unit0; unit < total && ok; unit += step) {
          int nt, mt;
          p.by_n.divmod(unit, mt, nt);
          for (int kb = 0; kb < stages; ++kb, ++i) {
            const int s = i % ST;
            if (i >= early) {  // (of the first, the weights are on their way already)
              if (!(ok = tc::mbar_wait(&bars->empty[s], ((i / ST) & 1) ^ 1, abort, p.status))) break;
              load_w(s, kb, nt);
            }
            load_x(s, kb, mt);
          }
        }
        if (*abort)  // every copy issued has landed before shared memory goes to another block
          for (int j = max(0, i - ST); j < i; ++j) drain_wait(&bars->full[j % ST], (j / ST) & 1);
      }
    } else {  // ---------------- products (the whole warp waits, one thread issues)
      constexpr uint32_t IDESC = tc::idesc_e4m3(TM, NTOK);
      int i = 0;
      bool ok = true;
      for (int unit = unit0; unit < total && ok; unit += step) {
        for (int kb = 0; kb < stages && ok; ++kb, ++i) {
          const int s = i % ST, d = i % DST;
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->tempty[d], ((i / DST) & 1) ^ 1, abort, p.status));
          ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(&bars->full[s], (i / ST) & 1, abort, p.status));
          if (ok && tc::elect_one()) {
            tc::fence_after_sync();
            const uint64_t wd = tc::sdesc_kmajor_sw128(tc::smem_u32(smem + s * C::STAGE));
            const uint64_t xd = tc::sdesc_kmajor_sw128(tc::smem_u32(smem + s * C::STAGE + C::W_STAGE));
#pragma unroll
            for (int k = 0; k < BK / 32; ++k)
              tc::umma_f8(tmem + d * C::D_COLS, tc::sdesc_advance(wd, k * 32), tc::sdesc_advance(xd, k * 32), IDESC, k > 0 ? 1u : 0u);
            tc::umma_commit(&bars->empty[s]);
            tc::umma_commit(&bars->tfull[d]);
          }
          __syncwarp();
        }
      }
      if (tc::elect_one()) {
        tc::umma_commit(&bars->drain);
        drain_wait(&bars->drain, 0);
      }
    }
  } else {  // ---------------- scales and sums: a warp has 32 channels and half of the tokens
    constexpr int CHUNK = HALF < 32 ? HALF : 32, PER = HALF < 32 ? 1 : HALF / 32;
    const int quarter = warp & 3, row = quarter * 32 + lane, first = warp < 6 ? 0 : HALF;
    float* mine = scales + (warp - 2) * 2 * HALF;
    // two channels of a token in one store, where they lie together in a word
    const bool words = p.y_type != JAB_FP32 && p.ldy % 2 == 0 && (reinterpret_cast<uintptr_t>(p.y) & 3) == 0;
    auto inside = [&](int64_t last) { return in_bounds(last, (p.M - 1) * p.ldy + p.N, p.status); };
    int i = 0;
    bool ok = true;
    for (int unit = unit0; unit < total && ok; unit += step) {
      int nt, mt;
      p.by_n.divmod(unit, mt, nt);
      const int n = nt * TM + row;
      const int64_t m0 = (int64_t)mt * NTOK + first;
      const int cols = (int)max((int64_t)0, min((int64_t)HALF, p.M - m0));
      const float* sw = p.sw + (ROWS ? (int64_t)min(n, p.N - 1) : (int64_t)nt) * p.stages + st0;
      const float* sx = p.sx + (int64_t)st0 * p.Mp + m0 + lane;
      float next_x[PER], next_w;
      auto fetch = [&](int kb) {  // the scales of a block of K: a lane has every 32nd token's
        if (kb >= stages) return;
        next_w = __ldg(sw + kb);
#pragma unroll
        for (int j = 0; j < PER; ++j) next_x[j] = lane + 32 * j < cols ? __ldg(sx + (int64_t)kb * p.Mp + 32 * j) : 0.f;
      };
      fetch(0);
      float2 acc[HALF / 2];
#pragma unroll
      for (int c = 0; c < HALF / 2; ++c) acc[c] = make_float2(0.f, 0.f);
      for (int kb = 0; kb < stages; ++kb, ++i) {
        const int d = i % DST;
        float* s = mine + (i & 1) * HALF;
        const float wn = next_w;
#pragma unroll
        for (int j = 0; j < PER; ++j)
          if (HALF >= 32 || lane < HALF) s[lane + 32 * j] = ROWS ? next_x[j] : __fmul_rn(next_x[j], wn);
        __syncwarp();
        fetch(kb + 1);
        if (!tc::mbar_wait(&bars->tfull[d], (i / DST) & 1, abort, p.status)) { ok = false; break; }
        tc::fence_after_sync();
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + d * C::D_COLS + first;
        const float2 w2 = make_float2(wn, wn);
#pragma unroll
        for (int c = 0; c < HALF; c += CHUNK) {
          uint32_t r[CHUNK];
          __syncwarp();
          tmem_ld(taddr + c, r);
          tc::tmem_ld_wait();
          if (c + CHUNK == HALF) {
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bars->tempty[d]);
          }
#pragma unroll
          for (int j = 0; j < CHUNK; j += 4) {
            const float4 f = *reinterpret_cast<const float4*>(s + c + j);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float2 v = make_float2(__uint_as_float(r[j + 2 * h]), __uint_as_float(r[j + 2 * h + 1]));
              const float2 x2 = h == 0 ? make_float2(f.x, f.y) : make_float2(f.z, f.w);
              float2& a = acc[(c + j) / 2 + h];
              a = ROWS ? tc::fma2(tc::mul2(v, x2), w2, a) : tc::fma2(v, x2, a);
            }
          }
        }
      }
      if (!ok) break;
      if (ranges > 1) {
        // Sums take the stages' place (all read: their products are done), every block adds up eight columns in turn.
        float* sums = reinterpret_cast<float*>(smem);  // [token, channel]
#pragma unroll
        for (int c = 0; c < HALF; ++c)
          if (c < cols) sums[(first + c) * TM + row] = c & 1 ? acc[c / 2].y : acc[c / 2].x;
        asm volatile("fence.acq_rel.cluster;" ::: "memory");
        __syncwarp();
        if (lane < ranges) tc::mbar_arrive_cluster(tc::mapa_shared(tc::smem_u32(&bars->joined), lane));
        if (!(ok = tc::mbar_wait_cluster(&bars->joined, 0, abort, p.status))) break;
        const int64_t t0 = (int64_t)mt * NTOK;
        const int all = (int)min((int64_t)NTOK, p.M - t0);
#pragma unroll 1
        for (int c0 = 8 * (rank + ranges * (warp < 6 ? 0 : 1)); c0 < all; c0 += 16 * ranges) {
          float sum[8] = {};
#pragma unroll 1
          for (int q = 0; q < ranges; ++q) {
            const uint32_t at = tc::mapa_shared(tc::smem_u32(sums + c0 * TM + row), q);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += c0 + j < all ? load_cluster(at + j * TM * 4) : 0.f;
          }
          if (n >= p.N) continue;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int64_t at = (t0 + c0 + j) * p.ldy + n;
            if (c0 + j < all && inside(at)) put(p.y, at, sum[j], p.y_type);
          }
        }
        break;
      }
      __syncwarp();
      if (words && cols == HALF && (nt + 1) * TM <= p.N) {
        // lanes 2i and 2i + 1 exchange a token: the even one stores the first of two, the odd one the second
        const bool odd = lane & 1;
        uint16_t* y = static_cast<uint16_t*>(p.y) + m0 * p.ldy + n + (odd ? p.ldy - 1 : 0);
#pragma unroll
        for (int c = 0; c < HALF / 2; ++c) {
          const float other = __shfl_xor_sync(0xffffffffu, odd ? acc[c].x : acc[c].y, 1);
          if (inside(y - static_cast<uint16_t*>(p.y) + 1))
            *reinterpret_cast<uint32_t*>(y) = odd ? pair_of(other, acc[c].y, p.y_type) : pair_of(acc[c].x, other, p.y_type);
          y += 2 * p.ldy;
        }
      } else if (n < p.N) {
#pragma unroll
        for (int c = 0; c < HALF; ++c) {
          const int64_t at = (m0 + c) * p.ldy + n;
          if (c < cols && inside(at)) put(p.y, at, c & 1 ? acc[c / 2].y : acc[c / 2].x, p.y_type);
        }
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  __syncwarp();
  if (ranges > 1) tc::cluster_sync();  // (the others have read this block's sums)
  tc::fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------ host side
PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return (PFN_cuTensorMapEncodeTiled_v12000) nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }();
  return fn;
}

// Boxes of 128 bytes of `rows` rows of a byte matrix [outer, K].
bool make_map(CUtensorMap* m, const void* base, uint64_t K, uint64_t outer, uint32_t rows) {
  auto fn = encode_fn();
  if (fn == nullptr || (reinterpret_cast<uintptr_t>(base) & 15u) || K % 16) return false;
  cuuint64_t dims[2] = {K, outer}, strides[1] = {K};
  cuuint32_t box[2] = {BK, rows}, estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tokens of a tile: the smallest that holds them all, 256 where there are two tiles of them for every SM.
int tile_tokens(int64_t M, int N, int sms) {
  if (M <= 16) return 16;
  if (M <= 32) return 32;
  if (M <= 64) return 64;
  return (M + 255) / 256 * ((N + TM - 1) / TM) >= 2 * (int64_t)sms ? 256 : 128;
}

struct Scratch {
  int64_t Mp;
  size_t sx, codes, total;
};
Scratch plan_scratch(int64_t M, int K) {
  Scratch s;
  s.Mp = (M + 31) / 32 * 32;
  s.sx = 0;
  s.codes = ((size_t)s.Mp * ((K + BK - 1) / BK) * 4 + 255) / 256 * 256;
  s.total = s.codes + (size_t)M * K;
  return s;
}

// K ranges of a tile: as many as leave no cluster waiting for another to end, of kLeast stages and more each.
constexpr int kLeast = 6;
template <class C, class Kernel>
int ranges_of(Kernel kern, const F8Params& p, int sms, int dev, Found& fit) {
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
  for (int s = (int)std::min<int64_t>({kMaxRanges, sms / tiles, p.stages / kLeast}); s > 1; --s) {
    const int clusters = fit.get(dev, s, [&] {  // of that many blocks, resident at once
      cudaLaunchConfig_t cfg = {};
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = s;
      at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
      cfg.gridDim = dim3((unsigned)(sms / s * s));
      cfg.blockDim = dim3(C::THREADS);
      cfg.dynamicSmemBytes = C::SMEM;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      int n = 0;
      if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) cudaGetLastError();
      return std::max(n, 1);
    });
    if (tiles <= clusters) return s;
  }
  return 1;
}

template <int NTOK, bool ROWS>
cudaError_t launch_as(const CUtensorMap& tw, const CUtensorMap& tx, F8Params p, int sms, cudaStream_t st) {
  using C = Cfg<NTOK>;
  auto kern = fp8_linear_kernel<NTOK, ROWS>;
  static SetUp ready;
  static Found fit;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = ready.once(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); });
  if (e != cudaSuccess) return e;
  p.ranges = C::SPLIT ? ranges_of<C>(kern, p, sms, dev, fit) : 1;
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = p.ranges;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(p.ranges > 1 ? tiles * p.ranges : std::min<int64_t>(tiles, sms)));
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = p.ranges > 1 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, kern, tw, tx, p);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}
template <bool ROWS>
cudaError_t launch_tokens(const CUtensorMap& tw, const CUtensorMap& tx, const F8Params& p, int ntok, int sms, cudaStream_t st) {
  return ntok == 16    ? launch_as<16, ROWS>(tw, tx, p, sms, st)
         : ntok == 32  ? launch_as<32, ROWS>(tw, tx, p, sms, st)
         : ntok == 64  ? launch_as<64, ROWS>(tw, tx, p, sms, st)
         : ntok == 128 ? launch_as<128, ROWS>(tw, tx, p, sms, st)
                       : launch_as<256, ROWS>(tw, tx, p, sms, st);
}

}  // namespace

size_t fp8_linear_scratch(int64_t M, int K) { return plan_scratch(M, K).total; }

cudaError_t launch_fp8_linear(const Fp8LinearArgs& a, int sms, cudaStream_t st) {
  const Scratch s = plan_scratch(a.M, a.K);
  char* w = static_cast<char*>(a.ws);
  const int ntok = tile_tokens(a.M, a.N, sms);
  F8Params p{};
  p.M = a.M, p.Mp = s.Mp, p.N = a.N, p.ldy = a.ldy;
  p.stages = (a.K + BK - 1) / BK;
  p.tiles_n = (a.N + TM - 1) / TM;
  p.tiles_m = (int)((a.M + ntok - 1) / ntok);
  if ((int64_t)p.tiles_n * p.tiles_m >= (int64_t)1 << 29) return cudaErrorInvalidValue;
  p.by_n = FastDiv(p.tiles_n);
  p.sx = reinterpret_cast<const float*>(w + s.sx);
  p.sw = a.w_scales;
  p.y = a.y;
  p.y_type = a.y_type;
  p.status = a.status;
  Fp8QuantArgs q{};
  q.M = a.M, q.K = a.K, q.x = a.x, q.type = a.x_type, q.ldx = a.ldx, q.block_rows = 1;
  q.codes = w + s.codes, q.scales = reinterpret_cast<float*>(w + s.sx);
  q.row_pitch = 1, q.block_pitch = s.Mp, q.status = a.status;
  CUtensorMap tw, tx;
  if (!make_map(&tw, a.codes, a.K, a.N, TM) || !make_map(&tx, w + s.codes, a.K, a.M, ntok)) return cudaErrorInvalidValue;
  const cudaError_t e = launch_fp8_quantize(q, sms, st);
  if (e != cudaSuccess) return e;
  return a.block_rows == 1 ? launch_tokens<true>(tw, tx, p, ntok, sms, st) : launch_tokens<false>(tw, tx, p, ntok, sms, st);
}

}  // namespace jab
