// Product in 8-bit floating point (e4m3) with a scale for every 128 of K, on the tensor cores of sm_103a:
//
//   y[m, n] = sum_b sx[m, b] sw[n / block_rows, b] sum_{k in block b} qx[m, k] qw[n, k]
//
// A block's sum is an accumulator of its own: four products of K = 32, then it is read out of tensor memory, multiplied by its
// scales and added to running sums in registers, while the next block's products fill another accumulator.
//
// Up to 128 tokens a tile, the output channels on the accumulator's 128 lanes and the tokens on its columns, so that one layout
// serves one token and many: a lane's channel has its own scale (block_rows = 1), a column's token another, which every lane
// reads from shared memory. Roles of a block: a warp that issues the copies (TMA, weights and token codes in one ring), two that
// issue the products of every other block of K (an issue with its waits is 400 clocks: one warp held 16 tokens up), one that
// brings the scales, eight that read out, scale and add up. Many tiles: persistent blocks. Few tiles: one a cluster, whose blocks
// take ranges of K and add their sums through shared memory in a fixed order. Many tokens: pairs of blocks, further down.
//
// Bound: 8192 tokens x 6144 x 4096 with scales for 128 x 128 weights take 238 us, 21 of them for the tokens' codes: 1.73 PFLOP/s, 0.45 of
// the 3.85 that an e4m3 product with one scale for all reaches here (8192^3). It is the round trip of the accumulators that takes the time
// (further down), not the products: the tensor pipe is 38 % active. With a scale for every row's 128 321 us (two operations an element in
// the read-out, 1700 clocks a block of K). One token (25 MB of codes) takes 9.3 us where the weights are in L2 (three sets in turn), 11.2
// where they are not (twelve), and the bytes take 3.8: two launches, the copies' latency and sixteen stages' products and read-outs on 96
// SMs (a third K range would need clusters of three, of which fewer than 48 fit). (Codes of up to 16 tokens made in the product's own
// kernel: no faster there, and 5.8 us instead of 5.0 for 1 x 2304 x 768, as the weights' copies cannot begin before the launch before has
// ended.)
#include <cudaTypedefs.h>

#include <algorithm>

#include "common.cuh"
#include "per_device.h"
#include "serve.h"
#include "tc.cuh"

namespace jab {
namespace {

constexpr int TM = 128, BK = 128;  // output channels of a tile; K of a stage, of a scale
constexpr int SST = 8;             // blocks of K whose scales are in shared memory
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
  static constexpr int ST = NTOK == 128 ? 6 : NTOK == 64 ? 8 : NTOK == 32 ? 9 : 11;
  static constexpr int D_COLS = NTOK < 32 ? 32 : NTOK, DST = 512 / D_COLS < 8 ? 512 / D_COLS : 8;  // accumulators
  static constexpr int HALF = NTOK / 2;                                                           // columns of a warp
  static constexpr int THREADS = 384;
  static constexpr int SMEM = ST * STAGE + 1024 + 1024 + SST * NTOK * 4;
  static_assert(NTOK * TM * 4 <= ST * STAGE, "a tile's sums take the stages' place");
};

struct Bars {
  uint64_t full[11], empty[11], tfull[8], tempty[8], sfull[SST], sempty[SST], joined, drain;
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

template <int REGS>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS)); }
template <int REGS>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS)); }

__device__ __forceinline__ float load_cluster(uint32_t at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// The pair's accumulator has been read: an arrival without a release at cluster scope, which has the thread wait for all that
// it has under way. The reads of tensor memory are complete, and nothing else is handed over.
__device__ __forceinline__ void arrive_read(uint32_t bar_cluster) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
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

// Waits for the columns that are on their way; they are not used before it.
template <int N>
__device__ __forceinline__ void tmem_arrived(uint32_t (&r)[N]) {
  tc::tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
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

// Results in fp16 that do not fit: from halfway past its largest (65504) on. (Sums of tokens and channels that are not there are 0, or NaN
// by what lies in the place of their scales; the maximum passes NaNs over.)
__device__ __forceinline__ float larger(float big, float2 v) { return fmaxf(big, fmaxf(fabsf(v.x), fabsf(v.y))); }
__device__ __forceinline__ void check_range(float big, const F8Params& p) {
  if (big >= 65520.f) report(p.status, JAB_ERR_RANGE);
}
template <int N>
__device__ __forceinline__ void check_range(const float2 (&sums)[N], const F8Params& p) {
  if (p.y_type != JAB_FP16) return;
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) big = larger(big, sums[i]);
  check_range(big, p);
}

template <int NTOK, bool ROWS>
__global__ void __launch_bounds__(Cfg<NTOK>::THREADS, 1)
    fp8_linear_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ F8Params p) {
  using C = Cfg<NTOK>;
  constexpr int ST = C::ST, DST = C::DST, HALF = C::HALF;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Bars* bars = reinterpret_cast<Bars*>(smem + ST * C::STAGE);
  float* scales = reinterpret_cast<float*>(smem + ST * C::STAGE + 1024);  // [SST, NTOK]
  const int warp = tc::warp_index(), lane = threadIdx.x & 31;
  const int ranges = p.ranges;
  // A block's tiles and its stages of each: [st0, st0 + stages)
  const int total = p.tiles_n * p.tiles_m, rank = ranges > 1 ? (int)tc::cluster_ctarank() : 0;
  const int unit0 = ranges > 1 ? blockIdx.x / ranges : blockIdx.x, step = ranges > 1 ? total : gridDim.x;
  const int st0 = p.stages * rank / ranges, stages = p.stages * (rank + 1) / ranges - st0;
  volatile int* abort = &bars->abort;
  auto load_w = [&](int s, int kb, int nt) {  // (past the end of K or of the rows: zeros)
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
    for (int s = 0; s < SST; ++s) {
      tc::mbar_init(&bars->sfull[s], 1);
      tc::mbar_init(&bars->sempty[s], 8);
    }
    tc::mbar_init(&bars->joined, 8 * ranges);
    tc::mbar_init(&bars->drain, 2);
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

  if (warp < 4) {
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
    } else if (warp < 3) {  // ---------------- products (the whole warp waits, one thread issues): two warps, a block of K each in turn
      constexpr uint32_t IDESC = tc::idesc_e4m3(TM, NTOK);
      const int n = (total - unit0 + step - 1) / step * stages;
      bool ok = true;
      for (int i = warp - 1; i < n; i += 2) {
        const int s = i % ST, d = i % DST;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->full[s], (i / ST) & 1, abort, p.status));
        if (i >= DST) ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(&bars->tempty[d], ((i / DST) & 1) ^ 1, abort, p.status));
        if (!ok) break;
        if (tc::elect_one()) {
          tc::fence_after_sync();
          const uint64_t wd = tc::sdesc_kmajor_sw128(tc::smem_u32(smem + s * C::STAGE));
          const uint64_t xd = tc::sdesc_kmajor_sw128(tc::smem_u32(smem + s * C::STAGE + C::W_STAGE));
#pragma unroll
          for (int k = 0; k < BK / 32; ++k)
            tc::umma_f8(tmem + d * C::D_COLS, tc::sdesc_advance(wd, k * 32), tc::sdesc_advance(xd, k * 32), IDESC, k > 0 ? 1u : 0u);
          tc::umma_commit(&bars->tfull[d]);
          tc::umma_commit(&bars->empty[s]);
        }
        __syncwarp();
      }
      if (tc::elect_one()) {
        tc::umma_commit(&bars->drain);
        drain_wait(&bars->drain, 0);
      }
    } else {  // ---------------- scales: a lane has four tokens' of a block of K; four blocks are on their way together
      const int c = 4 * lane;
      int i = 0;
      bool ok = true;
      for (int unit = unit0; unit < total && ok; unit += step) {
        int nt, mt;
        p.by_n.divmod(unit, mt, nt);
        const int64_t m = (int64_t)mt * NTOK + c;
        const bool there = c < NTOK && m < p.Mp;
        const float* sx = p.sx + (int64_t)st0 * p.Mp + m;
        const float* sw = p.sw + (int64_t)nt * p.stages + st0;
        for (int kb = 0; kb < stages && ok; kb += 4) {
          float4 v[4];
          float w[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const bool here = kb + u < stages;
            v[u] = there && here ? __ldcg(reinterpret_cast<const float4*>(sx + (int64_t)(kb + u) * p.Mp)) : make_float4(0.f, 0.f, 0.f, 0.f);
            w[u] = !ROWS && here ? __ldg(sw + kb + u) : 1.f;
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (kb + u >= stages) break;
            const int s = i % SST;
            if (!(ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->sempty[s], ((i / SST) & 1) ^ 1, abort, p.status)))) break;
            if (c < NTOK) {
              if (!ROWS) v[u] = make_float4(__fmul_rn(v[u].x, w[u]), __fmul_rn(v[u].y, w[u]), __fmul_rn(v[u].z, w[u]), __fmul_rn(v[u].w, w[u]));
              *reinterpret_cast<float4*>(scales + s * NTOK + c) = v[u];
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bars->sfull[s]);
            ++i;
          }
        }
      }
    }
  } else {  // ---------------- sums: a warp has 32 channels and half of the tokens
    constexpr int CHUNK = HALF < 32 ? HALF : 32;
    const int quarter = warp & 3, row = quarter * 32 + lane, first = warp < 8 ? 0 : HALF;
    // two channels of a token in one store, where they lie together in a word
    const bool words = p.y_type != JAB_FP32 && p.ldy % 2 == 0 && (reinterpret_cast<uintptr_t>(p.y) & 3) == 0;
    auto inside = [&](int64_t last) { return in_bounds(last, (p.M - 1) * p.ldy + p.N, p.status); };
    int i = 0;
    bool ok = true;
    for (int unit = unit0; unit < total && ok; unit += step) {
      int nt, mt;
      p.by_n.divmod(unit, mt, nt);
      const int n0 = nt * TM, n = n0 + row;
      const int64_t m0 = (int64_t)mt * NTOK + first;
      const int cols = (int)max((int64_t)0, min((int64_t)HALF, p.M - m0));
      const float* sw = p.sw + (int64_t)min(n, p.N - 1) * p.stages + st0;
      float next_w = 1.f, after_w = 1.f;  // a channel's scales come two blocks ahead
      if (ROWS) {
        next_w = __ldg(sw);
        if (stages > 1) after_w = __ldg(sw + 1);
      }
      float2 acc[HALF / 2];
#pragma unroll
      for (int c = 0; c < HALF / 2; ++c) acc[c] = make_float2(0.f, 0.f);
      for (int kb = 0; kb < stages; ++kb, ++i) {
        const int d = i % DST, s = i % SST;
        const float2 w2 = make_float2(next_w, next_w);
        next_w = after_w;
        if (ROWS && kb + 2 < stages) after_w = __ldg(sw + kb + 2);
        if (!tc::mbar_wait(&bars->sfull[s], (i / SST) & 1, abort, p.status) || !tc::mbar_wait(&bars->tfull[d], (i / DST) & 1, abort, p.status)) {
          ok = false;
          break;
        }
        tc::fence_after_sync();
        const float* sx = scales + s * NTOK + first;
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + d * C::D_COLS + first;
        uint32_t r[2][CHUNK];  // the next columns are on their way while some are worked on
        __syncwarp();
        tmem_ld(taddr, r[0]);
        tmem_arrived(r[0]);
#pragma unroll
        for (int c = 0; c < HALF; c += CHUNK) {
          const uint32_t(&now)[CHUNK] = r[(c / CHUNK) & 1];
          if (c + CHUNK < HALF) {
            tmem_ld(taddr + c + CHUNK, r[(c / CHUNK + 1) & 1]);
          } else {
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bars->tempty[d]);
          }
#pragma unroll
          for (int j = 0; j < CHUNK; j += 4) {
            const float4 f = *reinterpret_cast<const float4*>(sx + c + j);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float2 v = make_float2(__uint_as_float(now[j + 2 * h]), __uint_as_float(now[j + 2 * h + 1]));
              const float2 x2 = h == 0 ? make_float2(f.x, f.y) : make_float2(f.z, f.w);
              float2& a = acc[(c + j) / 2 + h];
              a = ROWS ? tc::fma2(tc::mul2(v, x2), w2, a) : tc::fma2(v, x2, a);
            }
          }
          if (c + CHUNK < HALF) tmem_arrived(r[(c / CHUNK + 1) & 1]);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->sempty[s]);
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
        for (int c0 = 8 * (rank + ranges * (warp < 8 ? 0 : 1)); c0 < all; c0 += 16 * ranges) {
          float sum[8] = {};
#pragma unroll 1
          for (int q = 0; q < ranges; ++q) {
            const uint32_t at = tc::mapa_shared(tc::smem_u32(sums + c0 * TM + row), q);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += c0 + j < all ? load_cluster(at + j * TM * 4) : 0.f;
          }
          if (n >= p.N) continue;
          if (p.y_type == JAB_FP16) {
            float big = 0.f;
#pragma unroll
            for (int j = 0; j < 8; j += 2) big = larger(big, make_float2(sum[j], sum[j + 1]));
            check_range(big, p);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int64_t at = (t0 + c0 + j) * p.ldy + n;
            if (c0 + j < all && inside(at)) put(p.y, at, sum[j], p.y_type);
          }
        }
        break;
      }
      check_range(acc, p);
      __syncwarp();
      if (words && cols == HALF && n0 + TM <= p.N) {
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

// ------------------------------------------------------------------ many tokens: pairs of blocks
// Two blocks of a cluster on two SMs share a tile of 256 tokens x 256 channels: either has 128 of the tokens (its lanes) and the codes of
// half of the channels, so that a stage is 32 KB a block. Lanes are tokens here: with channels on them every lane would read every token's
// scale from shared memory, a pass of its own each (8 warps x 128 columns: 1000 clocks for a block of K whose products would take 512 at
// the tensor cores' nominal rate). With block_rows = 128 a lane has one factor for a block of K; with block_rows = 1 tensor memory is read
// in the shape that gives a thread two of eight columns, whose scales are 32 passes a warp. Bound: a block of K takes 1130 clocks. Its
// products take 820 behind one another, as measured; with two accumulators of 256 columns (all of tensor memory) one is free again 500
// clocks for the barrier of its last product, 450 for the read-out and 400 for the arrival and the next issue after that. Three
// accumulators of 160 columns (263 us where this took 256) and one block a tile (277) were no faster: a pair's products take 1300 clocks
// from issue to the barrier however short they are, a block's own 48 KB a stage 950. (The form with block_rows = 128 has 104 bytes of a
// thread's state in local memory: registers are allotted for 168 a thread before they are moved.)
struct PairCfg {
  static constexpr int ST = 5, STAGE = 2 * TM * BK, THREADS = 384, DST = 2, COLS = 256;
  static constexpr int OUT = 32 * 128;  // a warp's place for 128 bytes of 32 rows on their way out
  static constexpr int EPI_REGS = 216, OTHER_REGS = 72;
  static constexpr int SMEM = ST * STAGE + 1024 + 1024 + SST * COLS * 4 + 8 * OUT;
  static_assert(128 * OTHER_REGS + 256 * EPI_REGS <= THREADS * (65536 / THREADS / 8 * 8), "registers");
};
constexpr int AHEAD = 4;  // blocks of K that a lane's factors come ahead

// 32 rows of 128 bytes from a warp's place (16-byte chunk c of row r at c ^ (r & 7)) to rows of `pitch` bytes: four rows a store, where
// lanes that store from their own rows touch 32 lines at a time (4000 clocks a tile: 256 us where this takes 238). `rows` of them are there.
template <class Inside>
__device__ __forceinline__ void rows_out(const uint8_t* place, uint8_t* y, int64_t pitch, int rows, int lane, Inside inside) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = 4 * i + (lane >> 3), c = lane & 7;
    const uint4 v = *reinterpret_cast<const uint4*>(place + r * 128 + ((c ^ (r & 7)) << 4));
    uint8_t* to = y + r * pitch + 16 * c;
    if (r < rows && inside(to)) *reinterpret_cast<uint4*>(to) = v;
  }
}

template <bool ROWS>
__global__ void __launch_bounds__(PairCfg::THREADS, 1)
    fp8_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ F8Params p) {
  using C = PairCfg;
  constexpr int ST = C::ST, DST = C::DST, COLS = C::COLS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Bars* bars = reinterpret_cast<Bars*>(smem + ST * C::STAGE);
  float* scales = reinterpret_cast<float*>(smem + ST * C::STAGE + 1024);  // [SST, COLS] of the channels (ROWS)
  const int warp = tc::warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)tc::cluster_ctarank(), total = p.tiles_n * p.tiles_m, unit0 = blockIdx.x / 2, step = gridDim.x / 2, stages = p.stages;
  const bool leads = rank == 0;  // issues the pair's products
  volatile int* abort = &bars->abort;
  const uint32_t full_lead = tc::mapa_shared(tc::smem_u32(&bars->full[0]), 0), tempty_lead = tc::mapa_shared(tc::smem_u32(&bars->tempty[0]), 0);
  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; ++s) {
      tc::mbar_init(&bars->full[s], 1);
      tc::mbar_init(&bars->empty[s], 1);
    }
    for (int d = 0; d < DST; ++d) {
      tc::mbar_init(&bars->tfull[d], 1);
      tc::mbar_init(&bars->tempty[d], 16);
    }
    for (int s = 0; s < SST; ++s) {
      tc::mbar_init(&bars->sfull[s], 1);
      tc::mbar_init(&bars->sempty[s], 8);
    }
    tc::mbar_init(&bars->drain, 2);
    bars->abort = 0;
    tc::fence_mbar_init();
  }
  if (warp == 1) {
    tc::tmem_alloc2(&bars->tmem_base, 512);
    tc::tmem_relinquish2();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  tc::cluster_sync();  // (both blocks' barriers and tensor memory are there)
  const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
  stream_order();

  if (warp < 4) {
    fewer_registers<C::OTHER_REGS>();
    if (warp == 0) {
      if (tc::elect_one()) {  // ---------------- copies, counted on the leading block's barriers
        int i = 0;
        bool ok = true;
        for (int unit = unit0; unit < total && ok; unit += step) {
          int nt, mt;
          p.by_n.divmod(unit, mt, nt);
          for (int kb = 0; kb < stages; ++kb, ++i) {
            const int s = i % ST;
            if (!(ok = tc::mbar_wait(&bars->empty[s], ((i / ST) & 1) ^ 1, abort, p.status))) break;
            if (leads) tc::mbar_expect_tx(&bars->full[s], 2 * C::STAGE);
            uint8_t* at = smem + s * C::STAGE;  // (past the end of K or of the rows: zeros)
            tc::tma_load_2d_pair(at, &tmX, full_lead + 8 * s, kb * BK, mt * 2 * TM + rank * TM);
            tc::tma_load_2d_pair(at + TM * BK, &tmW, full_lead + 8 * s, kb * BK, nt * COLS + rank * TM);
          }
        }
        if (*abort && leads)  // every copy of the pair has landed before shared memory goes to another block
          for (int j = max(0, i - ST); j < i; ++j) drain_wait(&bars->full[j % ST], (j / ST) & 1);
      }
    } else if (warp < 3) {  // ---------------- products (the whole warp waits, one thread issues): a warp for each accumulator
      constexpr uint32_t IDESC = tc::idesc_e4m3(2 * TM, COLS);
      const int n = leads ? (total - unit0 + step - 1) / step * stages : 0, d = warp - 1;
      bool ok = true;
      for (int i = d; i < n; i += DST) {
        const int s = i % ST;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->full[s], (i / ST) & 1, abort, p.status));
        if (i >= DST) ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(&bars->tempty[d], ((i / DST) & 1) ^ 1, abort, p.status));
        if (!ok) break;
        if (tc::elect_one()) {
          tc::fence_after_sync();
          const uint64_t xd = tc::sdesc_kmajor_sw128(tc::smem_u32(smem + s * C::STAGE));
          const uint64_t wd = tc::sdesc_kmajor_sw128(tc::smem_u32(smem + s * C::STAGE + TM * BK));
#pragma unroll
          for (int k = 0; k < BK / 32; ++k)
            tc::umma2_f8(tmem + d * COLS, tc::sdesc_advance(xd, k * 32), tc::sdesc_advance(wd, k * 32), IDESC, k > 0 ? 1u : 0u);
          tc::umma2_commit_mc(&bars->tfull[d], 0x3);
          tc::umma2_commit_mc(&bars->empty[s], 0x3);
        }
        __syncwarp();
      }
      if (leads && tc::elect_one()) {
        tc::umma2_commit_mc(&bars->drain, 0x1);
        drain_wait(&bars->drain, 0);
      }
    } else if (ROWS) {  // ---------------- channel scales: a lane has eight channels', two blocks of K at a time
      const int c = 8 * lane;
      int i = 0;
      bool ok = true;
      for (int unit = unit0; unit < total && ok; unit += step) {
        int nt, mt;
        p.by_n.divmod(unit, mt, nt);
        for (int kb = 0; kb < stages && ok; kb += 2) {
          float v[2][8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float* sw = p.sw + (int64_t)min(nt * COLS + c + j, p.N - 1) * stages;
#pragma unroll
            for (int u = 0; u < 2; ++u) v[u][j] = kb + u < stages ? __ldg(sw + kb + u) : 0.f;
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if (kb + u >= stages) break;
            const int s = i % SST;
            if (!(ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->sempty[s], ((i / SST) & 1) ^ 1, abort, p.status)))) break;
            float4* to = reinterpret_cast<float4*>(scales + s * COLS + c);
            to[0] = make_float4(v[u][0], v[u][1], v[u][2], v[u][3]), to[1] = make_float4(v[u][4], v[u][5], v[u][6], v[u][7]);
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bars->sfull[s]);
            ++i;
          }
        }
      }
    }
  } else {  // ---------------- sums: a warp has 32 tokens and half of the channels
    more_registers<C::EPI_REGS>();
    const int quarter = warp & 3, first = warp < 8 ? 0 : COLS / 2;
    const bool wide = ((p.y_type == JAB_FP32 ? p.ldy % 4 : p.ldy % 8) | (int64_t)(reinterpret_cast<uintptr_t>(p.y) & 15)) == 0;
    auto inside = [&](int64_t last) { return in_bounds(last, (p.M - 1) * p.ldy + p.N, p.status); };
    uint8_t* place = smem + ST * C::STAGE + 1024 + SST * COLS * 4 + (warp - 4) * C::OUT;
    const int size = p.y_type == JAB_FP32 ? 4 : 2;
    auto chunk_inside = [&](const uint8_t* to) { return inside((to - static_cast<const uint8_t*>(p.y)) / size + 16 / size - 1); };
    auto read = [&](int d) {  // the accumulator may be written again
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (leads)
          tc::mbar_arrive(&bars->tempty[d]);
        else
          arrive_read(tempty_lead + 8 * d);
      }
    };
    int i = 0;
    bool ok = true;
    for (int unit = unit0; unit < total && ok; unit += step) {
      int nt, mt;
      p.by_n.divmod(unit, mt, nt);
      const int64_t m0 = (int64_t)mt * 2 * TM + rank * TM + quarter * 32;
      const int n0 = nt * COLS + first;
      float2 acc[COLS / 4];
#pragma unroll
      for (int c = 0; c < COLS / 4; ++c) acc[c] = make_float2(0.f, 0.f);
      if constexpr (!ROWS) {
        const float* sx = p.sx + min(m0 + lane, p.Mp - 1);
        const float* sw = p.sw + (int64_t)min(n0 / TM, (p.N - 1) / TM) * stages;
        float fx[AHEAD], fw[AHEAD];
        auto fetch = [&](int u, int kb) {
          if (kb < stages) fx[u] = __ldcg(sx + (int64_t)kb * p.Mp), fw[u] = __ldg(sw + kb);
        };
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) fetch(u, u);
        for (int kb0 = 0; kb0 < stages && ok; kb0 += AHEAD) {
#pragma unroll
          for (int u = 0; u < AHEAD; ++u) {
            const int kb = kb0 + u;
            if (kb >= stages || !ok) break;
            const int d = i % DST;
            const float f = __fmul_rn(fx[u], fw[u]);
            const float2 f2 = make_float2(f, f);
            fetch(u, kb + AHEAD);
            if (!(ok = tc::mbar_wait(&bars->tfull[d], (i / DST) & 1, abort, p.status))) break;
            ++i;
            tc::fence_after_sync();
            const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + d * COLS + first;
            uint32_t r[2][32];  // the next columns are on their way while some are worked on
            __syncwarp();
            tmem_ld(taddr, r[0]);
            tmem_arrived(r[0]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if (c < 3)
                tmem_ld(taddr + 32 * (c + 1), r[(c + 1) & 1]);
              else
                read(d);
#pragma unroll
              for (int j = 0; j < 16; ++j)
                acc[16 * c + j] = tc::fma2(make_float2(__uint_as_float(r[c & 1][2 * j]), __uint_as_float(r[c & 1][2 * j + 1])), f2, acc[16 * c + j]);
              if (c < 3) tmem_arrived(r[(c + 1) & 1]);
            }
          }
        }
        if (!ok) break;
        check_range(acc, p);
        if (wide && n0 + COLS / 2 <= p.N) {
          uint8_t* y = static_cast<uint8_t*>(p.y) + (m0 * p.ldy + n0) * size;
          const int rows = (int)max((int64_t)0, min((int64_t)32, p.M - m0));
          auto put16 = [&](int c, const uint4& v) { *reinterpret_cast<uint4*>(place + lane * 128 + ((c ^ (lane & 7)) << 4)) = v; };
          if (size == 4) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              __syncwarp();
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                const float2 u = acc[16 * h + 2 * c], v = acc[16 * h + 2 * c + 1];
                put16(c, make_uint4(__float_as_uint(u.x), __float_as_uint(u.y), __float_as_uint(v.x), __float_as_uint(v.y)));
              }
              __syncwarp();
              rows_out(place, y + 128 * h, p.ldy * size, rows, lane, chunk_inside);
            }
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              __syncwarp();
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                const float2* v = acc + 32 * h + 4 * c;
                put16(c, make_uint4(pair_of(v[0].x, v[0].y, p.y_type), pair_of(v[1].x, v[1].y, p.y_type), pair_of(v[2].x, v[2].y, p.y_type),
                                    pair_of(v[3].x, v[3].y, p.y_type)));
              }
              __syncwarp();
              rows_out(place, y + 128 * h, p.ldy * size, rows, lane, chunk_inside);
            }
          }
        } else if (m0 + lane < p.M) {
          const int64_t at = (m0 + lane) * p.ldy + n0;
#pragma unroll
          for (int c = 0; c < COLS / 2; ++c)
            if (n0 + c < p.N && inside(at + c)) put(p.y, at + c, c & 1 ? acc[c / 2].y : acc[c / 2].x, p.y_type);
        }
      } else {
        // acc[4 c + t]: channels n0 + 8 c + 2 (lane % 4) and the next of token m0 + 8 t + lane / 4
        float fx[4], nx[4];  // of the thread's four tokens
        const int64_t m1 = m0 + (lane >> 2);
        auto fetch = [&](int kb) {
#pragma unroll
          for (int t = 0; t < 4; ++t)
            if (kb < stages) nx[t] = __ldcg(p.sx + (int64_t)kb * p.Mp + min(m1 + 8 * t, p.Mp - 1));
        };
        fetch(0);
        for (int kb = 0; kb < stages; ++kb, ++i) {
          const int d = i % DST, s = i % SST;
#pragma unroll
          for (int t = 0; t < 4; ++t) fx[t] = nx[t];
          fetch(kb + 1);
          if (!tc::mbar_wait(&bars->sfull[s], (i / SST) & 1, abort, p.status) || !tc::mbar_wait(&bars->tfull[d], (i / DST) & 1, abort, p.status)) {
            ok = false;
            break;
          }
          tc::fence_after_sync();
          const float* sw = scales + s * COLS + first + 2 * (lane & 3);
          const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + d * COLS + first;
#pragma unroll
          for (int c = 0; c < 2; ++c) {  // 64 columns
            uint32_t r[2][32];            // of the first and the second sixteen tokens
            __syncwarp();
            tc::tmem_ld_16x256b_x8(taddr + 64 * c, r[0]);
            tc::tmem_ld_16x256b_x8(taddr + 64 * c + (16u << 16), r[1]);
            tmem_arrived(r[0]);
            tmem_arrived(r[1]);
            if (c == 1) read(d);
#pragma unroll
            for (int n = 0; n < 8; ++n) {
              const float2 w2 = *reinterpret_cast<const float2*>(sw + 64 * c + 8 * n);
#pragma unroll
              for (int t = 0; t < 4; ++t) {  // tokens 16 (t / 2) + 8 (t & 1) + lane / 4
                const float2 v = make_float2(__uint_as_float(r[t >> 1][4 * n + 2 * (t & 1)]), __uint_as_float(r[t >> 1][4 * n + 2 * (t & 1) + 1]));
                float2& a = acc[32 * c + 4 * n + t];
                a = tc::fma2(tc::mul2(v, w2), make_float2(fx[t], fx[t]), a);
              }
            }
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&bars->sempty[s]);
        }
        if (!ok) break;
        check_range(acc, p);
        if (wide && n0 + COLS / 2 <= p.N) {
          uint8_t* y = static_cast<uint8_t*>(p.y) + (m0 * p.ldy + n0) * size;
          const int rows = (int)max((int64_t)0, min((int64_t)32, p.M - m0));
          if (size == 4) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              __syncwarp();
#pragma unroll
              for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  const int r = 8 * t + (lane >> 2), at = r * 128 + (((2 * c + ((lane & 3) >> 1)) ^ (r & 7)) << 4) + 8 * (lane & 1);
                  *reinterpret_cast<float2*>(place + at) = acc[4 * (4 * h + c) + t];
                }
              __syncwarp();
              rows_out(place, y + 128 * h, p.ldy * size, rows, lane, chunk_inside);
            }
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              __syncwarp();
#pragma unroll
              for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                  const int r = 8 * t + (lane >> 2), at = r * 128 + ((c ^ (r & 7)) << 4) + 4 * (lane & 3);
                  const float2 v = acc[4 * (8 * h + c) + t];
                  *reinterpret_cast<uint32_t*>(place + at) = pair_of(v.x, v.y, p.y_type);
                }
              __syncwarp();
              rows_out(place, y + 128 * h, p.ldy * size, rows, lane, chunk_inside);
            }
          }
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int64_t m = m1 + 8 * t;
            if (m >= p.M) continue;
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              const int n = n0 + 8 * c + 2 * (lane & 3);
              const int64_t at = m * p.ldy + n;
              const float2 v = acc[4 * c + t];
              if (n < p.N && inside(at)) put(p.y, at, v.x, p.y_type);
              if (n + 1 < p.N && inside(at + 1)) put(p.y, at + 1, v.y, p.y_type);
            }
          }
        }
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  __syncwarp();
  tc::cluster_sync();  // the pair's products are complete and no arrival is on its way to the other block
  tc::fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc2(tmem, 512);
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

// Tokens of a tile: the smallest that holds them all; past 128 the pairs' 256 where their rounds, each as long as 1.6 of the others',
// take less (768 x 6144 x 4096: 28 us, else 33; 1024: 47.3 and 46.7; 2048: 70 and 89).
int tile_tokens(int64_t M, int N, int sms) {
  if (M <= 16) return 16;
  if (M <= 32) return 32;
  if (M <= 64) return 64;
  if (M <= 128) return 128;
  const int64_t pairs = std::max(sms / 2, 1);
  const int64_t wide = ((M + 255) / 256 * ((N + 255) / 256) + pairs - 1) / pairs;
  const int64_t narrow = ((M + 127) / 128 * ((N + 127) / 128) + sms - 1) / sms;
  return 16 * wide < 10 * narrow ? 256 : 128;
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

// Clusters of s blocks that are resident at once.
template <class C, class Kernel>
int clusters_at_once(Kernel kern, int s, int sms, int dev, Found& fit) {
  return fit.get(dev, s, [&] {
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
}

// K ranges of a tile: as many as leave no cluster waiting for another to end, of kLeast stages and more each.
constexpr int kLeast = 6;
template <class C, class Kernel>
int ranges_of(Kernel kern, const F8Params& p, int sms, int dev, Found& fit) {
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
  for (int s = (int)std::min<int64_t>({kMaxRanges, sms / tiles, p.stages / kLeast}); s > 1; --s)
    if (tiles <= clusters_at_once<C>(kern, s, sms, dev, fit)) return s;
  return 1;
}

// `cluster` blocks a cluster, `grid` blocks.
template <class C, class Kernel>
cudaError_t launch(Kernel kern, const CUtensorMap& tw, const CUtensorMap& tx, const F8Params& p, int cluster, int64_t grid, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, tw, tx, p);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}
template <int NTOK, bool ROWS>
cudaError_t launch_as(const CUtensorMap& tw, const CUtensorMap& tx, F8Params p, int dev, int sms, cudaStream_t st) {
  using C = Cfg<NTOK>;
  auto kern = fp8_linear_kernel<NTOK, ROWS>;
  static SetUp ready;
  static Found fit;
  const cudaError_t e = ready.once(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); });
  if (e != cudaSuccess) return e;
  p.ranges = ranges_of<C>(kern, p, sms, dev, fit);
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
  return launch<C>(kern, tw, tx, p, p.ranges, p.ranges > 1 ? tiles * p.ranges : std::min<int64_t>(tiles, sms), st);
}
template <bool ROWS>
cudaError_t launch_pair(const CUtensorMap& tw, const CUtensorMap& tx, const F8Params& p, int dev, int sms, cudaStream_t st) {
  auto kern = fp8_pair_kernel<ROWS>;
  static SetUp ready;
  static Found fit;
  const cudaError_t e = ready.once(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, PairCfg::SMEM); });
  if (e != cudaSuccess) return e;
  const int pairs = std::min(clusters_at_once<PairCfg>(kern, 2, sms, dev, fit), std::max(sms / 2, 1));
  return launch<PairCfg>(kern, tw, tx, p, 2, 2 * std::min<int64_t>((int64_t)p.tiles_n * p.tiles_m, pairs), st);
}
template <bool ROWS>
cudaError_t launch_tokens(const CUtensorMap& tw, const CUtensorMap& tx, const F8Params& p, int ntok, int sms, cudaStream_t st) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  return ntok == 16    ? launch_as<16, ROWS>(tw, tx, p, dev, sms, st)
         : ntok == 32  ? launch_as<32, ROWS>(tw, tx, p, dev, sms, st)
         : ntok == 64  ? launch_as<64, ROWS>(tw, tx, p, dev, sms, st)
         : ntok == 128 ? launch_as<128, ROWS>(tw, tx, p, dev, sms, st)
                       : launch_pair<ROWS>(tw, tx, p, dev, sms, st);
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
  const int channels = ntok == 256 ? PairCfg::COLS : TM;
  p.tiles_n = (a.N + channels - 1) / channels;
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
  if (!make_map(&tw, a.codes, a.K, a.N, TM) || !make_map(&tx, w + s.codes, a.K, a.M, std::min(ntok, 128))) return cudaErrorInvalidValue;
  const cudaError_t e = launch_fp8_quantize(q, sms, st);
  if (e != cudaSuccess) return e;
  return a.block_rows == 1 ? launch_tokens<true>(tw, tx, p, ntok, sms, st) : launch_tokens<false>(tw, tx, p, ntok, sms, st);
}

}  // namespace jab
