// Product in 8-bit integers with a scale per token and per output channel, on the tensor cores of sm_103a:
//
//   y[m, n] = s_m w_n sum_k qx[m, k] qw[n, k],   s_m = fl32(max|x_m| / 127), qx = clip(rint(fl32(x / s_m)))
//
// The chip has no fast integer tensor form. Whole numbers up to 2^11 are exact in fp16, their products in the
// fp32 accumulator, and so is their sum while it stays below 2^24: 1024 products of codes at most (127^2 *
// 1024 < 2^24, and 128^2 * 1024 = 2^24). The accumulator is therefore read out every 1024 of K and added up in
// int32: the sum is exact, in any order of its parts, at the fp16 rate of the tensor cores.
//
// Two launches: the rows of X become codes (held in fp16, the operand's type) and scales; then the product, with the output
// channels on the accumulator's 128 lanes and the tokens on its columns. The weights travel as the bytes that they
// are: TMA brings a 128 x 128 tile of codes to shared memory, converter warps turn it into fp16 in tensor memory (a
// byte under the exponent of 1024, less 1152), and the products take it from there as their A operand. One layout
// serves one token and thousands. Many tiles: persistent blocks, two accumulators in turn, sums in registers. Few
// tiles: one a cluster, whose blocks take K ranges of it and add their sums through shared memory.
//
// Bound: 8192 tokens x 6144 x 4096 take 295 to 307 us, 26 of them for the tokens' codes (0.7 of HBM's rate) and 270 for the
// products, 1.53 PFLOP/s, 0.80 of the tensor cores' measured rate; without converters, drains and stores the products
// alone took 237 in all. One token (25 MB of codes) takes 12 us where the bytes take 3.7: the chain of launches, copy,
// conversion and products of 16 stages.
#include <cudaTypedefs.h>

#include <algorithm>

#include "kernels.h"
#include "per_device.h"
#include "quotient.cuh"
#include "serve.h"
#include "tc.cuh"

namespace jab {
namespace {

constexpr int TM = 128, BK = 64, LK = 2 * BK;  // output channels of a tile, K of a swizzled row, K of a stage
constexpr int kExactStages = 8;                // stages that one accumulator may take (1024 products)
constexpr int LST = 4;                         // stages of X in shared and of A in tensor memory
constexpr int kMaxRanges = 8;                  // K ranges of a tile (the portable cluster size)

// ------------------------------------------------------------------ tokens to codes
struct TokenParams {
  const void* x;
  int64_t ldx, M;
  int K, Kp;
  half_t* xh;     // [M, Kp]
  float* sx;      // [M]
  int* status;
};

template <class T>
__device__ __forceinline__ void unpack8(const uint4& u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<T, half_t>::value) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x, v[2 * i + 1] = f.y;
    } else {
      v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

// Scale of a row whose largest magnitude has the bits `big`; NaN where that is an infinity or a NaN.
template <class T>
__device__ __forceinline__ float row_scale(uint32_t big) {
  constexpr bool HALF = std::is_same<T, half_t>::value;
  const float a = HALF ? __half2float(__ushort_as_half((unsigned short)big)) : __uint_as_float(big << 16);
  return big < (HALF ? kHalfInf : kBf16Inf) ? __fdiv_rn(a, 127.f) : __uint_as_float(0x7fc00000u);
}
// Codes of 8 elements as fp16; 0 where the scale is 0 or NaN.
template <class T>
__device__ __forceinline__ uint4 row_codes(const uint4& u, float s) {
  float v[8];
  unpack8<T>(u, v);
  if (usual_scale(s)) {
    const float r1 = __frcp_rn(s);
    const float2 r = make_float2(r1, r1), ms = make_float2(-s, -s), up = make_float2(kToWhole, kToWhole);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 q = tc::sub2(tc::add2(quotients(make_float2(v[2 * j], v[2 * j + 1]), r, ms), up), up);
      w[j] = tc::pack_half2(q.x, q.y);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float r = fminf(fmaxf(rintf(__fdiv_rn(v[j], s)), -127.f), 127.f);
    v[j] = s > 0.f ? r : 0.f;
  }
  return make_uint4(tc::pack_half2(v[0], v[1]), tc::pack_half2(v[2], v[3]), tc::pack_half2(v[4], v[5]), tc::pack_half2(v[6], v[7]));
}

// A block per row; the row's first KEEP chunks of 8 elements a thread stay in registers between the maximum and
// the codes, what is longer is read again. Bound: bytes (8192 x 4096: 134 MB in 26 us; with a division for every element
// 32).
template <class T>
__global__ void __launch_bounds__(256) quantize_tokens_kernel(const __grid_constant__ TokenParams p) {
  constexpr int KEEP = 2;
  __shared__ uint32_t top[8];
  stream_order();
  const int tid = threadIdx.x, n8 = p.K / 8, n8p = p.Kp / 8;
  for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x) {
    const uint4* row = reinterpret_cast<const uint4*>(static_cast<const T*>(p.x) + m * p.ldx);
    uint4 keep[KEEP];
    uint32_t big = 0;
#pragma unroll
    for (int c = 0; c < KEEP; ++c) {
      keep[c] = make_uint4(0u, 0u, 0u, 0u);
      if (c * 256 + tid < n8) keep[c] = __ldg(row + c * 256 + tid);
      big = max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(big, keep[c].x), keep[c].y), keep[c].z), keep[c].w);
    }
    for (int i = KEEP * 256 + tid; i < n8; i += 256) {
      const uint4 u = __ldg(row + i);
      big = max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(big, u.x), u.y), u.z), u.w);
    }
    big = max(big & 0xffffu, big >> 16);
    big = __reduce_max_sync(0xffffffffu, big);
    __syncthreads();  // (the round before has read top)
    if ((tid & 31) == 0) top[tid >> 5] = big;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) big = max(big, top[w]);
    const float s = row_scale<T>(big);
    if (tid == 0) {
      p.sx[m] = s;
      if (!(s >= 0.f)) report(p.status, JAB_ERR_NONFINITE);
    }
    if (!in_bounds((m + 1) * p.Kp - 1, p.M * p.Kp, p.status)) continue;
    uint4* out = reinterpret_cast<uint4*>(p.xh + m * p.Kp);
#pragma unroll
    for (int c = 0; c < KEEP; ++c)
      if (c * 256 + tid < n8) out[c * 256 + tid] = row_codes<T>(keep[c], s);
    for (int i = KEEP * 256 + tid; i < n8; i += 256) out[i] = row_codes<T>(__ldg(row + i), s);
    for (int i = n8 + tid; i < n8p; i += 256) out[i] = make_uint4(0u, 0u, 0u, 0u);
  }
}

// ------------------------------------------------------------------ the product
struct LinParams {
  int64_t M, ldy;
  int N, stages, tiles_n, tiles_m, ranges;
  FastDiv by_n;
  const float *sx, *sw;
  void* y;
  int* status;
};

// Short tiles wait for the converters (16 products of 16 tokens take a tenth of a stage's conversion): four groups of
// them, where 128 tokens leave registers and time for two.
template <int NTOK>
struct Cfg {
  static constexpr int WST = NTOK == 128 ? 4 : 8;  // stages of weight codes
  static constexpr int W_STAGE = TM * LK, X_STAGE = NTOK * LK * 2;
  // Rows of a box of weights: half as many requests for the copy engine at 128 bytes (64 tokens x 6144 x 4096: 14.1 us, at 64
  // bytes 14.6), but the largest calls like the converters' reads of 64 better (8192 tokens: 297 us, at 128 bytes 306).
  static constexpr int W_ROW = NTOK == 128 ? BK : LK;
  static constexpr int D_COLS = NTOK < 32 ? 32 : NTOK;
  static constexpr int GROUPS = NTOK == 128 ? 2 : 4, THREADS = 32 * (4 + 8 + 4 * GROUPS);
  static constexpr int EPI_REGS = NTOK == 128 ? 128 : 96, CONV_REGS = NTOK == 128 ? 88 : 64;
  static constexpr bool SPLIT = NTOK < 128;  // whether clusters share a tile (128 tokens x 6144 x 4096: 18.2 us so, 18.3 without; the code costs 512 tokens and the largest calls 5 %)
  static constexpr int SMEM = WST * W_STAGE + LST * X_STAGE + 1024 + 512 + 8 * (NTOK / 2) * 4;
  static_assert(NTOK * TM * 4 <= WST * W_STAGE, "a tile's sums take the weights' place");
  static_assert(128 * 40 + 256 * EPI_REGS + 128 * GROUPS * CONV_REGS <= THREADS * (65536 / THREADS / 8 * 8), "registers");
};

struct Bars {
  uint64_t wfull[8], wempty[8], xfull[LST], ready[LST], empty[LST], tfull[2], tempty[2], joined, drain;
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(Bars) <= 512, "barrier block");

// Waits for a phase while leaving: bounded, whatever the abort flag says.
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity) {
  const uint64_t t0 = tc::globaltimer();
  while (!tc::mbar_test(bar, parity))
    if (tc::globaltimer() - t0 > tc::kWaitLimitNs) break;
}

template <class T>
__device__ __forceinline__ T out_as(float v);
template <>
__device__ __forceinline__ float out_as<float>(float v) { return v; }
template <>
__device__ __forceinline__ half_t out_as<half_t>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ bf16_t out_as<bf16_t>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ uint32_t pair_as(float a, float b, half_t) { return tc::pack_half2(a, b); }
__device__ __forceinline__ uint32_t pair_as(float a, float b, bf16_t) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// 4 signed bytes as two fp16 pairs.
__device__ __forceinline__ void codes_h2(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = w ^ 0x80808080u;
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  const uint32_t k = 0x64806480u;  // 1152
  const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&k));
  const __half2 y = __hsub2(*reinterpret_cast<const __half2*>(&b), *reinterpret_cast<const __half2*>(&k));
  lo = *reinterpret_cast<const uint32_t*>(&x);
  hi = *reinterpret_cast<const uint32_t*>(&y);
}

template <int REGS>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS)); }
template <int REGS>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS)); }

// 32 lanes x 16 columns.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                 "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
__device__ __forceinline__ int load_cluster(uint32_t at) {
  int v;
  asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

template <class T, int NTOK>
__global__ void __launch_bounds__(Cfg<NTOK>::THREADS, 1)
    qlinear_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ LinParams p) {
  using C = Cfg<NTOK>;
  constexpr int WST = C::WST;
  constexpr uint32_t A_COL = 2 * C::D_COLS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* w_smem = smem;
  uint8_t* x_smem = smem + WST * C::W_STAGE;
  Bars* bars = reinterpret_cast<Bars*>(x_smem + LST * C::X_STAGE);
  float* token_scales = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(bars) + 512);
  const int warp = tc::warp_index(), lane = threadIdx.x & 31;
  const int ranges = C::SPLIT ? p.ranges : 1;
  // A block's tiles and its stages of each: [st0, st0 + stages)
  const int total = p.tiles_n * p.tiles_m, rank = ranges > 1 ? (int)tc::cluster_ctarank() : 0;
  const int unit0 = ranges > 1 ? blockIdx.x / ranges : blockIdx.x, step = ranges > 1 ? total : gridDim.x;
  const int st0 = p.stages * rank / ranges, stages = p.stages * (rank + 1) / ranges - st0;
  volatile int* abort = &bars->abort;
  auto load_w = [&](int ws, int kb, int nt) {
    tc::mbar_expect_tx(&bars->wfull[ws], C::W_STAGE);
#pragma unroll
    for (int h = 0; h < LK / C::W_ROW; ++h)  // (past the end of K: zeros)
      tc::tma_load_2d(w_smem + ws * C::W_STAGE + h * TM * C::W_ROW, &tmW, &bars->wfull[ws], (st0 + kb) * LK + h * C::W_ROW, nt * TM);
  };
  if (threadIdx.x == 0) {
    for (int s = 0; s < WST; ++s) {
      tc::mbar_init(&bars->wfull[s], 1);
      tc::mbar_init(&bars->wempty[s], 4);
    }
    for (int s = 0; s < LST; ++s) {
      tc::mbar_init(&bars->xfull[s], 1);
      tc::mbar_init(&bars->ready[s], 4);
      tc::mbar_init(&bars->empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      tc::mbar_init(&bars->tfull[a], 1);
      tc::mbar_init(&bars->tempty[a], 8);
    }
    tc::mbar_init(&bars->joined, 8 * ranges);
    tc::mbar_init(&bars->drain, 1);
    bars->abort = 0;
    tc::fence_mbar_init();
    // (the kernel before, which made the codes of X, did not write the weights, and all before that one is complete)
    const int mt = p.by_n.quot(unit0), nt = unit0 - mt * p.tiles_n;
    for (int i = 0; i < min(WST, stages); ++i) load_w(i, i, nt);
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
    fewer_registers<40>();
    if (warp == 0) {
      if (tc::elect_one()) {  // ---------------- weights
        int i = 0;
        bool ok = true;
        for (int unit = unit0; unit < total && ok; unit += step) {
          int nt, mt;
          p.by_n.divmod(unit, mt, nt);
          for (int kb = 0; kb < stages; ++kb, ++i) {
            if (unit == unit0 && i < WST) continue;  // (on its way already)
            if (!(ok = tc::mbar_wait(&bars->wempty[i % WST], ((i / WST) & 1) ^ 1, abort, p.status))) break;
            load_w(i % WST, kb, nt);
          }
        }
        if (*abort)  // every copy issued has landed before shared memory goes to another block
          for (int j = max(0, i - WST); j < i; ++j) drain_wait(&bars->wfull[j % WST], (j / WST) & 1);
      }
    } else if (warp == 2) {
      if (tc::elect_one()) {  // ---------------- tokens
        int i = 0;
        bool ok = true;
        for (int unit = unit0; unit < total && ok; unit += step) {
          int nt, mt;
          p.by_n.divmod(unit, mt, nt);
          for (int kb = 0; kb < stages; ++kb, ++i) {
            const int xs = i % LST;
            if (!(ok = tc::mbar_wait(&bars->empty[xs], ((i / LST) & 1) ^ 1, abort, p.status))) break;
            tc::mbar_expect_tx(&bars->xfull[xs], C::X_STAGE);
#pragma unroll
            for (int h = 0; h < 2; ++h)  // (the second half of a last stage can lie past the end: zeros)
              tc::tma_load_2d(x_smem + xs * C::X_STAGE + h * (C::X_STAGE / 2), &tmX, &bars->xfull[xs], (st0 + kb) * LK + h * BK, mt * NTOK);
          }
        }
        if (*abort)
          for (int j = max(0, i - LST); j < i; ++j) drain_wait(&bars->xfull[j % LST], (j / LST) & 1);
      }
    } else if (warp == 1) {  // ---------------- products
      // The whole warp waits, one thread issues: behind a wait of its own a single thread issued four products in 450
      // clocks (the compiler no longer knows it to be alone and loops over every operand), this way in 210; those of 128
      // tokens take 256. One wait for eight products (the converters vouch for X): a wait is near 90 clocks.
      constexpr uint32_t IDESC = tc::idesc_f16(false, TM, NTOK);
      int i = 0, d = 0;
      bool ok = true;
      for (int unit = unit0; unit < total && ok; unit += step) {
        for (int c0 = 0; c0 < stages && ok; c0 += kExactStages, ++d) {
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->tempty[d & 1], ((d >> 1) & 1) ^ 1, abort, p.status));
          const int n = min(kExactStages, stages - c0);
          for (int b = 0; b < n && ok; ++b, ++i) {
            const int s = i % LST;
            ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->ready[s], (i / LST) & 1, abort, p.status));
            if (ok && tc::elect_one()) {
              tc::fence_after_sync();
              const uint64_t xd = tc::sdesc_kmajor_sw128(tc::smem_u32(x_smem + s * C::X_STAGE));
#pragma unroll
              for (int k = 0; k < LK / 16; ++k)
                tc::umma_f16_ts(tmem + (d & 1) * C::D_COLS, tmem + A_COL + s * (LK / 2) + k * 8,
                                tc::sdesc_advance(xd, (k & 3) * 32 + (k >> 2) * (C::X_STAGE / 2)), IDESC, b > 0 || k > 0 ? 1u : 0u);
              tc::umma_commit(&bars->empty[s]);
              if (b + 1 == n) tc::umma_commit(&bars->tfull[d & 1]);
            }
            __syncwarp();
          }
        }
      }
      if (tc::elect_one()) {
        tc::umma_commit(&bars->drain);
        drain_wait(&bars->drain, 0);
      }
    }
  } else if (warp < 12) {  // ---------------- epilogue: a warp has 32 channels and half of the tokens
    more_registers<C::EPI_REGS>();
    constexpr int HALF = NTOK / 2;
    const int quarter = warp & 3, row = quarter * 32 + lane, first = warp < 8 ? 0 : HALF;
    float* sx = token_scales + (warp - 4) * HALF;
    // two channels of a token in one store, where they lie together in a word
    const bool words = sizeof(T) == 2 && p.ldy % 2 == 0 && (reinterpret_cast<uintptr_t>(p.y) & 3) == 0;
    auto inside = [&](int64_t last) { return in_bounds(last, (p.M - 1) * p.ldy + p.N, p.status); };
    int d = 0;
    bool ok = true;
    for (int unit = unit0; unit < total && ok; unit += step) {
      int nt, mt;
      p.by_n.divmod(unit, mt, nt);
      const int n = nt * TM + row;
      const int64_t m0 = (int64_t)mt * NTOK + first;
      const int cols = (int)max((int64_t)0, min((int64_t)HALF, p.M - m0));
      const float wn = n < p.N ? __ldg(p.sw + n) : 0.f;
      __syncwarp();
      if (ranges == 1)
        for (int c = lane; c < cols; c += 32) sx[c] = p.sx[m0 + c];
      int acc[HALF];
#pragma unroll
      for (int c = 0; c < HALF; ++c) acc[c] = 0;
      for (int c0 = 0; c0 < stages; c0 += kExactStages, ++d) {
        if (!tc::mbar_wait(&bars->tfull[d & 1], (d >> 1) & 1, abort, p.status)) { ok = false; break; }
        tc::fence_after_sync();
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (d & 1) * C::D_COLS + first;
#pragma unroll
        for (int c = 0; c < HALF; c += 16) {  // (16 at a time: 32 would spill; of 8 columns the rest is not used)
          uint32_t r[16];
          __syncwarp();
          tmem_ld16(taddr + c, r);
          tc::tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16 && c + j < HALF; ++j) acc[c + j] += __float2int_rn(__uint_as_float(r[j]));
        }
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->tempty[d & 1]);
      }
      if (!ok) break;
      if (ranges > 1) {
        // Sums take the weights' place (all read: their products are done), every block adds up eight columns in turn.
        int* sums = reinterpret_cast<int*>(w_smem);  // [token, channel]
#pragma unroll
        for (int c = 0; c < HALF; ++c)
          if (c < cols) sums[(first + c) * TM + row] = acc[c];
        asm volatile("fence.acq_rel.cluster;" ::: "memory");
        __syncwarp();
        if (lane < ranges) tc::mbar_arrive_cluster(tc::mapa_shared(tc::smem_u32(&bars->joined), lane));
        if (!(ok = tc::mbar_wait_cluster(&bars->joined, 0, abort, p.status))) break;
        const int64_t t0 = (int64_t)mt * NTOK;
        const int all = (int)min((int64_t)NTOK, p.M - t0);
#pragma unroll 1
        for (int c0 = 8 * (rank + ranges * (warp < 8 ? 0 : 1)); c0 < all; c0 += 16 * ranges) {
          int sum[8] = {};
#pragma unroll 1
          for (int q = 0; q < ranges; ++q) {
            const uint32_t at = tc::mapa_shared(tc::smem_u32(sums + c0 * TM + row), q);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += c0 + j < all ? load_cluster(at + j * TM * 4) : 0;
          }
          if (n >= p.N) continue;
          T* y = static_cast<T*>(p.y) + (t0 + c0) * p.ldy + n;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (c0 + j < all && inside((t0 + c0 + j) * p.ldy + n)) y[j * p.ldy] = out_as<T>(__fmul_rn(__fmul_rn((float)sum[j], p.sx[t0 + c0 + j]), wn));
        }
        break;
      }
      __syncwarp();
      T* y = static_cast<T*>(p.y) + m0 * p.ldy + n;
      if (words && cols == HALF && (nt + 1) * TM <= p.N) {
        // lanes 2i and 2i + 1 exchange a token: the even one stores the first of two, the odd one the second
        const bool odd = lane & 1;
        y += odd ? p.ldy - 1 : 0;
#pragma unroll
        for (int c = 0; c < HALF; c += 2) {
          const float2 s = *reinterpret_cast<const float2*>(sx + c);
          const float u = __fmul_rn(__fmul_rn((float)acc[c], s.x), wn), v = __fmul_rn(__fmul_rn((float)acc[c + 1], s.y), wn);
          const float other = __shfl_xor_sync(0xffffffffu, odd ? u : v, 1);
          if constexpr (sizeof(T) == 2)
            if (inside(y - static_cast<T*>(p.y) + 1)) *reinterpret_cast<uint32_t*>(y) = odd ? pair_as(other, v, T()) : pair_as(u, other, T());
          y += 2 * p.ldy;
        }
      } else if (n < p.N) {
#pragma unroll
        for (int c = 0; c < HALF; ++c)
          if (c < cols && inside((m0 + c) * p.ldy + n)) y[c * p.ldy] = out_as<T>(__fmul_rn(__fmul_rn((float)acc[c], sx[c]), wn));
      }
    }
  } else {  // ---------------- converters
    fewer_registers<C::CONV_REGS>();
    const int quarter = warp & 3, grp = (warp - 12) >> 2, row = quarter * 32 + lane;
    int i = 0;
    bool ok = true;
    for (int unit = unit0; unit < total && ok; unit += step) {
      int nt, mt;
      p.by_n.divmod(unit, mt, nt);
      for (int kb = 0; kb < stages; ++kb, ++i) {
        if (i % C::GROUPS != grp) continue;
        const int ws = i % WST, s = i % LST;
        if (!tc::mbar_wait(&bars->wfull[ws], (i / WST) & 1, abort, p.status)) { ok = false; break; }
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const uint4* src = reinterpret_cast<const uint4*>(w_smem + ws * C::W_STAGE + (C::W_ROW == LK ? 0 : h * TM * BK) + row * C::W_ROW);
          uint4 v[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) v[c] = src[C::W_ROW == LK ? (4 * h + c) ^ (row & 7) : c ^ ((row >> 1) & 3)];  // TMA's swizzle of such rows
          if (h == 1) {
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bars->wempty[ws]);
          }
          uint32_t a[32];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            codes_h2(v[c].x, a[8 * c], a[8 * c + 1]);
            codes_h2(v[c].y, a[8 * c + 2], a[8 * c + 3]);
            codes_h2(v[c].z, a[8 * c + 4], a[8 * c + 5]);
            codes_h2(v[c].w, a[8 * c + 6], a[8 * c + 7]);
          }
          if (h == 0) {
            if (!tc::mbar_wait(&bars->empty[s], ((i / LST) & 1) ^ 1, abort, p.status)) { ok = false; break; }
            tc::fence_after_sync();
            __syncwarp();
          }
          tc::tmem_st32(tmem + ((uint32_t)(quarter * 32) << 16) + A_COL + s * (LK / 2) + h * 32, a);
        }
        if (!ok) break;
        tc::tmem_st_wait();
        tc::fence_before_sync();
        if (quarter == 0 && !tc::mbar_wait(&bars->xfull[s], (i / LST) & 1, abort, p.status)) { ok = false; break; }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->ready[s]);
      }
      if (!ok) break;
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

bool make_map(CUtensorMap* m, CUtensorMapDataType type, const void* base, uint64_t inner, uint64_t outer,
              uint64_t pitch_bytes, uint32_t box_inner, uint32_t box_outer, CUtensorMapSwizzle swizzle) {
  auto fn = encode_fn();
  if (fn == nullptr || (reinterpret_cast<uintptr_t>(base) & 15u) || pitch_bytes % 16) return false;
  cuuint64_t dims[2] = {inner, outer}, strides[1] = {pitch_bytes};
  cuuint32_t box[2] = {box_inner, box_outer}, estr[2] = {1, 1};
  return fn(m, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tokens of a tile: the smallest that holds them all, 128 at most.
int tile_tokens(int64_t M) { return M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128; }

struct Scratch {
  size_t sx, xh, total;
};
Scratch plan_scratch(int64_t M, int N, int K) {
  const int64_t Kp = (K + 63) / 64 * 64;
  Scratch s;
  s.sx = 0;
  s.xh = ((size_t)M * 4 + 255) / 256 * 256;
  s.total = s.xh + (size_t)M * Kp * 2;
  return s;
}

// K ranges of a tile: as many as leave no cluster waiting for another to end, of 1024 and more each. A cluster costs 2 us
// (its launch, the meeting of its blocks, the sums' way), a stage of 128 a quarter of one: 64 tokens x 6144 x 4096 take
// 14.1 us in two ranges and 15.6 in one, x 2304 x 768 9.3 in three and 6.8 in one.
template <class C, class Kernel>
int ranges_of(Kernel kern, const LinParams& p, int sms, int dev, Found& fit) {
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
  for (int s = (int)std::min<int64_t>({kMaxRanges, sms / tiles, p.stages / kExactStages}); s > 1; --s) {
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

template <class TX>
cudaError_t quantize_tokens(const TokenParams& t, int sms, cudaStream_t st) {
  return launch_after(quantize_tokens_kernel<TX>, (unsigned)std::min<int64_t>(t.M, (int64_t)sms * 8), 256, 0, st, t);
}

template <class T, int NTOK>
cudaError_t launch_as(const CUtensorMap& tw, const CUtensorMap& tx, LinParams p, int sms, cudaStream_t st) {
  using C = Cfg<NTOK>;
  auto kern = qlinear_kernel<T, NTOK>;
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
template <class T>
cudaError_t launch_tokens(const CUtensorMap& tw, const CUtensorMap& tx, const LinParams& p, int ntok, int sms, cudaStream_t st) {
  return ntok == 16   ? launch_as<T, 16>(tw, tx, p, sms, st)
         : ntok == 32 ? launch_as<T, 32>(tw, tx, p, sms, st)
         : ntok == 64 ? launch_as<T, 64>(tw, tx, p, sms, st)
                      : launch_as<T, 128>(tw, tx, p, sms, st);
}

}  // namespace

size_t quantized_linear_scratch(int64_t M, int N, int K) { return plan_scratch(M, N, K).total; }

cudaError_t launch_quantized_linear(const QLinearArgs& a, int sms, cudaStream_t st) {
  const Scratch s = plan_scratch(a.M, a.N, a.K);
  char* w = static_cast<char*>(a.ws);
  const int ntok = tile_tokens(a.M), Kp = (a.K + 63) / 64 * 64;
  LinParams p{};
  p.M = a.M;
  p.N = a.N;
  p.ldy = a.ldy;
  p.stages = (Kp + LK - 1) / LK;
  p.tiles_n = (a.N + TM - 1) / TM;
  p.tiles_m = (int)((a.M + ntok - 1) / ntok);
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
  if (tiles >= (int64_t)1 << 29) return cudaErrorInvalidValue;
  p.by_n = FastDiv(p.tiles_n);
  p.sx = reinterpret_cast<const float*>(w + s.sx);
  p.sw = a.w_scales;
  p.y = a.y;
  p.status = a.status;
  TokenParams t{};
  t.x = a.x;
  t.ldx = a.ldx;
  t.M = a.M;
  t.K = a.K;
  t.Kp = Kp;
  t.xh = reinterpret_cast<half_t*>(w + s.xh);
  t.sx = reinterpret_cast<float*>(w + s.sx);
  t.status = a.status;
  CUtensorMap tw, tx;
  if (!make_map(&tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.codes, a.K, a.N, a.K, ntok == 128 ? Cfg<128>::W_ROW : Cfg<16>::W_ROW, TM,
                ntok == 128 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B) ||
      !make_map(&tx, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, t.xh, Kp, a.M, (uint64_t)Kp * 2, BK, ntok, CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  const cudaError_t e = a.x_type == JAB_FP16 ? quantize_tokens<half_t>(t, sms, st) : quantize_tokens<bf16_t>(t, sms, st);
  if (e != cudaSuccess) return e;
  return a.y_type == JAB_FP16   ? launch_tokens<half_t>(tw, tx, p, ntok, sms, st)
         : a.y_type == JAB_BF16 ? launch_tokens<bf16_t>(tw, tx, p, ntok, sms, st)
                                : launch_tokens<float>(tw, tx, p, ntok, sms, st);
}

}  // namespace jab
