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
// are: TMA brings a 128 x 64 tile of codes to shared memory, converter warps turn it into fp16 in tensor memory (a
// byte under the exponent of 1024, less 1152), and the products take it from there as their A operand. One layout
// serves one token and thousands; the product is one of two kernels:
//   few tiles   one tile a block, K split over a cluster whose blocks add their sums through shared memory; all
//               accumulators of a block (1024 of K each) stay in tensor memory to the end
//   many tiles  persistent blocks, two accumulators in turn, sums in registers
#include <cudaTypedefs.h>

#include <algorithm>

#include "kernels.h"
#include "quotient.cuh"
#include "serve.h"
#include "tc.cuh"

namespace jab {
namespace {

constexpr int TM = 128, BK = 64;      // output channels of a tile, K of a block
constexpr int kExactBlocks = 16;      // K blocks that one accumulator may take (1024 products)
constexpr int AST = 8;                // A buffers in tensor memory and X stages
constexpr int W_BYTES = TM * BK;
constexpr int THREADS = 640;

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
// the codes, what is longer is read again.
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
  int N, k_blocks, tiles_n, tiles_m;
  FastDiv by_n;
  const float *sx, *sw;
  void* y;
  int* status;
};

constexpr int LK = 2 * BK, LST = 4;  // many tiles: K of a stage, and stages of X and of A
template <int NTOK>
struct Cfg {
  static constexpr int WST = NTOK == 128 ? 4 : 8;  // stages of weight codes
  static constexpr int W_STAGE = TM * LK, X_STAGE = NTOK * LK * 2;
  static constexpr int D_COLS = NTOK < 32 ? 32 : NTOK;
  static constexpr int SMEM = WST * W_STAGE + LST * X_STAGE + 1024 + 512 + 8 * (NTOK / 2) * 4;
};

struct Bars {
  uint64_t wfull[8], wempty[8], xfull[LST], ready[LST], empty[LST], tfull[2], tempty[2], drain;
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

template <class T, int NTOK>
__global__ void __launch_bounds__(THREADS, 1)
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
  const int total = p.tiles_n * p.tiles_m, stages = (p.k_blocks + 1) / 2;
  volatile int* abort = &bars->abort;
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
    tc::mbar_init(&bars->drain, 1);
    bars->abort = 0;
    tc::fence_mbar_init();
    tc::prefetch_tmap(&tmW);
    tc::prefetch_tmap(&tmX);
  }
  if (warp == 1) {
    tc::tmem_alloc(&bars->tmem_base, 512);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
  stream_order();

  if (warp < 4) {
    fewer_registers<40>();
    if (warp == 0 && tc::elect_one()) {  // ---------------- TMA producer
      int i = 0;
      bool ok = true;
      for (int unit = blockIdx.x; unit < total && ok; unit += gridDim.x) {
        int nt, mt;
        p.by_n.divmod(unit, mt, nt);
        for (int kb = 0; kb < stages; ++kb, ++i) {
          const int ws = i % WST, xs = i % LST;
          if (!tc::mbar_wait(&bars->wempty[ws], ((i / WST) & 1) ^ 1, abort, p.status)) { ok = false; break; }
          tc::mbar_expect_tx(&bars->wfull[ws], C::W_STAGE);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            tc::tma_load_2d(w_smem + ws * C::W_STAGE + h * W_BYTES, &tmW, &bars->wfull[ws], kb * LK + h * BK, nt * TM);
          if (!tc::mbar_wait(&bars->empty[xs], ((i / LST) & 1) ^ 1, abort, p.status)) {
            drain_wait(&bars->wfull[ws], (i / WST) & 1);
            ok = false;
            break;
          }
          tc::mbar_expect_tx(&bars->xfull[xs], C::X_STAGE);
#pragma unroll
          for (int h = 0; h < 2; ++h)  // (the second half of a last stage can lie past the end: zeros)
            tc::tma_load_2d(x_smem + xs * C::X_STAGE + h * (C::X_STAGE / 2), &tmX, &bars->xfull[xs], kb * LK + h * BK, mt * NTOK);
        }
      }
      if (*abort) {  // every copy issued has landed before shared memory goes to another block
        for (int j = max(0, i - WST); j < i; ++j) drain_wait(&bars->wfull[j % WST], (j / WST) & 1);
        for (int j = max(0, i - LST); j < i; ++j) drain_wait(&bars->xfull[j % LST], (j / LST) & 1);
      }
    } else if (warp == 1) {  // ---------------- products
      // The whole warp waits, one thread issues: behind a wait of its own a single thread issued four products in 450
      // clocks (the compiler no longer knows it to be alone and loops over every operand), this way in 210; they take 256.
      // One wait for eight products (the converters vouch for X): a wait is near 90 clocks.
      constexpr uint32_t IDESC = tc::idesc_f16(false, TM, NTOK);
      int i = 0, d = 0;
      bool ok = true;
      for (int unit = blockIdx.x; unit < total && ok; unit += gridDim.x) {
        for (int c0 = 0; c0 < stages && ok; c0 += kExactBlocks / 2, ++d) {
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->tempty[d & 1], ((d >> 1) & 1) ^ 1, abort, p.status));
          const int n = min(kExactBlocks / 2, stages - c0);
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
    more_registers<128>();
    constexpr int HALF = NTOK / 2;
    const int quarter = warp & 3, row = quarter * 32 + lane, first = warp < 8 ? 0 : HALF;
    float* sx = token_scales + (warp - 4) * HALF;
    // two channels of a token in one store, where they lie together in a word
    const bool words = sizeof(T) == 2 && p.ldy % 2 == 0 && (reinterpret_cast<uintptr_t>(p.y) & 3) == 0;
    int d = 0;
    bool ok = true;
    for (int unit = blockIdx.x; unit < total && ok; unit += gridDim.x) {
      int nt, mt;
      p.by_n.divmod(unit, mt, nt);
      const int n = nt * TM + row;
      const int64_t m0 = (int64_t)mt * NTOK + first;
      const int cols = (int)max((int64_t)0, min((int64_t)HALF, p.M - m0));
      const float wn = n < p.N ? __ldg(p.sw + n) : 0.f;
      __syncwarp();
      for (int c = lane; c < cols; c += 32) sx[c] = p.sx[m0 + c];
      int acc[HALF];
#pragma unroll
      for (int c = 0; c < HALF; ++c) acc[c] = 0;
      for (int c0 = 0; c0 < stages; c0 += kExactBlocks / 2, ++d) {
        if (!tc::mbar_wait(&bars->tfull[d & 1], (d >> 1) & 1, abort, p.status)) { ok = false; break; }
        tc::fence_after_sync();
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (d & 1) * C::D_COLS + first;
#pragma unroll
        for (int c = 0; c < HALF; c += 32) {
          uint32_t r[32];  // (8 or 16 columns: the rest of the 32 is not used)
          __syncwarp();
          tc::tmem_ld32(taddr + c, r);
          tc::tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32 && c + j < HALF; ++j) acc[c + j] += __float2int_rn(__uint_as_float(r[j]));
        }
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->tempty[d & 1]);
      }
      if (!ok) break;
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
          if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(y) = odd ? pair_as(other, v, T()) : pair_as(u, other, T());
          y += 2 * p.ldy;
        }
      } else if (n < p.N) {
#pragma unroll
        for (int c = 0; c < HALF; ++c)
          if (c < cols) y[c * p.ldy] = out_as<T>(__fmul_rn(__fmul_rn((float)acc[c], sx[c]), wn));
      }
    }
  } else {  // ---------------- converters
    fewer_registers<88>();
    const int quarter = warp & 3, grp = (warp - 12) >> 2, row = quarter * 32 + lane;
    int i = 0;
    bool ok = true;
    for (int unit = blockIdx.x; unit < total && ok; unit += gridDim.x) {
      int nt, mt;
      p.by_n.divmod(unit, mt, nt);
      for (int kb = 0; kb < stages; ++kb, ++i) {
        if ((i & 1) != grp) continue;
        const int ws = i % WST, s = i % LST;
        if (!tc::mbar_wait(&bars->wfull[ws], (i / WST) & 1, abort, p.status)) { ok = false; break; }
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const uint4* src = reinterpret_cast<const uint4*>(w_smem + ws * C::W_STAGE + h * W_BYTES + row * BK);
          uint4 v[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) v[c] = src[c ^ ((row >> 1) & 3)];  // TMA's 64-byte swizzle
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
  tc::fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------ few tiles
// Blocks of a cluster take K ranges of one tile. Loads of weights start before the codes of X are there (the weights
// were not written by the kernel before this one). Converters (16 warps, four groups that take K blocks in turn) become
// the epilogue: 8 columns at a time, the sums of a range's accumulators go to the shared memory of the block that has
// those columns, are added there and scaled. Loops over 8 columns rather than unrolled tiles: these calls are a few
// microseconds, and a cold SM fetches their code (unrolled, with the parts added in global memory: 14 us where the
// launch with everything in it takes 7, 37 tokens x 2304 x 768).
// FUSED: up to 16 tokens, whose rows every block quantises for itself (four more warps), its own K range into shared
// memory: the first launch and its end would be a third of the time.
constexpr int S_GROUPS = 4, S_THREADS = 32 * (4 + 4 * S_GROUPS), kMaxRanges = 8, kMaxA = 8, kFusedBlocks = 24;

template <int NTOK, bool FUSED>
struct SCfg {
  static constexpr int WST = NTOK <= 32 ? 16 : NTOK == 64 ? 10 : 8, XST = FUSED ? kFusedBlocks : NTOK == 128 ? 4 : AST;  // stages of weights and tokens
  static constexpr int X_BYTES = NTOK * BK * 2;
  static constexpr int D_COLS = NTOK < 32 ? 32 : NTOK, D_BUFS = NTOK == 128 ? 2 : 4, OCTS = NTOK / 8;
  static constexpr int SUM_BYTES = (OCTS + kMaxRanges - 1) * 8 * TM * 4;  // >= ranges * ceil(OCTS / ranges) octets
  static constexpr int SMEM = WST * W_BYTES + XST * X_BYTES + SUM_BYTES + 1024 + 1024;
};
static_assert(SCfg<128, false>::SMEM <= 226 * 1024 && SCfg<64, false>::SMEM <= 226 * 1024 && SCfg<32, false>::SMEM <= 226 * 1024 && SCfg<16, true>::SMEM <= 226 * 1024, "shared memory budget");

struct SBars {
  uint64_t wfull[16], wempty[16], xfull[AST], xempty[AST], afull[kMaxA], aempty[kMaxA], done, xready;
  uint32_t tmem_base;
  int abort;
  float sx[16];
};
static_assert(sizeof(SBars) <= 1024, "barrier block");

// 32 lanes x 8 columns.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void store_cluster(uint32_t at, int v) { asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }

// Rows of X (up to 16, by 128 threads): scales into sx, codes of K blocks [kb0, kb0 + n_kb) into x_smem.
template <class T>
__device__ __forceinline__ void quantize_range(const TokenParams& t, int kb0, int n_kb, uint8_t* x_smem, float* sx, int tid, int warp, int lane) {
  const int n8 = t.K / 8;
  // a warp has rows warp, warp + 4, ...
#pragma unroll 1
  for (int m = warp; m < t.M; m += 4) {
    const uint4* row = reinterpret_cast<const uint4*>(static_cast<const T*>(t.x) + m * t.ldx);
    uint32_t big = 0;
#pragma unroll 1
    for (int i0 = lane; i0 < n8; i0 += 32 * 8) {
      uint4 u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = i0 + 32 * j < n8 ? __ldg(row + i0 + 32 * j) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int j = 0; j < 8; ++j) big = max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(big, u[j].x), u[j].y), u[j].z), u[j].w);
    }
    big = __reduce_max_sync(0xffffffffu, max(big & 0xffffu, big >> 16));
    const float s = row_scale<T>(big);
    if (lane == 0) {
      sx[m] = s;
      if (!(s >= 0.f)) report(t.status, JAB_ERR_NONFINITE);
    }
#pragma unroll 1
    for (int i = lane; i < n_kb * 8; i += 32) {
      const int k8 = kb0 * 8 + i;
      const uint4 c = k8 < n8 ? row_codes<T>(__ldg(row + k8), s) : make_uint4(0u, 0u, 0u, 0u);
      *reinterpret_cast<uint4*>(x_smem + (i >> 3) * (16 * BK * 2) + m * 128 + (((i & 7) ^ (m & 7)) << 4)) = c;
    }
  }
}

template <class T, class TX, int NTOK, bool FUSED>
__global__ void __launch_bounds__(FUSED ? S_THREADS + 128 : S_THREADS, 1)
    qlinear_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ LinParams p,
                       const __grid_constant__ TokenParams tok, int ranges) {
  using C = SCfg<NTOK, FUSED>;
  constexpr int WST = C::WST, XST = C::XST, XB = C::X_BYTES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* w_smem = smem;
  uint8_t* x_smem = smem + WST * W_BYTES;
  int* sums = reinterpret_cast<int*>(x_smem + XST * XB);  // [range, own octet, 8, TM]
  SBars* bars = reinterpret_cast<SBars*>(x_smem + XST * XB + C::SUM_BYTES);
  const int warp = tc::warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)tc::cluster_ctarank(), unit = blockIdx.x / ranges;
  const int mt = p.by_n.quot(unit), nt = unit - mt * p.tiles_n;
  const int kb0 = p.k_blocks * rank / ranges, n_kb = p.k_blocks * (rank + 1) / ranges - kb0;
  // The four products of a K block go to D_BUFS accumulators in turn; A takes the columns behind them
  constexpr uint32_t a_col = C::D_BUFS * C::D_COLS;
  constexpr int na = kMaxA;
  constexpr bool SAME = XST == na;  // X's stages are free when A's are
  static_assert(a_col + na * 32 <= 512, "tensor memory");
  volatile int* abort = &bars->abort;
  if (threadIdx.x == 0) {
    for (int s = 0; s < WST; ++s) {
      tc::mbar_init(&bars->wfull[s], 1);
      tc::mbar_init(&bars->wempty[s], 4);
    }
    for (int s = 0; s < AST; ++s) {
      tc::mbar_init(&bars->xfull[s], 1);
      tc::mbar_init(&bars->xempty[s], 1);
    }
    for (int s = 0; s < kMaxA; ++s) {
      tc::mbar_init(&bars->afull[s], 4);
      tc::mbar_init(&bars->aempty[s], 1);
    }
    tc::mbar_init(&bars->done, 1);
    tc::mbar_init(&bars->xready, 4);
    bars->abort = 0;
    tc::fence_mbar_init();
    if (FUSED) stream_order();  // (weights too may have been written by the kernel before)
    for (int i = 0; i < min(WST, n_kb); ++i) {
      tc::mbar_expect_tx(&bars->wfull[i], W_BYTES);
      tc::tma_load_2d(w_smem + i * W_BYTES, &tmW, &bars->wfull[i], (kb0 + i) * BK, nt * TM);
    }
  }
  if (warp == 1) {
    tc::tmem_alloc(&bars->tmem_base, 512);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
  stream_order();

  if (warp == 0) {
    if (tc::elect_one()) {  // ---------------- TMA producer
      int w_next = min(WST, n_kb), i = 0;
      for (; i < n_kb; ++i) {
        if (!FUSED) {
          const int xs = i % XST;
          if (!tc::mbar_wait(SAME ? &bars->aempty[xs] : &bars->xempty[xs], ((i / XST) & 1) ^ 1, abort, p.status)) break;
          tc::mbar_expect_tx(&bars->xfull[xs], XB);
          tc::tma_load_2d(x_smem + xs * XB, &tmX, &bars->xfull[xs], (kb0 + i) * BK, mt * NTOK);
        }
        if (w_next < n_kb && w_next < i + WST) {
          const int ws = w_next % WST;
          if (!tc::mbar_wait(&bars->wempty[ws], ((w_next / WST) & 1) ^ 1, abort, p.status)) {
            ++i;
            break;
          }
          tc::mbar_expect_tx(&bars->wfull[ws], W_BYTES);
          tc::tma_load_2d(w_smem + ws * W_BYTES, &tmW, &bars->wfull[ws], (kb0 + w_next) * BK, nt * TM);
          ++w_next;
        }
      }
      if (*abort) {  // every copy issued has landed before shared memory goes to another block
        for (int j = max(0, w_next - WST); j < w_next; ++j) drain_wait(&bars->wfull[j % WST], (j / WST) & 1);
        if (!FUSED)
          for (int j = max(0, i - XST); j < i; ++j) drain_wait(&bars->xfull[j % XST], (j / XST) & 1);
      }
    }
  } else if (warp == 1) {  // ---------------- products (the whole warp waits, as below)
    constexpr uint32_t IDESC = tc::idesc_f16(false, TM, NTOK);
    bool ok = !FUSED || __all_sync(0xffffffffu, tc::mbar_wait(&bars->xready, 0, abort, p.status));
    for (int i = 0; i < n_kb && ok; ++i) {
      const int s = i % na, xs = i % XST;
      ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->afull[s], (i / na) & 1, abort, p.status));
      if (ok && tc::elect_one()) {
        tc::fence_after_sync();
        const uint64_t xd = tc::sdesc_kmajor_sw128(tc::smem_u32(x_smem + xs * XB));
#pragma unroll
        for (int k = 0; k < BK / 16; ++k)
          tc::umma_f16_ts(tmem + k % C::D_BUFS * C::D_COLS, tmem + a_col + s * 32 + k * 8, tc::sdesc_advance(xd, k * 32), IDESC,
                          i > 0 || k >= C::D_BUFS ? 1u : 0u);
        tc::umma_commit(&bars->aempty[s]);
        if (!FUSED && !SAME) tc::umma_commit(&bars->xempty[xs]);
      }
      __syncwarp();
    }
    if (tc::elect_one()) {
      tc::umma_commit(&bars->done);
      drain_wait(&bars->done, 0);
    }
  } else if (FUSED && warp >= 4 + 4 * S_GROUPS) {  // ---------------- tokens
    quantize_range<TX>(tok, kb0, n_kb, x_smem, bars->sx, threadIdx.x - S_THREADS, warp - 4 - 4 * S_GROUPS, lane);
    tc::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(&bars->xready);
  } else if (warp >= 4) {  // ---------------- converters, then epilogue
    const int quarter = warp & 3, grp = (warp - 4) >> 2, row = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    bool ok = true;
    for (int i = grp; i < n_kb && ok; i += S_GROUPS) {
      const int ws = i % WST, s = i % na;
      if (!(ok = tc::mbar_wait(&bars->wfull[ws], (i / WST) & 1, abort, p.status))) break;
      const uint4* src = reinterpret_cast<const uint4*>(w_smem + ws * W_BYTES + row * BK);
      uint4 v[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = src[c ^ ((row >> 1) & 3)];  // TMA's 64-byte swizzle
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars->wempty[ws]);
      uint32_t a[32];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        codes_h2(v[c].x, a[8 * c], a[8 * c + 1]);
        codes_h2(v[c].y, a[8 * c + 2], a[8 * c + 3]);
        codes_h2(v[c].z, a[8 * c + 4], a[8 * c + 5]);
        codes_h2(v[c].w, a[8 * c + 6], a[8 * c + 7]);
      }
      if (!(ok = tc::mbar_wait(&bars->aempty[s], ((i / na) & 1) ^ 1, abort, p.status))) break;
      tc::fence_after_sync();
      __syncwarp();
      tc::tmem_st32(tmem + lanes + a_col + s * 32, a);
      tc::tmem_st_wait();
      tc::fence_before_sync();
      // (vouches for X: one wait less for the warp that issues)
      if (!FUSED && quarter == 0 && !(ok = tc::mbar_wait(&bars->xfull[i % XST], (i / XST) & 1, abort, p.status))) break;
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars->afull[s]);
    }
    ok = ok && tc::mbar_wait(&bars->done, 0, abort, p.status);
    tc::fence_after_sync();
    const int own = (C::OCTS + ranges - 1) / ranges;
#pragma unroll 1
    for (int oct = grp; oct < C::OCTS && ok && (int64_t)mt * NTOK + oct * 8 < p.M; oct += S_GROUPS) {
      int acc[8] = {};
#pragma unroll 1
      for (int b = 0; b < C::D_BUFS; ++b) {
        uint32_t v[8];
        __syncwarp();
        tmem_ld8(tmem + lanes + b * C::D_COLS + oct * 8, v);
        tc::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += __float2int_rn(__uint_as_float(v[j]));
      }
      // to the block that has these columns
      const int place = oct / ranges, owner = oct - place * ranges;
      const uint32_t at = tc::mapa_shared(tc::smem_u32(sums + ((rank * own + place) * 8) * TM + row), owner);
#pragma unroll
      for (int j = 0; j < 8; ++j) store_cluster(at + j * TM * 4, acc[j]);
    }
  }
  tc::fence_before_sync();
  __syncwarp();
  tc::cluster_sync();  // every block's sums are where they belong
  tc::fence_after_sync();
  if (warp >= 4 && warp < 4 + 4 * S_GROUPS) {
    const int quarter = warp & 3, grp = (warp - 4) >> 2, row = quarter * 32 + lane, n = nt * TM + row;
    const int own = (C::OCTS + ranges - 1) / ranges;
    const float wn = n < p.N ? __ldg(p.sw + n) : 0.f;
#pragma unroll 1
    for (int place = grp; place < own; place += S_GROUPS) {
      const int oct = place * ranges + rank;
      const int64_t m0 = (int64_t)mt * NTOK + oct * 8;
      if (oct >= C::OCTS || m0 >= p.M) break;
      int acc[8] = {};
#pragma unroll 1
      for (int q = 0; q < ranges; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += sums[((q * own + place) * 8 + j) * TM + row];
      if (n >= p.N) continue;
      T* y = static_cast<T*>(p.y) + m0 * p.ldy + n;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (m0 + j < p.M) y[j * p.ldy] = out_as<T>(__fmul_rn(__fmul_rn((float)acc[j], FUSED ? bars->sx[m0 + j] : __ldcg(p.sx + m0 + j)), wn));
    }
  }
  __syncthreads();
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

// K ranges of the few-tiles kernel: as many as leave no cluster waiting for another to end; 0: the other kernel's case.
template <class C, class Kernel>
int ranges_of(Kernel kern, int threads, const LinParams& p, int sms, int (&fit)[kMaxRanges + 1]) {
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
  if (tiles > sms) return 0;
  for (int s = (int)std::min<int64_t>({kMaxRanges, sms / tiles, std::max(1, p.k_blocks / 2)}); s >= 1; --s) {
    if ((p.k_blocks + s - 1) / s > kExactBlocks * C::D_BUFS) continue;  // (1024 products an accumulator)
    if (fit[s] == 0) {  // clusters of that many blocks that are resident at once
      cudaLaunchConfig_t cfg = {};
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = s;
      at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
      cfg.gridDim = dim3((unsigned)(sms / s * s));
      cfg.blockDim = dim3(threads);
      cfg.dynamicSmemBytes = C::SMEM;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      int n = 0;
      if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) cudaGetLastError();
      fit[s] = std::max(n, s == 1 ? sms : 1);
    }
    if (tiles <= fit[s]) return s;
  }
  return 0;
}

// The few-tiles kernel, if it is its case: *done says so.
template <class T, class TX, int NTOK, bool FUSED>
cudaError_t launch_few(const CUtensorMap& tw, const CUtensorMap& tx, const LinParams& p, const TokenParams& t, int sms, cudaStream_t st, bool* done) {
  using C = SCfg<NTOK, FUSED>;
  auto kern = qlinear_few_kernel<T, TX, NTOK, FUSED>;
  constexpr int threads = FUSED ? S_THREADS + 128 : S_THREADS;
  static bool attr_set = false;
  static int fit[kMaxRanges + 1] = {};
  if (!attr_set) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e != cudaSuccess) return e;
    attr_set = true;
  }
  const int ranges = ranges_of<C>(kern, threads, p, sms, fit);
  *done = ranges > 0 && !(FUSED && (p.k_blocks + ranges - 1) / ranges > kFusedBlocks);
  if (!*done) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ranges;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)((int64_t)p.tiles_n * p.tiles_m * ranges));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, tw, tx, p, t, ranges);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}

template <class TX>
cudaError_t quantize_tokens(const TokenParams& t, int sms, cudaStream_t st) {
  return launch_after(quantize_tokens_kernel<TX>, (unsigned)std::min<int64_t>(t.M, (int64_t)sms * 8), 256, 0, st, t);
}

template <class T, class TX, int NTOK>
cudaError_t launch_as(const CUtensorMap& tw, const CUtensorMap& tx, const LinParams& p, const TokenParams& t, int sms, cudaStream_t st) {
  bool done = false;
  cudaError_t e;
  if constexpr (NTOK == 16) {
    e = launch_few<T, TX, NTOK, true>(tw, tx, p, t, sms, st, &done);
    if (e != cudaSuccess || done) return e;
  }
  if ((e = quantize_tokens<TX>(t, sms, st)) != cudaSuccess) return e;
  e = launch_few<T, half_t, NTOK, false>(tw, tx, p, t, sms, st, &done);
  if (e != cudaSuccess || done) return e;
  auto many = qlinear_kernel<T, NTOK>;
  static bool attr_set = false;
  if (!attr_set) {
    e = cudaFuncSetAttribute(many, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<NTOK>::SMEM);
    if (e != cudaSuccess) return e;
    attr_set = true;
  }
  return launch_after(many, (unsigned)std::min<int64_t>((int64_t)p.tiles_n * p.tiles_m, sms), THREADS, Cfg<NTOK>::SMEM, st, tw, tx, p);
}
template <class T, class TX>
cudaError_t launch_tokens(const CUtensorMap& tw, const CUtensorMap& tx, const LinParams& p, const TokenParams& t, int ntok, int sms, cudaStream_t st) {
  return ntok == 16   ? launch_as<T, TX, 16>(tw, tx, p, t, sms, st)
         : ntok == 32 ? launch_as<T, TX, 32>(tw, tx, p, t, sms, st)
         : ntok == 64 ? launch_as<T, TX, 64>(tw, tx, p, t, sms, st)
                      : launch_as<T, TX, 128>(tw, tx, p, t, sms, st);
}
template <class TX>
cudaError_t launch_out(const CUtensorMap& tw, const CUtensorMap& tx, const LinParams& p, const TokenParams& t, jab_dtype y, int ntok, int sms, cudaStream_t st) {
  return y == JAB_FP16   ? launch_tokens<half_t, TX>(tw, tx, p, t, ntok, sms, st)
         : y == JAB_BF16 ? launch_tokens<bf16_t, TX>(tw, tx, p, t, ntok, sms, st)
                         : launch_tokens<float, TX>(tw, tx, p, t, ntok, sms, st);
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
  p.k_blocks = Kp / BK;
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
  if (!make_map(&tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.codes, a.K, a.N, a.K, BK, TM, CU_TENSOR_MAP_SWIZZLE_64B) ||
      !make_map(&tx, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, t.xh, Kp, a.M, (uint64_t)Kp * 2, BK, ntok, CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  return a.x_type == JAB_FP16 ? launch_out<half_t>(tw, tx, p, t, a.y_type, ntok, sms, st) : launch_out<bf16_t>(tw, tx, p, t, a.y_type, ntok, sms, st);
}

}  // namespace jab
