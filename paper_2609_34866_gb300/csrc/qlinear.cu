// Product in 8-bit integers with a scale per token and per output channel, on the tensor cores of sm_103a:
//
//   y[m, n] = s_m w_n sum_k qx[m, k] qw[n, k],   s_m = fl32(max|x_m| / 127), qx = clip(rint(fl32(x / s_m)))
//
// The chip has no fast integer tensor form. Whole numbers up to 2^11 are exact in fp16, their products in the
// fp32 accumulator, and so is their sum while it stays below 2^24: 1024 products of codes at most (127^2 *
// 1024 < 2^24, and 128^2 * 1024 = 2^24). The accumulator is therefore read out every 1024 of K and added up in
// int32: the sum is exact, in any order of its parts, at the fp16 rate of the tensor cores.
//
// Two launches: the rows of X become codes (held in fp16, the operand's type) and scales; then a persistent
// kernel with the output channels on the accumulator's 128 lanes and the tokens on its columns. The weights
// travel as the bytes that they are: TMA brings a 128 x 64 tile of codes to shared memory, converter warps
// turn it into fp16 in tensor memory (a byte under the exponent of 1024, less 1152), and the products take
// it from there as their A operand. One layout serves one token and thousands: what changes with M is the
// number of columns and the K range of a unit.
//   warp 0        TMA producer
//   warp 1        tensor memory owner, issues the products
//   warps 4..7    epilogue: accumulators to int32 sums in registers, scaling, output
//   warps 8..15   converters, two groups that take K blocks in turn
#include <cudaTypedefs.h>

#include <algorithm>

#include "kernels.h"
#include "serve.h"
#include "tc.cuh"

namespace jab {
namespace {

constexpr int TM = 128, BK = 64;      // output channels of a tile, K of a block
constexpr int kExactBlocks = 16;      // K blocks that one accumulator may take (1024 products)
constexpr int AST = 8;                // A buffers in tensor memory and X stages
constexpr int W_BYTES = TM * BK;
constexpr int THREADS = 512;

// ------------------------------------------------------------------ tokens to codes
struct TokenParams {
  const void* x;
  int64_t ldx, M;
  int K, Kp;
  half_t* xh;     // [M, Kp]
  float* sx;      // [M]
  int* zero;      // the product's partial sums and counters, to 0
  int64_t n_zero;
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

// A block per row; the row's first KEEP chunks of 8 elements a thread stay in registers between the maximum and
// the codes, what is longer is read again.
template <class T>
__global__ void __launch_bounds__(256) quantize_tokens_kernel(const __grid_constant__ TokenParams p) {
  constexpr int KEEP = 2;
  __shared__ uint32_t top[8];
  stream_order();
  const int tid = threadIdx.x, n8 = p.K / 8, n8p = p.Kp / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < p.n_zero; i += (int64_t)gridDim.x * 256) p.zero[i] = 0;
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
    const bool fine = big < (std::is_same<T, half_t>::value ? kHalfInf : kBf16Inf);
    const float a = std::is_same<T, half_t>::value ? __half2float(__ushort_as_half((unsigned short)big)) : __uint_as_float(big << 16);
    const float s = fine ? __fdiv_rn(a, 127.f) : __uint_as_float(0x7fc00000u);
    if (tid == 0) {
      p.sx[m] = s;
      if (!fine) report(p.status, JAB_ERR_NONFINITE);
    }
    uint4* out = reinterpret_cast<uint4*>(p.xh + m * p.Kp);
    auto put = [&](int i, const uint4& u) {
      float v[8];
      unpack8<T>(u, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float r = fminf(fmaxf(rintf(__fdiv_rn(v[j], s)), -127.f), 127.f);
        v[j] = fine && s > 0.f ? r : 0.f;
      }
      out[i] = make_uint4(tc::pack_half2(v[0], v[1]), tc::pack_half2(v[2], v[3]), tc::pack_half2(v[4], v[5]), tc::pack_half2(v[6], v[7]));
    };
#pragma unroll
    for (int c = 0; c < KEEP; ++c)
      if (c * 256 + tid < n8) put(c * 256 + tid, keep[c]);
    for (int i = KEEP * 256 + tid; i < n8; i += 256) put(i, __ldg(row + i));
    for (int i = n8 + tid; i < n8p; i += 256) out[i] = make_uint4(0u, 0u, 0u, 0u);
  }
}

// ------------------------------------------------------------------ the product
struct LinParams {
  int64_t M, ldy;
  int N, k_blocks, tiles_n, tiles_m, splits;
  FastDiv by_tiles, by_n;
  const float *sx, *sw;
  void* y;
  int* part;      // int32 [M, N], zeroed (splits > 1)
  int* counters;  // [tiles, 4], zeroed (splits > 1)
  int* status;
};

template <int NTOK>
struct Cfg {
  static constexpr int WST = NTOK == 128 ? 8 : 16;  // stages of weight codes
  static constexpr int X_BYTES = NTOK * BK * 2;
  static constexpr int D_COLS = NTOK < 32 ? 32 : NTOK;
  static constexpr int SMEM = WST * W_BYTES + AST * X_BYTES + 1024 + 512;
};

struct Bars {
  uint64_t wfull[16], wempty[16], xfull[AST], afull[AST], empty[AST], tfull[2], tempty[2], drain;
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

__device__ __forceinline__ void unit_of(const LinParams& p, int unit, int& nt, int& mt, int& kb0, int& kb1) {
  int ks, t;
  p.by_tiles.divmod(unit, ks, t);
  p.by_n.divmod(t, mt, nt);
  kb0 = (int)((int64_t)p.k_blocks * ks / p.splits);
  kb1 = (int)((int64_t)p.k_blocks * (ks + 1) / p.splits);
}

template <class T>
__device__ __forceinline__ T out_as(float v);
template <>
__device__ __forceinline__ float out_as<float>(float v) { return v; }
template <>
__device__ __forceinline__ half_t out_as<half_t>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ bf16_t out_as<bf16_t>(float v) { return __float2bfloat16_rn(v); }

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
  constexpr int WST = C::WST, XB = C::X_BYTES;
  constexpr uint32_t A_COL = 2 * C::D_COLS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* w_smem = smem;
  uint8_t* x_smem = smem + WST * W_BYTES;
  Bars* bars = reinterpret_cast<Bars*>(x_smem + AST * XB);
  const int warp = tc::warp_index(), lane = threadIdx.x & 31;
  const int total = p.tiles_n * p.tiles_m * p.splits;
  volatile int* abort = &bars->abort;
  if (threadIdx.x == 0) {
    for (int s = 0; s < WST; ++s) {
      tc::mbar_init(&bars->wfull[s], 1);
      tc::mbar_init(&bars->wempty[s], 4);
    }
    for (int s = 0; s < AST; ++s) {
      tc::mbar_init(&bars->xfull[s], 1);
      tc::mbar_init(&bars->afull[s], 4);
      tc::mbar_init(&bars->empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      tc::mbar_init(&bars->tfull[a], 1);
      tc::mbar_init(&bars->tempty[a], 4);
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
        int nt, mt, kb0, kb1;
        unit_of(p, unit, nt, mt, kb0, kb1);
        for (int kb = kb0; kb < kb1; ++kb, ++i) {
          const int ws = i % WST, xs = i % AST;
          if (!tc::mbar_wait(&bars->wempty[ws], ((i / WST) & 1) ^ 1, abort, p.status)) { ok = false; break; }
          tc::mbar_expect_tx(&bars->wfull[ws], W_BYTES);
          tc::tma_load_2d(w_smem + ws * W_BYTES, &tmW, &bars->wfull[ws], kb * BK, nt * TM);
          if (!tc::mbar_wait(&bars->empty[xs], ((i / AST) & 1) ^ 1, abort, p.status)) {
            drain_wait(&bars->wfull[ws], (i / WST) & 1);
            ok = false;
            break;
          }
          tc::mbar_expect_tx(&bars->xfull[xs], XB);
          tc::tma_load_2d(x_smem + xs * XB, &tmX, &bars->xfull[xs], kb * BK, mt * NTOK);
        }
      }
      if (*abort) {  // every copy issued has landed before shared memory goes to another block
        for (int j = max(0, i - WST); j < i; ++j) drain_wait(&bars->wfull[j % WST], (j / WST) & 1);
        for (int j = max(0, i - AST); j < i; ++j) drain_wait(&bars->xfull[j % AST], (j / AST) & 1);
      }
    } else if (warp == 1 && tc::elect_one()) {  // ---------------- products
      constexpr uint32_t IDESC = tc::idesc_f16(false, TM, NTOK);
      int i = 0, d = 0;
      bool ok = true;
      for (int unit = blockIdx.x; unit < total && ok; unit += gridDim.x) {
        int nt, mt, kb0, kb1;
        unit_of(p, unit, nt, mt, kb0, kb1);
        for (int c0 = kb0; c0 < kb1 && ok; c0 += kExactBlocks, ++d) {
          if (!tc::mbar_wait(&bars->tempty[d & 1], ((d >> 1) & 1) ^ 1, abort, p.status)) { ok = false; break; }
          const int c1 = min(c0 + kExactBlocks, kb1);
          for (int kb = c0; kb < c1; ++kb, ++i) {
            const int s = i % AST;
            if (!tc::mbar_wait(&bars->xfull[s], (i / AST) & 1, abort, p.status) ||
                !tc::mbar_wait(&bars->afull[s], (i / AST) & 1, abort, p.status)) {
              ok = false;
              break;
            }
            tc::fence_after_sync();
            const uint64_t xd = tc::sdesc_kmajor_sw128(tc::smem_u32(x_smem + s * XB));
#pragma unroll
            for (int k = 0; k < BK / 16; ++k)
              tc::umma_f16_ts(tmem + (d & 1) * C::D_COLS, tmem + A_COL + s * 32 + k * 8, tc::sdesc_advance(xd, k * 32),
                              IDESC, kb > c0 || k > 0 ? 1u : 0u);
            tc::umma_commit(&bars->empty[s]);
          }
          if (ok) tc::umma_commit(&bars->tfull[d & 1]);
        }
      }
      tc::umma_commit(&bars->drain);
      drain_wait(&bars->drain, 0);
    }
  } else if (warp < 8) {  // ---------------- epilogue
    more_registers<216>();
    const int quarter = warp & 3, row = quarter * 32 + lane;
    int d = 0;
    bool ok = true;
    for (int unit = blockIdx.x; unit < total && ok; unit += gridDim.x) {
      int nt, mt, kb0, kb1;
      unit_of(p, unit, nt, mt, kb0, kb1);
      int acc[NTOK];
#pragma unroll
      for (int c = 0; c < NTOK; ++c) acc[c] = 0;
      for (int c0 = kb0; c0 < kb1; c0 += kExactBlocks, ++d) {
        if (!tc::mbar_wait(&bars->tfull[d & 1], (d >> 1) & 1, abort, p.status)) { ok = false; break; }
        tc::fence_after_sync();
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (d & 1) * C::D_COLS;
#pragma unroll
        for (int c = 0; c < NTOK; c += 32) {
          uint32_t r[32];  // (16 columns: the rest of the 32 belongs to nobody)
          __syncwarp();
          tc::tmem_ld32(taddr + c, r);
          tc::tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32 && c + j < NTOK; ++j) acc[c + j] += __float2int_rn(__uint_as_float(r[j]));
        }
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->tempty[d & 1]);
      }
      if (!ok) break;
      const int n = nt * TM + row;
      const int64_t m0 = (int64_t)mt * NTOK;
      const int cols = (int)min((int64_t)NTOK, p.M - m0);
      bool mine = true;
      if (p.splits > 1) {  // parts of the sum meet in memory; of the warps of these rows the last scales and stores
        if (n < p.N) {
#pragma unroll
          for (int c = 0; c < NTOK; ++c)
            if (c < cols) atomicAdd(p.part + (m0 + c) * p.N + n, acc[c]);
        }
        __threadfence();
        __syncwarp();
        int before = 0;
        if (lane == 0) before = atomicAdd(p.counters + (mt * p.tiles_n + nt) * 4 + quarter, 1);
        mine = __shfl_sync(0xffffffffu, before, 0) == p.splits - 1;
        __threadfence();
        if (mine && n < p.N) {
#pragma unroll
          for (int c = 0; c < NTOK; ++c)
            if (c < cols) acc[c] = __ldcg(p.part + (m0 + c) * p.N + n);
        }
      }
      if (mine && n < p.N) {
        const float wn = __ldg(p.sw + n);
        T* y = static_cast<T*>(p.y) + m0 * p.ldy + n;
#pragma unroll
        for (int c = 0; c < NTOK; ++c)
          if (c < cols) y[c * p.ldy] = out_as<T>(__fmul_rn(__fmul_rn((float)acc[c], p.sx[m0 + c]), wn));
      }
    }
  } else {  // ---------------- converters
    fewer_registers<104>();
    const int quarter = warp & 3, grp = (warp - 8) >> 2, row = quarter * 32 + lane;
    int i = 0;
    bool ok = true;
    for (int unit = blockIdx.x; unit < total && ok; unit += gridDim.x) {
      int nt, mt, kb0, kb1;
      unit_of(p, unit, nt, mt, kb0, kb1);
      for (int kb = kb0; kb < kb1; ++kb, ++i) {
        if ((i & 1) != grp) continue;
        const int ws = i % WST, s = i % AST;
        if (!tc::mbar_wait(&bars->wfull[ws], (i / WST) & 1, abort, p.status)) { ok = false; break; }
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
        if (!tc::mbar_wait(&bars->empty[s], ((i / AST) & 1) ^ 1, abort, p.status)) { ok = false; break; }
        tc::fence_after_sync();
        __syncwarp();
        tc::tmem_st32(tmem + ((uint32_t)(quarter * 32) << 16) + A_COL + s * 32, a);
        tc::tmem_st_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->afull[s]);
      }
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

constexpr int kMaxSplitTiles = 256;  // tiles that a split K is worth while for (fewer than the SMs)

struct Scratch {
  size_t sx, zero, xh, total;
  int64_t parts;  // int32 of partial sums that may be needed
};
Scratch plan_scratch(int64_t M, int N, int K) {
  const int64_t Kp = (K + 63) / 64 * 64;
  const int64_t tiles = (N + TM - 1) / TM * ((M + tile_tokens(M) - 1) / tile_tokens(M));
  Scratch s;
  s.parts = tiles <= kMaxSplitTiles ? M * N : 0;
  s.sx = 0;
  s.zero = ((size_t)M * 4 + 255) / 256 * 256;
  s.xh = s.zero + ((size_t)(4 * kMaxSplitTiles + s.parts) * 4 + 255) / 256 * 256;
  s.total = s.xh + (size_t)M * Kp * 2;
  return s;
}

template <class T, int NTOK>
cudaError_t launch_as(const CUtensorMap& tw, const CUtensorMap& tx, const LinParams& p, int sms, cudaStream_t st) {
  auto kern = qlinear_kernel<T, NTOK>;
  static bool attr_set = false;
  if (!attr_set) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<NTOK>::SMEM);
    if (e != cudaSuccess) return e;
    attr_set = true;
  }
  const int64_t total = (int64_t)p.tiles_n * p.tiles_m * p.splits;
  return launch_after(kern, (unsigned)std::min<int64_t>(total, sms), THREADS, Cfg<NTOK>::SMEM, st, tw, tx, p);
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
  p.k_blocks = Kp / BK;
  p.tiles_n = (a.N + TM - 1) / TM;
  p.tiles_m = (int)((a.M + ntok - 1) / ntok);
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
  if (tiles >= (int64_t)1 << 29) return cudaErrorInvalidValue;
  // K is split while tiles leave SMs idle, in ranges of at least four blocks
  p.splits = s.parts > 0 ? (int)std::max<int64_t>(1, std::min<int64_t>(sms / tiles, p.k_blocks / 4)) : 1;
  p.by_tiles = FastDiv((int)tiles);
  p.by_n = FastDiv(p.tiles_n);
  p.sx = reinterpret_cast<const float*>(w + s.sx);
  p.sw = a.w_scales;
  p.y = a.y;
  p.counters = reinterpret_cast<int*>(w + s.zero);
  p.part = p.counters + 4 * kMaxSplitTiles;
  p.status = a.status;
  TokenParams t{};
  t.x = a.x;
  t.ldx = a.ldx;
  t.M = a.M;
  t.K = a.K;
  t.Kp = Kp;
  t.xh = reinterpret_cast<half_t*>(w + s.xh);
  t.sx = reinterpret_cast<float*>(w + s.sx);
  t.zero = p.counters;
  t.n_zero = p.splits > 1 ? 4 * kMaxSplitTiles + s.parts : 0;
  t.status = a.status;
  CUtensorMap tw, tx;
  if (!make_map(&tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.codes, a.K, a.N, a.K, BK, TM, CU_TENSOR_MAP_SWIZZLE_64B) ||
      !make_map(&tx, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, t.xh, Kp, a.M, (uint64_t)Kp * 2, BK, ntok, CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  const unsigned rows = (unsigned)std::min<int64_t>(std::max<int64_t>(a.M, (t.n_zero + 2047) / 2048), (int64_t)sms * 8);
  cudaError_t e = a.x_type == JAB_FP16 ? launch_after(quantize_tokens_kernel<half_t>, rows, 256, 0, st, t)
                                       : launch_after(quantize_tokens_kernel<bf16_t>, rows, 256, 0, st, t);
  if (e != cudaSuccess) return e;
  if (a.y_type == JAB_FP16) return launch_tokens<half_t>(tw, tx, p, ntok, sms, st);
  if (a.y_type == JAB_BF16) return launch_tokens<bf16_t>(tw, tx, p, ntok, sms, st);
  return launch_tokens<float>(tw, tx, p, ntok, sms, st);
}

}  // namespace jab
