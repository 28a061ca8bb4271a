// Attention of new tokens over the quantised paged cache (single tokens, short runs of them, chunks).
//
//   s_ij = c k_j (q_i . K_j)          K_j, V_j whole numbers (codes), k_j, v_j their scales,
//   w_ij = 2^(s_ij - m_i) v_j         c = softmax scale * log2 e
//   o_i  = sum_j w_ij V_j / sum_j 2^(s_ij - m_i)
//
// The codes are exact in fp16 and the scales stay outside of the products: the one on K multiplies the
// score, the one on V the weight, so a byte of the cache costs one or two integer instructions and one
// subtraction on its way to the matrix instructions. m_i is a running maximum of s_ij + log2 v_j, not of
// s_ij: the weights that are rounded to fp16 are then at most 2^8 whatever the scales of V are.
//
// Rows of a tile are (token, query head) pairs that share a KV head, R = 8 NT of them. Keys go 16 at a time:
// S^T = K Q^T and O^T = V^T P^T by m16n8k16 products with the cache's side as the 16-row operand, because a
// decoding step has few rows (4 for a GQA ratio of 4: half of n8 idle, where they would leave three quarters
// of m16). Every operand goes from global memory to the registers that the instruction wants, with no pass
// through shared memory: the dimensions that a sum runs over may be permuted, so a lane takes head_dim / 4
// consecutive codes of its K row, and head_dim / 8 of each of its four V rows.
//
// Work is cut into equal numbers of 16-key tiles over a grid that is resident at once, whatever the lengths:
// block c takes the tiles [c per, (c + 1) per) of the list (KV head, sequence, row tile, key tile) and so
// parts of at most a few (sequence, head) items; parts of an item that went to several blocks are joined by a
// second kernel. Keys shared by all sequences are one more entry of the list, whose rows are those of
// all sequences.
#include <algorithm>
#include <type_traits>

#include "kv_attn.cuh"
#include "tc.cuh"

namespace jab {
namespace kv {
namespace {

constexpr int W = 4;  // warps of a block

// ------------------------------------------------------------------ codes to fp16
// A byte b under the exponent of 1024 is 1024 + b; less 1152 it is b - 128.
__device__ __forceinline__ uint32_t sub_h2(uint32_t a, uint32_t b) {
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t fma_h2(uint32_t a, uint32_t b, uint32_t c) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b), *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<const uint32_t*>(&r);
}
constexpr uint32_t k1152 = 0x64806480u, k1032 = 0x64086408u, kSixteenth = 0x2c002c00u, kMinus72 = 0xd480d480u;

// bytes (0, 1) and (2, 3) of w as fp16 pairs
__device__ __forceinline__ void bytes_h2(uint32_t w, uint32_t& lo, uint32_t& hi) {
  lo = sub_h2(__byte_perm(w, 0x64646464u, 0x4140), k1152);
  hi = sub_h2(__byte_perm(w, 0x64646464u, 0x4342), k1152);
}
// nibbles (j, j + 4) of w as fp16 pairs, j = 0 .. 3: those at bits 4 of a byte stand for 16 times as much
__device__ __forceinline__ void nibbles_h2(uint32_t w, uint32_t (&r)[4]) {
  const uint32_t u = w >> 8;
  r[0] = sub_h2((w & 0x000f000fu) | 0x64006400u, k1032);
  r[1] = fma_h2((w & 0x00f000f0u) | 0x64006400u, kSixteenth, kMinus72);
  r[2] = sub_h2((u & 0x000f000fu) | 0x64006400u, k1032);
  r[3] = fma_h2((u & 0x00f000f0u) | 0x64006400u, kSixteenth, kMinus72);
}

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

// BYTES consecutive bytes into 32-bit words.
template <int BYTES>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[BYTES / 4]) {
  if constexpr (BYTES >= 16) {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + i);
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  } else if constexpr (BYTES == 8) {
    const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
    w[0] = v.x, w[1] = v.y;
  } else {
    w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
  }
}

// A 16-key tile as a lane holds it: codes of K rows g and g + 8 (its quarter of the row) and of V rows 2q, 2q +
// 1, 2q + 8, 2q + 9 (its eighth), the scales of keys g and g + 8.
template <int DH, int BITS>
struct Tile {
  static constexpr int ROW = DH * BITS / 8, KB = ROW / 4, VB = ROW / 8;
  uint32_t k[2][KB / 4], v[4][VB / 4];
  float ks[2], vs[2];
};

template <int DH, int BITS>
__device__ __forceinline__ void load_tile(const AttnParams& p, int64_t row, int g, int q, Tile<DH, BITS>& t) {
  using TT = Tile<DH, BITS>;
#pragma unroll
  for (int i = 0; i < 2; ++i) load_words<TT::KB>(p.k_codes + (row + g + 8 * i) * TT::ROW + q * TT::KB, t.k[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) load_words<TT::VB>(p.v_codes + (row + 2 * q + (i & 1) + 8 * (i >> 1)) * TT::ROW + g * TT::VB, t.v[i]);
#pragma unroll
  for (int i = 0; i < 2; ++i) t.ks[i] = __ldg(p.k_scales + row + g + 8 * i), t.vs[i] = __ldg(p.v_scales + row + g + 8 * i);
}

// Q of row n of the tile, quarter q of the head, as the B operand of K's steps; returns the power of two that it
// was divided by (bf16: the row is brought into fp16's range; exact down to 2^-24 of its largest).
template <class T, int DH, int BITS>
__device__ __forceinline__ float load_q(const T* row, bool live, uint32_t (&b)[DH / 8]) {
  float f[DH / 4];
#pragma unroll
  for (int i = 0; i < DH / 4; i += 8) {
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (live) u = __ldg(reinterpret_cast<const uint4*>(row + i));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (std::is_same<T, half_t>::value) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        f[i + 2 * j] = x.x, f[i + 2 * j + 1] = x.y;
      } else {
        f[i + 2 * j] = __uint_as_float(w[j] << 16), f[i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  }
  float back = 1.f;
  if constexpr (!std::is_same<T, half_t>::value) {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < DH / 4; ++i) big = max(big, __float_as_uint(f[i]) & 0x7fffffffu);
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
    float by;
    row_power(big, by, back);
#pragma unroll
    for (int i = 0; i < DH / 4; ++i) f[i] *= by;
  }
#pragma unroll
  for (int i = 0; i < DH / 8; ++i) {
    // 8 bits: elements in their order; 4 bits: (j, j + 4) of each eight
    const int a = BITS == 8 ? 2 * i : 8 * (i / 4) + (i & 3), c = BITS == 8 ? a + 1 : a + 4;
    b[i] = tc::pack_half2(f[a], f[c]);
  }
  return back;
}

template <class T, int DH, int BITS, int NT>
__global__ void __launch_bounds__(32 * W) kv_attn_kernel(const __grid_constant__ AttnParams p) {
  constexpr int R = 8 * NT, MT = DH / 16, KS = DH / 16, PITCH = DH + 4;
  using TT = Tile<DH, BITS>;
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ int head[kPlanHead];
  __shared__ int row_lo[R], row_hi[R];
  __shared__ float2 sm_ml[W][R];
  float* sm_o = reinterpret_cast<float*>(dyn);               // [W][R][PITCH]
  const int E = entries(p);
  int* cum_t = reinterpret_cast<int*>(dyn + W * R * PITCH * 4);
  int* cum_i = cum_t + E + 1;
  stream_order();
  make_plan<R, 16, W, W>(p, cum_t, cum_i, head);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q4 = lane & 3;
  const int64_t all = (int64_t)head[kTotal] * p.n_kv;
  const int64_t x0 = (int64_t)blockIdx.x * head[kPer], x1 = min(all, x0 + head[kPer]);
  for (int64_t x = x0; x < x1;) {
    const Item it = item_at<R, 16>(p, cum_t, head, x, x1);
    const Entry& en = it.en;
    const int h = it.h, rt = it.rt, t0 = it.t0, s0 = it.s0, s1 = it.s1, rows = it.rows;
    __syncthreads();
    // what the rows see; rows past the end see all, of a Q of zeros
    if (tid < R) {
      int lo = 0, hi = INT32_MAX;
      if (tid < rows) {
        const int token = en.tok0 + p.by_g.quot(rt * R + tid);
        seen_by_row(p, en, en.all ? position_of(p, token) : en.len - en.nq + token - en.tok0, lo, hi);
      }
      row_lo[tid] = lo, row_hi[tid] = hi;
    }
    int all_lo, all_hi;
    seen_by_all(p, en, rt * R, rt * R + rows, head, all_lo, all_hi);
    // Q
    uint32_t qf[NT][DH / 8];
    float fac[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r = 8 * j + g, rr = rt * R + r, i = p.by_g.quot(rr);
      const T* row = static_cast<const T*>(p.q) + (int64_t)(en.tok0 + i) * p.ldq + (int64_t)(h * p.G + rr - i * p.G) * DH + q4 * (DH / 4);
      const float back = load_q<T, DH, BITS>(row, r < rows, qf[j]) * p.scale_log2;
      fac[j][0] = __shfl_sync(0xffffffffu, back, 8 * q4);
      fac[j][1] = __shfl_sync(0xffffffffu, back, 8 * q4 + 4);
    }
    __syncthreads();

    const int32_t* table = p.pages + (en.all ? 0 : (int64_t)(it.e - (p.list.all ? 1 : 0)) * p.max_pages);
    auto first_row = [&](int t) -> int64_t {  // row of the cache of the first key of tile t
      const int key = (t0 + t) * 16, pg = p.by_page.quot(key);
      if (key >= en.len) return (int64_t)h * p.page;  // a tile with nothing to see: any page, not the table's entry
      int id = __ldg(table + pg);
      if (id < 0 || id >= p.n_pages) {
        report(p.status, JAB_ERR_INVALID_ARG);
        id = 0;
      }
      return ((int64_t)id * p.n_kv + h) * p.page + (key - pg * p.page);
    };

    float o[NT][MT][4] = {}, m[NT][2], l[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j) m[j][0] = m[j][1] = -INFINITY, l[j][0] = l[j][1] = 0.f;
    TT cur;
    int t = s0 + warp;
    int64_t next_row = 0;
    if (t < s1) load_tile<DH, BITS>(p, first_row(t), g, q4, cur);
    if (t + W < s1) next_row = first_row(t + W);
    for (; t < s1; t += W) {
      TT nxt;
      if (t + W < s1) load_tile<DH, BITS>(p, next_row, g, q4, nxt);
      if (t + 2 * W < s1) next_row = first_row(t + 2 * W);
      // S^T = K Q^T
      float s[NT][4] = {};
#pragma unroll
      for (int i = 0; i < KS; i += BITS == 8 ? 1 : 2) {
        if constexpr (BITS == 8) {
          uint32_t a[4];
          bytes_h2(cur.k[0][i], a[0], a[2]);
          bytes_h2(cur.k[1][i], a[1], a[3]);
#pragma unroll
          for (int j = 0; j < NT; ++j) mma(s[j], a, qf[j][2 * i], qf[j][2 * i + 1]);
        } else {
          uint32_t u[4], w[4];
          nibbles_h2(cur.k[0][i / 2], u);
          nibbles_h2(cur.k[1][i / 2], w);
          const uint32_t a0[4] = {u[0], w[0], u[1], w[1]}, a1[4] = {u[2], w[2], u[3], w[3]};
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            mma(s[j], a0, qf[j][2 * i], qf[j][2 * i + 1]);
            mma(s[j], a1, qf[j][2 * i + 2], qf[j][2 * i + 3]);
          }
        }
      }
      // scores, their maxima with the weights' scales, weights
      const int key0 = (t0 + t) * 16;
      const bool masked = key0 < all_lo || key0 + 16 > all_hi;
      float lv[2];  // log2 of the V scales; a row of zeros counts as one of 2^-100
#pragma unroll
      for (int i = 0; i < 2; ++i) lv[i] = cur.vs[i] > 0.f ? __log2f(cur.vs[i]) : cur.vs[i] == 0.f ? -100.f : cur.vs[i];
      uint32_t pb[NT][4];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        bool see[4] = {true, true, true, true};
        if (masked) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int key = key0 + g + 8 * (c >> 1), col = 8 * j + 2 * q4 + (c & 1);
            see[c] = key >= row_lo[col] && key < row_hi[col];
          }
        }
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[j][c] = see[c] ? s[j][c] * (cur.ks[c >> 1] * fac[j][c & 1]) : -INFINITY;
          if (see[c]) top[c & 1] = fmaxf(top[c & 1], s[j][c] + lv[c >> 1]);
        }
        // (the first tile's maxima are above -inf + 8)
        if (__any_sync(0xffffffffu, top[0] > m[j][0] + 8.f || top[1] > m[j][1] + 8.f)) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float mx = fmaxf(top[c], m[j][c]);
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            const float f = shift2(m[j][c], mx);
            m[j][c] = mx;
            l[j][c] *= f;
#pragma unroll
            for (int i = 0; i < MT; ++i) o[j][i][c] *= f, o[j][i][c + 2] *= f;
          }
        }
        float wt[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float mm = m[j][c & 1];
          const float ex = see[c] ? tc::fast_exp2(s[j][c] - (mm == -INFINITY ? 0.f : mm)) : 0.f;
          l[j][c & 1] += ex;
          wt[c] = see[c] ? ex * cur.vs[c >> 1] : 0.f;
        }
        // A weight enters the products as its fp16 value and what that leaves over (2^-22 of it in all): rounded
        // once, a row with few keys would be 2^-12 off. The products are not what bounds this kernel.
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
          const uint32_t h = tc::pack_half2(wt[c], wt[c + 1]);
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
          pb[j][c >> 1] = transpose8x8(h);
          pb[j][2 + (c >> 1)] = transpose8x8(tc::pack_half2(wt[c] - f.x, wt[c + 1] - f.y));
        }
      }
      // O^T += V^T P^T
#pragma unroll
      for (int w = 0; w < TT::VB / 4; ++w) {
        uint32_t ab[2][2];  // [keys 2q.. / 2q + 8..]: dimensions interleaved, pairs of keys
        if constexpr (BITS == 8) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            ab[i][0] = __byte_perm(cur.v[2 * i][w], cur.v[2 * i + 1][w], 0x5140);  // a0 b0 a1 b1
            ab[i][1] = __byte_perm(cur.v[2 * i][w], cur.v[2 * i + 1][w], 0x7362);  // a2 b2 a3 b3
          }
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            uint32_t a[4];
            bytes_h2(ab[0][d], a[0], a[1]);
            bytes_h2(ab[1][d], a[2], a[3]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              mma(o[j][2 * w + d], a, pb[j][0], pb[j][1]);
              mma(o[j][2 * w + d], a, pb[j][2], pb[j][3]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            ab[i][0] = __byte_perm(cur.v[2 * i][w], cur.v[2 * i + 1][w], 0x5410);  // low halves
            ab[i][1] = __byte_perm(cur.v[2 * i][w], cur.v[2 * i + 1][w], 0x7632);  // high halves
          }
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            uint32_t u[4], x[4];
            nibbles_h2(ab[0][d], u);
            nibbles_h2(ab[1][d], x);
            const uint32_t a0[4] = {u[0], u[1], x[0], x[1]}, a1[4] = {u[2], u[3], x[2], x[3]};
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              mma(o[j][4 * w + 2 * d], a0, pb[j][0], pb[j][1]);
              mma(o[j][4 * w + 2 * d], a0, pb[j][2], pb[j][3]);
              mma(o[j][4 * w + 2 * d + 1], a1, pb[j][0], pb[j][1]);
              mma(o[j][4 * w + 2 * d + 1], a1, pb[j][2], pb[j][3]);
            }
          }
        }
      }
      cur = nxt;
    }
    // the warps' parts, joined in shared memory in a fixed order
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) l[j][c] += __shfl_xor_sync(0xffffffffu, l[j][c], w);
        const int col = 8 * j + 2 * q4 + c;
        if (g == 0) sm_ml[warp][col] = make_float2(m[j][c], l[j][c]);
        float* at = sm_o + (warp * R + col) * PITCH + g * (DH / 8);
#pragma unroll
        for (int i = 0; i < MT; ++i) *reinterpret_cast<float2*>(at + 2 * i) = make_float2(o[j][i][c], o[j][i][c + 2]);
      }
    __syncthreads();
    const bool whole = s0 == 0 && s1 == it.n && p.shared == 0;
    const int64_t slot = slot_of(p, blockIdx.x, h * head[kItems] + cum_i[it.e] + rt, x == x0);
    if (!whole && slot >= p.list.n_slots) report(p.status, JAB_ERR_INVALID_ARG);
    for (int r = warp; r < rows; r += W) {
      float mx = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) mx = fmaxf(mx, sm_ml[w][r].x);
      float f[W], lsum = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        f[w] = shift2(sm_ml[w][r].x, mx);
        lsum += f[w] * sm_ml[w][r].y;
      }
      const int rr = rt * R + r, i = p.by_g.quot(rr);
      const int64_t token = en.tok0 + i;
      const int qh = h * p.G + rr - i * p.G;
      const float inv = whole ? (lsum == 0.f ? 0.f : 1.f / lsum) : 1.f;
#pragma unroll
      for (int d = lane; d < DH; d += 32) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += f[w] * sm_o[(w * R + r) * PITCH + d];
        if (whole)
          store_out(static_cast<T*>(p.out) + token * p.ldo + (int64_t)qh * DH + d, v * inv);
        else if (slot < p.list.n_slots)
          p.list.part_o[(slot * R + r) * DH + d] = v;
      }
      if (lane == 0) {
        if (!whole) {
          if (slot < p.list.n_slots) p.list.part_ml[slot * R + r] = make_float2(mx, lsum);
        } else if (p.lse != nullptr) {
          p.lse[token * ((int64_t)p.n_kv * p.G) + qh] = lsum == 0.f ? -INFINITY : (mx + log2f(lsum)) * kLn2;
        }
      }
    }
    x += s1 - s0;
  }
}

// Adds to (mx, l, o) the parts that a list's blocks left of one (token, query head) in entry e. False: none, or the
// output is written already. A lane holds dimensions lane, lane + 32, ...
template <int DH, int R, int KT>
__device__ __forceinline__ bool join(AttnParams p, const List& list, int e, int token, int h, int gi, int lane, float& mx, float& l,
                                     float (&o)[DH / 32]) {
  p.list = list;
  const int E = entries(p);
  const int* head = list.plan;
  const int* cum_t = list.plan + kPlanHead;
  const int* cum_i = cum_t + E + 1;
  const Entry en = entry_of(p, e);
  if (token < en.tok0 || token >= en.tok0 + en.nq) return false;
  const int rr = (token - en.tok0) * p.G + gi, want = rr / R, r = rr - want * R;
  int base = cum_t[e], t0, n;
  if (en.all) {
    key_tiles<R, KT>(p, en, 0, head, t0, n);
    base += want * n;
  } else {
    for (int rt = 0;; ++rt) {
      key_tiles<R, KT>(p, en, rt, head, t0, n);
      if (rt == want) break;
      base += n;
    }
  }
  const int per = head[kPer];
  const int64_t y0 = (int64_t)h * head[kTotal] + base, y1 = y0 + n;
  const int c0 = (int)(y0 / per), c1 = (int)((y1 - 1) / per);
  if (c0 == c1 && p.shared == 0) return false;  // written by its block
  const int item = h * head[kItems] + cum_i[e] + want;
  // 32 parts at a time: a lane has the statistics of one, then all lanes add up the parts' rows
  for (int c = c0; c <= c1; c += 32) {
    const int mine = c + lane;
    const int64_t slot = slot_of(p, mine, item, (int64_t)mine * per >= y0);
    const bool have = mine <= c1 && slot < list.n_slots;
    const float2 ml = have ? list.part_ml[slot * R + r] : make_float2(-INFINITY, 0.f);
    float mn = ml.x;
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, w));
    mn = fmaxf(mn, mx);
    const float f = shift2(ml.x, mn), fa = shift2(mx, mn);
    mx = mn;
    l = l * fa + warp_sum(ml.y * f);
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) o[i] *= fa;
    const int64_t at = have ? (slot * R + r) * DH : 0;
    const int k1 = min(32, c1 - c + 1);
#pragma unroll 8
    for (int k = 0; k < k1; ++k) {
      const float fk = __shfl_sync(0xffffffffu, f, k);
      const float* part = list.part_o + __shfl_sync(0xffffffffu, at, k) + lane;
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) o[i] += fk == 0.f ? 0.f : fk * __ldcg(part + 32 * i);
    }
  }
  return true;
}

// Joins the parts of every (token, query head) whose keys went to several blocks or entries, in the lists' order; one
// warp each. by_keys: the list of kv_attn_kernel; by_tiles: of the tile kernel.
template <class T, int DH, int R>
__global__ void __launch_bounds__(128) kv_merge_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ List by_keys,
                                                       const __grid_constant__ List by_tiles) {
  stream_order();
  const int lane = threadIdx.x & 31, Hq = p.n_kv * p.G;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (unit >= (int64_t)p.n_tokens * Hq) return;
  const int token = (int)(unit / Hq), qh = (int)(unit - (int64_t)token * Hq), h = qh / p.G, gi = qh - h * p.G;
  const int b = sequence_of_warp(p, token, lane);
  float mx = -INFINITY, l = 0.f, o[DH / 32] = {};
  bool any = false;
  if (by_keys.used && by_keys.all) any |= join<DH, R, 16>(p, by_keys, 0, token, h, gi, lane, mx, l, o);
  if (by_tiles.used && by_tiles.all) any |= join<DH, kTileRows, kTileKeys>(p, by_tiles, 0, token, h, gi, lane, mx, l, o);
  if (by_keys.used) any |= join<DH, R, 16>(p, by_keys, b + (by_keys.all ? 1 : 0), token, h, gi, lane, mx, l, o);
  if (by_tiles.used) any |= join<DH, kTileRows, kTileKeys>(p, by_tiles, b + (by_tiles.all ? 1 : 0), token, h, gi, lane, mx, l, o);
  if (!any) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
    store_out(static_cast<T*>(p.out) + (int64_t)token * p.ldo + (int64_t)qh * DH + lane + 32 * i, o[i] * inv);
  if (lane == 0 && p.lse != nullptr) p.lse[(int64_t)token * Hq + qh] = l == 0.f ? -INFINITY : (mx + log2f(l)) * kLn2;
}

// ------------------------------------------------------------------ host side
constexpr int kMaxBlocks = 1216, kMaxTileBlocks = 512;
constexpr int kFewRows = 32;  // rows of a sequence up to which all of the work goes by 16 keys

int n_tiles_of_rows(int64_t rows) { return rows <= 8 ? 1 : rows <= 16 ? 2 : 4; }

// Which kernel takes what. Sequences of up to kFewRows (token, head) rows go by 16-key tiles: the cache's bytes bound
// them, not the products. Longer ones fill 128-row tiles; where lengths are mixed, those of up to 8 rows still go
// by keys, in a launch of their own.
struct Route {
  List keys, tiles;
  int nt;  // 8-row blocks of the by-keys kernel
  size_t keys_plan, keys_ml, keys_o, tiles_plan, tiles_ml, tiles_o, total;
};

Route route(int dh, int n_kv, int n_seqs, int64_t n_tokens, int G, int max_q, bool shared) {
  Route r{};
  const int64_t rows = (int64_t)max_q * G, all_rows = n_tokens * G;
  const bool tiles_own = rows > kFewRows, uniform = n_tokens == (int64_t)n_seqs * max_q;
  const bool tiles_all = shared && all_rows > kFewRows;
  const bool keys_own = !tiles_own || !uniform, keys_all = shared && !tiles_all;
  r.keys.used = keys_own || keys_all;
  r.tiles.used = tiles_own || tiles_all;
  r.keys.all = keys_all;
  r.tiles.all = tiles_all;
  r.nt = !tiles_own ? n_tiles_of_rows(keys_all ? std::max(rows, all_rows) : rows) : keys_all ? 4 : 1;
  const int split = !tiles_own ? INT32_MAX : uniform ? 0 : 8;  // rows up to which a sequence goes by keys
  r.keys.min_rows = 1, r.keys.max_rows = keys_own ? split : 0;
  r.tiles.min_rows = tiles_own ? split + 1 : INT32_MAX, r.tiles.max_rows = INT32_MAX;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = (at + bytes + 255) / 256 * 256;
    return o;
  };
  auto slots = [&](int blocks, int R, bool all, bool own) {
    if (!shared) return 2 * (int64_t)blocks;
    return blocks + (int64_t)n_kv * ((all ? (all_rows + R - 1) / R : 0) + (own ? (all_rows + R - 1) / R + n_seqs : 0));
  };
  const size_t plan_bytes = (size_t)(kPlanHead + 2 * (n_seqs + 2)) * 4;
  if (r.keys.used) {
    const int R = 8 * r.nt;
    const int64_t n = slots(kMaxBlocks, R, keys_all, keys_own);
    r.keys.n_slots = (int)std::min<int64_t>(n, INT32_MAX);
    r.keys_plan = take(plan_bytes), r.keys_ml = take((size_t)n * R * 8), r.keys_o = take((size_t)n * R * dh * 4);
  }
  if (r.tiles.used) {
    const int64_t n = slots(kMaxTileBlocks, kTileRows, tiles_all, tiles_own);
    r.tiles.n_slots = (int)std::min<int64_t>(n, INT32_MAX);
    r.tiles_plan = take(plan_bytes), r.tiles_ml = take((size_t)n * kTileRows * 8), r.tiles_o = take((size_t)n * kTileRows * dh * 4);
  }
  r.total = std::max<size_t>(at, 256);
  return r;
}

template <class T, int DH, int BITS, int NT>
cudaError_t launch_keys(const AttnParams& p, int64_t est_tiles, int sms, cudaStream_t st) {
  auto kern = kv_attn_kernel<T, DH, BITS, NT>;
  constexpr int R = 8 * NT;
  const size_t most = (size_t)W * R * (DH + 4) * 4 + (size_t)2 * (2048 + 2) * 4;
  static bool attr_set = false;
  if (!attr_set) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e != cudaSuccess) return e;
    attr_set = true;
  }
  const int E = p.n_seqs + (p.list.all ? 1 : 0);
  const size_t smem = (size_t)W * R * (DH + 4) * 4 + (size_t)2 * (E + 1) * 4;
  static size_t asked = 0;
  static int occ = 0;
  if (occ == 0 || asked != smem) {
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, 32 * W, smem);
    if (e != cudaSuccess) return e;
    occ = std::max(n, 1);
    asked = smem;
  }
  const int64_t grid = std::max<int64_t>(1, std::min<int64_t>({(int64_t)sms * occ, kMaxBlocks, (est_tiles + W - 1) / W}));
  return launch_after(kern, (unsigned)grid, 32 * W, smem, st, p);
}

template <class T, int DH>
cudaError_t launch_all(AttnParams p, const Route& r, int bits, jab_dtype type, int max_q, int max_len, int sms, cudaStream_t st) {
  cudaError_t e;
  if (r.keys.used) {
    p.list = r.keys;
    const int64_t est = (int64_t)p.n_kv * p.n_seqs * ((int64_t)max_len / 16 + 1) * std::max<int64_t>(1, (int64_t)max_q * p.G / (8 * r.nt));
    if (bits == 8)
      e = r.nt == 1 ? launch_keys<T, DH, 8, 1>(p, est, sms, st) : r.nt == 2 ? launch_keys<T, DH, 8, 2>(p, est, sms, st) : launch_keys<T, DH, 8, 4>(p, est, sms, st);
    else
      e = r.nt == 1 ? launch_keys<T, DH, 4, 1>(p, est, sms, st) : r.nt == 2 ? launch_keys<T, DH, 4, 2>(p, est, sms, st) : launch_keys<T, DH, 4, 4>(p, est, sms, st);
    if (e != cudaSuccess) return e;
  }
  if (r.tiles.used) {
    p.list = r.tiles;
    const int64_t rts = ((int64_t)max_q * p.G + kTileRows - 1) / kTileRows, kts = max_len / kTileKeys + 1;
    const int64_t est = p.n_kv * (p.n_seqs * rts * kts + (r.tiles.all ? ((int64_t)p.n_tokens * p.G / kTileRows + 1) * kts : 0));
    if ((e = launch_tiles(p, type, DH, bits, est, std::min(sms, kMaxTileBlocks), st)) != cudaSuccess) return e;
  }
  const unsigned blocks = (unsigned)(((int64_t)p.n_tokens * p.n_kv * p.G + 3) / 4);
  return r.nt == 1   ? launch_after(kv_merge_kernel<T, DH, 8>, blocks, 128, 0, st, p, r.keys, r.tiles)
         : r.nt == 2 ? launch_after(kv_merge_kernel<T, DH, 16>, blocks, 128, 0, st, p, r.keys, r.tiles)
                     : launch_after(kv_merge_kernel<T, DH, 32>, blocks, 128, 0, st, p, r.keys, r.tiles);
}

}  // namespace
}  // namespace kv

size_t kv_attention_scratch(int n_kv, int dh, int n_seqs, int64_t n_tokens, int n_q_heads, int max_q, int shared) {
  return kv::route(dh, n_kv, n_seqs, n_tokens, n_q_heads / n_kv, max_q, shared > 0).total;
}

cudaError_t launch_kv_attention(const KvAttnArgs& a, int sms, cudaStream_t st) {
  const jab_kv_cache& c = a.cache;
  kv::AttnParams p{};
  p.k_codes = static_cast<const uint8_t*>(c.k_codes);
  p.v_codes = static_cast<const uint8_t*>(c.v_codes);
  p.k_scales = c.k_scales;
  p.v_scales = c.v_scales;
  p.n_kv = c.n_kv_heads;
  p.G = a.n_q_heads / c.n_kv_heads;
  p.n_pages = (int)std::min<int64_t>(c.n_pages, INT32_MAX);
  p.max_pages = a.max_pages;
  p.page = c.page_tokens;
  p.copy_keys = std::min(c.page_tokens & -c.page_tokens, kv::kTileKeys);
  p.by_page = FastDiv(p.page);
  p.by_g = FastDiv(p.G);
  p.q = a.q;
  p.ldq = a.ldq;
  p.q_start = a.q_start;
  p.pages = a.pages;
  p.lens = a.lens;
  p.n_seqs = a.n_seqs;
  p.n_tokens = (int)a.n_tokens;
  p.shared = a.shared;
  p.window = a.window;
  p.scale_log2 = a.scale * kv::kLog2e;
  p.out = a.out;
  p.ldo = a.ldo;
  p.lse = a.lse;
  p.status = a.status;
  kv::Route r = kv::route(c.head_dim, p.n_kv, p.n_seqs, p.n_tokens, p.G, a.max_q, p.shared > 0);
  char* w = static_cast<char*>(a.ws);
  r.keys.plan = reinterpret_cast<int32_t*>(w + r.keys_plan);
  r.keys.part_ml = reinterpret_cast<float2*>(w + r.keys_ml);
  r.keys.part_o = reinterpret_cast<float*>(w + r.keys_o);
  r.tiles.plan = reinterpret_cast<int32_t*>(w + r.tiles_plan);
  r.tiles.part_ml = reinterpret_cast<float2*>(w + r.tiles_ml);
  r.tiles.part_o = reinterpret_cast<float*>(w + r.tiles_o);
  const bool wide = c.head_dim == 128;
  if (a.type == JAB_FP16)
    return wide ? kv::launch_all<half_t, 128>(p, r, c.bits, a.type, a.max_q, a.max_len, sms, st)
                : kv::launch_all<half_t, 64>(p, r, c.bits, a.type, a.max_q, a.max_len, sms, st);
  return wide ? kv::launch_all<bf16_t, 128>(p, r, c.bits, a.type, a.max_q, a.max_len, sms, st)
              : kv::launch_all<bf16_t, 64>(p, r, c.bits, a.type, a.max_q, a.max_len, sms, st);
}

}  // namespace jab
