// Softmax cross entropy of an output layer z = A B + bias without keeping the
// logits, and its gradient (maddness_linear_xent, maddness_linear_xent_grad).
//
// Forward: a tile of logits (outputs x rows) is formed on the matrix cores and
// reduced at once to each row's maximum and sum of exp(z - maximum) over the
// tile's outputs; a second kernel joins the tiles of a row.
// Backward: G = g (exp(z - lse) - onehot) is formed again tile by tile, a piece
// of the outputs at a time, and multiplied into dA += G B^T and dB = A^T G.
//
// One tile product serves all of them: C[i][j] = sum_k X[i][k] Y[j][k], each
// operand with k or its own index contiguous in memory.  fp32 matrices go
// through the matrix cores as three bf16 parts each (their exact sum), the six
// products whose terms reach 2^-24 of the result.
//
// What bounds it: the products, 2 N D M operations forward and 6 N D M back (a
// logit is formed again rather than kept: N M values written and read three
// times would cost more than 2 N D M from D of a few hundred on, and do not fit
// beside a large vocabulary's weights); few rows, the one reading of B.
// Measured, bf16: 8192 rows, 4096 -> 131072 forward 6.35 to 6.7 ms (1.31 to 1.38
// PFLOP/s); 8192 rows, 2048 -> 131072 back 10.6 to 11.1 ms (1.18 to 1.25); 63 rows,
// 1024 -> 50001 forward 33 us (24 of it the tiles, B at 4.2 TB/s).
#include "tile.hpp"

namespace mdn {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// what maxima are subtracted from: a row without a finite logit subtracts 0
__device__ __forceinline__ float base_of(float top) { return top == -__builtin_inff() ? 0.0f : top; }

struct XArgs {
  Operand W, A;             // weights (own index: outputs) and activations (own index: rows)
  int64_t N, D, M;
  const float* bias;        // [M] or null
  const int64_t* target;    // [N]
  float2* part;             // [N][tiles]: a tile's maximum and sum
  float* zt;                // [N]: the target's logit
  float* loss; float* lse_out;   // [N] (forward)
  int64_t m0;               // first output of this piece (gradient)
  const float* lse; const float* gloss;
  void* dz; int64_t ldz;    // [N][ldz]: the piece's G
  float* cpart;             // [row tiles][ldz]: sums of G over a tile's rows
  int64_t itiles, jtiles;
};

// where a row's target lies from output i0 on; out of every tile for rows without one
__device__ __forceinline__ int target_at(int64_t t, int64_t M, int64_t i0) {
  const int64_t d = t - i0;
  return t < 0 || t >= M || d < 0 || d >= (1 << 20) ? -1 : (int)d;
}

// a row's lse and loss from its maximum, its sum and its target's logit (looked
// at where there is one)
__device__ __forceinline__ void finish(const XArgs& a, int64_t n, float top, float sum, float z) {
  const float l = top + logf(sum);
  const int64_t t = a.target[n];
  a.lse_out[n] = l;
  a.loss[n] = t < 0 || t >= a.M ? 0.0f : l == -__builtin_inff() ? __builtin_inff() : l - z;
}

template <class T, class Tl>
__global__ void __launch_bounds__(Tl::NT, 1) xent_tile_kernel(XArgs a) {
  constexpr int BI = Tl::BI, BJ = Tl::BJ, WI = Tl::WI;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63;
  int64_t it, jt;
  tile_of(blockIdx.x, a.itiles, a.jtiles, it, jt);
  const int64_t i0 = it * BI, j0 = jt * BJ;
  typename Tl::Acc acc;
  Tl::product(a.W, a.A, i0, j0, 0, a.D, lds_address(lds), acc);
  const int bi = Tl::base_i(), bj = Tl::base_j();
  float b[Tl::MI][16];
  load_bias<Tl>(b, a.bias, i0 + bi, a.M);
  float2* red = reinterpret_cast<float2*>(lds);   // [WI][BJ]
  float* zl = reinterpret_cast<float*>(red + WI * BJ);   // [BJ]: targets' logits, and a place for what is none
#pragma unroll
  for (int nj = 0; nj < Tl::NJ; ++nj) {
    const int64_t j = j0 + bj + 32 * nj + (lane & 31);
    const int t = target_at(a.target[j < a.N ? j : a.N - 1], a.M, i0 + bi);
    float top = -__builtin_inff();
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi) {
#pragma unroll
      for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, acc[mi][nj][r] + b[mi][r]);
      if (__any(t >= 32 * mi && t < 32 * mi + 32)) {
        asm volatile("");   // (a branch: seldom taken)
        float z = 0.0f;
        bool mine = false;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool here = t == 32 * mi + entry_row(r, lane);
          z = here ? acc[mi][nj][r] + b[mi][r] : z;
          mine = mine || here;
        }
        zl[mine ? bj + 32 * nj + (lane & 31) : BJ] = z;
      }
    }
    top = __builtin_fmaxf(top, __shfl_xor(top, 32));
    const float base = base_of(top);
    float sum = 0.0f;
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum += exp_of(acc[mi][nj][r] + b[mi][r] - base);
    sum += __shfl_xor(sum, 32);
    red[Tl::wi() * BJ + bj + 32 * nj + (lane & 31)] = make_float2(top, sum);   // (the same from both halves)
  }
  __syncthreads();
  for (int j = threadIdx.x; j < BJ; j += Tl::NT) {
    if (j0 + j >= a.N) continue;
    float2 v = red[j];
#pragma unroll
    for (int w = 1; w < WI; ++w) {
      const float2 u = red[w * BJ + j];
      const float top = __builtin_fmaxf(v.x, u.x), b = base_of(top);
      v = make_float2(top, v.y * exp_of(v.x - b) + u.y * exp_of(u.x - b));
    }
    if (a.itiles == 1) {
      finish(a, j0 + j, v.x, v.y, zl[j]);
    } else {
      a.part[(j0 + j) * a.itiles + it] = v;
      const int t = target_at(a.target[j0 + j], a.M, i0);
      if (t >= 0 && t < BI) a.zt[j0 + j] = zl[j];
    }
  }
}

// One wavefront per row: lse and loss from the row's tiles.
__global__ void __launch_bounds__(256) xent_join_kernel(XArgs a) {
  const int lane = threadIdx.x & 63;
  for (int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); n < a.N; n += (int64_t)gridDim.x * 4) {
    const float2* part = a.part + n * a.itiles;
    float top = -__builtin_inff();
    for (int64_t t = lane; t < a.itiles; t += 64) top = __builtin_fmaxf(top, part[t].x);
    for (int o = 1; o < 64; o <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o));
    float sum = 0.0f;
    for (int64_t t = lane; t < a.itiles; t += 64) {
      const float2 v = part[t];
      sum += v.y * exp_of(v.x - base_of(top));
    }
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) finish(a, n, top, sum, a.zt[n]);
  }
}

// v plus what the lane `CTRL` (a rotation inside 16 lanes) says holds
template <int CTRL>
__device__ __forceinline__ float add_rotated(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}

// Sums of a and b over the 32 lanes of a half wavefront: a's in its lanes 0 to
// 15, b's in 16 to 31.
__device__ __forceinline__ float sums32(float a, float b) {
  // rows of 16 lanes 1 and 3 of the first change places with 0 and 2 of the second
  const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
  float v = __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]);
  v = add_rotated<0x121>(v);
  v = add_rotated<0x122>(v);
  v = add_rotated<0x124>(v);
  return add_rotated<0x128>(v);
}

// A tile of G: outputs m0 + i, rows j.  In bf16 G is rounded to it: that is
// what the two products take, and torch's own bf16 gradients of logits are no
// finer; its sums over rows are taken before.  Forming a tile's G, staging and
// writing it costs 18 us a round of workgroups beside 53 of products (2048 k);
// with scattered 8-byte stores and a shuffle per sum it was 33.
template <class T, class Tl>
__global__ void __launch_bounds__(Tl::NT, 1) xent_dz_kernel(XArgs a) {
  constexpr int BI = Tl::BI, BJ = Tl::BJ, WJ = Tl::WJ;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63;
  int64_t it, jt;
  tile_of(blockIdx.x, a.itiles, a.jtiles, it, jt);
  const int64_t i0 = a.m0 + it * BI, j0 = jt * BJ;
  typename Tl::Acc acc;
  Tl::product(a.W, a.A, i0, j0, 0, a.D, lds_address(lds), acc);
  const int bi = Tl::base_i(), bj = Tl::base_j();
  float b[Tl::MI][16], cols[Tl::MI][16];
  load_bias<Tl>(b, a.bias, i0 + bi, a.M);
  T* out = static_cast<T*>(a.dz) + j0 * a.ldz + it * BI;
#pragma unroll
  for (int nj = 0; nj < Tl::NJ; ++nj) {
    const int64_t j = j0 + bj + 32 * nj + (lane & 31);
    const int64_t at = j < a.N ? j : a.N - 1, target = a.target[at];   // (rows past the end are not written)
    const float l = a.lse[at], g = a.gloss[at];
    const bool live = j < a.N && target >= 0 && target < a.M && l != -__builtin_inff();
    const int t = live ? target_at(target, a.M, i0 + bi) : -1;
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi) {
      float v[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) v[r] = exp_of(acc[mi][nj][r] + b[mi][r] - l);
      if (__any(t >= 32 * mi && t < 32 * mi + 32)) {
        asm volatile("");   // (a branch: seldom taken)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          v[r] -= t == 32 * mi + entry_row(r, lane) ? 1.0f : 0.0f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        v[r] = live ? v[r] * g : 0.0f;   // (whatever a row without a gradient has for logits)
        cols[mi][r] = nj == 0 ? v[r] : cols[mi][r] + v[r];
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = bi + 32 * mi + entry_row(4 * q, lane);
        if (!Tl::lead()) continue;
        if constexpr (sizeof(T) == 2) stage4<T, Tl>(lds, i, (int)(j - j0), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        else if (j < a.N) write4(out + (j - j0) * a.ldz + i, a.ldz - it * BI - i, (f32x4){v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]});
      }
      __builtin_amdgcn_sched_barrier(0);   // (a block at a time: few registers)
    }
  }
  // sums over the tile's rows, for the bias gradient
  float* red = reinterpret_cast<float*>(lds + (sizeof(T) == 2 ? Tl::BI * Tl::BJ * 2 : 0));   // [WJ][BI]
#pragma unroll
  for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float s = sums32(cols[mi][r], cols[mi][r + 1]);
      if ((lane & 15) == 0 && Tl::lead()) red[Tl::wj() * BI + bi + 32 * mi + entry_row(r, lane) + ((lane >> 4) & 1)] = s;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < BI; i += Tl::NT) {
    float s = red[i];
#pragma unroll
    for (int w = 1; w < WJ; ++w) s += red[w * BI + i];
    if (it * BI + i < a.ldz) a.cpart[jt * a.ldz + it * BI + i] = s;
  }
  if constexpr (sizeof(T) == 2) write_staged<T, Tl>(lds, out, a.ldz, a.ldz - it * BI, a.N - j0);
}

// The bias gradient from the row tiles' sums: 32 outputs a workgroup, the tiles
// in 8 strands with 8 loads under way in each, the strands added in order.
__global__ void __launch_bounds__(256) xent_dbias_kernel(const float* cpart, int64_t jtiles, int64_t ldz, int64_t n, float* out) {
  __shared__ float red[8][32];
  const int strand = threadIdx.x >> 5, c = threadIdx.x & 31;
  for (int64_t i0 = (int64_t)blockIdx.x * 32; i0 < n; i0 += (int64_t)gridDim.x * 32) {
    const float* p = cpart + (i0 + c < n ? i0 + c : n - 1);
    float s = 0.0f;
    int64_t j = strand;
    for (; j + 56 < jtiles; j += 64) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p[(j + 8 * k) * ldz];
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
    for (; j < jtiles; j += 8) s += p[j * ldz];
    red[strand][c] = s;
    __syncthreads();
    if (strand == 0 && i0 + c < n) {
#pragma unroll
      for (int k = 1; k < 8; ++k) s += red[k][c];
      out[i0 + c] = s;
    }
    __syncthreads();
  }
}

// out[j][i] = sum_k X[i][k] Y[j][k], added to what `sum` holds where it is
// not the first piece; written to `sum` (32 bits) unless it is the last.
// splits > 1: blockIdx.y takes its share of k and leaves it in part[split].
struct GemmArgs {
  Operand X, Y;
  int64_t K;
  int64_t itiles, jtiles;
  void* out; int64_t ldo;
  float* sum;               // [rows of Y][rows of X] or null
  int first, last;
  float* part; int splits; int64_t kper;
};

enum GemmOut : int {
  kOut,      // the result, one piece
  kPart,     // 32-bit results: a share of k, or the first of several pieces
  kMore,     // a further piece: added to the sum
  kLast      // the last of several: the sum added, the result written
};

template <class T, class Tl, GemmOut MODE>
__global__ void __launch_bounds__(Tl::NT, 1) xent_gemm_kernel(GemmArgs a) {
  constexpr int BI = Tl::BI, BJ = Tl::BJ;
  extern __shared__ __align__(16) char lds[];
  int64_t it, jt;
  tile_of(blockIdx.x, a.itiles, a.jtiles, it, jt);
  const int64_t i0 = it * BI, j0 = jt * BJ, I = a.X.rows, J = a.Y.rows;
  const int64_t k0 = blockIdx.y * a.kper, kend = k0 + a.kper < a.K ? k0 + a.kper : a.K;
  typename Tl::Acc acc;
  Tl::product(a.X, a.Y, i0, j0, k0, kend, lds_address(lds), acc);
  float* sum = (a.splits > 1 ? a.part + blockIdx.y * I * J : a.sum) + j0 * I + i0;
  T* out = static_cast<T*>(a.out) + j0 * a.ldo + i0;
  if constexpr (MODE == kOut) write_tile<T, Tl>(acc, lds, out, a.ldo, I - i0, J - j0);
  else if constexpr (MODE == kPart) write_tile32<float, Tl, false>(acc, lds, sum, I, I - i0, J - j0);
  else if constexpr (MODE == kMore) write_tile32<float, Tl, true>(acc, lds, sum, I, I - i0, J - j0, sum, I);
  else write_tile32<T, Tl, true>(acc, lds, out, a.ldo, I - i0, J - j0, sum, I);
}

// Joins the shares of a split product, in order.
template <class T>
__global__ void __launch_bounds__(256) xent_join_splits_kernel(GemmArgs a) {
  const int64_t I = a.X.rows, all = I * a.Y.rows;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (int64_t)gridDim.x * 256) {
    float v = a.first ? 0.0f : a.sum[e];
    int s = 0;
    for (; s + 8 <= a.splits; s += 8) {   // eight loads under way at a time
      float u[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] = a.part[(s + k) * all + e];
#pragma unroll
      for (int k = 0; k < 8; ++k) v += u[k];
    }
    for (; s < a.splits; ++s) v += a.part[s * all + e];
    if (a.last) static_cast<T*>(a.out)[e / I * a.ldo + e % I] = from_float<T>(v);
    else a.sum[e] = v;
  }
}

template <class T>
__global__ void __launch_bounds__(256) xent_fill_kernel(T* p, int64_t n) {
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) p[e] = from_float<T>(0.0f);
}

constexpr int kWide = 128;   // outputs or columns of a tile
constexpr int kSlots = 512;  // workgroups that fill the card: two to a compute unit

// LDS of the kernel that forms G: the product's, or the staged tile and the sums behind it
template <class T, class Tl>
constexpr int kDzLds = sizeof(T) == 2 && Tl::BI * Tl::BJ * 2 + Tl::WJ * Tl::BI * 4 > (int)Tl::LDS ? Tl::BI * Tl::BJ * 2 + Tl::WJ * Tl::BI * 4 : (int)Tl::LDS;

template <class T, bool GRAD, class Tl>
hipError_t launch_logits(XArgs& a, int64_t outputs, hipStream_t s) {
  a.itiles = cdiv(outputs, Tl::BI);
  a.jtiles = cdiv(a.N, Tl::BJ);
  if constexpr (GRAD) return launch(xent_dz_kernel<T, Tl>, kDzLds<T, Tl>, a.itiles * a.jtiles, 1, Tl::NT, a, s);
  else return launch(xent_tile_kernel<T, Tl>, Tl::LDS, a.itiles * a.jtiles, 1, Tl::NT, a, s);
}

// Rows of a logits tile: 256 (large bf16 products with whole units in A), or
// 128, 64 or 32: the widest that the rows fill and that leaves every compute
// unit work.
template <class T>
int row_tile(const XArgs& a, int64_t outputs) {
  if (sizeof(T) == 2 && a.N >= 192 && direct(a.A, false) && cdiv(a.N, 256) * cdiv(outputs, 256) >= 192) return 256;
  if (a.N > 64 && cdiv(a.N, 128) * cdiv(outputs, 128) >= 256) return 128;
  return a.N > 32 && cdiv(a.N, 32) * cdiv(outputs, 128) > 256 ? 64 : 32;
}

template <class T, bool GRAD>
hipError_t logits(XArgs& a, int64_t outputs, int rows, bool md, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (rows == 256) {
      if (direct(a.W, !md)) return md ? launch_logits<T, GRAD, BigTile<T, kAlongK, kAlongK, false>>(a, outputs, s)
                                 : launch_logits<T, GRAD, BigTile<T, kAlongI, kAlongK, false>>(a, outputs, s);
      return md ? launch_logits<T, GRAD, BigTile<T, kAlongK, kAlongK, true>>(a, outputs, s)
                : launch_logits<T, GRAD, BigTile<T, kAlongI, kAlongK, true>>(a, outputs, s);
    }
  }
  if (rows >= 128) return md ? launch_logits<T, GRAD, Tile<T, kAlongK, kAlongK, 128, 128, 2, 2>>(a, outputs, s)
                             : launch_logits<T, GRAD, Tile<T, kAlongI, kAlongK, 128, 128, 2, 2>>(a, outputs, s);
  // Where every workgroup has a compute unit to itself: twice the wavefronts,
  // each for half of the k of a step twice as long, since one wavefront to a SIMD
  // waits for the stages of a step in turn (fp32 10000 x 512 -> 100, 157 workgroups:
  // 20.8 against 24.2 us; 20000 rows, 313 of them: 41 against 32 without).
  const bool alone = cdiv(a.N, rows) * cdiv(outputs, 128) <= 256;
  constexpr int BK = sizeof(T) == 2 ? 64 : 32;
  if (rows == 64) {
    if (alone) return md ? launch_logits<T, GRAD, Tile<T, kAlongK, kAlongK, 128, 64, 4, 1, 2 * BK, 2>>(a, outputs, s)
                         : launch_logits<T, GRAD, Tile<T, kAlongI, kAlongK, 128, 64, 4, 1, 2 * BK, 2>>(a, outputs, s);
    return md ? launch_logits<T, GRAD, Tile<T, kAlongK, kAlongK, 128, 64, 4, 1>>(a, outputs, s)
              : launch_logits<T, GRAD, Tile<T, kAlongI, kAlongK, 128, 64, 4, 1>>(a, outputs, s);
  }
  if (alone) return md ? launch_logits<T, GRAD, Tile<T, kAlongK, kAlongK, 128, 32, 4, 1, 2 * BK, 2>>(a, outputs, s)
                       : launch_logits<T, GRAD, Tile<T, kAlongI, kAlongK, 128, 32, 4, 1, 2 * BK, 2>>(a, outputs, s);
  return md ? launch_logits<T, GRAD, Tile<T, kAlongK, kAlongK, 128, 32, 4, 1>>(a, outputs, s)
            : launch_logits<T, GRAD, Tile<T, kAlongI, kAlongK, 128, 32, 4, 1>>(a, outputs, s);
}

// Shares of k for `tiles` tiles: workgroups for the whole card, at least 8 steps each.
int splits_for(int64_t tiles, int64_t slots, int64_t K, int bk) {
  int64_t s = slots / (tiles > 0 ? tiles : 1);
  const int64_t most = K / (8 * bk);
  if (s > most) s = most;
  return s < 1 ? 1 : (int)(s > 64 ? 64 : s);
}

template <class T, class Tl, bool PIECES>
hipError_t gemm(GemmArgs a, int64_t part_bytes, hipStream_t s) {
  a.itiles = cdiv(a.X.rows, Tl::BI);
  a.jtiles = cdiv(a.Y.rows, Tl::BJ);
  a.splits = splits_for(a.itiles * a.jtiles, Tl::BI == 256 ? kSlots / 2 : kSlots, a.K, Tl::BK);
  const int64_t fit = part_bytes / (a.X.rows * a.Y.rows * 4);
  if (a.splits > fit) a.splits = fit < 1 ? 1 : (int)fit;
  a.kper = up(cdiv(a.K, a.splits), Tl::BK);
  a.splits = (int)cdiv(a.K, a.kper);
  const GemmOut mode = a.splits > 1 || (a.first && !a.last) ? kPart : a.first ? kOut : a.last ? kLast : kMore;
  hipError_t e;
  if (mode == kOut) e = launch(xent_gemm_kernel<T, Tl, kOut>, Tl::LDS, a.itiles * a.jtiles, a.splits, Tl::NT, a, s);
  else if (mode == kPart) e = launch(xent_gemm_kernel<T, Tl, kPart>, Tl::LDS, a.itiles * a.jtiles, a.splits, Tl::NT, a, s);
  else if constexpr (PIECES) {
    if (mode == kLast) e = launch(xent_gemm_kernel<T, Tl, kLast>, Tl::LDS, a.itiles * a.jtiles, a.splits, Tl::NT, a, s);
    else e = launch(xent_gemm_kernel<T, Tl, kMore>, Tl::LDS, a.itiles * a.jtiles, a.splits, Tl::NT, a, s);
  } else {
    return hipErrorInvalidValue;
  }
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t b = cdiv(a.X.rows * a.Y.rows, 256);
  hipLaunchKernelGGL((xent_join_splits_kernel<T>), dim3((unsigned)(b < 4096 ? b : 4096)), dim3(256), 0, s, a);
  return hipGetLastError();
}

struct GradPlan {
  int64_t p;                                    // outputs per piece
  int64_t off_dz, off_c, off_sum, off_part, part, total;
};

// Outputs per piece of the gradient: G of a piece stays within 256 MiB, at least 256 outputs.
GradPlan grad_plan(int64_t N, int64_t D, int64_t M, int64_t elem) {
  GradPlan g{};
  int64_t p = (256ll << 20) / (N * elem) / 256 * 256;
  if (p < 256) p = 256;
  g.p = p < up(M, 64) ? p : up(M, 64);
  int64_t off = 0;
  auto take = [&](int64_t bytes) { const int64_t o = off; off += up(bytes, 256); return o; };
  g.off_dz = take(N * g.p * elem);
  g.off_c = take(cdiv(N, 32) * g.p * 4);
  g.off_sum = take(g.p < M ? N * D * 4 : 0);
  // shares of a product: at most 64 of its results, or a tile of 256 x 256 for
  // each compute unit
  const int64_t results = (N > g.p ? N : g.p) * D;
  g.part = results < 256 * 1024 ? results * 64 * 4 : 256ll * 256 * 256 * 4;
  g.off_part = take(g.part);
  g.total = off;
  return g;
}

template <class T>
hipError_t grad(XArgs a, bool md, void* dA, void* dB, float* dbias, char* ws, hipStream_t s) {
  const GradPlan g = grad_plan(a.N, a.D, a.M, sizeof(T));
  a.dz = ws + g.off_dz;
  a.cpart = reinterpret_cast<float*>(ws + g.off_c);
  T* B = static_cast<T*>(const_cast<void*>(a.W.p));
  for (int64_t m0 = 0; m0 < a.M; m0 += g.p) {
    const int64_t n = a.M - m0 < g.p ? a.M - m0 : g.p;
    XArgs z = a;
    z.m0 = m0;
    z.ldz = up(n, 64);
    hipError_t e = logits<T, true>(z, z.ldz, row_tile<T>(a, g.p), md, s);
    if (e != hipSuccess) return e;
    const int64_t b = cdiv(n, 32);
    hipLaunchKernelGGL(xent_dbias_kernel, dim3((unsigned)(b < 4096 ? b : 4096)), dim3(256), 0, s, z.cpart, z.jtiles, z.ldz, n, dbias + m0);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const Operand zk{z.dz, z.ldz, a.N, a.N}, zi{z.dz, z.ldz, n, z.ldz};
    GemmArgs x{};
    x.sum = reinterpret_cast<float*>(ws + g.off_sum);
    x.part = reinterpret_cast<float*>(ws + g.off_part);
    // dA [N][D] += G B^T over the piece's outputs
    x.X = Operand{md ? B + m0 * a.W.ld : B + m0, a.W.ld, a.D, a.D};
    x.Y = zk;
    x.K = n;
    x.out = dA; x.ldo = a.D;
    x.first = m0 == 0; x.last = m0 + n == a.M;
    bool done = false;
    if constexpr (sizeof(T) == 2) {
      // (as many tiles and shares of at least 1024 outputs as most compute units)
      if (a.N >= 192 && a.D >= 192 && cdiv(a.N, 256) * cdiv(a.D, 256) * cdiv(n, 1024) >= 192) {
        done = true;
        if (direct(x.X, md)) e = md ? gemm<T, BigTile<T, kAlongI, kAlongK, false>, true>(x, g.part, s) : gemm<T, BigTile<T, kAlongK, kAlongK, false>, true>(x, g.part, s);
        else e = md ? gemm<T, BigTile<T, kAlongI, kAlongK, true>, true>(x, g.part, s) : gemm<T, BigTile<T, kAlongK, kAlongK, true>, true>(x, g.part, s);
      }
    }
    // 64 rows where 128 give less than two rounds of workgroups (fp32, 316 tiles of
    // 10000 x 512 -> 100: the gradients 71 against 76 us; 512 tiles of 8192 x 1024
    // -> 1000: 371 with 128 against 380; only short products, 20000 x 512 -> 100,
    // would gain past that: 103 against 96)
    if (done) {}
    else if (cdiv(a.N, 128) * cdiv(a.D, 128) < 512) e = md ? gemm<T, Tile<T, kAlongI, kAlongK, 128, 64, 2, 2>, true>(x, g.part, s) : gemm<T, Tile<T, kAlongK, kAlongK, 128, 64, 2, 2>, true>(x, g.part, s);
    else e = md ? gemm<T, Tile<T, kAlongI, kAlongK, 128, 128, 2, 2>, true>(x, g.part, s) : gemm<T, Tile<T, kAlongK, kAlongK, 128, 128, 2, 2>, true>(x, g.part, s);
    if (e != hipSuccess) return e;
    // dB = A^T G: [D][M] columns m0.., or [M][D] rows m0..
    const Operand ai{a.A.p, a.A.ld, a.D, a.D};
    x.X = md ? ai : zi;
    x.Y = md ? zi : ai;
    x.K = a.N;
    x.out = static_cast<T*>(dB) + (md ? m0 * a.D : m0); x.ldo = md ? a.D : a.M;
    x.first = x.last = 1;
    done = false;
    if constexpr (sizeof(T) == 2) {
      if (direct(ai, true) && direct(zi, true) && cdiv(a.D, 256) * cdiv(n, 256) >= 192) {
        done = true;
        e = gemm<T, BigTile<T, kAlongI, kAlongI, false>, false>(x, g.part, s);
      }
    }
    if (!done) e = gemm<T, Tile<T, kAlongI, kAlongI, 128, 128, 2, 2>, false>(x, g.part, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t forward(XArgs a, bool md, float* loss, float* lse, hipStream_t s) {
  a.loss = loss;
  a.lse_out = lse;
  hipError_t e = logits<T, false>(a, a.M, row_tile<T>(a, a.M), md, s);
  if (e != hipSuccess || a.itiles == 1) return e;
  const int64_t b = cdiv(a.N, 4);
  hipLaunchKernelGGL(xent_join_kernel, dim3((unsigned)(b < 65536 ? b : 65536)), dim3(256), 0, s, a);
  return hipGetLastError();
}

int check(const void* A, int32_t dtype, int64_t N, int32_t D, int64_t lda, const void* B, int32_t M, int32_t outputs_first,
          const float* col_bias, const int64_t* target) {
  if (N < 0 || D <= 0 || M <= 0 || lda < D || (outputs_first != 0 && outputs_first != 1)) return MADDNESS_EINVAL;
  if (dtype != MADDNESS_F32 && dtype != MADDNESS_BF16) return MADDNESS_EINVAL;
  const uintptr_t al = dtype == MADDNESS_F32 ? 4 : 2;
  if (!B || !aligned(B, al) || (col_bias && !aligned(col_bias, 4))) return MADDNESS_EINVAL;
  if (N > 0 && (!A || !target || !aligned(A, al) || !aligned(target, 8))) return MADDNESS_EINVAL;
  return MADDNESS_OK;
}

XArgs args(const void* A, int64_t N, int32_t D, int64_t lda, const void* B, int32_t M, int32_t outputs_first,
           const float* col_bias, const int64_t* target) {
  XArgs a{};
  a.W = Operand{B, outputs_first ? D : M, M, M};
  a.A = Operand{A, lda, N, N};
  a.N = N; a.D = D; a.M = M;
  a.bias = col_bias; a.target = target;
  return a;
}

constexpr int64_t kMaxN = 1ll << 31;

}  // namespace
}  // namespace mdn

using namespace mdn;

extern "C" {

int64_t maddness_linear_xent_workspace_bytes(int64_t N, int32_t D, int32_t M, int32_t dtype) {
  if (N < 0 || N >= kMaxN || D <= 0 || M <= 0 || (dtype != MADDNESS_F32 && dtype != MADDNESS_BF16)) return -1;
  return up(N * 4, 256) + up(N * cdiv(M, kWide) * 8, 256) + 256;
}

int maddness_linear_xent(const void* A, int32_t dtype, int64_t N, int32_t D, int64_t lda, const void* B, int32_t M,
                         int32_t outputs_first, const float* col_bias, const int64_t* target, float* loss_out, float* lse_out,
                         void* workspace, int64_t workspace_bytes, void* stream) {
  const int rc = check(A, dtype, N, D, lda, B, M, outputs_first, col_bias, target);
  if (rc != MADDNESS_OK) return rc;
  if (N >= kMaxN) return MADDNESS_EUNSUPPORTED;
  if (N == 0) return MADDNESS_OK;
  if (!loss_out || !lse_out || !aligned(loss_out, 4) || !aligned(lse_out, 4)) return MADDNESS_EINVAL;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < maddness_linear_xent_workspace_bytes(N, D, M, dtype)) return MADDNESS_EINVAL;
  XArgs a = args(A, N, D, lda, B, M, outputs_first, col_bias, target);
  char* w = static_cast<char*>(workspace);
  a.zt = reinterpret_cast<float*>(w);
  a.part = reinterpret_cast<float2*>(w + up(N * 4, 256));
  hipStream_t s = static_cast<hipStream_t>(stream);
  return status_from(dtype == MADDNESS_F32 ? forward<float>(a, outputs_first, loss_out, lse_out, s) : forward<Bf16>(a, outputs_first, loss_out, lse_out, s));
}

int64_t maddness_linear_xent_grad_workspace_bytes(int64_t N, int32_t D, int32_t M, int32_t dtype) {
  if (N < 0 || N >= kMaxN || D <= 0 || M <= 0 || (dtype != MADDNESS_F32 && dtype != MADDNESS_BF16)) return -1;
  if (N == 0) return 256;
  return grad_plan(N, D, M, dtype == MADDNESS_F32 ? 4 : 2).total;
}

int maddness_linear_xent_grad(const void* A, int32_t dtype, int64_t N, int32_t D, int64_t lda, const void* B, int32_t M,
                              int32_t outputs_first, const float* col_bias, const int64_t* target, const float* lse,
                              const float* grad_loss, void* dA_out, void* dB_out, float* dbias_out, void* workspace,
                              int64_t workspace_bytes, void* stream) {
  const int rc = check(A, dtype, N, D, lda, B, M, outputs_first, col_bias, target);
  if (rc != MADDNESS_OK) return rc;
  if (N >= kMaxN) return MADDNESS_EUNSUPPORTED;
  const uintptr_t al = dtype == MADDNESS_F32 ? 4 : 2;
  if (!dB_out || !dbias_out || !aligned(dB_out, al) || !aligned(dbias_out, 4)) return MADDNESS_EINVAL;
  if (N > 0 && (!lse || !grad_loss || !dA_out || !aligned(lse, 4) || !aligned(grad_loss, 4) || !aligned(dA_out, al))) return MADDNESS_EINVAL;
  if (N > 0 && (!workspace || !aligned(workspace, 256) ||
                workspace_bytes < maddness_linear_xent_grad_workspace_bytes(N, D, M, dtype)))
    return MADDNESS_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (N == 0) {   // no rows: the gradients of B and the bias are zero
    const int64_t n = (int64_t)D * M, b = cdiv(n, 256);
    const dim3 grid((unsigned)(b < 4096 ? b : 4096));
    if (dtype == MADDNESS_F32) hipLaunchKernelGGL((xent_fill_kernel<float>), grid, dim3(256), 0, s, static_cast<float*>(dB_out), n);
    else hipLaunchKernelGGL((xent_fill_kernel<Bf16>), grid, dim3(256), 0, s, static_cast<Bf16*>(dB_out), n);
    hipLaunchKernelGGL((xent_fill_kernel<float>), dim3(64), dim3(256), 0, s, dbias_out, (int64_t)M);
    return status_from(hipGetLastError());
  }
  XArgs a = args(A, N, D, lda, B, M, outputs_first, col_bias, target);
  a.lse = lse; a.gloss = grad_loss;
  char* w = static_cast<char*>(workspace);
  return status_from(dtype == MADDNESS_F32 ? grad<float>(a, outputs_first, dA_out, dB_out, dbias_out, w, s)
                                           : grad<Bf16>(a, outputs_first, dA_out, dB_out, dbias_out, w, s));
}

}  // extern "C"
