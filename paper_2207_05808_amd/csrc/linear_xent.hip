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
#include "maddness.h"
#include "internal.hpp"
#include "mma.hpp"

namespace mdn {
namespace {

enum Order : int { kAlongK = 0, kAlongI = 1 };   // which index of an operand is contiguous

struct Operand {
  const void* p;
  int64_t ld;     // elements between rows (kAlongK) or between k steps (kAlongI)
  int64_t rows;   // extent of the operand's own index
};

// A tile of BI x BJ results of one workgroup of WI x WJ wavefronts, k in steps
// of BK through two LDS buffers.
template <class T, Order OX, Order OY, int BI, int BJ, int WI, int WJ>
struct Tile {
  static constexpr int P = Parts<T>::n;
  static constexpr int BK = P == 1 ? 64 : 32;
  static constexpr int CH = 16 / sizeof(T);          // elements of a 16-byte unit
  static constexpr int NT = WI * WJ * 64;
  static constexpr int MI = BI / WI / 32, NJ = BJ / WJ / 32;
  static constexpr int XU = BI * BK / CH / NT, YU = BJ * BK / CH / NT;   // units a thread moves per step
  static constexpr int XB = BI * BK * 2, YB = BJ * BK * 2;               // bytes of one part's LDS tile
  static constexpr int STAGE = P * (XB + YB);
  static constexpr int LDS = 2 * STAGE;
  static_assert(XU * CH * NT == BI * BK && YU * CH * NT == BJ * BK && MI * WI * 32 == BI && NJ * WJ * 32 == BJ, "tile");
  typedef f32x16 Acc[MI][NJ];

  // LDS address of element (r, k) of a part's tile.  Along k: rows of BK, their
  // 16-byte units permuted by the row so that 16 neighbouring rows' units lie
  // in different banks.  Along the row: one line of B rows per k, its 64-byte
  // blocks permuted by k for the transposing reads, which take 4 lines at once.
  template <Order O, int B>
  static __device__ __forceinline__ int at(int r, int k) {
    if constexpr (O == kAlongK) {
      constexpr int U = BK / 8;
      const int s = U == 8 ? (r >> 1) & 7 : (r >> 2) & 3;
      return r * (BK * 2) + (((k >> 3) ^ s) << 4) + (k & 7) * 2;
    } else {
      constexpr int NB = B / 32;
      const int s = NB >= 4 ? k & 3 : NB == 2 ? (k >> 1) & 1 : 0;
      return k * (B * 2) + (((r >> 5) ^ s) << 6) + (r & 31) * 2;
    }
  }

  // unit u of a step: its element's row and k inside the tile
  template <Order O, int B>
  static __device__ __forceinline__ void unit(int u, int& r, int& k) {
    if constexpr (O == kAlongK) {
      r = u / (BK / CH);
      k = (u % (BK / CH)) * CH;
    } else {
      k = u / (B / CH);
      r = (u % (B / CH)) * CH;
    }
  }

  template <Order O, int B, int U>
  static __device__ __forceinline__ void load(const Operand& o, int64_t r0, int64_t k0, int64_t kend, u32x4 (&v)[U]) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int r, k;
      unit<O, B>(threadIdx.x + i * NT, r, k);
      const T* p = static_cast<const T*>(o.p) + (O == kAlongK ? (r0 + r) * o.ld + (k0 + k) : (k0 + k) * o.ld + (r0 + r));
      // elements of the unit inside the matrix
      const bool in = r0 + r < o.rows && k0 + k < kend;
      const int64_t left = !in ? 0 : O == kAlongK ? kend - (k0 + k) : o.rows - (r0 + r);
      v[i] = (u32x4){0, 0, 0, 0};
      if (left >= CH) {
        v[i] = load16(p);
      } else if (left > 0) {
#pragma unroll
        for (int e = 0; e < CH; ++e)
          if (e < left) {
            if constexpr (CH == 4) v[i][e] = __float_as_uint(p[e]);
            else v[i][e >> 1] |= (uint32_t)p[e].bits << (16 * (e & 1));
          }
      }
    }
  }

  template <Order O, int B, int U>
  static __device__ __forceinline__ void store(char* lds, const u32x4 (&v)[U]) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int r, k;
      unit<O, B>(threadIdx.x + i * NT, r, k);
      char* p = lds + at<O, B>(r, k);
      if constexpr (P == 1) {
        *reinterpret_cast<u32x4*>(p) = v[i];
      } else {
        uint32_t a[P], b[P];
        split2<P>(__uint_as_float(v[i][0]), __uint_as_float(v[i][1]), a);
        split2<P>(__uint_as_float(v[i][2]), __uint_as_float(v[i][3]), b);
#pragma unroll
        for (int s = 0; s < P; ++s) *reinterpret_cast<u32x2*>(p + s * (B * BK * 2)) = (u32x2){a[s], b[s]};
      }
    }
  }

  // 8 consecutive k of row r (this lane's 8 of the 16 of step ks)
  template <Order O, int B>
  static __device__ __forceinline__ bf16x8 frag(const char* lds, int base, int ks, int lane) {
    if constexpr (O == kAlongK) {
      return *reinterpret_cast<const bf16x8*>(lds + at<O, B>(base + (lane & 31), ks * 16 + (lane >> 5) * 8));
    } else {
      // 16 lanes read 4 lines of 16 rows and get 4 k of one row each
      typedef __attribute__((address_space(3))) s16x4 Lds;
      const int k = ks * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2), r = base + (lane & 16) + (lane & 3) * 4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(lds + at<O, B>(r, k)));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(lds + at<O, B>(r, k + 4)));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      return __builtin_bit_cast(bf16x8, (s16x8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
  }

  // acc[mi][nj][r]: row i = base_i + 32 mi + 8 (r / 4) + 4 (lane / 32) + r % 4,
  // column j = base_j + 32 nj + lane % 32
  static __device__ __forceinline__ void product(const Operand& X, const Operand& Y, int64_t i0, int64_t j0, int64_t k0,
                                                 int64_t kend, char* lds, Acc& acc) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int bi = (wave / WJ) * 32 * MI, bj = (wave % WJ) * 32 * NJ;
    u32x4 xv[XU], yv[YU];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[mi][nj][r] = 0.0f;
    load<OX, BI>(X, i0, k0, kend, xv);
    load<OY, BJ>(Y, j0, k0, kend, yv);
    char* buf = lds;
    for (int64_t k = k0; k < kend; k += BK) {
      store<OX, BI>(buf, xv);
      store<OY, BJ>(buf + P * XB, yv);
      if (k + BK < kend) {
        load<OX, BI>(X, i0, k + BK, kend, xv);
        load<OY, BJ>(Y, j0, k + BK, kend, yv);
      }
      lds_only_barrier();   // a wavefront writes this buffer again only after the next barrier
#pragma unroll
      for (int ks = 0; ks < BK / 16; ++ks) {
        bf16x8 x[P][MI], y[P][NJ];
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
          for (int mi = 0; mi < MI; ++mi) x[p][mi] = frag<OX, BI>(buf + p * XB, bi + 32 * mi, ks, lane);
#pragma unroll
          for (int nj = 0; nj < NJ; ++nj) y[p][nj] = frag<OY, BJ>(buf + P * XB + p * YB, bj + 32 * nj, ks, lane);
        }
#pragma unroll
        for (int sum = P - 1; sum >= 0; --sum)   // smallest terms first
#pragma unroll
          for (int p = 0; p <= sum; ++p)
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
              for (int nj = 0; nj < NJ; ++nj)
                acc[mi][nj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[p][mi], y[sum - p][nj], acc[mi][nj], 0, 0, 0);
      }
      buf = buf == lds ? lds + STAGE : lds;
    }
    __syncthreads();   // the buffers are free
  }
};

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
  int64_t m0, m1;           // outputs of this piece (gradient)
  const float* lse; const float* gloss;
  void* dz; int64_t ldz;    // [N][ldz]: the piece's G
  float* cpart;             // [row tiles][ldz]: sums of G over a tile's rows
  int64_t itiles, jtiles;
};

// z of accumulator (mi, nj, r), -inf past the last output
template <class Tl>
__device__ __forceinline__ void add_bias(typename Tl::Acc& acc, const float* bias, int64_t i0, int64_t M) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int64_t i = i0 + 32 * mi + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
      const float b = i >= M ? -__builtin_inff() : bias ? bias[i] : 0.0f;
#pragma unroll
      for (int nj = 0; nj < Tl::NJ; ++nj) acc[mi][nj][r] = i >= M ? b : acc[mi][nj][r] + b;
    }
}

template <class T, Order OW, int BI, int BJ, int WI, int WJ>
__global__ void __launch_bounds__(WI * WJ * 64) xent_tile_kernel(XArgs a) {
  typedef Tile<T, OW, kAlongK, BI, BJ, WI, WJ> Tl;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t jt = blockIdx.x % a.jtiles, it = blockIdx.x / a.jtiles;
  const int64_t i0 = it * BI, j0 = jt * BJ;
  typename Tl::Acc acc;
  Tl::product(a.W, a.A, i0, j0, 0, a.D, lds, acc);
  const int bi = (wave / WJ) * 32 * Tl::MI, bj = (wave % WJ) * 32 * Tl::NJ;
  add_bias<Tl>(acc, a.bias, i0 + bi, a.M);
  float2* red = reinterpret_cast<float2*>(lds);   // [WI][BJ]
#pragma unroll
  for (int nj = 0; nj < Tl::NJ; ++nj) {
    const int64_t j = j0 + bj + 32 * nj + (lane & 31);
    const int64_t t = j < a.N ? a.target[j] : -1;
    float top = -__builtin_inff();
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        top = __builtin_fmaxf(top, acc[mi][nj][r]);
        if (t == i0 + bi + 32 * mi + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3) && t < a.M) a.zt[j] = acc[mi][nj][r];
      }
    top = __builtin_fmaxf(top, __shfl_xor(top, 32));
    float sum = 0.0f;
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum += exp_of(acc[mi][nj][r] - base_of(top));
    sum += __shfl_xor(sum, 32);
    if (lane < 32) red[(wave / WJ) * BJ + bj + 32 * nj + lane] = make_float2(top, sum);
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
    a.part[(j0 + j) * a.itiles + it] = v;
  }
}

// One wavefront per row: lse and loss from the row's tiles.
__global__ void __launch_bounds__(256) xent_join_kernel(const float2* part, const float* zt, const int64_t* target, int64_t N,
                                                        int64_t M, int64_t tiles, float* loss, float* lse) {
  const int lane = threadIdx.x & 63;
  for (int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); n < N; n += (int64_t)gridDim.x * 4) {
    float top = -__builtin_inff();
    for (int64_t t = lane; t < tiles; t += 64) top = __builtin_fmaxf(top, part[n * tiles + t].x);
    for (int o = 1; o < 64; o <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o));
    float sum = 0.0f;
    for (int64_t t = lane; t < tiles; t += 64) {
      const float2 v = part[n * tiles + t];
      sum += v.y * exp_of(v.x - base_of(top));
    }
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) {
      const float l = top + logf(sum);
      const int64_t t = target[n];
      lse[n] = l;
      loss[n] = t < 0 || t >= M ? 0.0f : l == -__builtin_inff() ? __builtin_inff() : l - zt[n];
    }
  }
}

// A tile of G: outputs m0 + i, rows j.
template <class T, Order OW, int BI, int BJ, int WI, int WJ>
__global__ void __launch_bounds__(WI * WJ * 64) xent_dz_kernel(XArgs a) {
  typedef Tile<T, OW, kAlongK, BI, BJ, WI, WJ> Tl;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t jt = blockIdx.x % a.jtiles, it = blockIdx.x / a.jtiles;
  const int64_t i0 = a.m0 + it * BI, j0 = jt * BJ;
  typename Tl::Acc acc;
  Tl::product(a.W, a.A, i0, j0, 0, a.D, lds, acc);
  const int bi = (wave / WJ) * 32 * Tl::MI, bj = (wave % WJ) * 32 * Tl::NJ;
  add_bias<Tl>(acc, a.bias, i0 + bi, a.M);
#pragma unroll
  for (int nj = 0; nj < Tl::NJ; ++nj) {
    const int64_t j = j0 + bj + 32 * nj + (lane & 31);
    const int64_t t = j < a.N ? a.target[j] : -1;
    const float l = j < a.N ? a.lse[j] : 0.0f;
    const bool live = t >= 0 && t < a.M && l != -__builtin_inff();
    const float g = live ? a.gloss[j] : 0.0f;
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t i = i0 + bi + 32 * mi + 8 * q + 4 * (lane >> 5);
        T out[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = exp_of(acc[mi][nj][4 * q + r] - l) - (t == i + r ? 1.0f : 0.0f);
          v = live ? v * g : 0.0f;
          acc[mi][nj][4 * q + r] = v;
          out[r] = from_float<T>(v);
        }
        if (j < a.N && i - a.m0 < a.ldz) {   // (ldz is a multiple of 64)
          T* p = static_cast<T*>(a.dz) + j * a.ldz + (i - a.m0);
          if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(p) = *reinterpret_cast<const u32x2*>(out);
          else *reinterpret_cast<u32x4*>(p) = *reinterpret_cast<const u32x4*>(out);
        }
      }
  }
  // sums over the tile's rows, for the bias gradient
  float* red = reinterpret_cast<float*>(lds);   // [WJ][BI]
#pragma unroll
  for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float s = acc[mi][0][r];
#pragma unroll
      for (int nj = 1; nj < Tl::NJ; ++nj) s += acc[mi][nj][r];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) s += __shfl_xor(s, o);
      if ((lane & 31) == 0) red[(wave % WJ) * BI + bi + 32 * mi + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)] = s;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < BI; i += Tl::NT) {
    float s = red[i];
#pragma unroll
    for (int w = 1; w < WJ; ++w) s += red[w * BI + i];
    if (it * BI + i < a.ldz) a.cpart[jt * a.ldz + it * BI + i] = s;
  }
}

__global__ void __launch_bounds__(256) xent_dbias_kernel(const float* cpart, int64_t jtiles, int64_t ldz, int64_t n, float* out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float s = 0.0f;
    for (int64_t j = 0; j < jtiles; ++j) s += cpart[j * ldz + i];
    out[i] = s;
  }
}

// out[i][j] = sum_k X[i][k] Y[j][k], added to what `sum` holds where it is
// not the first piece; written to `sum` (32 bits) unless it is the last.
// splits > 1: blockIdx.y takes its share of k and leaves it in part[split].
struct GemmArgs {
  Operand X, Y;
  int64_t K;
  int64_t itiles, jtiles;
  void* out; int64_t ldo;
  float* sum;               // [rows of X][rows of Y] or null
  int first, last;
  float* part; int splits; int64_t kper;
};

template <class T, Order OX, Order OY, int BI, int BJ, int WI, int WJ>
__global__ void __launch_bounds__(WI * WJ * 64) xent_gemm_kernel(GemmArgs a) {
  typedef Tile<T, OX, OY, BI, BJ, WI, WJ> Tl;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t jt = blockIdx.x % a.jtiles, it = blockIdx.x / a.jtiles;
  const int64_t i0 = it * BI, j0 = jt * BJ, I = a.X.rows, J = a.Y.rows;
  int64_t k0 = 0, kend = a.K;
  if (a.splits > 1) {
    k0 = blockIdx.y * a.kper;
    kend = k0 + a.kper < a.K ? k0 + a.kper : a.K;
  }
  typename Tl::Acc acc;
  Tl::product(a.X, a.Y, i0, j0, k0, kend, lds, acc);
  const int bi = (wave / WJ) * 32 * Tl::MI, bj = (wave % WJ) * 32 * Tl::NJ;
  float* part = a.splits > 1 ? a.part + blockIdx.y * I * J : nullptr;
#pragma unroll
  for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int64_t i = i0 + bi + 32 * mi + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
#pragma unroll
      for (int nj = 0; nj < Tl::NJ; ++nj) {
        const int64_t j = j0 + bj + 32 * nj + (lane & 31);
        if (i < I && j < J) {
          float v = acc[mi][nj][r];
          if (part) {
            part[i * J + j] = v;
          } else {
            if (!a.first) v += a.sum[i * J + j];
            if (a.last) static_cast<T*>(a.out)[i * a.ldo + j] = from_float<T>(v);
            else a.sum[i * J + j] = v;
          }
        }
      }
    }
}

// Joins the shares of a split product, in order.
template <class T>
__global__ void __launch_bounds__(256) xent_join_splits_kernel(GemmArgs a) {
  const int64_t I = a.X.rows, J = a.Y.rows;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < I * J; e += (int64_t)gridDim.x * 256) {
    float v = a.first ? 0.0f : a.sum[e];
    for (int s = 0; s < a.splits; ++s) v += a.part[s * I * J + e];
    if (a.last) static_cast<T*>(a.out)[e / J * a.ldo + e % J] = from_float<T>(v);
    else a.sum[e] = v;
  }
}

template <class T>
__global__ void __launch_bounds__(256) xent_fill_kernel(T* p, int64_t n) {
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) p[e] = from_float<T>(0.0f);
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int status_from(hipError_t e) { return e == hipSuccess ? MADDNESS_OK : MADDNESS_EHIP; }
int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
int64_t cdiv(int64_t v, int64_t m) { return (v + m - 1) / m; }

constexpr int64_t kMaxBlocks = (1ll << 31) - 1;
constexpr int kWide = 128;   // outputs or columns of a tile
constexpr int kSlots = 512;  // workgroups that fill the card: two to a compute unit

// rows of a logits tile: the wide one where that leaves enough workgroups
int row_tile(int64_t N, int64_t M) { return cdiv(N, kWide) * cdiv(M, kWide) >= 256 ? kWide : 32; }

// Outputs per piece of the gradient: G of a piece stays within 128 MiB (half
// of the memory-side cache), at least 256 outputs.
int64_t piece(int64_t N, int64_t M, int64_t elem) {
  int64_t p = (128ll << 20) / (N * elem) / 256 * 256;
  if (p < 256) p = 256;
  return p < up(M, 64) ? p : up(M, 64);
}

struct GradPlan {
  int64_t p, jt;                 // outputs per piece, row tiles
  int sa, sb;                    // shares of k of dA and dB
  int64_t off_dz, off_c, off_sum, off_part, total;
};

int splits_for(int64_t tiles, int64_t K, int bk) {
  int64_t s = kSlots / (tiles > 0 ? tiles : 1);
  const int64_t most = K / (8 * bk);   // at least 8 steps each
  if (s > most) s = most;
  return s < 1 ? 1 : (int)(s > 64 ? 64 : s);
}

GradPlan grad_plan(int64_t N, int64_t D, int64_t M, int64_t elem, bool md) {
  GradPlan g{};
  const int bk = elem == 2 ? 64 : 32;
  g.p = piece(N, M, elem);
  g.jt = cdiv(N, row_tile(N, g.p));
  g.sa = splits_for(cdiv(N, N <= 32 ? 32 : kWide) * cdiv(D, kWide), g.p, bk);
  g.sb = splits_for(cdiv(D, kWide) * cdiv(g.p, kWide), N, bk);
  int64_t off = 0;
  auto take = [&](int64_t bytes) { const int64_t o = off; off += up(bytes, 256); return o; };
  g.off_dz = take(N * g.p * elem);
  g.off_c = take(g.jt * g.p * 4);
  g.off_sum = take(g.p < M ? N * D * 4 : 0);
  const int64_t pa = g.sa > 1 ? g.sa * N * D * 4 : 0, pb = g.sb > 1 ? g.sb * D * g.p * 4 : 0;
  g.off_part = take(pa > pb ? pa : pb);
  g.total = off > 256 ? off : 256;
  return g;
}

template <class K, class Args>
hipError_t launch(K kernel, int lds, int64_t blocks, int splits, int threads, const Args& a, hipStream_t stream) {
  if (blocks > kMaxBlocks) return hipErrorInvalidValue;
  hipError_t err = hipSuccess;
  launch_prepare(reinterpret_cast<const void*>(kernel), threads, lds, &err);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks, (unsigned)splits), dim3(threads), lds, stream, a);
  return hipGetLastError();
}

template <class T, Order OW, bool GRAD, int BI, int BJ, int WI, int WJ>
hipError_t launch_logits(XArgs& a, int64_t outputs, hipStream_t s) {
  typedef Tile<T, OW, kAlongK, BI, BJ, WI, WJ> Tl;
  a.itiles = cdiv(outputs, BI);
  a.jtiles = cdiv(a.N, BJ);
  if constexpr (GRAD) return launch(xent_dz_kernel<T, OW, BI, BJ, WI, WJ>, Tl::LDS, a.itiles * a.jtiles, 1, Tl::NT, a, s);
  else return launch(xent_tile_kernel<T, OW, BI, BJ, WI, WJ>, Tl::LDS, a.itiles * a.jtiles, 1, Tl::NT, a, s);
}

template <class T, bool GRAD>
hipError_t logits(XArgs& a, int64_t outputs, int rows, bool md, hipStream_t s) {
  if (rows == kWide) return md ? launch_logits<T, kAlongK, GRAD, 128, 128, 2, 2>(a, outputs, s) : launch_logits<T, kAlongI, GRAD, 128, 128, 2, 2>(a, outputs, s);
  return md ? launch_logits<T, kAlongK, GRAD, 128, 32, 4, 1>(a, outputs, s) : launch_logits<T, kAlongI, GRAD, 128, 32, 4, 1>(a, outputs, s);
}

template <class T, Order OX, Order OY, int BI, int BJ, int WI, int WJ>
hipError_t gemm(GemmArgs a, hipStream_t s) {
  typedef Tile<T, OX, OY, BI, BJ, WI, WJ> Tl;
  a.itiles = cdiv(a.X.rows, BI);
  a.jtiles = cdiv(a.Y.rows, BJ);
  a.kper = up(cdiv(a.K, a.splits), Tl::BK);
  a.splits = (int)cdiv(a.K, a.kper);
  hipError_t e = launch(xent_gemm_kernel<T, OX, OY, BI, BJ, WI, WJ>, Tl::LDS, a.itiles * a.jtiles, a.splits, Tl::NT, a, s);
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t b = cdiv(a.X.rows * a.Y.rows, 256);
  hipLaunchKernelGGL((xent_join_splits_kernel<T>), dim3((unsigned)(b < 4096 ? b : 4096)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <class T>
hipError_t grad(XArgs a, bool md, void* dA, void* dB, float* dbias, char* ws, hipStream_t s) {
  const GradPlan g = grad_plan(a.N, a.D, a.M, sizeof(T), md);
  a.dz = ws + g.off_dz;
  a.cpart = reinterpret_cast<float*>(ws + g.off_c);
  T* B = static_cast<T*>(const_cast<void*>(a.W.p));
  for (int64_t m0 = 0; m0 < a.M; m0 += g.p) {
    const int64_t n = a.M - m0 < g.p ? a.M - m0 : g.p;
    a.m0 = m0;
    a.ldz = up(n, 64);
    hipError_t e = logits<T, true>(a, a.ldz, row_tile(a.N, g.p), md, s);
    if (e != hipSuccess) return e;
    const int64_t b = cdiv(n, 256);
    hipLaunchKernelGGL(xent_dbias_kernel, dim3((unsigned)(b < 4096 ? b : 4096)), dim3(256), 0, s, a.cpart, a.jtiles, a.ldz, n, dbias + m0);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const Operand zk{a.dz, a.ldz, a.N}, zi{a.dz, a.ldz, n};
    GemmArgs x{};
    x.sum = reinterpret_cast<float*>(ws + g.off_sum);
    x.part = reinterpret_cast<float*>(ws + g.off_part);
    // dA [N][D] += G B^T over the piece's outputs
    x.X = zk;
    x.Y = Operand{md ? B + m0 * a.W.ld : B + m0, a.W.ld, a.D};
    x.K = n;
    x.out = dA; x.ldo = a.D;
    x.first = m0 == 0; x.last = m0 + n == a.M;
    x.splits = g.sa;
    if (a.N <= 32) e = md ? gemm<T, kAlongK, kAlongI, 32, 128, 1, 4>(x, s) : gemm<T, kAlongK, kAlongK, 32, 128, 1, 4>(x, s);
    else e = md ? gemm<T, kAlongK, kAlongI, 128, 128, 2, 2>(x, s) : gemm<T, kAlongK, kAlongK, 128, 128, 2, 2>(x, s);
    if (e != hipSuccess) return e;
    // dB = A^T G: [D][M] columns m0.., or [M][D] rows m0..
    const Operand ai{a.A.p, a.A.ld, a.D};
    x.X = md ? zi : ai;
    x.Y = md ? ai : zi;
    x.K = a.N;
    x.out = static_cast<T*>(dB) + (md ? m0 * a.D : m0); x.ldo = md ? a.D : a.M;
    x.first = x.last = 1;
    x.splits = g.sb;
    if ((e = gemm<T, kAlongI, kAlongI, 128, 128, 2, 2>(x, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t forward(XArgs a, bool md, float* loss, float* lse, hipStream_t s) {
  hipError_t e = logits<T, false>(a, a.M, row_tile(a.N, a.M), md, s);
  if (e != hipSuccess) return e;
  const int64_t b = cdiv(a.N, 4);
  hipLaunchKernelGGL(xent_join_kernel, dim3((unsigned)(b < 65536 ? b : 65536)), dim3(256), 0, s, a.part, a.zt, a.target, a.N, a.M,
                     a.itiles, loss, lse);
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
  a.W = Operand{B, outputs_first ? D : M, M};
  a.A = Operand{A, lda, N};
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
  return grad_plan(N, D, M, dtype == MADDNESS_F32 ? 4 : 2, false).total;
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
