// Products with 4-bit block floating point weights, their quantizer, and the
// way back (maddness_quantize_w4, maddness_dequantize_w4, maddness_matmul_w4;
// the format is described in include/maddness.h).
//
// A weight is an E2M1 code times 2^e, e shared by 32 rows of a column.  Two
// bits of mantissa times a power of two are exact in bf16, and one instruction
// unpacks two codes and scales them, so a weight costs half an instruction and
// the scale none after the product.
//
// What bounds it: up to about 16 rows the reading of the weights (17 bytes per 32
// of them), from some hundred rows on the products.  Three kernels by rows, each
// with its figures: one column block per workgroup (8 rows and less), activations
// through LDS (up to about a thousand), weights unpacked to memory first.
// Measured, 4096 -> 65536: one bf16 row 43.7 us (3.3 TB/s from memory; 38 when
// the weights stay in the memory-side cache), 64 rows 53, 512 rows 307 (0.9
// PFLOP/s); 4096 rows of fp16, 4096 -> 8192 246 to 258 us (1.07 to 1.12).
#include "tile.hpp"

namespace mdn {
namespace {

constexpr int kWK = 128, kWM = 16;   // rows and columns of a packed block: 64 lanes x 16 bytes

// the 8 codes of one word as bf16, times the power of two
__device__ __forceinline__ bf16x8 unpack8(uint32_t w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return (bf16x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// biased exponent byte j as the power of two it stands for (255: NaN weights)
__device__ __forceinline__ float scale_of(uint32_t exps, int j) {
  return __uint_as_float(((exps >> (8 * j)) & 0xffu) << 23);
}

// 8 consecutive values of a row as bf16 parts; values at or past `left` are 0
template <class T>
__device__ __forceinline__ void load_parts(const T* p, int left, bf16x8 (&out)[Parts<T>::n]) {
  constexpr int P = Parts<T>::n;
  if constexpr (P == 1) {
    u32x4 v = {0, 0, 0, 0};
    if (left >= 8) {
      v = load16(p);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) v[i >> 1] |= (uint32_t)p[i].bits << (16 * (i & 1));
    }
    out[0] = __builtin_bit_cast(bf16x8, v);
  } else {
    float f[8];
    if (left >= 8) {
      if constexpr (sizeof(T) == 4) {
        const u32x4 a = load16(p), b = load16(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = __uint_as_float(a[i]); f[4 + i] = __uint_as_float(b[i]); }
      } else {
        const u32x4 a = load16(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = to_float(T{(uint16_t)(a[i >> 1] >> (16 * (i & 1)))});
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < left ? to_float(p[i]) : 0.0f;
    }
    u32x4 w[P];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t q[P];
      split2<P>(f[2 * i], f[2 * i + 1], q);
#pragma unroll
      for (int s = 0; s < P; ++s) w[s][i] = q[s];
    }
#pragma unroll
    for (int s = 0; s < P; ++s) out[s] = __builtin_bit_cast(bf16x8, w[s]);
  }
}

struct WArgs {
  const void* A; int64_t N, lda; int D, M;
  const uint8_t* codes; const uint8_t* exps;
  const float* bias; int act;   // 0 none, 1 bias, 2 bias + ReLU (a row softmax is a second pass)
  void* y;
  int nk, nm;                   // blocks of 128 rows / 16 columns of the weights
};

__device__ __forceinline__ float w4_sigma(const WArgs& a, float v, int m) {
  if (a.bias) v += a.bias[m];
  return a.act == 2 ? (v > 0.0f ? v : 0.0f) : v;
}

// Few rows: one workgroup takes 16 columns x 16 RT rows, the wavefronts the
// weight's 128-row blocks in turn; their sums are added through LDS.  A
// wavefront has its next four blocks under way at a time: what bounds a single
// row is how many bytes are (65536 columns of 4096 rows, one bf16 row: 43.7
// us, with one block under way 50).
template <class T, class Y, int RT>
__global__ void __launch_bounds__(512) w4_rows_kernel(WArgs a) {
  constexpr int P = Parts<T>::n, U = 4;
  extern __shared__ float red[];   // [wavefronts][RT][16 rows][16 columns]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int col = lane & 15, quarter = lane >> 4;
  const int mb = blockIdx.x;
  const u32x4* codes = reinterpret_cast<const u32x4*>(a.codes) + (int64_t)mb * a.nk * 64 + lane;
  const uint32_t* exps = reinterpret_cast<const uint32_t*>(a.exps) + (int64_t)mb * a.nk * 16 + col;
  const int64_t chunks = (a.N + 16 * RT - 1) / (16 * RT);
  for (int64_t c = blockIdx.y; c < chunks; c += gridDim.y) {
    const int64_t n0 = c * (16 * RT);
    f32x4 acc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r] = (f32x4){0, 0, 0, 0};
    for (int k0 = wave; k0 < a.nk; k0 += waves * U) {
      u32x4 w[U];
      uint32_t e[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int kb = k0 + u * waves < a.nk ? k0 + u * waves : k0;
        w[u] = codes[(int64_t)kb * 64];
        e[u] = exps[kb * 16];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int kb = k0 + u * waves;
        if (kb >= a.nk) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8 b = unpack8(w[u][j], scale_of(e[u], j));
          const int k = kb * kWK + 32 * j + 8 * quarter;
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const int64_t n = n0 + 16 * r + col < a.N ? n0 + 16 * r + col : a.N - 1;   // (results past the end are not written)
            bf16x8 x[P];
            load_parts(static_cast<const T*>(a.A) + n * a.lda + k, a.D - k, x);
#pragma unroll
            for (int p = P - 1; p >= 0; --p) acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[p], b, acc[r], 0, 0, 0);
          }
        }
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[((wave * RT + r) * 16 + 4 * quarter + i) * 16 + col] = acc[r][i];
    __syncthreads();
    for (int t = threadIdx.x; t < RT * 256; t += blockDim.x) {
      float v = red[t];
      for (int w = 1; w < waves; ++w) v += red[w * RT * 256 + t];
      const int64_t n = n0 + (t >> 4);
      const int m = mb * kWM + (t & 15);
      if (n < a.N && m < a.M) static_cast<Y*>(a.y)[n * a.M + m] = from_float<Y>(w4_sigma(a, v, m));
    }
    __syncthreads();
  }
}

// More rows: the activations' parts go through LDS, a 128-column block of 16 RT
// rows at a time (two buffers), and are shared by four wavefronts of 16 CT
// columns each, whose weights go from memory to registers and are unpacked
// there, once for all RT row blocks.  KG groups of four wavefronts take the
// 128-row blocks in turn (each with buffers of its own) where the columns alone
// do not fill the card; their sums are added through LDS.
template <class T, class Y, int RT, int CT, int KG>
__global__ void __launch_bounds__(256 * KG, KG == 1 && Parts<T>::n < 3 ? 2 : 1) w4_block_kernel(WArgs a) {
  constexpr int P = Parts<T>::n, ROWS = 16 * RT, BUF = P * ROWS * kWK * 2;   // bytes of a buffer
  constexpr int UNITS = ROWS * 16 / 256;   // 8-column units of a buffer per thread
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int group = threadIdx.x >> 8, t = threadIdx.x & 255, wave = t >> 6;
  char* buf = lds + group * (2 * BUF);
  const int mb0 = (blockIdx.x * 4 + wave) * CT;
  const int64_t n0 = (int64_t)blockIdx.y * ROWS;
  // a unit's row and place; rows past the end are read as the last one (their results are not written)
  auto load_unit = [&](int i, int kb, bf16x8 (&x)[P]) {
    const int u = t + 256 * i, r = u >> 4, k = kb * kWK + (u & 15) * 8;
    const int64_t n = n0 + r < a.N ? n0 + r : a.N - 1;
    load_parts(static_cast<const T*>(a.A) + n * a.lda + k, a.D - k, x);
  };
  auto store_unit = [&](int i, char* to, const bf16x8 (&x)[P]) {
    const int u = t + 256 * i, r = u >> 4, c = u & 15;
#pragma unroll
    for (int p = 0; p < P; ++p) *reinterpret_cast<bf16x8*>(to + p * (ROWS * kWK * 2) + r * (kWK * 2) + ((c ^ (r & 15)) << 4)) = x[p];
  };
  f32x4 acc[RT][CT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[r][c] = (f32x4){0, 0, 0, 0};
  const u32x4* codes = reinterpret_cast<const u32x4*>(a.codes) + lane;
  const uint32_t* exps = reinterpret_cast<const uint32_t*>(a.exps) + col;
  u32x4 w[CT];
  uint32_t e[CT];
  auto weights = [&](int kb) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const int64_t at = (int64_t)(mb0 + c < a.nm ? mb0 + c : a.nm - 1) * a.nk + kb;
      w[c] = codes[at * 64];
      e[c] = exps[at * 16];
    }
  };
  const int turns = (a.nk + KG - 1) / KG;   // the same for every group: they meet at the barriers
  auto block_of = [&](int s) { return s * KG + group < a.nk ? s * KG + group : a.nk - 1; };
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    bf16x8 x[P];
    load_unit(i, block_of(0), x);
    store_unit(i, buf, x);
  }
  weights(block_of(0));
  for (int s = 0; s < turns; ++s) {
    char* cur = buf + (s & 1) * BUF;
    lds_only_barrier();   // this block is in LDS, and everyone is done with the other buffer
    u32x4 wn[CT];
    uint32_t en[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) { wn[c] = w[c]; en[c] = e[c]; }
    const int next = s + 1 < turns ? block_of(s + 1) : block_of(s);
    weights(next);
    const bool mine = s * KG + group < a.nk;
    bf16x8 held[UNITS > 4 ? 4 : UNITS][P];   // the next block's first units, on their way under the products
#pragma unroll
    for (int i = 0; i < UNITS && i < 4; ++i) load_unit(i, next, held[i]);
    if (mine) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 b[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) b[c] = unpack8(wn[c][j], scale_of(en[c], j));
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const int row = 16 * r + col;
#pragma unroll
          for (int p = P - 1; p >= 0; --p) {
            const bf16x8 x = *reinterpret_cast<const bf16x8*>(cur + p * (ROWS * kWK * 2) + row * (kWK * 2) + (((4 * j + quarter) ^ (row & 15)) << 4));
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, b[c], acc[r][c], 0, 0, 0);
          }
        }
      }
    }
    char* to = buf + ((s + 1) & 1) * BUF;
#pragma unroll
    for (int i = 0; i < UNITS && i < 4; ++i) store_unit(i, to, held[i]);
#pragma unroll
    for (int i = 4; i < UNITS; ++i) {
      bf16x8 x[P];
      load_unit(i, next, x);
      store_unit(i, to, x);
    }
  }
  if constexpr (KG > 1) {
    float* red = reinterpret_cast<float*>(lds) + t;   // [group][r][c][i][256]
    __syncthreads();
    if (group > 0) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) red[(((group - 1) * RT + r) * CT + c) * 1024 + i * 256] = acc[r][c][i];
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int g = 1; g < KG; ++g) acc[r][c][i] += red[(((g - 1) * RT + r) * CT + c) * 1024 + i * 256];
  }
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int m = (mb0 + c) * kWM + col;
    if (m >= a.M) continue;
    const float bias = a.bias ? a.bias[m] : 0.0f;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t n = n0 + 16 * r + 4 * quarter + i;
        const float v = acc[r][c][i] + bias;
        if (n < a.N) static_cast<Y*>(a.y)[n * a.M + m] = from_float<Y>(a.act == 2 && !(v > 0.0f) ? 0.0f : v);
      }
  }
}

// Row softmax in place, one workgroup per row: three passes over a row that
// stays in the L2.
__global__ void __launch_bounds__(1024) w4_softmax_kernel(float* y, int64_t N, int M) {
  __shared__ float part[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    float* row = y + n * M;
    float top = -__builtin_inff();
    for (int m = threadIdx.x; m < M; m += blockDim.x) top = __builtin_fmaxf(top, row[m]);
    for (int o = 1; o < 64; o <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) part[wave] = top;
    __syncthreads();
    for (int w = 0; w < waves; ++w) top = __builtin_fmaxf(top, part[w]);
    __syncthreads();
    float sum = 0.0f;
    for (int m = threadIdx.x; m < M; m += blockDim.x) sum += expf(row[m] - top);
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0f;
    for (int w = 0; w < waves; ++w) sum += part[w];
    __syncthreads();
    for (int m = threadIdx.x; m < M; m += blockDim.x) row[m] = expf(row[m] - top) / sum;
  }
}

struct QArgs {
  const void* B; int64_t sd, sm;   // element (d, m) at d * sd + m * sm
  int D, M, nk, nm;
  uint8_t* codes; uint8_t* exps;
};

// The codes of 8 weights of a group with exponent e (0 where the group is not
// finite): the hardware's conversion, which divides by the power of two, rounds
// to the nearest code, ties to the even one, and stops at 6.  A weight that
// rounds to zero has no sign.
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], int e, bool bad) {
  const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
  const uint32_t some = (w | w >> 1 | w >> 2) & 0x11111111u;   // codes with a magnitude
  return bad ? 0u : w & (0x77777777u | some << 3);
}
// the smallest e with top <= 6 2^e: top = f 2^x, 1/2 <= f < 1, and 6 2^e = 3/4 2^(e + 3)
__device__ __forceinline__ int exponent_of(float top, bool inside) {
  int x = 0;
  const float f = frexpf(top, &x);
  const int e = f <= 0.75f ? x - 3 : x - 2;
  return top == 0.0f ? (inside ? -120 : 0) : e < -120 ? -120 : e > 125 ? 125 : e;
}

// Quantizing is bound by the reading of B and the writing of codes: [65536][4096]
// bf16 one row per output 166 us (4.1 TB/s; 565 with 2-byte loads, 223 with
// the codes found by comparisons), [1024][4096] fp32 about 7 us.
// B with its rows d contiguous (stride_d 1), or any strides.  One wavefront per
// packed block; lane (quarter, column) holds the 32 weights that it will write,
// 8 consecutive rows of each of the block's four groups: 16 or 32 bytes a load,
// a column's 128 rows in whole lines.
template <class T, bool DENSE>
__global__ void __launch_bounds__(256) w4_quantize_kernel(QArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, quarter = lane >> 4;
  const int64_t blocks = (int64_t)a.nk * a.nm;
  for (int64_t b = (int64_t)blockIdx.x * 4 + wave; b < blocks; b += (int64_t)gridDim.x * 4) {
    // neighbours: the next rows of the same columns, or (other strides) the next columns
    const int mb = (int)(DENSE ? b / a.nk : b % a.nm), kb = (int)(DENSE ? b % a.nk : b / a.nm);
    const int m = mb * kWM + col;
    const T* src = static_cast<const T*>(a.B) + m * a.sm;
    float v[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = kb * kWK + 32 * j + 8 * quarter;
      if (DENSE && m < a.M && d + 8 <= a.D) {
        if constexpr (sizeof(T) == 4) {
          const u32x4 x = load16(src + d), y = load16(src + d + 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) { v[j][i] = __uint_as_float(x[i]); v[j][4 + i] = __uint_as_float(y[i]); }
        } else {
          const u32x4 x = load16(src + d);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[j][i] = to_float(T{(uint16_t)(x[i >> 1] >> (16 * (i & 1)))});
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = d + i < a.D && m < a.M ? to_float(src[(d + i) * a.sd]) : 0.0f;
      }
    }
    u32x4 word;
    uint32_t exps = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float top = 0.0f;
      int odd = 0;   // not finite
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        top = __builtin_fmaxf(top, __builtin_fabsf(v[j][i]));
        odd |= !(__builtin_fabsf(v[j][i]) < __builtin_inff());
      }
      top = __builtin_fmaxf(top, __shfl_xor(top, 16));
      top = __builtin_fmaxf(top, __shfl_xor(top, 32));
      odd |= __shfl_xor(odd, 16);
      odd |= __shfl_xor(odd, 32);
      const int e = exponent_of(top, kb * kWK + 32 * j < a.D && m < a.M);
      exps |= (uint32_t)(odd ? 255 : e + 127) << (8 * j);
      word[j] = codes_of(v[j], e, odd);
    }
    const int64_t at = (int64_t)mb * a.nk + kb;
    reinterpret_cast<u32x4*>(a.codes)[at * 64 + lane] = word;
    if (quarter == 0) reinterpret_cast<uint32_t*>(a.exps)[at * 16 + col] = exps;
  }
}

// B with its columns contiguous (stride_m 1): a workgroup takes 64 columns of a
// block, a lane one of them and a wavefront one group of 32 rows, so that every
// load is 128 or 256 bytes of a row and a group's maximum stays in its lane; the
// codes are put together in LDS.
template <class T>
__global__ void __launch_bounds__(256) w4_quantize_rows_kernel(QArgs a) {
  __shared__ uint32_t words[4][4][64];   // [quarter][group][column]
  __shared__ uint8_t bytes[64][4];
  const int lane = threadIdx.x & 63, j = threadIdx.x >> 6;
  const int64_t strips = (a.nm + 3) / 4, blocks = (int64_t)a.nk * strips;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int kb = (int)(b / strips), m = (int)(b % strips) * 64 + lane, d = kb * kWK + 32 * j;
    const T* src = static_cast<const T*>(a.B) + m;
    float v[4][8], top = 0.0f;
    bool odd = false;   // not finite
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[q][i] = d + 8 * q + i < a.D && m < a.M ? to_float(src[(d + 8 * q + i) * a.sd]) : 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        top = __builtin_fmaxf(top, __builtin_fabsf(v[q][i]));
        odd = odd || !(__builtin_fabsf(v[q][i]) < __builtin_inff());
      }
    const int e = exponent_of(top, d < a.D && m < a.M);
    bytes[lane][j] = (uint8_t)(odd ? 255 : e + 127);
#pragma unroll
    for (int q = 0; q < 4; ++q) words[q][j][lane] = codes_of(v[q], e, odd);
    __syncthreads();
    // wavefront j writes quarter j of every column
    const int mb = m >> 4, col = lane & 15;
    if (mb < a.nm) {
      const int64_t at = (int64_t)mb * a.nk + kb;
      reinterpret_cast<u32x4*>(a.codes)[at * 64 + j * 16 + col] = (u32x4){words[j][0][lane], words[j][1][lane], words[j][2][lane], words[j][3][lane]};
      if (j == 0) reinterpret_cast<uint32_t*>(a.exps)[at * 16 + col] = *reinterpret_cast<const uint32_t*>(bytes[lane]);
    }
    __syncthreads();
  }
}

struct DArgs {
  const uint8_t* codes; const uint8_t* exps; int D, M, nk, nm;
  void* B;   // [D][M]
};

// A workgroup takes 64 columns of a block, a lane one of them, a wavefront one
// quarter of the rows: every store is 128 or 256 bytes of a row (4096 x 65536 to
// bf16 113 us, 6 TB/s; with 32-byte stores 197).
template <class T>
__global__ void __launch_bounds__(256) w4_dequantize_kernel(DArgs a) {
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6, col = lane & 15;
  const int64_t strips = (a.nm + 3) / 4, blocks = (int64_t)a.nk * strips;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int kb = (int)(b / strips), m = (int)(b % strips) * 64 + lane;
    if (m >= a.M) continue;
    const int64_t at = (int64_t)(m >> 4) * a.nk + kb;
    const uint32_t e = reinterpret_cast<const uint32_t*>(a.exps)[at * 16 + col];
    const u32x4 w = reinterpret_cast<const u32x4*>(a.codes)[at * 64 + q * 16 + col];
    T* out = static_cast<T*>(a.B) + ((int64_t)kb * kWK + 8 * q) * a.M + m;
    const int left = a.D - kb * kWK - 8 * q;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bf16x8 v = unpack8(w[j], scale_of(e, j));
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (32 * j + i < left) out[(int64_t)(32 * j + i) * a.M] = from_float<T>((float)v[i]);
    }
  }
}

// ------------------------------------------------------------ many rows
// The weights are unpacked to 16 bits once, k contiguous, and go through the
// tile product: bf16 (exact), or for fp16 activations fp16 with each column's
// weights scaled so that its largest exponent becomes 2^12 (its groups stay
// exact down to 35 octaves below that; the product is scaled back).  fp32
// activations become three bf16 parts side by side, over which the weights'
// k runs three times.

struct EArgs {
  const uint8_t* codes; const uint8_t* exps; int nk;
  int64_t rows;        // columns of the weights in this piece (rows of the result)
  void* W; int64_t ld; // [rows][ld], ld = 128 nk
  int32_t* shift;      // [16 * blocks]: the power of two a column's results are to be scaled by (fp16)
};

// One workgroup per 16 columns.
template <class T>
__global__ void __launch_bounds__(256) w4_unpack_kernel(EArgs a) {
  __shared__ int top[256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
  const int64_t mb = blockIdx.x;
  const uint32_t* exps = reinterpret_cast<const uint32_t*>(a.exps) + mb * a.nk * 16;
  int ref = 127;
  if constexpr (std::is_same<T, F16>::value) {
    int most = 0;   // largest exponent of the column, NaN groups (255) aside
    for (int e = threadIdx.x; e < a.nk * 16; e += 256) {
      const uint32_t w = exps[e];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int b = (int)((w >> (8 * j)) & 0xff);
        if (b != 255 && b > most) most = b;
      }
    }
    top[threadIdx.x] = most;
    __syncthreads();
    for (int t = 0; t < 16; ++t) most = top[t * 16 + col] > most ? top[t * 16 + col] : most;
    ref = most - 12;
    if (threadIdx.x < 16) a.shift[mb * 16 + threadIdx.x] = ref - 127;
  }
  const int64_t row = mb * 16 + col;
  T* out = static_cast<T*>(a.W) + row * a.ld;
  for (int kb = wave; kb < a.nk; kb += 4) {
    const u32x4 w = (reinterpret_cast<const u32x4*>(a.codes) + (mb * a.nk + kb) * 64)[lane];
    const uint32_t e = exps[kb * 16 + col];
    if (row >= a.rows) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u32x4 v;
      if constexpr (std::is_same<T, F16>::value) {
        const int b = (int)((e >> (8 * j)) & 0xff);
        const float s = b == 255 ? __uint_as_float(0x7f800000u) : ldexpf(1.0f, b - ref < -60 ? -60 : b - ref);
        v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[j], s, 0));
        v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[j], s, 1));
        v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[j], s, 2));
        v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[j], s, 3));
      } else {
        v = __builtin_bit_cast(u32x4, unpack8(w[j], scale_of(e, j)));
      }
      *reinterpret_cast<u32x4*>(out + kb * kWK + 32 * j + 8 * quarter) = v;
    }
  }
}

struct PArgs {
  const void* A; int64_t N, lda; int D;
  void* out; int64_t ld; int per;   // [N][parts * per], `per` columns a part, zeros behind the D there are
};

// Rows of A as 16-bit parts side by side, 8 columns a thread.
template <class T>
__global__ void __launch_bounds__(256) w4_parts_kernel(PArgs a) {
  const int units = a.per / 8;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < a.N * units; u += (int64_t)gridDim.x * 256) {
    const int64_t n = u / units;
    const int k = (int)(u % units) * 8;
    const T* p = static_cast<const T*>(a.A) + n * a.lda + k;
    uint16_t* out = static_cast<uint16_t*>(a.out) + n * a.ld + k;
    if constexpr (sizeof(T) == 2) {
      const Bf16* q = reinterpret_cast<const Bf16*>(p);   // (the bits as they are)
      bf16x8 x[1];
      load_parts<Bf16>(q, a.D - k, x);
      *reinterpret_cast<u32x4*>(out) = __builtin_bit_cast(u32x4, x[0]);
    } else {
      bf16x8 x[Parts<T>::n];
      load_parts<T>(p, a.D - k, x);
#pragma unroll
      for (int s = 0; s < Parts<T>::n; ++s) *reinterpret_cast<u32x4*>(out + s * a.per) = __builtin_bit_cast(u32x4, x[s]);
    }
  }
}

struct WTArgs {
  Operand W, A;
  int64_t K, N, M;             // M: outputs from this piece's first on
  const float* bias;           // of this piece, or null
  const int32_t* shift;        // of this piece (fp16)
  int act;
  void* y; int64_t ldy;
  int64_t itiles, jtiles;
};

template <class T, class Y, class Tl>
__global__ void __launch_bounds__(Tl::NT, 1) w4_tile_kernel(WTArgs a) {
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63;
  int64_t it, jt;
  tile_of(blockIdx.x, a.itiles, a.jtiles, it, jt);
  const int64_t i0 = it * Tl::BI, j0 = jt * Tl::BJ;
  typename Tl::Acc acc;
  Tl::product(a.W, a.A, i0, j0, 0, a.K, lds_address(lds), acc);
  const int bi = Tl::base_i();
#pragma unroll
  for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int64_t i = i0 + bi + 32 * mi + entry_row(r, lane), at = i < a.M ? i : a.M - 1;
      const float b = a.bias ? a.bias[at] : 0.0f;
      const int e = std::is_same<T, F16>::value ? a.shift[at] : 0;
#pragma unroll
      for (int nj = 0; nj < Tl::NJ; ++nj) {
        float v = acc[mi][nj][r];
        if constexpr (std::is_same<T, F16>::value) v = ldexpf(v, e);
        v += b;
        acc[mi][nj][r] = a.act == 2 && !(v > 0.0f) ? 0.0f : v;
      }
      if ((r & 3) == 3) __builtin_amdgcn_sched_barrier(0);
    }
  write_tile<Y, Tl>(acc, lds, static_cast<Y*>(a.y) + j0 * a.ldy + i0, a.ldy, a.M - i0, a.N - j0);
}

int blocks_for(int64_t waves, int per) {
  const int64_t b = (waves + per - 1) / per, most = 1 << 20;
  return (int)(b < most ? b : most);
}

template <class T>
hipError_t launch_quantize(const QArgs& a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.nk * a.nm;
  if (a.sm == 1 && a.sd != 1) hipLaunchKernelGGL((w4_quantize_rows_kernel<T>), dim3(blocks_for((int64_t)a.nk * ((a.nm + 3) / 4), 1)), dim3(256), 0, s, a);
  else if (a.sd == 1) hipLaunchKernelGGL((w4_quantize_kernel<T, true>), dim3(blocks_for(blocks, 4)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((w4_quantize_kernel<T, false>), dim3(blocks_for(blocks, 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <class T, class Y, int RT>
hipError_t launch_rows(const WArgs& a, hipStream_t stream) {
  const int waves = a.nk < 8 ? a.nk : 8;
  const int64_t chunks = (a.N + 16 * RT - 1) / (16 * RT);
  hipLaunchKernelGGL((w4_rows_kernel<T, Y, RT>), dim3((unsigned)a.nm, (unsigned)(chunks < 65535 ? chunks : 65535)), dim3(64 * waves),
                     waves * RT * 1024, stream, a);
  return hipGetLastError();
}

template <class T, class Y, int RT, int CT, int KG>
hipError_t launch_block(WArgs a, hipStream_t stream) {
  constexpr int kBuffers = KG * 2 * Parts<T>::n * 16 * RT * kWK * 2, kSums = (KG - 1) * RT * CT * 4096;
  constexpr int kLds = kBuffers > kSums ? kBuffers : kSums;
  static_assert(kLds <= kLdsBytes, "LDS");
  hipError_t err = hipSuccess;
  auto kernel = w4_block_kernel<T, Y, RT, CT, KG>;
  launch_prepare(reinterpret_cast<const void*>(kernel), 256 * KG, kLds, &err);
  if (err != hipSuccess) return err;
  constexpr int64_t kRows = 65535ll * 16 * RT;   // of one launch
  for (int64_t left = a.N; left > 0; left -= kRows) {
    a.N = left < kRows ? left : kRows;
    hipLaunchKernelGGL(kernel, dim3((unsigned)cdiv(a.nm, 4 * CT), (unsigned)cdiv(a.N, 16 * RT)), dim3(256 * KG), kLds, stream, a);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    a.A = static_cast<const T*>(a.A) + kRows * a.lda;
    a.y = static_cast<Y*>(a.y) + kRows * a.M;
  }
  return hipSuccess;
}

// From how many rows on the weights are unpacked first, which costs about 1.2
// ps a weight.  The block kernel then multiplies at 0.9 PFLOP/s a part of the
// activations (bf16 one, fp16 two, fp32 three) and the tiles at 1.2 to 1.3 (fp16
// one part): 4096 -> 65536, 512 rows of bf16 303 against 383 us, of fp32 827
// against 748.
constexpr int64_t many_rows(int32_t dtype) { return dtype == MADDNESS_BF16 ? 1536 : dtype == MADDNESS_F16 ? 448 : 1024; }

// The plan for many rows; bytes: workspace, 0 where the rows kernel takes the call.
struct Many {
  int parts; bool direct;   // 16-bit parts of A; A's rows go to LDS as they are
  int64_t per, rows, piece, off_shift, off_w, bytes;
};
Many plan_many(const void* A, int32_t dtype, int64_t N, int32_t D, int64_t lda, int32_t M) {
  Many p{};
  if (N <= many_rows(dtype)) return p;
  p.parts = dtype == MADDNESS_F32 ? 3 : 1;
  p.direct = dtype != MADDNESS_F32 && D % 64 == 0 && direct(Operand{A, lda, N, N, 0}, false);
  p.per = ((int64_t)D + kWK - 1) / kWK * kWK;
  // rows at a time whose parts are made: 256 MiB of them, at least 4096
  p.rows = (128ll << 20) / (p.parts * p.per) / 256 * 256;
  if (p.rows < 4096) p.rows = 4096;
  if (p.direct || p.rows > N) p.rows = N;
  // outputs at a time: their 16-bit weights within 256 MiB, at least 256 outputs
  p.piece = (128ll << 20) / p.per / 256 * 256;
  if (p.piece < 256) p.piece = 256;
  if (p.piece > up(M, 16)) p.piece = up(M, 16);
  int64_t off = p.direct ? 0 : up(p.rows * p.parts * p.per * 2, 256);
  p.off_shift = off;
  off += dtype == MADDNESS_F16 ? up(p.piece * 4, 256) : 0;
  p.off_w = off;
  p.bytes = off + up(p.piece * p.per * 2, 256);
  return p;
}

template <class T, class Y, class Tl>
hipError_t launch_tile(WTArgs& a, hipStream_t s) {
  a.itiles = cdiv(a.M, Tl::BI);
  a.jtiles = cdiv(a.N, Tl::BJ);
  return launch(w4_tile_kernel<T, Y, Tl>, Tl::LDS, a.itiles * a.jtiles, 1, Tl::NT, a, s);
}

// T: what the tiles multiply (bf16, or fp16 for fp16 activations)
template <class A, class T, class Y>
hipError_t launch_many(const WArgs& a, const Many& p, char* ws, hipStream_t s) {
  WTArgs t{};
  t.act = a.act; t.ldy = a.M;
  t.shift = reinterpret_cast<int32_t*>(ws + p.off_shift);
  const bool wide = p.direct || p.parts * p.per <= (1 << 22);   // offsets of a 256 x 256 tile fit in 32 bits
  for (int64_t n0 = 0; n0 < a.N; n0 += p.rows) {
    t.N = a.N - n0 < p.rows ? a.N - n0 : p.rows;
    t.A = Operand{a.A, a.lda, t.N, t.N, 0};
    t.K = a.D;
    if (!p.direct) {
      PArgs q{static_cast<const A*>(a.A) + n0 * a.lda, t.N, a.lda, a.D, ws, p.parts * p.per, (int)p.per};
      hipLaunchKernelGGL((w4_parts_kernel<A>), dim3(blocks_for(t.N * (p.per / 8), 256)), dim3(256), 0, s, q);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      t.A = Operand{ws, p.parts * p.per, t.N, t.N, 0};
      t.K = p.parts * p.per;
    }
    for (int64_t m0 = 0; m0 < a.M; m0 += p.piece) {
      const int64_t n = a.M - m0 < p.piece ? a.M - m0 : p.piece, at = m0 / kWM * a.nk;
      EArgs e{a.codes + at * 1024, a.exps + at * 64, a.nk, n, ws + p.off_w, p.per, reinterpret_cast<int32_t*>(ws + p.off_shift)};
      hipLaunchKernelGGL((w4_unpack_kernel<T>), dim3((unsigned)cdiv(n, kWM)), dim3(256), 0, s, e);
      hipError_t err = hipGetLastError();
      if (err != hipSuccess) return err;
      t.W = Operand{ws + p.off_w, p.per, n, n, p.per};
      t.M = n;
      t.bias = a.bias ? a.bias + m0 : nullptr;
      t.y = static_cast<Y*>(a.y) + n0 * a.M + m0;
      // 256 x 256 tiles where they leave work for most compute units
      if (wide && t.N >= 192 && cdiv(t.N, 256) * cdiv(n, 256) >= 192) err = launch_tile<T, Y, BigTile<T, kAlongK, kAlongK, false>>(t, s);
      else err = launch_tile<T, Y, Tile<T, kAlongK, kAlongK, 128, 128, 2, 2>>(t, s);
      if (err != hipSuccess) return err;
    }
  }
  return hipSuccess;
}

template <class T, class Y>
hipError_t launch_w4(const WArgs& a, const Many& p, char* ws, hipStream_t stream) {
  if (p.bytes > 0 && ws)
    return launch_many<T, typename std::conditional<std::is_same<T, F16>::value, F16, Bf16>::type, Y>(a, p, ws, stream);
  // (9 to 16 rows of a wide layer too: 4096 -> 65536, 16 of bf16 52 against 74 us)
  if (a.N <= 8 || (a.N <= 16 && cdiv(a.nm, 16) < 160)) return launch_rows<T, Y, 1>(a, stream);
  // more rows: the widest wavefronts that still leave a workgroup for most compute units
  const int64_t rows = cdiv(a.N, 64);
  if (cdiv(a.nm, 16) * rows >= 160) return launch_block<T, Y, 4, 4, 1>(a, stream);
  if (cdiv(a.nm, 8) * rows >= 160) return launch_block<T, Y, 4, 2, 1>(a, stream);
  if (cdiv(a.nm, 4) * rows >= 160 || a.nk == 1) return launch_block<T, Y, 4, 1, 1>(a, stream);
  // (as many groups as have LDS for their buffers)
  if constexpr (Parts<T>::n == 1) return launch_block<T, Y, 4, 1, 4>(a, stream);
  else if constexpr (Parts<T>::n == 2) return launch_block<T, Y, 2, 1, 4>(a, stream);
  else return launch_block<T, Y, 2, 1, 3>(a, stream);
}

}  // namespace
}  // namespace mdn

using namespace mdn;

// the kernels count rows and columns in 32 bits, whole blocks of them too
static bool too_large(int32_t D, int32_t M) { return D > INT32_MAX - kWK || M > INT32_MAX - kWK; }

extern "C" {

int64_t maddness_w4_code_bytes(int32_t D, int32_t M) {
  if (D <= 0 || M <= 0) return -1;
  return (((int64_t)D + kWK - 1) / kWK) * (((int64_t)M + kWM - 1) / kWM) * 1024;
}

int64_t maddness_w4_exponent_bytes(int32_t D, int32_t M) {
  const int64_t n = maddness_w4_code_bytes(D, M);
  return n < 0 ? -1 : n / 16;
}

int maddness_quantize_w4(const void* B, int32_t dtype, int32_t D, int32_t M, int64_t stride_d, int64_t stride_m,
                         uint8_t* codes_out, uint8_t* exps_out, void* stream) {
  if (D <= 0 || M <= 0 || stride_d < 0 || stride_m < 0 || !B || !codes_out || !exps_out) return MADDNESS_EINVAL;
  if (dtype < MADDNESS_F32 || dtype > MADDNESS_F16) return MADDNESS_EINVAL;
  if (!aligned(B, dtype == MADDNESS_F32 ? 4 : 2) || !aligned(codes_out, 16) || !aligned(exps_out, 4)) return MADDNESS_EINVAL;
  if (too_large(D, M)) return MADDNESS_EUNSUPPORTED;
  QArgs a{B, stride_d, stride_m, D, M, (int)(((int64_t)D + kWK - 1) / kWK), (int)(((int64_t)M + kWM - 1) / kWM), codes_out, exps_out};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return status_from(dtype == MADDNESS_F32 ? launch_quantize<float>(a, s) : dtype == MADDNESS_BF16 ? launch_quantize<Bf16>(a, s) : launch_quantize<F16>(a, s));
}

int maddness_dequantize_w4(const uint8_t* codes, const uint8_t* exps, int32_t D, int32_t M, void* B_out, int32_t dtype,
                           void* stream) {
  if (D <= 0 || M <= 0 || !codes || !exps || !B_out) return MADDNESS_EINVAL;
  if (dtype != MADDNESS_F32 && dtype != MADDNESS_BF16) return MADDNESS_EINVAL;
  if (!aligned(B_out, dtype == MADDNESS_F32 ? 4 : 2) || !aligned(codes, 16) || !aligned(exps, 4)) return MADDNESS_EINVAL;
  if (too_large(D, M)) return MADDNESS_EUNSUPPORTED;
  DArgs a{codes, exps, D, M, (int)(((int64_t)D + kWK - 1) / kWK), (int)(((int64_t)M + kWM - 1) / kWM), B_out};
  const dim3 grid(blocks_for((int64_t)a.nk * ((a.nm + 3) / 4), 1));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == MADDNESS_F32) hipLaunchKernelGGL((w4_dequantize_kernel<float>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((w4_dequantize_kernel<Bf16>), grid, dim3(256), 0, s, a);
  return status_from(hipGetLastError());
}

int64_t maddness_matmul_w4_workspace_bytes(const void* A, int32_t dtype, int64_t N, int32_t D, int64_t lda, int32_t M) {
  if (N < 0 || D <= 0 || M <= 0 || lda < D || dtype < MADDNESS_F32 || dtype > MADDNESS_F16) return -1;
  return plan_many(A, dtype, N, D, lda, M).bytes;
}

int maddness_matmul_w4(const void* A, int32_t dtype, int64_t N, int32_t D, int64_t lda, const uint8_t* codes,
                       const uint8_t* exps, int32_t M, const float* col_bias, int32_t act, void* y_out,
                       int32_t y_dtype, void* workspace, int64_t workspace_bytes, void* stream) {
  if (N < 0 || D <= 0 || M <= 0 || lda < D || act < 0 || act > 3) return MADDNESS_EINVAL;
  if (dtype < MADDNESS_F32 || dtype > MADDNESS_F16 || (y_dtype != dtype && y_dtype != MADDNESS_F32)) return MADDNESS_EINVAL;
  if (act == MADDNESS_ACT_SOFTMAX && y_dtype != MADDNESS_F32) return MADDNESS_EINVAL;
  if (too_large(D, M)) return MADDNESS_EUNSUPPORTED;
  if (N == 0) return MADDNESS_OK;
  if (!A || !codes || !exps || !y_out) return MADDNESS_EINVAL;
  if (!aligned(A, dtype == MADDNESS_F32 ? 4 : 2) || !aligned(y_out, y_dtype == MADDNESS_F32 ? 4 : 2) || !aligned(codes, 16) ||
      !aligned(exps, 4) || (col_bias && !aligned(col_bias, 4)))
    return MADDNESS_EINVAL;
  const Many p = plan_many(A, dtype, N, D, lda, M);
  if (workspace && p.bytes > 0 && (!aligned(workspace, 256) || workspace_bytes < p.bytes)) return MADDNESS_EINVAL;
  char* ws = static_cast<char*>(workspace);
  WArgs a{A, N, lda, D, M, codes, exps, act == MADDNESS_ACT_NONE ? nullptr : col_bias, act == MADDNESS_ACT_RELU ? 2 : 0, y_out,
          (int)(((int64_t)D + kWK - 1) / kWK), (int)(((int64_t)M + kWM - 1) / kWM)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (dtype == MADDNESS_F32) e = launch_w4<float, float>(a, p, ws, s);
  else if (dtype == MADDNESS_BF16) e = y_dtype == MADDNESS_F32 ? launch_w4<Bf16, float>(a, p, ws, s) : launch_w4<Bf16, Bf16>(a, p, ws, s);
  else e = y_dtype == MADDNESS_F32 ? launch_w4<F16, float>(a, p, ws, s) : launch_w4<F16, F16>(a, p, ws, s);
  if (e != hipSuccess || act != MADDNESS_ACT_SOFTMAX) return status_from(e);
  hipLaunchKernelGGL(w4_softmax_kernel, dim3((unsigned)(N < 65535 ? N : 65535)), dim3(1024), 0, s, static_cast<float*>(y_out), N, M);
  return status_from(hipGetLastError());
}

}  // extern "C"
