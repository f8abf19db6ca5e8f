// Tile products on the matrix cores, shared by the output layer's kernels
// (linear_xent.hip, w4_matmul.hip): C[i][j] = sum_k X[i][k] Y[j][k], each operand
// with k or its own index contiguous in memory, 32-bit sums, and the ways a tile
// leaves for memory as out[j][i].
#pragma once
#include "maddness.h"
#include "internal.hpp"
#include "mma.hpp"

#include <type_traits>

namespace mdn {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// 32 x 32 x 16 products of 8 values a lane, bf16 (fp32's parts too) or fp16
template <class T>
__device__ __forceinline__ f32x16 multiply_add(bf16x8 x, bf16x8 y, f32x16 c) {
  if constexpr (std::is_same<T, F16>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
}

enum Order : int { kAlongK = 0, kAlongI = 1 };   // which index of an operand is contiguous

struct Operand {
  const void* p;
  int64_t ld;     // elements between rows (kAlongK) or between k steps (kAlongI)
  int64_t rows;   // extent of the operand's own index
  int64_t pad;    // what of it memory holds (kAlongI: whole 16-byte units from `rows` on)
  int64_t wrap;   // k after which the operand begins again (a multiple of 64; 0: it does not)
};

// Where a tile's wavefronts stand: WI x WJ of them side by side, WK times over
// (each time for other k of a step; all WK end with the whole sums, and the
// first of them writes).
template <int WI, int WJ, int WK, int MI, int NJ>
struct Waves {
  // (read as scalars, so that the compiler knows them the same in every lane)
  static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % (WI * WJ); }
  static __device__ __forceinline__ int wk() { return WK == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / (WI * WJ); }
  static __device__ __forceinline__ bool lead() { return WK == 1 || wk() == 0; }
  static __device__ __forceinline__ int wi() { return wave() / WJ; }
  static __device__ __forceinline__ int wj() { return wave() % WJ; }
  static __device__ __forceinline__ int base_i() { return wi() * 32 * MI; }
  static __device__ __forceinline__ int base_j() { return wj() * 32 * NJ; }
};

// A tile of BI x BJ results of one workgroup, k in steps of BK through two LDS
// buffers.
template <class T, Order OX, Order OY, int BI_, int BJ_, int WI_, int WJ_, int BK_ = sizeof(T) == 2 ? 64 : 32, int WK = 1>
struct Tile : Waves<WI_, WJ_, WK, BI_ / WI_ / 32, BJ_ / WJ_ / 32> {
  typedef Waves<WI_, WJ_, WK, BI_ / WI_ / 32, BJ_ / WJ_ / 32> Place;
  static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_;
  static constexpr int P = sizeof(T) == 2 ? 1 : Parts<T>::n;   // 16-bit types as they are
  static constexpr int BK = BK_;
  static constexpr int CH = 16 / sizeof(T);          // elements of a 16-byte unit
  static constexpr int NT = WI * WJ * WK * 64;
  static constexpr int MI = BI / WI / 32, NJ = BJ / WJ / 32;
  static constexpr int XU = BI * BK / CH / NT, YU = BJ * BK / CH / NT;   // units a thread moves per step
  static constexpr int XB = BI * BK * 2, YB = BJ * BK * 2;               // bytes of one part's LDS tile
  static constexpr int STAGE = P * (XB + YB);
  static constexpr int LDS = 2 * STAGE;
  // steps loaded ahead into registers: memory takes longer than a step's products
  // (of 16-bit types; fp32's splits and six products take longer than it)
  static constexpr int AHEAD = P == 1 ? 3 : 1;
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
      const int s = U == 16 ? r & 15 : U == 8 ? (r >> 1) & 7 : (r >> 2) & 3;
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

  // The leading steps of k0 .. kend that lie in the operand's memory whole: rows
  // past its end are read as what stands there (along k: as its last row), and
  // reach only results that are not written.
  template <Order O, int B>
  static __device__ __forceinline__ int64_t whole_steps(const Operand& o, int64_t r0, int64_t k0, int64_t kend) {
    const int64_t full = (kend - k0) / BK;
    if (O == kAlongK) return full;
    // step s: (k0 + s BK + BK - 1) ld + r0 + B <= (kend - 1) ld + rows
    const int64_t over = r0 + B - o.rows, lines = over > 0 ? (over + o.ld - 1) / o.ld : 0, n = (kend - k0 - lines) / BK;
    return kend - k0 < lines ? 0 : n < full ? n : full;
  }

  // units of such a step
  template <Order O, int B, int U>
  static __device__ __forceinline__ void load_whole(const Operand& o, int64_t r0, int64_t k0, u32x4 (&v)[U]) {
    const T* base = static_cast<const T*>(o.p) + (O == kAlongK ? r0 * o.ld + k0 : k0 * o.ld + r0);
    const int64_t last = o.rows - 1 - r0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int r, k;
      unit<O, B>(threadIdx.x + i * NT, r, k);
      v[i] = load16(base + (O == kAlongK ? (r < last ? r : last) * o.ld + k : k * o.ld + r));
    }
  }

  // units of any step, zeros past the matrix and past kend: those inside first,
  // so that all of them are under way at once, then those that the end cuts
  template <Order O, int B, int U>
  static __device__ __forceinline__ void load(const Operand& o, int64_t r0, int64_t k0, int64_t kend, u32x4 (&v)[U]) {
    const T* base = static_cast<const T*>(o.p) + (O == kAlongK ? r0 * o.ld + k0 : k0 * o.ld + r0);
    bool cut = false;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int r, k;
      unit<O, B>(threadIdx.x + i * NT, r, k);
      const int64_t left = r0 + r >= o.rows || k0 + k >= kend ? 0 : O == kAlongK ? kend - (k0 + k) : o.rows - (r0 + r);
      v[i] = (u32x4){0, 0, 0, 0};
      if (left >= CH) v[i] = load16(base + (O == kAlongK ? r * o.ld + k : k * o.ld + r));
      cut |= left > 0 && left < CH;
    }
    if (__any(cut)) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        int r, k;
        unit<O, B>(threadIdx.x + i * NT, r, k);
        const int64_t left = r0 + r >= o.rows || k0 + k >= kend ? 0 : O == kAlongK ? kend - (k0 + k) : o.rows - (r0 + r);
        if (left <= 0 || left >= CH) continue;
        const T* p = base + (O == kAlongK ? r * o.ld + k : k * o.ld + r);
#pragma unroll
        for (int e = 0; e < CH - 1; ++e) {
          const T x = p[e < left ? e : 0];
          if constexpr (CH == 4) v[i][e] = e < left ? __float_as_uint(x) : 0u;
          else v[i][e >> 1] |= (e < left ? (uint32_t)x.bits : 0u) << (16 * (e & 1));
        }
      }
    }
  }

  // The same without a divergent branch (for BigTile, whose sums leave no
  // registers to save around one; its operands have 8 elements and more): units
  // inside are loaded as they are and the others' places from the operand's
  // start, then, where an end cuts units, every element from the nearest one.
  template <Order O, int B, int U>
  static __device__ __forceinline__ void load_flat(const Operand& o, int64_t r0, int64_t k0, int64_t kend, u32x4 (&v)[U]) {
    const T *origin = static_cast<const T*>(o.p), *base = origin + (O == kAlongK ? r0 * o.ld + k0 : k0 * o.ld + r0);
    const int64_t last_r = o.rows - 1 - r0, last_k = kend - 1 - k0;
    const bool cuts = (O == kAlongK ? kend - k0 : o.rows - r0) % CH != 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int r, k;
      unit<O, B>(threadIdx.x + i * NT, r, k);
      const bool full = O == kAlongK ? r <= last_r && k + CH - 1 <= last_k : r + CH - 1 <= last_r && k <= last_k;
      v[i] = load16(full ? base + (O == kAlongK ? r * o.ld + k : k * o.ld + r) : origin);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = full ? v[i][e] : 0u;
    }
    if (cuts) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        int r, k;
        unit<O, B>(threadIdx.x + i * NT, r, k);
        const bool cut = O == kAlongK ? r <= last_r && k <= last_k && k + CH - 1 > last_k : r <= last_r && r + CH - 1 > last_r && k <= last_k;
#pragma unroll
        for (int e = 0; e < CH - 1; ++e) {
          const int re = O == kAlongK ? r : r + e, ke = O == kAlongK ? k + e : k;
          const int64_t rc = re < last_r ? re : last_r, kc = ke < last_k ? ke : last_k;
          const T x = base[O == kAlongK ? rc * o.ld + kc : kc * o.ld + rc];
          const bool in = cut && re <= last_r && ke <= last_k;
          if constexpr (CH == 4) v[i][e] = in ? __float_as_uint(x) : v[i][e];
          else v[i][e >> 1] |= (in ? (uint32_t)x.bits : 0u) << (16 * (e & 1));
        }
        __builtin_amdgcn_sched_barrier(0);   // (a unit at a time: few registers)
      }
    }
  }

  template <Order O, int B, int U>
  static __device__ __forceinline__ void store(uint32_t lds, const u32x4 (&v)[U]) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int r, k;
      unit<O, B>(threadIdx.x + i * NT, r, k);
      const uint32_t p = lds + at<O, B>(r, k);
      if constexpr (P == 1) {
        *lds_at<u32x4>(p) = v[i];
      } else {
        uint32_t a[P], b[P];
        split2<P>(__uint_as_float(v[i][0]), __uint_as_float(v[i][1]), a);
        split2<P>(__uint_as_float(v[i][2]), __uint_as_float(v[i][3]), b);
#pragma unroll
        for (int s = 0; s < P; ++s) *lds_at<u32x2>(p + s * (B * BK * 2)) = (u32x2){a[s], b[s]};
      }
    }
  }

  // 8 consecutive k of row r (this lane's 8 of the 16 of step ks)
  template <Order O, int B>
  static __device__ __forceinline__ bf16x8 frag(uint32_t lds, int base, int ks, int lane) {
    if constexpr (O == kAlongK) {
      return *lds_at<const bf16x8>(lds + at<O, B>(base + (lane & 31), ks * 16 + (lane >> 5) * 8));
    } else {
      // 16 lanes read 4 lines of 16 rows and get 4 k of one row each
      const int k = ks * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2), r = base + (lane & 16) + (lane & 3) * 4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(lds + at<O, B>(r, k)));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(lds + at<O, B>(r, k + 4)));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      return __builtin_bit_cast(bf16x8, (s16x8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
  }

  // acc[mi][nj][r]: row i = base_i + 32 mi + 8 (r / 4) + 4 (lane / 32) + r % 4,
  // column j = base_j + 32 nj + lane % 32
  static __device__ __forceinline__ void product(const Operand& X, const Operand& Y, int64_t i0, int64_t j0, int64_t k0,
                                                 int64_t kend, uint32_t lds, Acc& acc) {
    const int lane = threadIdx.x & 63, bi = Place::base_i(), bj = Place::base_j();
    u32x4 xv[AHEAD][XU], yv[AHEAD][YU];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[mi][nj][r] = 0.0f;
    auto multiply = [&](uint32_t buf) {
#pragma unroll
      for (int n = 0; n < BK / 16 / WK; ++n) {
        const int ks = n * WK + Place::wk();
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
                acc[mi][nj] = multiply_add<T>(x[p][mi], y[sum - p][nj], acc[mi][nj]);
      }
    };
    if (k0 >= kend) return;
    // whole steps, loaded AHEAD of their use without a branch (so that a use
    // waits for its own step's loads alone; past the last, that one again)
    const int64_t sx = whole_steps<OX, BI>(X, i0, k0, kend), sy = whole_steps<OY, BJ>(Y, j0, k0, kend), whole = sx < sy ? sx : sy;
    uint32_t buf = lds;
    if (whole > 0) {
      int64_t kx = k0, ky = k0, left = whole;   // the next step to load
      auto fetch = [&](int u) {
        load_whole<OX, BI>(X, i0, kx, xv[u]);
        load_whole<OY, BJ>(Y, j0, ky, yv[u]);
        const int64_t d = --left > 0 ? BK : 0;
        kx += d;
        ky += d;
        kx = d && X.wrap && kx == X.wrap ? 0 : kx;
      };
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) fetch(u);
      for (int64_t s = 0; s < whole; s += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          if (s + u >= whole) break;
          store<OX, BI>(buf, xv[u]);
          store<OY, BJ>(buf + P * XB, yv[u]);
          fetch(u);
          lds_only_barrier();   // a wavefront writes this buffer again only after the next barrier
          multiply(buf);
          buf = buf == lds ? lds + STAGE : lds;
        }
      }
    }
    for (int64_t k = k0 + whole * BK; k < kend; k += BK) {   // what is left, with checks (X.wrap leaves none)
      load<OX, BI>(X, i0, k, kend, xv[0]);
      load<OY, BJ>(Y, j0, k, kend, yv[0]);
      store<OX, BI>(buf, xv[0]);
      store<OY, BJ>(buf + P * XB, yv[0]);
      lds_only_barrier();
      multiply(buf);
      buf = buf == lds ? lds + STAGE : lds;
    }
    __syncthreads();   // the buffers are free
    if constexpr (WK > 1) {   // the sums over k of all WK, in order
      static_assert(WK * BI * BJ * 4 <= LDS, "sums");
      float* own = (float*)lds_at<float>(lds) + Place::wave() * (MI * NJ * 1024) + lane;
#pragma unroll
      for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj)
#pragma unroll
          for (int r = 0; r < 16; ++r) own[Place::wk() * (BI * BJ) + (mi * NJ + nj) * 1024 + r * 64] = acc[mi][nj][r];
      __syncthreads();
#pragma unroll
      for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float v = own[(mi * NJ + nj) * 1024 + r * 64];
#pragma unroll
            for (int w = 1; w < WK; ++w) v += own[w * (BI * BJ) + (mi * NJ + nj) * 1024 + r * 64];
            acc[mi][nj][r] = v;
          }
      __syncthreads();
    }
  }
};

// The tile of large products of 16-bit matrices: 256 x 256 results of four wavefronts, 128 x
// 128 each, one to a SIMD with its sums in the accumulation registers.  LDS
// reads are then half of what the matrix cores take the time for (128 KB of
// reads and 64 KB of writes per 64 k against 2048 cycles of 128 bytes), where
// eight wavefronts of 128 x 64 would need all of it.  Steps of 64 k (whole
// 128-byte lines of rows along k) go from memory straight to LDS: five 32 KB
// slots hold this step's two operands, the next step's and the first of the one
// after.  A step's only barrier stands before its last quarter, whose operands
// are in registers by then; the two slots that it frees are filled in the three
// quarters that follow.  Reads and transfers are issued between products, a few
// at a time, since a wavefront waits where the memory pipeline's queue is full.
// STAGED_X: an operand X whose rows are not whole 16-byte units goes through
// registers instead (15% slower).
// Measured, 8192 x 4096 x 65536 with the logits reduced in the kernel: 1.36
// PFLOP/s, where the library's product alone reaches 1.51; two 64-k buffers
// filled in one burst 1.08, four buffers of 32 k (half lines of rows along k)
// 1.20.  The matrix cores are busy 70% of the time at 1.8 to 1.9 GHz, the clock
// that the card holds under them; waits at the barrier take 20%.
template <class T, Order OX, Order OY, bool STAGED_X>
struct BigTile : Waves<2, 2, 1, 4, 4> {
  static constexpr int BI = 256, BJ = 256, BK = 64, WI = 2, WJ = 2, MI = 4, NJ = 4, NT = 256;
  static constexpr uint32_t SLOT = 256 * BK * 2, LDS = 5 * SLOT;
  static constexpr int U = 8;                                     // 16-byte units per thread and operand of a step
  typedef f32x16 Acc[MI][NJ];
  typedef Tile<T, OX, OY, 256, 256, 2, 2, BK> Small;           // the LDS layout and guarded loads are its

  // byte offset of this lane's unit of transfer q from the step's origin; the
  // transfer fills 1 KB of LDS in lane order, so the lane fetches what the
  // layout has in its place.  Units past the matrix repeat its last ones: they
  // reach only results that are not written.
  template <Order O>
  static __device__ __forceinline__ uint32_t offset(const Operand& o, int64_t r0, int q) {
    const int lane = threadIdx.x & 63, block = (threadIdx.x >> 6) * U + q;
    if constexpr (O == kAlongK) {
      int64_t r = block * 8 + (lane >> 3);
      const int k = ((lane & 7) ^ ((r >> 1) & 7)) * 8;
      if (r > o.rows - 1 - r0) r = o.rows - 1 - r0;
      return (uint32_t)((r * o.ld + k) * 2);
    } else {
      const int k = block * 2 + (lane >> 5);
      int64_t r = ((((lane & 31) >> 2) ^ (k & 3)) * 4 + (lane & 3)) * 8;
      if (r > o.pad - 8 - r0) r = o.pad - 8 - r0;
      return (uint32_t)((k * o.ld + r) * 2);
    }
  }

  // 16 bytes a lane from base + off to LDS, 1 KB from `to` on (uniform).  In
  // assembly, since the compiler has every LDS read wait for all transfers under
  // way that it knows of; product() waits for those that a read needs.  (The
  // wait states cover a base that a vector instruction has just written, too.)
  static __device__ __forceinline__ void transfer(const char* base, uint32_t off, uint32_t to) {
#ifdef __OPTIMIZE__
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
#else   // (uniform values stay in vector registers there, which the assembly cannot take)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + off), lds_at<void>(to), 16, 0, 0);
#endif
  }

  template <Order O>
  struct Stream {
    const char* base;       // the next step's origin
    int64_t step;           // bytes from a step to the next
    uint32_t to;            // this wavefront's part of a slot
    int left, wrap;         // steps to the operand's end, steps it has (0: no end)
    uint32_t off[U];

    __device__ __forceinline__ void init(const Operand& o, int64_t r0, int64_t k0, uint32_t lds) {
      base = static_cast<const char*>(o.p) + (O == kAlongK ? r0 * o.ld + k0 : k0 * o.ld + r0) * 2;
      step = (O == kAlongK ? (int64_t)BK : BK * o.ld) * 2;
      to = __builtin_amdgcn_readfirstlane(lds + (threadIdx.x >> 6) * (U * 1024));
      left = wrap = (int)(o.wrap / BK);
#pragma unroll
      for (int q = 0; q < U; ++q) off[q] = offset<O>(o, r0, q);
    }
    // transfer q of the next step, into the slot at `at`; the last one moves on
    __device__ __forceinline__ void send(int q, uint32_t at) {
      transfer(base, off[q], to + at + q * 1024);
      if (q == U - 1) {
        base += step;
        if (--left == 0) {
          base -= wrap * step;
          left = wrap;
        }
      }
    }
  };

  static __device__ __forceinline__ void product(const Operand& X, const Operand& Y, int64_t i0, int64_t j0, int64_t k0,
                                                 int64_t kend, uint32_t lds, Acc& acc) {
    const int lane = threadIdx.x & 63, bi = Waves<2, 2, 1, 4, 4>::base_i(), bj = Waves<2, 2, 1, 4, 4>::base_j();
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[mi][nj][r] = 0.0f;
    const int steps = k0 < kend ? (int)((kend - k0) / BK) : 0;   // whole steps
    Stream<OX> sx;
    Stream<OY> sy;
    u32x4 held[STAGED_X ? U : 1];
    const int64_t whole_x = STAGED_X && steps > 0 ? Small::template whole_steps<OX, 256>(X, i0, k0, kend) : 0;
    if constexpr (!STAGED_X) sx.init(X, i0, k0, lds);
    sy.init(Y, j0, k0, lds);
    auto fetch = [&](int s) {   // a staged step to registers
      if constexpr (STAGED_X) {
        if (s < whole_x) Small::template load_whole<OX, 256, U>(X, i0, k0 + (int64_t)s * BK, held);
        else Small::template load_flat<OX, 256, U>(X, i0, k0 + (int64_t)s * BK, kend, held);
      }
    };
    auto put = [&](uint32_t at) {   // and from there to its slot
      if constexpr (STAGED_X) Small::template store<OX, 256, U>(lds + at, held);
    };
    bf16x8 x[2][MI], y[2][NJ];
    auto read = [&](uint32_t xs, uint32_t ys, int ks, int to, int n) {   // operand n = 0..7, in the order the products need them
      if (n == 0 || n > NJ) x[to][n == 0 ? 0 : n - NJ] = Small::template frag<OX, 256>(lds + xs, bi + 32 * (n == 0 ? 0 : n - NJ), ks, lane);
      else y[to][n - 1] = Small::template frag<OY, 256>(lds + ys, bj + 32 * (n - 1), ks, lane);
    };
    // the 16 products of one quarter step (16 k), the next quarter's reads
    // behind the first 8 of them and 4 transfers, send(0..3), behind the others
    auto quarter = [&](int from, uint32_t xs, uint32_t ys, int ks, auto send) {
#pragma unroll
      for (int n = 0; n < MI * NJ; ++n) {
        if (n < 8) read(xs, ys, ks, from ^ 1, n);
        else if ((n & 1) == 0) send((n - 8) / 2);
        __builtin_amdgcn_sched_barrier(0);
        acc[n / NJ][n % NJ] = multiply_add<T>(x[from][n / NJ], y[from][n % NJ], acc[n / NJ][n % NJ]);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (steps > 0) {
      // slots in turn: X0 Y0 X1 Y1 X2, then Y2 where X0 was, X3 where Y0 was, ...
#pragma unroll
      for (int s = 0; s < 3; ++s)
        if (s < steps) {
          if constexpr (STAGED_X) {
            fetch(s);
            put(2 * s * SLOT);
          } else {
#pragma unroll
            for (int q = 0; q < U; ++q) sx.send(q, 2 * s * SLOT);
          }
          if (s < 2) {
#pragma unroll
            for (int q = 0; q < U; ++q) sy.send(q, (2 * s + 1) * SLOT);
          }
        }
      if (!STAGED_X && steps > 2) asm volatile("s_waitcnt vmcnt(24)" ::: "memory");   // step 0 is there
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (STAGED_X && steps > 3) fetch(3);
      lds_only_barrier();
#pragma unroll
      for (int n = 0; n < 8; ++n) read(0, SLOT, 0, 0, n);
      auto next = [](uint32_t at) { return at + 2 * SLOT >= LDS ? at + 2 * SLOT - LDS : at + 2 * SLOT; };
      uint32_t xs = 0, ys = SLOT, xb = 0, yb = 0;   // this step's slots, and the step's before
      // ALL: a step that has one before it and three behind it
      auto step = [&](int s, auto all) {
        constexpr bool ALL = decltype(all)::value;
        const bool more_y = ALL || (s > 0 && s + 1 < steps), more_x = ALL || (s > 0 && s + 2 < steps), first_y = ALL || s + 2 < steps;
        if constexpr (STAGED_X) {
          if (more_x) {
            put(yb);
            if (ALL || s + 3 < steps) fetch(s + 3);
          }
        }
        quarter(0, xs, ys, 1, [&](int q) { if (more_y) sy.send(4 + q, xb); });
        quarter(1, xs, ys, 2, [&](int q) { if (!STAGED_X && more_x) sx.send(q, yb); });
        quarter(0, xs, ys, 3, [&](int q) { if (!STAGED_X && more_x) sx.send(4 + q, yb); });
        // every read of this step has arrived, and the next step's transfers
        // have landed: at most X of the step after it is on its way
        if constexpr (ALL && !STAGED_X) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_only_barrier();
        xb = xs;
        yb = ys;
        xs = next(xs);
        ys = next(ys);
        quarter(1, xs, ys, 0, [&](int q) { if (first_y) sy.send(q, xb); });   // (past the last step: reads of what is there, unused)
      };
      step(0, std::false_type{});
      int s = 1;
      for (; s + 3 < steps; ++s) step(s, std::true_type{});
      for (; s < steps; ++s) step(s, std::false_type{});
      __syncthreads();
    }
    if (k0 + (int64_t)steps * BK < kend) {   // the last, partial step
      u32x4 v[U];
      Small::template load_flat<OX, 256, U>(X, i0, k0 + (int64_t)steps * BK, kend, v);
      Small::template store<OX, 256, U>(lds, v);
      Small::template load_flat<OY, 256, U>(Y, j0, k0 + (int64_t)steps * BK, kend, v);
      Small::template store<OY, 256, U>(lds + SLOT, v);
      __syncthreads();
      for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
        for (int n = 0; n < 8; ++n) read(0, SLOT, ks, 0, n);
#pragma unroll
        for (int n = 0; n < MI * NJ; ++n)
          acc[n / NJ][n % NJ] = multiply_add<T>(x[0][n / NJ], y[0][n % NJ], acc[n / NJ][n % NJ]);
      }
      __syncthreads();
    }
  }
};

// Which tile a workgroup takes.  Neighbouring workgroups go to different XCDs,
// each with its own L2, so each XCD gets a run of tiles of its own; in a run, up
// to 8 columns of tiles are taken together, all their rows of tiles in turn, so
// that what runs at once on an XCD shares both operands.
__device__ __forceinline__ void tile_of(uint32_t block, int64_t itiles, int64_t jtiles, int64_t& it, int64_t& jt) {
  constexpr uint32_t kXcds = 8, kCols = 8;
  const uint32_t all = (uint32_t)(itiles * jtiles), per = all / kXcds, more = all % kXcds;
  const uint32_t xcd = block % kXcds, t = xcd * per + (xcd < more ? xcd : more) + block / kXcds;
  const uint32_t rows = (uint32_t)itiles, group = t / (kCols * rows), in = t % (kCols * rows);
  const uint32_t left = (uint32_t)jtiles - group * kCols, cols = left < kCols ? left : kCols;
  it = __builtin_amdgcn_readfirstlane(in / cols);   // (the same in every lane: kept in scalar registers)
  jt = __builtin_amdgcn_readfirstlane(group * kCols + in % cols);
}

// row of accumulator entry r inside its 32 x 32 block
__device__ __forceinline__ int entry_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// What is added to a wavefront's products, whose outputs begin at i0: the bias
// of each, -inf past the last output.  (No divergent branch while the sums fill
// the registers: see load_flat.)
template <class Tl>
__device__ __forceinline__ void load_bias(float (&b)[Tl::MI][16], const float* bias, int64_t i0, int64_t M) {
  const int lane = threadIdx.x & 63;
  const bool inside = i0 + 32 * Tl::MI <= M;   // (uniform)
#pragma unroll
  for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t i = i0 + 32 * mi + entry_row(4 * q, lane);
      if (inside) {
        const f32x4 v = bias ? __builtin_bit_cast(f32x4, load16(bias + i)) : (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) b[mi][4 * q + e] = v[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = bias ? bias[i + e < M ? i + e : M - 1] : 0.0f;
          b[mi][4 * q + e] = i + e < M ? v : -__builtin_inff();
        }
      }
    }
}

// A tile's results in 16 bits on their way to memory, out[j][i] with i contiguous:
// through LDS, so that every row is written in whole 16-byte units by
// neighbouring lanes.  A row's units are permuted by the row, so that 32 rows
// written at once go to different banks.
// two values rounded to 16 bits each
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (std::is_same<T, F16>::value) return from_float<F16>(a).bits | (uint32_t)from_float<F16>(b).bits << 16;
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(((f32x2){a, b}), bf16x2));
}

template <class T, class Tl>
__device__ __forceinline__ void stage4(char* lds, int i, int j, float a, float b, float c, float d) {   // results i .. i + 3 of row j
  constexpr int C = Tl::BI / 8;   // units of a row
  static_assert(Tl::BI * Tl::BJ * 2 <= Tl::LDS, "tile");
  *reinterpret_cast<u32x2*>(lds + j * (C * 16) + (((i >> 3) ^ (j & (C - 1))) << 4) + (i & 4) * 2) =
      (u32x2){pack2<T>(a, b), pack2<T>(c, d)};
}

template <class T, class Tl>
__device__ __forceinline__ void write_staged(const char* lds, T* out, int64_t ldo, int64_t I, int64_t J) {
  constexpr int C = Tl::BI / 8, STEP = Tl::NT / C, BATCH = Tl::BJ / STEP < 8 ? Tl::BJ / STEP : 8;
  const int c = threadIdx.x % C, left = I - c * 8 < 8 ? (int)(I - c * 8) : 8;
  if (left <= 0) return;
  for (int j0 = threadIdx.x / C; j0 < Tl::BJ; j0 += STEP * BATCH) {
    u32x4 v[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int j = j0 + k * STEP;
      v[k] = *reinterpret_cast<const u32x4*>(lds + j * (C * 16) + ((c ^ (j & (C - 1))) << 4));
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int j = j0 + k * STEP;
      if (j >= J) break;
      T* p = out + j * ldo + c * 8;
      if (left == 8) {
        store16(p, v[k]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < left) p[e] = T{(uint16_t)(v[k][e >> 1] >> (16 * (e & 1)))};
      }
    }
  }
}

// fp32 results i .. i + 3 of a row, `left` of them inside the matrix
__device__ __forceinline__ void write4(float* p, int64_t left, f32x4 v) {
  if (left >= 4) {
    store16(p, __builtin_bit_cast(u32x4, v));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = v[e];
  }
}

// A tile of I x J results from its own corner on, in 16 bits.
template <class T, class Tl>
__device__ __forceinline__ void write_tile16(typename Tl::Acc& acc, char* lds, T* out, int64_t ldo, int64_t I, int64_t J) {
  const int lane = threadIdx.x & 63, bi = Tl::base_i(), bj = Tl::base_j();
  if (Tl::lead()) {
#pragma unroll
    for (int nj = 0; nj < Tl::NJ; ++nj)
#pragma unroll
      for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          stage4<T, Tl>(lds, bi + 32 * mi + entry_row(4 * q, lane), bj + 32 * nj + (lane & 31), acc[mi][nj][4 * q], acc[mi][nj][4 * q + 1],
                        acc[mi][nj][4 * q + 2], acc[mi][nj][4 * q + 3]);
  }
  __syncthreads();
  write_staged<T, Tl>(lds, out, ldo, I, J);
}

// The same in 32 bits, through LDS too: in whole lines, and with no sums left
// in registers around the checks of the matrix's end.  A 256 x 256 tile goes in
// two halves, columns nj < NJ / 2 of every wavefront's blocks first.  ADD: the
// results are added to what `sum` [J][lds] holds; T: what is written.
template <class T, class Tl, bool ADD>
__device__ __forceinline__ void write_tile32(typename Tl::Acc& acc, char* lds, T* out, int64_t ldo, int64_t I, int64_t J, const float* sum = nullptr,
                                             int64_t ld_sum = 0) {
  constexpr int PASSES = Tl::BI * Tl::BJ * 4 > (int)Tl::LDS ? 2 : 1, NP = Tl::NJ / PASSES, ROWS = Tl::BJ / PASSES, C = Tl::BI / 4;
  static_assert(ROWS * Tl::BI * 4 <= (int)Tl::LDS && NP * PASSES == Tl::NJ, "tile");
  const int lane = threadIdx.x & 63, bi = Tl::base_i();
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    if (pass) __syncthreads();
    if (Tl::lead()) {
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const int j = (Tl::wj() * NP + n) * 32 + (lane & 31);   // row of LDS
#pragma unroll
        for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int c = (bi + 32 * mi + entry_row(4 * q, lane)) >> 2, nj = pass * NP + n;
            *reinterpret_cast<f32x4*>(lds + (j * C + (c ^ (j & 31))) * 16) =
                (f32x4){acc[mi][nj][4 * q], acc[mi][nj][4 * q + 1], acc[mi][nj][4 * q + 2], acc[mi][nj][4 * q + 3]};
          }
      }
    }
    __syncthreads();
    for (int u = threadIdx.x; u < ROWS * C; u += Tl::NT) {
      const int row = u / C, c = u % C;
      const int j = row / (32 * NP) * (32 * Tl::NJ) + pass * (32 * NP) + row % (32 * NP);   // row of the tile
      const int64_t left = I - c * 4;
      if (j >= J || left <= 0) continue;
      f32x4 v = *reinterpret_cast<const f32x4*>(lds + (row * C + (c ^ (row & 31))) * 16);
      if constexpr (ADD) {
        const float* p = sum + j * ld_sum + c * 4;
        if (left >= 4) {
          v += __builtin_bit_cast(f32x4, load16(p));
        } else {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (e < left) v[e] += p[e];
        }
      }
      T* to = out + j * ldo + c * 4;
      if constexpr (sizeof(T) == 4) {
        write4(to, left, v);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < left) to[e] = from_float<T>(v[e]);
      }
    }
  }
}

// as T, whichever that is
template <class T, class Tl>
__device__ __forceinline__ void write_tile(typename Tl::Acc& acc, char* lds, T* out, int64_t ldo, int64_t I, int64_t J) {
  if constexpr (sizeof(T) == 2) write_tile16<T, Tl>(acc, lds, out, ldo, I, J);
  else write_tile32<T, Tl, false>(acc, lds, out, ldo, I, J);
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int status_from(hipError_t e) { return e == hipSuccess ? MADDNESS_OK : MADDNESS_EHIP; }
int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
int64_t cdiv(int64_t v, int64_t m) { return (v + m - 1) / m; }

constexpr int64_t kMaxBlocks = (1ll << 31) - 1;
// Whether an operand's rows are whole 16-byte units (and a step's offsets fit
// in 32 bits), so that they can go straight to LDS.  along_i: its own index is
// the contiguous one.
bool direct(const Operand& o, bool along_i) {
  return aligned(o.p, 16) && o.ld % 8 == 0 && (!along_i || o.pad % 8 == 0) && o.ld <= (1 << 22);
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

}  // namespace
}  // namespace mdn
