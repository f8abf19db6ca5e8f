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

#include <type_traits>

namespace mdn {
namespace {

enum Order : int { kAlongK = 0, kAlongI = 1 };   // which index of an operand is contiguous

struct Operand {
  const void* p;
  int64_t ld;     // elements between rows (kAlongK) or between k steps (kAlongI)
  int64_t rows;   // extent of the operand's own index
  int64_t pad;    // what of it memory holds (kAlongI: whole 16-byte units from `rows` on)
};

// A tile of BI x BJ results of one workgroup of WI x WJ wavefronts, k in steps
// of BK through two LDS buffers.
template <class T, Order OX, Order OY, int BI_, int BJ_, int WI_, int WJ_, int BK_ = sizeof(T) == 2 ? 64 : 32>
struct Tile {
  static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_;
  static constexpr int P = Parts<T>::n;
  static constexpr int BK = BK_;
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
  static __device__ __forceinline__ void load(const Operand& o, int64_t r0, int64_t k0, int64_t kend, u32x4 (&v)[U], int first = 0) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int r, k;
      unit<O, B>(threadIdx.x + (first + i) * NT, r, k);
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
  static __device__ __forceinline__ void store(uint32_t lds, const u32x4 (&v)[U], int first = 0) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int r, k;
      unit<O, B>(threadIdx.x + (first + i) * NT, r, k);
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
    uint32_t buf = lds;
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

// The tile of large bf16 products: 256 x 256 results of four wavefronts, 128 x
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
// registers instead.
template <Order OX, Order OY, bool STAGED_X>
struct BigTile {
  static constexpr int BI = 256, BJ = 256, BK = 64, WI = 2, WJ = 2, MI = 4, NJ = 4, NT = 256;
  static constexpr uint32_t SLOT = 256 * BK * 2, LDS = 5 * SLOT;
  static constexpr int U = 8;                                     // 16-byte units per thread and operand of a step
  typedef f32x16 Acc[MI][NJ];
  typedef Tile<Bf16, OX, OY, 256, 256, 2, 2, BK> Small;           // the LDS layout and guarded loads are its

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

  // 16 bytes a lane from base + off to LDS, 1 KB from `to` on (uniform)
  static __device__ __forceinline__ void transfer(const void* base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
  }

  template <Order O>
  struct Stream {
    const char* base;       // the next step's origin
    int64_t step;           // bytes from a step to the next
    uint32_t to;            // this wavefront's part of a slot
    uint32_t off[U];

    __device__ __forceinline__ void init(const Operand& o, int64_t r0, int64_t k0, uint32_t lds) {
      base = static_cast<const char*>(o.p) + (O == kAlongK ? r0 * o.ld + k0 : k0 * o.ld + r0) * 2;
      step = (O == kAlongK ? (int64_t)BK : BK * o.ld) * 2;
      to = __builtin_amdgcn_readfirstlane(lds + (threadIdx.x >> 6) * (U * 1024));
#pragma unroll
      for (int q = 0; q < U; ++q) off[q] = offset<O>(o, r0, q);
    }
    // transfer q of the next step, into the slot at `at`; the last one moves on
    __device__ __forceinline__ void send(int q, uint32_t at) {
      transfer(base, off[q], to + at + q * 1024);
      if (q == U - 1) base += step;
    }
  };

  static __device__ __forceinline__ void product(const Operand& X, const Operand& Y, int64_t i0, int64_t j0, int64_t k0,
                                                 int64_t kend, uint32_t lds, Acc& acc) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int bi = (wave / WJ) * 128, bj = (wave % WJ) * 128;
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
    if constexpr (!STAGED_X) sx.init(X, i0, k0, lds);
    sy.init(Y, j0, k0, lds);
    auto fetch = [&](int s) {   // a staged step to registers
      if constexpr (STAGED_X) Small::template load<OX, 256, U>(X, i0, k0 + (int64_t)s * BK, kend, held);
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
        acc[n / NJ][n % NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[from][n / NJ], y[from][n % NJ], acc[n / NJ][n % NJ], 0, 0, 0);
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
      Small::template load<OX, 256, U>(X, i0, k0 + (int64_t)steps * BK, kend, v);
      Small::template store<OX, 256, U>(lds, v);
      Small::template load<OY, 256, U>(Y, j0, k0 + (int64_t)steps * BK, kend, v);
      Small::template store<OY, 256, U>(lds + SLOT, v);
      __syncthreads();
      for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
        for (int n = 0; n < 8; ++n) read(0, SLOT, ks, 0, n);
#pragma unroll
        for (int n = 0; n < MI * NJ; ++n)
          acc[n / NJ][n % NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[0][n / NJ], y[0][n % NJ], acc[n / NJ][n % NJ], 0, 0, 0);
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

// row of accumulator entry r inside its 32 x 32 block
__device__ __forceinline__ int entry_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// What is added to a wavefront's products, whose outputs begin at i0: the bias
// of each, -inf past the last output.
template <class Tl>
__device__ __forceinline__ void load_bias(float (&b)[Tl::MI][16], const float* bias, int64_t i0, int64_t M) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t i = i0 + 32 * mi + entry_row(4 * q, lane);
      if (i + 4 <= M) {
        const f32x4 v = bias ? __builtin_bit_cast(f32x4, load16(bias + i)) : (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) b[mi][4 * q + e] = v[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) b[mi][4 * q + e] = i + e >= M ? -__builtin_inff() : bias ? bias[i + e] : 0.0f;
      }
    }
}

// where a row's target lies from output i0 on; out of every tile for rows without one
__device__ __forceinline__ int target_at(int64_t t, int64_t M, int64_t i0) {
  const int64_t d = t - i0;
  return t < 0 || t >= M || d < 0 || d >= (1 << 20) ? -1 : (int)d;
}

template <class T, class Tl>
__global__ void __launch_bounds__(Tl::NT, 1) xent_tile_kernel(XArgs a) {
  constexpr int BI = Tl::BI, BJ = Tl::BJ, WI = Tl::WI, WJ = Tl::WJ;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t it, jt;
  tile_of(blockIdx.x, a.itiles, a.jtiles, it, jt);
  const int64_t i0 = it * BI, j0 = jt * BJ;
  typename Tl::Acc acc;
  Tl::product(a.W, a.A, i0, j0, 0, a.D, lds_address(lds), acc);
  const int bi = (wave / WJ) * 32 * Tl::MI, bj = (wave % WJ) * 32 * Tl::NJ;
  float b[Tl::MI][16];
  load_bias<Tl>(b, a.bias, i0 + bi, a.M);
  float2* red = reinterpret_cast<float2*>(lds);   // [WI][BJ]
#pragma unroll
  for (int nj = 0; nj < Tl::NJ; ++nj) {
    const int64_t j = j0 + bj + 32 * nj + (lane & 31);
    const int t = j < a.N ? target_at(a.target[j], a.M, i0 + bi) : -1;
    float top = -__builtin_inff();
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi) {
#pragma unroll
      for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, acc[mi][nj][r] + b[mi][r]);
      if (__any(t >= 32 * mi && t < 32 * mi + 32)) {
        asm volatile("");   // (a branch: seldom taken)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t == 32 * mi + entry_row(r, lane)) a.zt[j] = acc[mi][nj][r] + b[mi][r];
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

// A tile's results as bf16 on their way to memory, out[j][i] with i contiguous:
// through LDS, so that every row is written in whole 16-byte units by
// neighbouring lanes.  A row's units are permuted by the row, so that 32 rows
// written at once go to different banks.
template <class Tl>
__device__ __forceinline__ void stage4(char* lds, int i, int j, float a, float b, float c, float d) {   // results i .. i + 3 of row j
  constexpr int C = Tl::BI / 8;   // units of a row
  static_assert(Tl::BI * Tl::BJ * 2 <= Tl::LDS, "tile");
  *reinterpret_cast<u32x2*>(lds + j * (C * 16) + (((i >> 3) ^ (j & (C - 1))) << 4) + (i & 4) * 2) =
      (u32x2){__builtin_bit_cast(uint32_t, __builtin_convertvector(((f32x2){a, b}), bf16x2)),
              __builtin_bit_cast(uint32_t, __builtin_convertvector(((f32x2){c, d}), bf16x2))};
}

template <class Tl>
__device__ __forceinline__ void write_staged(const char* lds, Bf16* out, int64_t ldo, int64_t I, int64_t J) {
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
      Bf16* p = out + j * ldo + c * 8;
      if (left == 8) {
        store16(p, v[k]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < left) p[e] = Bf16{(uint16_t)(v[k][e >> 1] >> (16 * (e & 1)))};
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

// A tile of I x J results from its own corner on.
template <class T, class Tl>
__device__ __forceinline__ void write_tile(typename Tl::Acc& acc, char* lds, T* out, int64_t ldo, int64_t I, int64_t J) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bi = (wave / Tl::WJ) * 32 * Tl::MI, bj = (wave % Tl::WJ) * 32 * Tl::NJ;
#pragma unroll
  for (int nj = 0; nj < Tl::NJ; ++nj) {
    const int j = bj + 32 * nj + (lane & 31);
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = bi + 32 * mi + entry_row(4 * q, lane);
        const f32x4 v = {acc[mi][nj][4 * q], acc[mi][nj][4 * q + 1], acc[mi][nj][4 * q + 2], acc[mi][nj][4 * q + 3]};
        if constexpr (sizeof(T) == 2) stage4<Tl>(lds, i, j, v[0], v[1], v[2], v[3]);
        else if (j < J) write4(out + j * ldo + i, I - i, v);
        if (sizeof(T) == 4) __builtin_amdgcn_sched_barrier(0);
      }
  }
  if constexpr (sizeof(T) == 2) {
    __syncthreads();
    write_staged<Tl>(lds, out, ldo, I, J);
  }
}

// Adds what a tile of 32-bit sums (as write_tile writes them) holds.
template <class Tl>
__device__ __forceinline__ void add_tile(typename Tl::Acc& acc, const float* sum, int64_t ld, int64_t I, int64_t J) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bi = (wave / Tl::WJ) * 32 * Tl::MI, bj = (wave % Tl::WJ) * 32 * Tl::NJ;
#pragma unroll
  for (int nj = 0; nj < Tl::NJ; ++nj) {
    const int j = bj + 32 * nj + (lane & 31);
#pragma unroll
    for (int mi = 0; mi < Tl::MI; ++mi) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = bi + 32 * mi + 8 * q + 4 * (lane >> 5);
        const float* p = sum + j * ld + i;
        f32x4 v = {0, 0, 0, 0};
        if (j < J) {
          if (i + 4 <= I) {
            v = __builtin_bit_cast(f32x4, load16(p));
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (i + e < I) v[e] = p[e];
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mi][nj][4 * q + e] += v[e];
      }
      __builtin_amdgcn_sched_barrier(0);   // (a few loads at a time: few registers)
    }
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

// A tile of G: outputs m0 + i, rows j.
template <class T, class Tl>
__global__ void __launch_bounds__(Tl::NT, 1) xent_dz_kernel(XArgs a) {
  constexpr int BI = Tl::BI, BJ = Tl::BJ, WJ = Tl::WJ;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t it, jt;
  tile_of(blockIdx.x, a.itiles, a.jtiles, it, jt);
  const int64_t i0 = a.m0 + it * BI, j0 = jt * BJ;
  typename Tl::Acc acc;
  Tl::product(a.W, a.A, i0, j0, 0, a.D, lds_address(lds), acc);
  const int bi = (wave / WJ) * 32 * Tl::MI, bj = (wave % WJ) * 32 * Tl::NJ;
  float b[Tl::MI][16], cols[Tl::MI][16];
  load_bias<Tl>(b, a.bias, i0 + bi, a.M);
  T* out = static_cast<T*>(a.dz) + j0 * a.ldz + it * BI;
#pragma unroll
  for (int nj = 0; nj < Tl::NJ; ++nj) {
    const int64_t j = j0 + bj + 32 * nj + (lane & 31);
    const int64_t target = j < a.N ? a.target[j] : -1;
    const float l = j < a.N ? a.lse[j] : 0.0f;
    const bool live = target >= 0 && target < a.M && l != -__builtin_inff();
    const float g = live ? a.gloss[j] : 0.0f;
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
          if (t == 32 * mi + entry_row(r, lane)) v[r] -= 1.0f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        v[r] = live ? v[r] * g : 0.0f;   // (whatever a row without a gradient has for logits)
        cols[mi][r] = nj == 0 ? v[r] : cols[mi][r] + v[r];
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = bi + 32 * mi + entry_row(4 * q, lane);
        if constexpr (sizeof(T) == 2) stage4<Tl>(lds, i, (int)(j - j0), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
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
      if ((lane & 15) == 0) red[(wave % WJ) * BI + bi + 32 * mi + entry_row(r, lane) + ((lane >> 4) & 1)] = s;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < BI; i += Tl::NT) {
    float s = red[i];
#pragma unroll
    for (int w = 1; w < WJ; ++w) s += red[w * BI + i];
    if (it * BI + i < a.ldz) a.cpart[jt * a.ldz + it * BI + i] = s;
  }
  if constexpr (sizeof(T) == 2) write_staged<Tl>(lds, out, a.ldz, a.ldz - it * BI, a.N - j0);
}

__global__ void __launch_bounds__(256) xent_dbias_kernel(const float* cpart, int64_t jtiles, int64_t ldz, int64_t n, float* out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float s = 0.0f;
    int64_t j = 0;
    for (; j + 8 <= jtiles; j += 8) {   // eight loads under way at a time
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = cpart[(j + k) * ldz + i];
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
    for (; j < jtiles; ++j) s += cpart[j * ldz + i];
    out[i] = s;
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
  if constexpr (MODE == kMore || MODE == kLast) add_tile<Tl>(acc, sum, I, I - i0, J - j0);
  if constexpr (MODE == kOut || MODE == kLast) write_tile<T, Tl>(acc, lds, static_cast<T*>(a.out) + j0 * a.ldo + i0, a.ldo, I - i0, J - j0);
  else write_tile<float, Tl>(acc, lds, sum, I, I - i0, J - j0);
}

// Joins the shares of a split product, in order.
template <class T>
__global__ void __launch_bounds__(256) xent_join_splits_kernel(GemmArgs a) {
  const int64_t I = a.X.rows, J = a.Y.rows;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < I * J; e += (int64_t)gridDim.x * 256) {
    float v = a.first ? 0.0f : a.sum[e];
    for (int s = 0; s < a.splits; ++s) v += a.part[s * I * J + e];
    if (a.last) static_cast<T*>(a.out)[e / I * a.ldo + e % I] = from_float<T>(v);
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

template <class K, class Args>
hipError_t launch(K kernel, int lds, int64_t blocks, int splits, int threads, const Args& a, hipStream_t stream) {
  if (blocks > kMaxBlocks) return hipErrorInvalidValue;
  hipError_t err = hipSuccess;
  launch_prepare(reinterpret_cast<const void*>(kernel), threads, lds, &err);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks, (unsigned)splits), dim3(threads), lds, stream, a);
  return hipGetLastError();
}

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

// Whether an operand's rows are whole 16-byte units (and a step's offsets fit
// in 32 bits), so that they can go straight to LDS.  along_i: its own index is
// the contiguous one.
bool direct(const Operand& o, bool along_i) {
  return aligned(o.p, 16) && o.ld % 8 == 0 && (!along_i || o.pad % 8 == 0) && o.ld <= (1 << 22);
}

// Rows of a logits tile: 256 (large bf16 products with whole units in A), 128,
// or 32 where the wider ones would leave compute units without work.
template <class T>
int row_tile(const XArgs& a, int64_t outputs) {
  if (sizeof(T) == 2 && a.N >= 192 && direct(a.A, false) && cdiv(a.N, 256) * cdiv(outputs, 256) >= 192) return 256;
  return cdiv(a.N, 128) * cdiv(outputs, 128) >= 256 ? 128 : 32;
}

template <class T, bool GRAD>
hipError_t logits(XArgs& a, int64_t outputs, int rows, bool md, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (rows == 256) {
      if (direct(a.W, !md)) return md ? launch_logits<T, GRAD, BigTile<kAlongK, kAlongK, false>>(a, outputs, s)
                                 : launch_logits<T, GRAD, BigTile<kAlongI, kAlongK, false>>(a, outputs, s);
      return md ? launch_logits<T, GRAD, BigTile<kAlongK, kAlongK, true>>(a, outputs, s)
                : launch_logits<T, GRAD, BigTile<kAlongI, kAlongK, true>>(a, outputs, s);
    }
  }
  if (rows >= 128) return md ? launch_logits<T, GRAD, Tile<T, kAlongK, kAlongK, 128, 128, 2, 2>>(a, outputs, s)
                             : launch_logits<T, GRAD, Tile<T, kAlongI, kAlongK, 128, 128, 2, 2>>(a, outputs, s);
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
  // shares of a product: a tile of 256 x 256 for each compute unit
  g.part = 256ll * 256 * 256 * 4;
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
    const int64_t b = cdiv(n, 256);
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
      if (a.N >= 256 && a.D >= 256) {
        done = true;
        if (direct(x.X, md)) e = md ? gemm<T, BigTile<kAlongI, kAlongK, false>, true>(x, g.part, s) : gemm<T, BigTile<kAlongK, kAlongK, false>, true>(x, g.part, s);
        else e = md ? gemm<T, BigTile<kAlongI, kAlongK, true>, true>(x, g.part, s) : gemm<T, BigTile<kAlongK, kAlongK, true>, true>(x, g.part, s);
      }
    }
    if (done) {}
    else if (a.N <= 32) e = md ? gemm<T, Tile<T, kAlongI, kAlongK, 128, 32, 4, 1>, true>(x, g.part, s) : gemm<T, Tile<T, kAlongK, kAlongK, 128, 32, 4, 1>, true>(x, g.part, s);
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
      if (direct(ai, true) && cdiv(a.D, 256) * cdiv(n, 256) >= 192) {
        done = true;
        e = gemm<T, BigTile<kAlongI, kAlongI, false>, false>(x, g.part, s);
      }
    }
    if (!done) e = gemm<T, Tile<T, kAlongI, kAlongI, 128, 128, 2, 2>, false>(x, g.part, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t forward(XArgs a, bool md, float* loss, float* lse, hipStream_t s) {
  hipError_t e = logits<T, false>(a, a.M, row_tile<T>(a, a.M), md, s);
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
