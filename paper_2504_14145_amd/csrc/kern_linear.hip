// kern_linear.hip -- matrix products of the stage operators: out[m][n] =
// epilogue(sum_k a(m, k) b(n, k)), for dip_linear (x w^T) and its gradients (g w,
// g^T x), each operand lying along the contraction or across it.
//
// Bound by the matrix instructions where m, n and k are large, by the latency of
// memory where few tiles are, by memory where one side is short.  A large tile is
// 256 x 256 by four waves of 128 x 128, which reads least from LDS a product (with
// eight waves of 128 x 64 the LDS, reads and incoming tiles together, is as busy as
// the matrix units); an operand's tiles go from memory to LDS without passing
// registers, and across-lying ones are read through the transposing LDS read, so
// that no weight or activation is ever transposed in memory.  The product is taken
// as b a^T: a lane then holds eight consecutive columns of a row of the output,
// which its epilogue (bias, activation, eight dropout draws of one counter,
// residual) and its 16-byte stores want.
// bf16, 8192^3: 1.41 to 1.5 PFLOP/s forward, 1.45 to 1.51 and 1.44 to 1.5 for the
// gradients of x and w, the card's clock falling under the load; 65,536 x 3584 x
// 2560: 1.34, 1.33, 1.26, and 1.16 forward with bias, GELU and the value before it
// written.  Of a step's 2500 cycles 2048 are products, 280 waits at the two barriers;
// a tile's start and end take another 20,000.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "ops_internal.h"

namespace dipops {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) s16x8 lds_s16x8;

constexpr int kStep = 64;                  // contraction elements a staged tile
constexpr uint32_t kOutside = 0x80000000u; // a buffer offset that reads zeros

// A descriptor of `bytes` bytes from p: loads beyond them return zeros.
__device__ __forceinline__ i32x4 descriptor(const void *p, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  i32x4 d;
  d[0] = __builtin_amdgcn_readfirstlane(int(uint32_t(a)));
  d[1] = __builtin_amdgcn_readfirstlane(int(uint32_t(a >> 32) & 0xffffu));
  d[2] = __builtin_amdgcn_readfirstlane(int(bytes));
  d[3] = 0x00020000;
  return d;
}

// 16 bytes a lane from the buffer straight to LDS address to + OFF + 16 lane.
// Written out, because for the builtin the compiler waits for all loads before any
// LDS read that follows; the waits below are this file's own.  No register receives
// the data, the offset is read when the instruction issues, and the no-op is the wait
// that a new M0 needs.  M0, the LDS address, is a value that the first statement gives
// and the second takes, so the compiler leaves it alone between them (in one statement
// the allocation of the 256 x 256 forward's registers falls apart: 8192^3 1123 us
// against 752).
template <int OFF>
__device__ __forceinline__ void load_lds(const i32x4 &d, uint32_t offset, uint32_t to) {
  uint32_t at;
  asm volatile("s_add_u32 %0, %1, %2" : "={m0}"(at) : "s"(to), "n"(OFF) : "scc", "memory");
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(offset), "s"(d), "{m0}"(at) : "memory");
}

// Where a row's 16-byte chunks sit in LDS when the contraction runs along rows:
// 128 bytes a row, chunk c at slot c ^ spread(row).  The LDS serves a 16-byte read
// sixteen lanes at a time, eight rows at c and eight others at c ^ 1 (lanes 0-3,
// 12-15 of one sixteen with 4-11 of the next): with this those fall on all banks,
// for sixteen rows in a row and for the pairs of fragments below.
__device__ __forceinline__ uint32_t spread(uint32_t row) {
  return (row >> 1 & 1) | ((row >> 2 ^ row >> 4) & 1) << 1 | (row >> 3 & 1) << 2;
}

// One operand's share of a workgroup: ROWS output rows (or columns) times
// kStep contraction elements a step, THREADS threads.
//
// K_ROWS false: the array is [i][k].  LDS holds 128 bytes a row i, spread as above.
// K_ROWS true: the array is [k][i].  LDS holds 2 ROWS bytes a row k, 64-byte
// pieces of a row exchanged by k & 3, and the transposing LDS read gives a lane
// four consecutive k of its column.
template <bool K_ROWS, int ROWS, int THREADS>
struct Stage {
  static constexpr int kLoads = ROWS * kStep * 2 / 16 / THREADS;
  static constexpr int kBytes = ROWS * kStep * 2;
  static_assert(kLoads >= 1 && ROWS * kStep * 2 % (16 * THREADS) == 0);
  const unsigned char *base;   // of the next step to load
  uint32_t voff[kLoads];
  uint32_t k_at;               // K_ROWS: first k row of the thread; else its first k in the step
  uint32_t valid_rows, row_bytes;   // rows inside the array, bytes a row
  i32x4 desc;
  uint32_t to;                 // LDS address of the wave's first load

  __device__ void init(const Operand &o, int64_t i0, int64_t rows, int64_t k0, int t) {
    row_bytes = uint32_t(o.ld) * 2;
    valid_rows = uint32_t(min(int64_t(ROWS), rows - i0));
    desc = descriptor(o.p, bytes(kStep));
    if constexpr (!K_ROWS) {
      base = static_cast<const unsigned char *>(o.p) + (i0 * o.ld + k0) * 2;
      const uint32_t row = t / 8, chunk = (t % 8) ^ spread(row);
      k_at = chunk * 8;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const uint32_t r = row + i * (THREADS / 8);
        voff[i] = r < valid_rows ? r * row_bytes + chunk * 16 : kOutside;
      }
    } else {
      base = static_cast<const unsigned char *>(o.p) + (k0 * o.ld + i0) * 2;
      constexpr int per_row = ROWS * 2 / 16;
      const uint32_t kr = t / per_row, slot = (t % per_row) ^ ((kr & 3) << 2);
      k_at = kr;
      static_assert(THREADS / per_row % 4 == 0);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        voff[i] = slot * 8 < valid_rows ? (kr + i * (THREADS / per_row)) * row_bytes + slot * 16 : kOutside;
    }
  }
  // from `base` to the end of a step of which kl contraction elements exist
  __device__ __forceinline__ uint32_t bytes(uint32_t kl) const {
    const uint32_t b = K_ROWS ? (kl - 1) * row_bytes + valid_rows * 2 : (valid_rows - 1) * row_bytes + kl * 2;
    return kl ? (b + 3) & ~3u : 0u;
  }
  // Makes the step at `base` ready to load: to LDS address lds (of the workgroup's
  // tile), with kl of its contraction elements present (none: all zeros; fewer
  // than kStep only where no step follows).
  __device__ __forceinline__ void begin(uint32_t lds, uint32_t kl, uint32_t wave) {
    if (kl < kStep) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const uint32_t k = K_ROWS ? k_at + i * (THREADS / (ROWS * 2 / 16)) : k_at;
        voff[i] = k < kl ? voff[i] : kOutside;
      }
      desc[2] = __builtin_amdgcn_readfirstlane(int(bytes(kl)));
    }
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    desc[0] = __builtin_amdgcn_readfirstlane(int(uint32_t(at)));
    desc[1] = __builtin_amdgcn_readfirstlane(int(uint32_t(at >> 32)));
    to = __builtin_amdgcn_readfirstlane(lds + wave * 1024);
    base += K_ROWS ? uint64_t(row_bytes) * kStep : uint64_t(kStep) * 2;
  }
  // Whether load i brings what the last L steps before a tile read of it: the
  // first 32 k, and of a row operand read by fragment (x) its waves' first rows.
  template <bool BY_FRAGMENT>
  static constexpr bool early(int i, int wave_rows, int l) {
    if (K_ROWS) return i < kLoads / 2;
    return !BY_FRAGMENT || i * (THREADS / 8) % wave_rows < 16 * l;
  }
};

// Reads fragments (16 rows x 32 k) of a wave's rows r0 .. from a staged tile.
// PAIRED: fragment 2 p + f holds, as its row 4 q + i, row 32 p + 8 q + 4 f + i,
// so that the two fragments' results give a lane eight consecutive rows.
// Addresses are a few registers and offsets known at compile time.
template <class V, bool K_ROWS, int ROWS, bool PAIRED, int FRAGS>
struct Reader {
  static constexpr int kBases = !K_ROWS ? 4 : (FRAGS + 1) / 2;
  uint32_t at[kBases];
  __device__ __forceinline__ void init(uint32_t lds, uint32_t r0, int lane) {
    const uint32_t l = lane % 16, g = lane / 16;
    if constexpr (!K_ROWS) {
#pragma unroll
      for (int j = 0; j < kBases; ++j) {
        const uint32_t kk = j & 1, f = j >> 1;
        const uint32_t row = r0 + (PAIRED ? 8 * (l / 4) + 4 * f + l % 4 : 16 * f + l);
        at[j] = lds + row * 128 + (((kk * 4 + g) ^ spread(row)) << 4);
      }
    } else {
      const uint32_t kx = l / 4, q = l % 4, k = 8 * g + kx;
#pragma unroll
      for (int j = 0; j < kBases; ++j) {
        const uint32_t col = r0 + 32 * j + (PAIRED ? 8 * q : 4 * q);
        at[j] = lds + k * (ROWS * 2) + (((col / 8) ^ (kx << 2)) << 4) + (col % 8) * 2;
      }
    }
  }
  // the tile in the other of two buffers `by` bytes apart
  __device__ __forceinline__ void move(uint32_t by) {
#pragma unroll
    for (int j = 0; j < kBases; ++j) at[j] += by;
  }
  __device__ __forceinline__ V read(int frag, int kk) const {
    if constexpr (!K_ROWS) {
      return __builtin_bit_cast(
          V, *reinterpret_cast<lds_s16x8 *>(uintptr_t(at[(frag & 1) * 2 + kk] + (frag >> 1) * 32 * 128)));
    } else {
      const uint32_t off = (frag & 1) * (PAIRED ? 8 : 32) + kk * 32 * (ROWS * 2);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          reinterpret_cast<lds_s16x4 *>(uintptr_t(at[frag >> 1] + off)));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          reinterpret_cast<lds_s16x4 *>(uintptr_t(at[frag >> 1] + off + 4 * (ROWS * 2))));
      return __builtin_bit_cast(V, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// f(0) .. f(N - 1), the argument known at compile time.
template <class F, int... I>
__device__ __forceinline__ void unrolled_(F &&f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int P, class F>
__device__ __forceinline__ void each(F &&f) {
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int q = 0; q < 8; ++q) f(p, q);
}
template <int N, class F>
__device__ __forceinline__ void unrolled(F &&f) {
  unrolled_(f, std::make_integer_sequence<int, N>{});
}

__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return uint32_t(reinterpret_cast<uintptr_t>((lds_byte *)p));
}

// The order of a tile's loads: first those that its first fragments need.
template <class A, class B, int WAVE_ROWS, int L>
struct LoadOrder {
  static constexpr int kLoads = A::kLoads + B::kLoads;
  static constexpr bool early(int i) {
    return i < B::kLoads ? B::template early<false>(i, 1, L) : A::template early<true>(i - B::kLoads, WAVE_ROWS, L);
  }
  static constexpr int count(bool e) {
    int n = 0;
    for (int i = 0; i < kLoads; ++i) n += early(i) == e;
    return n;
  }
  static constexpr int kLate = count(false);
  static constexpr int nth(int j) {   // b's loads, then a's
    for (int e = 1; e >= 0; --e)
      for (int i = 0; i < kLoads; ++i)
        if (early(i) == bool(e) && j-- == 0) return i;
    return 0;
  }
  static constexpr bool of_a(int j) { return nth(j) >= B::kLoads; }
  static constexpr int index(int j) { return of_a(j) ? nth(j) - B::kLoads : nth(j); }
};

struct Split {
  float *partial;       // [splits][m][n4], n4 = n rounded up to 8
  int64_t steps;        // contraction steps a split
  int64_t n8;
};

// Tiles in the order in which the eight XCDs, which take workgroups in turn, see
// each a contiguous run of them, in strips of kGroup tile rows.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t &tm,
                                        uint32_t &tn) {
  const uint32_t all = tiles_m * tiles_n, x = id % 8, each = all / 8, rest = all % 8;
  id = x * each + min(x, rest) + id / 8;
  constexpr uint32_t kGroup = 4;
  const uint32_t strip = id / (kGroup * tiles_n), first = strip * kGroup;
  const uint32_t high = min(kGroup, tiles_m - first), in = id % (kGroup * tiles_n);
  tm = first + in % high;
  tn = in / high;
}

// what a workgroup does with its tile: the epilogue, a plain output of the
// operands' type, one of either type or added to, a part of a split
constexpr int kForward = 0, kGradient = 1, kGradientAny = 2, kPartial = 3;

// out tile BM x BN by WM x WN waves.
template <class T, bool A_K, bool B_K, int BM, int BN, int WM, int WN, int R, int KIND>
__global__ __launch_bounds__(64 * WM * WN, 1) void gemm_kernel(int64_t m, int64_t n, int64_t k, Operand a,
                                                            Operand b, Epilogue e, Split split) {
  typedef typename Vec8<T>::type V;
  constexpr int kThreads = 64 * WM * WN;
  constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  typedef Stage<A_K, BM, kThreads> StageA;
  typedef Stage<B_K, BN, kThreads> StageB;
  constexpr int kBuf = StageA::kBytes + StageB::kBytes;
  __shared__ __align__(1024) unsigned char s[R * kBuf];
  const uint32_t lds = lds_address(s);
  const int t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64);
  uint32_t tm, tn;
  tile_of(blockIdx.x, uint32_t((m + BM - 1) / BM), uint32_t((n + BN - 1) / BN), tm, tn);
  const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
  int64_t k0 = 0, k1 = k;
  if constexpr (KIND == kPartial) {
    k0 = int64_t(blockIdx.y) * split.steps * kStep;
    k1 = min(k, k0 + split.steps * kStep);
  }
  StageA sa;
  StageB sb;
  sa.init(a, m0, m, k0, t);
  sb.init(b, n0, n, k0, t);
  const uint32_t wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  const uint32_t lds_a = lds, lds_b = lds + R * StageA::kBytes;
  Reader<V, A_K, BM, false, FM> ra;
  Reader<V, B_K, BN, true, FN> rb;
  ra.init(lds_a, wm, lane);
  rb.init(lds_b, wn, lane);
  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // LDS is a ring of R staged tiles.  One is NS steps of one x fragment and FN
  // products.  x is read L steps ahead of its products, w half a tile ahead,
  // across tiles: L steps before a tile's end nothing of it is left to read, and
  // from there its place is filled again, with the tile R further on, and the next
  // one's first fragments are read.  Nothing but that point waits.  With few waves
  // a SIMD a product covers the issue of three other instructions, so the reads
  // and loads of a step are dealt out between its products.
  constexpr int NS = 2 * FM, L = FM / 2 > 1 ? FM / 2 : 1, X = 2 * L;
  // The loads of a tile are spread over D steps: all at once they would fill the
  // address queue and hold up the products behind them.  Those that the tile's
  // first fragments need come first, and the others may arrive L steps later.
  typedef LoadOrder<StageA, StageB, BM / WM, L> Order;
  constexpr int kLoads = Order::kLoads, kLate = Order::kLate, D = NS * 3 / 4;
  constexpr int kFirst = L * kLoads / D;                  // loads before the tile's end
  constexpr int kWay = (FN + L - 1) / L;
  constexpr bool kSplit = R == 2 && kLate > 0;            // a longer ring has time for all of them
  static_assert(NS % X == 0);
  V w[2][FN], x[X];
  // steps to take, and the contraction elements of the last one
  int left = __builtin_amdgcn_readfirstlane(int((k1 - k0 + kStep - 1) / kStep));
  const uint32_t last = uint32_t(k1 - k0 - int64_t(left - 1) * kStep);
  auto present = [&](int steps) { return steps > 1 ? uint32_t(kStep) : steps == 1 ? last : 0u; };
  auto load = [&](auto j_) __attribute__((always_inline)) {
    constexpr int j = decltype(j_)::value, i = Order::index(j);
    if constexpr (Order::of_a(j)) load_lds<i * kThreads * 16>(sa.desc, sa.voff[i], sa.to);
    else load_lds<i * kThreads * 16>(sb.desc, sb.voff[i], sb.to);
  };
  if (left > 0) {
    unrolled<R>([&](auto p_) __attribute__((always_inline)) {
      constexpr int p = decltype(p_)::value;
      sa.begin(lds_a + p * StageA::kBytes, present(left - p), wave);
      sb.begin(lds_b + p * StageB::kBytes, present(left - p), wave);
      unrolled<p + 1 < R ? kLoads : kFirst>(load);
    });
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((R - 2) * kLoads + kFirst) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int j = 0; j < FN; ++j) w[0][j] = rb.read(j, 0);
#pragma unroll
    for (int j = 0; j < L; ++j) x[j] = ra.read(j, 0);
  }
  uint32_t now = 0;   // place in the ring
  for (; left > 0; --left) {
    unrolled<NS>([&](auto s_) __attribute__((always_inline)) {
      constexpr int s = decltype(s_)::value, r = s - (NS - L);
      constexpr bool ahead = r >= 0;
      if constexpr (s == 0 && kSplit) {
        // the rest of this tile
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((R - 2) * kLoads + kFirst) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      if constexpr (r == 0) {
        // the first part of the next tile; and every wave has read this one
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((R - 2) * kLoads + (kSplit ? kLate : 0)) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        sa.begin(lds_a + now * StageA::kBytes, present(left - R), wave);
        sb.begin(lds_b + now * StageB::kBytes, present(left - R), wave);
        const uint32_t by = now == R - 1 ? uint32_t(1 - R) : 1u;
        ra.move(by * StageA::kBytes);
        rb.move(by * StageB::kBytes);
        now += by;
      }
      // the step's other work: one x fragment, w fragments, loads
      constexpr int q = (r + NS) % NS, d0 = q < D ? q * kLoads / D : 0, d1 = q < D ? (q + 1) * kLoads / D : 0;
      constexpr int n_w = s < L || ahead ? kWay : 0, others = 1 + n_w + d1 - d0;
      unrolled<FN>([&](auto j_) __attribute__((always_inline)) {
        constexpr int j = decltype(j_)::value, o0 = j * others / FN, o1 = (j + 1) * others / FN;
        unrolled<o1 - o0>([&](auto o_) __attribute__((always_inline)) {
          constexpr int o = o0 + decltype(o_)::value;
          if constexpr (o == 0) {
            x[(s + L) % X] = ra.read((s + L) % FM, (s + L) % NS / FM);
          } else if constexpr (o <= n_w) {
            constexpr int at = (ahead ? r : s) * kWay + o - 1;
            if constexpr (at < FN) w[ahead ? 0 : 1][at] = rb.read(at, ahead ? 0 : 1);
          } else {
            load(std::integral_constant<int, d0 + o - 1 - n_w>{});
          }
        });
        mfma16(w[s / FM][j], x[s % X], acc[s % FM][j]);
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  }
  // the loads after the last tile write zeros to LDS: they end before the wave
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  products_wait();
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int p = 0; p < FN / 2; ++p) in_accumulators(acc[i][2 * p], acc[i][2 * p + 1]);
  // A wave takes a row of fragments at a time, all of a row's loads ahead of their
  // use: it has the SIMD to itself, so nothing else covers them.  Of a long
  // epilogue there is one copy, looped over the rows: the loop picks its fragments
  // by uniform branches, since registers have no index.
  constexpr int P = FN / 2;
  const int64_t col0 = n0 + wn + 8 * (lane / 16), row0 = m0 + wm + lane % 16;
  int cols[P];   // columns of each eight that exist
#pragma unroll
  for (int p = 0; p < P; ++p) cols[p] = int(max(int64_t(0), min(int64_t(8), n - col0 - 32 * p)));
  V bias[P];
  if (KIND == kForward && e.bias) {
#pragma unroll
    for (int p = 0; p < P; ++p) bias[p] = take8(static_cast<const T *>(e.bias) + col0 + 32 * p, cols[p]);
  }
  // the residual's rows are asked for all at once where there are few, else one
  // round ahead
  constexpr int kRows = FM <= 4 ? FM : 1;
  V r[kRows][P];
  auto residual = [&](int at, int i) __attribute__((always_inline)) {
    const int64_t row = row0 + 16 * i;
    const T *q = static_cast<const T *>(e.residual) + row * e.ldr + col0;
#pragma unroll
    for (int p = 0; p < P; ++p) r[at][p] = take8(q + 32 * p, row < m ? cols[p] : 0);
  };
  if (KIND == kForward && e.residual) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) residual(i, i);
  }
  auto finish = [&](int i, float(&v)[P][8]) __attribute__((always_inline)) {
    const int64_t row = row0 + 16 * i;
    auto store = [&](auto *base, int64_t ld) __attribute__((always_inline)) {
      auto *q = base + row * ld + col0;
#pragma unroll
      for (int p = 0; p < P; ++p) store8(q + 32 * p, row < m ? cols[p] : 0, v[p]);
    };
    if constexpr (KIND == kPartial) {
      // rows of the partial product are padded to eight columns
      float *q = split.partial + (int64_t(blockIdx.y) * m + row) * split.n8 + col0;
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (row < m && cols[p] > 0) store8(q + 32 * p, 8, v[p]);
      return;
    }
    if constexpr (KIND == kForward) {
      if (e.bias) each<P>([&](int p, int q) { v[p][q] += float(bias[p][q]); });
      if (e.pre) store(static_cast<T *>(e.pre), e.ldp);
      if (e.act == DIP_ACT_SILU) each<P>([&](int p, int q) { v[p][q] = act_of(v[p][q], DIP_ACT_SILU); });
      else if (e.act == DIP_ACT_GELU) each<P>([&](int p, int q) { v[p][q] = act_of(v[p][q], DIP_ACT_GELU); });
      else if (e.act == DIP_ACT_RELU) each<P>([&](int p, int q) { v[p][q] = act_of(v[p][q], DIP_ACT_RELU); });
      if (e.drop.drop_of) {
#pragma unroll
        for (int p = 0; p < P; ++p) drop8(e.drop, uint32_t(col0 >> 3) + 4 * p, uint32_t(row), v[p]);
      }
      if (e.residual) {
        each<P>([&](int p, int q) { v[p][q] += float(r[i % kRows][p][q]); });
        if (kRows < FM && i + 1 < FM) residual(0, i + 1);
      }
    }
    if constexpr (KIND == kGradientAny) {
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (row < m && cols[p] > 0) finish8<T>(e, row, col0 + 32 * p, cols[p], v[p]);
    } else {
      if constexpr (KIND == kGradient) each<P>([&](int p, int q) { v[p][q] *= e.scale; });
      store(static_cast<T *>(e.out), e.ldo);
    }
  };
  auto fragments = [&](auto i_, float(&v)[P][8]) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int q = 0; q < 8; ++q) v[p][q] = acc[decltype(i_)::value][2 * p + q / 4][q % 4];
  };
  if constexpr ((KIND == kForward && kRows < FM) || KIND == kGradientAny) {
#pragma unroll 1
    for (int i = 0; i < FM; ++i) {
      // read by instructions written out: the compiler would make one array
      // indexed by i of the branches, and put it into memory
      float v[P][8];
      unrolled<FM>([&](auto i_) __attribute__((always_inline)) {
        if (i == decltype(i_)::value)
          each<P>([&](int p, int q) { v[p][q] = from_accumulator(acc[decltype(i_)::value][2 * p + q / 4][q % 4]); });
      });
      finish(i, v);
    }
  } else {
    unrolled<FM>([&](auto i_) __attribute__((always_inline)) {
      float v[P][8];
      fragments(i_, v);
      finish(decltype(i_)::value, v);
    });
  }
}

// Sums the splits' partial products in their order and finishes.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(int64_t m, int64_t n, Epilogue e, Split split, int splits) {
  const int64_t per = split.n8 / 8, all = m * per;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= all) return;
  const int64_t row = i / per, col = i % per * 8;
  float v[8];
  load8(split.partial + row * split.n8 + col, 8, v);
  for (int s = 1; s < splits; ++s) {
    float q[8];
    load8(split.partial + (int64_t(s) * m + row) * split.n8 + col, 8, q);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += q[j];
  }
  finish8<T>(e, row, col, int(min(int64_t(8), n - col)), v);
}

template <class T, bool A_K, bool B_K, int BM, int BN, int WM, int WN, int R>
hipError_t run(int64_t m, int64_t n, int64_t k, const Operand &a, const Operand &b, const Epilogue &e,
               const GemmPlan &plan, float *partial, hipStream_t stream) {
  const int64_t tiles = ((m + BM - 1) / BM) * ((n + BN - 1) / BN);
  const dim3 block(64 * WM * WN);
  Split s{partial, plan.steps, (n + 7) / 8 * 8};
  if (plan.splits <= 1) {
    auto go = [&](auto kernel) { kernel<<<dim3(uint32_t(tiles)), block, 0, stream>>>(m, n, k, a, b, e, s); };
    if constexpr (!B_K) go(gemm_kernel<T, A_K, B_K, BM, BN, WM, WN, R, kForward>);
    else if (e.out_f32 || e.accumulate) go(gemm_kernel<T, A_K, B_K, BM, BN, WM, WN, R, kGradientAny>);
    else go(gemm_kernel<T, A_K, B_K, BM, BN, WM, WN, R, kGradient>);
    return hipGetLastError();
  }
  gemm_kernel<T, A_K, B_K, BM, BN, WM, WN, R, kPartial>
      <<<dim3(uint32_t(tiles), uint32_t(plan.splits)), block, 0, stream>>>(m, n, k, a, b, e, s);
  const hipError_t rc = hipGetLastError();
  if (rc != hipSuccess) return rc;
  join_kernel<T><<<dim3(uint32_t((m * (s.n8 / 8) + 255) / 256)), dim3(256), 0, stream>>>(m, n, e, s, plan.splits);
  return hipGetLastError();
}

template <class T, bool A_K, bool B_K>
hipError_t pick(int64_t m, int64_t n, int64_t k, const Operand &a, const Operand &b, const Epilogue &e,
                const GemmPlan &plan, float *partial, hipStream_t stream) {
  switch (plan.tile) {
    case 0: return run<T, A_K, B_K, 256, 256, 2, 2, 2>(m, n, k, a, b, e, plan, partial, stream);
    case 1: return run<T, A_K, B_K, 128, 128, 2, 2, 2>(m, n, k, a, b, e, plan, partial, stream);
    case 3:
      if constexpr (!A_K) return run<T, A_K, B_K, 192, 128, 2, 2, 4>(m, n, k, a, b, e, plan, partial, stream);
    default: return run<T, A_K, B_K, 128, 128, 2, 2, 4>(m, n, k, a, b, e, plan, partial, stream);
  }
}

// Copies one or two arrays to where the products can take them: 16-byte aligned,
// the stride a multiple of 8, zeros in the columns up to it.  One launch for both.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(PackJob a, PackJob b, uint32_t blocks_a) {
  const bool second = blockIdx.x >= blocks_a;
  const PackJob &j = second ? b : a;
  const uint32_t per = uint32_t(j.ldo / 8);
  const int64_t i = int64_t(blockIdx.x - (second ? blocks_a : 0)) * 256 + threadIdx.x;
  if (i >= j.rows * per) return;
  const int64_t row = i / per, col = (i - row * per) * 8;
  float v[8];
  load8(static_cast<const T *>(j.p) + row * j.ld + col, int(min(int64_t(8), j.cols - col)), v);
  store8(static_cast<T *>(j.out) + row * j.ldo + col, 8, v);
}

}  // namespace

// The tile and the number of splits of the contraction with the least expected
// time.  256 x 256, one workgroup a CU, reaches the highest rate; 128 x 128 with
// two workgroups a CU fills the card with a quarter of the output; 128 x 128 and
// 192 x 128 with a longer ring of loads, one workgroup a CU, hide the latency of
// memory better where they suffice (192 only for rows of a that lie along the
// contraction: the other layout's loads do not divide by it).  Microseconds a step
// and a workgroup's start and end as measured in bf16, in that order: 2048^3 44 /
// 28 / 20 / 25 us; 1500 x 3584 x 3584 71 / 46 / 55 / 39; 1152 x 1792 x 3840 43 / 26
// / 33 / 23; 149 x 4096 x 14336 81 / 49 / 32 / 41; 4096^3 94 / 110 / 136 / -.  A split
// costs its partial products' way through the caches: 65,536 x 3584 x 2560's
// weight gradient takes 1328 us whole, 932 in 7 parts; 1152 x 1792 x 3840 26 whole,
// 40 in 2.
GemmPlan plan_gemm(int64_t m, int64_t n, int64_t k, bool a_rows) {
  struct Shape {
    int64_t bm, bn, slots;
    double step_us, fixed_us;
  };
  constexpr Shape shapes[] = {
      {256, 256, 256, 1.35, 8.0}, {128, 128, 512, 0.78, 4.0}, {128, 128, 256, 0.45, 3.5}, {192, 128, 256, 0.62, 4.5}};
  const int64_t steps = (k + kStep - 1) / kStep;
  GemmPlan best;
  double least = 0;
  for (int tile = 0; tile < (a_rows ? 4 : 3); ++tile) {
    const Shape &s = shapes[tile];
    const int64_t tiles = ((m + s.bm - 1) / s.bm) * ((n + s.bn - 1) / s.bn);
    if (tiles >= kMaxTiles) continue;   // the largest tile fits by the caller's check
    for (int64_t splits = 1; splits <= 16 && (splits == 1 || splits * 2 <= steps); ++splits) {
      const int64_t each = (steps + splits - 1) / splits;
      if (splits > 1 && (steps + each - 1) / each != splits) continue;
      const double rounds = double((tiles * splits + s.slots - 1) / s.slots);
      const double join = splits > 1 ? 4.0 + double(splits) * double(m) * double(n) * 8 / 6e6 : 0.0;
      const double us = rounds * (double(each) * s.step_us + s.fixed_us) + join;
      if (least != 0 && us >= least) continue;
      least = us;
      best.tile = tile;
      best.splits = int(splits);
      best.steps = each;
    }
  }
  best.bytes = best.splits > 1 ? up16(int64_t(best.splits) * m * ((n + 7) / 8 * 8) * 4) : 0;
  return best;
}

hipError_t launch_gemm(int dtype, int64_t m, int64_t n, int64_t k, const Operand &a, const Operand &b,
                       const Epilogue &e, const GemmPlan &plan, float *partial, hipStream_t stream) {
  if (dtype == DIP_BF16) {
    if (!a.k_rows && !b.k_rows) return pick<__bf16, false, false>(m, n, k, a, b, e, plan, partial, stream);
    if (!a.k_rows) return pick<__bf16, false, true>(m, n, k, a, b, e, plan, partial, stream);
    return pick<__bf16, true, true>(m, n, k, a, b, e, plan, partial, stream);
  }
  if (!a.k_rows && !b.k_rows) return pick<_Float16, false, false>(m, n, k, a, b, e, plan, partial, stream);
  if (!a.k_rows) return pick<_Float16, false, true>(m, n, k, a, b, e, plan, partial, stream);
  return pick<_Float16, true, true>(m, n, k, a, b, e, plan, partial, stream);
}

hipError_t launch_pack(int dtype, const PackJob &a, const PackJob &b, hipStream_t stream) {
  const int64_t na = (a.rows * (a.ldo / 8) + 255) / 256, nb = (b.rows * (b.ldo / 8) + 255) / 256;
  if (na + nb >= kMaxTiles) {   // a launch's workgroups: one array after the other, by rows
    for (const PackJob *j : {&a, &b}) {
      const int64_t most = (kMaxTiles - 1) * 256 / (j->ldo / 8);
      for (int64_t row = 0; row < j->rows; row += most) {
        PackJob q = *j;
        q.rows = std::min(most, j->rows - row);
        q.p = static_cast<const char *>(j->p) + row * j->ld * 2;
        q.out = static_cast<char *>(j->out) + row * j->ldo * 2;
        const hipError_t e = launch_pack(dtype, q, PackJob{}, stream);
        if (e != hipSuccess) return e;
      }
    }
    return hipSuccess;
  }
  const dim3 grid(uint32_t(na + nb));
  if (dtype == DIP_BF16)
    pack_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(a, b, uint32_t(na));
  else
    pack_kernel<_Float16><<<grid, dim3(256), 0, stream>>>(a, b, uint32_t(na));
  return hipGetLastError();
}

}  // namespace dipops
