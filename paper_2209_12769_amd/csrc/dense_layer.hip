// Dense layer on the rows of a batch, Y = act(X W + b) + R, and its gradients (gfx950).
//
//   forward   Z = X W + b, Y = act(Z) + R                                   contraction over the columns of X
//   data      dX = dZ W^T, dZ = dY act'(Z) formed as the rows are loaded    contraction over the columns of dY
//   weights   dW = X^T dZ, db = column sums of dZ                           contraction over the rows, split into slabs
//
// All three are tiles on the bf16 matrix cores (32 x 32 x 16), operands staged through LDS in the layout that the
// instruction reads: units of eight consecutive contraction indices (16 bytes).
// fp32: a number is the sum of three bf16 numbers; the six products of pieces with i + j <= 4 are formed (what is left
// out is below 2^-25 of |x w|), sums of 64 indices go to a total of their own, and every other one is formed negated, so
// that what the matrix cores drop below an accumulator's 24 bits (always downwards) cancels.  Kept rows are one exact
// piece: three products instead of six.  Sums that come out not finite in pieces are formed again in fp32.
// dZ: with ReLU formed as rows are loaded (a comparison).  The slopes of GELU and SiLU cost some twenty instructions a
// value and every value is loaded by several tiles, so a pass of its own forms dZ once and leaves it in the workspace.
// bf16: the operand has to be bf16, and dZ is left as the sum of two of its numbers, 16 bits, in two arrays: dX = [dZ0 | dZ1] [W | W]^T,
// dW by two products of one load of X.  Rounded to one (off by 2^-8 at most, the caller's choice) dX and dW are further from 64 bits
// than their own rounding has them, 0.0024 in norm for 0.0017, in two thirds of the time (524309 x 768 -> 256: 820 us for 1190).
// db is summed from the fp32 values in 64 bits.
#include "operators.h"

namespace dc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16;

// storage types of an operand
struct F32 { static constexpr int kBytes = 4, kPieces = 3; };
struct Bf16 { static constexpr int kBytes = 2, kPieces = 1; };
struct Kept { static constexpr int kBytes = 1, kPieces = 1; };
struct Bf16Pair { static constexpr int kBytes = 2, kPieces = 2; };      // a number is the sum of one of p and one of z

// An operand as it lies in memory: `rows` x `cols`, up to three matrices of d columns side by side; with z (kDz) the values are p
// where z > 0, else 0 (Bf16Pair: p + z).
struct Source {
  const char* p[3];
  const char* z;
  const unsigned char* exponent;
  long long ld, ldz, ld_exponent;
  long long rows;
  int cols, d;
};

// kN consecutive columns of one row, as they come from memory
template <class E, int kN, bool kDz>
struct Raw {
  static constexpr int kWords = (kN * E::kBytes + 3) / 4;
  unsigned w[kWords];
  unsigned z[kDz ? kWords : 1];
  unsigned e;
};

// Rows may start anywhere an element may: global loads of several words need no more than that on this machine.
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
typedef unsigned u32_any __attribute__((aligned(1)));
typedef u16 u16_any __attribute__((aligned(1)));
template <int kBytes>
__device__ __forceinline__ void read_words(unsigned* w, const char* p) {
  if constexpr (kBytes == 1) w[0] = *reinterpret_cast<const unsigned char*>(p);
  else if constexpr (kBytes == 2) w[0] = *reinterpret_cast<const u16_any*>(p);
  else if constexpr (kBytes == 4) w[0] = *reinterpret_cast<const u32_any*>(p);
  else if constexpr (kBytes == 8) {
    const u32x2 v = *reinterpret_cast<const u32x2_any*>(p);
    w[0] = v.x;
    w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i) {
      const u32x4 v = reinterpret_cast<const u32x4_any*>(p)[i];
      w[4 * i] = v.x;
      w[4 * i + 1] = v.y;
      w[4 * i + 2] = v.z;
      w[4 * i + 3] = v.w;
    }
  }
}
// Value k of the words.
template <class E>
__device__ __forceinline__ float value_of(const unsigned* w, int k, float scale) {
  if constexpr (E::kBytes == 4) return __uint_as_float(w[k]);
  else if constexpr (E::kBytes == 2) return __uint_as_float(k & 1 ? w[k >> 1] & 0xFFFF0000u : w[k >> 1] << 16);
  else return (float)(signed char)(w[k >> 2] >> (8 * (k & 3))) * scale;
}
// The matrix of a part, chosen among values: a choice among places would move the arguments to scratch memory.
__device__ __forceinline__ const char* part_of(const Source& s, int seg) {
  const size_t p0 = (size_t)s.p[0], p1 = (size_t)s.p[1], p2 = (size_t)s.p[2];
  return reinterpret_cast<const char*>(seg == 0 ? p0 : (seg == 1 ? p1 : p2));
}
template <class E, bool kDz>
__device__ __forceinline__ float single(const Source& s, long long row, int col) {
  const int seg = col / s.d;
  const char* p = part_of(s, seg);
  unsigned w[1], z[1];
  read_words<E::kBytes>(w, p + (row * s.ld + col - seg * s.d) * E::kBytes);
  float scale = 1.f;
  if constexpr (E::kBytes == 1) scale = kept_scale(s.exponent[row * s.ld_exponent + col / kKeptBlock]);
  float x = value_of<E>(w, 0, scale);
  if constexpr (kDz) {
    read_words<E::kBytes>(z, s.z + (row * s.ldz + col) * E::kBytes);
    x = value_of<E>(z, 0, 1.f) > 0.f ? x : 0.f;
  }
  return x;
}
// kN neighbouring values at p + off (and z + offz).
template <class E, int kN, bool kDz>
__device__ __forceinline__ void fetch(Raw<E, kN, kDz>& r, const char* p, const char* z, unsigned off, unsigned offz) {
  read_words<kN * E::kBytes>(r.w, p + off);
  if constexpr (kDz) read_words<kN * E::kBytes>(r.z, z + offz);
}
// The same value by value where only `left` (at least one) are there: the last one again behind them, no request in a branch.
template <class E, int kN, bool kDz>
__device__ __forceinline__ void fetch_some(Raw<E, kN, kDz>& r, const char* p, const char* z, unsigned off, unsigned offz, int left) {
  constexpr int kPer = 4 / E::kBytes;
  unsigned x[kN][1], y[kN][1];
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    const unsigned at = (unsigned)min(k, left - 1) * E::kBytes;
    read_words<E::kBytes>(x[k], p + off + at);
    if constexpr (kDz) read_words<E::kBytes>(y[k], z + offz + at);
  }
#pragma unroll
  for (int i = 0; i < Raw<E, kN, kDz>::kWords; ++i) {
    r.w[i] = 0;
    if constexpr (kDz) r.z[i] = 0;
  }
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    r.w[k / kPer] |= x[k][0] << (8 * E::kBytes * (k % kPer) % 32);
    if constexpr (kDz) r.z[k / kPer] |= y[k][0] << (8 * E::kBytes * (k % kPer) % 32);
  }
}
template <class E, int kN, bool kDz>
__device__ __forceinline__ void clear(Raw<E, kN, kDz>& r) {
#pragma unroll
  for (int i = 0; i < Raw<E, kN, kDz>::kWords; ++i) {
    r.w[i] = 0;
    if constexpr (kDz) r.z[i] = 0;
  }
  r.e = 0;
}
// Clears the first `n` values.
template <class E, int kN, bool kDz>
__device__ __forceinline__ void clear_front(Raw<E, kN, kDz>& r, int n) {
  constexpr int kPer = 4 / E::kBytes;
#pragma unroll
  for (int i = 0; i < Raw<E, kN, kDz>::kWords; ++i) {
    const int c = n - i * kPer;                         // values of this word that go
    const unsigned keep = c <= 0 ? ~0u : (c >= kPer ? 0u : ~0u << (8 * E::kBytes * c % 32));
    r.w[i] &= keep;
    if constexpr (kDz) r.z[i] &= keep;
  }
}
template <class E, int kN, bool kDz>
__device__ __forceinline__ float value(const Raw<E, kN, kDz>& r, int k) {
  float scale = 1.f;
  if constexpr (E::kBytes == 1) scale = kept_scale(r.e);
  const float x = value_of<E>(r.w, k, scale);
  if constexpr (kDz) return value_of<E>(r.z, k, 1.f) > 0.f ? x : 0.f;
  else return x;
}
template <class E, int kN, bool kDz>
__device__ __forceinline__ void values(float (&x)[kN], const Raw<E, kN, kDz>& r) {
#pragma unroll
  for (int k = 0; k < kN; ++k) x[k] = value(r, k);
}

// ---- pieces ----
// Three pieces of two values; what is not finite in its first piece has no others.
__device__ __forceinline__ void split_pair(unsigned (&p)[3], float x, float y) {
  const unsigned a = pack_bf16x2(x, y);
  const float rx = x - __uint_as_float(a << 16), ry = y - __uint_as_float(a & 0xFFFF0000u);
  const unsigned b = pack_bf16x2(rx, ry);
  p[0] = a;
  p[1] = b;
  p[2] = pack_bf16x2(rx - __uint_as_float(b << 16), ry - __uint_as_float(b & 0xFFFF0000u));
}
template <int kPieces>
__device__ __forceinline__ void pieces_of(u32x4 (&u)[kPieces], const float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (kPieces == 1) {
      u[0][k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
    } else {
      unsigned p[3];
      split_pair(p, x[2 * k], x[2 * k + 1]);
      u[0][k] = p[0];
      u[1][k] = p[1];
      u[2][k] = p[2];
    }
  }
}

// ---- LDS: units of eight contraction indices, R rows of KS / 8 units ----
// Two neighbouring rows share a line of eight units where KS = 32.  The exclusive or spreads over the banks both the
// reads (32 rows, one unit each) and the writes (units of one row, or one unit of rows kVC apart).
template <int KS>
__device__ __forceinline__ int unit_at(int r, int c) {
  if constexpr (KS == 64) return r * 8 + (c ^ ((r ^ (r >> 3)) & 7));
  const int line = r >> 1, u = (r & 1) << 2 | c;
  return line * 8 + (u ^ ((line ^ (line >> 3)) & 7));
}

// Byte addresses in such a tile follow from one another by exclusive ors and constants, which keeps a step's addresses in a
// handful of registers (kept apart, they did not fit, and a register read back from scratch memory waits for every load that
// was requested before it):
//  - n rows on (n a multiple of 32; KS = 32: of 16 within two such steps): rows_on<KS>(n) exclusive or, n * KS * 2 on;
//  - chunk c on from chunk lh (0 or 1), in pairs: exclusive or c * 16.
template <int KS>
constexpr unsigned rows_on(int n) {
  return (unsigned)((KS == 64 ? n >> 3 : n >> 4) & 7) << 4;
}

constexpr int kThreads = 256;             // of the kernels whose workgroups have four waves

// A tile of kR rows (of the product's operand) by KS contraction indices, from memory through registers of kT threads to LDS.
// kCols = false: the operand's rows are the rows of the matrix; true: its columns, and the contraction runs over the rows.
template <class E, bool kCols, bool kDz, int kR, int KS, int kT>
struct Stager {
  static constexpr int kP = E::kPieces, kC = KS / 8;
  static constexpr int kUnits = kR * kC / kT;                   // per thread
  static constexpr int kN = kCols ? kUnits : 8;                 // columns per vector
  static constexpr int kRaws = kCols ? 8 : kUnits;
  static constexpr int kPlane = kR * kC;                        // units per piece
  static constexpr int kRowsOn = kT / kC;                       // rows between a thread's units (kCols = false)
  Raw<E, kN, kDz> raw[kRaws];
  unsigned off, offz;    // of the thread's first vector from the tile's first row and index, in bytes
  unsigned at;           // of its first unit in LDS, in bytes

  // ld, ldz: bytes from row to row
  __device__ __forceinline__ void start(unsigned ld, unsigned ldz) {
    const unsigned t = threadIdx.x;
    const unsigned row = kCols ? t / (kR / kN) * 8 : t / kC, col = kCols ? t % (kR / kN) * kN : t % kC * 8;
    off = row * ld + col * E::kBytes;
    offz = kDz ? row * ldz + col * E::kBytes : 0;
    at = (unsigned)(kCols ? unit_at<KS>(col, row / 8) : unit_at<KS>(row, col / 8)) * 16;
  }
  // Requests are whole vectors, none behind a branch:
  //  - a unit that reaches behind index d is taken so much earlier that it ends there, in both operands alike, and mask()
  //    clears the indices that the unit before has; d is at least eight;
  //  - past the last row the last one is read again, and not stored; of columns the last whole vector (place() says which).
  static __device__ __forceinline__ int first(int k, int d) { return min(k, d - 8); }
  // Place of the thread's first column in a tile of that many; below zero where they are fewer than a vector has.
  static __device__ __forceinline__ int place(int t, int cols) { return min(t % (kR / kN) * kN, cols - kN); }
  // The thread's number, not to be computed with ahead of time: what the last tiles need is formed where they need it.
  static __device__ __forceinline__ int thread_now() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
  }
  // p (and z): the tile's first row at index k0 (kCols: index k0 at the tile's first column), a place that all lanes share;
  // rows from there to the end; the indices end at d.
  __device__ __forceinline__ void load(const char* p, const char* z, unsigned ld, unsigned ldz, int rows, int k0, int d) {
    if (rows >= kR && k0 + KS <= d) {                  // the same for all lanes
#pragma unroll
      for (int i = 0; i < kRaws; ++i) {
        const size_t on = (size_t)(kCols ? i : i * kRowsOn);
        fetch<E, kN, kDz>(raw[i], p + on * ld, kDz ? z + on * ldz : nullptr, off, offz);
      }
      return;
    }
    const int t = thread_now();
    if constexpr (kCols) {
      const int k = first(k0 + t / (kR / kN) * 8, d) - k0;
#pragma unroll
      for (int i = 0; i < 8; ++i) fetch<E, kN, kDz>(raw[i], p + (long long)(k + i) * ld + place(t, rows) * E::kBytes, nullptr, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const long long r = min(t / kC + i * kRowsOn, rows - 1);
        const int c = (first(k0 + t % kC * 8, d) - k0) * E::kBytes;
        fetch<E, kN, kDz>(raw[i], p + r * ld + c, kDz ? z + r * ldz + c : nullptr, 0, 0);
      }
    }
  }
  // Of the tile that was loaded; nothing to do where all its indices are there.
  __device__ __forceinline__ void mask(int k0, int d) {
    if (k0 + KS <= d) return;
    const int t = thread_now();
    if constexpr (kCols) {
      const int k = k0 + t / (kR / kN) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < k - first(k, d)) clear(raw[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int k = k0 + (t + kT * i) % kC * 8;
        clear_front(raw[i], k - first(k, d));
      }
    }
  }
  __device__ __forceinline__ void put(u32x4* lds, unsigned byte, const u32x4 (&p)[kP]) const {
#pragma unroll
    for (int q = 0; q < kP; ++q) *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(lds + q * kPlane) + byte) = p[q];
  }
  // cols (kCols): of the tile
  __device__ __forceinline__ void store(u32x4* lds, float sign, int cols) const {
    if constexpr (!kCols) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        u32x4 p[kP];
        unit(p, raw[i], sign);
        put(lds, (at ^ rows_on<KS>(i * kRowsOn)) + (unsigned)(i * kRowsOn * KS * 2), p);
      }
    } else if (cols >= kR) {
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        u32x4 p[kP];
        column(p, j, sign);
        // a row on within a vector: KS = 64 the next line and bit j of the spread, KS = 32 the other half of the line
        put(lds, KS == 64 ? (at ^ (unsigned)(j << 4)) + (unsigned)(j * 128) : at ^ (unsigned)(j << 6), p);
      }
    } else {
      store_at(lds, sign, place(thread_now(), cols));
    }
  }
  // The thread's first column at that place; what lies in front of the tile is left out.
  __device__ __forceinline__ void store_at(u32x4* lds, float sign, int place) const {
    const int c = thread_now() / (kR / kN);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      u32x4 p[kP];
      column(p, j, sign);
      if (place + j >= 0) put(lds, (unsigned)unit_at<KS>(place + j, c) * 16, p);
    }
  }
  __device__ __forceinline__ void column(u32x4 (&p)[kP], int j, float sign) const {
    if constexpr (E::kBytes == 2 && (!kDz || kP == 2)) {            // halves of the words of two rows
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kP == 2) p[1][i] = __builtin_amdgcn_perm(raw[2 * i + 1].z[j / 2], raw[2 * i].z[j / 2], j & 1 ? 0x07060302u : 0x05040100u);
        p[0][i] = __builtin_amdgcn_perm(raw[2 * i + 1].w[j / 2], raw[2 * i].w[j / 2], j & 1 ? 0x07060302u : 0x05040100u);
      }
    } else {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = value<E, kN, kDz>(raw[i], j);
        y[i] = kP == 1 ? x : x * sign;
      }
      pieces_of<kP>(p, y);
    }
  }
  // Adds the columns' values of the tile (kCols).
  __device__ __forceinline__ void add_columns(double (&sums)[kN]) const {
    float x[8][kN];
#pragma unroll
    for (int i = 0; i < 8; ++i) values<E, kN, kDz>(x[i], raw[i]);
#pragma unroll
    for (int j = 0; j < kN; ++j)
      sums[j] += (double)(((x[0][j] + x[1][j]) + (x[2][j] + x[3][j])) + ((x[4][j] + x[5][j]) + (x[6][j] + x[7][j])));
  }
  static __device__ __forceinline__ void unit(u32x4 (&p)[kP], const Raw<E, 8, kDz>& raw, float sign) {
    if constexpr (E::kBytes == 2 && !kDz) {
      p[0] = u32x4{raw.w[0], raw.w[1], raw.w[2], raw.w[3]};
    } else {
      float x[8];
      values<E, 8, kDz>(x, raw);
      if constexpr (kP > 1)
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= sign;
      pieces_of<kP>(p, x);
    }
  }
};

// The same for the columns of a matrix whose rows are walked: every thread keeps the place of its own columns, and steps from
// row to row.
template <class E, bool kDz, int kR, int KS, int kT>
struct ColumnStager : Stager<E, true, kDz, kR, KS, kT> {
  typedef Stager<E, true, kDz, kR, KS, kT> Base;
  using Base::kN;
  using Base::raw;
  const char *p, *z;
  const unsigned char* e;
  int here;              // place of the thread's first column in the tile
  int some;              // fewer columns than a vector has: so many; else 0
  bool whole;            // the tile's columns are all there

  __device__ __forceinline__ void start(const Source& s, int col0, long long row0) {
    Base::start(0, 0);
    // the last whole vector again where the columns end inside one (of kept rows, which are filled up to whole blocks, the
    // last of its block)
    const int cols = E::kBytes == 1 ? (s.cols + kKeptBlock - 1) / kKeptBlock * kKeptBlock : s.cols;
    const int col = max(0, min(col0 + (int)(threadIdx.x % (kR / kN)) * kN, cols - kN));
    here = col - col0;
    whole = col0 + kR <= cols;
    some = cols < kN ? cols : 0;
    p = s.p[0] + (row0 * s.ld + col) * E::kBytes;
    z = kDz ? s.z + (row0 * s.ldz + col) * E::kBytes : nullptr;
    e = E::kBytes == 1 ? s.exponent + row0 * s.ld_exponent + col / kKeptBlock : nullptr;
  }
  // rows: from the thread's place to the end of the slab; the place moves on by a step
  __device__ __forceinline__ void load(const Source& s, long long rows) {
    const int c = threadIdx.x / (kR / kN) * 8, most = (int)min(rows, (long long)KS) - 1;
    const unsigned ld = (unsigned)s.ld * E::kBytes, ldz = (unsigned)s.ldz * E::kBytes, lde = (unsigned)s.ld_exponent;
    if (some == 0) {
      // one offset a thread, of the last rows' steps one for each
      unsigned r = c;
      asm volatile("" : "+v"(r));
      if (most == KS - 1) {
        const unsigned o = r * ld, oz = r * ldz, oe = r * lde;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          fetch<E, kN, kDz>(raw[i], p + (size_t)i * ld, kDz ? z + (size_t)i * ldz : nullptr, o, oz);
          if constexpr (E::kBytes == 1) raw[i].e = (e + (size_t)i * lde)[oe];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const unsigned q = (unsigned)min((int)r + i, most);
          fetch<E, kN, kDz>(raw[i], p, z, q * ld, q * ldz);
          if constexpr (E::kBytes == 1) raw[i].e = e[q * lde];
        }
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const unsigned r = (unsigned)min(c + i, most);
        Raw<E, kN, kDz> x;
        fetch_some<E, kN, kDz>(x, p, z, r * ld, r * ldz, some);
        if constexpr (E::kBytes == 1) x.e = e[r * lde];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k == i) raw[k] = x;
      }
    }
    p += (size_t)KS * ld;
    if constexpr (kDz) z += (size_t)KS * ldz;
    if constexpr (E::kBytes == 1) e += (size_t)KS * lde;
  }
  __device__ __forceinline__ void mask(int rows) {
    if (rows >= KS) return;
    const int c = Base::thread_now() / (kR / kN) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i >= rows) clear(raw[i]);
  }
  __device__ __forceinline__ void store(u32x4* lds, float sign) const {
    if (whole) Base::store(lds, sign, kR);
    else Base::store_at(lds, sign, here);
  }
};

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.f;
  return z;
}
__device__ __forceinline__ f32x16 mfma(const u32x4& b, const u32x4& a, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
}

// Where a lane's operands of a wave's first 32 rows lie, in bytes: row `row0` (a multiple of 32 kI) + lane % 32, chunk lane / 32.
template <int KS>
__device__ __forceinline__ unsigned operands_at(int row0) {
  const int lane = threadIdx.x & 63;
  return (unsigned)unit_at<KS>(row0 + (lane & 31), lane >> 5) * 16;
}
// One staged step: acc[i][j] += A (rows a0 + 32 i ..) times B (rows b0 + 32 j ..), from where operands_at() says for a0 and
// b0.  The small products first.
template <int kPA, int kPB, int KS, int kRA, int kRB, int kI, int kFrom = 0, int kTo = KS / 16>      // part of the step, in 16 indices
__device__ __forceinline__ void multiply(f32x16 (&acc)[kI][2], const u32x4* A, const u32x4* B, unsigned a0, unsigned b0) {
  constexpr int kMost = kPA > kPB ? kPA : kPB;
  asm volatile("" : "+v"(a0), "+v"(b0));               // the addresses that follow are formed here, not kept from step to step
#pragma unroll
  for (int k = kFrom; k < kTo; ++k) {
    u32x4 a[kPA][kI], b[kPB][2];
#pragma unroll
    for (int p = 0; p < kPA; ++p)
#pragma unroll
      for (int i = 0; i < kI; ++i)
        a[p][i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(A + p * (kRA * KS / 8)) + (a0 ^ (unsigned)(k << 5) ^ rows_on<KS>(32 * i)) + i * KS * 64);
#pragma unroll
    for (int p = 0; p < kPB; ++p)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        b[p][j] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(B + p * (kRB * KS / 8)) + (b0 ^ (unsigned)(k << 5) ^ rows_on<KS>(32 * j)) + j * KS * 64);
#pragma unroll
    for (int sum = kMost - 1; sum >= 0; --sum)
#pragma unroll
      for (int p = 0; p < kPA; ++p) {
        const int q = sum - p;
        if (q < 0 || q >= kPB) continue;
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = mfma(b[q][j], a[p][i], acc[i][j]);
      }
    __builtin_amdgcn_sched_barrier(0);                // one index's operands in registers at a time
  }
}
template <int kI>
__device__ __forceinline__ void add_section(f32x16 (&total)[kI][2], f32x16 (&acc)[kI][2], float sign) {
#pragma unroll
  for (int i = 0; i < kI; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        total[i][j][v] = fmaf(acc[i][j][v], sign, total[i][j][v]);
        acc[i][j][v] = 0.f;
      }
}

// The part of a 1-D list of tiles that this workgroup takes: a contiguous eighth per XCD.
struct TileRange {
  long long first, end, step;
};
__device__ __forceinline__ TileRange tiles_of(long long ntiles) {
  const int xcd = blockIdx.x & 7;
  return {ntiles * xcd / 8 + (blockIdx.x >> 3), ntiles * (xcd + 1) / 8, gridDim.x >> 3};
}

struct ProductArgs {
  Source a;              // [rows, K]
  Source b;              // kColsB: [K, N]; else [N, K]
  const int* nrows;
  int K, N, act;
  const float* bias;
  const char* R;
  long long ldr;
  char* Z;
  long long ldz;
  char* Y;
  long long ldy;
  const int* stop;
};

template <class E>
__device__ __forceinline__ float load_value(const char* p, long long i) {
  unsigned w[1];
  read_words<E::kBytes>(w, p + i * E::kBytes);
  return value_of<E>(w, 0, 1.f);
}
template <class E>
__device__ __forceinline__ void store_value(char* p, long long i, float x) {
  if constexpr (E::kBytes == 4) reinterpret_cast<float*>(p)[i] = x;
  else reinterpret_cast<u16*>(p)[i] = to_bf16(x);
}
// 16 bytes of values
template <class E>
__device__ __forceinline__ void store_wide(char* p, long long i, const float (&x)[16 / E::kBytes]) {
  u32x4 w;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (E::kBytes == 4) w[k] = __float_as_uint(x[k]);
    else w[k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
  }
  *reinterpret_cast<u32x4_any*>(p + i * E::kBytes) = w;
}

// What becomes of 16 / kBytes neighbouring sums z of a row: a layer's results (kColsB), or a gradient, which is the sums.
// r: the residual's 16 bytes, where all of them are columns.  The bias comes in registers: a load here would wait for the
// stores of the rows before it.
template <class E>
__device__ __forceinline__ void bias_at(float (&bias)[16 / E::kBytes], const ProductArgs& g, int col) {
#pragma unroll
  for (int k = 0; k < 16 / E::kBytes; ++k) bias[k] = g.bias && col + k < g.N ? g.bias[col + k] : 0.f;
}
template <class E, bool kDz, bool kColsB>
__device__ __forceinline__ void finish(const ProductArgs& g, long long row, int col, float (&z)[16 / E::kBytes],
                                       const float (&bias)[16 / E::kBytes], const unsigned (&r)[4]) {
  constexpr int kW = 16 / E::kBytes;
  if constexpr (E::kPieces > 1) {
    unsigned bad = 0;
#pragma unroll
    for (int k = 0; k < kW; ++k) bad |= !__builtin_isfinite(z[k]) && col + k < g.N ? 1u << k : 0u;
    for (; bad; bad &= bad - 1) {                      // formed again in fp32
      const int c = __ffs(bad) - 1;
      float s = 0.f;
      for (int i = 0; i < g.K; ++i)
        s = fmaf(single<E, kDz>(g.a, row, i), kColsB ? single<E, false>(g.b, i, col + c) : single<E, false>(g.b, col + c, i), s);
#pragma unroll
      for (int k = 0; k < kW; ++k) z[k] = k == c ? s : z[k];
    }
  }
  if (col + kW <= g.N) {
    if constexpr (kColsB) {
#pragma unroll
      for (int k = 0; k < kW; ++k) z[k] += bias[k];
      if (g.Z) store_wide<E>(g.Z, row * g.ldz + col, z);
      activate<kW>(z, g.act);
      if (g.R)
#pragma unroll
        for (int k = 0; k < kW; ++k) z[k] += value_of<E>(r, k, 1.f);
    }
    store_wide<E>(g.Y, row * g.ldy + col, z);
    return;
  }
  if constexpr (kColsB) {
#pragma unroll
    for (int k = 0; k < kW; ++k) z[k] += bias[k];
    if (g.Z)
#pragma unroll
      for (int k = 0; k < kW; ++k)
        if (col + k < g.N) store_value<E>(g.Z, row * g.ldz + col + k, z[k]);
    activate<kW>(z, g.act);
  }
#pragma unroll
  for (int k = 0; k < kW; ++k)
    if (col + k < g.N) {
      if (kColsB && g.R) z[k] += load_value<E>(g.R, row * g.ldr + col + k);
      store_value<E>(g.Y, row * g.ldy + col + k, z[k]);
    }
}

// Few rows: a workgroup per 32 x 32 tile, operands straight from memory, the contraction dealt to its four waves in chunks of
// 16; their sums meet in LDS.  A tile of the kernel below would keep one CU busy while the others have nothing to do.
// Bound by latency: the launch, two or three rounds of requests, the exchange (1 x 256 -> 256 in bf16 and 437 x 384 -> 128 in
// fp32 take 5 to 8 us).
constexpr int kFewLd = 36;             // floats from row to row of a tile in LDS
template <class E, bool kDz, bool kColsB, bool kVec>      // kVec: the contraction is at least eight
__global__ __launch_bounds__(kThreads, 2) void few_rows_kernel(const ProductArgs g, long long few) {
  if (g.stop && g.stop[0] != 0) return;
  constexpr int kP = E::kPieces, kW = 16 / E::kBytes;
  __shared__ float lds[4 * 32 * kFewLd];
  const long long rows = g.nrows ? g.nrows[0] : g.a.rows;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, l32 = lane & 31, lh = lane >> 5;
  const int nct = (g.N + 31) >> 5, d = g.a.d, per = (d + 15) >> 4, chunks = g.K / d * per;      // the parts of a row one after another
  const long long ntiles = ((rows + 31) >> 5) * nct;
  if (ntiles > few) return;                           // the tiles of product_kernel
  const float sign = wave & 1 ? -1.f : 1.f;           // what the pieces' sums drop cancels between the waves
  for (long long tile = blockIdx.x; tile < ntiles; tile += gridDim.x) {
    const long long m0 = tile / nct * 32, row = min(m0 + l32, rows - 1);
    const int n0 = (int)(tile % nct) * 32, col = min(n0 + l32, g.N - 1);
    struct Chunk {
      Raw<E, 8, kDz> a;
      Raw<E, kColsB ? 1 : 8, false> b[kColsB ? 8 : 1];
    };
    // past the end the last chunk again, so that no request waits behind a branch; eight indices that reach behind the last
    // one are taken earlier, and those that the eight before have are cleared
    const unsigned ldb = (unsigned)g.b.ld * E::kBytes;
    const char* pb = g.b.p[0] + (kColsB ? (long long)col * E::kBytes : (long long)col * ldb);
    auto load = [&](Chunk& x, int c) {
      c = min(c, chunks - 1);
      const int seg = c >= 2 * per ? 2 : (c >= per ? 1 : 0), k = (c - seg * per) * 16 + 8 * lh, ka = kVec ? min(k, d - 8) : 0;
      const char* pa = part_of(g.a, seg) + (row * g.a.ld + ka) * E::kBytes;
      const char* pz = kDz ? g.a.z + (row * g.a.ldz + ka) * E::kBytes : nullptr;
      if constexpr (kVec) fetch<E, 8, kDz>(x.a, pa, pz, 0, 0);
      else fetch_some<E, 8, kDz>(x.a, pa, pz, 0, 0, min(d - ka, 8));
      if constexpr (kColsB) {
        const int kb = seg * d;
#pragma unroll
        for (int i = 0; i < 8; ++i) fetch<E, 1, false>(x.b[i], pb + (long long)(kb + (kVec ? ka + i : min(k + i, d - 1))) * ldb, nullptr, 0, 0);
      } else {
        if constexpr (kVec) fetch<E, 8, false>(x.b[0], pb, nullptr, (unsigned)(ka * E::kBytes), 0);
        else fetch_some<E, 8, false>(x.b[0], pb, nullptr, (unsigned)(ka * E::kBytes), 0, min(d - ka, 8));
      }
    };
    f32x16 acc = zero16();
    auto step = [&](const Chunk& x, int c) {
      const int k = c % per * 16 + 8 * lh, from = kVec ? k - min(k, d - 8) : 0, to = kVec ? 8 : d - k;      // the indices that count
      u32x4 a[kP], b[kP];
      float y[8];
      values<E, 8, kDz>(y, x.a);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = i >= from && i < to ? y[i] : 0.f;
      pieces_of<kP>(a, y);
      if constexpr (kColsB) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = value_of<E>(x.b[i].w, 0, 1.f);
      } else {
        values<E, 8, false>(y, x.b[0]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = i >= from && i < to ? (kP > 1 ? y[i] * sign : y[i]) : 0.f;
      pieces_of<kP>(b, y);
#pragma unroll
      for (int sum = kP - 1; sum >= 0; --sum)
#pragma unroll
        for (int p = 0; p <= sum; ++p) acc = mfma(b[sum - p], a[p], acc);
    };
    Chunk x0, x1, x2;
    load(x0, wave);
    load(x1, wave + 4);
    load(x2, wave + 8);
    for (int c = wave; c < chunks; c += 12) {
      step(x0, c);
      load(x0, c + 12);
      if (c + 4 < chunks) step(x1, c + 4);
      load(x1, c + 16);
      if (c + 8 < chunks) step(x2, c + 8);
      load(x2, c + 20);
    }
    __syncthreads();                                  // the last tile has been read
    // register v of a lane: row l32, column 8 (v / 4) + 4 lh + v % 4
    float* mine = lds + wave * 32 * kFewLd;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int v = 0; v < 4; ++v) mine[l32 * kFewLd + 8 * q + 4 * lh + v] = acc[4 * q + v];
    __syncthreads();
    const int r = t / (32 / kW), c0 = t % (32 / kW) * kW;
    if (r < 32 && m0 + r < rows && n0 + c0 < g.N) {
      float z[kW], bias[kW];
      if constexpr (kColsB) bias_at<E>(bias, g, n0 + c0);
      unsigned res[4] = {0, 0, 0, 0};
      if (kColsB && g.R && n0 + c0 + kW <= g.N) read_words<16>(res, g.R + ((m0 + r) * g.ldr + n0 + c0) * E::kBytes);
#pragma unroll
      for (int k = 0; k < kW; ++k) {
        const float* p = lds + r * kFewLd + c0 + k;
        const float u0 = p[0], u1 = p[32 * kFewLd], u2 = p[64 * kFewLd], u3 = p[96 * kFewLd];
        z[k] = kP > 1 ? (u0 - u1) + (u2 - u3) : (u0 + u1) + (u2 + u3);
      }
      finish<E, kDz, kColsB>(g, m0 + r, n0 + c0, z, bias, res);
    }
  }
}

// rows x N outputs, contraction over K columns of a.  Tiles of 64 kI rows x 32 kWaves columns, waves of 32 kI x 64: two
// side by side in rows, the others in columns.  kShort: of half the rows.
// What bounds it is how much is requested at a time: a step's loads (64 KB per CU) are on their way while the step before is
// multiplied, some 2 us, so that every byte loaded twice shows.  Eight waves take 256 columns, and the rows of a layer of
// that width are read once; LDS then holds two steps, and a step needs one barrier.  The residual's rows are requested 32 at a
// time before the sums go through LDS.
// Measured: bf16 2000003 x 768 -> 256 with residual 1.25 ms (4.1 TB/s, 630 TFLOP/s; library product alone 0.97 ms); fp32
// 196311 x 201 -> 139 with GELU, residual and Z 0.212 ms (matrix cores 25 % busy; the rest is conversions, the
// epilogue's instructions and waiting); dX of 524309 x 256 -> 768 in bf16 0.36 ms, of two arrays of dZ 0.56 ms (740 TFLOP/s).
template <class E, int kWaves, bool kShort>
struct ProductShape {
  static constexpr int kI = (E::kPieces == 1 ? 4 : 2) / (kShort ? 2 : 1), kTileM = 64 * kI, kTileN = 32 * kWaves, KS = E::kPieces == 1 ? 64 : 32;
  static constexpr int kUnitsA = E::kPieces * kTileM * KS / 8, kUnitsB = E::kPieces * kTileN * KS / 8, kBuffers = kWaves / 4;
  static constexpr int kLd = 68, kEnd = kWaves * 32 * kLd / 4;                    // of a wave's 32 x 64 sums, in units
  static constexpr int kStep = kUnitsA + kUnitsB, kLds = kBuffers * kStep > kEnd ? kBuffers * kStep : kEnd;
};
template <class E, bool kDz, bool kColsB, int kWaves, bool kShort>
__global__ __launch_bounds__(64 * kWaves, 2) void product_kernel(const ProductArgs g, long long few) {
  if (g.stop && g.stop[0] != 0) return;
  typedef ProductShape<E, kWaves, kShort> Shape;
  constexpr int kP = E::kPieces, KS = Shape::KS, kI = Shape::kI, kTileM = Shape::kTileM, kTileN = Shape::kTileN, kW = 16 / E::kBytes, kLd = Shape::kLd;
  extern __shared__ u32x4 lds[];
  const long long rows = g.nrows ? g.nrows[0] : g.a.rows;
  if (((rows + 31) >> 5) * ((g.N + 31) >> 5) <= few) return;      // few_rows_kernel
  const int wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1, lane = threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5;
  // the parts of a row one after another, each with steps of its own
  const int nct = (g.N + kTileN - 1) / kTileN, d = g.a.d, per = (d + KS - 1) / KS, steps = g.K / d * per;
  const unsigned lda = (unsigned)g.a.ld * E::kBytes, ldz = (unsigned)g.a.ldz * E::kBytes, ldb = (unsigned)g.b.ld * E::kBytes;
  const TileRange tr = tiles_of((rows + kTileM - 1) / kTileM * nct);
  Stager<E, false, kDz, kTileM, KS, 64 * kWaves> sa;
  Stager<E, kColsB, false, kTileN, KS, 64 * kWaves> sb;
  sa.start(lda, ldz);
  sb.start(ldb, 0);
  const unsigned a0 = operands_at<KS>(wm * 32 * kI), b0 = operands_at<KS>(wn * 64);
  auto load = [&](long long tile, int step) {
    const long long m0 = tile / nct * kTileM;
    const int n0 = (int)(tile % nct) * kTileN;
    const int seg = step >= 2 * per ? 2 : (step >= per ? 1 : 0), k0 = (step - seg * per) * KS;
    sa.load(part_of(g.a, seg) + m0 * lda + k0 * E::kBytes, kDz ? g.a.z + m0 * ldz + k0 * E::kBytes : nullptr, lda, ldz,
            (int)min(rows - m0, (long long)kTileM), k0, d);
    const long long kb = kColsB ? (long long)seg * d + k0 : k0;      // the parts of a gradient meet the same columns of W
    sb.load(kColsB ? g.b.p[0] + kb * ldb + n0 * E::kBytes : g.b.p[0] + (long long)n0 * ldb + kb * E::kBytes, nullptr, ldb, 0,
            min(g.N - n0, kTileN), k0, d);
  };
  for (long long tile = tr.first; tile < tr.end; tile += tr.step) {
    const long long m0 = tile / nct * kTileM;
    const int n0 = (int)(tile % nct) * kTileN;
    f32x16 acc[kI][2], total[kP > 1 ? kI : 1][2];
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        acc[i][j] = zero16();
        if (kP > 1) total[i][j] = zero16();
      }
    auto sign_of = [](int step) { return (step >> 1) & 1 ? -1.f : 1.f; };
    auto stash = [&](int step, u32x4* A) {
      const int k0 = step % per * KS;
      sa.mask(k0, d);
      sb.mask(k0, d);
      sa.store(A, 1.f, 0);
      sb.store(A + Shape::kUnitsA, sign_of(step), kColsB ? min(g.N - n0, kTileN) : 0);
    };
    auto section = [&](int step) {
      if constexpr (kP > 1) {
        if ((step & 1) || step + 1 == steps) add_section<kI>(total, acc, sign_of(step));
      }
    };
    load(tile, 0);
    __syncthreads();                                   // the last tile's sums have been read
    if constexpr (Shape::kBuffers > 1) {
      // the next step's rows go to the other half of LDS between the two halves of a step's products, so that one wave's
      // conversions run beside another's products; then the step after is requested
      stash(0, lds);
      if (steps > 1) load(tile, 1);
      __syncthreads();
      for (int step = 0; step < steps; ++step) {
        const u32x4* A = lds + (step & 1) * Shape::kStep;
        const u32x4* B = A + Shape::kUnitsA;
        multiply<kP, kP, KS, kTileM, kTileN, kI, 0, KS / 32>(acc, A, B, a0, b0);
        if (step + 1 < steps) stash(step + 1, lds + ((step + 1) & 1) * Shape::kStep);
        if (step + 2 < steps) load(tile, step + 2);
        multiply<kP, kP, KS, kTileM, kTileN, kI, KS / 32, KS / 16>(acc, A, B, a0, b0);
        section(step);
        __syncthreads();
      }
    } else {
      for (int step = 0; step < steps; ++step) {
        if (step > 0) __syncthreads();                 // the last step's operands have been read
        stash(step, lds);
        __syncthreads();
        if (step + 1 < steps) load(tile, step + 1);
        multiply<kP, kP, KS, kTileM, kTileN, kI>(acc, lds, lds + Shape::kUnitsA, a0, b0);
        section(step);
      }
      __syncthreads();
    }
    // register v of a lane: row l32, column 8 (v / 4) + 4 lh + v % 4 of a block; through LDS, 32 rows of a wave at a time, so
    // that a wave reads and writes whole rows of its 64 columns
    float* end = reinterpret_cast<float*>(lds) + wave * 32 * kLd;
    constexpr int kLanes = 64 / kW, kRounds = 32 / kW;
    // a vector that the columns end in starts earlier, so that it is whole: some results are written twice, alike (value by
    // value, a layer of 32 x 127 took 140 us where one of 32 x 128 took 73, each of 196311 rows)
    const int at = lane % kLanes * kW, have = g.N - n0 - wn * 64;
    const int c0 = have < kW ? at : min(at, have - kW), col = n0 + wn * 64 + c0;
    const bool wide = col + kW <= g.N;
    float bias[kW];
    if constexpr (kColsB) bias_at<E>(bias, g, col);
    for (int part = 0; part < kI; ++part) {
      const long long r0 = m0 + wm * 32 * kI + part * 32 + lane / kLanes;
      unsigned res[kRounds][4];
      if (kColsB && g.R && wide) {                     // requested together; past the end the last row again
#pragma unroll
        for (int u = 0; u < kRounds; ++u) read_words<16>(res[u], g.R + (min(r0 + u * kW, rows - 1) * g.ldr + col) * E::kBytes);
      }
#pragma unroll
      for (int i = 0; i < kI; ++i)
        if (i == part) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float4 v;
              if constexpr (kP > 1) v = make_float4(total[i][j][4 * q], total[i][j][4 * q + 1], total[i][j][4 * q + 2], total[i][j][4 * q + 3]);
              else v = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
              *reinterpret_cast<float4*>(end + l32 * kLd + j * 32 + 8 * q + 4 * lh) = v;
            }
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < kRounds; ++u) {
        if (r0 + u * kW >= rows || at >= have) continue;
        float z[kW];
#pragma unroll
        for (int k = 0; k < kW; ++k) z[k] = end[(lane / kLanes + u * kW) * kLd + c0 + k];
        finish<E, kDz, kColsB>(g, r0 + u * kW, col, z, bias, res[u]);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// ---- dZ of the smooth activations ----
// dz = dy act'(z), and its column sums over the rows of a block: 32 vectors of columns x 8 rows of threads.  Bound by memory:
// 524309 x 256 in bf16 0.15 ms, 5.3 TB/s, with the second number 0.20 ms.
struct SlopeArgs {
  long long rows;
  int N, act;
  const char* dy;
  long long lddy;
  const char* z;
  long long ldz;
  char* dz;              // [rows, N]; with pair (bf16) behind it what each value's rounding left, as bf16
  int pair;
  float* part;           // [row blocks][N]
  int row_blocks;
};
template <class E, int kV>
__global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs g) {
  __shared__ double red[8][32 * kV];
  const long long rows = g.rows;
  const int t = threadIdx.x, cb = blockIdx.x / g.row_blocks, rb = blockIdx.x % g.row_blocks;
  const int col = (cb * 32 + (t & 31)) * kV;
  double sum[kV];
#pragma unroll
  for (int k = 0; k < kV; ++k) sum[k] = 0.0;
  if (col < g.N)
    for (long long r = (long long)rb * 8 + (t >> 5); r < rows; r += (long long)g.row_blocks * 16) {
      unsigned y[2][(kV * E::kBytes + 3) / 4], z[2][(kV * E::kBytes + 3) / 4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {                    // two rows requested together; past the end the last one again
        const long long row = min(r + (long long)u * g.row_blocks * 8, rows - 1);
        read_words<kV * E::kBytes>(y[u], g.dy + (row * g.lddy + col) * E::kBytes);
        read_words<kV * E::kBytes>(z[u], g.z + (row * g.ldz + col) * E::kBytes);
      }
      float d[2][kV];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const long long row = r + (long long)u * g.row_blocks * 8;
#pragma unroll
        for (int k = 0; k < kV; ++k) d[u][k] = value_of<E>(z[u], k, 1.f);
        slopes<kV>(d[u], g.act);
#pragma unroll
        for (int k = 0; k < kV; ++k) d[u][k] = row < rows ? d[u][k] * value_of<E>(y[u], k, 1.f) : 0.f;
        if (row < rows) {
          const long long i = row * g.N + col;
          float left[kV];
#pragma unroll
          for (int k = 0; k < kV; ++k) {                 // what is not finite in its first number has no second
            const float first = __uint_as_float((unsigned)to_bf16(d[u][k]) << 16);
            left[k] = __builtin_isfinite(first) ? d[u][k] - first : 0.f;
          }
          if constexpr (kV * E::kBytes == 16) {
            store_wide<E>(g.dz, i, d[u]);
            if (E::kBytes == 2 && g.pair) store_wide<E>(g.dz, rows * g.N + i, left);
          } else {
#pragma unroll
            for (int k = 0; k < kV; ++k) {
              store_value<E>(g.dz, i + k, d[u][k]);
              if (E::kBytes == 2 && g.pair) store_value<E>(g.dz, rows * g.N + i + k, left[k]);
            }
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kV; ++k) sum[k] += (double)(d[0][k] + d[1][k]);
    }
  if (!g.part) return;
#pragma unroll
  for (int k = 0; k < kV; ++k) red[t >> 5][(t & 31) * kV + k] = sum[k];
  __syncthreads();
  for (int i = t; i < 32 * kV; i += 256) {
    const int c = cb * 32 * kV + i;
    if (c >= g.N) continue;
    double s = 0.0;
#pragma unroll
    for (int p = 0; p < 8; ++p) s += red[p][i];
    g.part[(size_t)rb * g.N + c] = (float)s;
  }
}

// ---- weight gradients ----
struct WeightArgs {
  Source a;              // X  [rows, M]
  Source b;              // dZ [rows, N]
  int M, N, S;
  float* part;           // [S][M * N + N]
  int sums;              // column sums of dZ are wanted
};
struct Slab {
  long long r0, r1;
};
__device__ __forceinline__ Slab slab_rows(const WeightArgs& g, long long rows, int slab, int KS) {
  long long per = (rows + g.S - 1) / g.S;
  per = (per + KS - 1) / KS * KS;
  const long long r0 = min((long long)slab * per, rows);
  return {r0, min(r0 + per, rows)};
}
// Tiles of dW: 64 kI x 32 kWaves, as above; every tile of a slab loads the slab's rows, so that wide ones load less.  Measured:
// 524309 rows, 768 x 256 in bf16 0.29 ms (710 TFLOP/s), with dZ in two numbers 0.41 ms (1000 TFLOP/s); 474011 rows, 384 x 128, kept rows times fp32 ones 0.32 ms.
template <class EA, class EB, int kWaves>
struct WeightShape {
  static constexpr int KS = EB::kPieces == 1 ? 64 : 32, kI = EB::kBytes == 2 ? kWaves / 2 : 2;
  static constexpr bool kSections = EB::kBytes == 4;
  static constexpr int kTileM = 64 * kI, kTileN = 32 * kWaves, kT = 64 * kWaves, kBuffers = kWaves / 4;
  static constexpr int kUnitsA = EA::kPieces * kTileM * KS / 8, kUnitsB = EB::kPieces * kTileN * KS / 8, kStep = kUnitsA + kUnitsB;
  static constexpr int kLds = kBuffers * kStep;
};
template <class EB>
constexpr int kSlabStep = EB::kPieces == 1 ? 64 : 32;

template <class EA, class EB, bool kDz, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void weight_kernel(const WeightArgs g) {
  typedef WeightShape<EA, EB, kWaves> Shape;
  constexpr int kPA = EA::kPieces, kPB = EB::kPieces, KS = Shape::KS, kI = Shape::kI, kHold = 256 / KS, kT = Shape::kT;
  constexpr int kTileM = Shape::kTileM, kTileN = Shape::kTileN;
  extern __shared__ u32x4 lds[];
  const long long rows = g.a.rows;
  const int wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1, lane = threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5;
  const int tiles_n = (g.N + kTileN - 1) / kTileN, tiles_m = max(1, (g.M + kTileM - 1) / kTileM), ntile = tiles_m * tiles_n;
  // the tiles of a slab read the same rows: they run on one XCD (the grid is ntile * S, S a multiple of eight)
  const int item = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  const int tile = item % ntile, slab = item / ntile;
  const int m0 = tile / tiles_n * kTileM, n0 = tile % tiles_n * kTileN;
  const Slab sl = slab_rows(g, rows, slab, KS);
  const int steps = (int)((sl.r1 - sl.r0 + KS - 1) / KS);
  // fp32: sections of 256 rows into a total of their own, every other one negated, and so is the first of every other slab
  f32x16 acc[kI][2], total[Shape::kSections ? kI : 1][2];
#pragma unroll
  for (int i = 0; i < kI; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      acc[i][j] = zero16();
      if (Shape::kSections) total[i][j] = zero16();
    }
  const bool want_sums = g.sums && m0 == 0;
  ColumnStager<EA, false, kTileM, KS, kT> sa;
  ColumnStager<EB, kDz, kTileN, KS, kT> sb;
  constexpr int kN = ColumnStager<EB, kDz, kTileN, KS, kT>::kN;
  double sums[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) sums[j] = 0.0;
  const bool product = g.M > 0;
  const unsigned a0 = operands_at<KS>(wm * 32 * kI), b0 = operands_at<KS>(wn * 64);
  if (product) sa.start(g.a, m0, sl.r0);
  sb.start(g.b, n0, sl.r0);
  const long long all = sl.r1 - sl.r0;
  auto load = [&](int step) {
    if (product) sa.load(g.a, all - (long long)step * KS);
    sb.load(g.b, all - (long long)step * KS);
  };
  auto sign_of = [&](int step) { return Shape::kSections && ((step / kHold) ^ slab) & 1 ? -1.f : 1.f; };
  auto stash = [&](int step, u32x4* A) {
    const int left = (int)min(all - (long long)step * KS, (long long)KS);
    sa.mask(left);
    sb.mask(left);
    if (product) sa.store(A, 1.f);
    sb.store(A + Shape::kUnitsA, sign_of(step));
    if constexpr (!(kPB == 2)) if (want_sums) sb.add_columns(sums);
  };
  auto section = [&](int step) {
    if constexpr (Shape::kSections) {
      if (step % kHold == kHold - 1 || step + 1 == steps) add_section<kI>(total, acc, sign_of(step));
    }
  };
  if (steps > 0) load(0);
  if constexpr (Shape::kBuffers > 1) {                 // as in product_kernel
    if (steps > 0) stash(0, lds);
    if (steps > 1) load(1);
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
      const u32x4* A = lds + (step & 1) * Shape::kStep;
      const u32x4* B = A + Shape::kUnitsA;
      if (product) multiply<kPA, kPB, KS, kTileM, kTileN, kI, 0, KS / 32>(acc, A, B, a0, b0);
      if (step + 1 < steps) stash(step + 1, lds + ((step + 1) & 1) * Shape::kStep);
      if (step + 2 < steps) load(step + 2);
      if (product) multiply<kPA, kPB, KS, kTileM, kTileN, kI, KS / 32, KS / 16>(acc, A, B, a0, b0);
      section(step);
      __syncthreads();
    }
  } else {
    for (int step = 0; step < steps; ++step) {
      if (step > 0) __syncthreads();
      stash(step, lds);
      __syncthreads();
      if (step + 1 < steps) load(step + 1);
      if (product) multiply<kPA, kPB, KS, kTileM, kTileN, kI>(acc, lds, lds + Shape::kUnitsA, a0, b0);
      section(step);
    }
  }
  float* P = g.part + (size_t)slab * ((size_t)g.M * g.N + g.N);
  const bool quads = g.N % 4 == 0;
#pragma unroll
  for (int i = 0; i < kI; ++i) {
    const int m = m0 + wm * 32 * kI + i * 32 + l32;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + wn * 64 + j * 32 + 8 * q + 4 * lh;
        const f32x16& s = Shape::kSections ? total[Shape::kSections ? i : 0][j] : acc[i][j];
        float* p = P + (size_t)m * g.N + n;
        if (m < g.M && n < g.N) {
          if (quads) {
            *reinterpret_cast<float4*>(p) = make_float4(s[4 * q], s[4 * q + 1], s[4 * q + 2], s[4 * q + 3]);
          } else {
#pragma unroll
            for (int v = 0; v < 4; ++v)
              if (n + v < g.N) p[v] = s[4 * q + v];
          }
        }
      }
  }
  if (want_sums) {                                   // the same for the whole workgroup
    double* red = reinterpret_cast<double*>(lds);    // [KS / 8][kTileN]
    constexpr int kBlocks = kTileN / kN;
    static_assert(KS / 8 * kTileN * 8 <= Shape::kLds * 16, "column sums in LDS");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kN; ++j)
      if (sb.here + j >= 0) red[threadIdx.x / kBlocks * kTileN + sb.here + j] = sums[j];
    __syncthreads();
    const int n = n0 + (int)threadIdx.x;
    if (threadIdx.x < kTileN && n < g.N) {
      double v = 0.0;
#pragma unroll
      for (int c = 0; c < KS / 8; ++c) v += red[c * kTileN + threadIdx.x];
      P[(size_t)g.M * g.N + n] = (float)v;
    }
  }
}

// dW [M, N] and db [N] = sums of the slabs' parts in 64 bits, ascending slabs.  A part in pieces that is not finite is
// formed again in fp32.
template <class EA, class EB, bool kDz>
__global__ __launch_bounds__(256) void weight_reduce_kernel(const WeightArgs g, char* dW, long long lddw, float* __restrict__ db) {
  const long long MN = (long long)g.M * g.N, stride = MN + g.N;
  const long long end = db ? stride : MN;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < end; i += (long long)gridDim.x * blockDim.x) {
    double s = 0.0;
    const float* __restrict__ p = g.part + i;
    for (int k = 0; k < g.S; k += 8, p += 8 * stride) {        // S is a multiple of eight; eight requested together
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = p[u * stride];
      if constexpr (EB::kBytes == 4) {
        float probe = 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) probe = fmaf(x[u], 0.f, probe);
        if (!(probe == 0.f) && i < MN) {
          const long long rows = g.a.rows;
          const int m = (int)(i / g.N), n = (int)(i % g.N);
          for (int u = 0; u < 8; ++u) {
            if (__builtin_isfinite(p[u * stride])) {
              s += (double)p[u * stride];
              continue;
            }
            const Slab sl = slab_rows(g, rows, k + u, kSlabStep<EB>);
            float v = 0.f;
            for (long long r = sl.r0; r < sl.r1; ++r) v = fmaf(single<EA, false>(g.a, r, m), single<EB, kDz>(g.b, r, n), v);
            s += (double)v;
          }
          continue;
        }
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) s += (double)x[u];
    }
    if (i < MN) store_value<EB>(dW, i / g.N * lddw + i % g.N, (float)s);
    else db[i - MN] = (float)s;
  }
}

// Eight waves where they compute no more columns than four would: N is at least 129, and its last tile of 256 is more than half
// full (200000 rows, fp32, 256 -> 384: 316 us by four waves, 391 by eight; 256 -> 512: 404 and 387; weight gradients 416 and
// 375 for 512, 240 and 220 for 256).
bool eight_waves(int N) { return (N + 255) / 256 * 256 == (N + 127) / 128 * 128; }
// For weight gradients; bf16 with a ReLU mask holds more of a step's rows than the registers of eight waves have room for.
bool eight_weight_waves(int N, bool bf16, bool relu) { return eight_waves(N) && !(bf16 && relu); }
// The slabs of a weight gradient: one round of workgroups (two of four waves per CU, or one of eight), at least 256 rows each.
int slabs_of(long long rows, int K, int N, int bf16, int act, int n_cu) {
  const bool eight = eight_weight_waves(N, bf16, act == DC_ACT_RELU);
  const int m = eight && bf16 ? 256 : 128, n = eight ? 256 : 128;
  const int ntile = ((K + m - 1) / m) * ((N + n - 1) / n);
  long long S = (eight ? 1 : 2) * n_cu / (ntile < 1 ? 1 : ntile) / 8 * 8, by_rows = (rows + 255) / 256;
  if (S > by_rows) S = (by_rows + 7) / 8 * 8;
  return S < 8 ? 8 : (int)S;
}
bool smooth(int act) { return act == DC_ACT_GELU || act == DC_ACT_SILU; }
int slope_blocks(long long rows, int n_cu) {           // row blocks of the pass that forms dZ
  const long long want = (rows + 63) / 64, most = (long long)n_cu * 8;
  return (int)(want < 1 ? 1 : (want < most ? want : most));
}

template <class K>
hipError_t allow_lds(K kernel, size_t bytes) {
  return bytes > 64 * 1024 ? hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : hipSuccess;
}
template <class E, bool kDz, bool kColsB, int kWaves, bool kShort>
hipError_t product_tiles(const ProductArgs& g, long long rows, int n_cu, long long few, hipStream_t s) {
  typedef ProductShape<E, kWaves, kShort> Shape;
  const long long most = (long long)n_cu * 8 / kWaves * (kShort ? 2 : 1), tiles = (rows + Shape::kTileM - 1) / Shape::kTileM * ((g.N + Shape::kTileN - 1) / Shape::kTileN);
  auto kernel = product_kernel<E, kDz, kColsB, kWaves, kShort>;
  const hipError_t e = allow_lds(kernel, Shape::kLds * 16);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles < most ? tiles : most) + 7) / 8 * 8), dim3(64 * kWaves), Shape::kLds * 16, s, g, few);
  return hipGetLastError();
}
// Up to `few` 32 x 32 tiles, each gets a workgroup: two rounds of two workgroups per CU (2048 x 256 -> 256 in fp32 9.9 us, by
// the larger tiles 28.3; 4096 rows 17.7 and 28.8; 8192 rows 31.5 and 29.8).  Where only the device knows the rows both
// kernels are launched, and one of them leaves at once.
template <class E, bool kDz, bool kColsB>
hipError_t product(const ProductArgs& g, long long rows, int n_cu, hipStream_t s) {
  const bool narrow = g.a.d < 8 || g.N < 4;            // less than a vector of the tiles' loads
  const long long small = (rows + 31) / 32 * ((g.N + 31) / 32);
  const long long few = narrow ? (1LL << 62) : 4 * n_cu;
  if (small <= few || g.nrows) {
    const dim3 grid((unsigned)(small < 4 * n_cu ? small : 4 * n_cu));
    if (g.a.d >= 8) hipLaunchKernelGGL((few_rows_kernel<E, kDz, kColsB, true>), grid, dim3(kThreads), 0, s, g, few);
    else hipLaunchKernelGGL((few_rows_kernel<E, kDz, kColsB, false>), grid, dim3(kThreads), 0, s, g, few);
  }
  if (small <= few) return hipGetLastError();
  // Eight waves where every CU gets a few of their tiles (2000003 x 768 -> 256 in bf16 1.24 ms, by four waves 1.33; 16384 x 256
  // -> 256 18.1 us, by four 14.6); of four waves, tiles of half the rows where those would not fill the CUs (16384 x 256 -> 256
  // in bf16 14.7 and 10.6 us; 9000 x 512 -> 256 in fp32 43 and 35; beyond, 60000 x 256 -> 128 in fp32 35 and 43).
  auto tiles = [&](int m, int n) { return (rows + m - 1) / m * ((g.N + n - 1) / n); };
  typedef ProductShape<E, 8, false> Wide;
  typedef ProductShape<E, 4, false> Tall;
  if (eight_waves(g.N) && tiles(Wide::kTileM, Wide::kTileN) >= 4 * n_cu) return product_tiles<E, kDz, kColsB, 8, false>(g, rows, n_cu, few, s);
  return tiles(Tall::kTileM, Tall::kTileN) > (E::kPieces > 1 ? n_cu : 2 * n_cu) ? product_tiles<E, kDz, kColsB, 4, false>(g, rows, n_cu, few, s)
                                                                             : product_tiles<E, kDz, kColsB, 4, true>(g, rows, n_cu, few, s);
}

template <class E>
hipError_t dense(const DenseArgs& a, hipStream_t s) {
  ProductArgs g{};
  const int K = a.nseg * a.d;
  for (int i = 0; i < a.nseg; ++i) g.a.p[i] = static_cast<const char*>(a.X[i]);
  g.a.ld = a.ldx;
  g.a.rows = a.rows;
  g.a.cols = K;
  g.a.d = a.d;
  g.b.p[0] = static_cast<const char*>(a.W);
  g.b.ld = a.ldw;
  g.b.rows = K;
  g.b.cols = g.b.d = a.N;
  g.nrows = a.nrows;
  g.K = K;
  g.N = a.N;
  g.act = a.act;
  g.bias = a.bias;
  g.R = static_cast<const char*>(a.R);
  g.ldr = a.ldr;
  g.Z = static_cast<char*>(a.Z);
  g.ldz = a.ldz;
  g.Y = static_cast<char*>(a.Y);
  g.ldy = a.ldy;
  g.stop = a.stop;
  return product<E, false, true>(g, a.rows, a.n_cu, s);
}

template <class E, class EX, bool kDz, int kWaves>
hipError_t weight_tiles(const WeightArgs& w, hipStream_t s) {
  typedef WeightShape<EX, E, kWaves> Shape;
  const int ntile = (w.M > 0 ? (w.M + Shape::kTileM - 1) / Shape::kTileM : 1) * ((w.N + Shape::kTileN - 1) / Shape::kTileN);
  auto kernel = weight_kernel<EX, E, kDz, kWaves>;
  const hipError_t e = allow_lds(kernel, Shape::kLds * 16);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(ntile * w.S), dim3(64 * kWaves), Shape::kLds * 16, s, w);
  return hipGetLastError();
}
template <class E, class EX, bool kDz>
hipError_t weight(const WeightArgs& w, const DenseBackArgs& a, float* db, hipStream_t s) {
  hipError_t e;
  if constexpr (kDz && E::kPieces == 1) e = weight_tiles<E, EX, kDz, 4>(w, s);
  else e = eight_weight_waves(w.N, E::kBytes == 2, kDz && E::kPieces != 2) ? weight_tiles<E, EX, kDz, 8>(w, s) : weight_tiles<E, EX, kDz, 4>(w, s);
  if (e != hipSuccess) return e;
  const long long total = (long long)w.M * w.N + w.N, most = (long long)a.n_cu * 8, want = (total + 255) / 256;
  hipLaunchKernelGGL((weight_reduce_kernel<EX, E, kDz>), dim3((unsigned)(want < most ? want : most)), dim3(256), 0, s, w,
                     static_cast<char*>(a.dW), a.lddw, db);
  return hipGetLastError();
}

template <class E, bool kDz>
hipError_t dense_back(const DenseBackArgs& a, hipStream_t s) {
  const int K = a.K;
  constexpr int kWide = 16 / E::kBytes;
  Source dz{};
  dz.p[0] = static_cast<const char*>(a.dY);
  dz.z = static_cast<const char*>(a.Z);
  dz.ld = a.lddy;
  dz.ldz = a.ldz;
  dz.rows = a.rows;
  dz.cols = dz.d = a.N;
  float* workspace = a.workspace;
  float* db = a.db;
  if (smooth(a.act)) {
    char* out = reinterpret_cast<char*>(workspace);
    workspace += dense_dz_floats(a.rows, a.N);
    SlopeArgs g{a.rows, a.N, a.act, dz.p[0], a.lddy, dz.z, a.ldz, out, a.bf16 && !a.round_dz, a.db ? workspace : nullptr, slope_blocks(a.rows, a.n_cu)};
    workspace += (size_t)g.row_blocks * a.N;
    const bool wide = a.N % kWide == 0;
    const int columns = 32 * (wide ? kWide : 1), cb = (a.N + columns - 1) / columns;
    if (wide) hipLaunchKernelGGL((slope_kernel<E, kWide>), dim3(cb * g.row_blocks), dim3(256), 0, s, g);
    else hipLaunchKernelGGL((slope_kernel<E, 1>), dim3(cb * g.row_blocks), dim3(256), 0, s, g);
    if (a.db) launch_column_sums(g.part, g.row_blocks, a.N, a.db, 0, nullptr, nullptr, s);
    db = nullptr;
    dz.p[0] = out;
    dz.z = nullptr;
    dz.ld = a.N;
    if (g.pair) dz.p[1] = out + a.rows * a.N * 2;
  }
  hipError_t e = hipSuccess;
  if (a.dX && a.rows > 0) {
    ProductArgs g{};
    g.a = dz;
    g.b.p[0] = static_cast<const char*>(a.W);
    g.b.ld = a.ldw;
    g.b.rows = K;
    g.b.cols = g.b.d = a.N;
    g.K = dz.p[1] ? 2 * a.N : a.N;
    g.N = K;
    g.act = DC_ACT_NONE;
    g.Y = static_cast<char*>(a.dX);
    g.ldy = a.lddx;
    e = product<E, kDz, false>(g, a.rows, a.n_cu, s);
  }
  if (e == hipSuccess && (a.dW || db)) {
    WeightArgs w{};
    w.a.rows = a.rows;
    w.M = a.dW ? K : 0;
    w.a.cols = w.a.d = K;
    if (a.kept.code) {
      w.a.p[0] = reinterpret_cast<const char*>(a.kept.code);
      w.a.exponent = a.kept.exponent;
      w.a.ld = a.kept.ld_code;
      w.a.ld_exponent = a.kept.ld_exponent;
    } else {
      w.a.p[0] = static_cast<const char*>(a.X);
      w.a.ld = a.ldx;
    }
    w.b = dz;
    w.N = a.N;
    w.S = slabs_of(a.rows, K, a.N, a.bf16, a.act, a.n_cu);
    w.part = workspace;
    w.sums = db != nullptr;
    if constexpr (E::kBytes == 2 && !kDz) {
      if (dz.p[1]) {
        w.b.z = dz.p[1];
        w.b.ldz = a.N;
        return a.kept.code ? weight<Bf16Pair, Kept, true>(w, a, db, s) : weight<Bf16Pair, E, true>(w, a, db, s);
      }
    }
    e = a.kept.code ? weight<E, Kept, kDz>(w, a, db, s) : weight<E, E, kDz>(w, a, db, s);
  }
  return e;
}

}  // namespace

hipError_t launch_dense(const DenseArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  return a.bf16 ? dense<Bf16>(a, s) : dense<F32>(a, s);
}

size_t dense_dz_floats(long long rows, int N) {
  return ((size_t)rows * N * 4 + 15) / 16 * 4;
}
size_t dense_back_floats(long long rows, int K, int N, int bf16, int act, int n_cu) {
  size_t n = (size_t)slabs_of(rows, K, N, bf16, act, n_cu) * ((size_t)K * N + N);
  if (smooth(act)) n += dense_dz_floats(rows, N) + (size_t)slope_blocks(rows, n_cu) * N;
  return n;
}

hipError_t launch_dense_back(const DenseBackArgs& a, hipStream_t s) {
  if (a.act == DC_ACT_RELU) return a.bf16 ? dense_back<Bf16, true>(a, s) : dense_back<F32, true>(a, s);
  return a.bf16 ? dense_back<Bf16, false>(a, s) : dense_back<F32, false>(a, s);
}

}  // namespace dc
