// Dense layer on the rows of a batch, Y = act(X W + b) + R, and its gradients (gfx950).
//
//   forward   Z = X W + b, Y = act(Z) + R                                   contraction over the columns of X
//   data      dX = dZ W^T, dZ = dY act'(Z) formed as the rows are loaded    contraction over the columns of dY
//   weights   dW = X^T dZ, db = column sums of dZ                           contraction over the rows, split into slabs
//
// All three are tiles of 128 x 128 on the bf16 matrix cores (32 x 32 x 16), operands staged through LDS in the layout
// that the instruction reads: units of eight consecutive contraction indices (16 bytes).
// fp32: a number is the sum of three bf16 numbers; the six products of pieces with i + j <= 4 are formed (what is left
// out is below 2^-25 of |x w|), sums of 64 indices go to a total of their own, and every other one is formed negated, so
// that what the matrix cores drop below an accumulator's 24 bits (always downwards) cancels.  Kept rows are one exact
// piece: three products instead of six.  Sums that come out not finite in pieces are formed again in fp32.
// bf16: dZ is rounded to bf16 as an operand (by at most 2^-8 of its size, as dX and dW are rounded by
// themselves); db is summed from dZ before that rounding, in 64 bits.
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

// An operand as it lies in memory: `rows` x `cols`, up to three matrices of d columns side by side; with z the values
// are p * act'(z).
struct Source {
  const char* p[3];
  const char* z;
  const unsigned char* exponent;
  long long ld, ldz, ld_exponent;
  long long rows;
  int cols, d, act;
};

// kN consecutive columns of one row, as they come from memory
template <class E, int kN, bool kDz>
struct Raw {
  static constexpr int kWords = (kN * E::kBytes + 3) / 4;
  unsigned w[kWords];
  unsigned z[kDz ? kWords : 1];
  unsigned e;
};

template <int kBytes>
__device__ __forceinline__ void read_words(unsigned* w, const char* p) {
  if constexpr (kBytes == 1) w[0] = *reinterpret_cast<const unsigned char*>(p);
  else if constexpr (kBytes == 2) w[0] = *reinterpret_cast<const u16*>(p);
  else if constexpr (kBytes == 4) w[0] = *reinterpret_cast<const unsigned*>(p);
  else if constexpr (kBytes == 8) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    w[0] = v.x;
    w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i) {
      const u32x4 v = reinterpret_cast<const u32x4*>(p)[i];
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
template <class E, bool kDz>
__device__ __forceinline__ float single(const Source& s, long long row, int col) {
  const int seg = col / s.d;
  unsigned w[1], z[1];
  read_words<E::kBytes>(w, s.p[seg] + (row * s.ld + col - seg * s.d) * E::kBytes);
  float scale = 1.f;
  if constexpr (E::kBytes == 1) scale = kept_scale(s.exponent[row * s.ld_exponent + col / kKeptBlock]);
  float x = value_of<E>(w, 0, scale);
  if constexpr (kDz) {
    read_words<E::kBytes>(z, s.z + (row * s.ldz + col) * E::kBytes);
    x *= activation_slope(value_of<E>(z, 0, 1.f), s.act);
  }
  return x;
}
// kVec: rows start at, and have a multiple of, whole vectors, and the vector lies inside the matrix; else value by value,
// zeros behind the last column.
template <class E, int kN, bool kDz, bool kVec>
__device__ __forceinline__ void fetch(Raw<E, kN, kDz>& r, const Source& s, long long row, int col) {
  if constexpr (kVec) {
    const int seg = (col >= s.d ? 1 : 0) + (col >= 2 * s.d ? 1 : 0);
    const char* p = seg == 0 ? s.p[0] : (seg == 1 ? s.p[1] : s.p[2]);
    read_words<kN * E::kBytes>(r.w, p + (row * s.ld + col - seg * s.d) * E::kBytes);
    if constexpr (kDz) read_words<kN * E::kBytes>(r.z, s.z + (row * s.ldz + col) * E::kBytes);
    if constexpr (E::kBytes == 1) r.e = s.exponent[row * s.ld_exponent + col / kKeptBlock];
  } else {
#pragma unroll
    for (int i = 0; i < Raw<E, kN, kDz>::kWords; ++i) {
      r.w[i] = 0;
      if constexpr (kDz) r.z[i] = 0;
    }
    r.e = 0;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      const int c = col + k;
      if (c >= s.cols) continue;
      const int seg = (c >= s.d ? 1 : 0) + (c >= 2 * s.d ? 1 : 0);
      const char* p = seg == 0 ? s.p[0] : (seg == 1 ? s.p[1] : s.p[2]);
      unsigned x[1];
      constexpr int kPer = 4 / E::kBytes;
      read_words<E::kBytes>(x, p + (row * s.ld + c - seg * s.d) * E::kBytes);
      r.w[k / kPer] |= x[0] << (8 * E::kBytes * (k % kPer) % 32);
      if constexpr (kDz) {
        read_words<E::kBytes>(x, s.z + (row * s.ldz + c) * E::kBytes);
        r.z[k / kPer] |= x[0] << (8 * E::kBytes * (k % kPer) % 32);
      }
      if constexpr (E::kBytes == 1) r.e = s.exponent[row * s.ld_exponent + c / kKeptBlock];
    }
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
template <class E, int kN, bool kDz>
__device__ __forceinline__ void values(float (&x)[kN], const Raw<E, kN, kDz>& r, int act) {
  float scale = 1.f;
  if constexpr (E::kBytes == 1) scale = kept_scale(r.e);
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    x[k] = value_of<E>(r.w, k, scale);
    if constexpr (kDz) x[k] *= activation_slope(value_of<E>(r.z, k, 1.f), act);
  }
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

constexpr int kTile = 128, kThreads = 256;

// A tile of kTile rows (of the product's operand) by KS contraction indices, from memory through registers to LDS.
// kCols = false: the operand's rows are the rows of the matrix; true: its columns, and the contraction runs over the rows.
template <class E, bool kCols, bool kDz, int KS, bool kVec>
struct Stager {
  static constexpr int kP = E::kPieces;
  static constexpr int kUnits = kTile * KS / 8 / kThreads;      // per thread: 4 or 2
  static constexpr int kN = kCols ? kUnits : 8;                 // columns per vector
  static constexpr int kRaws = kCols ? 8 : kUnits;
  Raw<E, kN, kDz> raw[kRaws];

  // r0: first row of the tile; k0 .. k_end: contraction indices
  __device__ __forceinline__ void load(const Source& s, long long r0, long long k0, long long k_end) {
    const int t = threadIdx.x;
    if constexpr (kCols) {
      constexpr int kBlocks = kTile / kN;
      const int c = t / kBlocks;
      int col = (int)r0 + (t % kBlocks) * kN;
      if constexpr (kVec) col = min(col, s.cols - kN);          // columns behind the last are not stored
      const long long k = k0 + c * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (k + i < k_end) fetch<E, kN, kDz, kVec>(raw[i], s, k + i, col);
        else clear(raw[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int u = t + kThreads * i, r = u / (KS / 8), c = u % (KS / 8);
        long long row = r0 + r;
        if (row >= s.rows) row = s.rows - 1;                    // rows behind the last are not stored
        const int k = (int)k0 + c * 8;
        if (k < k_end) fetch<E, kN, kDz, kVec>(raw[i], s, row, k);
        else clear(raw[i]);
      }
    }
  }
  // sums: column sums of the values (kCols), or null
  __device__ __forceinline__ void store(u32x4* lds, int act, float sign, double* sums) const {
    const int t = threadIdx.x;
    if constexpr (kCols) {
      constexpr int kBlocks = kTile / kN;
      const int c = t / kBlocks, r = (t % kBlocks) * kN;
      float x[8][kN];
#pragma unroll
      for (int i = 0; i < 8; ++i) values<E, kN, kDz>(x[i], raw[i], act);
      if (sums) {
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          double v = 0.0;
#pragma unroll
          for (int i = 0; i < 8; ++i) v += (double)x[i][j];
          sums[j] += v;
        }
      }
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = kP == 1 ? x[i][j] : x[i][j] * sign;
        u32x4 p[kP];
        pieces_of<kP>(p, y);
#pragma unroll
        for (int q = 0; q < kP; ++q) lds[q * kTile * KS / 8 + unit_at<KS>(r + j, c)] = p[q];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int u = t + kThreads * i, r = u / (KS / 8), c = u % (KS / 8);
        u32x4 p[kP];
        if constexpr (E::kBytes == 2 && !kDz) {
          p[0] = u32x4{raw[i].w[0], raw[i].w[1], raw[i].w[2], raw[i].w[3]};
        } else {
          float x[8];
          values<E, kN, kDz>(x, raw[i], act);
          if constexpr (kP > 1)
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= sign;
          pieces_of<kP>(p, x);
        }
#pragma unroll
        for (int q = 0; q < kP; ++q) lds[q * kTile * KS / 8 + unit_at<KS>(r, c)] = p[q];
      }
    }
  }
};

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.f;
  return z;
}

// One staged step: acc[i][j] += A (rows 64 wm + 32 i ..) times B (rows 64 wn + 32 j ..).  The small products first.
template <int kPA, int kPB, int KS>
__device__ __forceinline__ void multiply(f32x16 (&acc)[2][2], const u32x4* A, const u32x4* B, int wm, int wn) {
  constexpr int kMost = kPA > kPB ? kPA : kPB, kPlane = kTile * KS / 8;
  const int lane = threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5;
#pragma unroll
  for (int k = 0; k < KS / 16; ++k) {
    u32x4 a[kPA][2], b[kPB][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int p = 0; p < kPA; ++p) a[p][i] = A[p * kPlane + unit_at<KS>(wm * 64 + i * 32 + l32, 2 * k + lh)];
#pragma unroll
      for (int p = 0; p < kPB; ++p) b[p][i] = B[p * kPlane + unit_at<KS>(wn * 64 + i * 32 + l32, 2 * k + lh)];
    }
#pragma unroll
    for (int sum = kMost - 1; sum >= 0; --sum)
#pragma unroll
      for (int p = 0; p < kPA; ++p) {
        const int q = sum - p;
        if (q < 0 || q >= kPB) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b[q][j]),
                                                                __builtin_bit_cast(bf16x8, a[p][i]), acc[i][j], 0, 0, 0);
      }
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

// rows x N outputs, contraction over K columns of a
template <class E, bool kDz, bool kColsB, bool kVec>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(ProductArgs g) {
  if (g.stop && g.stop[0] != 0) return;
  constexpr int kP = E::kPieces, KS = kP == 1 ? 64 : 32;
  __shared__ u32x4 A[kP * kTile * KS / 8], B[kP * kTile * KS / 8];
  if (g.nrows) g.a.rows = g.nrows[0];
  const long long rows = g.a.rows;
  const int wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, lane = threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5;
  const int nct = (g.N + kTile - 1) / kTile, steps = (g.K + KS - 1) / KS;
  const TileRange tr = tiles_of((rows + kTile - 1) / kTile * nct);
  for (long long tile = tr.first; tile < tr.end; tile += tr.step) {
    const long long m0 = tile / nct * kTile;
    const int n0 = (int)(tile % nct) * kTile;
    f32x16 acc[2][2], total[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = total[i][j] = zero16();
    Stager<E, false, kDz, KS, kVec> sa;
    Stager<E, kColsB, false, KS, kVec> sb;
    sa.load(g.a, m0, 0, g.K);
    sb.load(g.b, n0, 0, g.K);
    for (int step = 0; step < steps; ++step) {
      const float sign = (step >> 1) & 1 ? -1.f : 1.f;
      __syncthreads();
      sa.store(A, g.a.act, 1.f, nullptr);
      sb.store(B, 0, sign, nullptr);
      __syncthreads();
      if (step + 1 < steps) {
        sa.load(g.a, m0, (step + 1) * KS, g.K);
        sb.load(g.b, n0, (step + 1) * KS, g.K);
      }
      multiply<kP, kP, KS>(acc, A, B, wm, wn);
      if (kP > 1 && ((step & 1) || step + 1 == steps)) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              total[i][j][v] = fmaf(acc[i][j][v], sign, total[i][j][v]);
              acc[i][j][v] = 0.f;
            }
      }
    }
    // register v of a lane: row l32, column 8 (v / 4) + 4 lh + v % 4 of the block
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const long long row = m0 + wm * 64 + i * 32 + l32;
      if (row >= rows) continue;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int col = n0 + wn * 64 + j * 32 + 8 * (v / 4) + 4 * lh + v % 4;
          if (col >= g.N) continue;
          float z = kP > 1 ? total[i][j][v] : acc[i][j][v];
          if (kP > 1 && !__builtin_isfinite(z)) {
            z = 0.f;
            for (int k = 0; k < g.K; ++k)
              z = fmaf(single<E, kDz>(g.a, row, k), kColsB ? single<E, false>(g.b, k, col) : single<E, false>(g.b, col, k), z);
          }
          if (g.bias) z += g.bias[col];
          if (g.Z) store_value<E>(g.Z, row * g.ldz + col, z);
          float y = activation(z, g.act);
          if (g.R) y += load_value<E>(g.R, row * g.ldr + col);
          store_value<E>(g.Y, row * g.ldy + col, y);
        }
    }
  }
}

// ---- weight gradients ----
struct WeightArgs {
  Source a;              // X  [rows, M]
  Source b;              // dZ [rows, N]
  const int* nrows;
  int M, N, S;
  float* part;           // [S][M * N + N]
  int sums;              // column sums of dZ are wanted
  const int* stop;
};

template <class EA, class EB, bool kDz, bool kVec>
__global__ __launch_bounds__(kThreads, 2) void weight_kernel(WeightArgs g) {
  if (g.stop && g.stop[0] != 0) return;
  constexpr int kPA = EA::kPieces, kPB = EB::kPieces, KS = kPA == 1 && kPB == 1 ? 64 : 32, kHold = 256 / KS;
  constexpr int kN = kTile * KS / 8 / kThreads;
  __shared__ u32x4 A[kPA * kTile * KS / 8], B[kPB * kTile * KS / 8];
  const long long rows = g.nrows ? g.nrows[0] : g.a.rows;
  const int wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, lane = threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5;
  const int tiles_n = (g.N + kTile - 1) / kTile, tiles_m = max(1, (g.M + kTile - 1) / kTile), ntile = tiles_m * tiles_n;
  // the tiles of a slab read the same rows: they run on one XCD (the grid is ntile * S, S a multiple of eight)
  const int item = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  const int tile = item % ntile, slab = item / ntile;
  const int m0 = tile / tiles_n * kTile, n0 = tile % tiles_n * kTile;
  long long per = (rows + g.S - 1) / g.S;
  per = (per + KS - 1) / KS * KS;
  const long long r0 = min((long long)slab * per, rows), r1 = min(r0 + per, rows);
  const int steps = (int)((r1 - r0 + KS - 1) / KS);
  f32x16 acc[2][2], total[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = total[i][j] = zero16();
  const bool want_sums = g.sums && m0 == 0;
  double sums[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) sums[j] = 0.0;
  Stager<EA, true, false, KS, kVec> sa;
  Stager<EB, true, kDz, KS, kVec> sb;
  if (steps > 0) {
    if (g.M > 0) sa.load(g.a, m0, r0, r1);
    sb.load(g.b, n0, r0, r1);
  }
  for (int step = 0; step < steps; ++step) {
    // sections of kHold steps; every other slab begins with the negated sign
    const float sign = ((step / kHold) ^ slab) & 1 ? -1.f : 1.f;
    __syncthreads();
    if (g.M > 0) sa.store(A, 0, 1.f, nullptr);
    sb.store(B, g.b.act, sign, want_sums ? sums : nullptr);
    __syncthreads();
    if (step + 1 < steps) {
      if (g.M > 0) sa.load(g.a, m0, r0 + (long long)(step + 1) * KS, r1);
      sb.load(g.b, n0, r0 + (long long)(step + 1) * KS, r1);
    }
    if (g.M > 0) multiply<kPA, kPB, KS>(acc, A, B, wm, wn);
    if (step % kHold == kHold - 1 || step + 1 == steps) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            total[i][j][v] = fmaf(acc[i][j][v], kPB > 1 ? sign : 1.f, total[i][j][v]);
            acc[i][j][v] = 0.f;
          }
    }
  }
  float* P = g.part + (size_t)slab * ((size_t)g.M * g.N + g.N);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int m = m0 + wm * 64 + i * 32 + l32;
    if (m >= g.M) continue;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int n = n0 + wn * 64 + j * 32 + 8 * (v / 4) + 4 * lh + v % 4;
        if (n >= g.N) continue;
        float z = total[i][j][v];
        if (kPB > 1 && !__builtin_isfinite(z)) {
          z = 0.f;
          for (long long r = r0; r < r1; ++r) z = fmaf(single<EA, false>(g.a, r, m), single<EB, kDz>(g.b, r, n), z);
        }
        P[(size_t)m * g.N + n] = z;
      }
  }
  if (want_sums) {                                   // the same for the whole workgroup
    __shared__ double red[KS / 8][kTile];
    constexpr int kBlocks = kTile / kN;
#pragma unroll
    for (int j = 0; j < kN; ++j) red[threadIdx.x / kBlocks][threadIdx.x % kBlocks * kN + j] = sums[j];
    __syncthreads();
    const int n = n0 + (int)threadIdx.x;
    if (threadIdx.x < kTile && n < g.N) {
      double v = 0.0;
#pragma unroll
      for (int c = 0; c < KS / 8; ++c) v += red[c][threadIdx.x];
      P[(size_t)g.M * g.N + n] = (float)v;
    }
  }
}

// dW [M, N] and db [N] = sums of the slabs' parts in 64 bits, ascending slabs.
template <class E>
__global__ __launch_bounds__(256) void weight_reduce_kernel(const float* __restrict__ part, int S, long long MN, int N, char* dW,
                                                            long long lddw, float* __restrict__ db, const int* stop) {
  if (stop && stop[0] != 0) return;
  const long long stride = MN + N;
  const long long first = dW ? 0 : MN, end = db ? stride : MN;
  for (long long i = first + (long long)blockIdx.x * blockDim.x + threadIdx.x; i < end; i += (long long)gridDim.x * blockDim.x) {
    double s = 0.0;
    const float* __restrict__ p = part + i;
    for (int k = 0; k < S; k += 8, p += 8 * stride) {        // S is a multiple of eight; eight requested together
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = p[u * stride];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += (double)x[u];
    }
    if (i < MN) store_value<E>(dW, i / N * lddw + i % N, (float)s);
    else db[i - MN] = (float)s;
  }
}

// The slabs of a weight gradient: one round of workgroups at two per CU, and at least 256 rows each.
int slabs_of(long long rows, int K, int N, int n_cu) {
  const int ntile = ((K + kTile - 1) / kTile) * ((N + kTile - 1) / kTile);
  long long S = 2 * n_cu / (ntile < 1 ? 1 : ntile), by_rows = (rows + 255) / 256;
  if (S > by_rows) S = by_rows;
  S = (S + 7) / 8 * 8;
  return S < 8 ? 8 : (int)S;
}

bool whole(const void* p, long long ld, int cols, int bytes, int n) {       // vectors of n values
  return cols % n == 0 && ld % n == 0 && reinterpret_cast<size_t>(p) % ((size_t)n * bytes) == 0;
}
unsigned grid_of(long long tiles, int n_cu) {
  const long long most = (long long)n_cu * 2;
  long long g = tiles < most ? tiles : most;
  return (unsigned)((g + 7) / 8 * 8);
}
long long tiles_count(long long rows, int N) { return (rows + kTile - 1) / kTile * ((N + kTile - 1) / kTile); }

template <class E>
hipError_t dense(const DenseArgs& a, hipStream_t s) {
  ProductArgs g{};
  const int K = a.nseg * a.d;
  bool vec = whole(a.W, a.ldw, a.N, E::kBytes, 4) && K % 8 == 0 && a.d % 8 == 0;
  for (int i = 0; i < a.nseg; ++i) {
    g.a.p[i] = static_cast<const char*>(a.X[i]);
    vec = vec && whole(a.X[i], a.ldx, a.d, E::kBytes, 16 / E::kBytes);
  }
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
  const dim3 grid(grid_of(tiles_count(a.rows, a.N), a.n_cu));
  if (vec) hipLaunchKernelGGL((product_kernel<E, false, true, true>), grid, dim3(kThreads), 0, s, g);
  else hipLaunchKernelGGL((product_kernel<E, false, true, false>), grid, dim3(kThreads), 0, s, g);
  return hipGetLastError();
}

template <class E, class EX, bool kDz, bool kVec>
void weight_launch(const WeightArgs& w, hipStream_t s) {
  const int ntile = (w.M > 0 ? (w.M + kTile - 1) / kTile : 1) * ((w.N + kTile - 1) / kTile);
  hipLaunchKernelGGL((weight_kernel<EX, E, kDz, kVec>), dim3(ntile * w.S), dim3(kThreads), 0, s, w);
}

template <class E, bool kDz>
hipError_t dense_back(const DenseBackArgs& a, hipStream_t s) {
  const int K = a.nseg * a.d;
  Source dz{};
  dz.p[0] = static_cast<const char*>(a.dY);
  dz.z = static_cast<const char*>(a.Z);
  dz.ld = a.lddy;
  dz.ldz = a.ldz;
  dz.rows = a.rows;
  dz.cols = dz.d = a.N;
  dz.act = a.act;
  constexpr int kWide = 16 / E::kBytes;
  const bool dz_vec = whole(a.dY, a.lddy, a.N, E::kBytes, kWide) && (!kDz || whole(a.Z, a.ldz, a.N, E::kBytes, kWide));
  if (a.dX && a.rows > 0) {
    ProductArgs g{};
    g.a = dz;
    g.b.p[0] = static_cast<const char*>(a.W);
    g.b.ld = a.ldw;
    g.b.rows = K;
    g.b.cols = g.b.d = a.N;
    g.nrows = a.nrows;
    g.K = a.N;
    g.N = K;
    g.act = DC_ACT_NONE;
    g.Y = static_cast<char*>(a.dX);
    g.ldy = a.lddx;
    g.stop = a.stop;
    const dim3 grid(grid_of(tiles_count(a.rows, K), a.n_cu));
    if (dz_vec && a.N % 8 == 0 && whole(a.W, a.ldw, a.N, E::kBytes, kWide))
      hipLaunchKernelGGL((product_kernel<E, kDz, false, true>), grid, dim3(kThreads), 0, s, g);
    else
      hipLaunchKernelGGL((product_kernel<E, kDz, false, false>), grid, dim3(kThreads), 0, s, g);
  }
  if (a.dW || a.db) {
    WeightArgs w{};
    w.a.rows = a.rows;
    w.M = a.dW ? K : 0;
    w.a.cols = K;
    w.a.d = a.d;
    bool vec = dz_vec;
    if (a.kept.code) {
      w.a.p[0] = reinterpret_cast<const char*>(a.kept.code);
      w.a.exponent = a.kept.exponent;
      w.a.ld = a.kept.ld_code;
      w.a.ld_exponent = a.kept.ld_exponent;
      vec = vec && whole(a.kept.code, a.kept.ld_code, K, 1, 4);
    } else {
      for (int i = 0; i < a.nseg; ++i) {
        w.a.p[i] = static_cast<const char*>(a.X[i]);
        if (w.M) vec = vec && whole(a.X[i], a.ldx, a.d, E::kBytes, 4);
      }
      w.a.ld = a.ldx;
    }
    w.b = dz;
    w.nrows = a.nrows;
    w.N = a.N;
    w.S = slabs_of(a.rows, K, a.N, a.n_cu);
    w.part = a.workspace;
    w.sums = a.db != nullptr;
    w.stop = a.stop;
    if (a.kept.code) {
      if (vec) weight_launch<E, Kept, kDz, true>(w, s);
      else weight_launch<E, Kept, kDz, false>(w, s);
    } else {
      if (vec) weight_launch<E, E, kDz, true>(w, s);
      else weight_launch<E, E, kDz, false>(w, s);
    }
    const long long MN = (long long)w.M * a.N, total = MN + a.N;
    const long long most = (long long)a.n_cu * 8, want = (total + 255) / 256;
    hipLaunchKernelGGL((weight_reduce_kernel<E>), dim3((unsigned)(want < most ? want : most)), dim3(256), 0, s, w.part, w.S, MN,
                       a.N, static_cast<char*>(a.dW), a.lddw, a.db, a.stop);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dense(const DenseArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  return a.bf16 ? dense<Bf16>(a, s) : dense<F32>(a, s);
}

size_t dense_back_floats(long long rows, int K, int N, int n_cu) {
  return (size_t)slabs_of(rows, K, N, n_cu) * ((size_t)K * N + N);
}

hipError_t launch_dense_back(const DenseBackArgs& a, hipStream_t s) {
  if (a.act == DC_ACT_NONE) return a.bf16 ? dense_back<Bf16, false>(a, s) : dense_back<F32, false>(a, s);
  return a.bf16 ? dense_back<Bf16, true>(a, s) : dense_back<F32, true>(a, s);
}

}  // namespace dc
