// Norm over the channels of each row with an activation, and its gradient (gfx950):
//
//   forward   mu = mean x, v = mean (x - mu)^2, r = 1 / sqrt(v + eps);  y = act(gamma (x - mu) r + beta)
//   backward  xh = (x - mu) r, dz = dy act'(gamma xh + beta), u = gamma dz, s1 = mean u, s2 = mean u xh;
//             dx = r (u - s1 - xh s2) [+ dres];  dgamma = sum over rows of dz xh, dbeta = sum of dz
//
// Bound by memory: a row is read once and stays in registers, eight or sixteen values a thread.  Rows of up to 512 channels take a
// power of two of a wave's lanes, several rows a wave, wider rows a workgroup.  The forward pass is one launch of as many
// workgroups as there are rows for, two rows a seat: they are handed out in the order of the addresses, and a copy of that kind
// gets 6.1 TB/s where one by resident workgroups that go on in strides gets 4.7.  (5.7 M rows of 256 in bf16 with SiLU, 5.8 GB:
// 982 us, 6.0 TB/s; by resident workgroups that request a row ahead a fifth more.)  The gradients keep to what is resident, since
// each workgroup hands on sums of 2 C numbers (2 M rows of 256 in bf16 with GELU and dres, 4.1 GB: 770 us, 5.3 TB/s; 474011 rows of
// 256 in fp32, x in 8 bits: 1.1 GB, 197 us, 5.6 TB/s).
// The variance is that of d = x - m, m the row's sum over C as fp32 has it: mean d is what m lacks, v = mean d^2 - (mean d)^2.
// So neither loses digits for values far from zero, and mu is m + mean d, rounded once where it is returned.  The gradients go by that
// rounded mu: their xh is off by up to 2^-24 |mu| r, the same for a whole row.
// Gradients of gamma and beta: 64 rows of a thread in fp32, these sums in fp32 again, a workgroup's rows and the workgroups
// in 64 bits and a fixed order.
#include <type_traits>

#include "row_vectors.h"

namespace dc {
namespace {

struct Kept8 {};               // x as codes

constexpr int kNarrow = 512;   // channels that a wave's lanes hold
constexpr int kRun = 64;       // rows whose terms are summed in fp32 before they join the others'
constexpr int kMostWaves = 16;

// How a thread's vectors lie in a row, vector j of kVector values at columns (j * lanes + t) * kVector:
//   kWhole  the row is all of them;
//   kBack   the row ends before the last: the vector that would reach beyond it ends with the row instead, and its first
//           `skip` values are its neighbour's, which it may write, being the same, but not count;
//   kShort  the row is shorter than one vector.
enum Fit { kWhole, kBack, kShort };
template <typename T, int NV>
struct Columns {
  int at[NV], skip[NV];        // skip: kVector<T> of a vector with no value of its own
};
template <typename T, int NV, Fit kFit>
__device__ __forceinline__ Columns<T, NV> columns_of(int t, int lanes, int C) {
  constexpr int kV = kVector<T>;
  Columns<T, NV> q;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * lanes + t) * kV;
    q.at[j] = kFit == kWhole ? c : max(min(c, C - kV), 0);
    q.skip[j] = kFit == kWhole ? 0 : min(c - q.at[j], kV);
  }
  return q;
}
// Whether value k of vector j is the thread's own.
template <typename T, int NV, Fit kFit>
__device__ __forceinline__ bool own(const Columns<T, NV>& q, int j, int k, int C) {
  return kFit == kWhole || (k >= q.skip[j] && (kFit == kBack || k < C));
}

template <typename T, typename X, int NV>
struct Fetched {
  u32x4 v[NV];
};
template <int NV>
struct Fetched<u16, Kept8, NV> {
  u32x2 v[NV];
  unsigned e[NV], e2[NV];      // exponents of its first and of its last value
};
template <int NV>
struct Fetched<float, Kept8, NV> {
  unsigned v[NV];
  unsigned e[NV], e2[NV];
};
// 16, 8 and 4 bytes from anywhere.  kOnce: as not used again soon.
template <bool kOnce>
__device__ __forceinline__ u32x4 read16(const void* p) {
  if constexpr (kOnce) return __builtin_nontemporal_load(static_cast<const u32x4_any*>(p));
  else return *static_cast<const u32x4_any*>(p);
}
template <bool kOnce>
__device__ __forceinline__ u32x2 read8(const void* p) {
  if constexpr (kOnce) return __builtin_nontemporal_load(static_cast<const u32x2_any*>(p));
  else return *static_cast<const u32x2_any*>(p);
}
template <bool kOnce>
__device__ __forceinline__ unsigned read4(const void* p) {
  if constexpr (kOnce) return __builtin_nontemporal_load(static_cast<const u32_any*>(p));
  else return *static_cast<const u32_any*>(p);
}
// `row` elements from p on: p is the same for the wave, so that only 32 bits are the lane's own.
template <bool kOnce, typename T, int NV, Fit kFit>
__device__ __forceinline__ void fetch(Fetched<T, T, NV>& f, const T* p, unsigned row, const Columns<T, NV>& q, int C) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (kFit == kShort) f.v[j] = load_vector<T, false>(p + row, q.at[j], C);
    else f.v[j] = read16<kOnce>(p + (row + (unsigned)q.at[j]));
  }
}
// A row of codes goes up to a multiple of 32, so a short one has a whole vector too.
template <bool kOnce, typename T, int NV, Fit kFit>
__device__ __forceinline__ void fetch(Fetched<T, Kept8, NV>& f, const signed char* p, unsigned row, const unsigned char* e, unsigned row_e, const Columns<T, NV>& q) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const unsigned at = q.at[j];
    if constexpr (sizeof(T) == 2) f.v[j] = read8<kOnce>(p + (row + at));
    else f.v[j] = read4<kOnce>(p + (row + at));
    f.e[j] = e[row_e + at / kKeptBlock];
    f.e2[j] = kFit == kBack ? e[row_e + (at + kVector<T> - 1) / kKeptBlock] : 0;
  }
}
template <typename T, int NV, Fit kFit>
__device__ __forceinline__ void values(float (&x)[NV * kVector<T>], const Fetched<T, T, NV>& f, const Columns<T, NV>&) {
  constexpr int kV = kVector<T>;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float w[kV];
    unpack(w, f.v[j], T());
#pragma unroll
    for (int k = 0; k < kV; ++k) x[j * kV + k] = w[k];
  }
}
template <typename T, int NV, Fit kFit>
__device__ __forceinline__ void values(float (&x)[NV * kVector<T>], const Fetched<T, Kept8, NV>& f, const Columns<T, NV>& q) {
  constexpr int kV = kVector<T>;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const float s = kept_scale(f.e[j]), s2 = kFit == kBack ? kept_scale(f.e2[j]) : 0.f;
    const int turn = kFit == kBack ? kKeptBlock - q.at[j] % kKeptBlock : kV;     // its first value of the second block
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      unsigned w;
      if constexpr (kV == 8) w = f.v[j][k / 4];
      else w = f.v[j];
      x[j * kV + k] = (float)(signed char)(w >> (8 * (k & 3))) * (kFit == kBack && k >= turn ? s2 : s);
    }
  }
}

// gamma or beta at a vector's columns.
template <typename T, Fit kFit>
__device__ __forceinline__ void vector_at(float (&g)[kVector<T>], const float* v, float none, int at, int C) {
#pragma unroll
  for (int k = 0; k < kVector<T>; k += 4) {
    float w[4] = {none, none, none, none};
    if (v) unpack(w, load_vector<float, kFit != kShort>(v, at + k, C), 0.f);
#pragma unroll
    for (int u = 0; u < 4; ++u) g[k + u] = w[u];
  }
}
template <typename T, int NV, Fit kFit>
__device__ __forceinline__ void vectors_at(float (&g)[NV * kVector<T>], const float* v, float none, const Columns<T, NV>& q, int C) {
  constexpr int kV = kVector<T>;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float w[kV];
    vector_at<T, kFit>(w, v, none, q.at[j], C);
#pragma unroll
    for (int k = 0; k < kV; ++k) g[j * kV + k] = w[k];
  }
}
// kOwn: a vector that ends with the row writes only what is its own, so that its neighbour's may be read until then.
template <bool kOnce, typename T, int NV, Fit kFit, bool kOwn = false>
__device__ __forceinline__ void put(const float (&y)[NV * kVector<T>], T* p, unsigned row, const Columns<T, NV>& q, int C) {
  constexpr int kV = kVector<T>;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float w[kV];
#pragma unroll
    for (int k = 0; k < kV; ++k) w[k] = y[j * kV + k];
    if (kFit == kWhole || q.skip[j] < kV) {
      if constexpr (kFit == kShort) {
        store_vector<T>(p + row, q.at[j], C, pack(w, T()));
      } else if (kOwn && kFit == kBack && q.skip[j] > 0) {
#pragma unroll
        for (int k = 0; k < kV; ++k)
          if (k >= q.skip[j]) narrow(w[k], p[row + (unsigned)(q.at[j] + k)]);
      } else if constexpr (kOnce) {
        __builtin_nontemporal_store(pack(w, T()), reinterpret_cast<u32x4_any*>(p + (row + (unsigned)q.at[j])));
      } else {
        *reinterpret_cast<u32x4_any*>(p + (row + (unsigned)q.at[j])) = pack(w, T());
      }
    }
  }
}

// Threads of a row: kLanes of a wave (0: a number that is not known when the kernel is built), or the workgroup.
constexpr int kGroup = 128;
// Sums over a row's threads, in all of them.  kGroup: `red` has room for a number of each wave, and another row's sums may use it
// only after one more barrier.
template <int kLanes>
__device__ __forceinline__ float row_sum(float x, int lanes, float* red) {
  if constexpr (kLanes == kGroup) {
    x = lane_sum<64>(x);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
    for (int w = 0; w < (int)blockDim.x >> 6; ++w) x += red[w];
    return x;
  } else {
    return lane_sum<kLanes>(x, lanes);
  }
}
template <int kLanes>
__device__ __forceinline__ void row_sums(float& x, float& y, int lanes, float* red) {
  if constexpr (kLanes == kGroup) {
    x = lane_sum<64>(x);
    y = lane_sum<64>(y);
    if ((threadIdx.x & 63) == 0) {
      red[threadIdx.x >> 6] = x;
      red[kMostWaves + (threadIdx.x >> 6)] = y;
    }
    __syncthreads();
    x = y = 0.f;
    for (int w = 0; w < (int)blockDim.x >> 6; ++w) {
      x += red[w];
      y += red[kMostWaves + w];
    }
  } else {
    x = lane_sum<kLanes>(x, lanes);
    y = lane_sum<kLanes>(y, lanes);
  }
}

// A product that is not made part of what it is subtracted from: m has to be the same number wherever it is taken.
__device__ __forceinline__ float rounded_product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}

// 1 / sqrt(x) off by one unit in the last place; what is no normal number goes the long way.
__device__ __forceinline__ float inverse_root(float x) {
  return x < 1.17549435e-38f ? 1.f / sqrtf(x) : __builtin_amdgcn_rsqf(x);
}

// The thread's place: `lanes` threads a row, `seats` rows of a workgroup at a time.
template <int kLanes>
struct Seat {
  int lanes, seats, seat, t;
  __device__ __forceinline__ explicit Seat(int l) {
    lanes = kLanes == kGroup ? (int)blockDim.x : (kLanes ? kLanes : l);
    seats = kLanes == kGroup ? 1 : 256 / lanes;
    seat = kLanes == kGroup ? 0 : (int)threadIdx.x / lanes;
    t = kLanes == kGroup ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
  }
};
// Elements between the workgroup's first row and the seat's: below 2^32 / sizeof(float), rows are at most 2^22 elements apart.
__device__ __forceinline__ unsigned rows_on(int seat, long long ld) { return (unsigned)seat * (unsigned)ld; }

// Rows of a seat in the forward pass, whose requests go out together (5.7 M rows of 256 in bf16 with SiLU: one 1090 us, two 995,
// four 1018; 20000 rows of 8192 in bf16 177, 136 and 135; 20011 of 5003 in fp32 186, 157 and 194).
constexpr int kSeatRows = 2;
template <typename T, int NV, int kLanes, Fit kFit, bool kOnce>
__global__ __launch_bounds__(kLanes == kGroup ? 1024 : 256) void row_norm_kernel(const RowNormArgs a, int row_lanes) {
  constexpr int kV = kVector<T>, kN = NV * kV, kRows = kSeatRows;
  __shared__ float red[kLanes == kGroup ? 3 * kMostWaves : 1];
  const Seat<kLanes> s(row_lanes);
  const Columns<T, NV> q = columns_of<T, NV, kFit>(s.t, s.lanes, a.C);
  const float share = 1.f / (float)a.C;
  const unsigned x_on = rows_on(s.seat, a.ldx), y_on = rows_on(s.seat, a.ldy);
  for (long long row0 = (long long)blockIdx.x * s.seats * kRows; row0 < a.rows; row0 += (long long)gridDim.x * s.seats * kRows) {
    const int left = (int)min(a.rows - row0, (long long)s.seats * kRows);     // rows of the workgroup
    const T* X = static_cast<const T*>(a.X) + row0 * a.ldx;
    T* Y = static_cast<T*>(a.Y) + row0 * a.ldy;
    // the requests of all its rows first; behind the last row the first one again
    Fetched<T, T, NV> f[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const bool there = u * s.seats + s.seat < left;
      fetch<kOnce, T, NV, kFit>(f[u], u * s.seats < left ? X + u * s.seats * a.ldx : X, there ? x_on : 0u, q, a.C);
    }
    float gamma[kN], beta[kN];
    vectors_at<T, NV, kFit>(gamma, a.gamma, 1.f, q, a.C);
    vectors_at<T, NV, kFit>(beta, a.beta, 0.f, q, a.C);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      if (u * s.seats + s.seat >= left) break;
      float x[kN];
      values<T, NV, kFit>(x, f[u], q);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < kV; ++k) sum += own<T, NV, kFit>(q, j, k, a.C) ? x[j * kV + k] : 0.f;
      const float m = rounded_product(row_sum<kLanes>(sum, s.lanes, red), share);
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < kV; ++k) {
          x[j * kV + k] -= m;
          const float d = own<T, NV, kFit>(q, j, k, a.C) ? x[j * kV + k] : 0.f;
          s1 += d;
          s2 = fmaf(d, d, s2);
        }
      row_sums<kLanes>(s1, s2, s.lanes, red + kMostWaves);
      // What is less than the rounding of the d's own (2^-24 of their size) says nothing about m: the d of one size are rounded alike,
      // which would move a mean that is far smaller than they are.
      const float square = s2 * share, found = s1 * share, lacks = found * found <= 0x1p-48f * square ? 0.f : found;
      const float var = fmaf(-lacks, lacks, square);
      const float r = inverse_root((var < 0.f ? 0.f : var) + a.eps);
      const float shift = -lacks * r;
#pragma unroll
      for (int k = 0; k < kN; ++k) x[k] = fmaf(fmaf(x[k], r, shift), gamma[k], beta[k]);
      activate<kN>(x, a.act);
      put<kOnce, T, NV, kFit>(x, Y + u * s.seats * a.ldy, y_on, q, a.C);
      if (a.mean && s.t == 0) {
        a.mean[row0 + u * s.seats + s.seat] = m + lacks;
        a.rstd[row0 + u * s.seats + s.seat] = r;
      }
    }
  }
}

template <typename T, typename X, int NV, int kLanes, Fit kFit, bool kOnce>
__global__ __launch_bounds__(kLanes == kGroup ? 1024 : 256) void row_norm_back_kernel(const RowNormArgs a, int row_lanes) {
  constexpr int kV = kVector<T>, kN = NV * kV;
  constexpr bool kKept = !std::is_same<T, X>::value, kWide = kLanes == kGroup;
  // Of sixteen values a thread the sums over rows stay in LDS, a thread's fours of both 1024 fours apart.  That is one workgroup a CU, of
  // which nothing covers the waits at its barrier, and in fp32 128 registers do not suffice (3 to 26 words of a thread in scratch memory):
  // with dres 20000 x 16384 in bf16 653 us, 4.0 TB/s, in fp32 935, 5.6; 20011 x 16383 833 and 1206; rows of 8192 in fp32 5.7 TB/s.
  constexpr bool kLds = kN > 8;
  __shared__ float red[kWide ? 4 * kMostWaves : 2 * 256 * kN];
  __shared__ float4 sums[kLds ? 1024 * kN / 2 : 1];
  const Seat<kLanes> s(row_lanes);
  const Columns<T, NV> q = columns_of<T, NV, kFit>(s.t, s.lanes, a.C);
  float gamma[kN], beta[kN], dg[kN], db[kN], dgs[kN], dbs[kN];     // of eight values a thread
  if (!kLds) {
    vectors_at<T, NV, kFit>(gamma, a.gamma, 1.f, q, a.C);
    vectors_at<T, NV, kFit>(beta, a.beta, 0.f, q, a.C);
  }
  float* out = a.workspace + (size_t)blockIdx.x * 2 * a.C;
  // the runs' sums: in registers, or where the workgroup's go
  auto join = [&](bool begin) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int v = 0; v < kV; ++v) {
        const int k = j * kV + v, c = q.at[j] + v;
        if constexpr (!kLds) {
          dgs[k] = begin ? 0.f : dgs[k] + dg[k];
          dbs[k] = begin ? 0.f : dbs[k] + db[k];
          dg[k] = db[k] = 0.f;
        } else {
          float4& g4 = sums[(k / 4 * 2) * 1024 + threadIdx.x];
          float4& b4 = sums[(k / 4 * 2 + 1) * 1024 + threadIdx.x];
          float& g = reinterpret_cast<float*>(&g4)[k & 3];
          float& b = reinterpret_cast<float*>(&b4)[k & 3];
          if (a.dgamma && own<T, NV, kFit>(q, j, v, a.C)) {
            out[c] = begin ? 0.f : out[c] + g;
            out[a.C + c] = begin ? 0.f : out[a.C + c] + b;
          }
          g = b = 0.f;
        }
      }
  };
  join(true);
  const float share = 1.f / (float)a.C;
  int run = 0, parity = 0;
  const unsigned x_on = kKept ? rows_on(s.seat, a.kept.ld_code) : rows_on(s.seat, a.ldx), e_on = rows_on(s.seat, a.kept.ld_exponent),
                 dy_on = rows_on(s.seat, a.lddy), res_on = rows_on(s.seat, a.lddres), dx_on = rows_on(s.seat, a.lddx);
  for (long long row0 = (long long)blockIdx.x * s.seats; row0 + s.seat < a.rows; row0 += (long long)gridDim.x * s.seats) {
    Fetched<T, X, NV> f;
    Fetched<T, T, NV> fd, fr;
    if constexpr (kKept) fetch<kOnce, T, NV, kFit>(f, a.kept.code + row0 * a.kept.ld_code, x_on, a.kept.exponent + row0 * a.kept.ld_exponent, e_on, q);
    else fetch<kOnce, T, NV, kFit>(f, static_cast<const T*>(a.X) + row0 * a.ldx, x_on, q, a.C);
    fetch<kOnce, T, NV, kFit>(fd, static_cast<const T*>(a.dY) + row0 * a.lddy, dy_on, q, a.C);
    if (!kLds && a.dRes) fetch<kOnce, T, NV, kFit>(fr, static_cast<const T*>(a.dRes) + row0 * a.lddres, res_on, q, a.C);
    const float m = a.mean[row0 + s.seat], r = a.rstd[row0 + s.seat];
    float xh[kN], dz[kN];
    values<T, NV, kFit>(xh, f, q);
    values<T, NV, kFit>(dz, fd, q);
    float s1 = 0.f, s2 = 0.f;
    // vector by vector: of sixteen values a thread there are no registers for all, nor for gamma, beta and dres all the time
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float gj[kV], bj[kV], z[kV];
      if (kLds) {
        vector_at<T, kFit>(gj, a.gamma, 1.f, q.at[j], a.C);
        vector_at<T, kFit>(bj, a.beta, 0.f, q.at[j], a.C);
      }
#pragma unroll
      for (int v = 0; v < kV; ++v) {
        const int k = j * kV + v;
        if (!kLds) {
          gj[v] = gamma[k];
          bj[v] = beta[k];
        }
        xh[k] = (xh[k] - m) * r;
        z[v] = fmaf(gj[v], xh[k], bj[v]);
      }
      if (a.act != DC_ACT_NONE) {
        slopes<kV>(z, a.act);
#pragma unroll
        for (int v = 0; v < kV; ++v) dz[j * kV + v] *= z[v];
      }
#pragma unroll
      for (int v = 0; v < kV; ++v) {
        const int k = j * kV + v;
        if constexpr (!kLds) {
          dg[k] = fmaf(dz[k], xh[k], dg[k]);
          db[k] += dz[k];
        } else if (k % 4 == 0) {
          float4 g = sums[(k / 4 * 2) * 1024 + threadIdx.x], b = sums[(k / 4 * 2 + 1) * 1024 + threadIdx.x];
          g.x = fmaf(dz[k], xh[k], g.x);
          g.y = fmaf(dz[k + 1], xh[k + 1], g.y);
          g.z = fmaf(dz[k + 2], xh[k + 2], g.z);
          g.w = fmaf(dz[k + 3], xh[k + 3], g.w);
          b.x += dz[k];
          b.y += dz[k + 1];
          b.z += dz[k + 2];
          b.w += dz[k + 3];
          sums[(k / 4 * 2) * 1024 + threadIdx.x] = g;
          sums[(k / 4 * 2 + 1) * 1024 + threadIdx.x] = b;
        }
        dz[k] *= gj[v];
        const float u = own<T, NV, kFit>(q, j, v, a.C) ? dz[k] : 0.f;
        s1 += u;
        s2 = fmaf(u, xh[k], s2);
      }
    }
    // dX may be dres, and a vector that ends with the row is its neighbour's too, which may be another wave's: read before that writes
    if (!kLds && kWide && kFit == kBack && a.dRes) {
#pragma unroll
      for (int j = 0; j < NV; ++j) asm volatile("" ::"v"(fr.v[j]));
    }
    row_sums<kLanes>(s1, s2, s.lanes, red + 2 * kMostWaves * parity);
    parity ^= 1;
    s1 *= share;
    s2 *= share;
    if (kLds && a.dRes) fetch<kOnce, T, NV, kFit>(fr, static_cast<const T*>(a.dRes) + row0 * a.lddres, res_on, q, a.C);
#pragma unroll
    for (int k = 0; k < kN; ++k) dz[k] = r * (dz[k] - s1 - xh[k] * s2);
    if (a.dRes) {
      float add[kN];
      values<T, NV, kFit>(add, fr, q);
#pragma unroll
      for (int k = 0; k < kN; ++k) dz[k] += add[k];
    }
    put<kOnce, T, NV, kFit, kLds>(dz, static_cast<T*>(a.dX) + row0 * a.lddx, dx_on, q, a.C);
    if (++run == kRun) {
      run = 0;
      join(false);
    }
  }
  if (!a.dgamma) return;
  join(false);
  if constexpr (kLds) return;
  if constexpr (kWide) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kV; ++k) {
        const int c = q.at[j] + k;
        if (own<T, NV, kFit>(q, j, k, a.C)) {
          out[c] = dgs[j * kV + k];
          out[a.C + c] = dbs[j * kV + k];
        }
      }
  } else {
    // the workgroup's rows: columns of a seat one behind the other
    const int width = s.lanes * kN, seats = 256 / s.lanes, seat = (int)threadIdx.x / s.lanes;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kV; ++k) {
        if (own<T, NV, kFit>(q, j, k, a.C)) {
          red[seat * width + q.at[j] + k] = dgs[j * kV + k];
          red[256 * kN + seat * width + q.at[j] + k] = dbs[j * kV + k];
        }
      }
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += 256) {
      double g = 0.0, b = 0.0;
      for (int q = 0; q < seats; ++q) {
        g += (double)red[q * width + c];
        b += (double)red[256 * kN + q * width + c];
      }
      out[c] = (float)g;
      out[a.C + c] = (float)b;
    }
  }
}

struct Plan {
  bool wide;
  int per;                     // values a thread
  int threads, lanes;          // of a workgroup; of a row
  long long blocks;
};
// `per` values a thread: in one row's lanes up to 64 threads, else in a workgroup.
Plan plan(long long rows, int C, int per) {
  Plan p{};
  p.per = per;
  const int need = (C + per - 1) / per;
  p.wide = need > 64;
  p.lanes = 1;
  while (!p.wide && p.lanes < need) p.lanes *= 2;
  if (p.wide) p.lanes = (need + 63) / 64 * 64;
  p.threads = p.wide ? p.lanes : 256;
  const long long seats = p.wide ? 1 : 256 / p.lanes;
  p.blocks = (rows + seats - 1) / seats;
  return p;
}
// A row a seat at a time, in the order in which the workgroups are handed out (a launch has less than 2^32 threads).  Wide rows in
// bf16 take sixteen values a thread, two requests, as rows in fp32 do with eight, and go faster by a tenth
// (50000 x 4096 in bf16, one row a seat: 211 us by eight, 189 by sixteen).  Rows beyond 8192 channels are one workgroup a CU (1024
// threads of 92 to 114 registers): 20000 x 16384 in bf16 350 us, 3.7 TB/s, in fp32 497, 5.3.
Plan forward_plan(long long rows, int C, bool bf16) {
  Plan p = plan(rows, C, C > 8192 || (bf16 && C > kNarrow) ? 16 : 8);
  p.blocks = (p.blocks + kSeatRows - 1) / kSeatRows;
  const long long most = (1LL << 31) / p.threads;
  if (p.blocks > most) p.blocks = most;
  return p;
}
// What a CU works on at a time, as each workgroup sums gradients of gamma and beta: rows of together 40 KB read and written, by 1024
// threads at most (60000 x 1536 in bf16 with dres by 2, 3 and 5 workgroups a CU 181, 143 and 155 us; 1000000 x 256 in fp32 with dres by
// 1 and 2 714 and 778; 2000003 x 256 in bf16 by 3 and 4 575 and 607).  bytes: of eight values of a row, read and written.
constexpr int kAtWork = 40000;
Plan back_plan(long long rows, int C, int n_cu, int bytes) {
  Plan p = plan(rows, C, C > 8192 ? 16 : 8);
  const int work = p.wide ? C * bytes / 8 : 256 * bytes;         // of a workgroup's rows
  int each = (kAtWork + work / 2) / work;
  if (each > 1024 / p.threads) each = 1024 / p.threads;
  if (each < 1) each = 1;
  const long long most = (long long)n_cu * each;
  if (p.blocks > most) p.blocks = most;
  return p;
}

// f gets kLanes and kFit as types: the lanes of 65 to 512 channels are known when the kernel is built.
template <int kI>
using Number = std::integral_constant<int, kI>;
template <typename T, typename F>
void each_fit(const Plan& p, int C, F f) {
  const bool whole = C == p.lanes * p.per;
  auto fit = [&](auto lanes) {
    if (whole) f(lanes, std::integral_constant<Fit, kWhole>());
    else f(lanes, std::integral_constant<Fit, kBack>());
  };
  if (p.wide) fit(Number<kGroup>());
  else if (p.lanes == 64) fit(Number<64>());
  else if (p.lanes == 32) fit(Number<32>());
  else if (p.lanes == 16) fit(Number<16>());
  else if (C >= kVector<T>) fit(Number<0>());
  else f(Number<0>(), std::integral_constant<Fit, kShort>());
}
// Whether rows go past the caches: whole ones (parts of lines are put together there) of which the memory's cache cannot hold all.
// 5.7 M rows of 256 in bf16, forward, 1025 -> 983 us; gradients of 2 M of them with dres 800 -> 768, of 474011 in fp32, x in 8 bits, 204 -> 197.
// Smaller ones may be there for the next operator: behind 200000 rows of 256 in bf16 past the caches a dense layer made it 102 us for 95.
constexpr long long kCached = 256 << 20;
template <Fit kFit>
bool once(const RowNormArgs& a) { return kFit == kWhole && a.rows * a.C * (a.bf16 ? 2LL : 4LL) > kCached; }
template <typename T>
void forward(const RowNormArgs& a, hipStream_t s) {
  constexpr int NV = 8 / kVector<T>;
  const Plan p = forward_plan(a.rows, a.C, a.bf16);
  const dim3 g((unsigned)p.blocks), b((unsigned)p.threads);
  each_fit<T>(p, a.C, [&](auto lanes, auto fit) {
    constexpr int kLanes = decltype(lanes)::value;
    constexpr Fit kFit = decltype(fit)::value;
    auto launch = [&](auto vectors, auto past) {
      hipLaunchKernelGGL((row_norm_kernel<T, decltype(vectors)::value, kLanes, kFit, decltype(past)::value != 0>), g, b, 0, s, a, p.lanes);
    };
    auto vectors = [&](auto past) {
      // sixteen values: a workgroup's rows, and a whole wave's in bf16
      if constexpr (kLanes == kGroup || (kLanes == 64 && sizeof(T) == 2)) {
        if (p.per == 16) return launch(Number<2 * NV>(), past);
      }
      launch(Number<NV>(), past);
    };
    if constexpr (kFit == kWhole) {
      if (once<kFit>(a)) return vectors(Number<1>());
    }
    vectors(Number<0>());
  });
}
template <typename T, typename X>
void backward(const RowNormArgs& a, const Plan& p, hipStream_t s) {
  constexpr int NV = 8 / kVector<T>;
  const dim3 g((unsigned)p.blocks), b((unsigned)p.threads);
  each_fit<T>(p, a.C, [&](auto lanes, auto fit) {
    constexpr int kLanes = decltype(lanes)::value;
    constexpr Fit kFit = decltype(fit)::value;
    auto launch = [&](auto vectors, auto past) {
      hipLaunchKernelGGL((row_norm_back_kernel<T, X, decltype(vectors)::value, kLanes, kFit, decltype(past)::value != 0>), g, b, 0, s, a, p.lanes);
    };
    auto vectors = [&](auto past) {
      if constexpr (kLanes == kGroup) {
        if (p.per == 16) return launch(Number<2 * NV>(), past);
      }
      launch(Number<NV>(), past);
    };
    if constexpr (kFit == kWhole) {
      if (once<kFit>(a)) return vectors(Number<1>());
    }
    vectors(Number<0>());
  });
}

}  // namespace

size_t row_norm_floats(long long rows, int C, int n_cu) { return (size_t)back_plan(rows, C, n_cu, 8 + 16 + 16).blocks * 2 * C; }

hipError_t launch_row_norm(const RowNormArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  if (a.bf16) forward<u16>(a, s);
  else forward<float>(a, s);
  return hipGetLastError();
}

hipError_t launch_row_norm_back(const RowNormArgs& a, hipStream_t s) {
  const int bytes = a.bf16 ? 16 : 32;              // of eight values
  const Plan p = back_plan(a.rows, a.C, a.n_cu, (a.kept.code ? 8 : bytes) + 2 * bytes + (a.dRes ? bytes : 0));
  if (a.rows > 0) {
    if (a.kept.code) {
      if (a.bf16) backward<u16, Kept8>(a, p, s);
      else backward<float, Kept8>(a, p, s);
    } else {
      if (a.bf16) backward<u16, u16>(a, p, s);
      else backward<float, float>(a, p, s);
    }
  }
  // without rows: zeros
  if (a.dgamma) launch_column_sums(a.workspace, (int)p.blocks, a.C, a.dgamma, a.C, a.dbeta, nullptr, s);
  return hipGetLastError();
}

}  // namespace dc
