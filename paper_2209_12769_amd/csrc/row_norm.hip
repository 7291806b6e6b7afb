// Norm over the channels of each row with an activation, and its gradient (gfx950):
//
//   forward   mu = mean x, v = mean (x - mu)^2, r = 1 / sqrt(v + eps);  y = act(gamma (x - mu) r + beta)
//   backward  xh = (x - mu) r, dz = dy act'(gamma xh + beta), u = gamma dz, s1 = mean u, s2 = mean u xh;
//             dx = r (u - s1 - xh s2) [+ dres];  dgamma = sum over rows of dz xh, dbeta = sum of dz
//
// Bound by memory: a row is read once and stays in registers, eight values a thread (sixteen beyond 8192 channels).  Rows of up
// to 512 channels take a power of two of a wave's lanes, several rows a wave, wider rows a workgroup; the grid is what is
// resident, each place takes one row after the other and requests the next one before it works on its own.
// The variance is that of d = x - m, m the row's sum over C as fp32 has it: mean d is what m lacks, v = mean d^2 - (mean d)^2.
// So neither loses digits for values far from zero, and mu is m + mean d, rounded once where it is returned.
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

// NV vectors of a row, vector j of a thread at columns (j * lanes + t) * kVector.
template <typename T, typename X, int NV>
struct Fetched {
  u32x4 v[NV];
};
template <int NV>
struct Fetched<u16, Kept8, NV> {
  u32x2 v[NV];
  unsigned e[NV];
};
template <int NV>
struct Fetched<float, Kept8, NV> {
  unsigned v[NV];
  unsigned e[NV];
};
template <typename T, int NV, bool kFull>
__device__ __forceinline__ void fetch(Fetched<T, T, NV>& f, const void* rows, long long ld, long long row, int t, int lanes, int C) {
  const T* p = static_cast<const T*>(rows) + row * ld;
#pragma unroll
  for (int j = 0; j < NV; ++j) f.v[j] = load_vector<T, kFull>(p, (j * lanes + t) * kVector<T>, C);
}
// A row of codes goes up to a multiple of 32: a vector that begins inside the row ends inside it.
template <typename T, int NV, bool kFull>
__device__ __forceinline__ void fetch(Fetched<T, Kept8, NV>& f, const KeptView& k, long long row, int t, int lanes, int C) {
  const signed char* p = k.code + row * k.ld_code;
  const unsigned char* e = k.exponent + row * k.ld_exponent;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * lanes + t) * kVector<T>;
    f.v[j] = decltype(f.v[j] + f.v[j]){};
    f.e[j] = 0;
    if (kFull || c < C) {
      if constexpr (sizeof(T) == 2) f.v[j] = *reinterpret_cast<const u32x2_any*>(p + c);
      else f.v[j] = *reinterpret_cast<const u32_any*>(p + c);
      f.e[j] = e[c / kKeptBlock];
    }
  }
}
template <typename T, int NV>
__device__ __forceinline__ void values(float (&x)[NV * kVector<T>], const Fetched<T, T, NV>& f) {
  constexpr int kV = kVector<T>;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float w[kV];
    unpack(w, f.v[j], T());
#pragma unroll
    for (int k = 0; k < kV; ++k) x[j * kV + k] = w[k];
  }
}
template <typename T, int NV>
__device__ __forceinline__ void values(float (&x)[NV * kVector<T>], const Fetched<T, Kept8, NV>& f) {
  constexpr int kV = kVector<T>;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const float s = kept_scale(f.e[j]);
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      unsigned w;
      if constexpr (kV == 8) w = f.v[j][k / 4];
      else w = f.v[j];
      x[j * kV + k] = (float)(signed char)(w >> (8 * (k & 3))) * s;
    }
  }
}

template <typename T, int NV>
__device__ __forceinline__ void vectors_at(float (&g)[NV * kVector<T>], const float* v, float none, int t, int lanes, int C) {
  constexpr int kV = kVector<T>;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      const int c = (j * lanes + t) * kV + k;
      g[j * kV + k] = v ? (c < C ? v[c] : 0.f) : none;
    }
}
template <typename T, int NV, bool kFull>
__device__ __forceinline__ void put(const float (&y)[NV * kVector<T>], void* rows, long long ld, long long row, int t, int lanes, int C) {
  constexpr int kV = kVector<T>;
  T* p = static_cast<T*>(rows) + row * ld;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float w[kV];
#pragma unroll
    for (int k = 0; k < kV; ++k) w[k] = y[j * kV + k];
    store_vector<T, kFull>(p, (j * lanes + t) * kV, C, pack(w, T()));
  }
}

// Sums over a row's threads, in all of them.  kWide: the workgroup; `red` has room for two numbers a wave, and another row's
// sums may use it only after one more barrier.
template <bool kWide>
__device__ __forceinline__ float row_sum(float x, int lanes, float* red) {
  x = lane_sum(x, kWide ? 64 : lanes);
  if constexpr (kWide) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
    for (int w = 0; w < (int)blockDim.x >> 6; ++w) x += red[w];
  }
  return x;
}
template <bool kWide>
__device__ __forceinline__ void row_sums(float& x, float& y, int lanes, float* red) {
  x = lane_sum(x, kWide ? 64 : lanes);
  y = lane_sum(y, kWide ? 64 : lanes);
  if constexpr (kWide) {
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

// Threads of a row: lanes of a wave, or the workgroup.
template <bool kWide>
struct Seat {
  int lanes, t;
  long long row, step;
  __device__ __forceinline__ explicit Seat(int l)
      : lanes(kWide ? (int)blockDim.x : l), t(kWide ? (int)threadIdx.x : (int)threadIdx.x & (l - 1)) {
    const int seats = kWide ? 1 : (int)blockDim.x / l;
    row = (long long)blockIdx.x * seats + (kWide ? 0 : (int)threadIdx.x / l);
    step = (long long)gridDim.x * seats;
  }
};

template <typename T, int NV, bool kWide, bool kFull>
__global__ __launch_bounds__(kWide ? 1024 : 256) void row_norm_kernel(const RowNormArgs a, int row_lanes) {
  constexpr int kV = kVector<T>, kN = NV * kV;
  __shared__ float red[kWide ? 3 * kMostWaves : 1];
  Seat<kWide> s(row_lanes);
  float gamma[kN], beta[kN];
  vectors_at<T, NV>(gamma, a.gamma, 1.f, s.t, s.lanes, a.C);
  vectors_at<T, NV>(beta, a.beta, 0.f, s.t, s.lanes, a.C);
  if (s.row >= a.rows) return;
  const float share = 1.f / (float)a.C;
  Fetched<T, T, NV> f;
  fetch<T, NV, kFull>(f, a.X, a.ldx, s.row, s.t, s.lanes, a.C);
  for (;;) {
    const long long next = s.row + s.step;
    Fetched<T, T, NV> ahead;
    fetch<T, NV, kFull>(ahead, a.X, a.ldx, next < a.rows ? next : s.row, s.t, s.lanes, a.C);
    float x[kN];
    values<T, NV>(x, f);
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kN; ++k) sum += x[k];
    const float m = rounded_product(row_sum<kWide>(sum, s.lanes, red), share);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kV; ++k) {
        float& d = x[j * kV + k];
        d -= m;
        if (!kFull && (j * s.lanes + s.t) * kV + k >= a.C) d = 0.f;
        s1 += d;
        s2 = fmaf(d, d, s2);
      }
    row_sums<kWide>(s1, s2, s.lanes, red + kMostWaves);
    const float lacks = s1 * share, var = fmaf(-lacks, lacks, s2 * share);
    const float r = inverse_root((var < 0.f ? 0.f : var) + a.eps);
    const float shift = -lacks * r;
#pragma unroll
    for (int k = 0; k < kN; ++k) x[k] = fmaf(fmaf(x[k], r, shift), gamma[k], beta[k]);
    activate<kN>(x, a.act);
    put<T, NV, kFull>(x, a.Y, a.ldy, s.row, s.t, s.lanes, a.C);
    if (a.mean && s.t == 0) {
      a.mean[s.row] = m + lacks;
      a.rstd[s.row] = r;
    }
    if (next >= a.rows) return;
    s.row = next;
    f = ahead;
  }
}

template <typename T, typename X, int NV, bool kWide, bool kFull>
__global__ __launch_bounds__(kWide ? 1024 : 256) void row_norm_back_kernel(const RowNormArgs a, int row_lanes) {
  constexpr int kV = kVector<T>, kN = NV * kV;
  constexpr bool kKept = !std::is_same<T, X>::value;
  __shared__ float red[kWide ? 4 * kMostWaves : 2 * 256 * kN];
  Seat<kWide> s(row_lanes);
  float gamma[kN], beta[kN], dg[kN], db[kN], dgs[kN], dbs[kN];
  if (kN == 8) {
    vectors_at<T, NV>(gamma, a.gamma, 1.f, s.t, s.lanes, a.C);
    vectors_at<T, NV>(beta, a.beta, 0.f, s.t, s.lanes, a.C);
  }
#pragma unroll
  for (int k = 0; k < kN; ++k) dg[k] = db[k] = dgs[k] = dbs[k] = 0.f;
  const float share = 1.f / (float)a.C;
  int run = 0, parity = 0;
  for (; s.row < a.rows; s.row += s.step) {
    Fetched<T, X, NV> f;
    Fetched<T, T, NV> fd, fr;
    if constexpr (kKept) fetch<T, NV, kFull>(f, a.kept, s.row, s.t, s.lanes, a.C);
    else fetch<T, NV, kFull>(f, a.X, a.ldx, s.row, s.t, s.lanes, a.C);
    fetch<T, NV, kFull>(fd, a.dY, a.lddy, s.row, s.t, s.lanes, a.C);
    if (a.dRes) fetch<T, NV, kFull>(fr, a.dRes, a.lddres, s.row, s.t, s.lanes, a.C);
    const float m = a.mean[s.row], r = a.rstd[s.row];
    if (kN > 8) {                                        // registers for eight values a thread only
      vectors_at<T, NV>(gamma, a.gamma, 1.f, s.t, s.lanes, a.C);
      vectors_at<T, NV>(beta, a.beta, 0.f, s.t, s.lanes, a.C);
    }
    float xh[kN], dz[kN], z[kN];
    values<T, NV>(xh, f);
    values<T, NV>(dz, fd);
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      xh[k] = (xh[k] - m) * r;
      z[k] = fmaf(gamma[k], xh[k], beta[k]);
    }
    if (a.act != DC_ACT_NONE) {
      slopes<kN>(z, a.act);
#pragma unroll
      for (int k = 0; k < kN; ++k) dz[k] *= z[k];
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      dg[k] = fmaf(dz[k], xh[k], dg[k]);
      db[k] += dz[k];
      dz[k] *= gamma[k];
      s1 += dz[k];
      s2 = fmaf(dz[k], xh[k], s2);
    }
    row_sums<kWide>(s1, s2, s.lanes, red + 2 * kMostWaves * parity);
    parity ^= 1;
    s1 *= share;
    s2 *= share;
#pragma unroll
    for (int k = 0; k < kN; ++k) dz[k] = r * (dz[k] - s1 - xh[k] * s2);
    if (a.dRes) {
      float add[kN];
      values<T, NV>(add, fr);
#pragma unroll
      for (int k = 0; k < kN; ++k) dz[k] += add[k];
    }
    put<T, NV, kFull>(dz, a.dX, a.lddx, s.row, s.t, s.lanes, a.C);
    if (++run == kRun) {
      run = 0;
#pragma unroll
      for (int k = 0; k < kN; ++k) {
        dgs[k] += dg[k];
        dbs[k] += db[k];
        dg[k] = db[k] = 0.f;
      }
    }
  }
  if (!a.dgamma) return;
  float* out = a.workspace + (size_t)blockIdx.x * 2 * a.C;
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    dgs[k] += dg[k];
    dbs[k] += db[k];
  }
  if constexpr (kWide) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kV; ++k) {
        const int c = (j * s.lanes + s.t) * kV + k;
        if (c < a.C) {
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
        const int c = (j * s.lanes + s.t) * kV + k;
        red[seat * width + c] = dgs[j * kV + k];
        red[256 * kN + seat * width + c] = dbs[j * kV + k];
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
  bool wide, full;
  int nv16;                    // sixteen values a thread instead of eight
  int threads, lanes;          // of a workgroup; of a row
  long long blocks;
};
Plan plan(long long rows, int C, int n_cu, bool back) {
  Plan p{};
  p.wide = C > kNarrow;
  p.nv16 = C > 8192;
  const int per = p.nv16 ? 16 : 8, need = (C + per - 1) / per;
  if (p.wide) {
    p.threads = p.lanes = (need + 63) / 64 * 64;
  } else {
    p.threads = 256;
    p.lanes = 1;
    while (p.lanes < need) p.lanes *= 2;
  }
  p.full = C == p.lanes * per;
  const long long seats = p.wide ? 1 : 256 / p.lanes, need_blocks = (rows + seats - 1) / seats;
  // what a CU holds at a time
  const int threads_of_cu = back ? 1024 : 2048, each = threads_of_cu / p.threads;
  const long long most = (long long)n_cu * (each < 1 ? 1 : each);
  p.blocks = need_blocks < most ? need_blocks : most;
  return p;
}

template <typename T>
void forward(const RowNormArgs& a, const Plan& p, hipStream_t s) {
  constexpr int NV = 8 / kVector<T>;
  const dim3 g((unsigned)p.blocks), b((unsigned)p.threads);
  if (p.nv16) {
    if (p.full) hipLaunchKernelGGL((row_norm_kernel<T, 2 * NV, true, true>), g, b, 0, s, a, p.lanes);
    else hipLaunchKernelGGL((row_norm_kernel<T, 2 * NV, true, false>), g, b, 0, s, a, p.lanes);
  } else if (p.wide) {
    if (p.full) hipLaunchKernelGGL((row_norm_kernel<T, NV, true, true>), g, b, 0, s, a, p.lanes);
    else hipLaunchKernelGGL((row_norm_kernel<T, NV, true, false>), g, b, 0, s, a, p.lanes);
  } else {
    if (p.full) hipLaunchKernelGGL((row_norm_kernel<T, NV, false, true>), g, b, 0, s, a, p.lanes);
    else hipLaunchKernelGGL((row_norm_kernel<T, NV, false, false>), g, b, 0, s, a, p.lanes);
  }
}
template <typename T, typename X>
void backward(const RowNormArgs& a, const Plan& p, hipStream_t s) {
  constexpr int NV = 8 / kVector<T>;
  const dim3 g((unsigned)p.blocks), b((unsigned)p.threads);
  if (p.nv16) {
    if (p.full) hipLaunchKernelGGL((row_norm_back_kernel<T, X, 2 * NV, true, true>), g, b, 0, s, a, p.lanes);
    else hipLaunchKernelGGL((row_norm_back_kernel<T, X, 2 * NV, true, false>), g, b, 0, s, a, p.lanes);
  } else if (p.wide) {
    if (p.full) hipLaunchKernelGGL((row_norm_back_kernel<T, X, NV, true, true>), g, b, 0, s, a, p.lanes);
    else hipLaunchKernelGGL((row_norm_back_kernel<T, X, NV, true, false>), g, b, 0, s, a, p.lanes);
  } else {
    if (p.full) hipLaunchKernelGGL((row_norm_back_kernel<T, X, NV, false, true>), g, b, 0, s, a, p.lanes);
    else hipLaunchKernelGGL((row_norm_back_kernel<T, X, NV, false, false>), g, b, 0, s, a, p.lanes);
  }
}

}  // namespace

size_t row_norm_floats(long long rows, int C, int n_cu) { return (size_t)plan(rows, C, n_cu, true).blocks * 2 * C; }

hipError_t launch_row_norm(const RowNormArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const Plan p = plan(a.rows, a.C, a.n_cu, false);
  if (a.bf16) forward<u16>(a, p, s);
  else forward<float>(a, p, s);
  return hipGetLastError();
}

hipError_t launch_row_norm_back(const RowNormArgs& a, hipStream_t s) {
  const Plan p = plan(a.rows, a.C, a.n_cu, true);
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
