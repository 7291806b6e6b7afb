// Rows kept in 8 bits for the backward pass, and read back (gfx950).
//
// Per row and 32 columns: m = max |x|, e = the smallest integer of [-126, 121] with m <= 127 * 2^e, codes
// q = x * 2^-e rounded to nearest even within +-127, and +-1 where x is not zero but would round to it (so that the
// sign, and with it ReLU's derivative, survives).  Off by at most half a step 2^e (a whole one for |x| below half of it or above 127 * 2^121).
// The scale is a power of two so that q * 2^e has at most seven significant bits: it is a bf16 number, and a
// product with kept rows needs one exact operand on the bf16 matrix cores where fp32 rows need three pieces.  A finer
// scale (m / 127) would gain half a bit on average and lose that.
// A block with a number that is not finite: exponent code 255, all its values NaN.
// Bound by memory: 4 or 2 bytes in, 1 + 1/32 out.  kV columns per lane, 32 / kV lanes per block.  Measured: 474011 x 256 in
// fp32 kept and read back 0.253 ms, 4.8 TB/s.
#include "operators.h"

namespace dc {
namespace {

template <typename T, int kV>
struct alignas(sizeof(T) * kV) Vec {
  T v[kV];
};
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(unsigned short x) { return __uint_as_float((unsigned)x << 16); }
__device__ __forceinline__ void narrow(float x, float& y) { y = x; }
__device__ __forceinline__ void narrow(float x, unsigned short& y) { y = to_bf16(x); }

template <typename T, int kV>
__global__ __launch_bounds__(256) void keep_kernel(const KeepArgs a) {
  if (a.stop && a.stop[0] != 0) return;
  constexpr int kLanes = kKeptBlock / kV;
  const long long rows = a.nrows ? a.nrows[0] : a.rows;
  const int nb = (a.cols + kKeptBlock - 1) / kKeptBlock;
  const T* __restrict__ src = static_cast<const T*>(a.src);
  const int lane = threadIdx.x % kLanes;
  const long long items = rows * nb;
  for (long long i = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / kLanes; i < items;
       i += (long long)gridDim.x * blockDim.x / kLanes) {
    const long long r = i / nb;
    const int b = (int)(i - r * nb), c = b * kKeptBlock + lane * kV;
    float x[kV];
    const T* p = src + r * a.ld + c;
    if (kV > 1) {                                    // a.cols is a multiple of kV
      Vec<T, kV> v{};
      if (c < a.cols) v = *reinterpret_cast<const Vec<T, kV>*>(p);
#pragma unroll
      for (int k = 0; k < kV; ++k) x[k] = widen(v.v[k]);
    } else {
      x[0] = c < a.cols ? widen(p[0]) : 0.f;
    }
    unsigned m = 0;                                  // the bits of |x| order as |x| does, what is not finite above all
#pragma unroll
    for (int k = 0; k < kV; ++k) m = max(m, __float_as_uint(x[k]) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, o, 64));
    const bool finite = m < 0x7F800000u;
    // 127 / 64 = 1.984375 = mantissa 0x7E0000
    int e = (int)(m >> 23) - 127 - 6 + ((m & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
    e = m == 0 ? kKeptLeast : min(max(e, kKeptLeast), kKeptMost);
    const float up = __uint_as_float((unsigned)(127 - e) << 23);
    Vec<signed char, kV> q;
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      float u = rintf(x[k] * up);
      u = fminf(fmaxf(u, -127.f), 127.f);
      if (u == 0.f && x[k] != 0.f) u = x[k] > 0.f ? 1.f : -1.f;
      q.v[k] = finite ? (signed char)(int)u : (signed char)0;
    }
    *reinterpret_cast<Vec<signed char, kV>*>(a.code + r * a.ld_code + c) = q;   // up to the end of the block
    if (lane == 0) a.exponent[r * a.ld_exponent + b] = (unsigned char)(finite ? e + 127 : kKeptNan);
  }
}

template <typename T, int kV>
__global__ __launch_bounds__(256) void restore_kernel(const KeepArgs a) {
  if (a.stop && a.stop[0] != 0) return;
  const long long rows = a.nrows ? a.nrows[0] : a.rows;
  const int per = (a.cols + kV - 1) / kV;
  T* __restrict__ dst = static_cast<T*>(a.dst);
  const long long items = rows * per;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < items; i += (long long)gridDim.x * blockDim.x) {
    const long long r = i / per;
    const int c = (int)(i - r * per) * kV;
    const Vec<signed char, kV> q = *reinterpret_cast<const Vec<signed char, kV>*>(a.code + r * a.ld_code + c);
    const float scale = kept_scale(a.exponent[r * a.ld_exponent + c / kKeptBlock]);
    Vec<T, kV> v;
#pragma unroll
    for (int k = 0; k < kV; ++k) narrow((float)q.v[k] * scale, v.v[k]);
    *reinterpret_cast<Vec<T, kV>*>(dst + r * a.ld + c) = v;
  }
}

// Vectors of kV columns need rows that start at a multiple of them.
bool vectors(const KeepArgs& a, const void* rows, int v) {
  const size_t bytes = (size_t)v * (a.bf16 ? 2 : 4);
  return a.cols % v == 0 && a.ld % v == 0 && a.ld_code % v == 0 && reinterpret_cast<size_t>(rows) % bytes == 0 &&
         reinterpret_cast<size_t>(a.code) % v == 0;
}
dim3 grid_of(long long threads, int n_cu) {
  const long long g = (threads + 255) / 256, most = (long long)n_cu * 32;
  return dim3((unsigned)(g < 1 ? 1 : (g > most ? most : g)));
}

}  // namespace

hipError_t launch_keep_rows(const KeepArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  const long long blocks = a.rows * ((a.cols + kKeptBlock - 1) / kKeptBlock);
  if (a.bf16) {
    if (vectors(a, a.src, 8)) hipLaunchKernelGGL((keep_kernel<unsigned short, 8>), grid_of(blocks * 4, a.n_cu), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((keep_kernel<unsigned short, 1>), grid_of(blocks * 32, a.n_cu), dim3(256), 0, s, a);
  } else {
    if (vectors(a, a.src, 4)) hipLaunchKernelGGL((keep_kernel<float, 4>), grid_of(blocks * 8, a.n_cu), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((keep_kernel<float, 1>), grid_of(blocks * 32, a.n_cu), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_restore_rows(const KeepArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  if (a.bf16) {
    if (vectors(a, a.dst, 8)) hipLaunchKernelGGL((restore_kernel<unsigned short, 8>), grid_of(a.rows * a.cols / 8, a.n_cu), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((restore_kernel<unsigned short, 1>), grid_of(a.rows * a.cols, a.n_cu), dim3(256), 0, s, a);
  } else {
    if (vectors(a, a.dst, 4)) hipLaunchKernelGGL((restore_kernel<float, 4>), grid_of(a.rows * a.cols / 4, a.n_cu), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((restore_kernel<float, 1>), grid_of(a.rows * a.cols, a.n_cu), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace dc
