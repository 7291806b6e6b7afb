// AdamW over many tensors in one launch (gfx950): per element, in fp32,
//
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   w = w - lr ((m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps) + decay w)
//
// Bound by memory.  The tensors are cut into chunks of 2048 elements, eight a thread, dealt to the resident workgroups; a chunk's
// tensor is found in a table that travels with the launch.  The step count t lies in device memory and the last workgroup counts
// it up, so that a captured step goes on counting.
// A bf16 parameter has the low 16 bits of its fp32 value w beside it (2 bytes where a copy of w would take 4): w is rounded to bf16
// with halves away from zero, so a low half of 0x8000 or more says that the bf16 number is one step above w's upper half, and the
// two are w itself.
//
// Moments in 8 bits: per 128 places an exponent x, and codes of floating-point values with three bits of mantissa: m a sign and four
// bits of exponent (1.875 2^x down to 2^(x - 17)), v, which has no sign, five (down to 2^(x - 33): v is of the size of m^2).  A
// code is the upper bits of the fp32 number that has its smallest steps among the denormals, so it is scaled, added to and cut.
// With beta2 = 0.999 v moves by a thousandth of itself a step and a code's step is a tenth: rounded to the nearest it would never move.
// It is rounded up or down by chance in proportion to what lies between (16 bits of a hash of seed, step and place for each
// number), so that it moves as it should on average.  v is never rounded to zero, which would make a step as large as eps allows.
// The moments of a step are those before they are rounded.  The hash: splitmix64's output function, one number for two places.
#include "row_vectors.h"

namespace dc {
namespace {

typedef unsigned long long u64;

constexpr int kPer = 8, kThreads = 256, kChunk = kPer * kThreads;
constexpr int kExponentNan = 255;              // of a block of moments that holds a number that is not finite

__host__ __device__ __forceinline__ u64 mix(u64 z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ULL;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBULL;
  return z ^ (z >> 31);
}

struct Place {
  const AdamwTensor* t;
  bool p16, g16;
  long long i;                 // the thread's first element in the tensor
  int left;                    // how many of its eight are there: 1 to 8
  long long at;                // its first place in the state arrays
  bool block;                  // its 128 places hold an element
};
__device__ __forceinline__ Place place_of(const AdamwArgs& a, int chunk) {
  int lo = 0, hi = a.tensors;  // the last tensor whose first chunk is not behind this one
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.first[mid] <= chunk) lo = mid;
    else hi = mid;
  }
  Place p;
  p.t = &a.t[lo];
  p.p16 = a.p16[lo] != 0;
  p.g16 = a.g16[lo] != 0;
  p.i = (long long)(chunk - a.first[lo]) * kChunk + threadIdx.x * kPer;
  const long long left = p.t->n - p.i;
  p.left = left > kPer ? kPer : (left < 0 ? 0 : (int)left);
  p.at = (long long)p.t->block * kMomentBlock + p.i;
  p.block = (p.i & ~(long long)(kMomentBlock - 1)) < p.t->n;
  return p;
}

// Eight elements from i, zeros behind the last.
__device__ __forceinline__ void load8(float (&x)[kPer], const void* from, long long i, int left, bool bf16) {
  if (bf16) {
    const u16* p = static_cast<const u16*>(from) + i;
    u32x4 v = {0, 0, 0, 0};
    if (left == kPer) {
      v = *reinterpret_cast<const u32x4_any*>(p);
    } else {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (k < left) v[k / 2] |= (unsigned)p[k] << (16 * (k & 1));
    }
    unpack(x, v, u16());
  } else {
    const float* p = static_cast<const float*>(from) + i;
    if (left == kPer) {
      const u32x4 lo = *reinterpret_cast<const u32x4_any*>(p), hi = *reinterpret_cast<const u32x4_any*>(p + 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = __uint_as_float(lo[k]);
        x[4 + k] = __uint_as_float(hi[k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kPer; ++k) x[k] = k < left ? p[k] : 0.f;
    }
  }
}
__device__ __forceinline__ void store8(const float (&x)[kPer], float* p, int left) {
  if (left == kPer) {
    *reinterpret_cast<u32x4_any*>(p) = u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    *reinterpret_cast<u32x4_any*>(p + 4) = u32x4{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (k < left) p[k] = x[k];
  }
}

// w from the bf16 number and the low half.  Zero has nothing below it to borrow from (its low half is less than 0x8000 unless the
// caller wrote the parameter anew).
__device__ __forceinline__ float whole(unsigned p, unsigned low) {
  const unsigned borrow = low >= 0x8000u && (p & 0x7FFFu) != 0 ? 1u : 0u;
  return __uint_as_float(((p - borrow) << 16) | low);
}
__device__ __forceinline__ void load_whole(float (&w)[kPer], const Place& p, const u16* low) {
  const u32x4 l = *reinterpret_cast<const u32x4*>(low + p.at);
  const u16* from = static_cast<const u16*>(p.t->p) + p.i;
  u32x4 v = {0, 0, 0, 0};
  if (p.left == kPer) {
    v = *reinterpret_cast<const u32x4_any*>(from);
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (k < p.left) v[k / 2] |= (unsigned)from[k] << (16 * (k & 1));
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    w[2 * k] = whole(v[k] & 0xFFFFu, l[k] & 0xFFFFu);
    w[2 * k + 1] = whole(v[k] >> 16, l[k] >> 16);
  }
}
__device__ __forceinline__ void store_whole(const float (&w)[kPer], const Place& p, u16* low) {
  unsigned hi[kPer], lo[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const unsigned b = __float_as_uint(w[k]);
    const bool nan = (b & 0x7FFFFFFFu) > 0x7F800000u;
    hi[k] = nan ? (b >> 16) | 0x40u : (b + 0x8000u) >> 16;
    lo[k] = nan || k >= p.left ? 0u : b & 0xFFFFu;
  }
  u16* to = static_cast<u16*>(p.t->p) + p.i;
  if (p.left == kPer) {
    *reinterpret_cast<u32x4_any*>(to) = u32x4{hi[0] | hi[1] << 16, hi[2] | hi[3] << 16, hi[4] | hi[5] << 16, hi[6] | hi[7] << 16};
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (k < p.left) to[k] = (u16)hi[k];
  }
  *reinterpret_cast<u32x4*>(low + p.at) = u32x4{lo[0] | lo[1] << 16, lo[2] | lo[3] << 16, lo[4] | lo[5] << 16, lo[6] | lo[7] << 16};
}

// ---- moments in 8 bits ----
// What a code's fp32 bits are times 2^(exponent - kUnit).
template <bool kM>
constexpr int kUnit = kM ? 15 : 31;
template <bool kM>
__device__ __forceinline__ void decode(float (&x)[kPer], u32x2 code, int exponent) {
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const unsigned c = code[k / 4] >> (8 * (k & 3)) & 0xFFu;
    const float f = __uint_as_float((kM ? c & 0x7Fu : c) << 20);
    const float y = exponent == kExponentNan ? __uint_as_float(0x7FC00000u) : __builtin_amdgcn_ldexpf(f, exponent - kUnit<kM>);
    x[k] = kM && (c & 0x80u) ? -y : y;
  }
}
__device__ __forceinline__ unsigned max_dpp16(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true));
}
// chance: 16 bits a place.  Returns the exponent of the 16 lanes' block.
template <bool kM>
__device__ __forceinline__ int encode(u32x2& code, const float (&x)[kPer], const unsigned (&chance)[kPer]) {
  constexpr int kMost = kM ? 127 : 255;
  unsigned top = 0;            // the bits of |x| order as |x| does, what is not finite above all
#pragma unroll
  for (int k = 0; k < kPer; ++k) top = max(top, __float_as_uint(x[k]) & 0x7FFFFFFFu);
  top = max_dpp16(top);
  // the smallest exponent whose largest value, 1.875 2^x, reaches the top
  int e = (int)(top >> 23) + ((top & 0x7FFFFFu) > 0x700000u ? 1 : 0);
  e = min(max(e, kM ? 1 : 11), 254);
  code = u32x2{0, 0};
  if (top >= 0x7F800000u) return kExponentNan;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const unsigned bits = __float_as_uint(__builtin_amdgcn_ldexpf(fabsf(x[k]), kUnit<kM> - e));
    unsigned c = min((bits + (chance[k] << 4 | 8u)) >> 20, (unsigned)kMost);
    if (!kM) c = max(c, x[k] > 0.f ? 1u : 0u);
    if (kM) c |= __float_as_uint(x[k]) >> 31 << 7;
    code[k / 4] |= c << (8 * (k & 3));
  }
  return e;
}

__device__ __forceinline__ double power(double b, unsigned n) {
  double r = 1.0;
  for (; n; n >>= 1, b *= b)
    if (n & 1) r *= b;
  return r;
}

template <bool kEight>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamwArgs a) {
  // the 8-bit codes are those of operations in fp32 rounded one by one
#pragma clang fp contract(off)
  const int before = a.steps[0], t = before < 2147483647 ? before + 1 : before;
  const float c1 = (float)(1.0 / (1.0 - power(a.beta1, (unsigned)t))), c2 = (float)(1.0 / (1.0 - power(a.beta2, (unsigned)t)));
  const float scale = a.grad_scale ? a.grad_scale[0] : 1.f;
  const u64 key = kEight ? mix(a.seed ^ mix((u64)t)) : 0;
  for (int chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const Place p = place_of(a, chunk);
    if (kEight ? !p.block : p.left == 0) continue;
    float g[kPer], w[kPer], m[kPer], v[kPer];
    load8(g, p.t->g, p.i, p.left, p.g16);
    if (p.p16) load_whole(w, p, a.low);
    else load8(w, p.t->p, p.i, p.left, false);
    if constexpr (kEight) {
      const u32x2 mc = *reinterpret_cast<const u32x2*>(static_cast<const unsigned char*>(a.m) + p.at);
      const u32x2 vc = *reinterpret_cast<const u32x2*>(static_cast<const unsigned char*>(a.v) + p.at);
      decode<true>(m, mc, a.m_exponent[p.at / kMomentBlock]);
      decode<false>(v, vc, a.v_exponent[p.at / kMomentBlock]);
    } else {
      load8(m, a.m, p.at, kPer, false);
      load8(v, a.v, p.at, kPer, false);
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const float gk = g[k] * scale;
      m[k] = m[k] * a.b1 + gk * a.o1;
      v[k] = v[k] * a.b2 + (gk * gk) * a.o2;
      const float step = (m[k] * c1) / (sqrtf(v[k] * c2) + a.eps);
      w[k] = fmaf(-a.lr, fmaf(p.t->decay, w[k], step), w[k]);
    }
    if constexpr (kEight) {
      unsigned cm[kPer], cv[kPer];
#pragma unroll
      for (int k = 0; k < kPer; k += 2) {
        const u64 r = mix(key + (u64)(p.at / 2 + k / 2) * 0xD1342543DE82EF95ULL);
        cm[k] = (unsigned)r & 0xFFFFu;
        cv[k] = (unsigned)r >> 16;
        cm[k + 1] = (unsigned)(r >> 32) & 0xFFFFu;
        cv[k + 1] = (unsigned)(r >> 48);
      }
#pragma unroll
      for (int k = 0; k < kPer; ++k)           // places behind the tensor's last element hold zeros
        if (k >= p.left) m[k] = v[k] = 0.f;
      u32x2 mc, vc;
      const int em = encode<true>(mc, m, cm), ev = encode<false>(vc, v, cv);
      *reinterpret_cast<u32x2*>(static_cast<unsigned char*>(a.m) + p.at) = mc;
      *reinterpret_cast<u32x2*>(static_cast<unsigned char*>(a.v) + p.at) = vc;
      if ((threadIdx.x & 15) == 0) {
        a.m_exponent[p.at / kMomentBlock] = (unsigned char)em;
        a.v_exponent[p.at / kMomentBlock] = (unsigned char)ev;
      }
    } else {
      store8(m, static_cast<float*>(a.m) + p.at, p.left);
      store8(v, static_cast<float*>(a.v) + p.at, p.left);
    }
    if (p.p16) {
      if (p.left > 0) store_whole(w, p, a.low);
    } else {
      store8(w, static_cast<float*>(p.t->p) + p.i, p.left);
    }
  }
  if (!a.count_up) return;
  __syncthreads();                             // every wave has read the count
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&a.steps[1], 1) == (int)gridDim.x - 1) {
      a.steps[1] = 0;
      a.steps[0] = t;
    }
  }
}

template <bool kEight>
__global__ __launch_bounds__(kThreads) void values_kernel(const AdamwArgs a) {
  for (int chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const Place p = place_of(a, chunk);
    if (!p.block) continue;
    float x[kPer];
    if (a.out_w) {
      if (p.p16) load_whole(x, p, a.low);
      else load8(x, p.t->p, p.i, p.left, false);
#pragma unroll
      for (int k = 0; k < kPer; ++k) x[k] = k < p.left ? x[k] : 0.f;
      store8(x, a.out_w + p.at, kPer);
    }
    if (a.out_m) {
      if constexpr (kEight) decode<true>(x, *reinterpret_cast<const u32x2*>(static_cast<const unsigned char*>(a.m) + p.at), a.m_exponent[p.at / kMomentBlock]);
      else load8(x, a.m, p.at, kPer, false);
#pragma unroll
      for (int k = 0; k < kPer; ++k) x[k] = k < p.left ? x[k] : 0.f;
      store8(x, a.out_m + p.at, kPer);
    }
    if (a.out_v) {
      if constexpr (kEight) decode<false>(x, *reinterpret_cast<const u32x2*>(static_cast<const unsigned char*>(a.v) + p.at), a.v_exponent[p.at / kMomentBlock]);
      else load8(x, a.v, p.at, kPer, false);
#pragma unroll
      for (int k = 0; k < kPer; ++k) x[k] = k < p.left ? x[k] : 0.f;
      store8(x, a.out_v + p.at, kPer);
    }
  }
}

unsigned blocks_of(const AdamwArgs& a) {
  const long long most = 8LL * a.n_cu;
  return (unsigned)(a.chunks < 1 ? 1 : (a.chunks < most ? a.chunks : most));
}

}  // namespace

long long adamw_chunks(long long n) { return (n + kChunk - 1) / kChunk; }

hipError_t launch_adamw(const AdamwArgs& a, bool eight, hipStream_t s) {
  static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");
  if (eight) hipLaunchKernelGGL((adamw_kernel<true>), dim3(blocks_of(a)), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((adamw_kernel<false>), dim3(blocks_of(a)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_adamw_values(const AdamwArgs& a, bool eight, hipStream_t s) {
  if (a.chunks < 1) return hipSuccess;
  if (eight) hipLaunchKernelGGL((values_kernel<true>), dim3(blocks_of(a)), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((values_kernel<false>), dim3(blocks_of(a)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace dc
