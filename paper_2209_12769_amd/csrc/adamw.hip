// AdamW over many tensors in one launch (gfx950): per element, in fp32,
//
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   w = w - lr ((m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps) + decay w)
//
// (the corrections as factors: k2 sqrt(v) and c1 m / (k2 sqrt(v) + eps), of which nothing is too small for fp32 before m and v are).
// Bound by memory (120 M parameters in bf16, moments in fp32, 3.1 GB: 545 us, 5.7 TB/s; 260 M with moments in 8 bits, 3.6 GB:
// 660 us, 5.5 TB/s, of which vector instructions are issued for 510).  The tensors are cut into chunks of 2048 elements, eight a
// thread, a workgroup each, so that memory is gone through in the order in which workgroups are handed out; a chunk's tensor is
// found in a table that travels with the launch.  The step count t lies in device memory, so that a captured step goes on counting: in
// a small call the last workgroup counts it up, otherwise a launch of its own (2.5 us of the host's time, which a small call is bound
// by; one by one would be 9 us of 500 workgroups).
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
constexpr u64 kDraw = 0xD1342543DE82EF95ULL;    // from one draw to the next
constexpr int kCounted = 2048;                 // chunks of a small call
constexpr int kSmall = 4;                      // and of its workgroups
constexpr int kExponentNan = 255;              // of a block of moments that holds a number that is not finite

__host__ __device__ __forceinline__ u64 mix(u64 z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ULL;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBULL;
  return z ^ (z >> 31);
}

// A part of a tensor, the same for a workgroup.
struct Chunk {
  char* p;                     // its first element
  const char* g;
  int n;                       // elements
  bool p16, g16;
  float decay;
  long long at;                // its first place in the state arrays
};
__device__ __forceinline__ Chunk chunk_of(const AdamwArgs& a, int chunk) {
  // the last tensor whose first chunk is not behind this one: all are looked at at once (a search would wait for the table in
  // every step)
  const int lane = threadIdx.x & 63;
  static_assert(kAdamwTensors <= 128, "two a lane");
  const bool in1 = lane < a.tensors, in2 = 64 + lane < a.tensors;
  const int f1 = a.t[in1 ? lane : 0].first, f2 = a.t[in2 ? 64 + lane : 0].first;
  const AdamwTensor t = a.t[__builtin_amdgcn_readfirstlane(__popcll(__ballot(in1 && f1 <= chunk)) + __popcll(__ballot(in2 && f2 <= chunk)) - 1)];
  const long long i = (long long)(chunk - t.first) * kChunk, left = t.n - i;
  Chunk c;
  c.p16 = t.types & 1;
  c.g16 = t.types & 2;
  c.p = static_cast<char*>(t.p) + i * (c.p16 ? 2 : 4);
  c.g = static_cast<const char*>(t.g) + i * (c.g16 ? 2 : 4);
  c.n = left < kChunk ? (int)left : kChunk;
  c.decay = t.decay;
  c.at = (long long)t.block * kMomentBlock + i;
  return c;
}

// Eight elements as they come from memory: fp32, or bf16 in the first four words.  kAll: all are there; else `left` of them, and
// zeros behind.
struct Raw {
  u32x4 v[2];
};
template <bool kAll>
__device__ __forceinline__ Raw request(const char* from, unsigned i, int left, bool bf16) {
  Raw r;
  if (kAll || left >= kPer) {
    if (bf16) {
      r.v[0] = *reinterpret_cast<const u32x4_any*>(from + 2 * i);
    } else {
      r.v[0] = *reinterpret_cast<const u32x4_any*>(from + 4 * i);
      r.v[1] = *reinterpret_cast<const u32x4_any*>(from + 4 * i + 16);
    }
    return r;
  }
  r.v[0] = r.v[1] = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (k < left) {
      if (bf16) r.v[0][k / 2] |= (unsigned)reinterpret_cast<const u16*>(from)[i + k] << (16 * (k & 1));
      else r.v[k / 4][k & 3] = reinterpret_cast<const unsigned*>(from)[i + k];
    }
  return r;
}
__device__ __forceinline__ void open(float (&x)[kPer], const Raw& r, bool bf16) {
  if (bf16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(r.v[0][k] << 16);
      x[2 * k + 1] = __uint_as_float(r.v[0][k] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k) x[k] = __uint_as_float(r.v[k / 4][k & 3]);
  }
}
template <bool kAll>
__device__ __forceinline__ void store8(const float (&x)[kPer], float* p, int left) {
  if (kAll || left >= kPer) {
    *reinterpret_cast<u32x4_any*>(p) = u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    *reinterpret_cast<u32x4_any*>(p + 4) = u32x4{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (k < left) p[k] = x[k];
  }
}

// w of a word of two halves, the bf16 number above, the low half below: where that is 0x8000 or more the number is one step too
// far.  Zero has nothing below it to give (its low half is less than 0x8000 unless the caller wrote the parameter anew).
__device__ __forceinline__ float whole(unsigned word) {
  return __uint_as_float(word - min(word << 1 & 0x10000u, word & 0x7FFF0000u));
}
__device__ __forceinline__ void wholes(float& w0, float& w1, unsigned p, unsigned low) {     // of two places
  w0 = whole(__builtin_amdgcn_perm(p, low, 0x05040100u));
  w1 = whole(__builtin_amdgcn_perm(p, low, 0x07060302u));
}
template <bool kAll>
__device__ __forceinline__ void store_whole(const float (&w)[kPer], u16* to, u16* low, int left) {
  unsigned hi[kPer], lo[kPer];       // a number's upper half of one, lower half of the other
  float sum = 0.f;                   // not a number if one of them is none
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    sum += w[k];
    hi[k] = __float_as_uint(w[k]) + 0x8000u;
    lo[k] = !kAll && k >= left ? 0u : __float_as_uint(w[k]);
  }
  if (__ballot(sum != sum) != 0) {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (w[k] != w[k]) {
        hi[k] = 0x7FC00000u;
        lo[k] = 0u;
      }
  }
  u32x4 h;
#pragma unroll
  for (int k = 0; k < 4; ++k) h[k] = __builtin_amdgcn_perm(hi[2 * k + 1], hi[2 * k], 0x07060302u);
  if (kAll || left >= kPer) {
    *reinterpret_cast<u32x4_any*>(to) = h;
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (k < left) to[k] = (u16)(hi[k] >> 16);
  }
  u32x4 l;
#pragma unroll
  for (int k = 0; k < 4; ++k) l[k] = __builtin_amdgcn_perm(lo[2 * k + 1], lo[2 * k], 0x05040100u);
  *reinterpret_cast<u32x4*>(low) = l;
}

// ---- moments in 8 bits ----
// What a code's fp32 bits are times 2^(exponent - kUnit).
template <bool kM>
constexpr int kUnit = kM ? 15 : 31;
// Four codes.
template <bool kM>
__device__ __forceinline__ void decode(float (&x)[4], unsigned code, int exponent) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const unsigned c = code >> (8 * k) & 0xFFu;
    // m: the sign stays at the top while the rest goes to the place of an exponent and three bits
    const unsigned bits = kM ? (unsigned)((int)(c << 24) >> 4) & 0x87F00000u : c << 20;
    x[k] = __builtin_amdgcn_ldexpf(__uint_as_float(bits), exponent - kUnit<kM>);
  }
  // a branch for the wave: it is all but never taken
  if (__ballot(exponent == kExponentNan) != 0 && exponent == kExponentNan) x[0] = x[1] = x[2] = x[3] = __uint_as_float(0x7FC00000u);
}
__device__ __forceinline__ unsigned max_dpp16(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true));
}
// 1 if x, which is not negative, is not zero; as one instruction (the compiler makes a comparison and a choice of it).
__device__ __forceinline__ unsigned not_zero(float x) {
  unsigned r;
  asm("v_min_u32 %0, 1, %1" : "=v"(r) : "v"(x));
  return r;
}
// r: a draw for two places, 16 bits for m and for v of the first and of the second.  Returns the exponent of the 16 lanes' block.
template <bool kM>
__device__ __forceinline__ int encode(u32x2& code, const float (&x)[kPer], const u64 (&r)[kPer / 2]) {
  unsigned top = 0;            // the bits of |x| order as |x| does, what is not finite above all; v has no sign
#pragma unroll
  for (int k = 0; k < kPer; ++k) top = max(top, kM ? __float_as_uint(x[k]) & 0x7FFFFFFFu : __float_as_uint(x[k]));
  top = max_dpp16(top);
  // the smallest exponent whose largest value, 1.875 2^x, reaches the top; beyond the largest of all, that
  int e = (int)(top >> 23) + ((top & 0x7FFFFFu) > 0x700000u ? 1 : 0);
  e = min(max(e, kM ? 1 : 11), 254);
  code = u32x2{0, 0};
  if (top >= 0x7F800000u) return kExponentNan;
  constexpr float kLargest = 0x1.Ep127f;
  float y[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) y[k] = fabsf(x[k]);
  if (top > __float_as_uint(kLargest)) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) y[k] = fminf(y[k], kLargest);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const unsigned half = (unsigned)(r[k / 2] >> (32 * (k & 1)));
    // 2^-17 of a step above the 16 bits, which leave 20 to be cut off
    const unsigned chance = kM ? (half & 0xFFFFu) << 4 : (half >> 16) << 4;
    unsigned c = (__float_as_uint(__builtin_amdgcn_ldexpf(y[k], kUnit<kM> - e)) + chance + 8u) >> 20;
    if constexpr (kM) c |= __float_as_uint(x[k]) >> 24 & 0x80u;
    else c = max(c, not_zero(x[k]));
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

// What all elements of a step share; worked out by one wave of a workgroup.
struct Step {
  float c1, k2;                // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  float scale;                 // of the gradients
  // Whether the machine's root and reciprocal serve, one unit in the last place each at a tenth of the instructions of exact ones.
  // They take what is no normal number as zero: a root of 1.1e-19 at most, times k2 a 16th of the rounding of eps or less.
  bool fast;
  u64 key;
};

// A chunk's step.  kAll: of kChunk elements.  `first`: the workgroup's first one, its requests go out before `step` is there; then
// counted() is called.
template <bool kEight, bool kAll, typename F>
__device__ __forceinline__ void update(const AdamwArgs& a, const Chunk& c, const Step& step, bool first, F counted) {
  // the 8-bit codes are those of operations in fp32 rounded one by one
#pragma clang fp contract(off)
  const unsigned i = threadIdx.x % kThreads * kPer;
  const int left = kAll ? kPer : min(max(c.n - (int)i, 0), kPer);
  const bool there = kAll || (kEight ? (int)(i & ~(unsigned)(kMomentBlock - 1)) < c.n : left > 0);
  unsigned char* const m8 = static_cast<unsigned char*>(a.m) + c.at;
  unsigned char* const v8 = static_cast<unsigned char*>(a.v) + c.at;
  float* const m32 = static_cast<float*>(a.m) + c.at;
  float* const v32 = static_cast<float*>(a.v) + c.at;
  unsigned char* const me = a.m_exponent + c.at / kMomentBlock;
  unsigned char* const ve = a.v_exponent + c.at / kMomentBlock;
  Raw rg, rw, rm, rv;
  u32x4 rl = {0, 0, 0, 0};
  u32x2 mc, vc;
  int em, ev;
  if (there) {
    rg = request<kAll>(c.g, i, left, c.g16);
    rw = request<kAll>(c.p, i, left, c.p16);
    if (c.p16) rl = *reinterpret_cast<const u32x4*>(a.low + c.at + i);
    if constexpr (kEight) {
      mc = *reinterpret_cast<const u32x2*>(m8 + i);
      vc = *reinterpret_cast<const u32x2*>(v8 + i);
      em = me[i / kMomentBlock];
      ev = ve[i / kMomentBlock];
    } else {
      rm = request<true>(reinterpret_cast<const char*>(m32), i, kPer, false);
      rv = request<true>(reinterpret_cast<const char*>(v32), i, kPer, false);
    }
  }
  if (first) {
    __syncthreads();
    counted();
  }
  if (!there) return;
  u64 r[kPer / 2];
  if constexpr (kEight) {      // the draws, while the requests are under way: kept in front of what waits for them
    u64 place = step.key + (u64)((c.at + i) / 2) * kDraw;
#pragma unroll
    for (int k = 0; k < kPer / 2; ++k, place += kDraw) {
      r[k] = mix(place);
      asm volatile("" : "+v"(r[k]));
    }
  }
  float g[kPer], w[kPer], m[kPer], v[kPer];
  open(g, rg, c.g16);
  if (c.p16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) wholes(w[2 * k], w[2 * k + 1], rw.v[0][k], rl[k]);
  } else {
    open(w, rw, false);
  }
  if constexpr (kEight) {
#pragma unroll
    for (int k = 0; k < kPer; k += 4) {
      float y[4], z[4];
      decode<true>(y, mc[k / 4], em);
      decode<false>(z, vc[k / 4], ev);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        m[k + u] = y[u];
        v[k + u] = z[u];
      }
    }
  } else {
    open(m, rm, false);
    open(v, rv, false);
  }
  if (a.grad_scale) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) g[k] *= step.scale;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    m[k] = m[k] * a.b1 + g[k] * a.o1;
    v[k] = v[k] * a.b2 + (g[k] * g[k]) * a.o2;
  }
  float by[kPer];              // m / (sqrt(v) k2 + eps)
  if (step.fast) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) by[k] = m[k] * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[k]), step.k2, a.eps));
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k) by[k] = m[k] / fmaf(sqrtf(v[k]), step.k2, a.eps);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) w[k] = fmaf(-a.lr, fmaf(c.decay, w[k], by[k] * step.c1), w[k]);
  if constexpr (kEight) {
    if (!kAll) {               // places behind the tensor's last element hold zeros
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (k >= left) m[k] = v[k] = 0.f;
    }
    em = encode<true>(mc, m, r);
    ev = encode<false>(vc, v, r);
    *reinterpret_cast<u32x2*>(m8 + i) = mc;
    *reinterpret_cast<u32x2*>(v8 + i) = vc;
    if ((threadIdx.x & 15) == 0) {
      me[i / kMomentBlock] = (unsigned char)em;
      ve[i / kMomentBlock] = (unsigned char)ev;
    }
  } else {
    store8<kAll>(m, m32 + i, left);
    store8<kAll>(v, v32 + i, left);
  }
  if (c.p16) {
    if (left > 0) store_whole<kAll>(w, reinterpret_cast<u16*>(c.p) + i, a.low + c.at + i, left);
  } else {
    store8<kAll>(w, reinterpret_cast<float*>(c.p) + i, left);
  }
}

// kMany: chunks of a workgroup side by side.  One, or four in small calls, which count the step up themselves.
template <bool kEight, int kMany>
__global__ __launch_bounds__(kThreads * kMany, kMany > 1 ? 4 : (kEight ? 5 : 8)) void adamw_kernel(const AdamwArgs a) {
  __shared__ Step step;
  const int before = a.steps[0], t = before < 2147483647 ? before + 1 : before;
  if (threadIdx.x < 64) {
    Step s;
    s.c1 = (float)(1.0 / (1.0 - power(a.beta1, (unsigned)t)));
    s.k2 = (float)sqrt(1.0 / (1.0 - power(a.beta2, (unsigned)t)));
    s.fast = a.eps >= 3e-11f * s.k2;
    s.scale = a.grad_scale ? a.grad_scale[0] : 1.f;
    s.key = mix(a.seed ^ mix((u64)t));
    if (threadIdx.x == 0) step = s;
  }
  if constexpr (kMany == 1) {
    for (int chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
      const Chunk c = chunk_of(a, chunk);
      if (c.n == kChunk) update<kEight, true>(a, c, step, chunk == (int)blockIdx.x, []() {});
      else update<kEight, false>(a, c, step, chunk == (int)blockIdx.x, []() {});
    }
  } else {
    // The last workgroup counts the step up.  Thread 0 counts its own once it has read the count of steps, and no other thread uses what
    // it read; nothing else is handed from one workgroup to another: no fence, which would write an XCD's whole L2 back for each of
    // them.  Additions to one place take 9 to 18 ns each, one after the other: hence four chunks each, and they are requested behind the
    // elements and waited for at the end (1.14 M parameters: 13.0 us by a chunk each and counted at the end, 9.1 so, 29 with a fence).
    unsigned before_it = 0;
    const int part = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
    update<kEight, false>(a, chunk_of(a, (int)blockIdx.x * kMany + part), step, true, [&]() {
      if (a.count_up && threadIdx.x == 0) before_it = atomicInc(reinterpret_cast<unsigned*>(&a.steps[1]), gridDim.x - 1);
    });
    if (a.count_up && threadIdx.x == 0 && before_it == gridDim.x - 1) a.steps[0] = t;       // its addition made the other 0 again
  }
}

__global__ void count_up_kernel(int* steps) {
  if (steps[0] < 2147483647) steps[0] += 1;
}

// Four values a thread, so that a wave's stores are neighbours: a workgroup takes half a chunk (all three of 260 M parameters with
// moments in 8 bits, 4.7 GB: 800 us, 5.9 TB/s).
template <bool kEight>
__global__ __launch_bounds__(kThreads) void values_kernel(const AdamwArgs a) {
  for (long long half = blockIdx.x; half < 2LL * a.chunks; half += gridDim.x) {
    const Chunk c = chunk_of(a, (int)(half / 2));
    const unsigned i = (unsigned)(half & 1) * (kChunk / 2) + threadIdx.x * 4;
    if ((int)(i & ~(unsigned)(kMomentBlock - 1)) >= c.n) continue;
    const int left = min(max(c.n - (int)i, 0), 4);
    auto put = [&](float* to, const float (&x)[4]) {
      u32x4 v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = k < left ? __float_as_uint(x[k]) : 0u;
      *reinterpret_cast<u32x4*>(to + c.at + i) = v;
    };
    float w[4], m[4], v[4];
    if (a.out_w) {
      if (c.p16) {
        const u32x2 l = *reinterpret_cast<const u32x2*>(a.low + c.at + i);
        const u16* from = reinterpret_cast<const u16*>(c.p) + i;
        u32x2 h = {0, 0};
        if (left == 4) {
          h = *reinterpret_cast<const u32x2_any*>(from);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (k < left) h[k / 2] |= (unsigned)from[k] << (16 * (k & 1));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) wholes(w[2 * k], w[2 * k + 1], h[k], l[k]);
      } else {
        const float* from = reinterpret_cast<const float*>(c.p) + i;
        if (left == 4) {
          unpack(w, *reinterpret_cast<const u32x4_any*>(from), 0.f);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = k < left ? from[k] : 0.f;
        }
      }
    }
    if (a.out_m) {
      if constexpr (kEight) decode<true>(m, *reinterpret_cast<const unsigned*>(static_cast<const unsigned char*>(a.m) + c.at + i), a.m_exponent[(c.at + i) / kMomentBlock]);
      else unpack(m, *reinterpret_cast<const u32x4*>(static_cast<const float*>(a.m) + c.at + i), 0.f);
    }
    if (a.out_v) {
      if constexpr (kEight) decode<false>(v, *reinterpret_cast<const unsigned*>(static_cast<const unsigned char*>(a.v) + c.at + i), a.v_exponent[(c.at + i) / kMomentBlock]);
      else unpack(v, *reinterpret_cast<const u32x4*>(static_cast<const float*>(a.v) + c.at + i), 0.f);
    }
    if (a.out_w) put(a.out_w, w);
    if (a.out_m) put(a.out_m, m);
    if (a.out_v) put(a.out_v, v);
  }
}

unsigned blocks_of(long long work) {
  const int most = 1 << 23;                    // a launch has less than 2^32 threads
  return (unsigned)(work < 1 ? 1 : (work < most ? work : most));
}

}  // namespace

long long adamw_chunks(long long n) { return (n + kChunk - 1) / kChunk; }

hipError_t launch_adamw(const AdamwArgs& a, bool eight, hipStream_t s) {
  static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");
  if (a.chunks > 0 && a.chunks <= kCounted) {
    const dim3 grid(blocks_of((a.chunks + kSmall - 1) / kSmall));
    if (eight) hipLaunchKernelGGL((adamw_kernel<true, kSmall>), grid, dim3(kThreads * kSmall), 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<false, kSmall>), grid, dim3(kThreads * kSmall), 0, s, a);
    return hipGetLastError();
  }
  if (a.chunks > 0) {
    if (eight) hipLaunchKernelGGL((adamw_kernel<true, 1>), dim3(blocks_of(a.chunks)), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<false, 1>), dim3(blocks_of(a.chunks)), dim3(kThreads), 0, s, a);
  }
  if (a.count_up) hipLaunchKernelGGL(count_up_kernel, dim3(1), dim3(1), 0, s, a.steps);
  return hipGetLastError();
}
hipError_t launch_adamw_values(const AdamwArgs& a, bool eight, hipStream_t s) {
  if (a.chunks < 1) return hipSuccess;
  if (eight) hipLaunchKernelGGL((values_kernel<true>), dim3(blocks_of(2LL * a.chunks)), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((values_kernel<false>), dim3(blocks_of(2LL * a.chunks)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace dc
