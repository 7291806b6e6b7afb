// Internal declarations of the operators on rows of a batch: dense layer (dense_layer.hip), norm over the rows of each
// graph (graph_norm.hip), rows kept in 8 bits (kept_rows.hip), and what they share.
#pragma once
#include "common.h"

namespace dc {

// ---- activations, in fp32 ----
// 1 / (1 + e^-z) from the machine's power of two and reciprocal, each off by one unit in the last place: relative to the result
// about (3 + |z|) 2^-24, where the library's exponential and an exact division would take three times the instructions
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
}
// The standard normal distribution at -|z| is e^(-z^2 / 2) times a smooth function of |z|, here a polynomial of degree 8 in
// t = 1 / (1 + p |z|) without a constant: the form of Abramowitz and Stegun 26.2.17 and its p, with three more
// coefficients, fitted for the smallest largest relative error over 0 <= |z| <= 14 (1.3e-7).  GELU
// by it is off by at most 4.9 roundings of |z|, and 0.5 z (1 + erf) in fp32 by up to 5.8, at about twice the
// instructions: those of the library's error function bound the norms with GELU and took 45 us of 0.33 ms for a layer of
// 27 M outputs.
struct NormalParts {
  float cdf, density;    // of the standard normal distribution at z
};
__device__ __forceinline__ NormalParts normal_parts(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.2316419f, fabsf(z), 1.f));
  const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * (z * z));
  float poly = fmaf(t, -0.0704237595f, 0.247685075f);
  poly = fmaf(t, poly, -0.201657608f);
  poly = fmaf(t, poly, 0.225250751f);
  poly = fmaf(t, poly, 0.0135532282f);
  poly = fmaf(t, poly, 0.102649979f);
  poly = fmaf(t, poly, 0.0904201567f);
  poly = fmaf(t, poly, 0.0925222412f);
  const float half = t * poly * e;
  return {z > 0.f ? 1.f - half : half, 0.39894228040143268f * e};
}
__device__ __forceinline__ float activation(float z, int act) {
  switch (act) {
    case DC_ACT_RELU: return z > 0.f ? z : (z != z ? z : 0.f);
    case DC_ACT_GELU: return z * normal_parts(z).cdf;
    case DC_ACT_SILU: return z * sigmoid(z);
    default: return z;
  }
}
__device__ __forceinline__ float activation_slope(float z, int act) {
  switch (act) {
    case DC_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case DC_ACT_GELU: {
      const NormalParts n = normal_parts(z);
      return fmaf(z, n.density, n.cdf);
    }
    case DC_ACT_SILU: {
      const float s = sigmoid(z);
      return s * fmaf(z, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}
// The same for kN values, the choice made once.
template <int kN>
__device__ __forceinline__ void activate(float (&z)[kN], int act) {
  switch (act) {
    case DC_ACT_RELU:
#pragma unroll
      for (int k = 0; k < kN; ++k) z[k] = activation(z[k], DC_ACT_RELU);
      break;
    case DC_ACT_GELU:
#pragma unroll
      for (int k = 0; k < kN; ++k) z[k] = activation(z[k], DC_ACT_GELU);
      break;
    case DC_ACT_SILU:
#pragma unroll
      for (int k = 0; k < kN; ++k) z[k] = activation(z[k], DC_ACT_SILU);
      break;
    default: break;
  }
}
template <int kN>
__device__ __forceinline__ void slopes(float (&z)[kN], int act) {
  switch (act) {
    case DC_ACT_RELU:
#pragma unroll
      for (int k = 0; k < kN; ++k) z[k] = activation_slope(z[k], DC_ACT_RELU);
      break;
    case DC_ACT_GELU:
#pragma unroll
      for (int k = 0; k < kN; ++k) z[k] = activation_slope(z[k], DC_ACT_GELU);
      break;
    case DC_ACT_SILU:
#pragma unroll
      for (int k = 0; k < kN; ++k) z[k] = activation_slope(z[k], DC_ACT_SILU);
      break;
    default:
#pragma unroll
      for (int k = 0; k < kN; ++k) z[k] = 1.f;
      break;
  }
}

// ---- kept rows: 8-bit codes, one power of two per row and 32 columns ----
constexpr int kKeptBlock = 32;
constexpr int kKeptNan = 255;                      // exponent code of a block that holds a number that is not finite
constexpr int kKeptLeast = -126, kKeptMost = 121;  // exponents: every code times its power of two is a normal, finite number
// The power of two of an exponent code (127 + exponent); NaN for kKeptNan.
__device__ __forceinline__ float kept_scale(unsigned code) {
  return code == kKeptNan ? __uint_as_float(0x7FC00000u) : __uint_as_float(code << 23);
}
struct KeptView {
  const signed char* code;       // [rows, ld_code]
  const unsigned char* exponent; // [rows, ld_exponent]
  long long ld_code, ld_exponent;
};

// ---- dense layer ----
// Y = act(X W + b) + R on the rows of a batch; X is up to three matrices of d columns side by side (K = nseg * d).
struct DenseArgs {
  long long rows;                // or, with nrows, the most rows there can be
  const int* nrows;              // device row count, or null
  int d, nseg, N, bf16, act;
  const void* X[3];
  long long ldx;
  const void* W;                 // [K, N]
  long long ldw;
  const float* bias;             // or null
  const void* R;                 // or null
  long long ldr;
  void* Z;                       // or null
  long long ldz;
  void* Y;
  long long ldy;
  const int* stop;               // device word: not 0 = leave everything alone; or null
  int n_cu;
};
hipError_t launch_dense(const DenseArgs& a, hipStream_t s);

// dZ = dY act'(Z); dX = dZ W^T, dW = X^T dZ, db = sum of the rows of dZ.
struct DenseBackArgs {
  long long rows;
  int K, N, bf16, act;
  int round_dz;                  // bf16, GELU and SiLU: dZ as one bf16 number, else as the sum of two
  const void* dY;
  long long lddy;
  const void* Z;                 // act other than none
  long long ldz;
  const void* X;                 // null where kept is taken
  long long ldx;
  KeptView kept;                 // code == null: X
  const void* W;
  long long ldw;
  void* dX;                      // [rows, K] or null
  long long lddx;
  void* dW;                      // [K, N] or null
  long long lddw;
  float* db;                     // [N] or null
  float* workspace;              // dense_back_floats() of them
  int n_cu;
};
size_t dense_back_floats(long long rows, int K, int N, int bf16, int act, int n_cu);
size_t dense_dz_floats(long long rows, int N);              // of them, dZ of a smooth activation: fp32, or two bf16 numbers
hipError_t launch_dense_back(const DenseBackArgs& a, hipStream_t s);

// ---- norm over the rows of each graph ----
struct GraphNormArgs {
  long long rows;                // rows of the arrays: a graph that reaches further is malformed
  int n_graphs;                  // or, with n_graphs_dev, the most there can be
  const int* n_graphs_dev;
  const int* node_off;
  int C, G, bf16, act;
  float eps;
  const void* X;                 // null where kept is taken (backward)
  long long ldx;
  KeptView kept;
  const float* gamma;            // or null: 1
  const float* beta;             // or null: 0
  float* mean;                   // [n_graphs, G]
  float* rstd;
  void* Y;                       // forward
  long long ldy;
  const void* dY;                // backward
  long long lddy;
  const void* dRes;              // backward: added to dX, or null
  long long lddres;
  void* dX;
  long long lddx;
  float* dgamma;                 // [C] or null (both or none)
  float* dbeta;
  char* workspace;
  int* status;                   // bad offsets set status[1] (and [0] if stop is taken)
  const int* stop;
  int n_cu;
};
size_t graph_norm_bytes(long long rows, int n_graphs, int C, int G, bool backward, int n_cu);
hipError_t launch_graph_norm(const GraphNormArgs& a, hipStream_t s);
hipError_t launch_graph_norm_back(const GraphNormArgs& a, hipStream_t s);

// out1 [n1] | out2 [n2] = sums over `blocks` rows of part [blocks, n1 + n2], in 64 bits and a fixed order.
void launch_column_sums(const float* part, int blocks, int n1, float* out1, int n2, float* out2, const int* stop, hipStream_t s);

// norm_layers.hip: the layers of a deep estimator, and the arguments of its norm in front of layer l
hipError_t launch_norm_layers(const GnnArgs& a, Profiler* prof, hipStream_t s, const void** h_last);
GraphNormArgs norm_args(const LayerNorms& n, int l, int H, int bf16, int n_cu);
void launch_row_major(const unsigned short* packed, long long n, int H, unsigned short* out, hipStream_t s);

// ---- kept rows ----
struct KeepArgs {
  long long rows;
  const int* nrows;
  int cols, bf16;                // type of x
  const void* src;               // keep: rows; restore: unused
  void* dst;                     // restore: rows
  long long ld;
  signed char* code;
  unsigned char* exponent;
  long long ld_code, ld_exponent;
  const int* stop;
  int n_cu;
};
hipError_t launch_keep_rows(const KeepArgs& a, hipStream_t s);
hipError_t launch_restore_rows(const KeepArgs& a, hipStream_t s);

}  // namespace dc
