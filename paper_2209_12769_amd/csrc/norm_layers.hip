// Layers of a deep estimator (dc_set_layer_norms), inference: after the first layer every layer adds to its input,
//     h_1 = [x | means of x] W_0 + b_0,   u = act(norm(h_l)),   h_{l+1} = h_l + [u | means of u] W_l + b_l,
// made of the operators: graph_norm.hip, the neighbour means of gnn.hip and the dense layer with a residual.  h stays in one
// buffer, to which each layer's product adds in place; u takes the other.
#include "operators.h"

namespace dc {

// The layer matrices in row-major bf16 from the fused layers' layout, [k / 8][H][8].
__global__ __launch_bounds__(256) void row_major_kernel(const unsigned short* __restrict__ packed, long long n, int H,
                                                        unsigned short* __restrict__ out) {
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
    const long long k = i / H;
    const int c = (int)(i - k * H);
    out[i] = packed[((k >> 3) * H + c) * 8 + (k & 7)];
  }
}
void launch_row_major(const unsigned short* packed, long long n, int H, unsigned short* out, hipStream_t s) {
  hipLaunchKernelGGL(row_major_kernel, dim3(512), dim3(256), 0, s, packed, n, H, out);
}

GraphNormArgs norm_args(const LayerNorms& n, int l, int H, int bf16, int n_cu) {
  GraphNormArgs a{};
  a.rows = n.rows;
  a.n_graphs = n.n_graphs;
  a.n_graphs_dev = n.n_graphs_dev;
  a.node_off = n.node_off;
  a.C = H;
  a.G = n.groups;
  a.bf16 = bf16;
  a.act = n.act;
  a.eps = n.eps;
  a.ldx = a.ldy = a.lddy = a.lddres = a.lddx = H;
  a.gamma = n.gamma + (size_t)(l - 1) * H;
  a.beta = n.beta + (size_t)(l - 1) * H;
  a.mean = n.mean;
  a.rstd = n.rstd;
  a.workspace = n.workspace;
  a.status = n.status;
  a.stop = n.status;
  a.n_cu = n_cu;
  return a;
}

hipError_t launch_norm_layers(const GnnArgs& a, Profiler* prof, hipStream_t s, const void** h_last) {
  const LayerNorms& n = *a.norms;
  const size_t es = a.bf16 ? 2 : 4;
  const char* W = static_cast<const char*>(a.bf16 ? n.W : a.W);
  const float* b = a.b;
  const void* src = a.Xc;
  int d = a.F;
  hipError_t e = hipSuccess;
  for (int l = 0; l < a.L && e == hipSuccess; ++l) {
    if (l > 0) {
      GraphNormArgs g = norm_args(n, l, a.H, a.bf16, a.n_cu);
      g.X = a.act[0];
      g.Y = a.act[1];
      if (prof) prof->begin(kFamGraphNorm, s);
      e = launch_graph_norm(g, s);
      if (prof) prof->end(s);
      if (e != hipSuccess) return e;
      src = a.act[1];
      d = a.H;
    }
    if (prof) prof->begin(kFamAggregate, s);
    launch_mean_aggregate(a, src, d, a.agg[0], a.agg[1], s);
    if (prof) prof->end(s);
    DenseArgs p{};
    p.rows = n.rows;
    p.nrows = a.node_off + a.n_cand;
    p.d = d;
    p.nseg = 3;
    p.N = a.H;
    p.bf16 = a.bf16;
    p.X[0] = src;
    p.X[1] = a.agg[0];
    p.X[2] = a.agg[1];
    p.ldx = d;
    p.W = W;
    p.ldw = a.H;
    p.bias = b;
    p.R = l > 0 ? a.act[0] : nullptr;
    p.ldr = a.H;
    p.Y = a.act[0];
    p.ldy = a.H;
    p.stop = a.status;
    p.n_cu = a.n_cu;
    if (prof) prof->begin(kFamUpdate, s);
    e = launch_dense(p, s);
    if (prof) prof->end(s);
    W += (size_t)3 * d * a.H * es;
    b += a.H;
  }
  *h_last = a.act[0];
  return e;
}

}  // namespace dc
