// Norm over the rows of each graph with an activation, and its gradient (gfx950): the channels of a row are in G groups
// of cg = C / G; a statistic runs over a graph's rows and a group's channels, m = rows * cg values.
//
//   forward   mu = mean x, v = mean (x - mu)^2, r = 1 / sqrt(v + eps);  y = act(gamma (x - mu) r + beta)
//   backward  xh = (x - mu) r, dz = dy act'(gamma xh + beta), u = gamma dz, s1 = mean u, s2 = mean u xh;
//             dx = r (u - s1 - xh s2) [+ dres];  dgamma = sum over rows of dz xh, dbeta = sum of dz
//
// Bound by memory, x read once and y written once: a workgroup takes a graph (or a slab of its channels, whole groups and
// whole cache lines), holds its rows in LDS between the sums and the second pass and reads again only what
// does not fit.  The forward's sums are formed in 64 bits, of x - x0 and its square, x0 the first value of the graph's group:
//   mu = x0 + mean (x - x0),  v = mean (x - x0)^2 - (mean (x - x0))^2
// Of x itself the two terms of v would be up to 2^46 times v (values may lie 2^23 times their spread from zero), and their
// rounding some percent of it.  Four instructions a value, which the loads hide.  mu is taken in two parts, the fp32 number that
// is returned and what it lacks, else a value next to mu would be off by mu's rounding; the second pass has two instructions a
// value in front of the activation: (gamma r) (x - mu) + (beta - (gamma r) lacks).  The gradient's sums are formed of a vector's
// values in fp32 and of the vectors in 64 bits; those of gamma and beta of 64 rows of a thread in fp32, of a workgroup's rows in
// 64 bits, rounded to fp32, and of the workgroups in 64 bits again.
// Measured: forward over 4096 graphs of 1390 rows, 256 channels in bf16, SiLU, 1.395 ms (4.2 TB/s; a copy 4.87); gradient over
// 52901 graphs of 9 rows, 256 channels in fp32, x as kept rows, 0.351 ms (3.1 TB/s).
// Graphs of more than long_rows rows would keep one workgroup busy while the others are done: the kernel of the short graphs
// only lists them, and their rows are dealt in chunks, counted from each graph's first row, to three kernels (sums of a chunk;
// sums of a graph; second pass).  The list's order is that of the workgroups' arrival; what is summed over several graphs is
// summed in the graphs' order.
#include <type_traits>

#include "operators.h"

namespace dc {
namespace {

typedef unsigned short u16;

template <typename T, int kV>
struct alignas(sizeof(T) * kV) Vec {
  T v[kV];
};
struct Kept8 {};       // x as codes

template <typename T, int kV>
struct Held {          // kV values as they come from memory
  Vec<T, kV> v;
};
template <int kV>
struct Held<Kept8, kV> {
  Vec<signed char, kV> v;
  unsigned char e;
};

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(u16 x) { return __uint_as_float((unsigned)x << 16); }
__device__ __forceinline__ void narrow(float x, float& y) { y = x; }
__device__ __forceinline__ void narrow(float x, u16& y) { y = to_bf16(x); }

struct Norm {
  GraphNormArgs a;
  int cg;                  // channels per group
  int slab;                // channels per slab: whole groups
  int nslab;
  int lanes;               // threads per row of a slab: a power of two
  int held;                // row steps of a thread that stay in LDS
  long long long_rows;     // graphs with more rows are left to the chunk kernels
  int chunk_rows;
  unsigned long long* found;   // long graphs << 32 | their chunks; null: there cannot be any
  int2* longs;             // [most_longs] graph and its first chunk, ascending in the chunks
  int most_longs, most_chunks; // offsets that ascend do not give more; what others give beyond is left out
  double2* part;           // [chunks][G] sums of a chunk
  float2* means;           // [long graphs][G] s1, s2; forward: what the mean lacks
  float* cols;             // [column blocks][2 C] parts of dgamma | dbeta
  int col_block0;          // first column block of this launch
};

// Where the rows of a graph (or of a chunk) begin, at the thread's columns: places that all lanes share, plus the columns; a row
// is a product of 24 bits away (rows of a graph: 4096 at most, 2^17 elements apart at most).
struct Places {
  const char *x, *dy, *res;
  const unsigned char* e;
  char* out;
  unsigned ldx, lddy, ldres, lde, ldo;       // bytes from row to row
};
template <typename T, typename X, bool kBack>
__device__ __forceinline__ Places places_of(const GraphNormArgs& a, long long row) {
  Places p{};
  constexpr bool kept = !std::is_same<T, X>::value;
  p.ldx = kept ? (unsigned)a.kept.ld_code : (unsigned)(a.ldx * sizeof(T));
  p.x = (kept ? reinterpret_cast<const char*>(a.kept.code) : static_cast<const char*>(a.X)) + row * p.ldx;
  p.lde = (unsigned)a.kept.ld_exponent;
  p.e = kept ? a.kept.exponent + row * p.lde : nullptr;
  p.lddy = (unsigned)(a.lddy * sizeof(T));
  p.dy = kBack ? static_cast<const char*>(a.dY) + row * p.lddy : nullptr;
  p.ldres = (unsigned)(a.lddres * sizeof(T));
  p.res = kBack && a.dRes ? static_cast<const char*>(a.dRes) + row * p.ldres : nullptr;
  p.ldo = (unsigned)((kBack ? a.lddx : a.ldy) * sizeof(T));
  p.out = static_cast<char*>(kBack ? a.dX : a.Y) + row * p.ldo;
  return p;
}
template <typename T, int kV>
__device__ __forceinline__ void hold(Held<T, kV>& h, const Places& p, unsigned row, int c) {
  h.v = *reinterpret_cast<const Vec<T, kV>*>(p.x + (__umul24(row, p.ldx) + (unsigned)(c * (int)sizeof(T))));
}
template <int kV>
__device__ __forceinline__ void hold(Held<Kept8, kV>& h, const Places& p, unsigned row, int c) {
  h.v = *reinterpret_cast<const Vec<signed char, kV>*>(p.x + (__umul24(row, p.ldx) + (unsigned)c));
  h.e = p.e[__umul24(row, p.lde) + (unsigned)(c / kKeptBlock)];
}
template <typename T, int kV>
__device__ __forceinline__ void values(float (&x)[kV], const Held<T, kV>& h) {
#pragma unroll
  for (int k = 0; k < kV; ++k) x[k] = widen(h.v.v[k]);
}
template <int kV>
__device__ __forceinline__ void values(float (&x)[kV], const Held<Kept8, kV>& h) {
  const float s = kept_scale(h.e);
#pragma unroll
  for (int k = 0; k < kV; ++k) x[k] = (float)h.v.v[k] * s;
}

struct Rows {
  long long lo, hi;
  bool ok;
};
// The rows of graph g; offsets that do not ascend inside the arrays are reported, and the graph is left alone.
__device__ __forceinline__ Rows rows_of(const GraphNormArgs& a, int g) {
  Rows r;
  r.lo = a.node_off[g];
  r.hi = a.node_off[g + 1];
  r.ok = r.lo >= 0 && r.hi >= r.lo && r.hi <= a.rows;
  if (!r.ok && threadIdx.x == 0) {
    if (a.stop) atomicCAS(&a.status[0], 0, (int)DC_ERR_BAD_GRAPH);
    atomicCAS(&a.status[1], 0, (int)DC_ERR_BAD_GRAPH);
  }
  return r;
}
__device__ __forceinline__ int graphs_of(const GraphNormArgs& a) {
  return a.n_graphs_dev ? min(a.n_graphs_dev[0], a.n_graphs) : a.n_graphs;
}

template <int kV>
struct Affine {
  float gamma[kV], beta[kV];
};
template <int kV>
__device__ __forceinline__ Affine<kV> affine_at(const GraphNormArgs& a, int c) {
  Affine<kV> f;
#pragma unroll
  for (int k = 0; k < kV; ++k) {
    f.gamma[k] = a.gamma ? a.gamma[c + k] : 1.f;
    f.beta[k] = a.beta ? a.beta[c + k] : 0.f;
  }
  return f;
}

// dy becomes dz.
template <int kV>
__device__ __forceinline__ void slope(float (&dy)[kV], const float (&xh)[kV], const Affine<kV>& f, int act) {
  float z[kV];
#pragma unroll
  for (int k = 0; k < kV; ++k) z[k] = fmaf(f.gamma[k], xh[k], f.beta[k]);
  slopes<kV>(z, act);
#pragma unroll
  for (int k = 0; k < kV; ++k) dy[k] *= z[k];
}

// What the sums of a group are counted from: its first value in row `row`, or zero if that is not finite.
template <typename T>
__device__ __forceinline__ T first_value(const GraphNormArgs& a, long long row, int channel) {
  return static_cast<const T*>(a.X)[row * a.ldx + channel];
}
// Not to be widened, and waited for, where it was requested.
template <typename T>
__device__ __forceinline__ double origin(T first) {
  unsigned bits = __builtin_bit_cast(std::conditional_t<sizeof(T) == 4, unsigned, u16>, first);
  asm volatile("" : "+v"(bits));
  const float x = __uint_as_float(sizeof(T) == 4 ? bits : bits << 16);
  return __builtin_isfinite(x) ? (double)x : 0.0;
}
// What a row's vector adds to the two sums.
template <bool kBack, int kV>
__device__ __forceinline__ void add_sums(double& s1, double& s2, const float (&x)[kV], float (&dy)[kV], double x0, float mu, float r,
                                         const Affine<kV>& f, int act, float (&dg)[kV], float (&db)[kV]) {
  if constexpr (!kBack) {
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      const double d = (double)x[k] - x0;
      s1 += d;
      s2 = fma(d, d, s2);
    }
  } else {
    float xh[kV];
#pragma unroll
    for (int k = 0; k < kV; ++k) xh[k] = (x[k] - mu) * r;
    slope<kV>(dy, xh, f, act);
    float v1 = 0.f, v2 = 0.f;                          // a vector's, before they go to the 64-bit sums
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      const float u = f.gamma[k] * dy[k];
      v1 += u;
      v2 = fmaf(u, xh[k], v2);
      dg[k] = fmaf(dy[k], xh[k], dg[k]);
      db[k] += dy[k];
    }
    s1 += (double)v1;
    s2 += (double)v2;
  }
}

// A run's sums of the gradients of gamma and beta go to the 64-bit ones.
template <int kV>
__device__ __forceinline__ void flush(double (&dgs)[kV], double (&dbs)[kV], float (&dg)[kV], float (&db)[kV]) {
#pragma unroll
  for (int k = 0; k < kV; ++k) {
    dgs[k] += (double)dg[k];
    dbs[k] += (double)db[k];
    dg[k] = db[k] = 0.f;
  }
}

// Sums over the workgroup by group.  Threads: `lanes` per row, of which `used` hold one vector each (gv vectors per group);
// every thread gives its two sums and gets its group's totals.  red: 2 * blockDim.x doubles.
__device__ __forceinline__ void group_sums(double& s1, double& s2, double2* red, int lanes, int used, int gv) {
  const int t = threadIdx.x, T = blockDim.x;
  for (int o = lanes; o < 64; o <<= 1) {               // the rows of a wave
    s1 += __shfl_xor(s1, o, 64);
    s2 += __shfl_xor(s2, o, 64);
  }
  // one entry per wave (or row, where a row takes several waves) and lane
  const int width = lanes > 64 ? lanes : 64, parts = T / width, lane = t & (lanes - 1);
  __syncthreads();                                     // the last totals have been read
  if (lanes > 64 || (t & 63) < lanes) red[t / width * lanes + lane] = make_double2(s1, s2);
  __syncthreads();
  if (parts > 1) {
    if (t < used) {
      double2 v = red[t];
      for (int p = 1; p < parts; ++p) {
        const double2 w = red[p * lanes + t];
        v.x += w.x;
        v.y += w.y;
      }
      red[t] = v;
    }
    __syncthreads();
  }
  if (gv > 1) {
    if (t < used && t % gv == 0) {
      double2 v = red[t];
      for (int i = 1; i < gv; ++i) {
        const double2 w = red[t + i];
        v.x += w.x;
        v.y += w.y;
      }
      red[t] = v;
    }
    __syncthreads();
  }
  const double2 v = red[lane < used ? lane / gv * gv : 0];
  s1 = v.x;
  s2 = v.y;
}

// mean (and what its fp32 value lacks) and 1 / sqrt(variance + eps) from the sums of x - x0 and (x - x0)^2 over m values.
__device__ __forceinline__ void statistics(double s1, double s2, double m, double x0, float eps, float& mu, float& lacks, float& rs) {
  const double from = m > 0 ? s1 / m : 0.0, var = m > 0 ? s2 / m - from * from : 0.0, mean = x0 + from;
  mu = (float)mean;
  lacks = (float)(mean - (double)mu);
  rs = (float)(1.0 / sqrt((var > 0.0 ? var : (var != var ? var : 0.0)) + (double)eps));
}

// What x - mu (mu as fp32) takes in the forward's second pass.
template <int kV>
__device__ __forceinline__ Affine<kV> of_graph(const Affine<kV>& f, float r, float lacks) {
  Affine<kV> h;
#pragma unroll
  for (int k = 0; k < kV; ++k) {
    h.gamma[k] = f.gamma[k] * r;
    h.beta[k] = fmaf(-lacks, h.gamma[k], f.beta[k]);
  }
  return h;
}
// The second pass of one vector.  Forward: f is of_graph's, r, s1 and s2 are not taken.
template <typename T, int kV, bool kBack>
__device__ __forceinline__ void finish(int act, const Places& p, const float (&x)[kV], float (&dy)[kV], unsigned row, int c, float mu, float r, float s1,
                                       float s2, const Affine<kV>& f) {
  Vec<T, kV> o;
  float xh[kV];
  if constexpr (!kBack) {
#pragma unroll
    for (int k = 0; k < kV; ++k) xh[k] = fmaf(f.gamma[k], x[k] - mu, f.beta[k]);
    activate<kV>(xh, act);
#pragma unroll
    for (int k = 0; k < kV; ++k) narrow(xh[k], o.v[k]);
  } else {
#pragma unroll
    for (int k = 0; k < kV; ++k) xh[k] = (x[k] - mu) * r;
    slope<kV>(dy, xh, f, act);
    Vec<T, kV> add{};
    if (p.res) add = *reinterpret_cast<const Vec<T, kV>*>(p.res + (__umul24(row, p.ldres) + (unsigned)(c * (int)sizeof(T))));
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      float d = r * (f.gamma[k] * dy[k] - s1 - xh[k] * s2);
      if (p.res) d += widen(add.v[k]);
      narrow(d, o.v[k]);
    }
  }
  *reinterpret_cast<Vec<T, kV>*>(p.out + (__umul24(row, p.ldo) + (unsigned)(c * (int)sizeof(T)))) = o;
}

template <typename T, typename X, int kV>
struct Two {
  Held<X, kV> x;
  Vec<T, kV> dy;
};
// LDS bytes of one row step of a thread: x, and dy for the gradient, in arrays of their own.
template <typename T, typename X, int kV, bool kBack>
constexpr int kItemBytes = (int)sizeof(Held<X, kV>) + (kBack ? (int)sizeof(Vec<T, kV>) : 0);
template <typename T, typename X, int kV, bool kBack>
__device__ __forceinline__ void fetch(Two<T, X, kV>& h, const Places& p, unsigned row, int c) {
  hold<>(h.x, p, row, c);
  if constexpr (kBack) h.dy = *reinterpret_cast<const Vec<T, kV>*>(p.dy + (__umul24(row, p.lddy) + (unsigned)(c * (int)sizeof(T))));
}
template <typename T, typename X, int kV, bool kBack>
__device__ __forceinline__ void open(float (&x)[kV], float (&dy)[kV], const Two<T, X, kV>& h) {
  values(x, h.x);
#pragma unroll
  for (int k = 0; k < kV; ++k) dy[k] = kBack ? widen(h.dy.v[k]) : 0.f;
}

// Column sums of the workgroup's rows: dg, db of every thread into cols[block][c], [C + c].
template <int kV>
__device__ __forceinline__ void column_sums(const Norm& n, double (&dg)[kV], double (&db)[kV], int lanes, int used, int c, int block,
                                            double2* red) {
  const int t = threadIdx.x, T = blockDim.x;
  for (int o = lanes; o < 64; o <<= 1) {
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      dg[k] += __shfl_xor(dg[k], o, 64);
      db[k] += __shfl_xor(db[k], o, 64);
    }
  }
  const int width = lanes > 64 ? lanes : 64, parts = T / width, lane = t & (lanes - 1);
  float* out = n.cols + (size_t)block * 2 * n.a.C;
#pragma unroll
  for (int k = 0; k < kV; ++k) {
    __syncthreads();
    if (lanes > 64 || (t & 63) < lanes) red[t / width * lanes + lane] = make_double2(dg[k], db[k]);
    __syncthreads();
    if (t < used) {
      double s1 = 0.0, s2 = 0.0;
      for (int p = 0; p < parts; ++p) {
        s1 += red[p * lanes + t].x;
        s2 += red[p * lanes + t].y;
      }
      out[c + k] = (float)s1;
      out[n.a.C + c + k] = (float)s2;
    }
  }
}

// A thread's rows first, first + step, .. (count of them) in groups of kStep: the requests of a group are made together, past the
// end the last row again (a request in a branch would make every wait wait for everything).
template <typename T, typename X, int kV, bool kBack, int kStep, typename F>
__device__ __forceinline__ void each_row(const Places& p, int first, int step, int from, int count, int c, F f) {
  for (int i = from; i < count; i += kStep) {
    Two<T, X, kV> h[kStep];
#pragma unroll
    for (int u = 0; u < kStep; ++u) fetch<T, X, kV, kBack>(h[u], p, (unsigned)(first + (int)__umul24(min(i + u, count - 1), step)), c);
#pragma unroll
    for (int u = 0; u < kStep; ++u)
      if (i + u < count) f(h[u], i + u);
  }
}

// Gradients of vectors: a thread's terms of so many rows are summed in fp32, these sums in 64 bits (1000 equal terms in fp32 alone were up
// to 250 roundings off; the runs cost at most 1.6 %, of 60000 graphs of 3 rows of 128).
constexpr int kRun = 64;
// each_row of all rows.  Forward: `begin` (which waits for a request made before) once the first group has been requested;
// gradient: `flush` behind each run.
template <typename T, typename X, int kV, bool kBack, int kStep, typename F, typename B, typename E>
__device__ __forceinline__ void each_run(const Places& p, int first, int step, int count, int c, F f, B begin, E flush) {
  for (int i = 0; i < count; i += kStep) {
    Two<T, X, kV> h[kStep];
#pragma unroll
    for (int u = 0; u < kStep; ++u) fetch<T, X, kV, kBack>(h[u], p, (unsigned)(first + (int)__umul24(min(i + u, count - 1), step)), c);
    if (!kBack && i == 0) begin();
#pragma unroll
    for (int u = 0; u < kStep; ++u)
      if (i + u < count) f(h[u], i + u);
    if (kBack && ((i + kStep) & (kRun - 1)) == 0) flush();
  }
  if (kBack) flush();
}

// One workgroup per (graph, slab), the slab fixed.  The first n.held row steps of every thread stay in LDS.
template <typename T, typename X, int kV, int kThreads, bool kBack>
__global__ __launch_bounds__(kThreads) void graph_norm_kernel(const Norm n) {
  if (n.a.stop && n.a.stop[0] != 0) return;
  typedef Two<T, X, kV> Item;
  extern __shared__ char lds[];
  double2* red = reinterpret_cast<double2*>(lds);
  const int slab = blockIdx.x % n.nslab, t = threadIdx.x;
  Held<X, kV>* held_x = reinterpret_cast<Held<X, kV>*>(lds + kThreads * sizeof(double2)) + t;
  Vec<T, kV>* held_dy = reinterpret_cast<Vec<T, kV>*>(lds + kThreads * (sizeof(double2) + n.held * sizeof(Held<X, kV>))) + t;
  const int c0 = slab * n.slab, width = min(n.slab, n.a.C - c0);
  const int used = width / kV, lane = t & (n.lanes - 1), rl = t / n.lanes, step = kThreads / n.lanes, gv = n.cg / kV;
  const bool in = lane < used;
  const int c = c0 + lane * kV, group = in ? c / n.cg : 0;
  const Affine<kV> f = affine_at<kV>(n.a, in ? c : c0);
  double dgs[kV], dbs[kV];
#pragma unroll
  for (int k = 0; k < kV; ++k) dgs[k] = dbs[k] = 0.0;
  const int ng = graphs_of(n.a);
  for (int g = blockIdx.x / n.nslab; g < ng; g += gridDim.x / n.nslab) {
    const Rows r = rows_of(n.a, g);
    if (!r.ok) continue;
    if (r.hi - r.lo > n.long_rows) {
      if (slab == 0 && t == 0) {
        const long long chunks = (r.hi - r.lo + n.chunk_rows - 1) / n.chunk_rows;
        const unsigned long long at = atomicAdd(n.found, (1ull << 32) + (unsigned long long)chunks);
        if ((at >> 32) < (unsigned)n.most_longs) n.longs[at >> 32] = make_int2(g, (int)(unsigned)at);
      }
      continue;
    }
    const double m = (double)(r.hi - r.lo) * n.cg;
    float mu = 0.f, rs = 0.f, s1f = 0.f, s2f = 0.f;
    if (kBack) {
      mu = n.a.mean[(size_t)g * n.a.G + group];
      rs = n.a.rstd[(size_t)g * n.a.G + group];
    }
    double s1 = 0.0, s2 = 0.0, x0 = 0.0;
    T first{};
    if (!kBack && r.hi > r.lo) first = first_value<T>(n.a, r.lo, group * n.cg);
    float dg[kV], db[kV];
#pragma unroll
    for (int k = 0; k < kV; ++k) dg[k] = db[k] = 0.f;
    const Places at = places_of<T, X, kBack>(n.a, r.lo);
    const int rows = (int)(r.hi - r.lo), count = in && rl < rows ? (rows - rl + step - 1) / step : 0;      // row steps of this thread
    auto add = [&](const Item& h, int i) {
      if (i < n.held) {
        held_x[i * kThreads] = h.x;
        if constexpr (kBack) held_dy[i * kThreads] = h.dy;
      }
      float x[kV], dy[kV];
      open<T, X, kV, kBack>(x, dy, h);
      add_sums<kBack, kV>(s1, s2, x, dy, x0, mu, rs, f, n.a.act, dg, db);
    };
    each_run<T, X, kV, kBack, kThreads == 64 ? 8 : 4>(at, rl, step, count, c, add, [&] { x0 = origin(first); }, [&] { flush<kV>(dgs, dbs, dg, db); });
    group_sums(s1, s2, red, n.lanes, used, gv);
    if constexpr (!kBack) {
      statistics(s1, s2, m, x0, n.a.eps, mu, s1f, rs);
      if (in && rl == 0 && lane % gv == 0) {
        n.a.mean[(size_t)g * n.a.G + group] = mu;
        n.a.rstd[(size_t)g * n.a.G + group] = rs;
      }
    } else {
      s1f = m > 0 ? (float)(s1 / m) : 0.f;
      s2f = m > 0 ? (float)(s2 / m) : 0.f;
    }
    const Affine<kV> fg = kBack ? f : of_graph(f, rs, s1f);
    auto second = [&](const Item& h, int i) {
      float x[kV], dy[kV];
      open<T, X, kV, kBack>(x, dy, h);
      finish<T, kV, kBack>(n.a.act, at, x, dy, (unsigned)(rl + i * step), c, mu, rs, s1f, s2f, fg);
    };
    const int here = min(count, n.held);
#pragma unroll 2
    for (int i = 0; i < here; ++i) {
      Item h;
      h.x = held_x[i * kThreads];
      if constexpr (kBack) h.dy = held_dy[i * kThreads];
      second(h, i);
    }
    each_row<T, X, kV, kBack, 4>(at, rl, step, here, count, c, second);
  }
  if (kBack && n.a.dgamma) column_sums<kV>(n, dgs, dbs, n.lanes, used, c, n.col_block0 + blockIdx.x / n.nslab, red);
}

// ---- long graphs: rows in chunks ----
__global__ __launch_bounds__(256) void no_longs_kernel(unsigned long long* found, int2* longs, int most) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i == 0) found[0] = 0;
  for (int k = i; k < most; k += gridDim.x * blockDim.x) longs[k] = make_int2(0, 0);
}

// The list comes in the order in which the graphs were found.  Gradients of gamma and beta are sums over the chunks as they are
// dealt out, so for them it is put in the graphs' order, a wave per entry, and a call gives the same bits each time.
__global__ __launch_bounds__(256) void order_longs_kernel(const Norm n, int2* __restrict__ ordered) {
  if (n.a.stop && n.a.stop[0] != 0) return;
  const int nlong = (int)min((unsigned)(n.found[0] >> 32), (unsigned)n.most_longs), lane = threadIdx.x & 63;
  for (int i = blockIdx.x * 4 + (threadIdx.x >> 6); i < nlong; i += gridDim.x * 4) {
    const int2 e = n.longs[i];
    int before = 0;
    long long chunks = 0;                              // of the graphs in front
    for (int k = lane; k < nlong; k += 64) {
      const int g = n.longs[k].x;
      if (g > e.x || (g == e.x && k >= i)) continue;
      const long long rows = (long long)n.a.node_off[g + 1] - n.a.node_off[g];
      ++before;
      chunks += rows > 0 ? (rows + n.chunk_rows - 1) / n.chunk_rows : 0;
    }
    for (int o = 32; o > 0; o >>= 1) {
      before += __shfl_xor(before, o, 64);
      chunks += __shfl_xor(chunks, o, 64);
    }
    if (lane == 0) ordered[before] = make_int2(e.x, (int)min(chunks, (long long)n.most_chunks));
  }
}

struct Segment {
  int entry, g;            // place in the list, graph
  long long first;         // its first row
  long long lo, hi;        // rows of the chunk
};
// The long graph of a chunk: the last entry whose first chunk is not behind it, found 64 entries at a time.
__device__ __forceinline__ Segment segment_of(const Norm& n, int nlong, int chunk) {
  const int lane = threadIdx.x & 63;
  int lo = 0, count = nlong;                           // the entry is one of lo .. lo + count - 1
  while (count > 1) {
    const int stride = (count + 63) >> 6, i = lo + lane * stride;
    const bool before = lane * stride < count && n.longs[i].y <= chunk;
    const int k = __popcll(__ballot(before)) - 1;      // ascending: the lanes in front
    count = min(stride, count - k * stride);
    lo += k * stride;
  }
  Segment s;
  s.entry = lo;
  const int2 e = n.longs[lo];
  s.g = e.x;
  const long long first = n.a.node_off[e.x], end = n.a.node_off[e.x + 1];
  s.first = first;
  s.lo = first + (long long)(chunk - e.y) * n.chunk_rows;
  s.hi = s.lo + n.chunk_rows < end ? s.lo + n.chunk_rows : end;
  // offsets that do not ascend can fill the list with more than it holds, and then a chunk's entry is not its graph
  if (first < 0 || end > n.a.rows || s.lo < first || s.lo >= end) s.hi = s.lo;
  return s;
}

constexpr int kChunkThreads = 512;

template <typename T, typename X, int kV, bool kBack>
__global__ __launch_bounds__(kChunkThreads) void chunk_sums_kernel(const Norm n) {
  if (n.a.stop && n.a.stop[0] != 0) return;
  __shared__ double2 red[kChunkThreads];
  const int slab = blockIdx.x % n.nslab, t = threadIdx.x;
  const int c0 = slab * n.slab, width = min(n.slab, n.a.C - c0);
  const int used = width / kV, lane = t & (n.lanes - 1), rl = t / n.lanes, step = kChunkThreads / n.lanes, gv = n.cg / kV;
  const bool in = lane < used;
  const int c = c0 + lane * kV, group = in ? c / n.cg : 0;
  const Affine<kV> f = affine_at<kV>(n.a, in ? c : c0);
  double dgs[kV], dbs[kV];
#pragma unroll
  for (int k = 0; k < kV; ++k) dgs[k] = dbs[k] = 0.0;
  const unsigned long long found = n.found[0];
  const int nchunk = (int)min((unsigned)found, (unsigned)n.most_chunks), nlong = (int)min((unsigned)(found >> 32), (unsigned)n.most_longs);
  for (int chunk = blockIdx.x / n.nslab; chunk < nchunk; chunk += gridDim.x / n.nslab) {
      const Segment seg = segment_of(n, nlong, chunk);
      if (seg.lo >= seg.hi) continue;
      float mu = 0.f, rs = 0.f;
      if (kBack) {
        mu = n.a.mean[(size_t)seg.g * n.a.G + group];
        rs = n.a.rstd[(size_t)seg.g * n.a.G + group];
      }
      double s1 = 0.0, s2 = 0.0, x0 = 0.0;
      T first{};
      if (!kBack) first = first_value<T>(n.a, seg.first, group * n.cg);
      float dg[kV], db[kV];
#pragma unroll
      for (int k = 0; k < kV; ++k) dg[k] = db[k] = 0.f;
      const Places at = places_of<T, X, kBack>(n.a, seg.lo);
      const int rows = (int)(seg.hi - seg.lo), count = in && rl < rows ? (rows - rl + step - 1) / step : 0;
      auto add = [&](const Two<T, X, kV>& h, int) {
        float x[kV], dy[kV];
        open<T, X, kV, kBack>(x, dy, h);
        add_sums<kBack, kV>(s1, s2, x, dy, x0, mu, rs, f, n.a.act, dg, db);
      };
      each_run<T, X, kV, kBack, 4>(at, rl, step, count, c, add, [&] { x0 = origin(first); }, [&] { flush<kV>(dgs, dbs, dg, db); });
      group_sums(s1, s2, red, n.lanes, used, gv);
      if (in && rl == 0 && lane % gv == 0) n.part[(size_t)chunk * n.a.G + group] = make_double2(s1, s2);
    }
  if (kBack && n.a.dgamma) column_sums<kV>(n, dgs, dbs, n.lanes, used, c, n.col_block0 + blockIdx.x / n.nslab, red);
}

// The sums of a long graph from its chunks': a wave each, `wide` (a power of two, at least the groups or 64) lanes side by side
// over the groups, the others over the chunks.
template <typename T, bool kBack>
__global__ __launch_bounds__(64) void long_sums_kernel(const Norm n, int wide) {
  if (n.a.stop && n.a.stop[0] != 0) return;
  const int nlong = (int)min((unsigned)(n.found[0] >> 32), (unsigned)n.most_longs), lane = threadIdx.x, q0 = lane & (wide - 1), k0 = lane / wide;
  for (int i = blockIdx.x; i < nlong; i += gridDim.x) {
    const int2 e = n.longs[i];
    const long long first = n.a.node_off[e.x], rows = (long long)n.a.node_off[e.x + 1] - first;
    if (rows <= n.long_rows || first < 0 || first + rows > n.a.rows || e.y < 0) continue;
    const int chunks = (int)min((rows + n.chunk_rows - 1) / n.chunk_rows, (long long)n.most_chunks - e.y);
    const double m = (double)rows * n.cg;
    for (int q = q0; q < n.a.G + q0; q += wide) {       // the same number of rounds for every lane
      double s1 = 0.0, s2 = 0.0;
      if (q < n.a.G)
        for (int k = k0; k < chunks; k += 64 / wide) {
          const double2 p = n.part[(size_t)(e.y + k) * n.a.G + q];
          s1 += p.x;
          s2 += p.y;
        }
      for (int o = 32; o >= wide; o >>= 1) {
        s1 += __shfl_xor(s1, o, 64);
        s2 += __shfl_xor(s2, o, 64);
      }
      if (k0 != 0 || q >= n.a.G) continue;
      if (kBack) {
        n.means[(size_t)i * n.a.G + q] = make_float2((float)(s1 / m), (float)(s2 / m));
      } else {
        float mu, lacks, rs;
        statistics(s1, s2, m, origin(first_value<T>(n.a, first, q * n.cg)), n.a.eps, mu, lacks, rs);
        n.means[(size_t)i * n.a.G + q] = make_float2(lacks, 0.f);
        n.a.mean[(size_t)e.x * n.a.G + q] = mu;
        n.a.rstd[(size_t)e.x * n.a.G + q] = rs;
      }
    }
  }
}

template <typename T, typename X, int kV, bool kBack>
__global__ __launch_bounds__(kChunkThreads) void chunk_finish_kernel(const Norm n) {
  if (n.a.stop && n.a.stop[0] != 0) return;
  const int slab = blockIdx.x % n.nslab, t = threadIdx.x;
  const int c0 = slab * n.slab, width = min(n.slab, n.a.C - c0);
  const int used = width / kV, lane = t & (n.lanes - 1), rl = t / n.lanes, step = kChunkThreads / n.lanes;
  const bool in = lane < used;                         // all lanes of a wave stay: they look for its segments together
  const int c = c0 + (in ? lane * kV : 0), group = c / n.cg;
  const Affine<kV> f = affine_at<kV>(n.a, c);
  const unsigned long long found = n.found[0];
  const int nchunk = (int)min((unsigned)found, (unsigned)n.most_chunks), nlong = (int)min((unsigned)(found >> 32), (unsigned)n.most_longs);
  for (int chunk = blockIdx.x / n.nslab; chunk < nchunk; chunk += gridDim.x / n.nslab) {
      const Segment seg = segment_of(n, nlong, chunk);
      if (seg.lo >= seg.hi) continue;
      const float mu = n.a.mean[(size_t)seg.g * n.a.G + group], rs = n.a.rstd[(size_t)seg.g * n.a.G + group];
      const float2 s = n.means[(size_t)seg.entry * n.a.G + group];
      const Affine<kV> fg = kBack ? f : of_graph(f, rs, s.x);
      const Places at = places_of<T, X, kBack>(n.a, seg.lo);
      const int rows = (int)(seg.hi - seg.lo), count = in && rl < rows ? (rows - rl + step - 1) / step : 0;
      each_row<T, X, kV, kBack, 4>(at, rl, step, 0, count, c, [&](const Two<T, X, kV>& h, int i) {
        float x[kV], dy[kV];
        open<T, X, kV, kBack>(x, dy, h);
        finish<T, kV, kBack>(n.a.act, at, x, dy, (unsigned)(rl + i * step), c, mu, rs, s.x, s.y, fg);
      });
    }
}

// One chain of additions per column would be a round trip per row: a workgroup takes 16 columns with 64 threads each, which
// request eight rows together.
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* __restrict__ part, int blocks, int n1, float* __restrict__ out1,
                                                           int n2, float* __restrict__ out2, const int* stop) {
  if (stop && stop[0] != 0) return;
  __shared__ double red[64][17];
  const int j = threadIdx.x & 15, p = threadIdx.x >> 4, c = blockIdx.x * 16 + j, n = n1 + n2;
  double s = 0.0;
  if (c < n)
    for (int b = p; b < blocks; b += 512) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = part[(size_t)min(b + 64 * u, blocks - 1) * n + c];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += b + 64 * u < blocks ? (double)x[u] : 0.0;
    }
  red[p][j] = s;
  __syncthreads();
  for (int o = 32; o > 0; o >>= 1) {
    if (p < o) red[p][j] += red[p + o][j];
    __syncthreads();
  }
  if (p == 0 && c < n) {
    if (c < n1) out1[c] = (float)red[0][j];
    else out2[c - n1] = (float)red[0][j];
  }
}

constexpr int most_threads(bool back) { return back ? 512 : 1024; }     // the gradient needs more than 128 registers
// Rows of a chunk: four chunks per CU, 64 to 512 rows.  Fewer than the shortest long graph.
int chunk_rows(long long rows, int n_cu) {
  const long long r = (rows / (4LL * n_cu) + 63) / 64 * 64;
  return (int)(r < 64 ? 64 : (r > 512 ? 512 : r));
}

struct Plan {
  int threads, slab, nslab, lanes, held;
  int chunk_slab, chunk_nslab, chunk_lanes;
  long long long_rows;
  bool chunks;             // there may be long graphs
  int blocks, chunk_blocks;    // column blocks: of the short graphs' kernel, of the chunk kernels
};
int pow2_at_least(int x) {
  int p = 1;
  while (p < x) p <<= 1;
  return p;
}
// Channels per slab: whole groups, at least a cache line of a row.
int slab_of(int C, int cg, int es) {
  const long long s = (long long)((128 / es + cg - 1) / cg) * cg;
  return s >= C ? C : (int)s;
}
// Workgroups of a launch: two rounds of the single waves, more of the larger ones, so that long and short graphs even out.
int blocks_most(int threads, int n_cu) { return n_cu * (threads == 64 ? 24 : 8); }
// LDS for rows of a workgroup of 64, 256 or more threads: twelve, three or one of them per CU
int held_bytes(int threads) { return threads == 64 ? 12 * 1024 : (threads == 256 ? 48 * 1024 : 140 * 1024); }

Plan plan_of(long long rows, int n_graphs, int C, int G, int es, int v, int item, bool back, int n_cu) {
  Plan p{};
  const int kMost = most_threads(back);
  const int cg = C / G;
  const long long mean = rows / (n_graphs > 0 ? n_graphs : 1), want = mean * 3 / 2;       // a graph of one and a half times the mean
  // whole rows and the fewest threads that hold it; else slabs
  p.slab = C;
  p.lanes = pow2_at_least((C + v - 1) / v);
  auto fits = [&](int threads, int lanes) {
    return lanes <= threads && want <= (long long)held_bytes(threads) / (threads * item) * (threads / lanes);
  };
  // A wave by itself needs no barriers, and what it does not hold it finds in L2: up to twice what it holds, in slabs of whole
  // groups where the rows are wider than its vectors (47207 graphs of 3 rows, 52 groups of 9 channels, bf16: 417 us, and 528
  // by workgroups).  Else 256 threads that hold whole rows; else narrower slabs (20000 graphs of 30 rows of 512 channels,
  // gradients in fp32: 883 us, and 2270 by workgroups of 512), for many graphs up to four times what a wave holds (6000 of
  // 120 rows of 256: 608 us, and 938).
  auto wave = [&](int most_lanes, long long times) {
    const int each = most_lanes * v / cg;              // groups
    if (each < 1) return false;
    const int slabs = (G + each - 1) / each, slab = (G + slabs - 1) / slabs * cg, lanes = pow2_at_least((slab + v - 1) / v);
    if ((slab * es < 64 && slabs > 1) || mean > times * (held_bytes(64) / (64 * item)) * (64 / lanes)) return false;
    p.slab = slab;
    p.lanes = lanes;
    return true;
  };
  auto narrower = [&](long long times) { return wave(32, times) || wave(16, times) || wave(8, times); };
  if (wave(64, 2)) p.threads = 64;
  else if (fits(256, p.lanes)) p.threads = 256;
  else if (narrower(2)) p.threads = 64;
  else if (n_graphs >= 4 * n_cu && !fits(kMost, p.lanes) && (narrower(4) || wave(64, 4))) p.threads = 64;
  else p.threads = kMost;
  const int narrow = slab_of(C, cg, es);
  // slabs also where whole rows would leave most CUs without work
  if (p.threads == kMost && (!fits(p.threads, p.lanes) || n_graphs < n_cu / 2)) {
    p.slab = narrow;
    p.lanes = pow2_at_least((p.slab + v - 1) / v);
  }
  // chunks are not held: whole rows if the workgroup is wide enough
  p.chunk_lanes = pow2_at_least((C + v - 1) / v);
  p.chunk_slab = p.chunk_lanes <= kChunkThreads ? C : narrow;
  p.chunk_lanes = pow2_at_least((p.chunk_slab + v - 1) / v);
  p.chunk_nslab = (C + p.chunk_slab - 1) / p.chunk_slab;
  p.held = held_bytes(p.threads) / (p.threads * item);
  p.nslab = (C + p.slab - 1) / p.slab;
  // twice what a workgroup would have if all had the same, 4096 rows at most (8 graphs of 9000 rows of 128 channels, fp32: 37
  // us, and 48 if none is cut; the gradient of 24 graphs of 20000 rows on average, 256 channels in bf16: 341 us, and 553 if those
  // up to 8191 rows are not; 64 graphs of 5000, which fill the CUs as they are, lose by it: 101 us, and 77)
  const long long share = 2 * rows * p.nslab / n_cu;
  p.long_rows = share < 1024 ? 1024 : (share > 4096 ? 4096 : share);
  p.chunks = rows > p.long_rows;
  auto blocks = [&](long long items, int threads, int nslab) {
    const int m = blocks_most(threads, n_cu);
    const long long most = m / nslab > 0 ? m / nslab : 1;
    return (int)(items < 1 ? 1 : (items < most ? items : most));
  };
  p.blocks = blocks(n_graphs, p.threads, p.nslab);
  p.chunk_blocks = p.chunks ? blocks((rows + chunk_rows(rows, n_cu) - 1) / chunk_rows(rows, n_cu), kChunkThreads, p.chunk_nslab) : 0;
  return p;
}

template <typename T, typename X, int kV, int kThreads, bool kBack>
hipError_t run_short(const Norm& n, int blocks, hipStream_t s) {
  const size_t bytes = kThreads * sizeof(double2) + (size_t)n.held * kThreads * kItemBytes<T, X, kV, kBack>;
  auto kernel = graph_norm_kernel<T, X, kV, kThreads, kBack>;
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3(blocks * n.nslab), dim3(kThreads), bytes, s, n);
  return hipGetLastError();
}

template <typename T, typename X, int kV, bool kBack>
hipError_t run(Norm n, hipStream_t s) {
  const Plan p = plan_of(n.a.rows, n.a.n_graphs, n.a.C, n.a.G, (int)sizeof(T), kV, kItemBytes<T, X, kV, kBack>, kBack, n.a.n_cu);
  n.slab = p.slab;
  n.nslab = p.nslab;
  n.lanes = p.lanes;
  n.held = p.held;
  n.long_rows = p.long_rows;
  n.chunk_rows = chunk_rows(n.a.rows, n.a.n_cu);
  char* w = n.a.workspace;
  int2* ordered = nullptr;
  if (p.chunks) {
    const size_t longs = (size_t)(n.a.rows / p.long_rows) + 1;
    n.found = reinterpret_cast<unsigned long long*>(w);
    n.longs = reinterpret_cast<int2*>(w + 16);
    w += 16 + (longs * sizeof(int2) + 15) / 16 * 16;
    n.part = reinterpret_cast<double2*>(w);
    n.most_longs = (int)longs;
    n.most_chunks = (int)(n.a.rows / n.chunk_rows + (long long)longs);
    w += (size_t)n.most_chunks * n.a.G * sizeof(double2);
    n.means = reinterpret_cast<float2*>(w);
    w += longs * n.a.G * sizeof(float2);
    if (kBack) {
      ordered = reinterpret_cast<int2*>(w);
      w += longs * sizeof(int2);
    }
    hipLaunchKernelGGL(no_longs_kernel, dim3((unsigned)(longs < 16384 ? (longs + 255) / 256 : 64)), dim3(256), 0, s, n.found, n.longs, n.most_longs);
  }
  n.cols = reinterpret_cast<float*>(w);
  hipError_t e = p.threads == 64    ? run_short<T, X, kV, 64, kBack>(n, p.blocks, s)
                 : p.threads == 256 ? run_short<T, X, kV, 256, kBack>(n, p.blocks, s)
                                    : run_short<T, X, kV, most_threads(kBack), kBack>(n, p.blocks, s);
  if (e != hipSuccess) return e;
  if (p.chunks) {
    n.col_block0 = p.blocks;
    n.slab = p.chunk_slab;
    n.nslab = p.chunk_nslab;
    n.lanes = p.chunk_lanes;
    const dim3 cgrid(p.chunk_blocks * n.nslab);
    if (kBack && n.a.dgamma) {
      hipLaunchKernelGGL(order_longs_kernel, dim3((unsigned)(n.most_longs < 16 * n.a.n_cu ? (n.most_longs + 3) / 4 : 4 * n.a.n_cu)), dim3(256), 0, s, n, ordered);
      n.longs = ordered;
    }
    hipLaunchKernelGGL((chunk_sums_kernel<T, X, kV, kBack>), cgrid, dim3(kChunkThreads), 0, s, n);
    const long long longs = n.a.rows / p.long_rows + 1, most = 4LL * n.a.n_cu;
    const int wide = n.a.G < 64 ? pow2_at_least(n.a.G) : 64;
    hipLaunchKernelGGL((long_sums_kernel<T, kBack>), dim3((unsigned)(longs < most ? longs : most)), dim3(64), 0, s, n, wide);
    hipLaunchKernelGGL((chunk_finish_kernel<T, X, kV, kBack>), cgrid, dim3(kChunkThreads), 0, s, n);
  }
  if (kBack && n.a.dgamma)
    launch_column_sums(n.cols, p.blocks + p.chunk_blocks, n.a.C, n.a.dgamma, n.a.C, n.a.dbeta, n.a.stop, s);
  return hipGetLastError();
}

template <typename T, typename X, bool kBack>
hipError_t dispatch(const GraphNormArgs& a, hipStream_t s) {
  Norm n{};
  n.a = a;
  n.cg = a.C / a.G;
  auto aligned = [&](const void* p, long long ld, size_t es, int v) {
    return !p || (ld % v == 0 && reinterpret_cast<size_t>(p) % (es * v) == 0);
  };
  // the widest vectors, up to 16 bytes, that no group's end cuts and every row starts on
  int v = 16 / (int)sizeof(T);
  for (; v > 1; v >>= 1) {
    bool ok = n.cg % v == 0 && aligned(a.Y, a.ldy, sizeof(T), v) && aligned(a.dY, a.lddy, sizeof(T), v) &&
              aligned(a.dX, a.lddx, sizeof(T), v) && aligned(a.dRes, a.lddres, sizeof(T), v);
    ok = ok && (a.kept.code ? aligned(a.kept.code, a.kept.ld_code, 1, v) : aligned(a.X, a.ldx, sizeof(T), v));
    if (ok) break;
  }
  switch (v) {
    case 8:
      if constexpr (sizeof(T) == 2) return run<T, X, 8, kBack>(n, s);
    case 4: return run<T, X, 4, kBack>(n, s);
    case 2: return run<T, X, 2, kBack>(n, s);
    default: return run<T, X, 1, kBack>(n, s);
  }
}

}  // namespace

void launch_column_sums(const float* part, int blocks, int n1, float* out1, int n2, float* out2, const int* stop, hipStream_t s) {
  hipLaunchKernelGGL(column_sums_kernel, dim3((n1 + n2 + 15) / 16), dim3(1024), 0, s, part, blocks, n1, out1, n2, out2, stop);
}

size_t graph_norm_bytes(long long rows, int n_graphs, int C, int G, bool backward, int n_cu) {
  // what any vector width and type would need, and any smaller number of rows: chunks of 512 rows, or four per CU and, as their
  // rows are rounded (from 64 on) before the last CU has its four, up to a 64th more
  const long long most = blocks_most(64, n_cu), by_rows = rows / 512 + 1, per_cu = 4LL * n_cu + n_cu / 16 + 2, nc = by_rows > per_cu ? by_rows : per_cu;
  const bool chunks = rows > 1024;
  const size_t longs = chunks ? (size_t)(rows / 1024) + 1 : 0;
  size_t b = chunks ? 16 + (longs * sizeof(int2) + 15) / 16 * 16 + ((size_t)nc + longs) * G * sizeof(double2) + longs * G * sizeof(float2) : 0;
  if (backward) {
    b += longs * sizeof(int2);
    b += (size_t)((n_graphs < most ? (n_graphs > 0 ? n_graphs : 1) : most) + (chunks ? (nc < most ? nc : most) : 0)) * 2 * C * sizeof(float);
  }
  return b;
}

hipError_t launch_graph_norm(const GraphNormArgs& a, hipStream_t s) {
  if (a.n_graphs <= 0) return hipSuccess;
  return a.bf16 ? dispatch<u16, u16, false>(a, s) : dispatch<float, float, false>(a, s);
}

hipError_t launch_graph_norm_back(const GraphNormArgs& a, hipStream_t s) {
  if (a.kept.code) return a.bf16 ? dispatch<u16, Kept8, true>(a, s) : dispatch<float, Kept8, true>(a, s);
  return a.bf16 ? dispatch<u16, u16, true>(a, s) : dispatch<float, float, true>(a, s);
}

}  // namespace dc
