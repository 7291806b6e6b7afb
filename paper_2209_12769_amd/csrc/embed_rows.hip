// Rows by kind: y_i = s T[id_i] (a row of zeros where id_i is -1), and the table's gradient dT_k = s sum of dy_i over id_i = k
// (gfx950).
//
// Forward: bound by the rows it writes; the table's used rows stay in the caches (5.7 M rows of 128 in bf16, 97 kinds, 1.5 GB:
// 264 us, 5.6 TB/s).
// Gradient: the row numbers are sorted by kind (stable radix sort, up to nine bits a pass; a short list by one workgroup), so that
// a kind's rows become neighbours, and the sorted list is cut into chunks of equal length.  A chunk sums its rows kind by kind in
// the list's order.  A kind that lies inside one chunk is written at once; what a chunk has of kinds that reach beyond it, the
// first and the last of its list at most, are entries of a second, shorter list, which is treated alike until it is short
// enough for one workgroup a kind.  No atomics: the same call gives the same bits.  Sums: up to 64 rows in fp32, up to four such runs
// in fp32, the chunks' in 64 bits, rounded to fp32 from list to list.  The table is cleared by the sort's launches, kinds that have
// rows are written after that.  Bound by memory in the rows' sums, which read rows at the sorted list's places, and by launches in
// the rest (474011 rows of 256 in fp32 to 97 kinds: 107 us, of them 77 the rows' sums, 6.3 TB/s; 65521 rows of 1031 in bf16 to
// 128001 kinds, by dY that take turns: 109 us, of them 52 the sort and the zeros, 35 the rows' sums).  Rows of up to 32 vectors, to 97
// kinds: 474011 rows of 256 in bf16 80 us, of them 45 the rows' sums (5.4 TB/s), of 128 in fp32 76 and 41 (5.9), of 128 in bf16 60 and
// 26 (4.6).
#include "row_vectors.h"

namespace dc {
namespace {

typedef unsigned long long u64;

// ---- forward ----
// The kind that an id names, -1 for none.
__device__ __forceinline__ int kind_of(const EmbedArgs& a, int id) {
  if (id >= 0 && id < a.kinds) return id;
  if (id != -1) atomicCAS(&a.status[1], 0, (int)DC_ERR_INVALID_ARG);
  return -1;
}

constexpr int kAtOnce = 8;     // rows of a thread, its columns are the same in all of them
// A workgroup takes `across` neighbouring rows of `used` vectors at a time, kAtOnce times; slabs of rows too wide for one are
// blockIdx.y.
template <typename T>
__global__ __launch_bounds__(1024) void embed_kernel(const EmbedArgs a, int used, int across) {
  constexpr int kV = kVector<T>;
  int seat = (int)((float)threadIdx.x / (float)used);          // the quotient put right where it is one off
  if ((seat + 1) * used <= (int)threadIdx.x) ++seat;
  if (seat * used > (int)threadIdx.x) --seat;
  const int t = (int)threadIdx.x - seat * used, column = ((int)blockIdx.y * used + t) * kV;
  if (seat >= across || column >= a.C) return;
  const unsigned c = max(min(column, a.C - kV), 0);            // the last vector ends with the row
  const unsigned y_on = (unsigned)seat * (unsigned)a.ldy + c;  // rows are at most 2^22 elements apart, seats 1024
  const T* table = static_cast<const T*>(a.table);
  for (long long row0 = (long long)blockIdx.x * across * kAtOnce; row0 < a.rows; row0 += (long long)gridDim.x * across * kAtOnce) {
    const int left = (int)min(a.rows - row0, (long long)across * kAtOnce);
    const int* id = a.id + row0;
    T* Y = static_cast<T*>(a.Y) + row0 * a.ldy;
    int kind[kAtOnce];
    u32x4 v[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) kind[u] = id[min(u * across + seat, left - 1)];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      kind[u] = kind_of(a, kind[u]);
      v[u] = load_vector<T, false>(table + (long long)max(kind[u], 0) * a.ldt, (int)c, a.C);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      if (u * across + seat >= left) break;
      float x[kV];
      unpack(x, v[u], T());
#pragma unroll
      for (int k = 0; k < kV; ++k) x[k] = kind[u] < 0 ? 0.f : x[k] * a.scale;
      T* to = Y + (long long)(u * across) * a.ldy;
      if (a.C >= kV) *reinterpret_cast<u32x4_any*>(to + y_on) = pack(x, T());
      else store_vector<T>(to + y_on, 0, a.C, pack(x, T()));
    }
  }
}

// ---- sort ----
constexpr int kRun = 64;       // rows that are summed in fp32 before they join the others of their chunk
constexpr int kSortThreads = 256, kSortWaves = kSortThreads / 64;
constexpr int kBits = 9, kBins = 1 << kBits;

struct Pair {
  int kind, row;
};
// Rows that stand for nothing, or for no kind of the table, come last, as kind `kinds`.
__device__ __forceinline__ Pair pair_at(const EmbedArgs& a, const Pair* in, int i) {
  if (in) return in[i];
  const int k = kind_of(a, a.id[i]);
  return Pair{k < 0 ? a.kinds : k, i};
}
// The lanes of the wave, among `active`, whose digit is the same.
__device__ __forceinline__ u64 same_digit(int digit, int bits, u64 active) {
  u64 m = active;
  for (int b = 0; b < bits; ++b) {
    const u64 set = __ballot(digit >> b & 1);
    m &= (digit >> b & 1) ? set : ~set;
  }
  return m;
}

// Between a wave's own accesses of LDS, which the hardware does in their order: nothing moves across.
__device__ __forceinline__ void in_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- zeros ----
// The launches of the sort wait for memory most of the time.  They clear the table besides, a part of it each, by further workgroups
// (3000 rows of 1024 in bf16 to 250000 kinds: the call 98 us, and 120 where the sums' launch looks for kinds without rows and clears no
// others; 65536 rows of 1024, one of each kind, 88 and 90).
struct Zeros {
  u16* table;                  // in halves of a word: rows of `width`, the last of `last`, `stride` from one to the next
  long long stride, rows;
  int width, last;
};
struct Part {
  Zeros z;
  long long from, to;          // rows
  int blocks;
};
constexpr int kClear = 8192;   // halves of a word that a wave clears
// A row by one wave, on 16-byte boundaries but for its first and last vector.  Zeros, and rows of kinds that lie inside one chunk, are
// stored as not used again soon: left in L2 they would be in the way of the rows that are summed (65521 rows of 1031 in bf16 to 128001
// kinds 125 -> 103 us; 100000 of 1024 to 100000 kinds 136 -> 114; tables of few kinds the same).
__device__ __forceinline__ void clear_row(u16* row, int n) {
  const int lane = threadIdx.x & 63;
  const u32x4 zero = {0, 0, 0, 0};
  if (n < 8) {
    if (lane < n) row[lane] = 0;
    return;
  }
  const int skip = (int)(-(reinterpret_cast<size_t>(row) / 2) & 7), whole = (n - skip) / 8;
  u32x4* to = reinterpret_cast<u32x4*>(row + skip);
  for (int at = lane; at < whole; at += 64) __builtin_nontemporal_store(zero, to + at);
  if (lane == 0 && skip != 0) *reinterpret_cast<u32x4_any*>(row) = zero;
  if (lane == 1 && skip + whole * 8 < n) *reinterpret_cast<u32x4_any*>(row + (n - 8)) = zero;
}
__device__ __forceinline__ void clear(const Part& p, int block) {
  const int waves = (int)blockDim.x >> 6;
  for (long long k = p.from + (long long)block * waves + ((int)threadIdx.x >> 6); k < p.to; k += (long long)p.blocks * waves)
    clear_row(p.z.table + k * p.z.stride, k == p.z.rows - 1 ? p.z.last : p.z.width);
}
// The table as one long row, cut, or its rows one by one.
Zeros zeros_of(const EmbedArgs& a) {
  const int halves = a.bf16 ? 1 : 2, width = a.C * halves;
  const long long stride = a.lddt * halves, all = (long long)a.kinds * width;
  u16* table = static_cast<u16*>(a.dtable);
  if (stride != width && a.kinds > 1) return Zeros{table, stride, a.kinds, width, width};
  const long long rows = (all + kClear - 1) / kClear;
  return Zeros{table, kClear, rows, kClear, (int)(all - (rows - 1) * kClear)};
}
// Part k of n; workgroups of `waves`.
Part part_of(const Zeros& z, int k, int n, int waves) {
  Part p{z, z.rows * k / n, z.rows * (k + 1) / n, 0};
  const long long each = (long long)waves * (z.width < kClear ? kClear / z.width : 1), need = (p.to - p.from + each - 1) / each;
  p.blocks = (int)(need < 1 << 20 ? need : 1 << 20);
  return p;
}

// How many pairs of each tile have each digit: count[digit][tile].
template <int kPer>
__global__ __launch_bounds__(kSortThreads) void count_kernel(const EmbedArgs a, const Pair* in, int shift, int bits, int tiles, int* count, Part zeros) {
  __shared__ int bin[kBins];
  if ((int)blockIdx.x >= tiles) return clear(zeros, blockIdx.x - tiles);
  const int bins = 1 << bits, n = (int)a.rows, tile = blockIdx.x;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) bin[i] = 0;
  __syncthreads();
#pragma unroll 4
  for (int k = 0; k < kPer; ++k) {
    const long long i = (long long)tile * (kSortThreads * kPer) + k * kSortThreads + threadIdx.x;
    const bool in_range = i < n;
    const int digit = in_range ? pair_at(a, in, (int)i).kind >> shift & (bins - 1) : 0;
    const u64 peers = same_digit(digit, bits, __ballot(in_range));
    // one addition for the lanes of a digit
    if (in_range && (peers & ((1ULL << (threadIdx.x & 63)) - 1)) == 0) atomicAdd(&bin[digit], __popcll(peers));
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) count[(size_t)i * tiles + tile] = bin[i];
}

// Exclusive sums over the workgroup's first 256 threads, the sum of all in `all`; every thread calls it.
__device__ __forceinline__ int scan256(int x, int* part, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int v = x;
  for (int o = 1; o < 64; o <<= 1) {
    const int w = __shfl_up(v, o, 64);
    if (lane >= o) v += w;
  }
  __syncthreads();
  if (lane == 63 && wave < 4) part[wave] = v;
  __syncthreads();
  int before = 0;
  all = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += part[w];
    all += part[w];
  }
  return before + v - x;
}

// A digit's counts become the number of its pairs in the tiles in front; total[digit].
__global__ __launch_bounds__(256) void scan_kernel(int* count, int bins, int tiles, int* total, Part zeros) {
  __shared__ int part[4];
  if ((int)blockIdx.x >= bins) return clear(zeros, blockIdx.x - bins);
  int* c = count + (size_t)blockIdx.x * tiles;
  int before = 0;
  for (int i0 = 0; i0 < tiles; i0 += 256) {
    const int i = i0 + threadIdx.x, x = i < tiles ? c[i] : 0;
    int all;
    const int at = scan256(x, part, all);
    if (i < tiles) c[i] = before + at;
    before += all;
  }
  if (threadIdx.x == 0) total[blockIdx.x] = before;
}

// Every pair to its place: its digit's first place, the tiles in front, the pairs of the tile in front.
template <int kPer>
__global__ __launch_bounds__(kSortThreads) void scatter_kernel(const EmbedArgs a, const Pair* in, int shift, int bits, int tiles, const int* count,
                                                               const int* total, Pair* out, Part zeros) {
  __shared__ int first[kBins];
  __shared__ int next[kSortWaves][kBins];
  __shared__ int part[4];
  if ((int)blockIdx.x >= tiles) return clear(zeros, blockIdx.x - tiles);
  const int bins = 1 << bits, n = (int)a.rows, tile = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = 0;
  for (int d0 = 0; d0 < bins; d0 += 256) {
    const int d = d0 + threadIdx.x, x = d < bins ? total[d] : 0;
    int all;
    const int at = scan256(x, part, all);
    if (d < bins) first[d] = before + at + count[(size_t)d * tiles + tile];
    before += all;
  }
  for (int i = threadIdx.x; i < kSortWaves * bins; i += kSortThreads) next[i / bins][i % bins] = 0;
  __syncthreads();
  // a wave's pairs are neighbours: 64 at a time
  Pair p[kPer];
  u64 peers[kPer];
  const long long base = (long long)tile * (kSortThreads * kPer) + wave * 64 * kPer + lane;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const long long i = base + k * 64;
    p[k] = i < n ? pair_at(a, in, (int)i) : Pair{0, -1};
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int digit = p[k].kind >> shift & (bins - 1);
    const bool in_range = base + k * 64 < n;
    peers[k] = same_digit(digit, bits, __ballot(in_range));
    if (in_range && (peers[k] & ((1ULL << lane) - 1)) == 0) next[wave][digit] += __popcll(peers[k]);
    in_order();
  }
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += kSortThreads) {
    int at = first[d];
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = next[w][d];
      next[w][d] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int digit = p[k].kind >> shift & (bins - 1);
    const bool in_range = base + k * 64 < n;
    const int rank = __popcll(peers[k] & ((1ULL << lane) - 1)), at = next[wave][digit];
    in_order();
    if (in_range) out[at + rank] = p[k];
    if (in_range && rank == 0) next[wave][digit] = at + __popcll(peers[k]);
    in_order();
  }
}

// The whole sort of a list of up to kSmall pairs by one workgroup, in LDS: the same passes, of up to kSmallBits bits.
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64, kSmallPer = 4, kSmall = kSmallThreads * kSmallPer, kSmallBits = 8, kSmallBins = 1 << kSmallBits;
__global__ __launch_bounds__(kSmallThreads) void sort_small_kernel(const EmbedArgs a, int bits, Pair* out, Part zeros) {
  __shared__ Pair list[kSmall];
  __shared__ int next[kSmallWaves][kSmallBins];
  __shared__ int part[4];
  if (blockIdx.x > 0) return clear(zeros, blockIdx.x - 1);
  const int n = (int)a.rows, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, base = wave * 64 * kSmallPer + lane;
  Pair p[kSmallPer];
#pragma unroll
  for (int k = 0; k < kSmallPer; ++k) p[k] = base + k * 64 < n ? pair_at(a, nullptr, base + k * 64) : Pair{0, -1};
  for (int shift = 0; shift < bits; shift += kSmallBits) {
    for (int i = threadIdx.x; i < kSmallWaves * kSmallBins; i += kSmallThreads) next[i / kSmallBins][i % kSmallBins] = 0;
    __syncthreads();
    u64 peers[kSmallPer];
#pragma unroll
    for (int k = 0; k < kSmallPer; ++k) {
      const int digit = p[k].kind >> shift & (kSmallBins - 1);
      const bool in_range = base + k * 64 < n;
      peers[k] = same_digit(digit, kSmallBits, __ballot(in_range));
      if (in_range && (peers[k] & ((1ULL << lane) - 1)) == 0) next[wave][digit] += __popcll(peers[k]);
      in_order();
    }
    __syncthreads();
    // the digits in front, then the waves in front: a thread a digit (the others take part in the barriers)
    int sum = 0, all;
    if (threadIdx.x < kSmallBins)
      for (int w = 0; w < kSmallWaves; ++w) sum += next[w][threadIdx.x];
    int at = scan256(sum, part, all);
    if (threadIdx.x < kSmallBins)
      for (int w = 0; w < kSmallWaves; ++w) {
        const int c = next[w][threadIdx.x];
        next[w][threadIdx.x] = at;
        at += c;
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSmallPer; ++k) {
      const int digit = p[k].kind >> shift & (kSmallBins - 1);
      const bool in_range = base + k * 64 < n;
      const int rank = __popcll(peers[k] & ((1ULL << lane) - 1)), place = next[wave][digit];
      in_order();
      if (in_range) list[place + rank] = p[k];
      if (in_range && rank == 0) next[wave][digit] = place + __popcll(peers[k]);
      in_order();
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSmallPer; ++k)
      if (base + k * 64 < n) p[k] = list[base + k * 64];
  }
#pragma unroll
  for (int k = 0; k < kSmallPer; ++k)
    if (base + k * 64 < n) out[base + k * 64] = p[k];
}

// ---- sums ----
struct Sums {
  EmbedArgs a;
  const Pair* sorted;          // [rows]
  int n;                       // entries of the list: rows, or entries of the level below
  int chunk;                   // entries of a chunk
  int nchunk;
  int lanes, nslab;            // places for a slab's vectors, slabs of a row
  int used;                    // places that are taken
  const float* in;             // levels above the first: [n][C]
  const int* in_kind;          // [n]: the kind, or ~kind of an entry without a sum
  float* out;                  // [2 nchunk][C]
  int* out_kind;
};

template <typename T>
__device__ __forceinline__ void write_kind(const EmbedArgs& a, int kind, int c, const float (&x)[kVector<T>]) {
  float y[kVector<T>];
#pragma unroll
  for (int k = 0; k < kVector<T>; ++k) y[k] = x[k] * a.scale;
  T* to = static_cast<T*>(a.dtable) + (long long)kind * a.lddt;
  if (c + kVector<T> <= a.C) __builtin_nontemporal_store(pack(y, T()), reinterpret_cast<u32x4_any*>(to + c));
  else store_vector<T>(to, c, a.C, pack(y, T()));
}
// Four columns of an entry from c.
__device__ __forceinline__ void read_entry(float (&x)[4], const float* row, int c, int C) { unpack(x, load_vector<float, false>(row, c, C), 0.f); }
template <int kV>
__device__ __forceinline__ void write_entry(float* row, int c, int C, const float (&x)[kV]) {
#pragma unroll
  for (int k = 0; k < kV; k += 4) {
    const float y[4] = {x[k], x[k + 1], x[k + 2], x[k + 3]};
    if (c + k < C) store_vector<float>(row, c + k, C, pack(y, 0.f));
  }
}
// Four columns of a kind.
__device__ __forceinline__ void write_kind4(const EmbedArgs& a, int kind, int c, const float (&x)[4]) {
  float y[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) y[k] = x[k] * a.scale;
  if (!a.bf16) {
    store_vector<float>(static_cast<float*>(a.dtable) + (long long)kind * a.lddt, c, a.C, pack(y, 0.f));
    return;
  }
  u16* row = static_cast<u16*>(a.dtable) + (long long)kind * a.lddt;
  const unsigned lo = pack_bf16x2(y[0], y[1]), hi = pack_bf16x2(y[2], y[3]);
  if (c + 4 <= a.C) {
    *reinterpret_cast<u32x2_any*>(row + c) = u32x2{lo, hi};
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < a.C) row[c + k] = (u16)((k < 2 ? lo : hi) >> (16 * (k & 1)));
  }
}

// What a chunk has of one kind is done with: kind and columns written at once, or an entry of the next list.
struct Close {
  int chunk;
  bool from_before, goes_on;   // the chunk's first kind began in front of it, its last one goes on behind
};
template <int kV, typename F>
__device__ __forceinline__ void close_kind(const Sums& s, const Close& k, int kind, int c, const float (&x)[kV], bool any, bool first, bool last, F write) {
  const bool up = (first && k.from_before) || (last && k.goes_on);
  const size_t entry = 2 * (size_t)k.chunk + (first ? 0 : 1);
  if (any) {
    if (up) write_entry<kV>(s.out + entry * s.a.C, c, s.a.C, x);
    else write(kind, x);
  }
  if (c == 0 && s.out_kind) {  // the thread of the row's first columns says what the entries are, if there is another list
    if (first) s.out_kind[2 * (size_t)k.chunk] = up && any ? kind : ~kind;
    if (last && first) s.out_kind[2 * (size_t)k.chunk + 1] = ~kind;
    if (last && !first) s.out_kind[2 * (size_t)k.chunk + 1] = up && any ? kind : ~kind;
  }
}
// A thread's first column of kV from place `at` of a row; below zero if it has none.  The last vector ends with the row, so that
// two threads may have the same columns and write the same.
template <int kV>
__device__ __forceinline__ int column_of(int at, int C) {
  const int c = at * kV;
  return c < C ? max(min(c, C - kV), 0) : -1;
}

// A pair of the sorted list.  kWave: the same for all lanes, by a scalar load, so that what follows from it takes no vector registers.
template <bool kWave>
__device__ __forceinline__ Pair sorted_at(const Sums& s, int i) {
  if constexpr (kWave) {
    const u64 w = ((const __attribute__((address_space(4))) u64*)reinterpret_cast<size_t>(s.sorted))[i];
    return Pair{(int)w, (int)(w >> 32)};
  } else {
    return s.sorted[i];
  }
}
// First level: chunks of the sorted rows.  kWave: a wave each, of rows or slabs of more than 32 vectors, so that the list comes by scalar
// loads and eight rows are on their way in the registers that this leaves (the whole call with and without: 65521 rows of 1031 in bf16 to
// 128001 kinds 103 and 111 us, 100000 of 1024 to 50000 93 and 95; 474011 of 256 in fp32 to 97 110 and 108.5).  kOnce: dY is read as not
// used again soon.
constexpr long long kCached = 256 << 20;       // bytes that the memory's cache holds
template <typename T, bool kWave, bool kOnce>
__global__ __launch_bounds__(256) void sum_rows_kernel(const Sums s) {
  constexpr int kV = kVector<T>, kAhead = kWave ? 8 : 4;
  const EmbedArgs& a = s.a;
  const int lanes = kWave ? 64 : s.lanes, t = threadIdx.x & (lanes - 1), seat = threadIdx.x / lanes;
  const long long item = (long long)blockIdx.x * (256 / lanes) + (kWave ? __builtin_amdgcn_readfirstlane(seat) : seat);
  if (item >= (long long)s.nchunk * s.nslab) return;
  Close close;
  close.chunk = (int)(item / s.nslab);
  const int c = t < s.used ? column_of<kV>((int)(item - (long long)close.chunk * s.nslab) * s.used + t, a.C) : -1;
  if (c < 0) return;
  const int p0 = (int)((long long)close.chunk * s.chunk), p1 = (int)min((long long)p0 + s.chunk, (long long)s.n), len = p1 - p0;
  const T* dY = static_cast<const T*>(a.dY);
  Pair e[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) e[u] = sorted_at<kWave>(s, p0 + min(u, len - 1));
  int kind = e[0].kind;
  close.from_before = p0 > 0 && sorted_at<kWave>(s, max(p0 - 1, 0)).kind == kind;
  const int past = p1 < s.n ? sorted_at<kWave>(s, min(p1, s.n - 1)).kind : -1;
  auto write = [&](int of, const float (&x)[kV]) { write_kind<T>(a, of, c, x); };
  float sum[kV], runs[kV];     // of up to kRun rows; of the kind's runs
#pragma unroll
  for (int k = 0; k < kV; ++k) sum[k] = runs[k] = 0.f;
  auto join = [&]() {
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      runs[k] += sum[k];
      sum[k] = 0.f;
    }
  };
  bool first = true;
  for (int q = 0; q < len; q += kAhead) {
    if (e[0].kind >= a.kinds) break;                     // only rows that stand for nothing are left
    u32x4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const T* row = dY + (long long)e[u].row * a.lddy;
      if constexpr (kOnce) v[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(row + c));
      else v[u] = load_vector<T, kWave>(row, c, a.C);
    }
    Pair next[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) next[u] = sorted_at<kWave>(s, p0 + min(q + kAhead + u, len - 1));
    if (q > 0 && q % kRun == 0) join();
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (q + u >= len || e[u].kind >= a.kinds) break;
      if (e[u].kind != kind) {
        join();
        close_kind(s, close, kind, c, runs, true, first, false, write);
#pragma unroll
        for (int k = 0; k < kV; ++k) runs[k] = 0.f;
        first = false;
        kind = e[u].kind;
      }
      float x[kV];
      unpack(x, v[u], T());
#pragma unroll
      for (int k = 0; k < kV; ++k) sum[k] += x[k];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) e[u] = next[u];
  }
  join();
  close.goes_on = past == kind;
  close_kind(s, close, kind, c, runs, kind < a.kinds, first, true, write);
}

__device__ __forceinline__ int kind_of_entry(int k) { return k < 0 ? ~k : k; }

// Levels between: chunks of a list of entries, four columns a thread, sums in 64 bits.
__global__ __launch_bounds__(256) void sum_entries_kernel(const Sums s) {
  constexpr int kAhead = 8;
  const EmbedArgs& a = s.a;
  const int t = threadIdx.x & (s.lanes - 1), seats = 256 / s.lanes;
  const long long item = (long long)blockIdx.x * seats + threadIdx.x / s.lanes;
  if (item >= (long long)s.nchunk * s.nslab) return;
  Close close;
  close.chunk = (int)(item / s.nslab);
  const int c = t < s.used ? column_of<4>((int)(item - (long long)close.chunk * s.nslab) * s.used + t, a.C) : -1;
  if (c < 0) return;
  const int p0 = close.chunk * s.chunk, p1 = min(p0 + s.chunk, s.n);
  int kind = kind_of_entry(s.in_kind[p0]);
  close.from_before = p0 > 0 && kind_of_entry(s.in_kind[p0 - 1]) == kind;
  const int past = p1 < s.n ? kind_of_entry(s.in_kind[p1]) : -1;
  auto write = [&](int of, const float (&x)[4]) { write_kind4(a, of, c, x); };
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  float x[4];
  bool first = true, any = false;
  for (int p = p0; p < p1; p += kAhead) {
    int e[kAhead];
    float v[kAhead][4];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) e[u] = s.in_kind[min(p + u, p1 - 1)];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (e[u] >= 0) read_entry(v[u], s.in + (size_t)min(p + u, p1 - 1) * a.C, c, a.C);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (p + u >= p1) break;
      const int of = kind_of_entry(e[u]);
      if (of != kind) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[k] = (float)sum[k];
          sum[k] = 0.0;
        }
        close_kind(s, close, kind, c, x, any, first, false, write);
        first = any = false;
        kind = of;
      }
      if (e[u] < 0) continue;
      any = true;
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] += (double)v[u][k];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = (float)sum[k];
  close.goes_on = past == kind;
  close_kind(s, close, kind, c, x, any, first, true, write);
}

// The last list: a workgroup for each entry that begins a kind, and 256 of its columns; its waves take the entries in turn.
constexpr int kLastWaves = 8;
__global__ __launch_bounds__(64 * kLastWaves) void last_sums_kernel(const Sums s) {
  constexpr int kAhead = 4;
  const EmbedArgs& a = s.a;
  const int p0 = blockIdx.x, kind = kind_of_entry(s.in_kind[p0]);
  if (kind >= a.kinds || (p0 > 0 && kind_of_entry(s.in_kind[p0 - 1]) == kind)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = (blockIdx.y * 64 + lane) * 4, c = max(min(at, a.C - 4), 0);
  __shared__ double part[kLastWaves][64][4];
  __shared__ int found[kLastWaves];
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  int any = 0;
  for (int p = p0 + wave; p < s.n; p += kLastWaves * kAhead) {
    int e[kAhead];
    float v[kAhead][4];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) e[u] = s.in_kind[min(p + u * kLastWaves, s.n - 1)];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (e[u] == kind) read_entry(v[u], s.in + (size_t)min(p + u * kLastWaves, s.n - 1) * a.C, c, a.C);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (p + u * kLastWaves >= s.n || e[u] != kind) continue;
      any = 1;
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] += (double)v[u][k];
    }
    if (kind_of_entry(e[kAhead - 1]) != kind) break;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[wave][lane][k] = sum[k];
  if (lane == 0) found[wave] = any;
  __syncthreads();
  if (wave != 0 || at >= a.C) return;
  for (int w = 1; w < kLastWaves; ++w) {
    any |= found[w];
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] += part[w][lane][k];
  }
  const float x[4] = {(float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]};
  if (any) write_kind4(a, kind, c, x);
}

constexpr int kLastMost = 1024;        // entries that the last launch takes
constexpr int kEntryChunk = 16;        // by 32, and 2048: 100000 rows of 1024 to 50000 kinds 112 us for 108, 1 M of 16 131 for 120

int lanes_of(int vectors) {
  int l = 1;
  while (l < vectors && l < 64) l *= 2;
  return l;
}

struct Plan {
  int all_bits, passes, bits;
  int per, tiles;              // pairs of a thread; workgroups of the sort; 0: it is one
  int lanes, nslab;            // threads of a row's slab, slabs
  int chunk, nchunk;
  long long entries[8];        // of each level's list
  int levels;                  // lists of entries
};
Plan plan(long long rows, int kinds, int C, int bytes) {
  Plan p{};
  p.all_bits = 1;
  while (p.all_bits < 31 && (kinds >> p.all_bits) != 0) ++p.all_bits;          // values 0 .. kinds
  p.passes = rows <= kSmall ? 1 : (p.all_bits + kBits - 1) / kBits;
  p.bits = (p.all_bits + p.passes - 1) / p.passes;
  // Small tiles until there are some hundred of them (65521 rows by tiles of 4096: 16 us a kernel, by tiles of 256: 5).  The whole call,
  // rows of 32 in bf16 to 100000 kinds, by tiles of 256, 1024 and 4096 pairs: 65521 rows 50, 53 and 84 us, 131072 65, 65 and 95, 262144
  // 81, 70 and 100, 1 M 155, 109 and 122, 3 M 372, 212 and 191.
  p.per = rows <= 65536 ? 1 : (rows <= 1048576 ? 4 : 16);
  p.tiles = rows <= kSmall ? 0 : (int)((rows + kSortThreads * p.per - 1) / (kSortThreads * p.per));
  const int vectors = (C * bytes + 15) / 16;
  p.lanes = lanes_of(vectors);
  p.nslab = (vectors + p.lanes - 1) / p.lanes;
  // Two waves a SIMD, eight rows on their way each, but 16 to 256 rows a chunk (474011 rows of 256 in fp32 to 97 kinds, the whole call:
  // 123 us by 2048 waves, 131 by 2560, 130 by 4096, 137 by 8192; 1024 make 65521 rows of 1031 in bf16 slower, 140 us for 127).
  const long long seats = 2048LL * (64 / p.lanes), chunk = (rows * p.nslab + seats - 1) / seats;
  p.chunk = (int)(chunk < 16 ? 16 : (chunk > 4 * kRun ? 4 * kRun : (chunk + 7) / 8 * 8));
  p.nchunk = (int)((rows + p.chunk - 1) / p.chunk);
  long long e = p.nchunk > 1 ? 2LL * p.nchunk : 0;           // of one chunk nothing is left to sum
  while (e > 0) {
    p.entries[p.levels++] = e;
    if (e <= kLastMost) break;
    e = 2 * ((e + kEntryChunk - 1) / kEntryChunk);
  }
  return p;
}
size_t round_up(size_t x) { return (x + 255) & ~(size_t)255; }

// Where the arrays of a call lie in its workspace; its size.
struct Room {
  size_t pair[2], count, total, kind[8], sum[8], bytes;
};
Room room(const Plan& p, long long rows, int C) {
  Room r{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round_up(bytes);
    return here;
  };
  r.pair[0] = take(rows * sizeof(Pair));
  r.pair[1] = p.passes > 1 ? take(rows * sizeof(Pair)) : 0;
  r.count = take(((size_t)p.tiles << p.bits) * sizeof(int));
  r.total = take(p.tiles > 0 ? ((size_t)1 << p.bits) * sizeof(int) : 0);
  for (int l = 0; l < p.levels; ++l) {
    r.kind[l] = take(p.entries[l] * sizeof(int));
    r.sum[l] = take((size_t)p.entries[l] * C * sizeof(float));
  }
  r.bytes = at;
  return r;
}

template <typename T>
void gradient(const EmbedArgs& a, const Plan& p, const Room& r, const Pair* sorted, hipStream_t s) {
  Sums m{};
  m.a = a;
  m.sorted = sorted;
  m.n = (int)a.rows;
  m.chunk = p.chunk;
  m.nchunk = p.nchunk;
  m.lanes = p.lanes;
  m.nslab = p.nslab;
  m.used = ((a.C + kVector<T> - 1) / kVector<T> + p.nslab - 1) / p.nslab;
  if (p.levels > 0) {
    m.out = reinterpret_cast<float*>(a.workspace + r.sum[0]);
    m.out_kind = reinterpret_cast<int*>(a.workspace + r.kind[0]);
  }
  const long long seats = 256 / p.lanes, items = (long long)p.nchunk * p.nslab;
  const dim3 grid((unsigned)((items + seats - 1) / seats));
  // A dY that the memory's cache cannot hold goes past the others: 474011 rows of 256 in fp32 to 97 kinds 122 -> 109 us, 2 M of 512 in
  // bf16 to 200000 623 -> 582.  A smaller one, which may be there from the launch that wrote it, does not: 100000 rows of 1024 in bf16
  // to 50000 kinds, read again and again, 93 us, past the caches 107.
  if (p.lanes < 64) hipLaunchKernelGGL((sum_rows_kernel<T, false, false>), grid, dim3(256), 0, s, m);
  else if (a.rows * a.C * (long long)sizeof(T) > kCached) hipLaunchKernelGGL((sum_rows_kernel<T, true, true>), grid, dim3(256), 0, s, m);
  else hipLaunchKernelGGL((sum_rows_kernel<T, true, false>), grid, dim3(256), 0, s, m);
  // entries: four columns a thread
  const int fours = (a.C + 3) / 4;
  m.lanes = lanes_of(fours);
  m.nslab = (fours + m.lanes - 1) / m.lanes;
  m.used = (fours + m.nslab - 1) / m.nslab;
  for (int l = 0; l < p.levels; ++l) {
    m.n = (int)p.entries[l];
    m.in = m.out;
    m.in_kind = m.out_kind;
    if (l + 1 < p.levels) {
      m.chunk = kEntryChunk;
      m.nchunk = (int)(p.entries[l + 1] / 2);
      m.out = reinterpret_cast<float*>(a.workspace + r.sum[l + 1]);
      m.out_kind = reinterpret_cast<int*>(a.workspace + r.kind[l + 1]);
      const long long seats = 256 / m.lanes, items = (long long)m.nchunk * m.nslab;
      hipLaunchKernelGGL(sum_entries_kernel, dim3((unsigned)((items + seats - 1) / seats)), dim3(256), 0, s, m);
    } else {
      hipLaunchKernelGGL(last_sums_kernel, dim3((unsigned)m.n, (fours + 63) / 64), dim3(64 * kLastWaves), 0, s, m);
    }
  }
}

template <int kPer>
const Pair* sort(const EmbedArgs& a, const Plan& p, const Room& r, hipStream_t s) {
  Pair* pair[2] = {reinterpret_cast<Pair*>(a.workspace + r.pair[0]), reinterpret_cast<Pair*>(a.workspace + r.pair[1])};
  int* count = reinterpret_cast<int*>(a.workspace + r.count);
  int* total = reinterpret_cast<int*>(a.workspace + r.total);
  if (p.tiles == 0) {
    const Part all = part_of(zeros_of(a), 0, 1, kSmallWaves);
    hipLaunchKernelGGL(sort_small_kernel, dim3(1 + all.blocks), dim3(kSmallThreads), 0, s, a, p.all_bits, pair[0], all);
    return pair[0];
  }
  const Zeros zeros = zeros_of(a);
  int launch = 0;
  auto next = [&]() { return part_of(zeros, launch++, 3 * p.passes, kSortWaves); };
  const Pair* in = nullptr;
  for (int k = 0; k < p.passes; ++k) {
    const int shift = k * p.bits;
    Pair* out = pair[k & 1];
    Part z = next();
    hipLaunchKernelGGL((count_kernel<kPer>), dim3(p.tiles + z.blocks), dim3(kSortThreads), 0, s, a, in, shift, p.bits, p.tiles, count, z);
    z = next();
    hipLaunchKernelGGL(scan_kernel, dim3((1 << p.bits) + z.blocks), dim3(256), 0, s, count, 1 << p.bits, p.tiles, total, z);
    z = next();
    hipLaunchKernelGGL((scatter_kernel<kPer>), dim3(p.tiles + z.blocks), dim3(kSortThreads), 0, s, a, in, shift, p.bits, p.tiles, (const int*)count,
                       (const int*)total, out, z);
    in = out;
  }
  return in;
}

}  // namespace

size_t embed_rows_bytes(long long rows, int kinds, int C) {
  const Plan p2 = plan(rows, kinds, C, 2), p4 = plan(rows, kinds, C, 4);
  const size_t b2 = room(p2, rows, C).bytes, b4 = room(p4, rows, C).bytes;
  return b2 > b4 ? b2 : b4;
}

hipError_t launch_embed_rows(const EmbedArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const int vectors = (a.C * (a.bf16 ? 2 : 4) + 15) / 16, slabs = (vectors + 1023) / 1024, used = (vectors + slabs - 1) / slabs;
  // rows of a workgroup: the fewest that leave less than an eighth of its waves' places empty, at least 256 places
  int across = 1;
  for (int best = 0, n = 1; n * used <= 1024; ++n) {
    const int fill = n * used * 1000 / ((n * used + 63) / 64 * 64);
    if (n * used < 192 && (n + 1) * used <= 1024) continue;
    if (fill > best) {
      best = fill;
      across = n;
    }
    if (fill >= 875) break;
  }
  const int threads = (across * used + 63) / 64 * 64;
  const long long need = (a.rows + across * kAtOnce - 1) / (across * kAtOnce), most = (1LL << 31) / threads;     // a launch has less than 2^32 threads
  const dim3 grid((unsigned)(need < most ? need : most), (unsigned)slabs), block((unsigned)threads);
  if (a.bf16) hipLaunchKernelGGL((embed_kernel<u16>), grid, block, 0, s, a, used, across);
  else hipLaunchKernelGGL((embed_kernel<float>), grid, block, 0, s, a, used, across);
  return hipGetLastError();
}

hipError_t launch_embed_rows_back(const EmbedArgs& a, hipStream_t s) {
  const Plan p = plan(a.rows, a.kinds, a.C, a.bf16 ? 2 : 4);
  const Room r = room(p, a.rows, a.C);
  const Pair* sorted = p.per == 1 ? sort<1>(a, p, r, s) : p.per == 4 ? sort<4>(a, p, r, s) : sort<16>(a, p, r, s);
  if (a.rows == 0) return hipGetLastError();
  if (a.bf16) gradient<u16>(a, p, r, sorted, s);
  else gradient<float>(a, p, r, sorted, s);
  return hipGetLastError();
}

}  // namespace dc
