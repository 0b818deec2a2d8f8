// Draws under temperature, top-k, top-p and min-p for gfx950, over rows of fp32 logits.
//
// With z = logit * scale / temperature and w = exp(z - max z), a row keeps, in the order of falling logits (equal ones by rising
// id): of the first k ids the shortest prefix that holds at least top_p of their mass, and of that the ids with w >= min_p.
// What is kept is renormalised; a draw is the first id, ascending, at which the running sum passes u times the total.
//
// Which id is the last one is decided at a border, and a draw next to one, so z and w are 64-bit.  Where atomics add weights up
// they are integers, in units of 2^-43 (2^20 of them fit 64 bits): the same sum in whatever order; all other sums have a fixed
// order.
//
// A row is cut into chunks of 2048 to 8192 ids (a workgroup each), so that few rows use many compute units.  By what is asked for:
//   greedy, or temperature alone   top (a chunk's largest logit, sum of weights), finish
//   min-p alone                    top, mass (what a chunk keeps), finish
//   top-k up to 1024 ids           groups (largest logit of every 16 ids), few.  The k-th largest group is no more than the k-th
//                                  largest logit, so whatever counts lies in the groups that reach it: one workgroup per row
//                                  reads those, resolves the borders among them, draws, and writes q over a row that `groups`
//                                  has cleared.
//   else                           bins, collect, resolve, finish.  Borders are first narrowed down by classes of z, 1/8 wide on a
//                                  fixed grid: `bins` has a chunk's masses and counts by class; in `collect` every workgroup adds
//                                  the chunks up, ids above the border classes are in, those inside are listed; `resolve`, a
//                                  workgroup per row, finds the border among them.
// `finish` writes the distribution or the truncated logits and draws inside the chunk that the draw falls into.
//
// Few rows are bound by launches that depend on each other, many by the row's one workgroup (kernels alone, us):
//   1 row of 32000, a top-k that goes by groups     groups 2.9, few 7.9
//   64 rows of 128256, top-k 1000                   groups 10.9 (66 MB read and written), few 22.8
//   8 rows of 128256, by classes                    bins 5.2, collect 8.1, resolve 3.0, finish 7.1
// Classes end 31.9 below the largest z.  Where fewer than k groups (ids) lie that near, or a border's class has more ids than a list
// holds, the row's one workgroup reads the row again in every pass (whole calls): 32000 ids, top-k 50, temperature 0.1 138 (0.25 and
// up: 10), 128256 ids 324; one level of 128256 ids, or 640 above -inf and top-k 1000, 1650.
#include <float.h>

#include "spec_internal.h"

#define FL_THREADS 512
#define FL_WAVES (FL_THREADS / 64)
#define FL_QUAD (FL_THREADS * 4)           // ids that a workgroup takes at a time, 4 neighbours per thread
#define FL_QUADS_MAX 4                     // of them in a chunk: 1, 2 or 4
#define FL_CHUNKS_MAX (SPEC_SAMPLE_VOCAB_MAX / (FL_QUAD * FL_QUADS_MAX))
#define FL_BINS 256
#define FL_GRID 8.0                       // classes per unit of z
#define FL_LIST 8192                      // most candidates that are kept as a list; beyond, the row is read again
#define FL_GROUP 16
#define FL_FEW 1024                       // largest top-k that goes by groups
#define FL_ONE 0x1p43                     // units of a weight of 1
typedef unsigned long long u64;
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
static_assert(SPEC_SAMPLE_VOCAB_MAX <= 1 << 20, "sums of weights fit 64 bits");
static_assert(FL_CHUNKS_MAX <= 128, "two chunks per lane");

struct FilterInfo {              // of a row: borders by classes, masses relative to its largest weight
  int kbin, plo, phi, low, n_before;  // class of the k-th id; classes that top-p may end in; first that min-p leaves out; ids before kbin
  double m_before_k, m_before_p, mass;  // mass: that of the ids top-p counts, where no kbin says which
};
struct FilterEnd {
  u64 last;                      // order of the last kept id
  double total;                  // units kept
};
struct FilterWork {              // arrays over the rows of a call
  float* top;                    // [row][C]: largest logit of a chunk; +inf for one with a NaN, unless greedy
  int* top_id;                   // [row][C]: greedy: its lowest id
  double* sum;                   // [row][C]: sum of exp(z - the chunk's largest z)
  double* kept;                  // [row][C]: units kept
  u64* mass;                     // [row][C][FL_BINS]
  unsigned* count;               // [row][C][FL_BINS]
  u64* list;                     // [row][L]
  FilterInfo* info;              // [row]
  FilterEnd* end;                // [row]
  unsigned* listed;              // [row]
  float* group;                  // [row][G]: largest logit of 16 ids, +inf with a NaN
};
struct FilterArgs {
  const float* logits;
  size_t ld;
  int V, chunk, C, G, L, greedy, top_k;    // ids of a chunk, chunks, groups, room of a list; top_k 0: off
  double mult, top_p, min_p;     // top_p 1: off
  const float* u;
  float *q, *masked;
  int* tok;
  FilterWork w;
};

// ---- one id ---------------------------------------------------------------------------------------------------------
// 64 bits that rise as an id falls in the order: logits by falling value, then ids
__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned b = __float_as_uint(x + 0.0f);               // -0 counts as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ u64 order_of(float x, int id) { return (u64)~key_of(x) << 32 | (unsigned)id; }
__device__ __forceinline__ float logit_of(u64 order) {
  const unsigned key = ~(unsigned)(order >> 32);
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// Bounds of the orders of logits up to / from a value that roundings have moved by less than 1e-6 of it; the edge of a class that is
// wider than fp32 may have become infinite, which has no 1e-6.
__device__ __forceinline__ u64 first_order(float x) {
  x = fmaxf(x, -FLT_MAX);
  return order_of(x + (fabsf(x) * 1e-6f + 1e-44f), 0);
}
__device__ __forceinline__ u64 last_order(float x) {
  x = fminf(x, FLT_MAX);
  return order_of(x - (fabsf(x) * 1e-6f + 1e-44f), -1);
}
// exp(-d), d >= 0: 2^-n times the Taylor series of 2^f, |f| <= 1/2, to the 12th power.  Against 60 digits off by up to 3e-16 of the
// value below d = 1, and by 1.2e-16 d beyond, the rounding of y (1.1e-14 up to 100, 4.9e-14 up to 700); d itself has two roundings.
__device__ __forceinline__ double weight(double d) {
  const double y = fmin(d, 1000.0) * 1.4426950408889634074, n = rint(y), t = (n - y) * 0.69314718055994530942;
  double p = 1.0 / 479001600.0;
  p = fma(p, t, 1.0 / 39916800.0);
  p = fma(p, t, 1.0 / 3628800.0);
  p = fma(p, t, 1.0 / 362880.0);
  p = fma(p, t, 1.0 / 40320.0);
  p = fma(p, t, 1.0 / 5040.0);
  p = fma(p, t, 1.0 / 720.0);
  p = fma(p, t, 1.0 / 120.0);
  p = fma(p, t, 1.0 / 24.0);
  p = fma(p, t, 1.0 / 6.0);
  p = fma(p, t, 0.5);
  p = fma(p, t, 1.0);
  p = fma(p, t, 1.0);
  return ldexp(p, -(int)n);
}
__device__ __forceinline__ double distance(float top, float x, double mult) { return ((double)top - (double)x) * mult; }
// w <= 1: added to 2^52, the units are the low bits of the sum
__device__ __forceinline__ u64 units(double w) { return (u64)__double_as_longlong(fma(w, FL_ONE, 0x1p52)) & 0xfffffffffffffull; }
__device__ __forceinline__ double line_of(float x, double mult) { return floor((double)x * mult * FL_GRID); }
__device__ __forceinline__ int class_of(double line, float x, double mult) {
  const double b = line - line_of(x, mult);
  return b < FL_BINS - 1 ? (int)b : FL_BINS - 1;
}

// ---- a wave, a workgroup --------------------------------------------------------------------------------------------
// Neighbours' values inside rows of 16 lanes and on to the rows behind: no trip through LDS.  `rest` where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_32(unsigned rest, unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp((int)rest, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T dpp_add(T v) {
  if constexpr (sizeof(T) == 4) {
    return v + __builtin_bit_cast(T, dpp_32<CTRL, ROWS>(0u, __builtin_bit_cast(unsigned, v)));
  } else {
    const u64 b = __builtin_bit_cast(u64, v);
    const u64 n = (u64)dpp_32<CTRL, ROWS>(0u, (unsigned)(b >> 32)) << 32 | dpp_32<CTRL, ROWS>(0u, (unsigned)b);
    return v + __builtin_bit_cast(T, n);
  }
}
template <typename T>
__device__ __forceinline__ T wave_scan_t(T v) {               // inclusive
  v = dpp_add<0x111, 0xf>(v);
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);
  return dpp_add<0x143, 0xc>(v);
}
template <typename T>
__device__ __forceinline__ T lane_t(T v, int lane) {          // lane: uniform
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  } else {
    const u64 b = __builtin_bit_cast(u64, v);
    const unsigned hi = __builtin_amdgcn_readlane((int)(b >> 32), lane), lo = __builtin_amdgcn_readlane((int)b, lane);
    return __builtin_bit_cast(T, (u64)hi << 32 | lo);
  }
}
template <typename T>
__device__ __forceinline__ T wave_sum_t(T v) { return lane_t(wave_scan_t(v), 63); }
template <typename T>
__device__ __forceinline__ T wave_before_t(T scan) {          // the lane before's; 0 in the first
  const T up = __shfl_up(scan, 1);
  return (threadIdx.x & 63) ? up : T(0);
}
__device__ __forceinline__ float wave_max_f(float v) {
  const unsigned none = __float_as_uint(-INFINITY);
  v = fmaxf(v, __uint_as_float(dpp_32<0x111, 0xf>(none, __float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(dpp_32<0x112, 0xf>(none, __float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(dpp_32<0x114, 0xf>(none, __float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(dpp_32<0x118, 0xf>(none, __float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(dpp_32<0x142, 0xa>(none, __float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(dpp_32<0x143, 0xc>(none, __float_as_uint(v))));
  return lane_t(v, 63);
}
__device__ __forceinline__ unsigned wave_or(unsigned v) {
  v |= dpp_32<0x111, 0xf>(0u, v);
  v |= dpp_32<0x112, 0xf>(0u, v);
  v |= dpp_32<0x114, 0xf>(0u, v);
  v |= dpp_32<0x118, 0xf>(0u, v);
  v |= dpp_32<0x142, 0xa>(0u, v);
  v |= dpp_32<0x143, 0xc>(0u, v);
  return lane_t(v, 63);
}
// sh is free again for whoever has passed one more barrier
template <int W = FL_WAVES, typename T>
__device__ __forceinline__ T block_sum_t(T v, T* sh) {        // to every thread
  v = wave_sum_t(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  T t = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) t += sh[i];
  return t;
}

// the chunk's ids j * 2048 + 4 * thread + i; beyond V: -inf, which has no weight and comes last
template <int Q>
__device__ __forceinline__ int id_of(int chunk, int j, int i) { return (chunk * Q + j) * FL_QUAD + threadIdx.x * 4 + i; }
template <int Q>
__device__ __forceinline__ void load_chunk(const FilterArgs& a, int row, int chunk, float (&x)[Q][4]) {
  const float* p = a.logits + (size_t)row * a.ld;
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    const int id = id_of<Q>(chunk, j, 0);
    if (id + 4 <= a.V) {
      const f32x4u v = *reinterpret_cast<const f32x4u*>(p + id);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[j][i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[j][i] = id + i < a.V ? p[id + i] : -INFINITY;
    }
  }
}
// four results from the id of i = 0 on
__device__ __forceinline__ void put4(float* out, const FilterArgs& a, int row, int id, const float (&v)[4]) {
  float* p = out + (size_t)row * a.V + id;
  if (id + 4 <= a.V) {
    *reinterpret_cast<f32x4u*>(p) = f32x4u{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (id + i < a.V) p[i] = v[i];
  }
}

// largest logit of the chunk, to every thread; +inf if there is a NaN
template <int Q>
__device__ __forceinline__ float chunk_top(const float (&x)[Q][4], float* sh) {
  float t = -INFINITY;
#pragma unroll
  for (int j = 0; j < Q; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) t = x[j][i] < INFINITY ? fmaxf(t, x[j][i]) : INFINITY;
  t = wave_max_f(t);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = t;
  __syncthreads();
  t = sh[0];
#pragma unroll
  for (int i = 1; i < FL_WAVES; ++i) t = fmaxf(t, sh[i]);
  return t;
}
__device__ __forceinline__ bool has_none(float top) { return !(top < INFINITY) || top == -INFINITY; }   // no distribution
__device__ __forceinline__ float row_top(const FilterArgs& a, int row) {     // by every wave for itself
  const int lane = threadIdx.x & 63;
  const float* p = a.w.top + (size_t)row * a.C;
  float t = lane < a.C ? p[lane] : -INFINITY;
  if (64 + lane < a.C) t = fmaxf(t, p[64 + lane]);
  return wave_max_f(t);
}

// ---- greedy, temperature alone, min-p alone -------------------------------------------------------------------------
template <int Q>
__global__ __launch_bounds__(FL_THREADS) void filter_top_kernel(FilterArgs a, int sum) {
  __shared__ float sh[FL_WAVES];
  __shared__ double shd[FL_WAVES];
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[Q][4];
  load_chunk(a, row, chunk, x);
  const float t = chunk_top(x, sh);
  if (sum && !has_none(t)) {
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < Q; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) s += weight(distance(t, x[j][i], a.mult));
    s = block_sum_t(s, shd);
    if (threadIdx.x == 0) a.w.sum[(size_t)row * a.C + chunk] = s;
  }
  if (threadIdx.x == 0) a.w.top[(size_t)row * a.C + chunk] = t;
}
// the lowest id of the largest logit, NaN counting as none; id 0 where nothing is above -inf
template <int Q>
__global__ __launch_bounds__(FL_THREADS) void filter_greedy_kernel(FilterArgs a) {
  __shared__ float sh[FL_WAVES];
  __shared__ int lowest;
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[Q][4];
  load_chunk(a, row, chunk, x);
  if (threadIdx.x == 0) lowest = 0x7fffffff;
#pragma unroll
  for (int j = 0; j < Q; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[j][i] = x[j][i] >= -INFINITY ? x[j][i] : -INFINITY;
  float t = -INFINITY;
#pragma unroll
  for (int j = 0; j < Q; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) t = fmaxf(t, x[j][i]);
  t = wave_max_f(t);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = t;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < FL_WAVES; ++i) t = fmaxf(t, sh[i]);
  int id = 0x7fffffff;
#pragma unroll
  for (int j = Q - 1; j >= 0; --j)
#pragma unroll
    for (int i = 3; i >= 0; --i)
      if (x[j][i] == t) id = id_of<Q>(chunk, j, i);
  if (id < 0x7fffffff) atomicMin(&lowest, id);
  __syncthreads();
  if (threadIdx.x == 0) {
    a.w.top[(size_t)row * a.C + chunk] = t;
    a.w.top_id[(size_t)row * a.C + chunk] = t == -INFINITY ? 0 : lowest;
  }
}
template <int Q>
__global__ __launch_bounds__(FL_THREADS) void filter_mass_kernel(FilterArgs a) {
  __shared__ u64 sh[FL_WAVES];
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[Q][4];
  load_chunk(a, row, chunk, x);
  const float top = row_top(a, row);
  if (has_none(top)) return;
  u64 sum = 0;
#pragma unroll
  for (int j = 0; j < Q; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double w = weight(distance(top, x[j][i], a.mult));
      if (w >= a.min_p) sum += units(w);
    }
  sum = block_sum_t(sum, sh);
  if (threadIdx.x == 0) a.w.kept[(size_t)row * a.C + chunk] = (double)sum;
}

// ---- classes --------------------------------------------------------------------------------------------------------
template <int Q>
__global__ __launch_bounds__(FL_THREADS) void filter_bins_kernel(FilterArgs a) {
  __shared__ float sh[FL_WAVES];
  __shared__ u64 mass[FL_BINS];
  __shared__ unsigned count[FL_BINS];
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[Q][4];
  load_chunk(a, row, chunk, x);
  if (threadIdx.x < FL_BINS) mass[threadIdx.x] = 0, count[threadIdx.x] = 0;
  const float t = chunk_top(x, sh);
  if (threadIdx.x == 0) {
    a.w.top[(size_t)row * a.C + chunk] = t;
    if (chunk == 0) a.w.listed[row] = 0;
  }
  if (!(t < INFINITY)) return;
  if (t > -INFINITY) {
    const double line = line_of(t, a.mult);
#pragma unroll
    for (int j = 0; j < Q; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int b = class_of(line, x[j][i], a.mult);
        if (a.top_k && b < FL_BINS - 1) atomicAdd(&count[b], 1u);
        const u64 m = units(weight(distance(t, x[j][i], a.mult)));
        if (m) atomicAdd(&mass[b], m);
      }
  }
  __syncthreads();
  if (threadIdx.x < FL_BINS) {
    const size_t at = ((size_t)row * a.C + chunk) * FL_BINS + threadIdx.x;
    a.w.mass[at] = mass[threadIdx.x];
    if (a.top_k) a.w.count[at] = count[threadIdx.x];
  }
}

// The borders of a row by classes, by the first wave: lane l holds classes 4 l .. 4 l + 3 of mass and count.  The last class takes
// all that lies further below, more than 31 in z: no mass in units, and the k-th id if no earlier class has it.
__device__ __forceinline__ FilterInfo find_classes(const FilterArgs& a, float top, double line, const double* mass, const unsigned* count) {
  const int lane = threadIdx.x;
  double m[4], sm = 0.0;
  unsigned n[4], sn = 0;                           // inclusive sums inside the lane
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sm += mass[lane * 4 + i];
    sn += count[lane * 4 + i];
    m[i] = sm;
    n[i] = sn;
  }
  const double im = wave_scan_t(sm), bm = wave_before_t(im);
  const unsigned in = wave_scan_t(sn), bn = in - sn;
  FilterInfo f;
  f.mass = lane_t(im, 63);
  // first class whose inclusive sums `reached` accepts, else the last one, and the sums before it
  auto first = [&](auto reached, double* before_m, int* before_n, double* upto) {
    int k = -1;
#pragma unroll
    for (int i = 3; i >= 0; --i)
      if (reached(bm + m[i], bn + n[i])) k = i;
    const u64 some = __ballot(k >= 0);
    const int at = some ? __ffsll((long long)some) - 1 : 63, pick = some ? k : 3;
    double pm = bm, um = bm + m[0];
    unsigned pn = bn;
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (pick == i) pm = bm + m[i - 1], pn = bn + n[i - 1], um = bm + m[i];
    *before_m = lane_t(pm, at);
    *before_n = (int)lane_t(pn, at);
    *upto = lane_t(um, at);
    return lane_t(lane * 4 + pick, at);
  };
  double upto = f.mass, skip_m;
  int skip_n;
  f.kbin = FL_BINS;
  f.m_before_k = f.mass;
  f.n_before = 0;
  if (a.top_k) f.kbin = first([&](double, unsigned c) { return c >= (unsigned)a.top_k; }, &f.m_before_k, &f.n_before, &upto);
  f.plo = f.phi = FL_BINS;
  f.m_before_p = 0.0;
  if (a.top_p < 1.0) {                             // the k ids' mass lies between these two
    const double lo = a.top_p * f.m_before_k, hi = a.top_p * upto;
    double skip;
    f.plo = first([&](double s, unsigned) { return s >= lo; }, &f.m_before_p, &skip_n, &skip);
    f.phi = first([&](double s, unsigned) { return s >= hi; }, &skip_m, &skip_n, &skip);
  }
  f.low = FL_BINS;
  if (a.min_p > 0.0) {                             // a class's largest z is that of the grid line above it
    int k = 4;
#pragma unroll
    for (int i = 3; i >= 0; --i)
      if (weight(fmax((double)top * a.mult - (line - (lane * 4 + i) + 1.0) / FL_GRID, 0.0)) < a.min_p * 0.999) k = i;
    const u64 some = __ballot(k < 4);
    if (some) {
      const int at = __ffsll((long long)some) - 1;
      f.low = at * 4 + lane_t(k, at);
    }
    // Borders among ids that min-p leaves out anyway; but as long as top-p's counts, it takes its share of the mass of the first k
    // ids, so the k-th is still looked for (not in the last class, whose ids have no units).
    if (f.plo >= f.low) f.plo = f.phi = FL_BINS;
    if (f.kbin >= f.low && (f.plo == FL_BINS || f.kbin == FL_BINS - 1)) {
      f.mass = f.m_before_k;
      f.kbin = FL_BINS;
    }
  }
  return f;
}

template <int Q>
__global__ __launch_bounds__(FL_THREADS) void filter_collect_kernel(FilterArgs a) {
  __shared__ double mass[2][FL_BINS], factor[FL_CHUNKS_MAX];
  __shared__ unsigned count[2][FL_BINS], listed[FL_WAVES], base;
  __shared__ int shift[FL_CHUNKS_MAX];
  __shared__ u64 sums[FL_WAVES];
  __shared__ FilterInfo info;
  const int chunk = blockIdx.x, row = blockIdx.y, w = threadIdx.x >> 6;
  float x[Q][4];
  load_chunk(a, row, chunk, x);
  const float t = threadIdx.x < a.C ? a.w.top[(size_t)row * a.C + threadIdx.x] : -INFINITY;
  const float top = row_top(a, row);
  if (has_none(top)) return;
  const double line = line_of(top, a.mult);
  if (threadIdx.x < a.C) {                         // chunk c's classes count from its own largest z, on the same grid
    const double s = line - line_of(t, a.mult);
    shift[threadIdx.x] = s < FL_BINS ? (int)s : FL_BINS;
    factor[threadIdx.x] = weight(distance(top, t, a.mult)) / FL_ONE;
  }
  __syncthreads();
  {
    const int b = threadIdx.x & (FL_BINS - 1), half = threadIdx.x / FL_BINS;
    const size_t rows = (size_t)row * a.C * FL_BINS;
    double m = 0.0;
    unsigned n = 0;
    for (int c = half; c < a.C; c += 16) {         // eight chunks' loads at a time
      u64 v[8];
      unsigned k[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = min(c + 2 * i, a.C - 1), from = max(b - shift[d], 0);
        v[i] = a.w.mass[rows + (size_t)d * FL_BINS + from];
        k[i] = 0;
        if (a.top_k) k[i] = a.w.count[rows + (size_t)d * FL_BINS + from];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = c + 2 * i;
        if (d < a.C && b >= shift[d]) {
          m += (double)v[i] * factor[d];
          n += k[i];
        }
      }
    }
    mass[half][b] = m;
    count[half][b] = n;
  }
  __syncthreads();
  if (threadIdx.x < FL_BINS) {
    mass[0][threadIdx.x] += mass[1][threadIdx.x];
    count[0][threadIdx.x] += count[1][threadIdx.x];
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const FilterInfo f = find_classes(a, top, line, mass[0], count[0]);
    if (threadIdx.x == 0) {
      info = f;
      if (chunk == 0) a.w.info[row] = f;
    }
  }
  __syncthreads();
  const int kbin = info.kbin, plo = info.plo, phi = info.phi, sure_below = min(min(plo, kbin), info.low);
  u64 sum = 0;
  unsigned mine = 0;
#pragma unroll
  for (int j = 0; j < Q; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = class_of(line, x[j][i], a.mult);
      if (b < sure_below) {
        const double v = weight(distance(top, x[j][i], a.mult));
        if (v >= a.min_p) sum += units(v);
      }
      if (id_of<Q>(chunk, j, i) < a.V && (b == kbin || (b >= plo && b <= phi))) mine |= 1u << (j * 4 + i);
    }
  sum = wave_sum_t(sum);
  const unsigned n = __popc(mine), in = wave_scan_t(n);
  if ((threadIdx.x & 63) == 63) sums[w] = sum, listed[w] = in;
  __syncthreads();
  unsigned at = in - n, all = 0;
#pragma unroll
  for (int i = 0; i < FL_WAVES; ++i) {
    if (i == w) at += all;
    all += listed[i];
  }
  if (threadIdx.x == 0) {
    base = all ? atomicAdd(&a.w.listed[row], all) : 0;
    sum = 0;
#pragma unroll
    for (int i = 0; i < FL_WAVES; ++i) sum += sums[i];
    a.w.kept[(size_t)row * a.C + chunk] = (double)sum;
  }
  __syncthreads();
  at += base;
#pragma unroll
  for (int j = 0; j < Q; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (mine >> (j * 4 + i) & 1) {
        if (at < (unsigned)a.L) a.w.list[(size_t)row * a.L + at] = order_of(x[j][i], id_of<Q>(chunk, j, i));
        ++at;
      }
}

// Of the keys that each(visit(key, amount)) goes through (amount > 0, every key once, `first` to `last`), the one at which the
// running sum of the amounts, by rising key, is first accepted by reached(sum); the last key, should none be; 0 without keys.
// Digits of 8 bits from the highest bit that is not the same in `first` and `last`; once few are left, they are compared with
// each other.
#define FL_RANK 128               // keys that are compared with each other instead
struct SelectLds {
  u64 hist[2][256], keys[FL_RANK], amounts[FL_RANK], upto[FL_RANK], before, key;
  unsigned count[2][256], rank[FL_RANK], pick, left, filled;
};
// For each of n <= FL_RANK different keys, how many are no larger (rank) and what these amount to (upto; both cleared before): a
// lane's two keys against an eighth of them per wave.
template <int W>
__device__ __forceinline__ void rank_keys(int n, const u64* keys, const u64* amounts, SelectLds& s) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const u64 k0 = lane < n ? keys[lane] : 0, k1 = 64 + lane < n ? keys[64 + lane] : 0;
  u64 u0 = 0, u1 = 0;
  unsigned r0 = 0, r1 = 0;
#pragma unroll 4
  for (int i = w * n / W; i < (w + 1) * n / W; ++i) {
    const u64 k = keys[i], m = amounts[i];
    u0 += k <= k0 ? m : 0;
    u1 += k <= k1 ? m : 0;
    r0 += k <= k0;
    r1 += k <= k1;
  }
  if (lane < n) atomicAdd(&s.upto[lane], u0), atomicAdd(&s.rank[lane], r0);
  if (64 + lane < n) atomicAdd(&s.upto[64 + lane], u1), atomicAdd(&s.rank[64 + lane], r1);
  __syncthreads();
}
template <int W, typename E, typename R>
__device__ u64 select_key(const E& each, const R& reached, u64 first, u64 last, unsigned left, SelectLds& s) {
  const int lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < 256; i += (W * 64)) s.hist[0][i] = 0, s.count[0][i] = 0;
  if (threadIdx.x < FL_RANK) s.upto[threadIdx.x] = 0, s.rank[threadIdx.x] = 0;
  if (threadIdx.x == 0) s.key = 0, s.filled = 0;
  __syncthreads();
  int shift = (first ^ last) >> 8 ? 56 - __clzll((long long)(first ^ last)) : 0;
  u64 before = 0;                                  // sum of what comes before `first`
  for (int b = 0;; b ^= 1) {
    if (left <= FL_RANK) {
      each([&](u64 k, u64 amount) {
        if (k >= first && k <= last) {
          const unsigned at = atomicAdd(&s.filled, 1u);
          s.keys[at] = k;
          s.amounts[at] = amount;
        }
      });
      __syncthreads();
      left = s.filled;
      rank_keys<W>(left, s.keys, s.amounts, s);
      if (threadIdx.x < left) {
        const u64 upto = before + s.upto[threadIdx.x];
        const unsigned rank = s.rank[threadIdx.x];
        const bool good = reached(upto);
        if (good ? rank == 1 || !reached(upto - s.amounts[threadIdx.x]) : rank == left) s.key = s.keys[threadIdx.x];
      }
      __syncthreads();
      first = s.key;
      break;
    }
    each([&](u64 k, u64 amount) {
      if (k >= first && k <= last) {
        atomicAdd(&s.hist[b][k >> shift & 255], amount);
        atomicAdd(&s.count[b][k >> shift & 255], 1u);
      }
    });
    __syncthreads();
    if (threadIdx.x < 64) {
      u64 h[4], sum = 0;
      unsigned c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum += s.hist[b][lane * 4 + i];
        h[i] = sum;
        c[i] = s.count[b][lane * 4 + i];
      }
      const u64 start = before + wave_scan_t(sum) - sum;
      int k = -1, some = -1;
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        if (c[i] && some < 0) some = i;
        if (c[i] && reached(start + h[i])) k = i;
      }
      const u64 good = __ballot(k >= 0), filled = __ballot(some >= 0);
      const int at = good ? __ffsll((long long)good) - 1 : filled ? 63 - __clzll((long long)filled) : 0, pick = good ? k : some < 0 ? 0 : some;
      u64 pm = start;
      unsigned n = c[0];
#pragma unroll
      for (int i = 1; i < 4; ++i)
        if (pick == i) pm = start + h[i - 1], n = c[i];
      if (lane == at) s.pick = lane * 4 + pick, s.before = pm, s.left = n;
    } else if (threadIdx.x >= (W * 64) - 256) {
      s.hist[b ^ 1][threadIdx.x - ((W * 64) - 256)] = 0;
      s.count[b ^ 1][threadIdx.x - ((W * 64) - 256)] = 0;
    }
    __syncthreads();
    first = (first >> shift & ~255ull | s.pick) << shift;
    last = first | ((1ull << shift) - 1);
    before = s.before;
    left = s.left;
    if (shift == 0) break;
    shift = shift > 8 ? shift - 8 : 0;
  }
  __syncthreads();
  return first;
}

// The border of a row among its candidates: the list, or where it did not hold them the row itself.
__global__ __launch_bounds__(FL_THREADS) void filter_resolve_kernel(FilterArgs a) {
  extern __shared__ u64 filter_lds[];              // FL_LIST orders, FL_LIST units
  u64 *list = filter_lds, *amount = filter_lds + FL_LIST;
  __shared__ u64 sh[FL_WAVES], chunk_mass[FL_CHUNKS_MAX];
  __shared__ SelectLds lds;
  const int row = blockIdx.x;
  const float top = row_top(a, row);
  if (has_none(top)) return;
  const FilterInfo f = a.w.info[row];
  const double line = line_of(top, a.mult);
  // orders of a class's ids lie between these (class 0 starts at the row's largest, the last one has no end)
  auto from = [&](int b) { return b <= 0 ? order_of(top, 0) : first_order((float)((line - b + 1.0) / FL_GRID / a.mult)); };
  auto to = [&](int b) { return b >= FL_BINS - 1 ? last_order(-INFINITY) : last_order((float)((line - b) / FL_GRID / a.mult)); };
  const float* x = a.logits + (size_t)row * a.ld;
  const unsigned listed = a.w.listed[row];
  const bool whole = listed > (unsigned)a.L;
  const int n = whole ? a.V : (int)listed;
  for (int c = threadIdx.x; c < a.C; c += FL_THREADS) chunk_mass[c] = 0;
  if (!whole)
    for (int i = threadIdx.x; i < n; i += FL_THREADS) {
      const u64 o = a.w.list[(size_t)row * a.L + i];
      list[i] = o;
      amount[i] = units(weight(distance(top, logit_of(o), a.mult)));
    }
  __syncthreads();
  // use(order, class, units) of every candidate
  auto candidates = [&](auto use) {
    for (int i = threadIdx.x; i < n; i += FL_THREADS) {
      const float v = whole ? x[i] : logit_of(list[i]);
      const int b = class_of(line, v, a.mult);
      if (!whole) use(list[i], b, amount[i]);
      else if (b == f.kbin || (b >= f.plo && b <= f.phi)) use(order_of(v, i), b, units(weight(distance(top, v, a.mult))));
    }
  };
  u64 last = ~0ull;
  double mass_k = f.mass;
  if (f.kbin < FL_BINS) {
    const u64 rank = (u64)(a.top_k - f.n_before);
    last = select_key<FL_WAVES>([&](auto visit) { candidates([&](u64 o, int b, u64) { if (b == f.kbin) visit(o, 1ull); }); },
                      [&](u64 s) { return s >= rank; }, from(f.kbin), to(f.kbin), listed, lds);
    u64 m = 0;
    candidates([&](u64 o, int b, u64 w) { if (b == f.kbin && o <= last) m += w; });
    mass_k = f.m_before_k + (double)block_sum_t(m, sh) / FL_ONE;
  }
  if (f.plo < FL_BINS) {
    const double goal = (a.top_p * mass_k - f.m_before_p) * FL_ONE;
    const u64 upto = last;
    last = select_key<FL_WAVES>([&](auto visit) { candidates([&](u64 o, int b, u64 w) { if (b >= f.plo && b <= f.phi && o <= upto && w) visit(o, w); }); },
                      [&](u64 s) { return (double)s >= goal; }, from(f.plo), to(f.phi), listed, lds);
  }
  candidates([&](u64 o, int, u64 w) {
    if (o <= last && weight(distance(top, logit_of(o), a.mult)) >= a.min_p && w) atomicAdd(&chunk_mass[(unsigned)o / (unsigned)a.chunk], w);
  });
  __syncthreads();
  for (int c = threadIdx.x; c < a.C; c += FL_THREADS) a.w.kept[(size_t)row * a.C + c] += (double)chunk_mass[c];
  if (threadIdx.x == 0) a.w.end[row].last = last;
}

// ---- results --------------------------------------------------------------------------------------------------------
enum { FINISH_ALL = 0 /* nothing truncated but by min-p = 0 */, FINISH_KEPT = 1 /* masses of the chunks */, FINISH_CLASSES = 2 /* and a border */,
       FINISH_WRITE = 3 /* border, total and token are there */ };
template <int Q>
__global__ __launch_bounds__(FL_THREADS) void filter_finish_kernel(FilterArgs a, int mode) {
  __shared__ u64 sums[Q][FL_WAVES];
  const int chunk = blockIdx.x, row = blockIdx.y, lane = threadIdx.x & 63;
  float x[Q][4];
  load_chunk(a, row, chunk, x);
  // whatever the row's passes have left, read at once
  const float* tops = a.w.top + (size_t)row * a.C;
  float t[2];
  double m[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = lane * 2 + i;
    t[i] = mode == FINISH_WRITE ? tops[0] : c < a.C ? tops[c] : -INFINITY;
    m[i] = 0.0;
    if (c < a.C && mode < FINISH_WRITE && !a.greedy) m[i] = (mode == FINISH_ALL ? a.w.sum : a.w.kept)[(size_t)row * a.C + c];
  }
  const float ref = tops[mode == FINISH_WRITE ? 0 : chunk];
  const u64 last = mode >= FINISH_CLASSES ? a.w.end[row].last : ~0ull;
  const double u = a.tok && a.u ? (double)a.u[row] : 0.0;
  const float top = wave_max_f(fmaxf(t[0], t[1]));
  if (a.greedy || has_none(top)) {
    int best = 0;
    if (a.greedy) {                                // the lowest chunk that has the largest logit
      const u64 even = __ballot(lane * 2 < a.C && t[0] == top), odd = __ballot(lane * 2 + 1 < a.C && t[1] == top);
      const int e = even ? __ffsll((long long)even) * 2 - 2 : 256, o = odd ? __ffsll((long long)odd) * 2 - 1 : 256;
      best = a.w.top_id[(size_t)row * a.C + min(e, o)];
    }
    if (a.tok && chunk == 0 && threadIdx.x == 0 && mode != FINISH_WRITE) a.tok[row] = a.greedy ? best : -1;
#pragma unroll
    for (int j = 0; j < Q; ++j) {
      float q[4], m[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool on = id_of<Q>(chunk, j, i) == best;
        q[i] = !a.greedy ? __builtin_nanf("") : on ? 1.0f : 0.0f;
        m[i] = !a.greedy ? __builtin_nanf("") : on ? x[j][i] : -INFINITY;
      }
      if (a.q) put4(a.q, a, row, id_of<Q>(chunk, j, 0), q);
      if (a.masked) put4(a.masked, a, row, id_of<Q>(chunk, j, 0), m);
    }
    return;
  }
  // units of every chunk, two per lane, and their running sums: the same in every wave and workgroup
  double before = 0.0, here = 0.0, total, goal = 0.0;
  bool mine = false;
  if (mode == FINISH_WRITE) {
    total = a.w.end[row].total;
  } else {
    if (mode == FINISH_ALL) {                      // sums that count from the chunk's own largest weight
#pragma unroll
      for (int i = 0; i < 2; ++i) m[i] = t[i] > -INFINITY ? m[i] * weight(distance(top, t[i], a.mult)) * FL_ONE : 0.0;
    }
    const double in = wave_scan_t(m[0] + m[1]), ex = wave_before_t(in);
    total = lane_t(in, 63);
    if (a.tok) {
      goal = fmin(fmax(u, 0.0), 1.0) * total;
      // the first chunk whose running sum passes the goal, else the last one with any mass
      const u64 p0 = __ballot(m[0] > 0.0 && ex + m[0] > goal), p1 = __ballot(m[1] > 0.0 && ex + m[0] + m[1] > goal);
      const u64 f0 = __ballot(m[0] > 0.0), f1 = __ballot(m[1] > 0.0);
      int c;
      if (p0 | p1) {
        const int l0 = p0 ? __ffsll((long long)p0) - 1 : 64, l1 = p1 ? __ffsll((long long)p1) - 1 : 64;
        c = l0 <= l1 ? l0 * 2 : l1 * 2 + 1;
      } else {
        const int l0 = f0 ? 63 - __clzll((long long)f0) : -1, l1 = f1 ? 63 - __clzll((long long)f1) : -1;
        c = l1 >= l0 ? l1 * 2 + 1 : l0 * 2;
      }
      mine = c == chunk;
      before = lane_t(chunk & 1 ? ex + m[0] : ex, chunk >> 1);
      here = lane_t(chunk & 1 ? m[1] : m[0], chunk >> 1);
    }
  }
  if (!a.q && !a.masked && !mine) return;
  const double inv = FL_ONE / total;
  unsigned kept = 0;
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    float q[4], m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int id = id_of<Q>(chunk, j, i);
      q[i] = 0.0f;
      m[i] = -INFINITY;
      if (id < a.V && (last == ~0ull || order_of(x[j][i], id) <= last)) {
        const double w = weight(distance(top, x[j][i], a.mult));
        if (w >= a.min_p) {
          kept |= 1u << (j * 4 + i);
          q[i] = (float)(w * inv);
          m[i] = x[j][i];
        }
      }
    }
    if (a.q) put4(a.q, a, row, id_of<Q>(chunk, j, 0), q);
    if (a.masked) put4(a.masked, a, row, id_of<Q>(chunk, j, 0), m);
  }
  if (!mine) return;
  // The id inside the chunk, in units of the chunk's own largest weight (it is kept if any of the chunk is), so that there are
  // some however small the chunk's share is.
  u64 start = 0, own[Q], scan[Q];
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    own[j] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) own[j] += kept >> (j * 4 + i) & 1 ? units(weight(distance(ref, x[j][i], a.mult))) : 0;
    scan[j] = wave_scan_t(own[j]);
    if (lane == 63) sums[j][threadIdx.x >> 6] = scan[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < Q; ++j)
#pragma unroll
    for (int i = 0; i < FL_WAVES; ++i) {
      if (i == (int)(threadIdx.x >> 6)) scan[j] += start - own[j];       // exclusive, from the chunk's first id on
      start += sums[j][i];
    }
  u64 want = (u64)(fmin(fmax((goal - before) / here, 0.0), 1.0) * (double)start);
  if (want >= start) want = start - 1;
#pragma unroll
  for (int j = 0; j < Q; ++j)
    if (scan[j] <= want && want < scan[j] + own[j]) {
      u64 at = scan[j];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u64 v = kept >> (j * 4 + i) & 1 ? units(weight(distance(ref, x[j][i], a.mult))) : 0;
        if (at <= want && want < at + v) a.tok[row] = id_of<Q>(chunk, j, i);
        at += v;
      }
    }
}

// ---- few ids --------------------------------------------------------------------------------------------------------
// The largest of every 16 ids (four lanes' quads), and the results cleared unless they replace the logits.
template <int Q>
__global__ __launch_bounds__(FL_THREADS) void filter_groups_kernel(FilterArgs a, int clear) {
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[Q][4];
  load_chunk(a, row, chunk, x);
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    float v = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) v = x[j][i] < INFINITY ? fmaxf(v, x[j][i]) : INFINITY;
    v = fmaxf(v, __shfl_xor(v, 1));
    v = fmaxf(v, __shfl_xor(v, 2));
    const int g = id_of<Q>(chunk, j, 0) / FL_GROUP;
    if ((threadIdx.x & 3) == 0) a.w.group[(size_t)row * a.G + g] = v;
    if (clear) {
      const float zero[4] = {0.f, 0.f, 0.f, 0.f}, none[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (a.q) put4(a.q, a, row, id_of<Q>(chunk, j, 0), zero);
      if (a.masked) put4(a.masked, a, row, id_of<Q>(chunk, j, 0), none);
    }
  }
}

// One workgroup per row: the groups that may matter, their ids, the borders, the draw and the results.
#define FL_FEW_LIST 4096
template <int W>
__global__ __launch_bounds__(W * 64) void filter_few_kernel(FilterArgs a, int clear) {
  constexpr int THREADS = W * 64;
  __shared__ u64 list[FL_FEW_LIST], amount[FL_FEW_LIST], sh[W];
  __shared__ float shf[W];
  __shared__ unsigned count[FL_BINS], picked, listed;
  __shared__ int bin;
  __shared__ SelectLds lds;
  int* groups = reinterpret_cast<int*>(amount);    // until the ids are listed
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const float* g = a.w.group + (size_t)row * a.G;
  const float* x = a.logits + (size_t)row * a.ld;
  // use(group, largest logit) of all of them: sixteen of a thread's at a time, the first sixteen stay in registers
  f32x4 own_groups[4];
  auto load_groups = [&](int i0, f32x4 (&v)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + k * THREADS * 4;
      v[k] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (i < a.G) v[k] = *reinterpret_cast<const f32x4*>(g + i);         // a multiple of 128 of them
    }
  };
  auto use_groups = [&](int i0, const f32x4 (&v)[4], auto use) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + k * THREADS * 4 + e;
        if (i < a.G) use(i, v[k][e]);
      }
  };
  load_groups(threadIdx.x * 4, own_groups);
  auto all_groups = [&](auto use) {
    use_groups(threadIdx.x * 4, own_groups, use);
    for (int i0 = threadIdx.x * 4 + THREADS * 16; i0 < a.G; i0 += THREADS * 16) {
      f32x4 v[4];
      load_groups(i0, v);
      use_groups(i0, v, use);
    }
  };
  float mx = -INFINITY;
  all_groups([&](int, float v) { mx = fmaxf(mx, v); });
  mx = wave_max_f(mx);
  if (lane == 0) shf[threadIdx.x >> 6] = mx;
  if (threadIdx.x < FL_BINS) count[threadIdx.x] = 0;
  if (threadIdx.x == 0) picked = listed = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) mx = fmaxf(mx, shf[i]);
  if (has_none(mx)) {
    if (threadIdx.x == 0) {
      if (a.tok) a.tok[row] = -1;
      a.w.top[(size_t)row * a.C] = INFINITY;
    }
    if (clear)
      for (int i = threadIdx.x; i < a.V; i += THREADS) {
        if (a.q) a.q[(size_t)row * a.V + i] = __builtin_nanf("");
        if (a.masked) a.masked[(size_t)row * a.V + i] = __builtin_nanf("");
      }
    return;
  }
  // The class of the k-th largest group; where fewer groups are that near, everything.  Any classes will do whose number falls
  // with the logit: these, in fp32, are about 1/8 wide in z.
  const float per = (float)fmin(fmax(a.mult * FL_GRID, 1e-30), 1e30);
  auto class_f = [&](float v) { return fminf((mx - v) * per, FL_BINS - 1.0f); };
  all_groups([&](int, float v) {
    const int b = (int)class_f(v);
    if (b < FL_BINS - 1) atomicAdd(&count[b], 1u);
  });
  __syncthreads();
  if (threadIdx.x < 64) {
    unsigned n[4], s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s += count[lane * 4 + i];
      n[i] = s;
    }
    const unsigned b = wave_scan_t(s) - s;
    int k = 4;
#pragma unroll
    for (int i = 3; i >= 0; --i)
      if (b + n[i] >= (unsigned)a.top_k) k = i;
    const u64 some = __ballot(k < 4);
    if (some ? lane == __ffsll((long long)some) - 1 : lane == 0) bin = some ? lane * 4 + k : FL_BINS - 1;
  }
  __syncthreads();
  const float beyond = (float)(bin + 1);
  const u64 edge = bin == FL_BINS - 1 ? last_order(-INFINITY) : last_order(mx - beyond / per - fabsf(mx) * 1e-6f);
  all_groups([&](int i, float v) {
    if (class_f(v) < beyond) {
      const unsigned at = atomicAdd(&picked, 1u);
      if (at < 2 * FL_FEW_LIST) groups[at] = i;
    }
  });
  __syncthreads();
  bool whole = picked > 2 * FL_FEW_LIST;           // then every id of the row is looked at
  if (!whole) {
    const int n = (int)picked * 4;                 // quads, four loads of a thread at a time
    for (int i0 = 0; i0 < n; i0 += THREADS * 4) {          // whole waves: they count together
      f32x4 v[4];
      int id[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = i0 + k * THREADS + threadIdx.x;
        id[k] = i < n ? groups[i >> 2] * FL_GROUP + (i & 3) * 4 : a.V;
        if (id[k] + 4 <= a.V) {
          v[k] = *reinterpret_cast<const f32x4u*>(x + id[k]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[k][e] = id[k] + e < a.V ? x[id[k] + e] : -INFINITY;
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i0 + k * THREADS >= n) break;
        unsigned mine = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (id[k] + e < a.V && class_f(v[k][e]) < beyond) mine |= 1u << e;
        const unsigned in = wave_scan_t((unsigned)__popc(mine)), all = lane_t(in, 63);
        unsigned at = 0;
        if (lane == 0 && all) at = atomicAdd(&listed, all);
        at = lane_t(at, 0) + in - __popc(mine);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (mine >> e & 1) {
            if (at < FL_FEW_LIST) list[at] = order_of(v[k][e], id[k] + e);
            ++at;
          }
      }
    }
    __syncthreads();
    whole = listed > FL_FEW_LIST;
  }
  const int n = whole ? a.V : (int)listed;
  if (!whole)
    for (int i = threadIdx.x; i < n; i += THREADS) amount[i] = units(weight(distance(mx, logit_of(list[i]), a.mult)));
  if (threadIdx.x < FL_RANK) lds.upto[threadIdx.x] = 0, lds.rank[threadIdx.x] = 0;
  __syncthreads();
  auto candidates = [&](auto use) {                // use(order, units) of every one
    for (int i = threadIdx.x; i < n; i += THREADS) {
      if (!whole) use(list[i], amount[i]);
      else if (class_f(x[i]) < beyond) use(order_of(x[i], i), units(weight(distance(mx, x[i], a.mult))));
    }
  };
  const double u = a.tok ? fmin(fmax((double)a.u[row], 0.0), 1.0) : 0.0;
  u64 last, total;
  auto kept = [&](u64 o) { return o <= last && (a.min_p == 0.0 || weight(distance(mx, logit_of(o), a.mult)) >= a.min_p); };
  if (n <= FL_RANK) {                              // one comparison of all with all gives both borders, a second one the draw
    rank_keys<W>(n, list, amount, lds);
    const bool in = (int)threadIdx.x < n;
    const u64 own = in ? list[threadIdx.x] : ~0ull, w = in ? amount[threadIdx.x] : 0, upto = in ? lds.upto[threadIdx.x] : 0;
    const int rank = in ? (int)lds.rank[threadIdx.x] : n + 1;
    if (rank == min(a.top_k, n)) lds.key = own, lds.before = upto;
    __syncthreads();
    last = lds.key;
    if (a.top_p < 1.0) {
      const double goal = a.top_p * (double)lds.before;
      __syncthreads();
      if (own <= last && (double)upto >= goal && (rank == 1 || (double)(upto - w) < goal)) lds.key = own;
      __syncthreads();
      last = lds.key;
    }
    const u64 mine = in && kept(own) ? w : 0;
    if (threadIdx.x < FL_RANK) {
      lds.keys[threadIdx.x] = (unsigned)own;
      lds.amounts[threadIdx.x] = mine;
      lds.upto[threadIdx.x] = 0;
    }
    total = block_sum_t<W>(mine, sh);
    rank_keys<W>(n, lds.keys, lds.amounts, lds);
    u64 goal = (u64)(u * (double)total);
    if (goal >= total) goal = total - 1;
    const u64 sum = in ? lds.upto[threadIdx.x] : 0;
    if (a.tok && sum > goal && sum - mine <= goal) a.tok[row] = (int)(unsigned)own;
  } else {
    const u64 like = order_of(mx, 0);
    last = select_key<W>([&](auto visit) { candidates([&](u64 o, u64) { visit(o, 1ull); }); },
                      [&](u64 s) { return s >= (u64)a.top_k; }, like, edge, n, lds);
    if (a.top_p < 1.0) {
      u64 m = 0;
      const u64 upto = last;
      candidates([&](u64 o, u64 w) { if (o <= upto) m += w; });
      const double goal = a.top_p * (double)block_sum_t<W>(m, sh);
      last = select_key<W>([&](auto visit) { candidates([&](u64 o, u64 w) { if (o <= upto && w) visit(o, w); }); },
                        [&](u64 s) { return (double)s >= goal; }, like, upto, n, lds);
    }
    u64 m = 0;
    candidates([&](u64 o, u64 w) { if (kept(o)) m += w; });
    total = block_sum_t<W>(m, sh);
    if (a.tok) {
      u64 goal = (u64)(u * (double)total);
      if (goal >= total) goal = total - 1;
      const u64 id = select_key<W>([&](auto visit) { candidates([&](u64 o, u64 w) { if (w && kept(o)) visit((u64)(unsigned)o, w); }); },
                                [&](u64 s) { return s > goal; }, 0, a.V - 1, n, lds);
      if (threadIdx.x == 0) a.tok[row] = (int)id;
    }
  }
  if (!clear) {
    if (threadIdx.x == 0) {
      a.w.end[row] = FilterEnd{last, (double)total};
      a.w.top[(size_t)row * a.C] = mx;
    }
    return;
  }
  const double inv = FL_ONE / (double)total;
  candidates([&](u64 o, u64) {
    if (!kept(o)) return;
    const size_t at = (size_t)row * a.V + (unsigned)o;
    if (a.q) a.q[at] = (float)(weight(distance(mx, logit_of(o), a.mult)) * inv);
    if (a.masked) a.masked[at] = x[(unsigned)o];
  });
}

// ---- the call -------------------------------------------------------------------------------------------------------
// Quads of a chunk: as few as still leave no more than two workgroups per CU (256 of them), so that a workgroup's share of 64-bit
// work is small.  Every workgroup of `collect` reads all chunks' classes (3 KiB each), so there not beyond 25 MB of that: one row
// of 160000 ids, top-p 0.9, 39 -> 31 us.  At most 128 chunks: two per lane.  By rows and ids alone, so that the workspace can be
// sized.
static int filter_quads(int rows, int V, bool classes) {
  int q = FL_QUADS_MAX;
  while (q > 1) {
    const long long C = (V + FL_QUAD * (q / 2) - 1) / (FL_QUAD * (q / 2));
    if (C * rows > 512 || C > 128 || (classes && C * C * rows > 8192)) break;
    q /= 2;
  }
  return q;
}
static size_t filter_chunks(int V, int quads) { return ((size_t)V + FL_QUAD * quads - 1) / (FL_QUAD * quads); }
static int filter_room(int V) { return V < FL_LIST ? V : FL_LIST; }
static size_t filter_layout(int rows, int V, char* base, FilterWork* w) {
  const size_t n = rows, classes = filter_chunks(V, filter_quads(rows, V, true));
  const size_t few = filter_chunks(V, filter_quads(rows, V, false)), C = few > classes ? few : classes;
  const size_t groups = filter_chunks(V, FL_QUADS_MAX) * (FL_QUAD * FL_QUADS_MAX / FL_GROUP);      // whole chunks of any size
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = base + at;
    at += (bytes + 15) & ~(size_t)15;
    return p;
  };
  w->mass = (u64*)take(n * classes * FL_BINS * 8);
  w->list = (u64*)take(n * filter_room(V) * 8);
  w->count = (unsigned*)take(n * classes * FL_BINS * 4);
  w->kept = (double*)take(n * C * 8);
  w->top = (float*)take(n * C * 4);
  w->top_id = (int*)take(n * C * 4);
  w->sum = (double*)take(n * C * 8);
  w->info = (FilterInfo*)take(n * sizeof(FilterInfo));
  w->end = (FilterEnd*)take(n * sizeof(FilterEnd));
  w->listed = (unsigned*)take(n * 4);
  w->group = (float*)take(n * groups * 4);
  return at;
}
size_t filter_work_bytes(int rows, int V) {
  FilterWork w;
  return filter_layout(rows, V, nullptr, &w);
}
template <int Q>
static hipError_t launch_filter(FilterArgs a, int rows, hipStream_t st) {
  a.chunk = Q * FL_QUAD;
  a.C = (a.V + a.chunk - 1) / a.chunk;
  a.G = a.C * (a.chunk / FL_GROUP);                // whole chunks of them
  const dim3 grid(a.C, rows), block(FL_THREADS);
  if (!a.greedy && a.top_k && a.top_k <= FL_FEW) {
    const int clear = a.q != a.logits && a.masked != a.logits;
    filter_groups_kernel<Q><<<grid, block, 0, st>>>(a, clear);
    // 16 waves where many ids are compared digit by digit, or where the row is long: their barriers cost more than they share as long
    // as few ids count, but take less than the whole row does that is read again and again if the k-th group lies far below (us
    // with top-p 0.9375, 8 | 16 waves):
    //   32000 ids     k 300 16.2 | 16.9    500 19.1 | 18.2    1000 23.4 | 21.2    k 50 at temperature 0.1 188 | 136
    //   128256        k 50  11.1 | 11.8    500 20.7 | 19.6    1000 25.8 | 23.4                            655 | 462
    //   160000        k 50  12.8 | 12.0   (8 waves' registers hold the groups of 131072)
    if (a.top_k > 384 || a.V > 65536) filter_few_kernel<16><<<rows, 1024, 0, st>>>(a, clear);
    else filter_few_kernel<8><<<rows, 512, 0, st>>>(a, clear);
    if (!clear) filter_finish_kernel<Q><<<grid, block, 0, st>>>(a, FINISH_WRITE);
    return hipGetLastError();
  }
  if (!a.greedy && (a.top_k || a.top_p < 1.0)) {
    const int bytes = 2 * FL_LIST * 8;
    hipError_t e = hipFuncSetAttribute((const void*)filter_resolve_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    filter_bins_kernel<Q><<<grid, block, 0, st>>>(a);
    filter_collect_kernel<Q><<<grid, block, 0, st>>>(a);
    filter_resolve_kernel<<<rows, block, bytes, st>>>(a);
    filter_finish_kernel<Q><<<grid, block, 0, st>>>(a, FINISH_CLASSES);
    return hipGetLastError();
  }
  const int all = !a.greedy && a.min_p == 0.0;
  if (a.greedy) filter_greedy_kernel<Q><<<grid, block, 0, st>>>(a);
  else filter_top_kernel<Q><<<grid, block, 0, st>>>(a, all);
  if (!a.greedy && !all) filter_mass_kernel<Q><<<grid, block, 0, st>>>(a);
  filter_finish_kernel<Q><<<grid, block, 0, st>>>(a, all ? FINISH_ALL : FINISH_KEPT);
  return hipGetLastError();
}
hipError_t launch_sample_rows(const float* logits, size_t ld, int rows, int V, const spec_sampling& s, const float* u, float* q,
                              float* masked, int* tok, void* work, hipStream_t st) {
  FilterArgs a = {};
  a.logits = logits;
  a.ld = ld;
  a.V = V;
  a.L = filter_room(V);
  a.greedy = s.temperature == 0.0f;
  a.mult = a.greedy ? 1.0 : (double)s.logit_scale / (double)s.temperature;
  a.top_k = s.top_k > 0 && s.top_k < V ? s.top_k : 0;
  a.top_p = s.top_p;
  a.min_p = s.min_p;
  a.u = u;
  a.q = q;
  a.masked = masked;
  a.tok = tok;
  filter_layout(rows, V, (char*)work, &a.w);
  const bool classes = !a.greedy && (a.top_k > FL_FEW || (!a.top_k && a.top_p < 1.0));
  const int quads = filter_quads(rows, V, classes);
  if (quads == 1) return launch_filter<1>(a, rows, st);
  if (quads == 2) return launch_filter<2>(a, rows, st);
  return launch_filter<4>(a, rows, st);
}
