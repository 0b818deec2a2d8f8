// Draws under temperature, top-k, top-p and min-p for gfx950, over rows of fp32 logits.
//
// With z = logit * scale / temperature and w = exp(z - max z), a row keeps, in the order of falling logits (equal ones by rising
// id): of the first k ids the shortest prefix that holds at least top_p of their mass, and of that the ids with w >= min_p.
// What is kept is renormalised; a draw is the first id, ascending, at which the running sum passes u times the total.
//
// Which id is the last one is decided at a border, and a draw next to one, so z and w are 64-bit and sums of w are integers, in
// units of 2^-43 (a sum of 2^20 of them fits 64 bits): exact, whatever order atomics come in.
//
// A row is cut into chunks of 8192 ids, so that one row uses many compute units.  Passes, each a launch over (chunk, row) unless
// said otherwise:
//   top      the chunk's largest logit
//   bins     counts and masses of 256 classes of z's distance from the row's largest (1/16 up to 12, then 1/4)
//   collect  every workgroup adds the chunks' classes up and finds those that hold the two borders; ids above them are in, those of
//            the border classes go to the row's list of candidates
//   resolve  one workgroup per row: the borders among the candidates by radix selection on (logit, id), masses of what is kept,
//            and the draw: the chunk, then the id inside it
//   write    the distribution, or the logits with -inf where an id is not kept
// Without top-k and top-p nothing has to be sorted: `bins` sums what min-p keeps and `resolve` follows.
#include "spec_internal.h"

#define FL_THREADS 512
#define FL_WAVES (FL_THREADS / 64)
#define FL_CHUNK 8192                     // ids of a chunk: 16 per thread, 4 neighbours at a time
#define FL_QUADS (FL_CHUNK / FL_THREADS / 4)
#define FL_CHUNKS_MAX (SPEC_SAMPLE_VOCAB_MAX / FL_CHUNK)
#define FL_BINS 256
#define FL_LIST 4096                      // candidates that are kept as a list; beyond, the row is read again
#define FL_ONE 0x1p43                     // a weight of 1
typedef unsigned long long u64;
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
static_assert(SPEC_SAMPLE_VOCAB_MAX <= 1 << 20, "sums of weights fit 64 bits");

struct FilterTop { float v; int id, bad, pad; };              // largest logit of a chunk, its lowest id, NaN or +inf seen
struct FilterInfo {                                           // borders of a row by classes
  int kbin, plo, phi, n_before;                               // class of the k-th id; classes that top-p may end in; ids before kbin
  u64 m_before_k, m_before_p, mass;                           // mass before kbin, before plo, of all
};
struct FilterEnd { u64 last, total; int bad, tok; };         // (logit, id) of the last kept id, mass of what is kept
struct FilterWork {                                           // arrays over the rows of a call
  FilterTop* top;      // [row][C]
  u64* mass;           // [row][C][FL_BINS]
  unsigned* count;     // [row][C][FL_BINS]
  u64* sure;           // [row][C]: mass that is kept whatever the candidates
  u64* list;           // [row][FL_LIST]
  FilterInfo* info;    // [row]
  FilterEnd* end;      // [row]
  unsigned* listed;    // [row]
};
struct FilterArgs {
  const float* logits;
  size_t ld;
  int V, C, greedy, top_k;       // top_k 0: off
  double mult, top_p, min_p;     // top_p 1: off
  const float* u;
  float *q, *masked;
  int* tok;
  FilterWork w;
};

// ---- one id ---------------------------------------------------------------------------------------------------------
// 64 bits that rise as an id falls in the order: logits by falling value, then ids
__device__ __forceinline__ u64 order_of(float x, int id) {
  const unsigned b = __float_as_uint(x + 0.0f);               // -0 counts as 0
  const unsigned key = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (u64)~key << 32 | (unsigned)id;
}
__device__ __forceinline__ float logit_of(u64 order) {
  const unsigned key = ~(unsigned)(order >> 32);
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
__device__ __forceinline__ double distance(float top, float x, double mult) { return ((double)top - (double)x) * mult; }
__device__ __forceinline__ double weight(double dist) { return exp(-dist); }
__device__ __forceinline__ u64 units(double w) { return (u64)(w * FL_ONE + 0.5); }
__device__ __forceinline__ int bin_of(double dist) {
  const double b = dist < 12.0 ? dist * 16.0 : 192.0 + (dist - 12.0) * 4.0;
  return b < FL_BINS - 1 ? (int)b : FL_BINS - 1;
}

// ---- a workgroup ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ u64 wave_sum_u(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ u64 wave_scan_u(u64 v) {           // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  return v;
}
__device__ __forceinline__ u64 block_sum_u(u64 v, u64* sh) {  // to every thread
  v = wave_sum_u(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 t = 0;
#pragma unroll
  for (int i = 0; i < FL_WAVES; ++i) t += sh[i];
  return t;
}
__device__ __forceinline__ u64 block_scan_u(u64 v, u64* sh, u64* total) {   // exclusive
  const int w = threadIdx.x >> 6;
  const u64 s = wave_scan_u(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sh[w] = s;
  __syncthreads();
  u64 before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < FL_WAVES; ++i) {
    if (i == w) before = all;
    all += sh[i];
  }
  *total = all;
  return before + s - v;
}

// the chunk's ids j * 2048 + 4 * thread + i; beyond V: -inf, which has no weight and comes last
__device__ __forceinline__ void load_chunk(const FilterArgs& a, int row, int chunk, float (&x)[FL_QUADS][4]) {
  const float* p = a.logits + (size_t)row * a.ld;
#pragma unroll
  for (int j = 0; j < FL_QUADS; ++j) {
    const int id = chunk * FL_CHUNK + j * FL_THREADS * 4 + threadIdx.x * 4;
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
__device__ __forceinline__ int id_of(int chunk, int j, int i) { return chunk * FL_CHUNK + j * FL_THREADS * 4 + threadIdx.x * 4 + i; }

struct RowTop { float v; int id; bool none; };                // none: no distribution
__device__ __forceinline__ FilterTop better(FilterTop a, FilterTop b) {
  const bool take = b.v > a.v || (b.v == a.v && b.id < a.id);
  a.v = take ? b.v : a.v;
  a.id = take ? b.id : a.id;
  a.bad |= b.bad;
  return a;
}
__device__ __forceinline__ FilterTop wave_better(FilterTop t) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    FilterTop s;
    s.v = __shfl_xor(t.v, o);
    s.id = __shfl_xor(t.id, o);
    s.bad = __shfl_xor(t.bad, o);
    t = better(t, s);
  }
  return t;
}
__device__ __forceinline__ RowTop row_top(const FilterArgs& a, int row) {    // by every wave for itself
  FilterTop t = {-INFINITY, 0, 0, 0};
  for (int c = threadIdx.x & 63; c < a.C; c += 64) t = better(t, a.w.top[(size_t)row * a.C + c]);
  t = wave_better(t);
  return RowTop{t.v, t.id, t.bad || t.v == -INFINITY};
}

// ---- the passes -----------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(FL_THREADS) void filter_top_kernel(FilterArgs a) {
  __shared__ FilterTop sh[FL_WAVES];
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[FL_QUADS][4];
  load_chunk(a, row, chunk, x);
  FilterTop t = {-INFINITY, 0x7fffffff, 0, 0};
#pragma unroll
  for (int j = 0; j < FL_QUADS; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (x[j][i] > t.v) t.v = x[j][i], t.id = id_of(chunk, j, i);     // a thread's ids ascend; NaN is never larger
      t.bad |= !(x[j][i] < INFINITY);
    }
  t = wave_better(t);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < FL_WAVES; ++i) t = better(t, sh[i]);
    if (t.id == 0x7fffffff) t.id = 0;
    a.w.top[(size_t)row * a.C + chunk] = t;
    if (chunk == 0) a.w.listed[row] = 0;
  }
}

__global__ __launch_bounds__(FL_THREADS) void filter_bins_kernel(FilterArgs a, int classes) {
  __shared__ u64 mass[FL_BINS], sh[FL_WAVES];
  __shared__ unsigned count[FL_BINS];
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[FL_QUADS][4];
  load_chunk(a, row, chunk, x);
  const RowTop top = row_top(a, row);
  if (top.none) return;
  if (!classes) {
    u64 sum = 0;
#pragma unroll
    for (int j = 0; j < FL_QUADS; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double w = weight(distance(top.v, x[j][i], a.mult));
        if (w >= a.min_p) sum += units(w);
      }
    sum = block_sum_u(sum, sh);
    if (threadIdx.x == 0) a.w.sure[(size_t)row * a.C + chunk] = sum;
    return;
  }
  if (threadIdx.x < FL_BINS) mass[threadIdx.x] = 0, count[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < FL_QUADS; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (id_of(chunk, j, i) < a.V) {
        const double d = distance(top.v, x[j][i], a.mult);
        const int b = bin_of(d);
        atomicAdd(&count[b], 1u);
        const u64 m = units(weight(d));
        if (m) atomicAdd(&mass[b], m);
      }
  __syncthreads();
  if (threadIdx.x < FL_BINS) {
    const size_t at = ((size_t)row * a.C + chunk) * FL_BINS + threadIdx.x;
    a.w.mass[at] = mass[threadIdx.x];
    a.w.count[at] = count[threadIdx.x];
  }
}

// first class whose inclusive sum reaches a target, by one wave of which lane l holds classes 4 l .. 4 l + 3
__global__ __launch_bounds__(FL_THREADS) void filter_collect_kernel(FilterArgs a) {
  __shared__ u64 mass[2][FL_BINS], sh[FL_WAVES];
  __shared__ unsigned count[2][FL_BINS], base;
  __shared__ FilterInfo info;
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[FL_QUADS][4];
  load_chunk(a, row, chunk, x);
  const RowTop top = row_top(a, row);
  if (top.none) return;
  {
    const int b = threadIdx.x & (FL_BINS - 1), half = threadIdx.x / FL_BINS;
    u64 m = 0;
    unsigned n = 0;
    for (int c = half; c < a.C; c += FL_THREADS / FL_BINS) {
      const size_t at = ((size_t)row * a.C + c) * FL_BINS + b;
      m += a.w.mass[at];
      n += a.w.count[at];
    }
    mass[half][b] = m;
    count[half][b] = n;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    u64 m[4], n[4], sm = 0, sn = 0;                // inclusive sums inside the lane
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sm += mass[0][lane * 4 + i] + mass[1][lane * 4 + i];
      sn += count[0][lane * 4 + i] + count[1][lane * 4 + i];
      m[i] = sm;
      n[i] = sn;
    }
    const u64 bm = wave_scan_u(sm) - sm, bn = wave_scan_u(sn) - sn;
    const u64 all = __shfl(bm + sm, 63);
    // class (and the sums before it) of the first inclusive sum that `reached` accepts; the sums rise, so it is one lane's
    auto first = [&](auto reached, int* bin, u64* before_m, u64* before_n) {
      int k = -1;
#pragma unroll
      for (int i = 3; i >= 0; --i)
        if (reached(bm + m[i], bn + n[i])) k = i;
      const u64 some = __ballot(k >= 0);
      const int at = some ? __ffsll((long long)some) - 1 : 63;
      u64 pm = bm, pn = bn;
#pragma unroll
      for (int i = 1; i < 4; ++i)
        if (k == i) pm = bm + m[i - 1], pn = bn + n[i - 1];
      *bin = __shfl(lane * 4 + (k < 0 ? 3 : k), at);
      *before_m = __shfl(pm, at);
      *before_n = __shfl(pn, at);
    };
    FilterInfo f;
    u64 nb = 0, unused_m, unused_n;
    f.mass = all;
    f.kbin = FL_BINS;
    f.m_before_k = all;
    if (a.top_k) first([&](u64, u64 c) { return c >= (u64)a.top_k; }, &f.kbin, &f.m_before_k, &nb);
    f.n_before = (int)nb;
    f.plo = f.phi = FL_BINS;
    f.m_before_p = 0;
    if (a.top_p < 1.0) {
      u64 upto = all;                              // mass of the k ids at most: what kbin holds counted whole
      if (a.top_k) {
        u64 b0 = 0, b1 = 0;
        int bin = 0;
        first([&](u64, u64 c) { return c >= (u64)a.top_k; }, &bin, &b0, &b1);
        upto = b0 + mass[0][bin] + mass[1][bin];
      }
      const double lo = a.top_p * (double)f.m_before_k, hi = a.top_p * (double)upto;
      first([&](u64 s, u64) { return (double)s >= lo; }, &f.plo, &f.m_before_p, &unused_n);
      first([&](u64 s, u64) { return (double)s >= hi; }, &f.phi, &unused_m, &unused_n);
    }
    if (lane == 0) {
      info = f;
      if (chunk == 0) a.w.info[row] = f;
    }
  }
  __syncthreads();
  const int kbin = info.kbin, plo = info.plo, phi = info.phi, sure_below = plo < kbin ? plo : kbin;
  u64 sum = 0;
  unsigned mine = 0;
#pragma unroll
  for (int j = 0; j < FL_QUADS; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double d = distance(top.v, x[j][i], a.mult);
      const int b = bin_of(d);
      if (b < sure_below) {
        const double w = weight(d);
        if (w >= a.min_p) sum += units(w);
      }
      if (id_of(chunk, j, i) < a.V && (b == kbin || (b >= plo && b <= phi))) mine |= 1u << (j * 4 + i);
    }
  sum = block_sum_u(sum, sh);
  u64 n;
  u64 at = block_scan_u(__popc(mine), sh, &n);
  if (threadIdx.x == 0) {
    a.w.sure[(size_t)row * a.C + chunk] = sum;
    base = n ? atomicAdd(&a.w.listed[row], (unsigned)n) : 0;
  }
  __syncthreads();
  at += base;
#pragma unroll
  for (int j = 0; j < FL_QUADS; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (mine >> (j * 4 + i) & 1) {
        if (at < FL_LIST) a.w.list[(size_t)row * FL_LIST + at] = order_of(x[j][i], id_of(chunk, j, i));
        ++at;
      }
}

// The candidates of a row, from the list or, where it did not hold them, from the row itself.
struct Candidates {
  const FilterArgs& a;
  const FilterInfo& f;
  const u64* list;
  const float* row;
  int n;
  bool whole;
  float top;
  template <typename F>
  __device__ __forceinline__ void each(F&& use) const {        // use(order, class, distance)
    for (int i = threadIdx.x; i < n; i += FL_THREADS) {
      const u64 o = whole ? order_of(row[i], i) : list[i];
      const double d = distance(top, whole ? row[i] : logit_of(o), a.mult);
      const int b = bin_of(d);
      if (!whole || b == f.kbin || (b >= f.plo && b <= f.phi)) use(o, b, d);
    }
  }
};

// The candidate at which the running sum, in order, of amount(order, class, distance) first reaches `target` (`base` before
// the first); the last one that has any, should none.  Digits of 8 bits, from the highest down.
template <typename A, typename T>
__device__ u64 select(const Candidates& c, A amount, u64 base, T target, u64* hist, u64* sh) {
  u64 prefix = 0;
  for (int shift = 56; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += FL_THREADS) hist[i] = 0;
    __syncthreads();
    c.each([&](u64 o, int b, double d) {
      if (shift == 56 || (o ^ prefix) >> (shift + 8) == 0) {
        const u64 v = amount(o, b, d);
        if (v) atomicAdd((u64*)&hist[o >> shift & 255], v);
      }
    });
    __syncthreads();
    if (threadIdx.x < 64) {
      const int lane = threadIdx.x;
      u64 h[4], s = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s += hist[lane * 4 + i];
        h[i] = s;
      }
      const u64 before = base + wave_scan_u(s) - s;
      int k = -1, last = -1;
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        if (h[i] != (i ? h[i - 1] : 0) && last < 0) last = i;
        if (h[i] != (i ? h[i - 1] : 0) && target(before + h[i])) k = i;
      }
      const u64 some = __ballot(k >= 0), any = __ballot(last >= 0);
      const int at = some ? __ffsll((long long)some) - 1 : any ? 63 - __clzll((long long)any) : 0;
      const int pick = some ? k : last < 0 ? 0 : last;
      u64 pm = before;
#pragma unroll
      for (int i = 1; i < 4; ++i)
        if (pick == i) pm = before + h[i - 1];
      if (lane == at) {
        sh[0] = (u64)(lane * 4 + pick);
        sh[1] = pm;
      }
    }
    __syncthreads();
    prefix |= sh[0] << shift;
    base = sh[1];
    __syncthreads();
  }
  return prefix;
}

__global__ __launch_bounds__(FL_THREADS) void filter_resolve_kernel(FilterArgs a, int classes) {
  __shared__ u64 list[FL_LIST], hist[256], sh[FL_WAVES], chunk_mass[FL_CHUNKS_MAX];
  __shared__ FilterInfo f;
  __shared__ int place;
  const int row = blockIdx.x;
  const RowTop top = row_top(a, row);
  if (a.greedy || top.none) {
    if (threadIdx.x == 0) {
      FilterEnd e;
      e.tok = a.greedy ? top.id : -1;
      e.bad = a.greedy ? 0 : 1;
      e.last = 0;
      e.total = 0;
      a.w.end[row] = e;
      if (a.tok) a.tok[row] = e.tok;
    }
    return;
  }
  u64 last = ~0ull;
  for (int c = threadIdx.x; c < a.C; c += FL_THREADS) chunk_mass[c] = a.w.sure[(size_t)row * a.C + c];
  if (classes) {
    if (threadIdx.x == 0) f = a.w.info[row];
    const unsigned n = a.w.listed[row];
    const bool whole = n > FL_LIST;
    if (!whole)
      for (unsigned i = threadIdx.x; i < n; i += FL_THREADS) list[i] = a.w.list[(size_t)row * FL_LIST + i];
    __syncthreads();
    const Candidates c = {a, f, list, a.logits + (size_t)row * a.ld, whole ? a.V : (int)n, whole, top.v};
    u64 mass_k = f.mass;
    if (a.top_k) {
      const u64 rank = (u64)a.top_k - f.n_before;
      last = select(c, [&](u64, int b, double) { return (u64)(b == f.kbin); }, 0, [&](u64 s) { return s >= rank; }, hist, sh);
      u64 m = 0;
      c.each([&](u64 o, int b, double d) {
        if (b == f.kbin && o <= last) m += units(weight(d));
      });
      mass_k = f.m_before_k + block_sum_u(m, sh);
    }
    if (a.top_p < 1.0) {
      const double goal = a.top_p * (double)mass_k;
      const u64 upto = last;
      last = select(c, [&](u64 o, int b, double d) { return b >= f.plo && b <= f.phi && o <= upto ? units(weight(d)) : 0ull; },
                    f.m_before_p, [&](u64 s) { return (double)s >= goal; }, hist, sh);
    }
    c.each([&](u64 o, int, double d) {
      if (o <= last) {
        const double w = weight(d);
        if (w >= a.min_p) atomicAdd(&chunk_mass[(unsigned)o / FL_CHUNK], units(w));
      }
    });
  }
  __syncthreads();
  // the chunk that the draw falls into
  u64 m = 0, total;
  static_assert(FL_CHUNKS_MAX <= FL_THREADS, "a thread per chunk");
  if (threadIdx.x < a.C) m = chunk_mass[threadIdx.x];
  u64 before = block_scan_u(m, sh, &total);
  if (threadIdx.x == 0) {
    FilterEnd e;
    e.last = last;
    e.total = total;
    e.bad = 0;
    e.tok = 0;
    a.w.end[row] = e;
  }
  if (!a.tok) return;
  double u = (double)a.u[row];
  if (!(u > 0.0)) u = 0.0;
  u64 goal = (u64)(u * (double)total);
  if (goal >= total) goal = total - 1;
  if (before <= goal && goal < before + m) place = threadIdx.x;
  __syncthreads();
  const int chunk = place;
  if (threadIdx.x == chunk) sh[0] = goal - before;          // (after the last read of sh in block_scan_u: a barrier lies between)
  __syncthreads();
  goal = sh[0];
  float x[FL_QUADS][4];
  load_chunk(a, row, chunk, x);
  u64 start = 0;
#pragma unroll
  for (int j = 0; j < FL_QUADS; ++j) {
    u64 v[4], s = 0, all;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double w = weight(distance(top.v, x[j][i], a.mult));
      v[i] = order_of(x[j][i], id_of(chunk, j, i)) <= last && w >= a.min_p ? units(w) : 0;
      s += v[i];
    }
    u64 at = start + block_scan_u(s, sh, &all);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (at <= goal && goal < at + v[i]) a.tok[row] = id_of(chunk, j, i);
      at += v[i];
    }
    start += all;
  }
}

__global__ __launch_bounds__(FL_THREADS) void filter_write_kernel(FilterArgs a) {
  const int chunk = blockIdx.x, row = blockIdx.y;
  float x[FL_QUADS][4];
  load_chunk(a, row, chunk, x);
  const FilterEnd e = a.w.end[row];
  const RowTop top = row_top(a, row);
  const double inv = 1.0 / ((double)e.total / FL_ONE);
#pragma unroll
  for (int j = 0; j < FL_QUADS; ++j) {
    float q[4], m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int id = id_of(chunk, j, i);
      if (a.greedy) {
        q[i] = id == e.tok ? 1.0f : 0.0f;
        m[i] = id == e.tok ? x[j][i] : -INFINITY;
      } else if (e.bad) {
        q[i] = m[i] = __builtin_nanf("");
      } else {
        q[i] = 0.0f;
        m[i] = -INFINITY;
        if (order_of(x[j][i], id) <= e.last) {
          const double w = weight(distance(top.v, x[j][i], a.mult));
          if (w >= a.min_p) {
            q[i] = (float)(w * inv);
            m[i] = x[j][i];
          }
        }
      }
    }
    const int id = id_of(chunk, j, 0);
    const size_t at = (size_t)row * a.V + id;
    if (id + 4 <= a.V) {
      if (a.q) *reinterpret_cast<f32x4u*>(a.q + at) = f32x4u{q[0], q[1], q[2], q[3]};
      if (a.masked) *reinterpret_cast<f32x4u*>(a.masked + at) = f32x4u{m[0], m[1], m[2], m[3]};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (id + i < a.V) {
          if (a.q) a.q[at + i] = q[i];
          if (a.masked) a.masked[at + i] = m[i];
        }
    }
  }
}

// ---- the call -------------------------------------------------------------------------------------------------------
static size_t filter_layout(int rows, int V, char* base, FilterWork* w) {
  const size_t C = (V + FL_CHUNK - 1) / FL_CHUNK, n = rows;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = base + at;
    at += (bytes + 15) & ~(size_t)15;
    return p;
  };
  w->mass = (u64*)take(n * C * FL_BINS * 8);
  w->list = (u64*)take(n * FL_LIST * 8);
  w->count = (unsigned*)take(n * C * FL_BINS * 4);
  w->sure = (u64*)take(n * C * 8);
  w->top = (FilterTop*)take(n * C * sizeof(FilterTop));
  w->info = (FilterInfo*)take(n * sizeof(FilterInfo));
  w->end = (FilterEnd*)take(n * sizeof(FilterEnd));
  w->listed = (unsigned*)take(n * 4);
  return at;
}
size_t filter_work_bytes(int rows, int V) {
  FilterWork w;
  return filter_layout(rows, V, nullptr, &w);
}
hipError_t launch_sample_rows(const float* logits, size_t ld, int rows, int V, const spec_sampling& s, const float* u, float* q,
                              float* masked, int* tok, void* work, hipStream_t st) {
  FilterArgs a;
  a.logits = logits;
  a.ld = ld;
  a.V = V;
  a.C = (V + FL_CHUNK - 1) / FL_CHUNK;
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
  const int classes = a.top_k || a.top_p < 1.0;
  const dim3 grid(a.C, rows);
  filter_top_kernel<<<grid, FL_THREADS, 0, st>>>(a);
  if (!a.greedy) filter_bins_kernel<<<grid, FL_THREADS, 0, st>>>(a, classes);
  if (!a.greedy && classes) filter_collect_kernel<<<grid, FL_THREADS, 0, st>>>(a);
  filter_resolve_kernel<<<rows, FL_THREADS, 0, st>>>(a, classes);
  if (q || masked) filter_write_kernel<<<grid, FL_THREADS, 0, st>>>(a);
  return hipGetLastError();
}
