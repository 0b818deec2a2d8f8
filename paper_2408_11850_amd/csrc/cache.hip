// Attention over a paged cache of keys and values in e4m3, for gfx950: the append that fills it, attention of the last rows of
// every sequence (whole or with a sliding window and first entries that stay visible), the attention weight of its entries, and
// eviction by that weight.
//
// A page holds 64 entries: keys [64][d] and values [d][64] of each KV head, so that 16 bytes of either are what a lane of an MFMA
// operand wants: keys are contracted over d, values over entries.  One scale for the keys and one for the values of a page and
// head, powers of two: a code times a scale is a multiplication that rounds nothing, and a code moves to another scale exactly
// unless it becomes denormal.
//
// Entries are held in the order of their sequence; the rows of a call are its last ones.  Row j of M sees the entries up to its
// own, len - M + j, and of those, with a window, the last `window` and the first `sinks`.
#include <float.h>
#include <limits.h>

#include <type_traits>

#include "spec_internal.h"

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4a;
typedef __attribute__((ext_vector_type(8), aligned(2))) unsigned short bf16x8a;

#define PAGE SPEC_PAGE_TOKENS
#define LEAST_EXP (-100)            // scales are 2^e, e >= this
#define FINITE_MAX 0x1p120f         // keys and values from here on count as infinite: their scales would leave fp32's range
#define NONE (-3.0e38f)             // running maximum of a row that has seen nothing; scores below it cannot be told from it
// A row's reference stays until a score is so far above it (to the base 2): weights reach 2^8.  Their rounding to bf16 is as large relative to
// them as ever, but the largest is no longer 1 and free of it.  Distance from 64 bits in the 2-norm for normal q and codes, of which the
// result's own rounding is 0.0017: 0.0021 to 0.0024, with the exact maximum 0.0020 to 0.0023, with weights in two bf16 parts that rounding alone.
// us (this | exact maximum | two parts): a 4095-token prompt 283 | 299 | 395, 8 rows behind 131072 73 | 75 | 88, one token 9.6 | 9.5 | 10.1.
#define LAG 8.f
#define FAR 0x1p20f                 // references from here on: see where it is used
#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f

// Eight codes times a power of two, exactly.  Keys take their page's scale here, not in the factor of their scores: 2^-100 or 2^112 times a
// softmax's scale may be 0 or infinite, and that times a hidden score, or a zero, NaN.
__device__ __forceinline__ bf16x8 to_bf16x8(unsigned lo, unsigned hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// 2^e for -126 <= e <= 127
__device__ __forceinline__ float power(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__float_as_uint(scale) >> 23 & 255u) - 127; }
// the least e >= LEAST_EXP with top <= 448 * 2^e: 448 = 1.75 * 2^8
__device__ __forceinline__ int page_exponent(float top) {
  return max((int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 127 - 8, LEAST_EXP);
}
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// four codes times a power of two, rounded again
__device__ __forceinline__ unsigned moved4(unsigned w, float by) {
  return codes4(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * by, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * by,
                __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * by, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * by);
}
__device__ __forceinline__ float move_by(int from, int to) { return power(max(from - to, -126)); }

// a * b - c with both roundings
__device__ __forceinline__ float difference(float a, float b, float c) {
#pragma clang fp contract(off)
  const float p = a * b;
  return p - c;
}

// over a wave, the same bits in every lane
template <int CTRL>
__device__ __forceinline__ float rotated(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, rotated<0x128>(v));
  v = fmaxf(v, rotated<0x124>(v));
  v = fmaxf(v, rotated<0x122>(v));
  return fmaxf(v, rotated<0x121>(v));
}
__device__ __forceinline__ float row_sum(float v) {
  v += rotated<0x128>(v);
  v += rotated<0x124>(v);
  v += rotated<0x122>(v);
  return v + rotated<0x121>(v);
}
__device__ __forceinline__ float wave_max(float v) { return groups_max(row_max(v)); }
__device__ __forceinline__ float wave_sum(float v) { return groups_sum(row_sum(v)); }

// ---- which rows a workgroup works on --------------------------------------------------------------------------------------
struct Span {
  int s;          // sequence, or -1: none
  int t;          // which of its tiles
  int row, M;     // its first row and their number
  int len;        // what the cache says of its length
};
// sums of a value over the lanes up to one's own
__device__ __forceinline__ int lanes_upto(int v) {
  const int lane = threadIdx.x & 63;
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);            // one, two, four and eight lanes down in a row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  const int a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31), c = __builtin_amdgcn_readlane(v, 47);
  return v + (lane >= 16 ? a : 0) + (lane >= 32 ? b : 0) + (lane >= 48 ? c : 0);
}
// Tile `id` of all sequences' tiles one behind the other; tiles(M) of a sequence with M rows.  Called by whole waves, the same in all lanes.
template <class Tiles>
__device__ __forceinline__ Span find_span(const QuantCache& c, const int* rows, int n_rows, int id, Tiles tiles) {
  if (!rows) {
    const int M = n_rows / c.n_seqs, per = tiles(M), s = id / per;
    return s < c.n_seqs ? Span{s, id - s * per, s * M, M, c.len[s]} : Span{-1, 0, 0, 0, 0};
  }
  int before = 0;
  for (int base = 0; base < c.n_seqs; base += 64) {
    const int s = base + (int)(threadIdx.x & 63);
    int first = 0, M = 0, len = 0;
    if (s < c.n_seqs) {                       // whatever the numbers are, the rows are rows of the call
      first = min(max(rows[s], 0), n_rows);
      M = min(max(rows[s + 1], first), n_rows) - first;
      len = c.len[s];
    }
    const int mine = M > 0 ? tiles(M) : 0, upto = lanes_upto(mine), all = __builtin_amdgcn_readlane(upto, 63);
    if (id - before < all) {
      const int at = __ffsll((long long)__ballot(upto > id - before)) - 1;
      return Span{base + at, id - before - __builtin_amdgcn_readlane(upto - mine, at), __builtin_amdgcn_readlane(first, at),
                  __builtin_amdgcn_readlane(M, at), __builtin_amdgcn_readlane(len, at)};
    }
    before += all;
  }
  return Span{-1, 0, 0, 0, 0};
}

// Pages that rows at the entries lo .. hi see: the first `a` (with a window: those of the sinks), then from `b` on.
struct Seen {
  int a, b, n;
  __device__ __forceinline__ int page(int i) const { return i < a ? i : b + i - a; }
};
__device__ __forceinline__ Seen seen_pages(int lo, int hi, int window, int sinks) {
  if (hi < 0) return Seen{0, 0, 0};
  int a = 0, b = 0;
  if (window > 0) {
    b = max(0, lo - window + 1) / PAGE;
    a = min(b, sinks / PAGE + (sinks % PAGE != 0));
  }
  return Seen{a, b, a + hi / PAGE - b + 1};
}

// Ids and scales of the pages that a wave goes over, 64 at a time: a lane holds those of a page, so that none of them is waited for
// on the way to a page's codes.
struct PageList {
  const QuantCache& c;
  const int* table;
  Seen seen;
  int h, step, first;     // the wave's pages are first, first + step, ... of `seen`
  int base, id;
  float ks, vs;
  __device__ __forceinline__ PageList(const QuantCache& c, int s, const Seen& seen, int h, int first, int step)
      : c(c), table(c.table + (size_t)s * c.table_ld), seen(seen), h(h), step(step), first(first), base(-64), id(0), ks(0.f), vs(0.f) {}
  __device__ __forceinline__ void fetch(int from) {
    base = from;
    const int i = first + (from + (int)(threadIdx.x & 63)) * step;
    id = i < seen.n ? table[seen.page(i)] : -1;
    const bool there = (unsigned)id < (unsigned)c.n_pages;
    const float2 x = *reinterpret_cast<const float2*>(c.scale + ((size_t)(there ? id : 0) * c.n_kv_heads + h) * 2);
    id = there ? id : -1;
    ks = x.x, vs = x.y;
  }
  // waits for what was fetched: no wait in the loop around, where codes are on their way
  __device__ __forceinline__ void settle() { asm volatile("" : "+v"(id), "+v"(ks), "+v"(vs)); }
  __device__ __forceinline__ int first_id(int i = 0) const { return __builtin_amdgcn_readlane(id, i); }
  // page i of the wave: its id, -1 if it is none of the cache, and its scales
  __device__ __forceinline__ int get(int i, float* k, float* v) {
    if (i >= base + 64) fetch(i), settle();
    *k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), i - base));
    *v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), i - base));
    return __builtin_amdgcn_readlane(id, i - base);
  }
};

// ---- append ---------------------------------------------------------------------------------------------------------------
// A workgroup takes the entries of a call that fall into one page: keys and values of a KV head, or eight query heads.  The
// angles' cosines and sines are made once per workgroup, in revolutions in 64 bits up to the reduction.
// Bound by memory for many rows: 4095 tokens of 8 heads with 64 query heads (159 MB read and written) 32.8 us, 4.8 TB/s; rows in fp32 (243 MB)
// 41.6 us, 5.8 TB/s.  One token: 5.1 us, the trips to its length, its page's id, the scale, and the codes that move if it grows.
template <int T>
__device__ __forceinline__ void load8(const void* p, size_t at, float (&v)[8]) {
  if (T == SPEC_F32) {
    const f32x4a* s = reinterpret_cast<const f32x4a*>(reinterpret_cast<const float*>(p) + at);
    const f32x4a a = s[0], b = s[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
    const bf16x8a a = *reinterpret_cast<const bf16x8a*>(reinterpret_cast<const unsigned short*>(p) + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float((unsigned)a[i] << 16);
  }
}

#define APPEND_THREADS 256
#define APPEND_HEADS 8             // query heads of a workgroup

template <int DH, int T>
__global__ __launch_bounds__(APPEND_THREADS) void append_kernel(QuantCache c, AppendArgs a) {
  constexpr int SUB = DH / 16;                   // lanes of a token: each 8 elements of the first half and their partners
  constexpr int PER = APPEND_THREADS / SUB;      // tokens at a time
  constexpr int STEPS = PAGE / PER;
  __shared__ float2 turn[PAGE][DH / 2];
  __shared__ __align__(16) unsigned char vt[DH][PAGE + 4];
  __shared__ int odd[PAGE];                      // entries with a key or value that is not finite
  __shared__ float tops[APPEND_THREADS / 64][2];
  const Span sp = find_span(c, a.rows, a.n_rows, blockIdx.x, [](int M) { return (M + 2 * PAGE - 2) / PAGE; });
  if (sp.s < 0) return;
  const int len = min(max(sp.len, 0), INT_MAX / 2), first = len - sp.M, capacity = c.max_pages * PAGE;
  const int page0 = ((first >> 6) + sp.t) * PAGE;                    // first may be negative
  const int lo = max(first, page0), hi = min(len, page0 + PAGE);     // the entries of this page
  if (lo >= hi) return;
  const int row0 = sp.row + lo - first, n = hi - lo;
  const int tid = threadIdx.x, sub = tid % SUB;
  if (a.theta > 0.f) {
    const int pos0 = a.position ? a.position[sp.s] + (lo - first) : lo;
    for (int i = tid; i < n * (DH / 2); i += APPEND_THREADS) {
      const int t = i / (DH / 2), p = i % (DH / 2);
      const double rev = (double)(pos0 + t) * exp2(-(double)p * a.log2_theta / (DH / 2)) * 0.15915494309189535;
      const double left = rev - rint(rev);
      const float near = (float)left, rest = 6.2831855f * (float)(left - (double)near);
      float sn, cs;
      sincospif(2.f * near, &sn, &cs);
      // what fp32 leaves of the angle, up to 2^-26 of a turn, to first order: beside a quarter turn it is 80 roundings of a cosine of 0.02
      turn[t][p] = make_float2(fmaf(-sn, rest, cs), fmaf(cs, rest, sn));
    }
  }
  const int y = blockIdx.y;
  if (y >= c.n_kv_heads) {                                           // query heads
    if (a.theta > 0.f) __syncthreads();
    const int h0 = (y - c.n_kv_heads) * APPEND_HEADS, nh = min(APPEND_HEADS, a.n_heads - h0);
    for (int i = tid; i < n * nh * SUB; i += APPEND_THREADS) {
      const int h = h0 + i / SUB % nh, t = i / (SUB * nh);
      float x0[8], x1[8];
      const size_t at = (size_t)(row0 + t) * a.ldq + (size_t)h * DH + sub * 8;
      load8<T>(a.q, at, x0);
      load8<T>(a.q, at + DH / 2, x1);
      bf16x8 o0, o1;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float r0 = x0[j], r1 = x1[j];
        if (a.theta > 0.f) {
          const float2 w = turn[t][sub * 8 + j];
          r0 = x0[j] * w.x - x1[j] * w.y;
          r1 = x1[j] * w.x + x0[j] * w.y;
        }
        o0[j] = (__bf16)r0;
        o1[j] = (__bf16)r1;
      }
      bf16* out = a.q_out + ((size_t)(row0 + t) * a.n_heads + h) * DH + sub * 8;
      *reinterpret_cast<bf16x8*>(out) = o0;
      *reinterpret_cast<bf16x8*>(out + DH / 2) = o1;
    }
    return;
  }
  const int page = page0 >= 0 && hi <= capacity && len <= capacity ? c.table[(size_t)sp.s * c.table_ld + page0 / PAGE] : -1;
  if ((unsigned)page >= (unsigned)c.n_pages) return;                 // no page of this cache: nothing is stored
  const size_t block = ((size_t)page * c.n_kv_heads + y) * PAGE * DH;
  float* scale = c.scale + ((size_t)page * c.n_kv_heads + y) * 2;
  if (tid < PAGE) odd[tid] = 0;
  float k0[STEPS][8], k1[STEPS][8], v0[STEPS][8], v1[STEPS][8];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int t = s * PER + tid / SUB;
    if (t < n) {
      const size_t ak = (size_t)(row0 + t) * a.ldk + (size_t)y * DH + sub * 8, av = (size_t)(row0 + t) * a.ldv + (size_t)y * DH + sub * 8;
      load8<T>(a.k, ak, k0[s]);
      load8<T>(a.k, ak + DH / 2, k1[s]);
      load8<T>(a.v, av, v0[s]);
      load8<T>(a.v, av + DH / 2, v1[s]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) k0[s][j] = k1[s][j] = v0[s][j] = v1[s][j] = 0.f;
    }
  }
  const int slot = lo - page0;
  const int e_old[2] = {slot ? exponent_of(scale[0]) : LEAST_EXP, slot ? exponent_of(scale[1]) : LEAST_EXP};
  __syncthreads();
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int t = s * PER + tid / SUB;
    if (t >= n) continue;
    bool fine = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (a.theta > 0.f) {
        const float2 w = turn[t][sub * 8 + j];
        const float x0 = k0[s][j], x1 = k1[s][j];
        k0[s][j] = x0 * w.x - x1 * w.y;
        k1[s][j] = x1 * w.x + x0 * w.y;
      }
      fine = fine && fabsf(k0[s][j]) < FINITE_MAX && fabsf(k1[s][j]) < FINITE_MAX && fabsf(v0[s][j]) < FINITE_MAX && fabsf(v1[s][j]) < FINITE_MAX;
    }
    if (!fine) odd[t] = 1;
  }
  __syncthreads();
  float top[2] = {0.f, 0.f};
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int t = s * PER + tid / SUB;
    if (t >= n) continue;
    if (odd[t]) {                                // its key becomes NaN, its value 0: whoever sees it becomes NaN, nobody else
#pragma unroll
      for (int j = 0; j < 8; ++j) k0[s][j] = k1[s][j] = __uint_as_float(0x7fc00000u), v0[s][j] = v1[s][j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      top[0] = fmaxf(top[0], fmaxf(fabsf(k0[s][j]), fabsf(k1[s][j])));          // without the NaN
      top[1] = fmaxf(top[1], fmaxf(fabsf(v0[s][j]), fabsf(v1[s][j])));
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    top[i] = wave_max(top[i]);
    if ((tid & 63) == 0) tops[tid >> 6][i] = top[i];
  }
  __syncthreads();
  int e[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float m = 0.f;
#pragma unroll
    for (int w = 0; w < APPEND_THREADS / 64; ++w) m = fmaxf(m, tops[w][i]);
    e[i] = max(page_exponent(m), e_old[i]);
  }
  uint8_t* kp = c.k + block;
  uint8_t* vp = c.v + block;
  // codes of earlier entries move to a larger scale
  if (slot && e[0] != e_old[0]) {
    const float by = move_by(e_old[0], e[0]);
    unsigned* p = reinterpret_cast<unsigned*>(kp);
    for (int i = tid; i < slot * DH / 4; i += APPEND_THREADS) p[i] = moved4(p[i], by);
  }
  if (slot && e[1] != e_old[1]) {
    const float by = move_by(e_old[1], e[1]);
    const int words = (slot + 3) / 4;
    for (int i = tid; i < DH * words; i += APPEND_THREADS) {
      const int at = i % words;
      unsigned* p = reinterpret_cast<unsigned*>(vp + (i / words) * PAGE) + at;
      const unsigned was = *p, keep = slot - at * 4 >= 4 ? 0xffffffffu : (1u << (slot - at * 4) * 8) - 1;
      *p = (moved4(was, by) & keep) | (was & ~keep);
    }
  }
  const float ik = power(-e[0]), iv = power(-e[1]);
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int t = s * PER + tid / SUB;
    if (t >= n) continue;
    uint8_t* kr = kp + (slot + t) * DH + sub * 8;
    *reinterpret_cast<uint2*>(kr) = make_uint2(codes4(k0[s][0] * ik, k0[s][1] * ik, k0[s][2] * ik, k0[s][3] * ik),
                                               codes4(k0[s][4] * ik, k0[s][5] * ik, k0[s][6] * ik, k0[s][7] * ik));
    *reinterpret_cast<uint2*>(kr + DH / 2) = make_uint2(codes4(k1[s][0] * ik, k1[s][1] * ik, k1[s][2] * ik, k1[s][3] * ik),
                                                        codes4(k1[s][4] * ik, k1[s][5] * ik, k1[s][6] * ik, k1[s][7] * ik));
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      const unsigned x0 = codes4(v0[s][j] * iv, v0[s][j + 1] * iv, v0[s][j + 2] * iv, v0[s][j + 3] * iv);
      const unsigned x1 = codes4(v1[s][j] * iv, v1[s][j + 1] * iv, v1[s][j + 2] * iv, v1[s][j + 3] * iv);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        vt[sub * 8 + j + b][slot + t] = (unsigned char)(x0 >> b * 8);
        vt[DH / 2 + sub * 8 + j + b][slot + t] = (unsigned char)(x1 >> b * 8);
      }
    }
  }
  __syncthreads();
  // values: whole words of new entries, bytes at the ends
  const int w0 = slot / 4, words = (slot + n + 3) / 4 - w0;
  for (int i = tid; i < DH * words; i += APPEND_THREADS) {
    const int d = i / words, w = w0 + i % words;
    uint8_t* p = vp + d * PAGE + w * 4;
    if (w * 4 >= slot && w * 4 + 4 <= slot + n) *reinterpret_cast<unsigned*>(p) = *reinterpret_cast<const unsigned*>(&vt[d][w * 4]);
    else
      for (int b = max(slot - w * 4, 0); b < min(slot + n - w * 4, 4); ++b) p[b] = vt[d][w * 4 + b];
  }
  if (tid < 2) scale[tid] = power(tid ? e[1] : e[0]);
}

hipError_t launch_append_quant(const QuantCache& c, const AppendArgs& a, int type, hipStream_t st) {
  const int per = a.rows ? 0 : a.n_rows / c.n_seqs;
  const long long tiles = a.rows ? a.n_rows / PAGE + 2ll * c.n_seqs : (long long)c.n_seqs * ((per + 2 * PAGE - 2) / PAGE);
  const dim3 grid((unsigned)tiles, c.n_kv_heads + (a.q ? (a.n_heads + APPEND_HEADS - 1) / APPEND_HEADS : 0));
  if (c.head_dim == 128) {
    if (type == SPEC_F32) append_kernel<128, SPEC_F32><<<grid, APPEND_THREADS, 0, st>>>(c, a);
    else append_kernel<128, SPEC_BF16><<<grid, APPEND_THREADS, 0, st>>>(c, a);
  } else {
    if (type == SPEC_F32) append_kernel<64, SPEC_F32><<<grid, APPEND_THREADS, 0, st>>>(c, a);
    else append_kernel<64, SPEC_BF16><<<grid, APPEND_THREADS, 0, st>>>(c, a);
  }
  return hipGetLastError();
}

// ---- attention ------------------------------------------------------------------------------------------------------------
// Rows are the M * G pairs (row, head of the group) of a KV head.  S^T = K Q^T and O^T += V^T P^T, both 16 x 16 x 32: row r of
// key tile t is entry 16 (r / 4) + 4 t + r % 4 of the page, so that the scores that a lane gets are the P operand it has to give,
// and 16 neighbouring bytes of a value's row its partner.  16 neighbouring bytes of a key likewise: the contraction over d takes
// them in that order on both sides.
template <int DH>
__device__ __forceinline__ void load_keys(const QuantCache& c, u32x4 (&k)[4][DH / 64], int page, int h, int lane) {
  const int r = lane & 15, g = lane >> 4;
  const uint8_t* p = c.k + ((size_t)max(page, 0) * c.n_kv_heads + h) * PAGE * DH + (16 * (r >> 2) + (r & 3)) * DH + g * 16;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int f = 0; f < DH / 64; ++f) k[t][f] = *reinterpret_cast<const u32x4*>(p + 4 * t * DH + f * 64);
}
template <int DH>
__device__ __forceinline__ void load_values(const QuantCache& c, u32x4 (&v)[DH / 16], int page, int h, int lane) {
  const uint8_t* p = c.v + ((size_t)max(page, 0) * c.n_kv_heads + h) * PAGE * DH + (lane & 15) * PAGE + (lane >> 4) * 16;
#pragma unroll
  for (int d = 0; d < DH / 16; ++d) v[d] = *reinterpret_cast<const u32x4*>(p + d * 16 * PAGE);
}
#define NAN32 __uint_as_float(0x7fc00000u)

// the first n of 16 bytes, 0 behind them
__device__ __forceinline__ u32x4 first_bytes(u32x4 v, int n) {
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int k = n - 4 * x;
    v[x] &= k >= 4 ? 0xffffffffu : k <= 0 ? 0u : (1u << k * 8) - 1;
  }
  return v;
}
// A page's scores s (times `by`, the call's scale, to the base 2; of the entries from `from` on) into weights pf, their sum l and reference m; o follows m.
// all: every row sees the whole page, else up to pos, above low or below sinks.
template <int DH>
__device__ __forceinline__ void softmax_step(f32x4 (&s)[4], f32x4 (&o)[DH / 16], float& m, float& l, bf16x8 (&pf)[2], float by, bool all,
                                             int from, int pos, int low, int sinks) {
  if (!all) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int e = from + 4 * t + x;
        s[t][x] = (e <= pos) & ((e > low) | (e < sinks)) ? s[t][x] : -INFINITY;
      }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int x = 0; x < 4; ++x) mx = fmaxf(mx, s[t][x]);
  mx = groups_max(mx) * by;
  if (__any(mx > m + LAG)) {                       // maxima settle after a few pages
    asm volatile("" ::: "memory");                 // and what is to do then stays here
    const float m_new = mx > m + LAG ? mx : m, corr = __builtin_amdgcn_exp2f(m - m_new);      // of the rows that need it: no row's bits
    m = m_new;                                                                               // depend on its neighbours
    l *= corr;
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) o[d] *= corr;
  }
  // the product with the scale in one rounding with the difference, unless its own rounding, left in the largest score, would count
  const bool far = fabsf(m) > FAR;
  float mul = by, less = m;
  if (__any(far)) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int x = 0; x < 4; ++x) s[t][x] = far ? difference(s[t][x], by, m) : s[t][x];
    mul = far ? 1.f : by, less = far ? 0.f : m;
  }
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float v = __builtin_amdgcn_exp2f(fmaf(s[t][x], mul, -less));
      sum += v;
      pf[t >> 1][(t & 1) * 4 + x] = (__bf16)v;
    }
  l += sum;
}
// a row's result, or its part: 4 elements of every 16 in this lane
template <int DH>
__device__ __forceinline__ void store_rows(const AttendArgs& a, const f32x4 (&o)[DH / 16], float m, float l, int pos, int split, size_t row_at, size_t part_at, int g) {
  if (a.splits == 1) {
    const bool empty = pos < 0;
    const float inv = empty ? 0.f : 1.f / l;
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) {
      bf16 b[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) b[x] = __float2bfloat16(o[d][x] * inv);
      *reinterpret_cast<uint2*>(a.out + row_at * DH + d * 16 + g * 4) = *reinterpret_cast<const uint2*>(b);
    }
    if (a.lse && g == 0) a.lse[row_at] = empty ? -INFINITY : (m + __log2f(l)) * LN2;
  } else {
    const size_t at = split * a.part_rows + part_at;
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) *reinterpret_cast<f32x4*>(a.part + at * DH + d * 16 + g * 4) = o[d];
    if (g == 0) a.part_ml[at] = make_float2(pos < 0 ? -INFINITY : m, l);       // -inf: the row sees nothing
  }
}

// Few rows of a KV head: the codes go to registers as operands, RT tiles of 16 rows share them in a wave.  The waves of a workgroup have
// row_waves sets of rows and take pages in turn.  No LDS on the way, as no other wave wants these codes: pages that four waves share
// through LDS, a tile of rows each, were slower (81 us against 69 for 64 rows of heads behind 131072), since every wave converts them.
// One row each of 16 sequences, 32 heads: 627 MB in 115 us, 5.4 TB/s.  64 rows of 8 heads behind 131072: 268 MB in 69 us, 3.9 TB/s, with one wave
// a SIMD, a page of it in flight, vector instructions in 40 % of the cycles and products in 23.  One token behind 4096: 6.9 us, four dependent
// trips to memory.
#define FEW_WAVES 4
template <int DH, int RT>
__global__ __launch_bounds__(FEW_WAVES * 64, RT == 1 ? 3 : 2) void attend_few_kernel(QuantCache c, AttendArgs a) {
  constexpr int KS = DH / 32, DT = DH / 16;
  __shared__ f32x4 osh[FEW_WAVES - 1][RT][DT][64];
  __shared__ float2 mlsh[FEW_WAVES][RT][16];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const unsigned parts = c.n_kv_heads * a.splits, part = blockIdx.x % parts;
  const int h = part % c.n_kv_heads, split = part / c.n_kv_heads, G = a.G;
  // sets of rows of a sequence with R: as the call says, or where its sequences differ as the sequence does
  auto row_waves = [&](int R) { return a.row_waves ? a.row_waves : R > 32 * RT ? 4 : R > 16 * RT ? 2 : 1; };
  Span sp = find_span(c, a.rows, a.n_rows, blockIdx.x / parts, [&](int M) {
    const int tile_rows = 16 * RT * row_waves(M * G);
    return M * G <= a.upto ? (M * G + tile_rows - 1) / tile_rows : 0;
  });
  sp.s = __builtin_amdgcn_readfirstlane(sp.s);
  if (sp.s < 0) return;
  sp.t = __builtin_amdgcn_readfirstlane(sp.t), sp.row = __builtin_amdgcn_readfirstlane(sp.row), sp.M = __builtin_amdgcn_readfirstlane(sp.M);
  const size_t part_from = a.per ? ((size_t)sp.s * a.per - sp.row) * a.n_heads : 0;       // of the parts, less that of the rows
  const int given = __builtin_amdgcn_readfirstlane(sp.len);
  const bool beyond = given > c.max_pages * PAGE;    // nothing is read; the rows become NaN
  const int len = max(given, 0), first = len - sp.M, R = sp.M * G;
  const int sets = row_waves(R), tile_rows = 16 * RT * sets, phases = FEW_WAVES / sets, rw = w % sets, phase = w / sets;
  const int wg0 = sp.t * tile_rows, wg_last = min(wg0 + tile_rows, R) - 1, r0 = wg0 + rw * 16 * RT, r_last = min(r0 + 16 * RT, R) - 1;
  const Seen seen = seen_pages(first + wg0 / G, beyond ? -1 : first + wg_last / G, a.window, a.sinks);
  const int per = (seen.n + a.splits - 1) / a.splits, i0 = split * per + phase;
  const int n = r0 < R ? max(0, (min(split * per + per, seen.n) - i0 + phases - 1) / phases) : 0;         // pages of this wave
  const int see_all = first + r0 / G, low_all = a.window ? first + max(r_last, 0) / G - a.window + 1 : 0;

  int pos[RT];
  size_t row_at[RT];                                 // (row, head), counted through
  bf16x8 qf[RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + rt * 16 + r16;
    const bool valid = r < R;
    const int tok = valid ? r / G : 0, hq = h * G + (valid ? r % G : 0);
    pos[rt] = valid ? first + tok : -1;
    row_at[rt] = (size_t)(sp.row + tok) * a.n_heads + hq;
#pragma unroll
    for (int j = 0; j < KS; ++j)
      qf[rt][j] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(a.q + (size_t)(sp.row + tok) * a.ldq + (size_t)hq * DH + g * 16 + (j >> 1) * 64 + (j & 1) * 8));
  }
  float m[RT], l[RT];
  f32x4 o[RT][DT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = pos[rt] < 0 ? 0.f : NONE, l[rt] = 0.f;       // a lane without a row is not FAR: its neighbours' scores are as in a full tile
#pragma unroll
    for (int d = 0; d < DT; ++d) o[rt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  PageList pages(c, sp.s, seen, h, i0, phases);
  u32x4 kd[4][DH / 64], vd[DT];
  float ks = 0.f, vs = 0.f;
  int id = -1;
  if (n > 0) {
    pages.fetch(0);                                  // the first codes are asked for behind the scales, and waited for with them
    load_keys<DH>(c, kd, pages.first_id(), h, lane);
    load_values<DH>(c, vd, pages.first_id(), h, lane);
    pages.settle();
    id = pages.get(0, &ks, &vs);
  }
  for (int i = 0; i < n; ++i) {
    const int e0 = seen.page(i0 + i * phases) * PAGE;
    const bool there = id >= 0, more = i + 1 < n;
    const float kscale = ks, vscale = there ? vs : 0.f;
    if (more) id = pages.get(i + 1, &ks, &vs);
    f32x4 s[RT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const bf16x8 kf = to_bf16x8(kd[t][j >> 1][(j & 1) * 2], kd[t][j >> 1][(j & 1) * 2 + 1], kscale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rt][j], s[rt][t], 0, 0, 0);
      }
    }
    if (more) load_keys<DH>(c, kd, id, h, lane);
    if (!there) {                                    // no such page: whoever sees it becomes NaN
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[rt][t] = f32x4{NAN32, NAN32, NAN32, NAN32};
    }
    const bool all = e0 + PAGE - 1 <= see_all && (!a.window || e0 >= low_all || e0 + PAGE <= a.sinks);
    bf16x8 pf[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
      softmax_step<DH>(s[rt], o[rt], m[rt], l[rt], pf[rt], a.scale_log2e, all, e0 + 16 * g, pos[rt], a.window ? pos[rt] - a.window : INT_MIN, a.sinks);
    // entries behind the last one, or of no page, may hold anything: 0 times a NaN would be one
    if (!there || e0 + PAGE > len) {
      const int live = there ? min(len - e0, PAGE) - 16 * g : 0;
#pragma unroll
      for (int d = 0; d < DT; ++d) vd[d] = first_bytes(vd[d], live);
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const bf16x8 vf = to_bf16x8(vd[d][x * 2], vd[d][x * 2 + 1], vscale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt][x], o[rt][d], 0, 0, 0);
      }
    if (more) load_values<DH>(c, vd, id, h, lane);
  }
  // the waves of a set of rows together
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] = groups_sum(l[rt]);
    if (g == 0) mlsh[w][rt][r16] = make_float2(m[rt], l[rt]);
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = NONE, sum = 0.f;
    for (int x = rw; x < FEW_WAVES; x += sets) top = fmaxf(top, mlsh[x][rt][r16].x);
    for (int x = rw; x < FEW_WAVES; x += sets) sum += mlsh[x][rt][r16].y * __builtin_amdgcn_exp2f(mlsh[x][rt][r16].x - top);
    const float f = __builtin_amdgcn_exp2f(m[rt] - top);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      o[rt][d] *= f;
      if (phase) osh[w - sets][rt][d][lane] = o[rt][d];
    }
    m[rt] = top, l[rt] = sum;
  }
  __syncthreads();
  if (phase) return;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    for (int x = rw; x < FEW_WAVES - sets; x += sets)
#pragma unroll
      for (int d = 0; d < DT; ++d) o[rt][d] += osh[x][rt][d][lane];
    if (r0 + rt * 16 + r16 < R) store_rows<DH>(a, o[rt], m[rt], beyond ? NAN32 : l[rt], pos[rt], split, row_at[rt], row_at[rt] + part_from, g);
  }
}

// Many rows: a workgroup of 8 waves has 256 rows of a KV head, a wave 32 of them, and a page is converted to bf16 once for all, on its
// way to LDS.  S^T = K Q^T and O^T += V^T P^T, 32 x 32 x 16: row 8 b + 4 c + i of a key tile is entry 16 (b / 2) + 8 c + 4 (b % 2) + i, so that
// again a lane's scores are the operand it gives, here against eight neighbouring entries of a value's row.  Scores of the next page
// are formed while the softmax of the present one runs: keys are in LDS one page ahead of values.
// A prompt of 4095 tokens, 64 heads over 8, d 128: 284 us back to back, 0.98 PFLOP/s (334 under the tracer).  Of a compute unit's busy cycles
// the products take 44 %, vector instructions 45, LDS 28, partly one behind the other; it is no single one of them: without products, without
// LDS reads, without the maxima or without the barrier the time stays, without conversion it falls by 15 %.  Slower were 64 rows a wave on half
// the waves (538: accumulators and queries exceed the registers that vector instructions reach), two workgroups of 4 waves (317
// against 303: each converts the page), values a page behind, so that all products run beside the softmax (317).
#define MANY_WAVES 8
#define MANY_ROWS (MANY_WAVES * 32)
typedef __attribute__((ext_vector_type(16))) float f32x16;
__device__ __forceinline__ int many_tiles(int R, int above) { return R > above ? (R + MANY_ROWS - 1) / MANY_ROWS : 0; }

template <int DH>
__global__ __launch_bounds__(MANY_WAVES * 64, 2) void attend_many_kernel(QuantCache c, AttendArgs a) {
  constexpr int KS = DH / 16, DT = DH / 32;
  constexpr int KB = 65, VB = 66;              // 16-byte units of an operand block: 64, and what keeps the writes of 8 lanes apart
  constexpr bool BOTH = DH == 128;             // a thread brings 16 bytes of the keys and of the values; with 64 either
  __shared__ u32x4 ksh[2][2 * KS * KB], vsh[2][DT * 4 * VB];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, half = lane >> 5;
  const int h = blockIdx.x % c.n_kv_heads, at = blockIdx.x / c.n_kv_heads, G = a.G;
  int split = at % a.splits, splits = a.splits, tile = gridDim.x / (c.n_kv_heads * a.splits) - 1 - at / a.splits;       // the longest first
  if (a.tiled) {                               // the others are not split
    if (at < a.tiled * a.splits) tile = a.tiled - 1 - at / a.splits;
    else tile = at - a.tiled * (a.splits - 1), split = 0, splits = 1;
  }
  Span sp = find_span(c, a.rows, a.n_rows, tile, [&](int M) { return many_tiles(M * G, a.above); });
  sp.s = __builtin_amdgcn_readfirstlane(sp.s);
  if (sp.s < 0) return;
  sp.t = __builtin_amdgcn_readfirstlane(sp.t), sp.row = __builtin_amdgcn_readfirstlane(sp.row), sp.M = __builtin_amdgcn_readfirstlane(sp.M);
  const int given = __builtin_amdgcn_readfirstlane(sp.len);
  const bool beyond = given > c.max_pages * PAGE;
  const int len = max(given, 0), first = len - sp.M, R = sp.M * G;
  const int wg0 = sp.t * MANY_ROWS, wg_last = min(wg0 + MANY_ROWS, R) - 1, r0 = wg0 + w * 32, r_last = min(r0 + 32, R) - 1;
  const Seen seen = seen_pages(first + wg0 / G, beyond ? -1 : first + wg_last / G, a.window, a.sinks);
  const int per = (seen.n + splits - 1) / splits, i0 = split * per, n = min(i0 + per, seen.n) - i0;
  const int see_all = first + r0 / G, low_all = a.window ? first + max(r_last, 0) / G - a.window + 1 : 0;

  const int r = r0 + r32;
  const bool valid = r < R;
  const int tok = valid ? r / G : 0, hq = h * G + (valid ? r % G : 0), pos = valid ? first + tok : -1;
  const size_t row_at = (size_t)(sp.row + tok) * a.n_heads + hq;
  bf16x8 qf[KS];
#pragma unroll
  for (int j = 0; j < KS; ++j)
    qf[j] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(a.q + (size_t)(sp.row + tok) * a.ldq + (size_t)hq * DH + half * 8 + j * 16));
  float m = pos < 0 ? 0.f : NONE, l = 0.f;      // as in tiles of 16: lanes without a row are not FAR
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x16{};

  // what this thread brings of a page, and where it goes
  const bool has_k = BOTH || tid < 256, has_v = BOTH || tid >= 256;
  const int kt = tid / KS % 64, kj = tid % KS, ku = kt & 31;
  const int kto = ((kt >> 5) * KS + kj) * KB + 8 * (2 * (ku >> 4) + ((ku >> 2) & 1)) + 4 * ((ku >> 3) & 1) + (ku & 3);
  const int vd = tid / 4 % DH, vj = tid & 3, vto = ((vd >> 5) * 4 + vj) * VB + (vd & 31);
  PageList pages(c, sp.s, seen, h, i0, 1);
  struct Raw {
    u32x4 k, v;
    float ks, vs;
    int id;
  };
  // keys are asked for first, the values of the same page a step later
  auto load_k = [&](Raw& p, int i) {
    p.id = pages.get(i, &p.ks, &p.vs);
    if (has_k) p.k = *reinterpret_cast<const u32x4*>(c.k + ((size_t)max(p.id, 0) * c.n_kv_heads + h) * PAGE * DH + kt * DH + kj * 16);
  };
  auto load_v = [&](Raw& p) {
    if (has_v) p.v = *reinterpret_cast<const u32x4*>(c.v + ((size_t)max(p.id, 0) * c.n_kv_heads + h) * PAGE * DH + vd * PAGE + vj * 16);
  };
  auto put_keys = [&](const Raw& p, int to) {
    if (!has_k) return;
    u32x4 lo, hi;
    if (p.id >= 0) {
      lo = __builtin_bit_cast(u32x4, to_bf16x8(p.k[0], p.k[1], p.ks));
      hi = __builtin_bit_cast(u32x4, to_bf16x8(p.k[2], p.k[3], p.ks));
    } else lo = hi = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};      // no such page: whoever sees it becomes NaN
    ksh[to][kto] = lo;
    ksh[to][kto + 32] = hi;
  };
  auto put_values = [&](Raw& p, int i, int to) {
    if (!has_v) return;
    const int e0 = seen.page(i0 + i) * PAGE;
    if (p.id < 0 || e0 + PAGE > len) {         // entries behind the last one, or of no page, may hold anything: 0 times a NaN would be one
      p.v = first_bytes(p.v, p.id >= 0 ? min(len - e0, PAGE) - 16 * vj : 0);
    }
    const float scale = p.id >= 0 ? p.vs : 0.f;
    vsh[to][vto] = __builtin_bit_cast(u32x4, to_bf16x8(p.v[0], p.v[1], scale));
    vsh[to][vto + 32] = __builtin_bit_cast(u32x4, to_bf16x8(p.v[2], p.v[3], scale));
  };
  auto scores = [&](f32x16 (&s)[2], int from) {
    s[0] = f32x16{}, s[1] = f32x16{};
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ksh[from][(t * KS + j) * KB + lane]), qf[j], s[t], 0, 0, 0);
  };
  Raw rk = {}, rv = {};                        // of the page whose keys go to LDS next, and of the one before it
  const int low = a.window ? pos - a.window : INT_MIN;
  auto step = [&](f32x16 (&s)[2], f32x16 (&ahead)[2], int i) {
    __syncthreads();                           // keys of page i + 1 and values of page i are there, their other places free
    if (i + 2 < n) put_keys(rk, i & 1);
    if (i + 1 < n) put_values(rv, i + 1, (i + 1) & 1);
    rv = rk;
    if (i + 2 < n) load_v(rv);
    if (i + 3 < n) load_k(rk, i + 3);
    const int e0 = seen.page(i0 + i) * PAGE;
    if (!(e0 + PAGE - 1 <= see_all && (!a.window || e0 >= low_all || e0 + PAGE <= a.sinks))) {
      const int mine = e0 + 8 * half;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int e = mine + 32 * t + 16 * (x >> 3) + (x & 7);
          s[t][x] = (e <= pos) & ((e > low) | (e < a.sinks)) ? s[t][x] : -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int x = 0; x < 16; ++x) mx = fmaxf(mx, s[t][x]);
    auto other = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = fmaxf(__uint_as_float(other[0]), __uint_as_float(other[1])) * a.scale_log2e;
    if (__any(mx > m + LAG)) {                 // maxima settle after a few pages
      asm volatile("" ::: "memory");           // and what is to do then stays here
      const float m_new = mx > m + LAG ? mx : m, corr = __builtin_amdgcn_exp2f(m - m_new);      // of the rows that need it
      m = m_new;
      l *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= corr;
    }
    // the product with the scale in one rounding with the difference, unless its own rounding, left in the largest score, would count
    const bool far = fabsf(m) > FAR;
    float by = a.scale_log2e, less = m;
    if (__any(far)) {
      asm volatile("" ::: "memory");
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int x = 0; x < 16; ++x) s[t][x] = far ? difference(s[t][x], a.scale_log2e, m) : s[t][x];
      by = far ? 1.f : by, less = far ? 0.f : m;
    }
    scores(ahead, (i + 1) & 1);                // behind the last page: of nothing, for nobody
    bf16x8 pf[4];
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float v = __builtin_amdgcn_exp2f(fmaf(s[t][x], by, -less));
        sum += v;
        pf[t * 2 + (x >> 3)][x & 7] = (__bf16)v;
      }
    l += sum;
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vsh[i & 1][(d * 4 + y) * VB + lane]), pf[y], o[d], 0, 0, 0);
    // operands are asked for six products ahead; the softmax goes between the products of the next scores
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
    for (int j = 0; j < 2 * KS; ++j) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x2, 112 / (2 * KS), 0);
    }
#pragma unroll
    for (int j = 0; j < 4 * DT; ++j) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
  };
  if (n > 0) {
    f32x16 s0[2], s1[2];
    load_k(rv, 0);
    load_v(rv);
    if (n > 1) load_k(rk, 1);
    put_keys(rv, 0);
    put_values(rv, 0, 0);
    if (n > 1) put_keys(rk, 1);
    rv = rk;
    if (n > 1) load_v(rv);
    if (n > 2) load_k(rk, 2);
    __syncthreads();
    scores(s0, 0);
    for (int i = 0; i < n; i += 2) {
      step(s0, s1, i);
      if (i + 1 < n) step(s1, s0, i + 1);
    }
  }
  auto other = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(other[0]) + __uint_as_float(other[1]);
  if (!valid) return;
  if (beyond) l = __uint_as_float(0x7fc00000u);
  if (splits == 1) {
    const bool empty = pos < 0;
    const float inv = empty ? 0.f : 1.f / l;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        bf16 b[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) b[y] = __float2bfloat16(o[d][x * 4 + y] * inv);
        *reinterpret_cast<uint2*>(a.out + row_at * DH + d * 32 + x * 8 + half * 4) = *reinterpret_cast<const uint2*>(b);
      }
    if (a.lse && half == 0) a.lse[row_at] = empty ? -INFINITY : (m + __log2f(l)) * LN2;
  } else {
    const size_t at = split * a.part_rows + (a.tiled ? ((size_t)tile * c.n_kv_heads + h) * MANY_ROWS + r - wg0 : row_at);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<f32x4*>(a.part + at * DH + d * 32 + x * 8 + half * 4) = f32x4{o[d][x * 4], o[d][x * 4 + 1], o[d][x * 4 + 2], o[d][x * 4 + 3]};
    if (half == 0) a.part_ml[at] = make_float2(pos < 0 ? -INFINITY : m, l);
  }
}

// Parts of a row's attention together.  WAVES waves have a row and head: a lane the maximum and sum of a part (there are at most 64), then
// 4 elements of some of the parts, the first eight of them asked for beside the sums.  64 parts of 64 rows: 4.8 us (a wave that adds
// one part after the other: 62); two trips to memory and the launch.
#define MERGE_WAVES 4
#define MERGE_PARTS 64
template <int DH, int WAVES>
__global__ __launch_bounds__(MERGE_WAVES * 64) void attend_merge_kernel(QuantCache c, AttendArgs a) {
  constexpr int LANES = DH / 4, WAYS = 64 / LANES * WAVES, AHEAD = 8;
  __shared__ f32x4 osh[MERGE_WAVES][LANES];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, way = w % WAVES * (64 / LANES) + lane / LANES;
  const size_t all = a.part_rows, at = (size_t)blockIdx.x * (MERGE_WAVES / WAVES) + w / WAVES;
  if (at >= all) return;                                                        // WAVES == 4: the whole workgroup
  int row = (int)(at / a.n_heads), head = (int)(at % a.n_heads);
  if (a.tiled) {
    const int h = (int)(at / MANY_ROWS) % c.n_kv_heads, tile = (int)(at / MANY_ROWS) / c.n_kv_heads;
    const Span sp = find_span(c, a.rows, a.n_rows, tile, [&](int M) { return many_tiles(M * a.G, a.above); });
    const int r = sp.t * MANY_ROWS + (int)(at % MANY_ROWS);
    if (sp.s < 0 || r >= sp.M * a.G) return;
    row = sp.row + r / a.G, head = h * a.G + r % a.G;
  } else if (a.per) {
    const int s = row / a.per, first = min(max(a.rows[s], 0), a.n_rows), M = min(max(a.rows[s + 1], first), a.n_rows) - first;
    row -= s * a.per;
    if (row >= M || M * a.G > a.upto) return;
    row += first;
  } else if (a.rows) {
    if (row >= a.rows[c.n_seqs] || row < a.rows[0]) return;                   // rows of no sequence have no parts and stay as they are
  }
  const size_t to = (size_t)row * a.n_heads + head;
  const float2 ml = lane < a.splits ? a.part_ml[lane * all + at] : make_float2(-INFINITY, 0.f);
  const float* from = a.part + at * DH + (lane % LANES) * 4;
  f32x4 ahead[AHEAD];
#pragma unroll
  for (int x = 0; x < AHEAD; ++x) {
    const int s = way + x * WAYS;
    ahead[x] = s < a.splits ? *reinterpret_cast<const f32x4*>(from + s * all * DH) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float top = wave_max(ml.x);
  const bool empty = top == -INFINITY;                                          // in every part: the row sees nothing
  const float f = empty || lane >= a.splits ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
  const float sum = wave_sum(ml.y * f);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < AHEAD; ++x) o += ahead[x] * __shfl(f, (way + x * WAYS) & 63);
  if (AHEAD * WAYS < MERGE_PARTS)
#pragma unroll 8
    for (int s = way + AHEAD * WAYS; s < a.splits; s += WAYS) o += *reinterpret_cast<const f32x4*>(from + s * all * DH) * __shfl(f, s);
#pragma unroll
  for (int d = LANES; d < 64; d <<= 1)
#pragma unroll
    for (int x = 0; x < 4; ++x) o[x] += __shfl_xor(o[x], d);
  if (WAVES > 1) {
    if (lane < LANES) osh[w][lane] = o;
    __syncthreads();
    if (w % WAVES) return;
#pragma unroll
    for (int x = 1; x < WAVES; ++x) o += osh[w + x][lane % LANES];
  }
  if (lane >= LANES) return;
  const float inv = empty ? 0.f : 1.f / sum;
  bf16 b[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) b[x] = __float2bfloat16(o[x] * inv);
  *reinterpret_cast<uint2*>(a.out + to * DH + lane * 4) = *reinterpret_cast<const uint2*>(b);
  if (a.lse && lane == 0) a.lse[to] = empty ? -INFINITY : (top + __log2f(sum)) * LN2;
}

// ---- attention weight of the entries ------------------------------------------------------------------------------------------
// w[entry] = sum over the rows and heads of a group of exp(score - lse).
struct Rows {
  int row, M, len, first, R;
  bool none;
};
__device__ __forceinline__ Rows rows_of(const QuantCache& c, const int* rows, int n_rows, int s, int G) {
  Rows r;
  r.M = n_rows / c.n_seqs, r.row = s * r.M;
  if (rows) {
    r.row = min(max(rows[s], 0), n_rows);
    r.M = min(max(rows[s + 1], r.row), n_rows) - r.row;
  }
  const int given = c.len[s];
  r.len = max(given, 0), r.first = r.len - r.M, r.R = r.M * G;
  r.none = r.M == 0 || given > c.max_pages * PAGE || given <= 0;
  return r;
}

// slices of a sequence's tiles of 64 rows where sequences differ, 0 if its rows are few
__device__ __forceinline__ int slices_of(const WeighArgs& a, int M) {
  const int R = M * a.G;
  return R > a.above ? ((R + 63) / 64 + a.tiles - 1) / a.tiles : 0;
}

// Few rows: their queries stay in registers, up to RT tiles of 16 at a time, and a wave goes over pages.  S^T = K Q^T as in the attention:
// a lane's scores belong to one row, so that sums over the rows of a tile are sums over 16 lanes, once per page.  One row each of 8
// sequences, 64 heads over 8, 34 MB of keys: 13.6 us, trips to memory before the first page and one or two pages a wave.
#define WEIGH_WAVES 4
template <int DH, int RT>
__global__ __launch_bounds__(WEIGH_WAVES * 64, 2) void weigh_few_kernel(QuantCache c, WeighArgs a) {
  constexpr int KS = DH / 32;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.y, s = blockIdx.z, G = a.G;
  const Rows rs = rows_of(c, a.rows, a.n_rows, s, G);
  if (rs.none || rs.R > a.upto) return;
  const int first = rs.first, len = rs.len;
  const Seen seen = seen_pages(first, len - 1, a.window, a.sinks);
  const int from = blockIdx.x * WEIGH_WAVES + w, step = gridDim.x * WEIGH_WAVES;
  const int mine = (seen.n - from + step - 1) / step;
  if (mine <= 0) return;
  float* to = a.weight + ((size_t)s * c.n_kv_heads + h) * a.ldw;
  for (int r0 = 0; r0 < rs.R; r0 += 16 * RT) {                // once, unless the rows are far more than those of other sequences
    bf16x8 qf[RT][KS];
    float lse[RT];
    int pos[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = r0 + rt * 16 + r16;
      const bool valid = r < rs.R;
      const int tok = valid ? r / G : 0, hq = h * G + (valid ? r % G : 0);
      pos[rt] = valid ? first + tok : -1;
      lse[rt] = valid ? a.lse[(size_t)(rs.row + tok) * a.n_heads + hq] * LOG2E : 0.f;
      const bf16* q = a.q + (size_t)(rs.row + tok) * a.ldq + (size_t)hq * DH + g * 16;
#pragma unroll
      for (int j = 0; j < KS; ++j) qf[rt][j] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(q + (j >> 1) * 64 + (j & 1) * 8));
    }
    const int see_all = first + r0 / G, low_all = a.window ? first + min(r0 + 16 * RT, rs.R) / G - a.window + 1 : 0;
    PageList pages(c, s, seen, h, from, step);
    u32x4 kd[4][DH / 64];
    float ks, vs;
    pages.fetch(0);
    load_keys<DH>(c, kd, pages.first_id(), h, lane);
    pages.settle();
    int id = pages.get(0, &ks, &vs);
    for (int i = 0; i < mine; ++i) {
      const int e0 = seen.page(from + i * step) * PAGE;
      const float kscale = ks, by = id >= 0 ? a.scale_log2e : NAN32;      // no such page: whoever sees it becomes NaN
      u32x4 now[4][DH / 64];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int f = 0; f < DH / 64; ++f) now[t][f] = kd[t][f];
      if (i + 1 < mine) {
        id = pages.get(i + 1, &ks, &vs);
        load_keys<DH>(c, kd, id, h, lane);
      }
      const bool all = e0 + PAGE - 1 <= see_all && (!a.window || e0 >= low_all || e0 + PAGE <= a.sinks) && r0 + 16 * RT <= rs.R;
      f32x4 sum[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f32x4 x[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) x[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          const bf16x8 kf = to_bf16x8(now[t][j >> 1][(j & 1) * 2], now[t][j >> 1][(j & 1) * 2 + 1], kscale);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) x[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rt][j], x[rt], 0, 0, 0);
        }
        sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const int low = a.window ? pos[rt] - a.window : INT_MIN;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            float v = __builtin_amdgcn_exp2f(difference(x[rt][y], by, lse[rt]));
            if (!all) {
              const int e = e0 + 16 * g + 4 * t + y;
              v = (e <= pos[rt]) & ((e > low) | (e < a.sinks)) ? v : 0.f;
            }
            sum[t][y] += v;
          }
        }
      }
      float v = 0.f;                                          // lane 16 g + 4 t + y: that entry of the page
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const float x = row_sum(sum[t][y]);
          v = r16 == 4 * t + y ? x : v;
        }
      const int e = e0 + lane;
      if (e < len) to[e] = e < first || r0 ? to[e] + v : v;    // an entry of these rows begins here
    }
  }
}

// Many rows: a wave keeps the 64 keys of a page as operands and the workgroup goes over tiles of 64 rows, whose queries, logarithms and
// entries pass through LDS.  S = Q K^T, 32 x 32 x 16: a lane's scores belong to one entry.  The tiles that see a group of pages are dealt to
// `slices` workgroups, or to as many of them as `a.tiles` asks for where sequences differ; sums of slices are added in their order.  2047 rows,
// 64 heads over 8, 34.9 GFLOP: 61 us traced (58 back to back, with 4.8 for the slices' sums), products in 35 % of the cycles, vector instructions in
// 52; about 6 us of it before the first product and nine tiles behind; three workgroups a CU do not fit the registers (142, spilling).
template <int DH>
__global__ __launch_bounds__(WEIGH_WAVES * 64, 2) void weigh_many_kernel(QuantCache c, WeighArgs a) {
  constexpr int KS = DH / 16, QB = 66, CH = DH / 8, LOADS = 64 * CH / (WEIGH_WAVES * 64);
  __shared__ u32x4 qsh[2][2 * KS * QB];
  __shared__ __align__(16) float lsh[2][64];
  __shared__ __align__(16) int psh[2][64];
  __shared__ int nans[2];                                      // whether a row of the tile has a NaN as its logarithm
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, half = lane >> 5;
  // pages that most rows see first
  const int h = blockIdx.x % c.n_kv_heads, G = a.G, group = blockIdx.x / c.n_kv_heads / a.slices;
  int s = blockIdx.y, slice = blockIdx.x / c.n_kv_heads % a.slices, slices = a.slices;
  if (a.tiles) {
    const Span sp = find_span(c, a.rows, a.n_rows, blockIdx.y, [&](int M) { return slices_of(a, M); });
    s = __builtin_amdgcn_readfirstlane(sp.s);
    if (s < 0) return;
    slice = __builtin_amdgcn_readfirstlane(sp.t), slices = slices_of(a, __builtin_amdgcn_readfirstlane(sp.M));
  }
  const Rows rs = rows_of(c, a.rows, a.n_rows, s, G);
  if (rs.none) return;
  const int first = rs.first, len = rs.len, R = rs.R;
  const Seen seen = seen_pages(first, len - 1, a.window, a.sinks);
  const int i = group * WEIGH_WAVES + w;
  if (group * WEIGH_WAVES >= seen.n) return;
  const bool has = i < seen.n;
  const int page = seen.page(min(i, seen.n - 1)), e0 = page * PAGE;
  const int id = c.table[(size_t)s * c.table_ld + page];
  const bool there = (unsigned)id < (unsigned)c.n_pages;
  const size_t block = (size_t)(there ? id : 0) * c.n_kv_heads + h;
  const float kscale = c.scale[block * 2];
  bf16x8 kf[2][KS];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int j = 0; j < KS; j += 2) {                          // 16 bytes of a key are two operands: d in that order on both sides
      const u32x4 x = *reinterpret_cast<const u32x4*>(c.k + block * PAGE * DH + (t * 32 + r32) * DH + j * 16 + half * 16);
      kf[t][j] = to_bf16x8(x[0], x[1], kscale);
      kf[t][j + 1] = to_bf16x8(x[2], x[3], kscale);
    }
  const float by = a.scale_log2e;
  if (!there) {                                                // no such page: whoever sees it becomes NaN
    constexpr unsigned NANS = 0x7fc07fc0u;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < KS; ++j) kf[t][j] = __builtin_bit_cast(bf16x8, u32x4{NANS, NANS, NANS, NANS});
  }
  // tiles with rows that see any of the group's pages
  const int lo_e = seen.page(group * WEIGH_WAVES) * PAGE, hi_e = seen.page(min(group * WEIGH_WAVES + WEIGH_WAVES, seen.n) - 1) * PAGE + PAGE - 1;
  const int tiles = (R + 63) / 64, tile0 = max(0, lo_e - first) * G / 64;
  int tile1 = tiles;
  if (a.window && lo_e >= a.sinks && hi_e + a.window - first < rs.M) tile1 = min(tiles, max(0, hi_e + a.window - first) * G / 64 + 1);
  const int all_tiles = max(0, tile1 - tile0), t0 = tile0 + (int)((long long)slice * all_tiles / slices), t1 = tile0 + (int)((long long)(slice + 1) * all_tiles / slices);
  auto token = [&](int r) { return (int)((unsigned long long)(unsigned)r * a.by_group >> 38); };      // r / G
  // rows that see all of this wave's page
  const int see_from = max(0, e0 + PAGE - 1 - first) * G;
  const int see_to = a.window && e0 + PAGE > a.sinks ? (int)min((long long)R, max(0ll, (long long)e0 + a.window - first) * G) : R;
  u32x4 raw[LOADS];
  const bf16* from[LOADS];
  float lse = 0.f;
  int pos = -1;
  // where a tile's rows stand: 64 rows further on where they are whole tokens, else worked out anew
  const bool whole = 64 % G == 0;
  const size_t on = (size_t)(64 / min(G, 64)) * a.ldq;
  auto load = [&](int tile) {
    if (whole && tile > t0 && tile * 64 + 64 <= R) {
#pragma unroll
      for (int x = 0; x < LOADS; ++x) from[x] += on;
    } else {
#pragma unroll
      for (int x = 0; x < LOADS; ++x) {
        const int at = x * WEIGH_WAVES * 64 + tid, r = min(tile * 64 + at / CH, R - 1), tok = token(r);
        from[x] = a.q + (size_t)(rs.row + tok) * a.ldq + (size_t)(h * G + r - tok * G) * DH + at % CH * 8;
      }
    }
#pragma unroll
    for (int x = 0; x < LOADS; ++x) raw[x] = *reinterpret_cast<const u32x4*>(from[x]);
    if (tid < 64) {
      const int r = min(tile * 64 + tid, R - 1), tok = token(r);
      lse = a.lse[(size_t)(rs.row + tok) * a.n_heads + h * G + r - tok * G] * LOG2E;
      pos = tile * 64 + tid < R ? first + tok : -1;
    }
  };
  auto put = [&](int to) {
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
      // 8 elements: 32 j + 16 c + 8 b are those of step 2 j + b in the lanes of half c
      const int at = x * WEIGH_WAVES * 64 + tid, r = at / CH, ch = at % CH;
      qsh[to][((r >> 5) * KS + ch / 4 * 2 + (ch & 1)) * QB + (ch >> 1 & 1) * 33 + (r & 31)] = raw[x];
    }
    // -inf, the score of what a row does not see, less its logarithm has to be -inf: that of a row that sees nothing becomes finite here, a
    // NaN where scores are hidden
    if (tid < 64) {
      lsh[to][tid] = lse < -FLT_MAX ? -FLT_MAX : lse, psh[to][tid] = pos;
      nans[to] = __ballot(lse != lse) != 0;
    }
  };
  float sum[2][2] = {};
  // 32 of the 64 rows: their scores, what they do not see, and their logarithms, which the tile's place will not keep
  struct Part {
    f32x16 x[2];
    float lse[16];
    int nans;
  } p0, p1;
  auto mask = [&](Part& p, int at, int r0) {
    if (r0 >= see_from && r0 + 32 <= see_to) return;
    if (__builtin_amdgcn_readfirstlane(p.nans)) {              // to the scores, of which only those that count stay
#pragma unroll
      for (int y = 0; y < 16; ++y)
        if (p.lse[y] != p.lse[y]) p.x[0][y] = p.x[1][y] = p.lse[y], p.lse[y] = 0.f;
    }
#pragma unroll
    for (int y = 0; y < 16; ++y) {
      const int pos = psh[at][(r0 & 32) + 8 * (y >> 2) + 4 * half + (y & 3)], low = a.window ? pos - a.window : INT_MIN;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int e = e0 + t * 32 + r32;
        p.x[t][y] = (e <= pos) & ((e > low) | (e < a.sinks)) ? p.x[t][y] : -INFINITY;
      }
    }
  };
  auto weights = [&](const Part& p, int y) {
#pragma unroll
    for (int t = 0; t < 2; ++t) sum[t][y & 1] += __builtin_amdgcn_exp2f(fmaf(p.x[t][y], by, -p.lse[y]));
  };
  // scores of `p`, and between their products the weights of `done`
  auto scores = [&](Part& p, int at, int b, const Part& done, auto both) {
    constexpr int AHEAD = 4;
    bf16x8 qf[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) qf[j] = __builtin_bit_cast(bf16x8, qsh[at][(b * KS + j) * QB + half * 33 + r32]);
    p.x[0] = f32x16{}, p.x[1] = f32x16{};
#pragma unroll
    for (int j = 0; j < KS; ++j) {
#pragma unroll
      for (int t = 0; t < 2; ++t) p.x[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[j % AHEAD], kf[t][j], p.x[t], 0, 0, 0);
      if (j + AHEAD < KS) qf[j % AHEAD] = __builtin_bit_cast(bf16x8, qsh[at][(b * KS + j + AHEAD) * QB + half * 33 + r32]);
      if (both.value) {
#pragma unroll
        for (int y = 0; y < 16; ++y)
          if (y * KS / 16 == j) weights(done, y);
      }
      __builtin_amdgcn_sched_barrier(0);                       // left alone the products come first, one chain behind the other
    }
#pragma unroll
    for (int y = 0; y < 16; ++y) p.lse[y] = lsh[at][b * 32 + 8 * (y >> 2) + 4 * half + (y & 3)];
    p.nans = nans[at];
  };
  if (t0 < t1) {
    load(t0);
    put(0);
    if (t0 + 1 < t1) load(t0 + 1);
    __syncthreads();
    scores(p0, 0, 0, p1, std::false_type());
    for (int tile = t0;; ++tile) {
      const int at = (tile - t0) & 1;
      mask(p0, at, tile * 64);
      scores(p1, at, 1, p0, std::true_type());
      mask(p1, at, tile * 64 + 32);
      if (tile + 1 == t1) break;
      put(at ^ 1);                                             // read last in front of the barrier before
      if (tile + 2 < t1) load(tile + 2);
      __syncthreads();
      scores(p0, at ^ 1, 0, p1, std::true_type());
    }
#pragma unroll
    for (int y = 0; y < 16; ++y) weights(p1, y);
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const unsigned x = __float_as_uint(sum[t][0] + sum[t][1]);
    auto o = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    sum[t][0] = __uint_as_float(o[0]) + __uint_as_float(o[1]);
  }
  const float v = half ? sum[1][0] : sum[0][0];
  const int e = e0 + lane;
  if (!has || e >= len) return;
  if (slices == 1) {
    float* to = a.weight + ((size_t)s * c.n_kv_heads + h) * a.ldw + e;
    *to = e < first ? *to + v : v;                             // an entry of these rows begins here
  } else a.part[(((a.tiles ? blockIdx.y : (size_t)slice * c.n_seqs + s) * c.n_kv_heads + h) * a.pages + i) * PAGE + lane] = v;
}

__global__ __launch_bounds__(256) void weigh_add_kernel(QuantCache c, WeighArgs a) {
  const int h = blockIdx.y, s = blockIdx.z;
  const Rows rs = rows_of(c, a.rows, a.n_rows, s, a.G);
  if (rs.none) return;
  int slices = a.slices, from = s;                             // the first of its slices
  if (a.tiles) {
    slices = slices_of(a, rs.M), from = 0;
    if (slices < 2) return;                                    // written by its only slice, or by the other pass
    for (int base = 0; base < s; base += 64) {
      const int x = base + (int)(threadIdx.x & 63), first = x < s ? min(max(a.rows[x], 0), a.n_rows) : 0;
      const int mine = x < s ? slices_of(a, min(max(a.rows[x + 1], first), a.n_rows) - first) : 0;
      from += __builtin_amdgcn_readlane(lanes_upto(mine), 63);
    }
    if (from + slices > a.ids) return;                         // beyond: row numbers that do not rise
  }
  const Seen seen = seen_pages(rs.first, rs.len - 1, a.window, a.sinks);
  const int i = blockIdx.x * 4 + threadIdx.x / PAGE;
  if (i >= seen.n) return;
  const int e = seen.page(i) * PAGE + threadIdx.x % PAGE;
  if (e >= rs.len) return;
  const size_t block = (size_t)c.n_kv_heads * a.pages * PAGE, all = a.tiles ? block : c.n_seqs * block;
  const float* p = a.part + (((size_t)from * c.n_kv_heads + h) * a.pages + i) * PAGE + threadIdx.x % PAGE;
  float* to = a.weight + ((size_t)s * c.n_kv_heads + h) * a.ldw + e;
  float v = e < rs.first ? *to : 0.f;                          // an entry of these rows begins here
#pragma unroll 8
  for (int x = 0; x < slices; ++x) v += p[x * all];
  *to = v;
}

// ---- eviction -----------------------------------------------------------------------------------------------------------------
// One workgroup per sequence and head finds the weight of the last entry that is kept, 11 bits of an ordered key at a time (the first
// ones are sign, exponent and two more, so that few entries of a wave meet in a counter), and lists the entries that are kept in their
// order; then a workgroup per page of 64 of them moves their codes.  A wave has a stretch of entries, in registers where that is up to 1024.
// Select: 4096 entries of one sequence 11 us, 16 ragged sequences of up to 16384 17 us; barriers and counters in LDS.  Gather of 2048
// entries of those 16, 8 heads of 128: 55 us; a value's elements are 64 bytes apart, so nearly all pages of values are read whole.
#define SELECT_THREADS 1024
#define SELECT_WAVES (SELECT_THREADS / 64)
#define SELECT_KEYS 16

// larger weights have larger keys, equal ones the same; a NaN counts as the least
__device__ __forceinline__ unsigned weight_key(float w) {
  const unsigned b = __float_as_uint(w + 0.f);
  return w != w ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(SELECT_THREADS) void evict_select_kernel(QuantCache c, EvictArgs a) {
  __shared__ int hist[2048];
  __shared__ int found[2];
  __shared__ int counts[SELECT_WAVES][2];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x, s = blockIdx.y;
  const int given = c.len[s], len = given > c.max_pages * PAGE ? 0 : max(given, 0);
  const float* weight = a.weight + ((size_t)s * c.n_kv_heads + h) * a.ldw;
  float* to_weight = a.to_weight + ((size_t)s * c.n_kv_heads + h) * a.ldt;
  int* kept = a.kept + ((size_t)s * c.n_kv_heads + h) * a.budget;
  const int n = min(len, a.budget);
  if (h == 0 && tid == 0) a.to_len[s] = given > c.max_pages * PAGE ? INT_MAX / 2 : n;
  for (int i = n + tid; i < a.budget; i += SELECT_THREADS) kept[i] = -1;
  if (len <= a.budget) {
    for (int i = tid; i < n; i += SELECT_THREADS) kept[i] = i, to_weight[i] = weight[i];
    return;
  }
  const int lo = a.sinks, hi = len - a.recent;                  // between them by weight
  int want = a.budget - a.sinks - a.recent;                     // so many of them, fewer than there are
  const int stretch = ((hi - lo + SELECT_WAVES - 1) / SELECT_WAVES + 63) / 64 * 64;
  const int from = lo + w * stretch, to = min(from + stretch, hi);
  const bool fits = stretch <= 64 * SELECT_KEYS;
  unsigned keys[SELECT_KEYS];
  if (fits) {
    float v[SELECT_KEYS];
#pragma unroll
    for (int x = 0; x < SELECT_KEYS; ++x) {
      const int i = from + x * 64 + lane;
      v[x] = i < to ? weight[i] : 0.f;
    }
#pragma unroll
    for (int x = 0; x < SELECT_KEYS; ++x) keys[x] = weight_key(v[x]);
  }
  // f(entry, key, whether there is one) for the wave's entries, 64 at a time in their order
  auto each = [&](auto f) {
    if (fits) {
#pragma unroll
      for (int x = 0; x < SELECT_KEYS; ++x) {
        const int i = from + x * 64 + lane;
        if (from + x * 64 < to) f(i, keys[x], i < to);
      }
    } else {
      for (int i = from + lane; i - lane < to; i += 64) f(i, i < to ? weight_key(weight[i]) : 0u, i < to);
    }
  };
  unsigned key = 0, mask = 0;                                   // the bits of the last kept key that are known
  if (want > 0) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const unsigned bits = pass == 2 ? 1023u : 2047u;
      hist[tid] = hist[tid + SELECT_THREADS] = 0;
      __syncthreads();
      each([&](int, unsigned k, bool in) {
        if (in && (k & mask) == key) atomicAdd(&hist[k >> shift & bits], 1);
      });
      __syncthreads();
      const int first = hist[2047 - 2 * tid], second = hist[2046 - 2 * tid];       // from the largest digit down
      const int upto = lanes_upto(first + second);
      if (lane == 63) counts[w][0] = upto;
      __syncthreads();
      const int waves = lanes_upto(counts[lane % SELECT_WAVES][0]);             // of the waves up to lane's in the first row of lanes
      const int before = upto - first - second + (w ? __builtin_amdgcn_readlane(waves, max(w - 1, 0)) : 0);
      if (before < want && before + first >= want) found[0] = 2047 - 2 * tid, found[1] = want - before;
      else if (before + first < want && before + first + second >= want) found[0] = 2046 - 2 * tid, found[1] = want - before - first;
      __syncthreads();
      key |= (unsigned)found[0] << shift;
      mask |= bits << shift;
      want = found[1];                                          // so many of those with this digit
    }
  } else key = 0xffffffffu;                                     // above every key (a NaN's bits do not reach it)
  // larger keys are kept, and the first `want` equal ones
  int more = 0, equal = 0;
  each([&](int, unsigned k, bool in) {
    more += __popcll(__ballot(in && k > key));
    equal += __popcll(__ballot(in && k == key));
  });
  __syncthreads();                                              // counts have been read
  if (lane == 0) counts[w][0] = more, counts[w][1] = equal;
  __syncthreads();
  int at = a.sinks, equals = 0;                                 // places and equal ones in front of this wave
  {
    const int m = lanes_upto(counts[lane % SELECT_WAVES][0]), e = lanes_upto(counts[lane % SELECT_WAVES][1]);
    equals = w ? __builtin_amdgcn_readlane(e, max(w - 1, 0)) : 0;
    at += (w ? __builtin_amdgcn_readlane(m, max(w - 1, 0)) : 0) + min(equals, max(want, 0));
  }
  const unsigned long long below = (1ull << lane) - 1;
  each([&](int i, unsigned k, bool in) {
    const unsigned long long eq = __ballot(in && k == key);
    const bool keep = in && (k > key || (k == key && equals + __popcll(eq & below) < want));
    const unsigned long long all = __ballot(keep);
    if (keep) {
      const int to_at = at + __popcll(all & below);
      kept[to_at] = i;
      to_weight[to_at] = weight[i];
    }
    at += __popcll(all);
    equals += __popcll(eq);
  });
  for (int i = tid; i < a.sinks; i += SELECT_THREADS) kept[i] = i, to_weight[i] = weight[i];
  for (int i = tid; i < a.recent; i += SELECT_THREADS) kept[a.budget - a.recent + i] = hi + i, to_weight[a.budget - a.recent + i] = weight[hi + i];
}

// What moves codes from a page's scale to 2^e.  A code that is not 0 is at least 2^-9, so that e is above its scale's exponent less 18: only
// zeros, of which the new scale knows nothing, meet a factor beyond fp32, and it has to stay finite for them.
__device__ __forceinline__ float moved_by(float scale, int e) { return fminf(scale * power(-e), 0x1p127f); }

#define GATHER_THREADS 256
template <int DH>
__global__ __launch_bounds__(GATHER_THREADS) void evict_gather_kernel(QuantCache c, QuantCache o, EvictArgs a) {
  constexpr int WAVES = GATHER_THREADS / 64, VS = DH / WAVES;          // values: a lane per entry, VS elements per wave
  constexpr int CH = DH / 16, KSTEPS = PAGE * CH / GATHER_THREADS;     // keys: 16 bytes a lane
  __shared__ size_t from[PAGE];                                        // block of the source page and head
  __shared__ int slot_of[PAGE];
  __shared__ float scales[PAGE][2];
  __shared__ float tops[WAVES][2];
  __shared__ __align__(16) unsigned char vt[DH][PAGE];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int h = blockIdx.y, s = blockIdx.z, e0 = blockIdx.x * PAGE;
  const int given = c.len[s], len = given > c.max_pages * PAGE ? 0 : max(given, 0), n = min(min(len, a.budget) - e0, PAGE);
  if (n <= 0) return;
  const int page = o.table[(size_t)s * o.table_ld + blockIdx.x];
  if ((unsigned)page >= (unsigned)o.n_pages) return;
  if (tid < PAGE) {
    int id = -1, e = 0;
    if (tid < n) {
      e = a.kept[((size_t)s * c.n_kv_heads + h) * a.budget + e0 + tid];
      id = c.table[(size_t)s * c.table_ld + e / PAGE];
    }
    const bool there = (unsigned)id < (unsigned)c.n_pages;
    const size_t at = (size_t)(there ? id : 0) * c.n_kv_heads + h;
    from[tid] = at * PAGE * DH;
    slot_of[tid] = there ? e % PAGE : -1;                              // no such page: a NaN as the key, 0 as the value
    scales[tid][0] = there ? c.scale[at * 2] : 1.f;
    scales[tid][1] = there ? c.scale[at * 2 + 1] : 1.f;
  }
  __syncthreads();
  u32x4 k[KSTEPS];
  unsigned char v[VS];
  float top[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < KSTEPS; ++i) {
    const int t = (i * GATHER_THREADS + tid) / CH, ch = tid % CH;
    k[i] = u32x4{0u, 0u, 0u, 0u};
    if (t < n) {
      if (slot_of[t] >= 0) k[i] = *reinterpret_cast<const u32x4*>(c.k + from[t] + slot_of[t] * DH + ch * 16);
      else k[i] = u32x4{0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
    }
    float m = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      m = fmaxf(m, fmaxf(fabsf(__builtin_amdgcn_cvt_f32_fp8((int)k[i][x], 0)), fabsf(__builtin_amdgcn_cvt_f32_fp8((int)k[i][x], 1))));
      m = fmaxf(m, fmaxf(fabsf(__builtin_amdgcn_cvt_f32_fp8((int)k[i][x], 2)), fabsf(__builtin_amdgcn_cvt_f32_fp8((int)k[i][x], 3))));
    }
    if (t < n) top[0] = fmaxf(top[0], m * scales[t][0]);
  }
  {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < VS; ++i) {
      v[i] = lane < n && slot_of[lane] >= 0 ? c.v[from[lane] + (w * VS + i) * PAGE + slot_of[lane]] : (unsigned char)0;
      m = fmaxf(m, fabsf(__builtin_amdgcn_cvt_f32_fp8((int)v[i], 0)));
    }
    top[1] = m * scales[lane][1];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    top[i] = wave_max(top[i]);
    if (lane == 0) tops[w][i] = top[i];
  }
  __syncthreads();
  int e[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float m = 0.f;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) m = fmaxf(m, tops[x][i]);
    e[i] = page_exponent(m);
  }
  const size_t block = ((size_t)page * o.n_kv_heads + h) * PAGE * DH;
#pragma unroll
  for (int i = 0; i < KSTEPS; ++i) {
    const int t = (i * GATHER_THREADS + tid) / CH, ch = tid % CH;
    if (t >= n) continue;
    const float by = moved_by(scales[t][0], e[0]);
    u32x4 x;
#pragma unroll
    for (int y = 0; y < 4; ++y) x[y] = moved4(k[i][y], by);
    *reinterpret_cast<u32x4*>(o.k + block + t * DH + ch * 16) = x;
  }
  const float by = moved_by(scales[lane][1], e[1]);
#pragma unroll
  for (int i = 0; i < VS; ++i)
    vt[w * VS + i][lane] = (unsigned char)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8((int)v[i], 0) * by, 0.f, 0, false);
  __syncthreads();
  const int words = (n + 3) / 4;
  for (int i = tid; i < DH * words; i += GATHER_THREADS) {
    const int d = i / words, x = i % words;
    uint8_t* p = o.v + block + d * PAGE + x * 4;
    if (x * 4 + 4 <= n) *reinterpret_cast<unsigned*>(p) = *reinterpret_cast<const unsigned*>(&vt[d][x * 4]);
    else
      for (int b = 0; b < n - x * 4; ++b) p[b] = vt[d][x * 4 + b];
  }
  if (tid < 2) o.scale[((size_t)page * o.n_kv_heads + h) * 2 + tid] = power(tid ? e[1] : e[0]);
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
// Splits go by the part's 256 compute units, not by what spec_init finds: workspaces and the order of sums follow from a call's arguments alone.
#define CUS 256
// most pages that rows of one tile can see, of `rows_seen` neighbouring entries
static int most_pages(const QuantCache& c, int rows_seen, int window, int sinks) {
  if (!window) return c.max_pages;
  const long long n = ((long long)window + rows_seen) / PAGE + 2 + (sinks + PAGE - 1) / PAGE;
  return (int)(n < c.max_pages ? n : c.max_pages);
}
// Tiles of `tile` rows: as many as there can be, and as many as there are where sequences have the same number of rows.
static long long most_tiles(const QuantCache& c, bool ragged, int n_rows, int G, int tile) {
  const long long each = ((long long)(n_rows / c.n_seqs) * G + tile - 1) / tile;
  return ragged ? ((long long)n_rows * G + (long long)c.n_seqs * (tile - 1)) / tile : c.n_seqs * each;
}
static long long mean_tiles(const QuantCache& c, int n_rows, int G, int tile) {
  return (long long)c.n_seqs * ((((long long)n_rows * G + c.n_seqs - 1) / c.n_seqs + tile - 1) / tile);
}
// Kernel and split of an attention, by the rows of a sequence in the mean, tiles and pages (us, back to back; 64 heads over 8 unless said).
//   two tiles of 16 rows share a wave's codes where one each would be more than 12 waves a CU, one page a wave (one tile | two):
//     64 rows of heads behind 1000 entries  11.1 | 13.5      8 sequences, 64 rows behind 4096   39.8 | 27.2      1, 64 behind 8192  20.3 | 18.9
//   from 160 rows on, and 8 waves a CU, pages pass through LDS (registers | LDS):
//     256 rows behind 1000   22.1 | 25.8 and 32 heads over 4  11.7 | 20.4      8 sequences, 256 behind 4096   70.0 | 57.0
//   parts of a sequence so that every CU has a workgroup (one a CU | two):
//     8 sequences, 64 rows behind 4096   27.0 | 28.6      64 rows behind 8192   18.9 | 23.9      windows of 8 requests   18.7 | 22.2
//     against it  64 rows behind 131072   76.9 | 71.3
// One launch (and a merge) takes all sequences, or where they may differ two of them those of more than SHORT rows of a KV head and the others.
// The host does not know which there are: rows of heads have to be so many that a launch with nothing to do counts for little.  As many rows as
// sequences, or so few more that none is long beside single ones, are taken for single tokens; fewer may be a prompt among sequences that rest.
// One | two:
//     a prompt of 2048 tokens and 31 single ones behind 8192   325 | 186      a prompt of 300 and 16 single ones behind 4000   145 | 93
//     512 behind 3584 and the same 31   275 | 193      a prompt of 2048 and 4 windows of 8 behind 32768   877 | 169
//     a prompt of 300 behind 16384 and 1000 single ones behind 512   620 | 462
//     against it  256 behind 768 and 63 single ones behind 2048   63 | 80      8 times 64 behind 2048   56 | 63      64 windows of 8   129 | 134
//     2048 windows of 2 behind 512   758 | 770      512 single tokens behind 2048 (were they not left out)   395 | 407      2048 behind 512   615 | 696
#define SHORT 160
struct AttendPass {
  int row_tiles;    // of 16 rows in a wave; 0: many rows
  int row_waves;    // waves of a workgroup that have rows of their own; the others take other pages of theirs
  int splits;
  long long tiles;
  int above, upto, per, tiled;
  size_t part_rows;
};
struct AttendPlan {
  AttendPass pass[2];
  int n;
};
static AttendPlan attend_plan(const QuantCache& c, bool ragged, int n_rows, int n_heads, int window, int sinks) {
  AttendPlan p;
  const int G = n_heads / c.n_kv_heads;
  const long long total = (long long)n_rows * G, rows = (total + c.n_seqs - 1) / c.n_seqs;      // of a sequence, in the mean
  const long long waves = mean_tiles(c, n_rows, G, 16) * c.n_kv_heads * most_pages(c, (int)(rows / G) + 1, window, sinks);
  const long long more = total - (long long)c.n_seqs * G;                                       // than a row each
  const bool mixed = ragged && c.n_seqs > 1 && G <= SHORT && total > 2048 && (more < 0 || more > SHORT) && waves > 8ll * CUS;
  p.n = mixed ? 2 : 1;
  for (int i = 0; i < p.n; ++i) {
    AttendPass& x = p.pass[i];
    const bool many = mixed ? i == 0 : rows > SHORT && waves > 8ll * CUS;
    x.row_tiles = many ? 0 : mixed || (rows > 16 && waves > 12ll * CUS) ? 2 : 1;
    x.row_waves = mixed ? 0 : rows > 64 ? 4 : rows > 32 ? 2 : 1;
    x.above = mixed && many ? SHORT : 0, x.upto = mixed && !many ? SHORT : INT_MAX, x.per = mixed && !many ? SHORT / G : 0;
    // rows of a workgroup, the most tiles there can be, and how many there will be about: a row of every sequence is not the long ones'
    const int tile = many ? MANY_ROWS : 16 * x.row_tiles * max(x.row_waves, 1);
    x.tiles = !mixed ? most_tiles(c, ragged, n_rows, G, tile) : many ? total / (MANY_ROWS / 2) : c.n_seqs + min((long long)c.n_seqs, total / 129);
    const long long about = !mixed ? mean_tiles(c, n_rows, G, tile) : many ? max(1ll, (total - (long long)c.n_seqs * G + tile - 1) / tile) : c.n_seqs;
    const long long groups = about * c.n_kv_heads, pages = most_pages(c, (tile + G - 1) / G, window, sinks), phases = FEW_WAVES / max(x.row_waves, 1);
    const long long most = many ? pages / 8 : (pages + phases - 1) / phases;
    const long long want = many ? CUS / groups : (CUS + groups - 1) / groups;
    x.splits = (int)max(1ll, min(min(want, most), (long long)MERGE_PARTS));
    // parts of a mixed call's long sequences are for as many tiles as there will be about, so that they stay below 256 * MANY_ROWS rows whatever
    // the call's rows are; tiles beyond, where other sequences have none, are not split
    x.tiled = mixed && many && x.splits > 1 ? (int)min(about, x.tiles) : 0;
    x.part_rows = x.tiled ? (size_t)x.tiled * c.n_kv_heads * MANY_ROWS : (size_t)(x.per ? (long long)c.n_seqs * x.per : n_rows) * n_heads;
  }
  return p;
}
size_t attend_quant_work_bytes(const QuantCache& c, bool ragged, int n_rows, int n_heads, int window, int sinks) {
  const AttendPlan p = attend_plan(c, ragged, n_rows, n_heads, window, sinks);
  size_t most = 0;                                     // passes run one behind the other
  for (int i = 0; i < p.n; ++i)
    if (p.pass[i].splits > 1) most = std::max(most, p.pass[i].splits * p.pass[i].part_rows * (c.head_dim + 2) * sizeof(float));
  return most;
}
template <int DH>
static hipError_t launch_attend(const QuantCache& c, const AttendArgs& a, const AttendPass& p, hipStream_t st) {
  const unsigned groups = (unsigned)((p.tiled ? p.tiled * (p.splits - 1) + p.tiles : p.tiles * p.splits) * c.n_kv_heads);
  if (p.row_tiles == 1) attend_few_kernel<DH, 1><<<groups, FEW_WAVES * 64, 0, st>>>(c, a);
  else if (p.row_tiles == 2) attend_few_kernel<DH, 2><<<groups, FEW_WAVES * 64, 0, st>>>(c, a);
  else attend_many_kernel<DH><<<groups, MANY_WAVES * 64, 0, st>>>(c, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  // four waves a row from 17 parts on, unless rows alone fill the chip
  if (p.splits > 16 && a.part_rows <= (1u << 16)) attend_merge_kernel<DH, 4><<<(unsigned)a.part_rows, MERGE_WAVES * 64, 0, st>>>(c, a);
  else attend_merge_kernel<DH, 1><<<(unsigned)((a.part_rows + MERGE_WAVES - 1) / MERGE_WAVES), MERGE_WAVES * 64, 0, st>>>(c, a);
  return hipGetLastError();
}
hipError_t launch_attend_quant(const QuantCache& c, AttendArgs a, void* work, hipStream_t st) {
  const AttendPlan p = attend_plan(c, a.rows != nullptr, a.n_rows, a.n_heads, a.window, a.sinks);
  a.G = a.n_heads / c.n_kv_heads;
  a.part = (float*)work;
  for (int i = 0; i < p.n; ++i) {
    const AttendPass& x = p.pass[i];
    a.splits = x.splits, a.row_waves = x.row_waves, a.above = x.above, a.upto = x.upto, a.per = x.per, a.tiled = x.tiled, a.part_rows = x.part_rows;
    a.part_ml = (float2*)(a.part + x.splits * x.part_rows * c.head_dim);
    const hipError_t e = c.head_dim == 128 ? launch_attend<128>(c, a, x, st) : launch_attend<64>(c, a, x, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
struct WeighPass {
  int row_tiles;    // of 16 rows, in registers; 0: many rows
  int groups;       // workgroups in x, over the slices' number
  int slices;       // of every sequence, or
  int tiles, ids;   // tiles of 64 rows in one, and how many of them there can be
  int above, upto;  // sequences with more than `above` and at most `upto` rows of a KV head are taken
};
struct WeighPlan {
  WeighPass pass[2];
  int n, pages;     // most that are seen
  size_t parts;     // rows of 64 * pages
};
// As for the attention two passes where sequences may differ and rows of heads are many, those of more than 64 of them and the others, and
// slices that follow a sequence's rows (one pass, and the same number of slices for all, | two):
//     a prompt of 2048 tokens and 31 single ones behind 8192   386 | 132      256 behind 768 and 63 single ones behind 2048   274 | 96
//     512 behind 3584 and the same 31   137 | 109      a prompt of 2048 and 4 windows of 8 behind 32768   374 | 156
//     a prompt of 300 behind 16384 and 1000 single ones behind 512   14680 | 1157
//     a prompt of 400 behind 4000 among 511 sequences that rest   4552 | 80
//     against it  64 windows of 8 behind 4096   79 | 94      2048 windows of 2 behind 512   244 | 498: workgroups that look for long sequences
//     512 single tokens behind 2048   236 | 278      2048 behind 512   237 | 382, left here, as a prompt of as many rows as sequences would take ms
static WeighPlan weigh_plan(const QuantCache& c, bool ragged, int n_rows, int n_heads, int window, int sinks) {
  WeighPlan p;
  const int G = n_heads / c.n_kv_heads, M = (n_rows + c.n_seqs - 1) / c.n_seqs;
  const long long total = (long long)n_rows * G, rows = (long long)M * G, lines = (long long)c.n_seqs * c.n_kv_heads;
  p.pages = most_pages(c, ragged ? n_rows : M, window, sinks);
  const int fours = (p.pages + WEIGH_WAVES - 1) / WEIGH_WAVES;
  // of long sequences, of 64 rows in all of them, and of slices: 16 tiles or more each, and at most 64 more than there are sequences
  const long long longs = min((long long)c.n_seqs, total / 65), all = total / 64 + longs, tiles = max(16ll, (all + 63) / 64), ids = all / tiles + longs;
  const bool mixed = ragged && c.n_seqs > 1 && c.n_seqs <= 32768 && total > 2048 && ids * c.n_kv_heads * p.pages <= 1 << 20;      // 256 MiB
  p.n = mixed ? 2 : 1, p.parts = 0;
  for (int i = 0; i < p.n; ++i) {
    WeighPass& x = p.pass[i];
    x = {0, fours, 1, 0, 0, 0, INT_MAX};
    if (mixed ? i == 1 : rows <= 64) {
      x.row_tiles = rows <= 16 ? 1 : rows <= 32 || rows > 64 ? 2 : 4;
      x.groups = (int)max(1ll, min((long long)fours, (3ll * CUS + lines - 1) / lines));
      if (mixed) x.upto = 64;
    } else if (mixed) {
      x.tiles = (int)tiles, x.ids = (int)ids, x.above = 64;
      p.parts = ids * c.n_kv_heads;
    } else {
      // many rows: tiles of 64 to so many slices that every CU has four workgroups, each at least 4 tiles (2047 rows of 64 heads over 8, us):
      //   4 slices 192, 8 100, 16 to 32 58 to 65
      // The table's width stands for the length, which the host does not know.  The same rows behind tables of 33 pages 62, 65 95, 129 157,
      // 513 and more 373: columns that are not needed yet are better left out of max_pages.
      x.slices = (int)max(1ll, min(min(4ll * CUS / (lines * fours), (rows + 255) / 256), 64ll));
      if (x.slices > 1) p.parts = x.slices * lines;
    }
  }
  return p;
}
size_t weigh_quant_work_bytes(const QuantCache& c, bool ragged, int n_rows, int n_heads, int window, int sinks) {
  const WeighPlan p = weigh_plan(c, ragged, n_rows, n_heads, window, sinks);
  return p.parts * p.pages * PAGE * sizeof(float);
}
template <int DH>
static hipError_t launch_weigh(const QuantCache& c, const WeighArgs& a, const WeighPass& p, int pages, hipStream_t st) {
  const dim3 grid(p.groups, c.n_kv_heads, c.n_seqs);
  if (p.row_tiles == 1) weigh_few_kernel<DH, 1><<<grid, WEIGH_WAVES * 64, 0, st>>>(c, a);
  else if (p.row_tiles == 2) weigh_few_kernel<DH, 2><<<grid, WEIGH_WAVES * 64, 0, st>>>(c, a);
  else if (p.row_tiles == 4) weigh_few_kernel<DH, 4><<<grid, WEIGH_WAVES * 64, 0, st>>>(c, a);
  else weigh_many_kernel<DH><<<dim3((unsigned)p.groups * p.slices * c.n_kv_heads, p.tiles ? p.ids : c.n_seqs), WEIGH_WAVES * 64, 0, st>>>(c, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (p.slices == 1 && !p.tiles)) return e;
  weigh_add_kernel<<<dim3((pages + 3) / 4, c.n_kv_heads, c.n_seqs), 256, 0, st>>>(c, a);
  return hipGetLastError();
}
hipError_t launch_weigh_quant(const QuantCache& c, WeighArgs a, void* work, hipStream_t st) {
  const WeighPlan p = weigh_plan(c, a.rows != nullptr, a.n_rows, a.n_heads, a.window, a.sinks);
  a.G = a.n_heads / c.n_kv_heads;
  a.part = (float*)work;
  a.pages = p.pages;
  a.by_group = ((1ull << 38) + a.G - 1) / a.G;           // r * G < 2^38: (r * this) >> 38 is r / G
  for (int i = 0; i < p.n; ++i) {
    const WeighPass& x = p.pass[i];
    a.slices = x.slices, a.tiles = x.tiles, a.ids = x.ids, a.above = x.above, a.upto = x.upto;
    const hipError_t e = c.head_dim == 128 ? launch_weigh<128>(c, a, x, p.pages, st) : launch_weigh<64>(c, a, x, p.pages, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
hipError_t launch_evict_quant(const QuantCache& c, const QuantCache& to, const EvictArgs& a, hipStream_t st) {
  evict_select_kernel<<<dim3(c.n_kv_heads, c.n_seqs), SELECT_THREADS, 0, st>>>(c, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((a.budget + PAGE - 1) / PAGE, c.n_kv_heads, c.n_seqs);
  if (c.head_dim == 128) evict_gather_kernel<128><<<grid, GATHER_THREADS, 0, st>>>(c, to, a);
  else evict_gather_kernel<64><<<grid, GATHER_THREADS, 0, st>>>(c, to, a);
  return hipGetLastError();
}
