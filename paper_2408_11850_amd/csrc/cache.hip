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
#include <limits.h>

#include "spec_internal.h"

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4a;
typedef __attribute__((ext_vector_type(8), aligned(2))) unsigned short bf16x8a;

#define PAGE SPEC_PAGE_TOKENS
#define LEAST_EXP (-100)            // scales are 2^e, e >= this
#define FINITE_MAX 0x1p120f         // keys and values from here on count as infinite: their scales would leave fp32's range
#define NONE (-3.0e38f)             // running maximum of a row that has seen nothing; scores below it cannot be told from it
#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f

// eight codes times a power of two, exactly
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

// ---- which rows a workgroup works on --------------------------------------------------------------------------------------
struct Span {
  int s;          // sequence, or -1: none
  int t;          // which of its tiles
  int row, M;     // its first row and their number
};
// Tile `id` of all sequences' tiles one behind the other; tiles(M) of a sequence with M rows.  Called by whole waves.
template <class Tiles>
__device__ __forceinline__ Span find_span(const QuantCache& c, const int* rows, int n_rows, int id, Tiles tiles) {
  if (!rows) {
    const int M = n_rows / c.n_seqs, per = tiles(M), s = id / per;
    return s < c.n_seqs ? Span{s, id - s * per, s * M, M} : Span{-1, 0, 0, 0};
  }
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < c.n_seqs; base += 64) {
    const int s = base + lane;
    int first = 0, M = 0;
    if (s < c.n_seqs) {                       // whatever the numbers are, the rows are rows of the call
      first = min(max(rows[s], 0), n_rows);
      M = min(max(rows[s + 1], first), n_rows) - first;
    }
    const int mine = M > 0 ? tiles(M) : 0;
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      upto += lane >= d ? o : 0;
    }
    const int all = __shfl(upto, 63);
    if (id - before < all) {
      const int at = __ffsll((long long)__ballot(upto > id - before)) - 1;
      return Span{base + at, id - before - __shfl(upto - mine, at), __shfl(first, at), __shfl(M, at)};
    }
    before += all;
  }
  return Span{-1, 0, 0, 0};
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

// ---- append ---------------------------------------------------------------------------------------------------------------
// A workgroup takes the entries of a call that fall into one page: keys and values of a KV head, or eight query heads.  The
// angles' cosines and sines are made once per workgroup, in revolutions in 64 bits up to the reduction.
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
  const int len = min(max(c.len[sp.s], 0), INT_MAX / 2), first = len - sp.M, capacity = c.max_pages * PAGE;
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
      float sn, cs;
      sincospif(2.f * (float)(rev - rint(rev)), &sn, &cs);
      turn[t][p] = make_float2(cs, sn);
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
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top[i] = fmaxf(top[i], __shfl_xor(top[i], d));
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
struct PageData {
  u32x4 k[4][DH / 64], v[DH / 16];
  float ks, vs;
  bool there;
};

template <int DH>
__device__ __forceinline__ void load_keys(const QuantCache& c, PageData<DH>& p, int page, int h, int lane) {
  const int r = lane & 15, g = lane >> 4;
  p.there = (unsigned)page < (unsigned)c.n_pages;
  const size_t at = (size_t)(p.there ? page : 0) * c.n_kv_heads + h;
  const uint8_t* k = c.k + at * PAGE * DH + (16 * (r >> 2) + (r & 3)) * DH + g * 16;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int f = 0; f < DH / 64; ++f) p.k[t][f] = *reinterpret_cast<const u32x4*>(k + 4 * t * DH + f * 64);
  p.ks = p.there ? c.scale[at * 2] : __uint_as_float(0x7fc00000u);       // no such page: whoever sees it becomes NaN
}
template <int DH>
__device__ __forceinline__ void load_values(const QuantCache& c, PageData<DH>& p, int page, int h, int lane) {
  const bool there = (unsigned)page < (unsigned)c.n_pages;
  const size_t at = (size_t)(there ? page : 0) * c.n_kv_heads + h;
  const uint8_t* v = c.v + at * PAGE * DH + (lane & 15) * PAGE + (lane >> 4) * 16;
#pragma unroll
  for (int d = 0; d < DH / 16; ++d) p.v[d] = *reinterpret_cast<const u32x4*>(v + d * 16 * PAGE);
  p.vs = c.scale[at * 2 + 1];
}

#define FEW_WAVES 4
template <int DH, int RT>
__global__ __launch_bounds__(FEW_WAVES * 64, 2) void attend_few_kernel(QuantCache c, AttendArgs a) {
  constexpr int KS = DH / 32, DT = DH / 16;
  __shared__ f32x4 osh[FEW_WAVES - 1][RT][DT][64];
  __shared__ float2 mlsh[FEW_WAVES][RT][16];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const unsigned parts = c.n_kv_heads * a.splits, part = blockIdx.x % parts;
  const int h = part % c.n_kv_heads, split = part / c.n_kv_heads;
  const int G = a.G, tile_rows = 16 * RT * a.row_waves;
  Span sp = find_span(c, a.rows, a.n_rows, blockIdx.x / parts, [&](int M) { return (M * G + tile_rows - 1) / tile_rows; });
  sp.s = __builtin_amdgcn_readfirstlane(sp.s);
  if (sp.s < 0) return;
  sp.t = __builtin_amdgcn_readfirstlane(sp.t), sp.row = __builtin_amdgcn_readfirstlane(sp.row), sp.M = __builtin_amdgcn_readfirstlane(sp.M);
  const int capacity = c.max_pages * PAGE, given = c.len[sp.s];
  const bool beyond = given > capacity;              // nothing is read; the rows become NaN
  const int len = max(given, 0), first = len - sp.M, R = sp.M * G;
  const int phases = FEW_WAVES / a.row_waves, rw = w % a.row_waves, phase = w / a.row_waves;
  const int wg0 = sp.t * tile_rows, wg_last = min(wg0 + tile_rows, R) - 1;
  const int r0 = wg0 + rw * 16 * RT, r_last = min(r0 + 16 * RT, R) - 1;      // r_last < r0: a wave without rows
  const Seen seen = seen_pages(first + wg0 / G, beyond ? -1 : first + wg_last / G, a.window, a.sinks);
  const int per = (seen.n + a.splits - 1) / a.splits, i0 = split * per, i1 = min(i0 + per, seen.n);
  const int see_all = first + r0 / G;                                         // entries up to here are seen by all of the wave's rows
  const int low_all = a.window ? first + max(r_last, 0) / G - a.window + 1 : 0;

  int pos[RT];
  bool valid[RT];
  size_t row_at[RT];                                                          // (row, head), counted through
  bf16x8 qf[RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + rt * 16 + r16;
    valid[rt] = r < R;
    const int tok = valid[rt] ? r / G : 0, hq = h * G + (valid[rt] ? r % G : 0);
    pos[rt] = valid[rt] ? first + tok : -1;
    row_at[rt] = (size_t)(sp.row + tok) * a.n_heads + hq;
    const bf16* q = a.q + (size_t)(sp.row + tok) * a.ldq + (size_t)hq * DH + g * 16;
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      u32x4 x = {0u, 0u, 0u, 0u};
      if (valid[rt]) x = *reinterpret_cast<const u32x4*>(q + (j >> 1) * 64 + (j & 1) * 8);
      qf[rt][j] = __builtin_bit_cast(bf16x8, x);
    }
  }
  float m[RT], l[RT];
  f32x4 o[RT][DT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = NONE, l[rt] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[rt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int* table = c.table + (size_t)sp.s * c.table_ld;
  PageData<DH> p;
  int i = i0 + phase;
  if (i < i1) {
    const int id = table[seen.page(i)];
    load_keys<DH>(c, p, id, h, lane);
    load_values<DH>(c, p, id, h, lane);
  }
  for (; i < i1; i += phases) {
    const int e0 = seen.page(i) * PAGE;
    const bool more = i + phases < i1;
    const int next = more ? table[seen.page(i + phases)] : 0;
    const float by = p.ks * a.scale_log2e;
    const bool there = p.there;
    f32x4 s[RT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const bf16x8 kf = to_bf16x8(p.k[t][j >> 1][(j & 1) * 2], p.k[t][j >> 1][(j & 1) * 2 + 1], 1.f);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rt][j], s[rt][t], 0, 0, 0);
      }
    }
    if (more) load_keys<DH>(c, p, next, h, lane);
    const bool all = e0 + PAGE - 1 <= see_all && (!a.window || e0 >= low_all || e0 + PAGE <= a.sinks);
    bf16x8 pf[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          float v = s[rt][t][x] * by;
          if (!all) {
            const int e = e0 + 16 * g + 4 * t + x;
            const bool see = e <= pos[rt] && (!a.window || e > pos[rt] - a.window || e < a.sinks);
            v = see ? v : -INFINITY;
          }
          s[rt][t][x] = v;
          mx = fmaxf(mx, v);
        }
      const float m_new = fmaxf(m[rt], groups_max(mx));
      const float corr = __builtin_amdgcn_exp2f(m[rt] - m_new);
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float v = __builtin_amdgcn_exp2f(s[rt][t][x] - m_new);
          sum += v;
          pf[rt][t >> 1][(t & 1) * 4 + x] = (__bf16)v;
        }
      l[rt] = l[rt] * corr + sum;
      m[rt] = m_new;
      if (!__all(corr == 1.f)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) o[rt][d] *= corr;
      }
    }
    // entries behind the last one, or of no page, may hold anything: 0 times a NaN would be one
    const int live = there ? min(len - e0, PAGE) - 16 * g : 0;
    if (!there || e0 + PAGE > len) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int n = live - 4 * x;
        const unsigned keep = n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << n * 8) - 1;
#pragma unroll
        for (int d = 0; d < DT; ++d) p.v[d][x] &= keep;
      }
    }
    const float vs = there ? p.vs : 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const bf16x8 vf = to_bf16x8(p.v[d][x * 2], p.v[d][x * 2 + 1], vs);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt][x], o[rt][d], 0, 0, 0);
      }
    if (more) load_values<DH>(c, p, next, h, lane);
  }
  // the waves of a row tile together
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] = groups_sum(l[rt]);
    if (g == 0) mlsh[w][rt][r16] = make_float2(m[rt], l[rt]);
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = NONE;
    for (int x = 0; x < phases; ++x) top = fmaxf(top, mlsh[x * a.row_waves + rw][rt][r16].x);
    const float f = __builtin_amdgcn_exp2f(m[rt] - top);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      o[rt][d] *= f;
      if (phase) osh[w - a.row_waves][rt][d][lane] = o[rt][d];
    }
    float sum = 0.f;
    for (int x = 0; x < phases; ++x) {
      const float2 ml = mlsh[x * a.row_waves + rw][rt][r16];
      sum += ml.y * __builtin_amdgcn_exp2f(ml.x - top);
    }
    m[rt] = top, l[rt] = sum;
  }
  __syncthreads();
  if (phase) return;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    for (int x = 1; x < phases; ++x)
#pragma unroll
      for (int d = 0; d < DT; ++d) o[rt][d] += osh[(x - 1) * a.row_waves + rw][rt][d][lane];
    if (!valid[rt]) continue;
    if (beyond) l[rt] = __uint_as_float(0x7fc00000u);
    if (a.splits == 1) {
      const bool empty = pos[rt] < 0;
      const float inv = empty ? 0.f : 1.f / l[rt];
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        bf16 b[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) b[x] = __float2bfloat16(o[rt][d][x] * inv);
        *reinterpret_cast<uint2*>(a.out + row_at[rt] * DH + d * 16 + g * 4) = *reinterpret_cast<const uint2*>(b);
      }
      if (a.lse && g == 0) a.lse[row_at[rt]] = empty ? -INFINITY : (m[rt] + __log2f(l[rt])) * LN2;
    } else {
      const size_t at = (size_t)split * a.n_rows * a.n_heads + row_at[rt];
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(a.part + at * DH + d * 16 + g * 4) = o[rt][d];
      if (g == 0) a.part_ml[at] = make_float2(pos[rt] < 0 ? -INFINITY : m[rt], l[rt]);      // -inf: the row sees nothing
    }
  }
}

// Parts of a row's attention together; a lane has 4 elements, 64 * 4 / DH rows share a wave.
template <int DH>
__global__ __launch_bounds__(256) void attend_merge_kernel(QuantCache c, AttendArgs a) {
  constexpr int LANES = DH / 4;
  const size_t all = (size_t)a.n_rows * a.n_heads, at = (size_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (at >= all) return;
  const int row = (int)(at / a.n_heads);
  // rows behind the last sequence have no parts and stay as they are; a row in front of the first entry sees nothing
  if (a.rows && (row >= a.rows[c.n_seqs] || row < a.rows[0])) return;
  float top = -INFINITY;
  for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.part_ml[s * all + at].x);
  const bool empty = top == -INFINITY;
  float sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const int lane = threadIdx.x % LANES;
  for (int s = 0; s < a.splits; ++s) {
    const float2 ml = a.part_ml[s * all + at];
    const float f = __builtin_amdgcn_exp2f(ml.x - top);
    sum += ml.y * f;
    if (ml.y != 0.f) o += *reinterpret_cast<const f32x4*>(a.part + (s * all + at) * DH + lane * 4) * f;
  }
  const float inv = empty ? 0.f : 1.f / sum;
  bf16 b[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) b[x] = __float2bfloat16(o[x] * inv);
  *reinterpret_cast<uint2*>(a.out + at * DH + lane * 4) = *reinterpret_cast<const uint2*>(b);
  if (a.lse && lane == 0) a.lse[at] = empty ? -INFINITY : (top + __log2f(sum)) * LN2;
}

// ---- attention weight of the entries ------------------------------------------------------------------------------------------
// w[entry] = sum over the rows and heads of a group of exp(score - lse).  A wave holds the 64 keys of a page as operands and goes
// over row tiles of 16; a lane's scores belong to one row, so sums over rows stay in registers until the end.
#define WEIGH_WAVES 4
template <int DH, bool SHARE>
__global__ __launch_bounds__(WEIGH_WAVES * 64, 2) void weigh_kernel(QuantCache c, WeighArgs a) {
  constexpr int KS = DH / 32;
  __shared__ float wsh[WEIGH_WAVES][PAGE];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.y, s = blockIdx.z, G = a.G;
  int row = s * (a.n_rows / c.n_seqs), M = a.n_rows / c.n_seqs;
  if (a.rows) {
    row = min(max(a.rows[s], 0), a.n_rows);
    M = min(max(a.rows[s + 1], row), a.n_rows) - row;
  }
  const int len = max(c.len[s], 0), first = len - M, R = M * G;
  if (M == 0 || len > c.max_pages * PAGE) return;
  const Seen seen = seen_pages(first, len - 1, a.window, a.sinks);
  const int i = SHARE ? blockIdx.x : blockIdx.x * WEIGH_WAVES + w;
  if (i >= seen.n) return;                                     // SHARE: the whole workgroup
  const int page = seen.page(i), e0 = page * PAGE;
  PageData<DH> p;
  load_keys<DH>(c, p, c.table[(size_t)s * c.table_ld + page], h, lane);
  bf16x8 kf[4][KS];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int j = 0; j < KS; ++j) kf[t][j] = to_bf16x8(p.k[t][j >> 1][(j & 1) * 2], p.k[t][j >> 1][(j & 1) * 2 + 1], 1.f);
  const float by = p.ks * a.scale_log2e;
  f32x4 sum[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  // the first row that sees the page's first entry
  const int tile0 = max(0, e0 - first) * G / 16, tiles = (R + 15) / 16;
  for (int tile = tile0 + (SHARE ? w : 0); tile < tiles; tile += SHARE ? WEIGH_WAVES : 1) {
    const int r = tile * 16 + r16;
    const bool valid = r < R;
    const int tok = valid ? r / G : 0, hq = h * G + (valid ? r % G : 0);
    const int pos = valid ? first + tok : -1;
    const bf16* q = a.q + (size_t)(row + tok) * a.ldq + (size_t)hq * DH + g * 16;
    const float lse = valid ? a.lse[(size_t)(row + tok) * a.n_heads + hq] * LOG2E : 0.f;
    bf16x8 qf[KS];
#pragma unroll
    for (int j = 0; j < KS; ++j) qf[j] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(q + (j >> 1) * 64 + (j & 1) * 8));
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][j], qf[j], x, 0, 0, 0);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int e = e0 + 16 * g + 4 * t + y;
        const bool see = e <= pos && (!a.window || e > pos - a.window || e < a.sinks);
        sum[t][y] += see ? __builtin_amdgcn_exp2f(fmaf(x[y], by, -lse)) : 0.f;
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      float v = sum[t][y];
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) v += __shfl_xor(v, d);
      if (r16 == 0) wsh[w][16 * g + 4 * t + y] = v;
    }
  if (SHARE) {
    __syncthreads();
    if (w) return;
  }
  const int e = e0 + lane;
  if (e >= len) return;
  float v = wsh[w][lane];
  if (SHARE)
    for (int x = 1; x < WEIGH_WAVES; ++x) v += wsh[x][lane];
  float* to = a.weight + ((size_t)s * c.n_kv_heads + h) * a.ldw + e;
  *to = e < first ? *to + v : v;                               // an entry of these rows begins here
}

// ---- eviction -----------------------------------------------------------------------------------------------------------------
// One workgroup per sequence and head finds the weight of the last entry that is kept, eight bits of an ordered key at a time, and
// lists the entries that are kept in their order; then a workgroup per page of 64 of them moves their codes.
#define SELECT_THREADS 1024
#define SELECT_WAVES (SELECT_THREADS / 64)

// larger weights have larger keys, equal ones the same; a NaN counts as the least
__device__ __forceinline__ unsigned weight_key(float w) {
  const unsigned b = __float_as_uint(w + 0.f);
  return w != w ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(SELECT_THREADS) void evict_select_kernel(QuantCache c, EvictArgs a) {
  __shared__ int hist[256];
  __shared__ int found[2];
  __shared__ int counts[SELECT_WAVES][2];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
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
  unsigned key = 0, mask = 0;                                   // the bits of the last kept key that are known
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += SELECT_THREADS) {
        const unsigned k = weight_key(weight[i]);
        if ((k & mask) == key) atomicAdd(&hist[k >> shift & 255u], 1);
      }
      __syncthreads();
      if (w == 0) {                                             // 4 digits a lane, from the largest down
        int four[4], mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) four[j] = hist[255 - (lane * 4 + j)], mine += four[j];
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int o = __shfl_up(upto, d);
          upto += lane >= d ? o : 0;
        }
        int before = upto - mine;
        if (before < want && upto >= want) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (before < want && before + four[j] >= want) found[0] = 255 - (lane * 4 + j), found[1] = want - before;
            before += four[j];
          }
        }
      }
      __syncthreads();
      key |= (unsigned)found[0] << shift;
      mask |= 255u << shift;
      want = found[1];                                          // so many of those with this digit
      __syncthreads();
    }
  } else key = 0xffffffffu;                                     // above every key (a NaN's bits do not reach it)
  // every wave has a stretch of entries; larger keys are kept, and the first `want` equal ones
  const int stretch = ((hi - lo + SELECT_WAVES - 1) / SELECT_WAVES + 63) / 64 * 64;
  const int from = lo + w * stretch, to = min(from + stretch, hi);
  int more = 0, equal = 0;
  for (int i = from; i < to; i += 64) {
    const unsigned k = i + lane < to ? weight_key(weight[i + lane]) : 0u;
    more += __popcll(__ballot(i + lane < to && k > key));
    equal += __popcll(__ballot(i + lane < to && k == key));
  }
  if (lane == 0) counts[w][0] = more, counts[w][1] = equal;
  __syncthreads();
  int at = a.sinks, equals = 0;                                 // places and equal ones in front of this wave
  for (int x = 0; x < w; ++x) {
    const int take = min(counts[x][1], max(want - equals, 0));
    at += counts[x][0] + take;
    equals += counts[x][1];
  }
  const unsigned long long below = (1ull << lane) - 1;
  for (int i = from; i < to; i += 64) {
    const bool in = i + lane < to;
    const float v = in ? weight[i + lane] : 0.f;
    const unsigned k = weight_key(v);
    const unsigned long long eq = __ballot(in && k == key);
    const bool keep = in && (k > key || (k == key && equals + __popcll(eq & below) < want));
    const unsigned long long all = __ballot(keep);
    if (keep) {
      const int to_at = at + __popcll(all & below);
      kept[to_at] = i + lane;
      to_weight[to_at] = v;
    }
    at += __popcll(all);
    equals += __popcll(eq);
  }
  for (int i = tid; i < a.sinks; i += SELECT_THREADS) kept[i] = i, to_weight[i] = weight[i];
  for (int i = tid; i < a.recent; i += SELECT_THREADS) kept[a.budget - a.recent + i] = hi + i, to_weight[a.budget - a.recent + i] = weight[hi + i];
}

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
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top[i] = fmaxf(top[i], __shfl_xor(top[i], d));
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
    const float by = scales[t][0] * power(-e[0]);
    u32x4 x;
#pragma unroll
    for (int y = 0; y < 4; ++y) x[y] = moved4(k[i][y], by);
    *reinterpret_cast<u32x4*>(o.k + block + t * DH + ch * 16) = x;
  }
  const float by = scales[lane][1] * power(-e[1]);
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
// most pages that rows of one tile can see, of `rows_seen` neighbouring entries
static int most_pages(const QuantCache& c, int rows_seen, int window, int sinks) {
  if (!window) return c.max_pages;
  const long long n = ((long long)window + rows_seen) / PAGE + 2 + (sinks + PAGE - 1) / PAGE;
  return (int)(n < c.max_pages ? n : c.max_pages);
}
static long long most_tiles(const QuantCache& c, bool ragged, int n_rows, int G, int tile) {
  if (ragged) return (long long)n_rows * G / tile + c.n_seqs;
  return (long long)c.n_seqs * (((long long)(n_rows / c.n_seqs) * G + tile - 1) / tile);
}
struct AttendPlan {
  int row_tiles;    // of 16 rows per wave
  int row_waves;    // waves of a workgroup that have rows of their own; the others take other pages of theirs
  int splits;
  long long tiles;
};
static AttendPlan attend_plan(const QuantCache& c, bool ragged, int n_rows, int n_heads, int window, int sinks) {
  AttendPlan p;
  const int G = n_heads / c.n_kv_heads, rows = (n_rows / c.n_seqs + 1) * G;
  p.row_tiles = rows > 16 ? 2 : 1;
  p.row_waves = rows > 64 ? 4 : rows > 32 ? 2 : 1;
  const int tile = 16 * p.row_tiles * p.row_waves;
  p.tiles = most_tiles(c, ragged, n_rows, G, tile);
  const int pages = most_pages(c, (tile + G - 1) / G, window, sinks), phases = FEW_WAVES / p.row_waves;
  const long long groups = p.tiles * c.n_kv_heads, want = 4ll * spec_num_cu();
  p.splits = (int)max(1ll, min(min((want + groups - 1) / groups, (long long)((pages + phases - 1) / phases)), 64ll));
  return p;
}
size_t attend_quant_work_bytes(const QuantCache& c, bool ragged, int n_rows, int n_heads, int window, int sinks) {
  const AttendPlan p = attend_plan(c, ragged, n_rows, n_heads, window, sinks);
  return p.splits == 1 ? 0 : (size_t)p.splits * n_rows * n_heads * (c.head_dim + 2) * sizeof(float);
}
template <int DH, int RT>
static void launch_few(const QuantCache& c, const AttendArgs& a, long long tiles, hipStream_t st) {
  attend_few_kernel<DH, RT><<<(unsigned)(tiles * c.n_kv_heads * a.splits), FEW_WAVES * 64, 0, st>>>(c, a);
}
hipError_t launch_attend_quant(const QuantCache& c, AttendArgs a, void* work, hipStream_t st) {
  const AttendPlan p = attend_plan(c, a.rows != nullptr, a.n_rows, a.n_heads, a.window, a.sinks);
  a.G = a.n_heads / c.n_kv_heads;
  a.splits = p.splits, a.row_waves = p.row_waves;
  const size_t all = (size_t)a.n_rows * a.n_heads;
  a.part = (float*)work;
  a.part_ml = (float2*)(a.part + (size_t)p.splits * all * c.head_dim);
  if (c.head_dim == 128) {
    if (p.row_tiles == 1) launch_few<128, 1>(c, a, p.tiles, st);
    else launch_few<128, 2>(c, a, p.tiles, st);
  } else {
    if (p.row_tiles == 1) launch_few<64, 1>(c, a, p.tiles, st);
    else launch_few<64, 2>(c, a, p.tiles, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const size_t per = 256 / (c.head_dim / 4);
  if (c.head_dim == 128) attend_merge_kernel<128><<<(unsigned)((all + per - 1) / per), 256, 0, st>>>(c, a);
  else attend_merge_kernel<64><<<(unsigned)((all + per - 1) / per), 256, 0, st>>>(c, a);
  return hipGetLastError();
}
hipError_t launch_weigh_quant(const QuantCache& c, WeighArgs a, hipStream_t st) {
  a.G = a.n_heads / c.n_kv_heads;
  const long long rows = (long long)(a.n_rows / c.n_seqs + 1) * a.G;
  const int pages = a.rows || !a.window ? c.max_pages : most_pages(c, a.n_rows / c.n_seqs, a.window, a.sinks);
  if (rows > 64) {
    const dim3 grid(pages, c.n_kv_heads, c.n_seqs);
    if (c.head_dim == 128) weigh_kernel<128, true><<<grid, WEIGH_WAVES * 64, 0, st>>>(c, a);
    else weigh_kernel<64, true><<<grid, WEIGH_WAVES * 64, 0, st>>>(c, a);
  } else {
    const dim3 grid((pages + WEIGH_WAVES - 1) / WEIGH_WAVES, c.n_kv_heads, c.n_seqs);
    if (c.head_dim == 128) weigh_kernel<128, false><<<grid, WEIGH_WAVES * 64, 0, st>>>(c, a);
    else weigh_kernel<64, false><<<grid, WEIGH_WAVES * 64, 0, st>>>(c, a);
  }
  return hipGetLastError();
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
