// 8-bit operands for gfx950: residual add + RMS norm to e4m3, rows to e4m3, weights to e4m3 and into operand order, and the
// products of the two.
//
// e4m3 is the OCP type (largest value 448).  A row has one fp32 scale per 128 columns, a weight matrix one per 128 x 128
// block, so a product is  y[m][n] = sum_b sx[b][m] sw[n / 128][b] sum_{k in block b} x[m][k] w[n][k]:  the inner sum is one
// v_mfma_f32_16x16x128_f8f6f4 (K = 128, fp32 sums of exact products), the outer one an fp32 multiply-add per result.
#include <type_traits>

#include "spec_internal.h"

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4a;
typedef __attribute__((ext_vector_type(8), aligned(2))) unsigned short bf16x8a;

#define E4M3_MAX 448.0f
#define FP8_LEAST 0x1p-100f       // blocks whose largest magnitude is below take this one's scale: no scale is 0 or denormal
#define FP8_EXACT 0x1p-90f        // a residual of a division by a smaller scale may need bits that fp32 does not have

// ---- rows -----------------------------------------------------------------------------------------------------------
// A lane takes 8 neighbouring columns, so that 16 lanes share a block of 128 and its largest magnitude is four rotations
// inside a row of lanes.

template <int CTRL>
__device__ __forceinline__ float dpp_ror(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, dpp_ror<0x128>(v));
  v = fmaxf(v, dpp_ror<0x124>(v));
  v = fmaxf(v, dpp_ror<0x122>(v));
  return fmaxf(v, dpp_ror<0x121>(v));
}
// every step adds the same two numbers in both lanes of a pair: all lanes hold the same bits
__device__ __forceinline__ float wave64_sum(float v) {
  v += dpp_ror<0x128>(v);
  v += dpp_ror<0x124>(v);
  v += dpp_ror<0x122>(v);
  v += dpp_ror<0x121>(v);
  return groups_sum(v);
}

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
// v becomes what is stored
template <int T>
__device__ __forceinline__ void store8(void* p, size_t at, float (&v)[8]) {
  if (T == SPEC_F32) {
    f32x4a* s = reinterpret_cast<f32x4a*>(reinterpret_cast<float*>(p) + at);
    s[0] = f32x4a{v[0], v[1], v[2], v[3]};
    s[1] = f32x4a{v[4], v[5], v[6], v[7]};
  } else {
    bf16x8a a;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bf16 b = __float2bfloat16(v[i]);
      a[i] = *reinterpret_cast<const unsigned short*>(&b);
      v[i] = __uint_as_float((unsigned)a[i] << 16);
    }
    *reinterpret_cast<bf16x8a*>(reinterpret_cast<unsigned short*>(p) + at) = a;
  }
}

// v / by, correctly rounded, for inv = 1 / by correctly rounded (Markstein): t is off by less than two steps, v - t * by is exact in a
// multiply-add as long as no bit of it is below 2^-149 (for quotients that a code can tell from 0, from 2^-10 on: by >= 2^-93), and
// its share of the quotient added once rounds to the nearest.  Infinities give NaN.  Scales and codes are thus
// those of IEEE divisions (a zero loses its sign).  Products with rounded reciprocals instead take 61 of 63 million normed values for the other neighbour
// of a border, divisions 41, a single rounding of the exact quotients 37; they cost 17.5 us where such products took 16.6
// (2047 rows of 11008 bf16), 1 to 2 % at other sizes.
__device__ __forceinline__ float quotient(float v, float by, float inv) {
  const float t = v * inv;
  return fmaf(fmaf(-t, by, v), inv, t);
}
__device__ __forceinline__ float scale_of(float top) { return quotient(fmaxf(top, FP8_LEAST), E4M3_MAX, 1.0f / E4M3_MAX); }

// 8 columns of a block of 128 to e4m3; the 16 lanes of the block share its scale.  A NaN is none of the magnitudes and stays
// NaN; an infinite one makes the scale NaN, and the block with it.
__device__ __forceinline__ float block_scale(const float (&v)[8]) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(v[i]));
  return scale_of(row16_max(a));
}
__device__ __forceinline__ uint2 to_e4m3(const float (&v)[8], float scale) {
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = v[i];
  if (__any(scale < FP8_EXACT)) {                  // both by a power of two, exactly; the test costs 0.5 to 0.9 % of 4096 x 8192 and the like
    const float up = scale < FP8_EXACT ? 0x1p64f : 1.0f;
    scale *= up;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] *= up;
  }
  const float inv = 1.0f / scale;                  // the quotients reach 448 up to the scale's rounding, which rounds to 448
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = quotient(t[i], scale, inv);
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], hi, true);
  return make_uint2((unsigned)lo, (unsigned)hi);
}

// XT: type of the rows; DT: of what is added first, -1 none; NORM: RMS norm and gain, else the rows as they are.
// A row belongs to `wpr` waves of a workgroup; a chunk is the 512 columns a wave takes at a time, at most G per wave.  The sum of
// squares is formed per chunk and over the chunks in ascending order, so a row's bits do not depend on how it is dealt out.
// Everything stays in registers between one read and one write, so HBM bounds it: 4096 x 8192 bf16 and a bf16 delta, 236 MB, 47 us
// (5.0 TB/s, as a copy), 1023 x 4096 fp32 11.1 us; one row of 8192 takes 3.6, of which the launch is most.
#define ROWS_CHUNK 512
#define ROWS_WAVES_MAX 16
template <int XT, int DT, bool NORM, int G>
__global__ __launch_bounds__(ROWS_WAVES_MAX * 64) void rows_fp8_kernel(void* x, size_t ldx, const void* delta, size_t ldd,
                                                                      const bf16* gain, float eps, int M, int d, int wpr,
                                                                      uint8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ float sums[ROWS_WAVES_MAX * G];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int rpw = (blockDim.x >> 6) / wpr;          // rows of a workgroup
  const int rw = w / wpr, wr = w % wpr, row = blockIdx.x * rpw + rw;
  const bool live = row < M;
  const int chunks = (d + ROWS_CHUNK - 1) / ROWS_CHUNK;
  float v[G][8];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int col = (g * wpr + wr) * ROWS_CHUNK + lane * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[g][i] = 0.f;
    if (live && col < d) load8<XT>(x, row * ldx + col, v[g]);
  }
  if (DT >= 0) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int col = (g * wpr + wr) * ROWS_CHUNK + lane * 8;
      if (live && col < d) {
        float a[8];
        load8<DT>(delta, row * ldd + col, a);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[g][i] += a[i];
        store8<XT>(x, row * ldx + col, v[g]);
      }
    }
  }
  if (NORM) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int chunk = g * wpr + wr;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[g][i] * v[g][i];
      s = wave64_sum(s);
      if (chunk < chunks && lane == 0) sums[rw * chunks + chunk] = s;
    }
    __syncthreads();
    float tot = 0.f;
    for (int c = 0; c < chunks; ++c) tot += sums[rw * chunks + c];
    const float inv = 1.0f / sqrtf(tot / (float)d + eps);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int col = (g * wpr + wr) * ROWS_CHUNK + lane * 8;
      if (col < d) {
        float b[8];
        load8<SPEC_BF16>(gain, col, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[g][i] = v[g][i] * inv * b[i];
      }
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int col = (g * wpr + wr) * ROWS_CHUNK + lane * 8;
    const float s = block_scale(v[g]);
    if (live && col < d) {
      *reinterpret_cast<uint2*>(q + (size_t)row * d + col) = to_e4m3(v[g], s);
      if ((lane & 15) == 0) scale[(size_t)(col >> 7) * M + row] = s;
    }
  }
}

template <int XT, int DT, bool NORM>
static hipError_t launch_rows(void* x, size_t ldx, const void* delta, size_t ldd, const bf16* gain, float eps, int M, int d,
                              uint8_t* q, float* scale, hipStream_t st) {
  const int chunks = (d + ROWS_CHUNK - 1) / ROWS_CHUNK;
  const int G = chunks <= ROWS_WAVES_MAX ? 1 : 4;
  const int wpr = (chunks + G - 1) / G;
  const int rpw = wpr >= 4 ? 1 : 4 / wpr;
  const dim3 grid((M + rpw - 1) / rpw), block(rpw * wpr * 64);
  if (G == 1) rows_fp8_kernel<XT, DT, NORM, 1><<<grid, block, 0, st>>>(x, ldx, delta, ldd, gain, eps, M, d, wpr, q, scale);
  else rows_fp8_kernel<XT, DT, NORM, 4><<<grid, block, 0, st>>>(x, ldx, delta, ldd, gain, eps, M, d, wpr, q, scale);
  return hipGetLastError();
}

hipError_t launch_add_norm_fp8(void* h, int h_type, size_t ldh, const void* delta, int delta_type, size_t ldd, const bf16* gain,
                               float eps, int M, int d, uint8_t* q, float* scale, hipStream_t st) {
#define NORM_CASE(XT, DT) return launch_rows<XT, DT, true>(h, ldh, delta, ldd, gain, eps, M, d, q, scale, st)
  if (h_type == SPEC_F32) {
    if (!delta) NORM_CASE(SPEC_F32, -1);
    if (delta_type == SPEC_F32) NORM_CASE(SPEC_F32, SPEC_F32);
    NORM_CASE(SPEC_F32, SPEC_BF16);
  }
  if (!delta) NORM_CASE(SPEC_BF16, -1);
  if (delta_type == SPEC_F32) NORM_CASE(SPEC_BF16, SPEC_F32);
  NORM_CASE(SPEC_BF16, SPEC_BF16);
#undef NORM_CASE
}
hipError_t launch_quant_fp8(const void* x, int x_type, size_t ldx, int M, int K, uint8_t* q, float* scale, hipStream_t st) {
  void* p = const_cast<void*>(x);                   // only read without a delta
  if (x_type == SPEC_F32) return launch_rows<SPEC_F32, -1, false>(p, ldx, nullptr, 0, nullptr, 0.f, M, K, q, scale, st);
  return launch_rows<SPEC_BF16, -1, false>(p, ldx, nullptr, 0, nullptr, 0.f, M, K, q, scale, st);
}

// ---- weights --------------------------------------------------------------------------------------------------------
// One workgroup of 256 threads per block of 128 x 128: 16 lanes a row of it, 16 rows at a time.
__global__ __launch_bounds__(256) void quant_weight_kernel(const bf16* __restrict__ w, int N, int K, uint8_t* __restrict__ q,
                                                           float* __restrict__ scale) {
  __shared__ float top[16];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, col = blockIdx.x * 128 + c * 8;
  float v[8][8], a = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int n = blockIdx.y * 128 + j * 16 + r;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] = 0.f;
    if (n < N && col < K) load8<SPEC_BF16>(w, (size_t)n * K + col, v[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(v[j][i]));
  }
  a = row16_max(a);
  if (c == 0) top[r] = a;
  __syncthreads();
  a = row16_max(top[c]);
  const float s = scale_of(a);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int n = blockIdx.y * 128 + j * 16 + r;
    if (n < N && col < K) *reinterpret_cast<uint2*>(q + (size_t)n * K + col) = to_e4m3(v[j], s);
  }
  if (threadIdx.x == 0) scale[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}
hipError_t launch_quant_weight_fp8(const bf16* w, int N, int K, uint8_t* q, float* scale, hipStream_t st) {
  quant_weight_kernel<<<dim3((K + 127) / 128, (N + 127) / 128), 256, 0, st>>>(w, N, K, q, scale);
  return hipGetLastError();
}

// Packed order: panel p (16 weight rows), block b of 128 columns: 2 KiB in operand order, 16 bytes per lane, the 16-byte pieces
// 0-3 of the rows and then the pieces 4-7: lane (c, g) = (lane % 16, lane / 16) has piece g, then g + 4, of row c; zeros behind K.
// A load of a wave is 1 KiB in one run, whole lines of it.  Once per model: 8192 x 28672 takes 76 us, 6.2 TB/s read and written.  The scales come along per panel, [panel][block], so that matrices
// can be concatenated and interleaved by panels.
__global__ __launch_bounds__(128) void pack_weight_fp8_kernel(const uint8_t* __restrict__ src, const float* __restrict__ src_scale,
                                                              int N, int K, int panel_start, int panel_step,
                                                              uint8_t* __restrict__ dst, float* __restrict__ dst_scale) {
  const int b = blockIdx.x, panel = blockIdx.y, KB = gridDim.x;
  const int r = threadIdx.x >> 3, i = threadIdx.x & 7, k = b * 128 + i * 16;
  const size_t to = (size_t)(panel_start + panel * panel_step) * KB + b;
  u32x4 v = {0, 0, 0, 0};
  typedef __attribute__((ext_vector_type(4), aligned(1))) unsigned u32x4b;
  if (k < K) v = *reinterpret_cast<const u32x4b*>(src + (size_t)(panel * 16 + r) * K + k);
  *reinterpret_cast<u32x4*>(dst + to * 2048 + (i >> 2) * 1024 + ((i & 3) * 16 + r) * 16) = v;
  if (threadIdx.x == 0) dst_scale[to] = src_scale[(size_t)(panel / 8) * KB + b];
}
hipError_t launch_pack_weight_fp8(void* dst, float* dst_scale, const void* src, const float* src_scale, int N, int K,
                                  int panel_start, int panel_step, hipStream_t st) {
  pack_weight_fp8_kernel<<<dim3((K + 127) / 128, N / 16), 128, 0, st>>>((const uint8_t*)src, src_scale, N, K, panel_start,
                                                                        panel_step, (uint8_t*)dst, dst_scale);
  return hipGetLastError();
}

// ---- products -------------------------------------------------------------------------------------------------------
// Operand order: lane (c, g) = (lane % 16, lane / 16) holds 32 bytes of row c; which 32 of the block's 128 does not matter as
// long as both operands agree: the 16-byte pieces g and g + 4.  A result's lane (c, g) holds column c (a token), rows 4 g ..
// 4 g + 3 (outputs): the scale of a token is one value per lane, that of a panel one per wave.
//
// Two ways to the inner sum of a block.  v_mfma_f32_16x16x128_f8f6f4 takes e4m3 as it is, at twice the rate of bf16; but inside
// each group of 8 products it drops what lies about 2^-14 below the largest of them: 1.5e-5 of the result (2-norm, normal
// operands), nothing beside a rounding to bf16 (2e-3), too much for an fp32 result.  So fp32 results, and decode-time ones of
// either type (which wait for the weights anyway), turn e4m3 into bf16 (exact) and use v_mfma_f32_16x16x32_bf16 (1e-8 there).
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
enum { FP8_STORE = 0, FP8_STORE16 = 1, FP8_SWIGLU = 2 };

struct Operand { u32x4 lo, hi; };
__device__ __forceinline__ f32x4 block_product(const Operand& w, const Operand& x) {
  const i32x8 a = {(int)w.lo[0], (int)w.lo[1], (int)w.lo[2], (int)w.lo[3], (int)w.hi[0], (int)w.hi[1], (int)w.hi[2], (int)w.hi[3]};
  const i32x8 b = {(int)x.lo[0], (int)x.lo[1], (int)x.lo[2], (int)x.lo[3], (int)x.hi[0], (int)x.hi[1], (int)x.hi[2], (int)x.hi[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}
struct Half16 { bf16x8 part[2]; };               // 16 columns of a lane
__device__ __forceinline__ bf16x8 to_bf16(unsigned a, unsigned b) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], t[0], t[1]};
}
__device__ __forceinline__ Half16 to_bf16(u32x4 v) { return Half16{{to_bf16(v[0], v[1]), to_bf16(v[2], v[3])}}; }
__device__ __forceinline__ f32x4 half_product(const Half16& w, const Half16& x, f32x4 d) {
#pragma unroll
  for (int i = 0; i < 2; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.part[i], x.part[i], d, 0, 0, 0);
  return d;
}
struct Operand16 { Half16 lo, hi; };
__device__ __forceinline__ f32x4 block_product(const Operand16& w, const Operand16& x) {
  return half_product(w.hi, x.hi, half_product(w.lo, x.lo, f32x4{0.f, 0.f, 0.f, 0.f}));
}
__device__ __forceinline__ f32x4 scaled_add(f32x4 d, float s, f32x4 acc) {
#pragma unroll
  for (int r = 0; r < 4; ++r) acc[r] = fmaf(d[r], s, acc[r]);
  return acc;
}

template <typename T> __device__ __forceinline__ T as_operand(const Operand& o);
template <> __device__ __forceinline__ Operand as_operand<Operand>(const Operand& o) { return o; }
template <> __device__ __forceinline__ Operand16 as_operand<Operand16>(const Operand& o) { return Operand16{to_bf16(o.lo), to_bf16(o.hi)}; }

struct Fp8Args {
  const uint8_t* x;      // [M][K]
  const float* xs;       // [KB][M]
  const uint8_t* w;      // packed
  const float* ws;       // [NT][KB]
  void* out;             // STORE: fp32 [M][N];  STORE16: bf16 [M][N];  SWIGLU: bf16 [M][N / 2]
  int M, N, K, KB, NT;
};

// outputs 4 g .. 4 g + 3 of a panel (SWIGLU: v, up = the gate and the up panel) for one token
template <int EPI>
__device__ __forceinline__ void fp8_store(const Fp8Args& a, int m, int panel, int g, f32x4 v, f32x4 up) {
  if (EPI == FP8_STORE) {
    *reinterpret_cast<f32x4*>((float*)a.out + (size_t)m * a.N + panel * 16 + g * 4) = v;
    return;
  }
  bf16 o[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) o[r] = __float2bfloat16(EPI == FP8_SWIGLU ? v[r] / (1.0f + __expf(-v[r])) * up[r] : v[r]);
  const size_t at = EPI == FP8_SWIGLU ? (size_t)m * (a.N / 2) + (panel >> 1) * 16 : (size_t)m * a.N + panel * 16;
  *reinterpret_cast<uint2*>((bf16*)a.out + at + g * 4) = *reinterpret_cast<const uint2*>(o);
}

// Up to 32 tokens: bound by the stream of the weights.  A workgroup of 4 waves owns a contiguous range of units (RP panels, SWIGLU:
// gate and up panels); wave w takes its quarter of a unit's blocks of 128, through a ring of D register stages of one block
// that runs on from unit to unit.  All ring loads are buffer loads whose range check turns "past the end" (blocks, rows, columns)
// into zeros without traffic: unconditional, so that a stage waits for its own loads only.  The two halves of a block (pieces 0-3
// and 4-7) are summed apart, and the waves' sums are added through LDS in a fixed order: a row's sums depend on K alone.
//
// What counts next to HBM is the address unit, which takes a load line by line.  Weights come 8 whole lines to a load.  Rows of x
// are 128 bytes apart by K: of 16 of them a load brings half a line each.  PAIR (up to 8 tokens) loads 8 whole ones instead, lanes
// c < 8 with the first half of a block and c >= 8 with the second, as one operand: of the product with the weights' first half
// the columns 0-7 count, of the other one the columns 8-15.
// 8192 x 28672 over 7 rows: 38 us, 6.2 TB/s of weights (a plain read reaches 6.7); 2048 x 2048 over one 3.6 in a graph.
#define SK_WAVES 4
#define SK_SKIP 0x7f000000u            // beyond every buffer
template <bool PAIR, int MT, int EPI, int RP, int D, int OCC>
__global__ __launch_bounds__(SK_WAVES * 64, OCC) void fp8_skinny_kernel(Fp8Args a, int per, int rem) {
  static_assert(!PAIR || MT == 1, "one tile of 8 tokens");
  __shared__ f32x4 red[2][SK_WAVES][RP][MT][64];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int b = blockIdx.x, u0 = b * per + min(b, rem), u1 = u0 + per + (b < rem ? 1 : 0);
  const int s0 = w * a.KB / SK_WAVES, ns = (w + 1) * a.KB / SK_WAVES - s0;
  const int rounds = ns > D ? (ns + D - 1) / D : 1;
  const unsigned pbytes = (unsigned)a.KB * 2048u, wlane = lane * 16u;
  const __amdgpu_buffer_rsrc_t xr =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.x), 0, (unsigned)a.M * (unsigned)a.K, 0x00020000);
  const __amdgpu_buffer_rsrc_t sr =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(a.xs), 0, (unsigned)a.KB * (unsigned)a.M * 4u, 0x00020000);
  const __amdgpu_buffer_rsrc_t pr =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(a.ws), 0, (unsigned)a.NT * (unsigned)a.KB * 4u, 0x00020000);
  constexpr int XL = PAIR ? 1 : 2;                       // loads of x per tile
  const int xcol = g * 16 + (PAIR ? (c >> 3) * 64 : 0);  // this lane's first column of a block
  unsigned xoff[MT], soff[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = PAIR ? c & 7 : t * 16 + c;
    xoff[t] = m < a.M ? (unsigned)m * (unsigned)a.K + xcol : SK_SKIP;
    soff[t] = m < a.M ? m * 4u : SK_SKIP;
  }
  u32x4 wq[D][RP][2], xq[D][MT][XL];
  float xs[D][MT], ws[RP], wn[RP];     // lane l of ws, wn: the panel's scale in stage l of this round, of the next one
  // no scale where the wave has no block: the next one, of another wave or panel, may be a NaN, which the zeros there would become
  auto load_ws = [&](int u, int r, float (&to)[RP]) {
    const unsigned mine = lane < min(D, ns - r * D) ? lane * 4u : SK_SKIP;
#pragma unroll
    for (int p = 0; p < RP; ++p) {
      const unsigned at = (unsigned)min(u * RP + p, a.NT - 1) * (unsigned)a.KB + min(s0 + r * D, a.KB - 1);
      to[p] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(pr, mine, at * 4u, 0));
    }
  };
  // stage s: block r * D + s of the wave's share of unit u.  What is not there is skipped by the lanes' offsets; the scalar ones
  // stay inside the buffers (a range check subtracts them from the size).
  auto load = [&](int s, int u, int r) {
    const int i = r * D + s, blk = min(s0 + i, a.KB - 1);
    const bool on = i < ns && u < u1;
#pragma unroll
    for (int p = 0; p < RP; ++p) {
      const int panel = min(u * RP + p, a.NT - 1);
      const unsigned at = wlane | (on && u * RP + p < a.NT ? 0u : SK_SKIP);
      const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>(a.w) + (size_t)panel * pbytes, 0, pbytes, 0x00020000);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        wq[s][p][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wr, at + h * 1024, blk * 2048, 2));
    }
    const unsigned skip = on ? 0u : SK_SKIP;
    const int left = a.K - blk * 128 - xcol;         // columns behind this lane's first one
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const unsigned at = skip | xoff[t];
#pragma unroll
      for (int h = 0; h < XL; ++h)
        xq[s][t][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xr, left > h * 64 ? at + h * 64 : SK_SKIP, blk * 128, 0));
      xs[s][t] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, skip | soff[t], blk * a.M * 4, 0));
    }
  };
#pragma unroll
  for (int s = 0; s < D; ++s) load(s, u0, 0);
  load_ws(u0, 0, ws);
  f32x4 acc[RP][MT][2];
#pragma unroll
  for (int p = 0; p < RP; ++p)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[p][t][0] = acc[p][t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  int buf = 0;
#pragma unroll 1
  for (int u = u0, r = 0; u < u1;) {
    const bool last = r + 1 == rounds;
    const int nu = last ? u + 1 : u, nr = last ? 0 : r + 1;
    load_ws(nu, nr, wn);
#pragma unroll
    for (int s = 0; s < D; ++s) {
      Half16 x16[MT][XL];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int h = 0; h < XL; ++h) x16[t][h] = to_bf16(xq[s][t][h]);
#pragma unroll
      for (int p = 0; p < RP; ++p) {
        const float wscale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ws[p]), s));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const Half16 w16 = to_bf16(wq[s][p][h]);
#pragma unroll
          for (int t = 0; t < MT; ++t)
            acc[p][t][h] = scaled_add(half_product(w16, x16[t][PAIR ? 0 : h], f32x4{0.f, 0.f, 0.f, 0.f}), xs[s][t] * wscale, acc[p][t][h]);
        }
      }
      load(s, nu, nr);
      __builtin_amdgcn_sched_barrier(0);              // stage by stage: the ring holds most registers
    }
    if (last) {
#pragma unroll
      for (int p = 0; p < RP; ++p)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          f32x4 v = acc[p][t][0] + acc[p][t][1];
          if (PAIR) v = c < 8 ? acc[p][t][0] : acc[p][t][1];      // a token's halves meet when they are read
          red[buf][w][p][t][lane] = v;
          acc[p][t][0] = acc[p][t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      // two buffers: nobody writes this one again before everybody has passed the next unit's barrier
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      // a wave adds and stores a tile at a time (SWIGLU: those of a pair of panels)
      constexpr int UP = EPI == FP8_SWIGLU ? 2 : 1, JOBS = RP / UP * MT;
      for (int job = (w + u) & (SK_WAVES - 1); job < JOBS; job += SK_WAVES) {
        const int t = job % MT, p0 = job / MT * UP, m = t * 16 + c;
        f32x4 sum[2];
#pragma unroll
        for (int q = 0; q < UP; ++q) {
          f32x4 e[SK_WAVES];
#pragma unroll
          for (int i = 0; i < SK_WAVES; ++i) {
            e[i] = red[buf][i][p0 + q][t][lane];
            if (PAIR) e[i] += red[buf][i][p0 + q][t][lane ^ 8];
          }
          sum[q] = (e[0] + e[1]) + (e[2] + e[3]);
        }
        if (m < a.M && u * RP + p0 < a.NT) fp8_store<EPI>(a, m, u * RP + p0, g, sum[0], sum[UP - 1]);
      }
      buf ^= 1;
    }
    u = nu, r = nr;
#pragma unroll
    for (int p = 0; p < RP; ++p) ws[p] = wn[p];
  }
}

// From 33 tokens on: BMT tiles of 16 tokens x BNP panels per workgroup of WM x WN waves, a block of 128 columns per stage, ST stages.
// Both operands, and their scales, go global -> LDS without a stop in registers: rows of x as 128 bytes, piece i of row r at
// place i ^ (r % 8), so that no read of a fragment meets a bank twice; weights as they are packed.  The loads are inline asm
// (they write no register), so that the compiler, which would wait for all of them before any LDS read, leaves the waiting to
// the explicit counts; everything else is ordinary code.
// Buffer range checks turn rows behind M, panels behind NT and columns behind K into zeros.
#define DMA_SKIP 0x7f000000u          // beyond every buffer
__device__ __forceinline__ u32x4 dma_rsrc(const void* base, unsigned bytes) {
  const uint64_t p = (uint64_t)base;
  return u32x4{(unsigned)p, (unsigned)(p >> 32) & 0xffffu, bytes, 0x00020000u};
}
// A wave's 64 x 16 (4) bytes to consecutive LDS addresses from `lds` on.  The s_nop keeps a scalar register that a vector
// instruction has just written five cycles from its use as an offset: the compiler looks for that outside asm only.
__device__ __forceinline__ void dma16(unsigned lds, u32x4 rsrc, unsigned voff, unsigned soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(soff)));
}
__device__ __forceinline__ void dma4(unsigned lds, u32x4 rsrc, unsigned voff, unsigned soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, %3 offen lds"
               ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(soff)));
}

template <int BMT, int BNP, int WM, int WN, int ST>
struct DenseShape {
  static constexpr int WAVES = WM * WN, MT = BMT / WM, NP = BNP / WN;
  static constexpr int XB = BMT * 2048, WB = BNP * 2048, SB = 2048;   // a stage: rows, panels, scales (of tokens, then of panels)
  static constexpr int STAGE = XB + WB + SB, BYTES = ST * STAGE;
  static constexpr int JOBS = (BMT + BNP) * 2 / WAVES + 1;            // loads of a wave per stage: operands, one of scales
  static_assert((BMT + BNP) * 2 % WAVES == 0 && BMT * 2 % WAVES == 0, "even shares");
  static_assert(BMT / 4 + 1 <= WAVES && BMT * 64 + BNP * 4 <= SB && BNP <= 64, "a load of scales per wave");
};

template <int EPI, int BMT, int BNP, int WM, int WN, int ST>
__global__ __launch_bounds__(WM * WN * 64) void fp8_dense_kernel(Fp8Args a, int TM, int TN, int chunk) {
  typedef DenseShape<BMT, BNP, WM, WN, ST> S;
  extern __shared__ u32x4 fp8_lds[];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  // XCD x (workgroups are dealt round-robin) takes the tiles [x chunk, (x + 1) chunk), row-major in groups of 4 columns
  const int j = blockIdx.x >> 3, tile = (blockIdx.x & 7) * chunk + j;
  if (j >= chunk || tile >= TM * TN) return;
  const int grp = tile / (TM * 4), idx = tile % (TM * 4), gw = min(4, TN - grp * 4);
  const int tm = idx / gw, tn = grp * 4 + idx % gw;
  const int m0 = tm * BMT * 16, p0 = tn * BNP;
  const int rows = min(BMT * 16, a.M - m0), panels = min(BNP, a.NT - p0);
  const u32x4 xr = dma_rsrc(a.x + (size_t)m0 * a.K, (unsigned)rows * (unsigned)a.K);
  const u32x4 wr = dma_rsrc(a.w + (size_t)p0 * a.KB * 2048, (unsigned)panels * (unsigned)a.KB * 2048u);
  const u32x4 sxr = dma_rsrc(a.xs + m0, (unsigned)((a.KB - 1) * (size_t)a.M + rows) * 4u);
  const u32x4 swr = dma_rsrc(a.ws + (size_t)p0 * a.KB, (unsigned)panels * (unsigned)a.KB * 4u);
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) u32x4*)fp8_lds;
  constexpr int XJ = BMT * 2 / S::WAVES, WJ = BNP * 2 / S::WAVES;
  // x: job i covers rows 8 i .. 8 i + 7, lane l row l / 8, place l % 8
  unsigned xoff[XJ], woff[WJ], soff;
  const int xpiece = (lane & 7) ^ (lane >> 3);
#pragma unroll
  for (int i = 0; i < XJ; ++i) {
    const int r = (w * XJ + i) * 8 + (lane >> 3);
    xoff[i] = r < rows ? (unsigned)r * (unsigned)a.K + xpiece * 16 : DMA_SKIP;
  }
#pragma unroll
  for (int i = 0; i < WJ; ++i) {
    const int job = w * WJ + i;
    woff[i] = (unsigned)(job >> 1) * (unsigned)a.KB * 2048u + (job & 1) * 1024 + lane * 16;
  }
  const bool tokens = w < BMT / 4;              // this wave's load of scales: of 64 tokens, or of the panels
  soff = tokens ? (w * 64 + lane < rows ? (w * 64 + lane) * 4u : DMA_SKIP)
                : (lane < panels ? (unsigned)lane * (unsigned)a.KB * 4u : DMA_SKIP);
  const bool tail = (a.K & 127) != 0;
  const unsigned cut = tail && xpiece * 16 >= (a.K & 127) ? DMA_SKIP : 0u;      // for the last block
  const u32x4 sr = tokens ? sxr : swr;
  const unsigned slds = S::XB + S::WB + (tokens ? w * 256 : BMT * 64), sstep = tokens ? (unsigned)a.M * 4u : 4u;
  // Load q of a wave for block b into a slot.  Past the last block the buffers have no bytes: zeros into a slot that nobody reads,
  // without traffic, so that one count of loads in flight serves every iteration.
  auto issue = [&](unsigned b, bool there, unsigned last, unsigned base, int q) {
    const unsigned o = there ? b : 0u;
    auto cut_off = [&](u32x4 r) { return u32x4{r[0], r[1], there ? r[2] : 0u, r[3]}; };
    if (q < XJ) dma16(base + (w * XJ + q) * 1024, cut_off(xr), xoff[q] | last, o * 128);
    else if (q < XJ + WJ) dma16(base + S::XB + (w * WJ + q - XJ) * 1024, cut_off(wr), woff[q - XJ], o * 2048);
    else dma4(base + slds, cut_off(sr), soff, o * sstep);
  };
  const int wm = w / WN, wn = w % WN;
  f32x4 acc[S::NP][S::MT];
#pragma unroll
  for (int p = 0; p < S::NP; ++p)
#pragma unroll
    for (int t = 0; t < S::MT; ++t) acc[p][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < ST - 1; ++s)
#pragma unroll
    for (int q = 0; q < S::JOBS; ++q) issue(s, s < a.KB, s == a.KB - 1 ? cut : 0u, lds0 + s * S::STAGE, q);
  int slot = 0, next = ST - 1;
  for (int i = 0; i < a.KB; ++i) {
    // this wave's loads of block i have landed, then everybody's; everybody is past reading the slot that is filled next
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((ST - 2) * S::JOBS) : "memory");
    const int ahead = i + ST - 1;
    const bool more = ahead < a.KB;
    const unsigned cut_now = ahead == a.KB - 1 ? cut : 0u, to = lds0 + next * S::STAGE;
    const u32x4* xl = fp8_lds + slot * (S::STAGE / 16) + wm * S::MT * 128 + c * 8;
    const u32x4* wl = fp8_lds + slot * (S::STAGE / 16) + S::XB / 16 + wn * S::NP * 128 + lane;
    const float* sl = reinterpret_cast<const float*>(fp8_lds + slot * (S::STAGE / 16) + (S::XB + S::WB) / 16);
    const int lo = g ^ (c & 7), hi = lo ^ 4;
    typedef typename std::conditional<EPI == FP8_STORE, Operand16, Operand>::type Op;
    // Panel p is multiplied while the fragments of the next ones come from LDS and the sums of the one before are scaled and added.
    // What the first products need is read first.  The loads go between panels (a wave that issues them back to back waits for the
    // address unit meanwhile), early in the step if it is all the time they have.
    constexpr int AHEAD = S::NP > 4 ? 2 : 1, SPREAD = ST == 2 ? (S::NP + 1) / 2 : S::NP;
    Op xf[S::MT], wf[AHEAD + 1];
    float xs[S::MT], ws[S::NP];
    f32x4 d[2][S::MT];
    wf[0] = as_operand<Op>(Operand{wl[0], wl[64]});
#pragma unroll
    for (int t = 0; t < S::MT; ++t) {
      xf[t] = as_operand<Op>(Operand{xl[t * 128 + lo], xl[t * 128 + hi]});
      __builtin_amdgcn_sched_barrier(0);                   // LDS reads stay in this order
    }
#pragma unroll
    for (int p = 1; p < AHEAD; ++p) wf[p] = as_operand<Op>(Operand{wl[p * 128], wl[p * 128 + 64]});
#pragma unroll
    for (int t = 0; t < S::MT; ++t) xs[t] = sl[(wm * S::MT + t) * 16 + c];
#pragma unroll
    for (int p = 0; p < S::NP; ++p) ws[p] = sl[BMT * 16 + wn * S::NP + p];
#pragma unroll
    for (int p = 0; p <= S::NP; ++p) {
      if (p + AHEAD < S::NP)
        wf[(p + AHEAD) % (AHEAD + 1)] = as_operand<Op>(Operand{wl[(p + AHEAD) * 128], wl[(p + AHEAD) * 128 + 64]});
#pragma unroll
      for (int t = 0; t < S::MT; ++t) {
        if (p < S::NP) d[p & 1][t] = block_product(wf[p % (AHEAD + 1)], xf[t]);
        if (p > 0) acc[p - 1][t] = scaled_add(d[(p - 1) & 1][t], xs[t] * ws[p - 1], acc[p - 1][t]);
      }
      if (p > 0 && p < S::NP && EPI != FP8_STORE) {
#pragma unroll
        for (int t = 0; t < S::MT; ++t) { __builtin_amdgcn_sched_group_barrier(0x8, 1, 0); __builtin_amdgcn_sched_group_barrier(0x2, 5, 0); }
      }
      if (p < SPREAD)
#pragma unroll
        for (int q = p * S::JOBS / SPREAD; q < (p + 1) * S::JOBS / SPREAD; ++q) issue(ahead, more, cut_now, to, q);
      __builtin_amdgcn_sched_barrier(0);
    }
    // its LDS reads are done before this wave meets the next barrier
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    slot = slot + 1 == ST ? 0 : slot + 1;
    next = next + 1 == ST ? 0 : next + 1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // the last loads must not outlive the workgroup's LDS
#pragma unroll
  for (int t = 0; t < S::MT; ++t) {
    const int m = m0 + (wm * S::MT + t) * 16 + c;
    if (m >= a.M) continue;
    constexpr int UP = EPI == FP8_SWIGLU ? 2 : 1;
    static_assert(S::NP % UP == 0, "whole pairs per wave");
#pragma unroll
    for (int p = 0; p < S::NP; p += UP) {
      const int panel = p0 + wn * S::NP + p;
      if (panel + UP <= a.NT) fp8_store<EPI>(a, m, panel, g, acc[p][t], acc[p + UP - 1][t]);
    }
  }
}

template <int EPI, int BMT, int BNP, int WM, int WN, int ST>
static hipError_t launch_dense(const Fp8Args& a, hipStream_t st) {
  typedef DenseShape<BMT, BNP, WM, WN, ST> S;
  const int TM = (a.M + BMT * 16 - 1) / (BMT * 16), TN = (a.NT + BNP - 1) / BNP, chunk = (TM * TN + 7) / 8;
  auto kernel = fp8_dense_kernel<EPI, BMT, BNP, WM, WN, ST>;
  const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::BYTES);
  if (e != hipSuccess) return e;
  kernel<<<chunk * 8, S::WAVES * 64, S::BYTES, st>>>(a, TM, TN, chunk);
  return hipGetLastError();
}

template <int EPI, bool PAIR, int MT, int RP, int D, int OCC, int WGS>
static hipError_t launch_units(const Fp8Args& a, hipStream_t st) {
  const int units = (a.NT + RP - 1) / RP, G = min(units, WGS * spec_num_cu());
  fp8_skinny_kernel<PAIR, MT, EPI, RP, D, OCC><<<G, SK_WAVES * 64, 0, st>>>(a, units / G, units % G);
  return hipGetLastError();
}
// Two panels share what is read of x where that counts (beyond 8 rows; SiLU * up has a pair anyway) and units suffice, four where
// x is as much again (beyond 16); else single panels, more of them in flight (us, RP = 1 | 2 | 4 panels, weights from HBM):
//   7 x 10240 x 8192   19.0 | 21.7        16 x 4096 x 11008  13.5 | 18.7         32 x 4096 x 4096     8.9 | 10.0 | 12.8
//   7 x 8192 x 28672   41.2 | 40.6        16 x 8192 x 8192   17.1 | 16.7         32 x 8192 x 8192    23.7 | 19.4 | 25.5
//                                         16 x 32000 x 8192  56.2 | 50.8         32 x 32000 x 8192   78.5 | 60.1 | 56.2
template <int EPI>
static hipError_t launch_skinny(const Fp8Args& a, hipStream_t st) {
  if (a.M > 16 && a.NT >= 1024) return launch_units<EPI, false, 2, 4, 2, 2, 2>(a, st);
  if constexpr (EPI == FP8_SWIGLU) {
    if (a.M <= 8) return launch_units<EPI, true, 1, 2, 4, 2, 2>(a, st);
    if (a.M <= 16) return launch_units<EPI, false, 1, 2, 4, 2, 2>(a, st);
    return launch_units<EPI, false, 2, 2, 4, 2, 2>(a, st);
  } else {
    if (a.M <= 8) return launch_units<EPI, true, 1, 1, 4, 4, 4>(a, st);
    if (a.M <= 16) return a.NT < 512 ? launch_units<EPI, false, 1, 1, 4, 2, 4>(a, st) : launch_units<EPI, false, 1, 2, 4, 2, 2>(a, st);
    return a.NT < 512 ? launch_units<EPI, false, 2, 1, 4, 2, 4>(a, st) : launch_units<EPI, false, 2, 2, 4, 2, 2>(a, st);
  }
}
// Tile by the time a launch takes (us): rounds of as many workgroups as fit, each a fixed part and a time per block of 128 columns
// that grows with the share of them in use, fitted to 27 shapes of bf16 results (256 x 256 | 256 x 192 | 128 x 256 | 128 x 128 |
// 64 x 64), of which it takes the fastest in 26, else one 1 % behind, and to 17 of fp32 ones (the last three):
//   64 x 4096 x 4096       43 |  38 |  30 | 20.4 | 13.6     1023 x 12288 x 4096   66 |  61 |  74 |  79 | 108
//   256 x 12288 x 4096     60 |  55 |  38 | 26.2 | 32.2     1023 x 8192 x 8192   107 | 101 |  79 |  91 | 139
//   512 x 8192 x 8192     107 | 100 |  64 | 49.5 | 74.6     4095 x 8192 x 8192   248 | 292 | 293 | 346 | 501
// and of few blocks, where the fixed part counts:
//   288 x 1024 x 128     10.2 | 8.4 | 6.7 |  4.7 |  3.1     898 x 4448 x 304    13.5 | 11.4 |  9.6 | 10.2 | 10.7
//   377 x 19616 x 416    16.7 | 14.4 | 12.2 | 14.1 | 17.9   2339 x 26896 x 384  58.9 | 63.9 | 63.0 | 76.1 | 96.0
// Off by more: 519 x 32448 x 22352 takes 256 x 192, 605, where 128 x 256 takes 547; 151 x 19200 x 512 128 x 256, 11.1, where 64 x 64
// takes 9.6.
// 256 x 256 runs at 2.3 to 2.4 PFLOP/s (zeros instead of data: 3.0, so the chip's power is a part of what bounds it); 4 vector instructions
// per MFMA scale and add, and every block passes LDS once per wave that uses it.
int fp8_tile(int M, int NT, int KB, bool exact) {
  static const struct { int tokens, panels, per_cu; float round, step, busy; } T[2][5] = {
      {{256, 16, 1, 3.0f, 1.415f, 0.480f}, {256, 12, 1, 3.0f, 1.274f, 0.339f}, {128, 16, 1, 4.2f, 0.854f, 0.255f}, {128, 8, 1, 3.2f, 0.537f, 0.124f}, {64, 4, 2, 3.2f, 0.304f, 0.151f}},
      {{0, 0, 0, 0.f, 0.f, 0.f}, {0, 0, 0, 0.f, 0.f, 0.f}, {128, 16, 1, 4.4f, 1.525f, 0.315f}, {128, 8, 1, 3.4f, 0.969f, 0.170f}, {64, 4, 2, 2.9f, 0.479f, 0.210f}}};
  int best = 4;
  double best_us = 0.0;
  for (int i = exact ? 2 : 0; i < 5; ++i) {
    const auto& t = T[exact][i];
    const long long tiles = (long long)((M + t.tokens - 1) / t.tokens) * ((NT + t.panels - 1) / t.panels);
    const long long slots = (long long)t.per_cu * spec_num_cu(), rounds = (tiles + slots - 1) / slots;
    const double us = rounds * (t.round + KB * (t.step + t.busy * (double)tiles / ((double)rounds * slots)));
    if (i == (exact ? 2 : 0) || us < best_us) best = i, best_us = us;
  }
  return best;
}
template <int EPI>
static hipError_t launch_fp8(const Fp8Args& a, hipStream_t st) {
  if (a.M <= 32) return launch_skinny<EPI>(a, st);
  const int tile = fp8_tile(a.M, a.NT, a.KB, EPI == FP8_STORE);
  if constexpr (EPI != FP8_STORE) {
    if (tile == 0) return launch_dense<EPI, 16, 16, 4, 2, 2>(a, st);
    if (tile == 1) return launch_dense<EPI, 16, 12, 4, 2, 2>(a, st);
  }
  if (tile == 2) return launch_dense<EPI, 8, 16, 2, 4, 3>(a, st);
  if (tile == 3) return launch_dense<EPI, 8, 8, 4, 2, 4>(a, st);
  return launch_dense<EPI, 4, 4, 2, 2, 4>(a, st);
}
hipError_t launch_gemm_fp8(const uint8_t* x, const float* xs, const void* w, const float* ws, int M, int N, int K, int swiglu,
                           void* out, int out_type, hipStream_t st) {
  const Fp8Args a = {x, xs, (const uint8_t*)w, ws, out, M, N, K, (K + 127) / 128, N / 16};
  if (swiglu) return launch_fp8<FP8_SWIGLU>(a, st);
  if (out_type == SPEC_F32) return launch_fp8<FP8_STORE>(a, st);
  return launch_fp8<FP8_STORE16>(a, st);
}
