// Attention of a batch's queries over the paged low-bit cache:
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - m_i),   j visible: j <= pos_i and (no window, or
//   j > pos_i - window, or j < sinks)
// in one pass over the keys, with the running maximum and sum of the softmax in float32.
//
// Both products run on the block-float instruction 16 x 16 x 128, which contracts over a page's 128 tokens.  The cache's codes are
// sign and two magnitude bits: the nibble of the E2M1 value code / 2, so 32 codes widen to an operand with 11 shifts and masks and
// are exact.
//   Queries are sums of three E2M3 numbers, a sixteenth apart through the instruction's scale operand: with the row's largest channel at
// 7.5, the first leaves at most a quarter, the second, of that times 16, an eighth of its unit, the third half of its smallest step:
// 1 / 30720 of the largest channel is lost.  6-bit x 4-bit products take half the time of 8-bit x 4-bit ones: three of them 51 cycles, two
// E4M3 parts (8 significand bits of every channel) 66.  4-bit queries (absmax, 7 levels) are one digit, in eighths.
//   Probabilities, times the value's scale, need relative precision: each is the sum of two E4M3 numbers, the second scaled by 2^-5,
// which is one rounding to 8 significand bits, as bfloat16 operands would have it, down to 2^-14 of the query's largest in the page; what
// is smaller ends at 2^-22 of that.  (Where many rows share a page the values widen to bfloat16 and the probabilities are rounded to that
// instead.)
// Products are exact, sums float32.
//
// Keys are the row operand, queries the column operand: a lane ends up with the scores of one query against 4 consecutive tokens
// of every 16, which is, byte for byte, the eight-bit column operand of the second product (kp_slot: keys are stored in the order
// that makes it so).  Scores and probabilities never leave the lane but for their maxima.
//
// The first token has 4 bits, level = sign (2 mag + low): its scale is doubled, and one more instruction with the low bits in
// place of the codes and the scale operand 1/2 adds the rest, in the sequence's first page only.
#include "kv_pages.h"

#define KA_THREADS 256
#define KA_WAVES 4

typedef float v2f __attribute__((ext_vector_type(2)));
typedef short v2s __attribute__((ext_vector_type(2)));

struct KaArgs {
  const void* Q;
  int64_t ldq, n_pos;
  int q_f32, Hq, H, G, D;          // H: key / value heads, G = Hq / H query heads each
  KvBatch b;
  const float* rope;
  float cs, eps;                          // cs = scale * log2(e)
  int64_t window;                         // 0: none
  int sinks;
  const unsigned char* pages;
  uint16_t* O;
  float* part;                            // partial results of split rows (ka_part_floats)
  int splits;
  int slots;                              // items a sequence, where all have as many (order below); else 1
};

__device__ __forceinline__ v4f ka_mfma_pv(const u32 (&a)[4], v8i b, v4f c, int sa, int sb) {
  const v8i av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, b, c, 4 /* rows: E2M1 */, 0 /* columns: E4M3 */, 0, sa, 0, sb);
}
__device__ __forceinline__ v4f ka_mfma_qk(const u32 (&a)[4], v8i b, v4f c, int sa, int sb) {      // (six words of b)
  const v8i av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, b, c, 4 /* rows: E2M1 */, 2 /* columns: E2M3 */, 0, sa, 0, sb);
}

// Four floats below 2^8 as hi + 2^-5 lo, both E4M3.  `old`: any value (the conversions write a half each).
__device__ __forceinline__ void ka_split4(const float (&x)[4], int old, int& hi, int& lo) {
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], old, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], hi, true);
  const v2f b0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, 32.0f, false), b1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, 32.0f, true);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_fmaf(x[0], 32.0f, -b0.x), __builtin_fmaf(x[1], 32.0f, -b0.y), hi, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_fmaf(x[2], 32.0f, -b1.x), __builtin_fmaf(x[3], 32.0f, -b1.y), lo, true);
}

// (fmaxf would first make each argument canonical: twice the instructions over scores that come out of a select)
__device__ __forceinline__ float ka_max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// v of the lane 4 or 8 further in its row of 16, wrapping round
template <int O>
__device__ __forceinline__ float ka_ror(float v) {
  return __uint_as_float((u32)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + O, 0xF, 0xF, false));
}
// over the lanes of a query: R = 16 the four of a column, R < 16 also those R columns apart
template <int R = 16>
__device__ __forceinline__ float ka_max_groups(float v) {
  if (R <= 8) v = fmaxf(v, ka_ror<8>(v));
  if (R <= 4) v = fmaxf(v, ka_ror<4>(v));
  // (both halves, then both rows of 16, of a copy exchanged: no trip through LDS)
  auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}

// the same over the four lane groups for magnitudes, a NaN being the largest
__device__ __forceinline__ float ka_top_groups(float v) {
  const u32 b = __float_as_uint(v) & 0x7FFFFFFFu;
  auto x = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  const u32 t = max((u32)x[0], (u32)x[1]);
  x = __builtin_amdgcn_permlane16_swap(t, t, false, false);
  return __uint_as_float(max((u32)x[0], (u32)x[1]));
}

__device__ __forceinline__ float ka_q_at(const KaArgs& p, int64_t at) {
  return p.q_f32 ? reinterpret_cast<const float*>(p.Q)[at] : bl_bf16_to_f32(reinterpret_cast<const uint16_t*>(p.Q)[at]);
}
// 16 bfloat16 channels at a 16-byte boundary
__device__ __forceinline__ void ka_bf16x16(const uint4 (&w)[2], float (&x)[16]) {
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const u32 ww[4] = {w[e].x, w[e].y, w[e].z, w[e].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[8 * e + 2 * i] = __uint_as_float(ww[i] << 16);
      x[8 * e + 2 * i + 1] = __uint_as_float(ww[i] & 0xFFFF0000u);
    }
  }
}

// 32 channels, even and odd, as E2M3 codes in order: the nearest to x / unit (a power of two), and the way back.
// (Written out because the results must not share registers with arguments: the builtins let them, and the last channels, read after
// the first results are written, then come out wrong.)
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v32f __attribute__((ext_vector_type(32)));
typedef u32 v6u __attribute__((ext_vector_type(6)));
__device__ __forceinline__ v6u ka_pack6(v16f even, v16f odd, float unit) {
  v6u w;
  asm("v_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3\n\ts_nop 1" : "=&v"(w) : "v"(even), "v"(odd), "v"(unit));
  return w;
}
__device__ __forceinline__ v32f ka_unpack6(v6u w, float unit) {
  v32f x;
  asm("v_cvt_scalef32_pk32_f32_fp6 %0, %1, %2\n\ts_nop 1" : "=&v"(x) : "v"(w), "v"(unit));
  return x;
}

// One query's operands: lane group g holds the digits of channels 32 g .. 32 g + 31 of every 128.  DT = 64: the second half of the
// contraction takes the second digit against the same codes, so two instructions do.
// QV: bfloat16 rows at 16-byte boundaries with D % 32 == 0 (16 channels then lie in one half of the rotation's pairs): all loads of a
// row go out together.  Other rows go channel by channel.
template <int DT, bool Q4, bool QV>
struct KaQuery {
  static constexpr int KS = DT == 256 ? 2 : 1;
  static constexpr int PARTS = Q4 ? 1 : DT == 64 ? 2 : 3;
  static constexpr int WORDS = KS * PARTS * 6;
  v8i op[KS][PARTS];                       // six words each
  float c;                                 // log2 units of a score that is product * key scale
  int pos;                                 // position; -1: no such row

  // scale operand of a part (E8M0)
  static __device__ __forceinline__ int scale(int part, int g) {
    return DT == 64 ? (part == 0 ? (g < 2 ? 127 : 123) : 119) : 127 - 4 * part;
  }

  __device__ __forceinline__ void load(const KaArgs& p, const KvSeq& q, int r, int rows, int h) {
    const int g = (threadIdx.x & 63) >> 4;
    const bool have = r < rows;
    const int i = have ? r / p.G : 0, head = h * p.G + (have ? r - i * p.G : 0);
    const int64_t at = (q.q0 + i) * p.ldq + (int64_t)head * p.D;
    const int64_t ps = q.pos0 + i;
    pos = have ? (int)ps : -1;
    float x[KS][2][16];
    const int half = p.D >> 1;
    const float* rr = p.rope ? p.rope + min(max(ps, (int64_t)0), p.n_pos - 1) * p.D : nullptr;
    if (QV) {
      const uint16_t* row = reinterpret_cast<const uint16_t*>(p.Q) + at;
      uint4 w[KS][2][2], o[KS][2][2];
      float4 cs[KS][2][4], sn[KS][2][4];
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int ch = min(128 * k + 32 * (DT == 64 ? g & 1 : g) + 16 * v, p.D - 16);
          const int other = ch < half ? ch + half : ch - half, pair = ch < half ? ch : ch - half;
#pragma unroll
          for (int e = 0; e < 2; ++e) w[k][v][e] = reinterpret_cast<const uint4*>(row + ch)[e];
          if (rr) {
#pragma unroll
            for (int e = 0; e < 2; ++e) o[k][v][e] = reinterpret_cast<const uint4*>(row + other)[e];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              cs[k][v][e] = reinterpret_cast<const float4*>(rr + pair)[e];
              sn[k][v][e] = reinterpret_cast<const float4*>(rr + half + pair)[e];
            }
          }
        }
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int ch = 128 * k + 32 * (DT == 64 ? g & 1 : g) + 16 * v;
          float (&y)[16] = x[k][v];
          ka_bf16x16(w[k][v], y);
          if (rr) {                        // kp_rotate's steps; the first half subtracts
            float t[16];
            ka_bf16x16(o[k][v], t);
            const u32 flip = ch < half ? 0x80000000u : 0u;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float4 c4 = cs[k][v][e >> 2], s4 = sn[k][v][e >> 2];
              const float cc = (e & 3) == 0 ? c4.x : (e & 3) == 1 ? c4.y : (e & 3) == 2 ? c4.z : c4.w;
              const float ss = (e & 3) == 0 ? s4.x : (e & 3) == 1 ? s4.y : (e & 3) == 2 ? s4.z : s4.w;
              y[e] = y[e] * cc + __uint_as_float(__float_as_uint(t[e]) ^ flip) * ss;
            }
          }
          if (ch >= p.D) {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = 0.0f;
          }
        }
    } else {
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int ch = 128 * k + 32 * (DT == 64 ? g & 1 : g) + 16 * v + e;
            float y = 0.0f;
            if (ch < p.D) {
              y = ka_q_at(p, at + ch);
              if (rr) y = kp_rotate(y, ka_q_at(p, at + (ch < half ? ch + half : ch - half)), rr, ch, half);
            }
            x[k][v][e] = y;
          }
    }
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = __builtin_elementwise_maximum(top, fabsf(x[k][v][e]));      // (a NaN stays)
    top = ka_top_groups(top);
    // digits are E2M3 values up to 7.5 (4-bit levels: eighths), codes halves; c is never 0 (times -inf)
    float f = Q4 ? 7.0f / (top + p.eps) : top > 0.0f ? 7.5f / top : 0.0f;
    if (!have) f = 0.0f;
    c = fmaxf(16.0f * p.cs * (top / (Q4 ? 7.0f : 60.0f)), 1.17549435e-38f);
    // A NaN or an infinity in the query: whatever its digits are, the largest score times this, less itself, is no number, and so are
    // the row's sum and outputs.  What is not seen stays -inf: a row that sees nothing still has sum 0.
    if (!(top < INFINITY)) c = INFINITY;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      v16f a, b;                           // even and odd channels
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        a[e] = x[k][e >> 3][2 * (e & 7)] * f;
        b[e] = x[k][e >> 3][2 * (e & 7) + 1] * f;
        if (Q4) {
          a[e] = fminf(fmaxf(rintf(a[e]), -7.0f), 7.0f);
          b[e] = fminf(fmaxf(rintf(b[e]), -7.0f), 7.0f);
        }
      }
      v6u w[3];
      if (Q4) {
        w[0] = ka_pack6(a, b, 8.0f);
      } else {
#pragma unroll
        for (int d = 0; d < 3; ++d) {      // each digit is the nearest to what the ones before it leave
          const float unit = d == 0 ? 1.0f : d == 1 ? 0.0625f : 0.00390625f;
          w[d] = ka_pack6(a, b, unit);
          if (d == 2) break;
          const v32f y = ka_unpack6(w[d], unit);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            a[e] -= y[2 * e];
            b[e] -= y[2 * e + 1];
          }
        }
      }
#pragma unroll
      for (int d = 0; d < PARTS; ++d) {
        u32 o[6];
#pragma unroll
        for (int i = 0; i < 6; ++i)
          o[i] = DT != 64 ? w[d][i] : d == 1 ? (g < 2 ? w[2][i] : 0u) : g < 2 ? w[0][i] : Q4 ? 0u : w[1][i];
        op[k][d] = (v8i){(int)o[0], (int)o[1], (int)o[2], (int)o[3], (int)o[4], (int)o[5], 0, 0};
      }
    }
  }
};

// Running state of 16 queries: a lane has one query (column lane % 16) and, of the output, channels 16 t + 4 (lane / 16) + r.
template <int DT>
struct KaState {
  v4f o[DT / 16];
  float m, l;                              // maximum of product * key scale (without c); the lane's part of the sum
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < DT / 16; ++t) o[t] = (v4f){0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.0f;
  }
};

struct KaRange {                           // pages a wave walks: sinks first, then the window
  int n_sink, lo, n;
  int64_t min_pos, max_pos;
};

__device__ __forceinline__ KaRange ka_range(const KaArgs& p, const KvSeq& q, int r0, int rows_here, int rows) {
  KaRange w;
  const int last = min(r0 + rows_here, rows) - 1;
  w.min_pos = q.pos0 + r0 / p.G;
  w.max_pos = q.pos0 + last / p.G;
  const int64_t hi = min(w.max_pos >> 7, (int64_t)p.b.max_pages - 1);       // last page (-1: none)
  int64_t lo = 0, sink = 0;
  if (p.window) {
    lo = max(w.min_pos - p.window + 1, (int64_t)0) >> 7;
    sink = min((int64_t)((p.sinks + KP_TOKENS - 1) >> 7), min(lo, hi + 1));
  }
  w.lo = (int)lo;
  w.n_sink = (int)sink;
  w.n = (int)sink + (int)max(hi - lo + 1, (int64_t)0);
  return w;
}

// A page's codes as they come: 12 bytes for 32 codes.
struct __align__(4) KaWords { u32 a, b, c; };

template <int DT>
__device__ __forceinline__ void ka_load_keys(const unsigned char* head, int U, KaWords (&r)[DT == 256 ? 16 : 8]) {
  constexpr int KS = DT == 256 ? 2 : 1;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    // groups of channels that the head lacks meet zeros in the query: any codes will do
    const int u = min(DT == 64 ? g & 1 : 4 * k + g, U - 1);
    const u32 off = (u32)(n * U + u) * 12;
#pragma unroll
    for (int t = 0; t < 8; ++t) r[t * KS + k] = *reinterpret_cast<const KaWords*>(head + off + t * 16 * 12 * U);
  }
}
// codes of 16 of the values' channels
template <int DT>
__device__ __forceinline__ KaWords ka_load_values(const unsigned char* head, int U, int d) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  // (channels that the head lacks are not stored; the group's place is the same for the wave: one offset register for all groups)
  return *reinterpret_cast<const KaWords*>(head + (kp_code_bytes(U) + 48 * min(16 * d, 32 * U - 16)) + (u32)(n * 4 + g) * 12);
}

// a * b, and 0 where either is 0, whatever the other is (the instruction, so that the compiler knows of it)
extern "C" __device__ float ka_mul_legacy(float a, float b) __asm("llvm.amdgcn.fmul.legacy");

// E of a largest weight: weights times ka_scale_factor(E) = 2^(134 - E) are below 2^8, E - 7 is the E8M0 of what that took away
__device__ __forceinline__ int ka_exponent(float top) { return min(max((int)(__float_as_uint(top) >> 23), 16), 254); }
__device__ __forceinline__ float ka_scale_factor(int E) { return __uint_as_float((u32)(261 - E) << 23); }

// Weights p * scale of 16 queries as the second product's operands; scales(t): the four value scales of scores t.  What is not seen has
// probability 0, and 0 times a scale that is infinite or no number is 0 here.  They are brought below 2^8 by a power of two that the
// instruction puts back: that of the column's largest weight in the page, not of its largest scale, for a key of next to no weight may be
// all that has a value.  -> E, its exponent (ka_exponent)
template <int N, typename F>
__device__ __forceinline__ int ka_weights(v4f (&S)[N], F scales, float c, float base, float& l, int (&ph)[N], int (&pl)[N]) {
  float sum[4] = {0.f, 0.f, 0.f, 0.f}, top = 0.0f;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const float4 s4 = scales(t);
    const float vs[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t][r], c, -base));
      sum[r] += e;
      S[t][r] = ka_mul_legacy(e, vs[r]);
    }
    top = ka_max3(ka_max3(top, S[t][0], S[t][1]), S[t][2], S[t][3]);
  }
  l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  const int E = ka_exponent(ka_max_groups(top));
  const float f = ka_scale_factor(E);
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const float w[4] = {S[t][0] * f, S[t][1] * f, S[t][2] * f, S[t][3] * f};
    ka_split4(w, __float_as_int(w[0]), ph[t], pl[t]);
  }
  return E;
}

// Operands of the first token's lowest magnitude bits (nibble 1 = half a level, of the sign in C): 32 channels of the key ...
__device__ __forceinline__ void ka_low_keys(u32 low, u32 C, u32 (&a)[4]) {
#pragma unroll
  for (int v = 0; v < 4; ++v) a[v] = (((low << v) & 0x88888888u) >> 3) | ((C << v) & 0x88888888u);
}
// ... and, of the values of channels 16 d ..., token 0 alone
__device__ __forceinline__ void ka_low_values(const u32* lows, int U, int d, u32 C, u32 (&a)[4]) {
  const int lane = threadIdx.x & 63, c0 = min(16 * d, 32 * U - 16);
  const u32 bit = (lows[U + (c0 >> 5)] >> kp_sign_bit((c0 & 16) + (lane & 15))) & 1u;
  a[0] = lane < 16 ? bit | (C & 8u) : 0u;
  a[1] = a[2] = a[3] = 0u;
}

// Scores of 16 queries against a page, masked where some are not seen; `hi` and so on are a row's own.
__device__ __forceinline__ bool ka_masked(const KaArgs& p, const KaRange& rg, int64_t t0) {
  return t0 + KP_TOKENS - 1 > rg.min_pos || (p.window && t0 <= rg.max_pos - p.window && t0 + KP_TOKENS > p.sinks);
}
// Places of the page that rows from position `first` to `last` see: lo + 1 .. hi, and those below snk, less 16 g
struct KaSeen {
  int hi, lo, snk;
  __device__ __forceinline__ KaSeen(const KaArgs& p, int64_t t0, int64_t first, int64_t last, int base) {
    auto clamp = [&](int64_t v) { return (int)min(max(v - t0, (int64_t)-1), (int64_t)KP_TOKENS); };
    hi = clamp(last) - base;
    lo = (p.window ? clamp(first - p.window) : -1) - base;
    snk = (int)min(max((int64_t)p.sinks - t0, (int64_t)0), (int64_t)KP_TOKENS) - base;
  }
  __device__ __forceinline__ bool at(int j) const { return j <= hi && (j > lo || j < snk); }
};
// Scores t, element r of lane group g are those of token 64 (t / 4) + 4 (t % 4) + r + 16 g of the page
__device__ __forceinline__ constexpr int ka_token(int t, int r) { return 64 * (t >> 2) + 4 * (t & 3) + r; }

// N scores of four, every STEP-th t; `see` less what the lane adds to ka_token
template <int STEP, int N>
__device__ __forceinline__ void ka_mask(v4f (&S)[N], KaSeen see) {
  // (without a window most comparisons are the same for every page: kept here, not held in registers over the loop)
  asm volatile("" : "+v"(see.hi), "+v"(see.lo), "+v"(see.snk));
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) S[t][r] = see.at(ka_token(STEP * t, r)) ? S[t][r] : -INFINITY;
}

// New maxima `mx` over a lane's scores of a page, what was summed so far brought to them; base: the maxima in log2 units
template <int DT, int R, int N>
__device__ __forceinline__ void ka_raise(const float* mx, const float* c, KaState<DT>* st, float* base) {
  float m[N];
  bool up = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    m[i] = fmaxf(st[i].m, ka_max_groups<R>(mx[i]));
    base[i] = m[i] == -INFINITY ? 0.0f : m[i] * c[i];      // nothing seen so far: all terms are exp2(-inf) = 0
    up |= m[i] > st[i].m;
  }
  if (__any(up)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float al = __builtin_amdgcn_exp2f(st[i].m * c[i] - base[i]);
      st[i].l *= al;
#pragma unroll
      for (int t = 0; t < DT / 16; ++t) st[i].o[t] *= al;
      st[i].m = m[i];
    }
  }
}
template <int DT, int R, int N>
__device__ __forceinline__ float ka_rescale(const v4f (&S)[N], float c, KaState<DT>& st) {
  float mx = -INFINITY, base;
#pragma unroll
  for (int t = 0; t < N; ++t) mx = ka_max3(ka_max3(mx, S[t][0], S[t][1]), S[t][2], S[t][3]);
  ka_raise<DT, R, 1>(&mx, &c, &st, &base);
  return base;
}

// A state that is not finite makes every row that sees it no number, as the formula does, whatever the sign of the product with an
// infinite key, and however small the weight of a value: the score is NaN for either.
__device__ __forceinline__ float ka_poison(float s, float v) {
  return fabsf(s) < INFINITY && fabsf(v) < INFINITY ? s : __uint_as_float(0x7FC00000u);
}

// A lane's scales: those of its scores' tokens
template <int STEP, int N>
__device__ __forceinline__ void ka_load_scales(const float* s, int base, float (&v)[N][4]) {
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const float4 w = *reinterpret_cast<const float4*>(s + base + ka_token(STEP * t, 0));
    v[t][0] = w.x; v[t][1] = w.y; v[t][2] = w.z; v[t][3] = w.w;
  }
}

// What a wave has of the page it works on.  Each part is replaced by the next page's as soon as it has been used, so that a page's
// loads are on their way for the time a whole page takes.
template <int DT, int N>
struct KaHeld {
  KaWords keys[DT == 256 ? 16 : 8], vals[DT / 16];
  float ks[N][4], vs[N][4];
};

// One page against R queries.  w: the page's; on return what `next` (a page that can be read) has.  FIRST: the sequence's page 0.
// R < 16: the products have 16 columns whatever is in them, so every query stands in 16 / R of them, and of these column j works on
// the scores t = j, j + 16 / R, ... alone: the softmax takes R / 16 of the instructions.  As the second product's operand a column has
// zeros for the others' tokens; the columns' outputs are added up after the last page.
template <bool FIRST, int DT, int R, bool Q4, bool QV>
__device__ __forceinline__ void ka_page(const KaArgs& p, const KaRange& rg, int page, const unsigned char* head,
                                        const unsigned char* next, int U, KaHeld<DT, R / 2>& w, const KaQuery<DT, Q4, QV>& qy,
                                        KaState<DT>& st) {
  typedef KaQuery<DT, Q4, QV> Query;
  constexpr int KS = Query::KS, PARTS = Query::PARTS, STEP = 16 / R, N = 8 / STEP;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, j = n / R;
  const int base_tok = 16 * g + 4 * j;
  const u32* lows = reinterpret_cast<const u32*>(head + kp_low_off(U));
  const float* next_scale = reinterpret_cast<const float*>(next + kp_scale_off(U));

  v4f S[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v4f T[STEP];
#pragma unroll
    for (int e = 0; e < STEP; ++e) {
      const int t = STEP * i + e;
      T[e] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        u32 a[4];
        const KaWords c = w.keys[t * KS + k];
        kp_expand(c.a, c.b, c.c, a);
#pragma unroll
        for (int d = 0; d < PARTS; ++d) T[e] = ka_mfma_qk(a, qy.op[k][d], T[e], 127, Query::scale(d, g));
        if (FIRST && t == 0) {             // the first token's lowest bits
          const u32 L = n == 0 ? lows[min(DT == 64 ? g & 1 : 4 * k + g, U - 1)] : 0u;
          ka_low_keys(L, c.c, a);
#pragma unroll
          for (int d = 0; d < PARTS; ++d) T[0] = ka_mfma_qk(a, qy.op[k][d], T[0], 126, Query::scale(d, g));
        }
      }
    }
    S[i] = T[0];
#pragma unroll
    for (int e = 1; e < STEP; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[i][r] = j == e ? T[e][r] : S[i][r];
  }
  ka_load_keys<DT>(next, U, w.keys);
  if (FIRST && base_tok == 0) { w.ks[0][0] *= 2.0f; w.vs[0][0] *= 2.0f; }

#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) S[t][r] *= w.ks[t][r];
  ka_load_scales<STEP>(next_scale, base_tok, w.ks);
  const int64_t t0 = (int64_t)page * KP_TOKENS;
  float odd = 0.0f;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      odd = __builtin_elementwise_maximum(odd, __builtin_elementwise_maximum(fabsf(S[t][r]), fabsf(w.vs[t][r])));
  u32 bits = __float_as_uint(odd);
  asm("" : "+v"(bits));                    // (floats compared under a vote: this compiler lets a NaN pass as less than infinity)
  const bool finite = __all((bits & 0x7FFFFFFFu) < 0x7F800000u);
  if (ka_masked(p, rg, t0) || !finite) {
    if (!finite) {
#pragma unroll
      for (int t = 0; t < N; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = ka_poison(S[t][r], w.vs[t][r]);
    }
    ka_mask<STEP>(S, KaSeen(p, t0, qy.pos, qy.pos, base_tok));
  }

  const float base = ka_rescale<DT, R>(S, qy.c, st);
  int wh[N], wl[N];
  auto scales = [&](int t) { return make_float4(w.vs[t][0], w.vs[t][1], w.vs[t][2], w.vs[t][3]); };
  const int E = ka_weights(S, scales, qy.c, base, st.l, wh, wl);
  ka_load_scales<STEP>(next_scale + KP_TOKENS, base_tok, w.vs);
  v8i ph, pl;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    ph[t] = STEP == 1 || j == t % STEP ? wh[t / STEP] : 0;
    pl[t] = STEP == 1 || j == t % STEP ? wl[t / STEP] : 0;
  }
  // (the scheduler would widen values above, between the weights, and fetch the next page's later for it: 131072 keys 33 us, 31 so)
  __builtin_amdgcn_sched_barrier(0);

#pragma unroll
  for (int d = 0; d < DT / 16; ++d) {
    const KaWords c = w.vals[d];
    u32 a[4];
    kp_expand(c.a, c.b, c.c, a);
    st.o[d] = ka_mfma_pv(a, ph, st.o[d], 127, E - 7);
    st.o[d] = ka_mfma_pv(a, pl, st.o[d], 127, E - 12);
    if (FIRST) {
      ka_low_values(lows, U, d, c.c, a);
      st.o[d] = ka_mfma_pv(a, ph, st.o[d], 126, E - 7);
      st.o[d] = ka_mfma_pv(a, pl, st.o[d], 126, E - 12);
    }
    w.vals[d] = ka_load_values<DT>(next, U, d);
  }
}

// The next page from turn k on, step by step, that is there; nullptr: none.  k is left at its turn.
__device__ __forceinline__ const unsigned char* ka_next(const KaArgs& p, const KvSeq& q, const KaRange& rg, int h, int head_bytes, int step,
                                                        int& k, int& page) {
  for (; k < rg.n; k += step) {
    page = k < rg.n_sink ? k : rg.lo + k - rg.n_sink;
    const int id = kp_scalar(p.b.table, (int64_t)q.s * p.b.max_pages + page);
    if (id >= 0 && id < p.b.n_pages) return p.pages + ((int64_t)id * p.H + h) * head_bytes;
  }
  return nullptr;
}

// All pages of a wave: turns k, k + step, ...
template <int DT, int R, bool Q4, bool QV>
__device__ __forceinline__ void ka_walk(const KaArgs& p, const KvSeq& q, const KaRange& rg, int h, int k, int step,
                                        const KaQuery<DT, Q4, QV>& qy, KaState<DT>& st) {
  constexpr int STEP = 16 / R;
  const int U = kp_units(p.D), hb = kp_head_bytes(U);
  KaHeld<DT, R / 2> w;
  int page = 0;
  const unsigned char* head = ka_next(p, q, rg, h, hb, step, k, page);
  if (!head) return;
  const int lane = threadIdx.x & 63, base_tok = 16 * (lane >> 4) + 4 * ((lane & 15) / R);
  const float* scales = reinterpret_cast<const float*>(head + kp_scale_off(U));
  ka_load_keys<DT>(head, U, w.keys);
  ka_load_scales<STEP>(scales, base_tok, w.ks);
  ka_load_scales<STEP>(scales + KP_TOKENS, base_tok, w.vs);
#pragma unroll
  for (int d = 0; d < DT / 16; ++d) w.vals[d] = ka_load_values<DT>(head, U, d);
  auto turn = [&](auto first) __attribute__((always_inline)) {
    int page2 = 0;
    k += step;
    const unsigned char* next = ka_next(p, q, rg, h, hb, step, k, page2);
    ka_page<decltype(first)::value, DT, R, Q4, QV>(p, rg, page, head, next ? next : head, U, w, qy, st);
    head = next;
    page = page2;
  };
  if (page == 0) turn(std::true_type());
  while (head) turn(std::false_type());
}

// What outputs are multiplied by (levels are halves): nothing seen, sum 0, gives zeros; a sum that is no number makes all outputs that.
__device__ __forceinline__ float ka_inverse(float sum) { return sum == 0.0f ? 0.0f : 2.0f / sum; }

template <int DT>
__device__ __forceinline__ void ka_store(const KaArgs& p, const KvSeq& q, int r, int h, const v4f (&o)[DT / 16], float inv) {
  const int g = (threadIdx.x & 63) >> 4;
  const int i = r / p.G;
  uint16_t* out = p.O + ((int64_t)(q.q0 + i) * p.Hq + h * p.G + (r - i * p.G)) * p.D;
#pragma unroll
  for (int d = 0; d < DT / 16; ++d) {
    const int c = 16 * d + 4 * g;
    if (c >= p.D) continue;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = o[d][e] * inv;
    if ((p.D & 3) == 0) {
      *reinterpret_cast<uint2*>(out + c) = make_uint2(bl_pack_bf16(v[0], v[1]), bl_pack_bf16(v[2], v[3]));
    } else {                               // D is even
      *reinterpret_cast<u32*>(out + c) = bl_pack_bf16(v[0], v[1]);
      if (c + 2 < p.D) *reinterpret_cast<u32*>(out + c + 2) = bl_pack_bf16(v[2], v[3]);
    }
  }
}

// Late rows have the most pages: they go first.  Where every sequence has as many items, all last ones go before all others: most are
// empty, and in turn with full ones they would leave half of the CUs without work (below; 32 sequences of 128 rows: 149 us in turn).
__device__ __forceinline__ int64_t ka_late_first(const KaArgs& p, unsigned at, int n_tiles) {
  if (p.slots > 1) return (int64_t)(at % (unsigned)p.b.n_seqs) * p.slots + (p.slots - 1 - (int)(at / (unsigned)p.b.n_seqs));
  return n_tiles - 1 - (int64_t)at;
}

// Many rows, more than 128 channels: a workgroup has 4 x QT x 16 rows (row = new token x query head of the group) of one key / value
// head and walks their pages; each wave widens a quarter of a page's codes into LDS, where all four read them as operands, while the
// page before is worked on.  (The kernel below it, for up to 128 channels, keeps the values in bfloat16, for which LDS has no room here.)
template <int DT>
struct KaStage {
  static constexpr int KT = DT / 16;                     // 1 KB pieces of key operands
  static constexpr int VT = DT / 16;                     // and of value operands
  uint4 keys[KT * 64], vals[VT * 64];
  float ks[KP_TOKENS], vs[KP_TOKENS];
};
template <int DT>
struct KaRaw {                                           // a wave's share of a page on its way
  KaWords k[KaStage<DT>::KT / 4], v[KaStage<DT>::VT / 4];
  float scale, value;                                    // value: for waves 0, 1 the value scale of the key's token
};

template <int DT>
__device__ __forceinline__ void ka_fetch(const unsigned char* head, int U, int wave, KaRaw<DT>& raw) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int i = 0; i < KaStage<DT>::KT / 4; ++i) {
    const int j = 4 * i + wave;                          // piece: 16 tokens x 4 groups of channels
    const int tok = 16 * (j >> 1) + n, u = min(4 * (j & 1) + g, U - 1);
    raw.k[i] = *reinterpret_cast<const KaWords*>(head + (u32)(tok * U + u) * 12);
  }
  const unsigned char* v = head + kp_code_bytes(U);
#pragma unroll
  for (int i = 0; i < KaStage<DT>::VT / 4; ++i) {
    const int ch = min(16 * (4 * i + wave), 32 * U - 16) + n;
    raw.v[i] = *reinterpret_cast<const KaWords*>(v + (u32)(ch * 4 + g) * 12);
  }
  const float* s = reinterpret_cast<const float*>(head + kp_scale_off(U));
  raw.scale = s[threadIdx.x];                            // waves 0, 1: keys; 2, 3: values
  raw.value = s[threadIdx.x | KP_TOKENS];
}

template <int DT>
__device__ __forceinline__ void ka_widen(int page, int wave, const KaRaw<DT>& raw, KaStage<DT>& to) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < KaStage<DT>::KT / 4; ++i) {
    u32 a[4];
    kp_expand(raw.k[i].a, raw.k[i].b, raw.k[i].c, a);
    to.keys[(4 * i + wave) * 64 + lane] = make_uint4(a[0], a[1], a[2], a[3]);
  }
#pragma unroll
  for (int i = 0; i < KaStage<DT>::VT / 4; ++i) {
    u32 a[4];
    kp_expand(raw.v[i].a, raw.v[i].b, raw.v[i].c, a);
    to.vals[(4 * i + wave) * 64 + lane] = make_uint4(a[0], a[1], a[2], a[3]);
  }
  float s = raw.scale;
  if (wave < 2) {
    if (page == 0 && threadIdx.x == 0) s *= 2.0f;
    to.ks[threadIdx.x] = ka_poison(s, raw.value);
  } else {
    const int tok = (int)threadIdx.x - KP_TOKENS;
    to.vs[tok] = page == 0 && tok == 0 ? 2.0f * s : s;
  }
}

// One page, from LDS, against a wave's QT x 16 queries
template <bool FIRST, int DT, int QT, bool Q4, bool QV>
__device__ __forceinline__ void ka_staged(const KaArgs& p, const KaRange& rg, int page, const unsigned char* head, int U,
                                          const KaStage<DT>& sg, const uint4* digits, const float (&qc)[QT], const int (&qp)[QT],
                                          KaState<DT> (&st)[QT]) {
  typedef KaQuery<DT, Q4, QV> Query;
  constexpr int KS = Query::KS, PARTS = Query::PARTS, WORDS = KS * PARTS * 6;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int64_t t0 = (int64_t)page * KP_TOKENS;
  // (The scheduler would fetch all operands at once and spill: fences between steps, the next operand fetched a step ahead.)
  u32 dg[QT * WORDS];
#pragma unroll
  for (int j = 0; j < QT * WORDS / 4; ++j) {
    const uint4 w = digits[64 * j];
    dg[4 * j] = w.x; dg[4 * j + 1] = w.y; dg[4 * j + 2] = w.z; dg[4 * j + 3] = w.w;
  }
  auto digit = [&](int i, int s, int d) {
    const u32* w = dg + ((i * KS + s) * PARTS + d) * 6;
    return (v8i){(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], 0, 0};
  };
  v4f S[QT][8];
  auto key = [&](int j) { return sg.keys[j * 64 + lane]; };
  uint4 ahead = key(0);
#pragma unroll
  for (int j = 0; j < 8 * KS; ++j) {
    const int t = j / KS, s = j % KS;
    const u32 a[4] = {ahead.x, ahead.y, ahead.z, ahead.w};
    if (j + 1 < 8 * KS) ahead = key(j + 1);
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      if (s == 0) S[i][t] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < PARTS; ++d) S[i][t] = ka_mfma_qk(a, digit(i, s, d), S[i][t], 127, Query::scale(d, g));
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  const u32* lows = reinterpret_cast<const u32*>(head + kp_low_off(U));
  if (FIRST) {                         // the first token's lowest bits (its scales are doubled in LDS)
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int u = min(4 * s + g, U - 1);
      u32 a[4];
      ka_low_keys(n == 0 ? lows[u] : 0u, n == 0 ? reinterpret_cast<const u32*>(head)[u * 3 + 2] : 0u, a);
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int d = 0; d < PARTS; ++d) S[i][0] = ka_mfma_qk(a, digit(i, s, d), S[i][0], 126, Query::scale(d, g));
    }
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const float4 s4 = *reinterpret_cast<const float4*>(sg.ks + 16 * g + ka_token(t, 0));
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      S[i][t][0] *= s4.x; S[i][t][1] *= s4.y; S[i][t][2] *= s4.z; S[i][t][3] *= s4.w;
    }
  }
  const bool masked = ka_masked(p, rg, t0);
  v8i ph[QT], pl[QT];
  int E[QT];
  auto scales = [&](int t) { return *reinterpret_cast<const float4*>(sg.vs + 16 * g + ka_token(t, 0)); };
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    if (masked) ka_mask<1>(S[i], KaSeen(p, t0, qp[i], qp[i], 16 * g));
    const float base = ka_rescale<DT, 16>(S[i], qc[i], st[i]);
    __builtin_amdgcn_sched_barrier(0);
    int wh[8], wl[8];
    E[i] = ka_weights(S[i], scales, qc[i], base, st[i].l, wh, wl);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      ph[i][t] = wh[t];
      pl[i][t] = wl[t];
    }
    asm volatile("" : "+v"(ph[i]), "+v"(pl[i]), "+v"(st[i].l));      // (done here, not where it is used)
    __builtin_amdgcn_sched_barrier(0);
  }
  ahead = sg.vals[lane];
#pragma unroll
  for (int d = 0; d < DT / 16; ++d) {
    const u32 a[4] = {ahead.x, ahead.y, ahead.z, ahead.w};
    if (d + 1 < DT / 16) ahead = sg.vals[64 * (d + 1) + lane];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      st[i].o[d] = ka_mfma_pv(a, ph[i], st[i].o[d], 127, E[i] - 7);
      st[i].o[d] = ka_mfma_pv(a, pl[i], st[i].o[d], 127, E[i] - 12);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (FIRST) {
#pragma unroll
    for (int d = 0; d < DT / 16; ++d) {
      const int ch = min(16 * d, 32 * U - 16) + n;
      u32 a[4];
      ka_low_values(lows, U, d, reinterpret_cast<const u32*>(head + kp_code_bytes(U))[ch * 12 + 2], a);
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        st[i].o[d] = ka_mfma_pv(a, ph[i], st[i].o[d], 126, E[i] - 7);
        st[i].o[d] = ka_mfma_pv(a, pl[i], st[i].o[d], 126, E[i] - 12);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < QT; ++i)
#pragma unroll
    for (int d = 0; d < DT / 16; ++d) asm volatile("" : "+v"(st[i].o[d]));
}

template <int DT, int QT, bool Q4, bool QV>
__global__ __launch_bounds__(KA_THREADS, 2) void kv_attention_wide_kernel(KaArgs p, int shift, int n_tiles) {
  extern __shared__ __align__(16) unsigned char ka_smem[];
  KaStage<DT>* stage = reinterpret_cast<KaStage<DT>*>(ka_smem);
  typedef KaQuery<DT, Q4, QV> Query;
  const int h = (int)(blockIdx.x % (unsigned)p.H);
  const int64_t item = ka_late_first(p, blockIdx.x / (unsigned)p.H, n_tiles);
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, shift, 1, q);
  if (local < 0) return;                   // (whole workgroup)
  const int rows = q.n * p.G;              // (at most T * G, which the host bounds)
  if ((local << shift) >= rows) return;
  const int block0 = (int)(local << shift), n = threadIdx.x & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = block0 + wave * (16 * QT);
  const bool live = r0 < rows;             // (a wave without rows still widens its share)
  // a wave's digits stay in LDS (36 words a lane that the registers have no room for), each lane's written and read by itself
  constexpr int WORDS = QT * Query::KS * Query::PARTS * 6;
  uint4* digits = reinterpret_cast<uint4*>(ka_smem + 2 * sizeof(KaStage<DT>)) + wave * (WORDS / 4 * 64) + (threadIdx.x & 63);
  float qc[QT];
  int qp[QT];
  KaState<DT> st[QT];
  {
    u32 w[WORDS];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      Query qy;
      qy.load(p, q, r0 + 16 * i + n, rows, h);
      qc[i] = qy.c;
      qp[i] = qy.pos;
#pragma unroll
      for (int e = 0; e < WORDS / QT; ++e) w[i * (WORDS / QT) + e] = (u32)qy.op[e / 6 / Query::PARTS][e / 6 % Query::PARTS][e % 6];
      st[i].clear();
    }
#pragma unroll
    for (int j = 0; j < WORDS / 4; ++j) digits[64 * j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  }
  const KaRange all = ka_range(p, q, block0, KA_WAVES * 16 * QT, rows), rg = ka_range(p, q, live ? r0 : block0, 16 * QT, rows);
  const int U = kp_units(p.D), hb = kp_head_bytes(U);
  KaRaw<DT> raw;
  int k = 0, page = 0, cur = 0;
  const unsigned char* head = ka_next(p, q, all, h, hb, 1, k, page);
  if (head) {
    ka_fetch<DT>(head, U, wave, raw);
    ka_widen<DT>(page, wave, raw, stage[0]);
  }
  __syncthreads();
  auto turn = [&](auto first) __attribute__((always_inline)) {
    int page2 = 0;
    ++k;
    const unsigned char* next = ka_next(p, q, all, h, hb, 1, k, page2);
    if (next) ka_fetch<DT>(next, U, wave, raw);
    ka_staged<decltype(first)::value, DT, QT, Q4, QV>(p, rg, page, head, U, stage[cur], digits, qc, qp, st);
    // the other buffer was last read a page ago, before the barrier that ended it
    if (next) ka_widen<DT>(page2, wave, raw, stage[cur ^ 1]);
    __syncthreads();
    head = next;
    page = page2;
    cur ^= 1;
  };
  if (head && page == 0) turn(std::true_type());
  while (head) turn(std::false_type());
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    float l = st[i].l;
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    const int r = r0 + 16 * i + n;
    if (r < rows) ka_store<DT>(p, q, r, h, st[i].o, ka_inverse(l));
  }
}

// Many rows, up to 128 channels: a workgroup has 8 x QT x 16 rows of one key / value head, one workgroup a CU.
// The matrix and the vector unit take about as long for a page, so a wave's instructions for them are interleaved: in turn q the scores
// of page q (made in the turn before) are scaled and their maximum found between the products of page q - 1's probabilities and values;
// then they become probabilities tile by tile, and page q + 1's scores take the registers of a tile as it is used up.  What turn q's
// products read is bundle q, the values of page q - 1 and the keys of page q + 1, in buffer q % 2; bundle q + 1 is widened into the
// other buffer meanwhile, from codes that each wave fetched a turn ago.  One barrier a turn.  2048 rows x 32 heads of 128 on 6144 cached:
// 248 us where calls follow each other (970 TFLOP/s of two products that would be bfloat16's), 290 with both products of a page behind
// one another and four waves; by the counters 9100 clocks a page of 256 rows, of which a matrix unit is busy 3650 and a vector unit issues
// for 6400, at 2.1 GHz: the vector unit's softmax bounds it.
// Probabilities times the values' scales are bfloat16 here: the values widen to bfloat16 once for 8 x QT x 16 rows (levels / 2, the
// first token's with its lowest bit, exact), and two conversions of the E4M3 pair that few rows take are saved for every score.
#define KR_WAVES 8
#define KR_THREADS (64 * KR_WAVES)
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

template <int DT>
struct KrBundle {
  uint4 keys[(DT == 64 ? 4 : 8) * 64];      // 16 tokens x 128 channels a KB (DT = 64: 32 tokens x 64)
  uint4 vals[DT / 16 * 4 * 64];             // 16 channels x 32 tokens a KB, [channels][tokens]
};
struct KrScales {
  float k[KP_TOKENS], v[KP_TOKENS];
};
struct KrRaw {                              // a wave's share of a bundle on its way
  KaWords k, v;
  float s, value;                           // value: for waves 0, 1 the value scale of the key's token
};
template <int DT, int QT, bool Q4, bool QV>
struct KrShared {
  static constexpr int WORDS = (QT * KaQuery<DT, Q4, QV>::WORDS + 3) / 4 * 4;
  KrBundle<DT> bundle[2];
  KrScales scales[4];                       // page q in q % 4
  uint4 digits[KR_WAVES][WORDS / 4][64];    // each lane's written and read by itself
};

template <int DT>
__device__ __forceinline__ KaWords kr_fetch_keys(const unsigned char* head, int U, int piece) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int slot = DT == 64 ? 32 * piece + 16 * (g >> 1) + n : 16 * piece + n, u = min(DT == 64 ? g & 1 : g, U - 1);
  return *reinterpret_cast<const KaWords*>(head + (u32)(slot * U + u) * 12);
}
// keys of page `pk`, values of page `pv`, scales of page `pk`
template <int DT>
__device__ __forceinline__ void kr_fetch(const unsigned char* pk, const unsigned char* pv, int U, int wave, KrRaw& raw) {
  if (DT == 128 || wave >= 4) raw.k = kr_fetch_keys<DT>(pk, U, DT == 64 ? wave - 4 : wave);
  if (DT == 128 || wave < 4) raw.v = ka_load_values<DT>(pv, U, wave);
  if (wave < 4) raw.s = reinterpret_cast<const float*>(pk + kp_scale_off(U))[threadIdx.x];      // waves 0, 1: keys'; 2, 3: values'
  if (wave < 2) raw.value = reinterpret_cast<const float*>(pk + kp_scale_off(U))[threadIdx.x + KP_TOKENS];
}
template <int DT>
__device__ __forceinline__ void kr_widen_keys(const KaWords& w, int piece, KrBundle<DT>& to) {
  u32 o[4];
  kp_expand(w.a, w.b, w.c, o);
  to.keys[piece * 64 + (threadIdx.x & 63)] = make_uint4(o[0], o[1], o[2], o[3]);
}
// 32 tokens of a channel: nibble word v is tokens 8 v .. of the 32, the operand of lane group 2 (g % 2) + v / 2, tokens' quarter
// 2 (g / 2) + v % 2.
template <int DT>
__device__ __forceinline__ void kr_widen_values(u32 o, int v, int d, KrBundle<DT>& to) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const u32 x[4] = {__builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(o, 1.0f, 0)),
                    __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(o, 1.0f, 1)),
                    __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(o, 1.0f, 2)),
                    __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(o, 1.0f, 3))};
  to.vals[(d * 4 + 2 * (g >> 1) + (v & 1)) * 64 + 16 * (2 * (g & 1) + (v >> 1)) + n] = make_uint4(x[0], x[1], x[2], x[3]);
}
// the sequence's first token, in place of its entry there: level / 2 = mag + low / 2, of the sign in C
template <int DT>
__device__ __forceinline__ void kr_first_value(const KaWords& w, int d, const u32* lows, int U, KrBundle<DT>& to) {
  const int lane = threadIdx.x & 63, c0 = min(16 * d, 32 * U - 16);
  const u32 low = (lows[U + (c0 >> 5)] >> kp_sign_bit((c0 & 16) + (lane & 15))) & 1u;
  const float m = (float)(w.a & 3u) + 0.5f * (float)low;
  if (lane < 16) reinterpret_cast<uint16_t*>(to.vals + d * 256 + lane)[0] = (uint16_t)(__float_as_uint(w.c & 8u ? -m : m) >> 16);
}
// a page's scales as its rows take them: no value weight where no row of the workgroup sees the place, whatever stands there
__device__ __forceinline__ void kr_scale(const KaArgs& p, const KaRange& all, int page, int wave, const KrRaw& raw, KrScales& to) {
  const float s = raw.s;
  if (wave < 2) {
    to.k[threadIdx.x] = ka_poison(page == 0 && threadIdx.x == 0 ? 2.0f * s : s, raw.value);
  } else {
    const int tok = (int)threadIdx.x - KP_TOKENS;
    to.v[tok] = KaSeen(p, (int64_t)page * KP_TOKENS, all.min_pos, all.max_pos, 0).at(tok) ? s : 0.0f;
  }
}

// Scores of 16 tokens (QT x PARTS products) from their keys
template <int DT, int QT, bool Q4, bool QV>
__device__ __forceinline__ void kr_scores(uint4 key, const u32* dg, int t, v4f (&S)[QT][8]) {
  typedef KaQuery<DT, Q4, QV> Query;
  const int g = (threadIdx.x & 63) >> 4;
  const u32 a[4] = {key.x, key.y, key.z, key.w};
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    S[i][t] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < Query::PARTS; ++d) {
      const u32* w = dg + (i * Query::PARTS + d) * 6;
      S[i][t] = ka_mfma_qk(a, (v8i){(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], 0, 0}, S[i][t], 127,
                           Query::scale(d, g));
    }
  }
}
template <int DT>
__device__ __forceinline__ uint4 kr_key(const KrBundle<DT>& bd, int t) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  return DT == 64 ? bd.keys[32 * t + 16 * (g & 1) + n] : bd.keys[t * 64 + lane];
}
template <int N>
__device__ __forceinline__ void kr_digits(const uint4 (*digits)[64], u32 (&dg)[N]) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    const uint4 w = digits[j][threadIdx.x & 63];
    dg[4 * j] = w.x; dg[4 * j + 1] = w.y; dg[4 * j + 2] = w.z; dg[4 * j + 3] = w.w;
  }
}
// N times: one matrix instruction, then V of the vector unit's
template <int N, int V>
__device__ __forceinline__ void kr_interleave() {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x402, V, 0);
  }
}

template <int DT, int QT, bool Q4, bool QV>
__global__ __launch_bounds__(KR_THREADS) void kv_attention_rows_kernel(KaArgs p, int shift, int n_tiles) {
  typedef KaQuery<DT, Q4, QV> Query;
  typedef KrShared<DT, QT, Q4, QV> Shared;
  extern __shared__ __align__(16) unsigned char ka_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(ka_smem);
  const int h = (int)(blockIdx.x % (unsigned)p.H);
  const int64_t item = ka_late_first(p, blockIdx.x / (unsigned)p.H, n_tiles);
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, shift, 1, q);
  if (local < 0) return;                   // (whole workgroup)
  const int rows = q.n * p.G;              // (at most T * G, which the host bounds)
  if ((local << shift) >= rows) return;
  const int block0 = (int)(local << shift), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = block0 + wave * (16 * QT);      // (a wave without rows has zero queries and does its share)
  const int U = kp_units(p.D), hb = kp_head_bytes(U);
  const KaRange all = ka_range(p, q, block0, KR_WAVES * 16 * QT, rows), rg = ka_range(p, q, r0 < rows ? r0 : block0, 16 * QT, rows);
  uint4 (*digits)[64] = sh.digits[wave];
  float qc[QT];
  int qp[QT];
  KaState<DT> st[QT];
  {
    u32 w[Shared::WORDS];
    w[Shared::WORDS - 2] = w[Shared::WORDS - 1] = 0;
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      Query qy;
      qy.load(p, q, r0 + 16 * i + n, rows, h);
      qc[i] = qy.c;
      qp[i] = qy.pos;
#pragma unroll
      for (int e = 0; e < Query::WORDS; ++e) w[i * Query::WORDS + e] = (u32)qy.op[0][e / 6][e % 6];
      st[i].clear();
    }
#pragma unroll
    for (int j = 0; j < Shared::WORDS / 4; ++j) digits[j][lane] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  }

  // the next four pages, nullptr behind the last
  int k = -1;
  int page[4] = {0, 0, 0, 0};
  const unsigned char* head[4];
  auto next = [&](int e) __attribute__((always_inline)) {
    ++k;
    head[e] = ka_next(p, q, all, h, hb, 1, k, page[e]);
  };
#pragma unroll
  for (int e = 0; e < 4; ++e) next(e);
  if (head[0]) {
    constexpr int MV = DT / 16 * QT / 2, MQ = QT * Query::PARTS;       // products beside a tile of scores: of values, of keys
    v4f S[QT][8];
    v4i P[QT][4];                          // bfloat16, column operands of 32 tokens each
    u32 dg[Shared::WORDS];
    KrRaw raw;
    const bool has_k = DT == 128 || wave >= 4, has_v = DT == 128 || wave < 4;
    const int kp = DT == 64 ? wave - 4 : wave;
    auto values = [&](int v, const u32 (&o)[4], KrBundle<DT>& to) __attribute__((always_inline)) {
      if (has_v) kr_widen_values<DT>(o[v], v, wave, to);
    };
    // bundle 0: the first page's values, which meet zeros, and the second's keys; the first's keys for now in the other buffer
    kr_fetch<DT>(head[0], head[0], U, wave, raw);
    {
      u32 o[4];
      if (has_k) kr_widen_keys<DT>(raw.k, kp, sh.bundle[1]);
      kp_expand(raw.v.a, raw.v.b, raw.v.c, o);
#pragma unroll
      for (int v = 0; v < 4; ++v) values(v, o, sh.bundle[0]);
      if (wave < 4) kr_scale(p, all, page[0], wave, raw, sh.scales[0]);
    }
    kr_fetch<DT>(head[1] ? head[1] : head[0], head[0], U, wave, raw);
    if (has_k) kr_widen_keys<DT>(raw.k, kp, sh.bundle[0]);
    if (wave < 4) kr_scale(p, all, page[1], wave, raw, sh.scales[1]);
    kr_fetch<DT>(head[2] ? head[2] : head[0], head[0], U, wave, raw);
    __syncthreads();
    kr_digits(digits, dg);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      kr_scores<DT, QT, Q4, QV>(kr_key(sh.bundle[1], t), dg, t, S);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (page[0] == 0) {                    // the first token's lowest bits (its scale is doubled in LDS)
      const int u = min(DT == 64 ? g & 1 : g, U - 1);
      const u32* lows = reinterpret_cast<const u32*>(head[0] + kp_low_off(U));
      u32 a[4];
      ka_low_keys(n == 0 ? lows[u] : 0u, n == 0 ? reinterpret_cast<const u32*>(head[0])[u * 3 + 2] : 0u, a);
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int d = 0; d < Query::PARTS; ++d) {
          const u32* w = dg + (i * Query::PARTS + d) * 6;
          S[i][0] = ka_mfma_qk(a, (v8i){(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], 0, 0}, S[i][0], 126,
                               Query::scale(d, g));
        }
    }
#pragma unroll
    for (int i = 0; i < QT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) P[i][e] = (v4i){0, 0, 0, 0};
    __syncthreads();

    for (int turn = 0; head[0]; ++turn) {
      const KrScales& sc = sh.scales[turn & 3];
      const KrBundle<DT>& bd = sh.bundle[turn & 1];
      KrBundle<DT>& to = sh.bundle[(turn & 1) ^ 1];
      const float* sk = sc.k + 16 * g;
      const float* sv = sc.v + 16 * g;
      float mx[QT], base[QT];
      {
        // last page's products, this page's scales and maximum, this wave's share of the next bundle
        constexpr int VP = DT / 32;        // operands of the values beside a tile of scores
        uint4 va[VP];
        float4 s4 = *reinterpret_cast<const float4*>(sk + ka_token(0, 0));
        u32 o[4];
#pragma unroll
        for (int e = 0; e < VP; ++e) va[e] = bd.vals[e * 64 + lane];
#pragma unroll
        for (int i = 0; i < QT; ++i) mx[i] = -INFINITY;
        KaWords first = raw.v;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          uint4 vb[VP];
          const float4 s = s4;
#pragma unroll
          for (int e = 0; e < VP; ++e) {
            vb[e] = va[e];
            if (t < 7) va[e] = bd.vals[((t + 1) * VP + e) * 64 + lane];
          }
          if (t < 7) s4 = *reinterpret_cast<const float4*>(sk + ka_token(t + 1, 0));
#pragma unroll
          for (int e = 0; e < VP; ++e) {
            const int at = t * VP + e;
#pragma unroll
            for (int i = 0; i < QT; ++i)
              st[i].o[at / 4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, vb[e]), __builtin_bit_cast(v8bf, P[i][at % 4]),
                                                                        st[i].o[at / 4], 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < QT; ++i) {
            S[i][t][0] *= s.x; S[i][t][1] *= s.y; S[i][t][2] *= s.z; S[i][t][3] *= s.w;
            mx[i] = ka_max3(ka_max3(mx[i], S[i][t][0], S[i][t][1]), S[i][t][2], S[i][t][3]);
          }
          if (t == 0 && has_k) kr_widen_keys<DT>(raw.k, kp, to);
          if (t == 1) kp_expand(raw.v.a, raw.v.b, raw.v.c, o);
          if (t >= 2 && t < 6) values(t - 2, o, to);
          kr_interleave<MV, 24 / MV>();
          __builtin_amdgcn_sched_barrier(0);
        }
        // (products done here, not where they are used)
#pragma unroll
        for (int i = 0; i < QT; ++i)
#pragma unroll
          for (int d = 0; d < DT / 16; ++d) asm volatile("" : "+v"(st[i].o[d]));
        if (wave < 4) kr_scale(p, all, page[2], wave, raw, sh.scales[(turn + 2) & 3]);
        if (page[0] == 0 && has_v) kr_first_value<DT>(first, wave, reinterpret_cast<const u32*>(head[0] + kp_low_off(U)), U, to);
      }
      kr_fetch<DT>(head[3] ? head[3] : head[0], head[1] ? head[1] : head[0], U, wave, raw);
      const int64_t t0 = (int64_t)page[0] * KP_TOKENS;
      if (ka_masked(p, rg, t0)) {
#pragma unroll
        for (int i = 0; i < QT; ++i) {
          ka_mask<1>(S[i], KaSeen(p, t0, qp[i], qp[i], 16 * g));
          mx[i] = -INFINITY;
#pragma unroll
          for (int t = 0; t < 8; ++t) mx[i] = ka_max3(ka_max3(mx[i], S[i][t][0], S[i][t][1]), S[i][t][2], S[i][t][3]);
        }
      }
      ka_raise<DT, 16, QT>(mx, qc, st, base);
      __builtin_amdgcn_sched_barrier(0);
      {
        float sum[QT][2];
        uint4 key = kr_key(bd, 0);
        float4 s4 = *reinterpret_cast<const float4*>(sv + ka_token(0, 0));
        kr_digits(digits, dg);
#pragma unroll
        for (int i = 0; i < QT; ++i) sum[i][0] = sum[i][1] = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const float vs[4] = {s4.x, s4.y, s4.z, s4.w};
          if (t < 7) s4 = *reinterpret_cast<const float4*>(sv + ka_token(t + 1, 0));
          if (t > 0) {
            const uint4 now = key;
            key = kr_key(bd, t);
            kr_scores<DT, QT, Q4, QV>(now, dg, t - 1, S);
          }
#pragma unroll
          for (int i = 0; i < QT; ++i) {
            float w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i][t][r], qc[i], -base[i]));
              sum[i][r & 1] += e;
              w[r] = ka_mul_legacy(e, vs[r]);
            }
            P[i][t >> 1][2 * (t & 1)] = __builtin_bit_cast(int, (v2bf){(__bf16)w[0], (__bf16)w[1]});
            P[i][t >> 1][2 * (t & 1) + 1] = __builtin_bit_cast(int, (v2bf){(__bf16)w[2], (__bf16)w[3]});
          }
          if (t > 0) kr_interleave<MQ, QT * 18 / MQ>();
          __builtin_amdgcn_sched_barrier(0);
        }
        kr_scores<DT, QT, Q4, QV>(key, dg, 7, S);          // (behind the last page: of nothing, for nobody)
#pragma unroll
        for (int i = 0; i < QT; ++i) {
          st[i].l += sum[i][0] + sum[i][1];
          asm volatile("" : "+v"(P[i][0]), "+v"(P[i][1]), "+v"(P[i][2]), "+v"(P[i][3]), "+v"(st[i].l));
#pragma unroll
          for (int t = 0; t < 8; ++t) asm volatile("" : "+v"(S[i][t]));
        }
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 3; ++e) { head[e] = head[e + 1]; page[e] = page[e + 1]; }
      next(3);
      if (!head[0]) {                      // the last page's products
        const KrBundle<DT>& last = sh.bundle[(turn & 1) ^ 1];
#pragma unroll
        for (int at = 0; at < DT / 4; ++at)
#pragma unroll
          for (int i = 0; i < QT; ++i)
            st[i].o[at / 4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, last.vals[at * 64 + lane]),
                                                                      __builtin_bit_cast(v8bf, P[i][at % 4]), st[i].o[at / 4], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    float l = st[i].l;
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    const int r = r0 + 16 * i + n;
    if (r < rows) ka_store<DT>(p, q, r, h, st[i].o, ka_inverse(l));
  }
}

// Few rows: the pages are dealt to the four waves of `splits` workgroups; waves join in LDS, workgroups in the kernel below.
// Partial results of (tile, head, split): R rows x (log2 maximum, sum), then R x DT outputs.
__host__ __device__ static inline int64_t ka_part_floats(int DT, int R) { return R * (DT + 2); }

// A decoding batch has one item with rows and one without for every sequence, in turn, and an XCD deals workgroups to its shader
// engines in turn as well: half of them got the empty ones (64 sequences x 8 heads: 32 of an XCD's 64 workgroups ran on 16 CUs, 77 us).
// Where every sequence has as many items, all first ones go before all second ones.
__device__ __forceinline__ int64_t ka_item(const KaArgs& p, unsigned i) {
  return p.slots > 1 ? (int64_t)(i % (unsigned)p.b.n_seqs) * p.slots + i / (unsigned)p.b.n_seqs : (int64_t)i;
}

template <int DT, int R, bool Q4, bool QV>
__global__ __launch_bounds__(KA_THREADS, DT == 256 ? 1 : 2) void kv_attention_split_kernel(KaArgs p) {
  constexpr int SHIFT = R == 16 ? 4 : R == 8 ? 3 : 2;
  __shared__ float lds_o[KA_WAVES - 1][R][DT + 4];
  __shared__ float lds_m[KA_WAVES][R], lds_l[KA_WAVES][R];
  const int h = (int)(blockIdx.x % (unsigned)p.H);
  const unsigned rest = blockIdx.x / (unsigned)p.H;
  const int split = (int)(rest % (unsigned)p.splits);
  const int64_t item = ka_item(p, rest / (unsigned)p.splits);
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, SHIFT, 1, q);
  if (local < 0) return;                   // (whole workgroup)
  const int rows = q.n * p.G;
  if ((local << SHIFT) >= rows) return;
  const int r0 = (int)(local << SHIFT), lane = threadIdx.x & 63, n = lane & (R - 1), g = lane >> 4;
  const bool mine = (lane & 15) < R;       // one of a query's columns writes
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  KaQuery<DT, Q4, QV> qy;
  KaState<DT> st;
  qy.load(p, q, r0 + n, rows, h);
  st.clear();
  ka_walk<DT, R, Q4, QV>(p, q, ka_range(p, q, r0, R, rows), h, split * KA_WAVES + wave, p.splits * KA_WAVES, qy, st);
  // a query's columns together
  auto columns = [](float v) {
    if (R <= 8) v += ka_ror<8>(v);
    if (R <= 4) v += ka_ror<4>(v);
    return v;
  };
  float l = columns(st.l);
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
#pragma unroll
  for (int d = 0; d < DT / 16; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) st.o[d][e] = columns(st.o[d][e]);
  const float m = st.m == -INFINITY ? -INFINITY : st.m * qy.c;     // log2 units
  if (lane < R) {
    lds_m[wave][n] = m;
    lds_l[wave][n] = l;
  }
  __syncthreads();
  float top = lds_m[0][n];
#pragma unroll
  for (int w = 1; w < KA_WAVES; ++w) top = fmaxf(top, lds_m[w][n]);
  const float base = top == -INFINITY ? 0.0f : top;
  const float f = __builtin_amdgcn_exp2f(m - base);
  if (wave > 0 && mine) {
#pragma unroll
    for (int d = 0; d < DT / 16; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) lds_o[wave - 1][n][16 * d + 4 * g + e] = st.o[d][e] * f;
  }
  __syncthreads();
  if (wave > 0 || !mine || r0 + n >= rows) return;
  float sum = 0.0f;
#pragma unroll
  for (int w = 0; w < KA_WAVES; ++w) sum += lds_l[w][n] * __builtin_amdgcn_exp2f(lds_m[w][n] - base);
#pragma unroll
  for (int d = 0; d < DT / 16; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = st.o[d][e] * f;
#pragma unroll
      for (int w = 0; w < KA_WAVES - 1; ++w) v += lds_o[w][n][16 * d + 4 * g + e];
      st.o[d][e] = v;
    }
  if (p.splits == 1) {
    ka_store<DT>(p, q, r0 + n, h, st.o, ka_inverse(sum));
    return;
  }
  float* part = p.part + ((item * p.H + h) * p.splits + split) * ka_part_floats(DT, R);
  if (g == 0) {
    part[n] = top;
    part[R + n] = sum;
  }
#pragma unroll
  for (int d = 0; d < DT / 16; ++d)
#pragma unroll
    for (int e = 0; e < 4; e += 2)
      *reinterpret_cast<float2*>(part + 2 * R + n * DT + 16 * d + 4 * g + e) = make_float2(st.o[d][e], st.o[d][e + 1]);
}

// Joins the workgroups' partial results: a workgroup has one row of a tile and head, its waves a quarter of the splits each.
template <int DT>
__global__ __launch_bounds__(KA_THREADS) void kv_attention_join_kernel(KaArgs p, int shift) {
  constexpr int PER = DT / 64;             // channels a lane
  __shared__ float lds_o[KA_WAVES][DT];
  const int R = 1 << shift, n = (int)(blockIdx.x & (unsigned)(R - 1));
  const unsigned rest = blockIdx.x >> shift;
  const int h = (int)(rest % (unsigned)p.H);
  const int64_t item = rest / (unsigned)p.H;
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, shift, 1, q);
  if (local < 0) return;
  const int rows = q.n * p.G;
  if ((local << shift) + n >= rows) return;    // (whole workgroup)
  const int64_t stride = ka_part_floats(DT, R);
  const float* part = p.part + (item * p.H + h) * p.splits * stride;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // every wave has all maxima and sums
  float top = -INFINITY;
  for (int s = lane; s < p.splits; s += 64) top = fmaxf(top, part[s * stride + n]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float base = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f;
  for (int s = lane; s < p.splits; s += 64)
    sum += part[s * stride + R + n] * __builtin_amdgcn_exp2f(part[s * stride + n] - base);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
  float acc[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) acc[e] = 0.0f;
#pragma unroll 4
  for (int s = wave; s < p.splits; s += KA_WAVES) {
    const float* ps = part + s * stride;
    const float f = __builtin_amdgcn_exp2f(ps[n] - base);
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] = __builtin_fmaf(ps[2 * R + n * DT + PER * lane + e], f, acc[e]);
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) lds_o[wave][PER * lane + e] = acc[e];
  __syncthreads();
  const int c = 2 * (int)threadIdx.x;
  if (c >= p.D) return;
  const float inv = ka_inverse(sum);
  float v[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) v[e] = (((lds_o[0][c + e] + lds_o[1][c + e]) + lds_o[2][c + e]) + lds_o[3][c + e]) * inv;
  const int r = (int)(local << shift) + n, i = r / p.G;
  uint16_t* out = p.O + ((int64_t)(q.q0 + i) * p.Hq + h * p.G + (r - i * p.G)) * p.D;
  *reinterpret_cast<u32*>(out + c) = bl_pack_bf16(v[0], v[1]);
}

// ---------------------------------------------------------------- which kernel
// Row tiles of BM rows of n_seqs sequences with T new tokens: at most floor(T G / BM) + n_seqs.
static int64_t ka_tiles(int64_t T, int64_t G, int64_t n_seqs, int shift) { return ((T * G) >> shift) + n_seqs; }
static int ka_dt(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// How a call is dealt out: `splits` workgroups along the keys for tiles of 2^shift rows, or (0) whole rows
struct KaPlan {
  int splits, shift;
};
static KaPlan ka_plan(int64_t T, int64_t n_seqs, int64_t G, int64_t H, int64_t D, int64_t max_pages) {
  // Whole rows where their workgroups (of 128, or 64, rows) are filled and fill the chip's turns: sequences taken to be alike, the share of
  // the row places of all turns that have a row.  A place of the whole rows does about 1.6 times the work of one of the split ones (128
  // channels; of more, 2.5).  Split / whole, 8 heads of 128: 1 sequence of 256 x 4 rows on 2000 cached (0.25 of the places) 25 / 53 us,
  // of 400 x 4 on 4000 (0.39) 68 / 90, of 512 x 4 (0.5) 69 / 93; 8 of 200 on 900, 16 heads of 64 (0.78) 53 / 36; 1000 on none, 32 heads
  // of 64 (0.98) 51 / 30; 16 heads of 256, 2 of 300 on 1000 (0.59) 73 / 52.
  const int unit = D > 128 ? 64 : 128;
  const int64_t rows = (T * G + n_seqs - 1) / n_seqs, blocks = (rows + unit - 1) / unit * n_seqs * H, turns = (blocks + 255) / 256;
  if ((double)T * G * H >= (D > 128 ? 0.4 : 0.6) * 256.0 * turns * unit) return {0, 0};
  // rows a sequence: tiles of 4 or 8 do without the softmax of empty columns
  const int shift = T * G <= 4 * n_seqs ? 2 : T * G <= 8 * n_seqs ? 3 : 4;
  const int64_t tiles = ka_tiles(T, G, n_seqs, shift) * H;
  const int64_t want = (512 + tiles - 1) / tiles, most = (max_pages + KA_WAVES - 1) / KA_WAVES;
  return {(int)(want < most ? want : most), shift};
}

// Whole rows, up to 128 channels: eight waves of 32 rows (8), whose turn of the chip takes 1.7 times that of eight waves of 16 (7).  Not
// for a single turn where the new rows are most of their sequences and so see very unlike numbers of pages.  With 16 and 32: 4 sequences
// of 256 x 4 rows on 2000 cached, 8 heads of 128: 58 and 84 us; 2048 x 4 on 6144, 279 and 249; 4096 on none, 16 heads, 108 and 139.
static int ka_rows_shift(int64_t T, int64_t n_seqs, int64_t G, int64_t H, int64_t max_pages) {
  const int64_t rows = (T * G + n_seqs - 1) / n_seqs;
  auto turns = [&](int64_t unit) { return ((rows + unit - 1) / unit * n_seqs * H + 255) / 256; };
  return 17 * turns(256) < 10 * turns(128) && (turns(256) > 1 || 2 * T <= n_seqs * max_pages * KP_TOKENS) ? 8 : 7;
}

size_t bl_kv_attention_ws_bytes(int64_t T, int64_t n_seqs, int64_t G, int64_t H, int64_t D, int64_t max_pages) {
  const KaPlan k = ka_plan(T, n_seqs, G, H, D, max_pages);
  if (k.splits <= 1) return 0;
  return (size_t)(ka_tiles(T, G, n_seqs, k.shift) * H * k.splits * ka_part_floats(ka_dt(D), 1 << k.shift) * 4);
}

int bl_launch_kv_attention(const void* Q, int64_t ldq, bl_dtype qdt, int Hq, int H, int D, int q_bits, const KvBatch& b,
                           const float* rope, int64_t n_pos, float scale, float eps, int64_t window, int64_t sinks,
                           const void* pages, void* O, void* ws, hipStream_t s) {
  KaArgs p;
  p.Q = Q; p.ldq = ldq; p.n_pos = n_pos;
  p.q_f32 = qdt == BL_F32;
  p.Hq = Hq; p.H = H; p.G = Hq / H; p.D = D;
  p.b = b; p.rope = rope;
  p.cs = scale * 1.44269504f;
  p.eps = eps;
  // (no position is that far behind another: all are in reach, and differences fit 64 bits)
  p.window = window > 0x7FFFFFFF ? 0 : window;
  p.sinks = (int)(sinks < 0x7FFFFF00 ? sinks : 0x7FFFFF00);
  p.pages = (const unsigned char*)pages;
  p.O = (uint16_t*)O; p.part = (float*)ws;
  const KaPlan plan = ka_plan(b.T, b.n_seqs, p.G, H, D, b.max_pages);
  p.splits = plan.splits;
  const int dt = ka_dt(D);
  const bool qv = qdt == BL_BF16 && D % 32 == 0 && bl_aligned16(Q) && ldq % 8 == 0 && bl_aligned16(rope);
#define KA_GO2(DT, Q4, QV)                                                                               \
  do {                                                                                                   \
    if (p.splits && shift == 2) kv_attention_split_kernel<DT, 4, Q4, QV><<<blocks, KA_THREADS, 0, s>>>(p); \
    else if (p.splits && shift == 3) kv_attention_split_kernel<DT, 8, Q4, QV><<<blocks, KA_THREADS, 0, s>>>(p); \
    else if (p.splits) kv_attention_split_kernel<DT, 16, Q4, QV><<<blocks, KA_THREADS, 0, s>>>(p);       \
    else if (DT == 256) {                                                                                \
      constexpr int lds = (int)(2 * sizeof(KaStage<256>)) + KA_WAVES * 64 * 4 * KaQuery<256, Q4, QV>::WORDS; \
      BL_SET_MAX_LDS_ONCE((kv_attention_wide_kernel<256, 1, Q4, QV>), lds);                              \
      kv_attention_wide_kernel<256, 1, Q4, QV><<<blocks, KA_THREADS, lds, s>>>(p, shift, (int)tiles);    \
    } else if (shift == 8) KA_ROWS((DT == 64 ? 64 : 128), 2, Q4, QV);                                    \
    else KA_ROWS((DT == 64 ? 64 : 128), 1, Q4, QV);                                                      \
  } while (0)
#define KA_ROWS(DT, QT, Q4, QV)                                                                          \
  do {                                                                                                   \
    constexpr int lds = (int)sizeof(KrShared<DT, QT, Q4, QV>);                                           \
    BL_SET_MAX_LDS_ONCE((kv_attention_rows_kernel<DT, QT, Q4, QV>), lds);                                \
    kv_attention_rows_kernel<DT, QT, Q4, QV><<<blocks, KR_THREADS, lds, s>>>(p, shift, (int)tiles);      \
  } while (0)
#define KA_GO(DT)                                                  \
  do {                                                             \
    if (q_bits == 4) {                                             \
      if (qv) KA_GO2(DT, true, true); else KA_GO2(DT, true, false); \
    } else {                                                       \
      if (qv) KA_GO2(DT, false, true); else KA_GO2(DT, false, false); \
    }                                                              \
  } while (0)
  const int shift = p.splits ? plan.shift : dt == 256 ? 6 : ka_rows_shift(b.T, b.n_seqs, p.G, H, b.max_pages);
  const int64_t tiles = ka_tiles(b.T, p.G, b.n_seqs, shift);
  const int64_t n_blocks = tiles * H * (p.splits ? p.splits : 1);
  p.slots = tiles % b.n_seqs == 0 ? (int)(tiles / b.n_seqs) : 1;
  if (!bl_grid_ok(n_blocks) || !bl_grid_ok(tiles * H * 16)) return BL_ESHAPE;
  const unsigned blocks = (unsigned)n_blocks;
  if (dt == 64) KA_GO(64); else if (dt == 128) KA_GO(128); else KA_GO(256);
  BL_HIP_CHECK_LAUNCH();
  if (p.splits > 1) {
    const unsigned joins = (unsigned)((tiles * H) << shift);
    if (dt == 64) kv_attention_join_kernel<64><<<joins, KA_THREADS, 0, s>>>(p, shift);
    else if (dt == 128) kv_attention_join_kernel<128><<<joins, KA_THREADS, 0, s>>>(p, shift);
    else kv_attention_join_kernel<256><<<joins, KA_THREADS, 0, s>>>(p, shift);
    BL_HIP_CHECK_LAUNCH();
  }
#undef KA_GO
#undef KA_GO2
#undef KA_ROWS
  return BL_OK;
}
