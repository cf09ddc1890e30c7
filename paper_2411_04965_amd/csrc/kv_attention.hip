// Attention of a batch's queries over the paged low-bit cache:
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - m_i),   j visible: j <= pos_i and (no window, or
//   j > pos_i - window, or j < sinks)
// in one pass over the keys, with the running maximum and sum of the softmax in float32.
//
// Both products run on the block-float instruction 16 x 16 x 128, which contracts over a page's 128 tokens.  The cache's codes are
// sign and two magnitude bits: the nibble of the E2M1 value code / 2, so 32 codes widen to an operand with 13 shifts and masks and
// are exact.
//   Queries are fixed-point numbers of the row's largest channel: three digits -15 .. 15, -8 .. 8, -8 .. 8 in E2M3 (whose codes 0 ..
// 15 are the values 0 .. 15 eighths), a sixteenth apart through the instruction's scale operand; what is lost is at most 1 / 7680
// of the largest channel.  6-bit x 4-bit products take half the time of 8-bit x 4-bit ones: three of them 51 cycles, two E4M3 parts (8
// significand bits of every channel) 66.  4-bit queries (absmax, 7 levels) are one digit.
//   Probabilities, times the value's scale, need relative precision: each is the sum of two E4M3 numbers, the second scaled by 2^-5,
// which is one rounding to 8 significand bits, as bfloat16 operands would have it.
// Products are exact, sums float32.
//
// Keys are the row operand, queries the column operand: a lane ends up with the scores of one query against 4 consecutive tokens
// of every 16, which is, byte for byte, the eight-bit column operand of the second product (kp_slot: keys are stored in the order
// that makes it so).  Scores and probabilities never leave the lane but for two maxima a page; nothing goes through LDS.
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
  int q_f32, q_vec, Hq, H, G, D;          // H: key / value heads, G = Hq / H query heads each
  KvBatch b;
  const float* rope;
  float cs, eps;                          // cs = scale * log2(e)
  int64_t window;                         // 0: none
  int sinks;
  const unsigned char* pages;
  uint16_t* O;
  float* part;                            // partial results of split rows (ka_part_floats)
  int splits;
};

__device__ __forceinline__ v4f ka_mfma_pv(const u32 (&a)[4], v8i b, v4f c, int sa, int sb) {
  const v8i av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, b, c, 4 /* rows: E2M1 */, 0 /* columns: E4M3 */, 0, sa, 0, sb);
}
__device__ __forceinline__ v4f ka_mfma_qk(const u32 (&a)[4], const u32 (&b)[6], v4f c, int sa, int sb) {
  const v8i av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const v8i bv = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], (int)b[4], (int)b[5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4 /* rows: E2M1 */, 2 /* columns: E2M3 */, 0, sa, 0, sb);
}

// Four floats below 2^8 as hi + 2^-5 lo, both E4M3
__device__ __forceinline__ void ka_split4(const float (&x)[4], int& hi, int& lo) {
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], hi, true);
  const v2f b0 = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), b1 = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32((x[0] - b0.x) * 32.0f, (x[1] - b0.y) * 32.0f, 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32((x[2] - b1.x) * 32.0f, (x[3] - b1.y) * 32.0f, lo, true);
}

__device__ __forceinline__ float ka_max_groups(float v) {      // over the four lanes of a query
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

__device__ __forceinline__ float ka_q_at(const KaArgs& p, int64_t at) {
  return p.q_f32 ? reinterpret_cast<const float*>(p.Q)[at] : bl_bf16_to_f32(reinterpret_cast<const uint16_t*>(p.Q)[at]);
}

// 16 channels from c on of the head that starts at element `at`
__device__ __forceinline__ void ka_load16(const KaArgs& p, int64_t at, int c, float (&x)[16]) {
  if (p.q_vec) {
    if (c >= p.D) {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = 0.0f;
    } else if (p.q_f32) {
      const float4* s = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.Q) + at + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 w = s[e];
        x[4 * e] = w.x; x[4 * e + 1] = w.y; x[4 * e + 2] = w.z; x[4 * e + 3] = w.w;
      }
    } else {
      const uint4* s = reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.Q) + at + c);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint4 w = s[e];
        const u32 ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[8 * e + 2 * i] = __uint_as_float(ww[i] << 16);
          x[8 * e + 2 * i + 1] = __uint_as_float(ww[i] & 0xFFFF0000u);
        }
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = c + e < p.D ? ka_q_at(p, at + c + e) : 0.0f;
  }
}

// One query's operands: lane group g holds the digits of channels 32 g .. 32 g + 31 of every 128.  DT = 64: the second half of the
// contraction takes the second digit against the same codes, so two instructions do.
template <int DT, bool Q4>
struct KaQuery {
  static constexpr int KS = DT == 256 ? 2 : 1;
  static constexpr int PARTS = Q4 ? 1 : DT == 64 ? 2 : 3;
  u32 op[KS][PARTS][6];
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
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const int ch = 128 * k + 32 * (DT == 64 ? g & 1 : g) + 16 * v;
        float (&y)[16] = x[k][v];
        ka_load16(p, at, ch, y);
        if (rr) {
          if (p.q_vec) {                            // D % 32 == 0: 16 channels lie in one half
            if (ch < p.D) {
              float o[16];
              ka_load16(p, at, ch < half ? ch + half : ch - half, o);
#pragma unroll
              for (int e = 0; e < 16; ++e) y[e] = kp_rotate(y[e], o[e], rr, ch + e, half);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int cc = ch + e;
              if (cc < p.D) y[e] = kp_rotate(y[e], ka_q_at(p, at + (cc < half ? cc + half : cc - half)), rr, cc, half);
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if (!have) y[e] = 0.0f;
          top = fmaxf(top, fabsf(y[e]));
        }
      }
    top = ka_max_groups(top);
    const float lv = Q4 ? 7.0f : 15.0f;
    const float f = Q4 ? 7.0f / (top + p.eps) : top > 0.0f ? 15.0f / top : 0.0f;
    c = fmaxf(16.0f * p.cs * (top / lv), 1.17549435e-38f);      // digits are eighths, codes halves; never 0 (times -inf)
#pragma unroll
    for (int k = 0; k < KS; ++k) {
#pragma unroll
      for (int w = 0; w < PARTS; ++w)
#pragma unroll
        for (int e = 0; e < 6; ++e) op[k][w][e] = 0;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const float y = x[k][e >> 4][e & 15] * f;
        float d[3];
        d[0] = fminf(fmaxf(rintf(y), -lv), lv);
        const float r1 = (y - d[0]) * 16.0f;
        d[1] = fminf(fmaxf(rintf(r1), -15.0f), 15.0f);
        d[2] = fminf(fmaxf(rintf((r1 - d[1]) * 16.0f), -15.0f), 15.0f);
        if (DT == 64 && !Q4) {
          if (g >= 2) { d[0] = d[1]; d[1] = 0.0f; } else d[1] = d[2];
        }
        if (DT == 64 && Q4 && g >= 2) d[0] = 0.0f;
#pragma unroll
        for (int w = 0; w < PARTS; ++w) {
          const u32 code = (u32)fabsf(d[w]) | (d[w] < 0.0f ? 32u : 0u);
          const int bit = 6 * e;
          op[k][w][bit >> 5] |= code << (bit & 31);
          if ((bit & 31) > 26) op[k][w][(bit >> 5) + 1] |= code >> (32 - (bit & 31));
        }
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

// A page's codes as they come: 12 bytes for 32 codes.  Loads are issued together and used later.
template <int N>
struct KaCodes {
  struct __align__(4) Words { u32 a, b, c; };
  Words w[N];
};

template <int DT>
__device__ __forceinline__ void ka_load_keys(const unsigned char* head, int U, KaCodes<DT == 256 ? 16 : 8>& r) {
  constexpr int KS = DT == 256 ? 2 : 1;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    // groups of channels that the head lacks meet zeros in the query: any codes will do
    const int u = min(DT == 64 ? g & 1 : 4 * k + g, U - 1);
    const u32 off = (u32)(n * U + u) * 12;
#pragma unroll
    for (int t = 0; t < 8; ++t) r.w[t * KS + k] = *reinterpret_cast<const typename KaCodes<DT == 256 ? 16 : 8>::Words*>(head + off + t * 16 * 12 * U);
  }
}
template <int DT>
__device__ __forceinline__ void ka_load_values(const unsigned char* head, int U, KaCodes<DT / 16>& r) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const unsigned char* v = head + kp_code_bytes(U);
#pragma unroll
  for (int d = 0; d < DT / 16; ++d) {
    const int ch = min(16 * d, 32 * U - 16) + n;    // (channels that the head lacks are not stored)
    r.w[d] = *reinterpret_cast<const typename KaCodes<DT / 16>::Words*>(v + (u32)(ch * 4 + g) * 12);
  }
}
// 128 scales: t of a lane are those of tokens 64 (t / 4) + 16 g + 4 (t % 4) ...
__device__ __forceinline__ void ka_load_scales(const float* s, float (&v)[8][4]) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const float4 w = *reinterpret_cast<const float4*>(s + 64 * (t >> 2) + 16 * g + 4 * (t & 3));
    v[t][0] = w.x; v[t][1] = w.y; v[t][2] = w.z; v[t][3] = w.w;
  }
}

// probabilities of 16 queries as the second product's operands; MASKED: what is not seen has no weight, whatever stands there
template <bool MASKED>
__device__ __forceinline__ void ka_weights(const v4f (&S)[8], const float (&vs)[8][4], float c, float base, float& l, v8i& ph, v8i& pl) {
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    float w[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t][r], c, -base));
      sum[r] += e;
      w[r] = e * vs[t][r];
      if (MASKED && e == 0.0f) w[r] = 0.0f;
    }
    int hi, lo;
    ka_split4(w, hi, lo);
    ph[t] = hi;
    pl[t] = lo;
  }
  l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// One page against QT x 16 queries.  keys: the page's; on return those of `next` (nullptr: none) are on their way.
template <int DT, int QT, bool Q4>
__device__ __forceinline__ void ka_page(const KaArgs& p, const KaRange& rg, int page, const unsigned char* head,
                                        const unsigned char* next, int U, KaCodes<DT == 256 ? 16 : 8>& keys,
                                        const KaQuery<DT, Q4> (&qy)[QT], KaState<DT> (&st)[QT]) {
  typedef KaQuery<DT, Q4> Query;
  constexpr int KS = Query::KS, PARTS = Query::PARTS;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const float* k_scale = reinterpret_cast<const float*>(head + kp_scale_off(U));
  const u32* lows = reinterpret_cast<const u32*>(head + kp_low_off(U));
  float ks[8][4], vs[8][4];
  KaCodes<DT / 16> vals;
  ka_load_scales(k_scale, ks);
  ka_load_values<DT>(head, U, vals);
  ka_load_scales(k_scale + KP_TOKENS, vs);

  // scores: S[i][t] = codes of 16 tokens x queries
  v4f S[QT][8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
#pragma unroll
    for (int i = 0; i < QT; ++i) S[i][t] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32 a[4];
      const auto w = keys.w[t * KS + k];
      kp_expand(w.a, w.b, w.c, a);
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int d = 0; d < PARTS; ++d) S[i][t] = ka_mfma_qk(a, qy[i].op[k][d], S[i][t], 127, Query::scale(d, g));
    }
  }
  if (page == 0) {                         // the first token's lowest bits
    ks[0][0] *= g == 0 ? 2.0f : 1.0f;
    vs[0][0] *= g == 0 ? 2.0f : 1.0f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const u32 L = n == 0 ? lows[min(DT == 64 ? g & 1 : 4 * k + g, U - 1)] : 0u, C = keys.w[k].c;
      u32 a[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) a[v] = (((L << v) & 0x88888888u) >> 3) | ((C << v) & 0x88888888u);
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int d = 0; d < PARTS; ++d) S[i][0] = ka_mfma_qk(a, qy[i].op[k][d], S[i][0], 126, Query::scale(d, g));
    }
  }
  if (next) ka_load_keys<DT>(next, U, keys);

#pragma unroll
  for (int i = 0; i < QT; ++i)
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[i][t][r] *= ks[t][r];
  // lane group g, scores t, element r: token 64 (t / 4) + 16 g + 4 (t % 4) + r of the page
  const int64_t t0 = (int64_t)page * KP_TOKENS;
  const bool masked = t0 + KP_TOKENS - 1 > rg.min_pos || (p.window && t0 <= rg.max_pos - p.window && t0 + KP_TOKENS > p.sinks);
  if (masked) {
    const int snk = (int)min(max((int64_t)p.sinks - t0, (int64_t)0), (int64_t)KP_TOKENS);
    auto clamp = [&](int64_t v) { return (int)min(max(v - t0, (int64_t)-1), (int64_t)KP_TOKENS); };
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      // a row sees tokens lo + 1 .. hi of the page, and those below snk
      const int hi = clamp(qy[i].pos) - 16 * g, lo = (p.window ? clamp(qy[i].pos - p.window) : -1) - 16 * g, sk = snk - 16 * g;
#pragma unroll
      for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = 64 * (t >> 2) + 4 * (t & 3) + r;
          S[i][t][r] = j <= hi && (j > lo || j < sk) ? S[i][t][r] : -INFINITY;
        }
    }
    // places that no query of the wave sees may hold anything
    const int hi = clamp(rg.max_pos) - 16 * g, lo = (p.window ? clamp(rg.min_pos - p.window) : -1) - 16 * g, sk = snk - 16 * g;
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 64 * (t >> 2) + 4 * (t & 3) + r;
        vs[t][r] = j <= hi && (j > lo || j < sk) ? vs[t][r] : 0.0f;
      }
  }

  // value scales, brought below 2^8 by a power of two 2^(E - 134) that the instruction puts back
  float vm = 0.0f;
#pragma unroll
  for (int t = 0; t < 8; ++t) vm = fmaxf(vm, fmaxf(fmaxf(vs[t][0], vs[t][1]), fmaxf(vs[t][2], vs[t][3])));
  vm = ka_max_groups(vm);
  const int E = min(max((int)(__float_as_uint(vm) >> 23), 16), 254);
  const float vf = __uint_as_float((u32)(261 - E) << 23);
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) vs[t][r] *= vf;

  v8i ph[QT], pl[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 8; ++t) mx = fmaxf(mx, fmaxf(fmaxf(S[i][t][0], S[i][t][1]), fmaxf(S[i][t][2], S[i][t][3])));
    const float m = fmaxf(st[i].m, ka_max_groups(mx));
    const float base = m == -INFINITY ? 0.0f : m * qy[i].c;      // nothing seen so far: all terms are exp2(-inf) = 0
    if (__any(m > st[i].m)) {
      const float al = __builtin_amdgcn_exp2f(st[i].m * qy[i].c - base);
      st[i].l *= al;
#pragma unroll
      for (int t = 0; t < DT / 16; ++t) st[i].o[t] *= al;
      st[i].m = m;
    }
    if (masked) ka_weights<true>(S[i], vs, qy[i].c, base, st[i].l, ph[i], pl[i]);
    else ka_weights<false>(S[i], vs, qy[i].c, base, st[i].l, ph[i], pl[i]);
  }

#pragma unroll
  for (int d = 0; d < DT / 16; ++d) {
    const auto w = vals.w[d];
    u32 a[4];
    kp_expand(w.a, w.b, w.c, a);
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      st[i].o[d] = ka_mfma_pv(a, ph[i], st[i].o[d], 127, E - 7);
      st[i].o[d] = ka_mfma_pv(a, pl[i], st[i].o[d], 127, E - 12);
    }
  }
  if (page == 0) {
#pragma unroll
    for (int d = 0; d < DT / 16; ++d) {
      const int ch = min(16 * d, 32 * U - 16) + n;
      const u32 bit = (lows[U + (ch >> 5)] >> kp_sign_bit(ch & 31)) & 1u;
      const u32 a[4] = {g == 0 ? bit | (vals.w[d].c & 8u) : 0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        st[i].o[d] = ka_mfma_pv(a, ph[i], st[i].o[d], 126, E - 7);
        st[i].o[d] = ka_mfma_pv(a, pl[i], st[i].o[d], 126, E - 12);
      }
    }
  }
}

// The next page from turn k on, step by step, that is there; nullptr: none.  k is left at its turn.
__device__ __forceinline__ const unsigned char* ka_next(const KaArgs& p, const KvSeq& q, const KaRange& rg, int h, int head_bytes, int step,
                                                        int& k, int& page) {
  for (; k < rg.n; k += step) {
    page = k < rg.n_sink ? k : rg.lo + k - rg.n_sink;
    const int id = p.b.table[(int64_t)q.s * p.b.max_pages + page];
    if (id >= 0 && id < p.b.n_pages) return p.pages + ((int64_t)id * p.H + h) * head_bytes;
  }
  return nullptr;
}

// All pages of a wave: turns k, k + step, ...
template <int DT, int QT, bool Q4>
__device__ __forceinline__ void ka_walk(const KaArgs& p, const KvSeq& q, const KaRange& rg, int h, int k, int step,
                                        const KaQuery<DT, Q4> (&qy)[QT], KaState<DT> (&st)[QT]) {
  const int U = kp_units(p.D), hb = kp_head_bytes(U);
  KaCodes<DT == 256 ? 16 : 8> keys;
  int page = 0;
  const unsigned char* head = ka_next(p, q, rg, h, hb, step, k, page);
  if (head) ka_load_keys<DT>(head, U, keys);
  while (head) {
    int page2 = 0;
    k += step;
    const unsigned char* next = ka_next(p, q, rg, h, hb, step, k, page2);
    ka_page<DT, QT, Q4>(p, rg, page, head, next, U, keys, qy, st);
    head = next;
    page = page2;
  }
}

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

// A wave: QT x 16 rows (row = new token x query head of the group) of one key / value head, all their pages.
template <int DT, int QT, bool Q4>
__global__ __launch_bounds__(KA_THREADS, DT == 256 ? 1 : 2) void kv_attention_rows_kernel(KaArgs p, int shift, int n_tiles) {
  const int h = (int)(blockIdx.x % (unsigned)p.H);
  // late rows have the most pages: they go first
  const int64_t item = n_tiles - 1 - (int64_t)(blockIdx.x / (unsigned)p.H);
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, shift, 1, q);
  if (local < 0) return;
  const int rows = q.n * p.G;              // (at most T * G, which the host bounds)
  const int64_t first = (local << shift) + (int64_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (16 * QT);
  if (first >= rows) return;               // (no barriers in this kernel)
  const int r0 = (int)first, n = threadIdx.x & 15;
  KaQuery<DT, Q4> qy[QT];
  KaState<DT> st[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    qy[i].load(p, q, r0 + 16 * i + n, rows, h);
    st[i].clear();
  }
  ka_walk<DT, QT, Q4>(p, q, ka_range(p, q, r0, 16 * QT, rows), h, 0, 1, qy, st);
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    float l = st[i].l;
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    const int r = r0 + 16 * i + n;
    if (r < rows) ka_store<DT>(p, q, r, h, st[i].o, l > 0.0f ? 2.0f / l : 0.0f);
  }
}

// Few rows: the pages are dealt to the four waves of `splits` workgroups; waves join in LDS, workgroups in the kernel below.
// Partial results of (tile, head, split): 16 rows x (log2 maximum, sum), then 16 x DT outputs.
__host__ __device__ static inline int64_t ka_part_floats(int DT) { return 16 * (DT + 2); }

template <int DT, bool Q4>
__global__ __launch_bounds__(KA_THREADS, DT == 256 ? 1 : 2) void kv_attention_split_kernel(KaArgs p) {
  __shared__ float lds_o[KA_WAVES - 1][16][DT + 4];
  __shared__ float lds_m[KA_WAVES][16], lds_l[KA_WAVES][16];
  const int h = (int)(blockIdx.x % (unsigned)p.H);
  const unsigned rest = blockIdx.x / (unsigned)p.H;
  const int split = (int)(rest % (unsigned)p.splits);
  const int64_t item = rest / (unsigned)p.splits;
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, 4, 1, q);
  if (local < 0) return;                   // (whole workgroup)
  const int rows = q.n * p.G;
  if ((local << 4) >= rows) return;
  const int r0 = (int)(local << 4), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  KaQuery<DT, Q4> qy[1];
  KaState<DT> st[1];
  qy[0].load(p, q, r0 + n, rows, h);
  st[0].clear();
  ka_walk<DT, 1, Q4>(p, q, ka_range(p, q, r0, 16, rows), h, split * KA_WAVES + wave, p.splits * KA_WAVES, qy, st);
  float l = st[0].l;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  const float m = st[0].m == -INFINITY ? -INFINITY : st[0].m * qy[0].c;     // log2 units
  if (g == 0) {
    lds_m[wave][n] = m;
    lds_l[wave][n] = l;
  }
  __syncthreads();
  float top = lds_m[0][n];
#pragma unroll
  for (int w = 1; w < KA_WAVES; ++w) top = fmaxf(top, lds_m[w][n]);
  const float base = top == -INFINITY ? 0.0f : top;
  const float mine = __builtin_amdgcn_exp2f(m - base);
  if (wave > 0) {
#pragma unroll
    for (int d = 0; d < DT / 16; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) lds_o[wave - 1][n][16 * d + 4 * g + e] = st[0].o[d][e] * mine;
  }
  __syncthreads();
  if (wave > 0) return;
  float sum = 0.0f;
#pragma unroll
  for (int w = 0; w < KA_WAVES; ++w) sum += lds_l[w][n] * __builtin_amdgcn_exp2f(lds_m[w][n] - base);
#pragma unroll
  for (int d = 0; d < DT / 16; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = st[0].o[d][e] * mine;
#pragma unroll
      for (int w = 0; w < KA_WAVES - 1; ++w) v += lds_o[w][n][16 * d + 4 * g + e];
      st[0].o[d][e] = v;
    }
  if (p.splits == 1) {
    if (r0 + n < rows) ka_store<DT>(p, q, r0 + n, h, st[0].o, sum > 0.0f ? 2.0f / sum : 0.0f);
    return;
  }
  float* part = p.part + ((item * p.H + h) * p.splits + split) * ka_part_floats(DT);
  if (g == 0) {
    part[n] = top;
    part[16 + n] = sum;
  }
#pragma unroll
  for (int d = 0; d < DT / 16; ++d) *reinterpret_cast<v4f*>(part + 32 + n * DT + 16 * d + 4 * g) = st[0].o[d];
}

// Joins the workgroups' partial results: a workgroup has one row of a tile and head, its waves a quarter of the splits each.
template <int DT>
__global__ __launch_bounds__(KA_THREADS) void kv_attention_join_kernel(KaArgs p) {
  constexpr int PER = DT / 64;             // channels a lane
  __shared__ float lds_o[KA_WAVES][DT];
  const int n = (int)(blockIdx.x & 15u);
  const unsigned rest = blockIdx.x >> 4;
  const int h = (int)(rest % (unsigned)p.H);
  const int64_t item = rest / (unsigned)p.H;
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, 4, 1, q);
  if (local < 0) return;
  const int rows = q.n * p.G;
  if ((local << 4) + n >= rows) return;    // (whole workgroup)
  const float* part = p.part + (item * p.H + h) * p.splits * ka_part_floats(DT);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // every wave has all maxima and sums
  float top = -INFINITY;
  for (int s = lane; s < p.splits; s += 64) top = fmaxf(top, part[s * ka_part_floats(DT) + n]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float base = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f;
  for (int s = lane; s < p.splits; s += 64)
    sum += part[s * ka_part_floats(DT) + 16 + n] * __builtin_amdgcn_exp2f(part[s * ka_part_floats(DT) + n] - base);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
  float acc[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) acc[e] = 0.0f;
#pragma unroll 4
  for (int s = wave; s < p.splits; s += KA_WAVES) {
    const float* ps = part + s * ka_part_floats(DT);
    const float f = __builtin_amdgcn_exp2f(ps[n] - base);
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] = __builtin_fmaf(ps[32 + n * DT + PER * lane + e], f, acc[e]);
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) lds_o[wave][PER * lane + e] = acc[e];
  __syncthreads();
  const int c = 2 * (int)threadIdx.x;
  if (c >= p.D) return;
  const float inv = sum > 0.0f ? 2.0f / sum : 0.0f;
  float v[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) v[e] = (((lds_o[0][c + e] + lds_o[1][c + e]) + lds_o[2][c + e]) + lds_o[3][c + e]) * inv;
  const int r = (int)(local << 4) + n, i = r / p.G;
  uint16_t* out = p.O + ((int64_t)(q.q0 + i) * p.Hq + h * p.G + (r - i * p.G)) * p.D;
  *reinterpret_cast<u32*>(out + c) = bl_pack_bf16(v[0], v[1]);
}

// ---------------------------------------------------------------- which kernel
// Row tiles of BM rows of n_seqs sequences with T new tokens: at most floor(T G / BM) + n_seqs.
static int64_t ka_tiles(int64_t T, int64_t G, int64_t n_seqs, int shift) { return ((T * G) >> shift) + n_seqs; }
static int ka_dt(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// Workgroups along the keys; 0: the rows fill the chip without
static int ka_splits(int64_t T, int64_t n_seqs, int64_t G, int64_t H, int64_t max_pages) {
  const int64_t tiles = ka_tiles(T, G, n_seqs, 4) * H;
  if (tiles >= 2048) return 0;
  const int64_t want = (512 + tiles - 1) / tiles, most = (max_pages + KA_WAVES - 1) / KA_WAVES;
  return (int)(want < most ? want : most);
}

size_t bl_kv_attention_ws_bytes(int64_t T, int64_t n_seqs, int64_t G, int64_t H, int64_t D, int64_t max_pages) {
  const int splits = ka_splits(T, n_seqs, G, H, max_pages);
  if (splits <= 1) return 0;
  return (size_t)(ka_tiles(T, G, n_seqs, 4) * H * splits * ka_part_floats(ka_dt(D)) * 4);
}

int bl_launch_kv_attention(const void* Q, int64_t ldq, bl_dtype qdt, int Hq, int H, int D, int q_bits, const KvBatch& b,
                           const float* rope, int64_t n_pos, float scale, float eps, int64_t window, int64_t sinks,
                           const void* pages, void* O, void* ws, hipStream_t s) {
  KaArgs p;
  p.Q = Q; p.ldq = ldq; p.n_pos = n_pos;
  p.q_f32 = qdt == BL_F32;
  p.q_vec = D % 32 == 0 && bl_aligned16(Q) && ldq * (qdt == BL_F32 ? 4 : 2) % 16 == 0;
  p.Hq = Hq; p.H = H; p.G = Hq / H; p.D = D;
  p.b = b; p.rope = rope;
  p.cs = scale * 1.44269504f;
  p.eps = eps; p.window = window;
  p.sinks = (int)(sinks < 0x7FFFFF00 ? sinks : 0x7FFFFF00);
  p.pages = (const unsigned char*)pages;
  p.O = (uint16_t*)O; p.part = (float*)ws;
  p.splits = ka_splits(b.T, b.n_seqs, p.G, H, b.max_pages);
  const int dt = ka_dt(D);
  if (p.splits) {
    const int64_t tiles = ka_tiles(b.T, p.G, b.n_seqs, 4) * H;
    if (!bl_grid_ok(tiles * p.splits) || !bl_grid_ok(tiles * 16)) return BL_ESHAPE;
    const unsigned blocks = (unsigned)(tiles * p.splits);
#define KA_GO(DT)                                                                    \
  do {                                                                               \
    if (q_bits == 4) kv_attention_split_kernel<DT, true><<<blocks, KA_THREADS, 0, s>>>(p); \
    else kv_attention_split_kernel<DT, false><<<blocks, KA_THREADS, 0, s>>>(p);      \
    BL_HIP_CHECK_LAUNCH();                                                           \
    if (p.splits > 1) kv_attention_join_kernel<DT><<<(unsigned)(tiles * 16), KA_THREADS, 0, s>>>(p); \
  } while (0)
    if (dt == 64) KA_GO(64); else if (dt == 128) KA_GO(128); else KA_GO(256);
#undef KA_GO
  } else {
    const int shift = 6;                   // four waves of 16 rows
    const int64_t tiles = ka_tiles(b.T, p.G, b.n_seqs, shift);
    if (!bl_grid_ok(tiles * H)) return BL_ESHAPE;
    const unsigned blocks = (unsigned)(tiles * H);
#define KA_GO(DT)                                                                    \
  do {                                                                               \
    if (q_bits == 4) kv_attention_rows_kernel<DT, 1, true><<<blocks, KA_THREADS, 0, s>>>(p, shift, (int)tiles); \
    else kv_attention_rows_kernel<DT, 1, false><<<blocks, KA_THREADS, 0, s>>>(p, shift, (int)tiles); \
  } while (0)
    if (dt == 64) KA_GO(64); else if (dt == 128) KA_GO(128); else KA_GO(256);
#undef KA_GO
  }
  BL_HIP_CHECK_LAUNCH();
  return BL_OK;
}
