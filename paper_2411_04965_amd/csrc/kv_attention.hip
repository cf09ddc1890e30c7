// Attention of a batch's queries over the paged low-bit cache:
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - m_i),   j visible: j <= pos_i and (no window, or
//   j > pos_i - window, or j < sinks)
// in one pass over the keys, with the running maximum and sum of the softmax in float32.
//
// Both products run on the block-float instruction 16 x 16 x 128, 4-bit x 8-bit, which contracts over a page's 128 tokens.  The
// cache's codes are sign and two magnitude bits: the nibble of the E2M1 value code / 2, so 32 codes widen to an operand with 13
// shifts and masks and are exact.  A bfloat16 query has 8 significand bits: the sum of two E4M3 numbers, the second scaled by
// 2^-5 through the instruction's scale operand; products with the codes are exact, sums float32.  (Float32 and rotated queries are
// rounded to those 8 bits.)  The probabilities, times the value's scale, are split the same way: the one rounding there is to 8
// bits, as bfloat16 operands would have it.  4-bit queries (absmax, 7 levels) are exact in one E4M3 operand.
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

__device__ __forceinline__ v4f ka_mfma(const u32 (&a)[4], v8i b, v4f c, int sa, int sb) {
  const v8i av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, b, c, 4 /* rows: E2M1 */, 0 /* columns: E4M3 */, 0, sa, 0, sb);
}

// Four floats of magnitude below 2^8 + 2^4 as hi + 2^-5 lo, both E4M3
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

// One query's operands: lane group g holds channels 16 g .. 16 g + 15 and 64 + 16 g .. of every 128 (DT = 64: the second half of
// the contraction takes the low parts against the same codes, one instruction instead of two).
template <int DT, bool Q4>
struct KaQuery {
  static constexpr int KS = DT == 256 ? 2 : 1;
  static constexpr int PARTS = Q4 || DT == 64 ? 1 : 2;
  v8i op[KS][PARTS];
  float c;                                 // log2 units of a score that is product * key scale
  int pos;                                 // position; -1: no such row

  __device__ __forceinline__ void load(const KaArgs& p, const KvSeq& q, int r, int rows, int h) {
    const int g = (threadIdx.x & 63) >> 4;
    const bool have = r < rows;
    const int i = have ? r / p.G : 0, head = h * p.G + (have ? r - i * p.G : 0);
    const int64_t at = (q.q0 + i) * p.ldq + (int64_t)head * p.D;
    const int64_t ps = q.pos0 + i;
    pos = have ? (int)ps : -1;
    constexpr int NC = DT == 64 ? 1 : 2 * KS;       // chunks of 16 channels
    float x[NC][16];
    const int half = p.D >> 1;
    const float* rr = p.rope ? p.rope + min(max(ps, (int64_t)0), p.n_pos - 1) * p.D : nullptr;
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int ch = 64 * k + 16 * g;
      ka_load16(p, at, ch, x[k]);
      if (rr) {
        if (p.q_vec) {                              // D % 32 == 0: a chunk lies in one half
          if (ch < p.D) {
            float o[16];
            ka_load16(p, at, ch < half ? ch + half : ch - half, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) x[k][e] = kp_rotate(x[k][e], o[e], rr, ch + e, half);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int cc = ch + e;
            if (cc < p.D) x[k][e] = kp_rotate(x[k][e], ka_q_at(p, at + (cc < half ? cc + half : cc - half)), rr, cc, half);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (!have) x[k][e] = 0.0f;
        top = fmaxf(top, fabsf(x[k][e]));
      }
    }
    top = ka_max_groups(top);
    float f;
    if (Q4) {
      f = 7.0f / (top + p.eps);
      c = 2.0f * p.cs * (top / 7.0f);
    } else {
      // a power of two brings the largest channel to 128 .. 256
      const int E = min(max((int)(__float_as_uint(top) >> 23), 16), 254);
      f = __uint_as_float((u32)(261 - E) << 23);
      c = 2.0f * p.cs * __uint_as_float((u32)(E - 7) << 23);
    }
#pragma unroll
    for (int k = 0; k < NC; ++k) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float y[4];
        int hi, lo = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = x[k][4 * w + e] * f;
          if (Q4) y[e] = fminf(fmaxf(rintf(y[e]), -7.0f), 7.0f);
        }
        ka_split4(y, hi, lo);                       // (lo = 0 for levels)
        if (DT == 64) {
          op[0][0][w] = hi;
          op[0][0][4 + w] = lo;
        } else {
          op[k >> 1][0][4 * (k & 1) + w] = hi;
          if (PARTS == 2) op[k >> 1][PARTS - 1][4 * (k & 1) + w] = lo;
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

// One page against QT x 16 queries
template <int DT, int QT, bool Q4>
__device__ __forceinline__ void ka_page(const KaArgs& p, const KaRange& rg, int page, const unsigned char* head, int U,
                                        const KaQuery<DT, Q4> (&qy)[QT], KaState<DT> (&st)[QT]) {
  constexpr int KS = KaQuery<DT, Q4>::KS, PARTS = KaQuery<DT, Q4>::PARTS;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int64_t t0 = (int64_t)page * KP_TOKENS;
  const float* k_scale = reinterpret_cast<const float*>(head + kp_scale_off(U));
  const float* v_scale = k_scale + KP_TOKENS;
  const u32* lows = reinterpret_cast<const u32*>(head + kp_low_off(U));
  const unsigned char* v_codes = head + kp_code_bytes(U);

  // scores: S[i][t] = codes of 16 tokens x queries
  v4f S[QT][8];
  const int sb = DT == 64 ? (g < 2 ? 127 : 122) : 127;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
#pragma unroll
    for (int i = 0; i < QT; ++i) S[i][t] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int u = DT == 64 ? g & 1 : 4 * k + g;
      u32 A = 0, B = 0, C = 0, a[4];
      if (u < U) {
        const u32* w = reinterpret_cast<const u32*>(head) + ((16 * t + n) * U + u) * 3;
        A = w[0]; B = w[1]; C = w[2];
      }
      kp_expand(A, B, C, a);
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        S[i][t] = ka_mfma(a, qy[i].op[k][0], S[i][t], 127, sb);
        if (PARTS == 2) S[i][t] = ka_mfma(a, qy[i].op[k][PARTS - 1], S[i][t], 127, 122);
      }
      if (t == 0 && page == 0) {
        const u32 L = n == 0 && u < U ? lows[u] : 0u;
#pragma unroll
        for (int v = 0; v < 4; ++v) a[v] = (((L << v) & 0x88888888u) >> 3) | ((C << v) & 0x88888888u);
#pragma unroll
        for (int i = 0; i < QT; ++i) {
          S[i][t] = ka_mfma(a, qy[i].op[k][0], S[i][t], 126, sb);
          if (PARTS == 2) S[i][t] = ka_mfma(a, qy[i].op[k][PARTS - 1], S[i][t], 126, 122);
        }
      }
    }
  }

  // lane group g, scores t, element r: token 64 (t / 4) + 16 g + 4 (t % 4) + r of the page
  const bool masked = t0 + KP_TOKENS - 1 > rg.min_pos || (p.window && t0 <= rg.max_pos - p.window && t0 + KP_TOKENS > p.sinks);
  float mx[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) mx[i] = -INFINITY;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const int tok = 64 * (t >> 2) + 16 * g + 4 * (t & 3);
    const float4 s4 = *reinterpret_cast<const float4*>(k_scale + tok);
    float sc[4] = {s4.x, s4.y, s4.z, s4.w};
    if (t == 0 && page == 0 && g == 0) sc[0] *= 2.0f;
#pragma unroll
    for (int i = 0; i < QT; ++i) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v = S[i][t][r] * sc[r];
        if (masked) {
          const int64_t j = t0 + tok + r;
          const bool see = j <= qy[i].pos && (!p.window || j > qy[i].pos - p.window || j < p.sinks);
          v = see ? v : -INFINITY;
        }
        S[i][t][r] = v;
        mx[i] = fmaxf(mx[i], v);
      }
    }
  }

  // value scales, brought below 2^8 by a power of two 2^(E - 134) that the instruction puts back
  float vs[8][4];
  float vm = 0.0f;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const int tok = 64 * (t >> 2) + 16 * g + 4 * (t & 3);
    const float4 s4 = *reinterpret_cast<const float4*>(v_scale + tok);
    vs[t][0] = s4.x; vs[t][1] = s4.y; vs[t][2] = s4.z; vs[t][3] = s4.w;
    if (t == 0 && page == 0 && g == 0) vs[0][0] *= 2.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (masked) {                        // places that no query of the wave sees may hold anything
        const int64_t j = t0 + tok + r;
        if (j > rg.max_pos || (p.window && j <= rg.min_pos - p.window && j >= p.sinks)) vs[t][r] = 0.0f;
      }
      vm = fmaxf(vm, vs[t][r]);
    }
  }
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
    const float m = fmaxf(st[i].m, ka_max_groups(mx[i]));
    const float base = m == -INFINITY ? 0.0f : m * qy[i].c;      // nothing seen so far: all terms are exp2(-inf) = 0
    if (__any(m > st[i].m)) {
      const float al = __builtin_amdgcn_exp2f(st[i].m * qy[i].c - base);
      st[i].l *= al;
#pragma unroll
      for (int t = 0; t < DT / 16; ++t) st[i].o[t] *= al;
      st[i].m = m;
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      float w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i][t][r], qy[i].c, -base));
        st[i].l += e;
        w[r] = e * vs[t][r];
        if (masked && e == 0.0f) w[r] = 0.0f;
      }
      int hi, lo;
      ka_split4(w, hi, lo);
      ph[i][t] = hi;
      pl[i][t] = lo;
    }
  }

#pragma unroll
  for (int d = 0; d < DT / 16; ++d) {
    if (16 * d < 32 * U) {                 // (uniform)
      const u32* w = reinterpret_cast<const u32*>(v_codes) + ((16 * d + n) * 4 + g) * 3;
      const u32 A = w[0], B = w[1], C = w[2];
      u32 a[4];
      kp_expand(A, B, C, a);
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        st[i].o[d] = ka_mfma(a, ph[i], st[i].o[d], 127, E - 7);
        st[i].o[d] = ka_mfma(a, pl[i], st[i].o[d], 127, E - 12);
      }
      if (page == 0) {
        const int ch = 16 * d + n;
        const u32 bit = g == 0 ? (lows[U + (ch >> 5)] >> kp_sign_bit(ch & 31)) & 1u : 0u;
        u32 x[4] = {bit | (C & 8u), 0u, 0u, 0u};
        if (g != 0) x[0] = 0u;
#pragma unroll
        for (int i = 0; i < QT; ++i) {
          st[i].o[d] = ka_mfma(x, ph[i], st[i].o[d], 126, E - 7);
          st[i].o[d] = ka_mfma(x, pl[i], st[i].o[d], 126, E - 12);
        }
      }
    }
  }
}

// The page's head, or nullptr where the table names no page of the pool
__device__ __forceinline__ const unsigned char* ka_page_head(const KaArgs& p, const KvSeq& q, int page, int h, int head_bytes) {
  const int id = p.b.table[(int64_t)q.s * p.b.max_pages + page];
  return id >= 0 && id < p.b.n_pages ? p.pages + ((int64_t)id * p.H + h) * head_bytes : nullptr;
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
__global__ __launch_bounds__(KA_THREADS) void kv_attention_rows_kernel(KaArgs p, int shift, int n_tiles) {
  const int h = (int)(blockIdx.x % (unsigned)p.H);
  // late rows have the most pages: they go first
  const int64_t item = n_tiles - 1 - (int64_t)(blockIdx.x / (unsigned)p.H);
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, shift, 1, q);
  if (local < 0) return;
  const int rows = q.n * p.G;              // (at most T * G, which the host bounds)
  const int64_t first = (local << shift) + (int64_t)(threadIdx.x >> 6) * (16 * QT);
  if (first >= rows) return;               // (no barriers in this kernel)
  const int r0 = (int)first, n = threadIdx.x & 15;
  const int U = kp_units(p.D), hb = kp_head_bytes(U);
  KaQuery<DT, Q4> qy[QT];
  KaState<DT> st[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    qy[i].load(p, q, r0 + 16 * i + n, rows, h);
    st[i].clear();
  }
  const KaRange rg = ka_range(p, q, r0, 16 * QT, rows);
  for (int k = 0; k < rg.n; ++k) {
    const int page = k < rg.n_sink ? k : rg.lo + k - rg.n_sink;
    const unsigned char* head = ka_page_head(p, q, page, h, hb);
    if (head) ka_page<DT, QT, Q4>(p, rg, page, head, U, qy, st);
  }
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
__global__ __launch_bounds__(KA_THREADS) void kv_attention_split_kernel(KaArgs p) {
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
  const int r0 = (int)(local << 4), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
  const int U = kp_units(p.D), hb = kp_head_bytes(U);
  KaQuery<DT, Q4> qy[1];
  KaState<DT> st[1];
  qy[0].load(p, q, r0 + n, rows, h);
  st[0].clear();
  const KaRange rg = ka_range(p, q, r0, 16, rows);
  for (int k = split * KA_WAVES + wave; k < rg.n; k += p.splits * KA_WAVES) {
    const int page = k < rg.n_sink ? k : rg.lo + k - rg.n_sink;
    const unsigned char* head = ka_page_head(p, q, page, h, hb);
    if (head) ka_page<DT, 1, Q4>(p, rg, page, head, U, qy, st);
  }
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

// Joins the workgroups' partial results: a workgroup has the 16 rows of one tile and head.
template <int DT>
__global__ __launch_bounds__(KA_THREADS) void kv_attention_join_kernel(KaArgs p) {
  const int h = (int)(blockIdx.x % (unsigned)p.H);
  const int64_t item = blockIdx.x / (unsigned)p.H;
  KvSeq q;
  const int64_t local = kp_find(p.b, item, p.G, 4, 1, q);
  if (local < 0) return;
  const int rows = q.n * p.G;
  if ((local << 4) >= rows) return;
  const float* part = p.part + (item * p.H + h) * p.splits * ka_part_floats(DT);
  const int live = min(16, rows - (int)(local << 4));
  for (int it = threadIdx.x; it < live * (DT / 2); it += KA_THREADS) {
    const int n = it / (DT / 2), c = 2 * (it - n * (DT / 2));
    if (c >= p.D) continue;
    float top = -INFINITY;
    for (int s = 0; s < p.splits; ++s) top = fmaxf(top, part[s * ka_part_floats(DT) + n]);
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, x = 0.0f, y = 0.0f;
    for (int s = 0; s < p.splits; ++s) {
      const float* ps = part + s * ka_part_floats(DT);
      const float f = __builtin_amdgcn_exp2f(ps[n] - base);
      const float2 o = *reinterpret_cast<const float2*>(ps + 32 + n * DT + c);
      sum += ps[16 + n] * f;
      x += o.x * f;
      y += o.y * f;
    }
    const float inv = sum > 0.0f ? 2.0f / sum : 0.0f;
    const int r = (int)(local << 4) + n, i = r / p.G;
    uint16_t* out = p.O + ((int64_t)(q.q0 + i) * p.Hq + h * p.G + (r - i * p.G)) * p.D;
    *reinterpret_cast<u32*>(out + c) = bl_pack_bf16(x * inv, y * inv);
  }
}

// ---------------------------------------------------------------- which kernel
// Row tiles of BM rows of n_seqs sequences with T new tokens: at most floor(T G / BM) + n_seqs.
static int64_t ka_tiles(int64_t T, int64_t G, int64_t n_seqs, int shift) { return ((T * G) >> shift) + n_seqs; }
static int ka_dt(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// Workgroups along the keys; 0: the rows fill the chip without
static int ka_splits(int64_t T, int64_t n_seqs, int64_t G, int64_t H, int64_t max_pages) {
  const int64_t tiles = ka_tiles(T, G, n_seqs, 4) * H;
  if (tiles >= 2048) return 0;
  const int64_t want = (1024 + tiles - 1) / tiles, most = (max_pages + KA_WAVES - 1) / KA_WAVES;
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
    if (!bl_grid_ok(tiles * p.splits)) return BL_ESHAPE;
    const unsigned blocks = (unsigned)(tiles * p.splits);
#define KA_GO(DT)                                                                    \
  do {                                                                               \
    if (q_bits == 4) kv_attention_split_kernel<DT, true><<<blocks, KA_THREADS, 0, s>>>(p); \
    else kv_attention_split_kernel<DT, false><<<blocks, KA_THREADS, 0, s>>>(p);      \
    BL_HIP_CHECK_LAUNCH();                                                           \
    if (p.splits > 1) kv_attention_join_kernel<DT><<<(unsigned)tiles, KA_THREADS, 0, s>>>(p); \
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
