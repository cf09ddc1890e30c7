// The paged form of the low-bit key / value cache (Section 4.2, Table 3): a batch's new keys and values are rotated (keys),
// quantized per head to 3 bits, or 4 at position 0, and put into their places; and the way back.
//   gamma = max |x| over the head,  q = RoundClip(x * (Q_b / (gamma + eps)), -Q_b, Q_b),  scale = gamma / Q_b
// 2 D bytes of a bfloat16 head in, 3 D / 8 + 4 out: HBM's to bound for prompts (4096 tokens x 32 heads of 128, keys and values: 31 us,
// 2.9 TB/s, beside vector units that issue for two thirds of the time that CUs hold work; 44 with the codes put together bit by bit),
// the chain of table, row and words for single tokens (32 sequences x 8 heads: 6.2 us).
//
// Workgroup = one head of one page.  Key codes are a token's own 12 byte groups.  Value codes of 32 tokens share words, so the
// page's new tokens are coded into LDS first and the words are then put together by one thread each, the bits of older tokens
// kept: no two workgroups write the same word, and no order of anything decides what is stored.
#include "kv_pages.h"

#define KP_THREADS 256

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

template <typename RawT>
__device__ __forceinline__ float kp_to_f32(RawT v) {
  return sizeof(RawT) == 2 ? __uint_as_float((u32)v << 16) : __uint_as_float((u32)v);
}

// 8 channels from c on of a head of D channels (zeros behind it)
template <typename RawT, bool VEC>
__device__ __forceinline__ void kp_load8(const RawT* x, int c, int D, float (&v)[8]) {
  if (VEC) {                                     // D % 16 == 0, 16-byte aligned
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    if (c < D) {
      if (sizeof(RawT) == 2) {
        const uint4 w = *reinterpret_cast<const uint4*>(x + c);
        const u32 ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[2 * e] = __uint_as_float(ww[e] << 16);
          v[2 * e + 1] = __uint_as_float(ww[e] & 0xFFFF0000u);
        }
      } else {
        const float4 a = *reinterpret_cast<const float4*>(x + c), b = *reinterpret_cast<const float4*>(x + c + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < D ? kp_to_f32<RawT>(x[c + e]) : 0.0f;
  }
}

// LPT lanes a token, 8 channels a lane.  A NaN is larger than any number, as where quantize_heads takes its maximum: it has to reach the
// scale.
template <int LPT>
__device__ __forceinline__ float kp_head_max(const float (&v)[8]) {
  float f = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f = __builtin_elementwise_maximum(f, fabsf(v[e]));
  u32 m = __float_as_uint(f) & 0x7FFFFFFFu;
  // neighbours, pairs, then mirrored halves and rows, whose quads are alike by then
  auto of = [](u32 x, auto ctrl) { return (u32)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, false); };
  m = max(m, of(m, std::integral_constant<int, 0xB1>{}));
  m = max(m, of(m, std::integral_constant<int, 0x4E>{}));
  m = max(m, of(m, std::integral_constant<int, 0x141>{}));
  if (LPT >= 16) m = max(m, of(m, std::integral_constant<int, 0x140>{}));
  if (LPT >= 32) m = max(m, (u32)__shfl_xor((int)m, 16, 64));
  return __uint_as_float(m);
}

// Levels RoundClip(v * s) of 8 channels, in nibbles: stored magnitude, sign (1: below zero), lowest magnitude bit of a 4-bit level.
// 3 bits: clipped before it is rounded (the bounds are integers), and rounded by an addition that leaves the level in the lowest bits;
// level + 4 of all channels then stand in one word, below 4 where the level is below zero.
__device__ __forceinline__ void kp_codes8(const float (&v)[8], float s, bool four, u32& mag, u32& sgn, u32& low) {
  u32 n = 0x44444444u;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = fminf(fmaxf(v[e] * s, -3.0f), 3.0f) + 12582912.0f;      // 1.5 x 2^23
    n += (__float_as_uint(p) - 0x4B400000u) << (4 * e);
  }
  sgn = (~n >> 2) & 0x11111111u;
  mag = ((n & 0x33333333u) ^ (sgn * 3u)) + sgn;
  low = 0u;
  if (__any(four)) {                             // (one token of a sequence)
    u32 m4 = 0u, s4 = 0u, l4 = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = fminf(fmaxf(rintf(v[e] * s), -7.0f), 7.0f);
      const u32 m = (u32)fabsf(p);
      m4 |= (m >> 1) << (4 * e);
      l4 |= (m & 1u) << (4 * e);
      s4 |= (p < 0.0f ? 1u : 0u) << (4 * e);
    }
    if (four) { mag = m4; sgn = s4; low = l4; }
  }
}

// Words of 4 channels from the codes of 32 tokens (t[i]: token i, a byte each): bytes of the words are made for all four at once and
// then transposed.  Byte j of A has tokens 2 j, 8 + 2 j, 2 j + 1, 9 + 2 j from its low end on, of B the same behind 16; of C the signs of
// 24 + 2 j, 16 + 2 j, 8 + 2 j, 2 j, then of the tokens behind them.
__device__ __forceinline__ void kp_words4(const u32 (&t)[32], u32 (&w)[4][3]) {
  u32 x[3][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const u32* y = t + 16 * o + 2 * j;
      x[o][j] = (y[0] & 0x03030303u) | (y[8] & 0x03030303u) << 2 | (y[1] & 0x03030303u) << 4 | (y[9] & 0x03030303u) << 6;
    }
    const u32* y = t + 2 * j;
    x[2][j] = (y[0] & 0x04040404u) << 1 | (y[8] & 0x04040404u) | (y[16] & 0x04040404u) >> 1 | (y[24] & 0x04040404u) >> 2 |
              (y[1] & 0x04040404u) << 5 | (y[9] & 0x04040404u) << 4 | (y[17] & 0x04040404u) << 3 | (y[25] & 0x04040404u) << 2;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const u32 a = __builtin_amdgcn_perm(x[k][1], x[k][0], 0x05010400u), b = __builtin_amdgcn_perm(x[k][1], x[k][0], 0x07030602u);
    const u32 c = __builtin_amdgcn_perm(x[k][3], x[k][2], 0x05010400u), d = __builtin_amdgcn_perm(x[k][3], x[k][2], 0x07030602u);
    w[0][k] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    w[1][k] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    w[2][k] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    w[3][k] = __builtin_amdgcn_perm(d, b, 0x07060302u);
  }
}

template <typename RawT, int LPT, bool VEC>
__global__ __launch_bounds__(KP_THREADS) void kv_append_kernel(
    const RawT* __restrict__ K, int64_t ldk, const RawT* __restrict__ V, int64_t ldv, int H, int D, KvBatch b,
    const float* __restrict__ rope, int64_t n_pos, float eps, unsigned char* __restrict__ pages) {
  constexpr int ROW = 8 * LPT;                   // LDS bytes a token
  __shared__ __align__(16) unsigned char vq[KP_TOKENS * ROW];
  const int h = (int)(blockIdx.x % (unsigned)H);
  KvSeq q;
  const int64_t local = kp_find(b, blockIdx.x / (unsigned)H, 1, 7, 2, q);
  if (local < 0) return;
  const int64_t pg = (q.pos0 > 0 ? q.pos0 >> 7 : 0) + local;
  if (pg >= b.max_pages || pg * KP_TOKENS >= q.len) return;
  const int id = kp_scalar(b.table, (int64_t)q.s * b.max_pages + pg);
  if (id < 0 || id >= b.n_pages) return;
  // tokens a .. e - 1 of the page are new
  const int a = (int)max(q.pos0 - pg * KP_TOKENS, (int64_t)0), e = (int)min(q.len - pg * KP_TOKENS, (int64_t)KP_TOKENS);
  const int U = kp_units(D), Dp = 32 * U, half = D >> 1;
  unsigned char* head = pages + ((int64_t)id * H + h) * kp_head_bytes(U);
  float* k_scale = reinterpret_cast<float*>(head + kp_scale_off(U));
  float* v_scale = k_scale + KP_TOKENS;
  u32* lows = reinterpret_cast<u32*>(head + kp_low_off(U));
  const int j = threadIdx.x % LPT, c = 8 * j, jq = j & 3, u = j >> 2;

  // older tokens' bits in the value words that this thread will put together: on their way before anything else
  constexpr int ITEMS = ROW * 4 / KP_THREADS;
  u32 old[ITEMS][3];
  u32* const v_words = reinterpret_cast<u32*>(head + kp_code_bytes(U));
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int it = (int)threadIdx.x + k * KP_THREADS, gr = it / Dp, d = it - gr * Dp;
    const int lo = max(a - 32 * gr, 0), hi = min(e - 32 * gr, 32);
    if (it < 4 * Dp && lo < hi && hi - lo < 32) {
#pragma unroll
      for (int i = 0; i < 3; ++i) old[k][i] = v_words[(d * 4 + gr) * 3 + i];
    } else {
      old[k][0] = old[k][1] = old[k][2] = 0u;
    }
  }

  for (int base = a; base < e; base += KP_THREADS / LPT) {      // (every lane stays: the quads exchange words)
    const int tok = base + (int)threadIdx.x / LPT;
    const bool have = tok < e;
    const int64_t pos = pg * KP_TOKENS + tok;
    const int64_t row = have ? q.q0 + (pos - q.pos0) : q.q0;
    const bool four = pos == 0;
    const float qb = four ? 7.0f : 3.0f;
    float v[8], y[8];
    u32 mag, sgn, low;
    // key and value
    const RawT* x = K + row * ldk + (int64_t)h * D;
    kp_load8<RawT, VEC>(x, c, D, v);
    kp_load8<RawT, VEC>(V + row * ldv + (int64_t)h * D, c, D, y);
    if (rope) {
      const float* rr = rope + min(pos, n_pos - 1) * D;
      if (VEC) {
        // 8 channels lie in one half of the pairs; the first half subtracts (kp_rotate's steps)
        float o[8], cs[8], sn[8];
        const int cc = min(c, D - 8), pair = cc < half ? cc : cc - half;
        kp_load8<RawT, true>(x, cc < half ? cc + half : cc - half, D, o);
        const f32x4_any* cp = reinterpret_cast<const f32x4_any*>(rr + pair);
        const f32x4_any* sp = reinterpret_cast<const f32x4_any*>(rr + half + pair);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f32x4_any c4 = cp[i], s4 = sp[i];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            cs[4 * i + k] = c4[k];
            sn[4 * i + k] = s4[k];
          }
        }
        const u32 flip = cc < half ? 0x80000000u : 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float r = v[i] * cs[i] + __uint_as_float(__float_as_uint(o[i]) ^ flip) * sn[i];
          v[i] = c < D ? r : 0.0f;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < D) v[i] = kp_rotate(v[i], kp_to_f32<RawT>(x[c + i < half ? c + i + half : c + i - half]), rr, c + i, half);
      }
    }
    float g = kp_head_max<LPT>(v);
    kp_codes8(v, qb / (g + eps), four, mag, sgn, low);
    if (have && j == 0) k_scale[tok] = g / qb;
    mag <<= 2 * (jq & 1);
    sgn <<= 3 - jq;
    low <<= 3 - jq;
    auto quad = [](u32 w, auto ctrl) { return (u32)__builtin_amdgcn_update_dpp(0, (int)w, decltype(ctrl)::value, 0xF, 0xF, false); };
    mag |= quad(mag, std::integral_constant<int, 0xB1>{});                  // lanes 0, 1: A; lanes 2, 3: B
    const u32 magB = quad(mag, std::integral_constant<int, 0xAA>{});        // B in every lane
    sgn |= quad(sgn, std::integral_constant<int, 0xB1>{});
    sgn |= quad(sgn, std::integral_constant<int, 0x4E>{});
    low |= quad(low, std::integral_constant<int, 0xB1>{});
    low |= quad(low, std::integral_constant<int, 0x4E>{});
    if (have && u < U) {
      u32* w = reinterpret_cast<u32*>(head) + (kp_slot(tok) * U + u) * 3;
      if (jq < 3) w[jq] = jq == 0 ? mag : jq == 1 ? magB : sgn;
      if (four && jq == 3) lows[u] = low;
    }
    g = kp_head_max<LPT>(y);
    kp_codes8(y, qb / (g + eps), four, mag, sgn, low);
    if (have) {
      if (j == 0) v_scale[tok] = g / qb;
      // a byte each: bits 0, 1 stored magnitude, bit 2 sign, bit 3 the lowest magnitude bit
      const u32 x = mag | sgn << 2 | low << 3, ev = x & 0x0F0F0F0Fu, od = (x >> 4) & 0x0F0F0F0Fu;
      *reinterpret_cast<uint2*>(vq + tok * ROW + c) =
          make_uint2(__builtin_amdgcn_perm(od, ev, 0x05010400u), __builtin_amdgcn_perm(od, ev, 0x07030602u));
    }
  }
  __syncthreads();
  if (pg == 0 && a == 0 && (int)threadIdx.x < U) {
    u32 w = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) w |= (u32)((vq[32 * threadIdx.x + i] >> 3) & 1) << kp_sign_bit(i);
    lows[U + threadIdx.x] = w;
  }
  // 32 new tokens: 4 channels a thread
  if ((int)threadIdx.x < Dp) {
    const int g = (int)threadIdx.x / (Dp >> 2), d = 4 * ((int)threadIdx.x - g * (Dp >> 2));
    if (a <= 32 * g && e >= 32 * g + 32) {
      u32 t[32], w[4][3];
#pragma unroll
      for (int i = 0; i < 32; ++i) t[i] = *reinterpret_cast<const u32*>(vq + (32 * g + i) * ROW + d);
      kp_words4(t, w);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < 3; ++k) v_words[((d + i) * 4 + g) * 3 + k] = w[i][k];
    }
  }
  // fewer, among older tokens or unused places: a channel a thread
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int it = (int)threadIdx.x + k * KP_THREADS, g = it / Dp, d = it - g * Dp;
    const int lo = max(a - 32 * g, 0), hi = min(e - 32 * g, 32);            // tokens lo .. hi - 1 of the 32
    if (it >= 4 * Dp || lo >= hi || hi - lo == 32) continue;
    u32* w = v_words + (d * 4 + g) * 3;
    u32 nw[3] = {0u, 0u, 0u}, keep[3] = {~0u, ~0u, ~0u};
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (i >= lo && i < hi) {
        const u32 v = vq[(32 * g + i) * ROW + d];
        nw[i >> 4] |= (v & 3u) << kp_mag_bit(i);
        nw[2] |= ((v >> 2) & 1u) << kp_sign_bit(i);
        keep[i >> 4] &= ~(3u << kp_mag_bit(i));
        keep[2] &= ~(1u << kp_sign_bit(i));
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (keep[i] != ~0u) w[i] = (old[k][i] & keep[i]) | nw[i];
  }
}

// Work items of the two kernels here: pages that hold rows of the call, at most two more a sequence than whole pages of rows.
static int64_t kp_items(int64_t T, int64_t n_seqs) { return (T >> 7) + 2 * n_seqs; }

int bl_launch_kv_append(const void* K, int64_t ldk, const void* V, int64_t ldv, bl_dtype dt, int H, int D, const KvBatch& b,
                        const float* rope, int64_t n_pos, float eps, void* pages, hipStream_t s) {
  const int64_t blocks = kp_items(b.T, b.n_seqs) * H;
  if (!bl_grid_ok(blocks)) return BL_ESHAPE;
  const int es = dt == BL_BF16 ? 2 : 4;
  const bool vec = D % 16 == 0 && bl_aligned16(K) && bl_aligned16(V) && ldk * es % 16 == 0 && ldv * es % 16 == 0;
#define KP_GO(T, LPT, VEC) \
  kv_append_kernel<T, LPT, VEC><<<(unsigned)blocks, KP_THREADS, 0, s>>>((const T*)K, ldk, (const T*)V, ldv, H, D, b, rope, n_pos, \
                                                                        eps, (unsigned char*)pages)
#define KP_LPT(T, VEC)                      \
  do {                                      \
    if (D <= 64) KP_GO(T, 8, VEC);          \
    else if (D <= 128) KP_GO(T, 16, VEC);   \
    else KP_GO(T, 32, VEC);                 \
  } while (0)
  if (dt == BL_BF16) { if (vec) KP_LPT(uint16_t, true); else KP_LPT(uint16_t, false); }
  else { if (vec) KP_LPT(u32, true); else KP_LPT(u32, false); }
#undef KP_LPT
#undef KP_GO
  BL_HIP_CHECK_LAUNCH();
  return BL_OK;
}

// ---------------------------------------------------------------- reading the codes back
// value = level * scale, one float32 multiply (bfloat16 outputs: one rounding more).  4096 tokens x 32 heads of 128: 26 us, 3.6 TB/s,
// beside vector units that issue for two thirds of the time; a wave stores whole lines of keys, rows of 256 bytes of values.
__device__ __forceinline__ float kp_level(u32 mag, u32 neg, u32 low, bool four) {
  const float m = (float)(four ? 2 * mag + low : mag);
  return neg ? -m : m;
}
template <typename OutT>
__device__ __forceinline__ void kp_store2(OutT* p, float x, float y) {
  if (sizeof(OutT) == 2) *reinterpret_cast<u32*>(p) = (u32)bl_f32_to_bf16_rne(x) | ((u32)bl_f32_to_bf16_rne(y) << 16);
  else *reinterpret_cast<float2*>(p) = make_float2(x, y);
}

template <typename OutT>
__global__ __launch_bounds__(KP_THREADS) void kv_read_kernel(const unsigned char* __restrict__ pages, int H, int D, KvBatch b,
                                                             OutT* __restrict__ K, OutT* __restrict__ V) {
  const int h = (int)(blockIdx.x % (unsigned)H);
  KvSeq q;
  const int64_t local = kp_find(b, blockIdx.x / (unsigned)H, 1, 7, 2, q);
  if (local < 0) return;
  const int64_t pg = (q.pos0 > 0 ? q.pos0 >> 7 : 0) + local;
  if (pg >= b.max_pages || pg * KP_TOKENS >= q.len) return;
  const int id = kp_scalar(b.table, (int64_t)q.s * b.max_pages + pg);
  if (id < 0 || id >= b.n_pages) return;
  const int a = (int)max(q.pos0 - pg * KP_TOKENS, (int64_t)0), e = (int)min(q.len - pg * KP_TOKENS, (int64_t)KP_TOKENS);
  const int U = kp_units(D);
  const unsigned char* head = pages + ((int64_t)id * H + h) * kp_head_bytes(U);
  const float* k_scale = reinterpret_cast<const float*>(head + kp_scale_off(U));
  const float* v_scale = k_scale + KP_TOKENS;
  const u32* lows = reinterpret_cast<const u32*>(head + kp_low_off(U));
  const int64_t row0 = q.q0 + pg * KP_TOKENS - q.pos0;      // row of the page's token 0
  if (K) {
    // a thread: 8 channels of one token
    const u32* words = reinterpret_cast<const u32*>(head);
    for (int it = threadIdx.x; it < (e - a) * 4 * U; it += KP_THREADS) {
      const int tok = a + it / (4 * U), o8 = it % (4 * U), u = o8 >> 2, k = o8 & 3;
      const u32* w = words + (kp_slot(tok) * U + u) * 3;
      const bool four = pg == 0 && tok == 0;
      const u32 m = w[k >> 1] >> (2 * (k & 1)), sg = w[2] >> (3 - k), lo = four ? lows[u] >> (3 - k) : 0u;
      const float d = k_scale[tok];
      OutT* out = K + ((row0 + tok) * H + h) * (int64_t)D;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const int c = 8 * o8 + i;
        if (c < D)                                         // (D is even)
          kp_store2<OutT>(out + c, kp_level((m >> (4 * i)) & 3u, (sg >> (4 * i)) & 1u, (lo >> (4 * i)) & 1u, four) * d,
                          kp_level((m >> (4 * i + 4)) & 3u, (sg >> (4 * i + 4)) & 1u, (lo >> (4 * i + 4)) & 1u, four) * d);
      }
    }
  }
  if (V) {
    // a thread: two channels of 32 tokens
    const u32* words = reinterpret_cast<const u32*>(head + kp_code_bytes(U));
    const int pairs = D >> 1;
    for (int it = threadIdx.x; it < 4 * pairs; it += KP_THREADS) {
      const int g = it / pairs, d = 2 * (it - g * pairs);
      const int lo = max(a - 32 * g, 0), hi = min(e - 32 * g, 32);
      if (lo >= hi) continue;
      u32 w[2][3];
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int k = 0; k < 3; ++k) w[p][k] = words[((d + p) * 4 + g) * 3 + k];
      u32 low[2] = {0u, 0u};
      if (pg == 0 && g == 0) {
#pragma unroll
        for (int p = 0; p < 2; ++p) low[p] = (lows[U + ((d + p) >> 5)] >> kp_sign_bit((d + p) & 31)) & 1u;
      }
      OutT* out = V + ((row0 + 32 * g) * H + h) * (int64_t)D + d;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        if (i < lo || i >= hi) continue;
        const bool four = pg == 0 && g == 0 && i == 0;
        const float sc = v_scale[32 * g + i];
        float x[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) x[p] = kp_level((w[p][i >> 4] >> kp_mag_bit(i)) & 3u, (w[p][2] >> kp_sign_bit(i)) & 1u, low[p], four) * sc;
        kp_store2<OutT>(out + (int64_t)i * H * D, x[0], x[1]);
      }
    }
  }
}

int bl_launch_kv_read(const void* pages, int H, int D, const KvBatch& b, void* K, void* V, bl_dtype odt, hipStream_t s) {
  const int64_t blocks = kp_items(b.T, b.n_seqs) * H;
  if (!bl_grid_ok(blocks)) return BL_ESHAPE;
  if (odt == BL_BF16) kv_read_kernel<uint16_t><<<(unsigned)blocks, KP_THREADS, 0, s>>>((const unsigned char*)pages, H, D, b, (uint16_t*)K, (uint16_t*)V);
  else kv_read_kernel<float><<<(unsigned)blocks, KP_THREADS, 0, s>>>((const unsigned char*)pages, H, D, b, (float*)K, (float*)V);
  BL_HIP_CHECK_LAUNCH();
  return BL_OK;
}
