// RMS norm in front of a quantized linear, and its gradient.
//   h = X + R (rounded to the stream's type), rstd = 1 / sqrt(mean h^2 + eps), y = (h * rstd) * gamma, codes of y by eq. 7 or eq. 3
// HBM bound: a bfloat16 channel takes 4 bytes in, 2 out, and half a byte (INT4) to one (INT8) of codes.  One workgroup has a row in
// registers, 16 channels a thread and turn (a thread then owns whole words of every code format), so the row is read once though
// it is passed over three times: squares, statistic, codes.  The two sums are float64 (as the quantizers' mean is), so that the
// codes do not depend on the order of the additions.  16384 x 4096 with a residual, six-bit codes: 102 us = 4.3 TB/s; 2000 x 5460, INT8:
// 24 us = 3.2 TB/s; one row of 4096: 3.6 us, launch and two exchanges between waves.
#include "common.h"

typedef u32 u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// 16 channels from c on of a row of K; zeros behind the row.  Rows may start at any element.
__device__ __forceinline__ void rn_load16(const uint16_t* x, int c, int K, float (&v)[16]) {
  if (c + 16 <= K) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4_any w = *reinterpret_cast<const u32x4_any*>(x + c + 8 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[8 * i + 2 * e] = __uint_as_float(w[e] << 16);
        v[8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = c + e < K ? bl_bf16_to_f32(x[c + e]) : 0.0f;
  }
}
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void rn_load16(const float* x, int c, int K, float (&v)[16]) {
  if (c + 16 <= K) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4_any w = *reinterpret_cast<const f32x4_any*>(x + c + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * i + e] = w[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = c + e < K ? x[c + e] : 0.0f;
  }
}
__device__ __forceinline__ void rn_store16(uint16_t* x, int c, int K, const float (&v)[16]) {
  if (c + 16 <= K) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u32x4_any w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = bl_pack_bf16(v[8 * i + 2 * e], v[8 * i + 2 * e + 1]);
      *reinterpret_cast<u32x4_any*>(x + c + 8 * i) = w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (c + e < K) x[c + e] = bl_f32_to_bf16_any(v[e]);
  }
}
__device__ __forceinline__ void rn_store16(float* x, int c, int K, const float (&v)[16]) {
  if (c + 16 <= K) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4_any w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = v[4 * i + e];
      *reinterpret_cast<f32x4_any*>(x + c + 4 * i) = w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (c + e < K) x[c + e] = v[e];
  }
}
__device__ __forceinline__ float rn_round(float v, const uint16_t*) { return bl_bf16_to_f32(bl_f32_to_bf16_any(v)); }
__device__ __forceinline__ float rn_round(float v, const float*) { return v; }

// sum and maximum (of numbers that are not negative; a NaN is the largest) over a workgroup of NT threads, in every thread; `red` is
// used once a call
template <int NT>
__device__ __forceinline__ double rn_sum(double v, double* red) {
  v = bl_wave_sum_f64_dpp(v);
  if (NT == 64) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) t += red[w];
  return t;
}
template <int NT>
__device__ __forceinline__ float rn_max(float x, u32* red) {
  u32 v = bl_wave_max_u32(__float_as_uint(x) & 0x7FFFFFFFu);
  if (NT == 64) return __uint_as_float(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = max(v, red[w]);
  return __uint_as_float(v);
}

enum { RN_INT4 = 0, RN_MX6 = 1, RN_INT8 = 2 };

// E3M2 code of an INT4 level (an integer value): its exponent field less 124 and its two top mantissa bits, the sign in bit 5
__device__ __forceinline__ u32 rn_e3m2(float p) {
  const u32 b = __float_as_uint(p);
  const u32 c = (((b >> 21) & 31u) ^ 16u) | ((b >> 26) & 32u);
  return (b << 1) != 0u ? c : 0u;
}

template <typename T, int NT, int NV, int OUT>
__global__ __launch_bounds__(NT) void rmsnorm_quantize_kernel(const T* __restrict__ X, const T* __restrict__ R, int64_t M, int K, int Kp,
                                                              const float* __restrict__ gamma, float norm_eps, float eps,
                                                              T* __restrict__ H, float* __restrict__ rstd_out,
                                                              u32* __restrict__ q_out, float* __restrict__ scale_out) {
  __shared__ double red0[NT / 64], red1[NT / 64];
  __shared__ u32 redm[NT / 64];
  // block-ordered codes: tokens that share lines go to one XCD, as in the quantizer
  int64_t m = blockIdx.x;
  if (OUT == RN_MX6) {
    m = (int64_t)(blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    if (m >= M) return;                          // (whole workgroup, before any barrier)
  }
  float h[NV][16];
  double ss = 0.0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 16 * (threadIdx.x + NT * j);
    rn_load16(X + m * K, c, K, h[j]);
    if (R) {
      float r[16];
      rn_load16(R + m * K, c, K, r);
#pragma unroll
      for (int e = 0; e < 16; ++e) h[j][e] = rn_round(h[j][e] + r[e], X);
    }
    if (H && c < K) rn_store16(H + m * K, c, K, h[j]);
#pragma unroll
    for (int e = 0; e < 16; ++e) ss = __builtin_fma((double)h[j][e], (double)h[j][e], ss);
  }
  ss = rn_sum<NT>(ss, red0);
  const float rstd = (float)(1.0 / sqrt(ss / (double)K + (double)norm_eps));
  if (rstd_out && threadIdx.x == 0) rstd_out[m] = rstd;
  double sum = 0.0;
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 16 * (threadIdx.x + NT * j);
    float g[16];
    rn_load16(gamma, c, K, g);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      h[j][e] = (h[j][e] * rstd) * g[e];
      if (OUT == RN_INT8) top = __builtin_elementwise_maximum(top, fabsf(h[j][e]));      // (a NaN stays, as in the quantizer)
      else sum += (double)fabsf(h[j][e]);
    }
  }
  float s, d;
  if (OUT == RN_INT8) {
    top = rn_max<NT>(top, redm);
    s = 127.0f / (top + eps);
    d = top / 127.0f;
  } else {
    sum = rn_sum<NT>(sum, red1);
    const float beta = (float)(sum / (double)K), sqrt7 = 2.6457512f;   // float32(sqrt(7))
    s = sqrt7 / (beta + eps);
    d = beta / sqrt7;
  }
  if (threadIdx.x == 0) scale_out[m] = d;

#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int hu = threadIdx.x + NT * j;         // half unit: channels 16 hu ..
    if (hu >= Kp / 16) continue;
    if (OUT == RN_INT8) {
      uint4 w;
      u32* ww = &w.x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ww[i] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) ww[i] |= ((u32)(int)fminf(fmaxf(rintf(h[j][4 * i + e] * s), -128.0f), 127.0f) & 255u) << (8 * e);
      }
      reinterpret_cast<uint4*>(q_out + m * (int64_t)(Kp / 4))[hu] = w;
    } else {
      float p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] = fminf(fmaxf(rintf(h[j][e] * s), -8.0f), 7.0f);
      if (OUT == RN_INT4) {                      // byte b of a word: level b, level 4 + b
        uint2 w;
        u32* ww = &w.x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ww[i] = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            ww[i] |= (((u32)(int)p[8 * i + e] & 15u) | (((u32)(int)p[8 * i + 4 + e] & 15u) << 4)) << (8 * e);
        }
        reinterpret_cast<uint2*>(q_out + m * (int64_t)(Kp / 8))[hu] = w;
      } else {                                   // 96 bits of the unit's stream
        u32 w3[3] = {0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const u32 c = rn_e3m2(p[e]);
          const int bit = 6 * e;
          w3[bit >> 5] |= c << (bit & 31);
          if ((bit & 31) > 26) w3[(bit >> 5) + 1] |= c >> (32 - (bit & 31));
        }
        const int r = (int)(m & 31), kb = hu >> 3, u = (hu >> 1) & 3;
        unsigned char* b = reinterpret_cast<unsigned char*>(q_out) + ((m >> 5) * (int64_t)(Kp / 128) + kb) * (32 * 96);
        u32* pp = reinterpret_cast<u32*>(b + r * 64 + ((u ^ ((r >> 2) & 3)) << 4));
        if ((hu & 1) == 0) {
          pp[0] = w3[0]; pp[1] = w3[1]; pp[2] = w3[2];
        } else {
          pp[3] = w3[0];
          u32* qq = reinterpret_cast<u32*>(b + 2048 + r * 32 + ((u ^ ((r >> 3) & 3)) << 3));
          qq[0] = w3[1]; qq[1] = w3[2];
        }
      }
    }
  }
}

template <typename T, int OUT>
static int rn_launch(const void* X, const void* R, int64_t M, int K, const float* gamma, float norm_eps, float eps, void* H,
                     float* rstd, void* q, float* scale, hipStream_t s) {
  const int Kp = (int)bl_round_up(K, BL_KPAD);
  const unsigned grid = (unsigned)(OUT == RN_MX6 ? bl_round_up(M, 8) : M);
#define RN_GO(NT, NV) \
  rmsnorm_quantize_kernel<T, NT, NV, OUT><<<grid, NT, 0, s>>>((const T*)X, (const T*)R, M, K, Kp, gamma, norm_eps, eps, (T*)H, rstd, (u32*)q, scale)
  if (Kp <= 1024) RN_GO(64, 1);
  else if (Kp <= 4096) RN_GO(256, 1);
  else if (Kp <= 8192) RN_GO(256, 2);
  else if (Kp <= 16384) RN_GO(512, 2);
  else RN_GO(512, 4);
#undef RN_GO
  BL_HIP_CHECK_LAUNCH();
  return BL_OK;
}

int bl_launch_rmsnorm_quantize(const void* X, const void* R, bl_dtype dt, int64_t M, int64_t K, const float* gamma, float norm_eps,
                               bl_act_mode mode, float eps, void* H, float* rstd, void* q, float* scale, hipStream_t s) {
#define RN_MODE(T)                                                                                                              \
  (mode == BL_ACT_TOPK_INT8_ABSMAX ? rn_launch<T, RN_INT8>(X, R, M, (int)K, gamma, norm_eps, eps, H, rstd, q, scale, s)         \
   : mode == BL_ACT_INT4_ABSMEAN_MX6 ? rn_launch<T, RN_MX6>(X, R, M, (int)K, gamma, norm_eps, eps, H, rstd, q, scale, s)        \
                                     : rn_launch<T, RN_INT4>(X, R, M, (int)K, gamma, norm_eps, eps, H, rstd, q, scale, s))
  return dt == BL_BF16 ? RN_MODE(uint16_t) : RN_MODE(float);
#undef RN_MODE
}

// ---------------------------------------------------------------- gradient
// With xh = h * rstd, a = dY * gamma:  dX = dH + rstd (a - xh mean(a xh)),  dgamma = sum over tokens of dY * xh.
// HBM's to bound: 8 bytes a bfloat16 channel (6 without dH); 4096 x 3200: 28 us = 3.7 TB/s, waves waiting for three quarters of their time
// (a token's loads start behind the sum of the one before).  A workgroup walks over its share of the tokens and keeps its sums of dgamma in
// registers; the partial sums are added in a fixed order by the second kernel.
#define RN_GROUPS 512

template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT) void rmsnorm_backward_kernel(const T* __restrict__ dY, const T* __restrict__ H,
                                                              const float* __restrict__ rstd, const float* __restrict__ gamma,
                                                              const T* __restrict__ dH, int64_t M, int K, T* __restrict__ dX,
                                                              float* __restrict__ part) {
  __shared__ double red[2][NT / 64];
  constexpr bool KEEP = NV < 4;                  // gamma in registers; four turns have no room (470 spilled): read a token
  float ga[KEEP ? NV : 1][16], dg[NV][16];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (KEEP) rn_load16(gamma, 16 * (threadIdx.x + NT * j), K, ga[KEEP ? j : 0]);
#pragma unroll
    for (int e = 0; e < 16; ++e) dg[j][e] = 0.0f;
  }
  int turn = 0;
  for (int64_t m = blockIdx.x; m < M; m += gridDim.x, turn ^= 1) {
    const float rs = rstd[m];
    float xh[NV][16], a[NV][16], sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = 16 * (threadIdx.x + NT * j);
      rn_load16(H + m * K, c, K, xh[j]);
      rn_load16(dY + m * K, c, K, a[j]);
      if (!KEEP) rn_load16(gamma, c, K, ga[0]);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        xh[j][e] *= rs;
        dg[j][e] = __builtin_fmaf(a[j][e], xh[j][e], dg[j][e]);
        a[j][e] *= ga[KEEP ? j : 0][e];
        sum = __builtin_fmaf(a[j][e], xh[j][e], sum);
      }
    }
    const float c0 = (float)(rn_sum<NT>((double)sum, red[turn]) / (double)K);    // (two buffers: one barrier a token)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = 16 * (threadIdx.x + NT * j);
      if (c >= K) continue;
      float o[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] = rs * (a[j][e] - xh[j][e] * c0);
      if (dH) {
        float d[16];
        rn_load16(dH + m * K, c, K, d);
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] += d[e];
      }
      rn_store16(dX + m * K, c, K, o);
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 16 * (threadIdx.x + NT * j);
    if (c < K) rn_store16(part + blockIdx.x * (int64_t)K, c, K, dg[j]);
  }
}

// A workgroup: 64 channels, its 16 waves every 16th partial sum each (512 x 3200 partial sums: 36 us with four waves, 4 with sixteen).  The order of the additions is fixed.
#define RN_SUM_WAVES 16
__global__ __launch_bounds__(64 * RN_SUM_WAVES) void rmsnorm_dgamma_kernel(const float* __restrict__ part, int groups, int K,
                                                                           float* __restrict__ dgamma) {
  __shared__ double red[RN_SUM_WAVES][64];
  const int l = threadIdx.x & 63, c = blockIdx.x * 64 + l, w = threadIdx.x >> 6;
  double s = 0.0;
  if (c < K) {
#pragma unroll 8
    for (int g = w; g < groups; g += RN_SUM_WAVES) s += (double)part[(int64_t)g * K + c];
  }
  red[w][l] = s;
  __syncthreads();
  if (w == 0 && c < K) {
#pragma unroll
    for (int i = 1; i < RN_SUM_WAVES; ++i) s += red[i][l];
    dgamma[c] = (float)s;
  }
}

static int64_t rn_groups(int64_t M) { return M < RN_GROUPS ? M : RN_GROUPS; }
size_t bl_rmsnorm_backward_ws_bytes(int64_t M, int64_t K) { return (size_t)(rn_groups(M) * K * 4); }

int bl_launch_rmsnorm_backward(const void* dY, const void* H, const float* rstd, const float* gamma, const void* dH, bl_dtype dt,
                               int64_t M, int64_t K64, void* dX, float* dgamma, void* ws, hipStream_t s) {
  const int K = (int)K64;
  const unsigned groups = (unsigned)rn_groups(M);
#define RN_GO(T, NT, NV) \
  rmsnorm_backward_kernel<T, NT, NV><<<groups, NT, 0, s>>>((const T*)dY, (const T*)H, rstd, gamma, (const T*)dH, M, K, (T*)dX, (float*)ws)
#define RN_K(T)                              \
  do {                                       \
    if (K <= 1024) RN_GO(T, 64, 1);          \
    else if (K <= 4096) RN_GO(T, 256, 1);    \
    else if (K <= 8192) RN_GO(T, 512, 1);    \
    else if (K <= 16384) RN_GO(T, 512, 2);   \
    else RN_GO(T, 512, 4);                   \
  } while (0)
  if (dt == BL_BF16) RN_K(uint16_t); else RN_K(float);
#undef RN_K
#undef RN_GO
  BL_HIP_CHECK_LAUNCH();
  rmsnorm_dgamma_kernel<<<(unsigned)((K + 63) / 64), 64 * RN_SUM_WAVES, 0, s>>>((const float*)ws, (int)groups, K, dgamma);
  BL_HIP_CHECK_LAUNCH();
  return BL_OK;
}
