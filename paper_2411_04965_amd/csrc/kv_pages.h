// Pages of the low-bit key / value cache (format: the public header): shared by the kernels that write, read back and attend
// over them.
#pragma once
#include "common.h"

#define KP_TOKENS 128            // BL_KV_PAGE: what one block-float matrix instruction contracts over
#define KP_MAX_D 256

// Bytes of one head in a page: key codes, value codes (32 channels or tokens = 12 bytes), 128 key scales, 128 value scales, the
// lowest magnitude bits of a first token (a word per 32 channels, keys then values, in 128 bytes).
__host__ __device__ static inline int kp_units(int D) { return (D + 31) >> 5; }
__host__ __device__ static inline int kp_code_bytes(int U) { return KP_TOKENS * 12 * U; }
__host__ __device__ static inline int kp_head_bytes(int U) { return 2 * kp_code_bytes(U) + 2 * KP_TOKENS * 4 + 128; }
__host__ __device__ static inline int kp_scale_off(int U) { return 2 * kp_code_bytes(U); }
__host__ __device__ static inline int kp_low_off(int U) { return 2 * kp_code_bytes(U) + 2 * KP_TOKENS * 4; }
// Key codes of token t stand in slot t with bits 2, 3 and 4, 5 exchanged: the order in which the first product's results, used
// as the second product's eight-bit operand, meet values in token order.
__host__ __device__ static inline int kp_slot(int t) { return (t & 0x43) | ((t & 0x0C) << 2) | ((t & 0x30) >> 2); }

// A batch: sequence s has the rows q_start[s] .. q_start[s + 1] - 1 of the call's T, its last row at position kv_len[s] - 1.
// Nothing read from these arrays is trusted: rows are clamped to T, pages outside the pool count as absent.
struct KvBatch {
  const int32_t* q_start;        // [n_seqs + 1]
  const int32_t* kv_len;         // [n_seqs]
  const int32_t* table;          // [n_seqs, max_pages]
  int n_seqs, max_pages, n_pages, T;
};

struct KvSeq {
  int s, q0, n;                  // sequence, its first row, its rows
  int64_t len, pos0;             // length with the new tokens, position of the first of them (negative if n > len)
};

// A batch's numbers at a place that is the same for a whole wave, through the scalar cache (nothing writes them while a kernel runs).
// As vector loads they would be waited for behind everything a wave has on its way: loads come back in order.
__device__ __forceinline__ int kp_scalar(const int32_t* p, int64_t i) {
  return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)p)[i];
}

// Work items are dealt to sequences without the host knowing their lengths: sequence s owns the items from
// floor(q_start[s] * mul / 2^shift) + per * s on.  That start grows by at least floor(rows * mul / 2^shift) + per, so every
// sequence has enough items and the total is known on the host.
__device__ __forceinline__ int64_t kp_first_item(const KvBatch& b, int s, int mul, int shift, int per) {
  const int q = min(max(b.q_start[s], 0), b.T);
  return (((int64_t)q * mul) >> shift) + (int64_t)per * s;
}
// The sequence that owns `item` (64 candidates a step, every lane of a wave takes part), and the item's number in it (-1: none).
__device__ __forceinline__ int64_t kp_find(const KvBatch& b, int64_t item, int mul, int shift, int per, KvSeq& q) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = b.n_seqs;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int i = lane * step;
    const bool le = i < n && kp_first_item(b, lo + i, mul, shift, per) <= item;
    const unsigned long long no = ~__ballot(le);
    const int ones = no ? __builtin_ctzll(no) : 64;
    const int at = max(ones - 1, 0) * step;
    lo += at;
    n = min(step, n - at);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  q.s = lo;
  q.q0 = min(max(kp_scalar(b.q_start, lo), 0), b.T);
  q.n = min(max(kp_scalar(b.q_start, lo + 1), 0), b.T) - q.q0;
  q.len = kp_scalar(b.kv_len, lo);
  q.pos0 = q.len - q.n;
  const int64_t local = item - ((((int64_t)q.q0 * mul) >> shift) + (int64_t)per * lo);
  return q.n > 0 && local >= 0 ? local : -1;
}

// Words A, B, C of 32 codes -> 32 E2M1 nibbles (code i in nibble i % 8 of word i / 8).  A code's two magnitude bits m are the
// nibble of the value m / 2, so nothing but shifts and masks is needed: 11 instructions for 32 codes (a sign word cleared of the
// bits between, then one bit-wise choice a nibble word).
__device__ __forceinline__ void kp_expand(u32 A, u32 B, u32 C, u32 (&o)[4]) {
  u32 even = C & 0xAAAAAAAAu, odd = (C << 1) & 0xAAAAAAAAu;
  asm("" : "+v"(even), "+v"(odd));                     // (known bits would turn the choices back into two instructions each)
  auto choose = [](u32 mag, u32 sign) { return (mag & 0x33333333u) | (sign & 0xCCCCCCCCu); };
  o[0] = choose(A, even);
  o[1] = choose(A >> 2, odd);
  o[2] = choose(B, even << 2);
  o[3] = choose(B >> 2, odd << 2);
}
// bit of code i in C and in a word of lowest magnitude bits
__host__ __device__ __forceinline__ int kp_sign_bit(int i) { return 4 * (i & 7) + 3 - (i >> 3); }
__host__ __device__ __forceinline__ int kp_mag_bit(int i) { return 4 * (i & 7) + 2 * ((i >> 3) & 1); }

// Rotary position embedding of channel c of a head: channels c and c + D / 2 are a pair; table row: cosines, then sines.
// Two multiplies and one addition in float32, not fused.
__device__ __forceinline__ float kp_rotate(float x, float partner, const float* row, int c, int half) {
  const int p = c < half ? c : c - half;
  const float cs = row[p], sn = row[half + p];
  return c < half ? x * cs - partner * sn : x * cs + partner * sn;
}
