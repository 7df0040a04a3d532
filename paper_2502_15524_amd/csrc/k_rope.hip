// Rotary positions of their own: the tables of a scaled rotation, and rotation
// with cache append at given positions and slots.
#include "hs_device.h"
#include "hs_kernels.h"

namespace hs {

// ------------------------------------------------------------------- tables
//
// Entry (p, i): cos and sin of p w_i, times a magnitude. The angle is formed in
// turns as a 64-bit fraction, p times w_i / 2 pi modulo 1 (at position 131072 a float32
// angle would be off by 0.008 rad), and whole quarter turns are taken off before the
// rounding to float32, which is of all 64 bits, so that a small sine has as many good bits as a
// large one. That leaves at most half a quarter, y, for the two Taylor polynomials of pi / 2 y (their
// first dropped terms are below 2e-9 and 2e-10). Bound by
// the stores, 8 bytes per entry: 131072 positions of 64 pairs 12.0 us, 5.6 TB/s, on MI355X
// (12.3 with the angles in float64, 11.9 of 32 bits of the fraction, whose least sines were 0.4 %
// off and more; a fill of the same bytes takes 9.8).

struct RopeFreq {
  uint64_t turns[64];  // w_i / 2 pi in units of 2^-64
};

__device__ __forceinline__ void sincos_turns(uint64_t turns, float m, float& c, float& s) {
  constexpr double H = 1.57079632679489661923;
  constexpr float h = (float)H, h_rest = (float)(H - (double)h);
  const uint32_t up = (uint32_t)(turns >> 32), low = (uint32_t)turns << 2;
  const uint32_t q = (up + 0x20000000u) >> 30;
  // the part of a quarter left, 2^32 big + rest in units of 2^-64 (big saturates half a unit early)
  const int big = __builtin_elementwise_add_sat((int)(turns >> 30), (int)(low >> 31)), rest = (int)low;
  const float y = fmaf((float)big, 0x1p-32f, (float)rest * 0x1p-64f);  // |y| <= 1 / 2
  const float z = y * y;
  float sp = fmaf(z, (float)(H * H * H * H * H * H * H * H * H / 362880), (float)(-H * H * H * H * H * H * H / 5040));
  sp = fmaf(z, sp, (float)(H * H * H * H * H / 120));
  sp = fmaf(z, sp, (float)(-H * H * H / 6));
  sp = fmaf(y, h, y * fmaf(z, sp, h_rest));
  float cp = fmaf(z, (float)(-H * H * H * H * H * H * H * H * H * H / 3628800), (float)(H * H * H * H * H * H * H * H / 40320));
  cp = fmaf(z, cp, (float)(-H * H * H * H * H * H / 720));
  cp = fmaf(z, cp, (float)(H * H * H * H / 24));
  cp = fmaf(z, cp, (float)(-H * H / 2));
  cp = fmaf(z, cp, 1.0f);
  const float a = q & 1 ? sp : cp, b = q & 1 ? cp : sp;
  // quarters 1 and 2 turn the cosine's sign, 2 and 3 the sine's
  c = __uint_as_float(__float_as_uint(a) ^ ((q + 1) << 30 & 0x80000000u)) * m;
  s = __uint_as_float(__float_as_uint(b) ^ (q << 30 & 0x80000000u)) * m;
}

// A thread takes four neighbouring pairs (half % 4 == 0) of four positions.
__global__ __launch_bounds__(256) void rope_tables_kernel(float* cos_t, float* sin_t, int max_pos,
                                                          int half, RopeFreq f, float magnitude) {
  const int q4 = half / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, p0 = i / q4 * 4;
  const int j = (int)(i % q4) * 4;
  if (p0 >= max_pos) return;
  uint64_t w[4], t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = f.turns[j + e];
    t[e] = w[e] * (uint64_t)p0;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (p0 + u >= max_pos) return;
    float c[4], s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sincos_turns(t[e], magnitude, c[e], s[e]);
      t[e] += w[e];
    }
    const int64_t to = (p0 + u) * half + j;
    *reinterpret_cast<float4*>(cos_t + to) = make_float4(c[0], c[1], c[2], c[3]);
    *reinterpret_cast<float4*>(sin_t + to) = make_float4(s[0], s[1], s[2], s[3]);
  }
}

hipError_t rope_tables(float* cos_t, float* sin_t, int max_pos, int half, const uint64_t* turns,
                       float magnitude, hipStream_t s) {
  if (max_pos < 1 || half < 4 || half > 64 || (half % 4) ||
      (((uintptr_t)cos_t | (uintptr_t)sin_t) & 15))
    return hipErrorInvalidValue;
  RopeFreq f;
  for (int i = 0; i < 64; ++i) f.turns[i] = i < half ? turns[i] : 0;
  const int64_t n = ((int64_t)max_pos + 3) / 4 * (half / 4);
  if (n >= (1ll << 32) - 256) return hipErrorInvalidValue;  // threads of a launch
  hipLaunchKernelGGL(rope_tables_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, cos_t,
                     sin_t, max_pos, half, f, magnitude);
  return hipGetLastError();
}

// ------------------------------------------------- rotation and cache append
//
// A head is D / 16 pairs of 16-byte chunks. Of a rotated pair the chunks hold
// the two partners of eight rotation pairs (half layout: elements 8 j and
// rot / 2 + 8 j; interleaved: 16 j and 16 j + 8); the pairs past the rotated part
// of a head and those of the value heads are copied as they are. Rotated in
// float32 with the two functions that every rotation of the library uses, one
// rounding to bf16. Bound by HBM: every input byte is read once, every output
// byte written once. A thread takes one chunk pair of one head of one token, whose values
// it requests before the position is known. MI355X: 8192 tokens of 32 + 8 heads with rows of
// keys 40.2 us, 5.5 TB/s; 1531 of 40 + 40 23.7 us (with two or four heads to a thread, which
// share the angles' loads, 41.9 and 43.6, 24.9 and 26.7).

template <bool HALF>
__device__ __forceinline__ void rotate_pair(pack8& u, pack8& v, const float* c, const float* s) {
  if constexpr (HALF) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a0 = lo_bf(u.w[w]), a1 = hi_bf(u.w[w]), b0 = lo_bf(v.w[w]), b1 = hi_bf(v.w[w]);
      u.w[w] = pack2bf(rope_first(a0, b0, c[2 * w], s[2 * w]),
                       rope_first(a1, b1, c[2 * w + 1], s[2 * w + 1]));
      v.w[w] = pack2bf(rope_second(a0, b0, c[2 * w], s[2 * w]),
                       rope_second(a1, b1, c[2 * w + 1], s[2 * w + 1]));
    }
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a0 = lo_bf(u.w[w]), b0 = hi_bf(u.w[w]), a1 = lo_bf(v.w[w]), b1 = hi_bf(v.w[w]);
      u.w[w] = pack2bf(rope_first(a0, b0, c[w], s[w]), rope_second(a0, b0, c[w], s[w]));
      v.w[w] = pack2bf(rope_first(a1, b1, c[4 + w], s[4 + w]),
                       rope_second(a1, b1, c[4 + w], s[4 + w]));
    }
  }
}

template <bool HALF>
__global__ __launch_bounds__(256) void rope_kv_at_kernel(RopeKvAtArgs a, int per_token) {
  const int pairs = a.D / 16;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int t = (int)(i / per_token), r = (int)(i - (int64_t)t * per_token), head = r / pairs, j = r % pairs;
  if (t >= a.T) return;
  const bool half_pair = HALF && j < a.rot / 16;
  const int e0 = half_pair ? 8 * j : 16 * j, e1 = half_pair ? a.rot / 2 + 8 * j : 16 * j + 8;
  const bf16_t* x = a.qkv + (int64_t)t * a.ldqkv + head * a.D;
  pack8 u = ld16(x + e0), v = ld16(x + e1);
  const int pos = a.pos[t], slot = a.slot[t];
  if (pos < 0 || pos >= a.max_pos) return;  // an empty row
  if (j < a.rot / 16 && head < a.n_heads + a.n_kv_heads) {
    const float* ct = a.cos_t + (int64_t)pos * (a.rot / 2) + 8 * j;
    const float* st = a.sin_t + (int64_t)pos * (a.rot / 2) + 8 * j;
    float c[8], s[8];
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 c4 = *reinterpret_cast<const float4*>(ct + e);
      const float4 s4 = *reinterpret_cast<const float4*>(st + e);
      c[e] = c4.x, c[e + 1] = c4.y, c[e + 2] = c4.z, c[e + 3] = c4.w;
      s[e] = s4.x, s[e + 1] = s4.y, s[e + 2] = s4.z, s[e + 3] = s4.w;
    }
    rotate_pair<HALF>(u, v, c, s);
  }
  const auto put = [&](bf16_t* y) {
    st16(y + e0, u);
    st16(y + e1, v);
  };
  if (head < a.n_heads) return put(a.q_out + (int64_t)t * a.ldq + head * a.D);
  const int kh = head - a.n_heads;  // values: from n_kv_heads on, as the pool has them
  if (kh < a.n_kv_heads && a.k_out) put(a.k_out + (int64_t)t * a.ldk + kh * a.D);
  const int blk = slot >> 4;  // negative slots give a negative block
  if (blk >= 0 && blk < a.pool_blocks)
    put(a.pool + ((int64_t)blk * 2 * a.n_kv_heads + kh) * 16 * a.D + (slot & 15) * a.D);
}

hipError_t rope_kv_at(const RopeKvAtArgs& a, hipStream_t s) {
  if (a.T <= 0) return hipSuccess;
  if ((a.D != 64 && a.D != 128) || a.rot < 16 || a.rot > a.D || (a.rot % 16) ||
      (a.ldqkv % 8) || (a.ldq % 8) || (a.ldk % 8))
    return hipErrorInvalidValue;
  const int64_t per = (int64_t)(a.n_heads + 2 * a.n_kv_heads) * (a.D / 16), n = (a.T * per + 255) / 256;
  if (per >= (1ll << 31) || n >= (1ll << 24)) return hipErrorInvalidValue;  // threads of a launch
  if (a.interleaved)
    hipLaunchKernelGGL(rope_kv_at_kernel<false>, dim3((unsigned)n), dim3(256), 0, s, a, (int)per);
  else
    hipLaunchKernelGGL(rope_kv_at_kernel<true>, dim3((unsigned)n), dim3(256), 0, s, a, (int)per);
  return hipGetLastError();
}

}  // namespace hs
