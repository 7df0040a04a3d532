// Rotary positions of their own: the tables of a scaled rotation, and rotation
// with cache append at given positions and slots.
#include "hs_device.h"
#include "hs_kernels.h"

namespace hs {

// ------------------------------------------------------------------- tables
//
// Entry (p, i): cos and sin of p w_i, times a magnitude. The angle is formed in
// turns in float64 (p w_i / 2 pi; at position 131072 a float32 angle would be
// off by 0.008 rad) and whole quarter turns are taken off before the rounding
// to float32, which leaves at most pi / 4 for the two Taylor polynomials (their
// first dropped terms are below 2e-9 and 2e-10). Bound by the stores: 8 bytes per
// entry.

struct RopeFreq {
  double turns[64];  // w_i / 2 pi
};

__device__ __forceinline__ void sincos_turns(double t, float m, float& c, float& s) {
  const double t4 = t * 4.0, k = __builtin_rint(t4);
  const float x = (float)((t4 - k) * 1.57079632679489661923);  // |x| <= pi / 4
  const int q = (int)k & 3;
  const float z = x * x;
  float sp = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
  sp = fmaf(z, sp, 8.33333333e-3f);
  sp = fmaf(z, sp, -1.66666667e-1f);
  sp = fmaf(x * z, sp, x);
  float cp = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
  cp = fmaf(z, cp, -1.38888889e-3f);
  cp = fmaf(z, cp, 4.16666667e-2f);
  cp = fmaf(z, cp, -0.5f);
  cp = fmaf(z, cp, 1.0f);
  const float a = q & 1 ? sp : cp, b = q & 1 ? cp : sp;
  c = ((q + 1) & 2 ? -a : a) * m;
  s = (q & 2 ? -b : b) * m;
}

// A thread takes four neighbouring pairs of one position (half % 4 == 0).
__global__ __launch_bounds__(256) void rope_tables_kernel(float* cos_t, float* sin_t, int max_pos,
                                                          int half, RopeFreq f, float magnitude) {
  const int q4 = half / 4;
  const int64_t n = (int64_t)max_pos * q4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int p = (int)(i / q4), j = (int)(i % q4) * 4;
  float c[4], s[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) sincos_turns((double)p * f.turns[j + e], magnitude, c[e], s[e]);
  *reinterpret_cast<float4*>(cos_t + i * 4) = make_float4(c[0], c[1], c[2], c[3]);
  *reinterpret_cast<float4*>(sin_t + i * 4) = make_float4(s[0], s[1], s[2], s[3]);
}

hipError_t rope_tables(float* cos_t, float* sin_t, int max_pos, int half, const double* turns,
                       float magnitude, hipStream_t s) {
  if (max_pos < 1 || half < 4 || half > 64 || (half % 4) ||
      (((uintptr_t)cos_t | (uintptr_t)sin_t) & 15))
    return hipErrorInvalidValue;
  RopeFreq f;
  for (int i = 0; i < 64; ++i) f.turns[i] = i < half ? turns[i] : 0.0;
  const int64_t n = (int64_t)max_pos * (half / 4);
  if ((n + 255) / 256 >= (1ll << 31)) return hipErrorInvalidValue;
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
// byte written once. One thread takes one chunk pair of one head of one token.

template <bool HALF>
__global__ __launch_bounds__(256) void rope_kv_at_kernel(RopeKvAtArgs a) {
  const int pairs = a.D / 16, rot_pairs = a.rot / 16;
  const int heads = a.n_heads + 2 * a.n_kv_heads;
  const int t = blockIdx.x, i = blockIdx.y * 256 + threadIdx.x;
  if (i >= heads * pairs) return;
  const int pos = a.pos[t];
  if (pos < 0 || pos >= a.max_pos) return;  // an empty row
  const int head = i / pairs, j = i % pairs;
  const int slot = a.slot[t];
  const int blk = slot >> 4;  // negative slots give a negative block
  const bool cached = blk >= 0 && blk < a.pool_blocks;
  const bool value = head >= a.n_heads + a.n_kv_heads;
  const bool turned = j < rot_pairs && !value;
  const int e0 = HALF && j < rot_pairs ? 8 * j : 16 * j;
  const int e1 = HALF && j < rot_pairs ? a.rot / 2 + 8 * j : 16 * j + 8;
  const bf16_t* x = a.qkv + (int64_t)t * a.ldqkv + head * a.D;
  pack8 u = ld16(x + e0), v = ld16(x + e1);
  if (turned) {
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
  if (head < a.n_heads) {
    bf16_t* y = a.q_out + (int64_t)t * a.ldq + head * a.D;
    st16(y + e0, u);
    st16(y + e1, v);
    return;
  }
  const int kv = value ? 1 : 0, kh = head - a.n_heads - kv * a.n_kv_heads;
  if (!value && a.k_out) {
    bf16_t* y = a.k_out + (int64_t)t * a.ldk + kh * a.D;
    st16(y + e0, u);
    st16(y + e1, v);
  }
  if (cached) {
    bf16_t* y = a.pool + (((int64_t)blk * 2 + kv) * a.n_kv_heads + kh) * 16 * a.D + (slot & 15) * a.D;
    st16(y + e0, u);
    st16(y + e1, v);
  }
}

hipError_t rope_kv_at(const RopeKvAtArgs& a, hipStream_t s) {
  if (a.T <= 0) return hipSuccess;
  const int64_t items = (int64_t)(a.n_heads + 2 * a.n_kv_heads) * (a.D / 16);
  if ((a.D != 64 && a.D != 128) || a.rot < 16 || a.rot > a.D || (a.rot % 16) ||
      (a.ldqkv % 8) || (a.ldq % 8) || (a.ldk % 8) || (items + 255) / 256 > 65535)
    return hipErrorInvalidValue;
  const dim3 grid(a.T, (unsigned)((items + 255) / 256));
  if (a.interleaved)
    hipLaunchKernelGGL(rope_kv_at_kernel<false>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(rope_kv_at_kernel<true>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hs
