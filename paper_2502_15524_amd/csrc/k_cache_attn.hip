// Decode attention over a paged cache whose sequences share a prefix, and with
// the weight that every cached token received.
//
// A sequence's tokens are the prefix's, then its own. They are taken in slots of
// whole blocks: slot v of the prefix's blocks, then of the sequence's own; the
// slots past a block's last token hold nothing. One workgroup takes 128 slots of
// one (sequence, kv head), two blocks per wave, and leaves for each query head
// the unnormalised P V, the largest score (log2 domain) and the sum of
// exp2(score - largest); a second kernel merges the splits and, where weights
// are asked for, turns the stored scores into probabilities with the merged
// statistics. All of it in float32; the probabilities are rounded to bf16 for
// the second matrix product only (an error of half a bf16 step, as the output's
// own rounding), their sum and the weights are of the unrounded ones.
#include "hs_device.h"
#include "hs_kernels.h"

#include <algorithm>

namespace hs {

namespace {
constexpr int kSplit = 128;
typedef short s16x4_v __attribute__((ext_vector_type(4)));

// The block that holds slots 16 j .. 16 j + 15 of sequence b, and how many
// of them are tokens. Entries that name no block of the pool hold no tokens.
struct Block {
  int at, n;
};
__device__ __forceinline__ Block block_of(const CacheAttnArgs& a, int b, int j, int ctx) {
  Block r{-1, 0};
  if (j < a.lead_blocks) {
    r.at = a.prefix[j];
    r.n = min(16, a.prefix_len - 16 * j);
  } else {
    const int o = j - a.lead_blocks;
    if (16 * o < ctx) {
      r.at = a.block_table[(int64_t)b * a.max_blocks + o];
      r.n = min(16, ctx - 16 * o);
    }
  }
  if (r.at < 0 || r.at >= a.pool_blocks) r = Block{0, 0};
  return r;
}

// Merged statistics of a query head of a sequence: the splits' largest score
// and the sum relative to it. Called by a whole wave; the order is fixed.
__device__ __forceinline__ void merge_ml(const float* ml, int n, float& M, float& L) {
  const int lane = threadIdx.x & 63;
  M = -INFINITY;
  for (int s = lane; s < n; s += 64) M = fmaxf(M, ml[2 * s]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  L = 0.f;
  for (int s = lane; s < n; s += 64) {
    const float m = ml[2 * s];
    if (m != -INFINITY) L += ml[2 * s + 1] * fast_exp2(m - M);
  }
  L = wave_sum(L);
}

// Splits of sequence b that hold anything.
__device__ __forceinline__ int splits_of(const CacheAttnArgs& a, int ctx) {
  return min(a.splits, (a.lead_blocks * 16 + ctx + kSplit - 1) / kSplit);
}
__device__ __forceinline__ int ctx_of(const CacheAttnArgs& a, int b) {
  return min(max(a.ctx[b], 0), a.max_ctx);
}
}  // namespace

// S^T = K Q^T and O^T = V^T P^T with 16x16x32 MFMAs: keys on the rows, the G query
// heads of the kv head on the columns (the other columns zero). Lane (r, g) =
// (lane % 16, lane / 16) ends with the scores of keys 4 g .. 4 g + 3 of each block
// for query head r, which are the second product's B operand as they are; its
// V^T fragments come from transposing LDS reads. Keys and values are read in
// whole rows, all of them requested before the first is used, and staged
// through the wave's own LDS buffer, the keys first, then the values over them.
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4))) void cache_attn_kernel(
    CacheAttnArgs a, float scale_log2) {
  constexpr int KS = D / 32, DT = D / 16, CH = D / 8;
  constexpr int RPL = 64 / CH;    // rows per load instruction
  constexpr int NL = 16 / RPL;    // load instructions per block
  constexpr int LV = D + 16;      // padded row: the transposing reads on distinct banks
  __shared__ __attribute__((aligned(16))) bf16_t sV[4][32 * LV];
  __shared__ float s_ml[4][16][2];
  static_assert(16 * D * 4 <= 32 * LV * 2, "a wave's partial fits its buffer");
  const auto s_acc = [&](int w) { return reinterpret_cast<float*>(sV[w]); };

  const int split = blockIdx.x / a.n_kv_heads, kh = blockIdx.x - split * a.n_kv_heads;
  const int b = blockIdx.y, G = a.G;
  const int ctx = ctx_of(a, b);
  if (split >= splits_of(a, ctx) && split > 0) return;  // uniform across the workgroup
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int fr = lane & 15, g = lane >> 4;
  const int64_t head_stride = (int64_t)16 * D, kv_stride = a.n_kv_heads * head_stride;
  const bf16_t* qrow = a.q + (int64_t)b * a.ldq + (int64_t)kh * G * D;
  const int crow = lane / CH, cch = lane % CH;

  Block blk[2];
  pack8 ck[2][NL], cv[2][NL], qf[KS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    blk[t] = block_of(a, b, split * (kSplit / 16) + wave * 2 + t, ctx);
    const bf16_t* base = a.pool + (int64_t)blk[t].at * 2 * kv_stride + kh * head_stride;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = RPL * i + crow;
      const bf16_t* krow = base + r * D + cch * 8;
      ck[t][i] = r < blk[t].n ? ld16_nt(krow) : zero8();
      cv[t][i] = r < blk[t].n ? ld16_nt(krow + kv_stride) : zero8();
    }
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = fr < G ? ld16(qrow + fr * D + ks * 32 + g * 8) : zero8();
  bf16_t* sv = sV[wave];
  pack8 kf[2][KS];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < NL; ++i) st16(sv + (16 * t + RPL * i + crow) * LV + cch * 8, ck[t][i]);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[t][ks] = ld16(sv + (16 * t + fr) * LV + ks * 32 + g * 8);
  asm volatile("" ::: "memory");  // the key reads before the value stores (one wave's LDS operations run in order)
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < NL; ++i) st16(sv + (16 * t + RPL * i + crow) * LV + cch * 8, cv[t][i]);

  f32x4_v s[2];
  float m = -INFINITY;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    s[t] = f32x4_v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[t][ks]), as_bf16x8(qf[ks]), s[t], 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[t][j] = 4 * g + j < blk[t].n ? s[t][j] * scale_log2 : -INFINITY;
      m = fmaxf(m, s[t][j]);
    }
    // the scores of the sequence's own tokens, for their weights
    const int own = (split * (kSplit / 16) + wave * 2 + t - a.lead_blocks) * 16;
    if (a.scores && own >= 0 && own < ctx && fr < G)
      *reinterpret_cast<f32x4_v*>(a.scores + ((int64_t)b * a.n_heads + kh * G + fr) * a.score_stride + own + 4 * g) = s[t];
  }
  m = fmaxf(m, __shfl_xor(m, 16, 64));
  m = fmaxf(m, __shfl_xor(m, 32, 64));
  const float m0 = m == -INFINITY ? 0.f : m;
  float l = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[t][j] = fast_exp2(s[t][j] - m0);
      l += s[t][j];
    }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  pack8 pk;
  pk.w[0] = pack2bf(s[0][0], s[0][1]);
  pk.w[1] = pack2bf(s[0][2], s[0][3]);
  pk.w[2] = pack2bf(s[1][0], s[1][1]);
  pk.w[3] = pack2bf(s[1][2], s[1][3]);
  const bf16x8_v pf = as_bf16x8(pk);
  asm volatile("" ::: "memory");  // the value stores before the fragment reads
  f32x4_v o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    const bf16_t* vp = sv + (4 * g + (fr >> 2)) * LV + dt * 16 + 4 * (fr & 3);
    const s16x4_v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4_v*)(vp));
    const s16x4_v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4_v*)(vp + 16 * LV));
    const bf16x8_v vb =
        __builtin_bit_cast(bf16x8_v, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, pf, f32x4_v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
  }
  asm volatile("" ::: "memory");  // the fragment reads before the partial goes over them
  if (fr < G) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<f32x4_v*>(s_acc(wave) + fr * D + dt * 16 + 4 * g) = o[dt];
    if (g == 0) {
      s_ml[wave][fr][0] = l == 0.f ? -INFINITY : m0;  // only NaN scores: a sum, of NaN, without a largest
      s_ml[wave][fr][1] = l;
    }
  }
  __syncthreads();
  for (int i = tid; i < G * D; i += 256) {
    const int gg = i / D, d = i % D;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, s_ml[w][gg][0]);
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = s_ml[w][gg][0];
      if (mw == -INFINITY) continue;
      const float f = fast_exp2(mw - M);
      L += s_ml[w][gg][1] * f;
      O += s_acc(w)[gg * D + d] * f;
    }
    const int64_t row = ((int64_t)b * a.n_heads + kh * G + gg) * a.splits + split;
    a.part_o[row * D + d] = O;
    if (d == 0) {
      a.part_ml[row * 2] = M;
      a.part_ml[row * 2 + 1] = L;
    }
  }
}

// The output of one (query head, sequence): 256 threads, four splits at a time.
template <int D>
__device__ __forceinline__ void merge_out(const CacheAttnArgs& a, int h, int b) {
  constexpr int W = 256 / D;
  __shared__ float s_o[256];
  const int ctx = ctx_of(a, b), n = splits_of(a, ctx);
  const int64_t row = ((int64_t)b * a.n_heads + h) * a.splits;
  const float* ml = a.part_ml + row * 2;
  float M, L;
  merge_ml(ml, n, M, L);
  const int d = threadIdx.x % D, w = threadIdx.x / D;
  float o = 0.f;
  for (int s = w; s < n; s += W) {
    const float m = ml[2 * s];
    if (m != -INFINITY) o += a.part_o[(row + s) * D + d] * fast_exp2(m - M);
  }
  s_o[threadIdx.x] = o;
  __syncthreads();
  if (w) return;
#pragma unroll
  for (int i = 1; i < W; ++i) o += s_o[i * D + d];
  // no token at all, or none with a score above -inf: zero
  a.out[(int64_t)b * a.ldo + h * D + d] = f2bf(L == 0.f ? 0.f : o / L);
}

// What a sequence's own tokens received: 1024 tokens of one kv head.
__device__ __forceinline__ void add_weights(const CacheAttnArgs& a, int kh, int b, int chunk) {
  __shared__ float s_m[16], s_r[16];
  const int ctx = ctx_of(a, b), n = splits_of(a, ctx), G = a.G;
  const int t0 = chunk * 1024;
  if (t0 >= ctx) return;  // uniform
  const int wave = threadIdx.x >> 6;
  for (int gg = wave; gg < G; gg += 4) {
    float M, L;
    merge_ml(a.part_ml + ((int64_t)b * a.n_heads + kh * G + gg) * a.splits * 2, n, M, L);
    s_m[gg] = M == -INFINITY ? 0.f : M;
    s_r[gg] = L == 0.f ? 0.f : 1.f / L;
  }
  __syncthreads();
  const int64_t row = ((int64_t)b * a.n_kv_heads + kh) * a.acc_stride;
  const float* sc = a.scores + ((int64_t)b * a.n_heads + kh * G) * a.score_stride;
  for (int t = t0 + threadIdx.x; t < min(t0 + 1024, ctx); t += 256) {
    float p = 0.f;
    for (int gg = 0; gg < G; ++gg) p += fast_exp2(sc[gg * a.score_stride + t] - s_m[gg]) * s_r[gg];
    if (t == ctx - 1) {
      if (a.pos) a.pos[row + t] = a.seen[b] - 1;
    } else {
      p += a.decay * a.acc[row + t];
    }
    a.acc_out[row + t] = p;
  }
}

// Workgroups [0, n_heads) of a sequence merge its outputs, the others its weights.
template <int D>
__global__ __launch_bounds__(256) void cache_attn_merge_kernel(CacheAttnArgs a) {
  const int i = blockIdx.x;
  if (i < a.n_heads) return merge_out<D>(a, i, blockIdx.y);
  add_weights(a, (i - a.n_heads) % a.n_kv_heads, blockIdx.y, (i - a.n_heads) / a.n_kv_heads);
}

CacheAttnPlan cache_attn_plan(int64_t B, int64_t n_heads, int64_t n_kv_heads, int64_t D,
                              int64_t prefix_len, int64_t max_ctx, bool weights) {
  CacheAttnPlan p;
  p.lead_blocks = (int)((prefix_len + 15) / 16);
  p.splits = std::max<int64_t>(1, (p.lead_blocks * 16ll + max_ctx + kSplit - 1) / kSplit);
  p.score_stride = weights ? (max_ctx + 15) / 16 * 16 : 0;
  p.part_o = 0;
  p.part_ml = p.part_o + B * n_heads * p.splits * D;
  p.scores = (p.part_ml + B * n_heads * p.splits * 2 + 3) / 4 * 4;
  p.floats = p.scores + B * n_heads * p.score_stride;
  return p;
}

hipError_t cache_attn(CacheAttnArgs a, const CacheAttnPlan& p, float* ws, hipStream_t s) {
  if (a.B <= 0) return hipSuccess;
  if ((a.D != 64 && a.D != 128) || a.G < 1 || a.G > 16 || a.n_heads != a.G * a.n_kv_heads ||
      (a.ldq % 8) || a.B > 65535 || p.splits < 1)
    return hipErrorInvalidValue;
  const int chunks = a.acc_out ? (a.max_ctx + 1023) / 1024 : 0;
  const int64_t gx = p.splits * a.n_kv_heads, gm = a.n_heads + (int64_t)chunks * a.n_kv_heads;
  if (gx >= (1ll << 31) || gm >= (1ll << 31)) return hipErrorInvalidValue;
  a.lead_blocks = p.lead_blocks;
  a.splits = (int)p.splits;
  a.part_o = ws + p.part_o;
  a.part_ml = ws + p.part_ml;
  a.scores = p.score_stride ? ws + p.scores : nullptr;
  a.score_stride = p.score_stride;
  const float sl = (float)(1.4426950408889634 / sqrt((double)a.D));
  const dim3 grid((unsigned)gx, a.B), merge((unsigned)gm, a.B);
  if (a.D == 128) {
    hipLaunchKernelGGL(cache_attn_kernel<128>, grid, dim3(256), 0, s, a, sl);
    hipLaunchKernelGGL(cache_attn_merge_kernel<128>, merge, dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL(cache_attn_kernel<64>, grid, dim3(256), 0, s, a, sl);
    hipLaunchKernelGGL(cache_attn_merge_kernel<64>, merge, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace hs
