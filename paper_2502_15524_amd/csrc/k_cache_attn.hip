// Decode attention over a paged cache whose sequences share a prefix, and with
// the weight that every cached token received.
//
// A sequence's tokens are the prefix's, then its own, in slots of whole blocks
// (the slots past a block's last token hold nothing). They are cut into splits;
// each leaves for each query head the unnormalised P V, the largest score (log2
// domain) and the sum of exp2(score - largest); a second kernel merges the splits
// and, where weights are asked for, turns the stored scores into probabilities
// with the merged statistics. All of it in float32; for the second matrix product,
// whose operands are bf16, a probability is the sum of two of them, 15 bits of it,
// so that an output is off by little more than its own rounding.
//
// Two kinds of workgroup: of one sequence and kv head, with the kv head's G query heads as the
// rows; and of a part of the prefix and one kv head, with the G query heads of all
// sequences as the rows, so that the prefix is read once for the batch. Short sequences
// are one split, whose workgroup writes output and weights without a second kernel.
//
// Bound by HBM: every cached key and value is read once. MI355X, merge included: 8B heads, 32
// sequences of 64 to 512 tokens behind 8192 22.1 us (72 MB: 3.3 TB/s; in a kernel trace 20.9 and 3.9 for the
// merge; a prefix of 2, 4, 8 and 16 steps to a workgroup with a token of their own takes 11.5, 13.8, 18.0 and
// 25.8 there: 9 and 1.0 to 1.2 a step); 13B heads, 24 of up to 300 behind 2011 27.8 us (4.2 TB/s); with weights,
// 24 of 512 to 4096 behind 1000 53.5 us (4.5 TB/s).
#include "hs_device.h"
#include "hs_kernels.h"

#include <algorithm>
#include <type_traits>

namespace hs {

namespace {
constexpr int kDirect = 1024;  // slots that one workgroup takes alone at most
typedef short s16x4_v __attribute__((ext_vector_type(4)));

// The block that holds slots 16 j .. 16 j + 15 of sequence b: its table entry (which does not
// wait for the sequence's length; past the table: the last one), and how many of the slots
// are tokens. Entries that name no block of the pool hold none.
struct Block {
  int at, n;
};
__device__ __forceinline__ int entry_of(const CacheAttnArgs& a, int b, int j) {
  if (j < a.lead_blocks) return a.prefix[j];
  return a.max_blocks > 0 ? a.block_table[(int64_t)b * a.max_blocks + min(j - a.lead_blocks, a.max_blocks - 1)] : -1;
}
__device__ __forceinline__ Block block_of(const CacheAttnArgs& a, int entry, int j, int ctx) {
  const int n = j < a.lead_blocks ? a.prefix_len - 16 * j : ctx - 16 * (j - a.lead_blocks);
  return entry < 0 || entry >= a.pool_blocks || n <= 0 ? Block{0, 0} : Block{entry, min(16, n)};
}

// A buffer descriptor of uniform values, kept in scalar registers.
__device__ __forceinline__ v4i_t scalar_rsrc(const void* p, uint32_t bytes) {
  v4i_t r = buf_rsrc(p, bytes);
#pragma unroll
  for (int i = 0; i < 3; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
  return r;
}

// Two probabilities as sums of two bf16 each: the upper 8 bits of the significand, and the
// rest rounded, at most 2^-15 of the probability off. The last bit is set, so that the rest is zero
// for zero alone (below 2^-103 it may underflow): an infinite value gives infinity, where zero times it were NaN.
// One rounding to bf16 instead left outputs 0.0020 to 0.0022 of the norm off, 0.0017 now, what their
// own rounding takes; MI355X: 8B heads, 32 sequences behind 8192 tokens 21.7 -> 22.7 us (a prefix
// of many query heads is near the matrix instructions' rate), 13B heads and single sequences unchanged.
__device__ __forceinline__ void split2bf(float x, float y, uint32_t& big, uint32_t& rest) {
  const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
  big = __builtin_amdgcn_perm(b, a, 0x07060302u);  // the upper halves
  rest = pack2bf(__uint_as_float(a | 1) - hi_bf(a), __uint_as_float(b | 1) - hi_bf(b));
}

// 16 bytes read once per call (a non-temporal load)
__device__ __forceinline__ pack8 ld16_once(__amdgpu_buffer_rsrc_t r, int off) {
  constexpr int kNonTemporal = 2;
  return __builtin_bit_cast(pack8, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kNonTemporal));
}

// (largest score, sum) of the split that the lane has among the first 64, requested without
// waiting for the sequence's length: past its splits it may be anything.
__device__ __forceinline__ float2 first_ml(const CacheAttnArgs& a, const float* ml) {
  const int s = min((int)(threadIdx.x & 63), a.splits - 1);
  return make_float2(ml[2 * s], ml[2 * s + 1]);
}
// Merged statistics of a query head of a sequence of n splits: the largest score and the
// sum relative to it. Called by a whole wave; the order is fixed.
__device__ __forceinline__ void merge_ml(const float* ml, float2 first, int n, float& M, float& L) {
  const int lane = threadIdx.x & 63;
  M = lane < n ? first.x : -INFINITY;
  for (int s = lane + 64; s < n; s += 64) M = fmaxf(M, ml[2 * s]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  L = lane < n && first.x != -INFINITY ? first.y * fast_exp2(first.x - M) : 0.f;
  for (int s = lane + 64; s < n; s += 64) {
    const float m = ml[2 * s];
    if (m != -INFINITY) L += ml[2 * s + 1] * fast_exp2(m - M);
  }
  L = wave_sum(L);
}

// Splits of a sequence that hold anything: those of the prefix, then its own.
__device__ __forceinline__ int splits_of(const CacheAttnArgs& a, int ctx) {
  return min(a.splits, a.prefix_splits + (a.lead_blocks + (ctx + 15) / 16 + a.own_blocks - 1) / a.own_blocks);
}
__device__ __forceinline__ int ctx_of(const CacheAttnArgs& a, int b) {
  return min(max(a.ctx[b], 0), a.max_ctx);
}
// What a token received, added to what it had; the newest starts with it, and gets its position.
__device__ __forceinline__ void put_weight(const CacheAttnArgs& a, int64_t at, int b, bool newest, float old, float p) {
  if (newest && a.pos) a.pos[at] = a.seen[b] - 1;
  a.acc_out[at] = newest ? p : a.decay * old + p;
}
}  // namespace

// S^T = K Q^T and O^T = V^T P^T with 16x16x32 MFMAs: keys on the rows, the G query
// heads of the kv head on the columns (the other columns zero). Lane (r, g) =
// (lane % 16, lane / 16) ends with the scores of keys 4 g .. 4 g + 3 of each block
// for query head r, which are the second product's B operand as they are; its
// V^T fragments come from transposing LDS reads. Keys and values are read in
// whole rows, all of them requested before the first is used, and staged
// through the wave's own LDS buffer, the keys first, then the values over them.
//
// NW waves, a step of 32 NW slots; LOOP: as many steps as the split has, the next one's rows
// requested before this one's products, else one. DIRECT: the sequence is one split, and the
// workgroup writes the output and the weights.

// bytes of LDS: the waves' buffers and statistics, the merged statistics of the direct form
constexpr int split_lds(int D, int NW) { return NW * 32 * (D + 16) * 2 + (NW + 1) * 16 * 2 * 4; }

template <int D, int NW, bool LOOP, bool DIRECT = false>
__device__ __forceinline__ void attn_split(const CacheAttnArgs& a, float scale_log2, int split, int kh,
                                           int b, char* smem) {
  constexpr int KS = D / 32, DT = D / 16, CH = D / 8;
  constexpr int RPL = 64 / CH;    // rows per load instruction
  constexpr int NL = 16 / RPL;    // load instructions per block
  constexpr int LV = D + 16;      // padded row: the transposing reads on distinct banks
  constexpr int CB = 2 * NW;      // blocks of a step
  static_assert(16 * D * 4 <= 32 * LV * 2, "a wave's partial fits its buffer");
  const auto sV = [&](int w) { return reinterpret_cast<bf16_t*>(smem) + w * 32 * LV; };
  const auto s_acc = [&](int w) { return reinterpret_cast<float*>(sV(w)); };
  float(*const s_ml)[16][2] = reinterpret_cast<float(*)[16][2]>(smem + NW * 32 * LV * 2);
  float* const s_fin = reinterpret_cast<float*>(s_ml + NW);  // [16][2]
  const int G = a.G, to = a.prefix_splits + split;
  const int tid = threadIdx.x, lane = tid & 63;
  const int j0 = split * a.own_blocks;  // the split's first block
  const int entry = entry_of(a, b, j0 + lane);
  const int ctx = ctx_of(a, b);
  asm volatile("" ::"v"(entry));  // not sunk below the branch
  if (!DIRECT && to > 0 && to >= splits_of(a, ctx)) return;  // uniform across the workgroup
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 15, g = lane >> 4;
  const int64_t head_stride = (int64_t)16 * D, kv_stride = a.n_kv_heads * head_stride;
  const bf16_t* qrow = a.q + (int64_t)b * a.ldq + (int64_t)kh * G * D;
  const int crow = lane / CH, cch = lane % CH;
  const int left = a.lead_blocks + (ctx + 15) / 16 - j0;
  const int chunks = LOOP ? (min(a.own_blocks, left) + CB - 1) / CB : 1;

  // lane i holds the split's block i (at most 64)
  const Block mine = block_of(a, entry, j0 + lane, ctx);
  Block blk[2];
  pack8 ck[2][NL], cv[2][NL];
  const auto load = [&](int c) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i = c * CB + wave * 2 + t;
      blk[t] = Block{__builtin_amdgcn_readlane(mine.at, i), __builtin_amdgcn_readlane(mine.n, i)};
      // rows past the block's last token read zeros
      const bf16_t* base = a.pool + (int64_t)blk[t].at * 2 * kv_stride + kh * head_stride;
      const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(base), 0, blk[t].n * D * 2, kRsrcWord3);
      const __amdgpu_buffer_rsrc_t rv =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(base + kv_stride), 0, blk[t].n * D * 2, kRsrcWord3);
#pragma unroll
      for (int i = 0; i < NL; ++i) ck[t][i] = ld16_once(rk, lane * 16 + i * 1024);
#pragma unroll
      for (int i = 0; i < NL; ++i) cv[t][i] = ld16_once(rv, lane * 16 + i * 1024);
    }
  };
  load(0);
  pack8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = fr < G ? ld16(qrow + fr * D + ks * 32 + g * 8) : zero8();
  bf16_t* sv = sV(wave);
  float m_run = -INFINITY, l_run = 0.f;
  f32x4_v o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4_v{0.f, 0.f, 0.f, 0.f};

  for (int c = 0; c < chunks; ++c) {
    pack8 kf[2][KS];
    const int n[2] = {blk[0].n, blk[1].n};
    // (a wave's LDS operations run in order: the last chunk's fragment reads come first)
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < NL; ++i) st16(sv + (16 * t + RPL * i + crow) * LV + cch * 8, ck[t][i]);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[t][ks] = ld16(sv + (16 * t + fr) * LV + ks * 32 + g * 8);
    asm volatile("" ::: "memory");  // the key reads before the value stores
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < NL; ++i) st16(sv + (16 * t + RPL * i + crow) * LV + cch * 8, cv[t][i]);
    if (LOOP && c + 1 < chunks) load(c + 1);  // on its way during this chunk's products

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
        s[t][j] = 4 * g + j < n[t] ? s[t][j] * scale_log2 : -INFINITY;
        m = fmaxf(m, s[t][j]);
      }
      // the scores of the sequence's own tokens, for their weights
      const int own = (j0 + c * CB + wave * 2 + t - a.lead_blocks) * 16;
      if (a.scores && own >= 0 && own < ctx && fr < G)
        *reinterpret_cast<f32x4_v*>(a.scores + ((int64_t)b * a.n_heads + kh * G + fr) * a.score_stride + own + 4 * g) = s[t];
    }
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float m_new = fmaxf(m_run, m), m0 = m_new == -INFINITY ? 0.f : m_new;
    const float corr = fast_exp2(m_run - m0);
    m_run = m_new;
    l_run *= corr;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[t][j] = fast_exp2(s[t][j] - m0);
        l_run += s[t][j];
      }
    pack8 pk, pr;
#pragma unroll
    for (int w = 0; w < 4; ++w) split2bf(s[w >> 1][2 * (w & 1)], s[w >> 1][2 * (w & 1) + 1], pk.w[w], pr.w[w]);
    const bf16x8_v pf = as_bf16x8(pk), pg = as_bf16x8(pr);
    asm volatile("" ::: "memory");  // the value stores before the fragment reads
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const bf16_t* vp = sv + (4 * g + (fr >> 2)) * LV + dt * 16 + 4 * (fr & 3);
      const s16x4_v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4_v*)(vp));
      const s16x4_v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4_v*)(vp + 16 * LV));
      const bf16x8_v vb =
          __builtin_bit_cast(bf16x8_v, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, pf, o[dt] * corr, 0, 0, 0);
      o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, pg, o[dt], 0, 0, 0);
    }
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  asm volatile("" ::: "memory");  // the fragment reads before the partial goes over them
  if (fr < G) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<f32x4_v*>(s_acc(wave) + fr * D + dt * 16 + 4 * g) = o[dt];
    if (g == 0) {
      // (only NaN scores: a sum, of NaN, without a largest)
      s_ml[wave][fr][0] = m_run == -INFINITY && l_run != 0.f ? 0.f : m_run;
      s_ml[wave][fr][1] = l_run;
    }
  }
  __syncthreads();
  for (int i = tid; i < G * D; i += 64 * NW) {
    const int gg = i / D, d = i % D;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, s_ml[w][gg][0]);
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float mw = s_ml[w][gg][0];
      if (mw == -INFINITY) continue;
      const float f = fast_exp2(mw - M);
      L += s_ml[w][gg][1] * f;
      O += s_acc(w)[gg * D + d] * f;
    }
    if constexpr (DIRECT) {
      // no token at all, or none with a score above -inf: zero
      a.out[(int64_t)b * a.ldo + (kh * G + gg) * D + d] = f2bf(L == 0.f ? 0.f : O / L);
      if (d == 0) {
        s_fin[2 * gg] = M == -INFINITY ? 0.f : M;
        s_fin[2 * gg + 1] = L == 0.f ? 0.f : 1.f / L;
      }
    } else {
      const int64_t row = ((int64_t)b * a.n_heads + kh * G + gg) * a.splits + to;
      a.part_o[row * D + d] = O;
      if (d == 0) {
        a.part_ml[row * 2] = M;
        a.part_ml[row * 2 + 1] = L;
      }
    }
  }
  if (DIRECT && a.scores) {
    __syncthreads();
    const int64_t row = ((int64_t)b * a.n_kv_heads + kh) * a.acc_stride;
    const float* sc = a.scores + ((int64_t)b * a.n_heads + kh * G) * a.score_stride;
    for (int t = tid; t < ctx; t += 64 * NW) {
      const float old = a.acc[row + t];
      float p = 0.f;
      for (int gg = 0; gg < G; ++gg) p += fast_exp2(sc[gg * a.score_stride + t] - s_fin[2 * gg]) * s_fin[2 * gg + 1];
      put_weight(a, row + t, b, t == ctx - 1, old, p);
    }
  }
}

// Rows of 32 query heads on the columns of 32x32x16 MFMAs, keys on the rows: lane
// (q, hi) = (lane % 32, lane / 32) gets row q's scores of keys 8 (i / 4) + 4 hi + i % 4
// (i = 0 .. 15) of 32, which are the second product's B operand as they are. The four
// waves are two groups of 32 rows by two groups of 32 keys of a step. Keys and values go
// from memory straight into a ring of NST stages of 64 keys, the request of a step
// NST - 1 steps ahead of its use; a wave's copies of a step cover one cache block, and
// read zeros past the block's last token or for a block outside the pool. The 16-byte
// chunks of a row are XOR-swizzled so that the fragment reads and the transposing
// reads of the values take different banks. Tiles of 64 rows, not 128 with 32 keys a
// step: the same keys come from L2 for the second tile (8B heads, 32 sequences behind
// 8192 tokens, MI355X, when this was chosen: 26.4 us with 128 rows, 24.1 with 64).
template <int D>
__device__ __forceinline__ int key_swz(int key) {
  return key & (D / 8 - 1);
}
template <int D>
__device__ __forceinline__ int value_swz(int key) {
  if constexpr (D == 128) return ((key & 3) << 2) | ((key >> 2) & 3);
  else return ((key & 3) << 1) | ((key >> 2) & 1);
}
constexpr int kPrefixBlocks = 64;  // of one workgroup at most: a lane each
constexpr int kTileRows = 64;
constexpr int prefix_stages(int D) { return D == 128 ? 2 : 4; }  // 64 KB: two workgroups per CU
constexpr int prefix_lds(int D) { return prefix_stages(D) * 64 * D * 4; }

template <int D>
__device__ __forceinline__ void attn_prefix(const CacheAttnArgs& a, float scale_log2, int split, int tile,
                                            int kh, char* smem) {
  constexpr int RW = kTileRows / 32, KB = 64, NST = prefix_stages(D);
  constexpr int CH = D / 8, ROW = D * 2, BLK = KB * ROW, STG = 2 * BLK;
  constexpr int KPI = 64 / CH, PER = KB / KPI / 4;  // keys per copy; copies per wave, operand and step
  static_assert(PER >= 1 && PER * KPI * 4 == KB && 16 % (PER * KPI) == 0, "a wave's copies stay within a block");
  static_assert(RW * 32 * D * 4 + 4 * 32 * 8 <= NST * STG, "the token groups' merge fits the ring");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, tw = wave / RW;
  const int q = lane & 31, hi = lane >> 5;
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) char*)smem;

  const int t0 = split * a.prefix_tokens, len = min(a.prefix_tokens, a.prefix_len - t0);
  const int steps = (len + KB - 1) / KB;
  // lane i holds the split's block i (at most 64), -1: none, or none of the pool
  int mine = 16 * lane < len ? a.prefix[t0 / 16 + lane] : -1;
  if (mine >= a.pool_blocks) mine = -1;
  // this lane's row
  const int G = a.G, row = (tile * RW + rw) * 32 + q, rows = a.B * G;
  const bool real = row < rows;
  const int rb = row / G, rh = kh * G + row - rb * G;
  int ko[PER], vo[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int key = (PER * wave + i) * KPI + lane / CH, at = lane % CH;
    ko[i] = (key & 15) * ROW + ((at ^ key_swz<D>(key)) * 16);
    vo[i] = (key & 15) * ROW + ((at ^ value_swz<D>(key)) * 16);
  }
  const int64_t head_bytes = 16ll * ROW, kv_bytes = a.n_kv_heads * head_bytes;
  const char* const base = reinterpret_cast<const char*>(a.pool) + kh * head_bytes;
  auto tokens_in = [&](int i) {  // of the split's block i
    return __builtin_amdgcn_readlane(mine, i & 63) < 0 ? 0 : min(16, len - 16 * i);
  };
  // a wave's copies of a step (PER of keys, then PER of values) are of one block
  v4i_t rk, rv;
  uint32_t to_lds;
  auto aim = [&](int step) {
    const int i = (step * KB + PER * wave * KPI) / 16;
    const int p = __builtin_amdgcn_readlane(mine, i & 63);
    const char* kp = base + (int64_t)max(p, 0) * 2 * kv_bytes;
    const uint32_t bytes = p < 0 ? 0u : (uint32_t)max(0, min(16, len - 16 * i)) * ROW;
    rk = scalar_rsrc(kp, bytes);
    rv = scalar_rsrc(kp + kv_bytes, bytes);
    to_lds = lds0 + (step % NST) * STG + wave * PER * 1024;
  };
  auto copy = [&](int j) {
    if (j < PER) dma16(rk, ko[j], to_lds + j * 1024);
    else dma16(rv, vo[j - PER], to_lds + BLK + (j - PER) * 1024);
  };
#pragma unroll
  for (int i = 0; i < NST - 1; ++i) {
    aim(i);
#pragma unroll
    for (int j = 0; j < 2 * PER; ++j) copy(j);
  }
  bf16x8_v qf[D / 16];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
    qf[ks] = as_bf16x8(real ? ld16(a.q + (int64_t)rb * a.ldq + rh * D + ks * 16 + hi * 8) : zero8());

  int ka[D / 16], va[D / 32][2];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
    ka[ks] = (32 * tw + q) * ROW + (((2 * ks + hi) ^ key_swz<D>(q)) * 16);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int key = 8 * u + 4 * hi + ((lane & 15) >> 2);
      const int chunk = dt * 4 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      va[dt][u] = BLK + (32 * tw + key) * ROW + ((chunk ^ value_swz<D>(key)) * 16) + (lane & 1) * 8;
    }
  f32x16_v o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const bool busy = (tile * RW + rw) * 32 < rows;  // of the wave

  // (the queries are waited for here, with the first step's copies: left to their first use, in
  // the loop, the wait would drain the copies in flight)
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) asm volatile("" : "+v"(qf[ks]));

  for (int k = 0; k < steps; ++k) {
    // this wave's copies of step k have landed (those of the NST - 2 steps after it may be
    // on their way), its reads of step k - 1 are complete; with everybody's at the
    // barrier the stage of step k - 1 takes the next request
    if constexpr (PER * 2 * (NST - 2) == 0) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PER * 2 * (NST - 2)) : "memory");
    asm volatile("s_barrier" ::: "memory");
    aim(k + NST - 1);
    if (!busy) {
#pragma unroll
      for (int j = 0; j < 2 * PER; ++j) copy(j);
      continue;
    }
    const char* st = smem + (k % NST) * STG;
    // (all key fragments are requested before the first product: left to the compiler, each
    // was read one product ahead, less than an LDS read takes)
    bf16x8_v kf[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) kf[ks] = as_bf16x8(ld16(st + ka[ks]));
    __builtin_amdgcn_sched_barrier(0);
    f32x16_v s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    // one copy behind each product: in a row, the four waves' copies keep one another waiting (MI355X, 32 sequences
    // behind 8192 tokens, in a graph: 20.3 -> 20.0 us without caches of their own, 23.5 -> 23.2 with 64 to 512; 24 ragged ones
    // behind 1000 53.3 and 53.4, 64 behind 4096 24.4 and 25.2)
    static_assert(2 * PER == D / 16, "as many copies as products");
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      copy(ks);
      __builtin_amdgcn_sched_barrier(0);
    }
    const int blk = (k * KB + 32 * tw) / 16, n0 = tokens_in(blk), n1 = tokens_in(blk + 1);
    if (n0 < 16 || n1 < 16) {  // uniform: blocks that are not full
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if ((8 * (e >> 2) & 15) + 4 * hi + (e & 3) >= (e < 8 ? n0 : n1)) s[e] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    {
      const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])) * scale_log2;
    }
    const float m_new = fmaxf(m_run, mx);
    const float m0 = m_new == -INFINITY ? 0.f : m_new;
    if (__any(m_new != m_run)) {
      const float corr = fast_exp2(m_run - m0);
      m_run = m_new;
      l_run *= corr;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] *= corr;
    }
    float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = fast_exp2(__builtin_fmaf(s[e], scale_log2, -m0));
      ps[e & 3] += s[e];
    }
    l_run += (ps[0] + ps[1]) + (ps[2] + ps[3]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      pack8 pb, pr;
#pragma unroll
      for (int w = 0; w < 4; ++w) split2bf(s[8 * h + 2 * w], s[8 * h + 2 * w + 1], pb.w[w], pr.w[w]);
      const bf16x8_v pf = as_bf16x8(pb), pg = as_bf16x8(pr);
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        const s16x4_v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4_v*)(st + va[dt][0] + h * 16 * ROW));
        const s16x4_v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4_v*)(st + va[dt][1] + h * 16 * ROW));
        const bf16x8_v vb =
            __builtin_bit_cast(bf16x8_v, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb, pf, o[dt], 0, 0, 0);
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb, pg, o[dt], 0, 0, 0);
      }
    }
  }
  {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
    l_run = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (m_run == -INFINITY && l_run != 0.f) m_run = 0.f;  // only NaN scores
  // Each token group hands half of its columns to the other, which merges and stores them,
  // through the ring, which the copies past the last step (they read nothing) have left.
  constexpr int HT = D / 64;  // tiles of 32 columns in a half
  f32x4_v* const s_o = reinterpret_cast<f32x4_v*>(smem);
  float2* const s_ml = reinterpret_cast<float2*>(s_o + 4 * HT * 4 * 64);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int i = 0; i < HT; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4_v x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = tw ? o[i][4 * g + e] : o[HT + i][4 * g + e];
      s_o[((wave * HT + i) * 4 + g) * 64 + lane] = x;
    }
  if (hi == 0) s_ml[wave * 32 + q] = make_float2(m_run, l_run);
  __syncthreads();
  if (!real) return;
  const int peer = rw + RW * (1 - tw);
  const float2 ml = s_ml[peer * 32 + q];
  const float m = fmaxf(m_run, ml.x);
  const float c0 = m_run == -INFINITY ? 0.f : fast_exp2(m_run - m);
  const float c1 = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m);
  const int64_t to = ((int64_t)rb * a.n_heads + rh) * a.splits + split;
#pragma unroll
  for (int i = 0; i < HT; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4_v y = s_o[((peer * HT + i) * 4 + g) * 64 + lane];
      f32x4_v x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (tw ? o[HT + i][4 * g + e] : o[i][4 * g + e]) * c0 + y[e] * c1;
      *reinterpret_cast<f32x4_v*>(a.part_o + to * D + (tw * HT + i) * 32 + g * 8 + hi * 4) = x;
    }
  if (hi == 0 && tw == 0) {
    a.part_ml[to * 2] = m;
    a.part_ml[to * 2 + 1] = l_run * c0 + ml.y * c1;
  }
}

template <int D, bool LOOP>
__device__ __forceinline__ void attn_sequences(const CacheAttnArgs& a, float scale_log2, int i, char* smem) {
  const int per = a.n_kv_heads * a.own_splits, b = i / per, r = i - b * per;
  attn_split<D, 4, LOOP>(a, scale_log2, r / a.n_kv_heads, r % a.n_kv_heads, b, smem);
}

// Every token through workgroups of one sequence.
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4))) void cache_attn_kernel(
    CacheAttnArgs a, float scale_log2) {
  __shared__ __attribute__((aligned(16))) char smem[split_lds(D, 4)];
  attn_sequences<D, false>(a, scale_log2, blockIdx.x, smem);
}
// One workgroup per (sequence, kv head), and no merge.
template <int D, int NW, bool LOOP>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2))) void cache_attn_direct_kernel(
    CacheAttnArgs a, float scale_log2) {
  __shared__ __attribute__((aligned(16))) char smem[split_lds(D, NW)];
  attn_split<D, NW, LOOP, true>(a, scale_log2, 0, blockIdx.x % a.n_kv_heads, blockIdx.x / a.n_kv_heads, smem);
}

// The prefix's workgroups first (the longest), then the sequences'.
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void cache_attn_shared_kernel(
    CacheAttnArgs a, float scale_log2) {
  __shared__ __attribute__((aligned(1024))) char smem[std::max(prefix_lds(D), split_lds(D, 4))];
  const int tiles = (a.B * a.G + kTileRows - 1) / kTileRows;
  const int i = blockIdx.x, first = a.prefix_splits * tiles * a.n_kv_heads;
  if (i < first) {
    const int j = i / a.n_kv_heads;
    return attn_prefix<D>(a, scale_log2, j / tiles, j % tiles, i % a.n_kv_heads, smem);
  }
  attn_sequences<D, true>(a, scale_log2, i - first, smem);
}

// The output of one (query head, sequence). A row of 16-byte loads takes D / 4 lanes, so
// the four waves take 4 * 256 / D splits at a time, up to 64 with all loads in flight; those of
// the first 64 do not wait for the sequence's length.
template <int D>
__device__ __forceinline__ void merge_out(const CacheAttnArgs& a, int h, int b) {
  constexpr int LPR = D / 4, RPP = 64 / LPR, U = 16 / RPP;  // lanes per row, rows per wave and load, loads
  __shared__ f32x4_v s_o[4][LPR];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = ((int64_t)b * a.n_heads + h) * a.splits;
  const float* ml = a.part_ml + row * 2;
  f32x4_v v[U], o = {0.f, 0.f, 0.f, 0.f};
  const auto load = [&](int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = min(s0 + (4 * u + wave) * RPP + lane / LPR, a.splits - 1);
      if (s0 + (4 * u + wave) * RPP < a.splits)  // uniform
        v[u] = *reinterpret_cast<const f32x4_v*>(a.part_o + (row + s) * D + (lane % LPR) * 4);
    }
  };
  load(0);
  const float2 first = first_ml(a, ml);
  const int ctx = ctx_of(a, b), n = splits_of(a, ctx);
  float M, L;
  merge_ml(ml, first, n, M, L);
  for (int s0 = 0; s0 < n; s0 += 64) {
    if (s0 > 0) load(s0);
    const float m = s0 + lane >= n ? -INFINITY : s0 == 0 ? first.x : ml[2 * (s0 + lane)];
    const float w = m == -INFINITY ? 0.f : fast_exp2(m - M);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float x = __shfl(w, (4 * u + wave) * RPP + lane / LPR, 64);
      if (x != 0.f) o += v[u] * x;  // (a split without weight may hold anything)
    }
  }
#pragma unroll
  for (int e = LPR; e < 64; e <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], e, 64);
  if (lane < LPR) s_o[wave][lane] = o;
  __syncthreads();
  if (threadIdx.x >= LPR) return;
  o = (s_o[0][lane] + s_o[1][lane]) + (s_o[2][lane] + s_o[3][lane]);
  // no token at all, or none with a score above -inf: zero
  const float r = n == 0 || L == 0.f ? 0.f : 1.f / L;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.out + (int64_t)b * a.ldo + h * D) + lane * 2;
  out[0] = pack2bf(o[0] * r, o[1] * r);
  out[1] = pack2bf(o[2] * r, o[3] * r);
}

// The same for up to 32 splits, a wave alone: no exchange through LDS (with the main kernel, MI355X, in a graph:
// 8B heads, 64 sequences behind 4096 tokens 26.9 -> 25.2 us, 32 behind 8192 24.0 -> 23.2; 13B, 24 behind 2011
// 28.7 -> 28.2).
template <int D>
__device__ __forceinline__ void merge_out_wave(const CacheAttnArgs& a, int h, int b) {
  constexpr int LPR = D / 4, RPP = 64 / LPR, U = 32 / RPP;
  const int lane = threadIdx.x & 63;
  const int64_t row = ((int64_t)b * a.n_heads + h) * a.splits;
  const __amdgpu_buffer_rsrc_t rows =  // past the last split: zeros, without traffic
      __builtin_amdgcn_make_buffer_rsrc(a.part_o + row * D, 0, a.splits * D * 4, kRsrcWord3);
  f32x4_v v[U], o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < U; ++u)
    v[u] = __builtin_bit_cast(f32x4_v, __builtin_amdgcn_raw_buffer_load_b128(rows, (u * 64 + lane) * 16, 0, 0));
  const float2 first = first_ml(a, a.part_ml + row * 2);
  const int n = splits_of(a, ctx_of(a, b));
  float M = lane < n ? first.x : -INFINITY;
#pragma unroll
  for (int e = 32; e > 0; e >>= 1) M = fmaxf(M, __shfl_xor(M, e, 64));
  const float w = lane < n && first.x != -INFINITY ? fast_exp2(first.x - M) : 0.f;
  const float L = wave_sum(lane < n && first.x != -INFINITY ? first.y * w : 0.f);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const float x = __shfl(w, u * RPP + lane / LPR, 64);
    if (x != 0.f) o += v[u] * x;  // (a split without weight may hold anything)
  }
#pragma unroll
  for (int e = LPR; e < 64; e <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], e, 64);
  if (lane >= LPR) return;
  const float r = n == 0 || L == 0.f ? 0.f : 1.f / L;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.out + (int64_t)b * a.ldo + h * D) + lane * 2;
  out[0] = pack2bf(o[0] * r, o[1] * r);
  out[1] = pack2bf(o[2] * r, o[3] * r);
}

// What a sequence's own tokens received: 1024 tokens of one kv head, four to a thread. The
// scores of the first four query heads and the old weights are requested with the splits'
// statistics (past the sequence's tokens they may be anything).
__device__ __forceinline__ void add_weights(const CacheAttnArgs& a, int kh, int b, int chunk) {
  __shared__ float s_m[16], s_r[16];
  const int G = a.G, t0 = chunk * 1024 + threadIdx.x, wave = threadIdx.x >> 6;
  const int64_t row = ((int64_t)b * a.n_kv_heads + kh) * a.acc_stride;
  const float* sc = a.scores + ((int64_t)b * a.n_heads + kh * G) * a.score_stride;
  float x[4][4], old[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) old[i] = a.acc[row + min(t0 + i * 256, a.max_ctx - 1)];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int gg = 0; gg < 4; ++gg) x[gg][i] = sc[min(gg, G - 1) * a.score_stride + min(t0 + i * 256, a.max_ctx - 1)];
  const float2 first = first_ml(a, a.part_ml + ((int64_t)b * a.n_heads + kh * G + min(wave, G - 1)) * a.splits * 2);
  const int ctx = ctx_of(a, b), n = splits_of(a, ctx);
  if (chunk * 1024 >= ctx) return;  // uniform
  for (int gg = wave; gg < G; gg += 4) {
    float M, L;
    const float* ml = a.part_ml + ((int64_t)b * a.n_heads + kh * G + gg) * a.splits * 2;
    merge_ml(ml, gg == wave ? first : first_ml(a, ml), n, M, L);
    s_m[gg] = M == -INFINITY ? 0.f : M;
    s_r[gg] = L == 0.f ? 0.f : 1.f / L;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + i * 256;
    if (t >= ctx) break;
    float p = 0.f;
#pragma unroll
    for (int gg = 0; gg < 4; ++gg)
      if (gg < G) p += fast_exp2(x[gg][i] - s_m[gg]) * s_r[gg];
    for (int gg = 4; gg < G; ++gg) p += fast_exp2(sc[gg * a.score_stride + t] - s_m[gg]) * s_r[gg];
    put_weight(a, row + t, b, t == ctx - 1, old[i], p);
  }
}

// The first workgroups of a sequence merge its outputs, the others its weights.
constexpr int kWaveSplits = 32;
__host__ __device__ __forceinline__ int merge_groups(int n_heads, int splits) {
  return splits <= kWaveSplits ? (n_heads + 3) / 4 : n_heads;
}
template <int D>
__global__ __launch_bounds__(256) void cache_attn_merge_kernel(CacheAttnArgs a) {
  const int i = blockIdx.x, groups = merge_groups(a.n_heads, a.splits);
  if (i >= groups) return add_weights(a, (i - groups) % a.n_kv_heads, blockIdx.y, (i - groups) / a.n_kv_heads);
  if (a.splits > kWaveSplits) return merge_out<D>(a, i, blockIdx.y);
  const int h = 4 * i + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (h < a.n_heads) merge_out_wave<D>(a, h, blockIdx.y);
}

CacheAttnPlan cache_attn_plan(int64_t B, int64_t n_heads, int64_t n_kv_heads, int64_t D,
                              int64_t prefix_len, int64_t max_ctx, bool weights) {
  CacheAttnPlan p;
  const int64_t rows = B * (n_heads / n_kv_heads), blocks = (prefix_len + 15) / 16;
  const int64_t slots = blocks * 16 + (max_ctx + 15) / 16 * 16;
  // Alone: a step of 256 slots at least as fast as splits and their merge at any batch; longer
  // ones where the workgroups fill the chip (128 and more for 3 and 4 steps), at two to a
  // CU in turn, or at one if each would read a prefix that the others have read. MI355X, in a graph, splits
  // and merge -> alone: 3 sequences of 97 tokens, 4 heads 6.2 -> 3.5 us; 32 of 200, 8 kv heads 10.9 -> 7.4;
  // 24 of 200, 40 heads 22.2 -> 18.1; 32 of 1000, 8 kv heads 27.5 -> 22.5; 28 of 400 behind 600 19.4 -> 14.1; 56 of
  // 1000 43.7 -> 38.1. Left to the splits: 8 of 1000 11.5 (13.8 alone); 36 of 100 behind 900 13.5 (22.2), 48 of 400
  // behind 600 21.7 (25.4).
  const int64_t groups = B * n_kv_heads;
  const bool prefixed = B > 1 && prefix_len > 0;
  p.direct = slots <= 256 || (groups <= (prefixed ? 256 : 512) && slots <= (groups < 128 ? 512 : kDirect));
  p.shared = !p.direct && prefixed;
  p.lead_blocks = p.shared ? 0 : (int)blocks;
  // (Without a prefix, splits of 128 tokens: the step of a workgroup, none looped. In splits of 384 tokens of the
  // looped form batches that fill the chip are faster and short ones slower: 24 of 512 to 4096 with weights 52.6 and
  // 50.3 us, 64 of 1000 to 2000 73.7 and 68.0; one of 1100, 32 heads 10.0 and 11.5, 4 of 4000 18.3 and 19.7.)
  p.own_blocks = p.direct ? kDirect / 16 : 8;
  p.prefix_tokens = 0;
  p.prefix_splits = 0;
  if (p.shared) {
    // Every split costs the batch a partial result (520 bytes per query head at D = 128, written
    // and read), so a split is as long as leaves 256 workgroups to the prefix, one per CU, and to
    // the sequences. MI355X, in a graph, splits of 128, 256, 512 and 1024 tokens: 32 sequences of 64 to 512 behind 8192 38.0,
    // 29.7, 22.5 and 28.5 us (512 taken), 64 of up to 200 behind 4096 36.8, 28.5, 23.8 and 27.4 (512), 16 of 500 behind
    // 32000 70.1, 56.4, 47.5 and 41.6 (1000), 13B heads, 24 of up to 300 behind 2011 32.7, 28.8, 28.3 and 28.7 (320).
    const int64_t tiles = (rows + kTileRows - 1) / kTileRows;
    p.prefix_tokens = (int)std::min<int64_t>(
        kPrefixBlocks * 16, std::max<int64_t>(128, (prefix_len * n_kv_heads * tiles / 256 + 63) / 64 * 64));
    p.prefix_splits = (prefix_len + p.prefix_tokens - 1) / p.prefix_tokens;
    // up to 512 of its slots in one split; longer ones in splits of 384. MI355X, in a graph, splits of 128, 256, 384, 512 and
    // 1024 tokens: 24 of 512 to 4096 63.0, 57.7, 53.5, 56.6 and 60.3 us with weights, 57.9, 49.0, 45.6, 47.3 and 48.1 without; 64
    // of 300 to 1000 52.8, 48.4, 42.7, 45.6 and 42.8; 16 of 600 to 1000 23.1, 22.4, 20.1, 21.3 and 23.2; 32 of 4096 124.5, 109.3, 106.7,
    // 103.8 and 104.7; 7B heads, 4 of 512 to 4096 35.8, 31.4, 30.2, 29.7 and 34.3. Up to 512: 128 of 400 to 500 64.9,
    // 56.3, 62.0, 53.5 and 53.4; 32 of 64 to 512 27.0, 24.3, 26.2, 22.4 and 22.5
    p.own_blocks = 8 * (int)std::min<int64_t>(max_ctx > 512 ? 3 : 4, std::max<int64_t>(1, groups * ((max_ctx + 127) / 128) / 256));
  }
  p.own_splits = (p.lead_blocks + (max_ctx + 15) / 16 + p.own_blocks - 1) / p.own_blocks;
  if (p.direct) p.own_splits = 1;
  p.splits = p.prefix_splits + p.own_splits;
  p.score_stride = weights ? (max_ctx + 15) / 16 * 16 : 0;
  const int64_t parts = p.direct ? 0 : B * n_heads * p.splits;
  p.part_o = 0;
  p.part_ml = parts * D;
  p.scores = (p.part_ml + parts * 2 + 3) / 4 * 4;
  p.floats = std::max<int64_t>(4, p.scores + B * n_heads * p.score_stride);
  p.groups = (p.prefix_splits * ((rows + kTileRows - 1) / kTileRows) + B * p.own_splits) * n_kv_heads;
  const int64_t chunks = weights ? (max_ctx + 1023) / 1024 : 0;
  p.merge_groups = merge_groups((int)n_heads, (int)p.splits) + chunks * n_kv_heads;
  p.fits = p.groups < (1ll << 23) && p.merge_groups < (1ll << 24);  // 2^32 threads of a launch
  return p;
}

hipError_t cache_attn(CacheAttnArgs a, const CacheAttnPlan& p, float* ws, hipStream_t s) {
  if (a.B <= 0) return hipSuccess;
  if ((a.D != 64 && a.D != 128) || a.G < 1 || a.G > 16 || a.n_heads != a.G * a.n_kv_heads ||
      (a.ldq % 8) || a.B > 65535 || p.splits < 1 || !p.fits)
    return hipErrorInvalidValue;
  a.lead_blocks = p.lead_blocks;
  a.prefix_tokens = p.prefix_tokens;
  a.prefix_splits = (int)p.prefix_splits;
  a.own_blocks = p.own_blocks;
  a.own_splits = (int)p.own_splits;
  a.splits = (int)p.splits;
  a.part_o = ws + p.part_o;
  a.part_ml = ws + p.part_ml;
  a.scores = p.score_stride ? ws + p.scores : nullptr;
  a.score_stride = p.score_stride;
  const float sl = (float)(1.4426950408889634 / sqrt((double)a.D));
  const dim3 grid((unsigned)p.groups), merge((unsigned)p.merge_groups, a.B);
  const auto launch = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (p.direct) {
      const int slots = a.lead_blocks * 16 + (a.max_ctx + 15) / 16 * 16;
      if (slots <= 128) hipLaunchKernelGGL((cache_attn_direct_kernel<D, 4, false>), grid, dim3(256), 0, s, a, sl);
      else if (slots <= 256) hipLaunchKernelGGL((cache_attn_direct_kernel<D, 8, false>), grid, dim3(512), 0, s, a, sl);
      else hipLaunchKernelGGL((cache_attn_direct_kernel<D, 8, true>), grid, dim3(512), 0, s, a, sl);
      return;
    }
    if (!p.shared)
      hipLaunchKernelGGL(cache_attn_kernel<D>, grid, dim3(256), 0, s, a, sl);
    else
      hipLaunchKernelGGL(cache_attn_shared_kernel<D>, grid, dim3(256), 0, s, a, sl);
    hipLaunchKernelGGL(cache_attn_merge_kernel<D>, merge, dim3(256), 0, s, a);
  };
  if (a.D == 128) launch(std::integral_constant<int, 128>{});
  else launch(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace hs
