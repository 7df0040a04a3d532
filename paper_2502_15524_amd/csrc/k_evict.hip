// Eviction from a paged KV cache by accumulated attention weight.
//
// A row is one kv head of one sequence. The `keep` best of its tokens stay:
// protected ones first, then by weight, then the lower slot. The order is that
// of 32-bit keys, so the `keep`-th largest key is found by a radix select, eight
// bits a pass, and the tokens that stay are known from it and from the rank
// among equal keys. A slot below `keep` whose token goes is a hole; the j-th hole
// takes the j-th token that stays at or past `keep`: as few rows move as can, the
// slots of the others do not change, and sources and holes never overlap.
#include "hs_device.h"
#include "hs_kernels.h"

namespace hs {

namespace {
constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Larger keys stay. A NaN is below every weight, a protected token above all.
__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sinks, int64_t recent_from) {
  if (pos < sinks || pos >= recent_from) return 0xFFFFFFFFu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 counts as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive sum of v over the workgroup's threads; *total: of all.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* s_wave, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();  // the last scan's totals have been read
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const uint32_t y = s_wave[w];
    before += w < wave ? y : 0;
    all += y;
  }
  *total = all;
  return before + x - v;
}
}  // namespace

__global__ __launch_bounds__(kThreads) void kv_evict_kernel(KvEvictArgs a) {
  __shared__ uint32_t s_hist[256], s_wave[kWaves], s_pick[2];
  const int kh = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int n = min(max(a.ctx[b], 0), a.max_ctx), kept = min(n, a.keep);
  const int64_t row = (int64_t)b * a.n_kv_heads + kh;
  const float* acc = a.acc + row * a.stride;
  const int32_t* pos = a.pos + row * a.stride;
  float* acc_out = a.acc_out + row * a.out_stride;
  int32_t* pos_out = a.pos_out + row * a.out_stride;
  if (kh == 0 && tid == 0) a.ctx_out[b] = kept;
  if (n <= a.keep) {
    for (int t = tid; t < n; t += kThreads) {
      acc_out[t] = acc[t];
      pos_out[t] = pos[t];
    }
    return;
  }
  const int64_t recent_from = (int64_t)a.seen[b] - a.recent;
  const auto key_at = [&](int t) { return evict_key(acc[t], pos[t], a.sinks, recent_from); };

  // the keep-th largest key, and how many of the tokens with that key stay
  uint32_t prefix = 0, mask = 0, need = a.keep;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
    for (int t = tid; t < n; t += kThreads) {
      const uint32_t k = key_at(t);
      if ((k & mask) == prefix) atomicAdd(&s_hist[(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t left = need;
      int bin = 255;
      for (; bin > 0 && s_hist[bin] < left; --bin) left -= s_hist[bin];
      s_pick[0] = bin;
      s_pick[1] = left;
    }
    __syncthreads();
    prefix |= s_pick[0] << shift;
    mask |= 255u << shift;
    need = s_pick[1];
  }

  // holes and the tokens that fill them, both in slot order
  int32_t* holes = a.lists + row * 2 * a.cap;
  int32_t* movers = holes + a.cap;
  uint32_t eq_seen = 0, n_holes = 0, n_movers = 0;
  for (int t0 = 0; t0 < n; t0 += kThreads) {
    const int t = t0 + tid;
    const uint32_t k = t < n ? key_at(t) : 0u;
    const bool eq = t < n && k == prefix;
    uint32_t all;
    const uint32_t er = eq_seen + block_scan(eq, s_wave, &all);
    eq_seen += all;
    const bool stays = t < n && (k > prefix || (eq && er < need));
    const bool hole = t < a.keep && !stays, mover = t >= a.keep && stays;
    const uint32_t hr = n_holes + block_scan(hole, s_wave, &all);
    n_holes += all;
    const uint32_t mr = n_movers + block_scan(mover, s_wave, &all);
    n_movers += all;
    if (hole && hr < (uint32_t)a.cap) holes[hr] = t;
    if (mover && mr < (uint32_t)a.cap) movers[mr] = t;
    if (t < a.keep && stays) {
      acc_out[t] = acc[t];
      pos_out[t] = pos[t];
    }
  }
  __syncthreads();
  const int moves = min((int)n_movers, a.cap);
  for (int j = tid; j < moves; j += kThreads) {
    acc_out[holes[j]] = acc[movers[j]];
    pos_out[holes[j]] = pos[movers[j]];
  }
  // the moved tokens' keys and values
  const int32_t* table = a.block_table + (int64_t)b * a.max_blocks;
  const int ch = a.D / 8, per = 2 * ch;
  for (int i = tid; i < moves * per; i += kThreads) {
    const int j = i / per, kv = (i % per) / ch, c = i % ch;
    const int from = movers[j], to = holes[j];
    const int pf = table[from >> 4], pt = table[to >> 4];
    if (pf < 0 || pf >= a.pool_blocks || pt < 0 || pt >= a.pool_blocks) continue;
    const int64_t head = (int64_t)kv * a.n_kv_heads + kh, unit = (int64_t)a.n_kv_heads * 2;
    st16(a.pool + ((pt * unit + head) * 16 + (to & 15)) * a.D + c * 8,
         ld16(a.pool + ((pf * unit + head) * 16 + (from & 15)) * a.D + c * 8));
  }
}

hipError_t kv_evict(const KvEvictArgs& a, hipStream_t s) {
  if (a.B <= 0) return hipSuccess;
  if ((a.D != 64 && a.D != 128) || a.n_kv_heads < 1 || a.B > 65535 || a.keep < 1 || a.cap < 0)
    return hipErrorInvalidValue;
  hipLaunchKernelGGL(kv_evict_kernel, dim3(a.n_kv_heads, a.B), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace hs
