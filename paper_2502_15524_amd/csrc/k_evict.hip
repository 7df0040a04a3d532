// Eviction from a paged KV cache by accumulated attention weight.
//
// A row is one kv head of one sequence. The `keep` best of its tokens stay:
// protected ones first, then by weight, then the lower slot. The order is that
// of 32-bit keys, so the `keep`-th largest key is found by a radix select, eight
// bits a pass, and the tokens that stay are known from it and from the rank
// among equal keys. A slot below `keep` whose token goes is a hole; the j-th hole
// takes the j-th token that stays at or past `keep`: as few rows move as can, the
// slots of the others do not change, and sources and holes never overlap.
//
// One workgroup selects for a row; its time is a chain of round trips and
// barriers (the weights of 2112 tokens are 17 KB). Rows with few moves move their
// keys and values there too; those with many leave the moves, as slots of the pool,
// to a second kernel that spreads the copies, which HBM bounds, over the chip.
#include "hs_device.h"
#include "hs_kernels.h"

#include <type_traits>

namespace hs {

namespace {
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMovesHere = 1024;  // per row at most, in the selecting workgroup
constexpr int kMovesPerGroup = 32;
constexpr int kHeld = 32;  // keys of a lane held in LDS, of longer rows

// Larger keys stay. A NaN is below every weight, a protected token above all.
__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sinks, int64_t recent_from) {
  if (pos < sinks || pos >= recent_from) return 0xFFFFFFFFu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 counts as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive sum over the lanes up to this one.
__device__ __forceinline__ uint32_t lane_scan(uint32_t v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast 15: rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast 31: rows 2 and 3
  return v;
}

// Sums of the waves' totals (s_wave[0 .. 15]) before this wave, and of all.
__device__ __forceinline__ uint32_t waves_before(const uint32_t* s_wave, int wave, uint32_t* all) {
  const uint32_t v = s_wave[threadIdx.x & (kWaves - 1)], sum = lane_scan(v);  // (the first row of lanes)
  *all = __builtin_amdgcn_readlane(sum, kWaves - 1);
  return __builtin_amdgcn_readlane(sum - v, wave);
}
__device__ __forceinline__ int rank_in(uint64_t ballot) {  // set lanes below this one
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(ballot >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)ballot, 0));
}
// 16 bytes of a token in slot (block * 16 + offset) of the pool: chunk c of its key (c < D / 8)
// or value
template <int D>
__device__ __forceinline__ bf16_t* chunk_of(const KvEvictArgs& a, int slot, int kh, int c) {
  constexpr int CH = D / 8;
  return a.pool + (((int64_t)(slot >> 4) * 2 + c / CH) * a.n_kv_heads + kh) * 16 * D + (slot & 15) * D + c % CH * 8;
}

// Moves [j0, j1) of a row, four chunks to a thread loaded before the first is stored; pair(j):
// from and to which slot of the pool (-1: left out).
template <int D, int THREADS, typename F>
__device__ __forceinline__ void move_tokens(const KvEvictArgs& a, F pair, int j0, int j1, int kh) {
  constexpr int CH = D / 4, U = 4;  // 16-byte chunks of a token
  const int c = threadIdx.x % CH;
  static_assert(THREADS % CH == 0, "a thread's chunks are alike");
  static_assert((int64_t)kEvictMoves * CH + U * THREADS < 1ll << 31, "chunks are counted in 32 bits");
  for (int i0 = j0 * CH; i0 < j1 * CH; i0 += U * THREADS) {
    pack8 v[U];
    int2 p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * THREADS + threadIdx.x;
      p[u] = i < j1 * CH ? pair(i / CH) : make_int2(-1, -1);
      if (p[u].y < 0) p[u].x = -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u].x >= 0) v[u] = ld16_nt(chunk_of<D>(a, p[u].x, kh, c));
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u].x >= 0) st16(chunk_of<D>(a, p[u].y, kh, c), v[u]);
  }
}
}  // namespace

// K > 0: max_ctx is at most K * 1024, and a token's weight, position and key stay in
// registers (wave w has tokens [64 w per, 64 (w + 1) per), per = ceil(max_ctx / 1024) to a
// lane; they are requested together with the row's length); up to K = 8 in 64 registers, so
// that a CU holds two workgroups (MI355X, K = 16 -> 8: 960 rows of 4097 to 4224 tokens down to 4096 63.9 -> 39.6
// us, 8 of 4500 to 5000 14.4 -> 12.0; K = 4 -> 2: 256 rows of 1025 to 1100 down to 1024 9.2 -> 8.6). K = 0: longer
// rows, whose keys stay in LDS, 32768 of them; the others are formed again in every pass, the next
// eight to a lane requested before these are used (all read again in every pass -> so: 8
// rows of 17536 tokens down to 4000 55.6 -> 33.2 us, of 60000 down to 8000 162 -> 90).
template <int D, int K, bool MOVE>
__global__ __launch_bounds__(kThreads, K == 0 || K == 16 ? 4 : 8) void kv_evict_select_kernel(KvEvictArgs a) {
  constexpr int R = K > 0 ? K : 1;
  // of the first pass's histogram, by lane: most weights share a few exponents. Eight copies are no
  // faster in any form (MI355X, 8 -> 4: 64 rows of 11000 to 12000 tokens 38.0 -> 38.0 us, 512 of 12000 to 16000
  // 297.2 -> 297.0, 256 of 2049 to 2176 12.4 -> 12.4, 960 of 4097 to 4224 41.2 -> 39.4)
  constexpr int kCopies = 4;
  constexpr int kMoves = MOVE || K == 0 ? kMovesHere : 4096;  // listed in LDS
  __shared__ __attribute__((aligned(16))) uint32_t s_hist[256 * (kCopies + 3)];
  __shared__ __attribute__((aligned(16))) uint32_t s_wave[3][kWaves];
  __shared__ uint32_t s_pick[4][3];
  __shared__ int s_table[R * 64], s_hole[kMoves], s_mover[kMoves];
  __shared__ uint32_t s_key[K > 0 ? 1 : kHeld * kThreads];
  const int kh = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = (int64_t)b * a.n_kv_heads + kh;
  const float* acc = a.acc + row * a.stride;
  const int32_t* pos = a.pos + row * a.stride;
  float* acc_out = a.acc_out + row * a.out_stride;
  int32_t* pos_out = a.pos_out + row * a.out_stride;
  const int32_t* table = a.block_table + (int64_t)b * a.max_blocks;
  float ws[R];
  int ps[R];
  int per = (a.max_ctx + kThreads - 1) / kThreads;
  if constexpr (K > 0) {
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const int t = min(wave * 64 * per + i * 64 + lane, a.max_ctx - 1);
      ws[i] = acc[t];
      ps[i] = pos[t];
    }
    if (tid < R * 64) s_table[tid] = table[min(tid, a.max_blocks - 1)];
  }
  const int n = min(max(a.ctx[b], 0), a.max_ctx), kept = min(n, a.keep);
  const int64_t recent_from = (int64_t)a.seen[b] - a.recent;
  if (tid < 64 * (kCopies + 3)) *reinterpret_cast<uint4*>(s_hist + 4 * tid) = make_uint4(0, 0, 0, 0);
  if (kh == 0 && tid == 0) a.ctx_out[b] = kept;
  if constexpr (K == 0) per = (n + kThreads - 1) / kThreads;
  const int first = wave * 64 * per + lane;
  uint32_t keys[R];
  if constexpr (K > 0) {
#pragma unroll
    for (int i = 0; i < K; ++i) keys[i] = evict_key(ws[i], ps[i], a.sinks, recent_from);
  }
  // f(token, key, index in the registers) for every token of the lane; for K = 0 from memory
  // from the lane's i0-th on
  const auto each_from = [&](int i0, auto f) {
    constexpr int U = 8;
    float w[U];
    int p[U];
    const auto load = [&](int i) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = min(first + (i + u) * 64, n - 1);
        w[u] = acc[t];
        p[u] = pos[t];
      }
    };
    if (i0 < per) load(i0);
    for (int i = i0; i < per; i += U) {
      uint32_t k[U];
#pragma unroll
      for (int u = 0; u < U; ++u) k[u] = evict_key(w[u], p[u], a.sinks, recent_from);
      load(i + U);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u < per) f(i + u, k[u]);
    }
  };
  const auto each = [&](auto f) {
    if constexpr (K > 0) {
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (i < per) f(first + i * 64, keys[i], i);
    } else {
#pragma unroll 4
      for (int i = 0; i < min(per, kHeld); ++i) f(first + i * 64, s_key[i * kThreads + tid], 0);
      each_from(kHeld, [&](int i, uint32_t k) { f(first + i * 64, k, 0); });
    }
  };
  const auto put = [&](int t, float w, int p) {
    if (acc_out != acc) acc_out[t] = w;
    if (pos_out != pos) pos_out[t] = p;
  };
  const auto copy = [&](int end) {  // K = 0
#pragma unroll 4
    for (int t = tid; t < end; t += kThreads)
      if (acc_out != acc) acc_out[t] = acc[t];
#pragma unroll 4
    for (int t = tid; t < end; t += kThreads)
      if (pos_out != pos) pos_out[t] = pos[t];
  };
  if (n <= a.keep) {
    if (!MOVE && tid == 0) a.counts[row] = 0;
    if constexpr (K == 0) return copy(n);
    return each([&](int t, uint32_t, int i) {
      if (t < n) put(t, ws[i], ps[i]);
    });
  }

  // the keep-th largest key, and how many of the tokens with that key stay
  uint32_t prefix = 0, mask = 0, need = a.keep;
  __syncthreads();
  const auto select = [&](int pass, auto copies_) {
    constexpr int copies = decltype(copies_)::value;
    const int shift = 24 - 8 * pass;
    uint32_t* const hist = s_hist + (pass ? 256 * (kCopies + pass - 1) : 0);
    const auto count = [&](int t, uint32_t k, int) {
      if (t < n && (k & mask) == prefix) atomicAdd(&hist[((k >> shift) & 255) * copies + (lane & (copies - 1))], 1u);
    };
    if constexpr (K == 0 && copies > 1) {  // the first pass
      each_from(0, [&](int i, uint32_t k) {
        if (i < kHeld) s_key[i * kThreads + tid] = k;
        count(first + i * 64, k, i);
      });
    } else {
      each(count);
    }
    __syncthreads();
    if (wave == 0) {  // lane l has bins 255 - 4 l down to 252 - 4 l
      uint32_t c[4], sum = 0;
      if constexpr (copies == 1) {
        const uint4 v = *reinterpret_cast<const uint4*>(hist + 252 - 4 * lane);
        c[0] = v.w, c[1] = v.z, c[2] = v.y, c[3] = v.x;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          c[j] = 0;
#pragma unroll
          for (int i = 0; i < copies; i += 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(hist + (255 - 4 * lane - j) * copies + i);
            c[j] += v.x + v.y + v.z + v.w;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j];
      const uint32_t above = lane_scan(sum) - sum;
      if (above < need && above + sum >= need) {  // one lane: its bins hold the key
        uint32_t left = need - above, j = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (j == (uint32_t)i && c[i] < left) {
            left -= c[i];
            ++j;
          }
        s_pick[pass][0] = 255 - 4 * lane - j;
        s_pick[pass][1] = left;
        s_pick[pass][2] = j == 0 ? c[0] : j == 1 ? c[1] : j == 2 ? c[2] : c[3];
      }
    }
    __syncthreads();
    prefix |= s_pick[pass][0] << shift;
    mask |= 255u << shift;
    need = s_pick[pass][1];
  };
  select(0, std::integral_constant<int, kCopies>{});
#pragma unroll 1  // (code that runs once comes from memory)
  for (int pass = 1; pass < 4; ++pass) select(pass, std::integral_constant<int, 1>{});

  // the first `need` of the tokens with that key in slot order stay
  uint32_t all, eq = 0;
  const bool ties = s_pick[3][2] != need;  // uniform
  if (ties) {
    each([&](int t, uint32_t k, int) { eq += __popcll(__ballot(t < n && k == prefix)); });
    if (lane == 0) s_wave[0][wave] = eq;
    __syncthreads();
    eq = waves_before(s_wave[0], wave, &all);
  }
  const uint32_t eq0 = eq;
  const auto stays = [&](uint32_t k, int t) {
    if (!ties) return t < n && k >= prefix;
    const bool same = t < n && k == prefix;
    const uint64_t m = __ballot(same);
    const bool s = t < n && (k > prefix || (same && eq + rank_in(m) < need));
    eq += __popcll(m);
    return s;
  };
  uint32_t holes = 0, movers = 0;
  each([&](int t, uint32_t k, int) {
    const bool s = stays(k, t);
    holes += __popcll(__ballot(t < a.keep && !s));
    movers += __popcll(__ballot(t >= a.keep && s));
  });
  if (lane == 0) {
    s_wave[1][wave] = holes;
    s_wave[2][wave] = movers;
  }
  __syncthreads();
  holes = waves_before(s_wave[1], wave, &all);
  movers = waves_before(s_wave[2], wave, &all);
  const int moves = min((int)all, a.cap);
  int2* const pairs = reinterpret_cast<int2*>(a.lists) + row * a.cap;
  const bool in_lds = a.cap <= kMoves;
  eq = eq0;
  if constexpr (K == 0) copy(a.keep);  // (a hole's are written again below)
  // the holes, the tokens that fill them, and the weights of what keeps its slot
  each([&](int t, uint32_t k, int i) {
    const bool s = stays(k, t);
    const int t_first = __builtin_amdgcn_readfirstlane(t);
    if (t_first < a.keep) {
      const bool hole = t < a.keep && !s;
      const uint64_t m = __ballot(hole);
      const uint32_t j = holes + rank_in(m);
      if (hole && j < (uint32_t)moves) {
        if (in_lds) s_hole[j] = t;
        else pairs[j].y = t;
      }
      holes += __popcll(m);
      if (K > 0 && t < a.keep && s) put(t, ws[i], ps[i]);
    }
    if (t_first + 63 >= a.keep) {
      const bool mover = t >= a.keep && s;
      const uint64_t m = __ballot(mover);
      const uint32_t j = movers + rank_in(m);
      if (mover && j < (uint32_t)moves) {
        if (in_lds) s_mover[j] = t;
        else pairs[j].x = t;
      }
      movers += __popcll(m);
    }
  });
  __syncthreads();
  const auto slot_of = [&](int t) {
    const int p = K > 0 ? s_table[t >> 4] : table[t >> 4];
    return p < 0 || p >= a.pool_blocks ? -1 : p * 16 + (t & 15);
  };
  if constexpr (MOVE)
    move_tokens<D, kThreads>(a, [&](int j) { return make_int2(slot_of(s_mover[j]), slot_of(s_hole[j])); }, 0, moves, kh);
  for (int j = tid; j < moves; j += kThreads) {
    const int from = in_lds ? s_mover[j] : pairs[j].x, to = in_lds ? s_hole[j] : pairs[j].y;
    acc_out[to] = acc[from];
    pos_out[to] = pos[from];
    if constexpr (!MOVE) pairs[j] = make_int2(slot_of(from), slot_of(to));
  }
  if (!MOVE && tid == 0) a.counts[row] = moves;
}

template <int D>
__global__ __launch_bounds__(256) void kv_evict_move_kernel(KvEvictArgs a) {
  const int kh = blockIdx.y, j0 = blockIdx.x * kMovesPerGroup;
  const int64_t row = (int64_t)blockIdx.z * a.n_kv_heads + kh;
  const int moves = a.counts[row];
  if (j0 >= moves) return;
  const int2* pairs = reinterpret_cast<const int2*>(a.lists) + row * a.cap;
  move_tokens<D, 256>(a, [&](int j) { return pairs[j]; }, j0, min(j0 + kMovesPerGroup, moves), kh);
}

hipError_t kv_evict(const KvEvictArgs& a, hipStream_t s) {
  if (a.B <= 0) return hipSuccess;
  if ((a.D != 64 && a.D != 128) || a.n_kv_heads < 1 || a.n_kv_heads > 65535 || a.B > 65535 ||
      a.keep < 1 || a.cap < 0 || a.cap > kEvictMoves)
    return hipErrorInvalidValue;
  const dim3 grid(a.n_kv_heads, a.B);
  // One launch for up to 512 moves a row, to 1024 where the rows fill the chip. MI355X, moved in the
  // second kernel -> in the first: 32 sequences of 600 to 900 down to 500, 8 kv heads 18.0 -> 15.8 us; 64 of
  // 1000 to 1500 down to 800 35.5 -> 32.8; 8 of 600 to 900 9.3 -> 9.7 and 1 of 1500 down to 1000, 32 kv heads
  // 10.1 -> 12.5, but a launch (4 us of the host's time) less.
  const bool here = a.cap <= 512 || (a.cap <= kMovesHere && (int64_t)a.B * a.n_kv_heads >= 256);
  const auto launch = [&](auto d) {
    constexpr int D = decltype(d)::value;
    const auto select = [&](auto k) {
      constexpr int K = decltype(k)::value;
      if (here) hipLaunchKernelGGL((kv_evict_select_kernel<D, K, true>), grid, dim3(kThreads), 0, s, a);
      else hipLaunchKernelGGL((kv_evict_select_kernel<128, K, false>), grid, dim3(kThreads), 0, s, a);  // (no use of D)
    };
    if (a.max_ctx <= 2 * kThreads) select(std::integral_constant<int, 2>{});
    else if (a.max_ctx <= 4 * kThreads) select(std::integral_constant<int, 4>{});
    else if (a.max_ctx <= 8 * kThreads) select(std::integral_constant<int, 8>{});
    else if (a.max_ctx <= 16 * kThreads) select(std::integral_constant<int, 16>{});
    else select(std::integral_constant<int, 0>{});
    if (!here)
      hipLaunchKernelGGL(kv_evict_move_kernel<D>, dim3((a.cap + kMovesPerGroup - 1) / kMovesPerGroup, a.n_kv_heads, a.B),
                         dim3(256), 0, s, a);
  };
  if (a.D == 128) launch(std::integral_constant<int, 128>{});
  else launch(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace hs
