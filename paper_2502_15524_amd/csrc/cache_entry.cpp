// Entry points of the cache operators (include/hs_kernel.h): argument checks,
// workspace sizes and the launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <string>

#include "../../include/hs_kernel.h"
#include "hs_host.h"
#include "hs_kernels.h"

using namespace hs;

namespace {
hs_status done(hipError_t e, const char* what) {
  if (e == hipErrorInvalidValue) return fail(HS_EINVAL, std::string(what) + ": unsupported shape");
  if (e != hipSuccess) return fail(HS_EHIP, std::string(what) + ": " + hipGetErrorString(e));
  return HS_OK;
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// HS_OK, or HS_EINVAL with the message set.
hs_status heads_ok(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (head_dim != 64 && head_dim != 128) return fail(HS_EINVAL, "head_dim must be 64 or 128");
  if (n_kv_heads < 1 || n_heads < 1 || n_heads % n_kv_heads || n_heads / n_kv_heads > 16 ||
      n_heads > 65536)
    return fail(HS_EINVAL, "bad head counts");
  return HS_OK;
}

// An argument in memory: `rows` of `width` bytes, `stride` bytes apart (of one row: any). Pools and
// rotary tables are left out of these checks: their sizes are bounds, which may be generous.
typedef __int128 wide;  // (strides are the caller's)
struct Array {
  const char* name;
  const void* at;
  int64_t rows;
  wide stride;
  int64_t width;
  bool written;
};
Array array(const char* name, const void* at, int64_t bytes, bool written = false) {
  return Array{name, at, 1, 0, bytes, written};
}

// Whether two arrays share a byte: exact where their strides are alike, so that an array may lie
// in the gaps of another's rows; else whether the ranges from first to last byte do.
bool overlap(const Array& a, const Array& b) {
  if (!a.at || !b.at || a.width <= 0 || b.width <= 0) return false;
  const wide d = (wide)reinterpret_cast<uintptr_t>(b.at) - (wide)reinterpret_cast<uintptr_t>(a.at);
  if (d >= (wide)(a.rows - 1) * a.stride + a.width || -d >= (wide)(b.rows - 1) * b.stride + b.width) return false;
  if (a.rows > 1 && b.rows > 1 && a.stride != b.stride) return true;
  const wide s = a.rows > 1 ? a.stride : b.stride;
  if (s <= 0) return true;
  // row j of b lies d + (j - i) s behind row i of a: the first j - i that is more than -b.width
  const wide x = -(wide)b.width - d;
  wide m = (x >= 0 ? x / s : -((-x + s - 1) / s)) + 1;
  m = std::max<wide>(m, -(wide)(a.rows - 1));
  return m <= b.rows - 1 && d + m * s < a.width;
}
// HS_EINVAL if one that the call writes overlaps another (one that is read and written in place is
// named once: its input is given without an address).
hs_status apart(std::initializer_list<Array> arrays) {
  for (auto a = arrays.begin(); a != arrays.end(); ++a)
    for (auto b = a + 1; b != arrays.end(); ++b) {
      if (!(a->written || b->written) || !overlap(*a, *b)) continue;
      return fail(HS_EINVAL, std::string(a->name) + " and " + b->name + " overlap");
    }
  return HS_OK;
}

hs_status ws_ok(const void* ws, uint64_t bytes, uint64_t need) {
  if (bytes < need)
    return fail(HS_ERANGE, "workspace of " + std::to_string(bytes) + " bytes, needs " + std::to_string(need));
  if (need && !ws) return fail(HS_EINVAL, "null workspace");
  if (!aligned(ws, 16)) return fail(HS_EINVAL, "workspace not 16-byte aligned");
  return HS_OK;
}

// Angle per position of every pair, in units of 2^-64 turns (whole turns do not count).
hs_status rope_turns(int32_t rot, double base, const hs_rope_scaling& c, uint64_t* turns) {
  constexpr double kTwoPi = 6.283185307179586476925;
  if (c.kind < HS_ROPE_PLAIN || c.kind > HS_ROPE_YARN) return fail(HS_EINVAL, "unknown rotary scaling");
  if (!(c.magnitude > 0) || !std::isfinite((float)c.magnitude))
    return fail(HS_EINVAL, "magnitude must be positive, and of float32");
  const bool banded = c.kind == HS_ROPE_BANDS || c.kind == HS_ROPE_YARN;
  if (c.kind != HS_ROPE_PLAIN && (!(c.factor > 0) || !std::isfinite(c.factor)))
    return fail(HS_EINVAL, "factor must be positive");
  if (banded && (c.original_ctx < 1 || !(c.low > 0) || !(c.low < c.high) || !std::isfinite(c.high)))
    return fail(HS_EINVAL, "needs original_ctx >= 1 and 0 < low < high");
  if (c.kind == HS_ROPE_NTK) base *= pow(c.factor, rot / (rot - 2.0));
  if (!(base > 1) || !std::isfinite(base)) return fail(HS_EINVAL, "base must be above 1");
  const auto at = [&](double x) { return rot * log(c.original_ctx / (kTwoPi * x)) / (2 * log(base)); };
  const double a = banded ? std::max(0.0, floor(at(c.high))) : 0.0;
  const double b = banded ? std::min(rot - 1.0, ceil(at(c.low))) : 0.0;
  for (int i = 0; i < rot / 2; ++i) {
    double w = pow(base, -2.0 * i / rot), keep = 1.0;  // the share of w that is not stretched
    if (c.kind == HS_ROPE_LINEAR) keep = 0.0;
    if (c.kind == HS_ROPE_BANDS) keep = (c.original_ctx * w / kTwoPi - c.low) / (c.high - c.low);
    if (c.kind == HS_ROPE_YARN) keep = 1.0 - (i - a) / std::max(b - a, 1e-3);
    keep = std::min(1.0, std::max(0.0, keep));
    if (keep < 1.0) w = (1.0 - keep) * w / c.factor + keep * w;
    if (!std::isfinite(w)) return fail(HS_EINVAL, "factor too small");
    const double t = w / kTwoPi;
    turns[i] = static_cast<uint64_t>(ldexp(t - floor(t), 64));
  }
  return HS_OK;
}
}  // namespace

extern "C" hs_status hs_k_rope_tables(float* cos_t, float* sin_t, int32_t max_pos, int32_t rot_dim,
                                      double base, const hs_rope_scaling* scaling, void* stream) {
  try {
    if (!cos_t || !sin_t || max_pos < 1) return fail(HS_EINVAL, "bad arguments");
    if (rot_dim < 8 || rot_dim > 128 || rot_dim % 8)
      return fail(HS_EINVAL, "rot_dim must be a multiple of 8 up to 128");
    if (!aligned(cos_t, 16) || !aligned(sin_t, 16)) return fail(HS_EINVAL, "tables not 16-byte aligned");
    const hs_rope_scaling plain{HS_ROPE_PLAIN, 0, 1.0, 0.0, 0.0, 1.0};
    const hs_rope_scaling& c = scaling ? *scaling : plain;
    uint64_t turns[64];
    const hs_status r = rope_turns(rot_dim, base, c, turns);
    if (r != HS_OK) return r;
    return done(rope_tables(cos_t, sin_t, max_pos, rot_dim / 2, turns, (float)c.magnitude,
                            static_cast<hipStream_t>(stream)),
                "rope_tables");
  } catch (...) {
    return fail(HS_EINVAL, "unexpected internal error");
  }
}

extern "C" hs_status hs_k_rope_kv(const void* qkv, int64_t ldqkv, const int32_t* pos,
                                  const int32_t* slot, const float* cos_t, const float* sin_t,
                                  int32_t max_pos, int32_t rot_dim, int32_t layout, void* q_out,
                                  int64_t ldq, void* k_out, int64_t ldk, void* pool,
                                  int32_t pool_blocks, int32_t T, int32_t n_heads,
                                  int32_t n_kv_heads, int32_t head_dim, void* stream) {
  try {
    if (!qkv || !pos || !slot || !cos_t || !sin_t || !q_out || !pool || T < 1 || max_pos < 1 ||
        pool_blocks < 1)
      return fail(HS_EINVAL, "bad arguments");
    const hs_status h = heads_ok(n_heads, n_kv_heads, head_dim);
    if (h != HS_OK) return h;
    if (rot_dim < 16 || rot_dim > head_dim || rot_dim % 16)
      return fail(HS_EINVAL, "rot_dim must be a multiple of 16 up to head_dim");
    if (layout != 0 && layout != 1) return fail(HS_EINVAL, "layout must be 0 or 1");
    if (ldqkv < (int64_t)(n_heads + 2 * n_kv_heads) * head_dim || ldq < (int64_t)n_heads * head_dim ||
        (k_out && ldk < (int64_t)n_kv_heads * head_dim))
      return fail(HS_EINVAL, "rows narrower than their heads");
    if (ldqkv % 8 || ldq % 8 || (k_out && ldk % 8) || !aligned(qkv, 16) || !aligned(q_out, 16) ||
        !aligned(k_out, 16) || !aligned(pool, 16) || !aligned(cos_t, 16) || !aligned(sin_t, 16) ||
        !aligned(pos, 4) || !aligned(slot, 4))
      return fail(HS_EINVAL, "pointers or row strides not aligned");
    // in place, or apart
    const int64_t nq = 2ll * n_heads * head_dim, nk = 2ll * n_kv_heads * head_dim, kv = nq + nk;
    const wide ld = 2 * (wide)ldqkv;
    const char* const x = static_cast<const char*>(qkv);
    const bool q_in_place = q_out == qkv && ldq == ldqkv, k_in_place = k_out == x + nq && ldk == ldqkv;
    const hs_status o = apart({{"the queries", q_in_place ? nullptr : x, T, ld, nq, false},
                               {"the keys", k_in_place ? nullptr : x + nq, T, ld, nk, false},
                               {"the values", x + kv, T, ld, nk, false},
                               {"q_out", q_out, T, 2 * (wide)ldq, nq, true},
                               {"k_out", k_out, T, 2 * (wide)ldk, nk, true},
                               array("pos", pos, 4ll * T), array("slot", slot, 4ll * T)});
    if (o != HS_OK) return o;
    RopeKvAtArgs a{static_cast<const bf16_t*>(qkv), ldqkv, pos, slot, cos_t, sin_t, max_pos, rot_dim,
                   layout == 1, static_cast<bf16_t*>(q_out), ldq, static_cast<bf16_t*>(k_out), k_out ? ldk : 0,
                   static_cast<bf16_t*>(pool), pool_blocks, T, n_heads, n_kv_heads, head_dim};
    return done(rope_kv_at(a, static_cast<hipStream_t>(stream)), "rope_kv");
  } catch (...) {
    return fail(HS_EINVAL, "unexpected internal error");
  }
}

namespace {
hs_status cache_attn_sizes(int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                           int32_t prefix_len, int32_t max_ctx) {
  if (B < 1 || B > 65535 || prefix_len < 0 || max_ctx < 0 || prefix_len > 1 << 30 || max_ctx > 1 << 30)
    return fail(HS_EINVAL, "bad arguments");
  const hs_status h = heads_ok(n_heads, n_kv_heads, head_dim);
  if (h != HS_OK) return h;
  // partial results and scores fit 2^50 bytes, so no size or index below overflows
  if ((double)B * n_heads * ((prefix_len + (double)max_ctx) / 128 + 2) * (head_dim + 130) > (double)(1ll << 48))
    return fail(HS_EINVAL, "too many sequences, heads and tokens");
  return HS_OK;
}

hs_status cache_attn_ws(int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                        int32_t prefix_len, int32_t max_ctx, bool weights, uint64_t* bytes) {
  if (!bytes) return fail(HS_EINVAL, "bad arguments");
  const hs_status r = cache_attn_sizes(B, n_heads, n_kv_heads, head_dim, prefix_len, max_ctx);
  if (r != HS_OK) return r;
  const CacheAttnPlan p = cache_attn_plan(B, n_heads, n_kv_heads, head_dim, prefix_len, max_ctx, weights);
  if (!p.fits) return fail(HS_EINVAL, "too many sequences, heads and tokens for a launch");
  *bytes = 4ull * p.floats;
  return HS_OK;
}

hs_status cache_attn_call(CacheAttnArgs a, bool weights, void* ws, uint64_t ws_bytes, void* stream) {
  const hs_status r = cache_attn_sizes(a.B, a.n_heads, a.n_kv_heads, a.D, a.prefix_len, a.max_ctx);
  if (r != HS_OK) return r;
  if (!a.q || !a.pool || !a.ctx || !a.out || a.pool_blocks < 1 || (a.prefix_len && !a.prefix) ||
      (a.max_ctx && !a.block_table))
    return fail(HS_EINVAL, "bad arguments");
  a.G = a.n_heads / a.n_kv_heads;
  if (!a.max_ctx) a.max_blocks = 0;  // no table to read
  if (a.max_ctx && a.max_blocks < (a.max_ctx + 15) / 16) return fail(HS_EINVAL, "block table too narrow");
  if (a.ldq < (int64_t)a.n_heads * a.D || a.ldo < (int64_t)a.n_heads * a.D)
    return fail(HS_EINVAL, "rows narrower than their heads");
  if (a.ldq % 8 || !aligned(a.q, 16) || !aligned(a.pool, 16) || !aligned(a.out, 4) || a.ldo % 2 ||
      !aligned(a.prefix, 4) || !aligned(a.block_table, 4) || !aligned(a.ctx, 4))
    return fail(HS_EINVAL, "pointers or row strides not aligned");
  if (weights) {
    if (a.max_ctx && (!a.acc || !a.acc_out)) return fail(HS_EINVAL, "null weights");
    if (a.acc_stride < a.max_ctx) return fail(HS_EINVAL, "rows of weights shorter than max_ctx");
    if (!(a.decay >= 0) || !std::isfinite(a.decay)) return fail(HS_EINVAL, "decay must be finite and not negative");
    if (a.pos && !a.seen) return fail(HS_EINVAL, "positions without the tokens seen");
    if (!aligned(a.acc, 4) || !aligned(a.acc_out, 4) || !aligned(a.pos, 4) || !aligned(a.seen, 4))
      return fail(HS_EINVAL, "pointers or row strides not aligned");
  }
  const CacheAttnPlan p =
      cache_attn_plan(a.B, a.n_heads, a.n_kv_heads, a.D, a.prefix_len, a.max_ctx, weights);
  if (!p.fits) return fail(HS_EINVAL, "too many sequences, heads and tokens for a launch");
  const hs_status w = ws_ok(ws, ws_bytes, 4ull * p.floats);
  if (w != HS_OK) return w;
  const int64_t width = 2ll * a.n_heads * a.D, rows = (int64_t)a.B * a.n_kv_heads, tokens = weights ? 4ll * a.max_ctx : 0;
  const hs_status o = apart({{"q", a.q, a.B, 2 * (wide)a.ldq, width, false},
                             {"out", a.out, a.B, 2 * (wide)a.ldo, width, true},
                             array("prefix", a.prefix, 4 * (((int64_t)a.prefix_len + 15) / 16)),
                             array("block_table", a.block_table, 4ll * a.B * a.max_blocks),
                             array("ctx", a.ctx, 4ll * a.B),
                             array("ws", ws, 4 * p.floats, true),
                             {"acc", a.acc == a.acc_out ? nullptr : a.acc, rows, 4 * (wide)a.acc_stride, tokens, false},
                             {"acc_out", a.acc_out, rows, 4 * (wide)a.acc_stride, tokens, true},
                             {"pos", a.pos, rows, 4 * (wide)a.acc_stride, tokens, true},
                             array("seen", a.pos ? a.seen : nullptr, 4ll * a.B)});
  if (o != HS_OK) return o;
  return done(cache_attn(a, p, static_cast<float*>(ws), static_cast<hipStream_t>(stream)), "cache attention");
}
}  // namespace

extern "C" hs_status hs_k_attn_decode_shared_ws(int32_t B, int32_t n_heads, int32_t n_kv_heads,
                                                int32_t head_dim, int32_t prefix_len,
                                                int32_t max_ctx, uint64_t* bytes) {
  try {
    return cache_attn_ws(B, n_heads, n_kv_heads, head_dim, prefix_len, max_ctx, false, bytes);
  } catch (...) {
    return fail(HS_EINVAL, "unexpected internal error");
  }
}

extern "C" hs_status hs_k_attn_decode_shared(
    const void* q, int64_t ldq, const void* pool, int32_t pool_blocks, const int32_t* prefix,
    int32_t prefix_len, const int32_t* block_table, const int32_t* ctx, void* out, int64_t ldo,
    int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_blocks,
    int32_t max_ctx, void* ws, uint64_t ws_bytes, void* stream) {
  try {
    CacheAttnArgs a{};
    a.q = static_cast<const bf16_t*>(q), a.ldq = ldq;
    a.pool = static_cast<const bf16_t*>(pool), a.pool_blocks = pool_blocks;
    a.prefix = prefix, a.prefix_len = prefix_len;
    a.block_table = block_table, a.ctx = ctx;
    a.out = static_cast<bf16_t*>(out), a.ldo = ldo;
    a.B = B, a.n_heads = n_heads, a.n_kv_heads = n_kv_heads, a.D = head_dim;
    a.max_blocks = max_blocks, a.max_ctx = max_ctx;
    return cache_attn_call(a, false, ws, ws_bytes, stream);
  } catch (...) {
    return fail(HS_EINVAL, "unexpected internal error");
  }
}

extern "C" hs_status hs_k_attn_decode_weights_ws(int32_t B, int32_t n_heads, int32_t n_kv_heads,
                                                 int32_t head_dim, int32_t prefix_len,
                                                 int32_t max_ctx, uint64_t* bytes) {
  try {
    return cache_attn_ws(B, n_heads, n_kv_heads, head_dim, prefix_len, max_ctx, true, bytes);
  } catch (...) {
    return fail(HS_EINVAL, "unexpected internal error");
  }
}

extern "C" hs_status hs_k_attn_decode_weights(
    const void* q, int64_t ldq, const void* pool, int32_t pool_blocks, const int32_t* prefix,
    int32_t prefix_len, const int32_t* block_table, const int32_t* ctx, void* out, int64_t ldo,
    const float* acc, float* acc_out, int64_t acc_stride, float decay, int32_t* pos,
    const int32_t* seen, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
    int32_t max_blocks, int32_t max_ctx, void* ws, uint64_t ws_bytes, void* stream) {
  try {
    CacheAttnArgs a{};
    a.q = static_cast<const bf16_t*>(q), a.ldq = ldq;
    a.pool = static_cast<const bf16_t*>(pool), a.pool_blocks = pool_blocks;
    a.prefix = prefix, a.prefix_len = prefix_len;
    a.block_table = block_table, a.ctx = ctx;
    a.out = static_cast<bf16_t*>(out), a.ldo = ldo;
    a.acc = acc, a.acc_out = acc_out, a.acc_stride = acc_stride, a.decay = decay;
    a.pos = pos, a.seen = seen;
    a.B = B, a.n_heads = n_heads, a.n_kv_heads = n_kv_heads, a.D = head_dim;
    a.max_blocks = max_blocks, a.max_ctx = max_ctx;
    return cache_attn_call(a, true, ws, ws_bytes, stream);
  } catch (...) {
    return fail(HS_EINVAL, "unexpected internal error");
  }
}

namespace {
// moves a row can have
int64_t evict_cap(int32_t keep, int32_t max_ctx) {
  return std::max<int64_t>(0, std::min<int64_t>(keep, (int64_t)max_ctx - keep));
}
hs_status evict_sizes(int32_t B, int32_t n_kv_heads, int32_t keep, int32_t max_ctx) {
  if (B < 1 || B > 65535 || n_kv_heads < 1 || n_kv_heads > 65535 || keep < 1 || max_ctx < 1 || max_ctx > 1 << 30)
    return fail(HS_EINVAL, "bad arguments");
  if ((double)B * n_kv_heads * max_ctx > (double)(1ll << 48))
    return fail(HS_EINVAL, "too many sequences, heads and tokens");
  if (evict_cap(keep, max_ctx) > kEvictMoves) return fail(HS_EINVAL, "more than 2^25 tokens of a row can move");
  return HS_OK;
}
uint64_t evict_bytes(int32_t B, int32_t n_kv_heads, int32_t keep, int32_t max_ctx) {
  return 4ull * B * n_kv_heads * (2 * evict_cap(keep, max_ctx) + 1);
}
}  // namespace

extern "C" hs_status hs_k_kv_evict_ws(int32_t B, int32_t n_kv_heads, int32_t keep, int32_t max_ctx,
                                      uint64_t* bytes) {
  try {
    if (!bytes) return fail(HS_EINVAL, "bad arguments");
    const hs_status r = evict_sizes(B, n_kv_heads, keep, max_ctx);
    if (r != HS_OK) return r;
    *bytes = evict_bytes(B, n_kv_heads, keep, max_ctx);
    return HS_OK;
  } catch (...) {
    return fail(HS_EINVAL, "unexpected internal error");
  }
}

extern "C" hs_status hs_k_kv_evict(void* pool, int32_t pool_blocks, const int32_t* block_table,
                                   const int32_t* ctx, const int32_t* seen, const float* acc,
                                   const int32_t* pos, int64_t stride, float* acc_out,
                                   int32_t* pos_out, int64_t out_stride, int32_t* ctx_out,
                                   int32_t keep, int32_t sinks, int32_t recent, int32_t B,
                                   int32_t n_kv_heads, int32_t head_dim, int32_t max_blocks,
                                   int32_t max_ctx, void* ws, uint64_t ws_bytes, void* stream) {
  try {
    const hs_status r = evict_sizes(B, n_kv_heads, keep, max_ctx);
    if (r != HS_OK) return r;
    if (!pool || !block_table || !ctx || !seen || !acc || !pos || !acc_out || !pos_out || !ctx_out ||
        pool_blocks < 1 || pool_blocks > 1 << 27 || sinks < 0 || recent < 0 || ctx_out == ctx)
      return fail(HS_EINVAL, "bad arguments");
    if (head_dim != 64 && head_dim != 128) return fail(HS_EINVAL, "head_dim must be 64 or 128");
    if (max_blocks < (max_ctx + 15) / 16) return fail(HS_EINVAL, "block table too narrow");
    if (stride < max_ctx || out_stride < std::min(keep, max_ctx))
      return fail(HS_EINVAL, "rows of weights shorter than their tokens");
    if ((static_cast<const void*>(acc) == acc_out || static_cast<const void*>(pos) == pos_out) && stride != out_stride)
      return fail(HS_EINVAL, "weights written in place need one stride");
    if (!aligned(pool, 16) || !aligned(block_table, 4) || !aligned(ctx, 4) || !aligned(seen, 4) ||
        !aligned(acc, 4) || !aligned(pos, 4) || !aligned(acc_out, 4) || !aligned(pos_out, 4) ||
        !aligned(ctx_out, 4))
      return fail(HS_EINVAL, "pointers not aligned");
    const hs_status w = ws_ok(ws, ws_bytes, evict_bytes(B, n_kv_heads, keep, max_ctx));
    if (w != HS_OK) return w;
    const int64_t rows = (int64_t)B * n_kv_heads, tokens = 4ll * max_ctx, kept = 4ll * std::min(keep, max_ctx);
    const hs_status o = apart({array("block_table", block_table, 4ll * B * max_blocks),
                               array("ctx", ctx, 4ll * B), array("seen", seen, 4ll * B),
                               {"acc", acc == acc_out ? nullptr : acc, rows, 4 * (wide)stride, tokens, false},
                               {"pos", pos == pos_out ? nullptr : pos, rows, 4 * (wide)stride, tokens, false},
                               {"acc_out", acc_out, rows, 4 * (wide)out_stride, acc == acc_out ? tokens : kept, true},
                               {"pos_out", pos_out, rows, 4 * (wide)out_stride, pos == pos_out ? tokens : kept, true},
                               array("ctx_out", ctx_out, 4ll * B, true),
                               array("ws", ws, (int64_t)evict_bytes(B, n_kv_heads, keep, max_ctx), true)});
    if (o != HS_OK) return o;
    KvEvictArgs a{static_cast<bf16_t*>(pool), pool_blocks, block_table, ctx, seen, acc, pos, stride,
                  acc_out, pos_out, out_stride, ctx_out, keep, sinks, recent, B, n_kv_heads, head_dim,
                  max_blocks, max_ctx, static_cast<int32_t*>(ws), (int)evict_cap(keep, max_ctx), nullptr};
    a.counts = a.lists + 2ll * B * n_kv_heads * a.cap;
    return done(kv_evict(a, static_cast<hipStream_t>(stream)), "kv_evict");
  } catch (...) {
    return fail(HS_EINVAL, "unexpected internal error");
  }
}
