"""The cache operators in the forms that long prefixes, ragged batches and long rows take: rings that
wrap, sequences of several steps, every selecting form of the eviction at its edges."""
import numpy as np
import pytest

from tests import gpu_util as G
from tests import test_gpu_cache_ops as base
from tests.test_gpu_cache_ops import BF, F32, Cache, _hs, bf, dev, host, workspace

pytestmark = pytest.mark.gpu


def cut(P, max_ctx, prefix_tokens, own_blocks):
    """Splits of a call whose prefix is cut into prefix_tokens and whose sequences into own_blocks."""
    return -(-P // prefix_tokens) + -(-(-(-max_ctx // 16)) // own_blocks)


def splits(hs, B, nh, nkv, d, P, max_ctx):
    """Splits of a call, from the size of its workspace: d + 2 floats a split and query head."""
    return hs.hs_k_attn_decode_shared_ws(B, nh, nkv, d, P, max_ctx) // (4 * B * nh * (d + 2))


# own tokens, prefix, query heads, kv heads, head dim; tokens of a prefix split, blocks of an own one
LONG = [
    # prefix splits of 2 (the least) to 16 steps, the last ones of neither whole steps nor blocks
    ([37, 0, 300] * 11, 3999, 16, 1, 128, 192, 8), ([37, 0, 300] * 11, 3999, 16, 1, 64, 192, 8),
    ([5, 0, 130] * 11, 8005, 16, 1, 128, 320, 8), ([5, 0, 130] * 11, 8005, 16, 1, 64, 320, 8),
    ([1, 0, 64] * 11, 20011, 16, 1, 64, 704, 8), ([2] * 33, 20011, 16, 1, 128, 704, 8),
    ([3, 0, 17] * 11, 30011, 16, 1, 128, 1024, 8), ([3, 0, 17] * 11, 30011, 16, 1, 64, 1024, 8),
    # own splits of 16, 24 and 32 blocks: several steps of a sequence, ended inside one
    ([200, 129, 1, 0] * 8, 1500, 16, 8, 128, 128, 16), ([200, 129, 1, 0] * 8, 1500, 16, 8, 64, 128, 16),
    ([2100, 1, 700, 0, 385, 1999], 500, 16, 8, 128, 128, 24), ([2100, 1, 700, 0, 385, 1999], 500, 16, 8, 64, 128, 24),
    ([500, 257, 0, 511] * 8, 700, 8, 8, 128, 128, 32), ([500, 257, 0, 511] * 8, 700, 16, 8, 64, 128, 32),
    # both
    ([2100, 0, 33, 1300, 5, 260, 1, 383, 384, 385, 768] * 3, 8005, 16, 1, 128, 320, 16),
]


class Long(Cache):
    """A cache behind a long prefix: its keys grow or fade along the tokens, so that the largest score
    moves on or back through the steps; blocks of the prefix and of a sequence that name none of the pool."""

    def __init__(self, lens, P, nh, nkv, d, shape, seed):
        rng = np.random.default_rng(seed)
        self.lens, self.P, self.nh, self.nkv, self.d, self.B = list(lens), P, nh, nkv, d, len(lens)
        self.max_ctx = max(lens)
        n_own, n_pre = [-(-n // 16) for n in lens], -(-P // 16)
        self.width = max(max(n_own), 1) + 1
        self.blocks = sum(n_own) + n_pre + 2
        perm = rng.permutation(self.blocks).astype(np.int32)
        self.pool = np.full((self.blocks, 2, nkv, 16, d), np.nan, np.float32)
        self.pool[:, 1, :, 1::2] = np.inf
        self.prefix, self.table = perm[:n_pre].copy(), np.full((self.B, self.width), -7, np.int32)
        self.table[:, ::2] = 2 ** 31 - 1

        def rows(n, pages):
            std = {"grows": np.linspace(0.1, 1.6, n), "fades": np.linspace(1.6, 0.1, n), "even": np.ones(n)}[shape].astype(np.float32)
            k, v = bf(rng, (n, nkv, d)), bf(rng, (n, nkv, d))
            k = base.gen.round_to_bf16(k * std[:, None, None])
            t = np.arange(n)
            self.pool[pages[t // 16], 0, :, t % 16], self.pool[pages[t // 16], 1, :, t % 16] = k, v
            return k, v

        self.pre = rows(P, self.prefix)
        self.own, at = [], n_pre
        for b, n in enumerate(lens):
            self.table[b, :n_own[b]] = perm[at:at + n_own[b]]
            at += n_own[b]
            self.own.append(rows(n, self.table[b]))
        self.q = bf(rng, (self.B, nh * d), 1.5)
        self.ctx = np.array(lens, np.int32)
        # a block of the prefix in its second half and one of the longest sequence that name no block
        self.drop = {b: [] for b in range(self.B)}
        if n_pre > 30:
            j = n_pre - 7
            self.prefix[j] = self.blocks
            for b in self.drop:
                self.drop[b] += range(16 * j, min(16 * j + 16, P))
        b = int(np.argmax(lens))
        if n_own[b] > 12:
            self.table[b, 11] = -1
            self.drop[b] += range(P + 176, P + 192)

    def exact(self, b):
        """Output and bound, probabilities and theirs: scores as in Cache.exact, 2^-15 of a probability in
        the second product, sums of n terms."""
        g, d = self.nh // self.nkv, self.d
        n = self.P + self.lens[b]
        if n == 0:
            return np.zeros(self.nh * d), np.zeros(self.nh * d), np.zeros((self.nh, 0)), np.zeros((self.nh, 0))
        k, v = (np.concatenate([x, y]).astype(np.float64) for x, y in zip(self.pre, self.own[b]))
        k, v = k.transpose(1, 2, 0), v.transpose(1, 0, 2)
        q = self.q[b].reshape(self.nkv, g, d).astype(np.float64)
        s = q @ k / np.sqrt(d)
        s[:, :, self.drop[b]] = -np.inf
        ds = (d + 8) * F32 * (np.abs(q) @ np.abs(k)).max(axis=2, keepdims=True) / np.sqrt(d)
        e = np.exp(s - s.max(axis=2, keepdims=True))
        p = e / e.sum(axis=2, keepdims=True)
        o = p @ v
        rel = 2 * ds + (n + 16) * F32
        tol = BF * np.abs(o) + (2.0 ** -15 + rel) * (p @ np.abs(v)) + 1e-30
        return o.reshape(-1), tol.reshape(-1), p.reshape(self.nh, n), (p * rel).reshape(self.nh, n)


def check_weights(c, out, acc, old, pos, old_pos, seen, decay, exact):
    g = c.nh // c.nkv
    for b, n in enumerate(c.lens):
        o, tol, p, dp = exact[b]
        assert np.all(np.abs(out[b] - o) <= tol), (b, np.nanmax(np.abs(out[b] - o) / tol))
        want = p[:, c.P:].reshape(c.nkv, g, n).sum(1)
        bound = dp[:, c.P:].reshape(c.nkv, g, n).sum(1) + (g + 2) * F32 * want
        if n:
            was = old[b, :, :n - 1].astype(np.float64) * np.float64(decay)
            want[:, :n - 1] += was
            bound[:, :n - 1] += 2 * F32 * (was + want[:, :n - 1])
            assert np.all(np.abs(acc[b, :, :n] - want) <= bound + 1e-37), (b, np.abs(acc[b, :, :n] - want).max())
            assert np.all(pos[b, :, n - 1] == seen[b] - 1)
        rest = np.ones(pos.shape[1:], bool)
        if n:
            rest[:, n - 1] = False
        assert np.array_equal(pos[b][rest], old_pos[b][rest])
        assert np.array_equal(acc[b, :, n:], old[b, :, n:], equal_nan=True)


def run_weights(c, seed):
    """In place; the host's copies of what check_weights wants."""
    torch = G.torch()
    hs = _hs()
    rng = np.random.default_rng(seed)
    dv, stride, decay = c.device(), c.max_ctx + 5, np.float32(0.9)
    old = np.exp(rng.standard_normal((c.B, c.nkv, stride)) * 2).astype(np.float32)
    for b, n in enumerate(c.lens):
        old[b, :, max(0, n - 1):] = np.nan
    old_pos, seen = rng.integers(0, 1000, old.shape).astype(np.int32), rng.integers(5000, 6000, c.B).astype(np.int32)
    acc, pos, dseen = dev(old), dev(old_pos), dev(seen)
    out = torch.full((c.B + 1, c.nh * c.d), 7.0, dtype=torch.bfloat16, device="cuda")
    nbytes = hs.hs_k_attn_decode_weights_ws(c.B, c.nh, c.nkv, c.d, c.P, c.max_ctx)
    ws = workspace(nbytes)
    hs.hs_k_attn_decode_weights(dv["q"].data_ptr(), c.nh * c.d, dv["pool"].data_ptr(), c.blocks, dv["prefix"].data_ptr() if c.P else 0, c.P,
                                dv["table"].data_ptr(), dv["ctx"].data_ptr(), out.data_ptr(), c.nh * c.d, acc.data_ptr(), acc.data_ptr(),
                                stride, float(decay), pos.data_ptr(), dseen.data_ptr(), c.B, c.nh, c.nkv, c.d, c.width, c.max_ctx,
                                ws.data_ptr(), nbytes, G.stream_ptr())
    torch.cuda.synchronize()
    assert np.all(host(out)[c.B] == 7.0)
    return host(out), host(acc), old, host(pos), old_pos, seen, decay


@pytest.mark.parametrize("shape", ["grows", "fades"])
@pytest.mark.parametrize("lens,prefix,nh,nkv,d,prefix_tokens,own_blocks", LONG)
def test_attention_behind_long_prefixes(lens, prefix, nh, nkv, d, prefix_tokens, own_blocks, shape):
    """With and without weights, in the form that the sizes are meant to take."""
    assert splits(_hs(), len(lens), nh, nkv, d, prefix, max(lens)) == cut(prefix, max(lens), prefix_tokens, own_blocks)
    c = Long(lens, prefix, nh, nkv, d, shape, prefix + nh + d)
    got = base.run_shared(c)
    exact = [c.exact(b) for b in range(c.B)]
    for b in range(c.B):
        assert np.all(np.abs(got[b] - exact[b][0]) <= exact[b][1]), (b, np.nanmax(np.abs(got[b] - exact[b][0]) / exact[b][1]))
    assert np.all(got[c.B] == 7.0)
    res = run_weights(c, 1)
    assert np.array_equal(res[0][:c.B], got[:c.B])
    check_weights(c, *res, exact)


@pytest.mark.parametrize("lens,prefix,nh,nkv,d", [
    ([2100, 5, 1024, 1025], 0, 16, 1, 128), ([1500, 0, 700], 0, 12, 2, 64), ([3000, 2049], 0, 32, 4, 128),  # splits
    ([300, 20, 256], 0, 32, 2, 128), ([250, 0, 3], 0, 16, 1, 64), ([900] * 8, 0, 96, 16, 64), ([900, 3] * 4, 0, 96, 16, 128),  # alone
    ([1500, 1000, 40], 333, 32, 2, 64), ([2500, 1, 1024], 90, 16, 1, 128)])  # behind a prefix
def test_weights_of_many_query_heads_on_long_sequences(lens, prefix, nh, nkv, d):
    """More than four query heads of a kv head, whose scores are read one after another, over more
    than the 1024 tokens of a workgroup."""
    c = Long(lens, prefix, nh, nkv, d, "even", 3)
    check_weights(c, *run_weights(c, 2), [c.exact(b) for b in range(c.B)])


# the selecting form goes by the longest row (2048, 4096, 8192, 16384 tokens in registers, then LDS), moves in it by
# how many a row can have (512; 1024 from 256 rows on), lists in LDS up to 4096
SELECT = [
    ([2100, 2049, 2048, 7], 2048, 4, 256, 2, 128), ([2100, 2049, 2048, 7], 2048, 4, 256, 2, 64),  # 4 x 1024 in registers, moves here
    ([4300, 4097, 4096, 10], 4096, 0, 9, 2, 128), ([4300, 4097, 4096, 10], 4096, 0, 9, 2, 64),    # 8
    ([8300, 8193, 100], 8192, 2, 30, 1, 128), ([8300, 8193, 100], 8192, 2, 30, 1, 64),            # 16
    ([16500, 16385, 50], 16384, 3, 3, 1, 128), ([16500, 16385, 50], 16384, 3, 3, 1, 64),          # LDS
    ([7000, 6001, 900], 2000, 4, 64, 1, 128), ([7000, 6001, 900], 2000, 4, 64, 1, 64),            # 8, moved by the second kernel
    ([2000, 1500, 899], 900, 4, 0, 2, 128), ([3500, 2000], 1300, 0, 40, 1, 64),                   # 2, 4
    ([12000, 100], 6000, 4, 64, 1, 128), ([12000, 11999], 6000, 4, 64, 1, 64),                    # 16, lists in memory
    ([16384, 9000], 8192, 0, 0, 1, 128), ([8192, 8000], 4096, 0, 7, 1, 64),                       # 16, 8: the most moves there are
    ([1700] * 3 + [900] * 61, 800, 2, 50, 4, 64), ([1700] * 3 + [900] * 61, 800, 2, 50, 4, 128),  # 900 moves, 256 rows
    ([2900] * 2 + [30] * 62, 1900, 2, 50, 4, 128), ([5096, 4200] + [5] * 62, 4096, 1, 9, 4, 64), ([8920] + [5] * 63, 8000, 1, 9, 4, 128)]
EDGES = [(n, keep) for top in (2048, 4096, 8192, 16384) for n in (top - 1, top, top + 1) for keep in (n - 1, 100, n // 2)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["plain", "ties", "odd"])
@pytest.mark.parametrize("lens,keep,sinks,recent,nkv,d", SELECT)
def test_evictions_of_every_form(lens, keep, sinks, recent, nkv, d, kind, in_place):
    base.test_kv_evict(lens, keep, sinks, recent, nkv, d, kind, in_place)


@pytest.mark.parametrize("n,keep", EDGES)
def test_evictions_at_the_edges_of_the_forms(n, keep):
    base.test_kv_evict([n, max(1, n - 3)], keep, 2, 5, 1, 64, "ties" if n % 2 else "odd", n % 3 == 0)
