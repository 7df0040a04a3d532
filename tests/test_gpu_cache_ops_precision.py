"""What the cache operators keep of float32: bounds without room for a rounding to
bf16 (2^-8 of the value) but the output's own."""
import numpy as np
import pytest

from tests import gpu_util as G
from tests.test_gpu_cache_ops import BF, F32, Cache, _hs, host, run_shared, turns

pytestmark = pytest.mark.gpu


def sharp(lens, prefix, nh, nkv, d, seed):
    """A cache whose queries and keys are multiples of 1/2 of at most 6: scores before their
    scale are sums of d multiples of 1/4 below 36 each, at most 2^15 of 1/4, exact in float32."""
    c = Cache(lens, prefix, nh, nkv, d, seed, std=1.5)
    few = lambda x: np.clip(np.round(2 * x) / 2, -6, 6).astype(np.float32)  # noqa: E731
    c.q = few(c.q)
    for b in range(c.B):
        c.k[b] = few(c.k[b])
    for t in range(prefix):
        c._put(c.prefix[t // 16], t % 16, c.k[0][t], c.v[0][t])
    for b, n in enumerate(lens):
        for t in range(n):
            c._put(c.table[b, t // 16], t % 16, c.k[b][prefix + t], c.v[b][prefix + t])
    return c


@pytest.mark.parametrize("lens,prefix,nh,nkv,d", [
    ([100, 5, 17], 0, 4, 4, 64), ([90, 30], 20, 32, 8, 128), ([250, 131], 0, 8, 8, 128), ([200, 3], 40, 16, 4, 64),  # alone
    ([1000, 700, 300] * 11, 0, 16, 4, 128), ([600] * 32, 0, 4, 4, 64),  # alone, several steps
    ([700, 1300], 0, 8, 8, 128), ([1100], 0, 8, 2, 64),  # splits
    ([40, 0, 33], 300, 8, 8, 128), ([700, 20], 900, 6, 2, 64), ([130] * 9, 1500, 16, 2, 128)])  # behind a prefix
def test_probabilities_keep_15_bits(lens, prefix, nh, nkv, d):
    """|error| <= half a bf16 step of the output, and of sum p |v|: 2^-15 (the probabilities of the
    second product), and float32's: a score's error is its scale's and its product's rounding, the
    maximum's and the subtraction's, 6 x 2^-24 of the largest score, twice (the probability's and
    the sum's); exp2 and the merges' factors 32 steps, the sums n. Rounded to bf16 the probabilities
    would be off by up to 2^-8, and outputs near zero by more than this."""
    c = sharp(lens, prefix, nh, nkv, d, 100 + len(lens) + prefix)
    got = run_shared(c)
    g = nh // nkv
    for b in range(c.B):
        o, _, p, _ = c.exact(b)
        n = prefix + lens[b]
        if n == 0:
            assert np.all(got[b] == 0)
            continue
        q = c.q[b].reshape(nkv, g, d).astype(np.float64)
        k, v = c.k[b].astype(np.float64).transpose(1, 2, 0), c.v[b].astype(np.float64).transpose(1, 0, 2)
        s = np.abs(q @ k).max(axis=2, keepdims=True) / np.sqrt(d) * 1.4426950408889634
        rel = 2.0 ** -15 + (12 * s + n + 32) * F32
        tol = BF * np.abs(o) + (rel * (p.reshape(nkv, g, n) @ np.abs(v))).reshape(-1)
        assert np.all(np.abs(got[b] - o) <= tol), (b, (np.abs(got[b] - o) / tol).max())


@pytest.mark.parametrize("lens,prefix", [([40, 3], 0), ([40, 3], 300), ([900] * 3, 0), ([900, 700], 1500)])
@pytest.mark.parametrize("d", [64, 128])
def test_an_infinite_value_gives_infinity(lens, prefix, d):
    """Infinite values of tokens with a probability above zero: the output is infinite with their
    sign, in the columns that have one, and finite in the others."""
    c = sharp(lens, prefix, 8, 2, d, 5)
    c.pool[c.table[0, 0], 1, 1, 2, 3] = np.inf
    c.pool[c.table[0, 2], 1, 1, 7, 9] = -np.inf
    if prefix:
        c.pool[c.prefix[8], 1, 0, 5, 21] = -np.inf
    got = run_shared(c)[:2].reshape(2, 2, 4, d)
    want = np.zeros((2, 2, 4, d))
    want[0, 1, :, 3], want[0, 1, :, 9] = np.inf, -np.inf
    if prefix:
        want[:, 0, :, 21] = -np.inf
    assert np.array_equal(np.where(np.isfinite(got), 0, got), want)


@pytest.mark.parametrize("lens,prefix", [([40, 3], 0), ([40, 3], 300), ([900] * 3, 0), ([900, 700], 1500)])
@pytest.mark.parametrize("d", [64, 128])
def test_a_large_value_without_probability_adds_nothing(lens, prefix, d):
    """A token whose score is several hundred below the others has probability zero in float32, and
    in float64 less than 10^-100: its values of 2^127 add nothing to any output."""
    c = sharp(lens, prefix, 4, 4, d, 6)
    c.k[0][prefix + 17] = -64 * np.where(c.q[0] < 0, -1, 1).reshape(4, d)
    c.v[0][prefix + 17] = 2.0 ** 127
    c._put(c.table[0, 1], 1, c.k[0][prefix + 17], c.v[0][prefix + 17])
    got = run_shared(c)
    q = c.q[0].reshape(4, 1, d).astype(np.float64)
    s = (q @ c.k[0].astype(np.float64).transpose(1, 2, 0)) / np.sqrt(d)
    assert np.all(s[:, :, prefix + 17] < s.max(axis=2) - 200)
    o, tol, _, _ = c.exact(0, [prefix + 17])
    assert np.all(np.abs(tol) < 1)
    assert np.all(np.abs(got[0] - o) <= tol), np.abs(got[0] - o).max()


@pytest.mark.parametrize("rot,base,kind,factor,original", [
    (128, 500000.0, "linear", 8.0, 0), (128, 500000.0, "bands", 8.0, 8192), (64, 10000.0, "plain", 1.0, 0), (16, 1e9, "plain", 1.0, 0),
    (128, 1e12, "linear", 1e4, 0), (96, 10000.0, "yarn", 16.0, 256), (8, 2.0, "ntk", 32.0, 0)])
def test_small_angles_are_as_exact_as_large_ones(rot, base, kind, factor, original):
    """|error| <= 6 x 2^-24 of the value: two half steps from the 64-bit fraction to float32, one of
    the polynomial's sum, one of its inner terms together (a fifth of it at most), the
    magnitude's and the product's. The fraction itself: 2^-64 of a turn and 2^-50 of the
    frequency (float64) a position. At the first positions the slowest pairs turn by less than
    2^-32, and their sines are that small."""
    torch = G.torch()
    hs = _hs()
    sc = hs.rope_scaling(kind, factor=factor, original_ctx=original)
    w = turns(rot, base, kind, factor, original, sc.low, sc.high)
    n = 200
    out = torch.zeros((2, n, rot // 2), dtype=torch.float32, device="cuda")
    hs.hs_k_rope_tables(out[0].data_ptr(), out[1].data_ptr(), n, rot, base, sc, G.stream_ptr())
    got = host(out).astype(np.float64)
    pos = np.arange(n, dtype=np.longdouble)[:, None]
    ang = pos * w
    for at, f in ((0, np.cos), (1, np.sin)):
        want = f(ang) * sc.magnitude
        tol = 6 * F32 * np.abs(want) + sc.magnitude * pos * (6.3 * 2.0 ** -64 + w * 2.0 ** -50)
        off = np.abs(got[at] - want)
        assert np.all(off <= tol), (at, np.unravel_index(np.argmax(off - tol), off.shape), (off / np.maximum(tol, 1e-30)).max())
