"""Arrays of the cache operators that lie in the gaps of one another's rows."""
import numpy as np
import pytest

from tests import gpu_util as G
from tests.test_gpu_cache_ops import Cache, _hs, bf, dev, dev_bf, host, workspace

pytestmark = pytest.mark.gpu


def test_rope_kv_output_in_the_gaps_of_its_input():
    """Queries and keys written behind the heads of the rows that they come from: the same bits as apart."""
    torch = G.torch()
    hs = _hs()
    T, nh, nkv, d, rot, blocks = 33, 8, 2, 64, 32, 4
    rng = np.random.default_rng(1)
    width, nq, nk = (nh + 2 * nkv) * d, nh * d, nkv * d
    ld = width + nq + nk + 24
    x = bf(rng, (T, ld))
    pos, slot = dev(rng.integers(0, 90, T).astype(np.int32)), dev(rng.permutation(blocks * 16)[:T].astype(np.int32))
    ang = rng.uniform(0, 6.28, (90, rot // 2))
    cos, sin = dev(np.cos(ang).astype(np.float32)), dev(np.sin(ang).astype(np.float32))
    got = []
    for gaps in (False, True):
        qkv, pool = dev_bf(x), torch.zeros((blocks, 2, nkv, 16, d), dtype=torch.bfloat16, device="cuda")
        q, k = torch.zeros((T, nq), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, nk), dtype=torch.bfloat16, device="cuda")
        if gaps:
            q, k = qkv[:, width:width + nq], qkv[:, width + nq:width + nq + nk]
        hs.hs_k_rope_kv(qkv.data_ptr(), ld, pos.data_ptr(), slot.data_ptr(), cos.data_ptr(), sin.data_ptr(), 90, rot, "interleaved", q.data_ptr(),
                        q.stride(0), k.data_ptr(), k.stride(0), pool.data_ptr(), blocks, T, nh, nkv, d, G.stream_ptr())
        got.append([host(t.contiguous()) for t in (q, k, pool, qkv[:, :width], qkv[:, width + nq + nk:])])
    assert np.abs(got[0][0]).max() > 0
    for a, b in zip(*got):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("lens,prefix", [([40, 7], 30), ([700, 1300], 900)])
def test_weights_and_positions_in_one_buffer(lens, prefix):
    """acc, acc_out and pos as columns of the same rows, in the attention and in the eviction."""
    torch = G.torch()
    hs = _hs()
    nh, nkv, d, keep = 8, 2, 64, 32
    c = Cache(lens, prefix, nh, nkv, d, 2, wild=False)
    dv, most, B = c.device(), c.max_ctx, c.B
    rng = np.random.default_rng(3)
    acc, pos = np.exp(rng.standard_normal((B, nkv, most))).astype(np.float32), np.tile(np.arange(most, dtype=np.int32), (B, nkv, 1))
    seen = dev(np.array(lens, np.int32))
    nw, ne = hs.hs_k_attn_decode_weights_ws(B, nh, nkv, d, prefix, most), hs.hs_k_kv_evict_ws(B, nkv, keep, most)
    w1, w2 = workspace(nw), workspace(ne)
    got = []
    for one in (False, True):
        pool = dv["pool"].clone()
        buf = torch.zeros((B, nkv, 5, most + 1), dtype=torch.float32, device="cuda")
        cols = [buf[:, :, i, :most] for i in range(5)]
        stride = 5 * (most + 1)
        if not one:
            cols, stride = [torch.zeros((B, nkv, most), dtype=torch.float32, device="cuda") for _ in range(5)], most
        a, a_out, a_end = cols[0], cols[1], cols[2]
        p, p_end = cols[3].view(torch.int32), cols[4].view(torch.int32)
        a.copy_(dev(acc))
        p.copy_(dev(pos))
        out = torch.zeros((B, nh * d), dtype=torch.bfloat16, device="cuda")
        left = torch.zeros(B, dtype=torch.int32, device="cuda")
        hs.hs_k_attn_decode_weights(dv["q"].data_ptr(), nh * d, pool.data_ptr(), c.blocks, dv["prefix"].data_ptr(), prefix, dv["table"].data_ptr(),
                                    dv["ctx"].data_ptr(), out.data_ptr(), nh * d, a.data_ptr(), a_out.data_ptr(), stride, 0.5, p.data_ptr(), seen.data_ptr(),
                                    B, nh, nkv, d, c.width, most, w1.data_ptr(), nw, G.stream_ptr())
        hs.hs_k_kv_evict(pool.data_ptr(), c.blocks, dv["table"].data_ptr(), dv["ctx"].data_ptr(), seen.data_ptr(), a_out.data_ptr(), p.data_ptr(), stride,
                         a_end.data_ptr(), p_end.data_ptr(), stride, left.data_ptr(), keep, 1, 4, B, nkv, d, c.width, most, w2.data_ptr(), ne,
                         G.stream_ptr())
        got.append([host(t.contiguous()) for t in (out, pool, left, *cols)])
        if one:
            assert not buf[:, :, :, most].any()
    assert (got[0][2] == np.minimum(lens, keep)).all()
    for x, y in zip(*got):
        assert np.array_equal(x, y)
