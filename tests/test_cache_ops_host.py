"""What the cache operators refuse, before anything reaches a GPU, and their workspace sizes."""
import math

import pytest

from paper_2502_15524_amd import hs

P = 1 << 20  # any aligned non-null value: nothing is dereferenced or launched


def refused(code, fn, *args, **kw):
    with pytest.raises(hs.HSError) as e:
        fn(*args, **kw)
    assert e.value.code == code, e.value


@pytest.mark.parametrize("change", [
    dict(cos_t=0), dict(sin_t=P + 4), dict(max_pos=0), dict(rot_dim=4), dict(rot_dim=136), dict(rot_dim=20), dict(base=1.0),
    dict(base=math.nan), dict(base=math.inf), dict(scaling=hs.hs_rope_scaling(5, 100, 2.0, 1.0, 4.0, 1.0)),
    dict(scaling=hs.rope_scaling("linear", factor=0.0)), dict(scaling=hs.rope_scaling("ntk", factor=math.inf)),
    dict(scaling=hs.rope_scaling("bands", factor=2.0)), dict(scaling=hs.rope_scaling("bands", factor=2.0, original_ctx=10, low=4.0)),
    dict(scaling=hs.rope_scaling("yarn", factor=2.0, original_ctx=10, low=0.0)),
    dict(scaling=hs.rope_scaling("yarn", factor=2.0, original_ctx=10, high=math.inf)),
    dict(scaling=hs.rope_scaling("linear", factor=2.0, magnitude=0.0)), dict(scaling=hs.rope_scaling("ntk", factor=1e300)),
    dict(scaling=hs.rope_scaling("linear", factor=2.0, magnitude=math.nan))])
def test_rope_tables_refuses(change):
    a = dict(cos_t=P, sin_t=P, max_pos=64, rot_dim=64, base=10000.0, scaling=None) | change
    refused(hs.HS_EINVAL, hs.hs_k_rope_tables, **a)


@pytest.mark.parametrize("change", [
    dict(qkv=0), dict(pos=0), dict(slot=0), dict(cos_t=0), dict(q_out=0), dict(pool=0), dict(T=0), dict(max_pos=0), dict(pool_blocks=0),
    dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144), dict(layout=2), dict(head_dim=96), dict(n_kv_heads=3), dict(n_kv_heads=0),
    dict(n_heads=0), dict(n_heads=136), dict(ldqkv=48 * 128 - 8), dict(ldq=32 * 128 - 8), dict(k_out=P, ldk=1016), dict(ldqkv=48 * 128 + 4),
    dict(ldq=32 * 128 + 2), dict(qkv=P + 2), dict(q_out=P + 8), dict(k_out=P + 4), dict(pool=P + 8), dict(cos_t=P + 8), dict(pos=P + 2)])
def test_rope_kv_refuses(change):
    a = dict(qkv=P, ldqkv=48 * 128, pos=P, slot=P, cos_t=P, sin_t=P, max_pos=64, rot_dim=128, layout="half", q_out=P, ldq=32 * 128,
             k_out=0, ldk=1024, pool=P, pool_blocks=4, T=3, n_heads=32, n_kv_heads=8, head_dim=128) | change
    refused(hs.HS_EINVAL, hs.hs_k_rope_kv, **a)


@pytest.mark.parametrize("change", [
    dict(q_out=P, ldq=48 * 128 + 8), dict(q_out=P + 256), dict(q_out=P - 4096), dict(k_out=P, ldk=48 * 128), dict(k_out=P + 32 * 256, ldk=1024),
    dict(k_out=P + 33 * 256, ldk=48 * 128)])
def test_rope_kv_refuses_rows_that_overlap(change):
    a = dict(qkv=P, ldqkv=48 * 128, pos=P, slot=P, cos_t=P, sin_t=P, max_pos=64, rot_dim=128, layout="half", q_out=16 * P, ldq=32 * 128,
             k_out=0, ldk=1024, pool=32 * P, pool_blocks=4, T=3, n_heads=32, n_kv_heads=8, head_dim=128) | change
    refused(hs.HS_EINVAL, hs.hs_k_rope_kv, **a)


def test_sizes_that_would_overflow_are_refused():
    for fn in (hs.hs_k_attn_decode_shared_ws, hs.hs_k_attn_decode_weights_ws):
        refused(hs.HS_EINVAL, fn, 65535, 65536, 65536, 128, 1 << 30, 1 << 30)
        refused(hs.HS_EINVAL, fn, 1, 32, 8, 128, (1 << 30) + 1, 1)
        assert fn(64, 32, 8, 128, 1 << 20, 1 << 20) > 0
    refused(hs.HS_EINVAL, hs.hs_k_kv_evict_ws, 65535, 65535, 1 << 29, 1 << 30)
    refused(hs.HS_EINVAL, hs.hs_k_kv_evict, **(EVICT | dict(pool_blocks=(1 << 27) + 1)))


ATTN = dict(q=P, ldq=4096, pool=P, pool_blocks=9, prefix=P, prefix_len=100, block_table=P, ctx=P, out=P, ldo=4096, B=2, n_heads=32,
            n_kv_heads=8, head_dim=128, max_blocks=4, max_ctx=64, ws=P, ws_bytes=1 << 40)
WEIGHTS = ATTN | dict(acc=P, acc_out=P, acc_stride=64, decay=1.0, pos=P, seen=P)
BAD = [dict(q=0), dict(pool=0), dict(ctx=0), dict(out=0), dict(prefix=0), dict(block_table=0), dict(pool_blocks=0), dict(prefix_len=-1),
       dict(max_ctx=-1), dict(B=0), dict(B=65536), dict(n_heads=30), dict(n_kv_heads=0), dict(n_heads=136, ldq=1 << 20, ldo=1 << 20),
       dict(head_dim=80), dict(max_ctx=65), dict(max_blocks=3), dict(ldq=4088), dict(ldo=4094), dict(ldq=4100), dict(ldo=4097), dict(q=P + 2),
       dict(pool=P + 8), dict(out=P + 2), dict(ctx=P + 1), dict(prefix=P + 2), dict(block_table=P + 2), dict(ws=P + 8), dict(ws=0)]


@pytest.mark.parametrize("change", BAD)
def test_attn_decode_shared_refuses(change):
    refused(hs.HS_EINVAL, hs.hs_k_attn_decode_shared, **(ATTN | change))


@pytest.mark.parametrize("change", BAD + [
    dict(acc=0), dict(acc_out=0), dict(acc_stride=63), dict(decay=-0.5), dict(decay=math.nan), dict(decay=math.inf), dict(seen=0),
    dict(acc=P + 2), dict(acc_out=P + 1), dict(pos=P + 2)])
def test_attn_decode_weights_refuses(change):
    refused(hs.HS_EINVAL, hs.hs_k_attn_decode_weights, **(WEIGHTS | change))


def test_attention_workspaces():
    """A byte less than the size given is refused, and the sizes grow with the call."""
    for fn, size, args in ((hs.hs_k_attn_decode_shared, hs.hs_k_attn_decode_shared_ws, ATTN),
                           (hs.hs_k_attn_decode_weights, hs.hs_k_attn_decode_weights_ws, WEIGHTS)):
        need = size(2, 32, 8, 128, 100, 64)
        assert need > 0
        refused(hs.HS_ERANGE, fn, **(args | dict(ws_bytes=need - 1)))
        assert size(64, 40, 40, 128, 100000, 100000) > 64 * 40 * 128 * 4
        for bad in ((0, 32, 8, 128, 1, 1), (2, 32, 8, 96, 1, 1), (2, 33, 8, 128, 1, 1), (2, 32, 8, 128, -1, 1), (2, 32, 8, 128, 1, -1)):
            refused(hs.HS_EINVAL, size, *bad)
    assert hs.hs_k_attn_decode_weights_ws(2, 32, 8, 128, 0, 64) > hs.hs_k_attn_decode_shared_ws(2, 32, 8, 128, 0, 64)


EVICT = dict(pool=P, pool_blocks=9, block_table=P, ctx=P, seen=P, acc=P, pos=2 * P, stride=64, acc_out=3 * P, pos_out=4 * P, out_stride=32,
             ctx_out=5 * P, keep=32, sinks=4, recent=8, B=2, n_kv_heads=8, head_dim=128, max_blocks=4, max_ctx=64, ws=P, ws_bytes=1 << 40)


@pytest.mark.parametrize("change", [
    dict(pool=0), dict(pool_blocks=0), dict(block_table=0), dict(ctx=0), dict(seen=0), dict(acc=0), dict(pos=0), dict(acc_out=0),
    dict(pos_out=0), dict(ctx_out=0), dict(ctx_out=P), dict(keep=0), dict(sinks=-1), dict(recent=-1), dict(B=0), dict(B=65536),
    dict(n_kv_heads=0), dict(head_dim=32), dict(max_blocks=3), dict(max_ctx=0), dict(max_ctx=65), dict(stride=63), dict(out_stride=31),
    dict(acc_out=P), dict(pos_out=2 * P), dict(pool=P + 2), dict(acc=P + 2), dict(ctx_out=P + 2), dict(ws=P + 4), dict(ws=0)])
def test_kv_evict_refuses(change):
    refused(hs.HS_EINVAL, hs.hs_k_kv_evict, **(EVICT | change))


def test_evict_workspace():
    need = hs.hs_k_kv_evict_ws(2, 8, 32, 64)
    assert need > 0
    refused(hs.HS_ERANGE, hs.hs_k_kv_evict, **(EVICT | dict(ws_bytes=need - 1)))
    refused(hs.HS_EINVAL, hs.hs_k_kv_evict_ws, 2, 8, 0, 64)
    refused(hs.HS_EINVAL, hs.hs_k_kv_evict_ws, 2, 8, 4, 0)


def test_evictions_of_more_than_2_25_moves_are_refused():
    """A row's moves are counted in 16-byte chunks, 32 of a token of 128 elements, in 32 bits: 2^26 of them
    would overflow. Few moves of a long row, or of one that keeps nearly all, are as before."""
    many = dict(max_blocks=1 << 26, stride=1 << 30, out_stride=1 << 30)
    for keep, max_ctx in ((1 << 26, 1 << 27), (1 << 27, 1 << 28), ((1 << 25) + 1, (1 << 26) + 2), (1 << 29, 1 << 30)):
        refused(hs.HS_EINVAL, hs.hs_k_kv_evict_ws, 1, 1, keep, max_ctx)
        refused(hs.HS_EINVAL, hs.hs_k_kv_evict, **(EVICT | many | dict(B=1, n_kv_heads=1, keep=keep, max_ctx=max_ctx)))
    for keep, max_ctx in ((1 << 25, 1 << 26), (1 << 25, 1 << 30), ((1 << 30) - (1 << 25), 1 << 30), (2048, 1 << 30)):
        moves = min(keep, max_ctx - keep)
        assert hs.hs_k_kv_evict_ws(1, 1, keep, max_ctx) == 4 * (2 * moves + 1)


def test_sizes_that_no_launch_takes_are_refused_with_their_workspace():
    """What a call refuses for its size has no workspace size, and what has one is not refused for its size."""
    refusing = 0
    for B in (1, 64, 1024, 65535):
        for nh, nkv in ((1, 1), (32, 8), (128, 128), (65536, 4096)):
            for prefix, own in ((0, 1 << 20), (1 << 20, 300), (1 << 30, 1 << 30), (300, 5), (0, 1 << 30)):
                for fn, size, args in ((hs.hs_k_attn_decode_shared, hs.hs_k_attn_decode_shared_ws, ATTN),
                                       (hs.hs_k_attn_decode_weights, hs.hs_k_attn_decode_weights_ws, WEIGHTS | dict(acc_stride=1 << 30))):
                    call = args | dict(B=B, n_heads=nh, n_kv_heads=nkv, ldq=nh * 128, ldo=nh * 128, prefix_len=prefix, max_ctx=own,
                                       max_blocks=1 << 26, ws_bytes=0)
                    try:
                        need = size(B, nh, nkv, 128, prefix, own)
                    except hs.HSError as e:
                        assert e.code == hs.HS_EINVAL
                        refused(hs.HS_EINVAL, fn, **(call | dict(ws_bytes=(1 << 64) - 1)))
                        refusing += 1
                    else:
                        assert need > 0
                        refused(hs.HS_ERANGE, fn, **call)
    assert 20 < refusing < 140
    size = hs.hs_k_attn_decode_shared_ws(64, 32, 8, 128, 0, 1 << 20)  # 2^22 workgroups: within a launch
    assert size > 0
    refused(hs.HS_EINVAL, hs.hs_k_attn_decode_shared_ws, 64, 32, 16, 128, 0, 1 << 20)  # 2^23


# arrays that lie apart, for the calls below: accepted ones end at the launch, which has no device here
APART_ATTN = WEIGHTS | dict(q=P, out=2 * P, pool=3 * P, prefix=4 * P, block_table=5 * P, ctx=6 * P, acc=7 * P, acc_out=8 * P, pos=9 * P, seen=10 * P,
                            ws=16 * P, ws_bytes=1 << 30)
APART_EVICT = EVICT | dict(pool=20 * P, block_table=6 * P, ctx=7 * P, seen=8 * P, ws=16 * P, ws_bytes=1 << 30)


@pytest.mark.parametrize("change", [
    dict(out=P), dict(out=P + 4096), dict(acc_out=7 * P + 4), dict(acc_out=7 * P - 252), dict(acc_out=9 * P), dict(pos=7 * P), dict(seen=9 * P + 8),
    dict(ctx=2 * P + 16), dict(ws=7 * P), dict(ws=P), dict(block_table=8 * P + 4), dict(prefix=2 * P)])
def test_attention_arrays_that_overlap_are_refused(change):
    refused(hs.HS_EINVAL, hs.hs_k_attn_decode_weights, **(APART_ATTN | change))


@pytest.mark.parametrize("change", [dict(out=P), dict(out=P + 8192 - 16), dict(ctx=2 * P), dict(ws=5 * P), dict(block_table=2 * P + 4)])
def test_shared_attention_arrays_that_overlap_are_refused(change):
    a = {k: v for k, v in APART_ATTN.items() if k in ATTN}
    refused(hs.HS_EINVAL, hs.hs_k_attn_decode_shared, **(a | change))


@pytest.mark.parametrize("change", [
    dict(acc_out=P + 4, out_stride=64), dict(acc_out=P - 4, out_stride=64), dict(acc_out=2 * P, out_stride=64), dict(pos_out=P, out_stride=64),
    dict(acc_out=4 * P + 64), dict(ctx_out=8 * P), dict(ctx_out=7 * P + 4), dict(ctx_out=P), dict(ctx_out=16 * P), dict(ws=P), dict(ws=6 * P),
    dict(acc_out=6 * P), dict(pos_out=2 * P + 256, out_stride=64)])
def test_evictions_whose_arrays_overlap_are_refused(change):
    refused(hs.HS_EINVAL, hs.hs_k_kv_evict, **(APART_EVICT | change))


@pytest.mark.parametrize("change", [
    dict(k_out=16 * P, ldk=1024), dict(k_out=16 * P + 8192 - 16, ldk=4096), dict(pos=16 * P + 64), dict(slot=16 * P), dict(q_out=P + 12288, ldq=48 * 128)])
def test_rope_kv_outputs_that_overlap_are_refused(change):
    a = dict(qkv=P, ldqkv=48 * 128, pos=2 * P, slot=3 * P, cos_t=4 * P, sin_t=5 * P, max_pos=64, rot_dim=128, layout="half", q_out=16 * P, ldq=32 * 128,
             k_out=0, ldk=1024, pool=32 * P, pool_blocks=4, T=3, n_heads=32, n_kv_heads=8, head_dim=128) | change
    refused(hs.HS_EINVAL, hs.hs_k_rope_kv, **a)


def accepted(fn, **kw):
    """Whether a call passes the checks: where there is no device, it then fails at the launch."""
    with pytest.raises(hs.HSError) as e:
        fn(**kw)
    assert e.value.code in (hs.HS_EINVAL, hs.HS_EHIP), e.value
    return e.value.code == hs.HS_EHIP


def without_device(f):
    import torch
    return pytest.mark.skipif(torch.cuda.is_available(), reason="would launch on memory that is not there")(f)


@without_device
def test_rows_are_refused_where_they_share_a_byte_and_only_there():
    """Against the sets of bytes, for arrays in the gaps of another's rows: two strides alike, or one row."""
    for B, nkv, most, stride in ((2, 2, 64, 150), (1, 1, 64, 64), (3, 1, 64, 70), (1, 5, 64, 200)):
        base = APART_ATTN | dict(B=B, n_heads=4 * nkv, n_kv_heads=nkv, max_ctx=most, acc_stride=stride)
        rows = B * nkv
        mine = {7 * P + 4 * (r * stride + t) for r in range(rows) for t in range(most)}
        for off in list(range(-2 * stride, 2 * stride, 7)) + [most, -most, most - 1, stride - most, stride - most + 1, rows * stride, -rows * stride]:
            at = 7 * P + 4 * off
            theirs = {at + 4 * (r * stride + t) for r in range(rows) for t in range(most)}
            assert accepted(hs.hs_k_attn_decode_weights, **(base | dict(acc_out=at))) == (off == 0 or not mine & theirs), (B, nkv, stride, off)
    for T, ld in ((3, 48 * 128 + 4096 + 64), (1, 48 * 128), (5, 48 * 128 + 1024)):
        base = dict(qkv=P, ldqkv=ld, pos=2 * P, slot=3 * P, cos_t=4 * P, sin_t=5 * P, max_pos=64, rot_dim=128, layout="half", q_out=16 * P, ldq=ld,
                    k_out=0, ldk=ld, pool=32 * P, pool_blocks=4, T=T, n_heads=32, n_kv_heads=8, head_dim=128)
        unit = lambda at, n: {at // 16 + r * ld // 8 + t for r in range(T) for t in range(n // 8)}  # noqa: E731
        whole, keys = unit(P, 48 * 128), unit(P + 8192, 1024)
        for off in [0, 8, 4096, 5 * 1024, 6 * 1024, 6 * 1024 + 8, 48 * 128 + 64, -4096, -4096 - 8, ld * T, ld * (T - 1) + 48 * 128]:
            got = accepted(hs.hs_k_rope_kv, **(base | dict(q_out=P + 2 * off)))
            assert got == (off == 0 or not unit(P + 2 * off, 4096) & whole), (T, ld, off)
            got = accepted(hs.hs_k_rope_kv, **(base | dict(k_out=P + 2 * off)))
            assert got == (off == 4096 or not unit(P + 2 * off, 1024) & whole), (T, ld, off)
        assert keys <= whole


@pytest.mark.parametrize("scaling", [
    hs.rope_scaling("linear", factor=1e-320), hs.rope_scaling("bands", factor=1e-310, original_ctx=10), hs.rope_scaling("linear", factor=2.0, magnitude=1e39),
    hs.hs_rope_scaling(0, 0, 0.0, 0.0, 0.0, 1e300)])
def test_scalings_whose_numbers_overflow_are_refused(scaling):
    """Frequencies above float64 have no fraction of a turn, a magnitude above float32 makes NaN of a zero."""
    refused(hs.HS_EINVAL, hs.hs_k_rope_tables, P, P, 64, 64, 10000.0, scaling)


def test_the_forms_meant_by_the_long_attention_tests_are_taken():
    """Each of them, if the rule that cuts a call changes: 2 to 16 steps of a prefix split, 8 to 32 blocks of an own one."""
    from tests.test_gpu_cache_ops_forms import LONG, cut, splits
    for lens, prefix, nh, nkv, d, prefix_tokens, own_blocks in LONG:
        assert splits(hs, len(lens), nh, nkv, d, prefix, max(lens)) == cut(prefix, max(lens), prefix_tokens, own_blocks)
    assert {x[5] for x in LONG} == {128, 192, 320, 704, 1024} and {x[6] for x in LONG} == {8, 16, 24, 32}
