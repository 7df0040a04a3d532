"""The gfx950 instructions of the cache operators: waits that a result that happens to be right would not show."""
from tests.test_device_code import kernels, pytestmark  # noqa: F401


def test_no_lds_read_passes_a_barrier(kernels):  # noqa: F811
    """The prefix's ring and the waves' buffers are refilled behind a barrier: every LDS read before it is
    complete there (lgkmcnt 0), not merely issued; and a copy into LDS is waited for (vmcnt) before the
    barrier that gives it to the other waves."""
    rings = 0
    for name, ins in kernels.items():
        if "cache_attn" not in name and "kv_evict" not in name:
            continue
        read = False
        copied = False  # since the last wait for vector memory
        for x in ins:
            if x.startswith("ds_read"):
                read = True
            elif x.startswith("s_waitcnt"):
                if "lgkmcnt(0)" in x:
                    read = False
                if "vmcnt" in x:
                    copied = False
            elif x.startswith("buffer_load") and x.endswith("lds"):
                copied = True
            elif x.startswith("s_barrier"):
                assert not read, name
                assert not copied, name
        rings += any(x.startswith("buffer_load") and x.endswith("lds") for x in ins)
    assert rings == 2  # of 64 and of 128 columns


def test_no_kernel_spills(kernels):  # noqa: F811
    """No scratch memory in any of them."""
    seen = 0
    for name, ins in kernels.items():
        if any(k in name for k in ("cache_attn", "kv_evict", "rope_kv_at", "rope_tables")):
            seen += 1
            assert not any(x.startswith(("scratch_", "buffer_store_dword off, off", "buffer_load_dword off")) for x in ins), name
    assert seen >= 15
