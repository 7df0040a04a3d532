"""The waits of the cache operators' gfx950 instructions along every path, loops included: how many
copies into LDS and how many LDS reads may be on their way at a barrier."""
import re
import struct
import subprocess

import pytest

from tests.test_device_code import LIB, MAGIC, OBJDUMP, pytestmark  # noqa: F401

MOST = 64  # of a counter


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    """{kernel: [(address, instruction, address it may branch to or None), ...]} of the cache operators."""
    data, out = open(LIB, "rb").read(), {}
    d = tmp_path_factory.mktemp("flow")
    for n, m in enumerate(re.finditer(MAGIC, data)):
        at = m.start() + len(MAGIC)
        (count,) = struct.unpack_from("<Q", data, at)
        at += 8
        for _ in range(count):
            off, size, tl = struct.unpack_from("<QQQ", data, at)
            triple = data[at + 24:at + 24 + tl].decode()
            at += 24 + tl
            if "gfx950" not in triple or not size:
                continue
            path = d / f"{n}.co"
            path.write_bytes(data[m.start() + off:m.start() + off + size])
            text = subprocess.run([OBJDUMP, "-d", "-C", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
            name, base = None, 0
            for line in text.splitlines():
                h = re.match(r"^([0-9a-f]+) <(.*)>:$", line.strip())
                if h:
                    base, name = int(h.group(1), 16), h.group(2)
                elif name and "//" in line and ("cache_attn" in name or "kv_evict" in name):
                    code, note = line.split("//", 1)
                    a = int(re.match(r"\s*([0-9A-F]+):", note).group(1), 16)
                    to = re.search(r"\+0x([0-9a-f]+)>\s*$", note) if "branch" in code else None
                    if "branch" in code and not to:  # to the first instruction
                        assert note.rstrip().endswith(">"), line
                    out.setdefault(name, []).append((a, code.strip(), None if "branch" not in code else base + (int(to.group(1), 16) if to else 0)))
    assert len(out) >= 15
    return out


def in_flight(ins, issues, counter):
    """{index of a barrier: the most operations issued (regex) that may not have completed there}, by
    the waits for `counter` along all paths. Operations of one counter complete in order, others of it
    count as none (which can only make the result larger)."""
    index = {a: i for i, (a, _, _) in enumerate(ins)}
    state, work = {0: 0}, [0]
    while work:
        i = work.pop()
        n = state[i]
        x, to = ins[i][1], ins[i][2]
        if re.match(issues, x):
            n = min(n + 1, MOST)
        elif x.startswith("s_waitcnt"):
            w = re.search(counter + r"\((\d+)\)", x)
            if w:
                n = min(n, int(w.group(1)))
        after = [] if x.startswith(("s_endpgm", "s_branch", "s_setpc")) else [i + 1]
        if to is not None:
            after.append(index[to])
        for j in after:
            if j < len(ins) and state.get(j, -1) < n:
                state[j] = n
                work.append(j)
    return {i: n for i, n in state.items() if ins[i][1].startswith("s_barrier")}


COPY, READ = r"buffer_load\w* .*\blds$", r"ds_read"


def ring_columns(name):
    m = re.search(r"cache_attn_shared_kernel<(\d+)>", name)
    return int(m.group(1)) if m else None


def too_many(name, ins):
    """What passes a barrier of a kernel: copies of the steps after the next of the prefix's ring (two stages
    of 128 columns: none; four of 64: two steps of 2 + 2 copies a wave) may, in its loop, and nothing else."""
    d = ring_columns(name)
    may = {None: 0, 128: 0, 64: 8}[d]
    copies = sorted(in_flight(ins, COPY, "vmcnt").values())
    return any(copies[:-1]) or any(n > may for n in copies) or any(in_flight(ins, READ, "lgkmcnt").values())


def test_what_is_on_its_way_at_a_barrier(listings):
    rings = 0
    for name, ins in listings.items():
        assert not too_many(name, ins), name
        rings += any(re.match(COPY, x) for _, x, _ in ins)
    assert rings == 2


def test_a_wait_that_leaves_more_is_found(listings):
    """The same listings with one wait changed: each ring's loop leaves one copy more, or waits for none."""
    for name, ins in listings.items():
        d = ring_columns(name)
        if d is None:
            continue
        loop = {128: "s_waitcnt vmcnt(0) lgkmcnt(0)", 64: "s_waitcnt vmcnt(8) lgkmcnt(0)"}[d]
        at = next(i for i, (_, x, _) in enumerate(ins) if x == loop)
        assert any(x.startswith("s_barrier") for _, x, _ in ins[at + 1:at + 6])
        for other in (f"s_waitcnt vmcnt({ {128: 1, 64: 9}[d] }) lgkmcnt(0)", "s_waitcnt lgkmcnt(0)", "s_waitcnt vmcnt(63) lgkmcnt(0)"):
            changed = list(ins)
            changed[at] = (ins[at][0], other, None)
            assert too_many(name, changed), (name, other)
