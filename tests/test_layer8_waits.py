"""As test_lds_waits, for the 8-bit layer's kernels; and the loads that go straight into LDS: a wavefront waits for its own
before the barrier behind which others read them."""
import os
import re
import subprocess

import pytest

from paper_2506_16235_amd import build as B
from test_lds_waits import _unfinished


@pytest.mark.parametrize("unit", B.LAYER8_UNITS)
def test_no_lds_write_in_flight_at_a_barrier(unit, tmp_path):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path / "k.s")
    flags = [f for f in B.HIP_FLAGS if f != "-fPIC"]
    subprocess.run([B.HIPCC, *flags, "-I", B.INCLUDE, "--cuda-device-only", "-S", os.path.join(B.LAYER8, unit + ".hip"), "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()
    assert text.count("s_barrier") >= 3
    assert _unfinished(text) == []
    assert not re.search(r"v_pk_(add|mul|fma)_f32", text)


# ---------------------------------------------------------------- loads that go straight into LDS

_MEMORY = ("global_", "buffer_", "flat_", "scratch_")


def _late_loads(text, ring_of):
    """(kernel, line of a barrier) where a wavefront may have more loads into LDS on their way than a ring of stages allows, over all paths;
    and how many barriers were looked at.  Of the loads of ring - 1 stages before the first barrier, ring - 2 stages' may be on their way
    there; at one behind a stage's requests as many; at one behind none (LDS is used for something else) none.  A wait for vmcnt(n) leaves
    the last n accesses to memory of any kind."""
    found, looked = set(), set()
    for m in re.finditer(r"^(_Z\w+):.*\n([\s\S]*?)^\.Lfunc_end", text, re.M):
        ring = ring_of(m.group(1))
        if ring is None:
            continue
        ins, label = [], {}
        for line in m.group(2).split("\n"):
            line = line.split(";")[0].strip()
            q = re.match(r"^(\.?\w+):$", line)
            if q:
                label[q.group(1)] = len(ins)
            elif line and not line.startswith("."):
                ins.append(line)
        # state: first barrier still to come, loads into LDS since the last one, and for each on its way how many accesses came after it
        seen, work = set(), [(0, (True, 0, ()))]
        while work:
            i, (first, issued, out) = work.pop()
            while (i, first, issued, out) not in seen:
                seen.add((i, first, issued, out))
                op = ins[i].split()[0]
                if op.startswith(_MEMORY):
                    out = tuple(n + 1 for n in out if n < 63)       # 64 may be on their way at most
                    if "_load_lds" in op:
                        out, issued = out + (0,), issued + 1
                elif op == "s_waitcnt":
                    w = re.search(r"vmcnt\((\d+)\)", ins[i])
                    if w:
                        out = tuple(n for n in out if n < int(w.group(1)))
                elif op == "s_barrier":
                    stage = issued // (ring - 1) if first else issued
                    looked.add((m.group(1), i))
                    if len(out) > stage * (ring - 2):
                        found.add((m.group(1), i))
                        out = ()
                    first, issued = False, 0
                if op == "s_endpgm":
                    break
                if op == "s_branch":
                    i = label[ins[i].split()[1]]
                    continue
                if op.startswith("s_cbranch"):
                    work.append((label[ins[i].split()[1]], (first, issued, out)))
                i += 1
    return found, looked


def test_follows_loads_into_lds():
    load = "\tglobal_load_lds_dwordx4 v1, s[0:1]\n"
    body = ("_Zk:\n" + load * 4 + "\tglobal_load_dword v2, v3, s[0:1]\n\ts_waitcnt vmcnt({0})\n\ts_barrier\n.LBB0:\n" + load * 2 +
            "\ts_waitcnt vmcnt({1})\n\ts_barrier\n\ts_cbranch_scc1 .LBB0\n\ts_waitcnt vmcnt({2})\n\ts_barrier\n\ts_endpgm\n.Lfunc_end0:\n")

    def late(*counts):
        return len(_late_loads(body.format(*counts), lambda name: 3)[0])
    assert late(2, 2, 0) == 0 and late(3, 2, 0) == 0        # the last access at the first barrier is none into LDS
    assert late(4, 2, 0) == 1 and late(2, 3, 0) == 1 and late(2, 2, 1) == 1 and late(63, 63, 63) == 3
    assert len(_late_loads(body.format(2, 2, 0), lambda name: 3)[1]) == 3


def test_loads_into_lds_are_there_before_the_barrier(tmp_path):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path / "k.s")
    flags = [f for f in B.HIP_FLAGS if f != "-fPIC"]
    subprocess.run([B.HIPCC, *flags, "-I", B.INCLUDE, "--cuda-device-only", "-S", os.path.join(B.LAYER8, "products.hip"), "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()

    def ring_of(kernel):
        if "k_product_large" in kernel:
            return 4
        m = re.search(r"k_productI\w+?Li\d+ELi(\d+)E", kernel)
        return int(m.group(1)) if m else None
    rings = [ring_of(k) for k in re.findall(r"^(_Z\w+):", text, re.M)]
    assert sum(r is not None for r in rings) == 12 and all(r for k, r in zip(re.findall(r"^(_Z\w+):", text, re.M), rings) if "few" not in k)
    for m in re.finditer(r"^(_Z\w+):.*\n([\s\S]*?)^\.Lfunc_end", text, re.M):
        assert ("_load_lds" in m.group(2)) == (ring_of(m.group(1)) is not None)
    late, looked = _late_loads(text, ring_of)
    assert late == set() and len(looked) >= 3 * 12
    # one request more on its way than allowed, and no wait at all, in the text that was read
    waits = re.compile(r"vmcnt\((\d+)\) lgkmcnt\(0\)(\n\ts_barrier)")
    more = waits.sub(lambda w: f"vmcnt({int(w.group(1)) + 1}) lgkmcnt(0){w.group(2)}", text)
    none = waits.sub(r"lgkmcnt(0)\2", text)
    assert len(waits.findall(text)) >= 3 * 12
    for worse in (more, none):
        assert {k for k, _ in _late_loads(worse, ring_of)[0]} == {k for k, _ in looked}
