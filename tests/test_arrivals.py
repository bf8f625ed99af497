"""Kernels whose workgroups leave partial results for the one that arrives last: from the compiler's own listing of every instantiation, a
wave has waited for its chip-coherent stores where its workgroup counts itself in (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2504_08242_amd import build as jbuild


def listing(tmp_path, source):
    """{kernel: its instructions and labels}"""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is not installed")
    out = tmp_path / "listing.s"
    subprocess.run([hipcc, *jbuild.HIPCC_FLAGS, "-S", "--offload-device-only", os.path.join(jbuild.CSRC, source), "-o", out],
                   check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    kernels, name = {}, None
    for line in out.read_text().splitlines():
        line = line.split(";")[0].strip()
        if m := re.match(r"(_ZN\S+):$", line):
            kernels[name := m.group(1)] = []
        elif re.match(r"\.Lfunc_end\d+:$", line):
            name = None
        elif name and line and (not line.startswith(".") or line.endswith(":")):
            kernels[name].append(line)
    return kernels


def arrivals(lines):
    """(line, this wave's coherent stores may be in flight, those of another wave may) of every arrival.  Every wave runs the same code, so
    what another wave has in flight is what this one may have had at the barrier in front of the arrival."""
    labels = {l[:-1]: i for i, l in enumerate(lines) if l.endswith(":")}
    state, todo, found = {0: (False, False)}, [0], {}
    while todo:
        i = todo.pop()
        mine, others = state[i]
        op, *args = lines[i].split()
        if re.match(r"(global|buffer|flat)_store", op) and "sc1" in args:
            mine = True
        elif op == "s_waitcnt" and re.search(r"vmcnt\(0\)", lines[i]):
            mine = False
        elif op == "s_barrier":
            others = mine
        elif re.match(r"(global|buffer|flat)_atomic_add$", op):
            found[i] = (i, mine, others)
        after = []
        if op.startswith(("s_branch", "s_cbranch")):
            after.append(labels[args[0]])
        if op not in ("s_branch", "s_endpgm") and i + 1 < len(lines):
            after.append(i + 1)
        for j in after:
            before = state.get(j)
            new = (mine, others) if before is None else (mine or before[0], others or before[1])
            if new != before:
                state[j] = new
                todo.append(j)
    return list(found.values())


@pytest.mark.parametrize("source,kernel,at_least", [("bf16_attention.hip", "attention", 6), ("paged_attention.hip", "attention_", 7),
                                                    ("paged_verify.hip", "verify", 4)])
def test_a_workgroup_arrives_behind_its_stores(tmp_path, source, kernel, at_least):
    seen = 0
    for name, lines in listing(tmp_path, source).items():
        stores = [l for l in lines if re.match(r"(global|buffer|flat)_store.* sc1$", l)]
        counted = arrivals(lines)
        if not counted:
            assert not stores, name   # nothing is left for others without an arrival
            continue
        seen += 1
        assert kernel in name and stores, name
        for at, mine, others in counted:
            assert not mine and not others, (name, lines[at - 3:at + 1])
    assert seen >= at_least


def test_the_listing_is_read_right():
    """Planted in small listings: no wait, a wait behind the barrier, a wait on one of two ways only."""
    store, wait, barrier, arrive = "global_store_dwordx2 v4, v[2:3], s[2:3] sc1", "s_waitcnt vmcnt(0)", "s_barrier", "global_atomic_add v3, v4, v3, s[4:5] sc0"
    result = lambda *lines: [x[1:] for x in arrivals([*lines, "s_endpgm"])]  # noqa: E731
    assert result(store, wait, barrier, arrive) == [(False, False)]
    assert result(store, barrier, arrive) == [(True, True)]
    assert result(store, barrier, wait, arrive) == [(False, True)]
    assert result(store, "s_waitcnt vmcnt(1)", barrier, arrive) == [(True, True)]
    assert result(store, "s_cbranch_vccnz .L1", wait, ".L1:", barrier, arrive) == [(True, True)]
    assert result(barrier, store, wait, arrive) == [(False, False)]
