"""Calls of more rows or sets than a launch has workgroups: the grid no longer grows with
the call, and its kernel goes on by the grid's size, which it then asks for among its
arguments (as the code object of librac.so says)."""
from __future__ import annotations

import os
import re
import subprocess

import pytest

import paper_2608_04991_amd as rac
from tests.test_kernel_resources import LLVM, MAGIC
from tests.test_more_dispatch import record  # noqa: F401  (a fixture)


@pytest.fixture(scope="module")
def asks(tmp_path_factory):
    """Kernels that ask for the grid's size."""
    tmp, out = str(tmp_path_factory.mktemp("code")), set()
    run = lambda *a: subprocess.run(a, check=True, capture_output=True, text=True).stdout
    run(f"{LLVM}/llvm-objcopy", "--dump-section", f".hip_fatbin={tmp}/fat", rac.library_path(), f"{tmp}/rest")
    data = open(f"{tmp}/fat", "rb").read()
    starts = [m.start() for m in re.finditer(MAGIC, data)]
    for i, (a, b) in enumerate(zip(starts, starts[1:] + [len(data)])):
        part = f"{tmp}/{i}"
        open(part, "wb").write(data[a:b])
        run(f"{LLVM}/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
            f"--input={part}", f"--output={part}.elf")
        for note in run(f"{LLVM}/llvm-readelf", "--notes", part + ".elf").split("  - .agpr_count")[1:]:
            if "hidden_block_count_x" in note:
                out.add(re.search(r"^    \.name:\s+(\S+)", note, re.M).group(1))
    plain = subprocess.run(["c++filt"], input="\n".join(sorted(out)), text=True, capture_output=True, check=True).stdout
    return {re.sub(r"\(anonymous namespace\)::|^void ", "", p).split("(")[0] for p in plain.splitlines()}


def of(rows, sets):
    """The same calls for some rows and some sets."""
    calls = [("rotary", [rows, 1, 0, 16, 16, 0], None), ("rotary", [rows, 64, 8, 256, 256, 2], None)]
    for type in (0, 1, 2):
        for vocab, top in ((1000, 0), (1000, 5), (40000, 0), (40000, 5), (2400001, 5)):
            calls.append(("logprobs", [rows, vocab, rows, top, type], [0, 1]))
            calls.append(("logprobs", [rows, vocab, 100, top, type], [1, 0]))
        calls.append(("backward", [rows, 40000, rows, 0, type], [1, 1]))
    heads = 1 << 10
    calls.append(("evict", [sets // heads, heads, 16, 8, 1 << 20, 2, 1], [sets, 0, 0]))
    calls.append(("append", [sets // heads, heads, 16, 8, 1 << 20, 2, 1], None))
    return calls


def test_a_grid_that_does_not_grow_is_of_a_kernel_that_goes_on(record, asks):  # noqa: F811
    some, more = of(1 << 22, 1 << 19), of(1 << 24, 1 << 20)
    logs = record(some + more)
    cut = set()
    for a, b in zip(logs[:len(some)], logs[len(some):]):
        assert [k for k, _, _ in a] == [k for k, _, _ in b]
        # (the eviction's one workgroup a call or a sequence, and a hundred scored tokens, are as many in both)
        cut |= {k for (k, x, _), (_, y, _) in zip(a, b) if x == y > 1 and k != "evict_demand_kernel"}
    assert {k.split("<")[0] for k in cut} >= {"rotary_kernel", "logprob_kernel", "logprob_join_kernel", "evict_pick_kernel"}
    assert cut - asks == set()
