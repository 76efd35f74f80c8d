"""The attention of token chunks: the last workgroup's reads of the others' partial results stand behind the ticket it drew, in the compiled
code too, and no register of its kernels spills."""
import os
import re
import subprocess

import pytest

TICKET = re.compile(r'atomicrmw add ptr.* syncscope\("agent(?:-one-as)?"\) monotonic')
ORDERS = re.compile(r"\bfence\b|~\{memory\}")
READS = re.compile(r"\bload atomic\b|@llvm\.amdgcn\.raw\.ptr\.buffer\.load")


SOURCES = ["chunk_attn.hip", "chunk_rows.hip"]


@pytest.mark.parametrize("source", SOURCES)
def test_reads_behind_the_ticket(tmp_path, source):
    from paper_2509_11815_amd import build
    out = str(tmp_path / "k.ll")
    subprocess.run([build._hipcc(), *build.HIPCC_FLAGS, "--cuda-device-only", "-S", "-emit-llvm", "-o", out, os.path.join(build.CSRC, source)], check=True, capture_output=True)
    with open(out) as f:
        lines = f.read().split("\n")
    found = 0
    for i, line in enumerate(lines):
        if not TICKET.search(line):
            continue
        found += 1
        for later in lines[i + 1:]:
            if ORDERS.search(later):
                break
            assert later != "}", (i, line)
            assert not READS.search(later), (line, later)
    assert found >= 8


@pytest.mark.parametrize("source", SOURCES)
def test_nothing_spills(source):
    from paper_2509_11815_amd import build
    usage = build.kernel_resource_usage(source)
    kernels = {k: v for k, v in usage.items() if "_kernel" in k}
    assert len(kernels) >= 8, sorted(usage)
    for name, u in kernels.items():
        assert u["scratch"] == 0 and u["lds"] <= 160 * 1024, (name, u)
