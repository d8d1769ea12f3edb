"""What the lanes of a wave exchange through LDS is ordered in the source, not by what the compiler happens to make of it
(no GPU): in the optimised intermediate code of the products whose waves turn their lines into fragments in LDS, a fence
stands between the stores and the reading, and between that and the next stores."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

ACCESS = re.compile(r"\b(store|load) (?:<4 x i32>|<4 x float>|i128).*addrspace\(3\)")


def unordered(lines):
    """LDS accesses of 16 bytes that follow one of the other kind with no fence between."""
    last, found = None, []
    for line in lines:
        if re.search(r"\bfence\b", line):
            last = None
            continue
        m = ACCESS.search(line)
        if m:
            if last not in (None, m.group(1)):
                found.append(line.strip())
            last = m.group(1)
    return found


def test_scanner_sees_the_pattern():
    put, get = "store <4 x i32> %1, ptr addrspace(3) %2, align 16", "%3 = load <4 x i32>, ptr addrspace(3) %4, align 16"
    fence = 'fence syncscope("wavefront") acq_rel, !mmra !24'
    assert unordered([put, get]) and unordered([put, fence, get, put])
    assert not unordered([put, put, fence, get, get, fence, put])


@pytest.fixture(scope="module")
def kernels():
    subprocess.run(["make", "-s", "-C", ROOT, "ir"], check=True)
    found, name = {}, None
    for line in open(os.path.join(ROOT, "_build", "fp8-gfx950.ll")):
        m = re.match(r"define .*@(_ZN\w+)\(", line)
        if m:
            name = m.group(1)
            found[name] = []
        elif line.startswith("}"):
            name = None
        elif name:
            found[name].append(line)
    return found


@pytest.mark.parametrize("kind", ["shared_tile_kernel", "few_rows_kernel"])
def test_lanes_exchange_behind_fences(kernels, kind):
    of_kind = {name: lines for name, lines in kernels.items() if kind in name}
    assert len(of_kind) >= 4
    for name, lines in of_kind.items():
        assert sum(bool(ACCESS.search(line)) for line in lines) >= 4, name
        assert not unordered(lines), (name, unordered(lines)[:3])
