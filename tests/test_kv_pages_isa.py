"""Checks on the generated gfx950 code of the kernels for shared pages and prefixes (no GPU needed: hipcc cross-compiles)."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2604_03950_amd import build as B


@pytest.fixture(scope="module", params=["dma_cache_pages.hip", "dma_cache_shared.hip"])
def source(request):
    flags = [f for f in B.HIPCC_FLAGS if f != "-fPIC"]
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "x.s")
        subprocess.run(["hipcc"] + flags + ["-S", "--cuda-device-only", "-o", out, os.path.join(B.CSRC, request.param)], check=True,
                       stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
        return request.param, open(out).read()


def test_registers(source):
    """No packed binary32 arithmetic; nothing spilled to memory but, outside the loops over the keys, by the kernel for shared prefixes where rows
    lie in tiles of 32 (D = 128); two workgroups per CU."""
    name, text = source
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    seen = 0
    for block in re.split(r"(?=- \.agpr_count)", text)[1:]:
        kernel = re.search(r"\.name:\s+(_ZN3dma\S+)", block).group(1)
        seen += 1
        count = {f: int(re.search(rf"\.{f}:\s+(\d+)", block).group(1)) for f in ("vgpr_count", "vgpr_spill_count", "group_segment_fixed_size")}
        args = [int(n) for n in re.findall(r"L[ib](\d+)E", kernel)]
        rows32 = "cache_shared_kernel" in kernel and args[0] == 128 and args[2] == 2                # <D, E5M2, tiles of 16 rows, ...>
        assert count["vgpr_spill_count"] <= (36 if rows32 else 0), (kernel, count)
        assert count["vgpr_count"] <= 256 and count["group_segment_fixed_size"] <= 80 * 1024, (kernel, count)
    assert seen == {"dma_cache_pages.hip": 5, "dma_cache_shared.hip": 24}[name]


def test_loops_over_keys(source):
    """No block with the matrix instructions of a step goes to scratch memory: a reload waits for the codes in flight.  (One reload at most where
    32 rows of D = 128 are a tile of an own part: what a group's sequences share, which most of the time goes to, has none.)"""
    name, text = source
    hot = 0
    for m in re.finditer(r"^(_ZN3dma19cache_shared_kernel\S+):", text, flags=re.M):
        body = text[m.end():text.index(".section", m.end())]
        args = [int(n) for n in re.findall(r"L[ib](\d+)E", m.group(1))]
        for b in re.split(r"^\.LBB\w+:", body, flags=re.M):
            if len(re.findall(r"\bv_mfma_", b)) >= 8:
                hot += 1
                own32 = args[0] == 128 and args[2] == 2 and len(re.findall(r"\bv_mfma_", b)) == 32
                assert len(re.findall(r"\bscratch_", b)) <= (1 if own32 else 0), m.group(1)
    assert hot >= 4 * 16 or name == "dma_cache_pages.hip"
