"""Checks on the generated gfx950 code of the cache's kernels (no GPU needed: hipcc cross-compiles)."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2604_03950_amd import build as B


@pytest.mark.parametrize("source", ["dma_cache.hip", "dma_cache_attn.hip", "dma_cache_prompt.hip"])
def test_registers(source):
    """No packed binary32 arithmetic; nothing spilled to memory but, outside the loop over the keys, by the kernel for few rows where it has 32:
    a reload in the loop would wait for the codes requested meanwhile.  Two waves per SIMD at least."""
    flags = [f for f in B.HIPCC_FLAGS if f != "-fPIC"]
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "x.s")
        subprocess.run(["hipcc"] + flags + ["-S", "--cuda-device-only", "-o", out, os.path.join(B.CSRC, source)], check=True,
                       stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
        text = open(out).read()
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    seen = 0
    for block in re.split(r"(?=- \.agpr_count)", text)[1:]:
        name = re.search(r"\.name:\s+(_ZN3dma\S+)", block)
        if not name:
            continue
        seen += 1
        count = {f: int(re.search(rf"\.{f}:\s+(\d+)", block).group(1)) for f in ("vgpr_count", "vgpr_spill_count", "group_segment_fixed_size")}
        args = [int(n) for n in re.findall(r"L[ib](\d+)E", name.group(1))]
        rows32 = "cache_attn_kernel" in name.group(1) and args[0] == 128 and args[2] == 2          # <D, E5M2, tiles of 16 rows, ...>
        assert count["vgpr_spill_count"] <= (12 if rows32 else 0), (name.group(1), count)
        assert count["vgpr_count"] <= 256 and count["group_segment_fixed_size"] <= 160 * 1024, (name.group(1), count)
    assert seen == {"dma_cache.hip": 8, "dma_cache_attn.hip": 52, "dma_cache_prompt.hip": 10}[source]


@pytest.mark.parametrize("uni", [0, 1])
@pytest.mark.parametrize("tiles", [1, 2])
def test_codes_stay_in_flight(uni, tiles):
    """The loop over the keys of the kernel for few rows never waits for everything: each block of it with the matrix instructions of a
    step and the requests of the next waits by count, and reloads nothing from scratch memory."""
    flags = [f for f in B.HIPCC_FLAGS if f != "-fPIC"]
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "x.s")
        subprocess.run(["hipcc"] + flags + ["-S", "--cuda-device-only", "-o", out, os.path.join(B.CSRC, "dma_cache_attn.hip")], check=True,
                       stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
        text = open(out).read()
    for waves in (4, 8):
        start = text.index(f"_ZN3dma17cache_attn_kernelILi128ELb0ELi{tiles}ELi{waves}ELb0ELb{uni}EEEvNS_13CacheAttnArgsE:")
        body = text[start:text.index(".section", start)]
        hot = [b for b in re.split(r"^\.LBB\w+:", body, flags=re.M) if len(re.findall(r"\bv_mfma_", b)) >= 16 * tiles and "global_load_dwordx4" in b]
        assert len(hot) == 2, len(hot)
        for b in hot:
            assert "scratch_" not in b and not re.search(r"s_waitcnt vmcnt\(0\)", b)
