"""The variant of cache_read for large outputs stores all of them past the caches: the hint is on
every store of the compiled kernels (a compiler may drop it, with no other trace than the time)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_17154_amd import build as b


@pytest.mark.skipif(not shutil.which(b.HIPCC), reason="no hipcc")
def test_every_store_of_the_streamed_reads_carries_the_hint(tmp_path):
    asm = tmp_path / "cache.s"
    subprocess.run([b.HIPCC] + b.FLAGS + ["--cuda-device-only", "-S", os.path.join(b.CSRC, "cache.hip"), "-o", str(asm)], check=True,
                   capture_output=True)
    seen = {}
    for part in re.split(r"\n(?=_ZN8ordermoe\S+:)", asm.read_text())[1:]:
        name = re.match(r"\S*cache_read_kernelI(\S+?)Li(\d+)ELi(\d)ELb(\d)E", part)
        if name:
            stores = re.findall(r"\s(?:global|flat|buffer)_store_\S+.*", part)
            assert stores, name.group(0)
            seen[name.groups()] = [bool(re.search(r"\bnt\b", s)) for s in stores]
    assert len(seen) == 2 * 3 * 2 * 2                           # types, head sizes, formats, both variants
    for (_, _, _, streamed), hints in seen.items():
        assert all(hints) if streamed == "1" else not any(hints)
