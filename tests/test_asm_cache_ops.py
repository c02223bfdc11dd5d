"""Static checks of the generated assembly of the cache's operators (CPU only, needs hipcc)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2512_10411_amd import build

needs_hipcc = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="hipcc not available")


def assembly(tmp_path, src):
    out = tmp_path / "k.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([build.hipcc_path(), *flags, "--cuda-device-only", "-S", "-o", str(out), os.path.join(build.CSRC, src)], check=True,
                   stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    return open(out).read()


@needs_hipcc
def test_weighing_kernels_own_all_lds_and_wait_for_their_copies(tmp_path):
    """They address LDS with plain byte addresses from 0 and copy rows straight into it.  Behind the barrier of a stage the buffer of the
    stage before is copied into: a wave's copies have landed in front of it (vmcnt), and so have its reads (lgkmcnt)."""
    text = assembly(tmp_path, "swaa_key_weights.hip")
    sizes = re.findall(r"\.amdhsa_group_segment_fixed_size\s+(\d+)", text)
    spills = re.findall(r"\.amdhsa_private_segment_fixed_size\s+(\d+)", text)
    names = re.findall(r"\.amdhsa_kernel\s+(\S+)", text)
    assert len(names) == len(sizes) == len(spills) and sum("key_weights_kernel" in n for n in names) >= 16
    for name, size, spill in zip(names, sizes, spills):
        assert int(size) == 0 and int(spill) == 0, name
    lines = text.splitlines()
    starts = [i for i, ln in enumerate(lines) if re.match(r"_Z\S*key_weights(_listed)?_kernel\S*:", ln)]
    assert len(starts) >= 32
    for first in starts:
        body = []
        for ln in lines[first:next(i for i in range(first, len(lines)) if lines[i].startswith(".Lfunc_end"))]:
            ln = ln.split(";")[0].strip()
            if ln and not ln.startswith(".") and not ln.endswith(":"):
                body.append(ln)
        barriers = [i for i, ln in enumerate(body) if ln.startswith("s_barrier")]
        waited = [i for i in barriers if body[i - 1].startswith("s_waitcnt") and "vmcnt(0)" in body[i - 1] and "lgkmcnt(0)" in body[i - 1]]
        assert waited, lines[first]  # (the listed kernels have a second one, between two items)
        assert len(barriers) - len(waited) <= 1


@needs_hipcc
@pytest.mark.parametrize("src", ["swaa_key_weights.hip", "swaa_norm_rope.hip", "swaa_evict.hip"])
def test_no_packed_arithmetic_of_32_bits(tmp_path, src):
    assert not re.search(r"v_pk_(add|mul|fma)_f32", assembly(tmp_path, src))
