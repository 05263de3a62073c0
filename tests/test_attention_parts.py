"""The scratch that a context has for parts of items is one for the attention over both
kinds of cache: a kernel whose parts would not fit does not compile."""
import os
import shutil
import subprocess

import pytest

from paper_2607_13500_amd import build

WAVES = ("constexpr int kManyWaves = DH == 256 ? 4 : 8;", "constexpr int kManyWaves = 16;")
CHANGES = {"as_they_are": None,
           "more_wavefronts": ("tr_attend.hip", *WAVES), "more_wavefronts_8": ("tr_attend8.hip", *WAVES),
           "more_workgroups": ("tr_attend.hip", "constexpr int kFewPerCu = DH == 64 ? 3 : DH == 128 ? 2 : 1;", "constexpr int kFewPerCu = 32;"),
           "more_tiles_8": ("tr_attend8.hip", "few<DH, 4, RT>(a, s)", "few<DH, 8, RT>(a, s)"),
           "less_scratch": ("tr_attend_work.h", "DH == 256 ? 128 : 256>;", "DH == 256 ? 64 : 128>;")}


@pytest.mark.parametrize("change", CHANGES)
def test_parts_fit_the_scratch(change, tmp_path):
    shutil.copytree(build.CSRC, tmp_path / "csrc")
    sources = ["tr_attend.hip", "tr_attend8.hip"]
    if CHANGES[change]:
        name, old, new = CHANGES[change]
        text = (tmp_path / "csrc" / name).read_text()
        assert text.count(old) == 1
        (tmp_path / "csrc" / name).write_text(text.replace(old, new))
        sources = [name] if name in sources else sources
    for source in sources:
        r = subprocess.run([build.hipcc(), "--offload-arch=" + build.ARCH, "--offload-host-only", "-std=c++17", "-fsyntax-only", "-I", build.INCLUDE,
                            "-I", str(tmp_path / "csrc"), str(tmp_path / "csrc" / source)], capture_output=True, text=True)
        if CHANGES[change]:
            assert r.returncode != 0 and "the parts' scratch is too small" in r.stderr, (source, r.stderr)
        else:
            assert r.returncode == 0, r.stderr
