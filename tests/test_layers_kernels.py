"""Of the kernels that are templates the library holds those that some call reaches (its symbols; no GPU)."""
import re
import shutil
import subprocess

import pytest

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.skipif(shutil.which("nm") is None, reason="needs nm")


def _kernels(name):
    """The template arguments of every kernel of that name in the library."""
    text = subprocess.run(["nm", qsr.lib_path()], check=True, capture_output=True, text=True, timeout=60).stdout
    return {m for m in re.findall(r"_ZN3qsr\d+%sI(\w+)EEEvNS_\w+Args?E\b" % name, text)}


def _norm_layouts():
    """(type, lanes, wavefronts, runs of 16 bytes to a lane) of every width: sixteen elements to a lane in bf16 from 513 on, eight in fp32 up to 8192."""
    seen = set()
    for name, E, unit in (("f", 4, 512), ("DF16b", 8, 1024)):
        for d in range(1, 16385):
            if d <= 512:
                seen.add((name, 16 if d <= 128 else 32 if d <= 256 else 64, 1, 0 if d < E else 8 // E))
                continue
            W = next((w for w in (1, 2, 4, 5, 8, 12 if E == 8 else 16) if d <= w * unit), 16)
            if E == 8 and 1536 < d <= 2048:
                W = 4
            narrow = (E == 8 and W == 4 and d <= 2048) or (E == 4 and d <= 8192)
            seen.add((name, 64, W, 8 // E if narrow else 16 // E))
    return seen


@pytest.mark.parametrize("kernel", ["layernorm_kernel", "layernorm_back_kernel"])
def test_layouts_of_the_norm(kernel):
    got = set()
    for args in _kernels(kernel):
        m = re.fullmatch(r"(f|DF16b)Li(\d+)ELi(\d+)ELi(\d+)ELb([01])", args)
        assert m, args
        got.add((m.group(1), int(m.group(2)), int(m.group(3)), int(m.group(4))))
    assert got == _norm_layouts()


def test_maps_of_the_recurrence():
    """Backward the maps are the same for both inputs."""
    got = _kernels("scan_maps_kernel")
    assert got == {"%sELb%dELb%d" % (t, comp, back) for t in ("fLi1", "DF16bLi1", "DF16bLi2") for comp, back in ((0, 0), (1, 0), (0, 1))}
