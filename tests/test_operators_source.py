"""Rules of the operators' kernels that are read off their source (no GPU)."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2310_14423_amd", "csrc")


def test_words_of_one_lane_are_read_behind_a_barrier():
    """A word in LDS that lane 0 writes for all (`if (tid == 0) se.x = ...`) is read by the others behind a barrier that no condition
    takes out, however few wavefronts a workgroup has."""
    lines = open(os.path.join(CSRC, "token_logprobs.hip")).read().splitlines()
    seen = 0
    for i, line in enumerate(lines):
        m = re.search(r"if \(tid == 0\) (se\.\w+) = (.*);", line)
        if not m:
            continue
        names = [m.group(1)] + re.findall(r"se\.\w+", m.group(2))
        for name in names:
            barrier = False
            for later in lines[i + 1:]:
                if later.strip().startswith("__syncthreads();"):
                    barrier = True
                if re.search(re.escape(name) + r"\b", later):
                    assert barrier, (i + 1, name)
                    seen += 1
                    break
    assert seen >= 3
