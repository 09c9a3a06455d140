"""Rules of the embedding's and the recurrence's kernels that are read off their source (no GPU)."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2310_14423_amd", "csrc")


def _kernel(source, name):
    """The text of a kernel, from its name to the brace that closes it."""
    start = source.index("void %s(" % name)
    return source[start:source.index("\n}\n", start)]


def test_sequences_without_steps_are_not_read():
    """x and gate of a sequence that has ended may lie where nothing is mapped: the kernel of single steps loads them under the condition that
    there is a step, and the others' rows are loaded by load_rows, row by row under `s < n`."""
    source = open(os.path.join(CSRC, "gated_scan.hip")).read()
    step = _kernel(source, "scan_step_kernel")
    loads = [m.start() for m in re.finditer(r"\*\(const Vec \*\)", step)]
    guard = re.search(r"if \(live\) \{(.*?)\n    \}", step, re.S)
    assert len(loads) == 2 and guard and all(guard.start(1) < at < guard.end(1) for at in loads)
    assert step.index("live = ") < guard.start()
    rows = source[source.index("void load_rows("):source.index("// A lane's place:")]
    assert rows.count("load_word<T, V>(") == 2 and "if (n >= STEPS) {" in rows and "if (s < n) w[s] = load_word<T, V>(" in rows
    assert source.count("load_word<T, V>(") == 2


def test_lanes_that_exchange_words_keep_their_order_by_a_fence():
    """Words in LDS that one lane of a wavefront writes and another reads, without a barrier of the workgroup: the order is kept by a fence
    of the wavefront, since a wave barrier by itself says nothing about memory."""
    source = open(os.path.join(CSRC, "embedding.hip")).read()
    barriers = re.findall(r"^.*\n.*__builtin_amdgcn_wave_barrier\(\);", source, re.M)
    assert barriers and all('__builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");' in b for b in barriers)
    for kernel in ("rank_keys", "embedding_direct_kernel"):
        text = _kernel(source, kernel)
        # read, fence, written, fence
        assert re.search(r"= (count\[digit\]|to\[wave\]\[row\]);.*?wave_in_order\(\);\s+if \(in && before == 0\) .*?;\s+wave_in_order\(\);", text, re.S)
