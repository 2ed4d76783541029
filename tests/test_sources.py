"""Rules that the CUDA sources keep and that no run can show."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_05076_b200", "csrc")


def code():
    """The sources without their comments, by file name."""
    out = {}
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        text = re.sub(r"/\*.*?\*/", " ", open(path).read(), flags=re.S)
        out[os.path.basename(path)] = re.sub(r"//[^\n]*", "", text)
    assert len(out) >= 5
    return out


def test_nothing_is_read_through_the_non_coherent_path():
    """Kernels begin while the one before them still writes (programmatic launches), so what they read changes during their life:
    neither __ldg nor what lets the compiler choose it (const __restrict__)."""
    for name, text in code().items():
        for word in (r"\b__ldg\b", r"ld\.global\.nc", r"ld\.global\S*\.nc\b", r"__restrict__"):
            assert not re.search(word, text), (name, word)


def test_every_device_function_is_called():
    text = " ".join(code().values())
    names = re.findall(r"__device__[^;{}()]*?(\w+)\s*\([^;{]*\)\s*\{", text)
    assert len(names) > 50
    unused = sorted({n for n in names if len(re.findall(r"\b%s\b" % n, text)) < 2})
    assert not unused, unused
