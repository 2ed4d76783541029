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


def test_no_warp_parts_over_a_wait():
    """Loads of TMEM and the choice of an issuing lane want all lanes of a warp: if a wait runs out for some of them and not for others, the rest must not go
    on without them. So the waits whose answer is a branch vote, the others' answers (bar_pass) decide no more than whether the chosen lane
    issues, and nobody tries a barrier elsewhere."""
    text = " ".join(code().values())
    wait = re.search(r"bool bar_wait\(.*?\n\}\n", text, flags=re.S).group()
    assert wait.count("return true") == wait.count("bar_try(") == wait.count("__all_sync(0xffffffffu, bar_try(") == 2
    assert wait.count("*gave_up)") == wait.count("__any_sync(0xffffffffu, *gave_up)") == 2
    assert len(re.findall(r"\bbar_try\(", text)) == 5                                            # its definition and the two waits
    rest = re.sub(r"bool bar_pass\(.*?\n\}\n", "", text, flags=re.S)
    for line in rest.splitlines():
        if "bar_pass<" in line:
            assert re.search(r"(^|;|\)|\{)\s*((bool )?ok = )?bar_pass<!?\w+>\([^;]*\)( && ok)?;", line) and not re.search(r"(if|while) \(!?bar_pass|&& bar_pass|return bar_pass|\? bar_pass", line), line
    assert not re.search(r"\bok && elected\(\)", text)


def test_attention_weights_meet_at_barriers_whatever_has_run_out():
    """A warp that has given up a wait leaves its loop: it must not be one that others meet at a barrier without a limit."""
    text = code()["weight_kernels.cuh"]
    loops = text[text.index("chunk_weights_kernel("):]
    loops = loops[loops.index("pdl_trigger"):loops.rindex("tmem_fence_before")]
    sums, rest = loops[loops.index("if (warp < 16)"):loops.index("if (warp == 16)")], loops[loops.index("if (warp == 16)"):]
    assert "bar.sync" in sums and "bar_pass<" in sums and not re.search(r"\bok\b|\bbreak\b|bar_wait|gave_up\)\s*(\)|&&)", sums)
    assert "bar_wait<" in rest and not re.search(r"bar\.sync|bar\.arrive|barrier\.|__syncthreads|cluster_wait", rest)


def test_attention_weights_read_a_tiles_bad_pages_before_they_let_go_of_it():
    """Behind the arrival nothing keeps the loading warps from the tag's place."""
    text = code()["weight_kernels.cuh"]
    sums = text[text.index("if (warp < 16)"):text.index("else if (warp == 16)")]
    assert sums.count("bad_pages[") == 1 and sums.index("bad_pages[") < sums.index("bar_arrive(smem_u32(&sh.d_empty")
