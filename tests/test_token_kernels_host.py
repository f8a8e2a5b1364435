"""What can be seen of the token-block kernels without a GPU: declarations that the compiler accepts and that only its
placement or luck in timing would make right."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2105_09080_b200" / "csrc"
FILES = ["gpga_dropout.cu", "gpga_norm.cu", "gpga_norm_grad.cu", "gpga_embed.cu"]


def code(name):
    """A source file without its comments."""
    text = (CSRC / name).read_text()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


@pytest.mark.parametrize("name", FILES)
def test_shared_arrays_that_are_read_wider_than_their_type_are_aligned(name):
    """An array of a type below eight bytes has that type's alignment unless it says more.  One that is only indexed needs
    no more; one that is handed on (a pointer to it, an argument) meets 64- and 128-bit accesses there."""
    found = 0
    for kernel in re.split(r"\b__global__\b", code(name))[1:]:
        for m in re.finditer(r"__shared__ (__align__\(\d+\) )?(float|uint32_t|int|T) ([^;]+);", kernel):
            found += 1
            for array in re.findall(r"(\w+)(?:\[[^,]*\])+", m[3]):
                rest = kernel[:m.start()] + kernel[m.end():]
                handed_on = re.search(rf"\b{array}\b(?!\s*\[)", rest)
                assert m[1] or not handed_on, f"{name}: {array} in '{m[0]}'"
    assert found




@pytest.mark.parametrize("name", FILES + ["gpga_token_api.cu", "gpga_launch.cuh"])
def test_host_statics_can_be_shared_by_threads(name):
    """The entries take no handle and may be called from several threads: what a host function keeps from one call to the
    next is initialised once by the language (const) or atomic."""
    kept = re.findall(r"^\s+static (?!__device__|inline\b|constexpr\b)[^;({]*", code(name), flags=re.M)
    assert all(re.match(r"\s+static (const |std::atomic<)", s) for s in kept), kept
