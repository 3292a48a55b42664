"""What the sequence kernels' sources have to keep to, checked without a GPU."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2212_11142_amd", "csrc")


@pytest.mark.parametrize("name", ["attend.hip", "attend_few.hip", "attend_grad.hip", "seq_dev.h"])
def test_no_vector_arithmetic_in_inline_assembly(name):
    """The results of a matrix or a transcendental instruction may be read a number of cycles
    later only. The compiler counts them for the instructions that it knows; inline assembly is
    read as soon as it stands there, so that the attention kernels have none that computes."""
    text = open(os.path.join(CSRC, name)).read()
    blocks = re.findall(r"\basm\s*(?:volatile)?\s*\(((?:[^()]|\([^()]*\))*)\)", text)
    assert blocks or name != "seq_dev.h"
    for b in blocks:
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', b.split(":")[0]))
        assert not re.search(r"(?<![A-Za-z0-9_])v_[a-z]", code), (name, code)


@pytest.mark.parametrize("name", ["attend_grad.hip", "seq_dev.h"])
def test_copies_wait_for_their_descriptor(name):
    """A buffer instruction reads scalar registers that a vector instruction may have written:
    5 cycles have to lie between, which the compiler does not see to before inline assembly."""
    text = open(os.path.join(CSRC, name)).read()
    blocks = re.findall(r"asm volatile\(((?:\s*\"[^\"]*\")+)", text)
    blocks = ["".join(re.findall(r'"([^"]*)"', b)) for b in blocks]
    blocks = [b.replace("\\n", "\n").replace("\\t", "\t") for b in blocks if "buffer_load" in b]
    assert blocks
    for b in blocks:
        code = b.split("buffer_load")[0].split("\n")
        waits = sum(int(l.split()[1]) + 1 if l.split()[0] == "s_nop" else 1 for l in code if l.strip())
        assert waits >= 5, b
