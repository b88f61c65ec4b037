"""CPU checks of the error query of the 4-bit linear (nothing reaches a GPU), and that each of its waits reports to both words."""
import os
import re

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def test_null_arguments(B):
    assert B.lib().w8a8_fp4_linear_error_word(None) == 1
    assert b"w8a8_fp4_linear_error_word" in B.lib().w8a8_last_error()


def test_every_wait_that_gives_up_says_so(B):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "paper_2608_28003_gb300", "csrc", "fp4_linear.cu")).read()
    assert re.findall(r"atomicOr\((.*?),", text) == ["a.err", "a.gave_up"]
    assert len(re.findall(r"give_up\(a, DEVERR_", text)) == 5
