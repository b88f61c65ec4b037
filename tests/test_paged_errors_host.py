"""CPU checks of the error queries of paged attention and of a model (nothing reaches a GPU)."""
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def test_null_arguments(B):
    assert B.lib().w8a8_model_check(None, None) == 1
    assert B.lib().w8a8_paged_attention_error_word(None) == 1
