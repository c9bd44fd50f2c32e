"""The example that uses the paged cache's operators together: decoding with drafted trees on
shared pages gives what decoding token by token gives, in fewer passes, and every page
comes back. In fp32, where the two ways' roundings (1e-6 of the logits) stay far below
the margins of random logits."""
import importlib.util
import os

import pytest

from paper_2505_14260_gb300 import build

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "shared_image.py")


@pytest.mark.parametrize("questions,tokens,nodes", [(1, 12, 16), (5, 20, 16), (3, 9, 7)])
def test_trees_give_the_tokens_of_plain_decoding(questions, tokens, nodes):
    build.build()
    spec = importlib.util.spec_from_file_location("shared_image", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got, fast, passes, pages = example.run(questions, tokens, "f32", nodes, seed=questions, say=lambda *a: None)
    for g, f in zip(got, fast):
        assert f[: len(g)] == g
    assert passes < tokens
    assert int(pages.refs.sum()) == 0 and int(pages.lens.sum()) == 0
    got, fast, _, pages = example.run(questions, tokens, "bf16", nodes, seed=questions, say=lambda *a: None)
    assert all(len(f) > tokens for f in fast) and int(pages.refs.sum()) == 0
