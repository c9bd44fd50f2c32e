"""The example with 4-bit weights and with a temperature: products, sampling and acceptance
beside the paged cache. At temperature 0 trees give the tokens of plain decoding, as with
whole weights."""
import importlib.util
import os

import pytest

from paper_2505_14260_gb300 import build

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "shared_image.py")


def example():
    build.build()
    spec = importlib.util.spec_from_file_location("shared_image", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("questions,tokens,nodes", [(1, 12, 16), (4, 16, 11)])
def test_four_bits_and_trees(questions, tokens, nodes):
    got, fast, passes, pages = example().run(questions, tokens, "f32", nodes, seed=questions, say=lambda *a: None, bits=4)
    assert all(f[: len(g)] == g for g, f in zip(got, fast))
    assert passes < tokens and int(pages.refs.sum()) == 0


@pytest.mark.parametrize("dtype,bits", [("bf16", 4), ("f32", 16)])
def test_a_temperature(dtype, bits):
    got, fast, _, pages = example().run(3, 12, dtype, 16, seed=7, say=lambda *a: None, bits=bits, temperature=0.8, top_p=0.9)
    assert all(len(f) > 12 and all(0 <= t < 1000 for t in f + g) for g, f in zip(got, fast))
    assert int(pages.refs.sum()) == 0 and int(pages.lens.sum()) == 0
