"""The serving example of the 4-bit cache: a captured step over contexts that grow and are cut, against 64 bits at every token.

Tolerance 4.4e-3: a rotated row or an output is off by half a step of bf16, 2^-8 of it at most, an output's probabilities by 2^-11."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_2608_17616_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("serve_cache4", os.path.join(ROOT, "examples", "serve_cache4.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kw", [
    {},
    dict(n_ctx=1, n_layers=1, n_kv=1, group=8, hd=128, page=64),
    dict(n_ctx=3, n_layers=2, prompt=70, page=8, tokens=150, most=100, keep=50, recent=0),
])
def test_every_token_of_the_example(example, kw):
    cuts, left, worst = example.serve(check=True, **kw)
    assert cuts >= 1
    assert worst <= 4.4e-3
    o = dict(dict(n_ctx=2, n_mem=16, prompt=150, tokens=60, most=192, keep=96, page=16), **kw)
    length = o["n_mem"] + o["prompt"]
    for _ in range(o["tokens"]):
        length = (o["keep"] if length == o["most"] else length) + 1
    width = -(-o["most"] // o["page"]) + 1
    assert left == o["n_ctx"] * (width + -(-o["keep"] // o["page"]) - -(-length // o["page"]))  # every page is somewhere
