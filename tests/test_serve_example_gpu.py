"""The serving example: learn, read, prefill over a window, decode over pages, evict, against 64 bits at every token.

Tolerance 5e-3: probabilities and outputs are rounded to bf16 once each (1.6e-3 together), times three."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_2608_17616_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("serve_cache", os.path.join(ROOT, "examples", "serve_cache.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kw", [
    {},
    dict(n_ctx=1, n_layers=1, n_kv=1, group=8, hd=128, page=64),
    dict(n_ctx=3, n_layers=2, prompt=70, window=5, page=8, tokens=150, most=100, keep=50, recent=0),
])
def test_every_token_of_the_example(example, kw):
    cuts, worst = example.serve(check=True, **kw)
    assert cuts >= 1
    assert worst <= 5e-3
