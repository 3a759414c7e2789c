"""The example of a server loop on the paged cache: mixed chunks and single tokens against dense attention without a cache."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")


@pytest.mark.parametrize("chunk", [1, 48, 500])
def test_serving_loop_agrees_with_dense_attention(chunk):
    print(f"[case] paged serving, chunks of {chunk}", flush=True)
    spec = importlib.util.spec_from_file_location("paged_serving", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # per block: probabilities, attention output, projection and residual each rounded to bf16 (2^-8), on both sides, two blocks
    assert example.main(["--chunk", str(chunk), "--new", "8"]) <= 16 * 2.0 ** -8
