"""The example that routes prompts and serves one worker's share from the paged cache."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)


def test_the_workers_steps_agree_with_plain_attention():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "worker_steps.py")
    spec = importlib.util.spec_from_file_location("worker_steps", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    # weights and outputs rounded to bf16 (2^-8 each) on values of at most about 5
    assert m.main(n_prompts=20, steps=3) <= 2 * 2.0 ** -8 * 5
