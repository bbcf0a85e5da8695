"""The example of a search where the prompt is no longer than what is kept: the first cut then meets beams that still share their prompt's pages."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests,beams,prompt,steps,keep", [(8, 4, 256, 10, 256), (3, 4, 64, 20, 64), (2, 3, 30, 30, 48), (2, 2, 33, 18, 33)])
def test_example_of_a_search_over_short_prompts(requests, beams, prompt, steps, keep):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("gpu-marked test run without a CUDA device")
    spec = importlib.util.spec_from_file_location("serving_step_example", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    cache, tokens, scores, _ = example.search(requests, beams, prompt, steps, keep)
    assert tuple(tokens.shape) == (requests, beams, steps) and cache.status_flags() == 0
    assert int(cache.length.min()) == int(cache.length.max()) <= keep + 8
