"""CPU: the positions that the serving example gives its tokens."""
import importlib.util
import os
import sys

import torch


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")
    spec = importlib.util.spec_from_file_location("paged_serving", path)
    module = importlib.util.module_from_spec(spec)
    sys.modules["paged_serving"] = module                            # its dataclasses look themselves up there
    spec.loader.exec_module(module)
    return module


def test_an_image_token_has_its_row_and_column():
    """Two sequences whose images begin behind 10 and 37 tokens, six tokens to a row."""
    positions = _example().positions
    begin = torch.tensor([10, 37])
    for i in range(20):
        time, row, column = positions(begin + i, i, 6)
        assert torch.equal(time, begin + i) and torch.equal(row, begin + i // 6) and torch.equal(column, begin + i % 6)


def test_a_prompts_token_has_its_time_on_every_axis():
    time = torch.arange(7)
    got = _example().positions(time, None, 6)
    assert got.dtype is torch.int32 and got.shape == (3, 7) and bool((got == time).all())
