"""The example that runs the token operators together on stitched canvases."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_patches_come_out_as_if_alone():
    """Whatever shares a patch's canvas does not change its tokens, nor the one after them. Each
    result passes four roundings to bfloat16 (embedding, queries and keys, heads, output), each of
    2^-8 at most, whose inputs may differ by one; a leak between patches changes whole values."""
    spec = importlib.util.spec_from_file_location(
        "canvas_layer", os.path.join(ROOT, "examples", "canvas_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main() <= 4 * 2.0 ** -8
