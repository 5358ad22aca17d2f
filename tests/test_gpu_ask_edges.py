"""Questions about regions: no words, no regions."""
import numpy as np
import pytest

from paper_2502_01277_amd import ask, binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def reader(octo):
    return ask.RegionReader("bf16", width=64, q_heads=4, kv_heads=2, capacity=12, seed=3)


def _regions(n):
    rois = np.zeros(n, binding.ROI_DTYPE)
    rois["x2"], rois["y2"], rois["frame"] = 50 + np.arange(n), 40, np.arange(n) % 2
    return rois


def test_no_words(reader):
    import torch
    frames = [torch.zeros(64, 80, 3, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ids = reader.look(frames, _regions(2))
    z = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    for q_start, regions in ((z(3), ids), (z(1), ids[:0])):          # two questions without words, no question
        assert tuple(reader.ask(z(0, 64, t=torch.bfloat16), q_start, regions, z(0)).shape) == (0, 64)
    assert reader.look(frames, _regions(0)).numel() == 0
