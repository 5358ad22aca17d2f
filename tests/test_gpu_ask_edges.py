"""Questions about regions: no words, no regions, and a host that does not wait."""
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


def test_look_does_not_wait_for_the_gpu(reader):
    import torch
    frames = [torch.zeros(64, 80, 3, dtype=torch.uint8, device="cuda") for _ in range(2)]
    reader.look(frames, _regions(3))
    torch.cuda.synchronize()
    busy = torch.cuda.Event()
    torch.cuda._sleep(int(1e9))                                      # some tenths of a second
    busy.record()
    reader.look(frames, _regions(3))
    waited = busy.query()
    torch.cuda.synchronize()
    assert not waited


def test_regions_keep_the_frames_of_their_call(reader):
    """The frame numbers' host copy may be gone or changed before the GPU reads it."""
    import torch
    frames = [torch.full((64, 80, 3), 30 * i, dtype=torch.uint8, device="cuda") for i in range(2)]
    held = []
    for change in (False, True):
        rois = _regions(4)
        if change:
            torch.cuda._sleep(int(1e8))
        ids = reader.look(frames, rois)
        if change:
            rois["frame"] = 0
            del rois
        at = ((ids % reader.capacity)[:, None] * ask.GRID ** 2 + torch.arange(ask.GRID ** 2, device="cuda")).view(-1)
        held.append([x[:, at].clone() for x in (reader.cache.k_codes, reader.cache.k_exps)])
    assert all(torch.equal(a, b) for a, b in zip(*held))
