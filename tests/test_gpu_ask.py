"""Questions about regions: the calls on tokens in a row, each step against the 64-bit oracle on what the step before gave."""
import numpy as np
import pytest

from oracle import tokens
from paper_2502_01277_amd import ask, binding

pytestmark = pytest.mark.gpu


def _np(x):
    return x.detach().double().cpu().numpy()


@pytest.mark.parametrize("dtype,half_step", [("bf16", 2.0 ** -8), ("f16", 2.0 ** -11)])
def test_regions_are_looked_at_and_read(octo, dtype, half_step):
    import torch
    rng = np.random.default_rng(5)
    frames = [torch.from_numpy(rng.integers(0, 256, (240, 320, 3)).astype(np.uint8)).cuda() for _ in range(3)]
    n = 9
    rois = np.zeros(n, binding.ROI_DTYPE)
    rois["frame"] = rng.integers(0, 3, n)
    rois["x1"], rois["y1"] = rng.uniform(0, 200, n), rng.uniform(0, 120, n)
    rois["x2"], rois["y2"] = rois["x1"] + rng.uniform(10, 110, n), rois["y1"] + rng.uniform(10, 110, n)
    reader = ask.RegionReader(dtype, width=64, q_heads=4, kv_heads=2, capacity=12, seed=3)
    reader.look(frames, rois[:6])
    ids = reader.look(frames, rois, first_frame=40)               # rows 6 .. 11, then 0 .. 2 again
    assert ids.tolist() == list(range(6, 15))
    cells, d = ask.GRID ** 2, reader.dim
    # the projection again, by hand from the patches, and what the cache should hold of it
    crops = octo.op_crop_resize(frames, rois, ask.GRID * ask.PATCH, ask.GRID * ask.PATCH, dtype)
    tok = torch.empty(n, ask.GRID, ask.GRID, 64, dtype=reader.torch_dtype, device="cuda")
    octo.op_conv(reader.patches, crops, tok)
    kv = reader._linear(reader.to_kv, tok.view(-1, 64)).view(n * cells, 4, d)
    pos = np.zeros((n, cells, 3), np.int32)
    pos[:, :, 0] = rois["frame"][:, None] + 40
    pos[:, :, 1], pos[:, :, 2] = np.arange(cells) // ask.GRID, np.arange(cells) % ask.GRID
    keys = tokens.rotate(_np(kv[:, :2]), np.ones(d), pos.reshape(-1, 3), ask.AXES, 10000.0)
    slots = ((ids % 12)[:, None] * cells + torch.arange(cells, device="cuda")).view(-1)
    k, v = torch.empty(n * cells, 2, d, device="cuda"), torch.empty(n * cells, 2, d, device="cuda")
    octo.op_cache4_load(reader.cache, slots, k, v)
    assert np.array_equal(_np(v), tokens.mx4_decode(*tokens.mx4_encode(_np(kv[:, 2:]), 140 if dtype == "f16" else 252)))
    # keys are rounded to 16 bits before the 4: a value within that rounding of a middle may take either neighbour
    ref = tokens.mx4_decode(*tokens.mx4_encode(keys))
    assert np.mean(np.abs(_np(k) - ref) > 0) < 0.05
    assert np.all(np.abs(_np(k) - keys) <= np.repeat(np.abs(keys.reshape(-1, 2, d // 32, 32)).max(-1) / 3.4, 32, -1).reshape(keys.shape))
    # questions of several lengths, one without words, two about one region
    lens, about = [3, 0, 5, 1, 2], [8, 2, 0, 0, 4]
    q_start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    text = torch.randn(sum(lens), 64, generator=torch.Generator().manual_seed(1)).to(reader.torch_dtype).cuda()
    when = torch.arange(sum(lens), dtype=torch.int32, device="cuda")
    regions = ids[torch.tensor(about, device="cuda")]
    answer = reader.ask(text, q_start, regions, when, max_q=5)
    q = reader.queries(text, when)
    start = _np(regions % 12).astype(np.int64) * cells
    pool_k, pool_v = np.zeros((12 * cells, 2, d)), np.zeros((12 * cells, 2, d))
    at = slots.cpu().numpy()
    pool_k[at], pool_v[at] = _np(k), _np(v)
    out, _ = tokens.attend(_np(q), pool_k, pool_v, _np(q_start).astype(int), start, [cells] * 5, d ** -0.5)
    # through the output layer in 64 bits: its inputs and the weights of the attention are rounded once each, its output once
    w = np.random.default_rng(3)
    shapes = [(64, 8, 8, 3), (2 * 2 * d, 1, 1, 64), (4 * d, 1, 1, 64), (64, 1, 1, 4 * d)]
    mats = [w.standard_normal(s).astype(np.float32) / np.float32(np.sqrt(np.prod(s[1:]))) for s in shapes]
    last = torch.from_numpy(mats[3].reshape(64, -1)).to(reader.torch_dtype).double().numpy()
    ref = out.reshape(len(text), -1) @ last.T
    size = np.abs(out).reshape(len(text), -1) @ np.abs(last).T
    spread = np.abs(pool_v).max() * np.abs(last).sum(1)
    assert np.all(np.abs(_np(answer) - ref) <= half_step * (np.abs(ref) + 2 * size + 2 * spread))


def test_command(octo, capsys):
    assert ask.main() == 0
    assert "regions of 49 tokens" in capsys.readouterr().out
