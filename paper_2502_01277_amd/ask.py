"""Questions about the regions a cascade finds: crops become tokens, their keys and values are kept in 4 bits, text tokens read them.

    frames, ROI table -> crop-resize -> patches (8 x 8 / stride 8 layer) -> keys and values (1x1 layer)
                      -> head norms and rotation by (frame, row, column) -> cache of 4 bits a value      RegionReader.look
    text tokens -> queries (1x1 layer) -> head norms and rotation -> attention to one region's tokens each
                -> output layer                                                                          RegionReader.ask

The layers, norms, rotations, cache and attention run in the library's kernels, indices and copies in torch's, all on the current stream; nothing
waits for the GPU.  The weights are random, as all of this package's: the module shows how the calls go together.

    python -m paper_2502_01277_amd.ask        # the tiny cascade's regions, one question each
"""
from __future__ import annotations

import math
import sys

import numpy as np

from . import binding
from .synth import to_storage

GRID = 7                # tokens along a side of a crop
PATCH = 8               # pixels along a side of a token
AXES = (8, 12, 12)      # pairs of a head turned by frame, row and column


class RegionReader:
    """Tokens of the last `capacity` regions, and the layers around them (width: channels of a token and of the text)."""

    def __init__(self, dtype="bf16", width=256, q_heads=8, kv_heads=2, capacity=1024, seed=0):
        import torch
        rng = np.random.default_rng(seed)
        self.dtype, self.width, self.q_heads, self.kv_heads, self.dim, self.capacity = dtype, width, q_heads, kv_heads, 2 * sum(AXES), capacity
        self.torch_dtype = binding.torch_dtype(dtype)

        def layer(cout, k, cin, stride=1):
            w = rng.standard_normal((cout, k, k, cin)).astype(np.float32) / math.sqrt(k * k * cin)
            return binding.ConvOp(to_storage(w, dtype), np.zeros(cout, np.float32), dtype, stride=stride)

        self.patches = layer(width, PATCH, 3, PATCH)
        self.to_kv = layer(2 * kv_heads * self.dim, 1, width)
        self.to_q = layer(q_heads * self.dim, 1, width)
        self.to_out = layer(width, 1, q_heads * self.dim)
        self.q_weight = torch.ones(self.dim, device="cuda")
        self.k_weight = torch.ones(self.dim, device="cuda")
        self.cache = binding.Cache4.zeros(kv_heads, capacity * GRID * GRID, self.dim)
        cell = torch.arange(GRID * GRID, dtype=torch.int32, device="cuda")
        self.cells = torch.stack([torch.zeros_like(cell), cell // GRID, cell % GRID], 1)          # (frame, row, column) inside a crop
        self.seen = 0

    def _linear(self, layer, x):
        """[n][cin] -> [n][cout] by a 1x1 layer."""
        n, cin = x.shape
        y = x.new_empty(n, layer.cout)
        if n:
            binding.op_conv(layer, x.view(n, 1, 1, cin), y.view(n, 1, 1, layer.cout))
        return y

    def look(self, frames, rois, first_frame=0):
        """Tokens of the regions `rois` (ROI records, as Pipeline.get_rois gives them) of `frames` into the cache.  Returns the numbers by which `ask` knows
        the regions; those of more than `capacity` regions ago are gone."""
        import torch
        n = len(rois)
        if n > self.capacity:
            raise ValueError("%d regions, room for %d" % (n, self.capacity))
        ids = torch.arange(self.seen, self.seen + n, device="cuda")
        self.seen += n
        if not n:
            return ids
        crops = binding.op_crop_resize(frames, rois, GRID * PATCH, GRID * PATCH, self.dtype)
        tokens = torch.empty(n, GRID, GRID, self.width, dtype=self.torch_dtype, device="cuda")
        binding.op_conv(self.patches, crops, tokens)
        kv = self._linear(self.to_kv, tokens.view(n * GRID * GRID, self.width)).view(-1, 2 * self.kv_heads, self.dim)
        pos = self.cells.repeat(n, 1, 1)
        # from pinned memory, so that the host goes on (torch keeps it until the copy is done)
        frame = torch.from_numpy(np.ascontiguousarray(rois["frame"])).pin_memory()
        pos[:, :, 0] = frame.to(pos.device, non_blocking=True)[:, None] + first_frame
        keys = kv[:, :self.kv_heads]
        binding.op_rotate([binding.RotatePart(keys, keys, self.k_weight)], pos.view(-1, 3), AXES)
        slots = (ids % self.capacity)[:, None] * (GRID * GRID) + torch.arange(GRID * GRID, device="cuda")
        binding.op_cache4_store(self.cache, keys, kv[:, self.kv_heads:], slots.view(-1))
        return ids

    def queries(self, text, frame):
        """Normed and turned queries of text tokens [n][width] asked at frame numbers [n]."""
        import torch
        q = self._linear(self.to_q, text).view(-1, self.q_heads, self.dim)
        pos = torch.zeros(text.shape[0], 3, dtype=torch.int32, device="cuda")
        pos[:, 0] = frame
        binding.op_rotate([binding.RotatePart(q, q, self.q_weight)], pos, AXES)
        return q

    def ask(self, text, q_start, regions, frame, max_q=None):
        """What question b, the rows q_start[b] .. q_start[b + 1] - 1 of text [n][width], reads in regions[b]: [n][width].  q_start int32 and regions (numbers from
        `look`) on the device; frame: int32 [n], when each token is asked; max_q: the longest question."""
        import torch
        q = self.queries(text, frame)
        out = torch.zeros_like(q)
        start = regions % self.capacity * (GRID * GRID)
        length = torch.full((regions.shape[0],), GRID * GRID, dtype=torch.int32, device="cuda")
        binding.op_attend(q, self.cache, out, q_start, start, length, max_q=max_q, max_kv=GRID * GRID)
        return self._linear(self.to_out, out.view(-1, self.q_heads * self.dim))


def main() -> int:
    import torch
    from . import synth, zoo
    spec = zoo.tiny_cascade()
    scene = synth.make_scene(np.random.default_rng(zoo.SEED0 + 1), 2, 320, 320, [6, 6], 16, 96, n_classes=8)
    frames = [torch.from_numpy(f).cuda() for f in scene.frames]
    pipe = binding.Pipeline(spec)
    pipe.submit(frames)
    pipe.run()
    pipe.collect()
    rois = pipe.get_rois(0)
    pipe.close()
    reader = RegionReader()
    regions = reader.look(frames, rois)
    n, words = len(rois), 6
    text = torch.randn(n * words, reader.width, device="cuda").to(reader.torch_dtype)
    q_start = torch.arange(0, n * words + 1, words, dtype=torch.int32, device="cuda")
    frame = torch.from_numpy(np.repeat(rois["frame"].astype(np.int32), words)).cuda()
    answer = reader.ask(text, q_start, regions, frame, max_q=words)
    print("%d regions of %d tokens in %.1f KiB, %d questions of %d tokens, answers %s, rms %.3f" % (
        n, GRID * GRID, n * GRID * GRID * reader.kv_heads * reader.dim * 2 * 17 / 32 / 1024, n, words, tuple(answer.shape), float(answer.float().pow(2).mean().sqrt())))
    return 0


if __name__ == "__main__":
    sys.exit(main())
