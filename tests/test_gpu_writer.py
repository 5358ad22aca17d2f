"""Words about regions: norm, product and draw as a model's layers call them, each call against the 64-bit definitions on what it was given."""
import types

import numpy as np
import pytest

import test_gpu_product as products
import test_gpu_sample as samples
from paper_2502_01277_amd import ask, binding

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _reader(octo, dtype, n=5, **kw):
    import torch
    rng = np.random.default_rng(9)
    frames = [torch.from_numpy(rng.integers(0, 256, (120, 160, 3)).astype(np.uint8)).cuda() for _ in range(2)]
    rois = np.zeros(n, binding.ROI_DTYPE)
    rois["frame"] = rng.integers(0, 2, n)
    rois["x1"], rois["y1"] = rng.uniform(0, 80, n), rng.uniform(0, 60, n)
    rois["x2"], rois["y2"] = rois["x1"] + rng.uniform(10, 60, n), rois["y1"] + rng.uniform(10, 50, n)
    reader = ask.RegionReader(dtype, width=64, q_heads=4, kv_heads=2, capacity=8, seed=3)
    return reader, reader.look(frames, rois), ask.RegionWriter(reader, vocab=1000, layers=2, hidden=96, **kw)


def _values(octo, x):
    import torch
    if not isinstance(x, binding.Mx8):
        return x.double()
    y = torch.empty(x.codes.shape, device="cuda")
    octo.op_mx8_load(x, y)
    return y.double()


class Checked:
    """The three calls, each of which is checked before the next one is made."""

    def __init__(self, octo, monkeypatch, dtype):
        self.octo, self.dtype, self.calls, self.half = octo, dtype, [], HALF[dtype]
        self.plain = types.SimpleNamespace(op_sample=binding.op_sample)
        for name in ("op_norm", "op_product", "op_sample"):
            monkeypatch.setattr(binding, name, self.wrap(name, getattr(binding, name)))

    def wrap(self, name, call):
        def checked(*args, **kw):
            import torch
            old = {k: v.double() for k, v in kw.items() if k in ("res",)}
            x = _values(self.octo, args[0])
            out = call(*args, **kw)
            self.calls.append(name)
            getattr(self, name)(x, args, kw, old, out)
            return out
        return checked

    def op_norm(self, x, args, kw, old, out):
        import torch
        y, weight = args[1], args[2]
        s = x + old["res"] if "res" in old else x
        ref = s / torch.sqrt((s * s).mean(-1, keepdim=True) + 1e-6) * weight.double()
        if "total" in kw:                                              # a sum in fp32, rounded to 16 bits
            assert bool(((kw["total"].double() - s).abs() <= (self.half + 2.0 ** -23) * s.abs()).all())
        # the sum's rounding to fp32, through the norm twice, and one rounding at the end
        off = 3 * 2.0 ** -24 * (x.abs() + (old["res"].abs() if "res" in old else 0)) * (ref / s).abs().nan_to_num(0.0) + 2.0 ** -22 * ref.abs()
        if isinstance(y, binding.Mx8):
            products._check_mx8(y, ref, off)
        else:
            products._check(y, ref, off, self.dtype)

    def op_product(self, x, args, kw, old, kernel):
        w, y = _values(self.octo, args[1]), args[2]
        eight = isinstance(args[0], binding.Mx8)
        assert kernel > 0
        ref, off = products._reference(x, w, None, kw.get("act", "none"), kw.get("gated", False), old.get("res"), False, products.GRAIN if eight and kernel < 10 else 0.0)
        if isinstance(y, binding.Mx8):
            products._check_mx8(y, ref, off)
        else:
            import torch
            products._check(y, ref, off, "f32" if y.dtype is torch.float32 else self.dtype)

    def op_sample(self, x, args, kw, old, out):
        logits, u, word = args
        settings = {k: v for k, v in kw.items() if k != "logprob"}
        got = samples._run(self.plain, logits, u, **settings)
        samples._check(got, logits, u, settings)
        assert np.array_equal(got[0], word.cpu().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens", [[3, 0, 5, 1, 2], [30, 1, 0, 40, 5]])
def test_every_call_of_a_draw(octo, monkeypatch, dtype, lens):
    import torch
    reader, ids, writer = _reader(octo, dtype)
    seen = Checked(octo, monkeypatch, dtype)
    n = sum(lens)
    g = torch.Generator().manual_seed(n)
    q_start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    words = torch.randint(0, writer.vocab, (n,), generator=g, dtype=torch.int32).cuda()
    x = writer.states(words, q_start, ids, torch.arange(n, dtype=torch.int32, device="cuda"), max_q=max(lens))
    assert x.shape == (n, 64) and bool(torch.isfinite(x).all())
    writer.draw(x, torch.rand(n, generator=g).cuda(), temperature=0.8, top_k=40, top_p=0.9, min_p=0.01)
    assert seen.calls == (["op_norm", "op_product", "op_product", "op_norm", "op_product", "op_product"] * 2 + ["op_norm", "op_product", "op_sample"])


def test_words_follow_words(octo):
    """Each word is drawn after the one before it, from the numbers it is given; without questions there are none."""
    import torch
    reader, ids, writer = _reader(octo, "bf16")
    first, frame = torch.arange(5, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    u = torch.rand(4, 5, generator=torch.Generator().manual_seed(2)).cuda()
    said = writer.write(first, ids, frame, u, temperature=1.2, top_p=0.95)
    assert said.shape == (4, 5) and bool(((said >= 0) & (said < writer.vocab)).all())
    again = writer.write(first, ids, frame, u, temperature=1.2, top_p=0.95)
    assert torch.equal(said, again)
    rest = writer.write(said[1], ids, frame, u[2:], temperature=1.2, top_p=0.95)
    assert torch.equal(rest, said[2:])
    assert not torch.equal(writer.write(first, ids, frame, 1 - u, temperature=1.2, top_p=0.95), said)
    assert writer.write(first[:0], ids[:0], frame[:0], u[:, :0]).shape == (4, 0)


def test_captured_step(octo):
    """A step of five questions, captured once: its replays give what eager steps give, with eager work between them."""
    import torch
    reader, ids, writer = _reader(octo, "bf16")
    frame = torch.zeros(5, dtype=torch.int32, device="cuda")
    q_start = torch.arange(6, dtype=torch.int32, device="cuda")
    word, u, logprob = torch.arange(5, dtype=torch.int32, device="cuda"), torch.rand(5, device="cuda"), torch.empty(5, device="cuda")

    def step():
        return writer.draw(writer.states(word, q_start, ids, frame, max_q=1), u, logprob, temperature=0.9, top_k=100)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for turn in range(4):
        u.copy_(torch.rand(5, generator=torch.Generator().manual_seed(turn)))
        word.copy_(torch.arange(5, dtype=torch.int32) * (turn + 1))
        graph.replay()
        torch.cuda.synchronize()
        got, share = captured.clone(), logprob.clone()
        assert torch.equal(got, step()) and torch.equal(share, logprob)
