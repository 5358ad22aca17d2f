"""octo_op_sample on rows whose words are ruled out by large finite numbers, and at temperatures that leave most words without weight: borders by count then lie among logits thousands of octaves
below the largest.  Against the definition, as in test_gpu_sample."""
import itertools

import numpy as np
import pytest

from test_gpu_sample import _check, _run, _t

pytestmark = pytest.mark.gpu
MASKS = {"f32": (-1e4, -1e9, -3.4028234663852886e38), "f16": (-1e4, -65504.0), "bf16": (-1e4, -1e9, -3.3895313892515355e38)}


def _masked(dtype, others, seed, allowed=(5, 300, 700)):
    """A row for each number of allowed words and each mask: the words at random places, in steps so that many are alike in half of the rows; what is left of the row may not be drawn."""
    import torch
    g = torch.Generator().manual_seed(seed)
    rows = []
    for i, (count, mask) in enumerate(itertools.product(allowed, MASKS[dtype])):
        row = torch.full((max(allowed) + others,), -float("inf"))
        place = torch.randperm(count + others, generator=g)
        words = torch.randn(count, generator=g) * 2
        row[place[:count]] = words if i % 2 else (words * 4).round() / 4
        row[place[count:]] = mask
        rows.append(row)
    return torch.stack(rows).to(_t(dtype)).cuda(), torch.rand(len(rows), generator=g).clamp_(min=0.01).cuda()


MORE = (dict(), dict(top_p=0.9), dict(min_p=0.01))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("others", [1500, 30000])
@pytest.mark.parametrize("top_k", [0, 50, 400, 700, 1000, 3500])
def test_words_ruled_out_by_finite_numbers(octo, dtype, others, top_k):
    logits, u = _masked(dtype, others, others + top_k)
    for temperature, more in itertools.product((1.0, 0.005, 1e-3), MORE):
        settings = dict(top_k=top_k, temperature=temperature, **more)
        _check(_run(octo, logits, u, **settings), logits, u, settings)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("top_k,temperature", [(0, 1.0), (50, 1.0), (700, 1.0), (1000, 0.005), (3500, 1e-3), (60000, 1.0)])
def test_the_same_in_long_rows(octo, dtype, top_k, temperature):
    """With a workspace, without one, and with the numbers of each row on the device."""
    import torch
    logits, u = _masked(dtype, 70000, top_k)
    n = logits.shape[0]
    token = torch.empty(n, dtype=torch.int32, device="cuda")
    each = torch.full((n,), top_k, dtype=torch.int32, device="cuda")
    for more in MORE:
        settings = dict(top_k=each, temperature=temperature, **more)
        work = torch.full((octo.sample_workspace_bytes(logits, u, token, **settings),), 0xFF, dtype=torch.uint8, device="cuda")
        got = _run(octo, logits, u, workspace=work, **settings)
        for other in (_run(octo, logits, u, workspace=work[:0], **settings), _run(octo, logits, u, **dict(settings, top_k=top_k))):
            assert all(np.array_equal(a, b) for a, b in zip(got, other))
        _check(got, logits, u, settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_most_words(octo, dtype):
    logits, u = _masked(dtype, (1 << 19) - 700, 3, allowed=(5, 700))
    for settings in (dict(top_k=1000, top_p=0.9), dict(top_k=400000, temperature=0.005), dict(top_k=50)):
        _check(_run(octo, logits, u, **settings), logits, u, settings)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [3000, 20000])
@pytest.mark.parametrize("temperature", [0.02, 0.005, 0.001, 1e-5])
def test_low_temperatures_and_many_words(octo, dtype, vocab, temperature):
    """Plain logits: few words have weight, the count goes on among those that have none."""
    import torch
    g = torch.Generator().manual_seed(vocab)
    logits = (torch.randn(8, vocab, generator=g) * 2).to(_t(dtype)).cuda()
    u = torch.rand(8, generator=g).clamp_(min=0.01).cuda()
    for top_k, more in itertools.product((513, 1000, 2500), MORE):
        settings = dict(top_k=top_k, temperature=temperature, **more)
        _check(_run(octo, logits, u, **settings), logits, u, settings)
