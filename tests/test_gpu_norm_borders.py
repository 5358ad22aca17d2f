"""octo_op_norm on the GPU, to its last bits: the residual's sum is one fp32 rounding, everything after it is in fp64 as far as a result shows it.

The reference takes that sum in fp32 and goes on in fp64; sums of squares in another order differ by a few 2^-53 of themselves.  Plain results: fp32 are rounded once; of 16 bits the factor and two products
are rounded to fp32 first, 3 * 2^-24 of the value (and the last rounding of that, 3 * 2^-24 (1 + 2^-8) in all).  Codes and exponents of 8 bits are those of the reference, except for values within 2^-40 of a middle between two codes, or of where an exponent changes."""
import numpy as np
import pytest

from oracle import answer
from test_gpu_norm import STEP, _np, _t

pytestmark = pytest.mark.gpu
NEAR = 2.0 ** -40


def _reference(x, res, w, eps):
    x = x.float().cpu().numpy()
    s = (x if res is None else x + res.float().cpu().numpy()).astype(np.float64)
    return s, s / np.sqrt((s * s).mean(-1, keepdims=True) + eps) * w.cpu().numpy().astype(np.float64)


def _same_codes(y8, ref):
    codes, exps = y8.codes.cpu().numpy(), y8.exps.cpu().numpy()
    best, best_exps = answer.mx8_encode(ref)
    off = exps != best_exps
    most = np.abs(ref).reshape(ref.shape[0], -1, 32).max(-1)
    border = 448.0 * np.exp2(np.minimum(exps, best_exps).astype(np.float64) - 127)
    assert np.all(np.abs(most / border - 1)[off] <= NEAR), np.argwhere(off)[:4]
    wrong = (codes != best) & ~np.repeat(off, 32, -1)
    if wrong.any():
        scale = np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, -1)[wrong]
        a, b = (answer.mx8_decode(c[wrong][:, None].repeat(32, 1), np.full((int(wrong.sum()), 1), 127, np.uint8))[:, 0] for c in (codes, best))
        assert np.all(np.abs(np.abs(ref[wrong] / scale) / np.abs((a + b) / 2) - 1) <= NEAR), (np.argwhere(wrong)[:4], int(wrong.sum()))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,width,with_res", [(2000, 4096, False), (2000, 4096, True), (700, 96, True), (60, 32768, False)])
def test_codes_are_the_definitions(octo, dtype, n, width, with_res):
    """Among eight million values some lie so near to a middle that fp32 takes the other code."""
    import torch
    g = torch.Generator().manual_seed(n + width)
    x, r = (torch.randn(n, width, generator=g).to(_t(dtype)).cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(width, generator=g)).cuda()
    y = octo.Mx8.empty(n, width)
    octo.op_norm(x, y, w, res=r if with_res else None)
    _same_codes(y, _reference(x, r if with_res else None, w, 1e-6)[1])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("eps", [1e-6, 3e-5, 0.37])
def test_codes_beside_every_border(octo, dtype, eps):
    """Weights that bring every value to within fp32's spacing of a middle between two codes, among those without a leading one too, and groups' largest values to where the exponent changes."""
    import torch
    v = answer.e4m3_decode(np.arange(127, dtype=np.uint8))
    mids = (v[1:] + v[:-1]) / 2
    factor = 1 / np.sqrt(1 + eps)                               # of rows of ones of either sign
    groups = []
    for e in (-7, 0, 5):
        for top in (448.0, 300.0, 224.1):
            for step in (-2, -1, 0, 1, 2):
                for first in range(0, len(mids) - 30, 31):
                    t = np.concatenate([[top], mids[first:first + 31]]) * 2.0 ** e / factor
                    near = t.astype(np.float32)
                    for _ in range(abs(step)):
                        near = np.nextafter(near, np.float32(np.inf if step > 0 else 0))
                    groups.append(near)
    w = torch.from_numpy(np.concatenate(groups)[:32768]).cuda()
    width = len(w) // 32 * 32
    w = w[:width].contiguous()
    g = torch.Generator().manual_seed(1)
    x = (torch.randint(0, 2, (6, width), generator=g) * 2 - 1).to(_t(dtype)).cuda()
    y = octo.Mx8.empty(6, width)
    octo.op_norm(x, y, w, eps=eps)
    # eps as the call takes it
    _same_codes(y, _reference(x, None, w, float(np.float32(eps)))[1])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,width", [(300, 4096), (50, 1001), (3, 32767), (200, 40)])
def test_plain_rows_are_rounded_once(octo, dtype, n, width):
    import torch
    g = torch.Generator().manual_seed(width)
    x, r = (torch.randn(n, width, generator=g).to(_t(dtype)).cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(width, generator=g)).cuda()
    y, total = torch.empty_like(x), torch.empty_like(x)
    octo.op_norm(x, y, w, res=r, total=total, eps=1e-5)
    s, ref = _reference(x, r, w, float(np.float32(1e-5)))
    rel, absolute = STEP[dtype]
    assert np.all(np.abs(_np(y) - ref) <= (rel + (2.0 ** -45 if dtype == "f32" else 3.02 * 2.0 ** -24)) * np.abs(ref) + absolute)
    assert torch.equal(total, torch.from_numpy(s.astype(np.float32)).to(_t(dtype)).cuda())
