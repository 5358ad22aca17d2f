"""Activations of octo_op_product on the GPU: what is no number, against the definition in 64 bits."""
import math

import pytest

from test_gpu_product import STEP, _t

pytestmark = pytest.mark.gpu


def _activate(act, v):
    import torch
    if act == "relu":
        return torch.where(v < 0, 0.0, v)
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return 0.5 * v * torch.special.erfc(-v * math.sqrt(0.5))
    return v


@pytest.mark.parametrize("rows,dtype", [("plain", "bf16"), ("plain", "f16"), ("plain", "f32"), ("mx8", "bf16")])
@pytest.mark.parametrize("n,cols", [(9, 96), (60, 96), (150, 4128), (4200, 4160)])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
def test_numbers_that_are_none_pass_every_activation(octo, rows, dtype, n, cols, act, gated):
    """NaN in a token, infinity in another (rows of 8 bits: both read as NaN), NaN in weights and in a bias: held tokens, operands from memory and tiles, both ways out of registers, and to 8 bits."""
    import torch
    k = 128
    g = torch.Generator().manual_seed(n)
    wide = cols * (2 if gated else 1)
    x, w = torch.randn(n, k, generator=g), torch.randn(wide, k, generator=g)
    x[1, 40], x[n - 1, 95], w[3, 2] = float("nan"), float("inf"), float("nan")
    b = torch.randn(wide, generator=g)
    b[7] = float("nan")
    if rows == "mx8":
        x64, w64 = x.double(), w.double()
        x64[n - 1, 64:96] = float("nan")
        x, w = (octo.Mx8(*(torch.from_numpy(a).cuda() for a in octo.quantize_mx8(v.numpy()))) for v in (x, w))
    else:
        x, w = x.to(_t(dtype)).cuda(), w.to(_t(dtype)).cuda()
        x64, w64 = x.double(), w.double()
    b = b.cuda()
    z = x64.cuda() @ w64.cuda().T + b.double()
    ref = _activate(act, z[:, :cols])
    if gated:
        ref = ref * z[:, cols:]
    nan = torch.isnan(ref)
    assert bool(nan[:, 3].all()) and bool(nan[1].all()) and bool(nan[:, 7].all())
    # rows whose addresses no vector divides leave the tiles through LDS
    odd = torch.empty(n * (cols + 1) + 1, dtype=_t(dtype), device="cuda")[1:1 + n * (cols + 1)].view(n, cols + 1)[:, :cols]
    for y in (torch.empty(n, cols, dtype=_t(dtype), device="cuda"), odd, torch.empty(n, cols, device="cuda")):
        octo.op_product(x, w, y, bias=b, act=act, gated=gated)
        assert torch.equal(torch.isnan(y), nan)
        assert torch.equal(torch.isinf(y), torch.isinf(ref))
    y8 = octo.Mx8.empty(n, cols)
    octo.op_product(x, w, y8, bias=b, act=act, gated=gated)
    sick = (~torch.isfinite(ref)).unflatten(1, (-1, 32)).any(-1)
    assert torch.equal(y8.exps == 255, sick)
    assert bool((y8.codes.unflatten(1, (-1, 32))[sick] == 0x7F).all())
    if rows == "mx8":
        y = torch.empty(n, cols, dtype=_t(dtype), device="cuda")
        octo.op_product(x, w, y, bias=b, act=act, gated=gated, fast8=True)
        assert torch.equal(torch.isnan(y), nan)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,cols", [(14, 96), (60, 96), (300, 4128), (4200, 4160)])
@pytest.mark.parametrize("gated", [False, True])
def test_gelu_of_negative_values(octo, dtype, n, cols, gated):
    """Its error is relative, also where the result is a millionth of the argument.  y = v/2 erfc(t), t = -v / sqrt 2, with v exact: t is off by 2^-23 of itself (the constant and the product), which erfc,
    whose logarithm has slopes up to 2 t + 1.13, makes (v^2 + 0.8 |v|) 2^-23; erfc itself is within 4 of its last bits, at most 2^-21; two products are 2^-24 each, and a gate is one more: (v^2 + |v| + 6) 2^-23 in
    all, then the type's rounding."""
    import torch
    v = torch.linspace(-12.0, 4.0, n).to(_t(dtype)).cuda()
    x = torch.zeros(n, 32, dtype=_t(dtype), device="cuda")
    x[:, 5] = v
    w = torch.ones(cols * (2 if gated else 1), 32, dtype=_t(dtype), device="cuda")
    v = v.double()
    ref = (_activate("gelu", v) * (v if gated else 1.0))[:, None].expand(n, cols)
    off = ref.abs() * (v * v + v.abs() + 6)[:, None] * 2.0 ** -23
    for kind in {dtype, "f32"}:
        y = torch.full((n, cols), float("nan"), dtype=_t(kind), device="cuda")
        octo.op_product(x, w, y, act="gelu", gated=gated)
        rel, absolute = STEP[kind]
        assert bool(((y.double() - ref).abs() <= off + rel * (ref.abs() + off) + absolute).all())
