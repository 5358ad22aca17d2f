"""octo_op_product on the GPU against the definition in 64 bits.

Bounds.  A sum of k products that are exact (16 and 8 bits) or rounded once (fp32) takes k additions in the matrix units, in an order and with an internal rounding or truncation that are
theirs: each is off by at most 2^-23 of what has been added up so far, at most the sum of |x w|, so (k + 1) 2^-23 sum |x w| in all (twice that with rounded products), and one rounding for the bias.
Activations have slopes of at most 1.13.  SiLU: its exponent is rounded (2^-24 of up to 1.45 |v|), exponential, sum, reciprocal and product are within 2^-23 each: (|v| + 6) 2^-23 of the result.
GELU: erf within 2^-21, a product and a sum: |v| 2^-20 absolutely.  A gate multiplies errors by the other half's size; the residual's sum is one rounding; then one rounding to the type.  All
of these are small beside the type's rounding for 16 bits.

Rows of 8 bits whose results are of 16 or 8 bits are multiplied by the 8-bit instructions where tokens are many (kernels 1 to 4).  Those add products in groups of eight aligned to the
largest, 2^E <= its size, and drop what lies below 2^(E - 13) (1 + 2^-13 comes out as it is, 1 + 2^-14 as 1; the largest has six bits of fraction and loses none): up to seven
products of a group lose less than 2^-13 of its largest, so a sum loses less than 7 * 2^-13 sum |x w|."""
import math

import numpy as np
import pytest

from oracle import answer

pytestmark = pytest.mark.gpu
STEP = {"f32": (2.0 ** -24, 0.0), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 0.0)}
E23 = 2.0 ** -23


def _t(dtype):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def _act(name, v):
    import torch
    if name == "relu":
        return torch.relu(v), torch.zeros_like(v)
    if name == "silu":
        y = v * torch.sigmoid(v)
        return y, (v.abs() + 6) * E23 * y.abs()
    if name == "gelu":
        return 0.5 * v * torch.special.erfc(-v * math.sqrt(0.5)), v.abs() * 8 * E23
    return v, torch.zeros_like(v)


GRAIN = 7 * 2.0 ** -13


def _reference(x, w, bias, act, gated, res, rounded_products, grain=0.0):
    """(y, how far fp32 may be off it) in float64 on the device."""
    z, size = x @ w.T, x.abs() @ w.abs().T
    off = size * ((x.shape[1] + 1) * E23 * (2 if rounded_products else 1) + grain)
    if bias is not None:
        z = z + bias
        off = off + z.abs() * E23
    cols = z.shape[1] // 2 if gated else z.shape[1]
    y, more = _act(act, z[:, :cols])
    off_y = 1.13 * off[:, :cols] + more
    if gated:
        u, off_u = z[:, cols:], off[:, cols:]
        off_y = off_y * (u.abs() + off_u) + y.abs() * off_u
        y = y * u
        off_y = off_y + y.abs() * E23
    if res is not None:
        y = y + res
        off_y = off_y + y.abs() * E23
    return y, off_y


def _check(got, y, off, dtype):
    import torch
    rel, absolute = STEP[dtype]
    err, bound = (got.double() - y).abs(), rel * (y.abs() + off) + absolute + off
    assert bool((err <= bound).all()), (float((err - bound).max()), torch.nonzero(err > bound)[:4].tolist(), torch.nonzero(~torch.isfinite(got))[:4].tolist())


def _check_mx8(y8, y, off):
    """What the eight bits hold is y up to half a step of its group and fp32's error."""
    import torch
    codes, exps = y8.codes.cpu().numpy(), y8.exps.cpu().numpy()
    got = torch.from_numpy(answer.mx8_decode(codes, exps)).cuda()
    scale = torch.from_numpy(np.exp2(exps.astype(np.float64) - 127)).cuda().repeat_interleave(32, 1)
    half = scale * torch.exp2(torch.floor(torch.log2((got.abs() / scale).clamp(min=2.0 ** -6))) - 4)
    err, bound = (got - y).abs(), half * (1 + 2.0 ** -20) + off
    assert bool((err <= bound).all()), (float((err - bound).max()), torch.nonzero(err > bound)[:4].tolist())
    # the exponent is the smallest that holds the group
    most = (y.abs() + off).unflatten(1, (-1, 32)).amax(-1)
    assert bool((most >= 224 * scale[:, ::32])[torch.from_numpy(exps > 1).cuda()].all())


def _mx8(octo, x):
    """(Mx8, its values in float64)."""
    import torch
    codes, exps = octo.quantize_mx8(x.float().cpu().numpy())
    held = octo.Mx8(torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda())
    return held, torch.from_numpy(answer.mx8_decode(codes, exps)).cuda()


def _inputs(octo, rows, dtype, n, k, cols, gated, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    wide = cols * (2 if gated else 1)
    x, w = torch.randn(n, k, generator=g), torch.randn(wide, k, generator=g) / math.sqrt(k)
    if rows == "mx8":
        (x8, x), (w8, w) = _mx8(octo, x), _mx8(octo, w)
        return x8, w8, x, w, g
    x, w = x.to(_t(dtype)).cuda(), w.to(_t(dtype)).cuda()
    return x, w, x.double(), w.double(), g


# tokens, k, outputs: one of each, one more and one less than blocks of 16, 32, 64, 128 and 256, rows that end inside a step, more steps than are in flight
SIZES = [(1, 32, 1), (1, 64, 64), (3, 32, 5), (2, 4096, 40), (16, 96, 32), (17, 160, 100), (31, 256, 33), (33, 1184, 127), (64, 128, 129), (65, 384, 64), (100, 32, 300), (129, 2080, 66), (7, 8224, 96),
         (308, 1184, 1100)]


@pytest.mark.parametrize("rows,dtype", [("plain", "bf16"), ("plain", "f16"), ("plain", "f32"), ("mx8", "bf16"), ("mx8", "f16"), ("mx8", "f32")])
@pytest.mark.parametrize("n,k,cols", SIZES)
@pytest.mark.parametrize("act,gated,bias,with_res,out", [("none", False, False, False, "same"), ("silu", True, True, True, "same"), ("gelu", False, True, True, "f32")])
def test_product(octo, rows, dtype, n, k, cols, act, gated, bias, with_res, out):
    import torch
    x, w, x64, w64, g = _inputs(octo, rows, dtype, n, k, cols, gated, n * 7 + k + cols)
    kind = "f32" if out == "f32" else dtype
    b = torch.randn(w64.shape[0], generator=g).cuda() if bias else None
    res = torch.randn(n, cols, generator=g).to(_t(kind)).cuda() if with_res else None
    y = torch.full((n, cols), float("nan"), dtype=_t(kind), device="cuda")
    kernel = octo.op_product(x, w, y, bias=b, act=act, gated=gated, res=res)
    assert kernel > 0
    ref, off = _reference(x64, w64, None if b is None else b.double(), act, gated, None if res is None else res.double(), rows == "plain" and dtype == "f32",
                          GRAIN if rows == "mx8" and kind != "f32" and kernel < 10 else 0.0)
    _check(y, ref, off, kind)


@pytest.mark.parametrize("rows,dtype", [("plain", "bf16"), ("plain", "f16"), ("plain", "f32"), ("mx8", "bf16")])
@pytest.mark.parametrize("n,k,cols", [(1, 32, 32), (5, 96, 64), (16, 4096, 96), (40, 288, 160), (130, 512, 128), (700, 1184, 1120)])
@pytest.mark.parametrize("act,gated", [("relu", False), ("silu", True)])
def test_product_to_eight_bits(octo, rows, dtype, n, k, cols, act, gated):
    x, w, x64, w64, _ = _inputs(octo, rows, dtype, n, k, cols, gated, n + k)
    y = octo.Mx8.empty(n, cols)
    y.codes.fill_(0x55)
    y.exps.fill_(0x55)
    kernel = octo.op_product(x, w, y, act=act, gated=gated)
    ref, off = _reference(x64, w64, None, act, gated, None, rows == "plain" and dtype == "f32", GRAIN if rows == "mx8" and kernel < 10 else 0.0)
    _check_mx8(y, ref, off)


@pytest.mark.parametrize("rows,dtype", [("plain", "bf16"), ("plain", "f16"), ("plain", "f32"), ("mx8", "bf16")])
@pytest.mark.parametrize("n,k,cols,gated", [(4100, 192, 4099, False), (4100, 192, 2080, True), (1100, 160, 7300, False), (2049, 96, 2050, False), (1030, 128, 1290, True)])
def test_large_products(octo, rows, dtype, n, k, cols, gated):
    """Enough blocks for the larger tiles, with ragged ends on both sides."""
    import torch
    x, w, x64, w64, g = _inputs(octo, rows, dtype, n, k, cols, gated, n)
    y = torch.full((n, cols), float("nan"), dtype=_t(dtype), device="cuda")
    res = torch.randn(n, cols, generator=g).to(_t(dtype)).cuda()
    kernel = octo.op_product(x, w, y, act="silu" if gated else "none", gated=gated, res=res)
    assert 0 < kernel < 10
    ref, off = _reference(x64, w64, None, "silu" if gated else "none", gated, res.double(), rows == "plain" and dtype == "f32", GRAIN if rows == "mx8" else 0.0)
    _check(y, ref, off, dtype)


HELD = [("plain", t, size, n) for t in ("bf16", "f16", "f32") for size, n in ((128, 16), (4096, 1), (4224, 16), (8192, 16), (8320, 5), (16384, 16), (16512, 2))]
HELD += [("mx8", "bf16", size, n) for size, n in ((128, 16), (4096, 16), (4224, 3), (8320, 5))]


@pytest.mark.parametrize("rows,dtype,bytes_of_k,n", HELD)
def test_held_tokens_and_more_weights_than_blocks(octo, rows, dtype, bytes_of_k, n):
    """Several groups of weights to a block, the last of them ragged, at and beyond the longest rows that are held."""
    import torch
    k = bytes_of_k // (1 if rows == "mx8" else _t(dtype).itemsize)
    for cols, gated, to8 in ((4230, False, False), (8300, False, False), (4230, True, False), (8352, False, True), (8352, True, True)):
        x, w, x64, w64, g = _inputs(octo, rows, dtype, n, k, cols, gated, n + k)
        y = octo.Mx8.empty(n, cols) if to8 else torch.full((n, cols), float("nan"), dtype=_t(dtype), device="cuda")
        kernel = octo.op_product(x, w, y, act="silu" if gated else "none", gated=gated)
        r = 4 if gated and to8 else 2 if gated or to8 or bytes_of_k <= 4096 and cols >= 8192 else 1
        room = (4 if rows == "mx8" else 8) if r == 4 else 8 if rows == "mx8" else 16
        assert (kernel == 10 * r) == (bytes_of_k <= 1024 * room), kernel
        ref, off = _reference(x64, w64, None, "silu" if gated else "none", gated, None, rows == "plain" and dtype == "f32")
        _check_mx8(y, ref, off) if to8 else _check(y, ref, off, dtype)


@pytest.mark.parametrize("n,k,cols,gated,to8,kernel", [(60, 100, 600, False, False, 22), (500, 260, 1030, False, False, 44), (130, 1028, 1504, True, True, 44), (70, 64, 96, True, True, 42), (1000, 36, 2100, False, False, 4)])
def test_fp32_in_blocks_of_every_size(octo, n, k, cols, gated, to8, kernel):
    import torch
    x, w, x64, w64, g = _inputs(octo, "plain", "f32", n, k, cols, gated, n)
    y = octo.Mx8.empty(n, cols) if to8 else torch.full((n, cols), float("nan"), device="cuda")
    assert octo.op_product(x, w, y, act="silu" if gated else "none", gated=gated) == kernel
    ref, off = _reference(x64, w64, None, "silu" if gated else "none", gated, None, True)
    _check_mx8(y, ref, off) if to8 else _check(y, ref, off, "f32")


@pytest.mark.parametrize("n,k,cols,gated,to8,kernel", [(60, 1120, 500, False, False, 11), (40, 2048, 2000, False, False, 21), (90, 1184, 600, True, False, 21), (20, 160, 640, False, True, 21),
                                                       (300, 288, 2000, False, False, 41), (70, 96, 320, True, True, 41), (90, 1024, 2016, True, True, 3), (1200, 96, 2060, False, False, 4)])
def test_rows_of_eight_bits_in_every_kernel(octo, n, k, cols, gated, to8, kernel):
    import torch
    x, w, x64, w64, g = _inputs(octo, "mx8", "bf16", n, k, cols, gated, n)
    y = octo.Mx8.empty(n, cols) if to8 else torch.full((n, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert octo.op_product(x, w, y, act="silu" if gated else "none", gated=gated) == kernel
    ref, off = _reference(x64, w64, None, "silu" if gated else "none", gated, None, False, GRAIN if kernel < 10 else 0.0)
    _check_mx8(y, ref, off) if to8 else _check(y, ref, off, "bf16")


def test_fp32_results_of_many_rows_in_eight_bits(octo):
    """They are added up in fp32, whichever kernel runs."""
    import torch
    for n, k, cols in ((2050, 544, 2060), (300, 256, 3300)):
        x, w, x64, w64, _ = _inputs(octo, "mx8", "bf16", n, k, cols, False, n)
        y = torch.full((n, cols), float("nan"), device="cuda")
        assert octo.op_product(x, w, y) in (2, 3)
        ref, off = _reference(x64, w64, None, "none", False, None, False)
        _check(y, ref, off, "f32")


@pytest.mark.parametrize("n", [4, 70, 600])
def test_strides_in_place_and_addresses(octo, n):
    """Rows of wider tensors, results over the residual at addresses and strides that no vector divides; what lies beside them stays."""
    import torch
    g = torch.Generator().manual_seed(n)
    k, cols = 136, 203
    xs, ws = torch.randn(n, 200, generator=g).bfloat16().cuda(), torch.randn(cols, 144, generator=g).bfloat16().cuda()
    flat = torch.randn(n * 211 + 8, generator=g).bfloat16().cuda()
    before = flat.clone()
    for offset in (0, 1, 3):
        flat.copy_(before)
        y = flat[offset:offset + n * 211].view(n, 211)[:, :cols]
        ref, off = _reference(xs[:, 64:64 + k].double(), ws[:, :k].double(), None, "none", False, y.double(), False)
        octo.op_product(xs[:, 64:64 + k], ws[:, :k], y, res=y)
        _check(y, ref, off, "bf16")
        mine = torch.zeros_like(flat, dtype=torch.bool)
        mine[offset:offset + n * 211].view(n, 211)[:, :cols] = True
        assert torch.equal(flat[~mine], before[~mine])
    # a bias at an address that no vector divides, and one row of weights for all (stride 0)
    b = torch.randn(cols + 1, generator=g).cuda()[1:]
    y = torch.empty(n, cols, dtype=torch.bfloat16, device="cuda")
    w = ws[:1, :k].expand(cols, k)
    octo.op_product(xs[:, :k], w, y, bias=b)
    ref, off = _reference(xs[:, :k].double(), w.double(), b.double(), "none", False, None, False)
    _check(y, ref, off, "bf16")


@pytest.mark.parametrize("n", [5, 90])
def test_exponents_at_any_address(octo, n):
    """Exponents of rows that are slices: their words are not aligned, and what lies behind the row's end is not read as one (it would be NaN)."""
    import torch
    g = torch.Generator().manual_seed(n)
    for k in (128, 160, 288):
        pair = []
        for rows in (n, 77):
            codes, exps = octo.quantize_mx8(torch.randn(rows, k, generator=g).numpy())
            c = torch.full((rows, k + 32), 0x7F, dtype=torch.uint8, device="cuda")
            e = torch.full((rows, k // 32 + 3), 255, dtype=torch.uint8, device="cuda")
            c[:, :k], e[:, 1:1 + k // 32] = torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda()
            pair.append((octo.Mx8(c[:, :k], e[:, 1:1 + k // 32]), torch.from_numpy(answer.mx8_decode(codes, exps)).cuda()))
        y = torch.empty(n, 77, dtype=torch.float32, device="cuda")
        octo.op_product(pair[0][0], pair[1][0], y)
        ref, off = _reference(pair[0][1], pair[1][1], None, "none", False, None, False)
        _check(y, ref, off, "f32")


@pytest.mark.parametrize("rows", ["plain", "mx8"])
@pytest.mark.parametrize("n", [9, 150, 4200])
def test_numbers_that_are_none_stay_in_their_rows(octo, rows, n):
    import torch
    k, cols = 96, 4160 if n > 4000 else 70
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(n, k, generator=g), torch.randn(cols, k, generator=g)
    x[1, 40], x[n - 1, 95], w[3, 2] = float("nan"), float("inf"), float("nan")
    if rows == "mx8":
        x, w = (octo.Mx8(*(torch.from_numpy(a).cuda() for a in octo.quantize_mx8(v.numpy()))) for v in (x, w))
    else:
        x, w = x.bfloat16().cuda(), w.bfloat16().cuda()
    y = torch.empty(n, cols, dtype=torch.bfloat16, device="cuda")
    octo.op_product(x, w, y)
    sick = torch.zeros(n, cols, dtype=torch.bool, device="cuda")
    sick[1] = sick[n - 1] = True
    sick[:, 3] = True
    assert torch.equal(~torch.isfinite(y), sick)


@pytest.mark.parametrize("n", [20, 300])
def test_a_count_on_the_device_and_another_stream(octo, n):
    import torch
    x, w = torch.randn(n, 64).half().cuda(), torch.randn(96, 64).half().cuda()
    side = torch.cuda.Stream()
    for count in (-1, 0, 1, n // 2, n, n + 5):
        m = max(0, min(count, n))
        y, y8 = torch.full((n, 96), 7.0, dtype=torch.float16, device="cuda"), octo.Mx8.empty(n, 96)
        y8.codes.fill_(3)
        y8.exps.fill_(5)
        d_n = torch.tensor([count], dtype=torch.int32, device="cuda")
        octo.op_product(x, w, y, n=d_n, stream=side)
        octo.op_product(x, w, y8, n=d_n, stream=side)
        side.synchronize()
        ref, off = _reference(x.double(), w.double(), None, "none", False, None, False)
        _check(y[:m], ref[:m], off[:m], "f16")
        _check_mx8(octo.Mx8(y8.codes[:m], y8.exps[:m]), ref[:m], off[:m])
        assert bool((y[m:] == 7).all()) and bool((y8.codes[m:] == 3).all()) and bool((y8.exps[m:] == 5).all())


@pytest.mark.parametrize("rows", ["plain", "mx8"])
def test_counts_around_the_tokens_of_a_first_kernel(octo, rows):
    """17 x 17 of the largest tiles: one round of 15 x 17 and smaller ones for the 360 tokens that are left over."""
    import torch
    n, k, cols = 4200, 64, 4160
    x, w, x64, w64, _ = _inputs(octo, rows, "f16", n, k, cols, False, 5)
    if rows == "mx8":
        x, w = octo.Mx8(torch.cat([x.codes, x.codes], 1), torch.cat([x.exps, x.exps], 1)), octo.Mx8(torch.cat([w.codes, w.codes], 1), torch.cat([w.exps, w.exps], 1))
        x64, w64 = torch.cat([x64, x64], 1), torch.cat([w64, w64], 1)
    ref, off = _reference(x64, w64, None, "none", False, None, False, GRAIN if rows == "mx8" else 0.0)
    for count in (-3, 0, 100, 3839, 3840, 3841, 4199, 4300):
        m = max(0, min(count, n))
        y, y8 = torch.full((n, cols), 7.0, dtype=torch.float16, device="cuda"), octo.Mx8.empty(n, cols)
        y8.codes.fill_(3)
        y8.exps.fill_(5)
        d_n = torch.tensor([count], dtype=torch.int32, device="cuda")
        assert octo.op_product(x, w, y, n=d_n) == octo.op_product(x, w, y8, n=d_n) == 1
        _check(y[:m], ref[:m], off[:m], "f16")
        _check_mx8(octo.Mx8(y8.codes[:m], y8.exps[:m]), ref[:m], off[:m])
        assert bool((y[m:] == 7).all()) and bool((y8.codes[m:] == 3).all()) and bool((y8.exps[m:] == 5).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("cols,width", [(4160, 4160), (4152, 4200), (4155, 4155)])
def test_residual_in_place_over_two_kernels(octo, dtype, cols, width):
    """Outputs that end inside a tile and inside what is asked for of a residual's row, rows further apart than their outputs."""
    import torch
    n, k = 4200, 64
    x, w, x64, w64, g = _inputs(octo, "plain", dtype, n, k, cols, False, cols)
    held = torch.randn(n, width, generator=g).to(_t(dtype)).cuda()
    before, y = held.clone(), held[:, :cols]
    assert octo.op_product(x, w, y, act="relu", res=y) == 1
    ref, off = _reference(x64, w64, None, "relu", False, before[:, :cols].double(), False)
    _check(y, ref, off, dtype)
    assert torch.equal(held[:, cols:], before[:, cols:])


def test_no_tokens_and_types_that_do_not_meet(octo):
    import torch
    w = torch.randn(96, 64, device="cuda")
    assert octo.op_product(torch.empty(0, 64, device="cuda"), w, torch.empty(0, 96, device="cuda")) == 0
    x, y = torch.randn(4, 64, device="cuda"), torch.empty(4, 96, device="cuda")
    for call in (lambda: octo.op_product(x, w.bfloat16(), y), lambda: octo.op_product(x, w, y.half()), lambda: octo.op_product(x[:, :60], w, y), lambda: octo.op_product(x, w, y[:, :95]),
                 lambda: octo.op_product(x, w, y, act="tanh"), lambda: octo.op_product(x, w, y, res=y.half()), lambda: octo.op_product(x, octo.Mx8.empty(96, 64), y),
                 lambda: octo.op_product(x, w, octo.Mx8.empty(4, 96), res=y), lambda: octo.op_product(x.cpu(), w, y), lambda: octo.op_product(x, w[:95], y[:, :47], gated=True),
                 lambda: octo.op_product(x, w, y, bias=y[0, :95])):
        with pytest.raises(octo.OctoError):
            call()


@pytest.mark.parametrize("n", [3, 200])
def test_captured_and_replayed(octo, n):
    import torch
    x, y = torch.zeros(n, 512, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 384, dtype=torch.bfloat16, device="cuda")
    w = torch.randn(768, 512).bfloat16().cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        octo.op_product(x, w, y, act="silu", gated=True)
    for seed in range(3):
        x.copy_(torch.randn(n, 512, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        again = torch.empty_like(y)
        octo.op_product(x, w, again, act="silu", gated=True)
        torch.cuda.synchronize()
        assert torch.equal(y, again)
