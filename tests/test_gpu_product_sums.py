"""Sums of rows in 8 bits on the GPU: in fp32 whichever kernel runs, those of the 8-bit matrix instructions only where the caller permits them.

Bounds are those of test_gpu_product: products of such rows are exact, a sum of k of them is off by (k + 1) 2^-23 of the sum of their sizes, then the result's rounding.  With fast8, 7 * 2^-13 of the sum
of the sizes more."""
import pytest

from test_gpu_product import GRAIN, _check, _check_mx8, _inputs, _reference, _t

pytestmark = pytest.mark.gpu

# tokens, k, outputs and the tile kernel that they take: the widest k of a step and several of them, ragged on both sides
TILES = [(4200, 128, 4160, 1), (4100, 896, 4128, 1), (2100, 384, 2080, 2), (129, 1024, 4096, 3), (70, 1152, 8224, 3), (1200, 256, 2080, 4)]


def _result(octo, out, n, cols):
    import torch
    return octo.Mx8.empty(n, cols) if out == "mx8" else torch.full((n, cols), float("nan"), dtype=_t(out), device="cuda")


@pytest.mark.parametrize("n,k,cols,kernel", TILES)
@pytest.mark.parametrize("out", ["bf16", "f16", "mx8"])
@pytest.mark.parametrize("fast8", [False, True])
def test_what_cancels_leaves_the_small_products(octo, n, k, cols, kernel, out, fast8):
    """Every four products hold one 2^14 times larger than the others, and those cancel each other in every eight."""
    import torch
    g = torch.Generator().manual_seed(n + k)
    x = torch.randint(8, 16, (n, k), generator=g).float() * 2.0 ** -9
    w = torch.randint(1, 3, (cols, k), generator=g).float() / 2
    x[:, ::4], w[:, ::8], w[:, 4::8] = 256.0, 1.0, -1.0
    x8, w8 = (octo.Mx8(*(torch.from_numpy(a).cuda() for a in octo.quantize_mx8(v.numpy()))) for v in (x, w))
    y = _result(octo, out, n, cols)
    assert octo.op_product(x8, w8, y, fast8=fast8) == kernel
    ref, off = _reference(x.double().cuda(), w.double().cuda(), None, "none", False, None, False, GRAIN if fast8 else 0.0)
    if not fast8:
        # An instruction adds 32 products, four of them 256, to a sum of small ones (all positive, up to ref): no partial sum is larger than 1024 + ref, and each addition is off by 2^-23 of it.
        off = (k + 1) * 2.0 ** -23 * (1024 + ref)
        assert float((off / ref).max()) < 0.1                      # well below what the small products come to
    _check_mx8(y, ref, off) if out == "mx8" else _check(y, ref, off, out)


@pytest.mark.parametrize("n,k,cols,kernel", TILES)
@pytest.mark.parametrize("out,act,gated,more", [("bf16", "none", False, True), ("f16", "silu", True, False), ("f16", "gelu", False, True), ("mx8", "silu", True, False), ("mx8", "relu", False, False)])
@pytest.mark.parametrize("fast8", [False, True])
def test_every_tile_and_epilogue(octo, n, k, cols, kernel, out, act, gated, more, fast8):
    import torch
    cols = cols // 64 * 32 if gated else cols
    x, w, x64, w64, g = _inputs(octo, "mx8", "bf16", n, k, cols, gated, n + cols)
    y = _result(octo, out, n, cols)
    b = torch.randn(w64.shape[0], generator=g).cuda() if more else None
    res = torch.randn(n, cols, generator=g).to(_t(out)).cuda() if more else None
    assert octo.op_product(x, w, y, bias=b, act=act, gated=gated, res=res, fast8=fast8) == kernel
    ref, off = _reference(x64, w64, None if b is None else b.double(), act, gated, None if res is None else res.double(), False, GRAIN if fast8 else 0.0)
    _check_mx8(y, ref, off) if out == "mx8" else _check(y, ref, off, out)


@pytest.mark.parametrize("n,k,cols,words", [(4200, 128, 4160, True), (2100, 384, 2080, True), (4200, 160, 4160, False), (300, 288, 3300, False)])
def test_what_is_in_fp32_with_fast8_too(octo, n, k, cols, words):
    """Results in fp32, and rows whose exponents are no aligned words: the same bits with and without."""
    import torch
    x, w, x64, w64, _ = _inputs(octo, "mx8", "bf16", n, k, cols, False, n)
    for out in ("f32",) if words else ("f32", "bf16"):
        y, fast = _result(octo, out, n, cols), _result(octo, out, n, cols)
        assert octo.op_product(x, w, y) == octo.op_product(x, w, fast, fast8=True)
        ref, off = _reference(x64, w64, None, "none", False, None, False)
        _check(y, ref, off, out)
        assert torch.equal(y, fast)


@pytest.mark.parametrize("n", [9, 60, 1200])
def test_the_same_bits_from_every_call(octo, n):
    import torch
    x, w, _, _, _ = _inputs(octo, "mx8", "bf16", n, 1024, 2080, False, n)
    first = _result(octo, "bf16", n, 2080)
    octo.op_product(x, w, first)
    for _ in range(4):
        y = _result(octo, "bf16", n, 2080)
        octo.op_product(x, w, y)
        assert torch.equal(y, first)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,k,cols,gated", [(308, 1160, 1100, False), (1000, 904, 470, False), (120, 72, 2300, False), (700, 1160, 700, False), (90, 800, 1495, True), (65, 1272, 4001, False)])
def test_short_rows_in_larger_blocks(octo, dtype, n, k, cols, gated):
    """Operands from memory, 64 tokens a block, where results would leave tiles through LDS."""
    x, w, x64, w64, g = _inputs(octo, "plain", dtype, n, k, cols, gated, n + k)
    import torch
    b, res = torch.randn(w64.shape[0], generator=g).cuda(), torch.randn(n, cols, generator=g).to(_t(dtype)).cuda()
    y = _result(octo, dtype, n, cols)
    assert octo.op_product(x, w, y, bias=b, act="gelu", gated=gated, res=res) == 24
    ref, off = _reference(x64, w64, b.double(), "gelu", gated, res.double(), False)
    _check(y, ref, off, dtype)


@pytest.mark.parametrize("rows,dtype", [("plain", "bf16"), ("plain", "f16"), ("plain", "f32"), ("mx8", "bf16")])
@pytest.mark.parametrize("n,k,cols", [(5, 1184, 96), (40, 1184, 96), (308, 1184, 1120), (300, 2048, 1120), (1200, 256, 2080), (2100, 384, 2080), (4200, 128, 4160)])
@pytest.mark.parametrize("gated,bias", [(False, True), (True, False), (True, True)])
def test_gelu_to_eight_bits(octo, rows, dtype, n, k, cols, gated, bias):
    """Groups of 32 outputs that leave tiles through LDS, and those of every other kernel."""
    import torch
    x, w, x64, w64, g = _inputs(octo, rows, dtype, n, k, cols, gated, n + k)
    b = torch.randn(w64.shape[0], generator=g).cuda() if bias else None
    y = octo.Mx8.empty(n, cols)
    y.codes.fill_(0x55)
    y.exps.fill_(0x55)
    octo.op_product(x, w, y, bias=b, act="gelu", gated=gated)
    ref, off = _reference(x64, w64, None if b is None else b.double(), "gelu", gated, None, rows == "plain" and dtype == "f32")
    _check_mx8(y, ref, off)
