"""octo_op_norm and octo_op_mx8_load on the GPU against the 64-bit oracle.

Bounds.  fp32 arithmetic: the residual's sum is one rounding (2^-24 of it; against |x| + |r| where they cancel), the sum of squares of up to 32768 values is added up in 8 to
32 steps a thread, then a tree of up to ten levels and up to 16 wavefronts, each step a rounding of 2^-24: under 80 of them, halved by the root; root, division and two
products are five more (the root and the division within 2^-23 each).  2.7e-6 of the value covers them all.  Then one rounding to the type."""
import numpy as np
import pytest

from oracle import answer

pytestmark = pytest.mark.gpu
STEP = {"f32": (2.0 ** -24, 0.0), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 0.0)}
LOOSE = 80 / 2 * 2.0 ** -24 + 5 * 2.0 ** -24


def _t(dtype):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def _np(x):
    return x.detach().double().cpu().numpy()


def _near(got, ref, size, dtype):
    rel, absolute = STEP[dtype]
    err, bound = np.abs(_np(got) - ref), rel * np.abs(ref) + absolute + LOOSE * size
    assert np.all(err <= bound), (float((err - bound).max()), np.argwhere(err > bound)[:4])


def _near_mx8(codes, exps, ref, size):
    """Codes and exponents stand for ref up to half a step of their group, or the value lies so near a border that fp32 may have taken the next one."""
    codes, exps = codes.cpu().numpy(), exps.cpu().numpy()
    got = answer.mx8_decode(codes, exps)
    best, best_exps = answer.mx8_encode(ref)
    off = exps != best_exps
    most = np.abs(ref).reshape(ref.shape[0], -1, 32).max(-1)
    # another exponent only where the group's largest value is within fp32's error of a border 448 * 2^e
    border = 448.0 * np.exp2(np.minimum(exps, best_exps).astype(np.float64) - 127)
    assert np.all(np.abs(most - border)[off] <= (LOOSE * size.reshape(ref.shape[0], -1, 32).max(-1))[off])
    scale = np.repeat(np.exp2(exps.astype(np.float64) - 127), 32, -1)
    a = np.abs(got) / scale
    half = scale * np.exp2(np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -9))), -6) - 4)      # half the step above a code's value
    assert np.all(np.abs(got - ref) <= half + LOOSE * size)
    same = codes == best
    assert same[~np.repeat(off, 32, -1)].mean() > 0.999 if ref.size > 4000 else True


# rows and widths: one value, one vector, widths that no vector divides, one more and one less than a wavefront's or a block's worth, the widest
PLAIN = [(1, 1), (3, 8), (5, 7), (1, 130), (70, 96), (33, 256), (2, 1095), (9, 1160), (301, 512), (1500, 264), (4, 4104), (3, 8191), (2, 16384), (2, 32768), (1, 32767), (1100, 2048)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,width", PLAIN)
@pytest.mark.parametrize("with_res", [True, False])
def test_norm(octo, dtype, n, width, with_res):
    import torch
    g = torch.Generator().manual_seed(n * 100 + width)
    x, r = (torch.randn(n, width, generator=g).to(_t(dtype)).cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(width, generator=g)).cuda()
    res, total = (r, torch.empty_like(x)) if with_res else (None, None)
    y = torch.full_like(x, float("nan"))
    octo.op_norm(x, y, w, res=res, total=total, eps=1e-5)
    s, ref = answer.norm(_np(x), _np(r) if with_res else None, _np(w), 1e-5)
    size = np.abs(_np(x)) + (np.abs(_np(r)) if with_res else 0)
    factor = np.abs(ref / np.where(s == 0, 1, s))
    _near(y, ref, factor * size, dtype)
    if with_res:
        _near(total, s, size, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,width", [(1, 32), (3, 64), (16, 4096), (7, 1184), (130, 96), (900, 512), (2, 32768), (5, 8224), (40, 2080)])
@pytest.mark.parametrize("with_res", [True, False])
def test_norm_to_eight_bits(octo, dtype, n, width, with_res):
    import torch
    g = torch.Generator().manual_seed(n * 100 + width)
    x, r = ((torch.randn(n, width, generator=g) * torch.exp2(torch.randint(-3, 4, (n, 1), generator=g).float())).to(_t(dtype)).cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(width, generator=g)).cuda()
    y = octo.Mx8.empty(n, width)
    y.codes.fill_(0x55)
    y.exps.fill_(0x55)
    total = torch.empty_like(x) if with_res else None
    octo.op_norm(x, y, w, res=r if with_res else None, total=total)
    s, ref = answer.norm(_np(x), _np(r) if with_res else None, _np(w))
    size = np.abs(_np(x)) + (np.abs(_np(r)) if with_res else 0)
    size = np.abs(ref / np.where(s == 0, 1, s)) * size
    _near_mx8(y.codes, y.exps, ref, size)
    if with_res:
        _near(total, s, np.abs(_np(x)) + np.abs(_np(r)), dtype)
    for kind in ("bf16", "f16", "f32"):
        back = torch.full((n, width), float("nan"), dtype=_t(kind), device="cuda")
        octo.op_mx8_load(y, back)
        held = answer.mx8_decode(y.codes.cpu().numpy(), y.exps.cpu().numpy())
        assert np.array_equal(_np(back), held.astype(np.float32).astype(np.float16).astype(np.float64) if kind == "f16" else held)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_eight_bits_without_a_norm_are_the_hosts(octo, dtype):
    """Conversion alone involves no arithmetic but the rounding: codes and exponents are the host's, at every border."""
    import torch
    rng = np.random.default_rng(4)
    v = answer.e4m3_decode(np.arange(127, dtype=np.uint8))
    mids = ((v[1:] + v[:-1]) / 2).astype(np.float32)
    rows = []
    for top in np.float32([224, 448, np.nextafter(np.float32(448), np.float32(999)), 256, 300, 447]):
        for e in (-100, -20, 0, 7, 100) if dtype != "f16" else (-15, -6, 0, 7):
            near = np.concatenate([mids, np.nextafter(mids, np.float32(0)), np.nextafter(mids, np.float32(999)), -mids[:3]])
            near = np.resize(near, (len(near) + 30) // 31 * 31).reshape(-1, 31)
            rows.append(np.concatenate([near, np.full((len(near), 1), top)], 1) * np.float32(2.0) ** e)
    x = np.concatenate(rows + [np.zeros((1, 32), np.float32), rng.standard_normal((200, 32)).astype(np.float32) * np.exp2(rng.integers(-14, 15, (200, 1))).astype(np.float32)])
    x = torch.from_numpy(x.astype(np.float32)).to(_t(dtype)).cuda()
    x = x[torch.isfinite(x).all(1)].contiguous()
    y = octo.Mx8.empty(*x.shape)
    octo.op_norm(x, y, norm=False)
    codes, exps = octo.quantize_mx8(x.float().cpu().numpy())
    assert np.array_equal(y.exps.cpu().numpy(), exps) and np.array_equal(y.codes.cpu().numpy(), codes)


def test_zeros_and_numbers_that_are_none(octo):
    """A row of zeros stays zeros, a NaN or an infinity stays in its row, and in its group of 32 where there is no norm."""
    import torch
    x = torch.randn(5, 96).cuda()
    x[1] = 0
    x[2, 40] = float("nan")
    x[3, 95] = float("-inf")
    for y in (torch.empty_like(x), octo.Mx8.empty(5, 96)):
        octo.op_norm(x, y, torch.ones(96, device="cuda"))
        out = y if isinstance(y, torch.Tensor) else torch.empty_like(x)
        if out is not y:
            octo.op_mx8_load(y, out)
        assert bool((out[1] == 0).all()) and bool(torch.isnan(out[2]).all()) and bool(torch.isnan(out[3, 95])) and bool(torch.isfinite(out[[0, 4]]).all())
    y, out = octo.Mx8.empty(5, 96), torch.empty_like(x)
    octo.op_norm(x, y, norm=False)
    octo.op_mx8_load(y, out)
    sick = torch.zeros(5, 96, dtype=torch.bool, device="cuda")
    sick[2, 32:64] = sick[3, 64:] = True
    assert torch.equal(torch.isnan(out), sick) and int((y.exps == 255).sum()) == 2
    huge = torch.full((1, 32), torch.finfo(torch.float32).max, device="cuda")
    y, out = octo.Mx8.empty(1, 32), torch.empty_like(huge)
    octo.op_norm(huge, y, norm=False)
    octo.op_mx8_load(y, out)
    assert bool(torch.isinf(out).all()) and int(y.exps[0, 0]) == 247      # it rounds to 256 * 2^120, which 8 bits hold and fp32 does not


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_in_place_and_any_address(octo, dtype):
    """Rows of wider tensors, at addresses and strides that no vector divides; the sum over the residual, the result over x."""
    import torch
    g = torch.Generator().manual_seed(5)
    for offset, stride, width, n in ((0, 512, 256, 40), (1, 301, 299, 40), (8, 264, 256, 7), (3, 97, 97, 300)):
        flat = [torch.randn(n * stride + 16, generator=g).to(_t(dtype)).cuda() for _ in range(2)]
        x, r = (f[offset:offset + n * stride].view(n, stride)[:, :width] for f in flat)
        before = [f.clone() for f in flat]
        s, ref = answer.norm(_np(x), _np(r))
        size = np.abs(_np(x)) + np.abs(_np(r))
        octo.op_norm(x, x, None, res=r, total=r)
        _near(x, ref, np.abs(ref / np.where(s == 0, 1, s)) * size, dtype)
        _near(r, s, size, dtype)
        for f, b in zip(flat, before):
            mine = torch.zeros_like(f, dtype=torch.bool)
            mine[offset:offset + n * stride].view(n, stride)[:, :width] = True
            assert torch.equal(f[~mine], b[~mine])


def test_a_count_on_the_device_another_stream_and_no_rows(octo):
    import torch
    x = torch.randn(50, 160).half().cuda()
    side = torch.cuda.Stream()
    for count in (-3, 0, 1, 33, 50, 99):
        m = max(0, min(count, 50))
        y, y8, back = torch.full_like(x, 7.0), octo.Mx8.empty(50, 160), torch.full_like(x, 7.0)
        y8.codes.fill_(3)
        y8.exps.fill_(5)
        n = torch.tensor([count], dtype=torch.int32, device="cuda")
        octo.op_norm(x, y, n=n, stream=side)
        octo.op_norm(x, y8, n=n, stream=side)
        octo.op_mx8_load(y8, back, n=n, stream=side)
        side.synchronize()
        _near(y[:m], answer.norm(_np(x[:m]))[1], 4.0, "f16")
        assert bool((y[m:] == 7).all()) and bool((back[m:] == 7).all()) and bool((y8.codes[m:] == 3).all()) and bool((y8.exps[m:] == 5).all())
        assert bool((y8.exps[:m] != 5).all())
    empty = torch.empty(0, 160, device="cuda")
    octo.op_norm(empty, empty)


def test_captured_and_replayed(octo):
    import torch
    x, y, total = (torch.zeros(33, 512, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    res = torch.randn(33, 512).bfloat16().cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        octo.op_norm(x, y, res=res, total=total)
    for seed in range(3):
        x.copy_(torch.randn(33, 512, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        y2, total2 = torch.empty_like(y), torch.empty_like(y)
        octo.op_norm(x, y2, res=res, total=total2)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(total, total2)
