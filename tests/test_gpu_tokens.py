"""Rotations, norms and the cache of 4 bits on the GPU against the 64-bit oracle.

Bounds.  An output is one rounding to its type (at most 2^-8 of the value in bf16, 2^-11 in fp16 and half its smallest step, 2^-24 in
fp32) of fp32 arithmetic: angle, sine and cosine are off by at most 4e-7 (fraction of a revolution rounded to fp32: 2 pi 2^-25;
the instructions: 1.3e-7), the norm's sum of up to 256 squares in a tree by less than 30 roundings, so 2e-6 of the two elements that are turned covers them.
What 4 bits hold is exact."""
import numpy as np
import pytest

from oracle import tokens

pytestmark = pytest.mark.gpu
STEP = {"f32": (2.0 ** -24, 0.0), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 0.0)}


def _types():
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _np(x):
    return x.detach().double().cpu().numpy()


def _check_rotation(got, x, weight, pos, sections, base, pairs, ladder, eps, dtype):
    ref = tokens.rotate(_np(x), None if weight is None else _np(weight), pos, sections, base, pairs, ladder, eps)
    u = tokens.rotate(_np(x), None if weight is None else _np(weight), pos, (), base, eps=eps)
    big = np.abs(u)
    total = sum(sections)
    for p in range(total):
        i, k = (p, p + total) if pairs == "split" else (2 * p, 2 * p + 1)
        big[..., i] = big[..., k] = np.abs(u[..., i]) + np.abs(u[..., k])
    rel, absolute = STEP[dtype]
    err = np.abs(_np(got) - ref)
    bound = rel * np.abs(ref) + absolute + 2e-6 * big
    assert np.all(err <= bound), (float((err - bound).max()), np.argwhere(err > bound)[:4])


# tokens, heads of the two tensors, dim, sections: vectors of 8, 4, 2 and 1 values, axes of no pairs, heads that fill a wavefront's step or not
SHAPES = [(1, (1, 0), 64, (32,)), (16, (32, 8), 128, (64,)), (97, (3, 2), 128, (16, 24, 24)), (33, (5, 1), 80, (10, 15, 15)), (29, (7, 7), 72, (9, 13, 14)), (300, (8, 8), 64, (16, 16)),
          (5, (2, 3), 36, (4, 0, 6)), (7, (1, 1), 6, (3,)), (9, (4, 0), 2, (1,)), (11, (3, 0), 256, (32, 40, 24, 32)), (13, (2, 2), 96, (8, 8)), (4, (70, 3), 128, (64,)), (1031, (9, 2), 64, (8, 12, 12))]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%d_%d_%d_%d" % (s[0], *s[1], s[2]))
@pytest.mark.parametrize("pairs,ladder,norm", [("split", "axis", True), ("interleaved", "axis", False), ("split", "shared", False), ("interleaved", "shared", True)])
def test_rotation(octo, dtype, shape, pairs, ladder, norm):
    import torch
    n, heads, dim, sections = shape
    g = torch.Generator().manual_seed(n * 1000 + dim)
    t = _types()[dtype]
    pos = torch.randint(-7, 70000, (n, len(sections)), generator=g, dtype=torch.int32)
    parts, xs = [], []
    for h in [h for h in heads if h]:
        x = torch.randn(n, h, dim, generator=g).to(t).cuda()
        w = (1 + 0.3 * torch.randn(dim, generator=g)).cuda() if norm else None
        xs.append((x, w))
        parts.append(octo.RotatePart(x, torch.full_like(x, float("nan")), w))
    octo.op_rotate(parts, pos.cuda(), sections, base=10000.0, pairs=pairs, ladder=ladder, eps=1e-5)
    for p, (x, w) in zip(parts, xs):
        _check_rotation(p.y, x, w, pos.numpy(), sections, 10000.0, pairs, ladder, 1e-5, dtype)


@pytest.mark.parametrize("offset", [0, 1, 2, 4])
def test_rotation_of_slices_in_place_and_with_one_norm(octo, offset):
    """Queries and keys as one projection writes them, at addresses that allow vectors of 8, 1, 2 and 4 values; only the keys have a norm; the values stay."""
    import torch
    n, hq, hk, dim = 37, 6, 2, 64
    flat = torch.randn(n * (hq + 2 * hk) * dim + 8, generator=torch.Generator().manual_seed(offset)).to(torch.bfloat16).cuda()
    fused = flat[offset:offset + n * (hq + 2 * hk) * dim].view(n, hq + 2 * hk, dim)
    before = fused.clone()
    w = torch.linspace(0.5, 1.5, dim).cuda()
    pos = torch.arange(2 * n, dtype=torch.int32).view(n, 2)
    q, k = fused[:, :hq], fused[:, hq:hq + hk]
    octo.op_rotate([octo.RotatePart(q, q), octo.RotatePart(k, k, w)], pos.cuda(), (16, 16))
    _check_rotation(q, before[:, :hq], None, pos.numpy(), (16, 16), 10000.0, "split", "axis", 1e-6, "bf16")
    _check_rotation(k, before[:, hq:hq + hk], w, pos.numpy(), (16, 16), 10000.0, "split", "axis", 1e-6, "bf16")
    assert torch.equal(fused[:, hq + hk:], before[:, hq + hk:])


def test_rotation_with_a_count_on_the_device_and_on_another_stream(octo):
    import torch
    n, dim = 50, 128
    x = torch.randn(n, 3, dim).half().cuda()
    pos = torch.arange(n, dtype=torch.int32)[:, None]
    side = torch.cuda.Stream()
    for count in (0, 1, 33, 50, 99):
        y = torch.full_like(x, 7.0)
        octo.op_rotate([octo.RotatePart(x, y)], pos.cuda(), (64,), n=torch.tensor([count], dtype=torch.int32, device="cuda"), stream=side)
        side.synchronize()
        m = min(count, n)
        _check_rotation(y[:m], x[:m], None, pos[:m].numpy(), (64,), 10000.0, "split", "axis", 1e-6, "f16")
        assert bool((y[m:] == 7).all())


def test_norm_without_rotation_zeros_and_numbers_that_are_none(octo):
    """A head of zeros stays zeros, a NaN or an infinity stays in its head."""
    import torch
    x = torch.randn(4, 9, 80).cuda()
    x[1, 2] = 0
    x[2, 3, 5] = float("nan")
    x[3, 8, 1] = float("inf")
    w = torch.ones(80, device="cuda")
    y = torch.empty_like(x)
    octo.op_rotate([octo.RotatePart(x, y, w)], None, ())
    ref = tokens.rotate(_np(x), np.ones(80), None, (), 1.0)
    assert bool((y[1, 2] == 0).all())
    sick = np.zeros((4, 9), bool)
    sick[2, 3] = sick[3, 8] = True
    assert np.isnan(_np(y)[2, 3]).all() and np.isnan(_np(y)[3, 8]).any()
    assert np.abs(_np(y) - ref)[~sick].max() < 1e-5
    empty = torch.empty(0, 9, 80, device="cuda")
    octo.op_rotate([octo.RotatePart(empty, empty.clone())], torch.empty(0, 1, dtype=torch.int32, device="cuda"), (40,))


def test_positions_far_into_a_text_lose_nothing(octo):
    """At position 2^31 - 1 the angle of the first pair is a number of whole turns that fp32 cannot tell from its neighbours."""
    import torch
    pos = torch.tensor([[2147483647], [-2147483648], [1000003]], dtype=torch.int32)
    x = torch.ones(3, 1, 8).cuda()
    y = torch.empty_like(x)
    octo.op_rotate([octo.RotatePart(x, y)], pos.cuda(), (4,), base=500000.0)
    _check_rotation(y, x, None, pos.numpy(), (4,), 500000.0, "split", "axis", 1e-6, "f32")


# ---- the cache of 4 bits ----
def _values(rng, n, heads, dim, dtype):
    import torch
    x = rng.standard_normal((n, heads, dim)) * np.exp2(rng.integers(-9, 9, (n, heads, 1)))
    g = x.reshape(n, heads, -1, 32)
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 7.0])
    g[::2, :, :, :10] = mids * 2.0 ** rng.integers(-6, 6, g[::2, :, :, :1].shape)       # middles between two codes
    g[::2, :, :, 10:] *= 0.01
    if n > 2:
        x[2] = 0
    return torch.from_numpy(x).to(_types()[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,heads,dim,rows", [(1, 1, 32, 1), (5, 3, 64, 40), (33, 8, 128, 64), (70, 2, 96, 71), (257, 5, 128, 999)])
def test_store_and_load(octo, dtype, n, heads, dim, rows):
    import torch
    rng = np.random.default_rng(n)
    k, v = _values(rng, n, heads, dim, dtype), _values(rng, n, heads, dim, dtype)
    slots = torch.from_numpy(rng.permutation(rows)[:n].astype(np.int64)).cuda()
    cache = octo.Cache4.zeros(heads, rows, dim)
    for x in (cache.k_codes, cache.k_exps, cache.v_codes, cache.v_exps):
        x.fill_(0xA5)
    octo.op_cache4_store(cache, k, v, slots)
    at = slots.cpu().numpy()
    rest = np.setdiff1d(np.arange(rows), at)
    held = []
    for x, codes, exps in ((k, cache.k_codes, cache.k_exps), (v, cache.v_codes, cache.v_exps)):
        ref_codes, ref_exps = tokens.mx4_encode(_np(x), 140 if dtype == "f16" else 252)
        c, e = codes.cpu().numpy().transpose(1, 0, 2), exps.cpu().numpy().transpose(1, 0, 2)
        assert np.array_equal(e[at], ref_exps) and np.array_equal(c[at], tokens.mx4_pack(ref_codes))
        assert np.all(c[rest] == 0xA5) and np.all(e[rest] == 0xA5)
        held.append(tokens.mx4_decode(ref_codes, ref_exps))
    k2, v2 = torch.full_like(k, 3), torch.full_like(v, 3)
    octo.op_cache4_load(cache, slots, k2, v2)
    assert np.array_equal(_np(k2), held[0]) and np.array_equal(_np(v2), held[1])


def test_store_skips_slots_outside_and_follows_strides_and_counts(octo):
    import torch
    rng = np.random.default_rng(8)
    heads, rows, dim = 2, 12, 64
    fused = _values(rng, 6, 3 * heads, dim, "bf16")
    k, v = fused[:, heads:2 * heads], fused[:, 2 * heads:]
    slots = torch.tensor([3, -1, 11, 12, 2 ** 40, 0], device="cuda")
    # rows outermost, heads inside, as a pool of whole tokens
    wide = [torch.full((rows, heads, dim // d), 0x11, dtype=torch.uint8, device="cuda") for d in (2, 32, 2, 32)]
    cache = octo.Cache4(*[w.transpose(0, 1) for w in wide])
    octo.op_cache4_store(cache, k, v, slots, n=torch.tensor([5], dtype=torch.int32, device="cuda"), stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    codes, exps = tokens.mx4_encode(_np(k))
    got = wide[0].cpu().numpy()
    assert np.array_equal(got[[3, 11]], tokens.mx4_pack(codes)[[0, 2]]) and np.all(got[[0, 1, 2, 4, 5, 6, 7, 8, 9, 10]] == 0x11)
    assert np.array_equal(wide[1].cpu().numpy()[[3, 11]], exps[[0, 2]])
    k2, v2 = torch.full((6, heads, dim), 5.0, device="cuda"), torch.full((6, heads, dim), 5.0, device="cuda")
    octo.op_cache4_load(cache, slots, k2, v2, n=torch.tensor([5], dtype=torch.int32, device="cuda"))
    ref = tokens.mx4_decode(*tokens.mx4_encode(_np(v)))
    assert np.array_equal(_np(v2)[[0, 2]], ref[[0, 2]]) and bool((v2[[1, 3, 4]] == 0).all()) and bool((v2[5] == 5).all())


def test_groups_of_numbers_that_are_none_read_as_such(octo):
    import torch
    x = torch.ones(3, 1, 64, device="cuda")
    x[0, 0, 40], x[1, 0, 3] = float("nan"), float("-inf")
    cache = octo.Cache4.zeros(1, 3, 64)
    slots = torch.arange(3, device="cuda")
    octo.op_cache4_store(cache, x, x, slots)
    for dtype in _types().values():
        k, v = torch.empty(3, 1, 64, dtype=dtype, device="cuda"), torch.empty(3, 1, 64, dtype=dtype, device="cuda")
        octo.op_cache4_load(cache, slots, k, v)
        want = np.ones((3, 1, 64))
        want[0, 0, 32:] = want[1, 0, :32] = np.nan
        assert np.array_equal(_np(k), want, equal_nan=True) and np.array_equal(_np(v), want, equal_nan=True)


def test_the_largest_fp16_values_stay_finite(octo):
    import torch
    x = torch.full((1, 1, 32), 65504.0, dtype=torch.float16, device="cuda")
    cache = octo.Cache4.zeros(1, 1, 32)
    octo.op_cache4_store(cache, x, -x, torch.zeros(1, dtype=torch.int64, device="cuda"))
    k, v = torch.empty_like(x), torch.empty_like(x)
    octo.op_cache4_load(cache, torch.zeros(1, dtype=torch.int64, device="cuda"), k, v)
    assert bool((k == 49152).all()) and bool((v == -49152).all())


def test_cache4_binding_refuses(octo):
    import torch
    cache = octo.Cache4.zeros(2, 4, 64)
    k = torch.zeros(3, 2, 64, device="cuda")
    slots = torch.arange(3, device="cuda")
    for bad in (dict(k=k.to(torch.float64), v=k.to(torch.float64)), dict(k=k[:, :1], v=k[:, :1]), dict(k=k, v=k[:2]), dict(k=k, v=k, slots=slots.int()), dict(k=k, v=k, slots=slots[:2])):
        with pytest.raises(octo.OctoError):
            octo.op_cache4_store(cache, bad["k"], bad["v"], bad.get("slots", slots))
    with pytest.raises(octo.OctoError):
        octo.op_rotate([octo.RotatePart(k, k)], torch.zeros(3, 2, device="cuda"), (16, 16))         # positions that are no integers
    with pytest.raises(octo.OctoError):
        octo.op_rotate([octo.RotatePart(k, k.transpose(0, 1))], torch.zeros(3, 1, dtype=torch.int32, device="cuda"), (16,))
