"""The calls around attention, as far as they need no GPU: the oracle's pins, the host's conversion to 8 bits, refusals."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import answer
from paper_2502_01277_amd import binding


# ---- the oracle ----
def test_norm_by_hand():
    s, y = answer.norm(np.array([[1.0, 4.0]]), np.array([[2.0, 0.0]]), np.array([2.0, 0.5]), eps=0.0)
    assert np.allclose(s, [[3, 4]]) and np.allclose(y, [[6 / math.sqrt(12.5), 2 / math.sqrt(12.5)]])
    assert np.allclose(answer.norm(np.array([[3.0, 4.0]]), norm=False)[1], [[3, 4]])


def test_product_by_hand():
    x, w = np.array([[1.0, 2.0]]), np.array([[3.0, 1.0], [0.0, -2.0]])
    assert np.allclose(answer.product(x, w, [0.5, 1.0], "relu", res=[[1.0, 1.0]]), [[6.5, 1.0]])
    assert np.allclose(answer.product(x, w, [0.5, 1.0], "silu", gated=True), [[5.5 / (1 + math.exp(-5.5)) * -3]])
    assert np.allclose(answer.activate("gelu", np.array([1.0])), 0.5 * (1 + math.erf(math.sqrt(0.5))))


def test_sampling_by_hand():
    x = np.log([0.1, 0.4, 0.3, 0.2])
    assert [answer.sample(x, u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.79, 0.81, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert answer.kept_tokens(x, top_k=2)[0] == [1, 2] and answer.kept_tokens(x, top_p=0.69)[0] == [1, 2] and answer.kept_tokens(x, top_p=0.71)[0] == [1, 2, 3]
    assert answer.kept_tokens(x, min_p=0.51)[0] == [1, 2] and answer.kept_tokens(x, top_p=0.0)[0] == [1] and answer.kept_tokens(x, temperature=0.0, top_k=3)[0] == [1]
    # top-p is a share of what top-k left
    assert answer.kept_tokens(x, top_k=2, top_p=0.56)[0] == [1] or math.isclose(0.4 / 0.7, 0.5714, abs_tol=1e-3)
    token, kept, logprob = answer.sample(x, 0.6, top_k=2)
    assert (token, kept) == (2, 2) and math.isclose(logprob, math.log(3 / 7))
    assert answer.sample([-np.inf, np.nan], 0.3) == (-1, 0, -np.inf)
    assert answer.kept_tokens([1.0, 2.0, 2.0, 2.0], top_k=2)[0] == [1, 2]
    assert answer.sample([5.0, np.inf, 3.0], 0.99) == (1, 3, 0.0)


def test_eight_bits_on_the_host_are_the_oracles():
    rng = np.random.default_rng(3)
    v = answer.e4m3_decode(np.arange(127, dtype=np.uint8))
    assert np.all(np.diff(v) > 0) and v[-1] == 448
    mids = ((v[1:] + v[:-1]) / 2).astype(np.float32)
    near = np.concatenate([mids, np.nextafter(mids, np.float32(0)), np.nextafter(mids, np.float32(999)), -mids])
    near = np.resize(near, 31 * 17).reshape(17, 31)
    rows = [np.zeros((1, 32), np.float32), np.full((1, 32), np.finfo(np.float32).max, np.float32), np.full((1, 32), 1e-45, np.float32)]
    for top in np.float32([224, 448, np.nextafter(np.float32(448), np.float32(999)), 256]):
        for e in (-120, -40, 0, 60):
            rows.append(np.concatenate([near, np.full((17, 1), top)], 1).astype(np.float32) * np.float32(2.0) ** e)
    rows.append(rng.standard_normal((300, 32)).astype(np.float32) * np.exp2(rng.integers(-60, 60, (300, 1))).astype(np.float32))
    x = np.concatenate(rows).astype(np.float32)
    codes, exps = binding.quantize_mx8(x)
    ref_codes, ref_exps = answer.mx8_encode(x.astype(np.float64))
    assert np.array_equal(exps, ref_exps) and np.array_equal(codes, ref_codes)
    back = binding.dequantize_mx8(codes, exps)
    assert np.array_equal(back.astype(np.float64), answer.mx8_decode(codes, exps).astype(np.float32).astype(np.float64))
    scale = np.exp2(exps.astype(np.float64) - 127)
    most = np.abs(x.astype(np.float64)).max(-1, keepdims=True)
    assert np.all(most <= 448 * scale) and np.all((most > 224 * scale)[exps > 1])


def test_eight_bits_of_what_is_no_number():
    x = np.ones((3, 32), np.float32)
    x[0, 5], x[1, 31] = np.nan, -np.inf
    codes, exps = binding.quantize_mx8(x)
    assert exps[:2, 0].tolist() == [255, 255] and np.all(codes[:2] == 0x7F)
    back = binding.dequantize_mx8(codes, exps)
    assert np.isnan(back[:2]).all() and np.all(back[2] == 1)
    for bad in (np.ones(31, np.float32), np.float32(1)):
        with pytest.raises(binding.OctoError):
            binding.quantize_mx8(bad)
    with pytest.raises(binding.OctoError):
        binding.dequantize_mx8(np.zeros(33, np.uint8), np.zeros(1, np.uint8))


# ---- what the calls refuse: nothing is launched, so no device is needed ----
def _norm_op(**changes):
    op = binding.OctoNormOp()
    op.dtype, op.y_format, op.n, op.width, op.norm, op.eps = 2, 0, 4, 64, 1, 1e-6
    op.d_x, op.d_y, op.x_row, op.y_row = 4096, 8192, 64, 64
    op.y8.d_codes, op.y8.d_exps, op.y8.code_row, op.y8.exp_row = 16384, 32768, 64, 2
    for name, v in changes.items():
        part = op.y8 if name in ("d_codes", "d_exps", "code_row", "exp_row") else op
        setattr(part, name, v)
    return binding.lib().octo_op_norm(C.byref(op), None)


def test_norm_refuses():
    assert binding.lib().octo_op_norm(None, None) == binding.EINVAL
    assert _norm_op(n=0) == binding.OK and _norm_op(n=0, y_format=1) == binding.OK
    for bad in (dict(dtype=3), dict(dtype=-1), dict(y_format=2), dict(n=-1), dict(width=0), dict(width=32769), dict(d_x=None), dict(d_y=None), dict(eps=-1.0), dict(eps=float("nan")), dict(x_row=-1),
                dict(y_row=-64), dict(d_res=512, res_row=-1), dict(d_sum=512, sum_row=-1), dict(d_sum=8192, sum_row=64), dict(d_x=4097), dict(d_weight=2), dict(d_n=2)):
        assert _norm_op(**bad) == binding.EINVAL, bad
    for bad in (dict(width=48), dict(d_codes=None), dict(d_exps=None), dict(d_codes=8), dict(code_row=72), dict(code_row=-64), dict(exp_row=-1), dict(x_row=68), dict(d_x=4104), dict(d_res=8, res_row=64),
                dict(d_sum=512, sum_row=65)):
        assert _norm_op(y_format=1, **bad) == binding.EINVAL, bad
    assert _norm_op(n=0, norm=0, eps=-1.0) == binding.OK


def _mx8_op(**changes):
    op = binding.OctoMx8Op()
    op.dtype, op.n, op.width, op.d_y, op.y_row = 2, 4, 64, 4096, 64
    op.x8.d_codes, op.x8.d_exps, op.x8.code_row, op.x8.exp_row = 16384, 32768, 64, 2
    for name, v in changes.items():
        part = op.x8 if name in ("d_codes", "d_exps", "code_row", "exp_row") else op
        setattr(part, name, v)
    return binding.lib().octo_op_mx8_load(C.byref(op), None)


def test_mx8_load_refuses():
    assert binding.lib().octo_op_mx8_load(None, None) == binding.EINVAL
    assert _mx8_op(n=0) == binding.OK
    for bad in (dict(dtype=3), dict(n=-1), dict(width=0), dict(width=40), dict(d_y=None), dict(d_y=4104), dict(y_row=65), dict(y_row=-64), dict(d_codes=None), dict(code_row=65), dict(exp_row=-2),
                dict(n=1 << 30, width=32768)):
        assert _mx8_op(**bad) == binding.EINVAL, bad


def test_layouts_of_the_packed_calls():
    assert binding._NORM.size == C.sizeof(binding.OctoNormOp) and binding._MX8.size == C.sizeof(binding.OctoMx8Op)


def _product_op(**changes):
    op = binding.OctoProductOp()
    op.dtype, op.x_format, op.y_format, op.n, op.k, op.cols = 2, 0, 0, 4, 64, 96
    op.d_x, op.d_w, op.x_row, op.w_row, op.d_y, op.y_row, op.res_row = 4096, 8192, 64, 64, 65536, 96, 96
    for rows, at in ((op.x8, 1), (op.w8, 2), (op.y8, 3)):
        rows.d_codes, rows.d_exps, rows.code_row, rows.exp_row = at << 20, (at << 20) + 65536, 96, 3
    for name, v in changes.items():
        part = op
        for p in name.split("__")[:-1]:
            part = getattr(part, p)
        setattr(part, name.split("__")[-1], v)
    kid = C.c_int32(7)
    st = binding.lib().octo_op_product(C.byref(op), None, C.byref(kid))
    assert kid.value == 0
    return st


def test_product_refuses():
    assert binding.lib().octo_op_product(None, None, None) == binding.EINVAL
    assert _product_op(n=0) == binding.OK and _product_op(n=0, x_format=1, y_format=1) == binding.OK and _product_op(n=0, gated=1, act=3, d_res=512) == binding.OK
    for bad in (dict(dtype=3), dict(dtype=-1), dict(x_format=2), dict(y_format=-1), dict(n=-1), dict(k=0), dict(cols=0), dict(cols=0x20000001), dict(act=4), dict(act=-1), dict(d_x=None), dict(d_w=None),
                dict(d_x=4104), dict(d_w=8200), dict(k=60), dict(k=2147483640), dict(k=(1 << 29) + 8), dict(x_row=60), dict(w_row=-8), dict(x_row=(8 << 20) // 2 + 8), dict(w_row=1 << 60), dict(d_y=None), dict(d_y=65537), dict(y_row=-1),
                dict(d_res=1), dict(d_res=512, res_row=-1), dict(d_bias=2), dict(d_n=2), dict(out_f32=1, d_y=65538)):
        assert _product_op(**bad) == binding.EINVAL, bad
    for bad in (dict(k=48), dict(k=(1 << 30) + 32), dict(x8__d_codes=None), dict(w8__d_exps=None), dict(x8__d_codes=8), dict(w8__code_row=72), dict(x8__code_row=-96), dict(w8__exp_row=-1), dict(x8__code_row=(8 << 20) + 16),
                dict(x8__exp_row=1 << 40)):
        assert _product_op(x_format=1, **bad) == binding.EINVAL, bad
    for bad in (dict(cols=100), dict(out_f32=1), dict(d_res=512), dict(y8__d_codes=None), dict(y8__code_row=100), dict(y8__exp_row=-1)):
        assert _product_op(y_format=1, **bad) == binding.EINVAL, bad
    assert _product_op(n=0x7FFFFFFF, cols=0x20000000) == binding.EINVAL       # more blocks than a launch takes


def test_layout_of_the_packed_product():
    assert binding._PRODUCT.size == C.sizeof(binding.OctoProductOp)


def _sample_op(**changes):
    op = binding.OctoSampleOp()
    op.dtype, op.n, op.vocab, op.d_logits, op.row, op.d_u, op.d_token = 2, 4, 100, 4096, 100, 8192, 16384
    op.temperature, op.top_p = 1.0, 1.0
    for name, v in changes.items():
        setattr(op, name, v)
    return binding.lib().octo_op_sample(C.byref(op), None)


def test_sample_refuses():
    assert binding.lib().octo_op_sample(None, None) == binding.EINVAL
    assert _sample_op(n=0) == binding.OK and _sample_op(n=0, d_logits=4098, row=0) == binding.OK
    for bad in (dict(dtype=3), dict(n=-1), dict(n=1 << 22), dict(vocab=0), dict(vocab=(1 << 19) + 1), dict(d_logits=None), dict(d_logits=4097), dict(dtype=0, d_logits=4098), dict(row=-1), dict(d_u=None),
                dict(d_token=None), dict(d_u=8194), dict(d_token=2), dict(d_temperature=1), dict(d_top_k=2), dict(d_top_p=3), dict(d_min_p=2), dict(d_logprob=1), dict(d_kept=2), dict(d_n=2)):
        assert _sample_op(**bad) == binding.EINVAL, bad


def test_workspace_of_a_sample():
    """Only few long rows of fp32 and fp16 have one, and not where the host knows that a short list is enough."""
    need = binding.lib().octo_op_sample_workspace_bytes
    op = binding.OctoSampleOp(dtype=0, n=4, vocab=70000)
    size = need(C.byref(op))
    assert size > 0 and size == 4 * need(C.byref(binding.OctoSampleOp(dtype=0, n=1, vocab=70000))) == need(C.byref(binding.OctoSampleOp(dtype=1, n=4, vocab=70000)))
    for none in (dict(dtype=2), dict(n=0), dict(n=65), dict(n=-1), dict(vocab=65535), dict(vocab=(1 << 19) + 1), dict(top_k=512), dict(dtype=3)):
        assert need(C.byref(binding.OctoSampleOp(**{**dict(dtype=0, n=4, vocab=70000), **none}))) == 0, none
    assert need(None) == 0 and need(C.byref(binding.OctoSampleOp(dtype=0, n=4, vocab=70000, top_k=512, d_top_k=4096))) == size
    long = dict(dtype=0, vocab=70000, row=70000)
    for bad in (dict(d_workspace=4096, workspace_bytes=size - 1), dict(d_workspace=4104, workspace_bytes=size)):
        assert _sample_op(**long, **bad) == binding.EINVAL, bad


def test_layout_of_the_packed_sample():
    assert binding._SAMPLE.size == C.sizeof(binding.OctoSampleOp)
