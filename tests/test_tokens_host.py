"""The calls on tokens, as far as they need no GPU: the oracle's pins, the host conversion to 4 bits, refusals."""
import ctypes as C

import numpy as np
import pytest

from oracle import tokens
from paper_2502_01277_amd import binding


# ---- the oracle ----
def test_rotation_keeps_lengths_and_depends_on_distances_alone():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 5, 2, 16))
    for pairs in ("split", "interleaved"):
        for ladder in ("axis", "shared"):
            pos = rng.integers(0, 50, (5, 3)).astype(np.int32)
            a = tokens.rotate(q, None, pos, (2, 3, 3), 100.0, pairs, ladder)
            assert np.allclose((a * a).sum(-1), (q * q).sum(-1))
            b = tokens.rotate(k, None, pos + np.int32([4, 1, 7]), (2, 3, 3), 100.0, pairs, ladder)
            a2, b2 = tokens.rotate(q, None, pos + 9, (2, 3, 3), 100.0, pairs, ladder), tokens.rotate(k, None, pos + np.int32([13, 10, 16]), (2, 3, 3), 100.0, pairs, ladder)
            assert np.allclose((a * b).sum(-1), (a2 * b2).sum(-1))


def test_rotation_by_hand():
    x = np.zeros((1, 1, 6))
    x[0, 0] = [1, 2, 3, 4, 5, 6]
    y = tokens.rotate(x, None, np.int32([[2, 3]]), (1, 1), 100.0, "split")
    c, s, c3, s3 = np.cos(2), np.sin(2), np.cos(3), np.sin(3)
    assert np.allclose(y[0, 0], [c - 3 * s, 2 * c3 - 4 * s3, 3 * c + s, 4 * c3 + 2 * s3, 5, 6])
    y = tokens.rotate(x, None, np.int32([[2]]), (2,), 100.0, "interleaved")
    c2, s2 = np.cos(0.2), np.sin(0.2)
    assert np.allclose(y[0, 0], [c - 2 * s, 2 * c + s, 3 * c2 - 4 * s2, 4 * c2 + 3 * s2, 5, 6])


def test_norm_by_hand():
    y = tokens.rotate(np.array([[[3.0, 4.0]]]), np.array([2.0, 0.5]), None, (), 1.0, eps=0.0)
    assert np.allclose(y, [[[6 / np.sqrt(12.5), 2 / np.sqrt(12.5)]]])


def test_attention_by_hand():
    q, k, v = np.ones((2, 2, 1)), np.array([[[0.0]], [[np.log(3.0)]], [[5.0]]]), np.array([[[1.0]], [[5.0]], [[9.0]]])
    out, lse = tokens.attend(q, k, v, [0, 1, 2], [0, 2], [2, 0], 1.0)
    assert np.allclose(out[0], 4.0) and np.allclose(lse[0], np.log(4.0)) and np.all(out[1] == 0) and np.all(np.isneginf(lse[1]))
    out, _ = tokens.attend(q[:1], k, v, [0, 1], [0], [3], 1.0, key_mask=[0, 1, 0])
    assert np.allclose(out, 5.0)


def _awkward(rng):
    """Groups at which the exponent or the rounding can go wrong: middles between values, 7 and its neighbours, zeros, the ends of the range."""
    mids = np.float32([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    base = np.concatenate([mids, np.nextafter(mids, np.float32(0)), np.nextafter(mids, np.float32(9)), np.float32([0, 6, 6.9])])
    rows = []
    for top in np.float32([3.5, np.nextafter(np.float32(3.5), np.float32(9)), 6, 6.5, 7, np.nextafter(np.float32(7), np.float32(9)), 8]):
        for e in (-40, -3, 0, 9, 60):
            rows.append(np.concatenate([base, -base[:7], [top]])[:32] * np.float32(2.0) ** e)
            rows[-1][-1] = top * np.float32(2.0) ** e
    rows.append(np.zeros(32, np.float32))
    rows.append(np.full(32, np.finfo(np.float32).max, np.float32))
    rows += [rng.standard_normal(32).astype(np.float32) * np.float32(2.0) ** int(e) for e in rng.integers(-30, 30, 200)]
    return np.stack(rows).astype(np.float32)


def test_four_bits_on_the_host_are_the_oracles():
    x = _awkward(np.random.default_rng(3))
    codes, exps = binding.quantize_mx4(x)
    ref_codes, ref_exps = tokens.mx4_encode(x.astype(np.float64))
    assert np.array_equal(exps, ref_exps)
    assert np.array_equal(codes, tokens.mx4_pack(ref_codes))
    back = binding.dequantize_mx4(codes, exps)
    assert np.array_equal(back.astype(np.float64), tokens.mx4_decode(ref_codes, ref_exps))
    # nothing is further off than half the widest step, and no group could do with a smaller exponent
    scale = np.exp2(exps.astype(np.float64) - 127)
    most = np.abs(x.astype(np.float64)).max(-1, keepdims=True)
    inside = exps < 252
    assert np.all((np.abs(back - x) <= scale)[inside[:, 0]]) and np.all((most <= 7 * scale)[inside]) and np.all((most > 3.5 * scale)[inside & (exps > 1)])


def test_four_bits_of_what_is_no_number():
    x = np.ones((3, 32), np.float32)
    x[0, 5], x[1, 31] = np.nan, -np.inf
    codes, exps = binding.quantize_mx4(x)
    assert exps[:, 0].tolist() == [255, 255, tokens.mx4_encode(x[2:].astype(np.float64))[1][0, 0]]
    back = binding.dequantize_mx4(codes, exps)
    assert np.isnan(back[:2]).all() and np.all(back[2] == 1)
    every = np.arange(256, dtype=np.uint8)                  # every byte of codes at every exponent
    for e in (1, 100, 127, 128, 252):
        got = binding.dequantize_mx4(every, np.full(16, e, np.uint8))
        assert np.array_equal(got, tokens.mx4_decode(tokens.mx4_unpack(every), np.full(16, e, np.uint8)).astype(np.float32))
    with pytest.raises(binding.OctoError):
        binding.quantize_mx4(np.ones(31, np.float32))


# ---- refusals: before any launch, so they need no GPU ----
def _rotate_op():
    op = binding.OctoRotateOp()
    op.dtype, op.n_tokens, op.dim, op.n_axes, op.n_parts, op.base, op.eps = 2, 4, 64, 2, 1, 100.0, 1e-6
    op.sections[:2] = (12, 20)
    op.d_pos = 4096
    p = op.part[0]
    p.d_x, p.d_y, p.heads, p.x_token, p.x_head, p.y_token, p.y_head = 8192, 16384, 2, 128, 64, 128, 64
    return op


ROTATE_BAD = [("dtype", 3), ("dtype", -1), ("n_tokens", -1), ("dim", 0), ("dim", 63), ("dim", 258), ("n_axes", 5), ("n_axes", -1), ("n_parts", 0), ("n_parts", 3), ("pairs", 2),
              ("ladder", -1), ("base", 0.0), ("base", -2.0), ("base", float("inf")), ("base", float("nan")), ("d_pos", 0), ("d_pos", 4097)]


@pytest.mark.parametrize("field,value", ROTATE_BAD)
def test_rotate_refuses(field, value):
    op = _rotate_op()
    setattr(op, field, value)
    assert binding.lib().octo_op_rotate(C.byref(op), None) == binding.EINVAL


@pytest.mark.parametrize("field,value", [("d_x", 0), ("d_y", 0), ("d_x", 8193), ("heads", 0), ("heads", -3), ("x_token", -1), ("y_head", -64), ("d_weight", 4098)])
def test_rotate_refuses_parts(field, value):
    op = _rotate_op()
    setattr(op.part[0], field, value)
    assert binding.lib().octo_op_rotate(C.byref(op), None) == binding.EINVAL


def test_rotate_refuses_sections_and_takes_nothing():
    L = binding.lib()
    op = _rotate_op()
    op.sections[1] = 21                                      # 33 pairs of 64 elements
    assert L.octo_op_rotate(C.byref(op), None) == binding.EINVAL
    op.sections[1] = -1
    assert L.octo_op_rotate(C.byref(op), None) == binding.EINVAL
    op = _rotate_op()
    op.part[0].d_weight, op.eps = 4096, float("nan")
    assert L.octo_op_rotate(C.byref(op), None) == binding.EINVAL
    op = _rotate_op()
    op.dim, op.part[0].d_x = 256, 8194                       # 128 pairs one by one: more than 64 lanes
    assert L.octo_op_rotate(C.byref(op), None) == binding.EINVAL
    assert L.octo_op_rotate(None, None) == binding.EINVAL
    op = _rotate_op()
    op.n_tokens = 0
    assert L.octo_op_rotate(C.byref(op), None) == binding.OK


def _cache_op():
    op = binding.OctoCache4Op()
    op.dtype, op.n, op.heads, op.dim, op.rows = 2, 3, 2, 64, 10
    for p in (op.k_plane, op.v_plane):
        p.d_codes, p.d_exps, p.code_row, p.code_head, p.exp_row, p.exp_head = 4096, 4097, 32, 320, 2, 20
    op.d_k, op.d_v, op.k_token, op.k_head, op.v_token, op.v_head, op.d_slots = 8192, 16384, 128, 64, 128, 64, 4096
    return op


@pytest.mark.parametrize("field,value", [("dtype", 3), ("n", -1), ("heads", 0), ("dim", 48), ("dim", 160), ("dim", 0), ("rows", 0), ("d_k", 0), ("d_v", 8), ("d_slots", 0), ("d_slots", 4), ("k_token", 4),
                                         ("v_head", -8)])
def test_cache4_refuses(field, value):
    L = binding.lib()
    op = _cache_op()
    setattr(op, field, value)
    assert L.octo_op_cache4_store(C.byref(op), None) == binding.EINVAL
    assert L.octo_op_cache4_load(C.byref(op), None) == binding.EINVAL


@pytest.mark.parametrize("field,value", [("d_codes", 0), ("d_codes", 4100), ("d_exps", 0), ("code_row", 8), ("code_head", -16), ("exp_row", -1)])
def test_cache4_refuses_planes(field, value):
    op = _cache_op()
    setattr(op.v_plane, field, value)
    assert binding.lib().octo_op_cache4_store(C.byref(op), None) == binding.EINVAL


def test_cache4_takes_nothing_and_refuses_too_much():
    L = binding.lib()
    op = _cache_op()
    op.n = 0
    assert L.octo_op_cache4_store(C.byref(op), None) == binding.OK and L.octo_op_cache4_load(C.byref(op), None) == binding.OK
    op.n, op.heads = 0x7FFFFFFF, 64                          # beyond 32-bit thread numbers
    assert L.octo_op_cache4_store(C.byref(op), None) == binding.EINVAL
    assert L.octo_op_cache4_store(None, None) == binding.EINVAL


def _attend_op(fmt=0):
    op = binding.OctoAttendOp()
    op.dtype, op.kv_format, op.dim, op.q_heads, op.kv_heads, op.n_seq, op.n_q, op.max_q, op.max_kv, op.scale, op.kv_rows = 2, fmt, 64, 8, 2, 3, 9, 4, 50, 0.1, 100
    op.d_q, op.q_row, op.q_head, op.d_out, op.out_row, op.out_head = 4096, 512, 64, 8192, 512, 64
    op.d_k, op.d_v, op.k_row, op.k_head, op.v_row, op.v_head = 4096, 4096, 128, 64, 128, 64
    for p in (op.k_plane, op.v_plane):
        p.d_codes, p.d_exps, p.code_row, p.code_head, p.exp_row, p.exp_head = 4096, 4097, 32, 3200, 2, 200
    op.d_q_start, op.d_kv_start, op.d_kv_len = 4096, 4096, 4096
    return op


ATTEND_BAD = [("dtype", 3), ("dtype", -1), ("kv_format", 2), ("dim", 60), ("dim", 136), ("dim", 0), ("q_heads", 7), ("q_heads", 0), ("kv_heads", 0), ("kv_heads", 16), ("n_seq", -1), ("n_q", -1), ("max_q", 10),
              ("max_q", -1), ("max_kv", -1), ("scale", 0.0), ("scale", -1.0), ("scale", float("inf")), ("kv_rows", -1), ("d_q", 0), ("d_q", 4098), ("q_row", 4), ("q_head", -64), ("d_out", 0), ("d_out", 4100),
              ("out_row", 12), ("d_q_start", 0), ("d_q_start", 4098), ("d_kv_start", 0), ("d_kv_start", 4100), ("d_kv_len", 0), ("d_lse", 2)]


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("field,value", ATTEND_BAD)
def test_attend_refuses(fmt, field, value):
    op = _attend_op(fmt)
    setattr(op, field, value)
    assert binding.lib().octo_op_attend(C.byref(op), None, None) == binding.EINVAL


@pytest.mark.parametrize("field,value", [("d_k", 0), ("d_v", 4104), ("k_row", 4), ("v_head", -8), ("k_row", 8 << 20), ("v_row", 1 << 40)])
def test_attend_refuses_pools(field, value):
    op = _attend_op()
    setattr(op, field, value)
    assert binding.lib().octo_op_attend(C.byref(op), None, None) == binding.EINVAL


@pytest.mark.parametrize("field,value", [("d_codes", 0), ("d_codes", 4104), ("d_exps", 0), ("code_row", 24), ("code_head", -16), ("exp_row", -2), ("code_row", 16 << 20), ("exp_row", 16 << 20)])
def test_attend_refuses_planes(field, value):
    op = _attend_op(1)
    setattr(op.k_plane, field, value)
    assert binding.lib().octo_op_attend(C.byref(op), None, None) == binding.EINVAL


def test_attend_refuses_fp32_on_four_bits_and_takes_nothing():
    L = binding.lib()
    op = _attend_op(1)
    op.dtype = 0
    assert L.octo_op_attend(C.byref(op), None, None) == binding.EINVAL and L.octo_op_attend_workspace_bytes(C.byref(op)) == 0
    kid = C.c_int32(5)
    for name in ("n_seq", "max_q"):
        op = _attend_op()
        setattr(op, name, 0)
        assert L.octo_op_attend(C.byref(op), None, C.byref(kid)) == binding.OK and kid.value == 0
        assert L.octo_op_attend_workspace_bytes(C.byref(op)) == 0
    assert L.octo_op_attend(None, None, None) == binding.EINVAL and L.octo_op_attend_workspace_bytes(None) == 0


def test_packed_arguments_have_the_layout_of_the_structs():
    for packed, cls in ((binding._ROTATE, binding.OctoRotateOp), (binding._CACHE4, binding.OctoCache4Op), (binding._ATTEND, binding.OctoAttendOp)):
        assert packed.size == C.sizeof(cls)
        flat = []

        def walk(kind, at):
            if hasattr(kind, "_fields_"):
                for name, sub in kind._fields_:
                    walk(sub, at + getattr(kind, name).offset)
            elif hasattr(kind, "_length_"):
                for i in range(kind._length_):
                    walk(kind._type_, at + i * C.sizeof(kind._type_))
            else:
                flat.append((at, kind))

        walk(cls, 0)
        for i, (at, kind) in enumerate(flat):                # each field alone at 1
            raw = packed.pack(*[1 if k == i else 0 for k in range(len(flat))])
            assert kind.from_buffer_copy(raw, at).value == 1 and raw.count(0) < len(raw), i
            other = bytearray(raw)
            other[at:at + C.sizeof(kind)] = bytes(C.sizeof(kind))
            assert not any(other), i
