"""Attention to ragged keys on the GPU against the 64-bit oracle.

Bounds.  With w the weights (sum 1) and E = 2^-8 (bf16), 2^-11 (fp16), 2^-24 (fp32) the largest rounding to the type:
  - a score is off by at most d = (dim + 8) 2^-24 scale sum |q| |k| of its key, so the weights by 2 d (their own and their sum's);
  - a weight is rounded once (E), in fp16 also by half its smallest step, 2^-25, where the largest weight is at least 1;
  - exponential and sums in fp32: at most (keys / 8 + 64) 2^-24;
  - nothing is held below the smallest normal number, 2^-126 (weights, values, results);
so |out - ref| <= (E + 2 d + (keys / 8 + 64) 2^-24) sum w |v| + E |ref| (+ fp16: 2^-24 (1 + sum |v| / sum exp(s - max))) + 2^-126 (1 + sum |v|), and
|lse - ref| <= d + (keys / 8 + 64) 2^-24 + 2^-22 (1 + |ref|)."""
import ctypes as C

import numpy as np
import pytest

from oracle import tokens

pytestmark = pytest.mark.gpu
E = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _types():
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _np(x):
    return x.detach().double().cpu().numpy()


class Problem:
    """Sequences with given lengths in a pool whose other rows, and whose hidden ones, hold NaN."""

    def __init__(self, octo, dtype, fmt, dim, kv_heads, group, q_len, kv_len, mask=None, seed=0, loud=1.0, gap=3):
        import torch
        rng = np.random.default_rng(seed)
        t = _types()[dtype]
        self.dtype, self.scale = dtype, dim ** -0.5
        n = len(q_len)
        self.q_start = np.concatenate([[gap], gap + np.cumsum(q_len)]).astype(np.int32)
        order, at, self.kv_start = rng.permutation(n), gap, np.zeros(n, np.int64)
        for b in order:
            self.kv_start[b] = at
            at += kv_len[b] + gap
        self.rows, self.kv_len = at, np.asarray(kv_len, np.int32)
        self.used = np.zeros(self.rows, bool)
        for b in range(n):
            self.used[self.kv_start[b]:self.kv_start[b] + kv_len[b]] = True
        self.mask = None
        if mask is not None:
            self.mask = (rng.random(self.rows) < mask).astype(np.uint8) * rng.integers(1, 256, self.rows).astype(np.uint8)
            if n > 1:
                self.mask[self.kv_start[0]:self.kv_start[0] + kv_len[0]] = 0        # the first sequence sees nothing
            self.used &= self.mask != 0
        n_q = int(self.q_start[-1]) + gap
        as_t = lambda x: torch.from_numpy(x).to(t).cuda()  # noqa: E731
        self.q = as_t(rng.standard_normal((n_q, kv_heads * group, dim)) * loud)
        k, v = rng.standard_normal((2, self.rows, kv_heads, dim)) * np.exp2(rng.integers(-2, 3, (2, 1, kv_heads, dim)))
        if fmt == "cache4":
            planes, self.kv = [], []
            for x in (k, v):
                codes, exps = tokens.mx4_encode(x.transpose(1, 0, 2))
                self.kv.append(tokens.mx4_decode(codes, exps).transpose(1, 0, 2))
                exps[:, ~self.used] = 255
                planes += [torch.from_numpy(tokens.mx4_pack(codes)).cuda(), torch.from_numpy(exps).cuda()]
            self.held = octo.Cache4(*planes)
        else:
            kt, vt = as_t(k), as_t(v)
            self.kv = [_np(kt), _np(vt)]
            sick = torch.from_numpy(~self.used).cuda()
            kt[sick], vt[sick] = float("nan"), float("nan")
            self.held = (kt, vt)
        self.out = torch.full((n_q, kv_heads * group, dim), 7.0, dtype=t, device="cuda")
        self.lse = torch.full((n_q, kv_heads * group), 7.0, device="cuda")
        self.dev = [torch.from_numpy(x).cuda() for x in (self.q_start, self.kv_start, self.kv_len)]
        self.dmask = None if self.mask is None else torch.from_numpy(self.mask).cuda()

    def run(self, octo, **kw):
        kw = dict(dict(max_q=int(np.diff(self.q_start).max()), max_kv=int(self.kv_len.max()), key_mask=self.dmask, lse=self.lse), **kw)
        return octo.op_attend(self.q, self.held, self.out, *self.dev, **kw)

    def check(self, sequences=None):
        q, (k, v) = _np(self.q), self.kv
        n = len(self.kv_len) if sequences is None else sequences
        ref, lse = tokens.attend(q, k, v, self.q_start[:n + 1], self.kv_start[:n], self.kv_len[:n], self.scale, self.mask)
        out, got_lse = _np(self.out), _np(self.lse)
        asked = np.zeros(len(q), bool)
        asked[self.q_start[0]:self.q_start[n]] = True
        assert np.all(out[~asked] == 7) and np.all(got_lse[~asked] == 7)
        group, dim, e = q.shape[1] // k.shape[1], q.shape[2], E[self.dtype]
        for b in range(n):
            rows = np.arange(self.kv_start[b], self.kv_start[b] + self.kv_len[b])
            rows = rows[self.used[rows]]
            lo, hi = self.q_start[b], self.q_start[b + 1]
            if not len(rows):
                assert np.all(out[lo:hi] == 0) and np.all(np.isneginf(got_lse[lo:hi])), b
                continue
            if lo == hi:
                continue
            for h in range(q.shape[1]):
                kk, vv = k[rows, h // group], v[rows, h // group]
                s = q[lo:hi, h] @ kk.T * self.scale
                d = (dim + 8) * 2.0 ** -24 * self.scale * (np.abs(q[lo:hi, h]) @ np.abs(kk).T).max(-1, keepdims=True)
                w = np.exp(s - lse[lo:hi, h, None])
                tiny = 2.0 ** -126 * (1 + np.abs(vv).sum(0))
                bound = (e + 2 * d + (len(rows) / 8 + 64) * 2.0 ** -24) * (w @ np.abs(vv)) + e * np.abs(ref[lo:hi, h]) + tiny
                if self.dtype == "f16":
                    bound = bound + 2.0 ** -24 * (1 + np.abs(vv).sum(0) / np.exp(s - s.max(-1, keepdims=True)).sum(-1, keepdims=True))
                err = np.abs(out[lo:hi, h] - ref[lo:hi, h])
                assert np.all(err <= bound), (b, h, float((err - bound).max()), float(bound.max()))
                off = np.abs(got_lse[lo:hi, h] - lse[lo:hi, h])
                assert np.all(off <= d[:, 0] + (len(rows) / 8 + 64) * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(lse[lo:hi, h]))), (b, h)


FORMS = [("bf16", "plain"), ("f16", "plain"), ("f32", "plain"), ("bf16", "cache4"), ("f16", "cache4")]
forms = pytest.mark.parametrize("dtype,fmt", FORMS, ids=lambda x: x)


@forms
@pytest.mark.parametrize("dim", [8, 32, 56, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("mask", [None, 0.6], ids=["all", "mask"])
def test_single_tokens(octo, dtype, fmt, dim, mask):
    if fmt == "cache4" and dim % 32:
        pytest.skip("the cache holds groups of 32")
    p = Problem(octo, dtype, fmt, dim, 2, 4, [1] * 9, [40, 0, 1, 31, 32, 33, 127, 128, 261], mask, seed=dim)
    assert p.run(octo)
    p.check()


@forms
@pytest.mark.parametrize("dim,kv_heads,group", [(64, 3, 1), (128, 1, 8), (96, 2, 5), (72, 2, 3)])
@pytest.mark.parametrize("mask", [None, 0.5], ids=["all", "mask"])
def test_questions_of_many_lengths(octo, dtype, fmt, dim, kv_heads, group, mask):
    if fmt == "cache4" and dim % 32:
        pytest.skip("the cache holds groups of 32")
    p = Problem(octo, dtype, fmt, dim, kv_heads, group, [5, 0, 1, 33, 16, 70], [65, 50, 300, 1, 96, 129], mask, seed=dim + group)
    assert p.run(octo)
    p.check()


SHORT, EDGES = [20, 3, 17, 16, 1, 0, 32, 31], [49, 0, 1, 33, 64, 65, 31, 96]
# every kernel on every type and format where there is one (the number of sequences and the keys decide): dim, key heads, group, queries, keys, kernel
KERNELS = [
    # a wavefront has rows of its own
    ("bf16", "plain", 128, 8, 1, SHORT * 8, EDGES * 8, 2), ("f16", "plain", 72, 8, 1, SHORT * 8, EDGES * 8, 2), ("f32", "plain", 64, 8, 1, SHORT * 8, EDGES * 8, 2), ("f32", "plain", 128, 8, 1, SHORT * 8, EDGES * 8, 2),
    ("bf16", "cache4", 128, 8, 1, SHORT * 8, EDGES * 8, 2), ("f16", "cache4", 64, 8, 1, SHORT * 8, EDGES * 8, 2),
    # 128 rows and tiles of 64 keys in LDS
    ("bf16", "plain", 128, 3, 1, [129, 1, 128, 33, 0, 97], [3000, 63, 1, 64, 65, 193], 3), ("f16", "plain", 64, 3, 1, [129, 1, 128, 33, 0, 97], [3000, 128, 0, 64, 65, 191], 3),
    ("bf16", "plain", 80, 2, 5, [26, 7, 1, 30, 5, 2], [3500, 64, 65, 1, 0, 640], 3), ("f16", "plain", 96, 1, 8, [40, 33, 3, 16], [4500, 31, 127, 129], 3), ("bf16", "plain", 24, 4, 2, [70, 5, 66], [3000, 64, 65], 3),
    ("bf16", "cache4", 128, 4, 1, [70, 64, 1, 49] * 16, [40, 64, 1, 65] * 16, 3), ("f16", "cache4", 64, 4, 1, [70, 64, 1, 49] * 16, [40, 64, 1, 130] * 16, 3), ("f16", "cache4", 96, 4, 1, [70, 64, 1, 49] * 16, [40, 0, 1, 63] * 16, 3),
    ("bf16", "cache4", 32, 4, 1, [70, 64, 1, 49] * 16, [40, 64, 1, 65] * 16, 3),
    # the same, with parts cut by the lengths on the device
    ("bf16", "plain", 128, 3, 1, [129, 1, 128, 33, 0, 97], [22000, 63, 1, 64, 65, 193], 5), ("f16", "plain", 64, 4, 5, [1, 30, 0, 26, 13], [0, 33100, 64, 30000, 127], 5),
    ("bf16", "cache4", 96, 3, 1, [1, 129, 128, 33, 0, 97], [0, 22000, 1, 6400, 65, 193], 5),
    ("f16", "cache4", 128, 3, 1, [1, 129, 128, 33, 0, 97], [0, 22000, 1, 6400, 65, 12289], 5), ("bf16", "cache4", 64, 2, 3, [40, 90, 7, 1, 43, 0, 90, 3, 50, 88], [25000, 1, 63, 64, 65, 9, 24999, 128, 2000, 0], 5),
    # 32 rows share their keys
    ("bf16", "plain", 128, 3, 1, [70, 33, 0, 48, 17, 1], [1500, 33, 9, 129, 1, 0], 4), ("f16", "plain", 64, 3, 2, [35, 16, 9, 1], [2500, 400, 31, 128], 4), ("f16", "plain", 88, 3, 1, [70, 33, 0, 48, 17, 1], [1500, 33, 9, 129, 1, 64], 4),
    ("f32", "plain", 64, 3, 1, [90, 33, 0, 48, 17, 1], [3700, 33, 9, 129, 1, 0], 4), ("f32", "plain", 96, 3, 1, [90, 33, 1], [7400, 64, 129], 4), ("f32", "plain", 128, 3, 1, [90, 33, 1], [7400, 65, 129], 4),
    ("bf16", "cache4", 128, 3, 1, [70, 33, 0, 48, 17, 1], [11600, 33, 9, 129, 1, 0], 4), ("f16", "cache4", 64, 3, 1, [70, 33, 0, 48, 17, 1], [11600, 33, 9, 129, 1, 64], 4),
    # 16 rows, tiles of rows of several blocks
    ("bf16", "plain", 96, 3, 1, [70, 33, 0, 48], [300, 33, 9, 129], 1), ("f32", "plain", 80, 3, 2, [35, 16, 9, 1], [300, 64, 31, 0], 1), ("f16", "cache4", 128, 3, 1, [70, 33, 0, 48], [900, 33, 9, 129], 1),
]


@pytest.mark.parametrize("mask", [None, 0.7], ids=["all", "mask"])
@pytest.mark.parametrize("case", KERNELS, ids=lambda c: "%s_%s_%d_k%d" % (c[0], c[1], c[2], c[7]))
def test_every_kernel_at_its_edges(octo, case, mask):
    dtype, fmt, dim, kv_heads, group, q_len, kv_len, kernel = case
    p = Problem(octo, dtype, fmt, dim, kv_heads, group, q_len, kv_len, mask, seed=dim)
    kid = p.run(octo)
    if octo.device_cu_count() == 256:
        assert kid // 1000 == kernel, kid
    p.check()


@forms
def test_one_long_sequence_is_split(octo, dtype, fmt):
    """Few rows and many keys: several parts, whose number depends on the GPU but not on the result."""
    p = Problem(octo, dtype, fmt, 128, 2, 4, [1, 2], [5000, 3301], 0.9, seed=4)
    assert p.run(octo) % 1000 > 1
    p.check()
    first = p.out.clone(), p.lse.clone()
    p.out.fill_(7)
    p.run(octo)
    import torch
    assert torch.equal(p.out, first[0]) and torch.equal(p.lse, first[1])


@forms
def test_sharp_and_growing_scores(octo, dtype, fmt):
    """Scores of hundreds, so that almost all weight is on single keys and the reference moves often."""
    p = Problem(octo, dtype, fmt, 64, 2, 2, [3, 40], [700, 333], seed=9, loud=60.0)
    if fmt == "plain":
        grow = np.linspace(0.01, 1.0, p.rows)[:, None, None]
        import torch
        k = torch.from_numpy(p.kv[0] * grow).to(p.q.dtype).cuda()
        p.held, p.kv[0] = (k, p.held[1]), _np(k)
        p.held[0][torch.from_numpy(~p.used).cuda()] = float("nan")
    p.run(octo)
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_infinite_scores_stay_in_their_rows(octo, dtype):
    """A key with an infinity: minus infinity is a weight of 0; plus infinity and NaN make their row NaN, and no other."""
    import torch
    p = Problem(octo, dtype, "plain", 64, 1, 1, [3], [70], seed=2)
    lo = int(p.q_start[0])
    p.q[lo:lo + 3, 0, 0] = torch.tensor([1.0, -1.0, 0.5], dtype=p.q.dtype)
    p.held[0][int(p.kv_start[0]) + 5, 0, 0] = float("-inf")
    p.run(octo)
    out = _np(p.out)
    assert np.isnan(out[lo + 1, 0]).all() and np.isfinite(out[[lo, lo + 2], 0]).all()
    p.kv[0][int(p.kv_start[0]) + 5] = 0
    p.used[int(p.kv_start[0]) + 5] = False
    keep = np.ones(p.rows, np.uint8)
    keep[int(p.kv_start[0]) + 5] = 0
    ref, _ = tokens.attend(_np(p.q), p.kv[0], p.kv[1], p.q_start, p.kv_start, p.kv_len, p.scale, keep)
    assert np.abs(out[[lo, lo + 2]] - ref[[lo, lo + 2]]).max() < 16 * E[dtype] + 1e-5


@pytest.mark.parametrize("dtype,dim,heads,q_len,kv_len,kernel", [("bf16", 64, 1, [16], [70], 1), ("f16", 128, 3, [70, 33, 0, 48, 17, 1], [1500, 33, 9, 129, 1, 0], 4), ("bf16", 128, 3, [129, 1, 128, 33, 0, 97], [3000, 63, 1, 64, 65, 193], 3), ("f32", 64, 8, [20, 3] * 32, [49, 20] * 32, 2)])
def test_a_query_that_is_no_number_stays_in_its_row(octo, dtype, dim, heads, q_len, kv_len, kernel):
    import torch
    p = Problem(octo, dtype, "plain", dim, heads, 1, q_len, kv_len, seed=7)
    p.run(octo)
    clean, lse = p.out.clone(), p.lse.clone()
    sick = torch.zeros(p.q.shape[:2], dtype=torch.bool, device="cuda")
    lo = int(p.q_start[0])
    sick[lo + 5, 0] = sick[lo + 9, heads - 1] = True
    p.q[sick] = torch.where(torch.arange(dim, device="cuda") == 3, float("nan"), 1.0).to(p.q.dtype)
    kid = p.run(octo)
    assert octo.device_cu_count() != 256 or kid // 1000 == kernel
    assert bool(torch.isnan(p.out[sick]).all()) and bool(torch.isnan(p.lse[sick]).all())
    # the reference of a wavefront's rows moves when one of them asks for it: the others agree within the bound, not bit for bit
    assert float((p.out - clean)[~sick].abs().max()) <= 8 * E[dtype] * float(clean.abs().max()) + 1e-5 and bool(torch.isclose(p.lse, lse, rtol=0, atol=1e-4)[~sick].all())


@forms
def test_counts_and_lengths_on_the_device_are_cut_to_what_the_host_stated(octo, dtype, fmt):
    import torch
    p = Problem(octo, dtype, fmt, 64, 1, 2, [2, 3, 4, 2], [50, 60, 70, 80], seed=1)
    p.run(octo, n_seq=torch.tensor([2], dtype=torch.int32, device="cuda"))
    p.check(2)
    p.out.fill_(7), p.lse.fill_(7)
    p.run(octo, n_seq=torch.tensor([0], dtype=torch.int32, device="cuda"))
    assert bool((p.out == 7).all()) and bool((p.lse == 7).all())
    # longer than stated: cut to max_kv; starts outside the pool and negative lengths: no keys; wild q_start: clamped
    p.run(octo, max_kv=40)
    p.kv_len = np.minimum(p.kv_len, 40)
    p.check()
    p.dev[1][1], p.dev[1][3] = -5, p.rows
    p.dev[2][2] = -1
    p.run(octo)
    p.kv_len[[1, 2, 3]] = 0
    p.check()
    p.dev[0][0], p.dev[0][4] = -100, 2 ** 30
    p.run(octo)
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["plain", "cache4"])
def test_parts_cut_on_the_device_follow_its_counts(octo, fmt):
    """A long call with fewer sequences present, lengths beyond what the host stated, starts outside the pool, and the same bits twice."""
    import torch
    p = Problem(octo, "bf16", fmt, 128, 3, 1, [129, 40, 0, 128, 1, 2], [22000, 900, 70, 9000, 5, 6], 0.8, seed=12)
    kw = dict(n_seq=torch.tensor([3], dtype=torch.int32, device="cuda"))
    need = octo.attend_workspace_bytes(p.q, p.held, p.out, *p.dev, max_q=129, max_kv=22000)
    kid = p.run(octo, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"), **kw)
    assert octo.device_cu_count() != 256 or kid // 1000 == 5
    p.check(3)
    first = p.out.clone()
    p.out.fill_(7)
    p.run(octo, **kw)
    assert torch.equal(p.out, first)
    p.out.fill_(7), p.lse.fill_(7)
    p.dev[1][3], p.dev[2][1] = -1, 2 ** 31 - 1
    p.kv_len[3] = 0
    p.kv_len[1] = min(22000, p.rows - int(p.kv_start[1]))
    p.used[int(p.kv_start[1]):int(p.kv_start[1]) + int(p.kv_len[1])] &= p.mask[int(p.kv_start[1]):int(p.kv_start[1]) + int(p.kv_len[1])] != 0
    if fmt == "plain":                          # rows between the sequences hold NaN: hide what the long sequence newly reads of them
        p.mask[np.isnan(_np(p.held[0]).sum((1, 2)))] = 0
        p.dmask.copy_(torch.from_numpy(p.mask))
    else:
        p.mask[(p.held.k_exps == 255).any(2).any(0).cpu().numpy()] = 0
        p.dmask.copy_(torch.from_numpy(p.mask))
    seen = np.arange(p.rows)
    p.used = (p.mask != 0) & (seen >= 0)
    p.run(octo)
    p.check()


@pytest.mark.parametrize("dtype,fmt,dim,heads,group,q_len,kv_len,kernel", [
    ("bf16", "plain", 128, 6, 4, [64, 64, 64], [22000, 22000, 21990], 5), ("f16", "cache4", 96, 6, 4, [64, 64, 64], [22000, 22000, 21990], 5),
    # the host takes them to be alike and they are not
    ("f16", "plain", 72, 6, 4, [64, 64, 64], [22000, 0, 700], 5), ("bf16", "plain", 64, 2, 1, [128] * 16, [3000] * 15 + [1], 3),
    ("bf16", "plain", 128, 3, 2, [300, 300], [2000, 2000], 3),
], ids=lambda v: str(v) if not isinstance(v, list) else "")
def test_parts_of_sequences_of_equal_length(octo, dtype, fmt, dim, heads, group, q_len, kv_len, kernel):
    p = Problem(octo, dtype, fmt, dim, heads, group, q_len, kv_len, None, seed=14)
    kid = p.run(octo)
    p.check()
    assert octo.device_cu_count() != 256 or (kid // 1000 == kernel and kid % 1000 > 1)
    first = p.out.clone()
    p.out.fill_(7)
    p.run(octo)
    import torch
    assert torch.equal(p.out, first)


def test_no_keys_for_many_equal_rows(octo):
    """max_kv of zero with the rows of a long call."""
    p = Problem(octo, "bf16", "plain", 64, 2, 1, [513] * 200, [0] * 200, None, seed=15)
    p.run(octo)
    p.check()


@forms
def test_strided_tensors_and_another_stream(octo, dtype, fmt):
    """Queries as slices of a wider projection, heads of the pool outermost, the result into a wider buffer."""
    import torch
    p = Problem(octo, dtype, fmt, 96, 2, 2, [3, 20], [90, 200], 0.8, seed=6)
    wide_q = torch.full((p.q.shape[0], 7, 128), float("nan"), dtype=p.q.dtype, device="cuda")
    wide_q[:, 2:6, 16:112] = p.q
    p.q = wide_q[:, 2:6, 16:112]
    wide_out = torch.full((5, p.q.shape[0], 96), 7.0, dtype=p.q.dtype, device="cuda")
    p.out = wide_out[1:].transpose(0, 1)
    if fmt == "plain":
        p.held = tuple(x.transpose(0, 1).contiguous().transpose(0, 1) for x in p.held)
    else:
        p.held = octo.Cache4(*[x.transpose(0, 1).contiguous().transpose(0, 1) for x in (p.held.k_codes, p.held.k_exps, p.held.v_codes, p.held.v_exps)])
    side = torch.cuda.Stream()
    p.run(octo, stream=side)
    side.synchronize()
    p.check()
    assert bool((wide_out[0] == 7).all())


@pytest.mark.parametrize("fmt", ["plain", "cache4"])
def test_a_pool_beyond_32_bit_offsets(octo, fmt):
    """Keys whose bytes lie beyond 4 GiB from the start of the pool."""
    import torch
    rows, heads, dim = (2_200_000, 8, 128) if fmt == "plain" else (9_000_000, 8, 128)
    small = Problem(octo, "bf16", fmt, dim, heads, 1, [2], [300], seed=3)
    move = rows - small.rows
    if fmt == "plain":
        big = [torch.empty(rows, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for x, y in zip(big, small.held):
            x[move:] = y
        assert big[0][move:].data_ptr() - big[0].data_ptr() > 2 ** 32
        small.held = tuple(big)
    else:
        big = []
        for y in (small.held.k_codes, small.held.k_exps, small.held.v_codes, small.held.v_exps):
            x = torch.empty(rows, heads, y.shape[2], dtype=torch.uint8, device="cuda")
            x[move:] = y.transpose(0, 1)
            big.append(x.transpose(0, 1))
        assert big[0][0, move:].data_ptr() - big[0].data_ptr() > 2 ** 32
        small.held = octo.Cache4(*big)
    small.dev[1] += move
    small.run(octo)
    small.check()


@pytest.mark.parametrize("q_len,kv_len", [([1, 1], [900, 700]), ([50, 3], [300, 999])])
def test_in_a_graph(octo, q_len, kv_len):
    """Captured with a workspace of the caller's, replayed with other inputs in the same memory."""
    import torch
    p = Problem(octo, "bf16", "cache4", 128, 2, 4, q_len, kv_len, 0.9, seed=11)
    p.out.fill_(7)
    need = octo.attend_workspace_bytes(p.q, p.held, p.out, *p.dev, max_q=max(q_len), max_kv=max(kv_len))
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    p.run(octo, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(octo, workspace=ws)
    for k in range(3):
        p.q.copy_(torch.randn_like(p.q))
        p.out.fill_(7), p.lse.fill_(7), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        p.check()
        again = p.out.clone()
        p.run(octo)
        assert torch.equal(again, p.out)


def test_nothing_to_do(octo):
    import torch
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    q, k = z(4, 2, 64), z(0, 2, 64)
    out = torch.full_like(q, 7)
    lse = z(4, 2, t=torch.float32)
    assert octo.op_attend(q, (k, k), out, z(1, t=torch.int32), z(0, t=torch.int64), z(0, t=torch.int32)) == 0
    assert bool((out == 7).all())
    # a pool without rows
    octo.op_attend(q, (k, k), out, torch.tensor([0, 4], dtype=torch.int32, device="cuda"), z(1, t=torch.int64), z(1, t=torch.int32) + 9, lse=lse)
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


def test_refusals(octo):
    import torch
    p = Problem(octo, "bf16", "plain", 64, 1, 2, [2], [5])
    k, v = p.held
    for held in ((k, v[:-1]), (k.half(), v.half()), (k[..., :32], v[..., :32]), (k[:, :, ::2], v[:, :, ::2])):
        with pytest.raises(octo.OctoError):
            octo.op_attend(p.q, held, p.out, *p.dev)
    for kw in (dict(scale=float("nan")), dict(scale=0.0), dict(max_q=p.q.shape[0] + 1), dict(max_kv=-1), dict(key_mask=torch.ones(3, dtype=torch.uint8, device="cuda")),
               dict(lse=torch.empty(3, device="cuda"))):
        with pytest.raises(octo.OctoError):
            octo.op_attend(p.q, p.held, p.out, *p.dev, **kw)
    long = Problem(octo, "bf16", "plain", 64, 1, 2, [1], [9000])
    assert octo.attend_workspace_bytes(long.q, long.held, long.out, *long.dev, max_q=1, max_kv=9000) > 64
    with pytest.raises(octo.OctoError) as e:
        long.run(octo, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == octo.ENOMEM
    assert bool((long.out == 7).all())
