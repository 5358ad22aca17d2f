"""Long calls of attention whose parts are cut on the device, of sizes at which the pieces of equal sequences fill more than three rounds of blocks, against the
definition in 64 bits (on the GPU: they are long).  The workspace holds NaN before each call, so a part that no block computes shows.  The bounds are those of
test_gpu_attend.py."""
import math

import pytest

pytestmark = pytest.mark.gpu
E = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


class Long:
    def __init__(self, octo, dtype, fmt, dim, q_heads, kv_heads, q_len, kv_len, seed=1):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        t = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        self.dtype, self.dim, self.q_len, self.kv_len, self.rows = dtype, dim, q_len, kv_len, sum(kv_len)
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=t)  # noqa: E731
        self.q, self.heads = randn(sum(q_len), q_heads, dim), kv_heads
        if fmt == "plain":
            self.held = (randn(self.rows, kv_heads, dim), randn(self.rows, kv_heads, dim))
        else:
            codes = lambda: torch.randint(0, 256, (kv_heads, self.rows, dim // 2), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
            exps = lambda: torch.randint(123, 127, (kv_heads, self.rows, dim // 32), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
            self.held = octo.Cache4(codes(), exps(), codes(), exps())
        self.starts = [sum(q_len[:i]) for i in range(len(q_len) + 1)]
        self.kv_starts = [sum(kv_len[:i]) for i in range(len(kv_len))]
        dev = lambda v, ty: torch.tensor(v, dtype=ty, device="cuda")  # noqa: E731
        self.dev = [dev(self.starts, torch.int32), dev(self.kv_starts, torch.int64), dev(kv_len, torch.int32)]
        self.out, self.lse = torch.full_like(self.q, 7.0), torch.full(self.q.shape[:2], 7.0, device="cuda")

    def run(self, octo):
        import torch
        most = dict(max_q=max(self.q_len), max_kv=max(self.kv_len))
        need = octo.attend_workspace_bytes(self.q, self.held, self.out, *self.dev, **most)
        return octo.op_attend(self.q, self.held, self.out, *self.dev, lse=self.lse, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None, **most)

    def values(self, which, head, lo, hi):
        """[rows][dim] in 64 bits."""
        import torch
        if isinstance(self.held, tuple):
            return self.held[which][lo:hi, head].double()
        codes, exps = ((self.held.k_codes, self.held.k_exps), (self.held.v_codes, self.held.v_exps))[which]
        c, e = codes[head, lo:hi], exps[head, lo:hi]
        v = torch.tensor(E2M1 + tuple(-x for x in E2M1), dtype=torch.float64, device="cuda")[torch.stack([c & 15, c >> 4], -1).flatten(1).long()]
        return v * torch.exp2(e.double() - 127).repeat_interleave(32, 1)

    def check(self):
        import torch
        group, e, scale = self.q.shape[1] // self.heads, E[self.dtype], self.dim ** -0.5
        for b, n in enumerate(self.kv_len):
            lo, hi = self.starts[b], self.starts[b + 1]
            if lo == hi:
                continue
            if not n:
                assert bool((self.out[lo:hi] == 0).all()) and bool(torch.isneginf(self.lse[lo:hi]).all())
                continue
            for h in range(self.heads):
                k, v = (self.values(i, h, self.kv_starts[b], self.kv_starts[b] + n) for i in (0, 1))
                mine = slice(h * group, (h + 1) * group)
                kt = k.t().contiguous()
                every = [x[lo:hi, mine].double().reshape((hi - lo) * group, -1) for x in (self.q, self.out, self.lse[:, :, None])]
                for q, out, got in zip(*[x.split(16384) for x in every]):
                    got = got[:, 0]
                    s = (q @ kt) * scale
                    d = (self.dim + 8) * 2.0 ** -24 * scale * (q.abs() @ kt.abs()).amax(1)
                    lse = torch.logsumexp(s, 1)
                    w = torch.exp(s - lse[:, None])
                    ref = w @ v
                    fp32 = (n / 8 + 64) * 2.0 ** -24
                    bound = (e + 2 * d + fp32)[:, None] * (w @ v.abs()) + e * ref.abs() + 2.0 ** -126 * (1 + v.abs().sum(0))
                    if self.dtype == "f16":
                        bound += 2.0 ** -24 * (1 + v.abs().sum(0) * torch.exp(s.amax(1) - lse)[:, None])
                    err = (out - ref).abs()
                    assert bool((err <= bound).all()), (b, h, float((err - bound).nan_to_num(nan=math.inf).max()))
                    off = (got - lse).abs()
                    assert bool((off <= d + fp32 + 2.0 ** -22 * (1 + lse.abs())).all()), (b, h)


@pytest.mark.parametrize("dtype,fmt,dim,q_heads,kv_heads,n,q_len,kv_len", [
    ("bf16", "plain", 128, 32, 8, 2, 2049, 12800), ("bf16", "plain", 72, 16, 1, 5, 900, 6400), ("f16", "plain", 32, 64, 2, 3, 520, 12800), ("f16", "plain", 80, 16, 8, 6, 642, 21877),
    ("bf16", "plain", 72, 40, 8, 36, 4, 16452), ("f16", "cache4", 128, 32, 8, 17, 96, 20440), ("bf16", "cache4", 96, 68, 4, 2, 520, 6400), ("f16", "cache4", 64, 64, 2, 3, 520, 12800),
    ("bf16", "cache4", 64, 136, 8, 100, 1, 6400),
    # 599552 rows to join
    ("bf16", "plain", 8, 512, 8, 1, 1171, 12800)])
def test_equal_sequences(octo, dtype, fmt, dim, q_heads, kv_heads, n, q_len, kv_len):
    p = Long(octo, dtype, fmt, dim, q_heads, kv_heads, [q_len] * n, [kv_len] * n)
    kid = p.run(octo)
    assert octo.device_cu_count() != 256 or (kid // 1000 == 5 and kid % 1000 > 1), kid
    p.check()


@pytest.mark.parametrize("dtype,fmt,dim,q_heads,kv_heads,q_len,kv_len", [
    # lengths of keys that the host takes to be equal and are not
    ("bf16", "plain", 72, 16, 1, [900] * 5, [6400, 10, 0, 6400, 3200]), ("f16", "cache4", 96, 68, 4, [520, 519], [6400, 700]),
    # just as equal as it takes for the host's number of parts, and just not
    ("f16", "plain", 32, 64, 2, [520, 519, 521], [12800, 12000, 11201]), ("bf16", "plain", 72, 16, 1, [900] * 5, [6400] * 4 + [4300])])
def test_nearly_equal_sequences(octo, dtype, fmt, dim, q_heads, kv_heads, q_len, kv_len):
    p = Long(octo, dtype, fmt, dim, q_heads, kv_heads, q_len, kv_len)
    kid = p.run(octo)
    assert octo.device_cu_count() != 256 or kid // 1000 == 5, kid
    p.check()


@pytest.mark.parametrize("dtype,fmt,dim,q_len,kv_len", [("bf16", "plain", 128, [1, 2], [700, 33]), ("f32", "plain", 64, [40, 3], [300, 65]), ("f16", "cache4", 96, [7] * 40, [500] * 40), ("bf16", "plain", 72, [300, 299], [900, 64])])
def test_no_limit_stated(octo, dtype, fmt, dim, q_len, kv_len):
    """Sequences of a few keys where the host states the largest number that is taken."""
    from test_gpu_attend import Problem
    p = Problem(octo, dtype, fmt, dim, 2, 4, q_len, kv_len, 0.8, seed=5)
    assert p.run(octo, max_kv=0x7FFFFF00) % 1000 > 1
    p.check()
