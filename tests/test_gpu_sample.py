"""octo_op_sample on the GPU against the 64-bit oracle.

Tokens and counts are whole numbers and have to be equal.  The kernel's weights are multiples of 2^-43 or less of the largest, each off by half of that and 1e-15 of itself: a sum of n of them is within
n * 2^-44 of the oracle's.  Random numbers of 24 bits and shares of random logits lie nearer to a border than that once in 10^8 rows; equal logits, where borders are exact, are
tested with weights that are exact.  logprob: fp32 of a logarithm that is within 1e-9."""
import math

import numpy as np
import pytest

from oracle import answer

pytestmark = pytest.mark.gpu


def _t(dtype):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def _run(octo, logits, u, **settings):
    import torch
    n = logits.shape[0]
    token, kept = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    logprob = torch.full((n,), float("nan"), device="cuda")
    octo.op_sample(logits, u, token, logprob=logprob, kept=kept, **settings)
    return token.cpu().numpy(), kept.cpu().numpy(), logprob.cpu().numpy()


def _expected(x, u, t, k, p, m):
    """The oracle's answer, with the sums of a row by numpy (the row may be long): (token, kept, logprob)."""
    x = np.where(np.isnan(x), -np.inf, x)
    words = np.nonzero(x > -np.inf)[0]
    if not len(words):
        return -1, 0, -np.inf
    words = words[np.lexsort((words, -x[words]))]
    if not t > 0:
        return int(words[0]), 1, 0.0
    top = x[words[0]]
    w = (x[words] == top).astype(np.float64) if np.isinf(top) else np.exp((x[words] - top) / t)
    if k > 0:
        words, w = words[:k], w[:k]
    up_to = np.cumsum(w)
    keep = len(w)
    if p < 1:
        keep = min(keep, max(1, int((up_to - w < p * up_to[-1]).sum())))
    if m > 0:
        keep = min(keep, max(1, int((w >= m).sum())))
    words, w = words[:keep], w[:keep]
    back = np.argsort(words)
    up_to = np.cumsum(w[back])
    at = min(int((up_to <= u * up_to[-1]).sum()), keep - 1)
    return int(words[back][at]), keep, math.log(w[back][at] / up_to[-1])


def _check(got, logits, u, settings):
    x, u = logits.double().cpu().numpy(), u.double().cpu().numpy()
    n = len(x)
    values = []
    for name, none in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)):
        v = settings.get(name, none)
        values.append(np.broadcast_to(v.cpu().numpy().astype(np.float64) if hasattr(v, "cpu") else np.float64(np.float32(v)), (n,)))
    for r in range(n):
        t, k, p, m = (v[r] for v in values)
        token, kept, logprob = _expected(x[r], u[r], t, int(k), p, m)
        assert (int(got[0][r]), int(got[1][r])) == (token, kept), (r, t, k, p, m, u[r])
        assert got[2][r] == logprob or abs(got[2][r] - logprob) <= 1e-6 + 2.0 ** -23 * abs(logprob), (r, got[2][r], logprob)


def test_the_expectation_is_the_oracles():
    rng = np.random.default_rng(0)
    for _ in range(200):
        x = np.round(rng.standard_normal(17) * 2, 1)
        x[rng.random(17) < 0.2] = -np.inf
        args = rng.random(), rng.choice([0.0, 0.5, 1.3]), int(rng.choice([0, 3, 9])), rng.choice([1.0, 0.61, 0.93]), rng.choice([0.0, 0.07])
        a, b = _expected(x, *args), answer.sample(x, *args)
        assert a[:2] == b[:2] and (a[2] == b[2] or abs(a[2] - b[2]) < 1e-12)


def _logits(n, vocab, dtype, seed, flat=2.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, vocab, generator=g) * flat
    likely = torch.randint(0, vocab, (n, min(vocab, 9)), generator=g)
    x.scatter_add_(1, likely, 6 * torch.rand(n, min(vocab, 9), generator=g))
    x[torch.rand(n, vocab, generator=g) < 0.02] = -math.inf
    return x.to(_t(dtype)).cuda(), torch.rand(n, generator=g).cuda(), g


VOCABS = [1, 2, 7, 63, 64, 65, 1000, 4097, 8192, 32769, 100003]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_settings_of_each_row(octo, dtype, vocab):
    import torch
    n = 24
    logits, u, g = _logits(n, vocab, dtype, vocab)
    pick = lambda v: torch.tensor(v)[torch.randint(0, len(v), (n,), generator=g)].cuda()  # noqa: E731
    settings = dict(temperature=pick([0.0, 0.3, 0.9, 1.7, 40.0]), top_k=pick([0, 0, 1, 2, 50, 1500, 5000, -3]).to(torch.int32), top_p=pick([1.0, 1.0, 0.3, 0.9, 0.993, 0.0, 1.5]), min_p=pick([0.0, 0.0, 0.05, 1e-4, 2.0]))
    logits[3] = -math.inf
    logits[5] = math.nan
    _check(_run(octo, logits, u, **settings), logits, u, settings)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("settings", [{}, dict(temperature=0.0), dict(temperature=0.7, top_k=40), dict(top_p=0.95), dict(min_p=0.02), dict(temperature=1.2, top_k=3000, top_p=0.9, min_p=0.001),
                                      dict(top_k=1), dict(top_p=1e-9), dict(temperature=1e-30, top_k=30), dict(temperature=1e30, top_p=0.5), dict(temperature=float("inf"), top_k=700)],
                         ids=lambda s: "_".join("%s%g" % p for p in s.items()) or "none")
def test_one_setting_for_all_rows(octo, dtype, settings):
    logits, u, _ = _logits(6, 20011, dtype, 5)
    _check(_run(octo, logits, u, **settings), logits, u, settings)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [100, 2048, 2049, 30000, 70001])
def test_equal_logits_go_by_their_index(octo, dtype, vocab):
    """All alike, two values, and a few ones above many alike: borders fall between equal logits, more of them than are sorted."""
    import torch
    rows = [torch.zeros(vocab), torch.full((vocab,), -3.5), (torch.arange(vocab) % 2).float() * 4, torch.where(torch.arange(vocab) % 31 == 3, 2.0, 1.0)]
    logits = torch.stack(rows).to(_t(dtype)).cuda()
    u = torch.tensor([0.37, 0.0, 0.51, 0.999]).cuda()
    for settings in (dict(top_k=vocab // 3 + 1), dict(top_k=vocab - 1), dict(temperature=1e30, top_p=0.625), dict(top_k=vocab // 2 + 1, temperature=1e30, top_p=0.3), dict(min_p=0.5)):
        _check(_run(octo, logits, u, **settings), logits, u, settings)


def test_a_long_flat_tail(octo):
    """A share that ends far down: bins of w with more tokens than are sorted, whose logits differ in their last bits alone."""
    import torch
    vocab = 120000
    x = 8.0 + torch.arange(vocab).double() * 2.0 ** -20
    logits = torch.stack([x, x.flip(0), -x]).float().cuda()
    assert len(torch.unique(logits[0])) == vocab
    u = torch.tensor([0.2, 0.5, 0.93]).cuda()
    for settings in (dict(top_p=0.7), dict(top_k=50001), dict(top_k=99999, top_p=0.6), dict(top_k=40000, top_p=0.97), {}):
        _check(_run(octo, logits, u, **settings), logits, u, settings)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_both_zeros_and_tiny_logits(octo, dtype):
    """Zeros of both signs are equal logits; magnitudes far below the largest one's lie between positive and negative ones."""
    import torch
    g = torch.Generator().manual_seed(6)
    n, vocab = 12, 5000
    x = torch.randn(n, vocab, generator=g)
    x[0::4] = torch.where(torch.rand(3, vocab, generator=g) < 0.5, 0.0, -0.0)
    x[0::4, ::997] = 1.0
    small = torch.randn(3, vocab, generator=g) * 2.0 ** -20
    x[1::4] = torch.where(torch.rand(3, vocab, generator=g) < 0.3, small, x[1::4])
    x[2::4] *= 2.0 ** -14                                       # all small: octaves follow the largest magnitude
    x[3::4] = -x[3::4].abs() - 0.5
    logits = x.to(_t(dtype)).cuda()
    u = torch.rand(n, generator=g).cuda()
    for settings in ({}, dict(top_k=700), dict(top_k=3000, top_p=0.9), dict(temperature=0.8, top_p=0.45), dict(top_p=0.62), dict(min_p=0.1), dict(min_p=0.999), dict(temperature=1e-3, top_p=0.97), dict(top_k=9), dict(top_k=2500, min_p=0.2)):
        _check(_run(octo, logits, u, **settings), logits, u, settings)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("min_p", [0.02, 0.3, 0.9])
def test_what_min_p_drops(octo, dtype, min_p):
    """Borders of min-p at, above and below logits of no magnitude, alone and beside the others."""
    import torch
    base = [3.0, 1.5, 0.25, 2.0 ** -22, 0.0, -(2.0 ** -23), -0.25, -1.5, -4.0]
    rows = [torch.tensor(base).repeat(400)] + [torch.tensor(base[i:]).repeat(400)[:2000] for i in (1, 2, 3, 4, 6)] + [torch.tensor([1.5, 2.0 ** -22, -1.5]).repeat(900)]
    n = max(len(r) for r in rows)
    logits = torch.full((len(rows), n), -math.inf)
    for i, r in enumerate(rows):
        logits[i, :len(r)] = r
    logits = logits.to(_t(dtype)).cuda()
    u = torch.linspace(0.03, 0.97, len(rows)).cuda()
    for settings in (dict(min_p=min_p), dict(min_p=min_p, top_k=1100), dict(min_p=min_p, top_p=0.6), dict(min_p=min_p, top_k=1500, top_p=0.83, temperature=0.7)):
        _check(_run(octo, logits, u, **settings), logits, u, settings)


def test_infinities(octo):
    import torch
    x = torch.randn(4, 500).cuda()
    x[0, 17] = x[0, 400] = math.inf
    x[1] = -math.inf
    x[1, 499] = -3e38
    x[2, 3] = 3e38
    x[3] = math.inf
    u = torch.tensor([0.6, 0.9, 0.5, 0.25]).cuda()
    token, kept, logprob = _run(octo, x, u)
    assert token.tolist() == [400, 499, 3, 125] and kept.tolist() == [500, 1, 500, 500]
    assert np.allclose(logprob, [math.log(0.5), 0, 0, -math.log(500)], atol=1e-6)
    assert _run(octo, x, u, temperature=float("inf"))[0].tolist() == [400, 499, 250, 125]


def test_random_numbers_at_the_ends(octo):
    """u of 0 draws the first kept token by index, the largest the last; numbers outside are taken as the ends."""
    import torch
    x = torch.zeros(6, 300).cuda()
    x[:, :40] = -math.inf
    u = torch.tensor([0.0, -5.0, math.nan, 1.0 - 2.0 ** -24, 1.0, 7.0]).cuda()
    assert _run(octo, x, u)[0].tolist() == [40, 40, 40, 299, 299, 299]


def test_shares_are_those_of_the_weights(octo):
    """Evenly spread random numbers draw every token as often as its weight says, up to one."""
    import torch
    n = 4000
    x = torch.tensor([0.5, -1.0, 2.0, 0.0, -math.inf, 1.0, 2.0]).repeat(n, 1).cuda()
    u = (torch.arange(n).float() / n + 0.5 / n).cuda()
    drawn = np.bincount(_run(octo, x, u, temperature=0.8)[0], minlength=7)
    w = torch.softmax(x[0].double() / np.float64(np.float32(0.8)), 0).cpu().numpy()
    assert np.abs(drawn - n * w).max() <= 1.01


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_wider_tensor_at_any_address(octo, dtype):
    import torch
    wide, u, _ = _logits(9, 3011, dtype, 8)
    for first, vocab in ((0, 3000), (1, 2999), (3, 1), (5, 64), (7, 3004)):
        logits = wide[:, first:first + vocab]
        settings = dict(temperature=0.9, top_k=30, top_p=0.97)
        _check(_run(octo, logits, u, **settings), logits, u, settings)


def test_a_count_on_the_device_another_stream_and_optional_outputs(octo):
    import torch
    logits, u, _ = _logits(10, 777, "f32", 2)
    side = torch.cuda.Stream()
    whole = _run(octo, logits, u)[0]
    for count in (-1, 0, 1, 7, 10, 30):
        m = max(0, min(count, 10))
        token = torch.full((10,), -7, dtype=torch.int32, device="cuda")
        octo.op_sample(logits, u, token, n=torch.tensor([count], dtype=torch.int32, device="cuda"), stream=side)
        side.synchronize()
        assert token.tolist() == whole[:m].tolist() + [-7] * (10 - m)
    octo.op_sample(torch.empty(0, 5, device="cuda"), u, token)
    for call in (lambda: octo.op_sample(logits.double(), u, token), lambda: octo.op_sample(logits, u[:9], token), lambda: octo.op_sample(logits, u, token.long()), lambda: octo.op_sample(logits.T, u, token),
                 lambda: octo.op_sample(logits, u, token, top_k=u), lambda: octo.op_sample(logits, u, token, top_p=u.half()), lambda: octo.op_sample(logits.cpu(), u, token),
                 lambda: octo.op_sample(logits, u, token, logprob=u.half())):
        with pytest.raises(octo.OctoError):
            call()


def test_captured_and_replayed(octo):
    import torch
    logits, u, _ = _logits(5, 5000, "bf16", 1)
    token, again = (torch.zeros(5, dtype=torch.int32, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        octo.op_sample(logits, u, token, top_p=0.9)
    for seed in range(3):
        fresh, u2, _ = _logits(5, 5000, "bf16", 30 + seed)
        logits.copy_(fresh)
        u.copy_(u2)
        graph.replay()
        octo.op_sample(logits, u, again, top_p=0.9)
        torch.cuda.synchronize()
        assert torch.equal(token, again)
        _check(_run(octo, logits, u, top_p=0.9), logits, u, dict(top_p=0.9))


def _hard_rows(dtype, vocab):
    """Rows on which borders fall among many equal logits, in steep and flat ones, with infinities, NaN and nothing."""
    import torch
    g = torch.Generator().manual_seed(vocab)
    rows = [torch.randn(vocab, generator=g) * s for s in (0.01, 2.0, 30.0)]
    rows.append(torch.randn(vocab, generator=g).mul(4).round())                        # thousands of equal logits on a step
    rows.append(torch.zeros(vocab))
    rows.append(torch.full((vocab,), -float("inf")))
    rows.append(torch.randn(vocab, generator=g).masked_fill(torch.rand(vocab, generator=g) < 0.9, float("nan")))
    some = torch.randn(vocab, generator=g)
    some[vocab // 3::9973] = float("inf")
    rows.append(some)
    last = torch.full((vocab,), -200.0)
    last[-1] = 3.0
    rows.append(last)
    rows.append(torch.arange(vocab).float().neg().mul(1e-4))
    return torch.stack(rows).to(_t(dtype)).cuda()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [65536, 70001, 131072, 524288])
@pytest.mark.parametrize("settings", [dict(), dict(top_p=0.9), dict(top_p=0.3, min_p=0.001), dict(min_p=0.2), dict(top_k=700), dict(top_k=20000, top_p=0.99), dict(top_k=40, top_p=0.9),
                                      dict(temperature=0.3, top_p=0.5), dict(temperature=0.0), dict(temperature=float("inf"), top_p=0.7), dict(min_p=1e-25)])
def test_rows_shared_among_workgroups(octo, dtype, vocab, settings):
    """Long rows with a workspace: the same as the definition says, and bit for bit the same as without one."""
    import torch
    x = _hard_rows(dtype, vocab)
    n = x.shape[0]
    settings = dict(settings)
    if settings.get("top_k", 0) and settings["top_k"] <= 512:
        settings["top_k"] = torch.tensor([settings["top_k"], 0] * (n // 2), dtype=torch.int32, device="cuda")      # rows of both kinds in a call
    u = torch.rand(n, generator=torch.Generator().manual_seed(7)).cuda()
    u[1], u[2] = 0.0, 0.99999994
    token = torch.empty(n, dtype=torch.int32, device="cuda")
    need = octo.sample_workspace_bytes(x, u, token, **settings)
    assert (need > 0) == (dtype != "bf16")
    work = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    got = _run(octo, x, u, workspace=work, **settings)
    alone = _run(octo, x, u, workspace=work[:0], **settings)
    for a, b in zip(got, alone):
        assert np.array_equal(a, b, equal_nan=True)
    _check(got, x, u, settings)


def test_workspaces(octo):
    """Sizes, refusals, rows that a count on the device leaves alone, and two captured calls that share one."""
    import torch
    g = torch.Generator().manual_seed(0)
    x, u, token = torch.randn(6, 70000, generator=g).cuda(), torch.rand(6, generator=g).cuda(), torch.full((6,), -7, dtype=torch.int32, device="cuda")
    need = octo.sample_workspace_bytes(x, u, token)
    assert need > 0
    assert octo.sample_workspace_bytes(x, u, token, top_k=50) == 0 == octo.sample_workspace_bytes(x[:, :5000], u, token)
    assert octo.sample_workspace_bytes(x[:1].expand(300, 70000), u[:1].expand(300).contiguous(), token[:1].expand(300).contiguous()) == 0
    work = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    for bad in (work[:need - 1], work[8:need + 8]):
        with pytest.raises(Exception):
            octo.op_sample(x, u, token, workspace=bad)
    octo.op_sample(x, u, token, top_p=0.9, n=torch.tensor([4], dtype=torch.int32, device="cuda"), workspace=work)
    assert bool((token[:4] >= 0).all()) and bool((token[4:] == -7).all())
    y = x.flip(1).contiguous()
    tokens, graphs = [torch.empty_like(token) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    torch.cuda.synchronize()
    for logits, t, graph in zip((x, y), tokens, graphs):
        with torch.cuda.graph(graph):
            octo.op_sample(logits, u, t, top_p=0.9, workspace=work)
    for turn in range(3):
        u.copy_(torch.rand(6, generator=g))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for logits, t in zip((x, y), tokens):
            octo.op_sample(logits, u, token, top_p=0.9)
            assert torch.equal(t, token)
