"""GPU checks of logprobs (log probabilities of given tokens, entropy, alternatives) and logprobs_grad against a plain
implementation in 64 bits, and of what they refuse.

Tolerances.  An exponential exp(x - r), |x - r| = a, is off by (2a + 2) * 2^-24 of its value: the difference and its product
with log2 e are rounded, and the instruction by one step.  A lane adds V / 512 / G * G of them in a row, a workgroup and its
parts at most 32 more partial sums, each sum with half a step: S is off by at most `terms` = V / 512 + 64 steps of 2^-24,
plus 2a of them for the terms that matter, which are those with a small a (a * exp(-a) < 0.37, and a reference lies at most
8 below the maximum: 24 more).  log S moves by as much.  x - m and the last difference add half a step of their size."""
import math

import pytest
import torch

gpu = pytest.mark.gpu
EPS = 2.0 ** -24
INF = math.inf


@pytest.fixture(scope="module")
def sp():
    from paper_2504_08850_amd import specee
    specee.lib()
    return specee


def plain(x, ids, n_top):
    """In 64 bits, from the definitions; x on the CPU."""
    z = x.double()
    N, V = z.shape
    m = z.amax(1)
    bad = z.isnan().any(1) | (m == INF)
    empty = ~bad & (m == -INF)
    t = z - torch.where(empty | bad, torch.zeros_like(m), m)[:, None]
    e = torch.where(bad[:, None], torch.zeros_like(t), t).exp()
    S = e.sum(1)
    log_sum = S.log()
    inner = torch.where(e > 0, e * torch.where(e > 0, t, torch.zeros_like(t)), torch.zeros_like(t)).sum(1)
    H = torch.where(S > 0, log_sum - inner / S, torch.zeros_like(S))
    lp = torch.where(empty[:, None], torch.full_like(t, -INF), t - log_sum[:, None])
    nan = torch.full((), math.nan, dtype=torch.float64)
    out = {k: torch.where(bad, nan, v) for k, v in dict(max_logit=m, log_sum=log_sum, entropy=H).items()}
    lp = torch.where(bad[:, None], nan, lp)
    if ids is not None:
        inside = (ids >= 0) & (ids < V)
        out["logprobs"] = torch.where(inside, lp.gather(1, ids.clamp(0, V - 1).long()), nan)
    if n_top:
        order = torch.argsort(torch.where(bad[:, None], torch.zeros_like(z), z), dim=1, descending=True, stable=True)
        order = order[:, :n_top]
        got = z.gather(1, order)
        none = bad[:, None] | (got == -INF)
        tid = torch.where(none, -1, order)
        tlp = torch.where(bad[:, None], nan, torch.where(none, torch.full_like(got, -INF), lp.gather(1, order)))
        pad = n_top - order.shape[1]
        out["top_ids"] = torch.nn.functional.pad(tid, (0, pad), value=-1)
        out["top_logprobs"] = torch.nn.functional.pad(tlp, (0, pad), value=-INF)
        out["top_logprobs"][bad] = math.nan
    return out, lp


def near(got, want, tol, what):
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = want.isfinite()
    assert torch.equal(fine, got.isfinite()), what
    assert torch.equal(want.isnan(), got.isnan()), what
    assert torch.equal(want[want.isinf()], got[want.isinf()]), what
    off = (got - want).abs()[fine]
    lim = (tol if isinstance(tol, torch.Tensor) else torch.full_like(want, tol))[fine]
    assert bool((off <= lim).all()), (what, float((off - lim).max()), float(off.max()))


def check(out, x, ids, n_top):
    want, _ = plain(x, ids, n_top)
    V = x.shape[1]
    steps = (V / 512 + 64 + 24) * EPS
    assert set(out) - {"_workspace"} == set(want)
    near(out["max_logit"], want["max_logit"], 0.0, "max_logit")
    # (the sum is at least 1, so log S moves by what S does; 2 steps of its own)
    near(out["log_sum"], want["log_sum"], steps + 2 * EPS * want["log_sum"].abs(), "log_sum")
    # sum of e * t over S: its terms are at most 0.37 S each in size, off like S, and moved to the maximum from up to 8 below
    size = 10 + 2 * want["log_sum"].abs()
    near(out["entropy"], want["entropy"], steps * size, "entropy")
    for k in ("logprobs", "top_logprobs"):
        if k in want:
            near(out[k], want[k], steps + 4 * EPS * (want[k].abs() + want["log_sum"].abs()[:, None]), k)
    if n_top:
        assert torch.equal(out["top_ids"].cpu().long(), want["top_ids"].long()), "top_ids"


def logits(N, V, dtype, seed, std=2.5):
    g = torch.Generator().manual_seed(seed)
    return (std * torch.randn((N, V), generator=g)).to(dtype)


def tokens(N, V, T, seed):
    return torch.randint(0, V, (N, T), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("N,V,T,n_top", [(1, 1, 1, 1), (2, 2, 3, 5), (3, 7, 1, 32), (5, 50, 4, 20), (1, 777, 16, 8),
                                         (60, 777, 64, 32), (1, 32000, 1, 5), (2, 32003, 4, 20), (7, 24001, 0, 1),
                                         (513, 4099, 2, 3), (33, 50280, 1, 0), (1, 128256, 8, 32), (9, 128255, 8, 8),
                                         (256, 2049, 1, 16), (300, 4097, 1, 31), (511, 9001, 1, 5), (64, 60001, 2, 9),
                                         (3, 300007, 2, 32), (1, 262080, 1, 20), (1030, 250, 1, 32),
                                         (1100, 777, 2, 20), (1025, 8003, 1, 8), (4, 200, 0, 32)])
def test_against_64_bits(sp, N, V, T, n_top, dtype):
    x = logits(N, V, dtype, N + V)
    ids = tokens(N, V, T, 3) if T else None
    out = sp.logprobs(x.cuda(), None if ids is None else ids.cuda(), n_top=n_top)
    check(out, x, ids, n_top)


ROWS = {
    "equal": lambda x: x.fill_(1.25),
    "ascending": lambda x: x.copy_(torch.arange(x.shape[1]) / 64.0),
    "descending": lambda x: x.copy_(-torch.arange(x.shape[1]) / 64.0),
    "few values": lambda x: x.copy_((x * 2).round() / 2),
    "lowest but one": lambda x: (x.fill_(torch.finfo(x.dtype).min), x.__setitem__(slice(x.numel() // 2, None), 0.5)),
    "all lowest": lambda x: x.fill_(torch.finfo(x.dtype).min),
    "masked half": lambda x: x.__setitem__((slice(None), slice(None, None, 2)), -INF),
    "one left": lambda x: (x.fill_(-INF), x.__setitem__((slice(None), x.shape[1] - 1), 3.0)),
    "none left": lambda x: x.fill_(-INF),
    "last rows none": lambda x: x.__setitem__(slice(1, None), -INF),
    "nan": lambda x: x.__setitem__((0, x.shape[1] // 3), math.nan),
    "all nan": lambda x: x.fill_(math.nan),
    "infinite": lambda x: x.__setitem__((0, x.shape[1] - 1), INF),
    "nan and masked": lambda x: (x.fill_(-INF), x.__setitem__((0, 0), math.nan)),
    "spread": lambda x: x.mul_(1000.0),
    "certain": lambda x: x.__setitem__((slice(None), 5 % x.shape[1]), 60000.0),
    "every 4096th": lambda x: x.__setitem__((slice(None), slice(3, None, 4096)), 40.0),
}


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("N,V", [(1, 8200), (2, 33), (3, 32003), (600, 1030), (2, 128257), (1100, 515)])
@pytest.mark.parametrize("what", sorted(ROWS))
def test_rows_that_are_special(sp, what, N, V, dtype):
    x = logits(N, V, dtype, 17)
    ROWS[what](x)
    ids = tokens(N, V, 4, 5)
    ids[:, 1] = -1
    ids[:, 2] = V
    check(sp.logprobs(x.cuda(), ids.cuda(), n_top=12), x, ids, 12)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("V", [2100, 6000, 20000, 128257])
@pytest.mark.parametrize("n_top", [1, 32])
def test_equal_logits_by_the_hundred(sp, n_top, V, dtype):
    counts = (31, 33, 255, 256, 257, 511, 512, 513, 2000)
    x = logits(len(counts), V, dtype, 23)
    for n, c in enumerate(counts):
        x[n, torch.randperm(V, generator=torch.Generator().manual_seed(c))[:c]] = 30.0
    x[3:, 7] = 31.0                                # and one above them
    check(sp.logprobs(x.cuda(), None, n_top=n_top), x, None, n_top)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 5), (0, 7), (7, 64), (5, 1)])
def test_rows_apart_and_off_any_alignment(sp, offset, pad, dtype):
    for N, V in ((4, 301), (3, 16411), (1, 16411), (2, 110011), (1026, 301)):
        buf = torch.full((offset + N * (V + pad),), 1000.0, dtype=dtype)   # what lies between would win
        x = buf[offset:].view(N, V + pad)[:, :V]
        x.copy_(logits(N, V, dtype, V + pad))
        on = buf.cuda()
        y = on[offset:].view(N, V + pad)[:, :V]
        ids = tokens(N, V, 2, 4)
        check(sp.logprobs(y, ids.cuda(), n_top=9), x, ids, 9)


@gpu
def test_offsets_beyond_32_bits(sp):
    V, stride = 4099, (1 << 31) + 3
    buf = torch.empty((2 * stride + V,), dtype=torch.float16, device="cuda")
    x = logits(3, V, torch.float16, 2)
    y = buf.as_strided((3, V), (stride, 1))
    y.copy_(x.cuda())
    ids = tokens(3, V, 2, 4)
    check(sp.logprobs(y, ids.cuda(), n_top=4), x, ids, 4)
    st = sp.logprobs(y, ids.cuda())
    g = torch.ones((3, 2), device="cuda")
    got = sp.logprobs_grad(y, ids.cuda(), st["max_logit"], st["log_sum"], g_logprobs=g, out=y)   # in place
    assert got.data_ptr() == buf.data_ptr()
    check_grad(got, x, ids, g.cpu(), None)


@gpu
@pytest.mark.parametrize("V", [50280, 128256])
def test_same_bits_every_time_and_however_the_outputs_are_asked_for(sp, V):
    x = logits(3, V, torch.float32, 8).cuda()
    ids = tokens(3, V, 4, 4).cuda()
    a = sp.logprobs(x, ids, n_top=20)
    b = sp.logprobs(x, ids, n_top=20, out={k: torch.full_like(v, 7) for k, v in a.items() if k != "_workspace"},
                    workspace=a["_workspace"])
    c = sp.logprobs(x)
    for k in a:
        if k != "_workspace":
            assert torch.equal(a[k], b[k]), k
            assert k not in c or torch.equal(a[k], c[k]), k


@gpu
@pytest.mark.parametrize("N,V,n_top", [(2, 32003, 6), (2, 128257, 6), (3, 128256, 20), (1100, 777, 20), (2, 262100, 9)])
def test_graph_replays_and_two_streams(sp, N, V, n_top):
    x = logits(N, V, torch.float32, 1).cuda()
    ids = tokens(N, V, 3, 4).cuda()
    g, gh = torch.randn(N, 3, device="cuda"), torch.randn(N, device="cuda")
    ref = sp.logprobs(x, ids, n_top=n_top)
    rg = sp.logprobs_grad(x, ids, ref["max_logit"], ref["log_sum"], ref["entropy"], g, gh)
    out, dx = sp.logprobs(x, ids, n_top=n_top), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = sp.logprobs(x, ids, n_top=n_top, stream=side)       # beside the next call, with a workspace of its own
    again = sp.logprobs(x, ids, n_top=n_top)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.logprobs(x, ids, n_top=n_top, out=out, workspace=out["_workspace"])
        sp.logprobs_grad(x, ids, out["max_logit"], out["log_sum"], out["entropy"], g, gh, out=dx)
    for _ in range(3):
        for k in ref:
            if k != "_workspace":
                out[k].fill_(-3)
        dx.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        for k in ref:
            if k != "_workspace":
                for o in (out, other, again):
                    assert torch.equal(ref[k], o[k]), k
        assert torch.equal(dx, rg)


# ---- confident rows ---------------------------------------------------------------------------------------------------

# each kernel and way of dealing rows out: rows in steps by 256, 512 and 1024 threads, rows in parts of four and of eight
# granules per thread
CONFIDENT = [(1100, 777), (300, 4100), (600, 9001), (200, 32003), (60, 128256), (24, 200001), (9, 60001)]


def confident(N, V, dtype, seed):
    """Rows whose largest logit stands by itself, `gap` above the log of the sum of the others: from -1 (no confidence) to 60; a
    few rows about 1000 and -3000, one with the largest twice."""
    x = logits(N, V, torch.float32, seed, std=1.0)
    gap = torch.linspace(-1.0, 60.0, N)
    at = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(seed + 1))
    at[:3] = torch.tensor([0, V - 1, 1])
    x[torch.arange(N), at] = torch.logsumexp(x, 1) + gap
    x[4::9] += 1000.0
    x[6::9] -= 3000.0
    x[N // 2, (at[N // 2] + V // 2) % V] = x[N // 2, at[N // 2]]
    return x.to(dtype)


def above_one(x):
    """(S - 1, sum of e * (M - x)) in 64 bits: one of the largest stays out of the sum."""
    z = x.double()
    M, at = z.max(1, keepdim=True)
    e = (z - M).exp()
    e.scatter_(1, at, 0.0)
    return e.sum(1), torch.where(e > 0, e * (M - z), torch.zeros_like(e)).sum(1)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("n_top", [0, 3, 12])
@pytest.mark.parametrize("N,V", CONFIDENT)
def test_confident_rows_keep_their_relative_precision(sp, N, V, n_top, dtype):
    """log S = log(1 + u), u the sum over all but one of the largest, entropy = log S + (sum of e a) / S, a = M - x: sums of terms
    above 0, so the relative error is that of the terms and of adding up.  A term exp(-a) is formed about a reference up to 8 off
    and moved to M: its exponents, up to a + 16 in all, are each rounded three times (difference, constant, product), which is
    2.5 steps of 2^-24 of them, and two exponentials and their product are 5 steps; rescaled by every rise of the reference, one per
    8 of a lane's spread (four at most here: std 1), 5 steps each.  Adding up: V / 512 + 64 steps.  The logarithm and the division:
    6 steps.  In the sum of e a, a itself is the difference of two such exponents: 3 * (a + 24) steps of 1 more, on the part
    that this sum has of the entropy."""
    x = confident(N, V, dtype, 5)
    u, ua = above_one(x)
    log_sum = torch.log1p(u)
    H = log_sum + ua / (1 + u)
    out = sp.logprobs(x.cuda(), x.argmax(1, keepdim=True).int().cuda(), n_top=n_top)
    got = {k: v.double().cpu() for k, v in out.items() if k != "_workspace"}
    steps = V / 512 + 64 + 2.5 * (ua / u + 16) + 5 * 5 + 6
    assert bool((got["log_sum"] >= 0).all()) and bool((got["entropy"] >= 0).all())
    off = (got["log_sum"] - log_sum).abs() / log_sum
    assert bool((off <= steps * EPS).all()), (float(off.max()), int(off.argmax()))
    off = (got["entropy"] - H).abs()
    lim = (steps * H + 3 * (ua + 24 * u) / (1 + u)) * EPS
    assert bool((off <= lim).all()), (float((off / H).max()), int((off / H).argmax()))
    assert torch.equal(got["logprobs"][:, 0], -got["log_sum"])
    if n_top:
        assert torch.equal(got["top_logprobs"][:, 0], -got["log_sum"])


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("n_top", [0, 3, 12])
@pytest.mark.parametrize("N,V", CONFIDENT)
def test_one_allowed_token_is_certain(sp, N, V, n_top, dtype):
    """As a grammar leaves a row: its log probability, log S and the entropy are 0, whatever the logit."""
    gen = torch.Generator().manual_seed(N)
    x = torch.full((N, V), -INF, dtype=dtype)
    ids = torch.randint(0, V, (N, 1), generator=gen)
    x.scatter_(1, ids, (torch.randn((N, 1), generator=gen) * 10.0 ** torch.linspace(-2, 4, N)[:, None]).to(dtype))
    out = sp.logprobs(x.cuda(), ids.int().cuda(), n_top=n_top)
    for k in ("log_sum", "entropy", "logprobs"):
        assert not bool(out[k].any()), (k, float(out[k].abs().max()))
    assert torch.equal(out["max_logit"].cpu(), x.gather(1, ids)[:, 0].float())
    if n_top:
        assert torch.equal(out["top_ids"][:, :1].cpu().long(), ids) and not bool(out["top_logprobs"][:, 0].any())


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("N,V", CONFIDENT)
def test_the_largest_many_times(sp, N, V, dtype):
    """S is their number where all else is forbidden, and log S and the entropy are its logarithm.  Of fp32 logits every term is
    exactly 1 and S a whole number: 6 steps of the logarithm.  Of fp16 logits the terms and their scale are off by two steps
    each, and adding them up rounds V / 512 + 64 times."""
    gen = torch.Generator().manual_seed(N)
    x = torch.full((N, V), -INF, dtype=dtype)
    count = torch.randint(1, V, (N,), generator=gen)
    count[:3] = torch.tensor([2, 3, V])
    value = (torch.randn((N,), generator=gen) * 30).to(dtype)
    for n in range(N):
        x[n, torch.randperm(V, generator=gen)[:count[n]]] = value[n]
    out = sp.logprobs(x.cuda(), n_top=2)
    want = count.double().log()
    for k in ("log_sum", "entropy"):
        off = (out[k].double().cpu() - want).abs()
        lim = 6 * EPS * want + (0.0 if dtype == torch.float32 else (V / 512 + 64 + 4) * EPS * (count > 1))
        assert bool((off <= lim).all()), (k, float(off.max()))


# ---- gradient ---------------------------------------------------------------------------------------------------------

def plain_grad(x, ids, g, gh):
    want, lp = plain(x, None, 0)
    p = torch.where(lp.isnan(), lp, lp.exp())
    N, V = x.shape
    inside = (ids >= 0) & (ids < V)
    g = torch.where(inside, g.double(), torch.zeros_like(g.double()))
    factor = g.sum(1, keepdim=True).expand(N, V).clone()
    size = g.abs().sum(1, keepdim=True).expand(N, V).clone()
    if gh is not None:
        inner = torch.where(p == 0, torch.zeros_like(lp), lp + want["entropy"][:, None])
        factor += gh.double()[:, None] * inner
        size += gh.double().abs()[:, None] * (torch.where(p == 0, torch.zeros_like(lp), lp).abs() + want["entropy"][:, None])
    hits, sizes = torch.zeros_like(lp), torch.zeros_like(lp)
    for t in range(ids.shape[1]):
        at = ids[:, t:t + 1].clamp(0, V - 1).long()
        hits.scatter_add_(1, at, g[:, t:t + 1])
        sizes.scatter_add_(1, at, g[:, t:t + 1].abs())
    d = hits - p * factor
    empty = want["max_logit"] == -INF
    d[empty] = 0
    return d, p, size, sizes


def check_grad(got, x, ids, g, gh):
    """p is off by (3 |log p| + 64 + what log S is off by) steps; the factor by 64 + 3 of its size (up to 64 ids add up);
    then the difference, and the rounding to the logits' type (2^-11; 2^-25 below the normal numbers).
    A probability below the normal numbers (2^-126) may be 0: off by that much of the factor's size.
    The gradients of an id that repeats are added one after the other: half a step of each sum on the way, which is as large
    as the sum of their sizes, also where the last sum is small.  (-0.8311 and 0.8353 for one id: a sum of 0.0043 that is
    off by up to 2^-25 = 3.0e-8 in whatever order; 1.9e-8 in fp32 on the CPU, where 70 steps of 0.0043 are 1.8e-8.)"""
    d, p, size, hits = plain_grad(x, ids, g, gh)
    got = got.double().cpu()
    assert torch.equal(d.isnan(), got.isnan())
    fine = ~d.isnan()
    lp = torch.where(p > 0, p, torch.ones_like(p)).log().abs()
    steps = (x.shape[1] / 512 + 256 + 6 * lp) * EPS
    lim = (steps * p + 2.0 ** -126) * size + 70 * EPS * hits + 1e-37
    if x.dtype == torch.float16:
        lim = lim + 2.0 ** -11 * d.abs() + 2.0 ** -25
    off = (got - d).abs()
    assert bool((off[fine] <= lim[fine]).all()), float((off - lim)[fine].max())


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("N,V,T", [(1, 1, 1), (2, 3, 2), (3, 50, 64), (60, 777, 4), (1, 32000, 1), (5, 32003, 4),
                                   (2, 128256, 8), (300, 1027, 1), (3, 16385, 0), (600, 1027, 5), (513, 2051, 2),
                                   (520, 3, 1)])
def test_gradient_against_64_bits(sp, N, V, T, entropy, dtype):
    x, ids = logits(N, V, dtype, N + V), tokens(N, V, T, 6)
    gen = torch.Generator().manual_seed(9)
    g, gh = torch.randn((N, T), generator=gen), torch.randn((N,), generator=gen) if entropy else None
    if T > 1:
        ids[:, 1] = ids[:, 0]                     # the same token twice
    if T > 3:
        ids[:, 2], ids[:, 3] = -1, V              # and tokens that are none
    y = x.cuda()
    st = sp.logprobs(y)
    got = sp.logprobs_grad(y, ids.cuda() if T else None, st["max_logit"], st["log_sum"], st["entropy"],
                           g.cuda() if T else None, None if gh is None else gh.cuda())
    check_grad(got, x, ids, g, gh)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("what", sorted(ROWS))
def test_gradient_of_rows_that_are_special(sp, what, dtype):
    x = logits(3, 4099, dtype, 17)
    ROWS[what](x)
    ids = tokens(3, 4099, 3, 5)
    gen = torch.Generator().manual_seed(9)
    g, gh = torch.randn((3, 3), generator=gen), torch.randn((3,), generator=gen)
    y = x.cuda()
    st = sp.logprobs(y)
    got = sp.logprobs_grad(y, ids.cuda(), st["max_logit"], st["log_sum"], st["entropy"], g.cuda(), gh.cuda())
    check_grad(got, x, ids, g, gh)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("T", [0, 3])
@pytest.mark.parametrize("N,V", [(3, 4099), (600, 515), (520, 3)])
@pytest.mark.parametrize("what", sorted(ROWS))
def test_gradient_of_special_rows_without_entropy(sp, what, N, V, T, dtype):
    """The ordinary loss, of log probabilities alone: a row with NaN or +inf has no gradient but NaN, its tokens' too."""
    x = logits(N, V, dtype, 17)
    ROWS[what](x)
    ids = tokens(N, V, T, 5)
    g = torch.randn((N, T), generator=torch.Generator().manual_seed(9))
    y = x.cuda()
    st = sp.logprobs(y)
    got = sp.logprobs_grad(y, ids.cuda() if T else None, st["max_logit"], st["log_sum"], g_logprobs=g.cuda() if T else None)
    check_grad(got, x, ids, g, None)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("repeats", [1, 2, 5])
@pytest.mark.parametrize("N,V", [(600, 515), (40, 515), (60, 32003)])
def test_gradient_of_a_confident_target(sp, N, V, repeats, dtype):
    """The target is the best token, alone or named several times: g (1 - p) there, whose relative error is that of log p
    (test_confident_rows_keep_their_relative_precision) and 6 steps more, and of the sum of the g, which are of one sign."""
    x = confident(N, V, dtype, 7)
    u, ua = above_one(x)
    g = torch.rand((N, repeats), generator=torch.Generator().manual_seed(3)) + 0.5
    ids = x.argmax(1, keepdim=True).int().expand(N, repeats).contiguous()
    y = x.cuda()
    st = sp.logprobs(y)
    got = sp.logprobs_grad(y, ids.cuda(), st["max_logit"], st["log_sum"], g_logprobs=g.cuda()).double().cpu()
    got = got.gather(1, ids[:, :1].long())[:, 0]
    want = g.double().sum(1) * u / (1 + u)
    lim = (V / 512 + 64 + 2.5 * (ua / u + 16) + 5 * 5 + 6 + 6 + repeats) * EPS * want
    if dtype == torch.float16:
        lim = lim + 2.0 ** -11 * want + 2.0 ** -25
    off = (got - want).abs()
    assert bool((off <= lim).all()), (float((off / want).max()), int((off / lim).argmax()))


@gpu
@pytest.mark.parametrize("N,V,dtype", [(800, 32003, torch.float32), (1700, 32000, torch.float16), (30001, 1030, torch.float32),
                                       (26000, 2050, torch.float16)])
def test_gradients_too_large_for_a_cache(sp, N, V, dtype):
    """100 MB and more: stores with the non-temporal hint, of rows by 512 and by 128 threads, in place too."""
    ids = tokens(N, V, 2, 6)
    g = torch.randn((N, 2), generator=torch.Generator().manual_seed(3))
    y = logits(64, V, dtype, 4).cuda().repeat(-(-N // 64), 1)[:N].contiguous()
    st = sp.logprobs(y)
    got = sp.logprobs_grad(y, ids.cuda(), st["max_logit"], st["log_sum"], g_logprobs=g.cuda())
    for rows in (slice(0, 40), slice(N // 2, N // 2 + 40), slice(N - 40, N)):
        check_grad(got[rows], y[rows].cpu(), ids[rows], g[rows], None)
    again = sp.logprobs_grad(y, ids.cuda(), st["max_logit"], st["log_sum"], g_logprobs=g.cuda(), out=y)
    assert again.data_ptr() == y.data_ptr() and torch.equal(again, got)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_gradient_strides_alignments_and_places(sp, dtype):
    N, V = 3, 2053
    x, ids = logits(N, V, dtype, 2), tokens(N, V, 2, 5)
    g = torch.randn((N, 2), generator=torch.Generator().manual_seed(3))
    for pad, opad, off in ((0, 0, 0), (5, 5, 0), (3, 0, 1), (0, 9, 3), (8, 16, 0)):
        buf = torch.full((N * (V + pad),), 1000.0, dtype=dtype, device="cuda")
        y = buf.view(N, V + pad)[:, :V]
        y.copy_(x.cuda())
        obuf = torch.full((off + N * (V + opad),), 7.0, dtype=dtype, device="cuda")
        o = obuf[off:].view(N, V + opad)[:, :V]
        st = sp.logprobs(y)
        got = sp.logprobs_grad(y, ids.cuda(), st["max_logit"], st["log_sum"], g_logprobs=g.cuda(), out=o)
        check_grad(got, x, ids, g, None)
        o.fill_(7.0)
        assert bool((obuf == 7.0).all())          # nothing between the rows was written
        if pad:
            got = sp.logprobs_grad(y, ids.cuda(), st["max_logit"], st["log_sum"], g_logprobs=g.cuda(), out=y)
            check_grad(got, x, ids, g, None)
            y.fill_(1000.0)
            assert bool((buf == 1000.0).all())


@gpu
def test_gradient_against_differences(sp):
    """Central differences of the 64-bit loss, step 1e-5: off by 1e-10 * third derivative (below 10 here), and by the
    kernel's own error."""
    N, V, T = 2, 41, 3
    x, ids = logits(N, V, torch.float32, 12, std=1.0), tokens(N, V, T, 6)
    gen = torch.Generator().manual_seed(9)
    g, gh = torch.randn((N, T), generator=gen).double(), torch.randn((N,), generator=gen).double()

    def loss(z):
        lp = torch.log_softmax(z, 1)
        return float((lp.gather(1, ids.long()) * g).sum() - (gh * (lp.exp() * lp).sum(1)).sum())

    num = torch.empty((N, V), dtype=torch.float64)
    for n in range(N):
        for v in range(V):
            a, b = x.double(), x.double()
            a[n, v] += 1e-5
            b[n, v] -= 1e-5
            num[n, v] = (loss(a) - loss(b)) / 2e-5
    y = x.cuda()
    st = sp.logprobs(y, ids.cuda())
    got = sp.logprobs_grad(y, ids.cuda(), st["max_logit"], st["log_sum"], st["entropy"], g.float().cuda(),
                           gh.float().cuda()).double().cpu()
    assert float((got - num).abs().max()) <= 1e-5


# ---- refusals ---------------------------------------------------------------------------------------------------------

def test_refusals_without_a_gpu(sp):
    import ctypes as C
    lib = sp.lib()
    a, b, odd = C.c_void_p(0x1000), C.c_void_p(0x2000), C.c_void_p(0x1001)
    ll, size = C.c_longlong, C.c_size_t

    def call(V=100, N=1, x=a, h=None, stride=100, ids=a, T=1, top=1, lp=b, tid=b, tlp=b, ws=b, n=1 << 20):
        return lib.specee_logprobs(C.byref(sp.Dims(8, V, 1, 1, 0.0, 0.5)), N, x, h, ll(stride), ids, T, top, lp, b, b, b, tid,
                                   tlp, ws, size(n), None)

    assert call(V=0) == -1 and call(N=-1) == -1 and call(N=65536) == -1 and call(T=-1) == -1 and call(T=65) == -1
    assert call(top=33) == -1 and call(top=-1) == -1 and call(stride=99) == -1
    assert call(x=None) == -1 and call(h=a) == -1 and call(ids=None) == -1 and call(lp=None) == -1
    assert call(tid=None) == -1 and call(tlp=None) == -1
    assert call(x=odd) == -2 and call(x=None, h=odd) == -2
    assert call(N=0, x=None) == 0
    big = dict(V=128256, stride=128256)                                # one row in parts: a workspace is needed
    assert call(**big, ws=None, n=0) == -3 and call(**big, n=16) == -3 and call(**big, ws=C.c_void_p(0x1004)) == -2

    def grad(V=100, N=1, x=a, h=None, stride=100, ids=a, T=1, m=a, s=a, H=a, g=a, gh=None, o=b, oh=None, ostride=100):
        return lib.specee_logprobs_grad(C.byref(sp.Dims(8, V, 1, 1, 0.0, 0.5)), N, x, h, ll(stride), ids, T, m, s, H, g, gh, o,
                                        oh, ll(ostride), None)

    assert grad(V=0) == -1 and grad(N=-1) == -1 and grad(T=65) == -1 and grad(m=None) == -1 and grad(s=None) == -1
    assert grad(ids=None) == -1 and grad(g=None) == -1 and grad(gh=a, H=None) == -1
    assert grad(o=None) == -1 and grad(oh=b) == -1 and grad(o=None, oh=b) == -1 and grad(x=None, h=a) == -1
    assert grad(ostride=99) == -1 and grad(o=odd) == -2
    assert grad(N=2, o=a, ostride=101) == -1                           # in place with another stride
    assert grad(N=0, x=None, o=None) == 0
    with pytest.raises(sp.SpeceeError):
        sp.workspace_bytes(sp.OP_LOGPROBS, sp.Dims(8, 100, 1, 1, 0.0, 0.5), 1, 33)
    assert sp.workspace_bytes(sp.OP_LOGPROBS, sp.Dims(8, 100, 1, 1, 0.0, 0.5), 1, 32) == 0
    assert 0 < sp.workspace_bytes(sp.OP_LOGPROBS, sp.Dims(8, 128256, 1, 1, 0.0, 0.5), 1, 32) < 1 << 14


@pytest.mark.parametrize("n_top", [0, 5, 32])
@pytest.mark.parametrize("V", [100, 60001, 128256, 200001, 262080, 300007])
def test_a_workspace_for_many_rows_serves_fewer(sp, V, n_top):
    dims = sp.Dims(8, V, 1, 1, 0.0, 0.5)
    sizes = [sp.workspace_bytes(sp.OP_LOGPROBS, dims, n, n_top) for n in range(1, 200)]
    assert sizes == sorted(sizes)
    assert sizes[-1] >= sp.workspace_bytes(sp.OP_LOGPROBS, dims, 64, max(n_top - 1, 0))


@gpu
def test_a_workspace_for_many_rows_is_taken_by_fewer(sp):
    V = 128256
    ws = torch.empty(sp.workspace_bytes(sp.OP_LOGPROBS, sp.Dims(8, V, 1, 1, 0.0, 0.5), 4096, 20), dtype=torch.uint8, device="cuda")
    for N, n_top in ((70, 20), (64, 20), (33, 5), (1, 20), (3, 0)):
        for dtype in (torch.float32, torch.float16):
            x = logits(N, V, dtype, N)
            check(sp.logprobs(x.cuda(), n_top=n_top, workspace=ws), x, None, n_top)


@gpu
def test_python_refusals(sp):
    x, ids = torch.zeros((2, 40), device="cuda"), torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    for bad in (x.double(), x.cpu(), x.t(), x[:, ::2], x[:1].expand(2, 40)):
        with pytest.raises(AssertionError):
            sp.logprobs(bad)
    with pytest.raises(AssertionError):
        sp.logprobs(x, ids.long())
    with pytest.raises(AssertionError):
        sp.logprobs(x, ids[:1])
    st = sp.logprobs(x, ids)
    with pytest.raises(AssertionError):
        sp.logprobs_grad(x, ids, st["max_logit"], st["log_sum"])
    with pytest.raises(AssertionError):
        sp.logprobs_grad(x, ids, st["max_logit"], st["log_sum"], g_logprobs=torch.zeros((2, 1), device="cuda"), out=x.half())
    none = sp.logprobs(x[:0], ids[:0], n_top=2)
    assert none["top_ids"].shape == (0, 2)
