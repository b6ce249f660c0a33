"""GPU checks of block_norm (norms around a block with its gate and residual scale) against a plain implementation in
64 bits, and of what it refuses.

Tolerances.  A rounding to fp16 is off by half a step, 2^-11 of the value (2^-25 below the normal numbers), one to e4m3 by
2^-4 (2^-10 of the scale below them).  In fp32 a row's mean of squares adds d terms over 8 or 16 of a lane, six steps of a
wavefront and up to 16 of a workgroup: at most 38 roundings, half of which reach the root; every factor and sum adds one.
64 * 2^-24 of the sizes that are added is above all of that."""
import pytest
import torch

gpu = pytest.mark.gpu
F32 = 64 * 2.0 ** -24


@pytest.fixture(scope="module")
def sp():
    from paper_2504_08850_amd import specee
    specee.lib()
    return specee


def inputs(N, d, seed, gate="none", post=True, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0, mean=0.0: (mean + std * torch.randn(s, generator=g)).half()
    return dict(hidden=n(N, d, std=spread), branch=n(N, d, std=3.0), gamma=n(d, std=0.1, mean=1.0),
                gamma_post=n(d, std=0.1, mean=1.0) if post else None,
                gate={"none": None, "all": n(d, std=0.5), "each": n(N, d, std=0.5)}[gate])


def plain(t, hidden_scale=1.0, branch_scale=1.0, eps=1e-5):
    """(s, size of what is added into s, x) in 64 bits."""
    def r(v):
        return 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)

    h = hidden_scale * t["hidden"].double()
    if t["branch"] is None:
        s, size = h, h.abs()
    else:
        b = t["branch"].double()
        if t["gamma_post"] is not None:
            b = b * r(b) * t["gamma_post"].double()
        if t["gate"] is not None:
            b = b * t["gate"].double()
        s, size = h + branch_scale * b, h.abs() + (branch_scale * b).abs()
    if t["gamma"] is None:
        return s, size, None, None
    return s, size, s * r(s) * t["gamma"].double(), size * r(s) * t["gamma"].double().abs()


def up(t):
    return {k: None if v is None else v.cuda() for k, v in t.items()}


def check(out, s, size, x, xsize, f8):
    off = (out["hidden"].double().cpu() - s).abs()
    assert bool((off <= 2.0 ** -11 * s.abs() + 2.0 ** -25 + F32 * size).all()), off.max()
    if "x" in out:
        off = (out["x"].double().cpu() - x).abs()
        assert bool((off <= 2.0 ** -11 * x.abs() + 2.0 ** -25 + F32 * (xsize + x.abs())).all()), off.max()
    if f8:
        N, d = x.shape
        nb = (d + 127) // 128
        slack = F32 * (xsize + x.abs())
        pad = lambda v: torch.nn.functional.pad(v, (0, nb * 128 - d)).view(N, nb, 128)
        scales = out["x8_scales"].double().cpu()
        top, most = pad(x.abs()).amax(2), pad(slack).amax(2)
        want = torch.where(top > 0, top / 448, torch.ones_like(top))
        assert bool(((scales - want).abs() <= most / 448 + 2.0 ** -23 * want).all())
        codes = pad(out["x8"].float().double().cpu())
        off = (codes * scales[..., None] - pad(x)).abs()
        assert bool((off <= 2.0 ** -4 * pad(x.abs()) * (1 + 2.0 ** -20) + 2.0 ** -10 * scales[..., None] + pad(slack)).all())
        assert float(codes.abs().max()) <= 448


@gpu
@pytest.mark.parametrize("N,d", [(1, 8), (3, 16), (2, 120), (1, 128), (5, 136), (3, 520), (7, 1032), (60, 2056), (1, 4096),
                                 (33, 5120), (2, 8192), (3, 8200), (1, 16384), (2000, 1032)])
@pytest.mark.parametrize("post,gate", [(True, "none"), (False, "all"), (True, "each")])
def test_against_64_bits(sp, N, d, post, gate):
    t = inputs(N, d, 7 * N + d, gate, post)
    out = sp.block_norm(**up(t), hidden_scale=0.75, branch_scale=-1.5, want_f8=True)
    check(out, *plain(t, 0.75, -1.5), True)


@gpu
@pytest.mark.parametrize("want_x,want_f8", [(False, False), (True, False), (False, True)])
def test_outputs_that_are_not_asked_for_are_not_there(sp, want_x, want_f8):
    t = inputs(5, 264, 3)
    out = sp.block_norm(**up(t), want_x=want_x, want_f8=want_f8)
    assert set(out) == {"hidden"} | ({"x"} if want_x else set()) | ({"x8", "x8_scales"} if want_f8 else set())
    check(out, *plain(t), want_f8)


@gpu
def test_without_branch_or_weight(sp):
    t = inputs(4, 1032, 5)
    t["branch"] = t["gamma_post"] = None
    check(sp.block_norm(**up(t), hidden_scale=0.5, want_f8=True), *plain(t, 0.5), True)
    t = dict(inputs(4, 1032, 6, "all"), gamma=None)
    check(sp.block_norm(**up(t), branch_scale=2.0), *plain(t, 1.0, 2.0), False)


@gpu
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), 3.0])
def test_without_a_branch_its_scale_means_nothing(sp, scale):
    t = inputs(4, 1032, 5)
    t["branch"] = t["gamma_post"] = None
    check(sp.block_norm(**up(t), branch_scale=scale, want_f8=True), *plain(t), True)


@gpu
def test_rows_of_zeros_and_far_apart_sizes(sp):
    t = inputs(6, 512, 8)
    t["hidden"][2] = 0
    t["branch"][2] = 0
    t["hidden"][3, 128:256] = 0
    t["branch"][3, 128:256] = 0          # a block of zeros in a row that is none
    t["hidden"][4] *= 2.0 ** -14
    t["branch"][4] *= 2.0 ** -14
    t["hidden"][5, 7] = 60000.0          # one outlier channel
    out = sp.block_norm(**up(t), want_f8=True)
    check(out, *plain(t), True)
    assert bool((out["x8_scales"][2] == 1).all()) and float(out["x8_scales"][3, 1]) == 1.0
    assert not bool(out["x8"][2].float().any()) and not bool(out["x"][2].any())


@gpu
def test_in_place_and_outputs_kept(sp):
    t = inputs(9, 2056, 10, "each")
    ref = sp.block_norm(**up(t), want_f8=True)
    u = up(t)
    out = dict(hidden=u["hidden"], x=u["branch"], x8=torch.empty_like(ref["x8"]), x8_scales=torch.empty_like(ref["x8_scales"]))
    got = sp.block_norm(**u, want_f8=True, out=out)
    assert got is out and out["hidden"].data_ptr() == u["hidden"].data_ptr()
    for k in ref:
        assert torch.equal(ref[k].float(), got[k].float()), k


# more rows than the GPU holds workgroups for: two to ten turns of each, the last of them uneven
TURNS = [(600, 16384), (1300, 8200), (2500, 5120), (5001, 4096), (12001, 1032), (41000, 128)]


@gpu
@pytest.mark.parametrize("N,d", TURNS)
@pytest.mark.parametrize("post,gate", [(True, "none"), (False, "all"), (True, "each"), (None, "none")])
def test_several_rows_per_workgroup(sp, N, d, post, gate):
    t = inputs(N, d, N + d, gate, bool(post))
    if post is None:
        t["branch"] = None
    want = plain(t, 0.75, -1.5)
    for asked in (dict(want_f8=True), dict(want_x=False)):
        out = sp.block_norm(**up(t), hidden_scale=0.75, branch_scale=-1.5, **asked)
        check(out, *want, "want_f8" in asked)


@gpu
@pytest.mark.parametrize("N,d", TURNS)
@pytest.mark.parametrize("gate", ["none", "each"])
def test_several_rows_per_workgroup_in_place(sp, N, d, gate):
    t = inputs(N, d, 3, gate)
    ref = sp.block_norm(**up(t), want_f8=True)
    for a, b in (("hidden", "branch"), ("branch", "hidden")):      # where the new state and x go
        u = up(t)
        out = dict(hidden=u[a], x=u[b], x8=torch.empty_like(ref["x8"]), x8_scales=torch.empty_like(ref["x8_scales"]))
        sp.block_norm(**u, want_f8=True, out=out)
        for k in ref:
            assert torch.equal(ref[k].view(torch.uint8), out[k].view(torch.uint8)), (k, a)


@gpu
def test_neighbouring_memory_is_left_alone(sp):
    N, d = 3, 136
    t = up(inputs(N, d, 11))
    buf = torch.full((N + 2, d), 7.0, dtype=torch.float16, device="cuda")
    x8 = torch.full((N + 2, d), 7, dtype=torch.uint8, device="cuda")
    scales = torch.full((N + 2, 2), 7.0, device="cuda")
    out = dict(hidden=torch.empty((N, d), dtype=torch.float16, device="cuda"), x=buf[:N],
               x8=x8.view(torch.float8_e4m3fn)[:N], x8_scales=scales[:N])
    sp.block_norm(**t, want_f8=True, out=out)
    assert bool((buf[N:] == 7).all()) and bool((x8[N:] == 7).all()) and bool((scales[N:] == 7).all())


@gpu
def test_nan_and_infinity_stay_in_their_rows_and_blocks(sp):
    N, d = 3, 384
    h = torch.randn((N, d), generator=torch.Generator().manual_seed(1)).half()
    h[0, 5] = float("nan")
    h[1, 200] = float("inf")
    gamma = torch.ones(d).half()
    gamma[130] = float("inf")
    out = {k: v.float().cpu() for k, v in sp.block_norm(h.cuda(), gamma.cuda(), want_f8=True).items()}
    assert bool(out["x"][0].isnan().all()) and bool(out["x8"][0].isnan().all())     # the norm of a row with NaN
    assert bool(out["x"][1, 200].isnan()) and bool(out["x8"][1, 200].isnan())       # inf * 0
    values = out["x8"][2] * out["x8_scales"][2].repeat_interleave(128)
    assert bool(values[128:256].isnan().all()) and bool(values[:128].isfinite().all()) and bool(values[256:].isfinite().all())


@gpu
def test_graph_replays_and_other_streams(sp):
    t = up(inputs(17, 1032, 12, "all"))
    ref = {k: v.float().clone() for k, v in sp.block_norm(**t, want_f8=True).items()}
    out = sp.block_norm(**t, want_f8=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = sp.block_norm(**t, want_f8=True, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.block_norm(**t, want_f8=True, out=out)
    for _ in range(3):
        for v in out.values():
            v.view(torch.uint8).fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        for k in ref:
            assert torch.equal(ref[k], out[k].float()) and torch.equal(ref[k], other[k].float()), k


def test_refusals_without_a_gpu(sp):
    import ctypes as C
    lib = sp.lib()
    a, b, odd = C.c_void_p(0x1000), C.c_void_p(0x2000), C.c_void_p(0x1008)
    f = C.c_float

    def call(d=64, N=1, eps=1e-5, hidden=a, branch=a, post=a, gate=None, rows=0, gamma=a, out=b, x=None, x8=None, xs=None):
        return lib.specee_block_norm(C.byref(sp.Dims(d, 1, 1, 1, eps, 0.5)), N, hidden, branch, post, gate, rows, f(1), f(1),
                                     gamma, out, x, x8, xs, None)

    assert call(d=12) == -1 and call(d=0) == -1 and call(d=16392) == -1 and call(eps=-1.0) == -1 and call(N=-1) == -1
    assert call(N=0, hidden=None) == 0
    assert call(hidden=None) == -1 and call(out=None) == -1
    assert call(branch=None) == -1 and call(branch=None, post=None, gate=a, rows=1) == -1
    assert call(gate=a, rows=2, N=3) == -1 and call(gate=a, rows=0) == -1
    assert call(x8=a) == -1 and call(xs=a) == -1 and call(gamma=None, x=a) == -1
    assert call(x=b) == -1                                            # x in the place of hidden_out
    assert call(hidden=odd) == -2 and call(x=odd) == -2 and call(gate=odd, rows=1) == -2 and call(gamma=odd) == -2


@gpu
def test_python_refusals(sp):
    t = up(inputs(3, 64, 1))
    with pytest.raises(AssertionError):
        sp.block_norm(t["hidden"].cpu(), t["gamma"])
    with pytest.raises(AssertionError):
        sp.block_norm(t["hidden"].float(), t["gamma"])
    with pytest.raises(AssertionError):
        sp.block_norm(**dict(t, gate=torch.zeros((2, 64), dtype=torch.float16, device="cuda")))
    with pytest.raises(AssertionError):
        sp.block_norm(**dict(t, gamma=t["gamma"][:32]))
    with pytest.raises(AssertionError):
        sp.block_norm(**dict(t, branch=t["branch"][:2]))
    with pytest.raises(sp.SpeceeError):
        sp.block_norm(t["hidden"], t["gamma"], gamma_post=t["gamma"])
    empty = sp.block_norm(t["hidden"][:0], t["gamma"], want_f8=True)
    assert empty["x8"].shape == (0, 64) and empty["x8_scales"].shape == (0, 1)
