"""GPU checks of matmul_f8 (product in 8-bit floating point with a scale per block of 128) against a plain implementation in
64 bits, of the 8-bit storage, and of what it refuses.

Tolerances.  Every product of two codes is exact.  fp32 results: a block is added up in four matrix steps of 32 products, the
blocks one by one, parts of the elements once more: at most 4 * 33 + 2 * blocks + 64 roundings, each of at most 2^-24 of the sum
of the absolute products.  fp16 results: the 8-bit matrix cores line the products of a block up with the largest one and cut
what lies below; measured on random codes, where it shows most, at most 3.2e-4 of the 2-norm of a block's products: 2^-10 of
it is allowed, and half a step of fp16 (2^-11 of the value, 2^-25 below the normal numbers)."""
import numpy as np
import pytest
import torch

from paper_2504_08850_amd import synth

gpu = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def sp():
    from paper_2504_08850_amd import specee
    specee.lib()
    return specee


def inputs(N, V, d, seed, codes="normal"):
    g = torch.Generator().manual_seed(seed)
    nb, nv = (d + 127) // 128, (V + 127) // 128
    if codes == "normal":
        draw = lambda n: (torch.randn((n, d), generator=g) * 150).clamp(-448, 448).to(F8)
    else:                                             # any code but NaN
        def draw(n):
            c = torch.randint(0, 254, (n, d), generator=g)
            return (c + (c >= 127)).to(torch.uint8).view(F8)
    scale = lambda *s: torch.exp(torch.randn(s, generator=g)) * 1e-2
    return dict(x=draw(N), x_scales=scale(N, nb), weight=draw(V), w_scales=scale(nv, nb))


def plain(t):
    """(out, sum of absolute products, 2-norm of the products), in 64 bits."""
    d, V = t["x"].shape[1], t["weight"].shape[0]
    at, rows = torch.arange(d) // 128, torch.arange(V) // 128
    x = t["x"].float().double() * t["x_scales"].double()[:, at]
    w = t["weight"].float().double() * t["w_scales"].double()[rows][:, at]
    return x @ w.t(), x.abs() @ w.abs().t(), ((x * x) @ (w * w).t()).sqrt()


def up(t):
    return {k: v.cuda() for k, v in t.items()}


def check(out, t, want=None):
    ref, size, norm = plain(t) if want is None else want
    d = t["x"].shape[1]
    off = (out.double().cpu() - ref).abs()
    lim = (132 + 2 * (d // 128 + 1) + 64) * 2.0 ** -24 * size
    if out.dtype == torch.float16:
        lim = lim + 2.0 ** -10 * norm + 2.0 ** -11 * ref.abs() + 2.0 ** -25
        # what rounds to 2^16 or more (from 65520 on) is an infinity of its sign in fp16
        over, under = ref.abs() - lim >= 65520, ref.abs() + lim < 65520
        assert torch.equal(out.cpu()[over].double(), torch.sign(ref[over]) * torch.inf)
        out, off, lim = out.cpu()[under], off[under], lim[under]
    assert bool(out.isfinite().all()) and bool((off <= lim).all()), float((off / lim.clamp_min(1e-300)).max())


SHAPES = [(1, 1, 16), (1, 128, 128), (2, 129, 144), (1, 1000, 4096), (3, 300, 32), (5, 3, 1040), (16, 515, 1024), (17, 127, 112),
          (31, 257, 2048), (33, 777, 528), (60, 1000, 640), (64, 128, 256), (65, 130, 272), (127, 1, 128), (128, 128, 128),
          (129, 129, 129 * 16), (200, 650, 400), (257, 513, 384), (300, 1025, 1536), (520, 260, 144), (1, 40, 16384),
          (20, 33, 28672), (4, 4099, 512), (1, 20011, 4112), (700, 1, 16), (1024, 1024, 1024),
          (33, 33024, 272), (60, 50281, 400), (40, 99000, 272), (64, 131072, 144), (50, 130050, 144), (64, 33001, 1040), (100, 40003, 272), (128, 33030, 528), (70, 31001, 144),
          (2100, 1100, 272), (4200, 2100, 144), (4000, 3100, 272)]


@gpu
@pytest.mark.parametrize("N,V,d", SHAPES)
def test_against_64_bits(sp, N, V, d):
    t = inputs(N, V, d, N + V + d)
    want = plain(t)
    for dtype in (torch.float32, torch.float16):
        out = sp.matmul_f8(**up(t), dtype=dtype)["out"]
        assert out.dtype == dtype
        check(out, t, want)


# every form of tile through at least six blocks of elements, so that loads run ahead of the products, wait their turn and go
# round, in one part and in several; with a whole last block and with a short one
STEADY = [(500, 1100, 4112), (600, 300, 16384), (60, 24001, 4608), (40, 8192, 8192), (50, 16500, 2064), (64, 131072, 768),
          (64, 131072, 784), (50, 33010, 784), (100, 8192, 8192), (100, 9001, 4112), (100, 33010, 784), (300, 5120, 5120),
          (200, 5200, 5136), (130, 12300, 2576), (4200, 2100, 1024), (4200, 2100, 1040), (4000, 3100, 1024), (4000, 3100, 1040),
          (2900, 2000, 16400), (2100, 2048, 12304)]


@gpu
@pytest.mark.parametrize("N,V,d", STEADY)
def test_many_blocks_in_every_form(sp, N, V, d):
    t = inputs(N, V, d, 11)
    on = up(t)
    want = tuple(v.cpu() for v in plain(on))
    for dtype in (torch.float32, torch.float16):
        check(sp.matmul_f8(**on, dtype=dtype)["out"], t, want)


@gpu
@pytest.mark.parametrize("N,V,d", [(60, 24001, 4608), (40, 8192, 8192), (64, 131072, 784), (100, 9001, 4112), (300, 5120, 5120),
                                   (4200, 2100, 1040), (4000, 3100, 1040)])
def test_many_blocks_give_the_same_bits_in_graphs(sp, N, V, d):
    t = up(inputs(N, V, d, 12))
    for dtype in (torch.float32, torch.float16):
        ref = sp.matmul_f8(**t, dtype=dtype)["out"].clone()
        kept = sp.matmul_f8(**t, dtype=dtype)
        assert torch.equal(ref, kept["out"])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sp.matmul_f8(**t, dtype=dtype, out=kept["out"], workspace=kept["_workspace"])
        for _ in range(3):
            kept["out"].fill_(3)
            kept["_workspace"].fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(ref, kept["out"])


@gpu
@pytest.mark.parametrize("N,V,d", [(1, 300, 4096), (16, 260, 1040), (40, 129, 528), (130, 257, 1168), (300, 300, 2048)])
def test_every_code(sp, N, V, d):
    t = inputs(N, V, d, 5, codes="any")
    t["x_scales"] *= 0.1                               # fp16 results stay below 65504
    t["w_scales"] *= 0.01
    want = plain(t)
    for dtype in (torch.float32, torch.float16):
        check(sp.matmul_f8(**up(t), dtype=dtype)["out"], t, want)


@gpu
@pytest.mark.parametrize("N,V,d", [(1, 257, 272), (16, 130, 400), (70, 300, 144), (257, 257, 272), (50, 33010, 400),
                                   (100, 33010, 400), (2100, 1100, 272), (4000, 3100, 272)])
def test_each_scale_reaches_its_own_block(sp, N, V, d):
    """One code of 1 per row of x, all weights 1: every output is one product of two scales, exactly."""
    nb, nv = (d + 127) // 128, (V + 127) // 128
    at = (torch.arange(N) * 37) % d
    x = torch.zeros((N, d))
    x[torch.arange(N), at] = 1.0
    t = dict(x=x.to(F8), weight=torch.ones((V, d)).to(F8), x_scales=2.0 ** (torch.arange(N * nb) % 7).float().view(N, nb),
             w_scales=2.0 ** -(torch.arange(nv * nb) % 5).float().view(nv, nb))
    want = t["x_scales"][torch.arange(N), at // 128][:, None] * t["w_scales"][:, at // 128].t().repeat_interleave(128, 1)[:, :V]
    for dtype in (torch.float32, torch.float16):
        assert torch.equal(sp.matmul_f8(**up(t), dtype=dtype)["out"].float().cpu(), want)


@gpu
@pytest.mark.parametrize("N", [1, 16, 60, 130, 300])
def test_a_nan_reaches_its_row_or_column_alone_and_neighbours_are_left(sp, N):
    V, d = 260, 400
    t = inputs(N, V, d, 9)
    t["x"].view(torch.uint8)[N - 1, 399] = 0x7f
    t["weight"].view(torch.uint8)[130, 0] = 0xff
    for dtype in (torch.float32, torch.float16):
        buf = torch.full((N + 3, V), 7.0, dtype=dtype, device="cuda")
        got = sp.matmul_f8(**up(t), dtype=dtype, out=buf[:N])["out"].isnan().cpu()
        want = torch.zeros((N, V), dtype=torch.bool)
        want[N - 1] = True
        want[:, 130] = True
        assert torch.equal(got, want) and bool((buf[N:] == 7).all())


@gpu
@pytest.mark.parametrize("N,V,d", [(1, 4096, 4096), (16, 1030, 2048), (60, 2100, 1040), (300, 300, 528), (50, 33010, 400),
                                   (2100, 1100, 528), (4000, 3100, 272)])
def test_same_bits_graphs_and_streams(sp, N, V, d):
    t = up(inputs(N, V, d, 3))
    for dtype in (torch.float32, torch.float16):
        ref = sp.matmul_f8(**t, dtype=dtype)["out"].clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        other = sp.matmul_f8(**t, dtype=dtype, stream=side)     # beside the next call, with a workspace of its own
        kept = sp.matmul_f8(**t, dtype=dtype)
        torch.cuda.synchronize()
        assert torch.equal(ref, other["out"]) and torch.equal(ref, kept["out"])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sp.matmul_f8(**t, dtype=dtype, out=kept["out"], workspace=kept["_workspace"])
        for _ in range(3):
            kept["out"].fill_(3)
            kept["_workspace"].fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(ref, kept["out"])


@pytest.mark.parametrize("V,d", [(1, 16), (300, 4096), (1000, 65536), (4096, 4096), (5120, 5120), (8192, 8192), (24001, 4608),
                                 (50280, 2048), (128256, 8192)])
def test_a_workspace_for_many_states_serves_fewer(sp, V, d):
    dims = sp.Dims(d, V, 1, 1, 0.0, 0.5)
    sizes = [sp.workspace_bytes(sp.OP_MATMUL_F8, dims, n) for n in list(range(1, 700)) + [1000, 2043, 4096, 8192, 40000]]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("d", [1296, 2576, 5136])
def test_parts_are_whole_quads(sp, d):
    """Results in parts are stored 16 bytes at a time: also where N V is odd each part begins at a multiple of them."""
    for V in (65, 129, 131, 515):
        for N in (17, 33, 61, 127, 129):
            assert sp.workspace_bytes(sp.OP_MATMUL_F8, sp.Dims(d, V, 1, 1, 0.0, 0.5), N) % 16 == 0


@gpu
@pytest.mark.parametrize("N,V,d", [(17, 129, 1296), (61, 131, 2576), (129, 515, 5136), (3, 129, 9360)])
def test_parts_of_an_odd_number_of_results(sp, N, V, d):
    t = inputs(N, V, d, 2)
    want = plain(t)
    for dtype in (torch.float32, torch.float16):
        check(sp.matmul_f8(**up(t), dtype=dtype)["out"], t, want)


@gpu
def test_a_workspace_for_many_states_is_taken_by_fewer(sp):
    V, d = 1100, 2064
    ws = torch.empty(sp.workspace_bytes(sp.OP_MATMUL_F8, sp.Dims(d, V, 1, 1, 0.0, 0.5), 8192), dtype=torch.uint8, device="cuda")
    for N in (8192, 1, 16, 17, 40, 64, 100, 200, 700):
        t = inputs(N, V, d, N)
        for dtype in (torch.float32, torch.float16):
            check(sp.matmul_f8(**up(t), dtype=dtype, workspace=ws)["out"], t)


@gpu
def test_weights_beyond_32_bits(sp):
    """The last rows of 4.3 GB of weights, and of 4.3 GB of states."""
    d, big = 16384, 262400
    t = inputs(2, 128, d, 4)
    w = torch.zeros((big, d), dtype=torch.uint8, device="cuda")
    w[-128:] = t["weight"].view(torch.uint8).cuda()
    scales = torch.ones((big // 128, d // 128), device="cuda")
    scales[-1] = t["w_scales"].cuda()[0]
    u = up(t)
    want = plain(t)
    out = sp.matmul_f8(u["x"], u["x_scales"], w.view(F8), scales)["out"]
    assert not bool(out[:, :-128].any())
    check(out[:, -128:], t, want)
    rows = torch.ones((big, d // 128), device="cuda")            # and the other way round: many states, few outputs
    rows[-128:] = t["w_scales"].cuda()
    out = sp.matmul_f8(w.view(F8), rows, u["x"], torch.ones((1, d // 128), device="cuda"), dtype=torch.float16)["out"]
    assert not bool(out[:-128].any())
    back = dict(x=t["weight"], x_scales=t["w_scales"].expand(128, -1), weight=t["x"], w_scales=torch.ones((1, d // 128)))
    check(out[-128:], back)


@gpu
@pytest.mark.parametrize("N", [1, 7, 60, 200])
def test_a_block_then_its_head_then_the_answer(sp, N):
    """The operators as they are used: the block's end writes the state and its 8-bit form, the head reads that, and the answer
    is read off the logits; each against 64 bits from what the one before it wrote."""
    d, V, T, n_top = 1040, 1003, 4, 5
    g = torch.Generator().manual_seed(N)
    half = lambda *s, std=1.0, mean=0.0: (mean + std * torch.randn(s, generator=g)).half()
    hidden, branch, gamma, post = half(N, d), half(N, d, std=2.0), half(d, std=0.1, mean=1.0), half(d, std=0.1, mean=1.0)
    w, ws = synth.quantize_f8(half(V, d, std=0.08).numpy().astype(np.float32))
    w, ws = torch.from_numpy(w).view(F8), torch.from_numpy(ws)
    s = sp.block_norm(hidden.cuda(), gamma.cuda(), branch=branch.cuda(), gamma_post=post.cuda(), want_x=False, want_f8=True)
    z = sp.matmul_f8(s["x8"], s["x8_scales"], w.cuda(), ws.cuda())["out"]
    ids = torch.randint(0, V, (N, T), generator=g, dtype=torch.int32)
    a = sp.logprobs(z, ids.cuda(), n_top=n_top)
    # the state's own predictor reads the same row
    got = sp.lm_head_gemv(s["hidden"], gamma.cuda(), half(16, d).cuda())
    assert bool(got.isfinite().all())
    t = dict(x=s["x8"].cpu(), x_scales=s["x8_scales"].cpu(), weight=w, w_scales=ws)
    check(z, t)
    lp = torch.log_softmax(z.double().cpu(), 1)
    assert float((a["logprobs"].double().cpu() - lp.gather(1, ids.long())).abs().max()) <= 1e-5
    assert torch.equal(a["top_ids"].cpu().long(), torch.argsort(z.cpu(), dim=1, descending=True, stable=True)[:, :n_top])
    # and against the head without any 8-bit form: x and w are each off by at most 2^-4, on average a third of that
    b = branch.double()
    full = hidden.double() + b / (b.pow(2).mean(1, keepdim=True) + 1e-5).sqrt() * post.double()
    full = full / (full.pow(2).mean(1, keepdim=True) + 1e-5).sqrt() * gamma.double()
    wide = torch.from_numpy(np.repeat(np.repeat(ws.numpy(), 128, 0)[:V], 128, 1)[:, :d])
    exact = full @ (w.float() * wide).double().t()
    assert float((z.double().cpu() - exact).norm() / exact.norm()) <= 2.0 ** -4
    dz = sp.logprobs_grad(z, ids.cuda(), a["max_logit"], a["log_sum"], g_logprobs=torch.ones((N, T), device="cuda"))
    want = -T * lp.exp()
    for k in range(T):
        want.scatter_add_(1, ids[:, k:k + 1].long(), torch.ones((N, 1), dtype=torch.float64))
    assert float((dz.double().cpu() - want).abs().max()) <= 1e-5


# ---- storage and refusals, without a GPU ------------------------------------------------------------------------------

def test_synthetic_storage_is_e4m3():
    codes = np.arange(256, dtype=np.uint8)
    v = torch.from_numpy(codes).view(F8).float().numpy()
    fine = ~np.isnan(v)
    assert np.array_equal(synth.e4m3(v[fine]), codes[fine])
    r = np.concatenate([np.linspace(-460, 460, 20011), np.geomspace(1e-5, 448, 4001)]).astype(np.float32)
    want = torch.from_numpy(np.clip(r, -448, 448)).to(F8).view(torch.uint8).numpy()
    assert np.array_equal(synth.e4m3(r), want)
    w = np.random.default_rng(1).standard_normal((130, 200)).astype(np.float32)
    w[:128, 128:] = 0
    q, s = synth.quantize_f8(w)
    assert q.shape == w.shape and s.shape == (2, 2) and s[0, 1] == 1.0 and q.dtype == np.uint8
    back = torch.from_numpy(q).view(F8).float().numpy() * np.repeat(np.repeat(s, 128, 0)[:130], 128, 1)[:, :200]
    assert np.all(np.abs(back - w) <= np.abs(w) * 2.0 ** -4 * 1.0001 + np.repeat(np.repeat(s, 128, 0)[:130], 128, 1)[:, :200] * 2.0 ** -10)


@pytest.mark.parametrize("size", [1e-45, 1e-42, 1e-38, 1e-35, 3e38])
def test_synthetic_storage_of_blocks_at_the_ends_of_fp32(size):
    w = (np.random.default_rng(2).uniform(-1, 1, (3, 256)) * size).astype(np.float32)
    w[0, 0] = w[1, 200] = size
    q, s = synth.quantize_f8(w)
    wide = np.repeat(np.repeat(s, 128, 0)[:3], 128, 1).astype(np.float64)
    back = torch.from_numpy(q).view(F8).float().numpy().astype(np.float64) * wide
    assert np.isfinite(s).all() and (s >= np.finfo(np.float32).tiny).all()
    assert np.all(np.abs(back - w) <= np.abs(w) * 2.0 ** -4 * 1.0001 + wide * 2.0 ** -10)


def test_refusals_without_a_gpu(sp):
    import ctypes as C
    lib = sp.lib()
    a, odd, size = C.c_void_p(0x1000), C.c_void_p(0x1008), C.c_size_t

    def call(d=128, V=64, N=1, x=a, xs=a, w=a, ws=a, out=a, h=None, wk=a, n=1 << 40):
        return lib.specee_matmul_f8(C.byref(sp.Dims(d, V, 1, 1, 0.0, 0.5)), N, x, xs, w, ws, out, h, wk, size(n), None)

    assert call(d=24) == -1 and call(d=0) == -1 and call(d=65552) == -1 and call(V=0) == -1 and call(N=-1) == -1
    assert call(x=None) == -1 and call(xs=None) == -1 and call(w=None) == -1 and call(ws=None) == -1
    assert call(out=None) == -1 and call(h=a) == -1
    assert call(x=odd) == -2 and call(w=odd) == -2 and call(out=odd) == -2 and call(wk=odd) == -2
    assert call(N=0, x=None, out=None) == 0
    assert sp.workspace_bytes(sp.OP_MATMUL_F8, sp.Dims(4096, 4096, 1, 1, 0.0, 0.5), 0) == 0
    with pytest.raises(sp.SpeceeError):
        sp.workspace_bytes(sp.OP_MATMUL_F8, sp.Dims(24, 64, 1, 1, 0.0, 0.5), 1)


@gpu
def test_python_refusals(sp):
    t = up(inputs(4, 130, 256, 1))
    for k, bad in (("x", t["x"].float()), ("x_scales", t["x_scales"][:, :1]), ("w_scales", t["w_scales"][:1]),
                   ("weight", t["weight"][:, :128]), ("x", t["x"].cpu()), ("x_scales", t["x_scales"].half()),
                   ("weight", t["weight"].view(torch.uint8))):
        with pytest.raises(AssertionError):
            sp.matmul_f8(**dict(t, **{k: bad}))
    with pytest.raises(AssertionError):
        sp.matmul_f8(**t, out=torch.empty((4, 130), dtype=torch.float16, device="cuda"))
    with pytest.raises(AssertionError):
        sp.matmul_f8(**t, dtype=torch.bfloat16)
    empty = sp.matmul_f8(t["x"][:0], t["x_scales"][:0], t["weight"], t["w_scales"])
    assert empty["out"].shape == (0, 130)
