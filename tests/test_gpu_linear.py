"""act(x W^T + bias) + resid against float64: few and many rows, odd sizes, strides, both types, every activation."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def make(m, k, n, dtype, seed, bias=True, resid=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    return (rand(m, k).to(dtype), (rand(n, k) * k ** -0.5).to(dtype), rand(n) if bias else None, rand(m, n).to(dtype) if resid else None)


ACTS = {
    "none": lambda t: t,
    "relu": lambda t: t.clamp(min=0),
    "silu": lambda t: t / (1 + (-t).exp()),
    "gelu": lambda t: 0.5 * t * (1 + torch.erf(t / math.sqrt(2))),
    "gelu_tanh": lambda t: 0.5 * t * (1 + torch.tanh(math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3))),
}


def check(y, x, w, bias, resid, act):
    pre = x.double() @ w.double().T + (bias.double() if bias is not None else 0)
    want = ACTS[act](pre) + (resid.double() if resid is not None else 0)
    # fp32 sums of k products and a bias, an ulp of the running sum each (the tensor core truncates): (k + 8) 2^-23 of the magnitudes;
    # the activations' slopes are below 1.2; what they compute is right to 2^-20 of their argument; two more fp32 additions
    mag = x.double().abs() @ w.double().abs().T + (bias.double().abs() if bias is not None else 0)
    bound = torch.finfo(y.dtype).eps / 2 * want.abs() + 1.2 * (x.shape[1] + 8) * 2.0 ** -23 * mag + 2.0 ** -20 * (pre.abs() + want.abs())
    bad = (y.double() - want).abs() / bound.clamp(min=1e-30)
    assert bool((bad <= 1).all()), bad.max().item()


SHAPES = [(1, 64, 16), (1, 4096, 1000), (2, 72, 8), (5, 128, 250), (16, 1024, 24), (37, 512, 4096), (64, 64, 1), (127, 200, 333),
          (128, 256, 256), (129, 264, 130), (300, 1000, 96), (640, 8, 40), (1000, 512, 2000), (2049, 320, 777), (5000, 136, 512)]


@pytest.mark.parametrize("m,k,n", SHAPES)
def test_bf16(dare, m, k, n):
    for act, bias, resid in (("none", True, True), ("silu", False, False)):
        x, w, b, r = make(m, k, n, BF16, m + k + n, bias, resid)
        check(dare.linear(x, w, bias=b, resid=r, act=dare.ACT[act]), x, w, b, r, act)


@pytest.mark.parametrize("m,k,n", SHAPES + [(3, 1, 1), (17, 33, 65), (70, 127, 64), (33, 4, 300)])
def test_f32(dare, m, k, n):
    for act, bias, resid in (("none", True, True), ("gelu", False, False)):
        x, w, b, r = make(m, k, n, F32, m + k + n, bias, resid)
        check(dare.linear(x, w, bias=b, resid=r, act=dare.ACT[act]), x, w, b, r, act)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("m", [1, 40, 400])
def test_activations(dare, dtype, act, m):
    x, w, b, r = make(m, 192, 200, dtype, 7)
    x, b = x * 3, b * 4                                   # arguments from about -20 to 20
    check(dare.linear(x, w, bias=b, resid=r, act=dare.ACT[act]), x, w, b, r, act)


@pytest.mark.parametrize("m,k,n", [(1, 33, 17), (3, 129, 65), (9, 7, 100), (50, 1001, 31), (200, 65, 129)])
def test_bf16_rows_off_the_grid(dare, m, k, n):
    x, w, b, r = make(m, k, n, BF16, 3)
    check(dare.linear(x, w, bias=b, resid=r), x, w, b, r, "none")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [1, 6, 70, 700])
def test_strides(dare, dtype, m):
    x, w, b, r = make(m, 128, 96, dtype, 11)
    want = dare.linear(x, w, bias=b, resid=r, act=dare.ACT["relu"])
    pad = lambda t, extra: torch.cat((t, torch.full((t.shape[0], extra), float("nan"), dtype=t.dtype, device="cuda")), 1)[:, :t.shape[1]]
    for extra in (8, 3):                                  # rows on and off the 16-byte grid
        y = pad(torch.zeros_like(want), extra)
        got = dare.linear(pad(x, extra), pad(w, extra), bias=b, resid=pad(r, extra), act=dare.ACT["relu"], out=y)
        assert got is y
        check(y, x, w, b, r, "relu")
        wide = y.as_strided((m, 96 + extra), (96 + extra, 1))[:, 96:]
        assert bool(wide.isnan().all())                   # nothing behind the rows is written
    # on top of the residual
    acc = r.clone()
    dare.linear(x, w, bias=b, resid=acc, act=dare.ACT["relu"], out=acc)
    assert torch.equal(acc, want)
    # one row for all (stride 0), more dimensions
    same = x[:1].expand(m, -1)
    check(dare.linear(same, w), same, w, None, None, "none")
    assert torch.equal(dare.linear(x.view(1, m, 128), w, bias=b, resid=r.view(1, m, 96), act=dare.ACT["relu"]).view(m, 96), want)
    # bias off the 16-byte grid
    odd = torch.zeros(97, device="cuda")[1:].copy_(b)
    assert torch.equal(dare.linear(x, w, bias=odd, resid=r, act=dare.ACT["relu"]), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [3, 40, 300])
def test_not_numbers_stay_in_their_rows_and_columns(dare, dtype, m):
    x, w, b, _ = make(m, 256, 130, dtype, 13, resid=False)
    want = dare.linear(x, w, bias=b)
    x2, w2 = x.clone(), w.clone()
    x2[1, 5], w2[7, 200], w2[129, 0] = float("inf"), float("nan"), float("-inf")
    got = dare.linear(x2, w2, bias=b)
    rows, cols = [i for i in range(m) if i != 1], [j for j in range(130) if j not in (7, 129)]
    assert torch.equal(got[rows][:, cols], want[rows][:, cols])
    ref = x2.double() @ w2.double().T + b.double()
    assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isinf(), ref.isinf())
    assert torch.equal(got[got.isinf()].double(), ref[ref.isinf()])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [1, 9, 200])
def test_rows_that_overlap_and_short_rows(dare, dtype, m):
    """Inputs whose rows share elements (a sliding window), and rows of one or three elements on the 16-byte grid."""
    g = torch.Generator(device="cuda").manual_seed(23)
    line = torch.randn(8 * m + 64, generator=g, device="cuda").to(dtype)
    x, w = line.as_strided((m, 64), (8, 1)), torch.randn((40, 64), generator=g, device="cuda").to(dtype)
    check(dare.linear(x, w), x, w, None, None, "none")
    check(dare.linear(w, line.as_strided((m, 64), (8, 1))), w, x, None, None, "none")
    for k in (1, 3):
        x, w = (torch.randn((n, 8), generator=g, device="cuda").to(dtype)[:, :k] for n in (m, 40))
        check(dare.linear(x, w), x, w, None, None, "none")


@pytest.mark.parametrize("m,k,n", [(20, 2048, 2048), (128, 8192, 200), (300, 4096, 1024), (601, 1024, 1000), (48, 4164, 130), (33, 516, 65),
                                   (90, 200, 64), (16, 12288, 64), (17, 2052, 500)])
def test_f32_few_tiles(dare, m, k, n):
    """Tiles of fewer rows, k-elements shared by several CTAs; with what is no number in one CTA's part."""
    x, w, b, r = make(m, k, n, F32, m + n)
    y = dare.linear(x, w, bias=b, resid=r, act=dare.ACT["silu"])
    check(y, x, w, b, r, "silu")
    assert torch.equal(dare.linear(x, w, bias=b, resid=r, act=dare.ACT["silu"]), y)
    plain = dare.linear(x, w)
    x[m - 1, k - 1], w[n - 1, 0], x[0, k // 2] = float("inf"), float("nan"), 3e38
    got, ref = dare.linear(x, w), x.double() @ w.double().T
    assert torch.equal(got[1:m - 1, :n - 1], plain[1:m - 1, :n - 1]) and bool(got[:, n - 1].isnan().all())
    assert bool(got[m - 1, :n - 1].isinf().all()) and torch.equal(got[m - 1, :n - 1].sign().double(), ref[m - 1, :n - 1].sign())
    check(got[:1, :n - 1], x[:1], w[:n - 1], None, None, "none")


@pytest.mark.parametrize("m,k,n", [(1, 4096, 6144), (3, 4096, 4096), (8, 12288, 4096), (20, 8200, 1000), (100, 10000, 200), (64, 1032, 1024),
                                   (130, 520, 530), (300, 4096, 1023), (257, 2048, 256), (512, 8192, 1024), (33, 2056, 17)])
def test_bf16_few_tiles(dare, m, k, n):
    """k-elements shared by several CTAs; y on and off the 16-byte grid, on top of the residual; what is no number in one CTA's part."""
    x, w, b, r = make(m, k, n, BF16, m + n)
    y = dare.linear(x, w, bias=b, resid=r, act=dare.ACT["silu"])
    check(y, x, w, b, r, "silu")
    off = torch.full((m, n + 3), 7.0, dtype=BF16, device="cuda")
    off[:, :n] = r
    dare.linear(x, w, bias=b, resid=off[:, :n], act=dare.ACT["silu"], out=off[:, :n])
    assert torch.equal(off[:, :n], y) and bool((off[:, n:] == 7.0).all())
    plain = dare.linear(x, w)
    check(plain, x, w, None, None, "none")
    x[m - 1, k - 1], w[n - 1, 0] = float("inf"), float("nan")
    got, ref = dare.linear(x, w), x.double() @ w.double().T
    assert torch.equal(got[:m - 1, :n - 1], plain[:m - 1, :n - 1]) and bool(got[:, n - 1].isnan().all())
    assert bool(got[m - 1, :n - 1].isinf().all()) and torch.equal(got[m - 1, :n - 1].sign().double(), ref[m - 1, :n - 1].sign())


def test_f32_of_wide_range(dare):
    """The tensor-core form splits operands of any size."""
    g = torch.Generator(device="cuda").manual_seed(17)
    x = torch.randn((600, 512), generator=g, device="cuda") * torch.logspace(-15, 15, 512, device="cuda")
    w = torch.randn((640, 512), generator=g, device="cuda") * torch.logspace(10, -20, 512, device="cuda")
    check(dare.linear(x, w), x, w, None, None, "none")


def test_capture_streams_and_nothing(dare):
    for dtype in (BF16, F32):
        x, w, b, r = make(33, 256, 512, dtype, 19)
        want = dare.linear(x, w, bias=b, resid=r, act=dare.ACT["gelu"])
        outs, side = [], [torch.cuda.Stream() for _ in range(2)]
        for s in side:
            s.wait_stream(torch.cuda.current_stream())
        for _ in range(4):
            for s in side:
                with torch.cuda.stream(s):
                    outs.append(dare.linear(x, w, bias=b, resid=r, act=dare.ACT["gelu"]))
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = dare.linear(x, w, bias=b, resid=r, act=dare.ACT["gelu"])
        x.neg_()
        graph.replay()
        assert torch.equal(y, dare.linear(x, w, bias=b, resid=r, act=dare.ACT["gelu"]))
        assert dare.linear(x[:0], w, bias=b).shape == (0, 512)
