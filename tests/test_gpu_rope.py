"""Rotary positions against float64: tables with every scaling, both layouts, parts of heads, strides, the way back."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def frequencies(r, theta, scaling, s, trained, low, high):
    """The header's formulas, pair by pair."""
    if scaling == "base":
        theta = theta * s ** (r / (r - 2))
    f = []
    if scaling == "index":
        at = lambda turns: r * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(theta))
        first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), r - 1)
    for j in range(r // 2):
        fj = theta ** (-2 * j / r)
        if scaling == "linear":
            fj /= s
        elif scaling == "turns":
            keep = min(max((trained * fj / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            fj = keep * fj + (1 - keep) * fj / s
        elif scaling == "index":
            keep = 1 - min(max((j - first) / max(last - first, 1e-3), 0.0), 1.0)
            fj = keep * fj + (1 - keep) * fj / s
        f.append(fj)
    return torch.tensor(f, dtype=torch.float64)


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "turns", "index"])
@pytest.mark.parametrize("positions,r", [(1, 2), (17, 58), (5000, 128), (131072, 64), (33, 256)])
def test_table(dare, scaling, positions, r):
    if scaling == "base" and r == 2:
        pytest.skip("no base scaling of a single pair (refused, below)")
    t = dare.rope_table(positions, r, 5e5, scaling=dare.ROPE_SCALE[scaling], factor=8.0, trained=4096, low=1.0, high=32.0,
                        magnitude=1.25)
    a = torch.outer(torch.arange(positions, dtype=torch.float64), frequencies(r, 5e5, scaling, 8.0, 4096, 1.0, 32.0))
    want = torch.stack((a.cos(), a.sin()), -1) * 1.25
    # rounding to fp32: half an ulp of values up to 1.25, 2^-24 (below 1) or 2^-23 * 1.25 / 2; the angles' own error: two
    # roundings of the frequency and one of the product, 3 * 2^-53 * 131072 < 2^-34
    assert (t.double().cpu() - want).abs().max().item() <= 2.0 ** -24 * 1.25 + 2.0 ** -33


def oracle(x, table, pos, r, layout, transpose):
    x, cs = x.double(), table.double()[pos.long()]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1] * (-1 if transpose else 1)
    y = x.clone()
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, b * c + a * s
    return y


def close(y, want, x, mag):
    # two products and a sum in fp32: 3 * 2^-24 of |a c| + |b s| <= sqrt(2) |x| mag; then the rounding to the type
    bound = torch.finfo(y.dtype).eps / 2 * want.abs() + 8 * 2.0 ** -24 * mag * x.double().abs().max()
    return bool(((y.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,hd,r", [(1, 1, 2, 2), (1, 40, 128, 128), (7, 5, 128, 64), (300, 3, 64, 58), (5, 9, 33, 22),
                                                (129, 33, 256, 256), (1023, 2, 32, 16), (64, 48, 128, 8), (3, 1, 96, 96)])
@pytest.mark.parametrize("transpose", [False, True])
def test_apply(dare, dtype, layout, tokens, heads, hd, r, transpose):
    g = torch.Generator(device="cuda").manual_seed(tokens * 1000 + heads * 10 + r)
    x = torch.randn((tokens, heads, hd), generator=g, device="cuda").to(dtype)
    table = dare.rope_table(4000, r, 1e4, magnitude=0.75)
    pos = torch.randint(0, 4000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = 3999
    before = x.clone()
    y = dare.rope(x, table, pos, layout=dare.ROPE_LAYOUT[layout], transpose=transpose)
    assert torch.equal(x, before)
    want = oracle(x, table, pos, r, layout, transpose)
    assert close(y, want, x, 0.75)
    assert torch.equal(y[..., r:], x[..., r:])
    # in place, and without positions: pos_begin + token
    z = x.clone()
    assert dare.rope(z, table, pos, layout=dare.ROPE_LAYOUT[layout], transpose=transpose, out=z) is z
    assert torch.equal(z, y)
    run = dare.rope(x, table, layout=dare.ROPE_LAYOUT[layout], transpose=transpose, pos_begin=11)
    assert close(run, oracle(x, table, torch.arange(11, 11 + tokens, device="cuda"), r, layout, transpose), x, 0.75)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(dare, dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    table = dare.rope_table(64, 64, 1e4)
    fused = torch.randn((50, 12, 64), generator=g, device="cuda").to(dtype)
    pos = torch.randint(0, 64, (50,), generator=g, device="cuda", dtype=torch.int32)
    want = oracle(fused, table, pos, 64, "half", False)
    # some heads of a fused row, in place: the other heads stay
    z = fused.clone()
    dare.rope(z[:, 2:7], table, pos, out=z[:, 2:7])
    assert torch.equal(z[:, :2], fused[:, :2]) and torch.equal(z[:, 7:], fused[:, 7:])
    assert close(z[:, 2:7], want[:, 2:7], fused, 1.0)
    # head-major memory in and out
    y = torch.empty((12, 50, 64), dtype=dtype, device="cuda").transpose(0, 1)
    dare.rope(fused.transpose(0, 1).contiguous().transpose(0, 1), table, pos, out=y)
    assert close(y, want, fused, 1.0)
    # rows that start off the 16-byte grid
    odd = torch.zeros(50 * 12 * 64 + 1, dtype=dtype, device="cuda")[1:].view(50, 12, 64)
    odd.copy_(fused)
    assert torch.equal(dare.rope(odd, table, pos), dare.rope(fused, table, pos))


def test_there_and_back_and_gradient(dare):
    g = torch.Generator(device="cuda").manual_seed(5)
    table = dare.rope_table(512, 48, 1e4)
    x = torch.randn((37, 6, 64), generator=g, device="cuda")
    pos = torch.randint(0, 512, (37,), generator=g, device="cuda", dtype=torch.int32)
    for layout in dare.ROPE_LAYOUT.values():
        back = dare.rope(dare.rope(x, table, pos, layout=layout), table, pos, layout=layout, transpose=True)
        # two passes of 8 * 2^-24 max |x| each, and cos^2 + sin^2 = 1 to 2 * 2^-24
        assert (back - x).abs().max().item() <= 20 * 2.0 ** -24 * x.abs().max().item()
        # the gradient of <w, rope(x)> in x is rope^T(w): against central differences of the (linear) forward call
        w, d = torch.randn(x.shape, generator=g, device="cuda"), torch.randn(x.shape, generator=g, device="cuda")
        slope = ((dare.rope(x + d, table, pos, layout=layout) - dare.rope(x - d, table, pos, layout=layout)).double() * w).sum() / 2
        grad = dare.rope(w, table, pos, layout=layout, transpose=True)
        scale = (w.abs().double() * (x.abs() + d.abs())).sum().item()
        assert abs(slope.item() - (grad.double() * d).sum().item()) <= 20 * 2.0 ** -24 * scale


def test_positions_outside_the_table(dare):
    table = dare.rope_table(100, 32, 1e4)
    x = torch.randn((6, 3, 32), device="cuda")
    pos = torch.tensor([0, -1, 99, 100, 2 ** 31 - 1, 5], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = torch.full_like(x, 7.0)
    dare.rope(x, table, pos, out=y, status=status)
    assert status.item() == dare.ERR_DEVICE_CHECK
    assert bool((y[[1, 3, 4]] == 7.0).all())
    ok = [0, 2, 5]
    assert close(y[ok], oracle(x[ok], table, pos[ok], 32, "half", False), x, 1.0)
    dare.rope(x, table, pos, out=y)                       # and without a status word


def test_empty_calls_capture_and_streams(dare):
    table = dare.rope_table(100, 32, 1e4)
    assert dare.rope(torch.empty((0, 3, 32), device="cuda"), table).shape == (0, 3, 32)
    assert dare.rope_table(0, 32, 1e4).shape == (0, 16, 2)
    x = torch.randn((40, 3, 32), device="cuda")
    want = dare.rope(x, table)
    y, side = torch.zeros_like(x), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dare.rope(x, table, out=y)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dare.rope(x, table, out=y)
    x.add_(1.0)
    graph.replay()
    assert torch.equal(y, dare.rope(x, table))
