"""Operators whose operands the kernel in front of them has just written, one behind the other without a wait on the host: the same bits
as with one after every call."""
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


def replays(step, inputs, n):
    """step() captured and replayed on n inputs, against the same step with a synchronisation after every call."""
    plain = lambda f, *a, **k: (f(*a, **k), torch.cuda.synchronize())[0]
    direct = lambda f, *a, **k: f(*a, **k)
    for x in inputs[1]:
        inputs[0].copy_(x)
        step(plain)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(direct)
    for i in range(n):
        x = inputs[1][i % len(inputs[1])]
        inputs[0].copy_(x)
        graph.replay()
        got = [t.clone() for t in out]
        inputs[0].copy_(x)
        want = step(plain)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


@pytest.mark.parametrize("dtype,m,d,last", [(BF16, 1, 1024, 1024), (BF16, 4, 512, 264), (BF16, 16, 2048, 512), (BF16, 300, 512, 520),
                                            (F32, 1, 1024, 1000), (F32, 3, 516, 260), (F32, 40, 512, 256), (F32, 200, 256, 512)])
def test_products(dare, dtype, m, d, last):
    """Each product reads what the one before wrote: as x, as residual, as W, as bias."""
    g = torch.Generator(device="cuda").manual_seed(m + d)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = torch.empty((m, d), dtype=dtype, device="cuda")
    xs = [rand(m, d).to(dtype) for _ in range(3)]
    w = [(rand(d, d) * d ** -0.5).to(dtype) for _ in range(3)]
    side = rand(last, d).to(dtype)
    bias_w = rand(d, 8)

    def step(call):
        a = call(dare.linear, x, w[0], act=dare.ACT["silu"])
        b = call(dare.linear, a, w[1], resid=a)
        c = call(dare.linear, b, w[2], act=dare.ACT["gelu"], resid=x)
        weights = call(dare.linear, side, w[0])                              # W, and a bias, of what was just computed
        bias = call(dare.linear, c[:1, :8].float(), bias_w)[0]
        e = call(dare.linear, c, w[0], bias=bias)
        return a, b, c, e, call(dare.linear, e, weights)
    replays(step, (x, xs), 30)


@pytest.mark.parametrize("dtype,hd,n", [(BF16, 128, 40), (BF16, 64, 700), (F32, 64, 40), (BF16, 128, 1), (F32, 128, 1)])
def test_table_rotation_attention(dare, dtype, hd, n):
    """Table, rotation with positions, attention with lengths, all written by the kernel in front."""
    g = torch.Generator(device="cuda").manual_seed(n + hd)
    cache = 1500
    x = torch.empty((n, 8 + 2 + 2, hd), dtype=dtype, device="cuda")
    xs = [torch.randn(x.shape, generator=g, device="cuda").to(dtype) for _ in range(3)]
    k, v = (torch.randn((cache, 2, hd), generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.empty((2048, hd // 2, 2), device="cuda")
    pos, lens = (torch.empty(s, dtype=torch.int32, device="cuda") for s in (n, 1))
    q_begin, k_begin = (torch.tensor(s, dtype=torch.int32, device="cuda") for s in ([0, n], [0]))
    arange = torch.arange(n, dtype=torch.int32, device="cuda")

    def step(call):
        call(dare.rope_table, 2048, hd, 1e4, out=table)
        torch.add(arange, (x[0, 0, 0].abs() * 100).to(torch.int32), out=pos)
        turned = call(dare.rope, x[:, :10], table, pos)
        call(dare.rope_table, 2048, hd, 5e5, out=table)
        again = call(dare.rope, turned, table, pos, layout=dare.ROPE_LAYOUT["interleaved"])
        torch.add(n, pos[:1], out=lens)
        out, lse = call(dare.attention, again[:, :8], k, v, q_begin, k_begin, k_len=lens, causal=True, return_lse=True)
        return turned, again, out, lse
    replays(step, (x, xs), 30)
