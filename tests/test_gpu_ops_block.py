"""The stand-alone operators as a caller strings them together: a pre-norm block with grouped heads, biases and its own rotary
layout, over packed prompts of different lengths and then one more token of each sequence against caches."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
D, H, KV, HD, FF, ROOM, R = 512, 8, 2, 64, 1408, 160, 48
LENS = [70, 133, 1, 32]


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def make(dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s, std=1.0: torch.randn(s, generator=g, device="cuda") * std
    w = {"qkv": n((H + 2 * KV) * HD, D, std=D ** -0.5), "o": n(D, H * HD, std=(H * HD) ** -0.5), "up": n(FF, D, std=D ** -0.5),
         "down": n(D, FF, std=FF ** -0.5)}
    w = {k: v.to(dtype) for k, v in w.items()}
    w |= {"b_qkv": n((H + 2 * KV) * HD, std=0.3), "b_up": n(FF, std=0.3), "gain1": n(D, std=0.1) + 1, "gain2": n(D, std=0.1) + 1}
    return w, n(sum(LENS), D).to(dtype), n(len(LENS), D).to(dtype)


def norm(dare, x, gain):
    y = torch.empty_like(x)
    assert dare.dare_rmsnorm(x.data_ptr(), gain.data_ptr(), y.data_ptr(), x.shape[0], D, 1e-5,
                             dare.BF16 if x.dtype == torch.bfloat16 else dare.F32, torch.cuda.current_stream().cuda_stream) == dare.OK
    return y


def block(dare, w, x, table, positions, keys):
    """keys(k, v) -> (k, v, k_begin, k_len): where the attention finds keys and values once this call's are known."""
    qkv = dare.linear(norm(dare, x, w["gain1"]), w["qkv"], bias=w["b_qkv"]).view(-1, H + 2 * KV, HD)
    turned = qkv[:, :H + KV]
    dare.rope(turned, table, positions, layout=dare.ROPE_LAYOUT["interleaved"], out=turned)
    k, v, q_begin, k_begin, k_len = keys(qkv[:, H:H + KV], qkv[:, H + KV:])
    o = dare.attention(qkv[:, :H], k, v, q_begin, k_begin, k_len=k_len, causal=True)
    y = dare.linear(o.view(-1, H * HD), w["o"], resid=x)
    up = dare.linear(norm(dare, y, w["gain2"]), w["up"], bias=w["b_up"], act=dare.ACT["gelu"])
    return dare.linear(up, w["down"], resid=y)


def oracle(w, x):
    """One sequence, float64."""
    w = {k: v.double() for k, v in w.items()}
    x = x.double()
    rms = lambda t, g: t / (t.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * g
    qkv = (rms(x, w["gain1"]) @ w["qkv"].T + w["b_qkv"]).view(-1, H + 2 * KV, HD)
    ang = torch.outer(torch.arange(len(x), dtype=torch.float64, device="cuda"),
                      1e4 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R))
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    a, b = qkv[:, :H + KV, 0:R:2].clone(), qkv[:, :H + KV, 1:R:2].clone()
    qkv[:, :H + KV, 0:R:2], qkv[:, :H + KV, 1:R:2] = a * c - b * s, b * c + a * s
    q, k, v = qkv[:, :H], qkv[:, H:H + KV].repeat_interleave(H // KV, 1), qkv[:, H + KV:].repeat_interleave(H // KV, 1)
    z = torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(HD)
    z = z.masked_fill(torch.ones(len(x), len(x), dtype=torch.bool, device="cuda").triu(1), -math.inf)
    o = torch.einsum("hqk,khd->qhd", z.softmax(-1), v).reshape(len(x), H * HD)
    y = x + o @ w["o"].T
    t = rms(y, w["gain2"]) @ w["up"].T + w["b_up"]
    return y + (0.5 * t * (1 + torch.erf(t / math.sqrt(2)))) @ w["down"].T


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompts_then_a_token(dare, dtype):
    w, x, x_next = make(dtype)
    # The chain rounds a dozen times (norms, projection, rotation, weights, outputs), each by at most 2^-8 (2^-24) of its result in the
    # 2-norm, and the branches add to a residual as large as they are: twelve of those.  fp32 sums of up to 1408 products: 2^-13 more.
    tol = 12 * 2.0 ** -8 if dtype == torch.bfloat16 else 12 * 2.0 ** -24 + 2.0 ** -13
    ints = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")
    begins = [sum(LENS[:i]) for i in range(len(LENS) + 1)]
    table = dare.rope_table(ROOM, R, 1e4)
    cache = torch.full((2, len(LENS), ROOM, KV, HD), float("nan"), dtype=dtype, device="cuda")
    begin_q, positions = ints(begins), ints([p for n in LENS for p in range(n)])

    def prompt_keys(k, v):
        for b, n in enumerate(LENS):
            cache[0, b, :n], cache[1, b, :n] = k[begins[b]:begins[b + 1]], v[begins[b]:begins[b + 1]]
        return k, v, begin_q, begin_q, None

    out = block(dare, w, x, table, positions, prompt_keys)
    where, begin_one, begin_cache, lens = ints(LENS), ints(range(len(LENS) + 1)), ints([b * ROOM for b in range(len(LENS))]), ints([n + 1 for n in LENS])
    rows = torch.arange(len(LENS), device="cuda")

    def token_keys(k, v):
        cache[0, rows, where.long()], cache[1, rows, where.long()] = k, v
        return cache[0].view(-1, KV, HD), cache[1].view(-1, KV, HD), begin_one, begin_cache, lens

    nxt = block(dare, w, x_next, table, where, token_keys)
    for b, n in enumerate(LENS):
        want = oracle(w, torch.cat((x[begins[b]:begins[b + 1]], x_next[b:b + 1])))
        got = torch.cat((out[begins[b]:begins[b + 1]], nxt[b:b + 1])).double()
        assert (got - want).norm().item() <= tol * want.norm().item(), (b, ((got - want).norm() / want.norm()).item())
        assert (got[-1] - want[-1]).norm().item() <= tol * want[-1].norm().item()
    # the step as a captured graph: the same bits, and new ones for a new input
    graph, x_in = torch.cuda.CUDAGraph(), x_next.clone()
    with torch.cuda.graph(graph):
        again = block(dare, w, x_in, table, where, token_keys)
    graph.replay()
    assert torch.equal(again, nxt)
    x_in.copy_(x_next.flip(0))
    graph.replay()
    assert torch.equal(again, block(dare, w, x_next.flip(0).contiguous(), table, where, token_keys))
