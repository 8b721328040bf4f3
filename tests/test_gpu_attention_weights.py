"""Softmax weights of packed attention in bf16: how many bits of them reach the product with the values."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# many rows (256 a CTA), few rows over many keys (shares of the keys), and heads on the CUDA cores
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,hd,nq,n", [(64, 8, 64, 700, 900), (16, 4, 64, 700, 900), (8, 8, 64, 1500, 1500), (16, 2, 64, 1, 3001), (8, 4, 64, 40, 2500),
                                                    (32, 8, 64, 128, 128), (4, 2, 32, 60, 333), (4, 1, 256, 60, 333)])
def test_heads_of_64_keep_16_bits(dare, heads, kv_heads, hd, nq, n, causal):
    """Values of both signs, so that outputs are small beside what is summed: a weight's error is not hidden by storing the output."""
    g = torch.Generator(device="cuda").manual_seed(heads + nq + n)
    q, k, v = (torch.randn((r, h, hd), generator=g, device="cuda").to(BF16) for r, h in ((nq, heads), (n, kv_heads), (n, kv_heads)))
    scale = hd ** -0.5
    out, lse = dare.attention(q, k, v, ints([0, nq]), ints([0, n]), causal=causal, return_lse=True)
    ks, vs = (t.double().repeat_interleave(heads // kv_heads, 1).transpose(0, 1) for t in (k, v))
    qs = q.double().transpose(0, 1)
    z = qs @ ks.transpose(1, 2) * scale
    mag = (qs.abs() @ ks.abs().transpose(1, 2) * scale).amax().item()
    if causal:
        z = z.masked_fill(torch.ones((nq, n), dtype=torch.bool, device="cuda").triu(n - nq + 1), float("-inf"))
    w = z.softmax(-1)
    want, size = w @ vs, w @ vs.abs()
    got = out.double().transpose(0, 1)
    # A score: hd products summed in fp32 and scaled (the tensor core truncates, an ulp an addition), (2 hd + 16) 2^-24 of the magnitudes; 2^x
    # with its argument 2^-20; sums over the keys, an ulp a key.  A weight in two bf16 parts: 2^-8 is left by the first (half a step of bf16),
    # 2^-8 of that by the second.  Storing the output: half a step.
    eps = (2 * hd + 16) * 2.0 ** -24 * mag + 2.0 ** -20 + (n + 16) * 2.0 ** -23
    bound = 2.0 ** -8 * want.abs() * (1 + eps) + (2.0 ** -16 + eps) * size
    assert bool(((got - want).abs() <= bound).all()), ((got - want).abs() / bound).max().item()
    # The errors' 2-norm: what rounding the exact output to bf16 leaves, and of each weight at most the above (of random signs, less).
    err, stored = (got - want).norm().item(), (want.to(BF16).double() - want).norm().item()
    assert err <= stored + (2.0 ** -16 + eps) * size.norm().item(), (err, stored)
